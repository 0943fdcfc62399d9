"""Which kernels of the cross entropy a size goes to, without a GPU (the launches are kept as in
test_launch_limits_host.py): the sizes of tests/test_gpu_vocab_loss_many.py reach the kernels that they are there for,
and those of tests/test_gpu_vocab_loss.py the few tokens' way, on both sides of its limits."""
import re

import pytest

import test_gpu_vocab_loss as few
import test_gpu_vocab_loss_many as many
import test_launch_limits_host as limits
from test_launch_limits_host import launches  # noqa: F401
from test_launch_limits_train_host import MORE, blocks


@pytest.fixture(autouse=True)
def more(monkeypatch):
    monkeypatch.setattr(limits, "RUN", limits.RUN.replace("\nassert eval", MORE + "\nassert eval"))


def kernels(got):
    """(name, template arguments) of the launches; the arguments as the compiler writes them."""
    return [re.search(r"\d([a-z][a-z_]*_kernel)(?:I(.+?)EEv|E)", g[0]).groups() for g in got]


def count(got, name, *arguments):
    return sum(k == name and all(a in (t or "") for a in arguments) for k, t in kernels(got))


@pytest.mark.parametrize("name", many.WAYS)
def test_many_tokens(name, launches):  # noqa: F811
    T, V, D, dtype, stands, table_pieces, g_pieces = many.WAYS[name]
    dt = int(dtype == many.BF16)
    planes, tiles = 1 if dt else 3, -(-T // 256)
    for smoothing in (0.0, 0.1):
        got = launches(f"loss({T}, {V}, {D}, {dt}, {smoothing})")
        assert count(got, "loss_kernel", f"Li{planes}E", f"Lb{int(smoothing > 0)}") == table_pieces
        assert count(got, "loss_few_kernel") == 0
        # the squares of 64 rows that are laid out: the tokens', and the table's unless it is read where it stands
        assert blocks(got, "pack_kernel") == 4 * tiles + (0 if stands else 4 * -(-V // 256))
    got = launches(f"loss_grad({T}, {V}, {D}, {dt})")
    assert count(got, "few_grad_kernel") == 0
    for kernel in ("grad_logits_kernel", "grad_table_kernel", "grad_rows_kernel"):
        assert count(got, kernel, f"Li{planes}E") == g_pieces


@pytest.mark.parametrize("T,V,D", few.SIZES)
@pytest.mark.parametrize("dt", [0, 1])
def test_few_tokens(T, V, D, dt, launches):  # noqa: F811
    assert count(launches(f"loss({T}, {V}, {D}, {dt})"), "loss_few_kernel") == 1
    assert count(launches(f"loss_grad({T}, {V}, {D}, {dt})"), "few_grad_kernel") == (T <= 64)


@pytest.mark.parametrize("dt", [0, 1])
def test_the_few_tokens_limits(dt, launches):  # noqa: F811
    """64 tokens of any vocabulary; more of them up to 4e9 operations; rows as wide as 136 KB hold 16 of."""
    for T, V, D, way in ((64, 1 << 20, 256, True), (65, 1 << 20, 256, False), (1000, 31250, 64, True),
                         (1000, 31251, 64, False), (1, 70, 4320 if dt else 1440, True), (1, 70, 4321 if dt else 1441, False)):
        got = launches(f"loss({T}, {V}, {D}, {dt})")
        assert count(got, "loss_few_kernel") == int(way) and (count(got, "loss_kernel") > 0) == (not way), (T, V, D)
