"""The launches of dropout, the norms around a block and the cross entropy at the ends of their sizes, without a GPU
(as in test_launch_limits_host.py, whose stand-ins keep every grid): every launch fits, and the kernels that are
launched several times over parts of their work cover all of it."""
import pytest

import paper_2110_09132_amd as emb
import test_launch_limits_host as limits
from test_launch_limits_host import MOST, blocks, launches  # noqa: F401


def fields(struct):
    return ", ".join(f"('{name}', ctypes.{kind.__name__})" for name, kind in struct._fields_)


MORE = f"""
class Block(ctypes.Structure):
    _fields_ = [{fields(emb.BlockNormArgs)}]


class BlockGrad(ctypes.Structure):
    _fields_ = [{fields(emb.BlockNormGradArgs)}]


def struct(kind, T, D_, st, bt, gate_rows, **more):
    a = kind(**more)
    for name, t in kind._fields_:
        if t is ctypes.c_void_p and name != "seed_dev":
            setattr(a, name, 4096)
        if name.startswith("ld"):
            setattr(a, name, D_)
    a.T, a.D, a.stream_dtype, a.dtype, a.gate_rows, a.alpha, a.p = T, D_, st, bt, gate_rows, 1.0, 0.1
    return a


def dropout(T, D_, dt):
    return lib.emb_dropout(FAKE, I(dt), L(D_), I(T), I(D_), D(0.1), ctypes.c_uint64(3), NULL, FAKE, L(D_), FAKE, L(D_), NULL)


def block(T, D_, st, bt, gate_rows=0):
    a = struct(Block, T, D_, st, bt, gate_rows, eps=1e-5)
    return lib.emb_block_norm(ctypes.byref(a), NULL)


def block_grad(T, D_, st, bt, gate_rows=0):
    a = struct(BlockGrad, T, D_, st, bt, gate_rows, workspace_bytes=1 << 62)
    return lib.emb_block_norm_backward(ctypes.byref(a), NULL)


def loss(T, V, D_, dt, e=0.1):
    return lib.emb_vocab_loss(FAKE, I(dt), L(D_), FAKE, L(D_), I(T), L(V), I(D_), FAKE, D(e), FAKE, FAKE, FAKE, ALL, NULL,
                              NULL)


def loss_grad(T, V, D_, dt, e=0.1):
    return lib.emb_vocab_loss_backward(FAKE, I(1), FAKE, I(dt), L(D_), FAKE, L(D_), I(T), L(V), I(D_), FAKE, D(e), FAKE, FAKE,
                                       L(D_), FAKE, L(D_), FAKE, ALL, NULL, NULL)

"""
WIDEST = (1 << 28) - 1
ROWS = [(1, WIDEST), (5, 1 << 26), (MOST, 1), (MOST, 300), (MOST, 1000), (1 << 20, 20000), (MOST, WIDEST)]


@pytest.fixture(autouse=True)
def more(monkeypatch):
    monkeypatch.setattr(limits, "RUN", limits.RUN.replace("\nassert eval", MORE + "\nassert eval"))


@pytest.mark.parametrize("T,D", [(T, D) for T, D in ROWS if T * D < 1 << 41])
@pytest.mark.parametrize("dt", [0, 1])
def test_dropout(T, D, dt, launches):  # noqa: F811
    got = launches(f"dropout({T}, {D}, {dt})")
    lanes = min(256, 1 << max(0, (-(-D // (8 if dt else 4)) - 1).bit_length()))
    assert blocks(got, "dropout_kernel") == -(-T // (256 // lanes))


@pytest.mark.parametrize("T,D", ROWS)
@pytest.mark.parametrize("st,bt", [(0, 0), (0, 1), (1, 1)])
def test_block_norm(T, D, st, bt, launches):  # noqa: F811
    if T * D < 1 << 41 or D > 20000:
        launches(f"block({T}, {D}, {st}, {bt})")
    got = launches(f"block_grad({T}, {D}, {st}, {bt})")
    assert blocks(got, "block_sum") == -(-5 * D // 32)
    for rows in (1, 7, T, 1 << 62):
        got = launches(f"block_grad({T}, {D}, {st}, {bt}, {rows})")
        assert blocks(got, "block_sum") >= -(-5 * D // 32)
    assert blocks(launches(f"block_grad(0, {D}, {st}, {bt}, 7)"), "block_sum") == -(-5 * D // 32)


@pytest.mark.parametrize("T,V,D", [(1, (1 << 31) - 1, 1), (64, (1 << 31) - 1, 64), (65, (1 << 31) - 1, 1), (1, 1, 1 << 16),
                                   (64, 1 << 20, 1 << 16), (1 << 22, 1, 1), (1 << 22, 1000, 1 << 16), (1 << 16, 30000, 1),
                                   (1 << 18, 1000, 1 << 16), (1 << 22, 100000, 64)])
@pytest.mark.parametrize("dt", [0, 1])
def test_vocab_loss(T, V, D, dt, launches):  # noqa: F811
    got = launches(f"loss({T}, {V}, {D}, {dt})")
    if any("loss_join_kernel" in g[0] for g in got):
        assert blocks(got, "loss_join_kernel") == -(-T // 4)
    got = launches(f"loss_grad({T}, {V}, {D}, {dt})")
    if any("grad_rows_join" in g[0] for g in got):
        width = [64 * w for w in (4, 2, 1) if f"Li{w}E" in next(g[0] for g in got if "grad_rows_join" in g[0])][0]
        tiles = -(-T // 256) * -(-D // width)
        assert blocks(got, "grad_rows_join") == tiles * width // 8 + -(-T // 64)
