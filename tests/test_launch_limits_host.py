"""The launches of the dense operators at the ends of their sizes, without a GPU: libemb.so is loaded after
stand-ins for the runtime's launch functions (tests/host_order/launches.cpp) that keep every grid.  A launch
holds less than 2^32 threads along x and at most 65535 workgroups along y and z, and the kernels that are
launched several times over parts of their work cover all of it."""
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(ROOT, "paper_2110_09132_amd", "libemb.so")

# One process per call, so that this one keeps its runtime: (call, arguments) -> the launches.
RUN = """
import ctypes, sys
shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
shim.launches_get.restype = ctypes.c_char_p
P, I, L, D, S = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t
FAKE, NULL, ALL = P(4096), None, S(-1)


def norm(T, D_, ids=NULL, V=0, xt=0, yt=0):
    return lib.emb_layer_norm(FAKE, I(xt), L(D_), ids, L(V), I(T), I(D_), NULL, NULL, D(1e-5), FAKE, I(yt), L(D_), FAKE,
                              FAKE, NULL, NULL)


def norm_grad(T, D_, xt=0, yt=0):
    return lib.emb_layer_norm_backward(FAKE, I(yt), L(D_), FAKE, I(xt), L(D_), NULL, L(0), I(T), I(D_), NULL, FAKE, FAKE,
                                       FAKE, L(D_), FAKE, FAKE, FAKE, ALL, NULL, NULL)


def bias(H, Q, K, R=100, B=32, dtype=0):
    return lib.emb_relative_bias(FAKE, I(B), I(H), FAKE, I(R), I(Q), I(K), L(0), FAKE, I(dtype), L(K), L(Q * K), NULL,
                                 NULL)


def bias_grad(N, H, Q, K, R=100, B=32, dtype=0):
    return lib.emb_relative_bias_backward(FAKE, I(dtype), I(N), I(H), I(Q), I(K), L(H * Q * K), L(Q * K), L(K), FAKE, I(R),
                                          I(B), L(0), FAKE, FAKE, ALL, NULL, NULL)


assert eval(sys.argv[3]) == 0
out = (ctypes.c_uint32 * 6)()
for i in range(shim.launches_count()):
    name = shim.launches_get(i, out).decode()
    print(name, *out)
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = tmp_path_factory.mktemp("launches")
    shim = d / "liblaunches.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "host_order", "launches.cpp"),
                    "-o", str(shim)], check=True)

    def run(call):
        r = subprocess.run([sys.executable, "-c", RUN, str(shim), LIB, call], capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        got = []
        for line in r.stdout.splitlines():
            name, *n = line.split()
            gx, gy, gz, bx, by, bz = map(int, n)
            assert gx >= 1 and gx * bx < 1 << 32 and 1 <= gy <= 65535 and 1 <= gz <= 65535 and bx * by * bz <= 1024, line
            got.append((name, gx, gy, gz, bx))
        return got
    return run


def blocks(got, kernel):
    return sum(gx for name, gx, *_ in got if kernel in name)


MOST = (1 << 30) - 1  # rows, queries, keys, the map's reach


@pytest.mark.parametrize("T,D", [(1, (1 << 28) - 1), (5, 1 << 26), (3, (1 << 26) + 1), (MOST, 1), (MOST, 1000),
                                 (MOST, 20000), (0, (1 << 28) - 1)])
def test_layer_norm(T, D, launches):
    for xt, yt in ((0, 0), (1, 1)):
        if T:
            launches(f"norm({T}, {D}, xt={xt}, yt={yt})")
        got = launches(f"norm_grad({T}, {D}, xt={xt}, yt={yt})")
        assert blocks(got, "norm_sum") == -(-2 * D // 32)  # 32 of the 2 D columns each


@pytest.mark.parametrize("H,Q,K", [(1, MOST, 1), (1, 1, MOST), (65535, 1, 1000), (1, 1 << 25, 1025), (1, MOST, 64),
                                   (1, 1 << 26, 1030), (2, 1 << 20, 1 << 17)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_relative_bias(H, Q, K, dtype, launches):
    got = launches(f"bias({H}, {Q}, {K}, dtype={dtype})")
    assert all(gy == H for _, _, gy, *_ in got)


@pytest.mark.parametrize("N,H,Q,K,R,B", [(1, 1, 1, 1 << 28, MOST, 32), (1, 1, 1, MOST, MOST, 32), (1, 2, MOST, 1, MOST, 32),
                                         (1, 65535, 3, 40, 100, 32), (1 << 20, 1, 10, 10, 100, 32),
                                         (1, 1, 700, 700, 5000, 1 << 26), (1, 1, 700, 700, 5000, (1 << 31) - 1),
                                         (1, 1, 10, 10, 5, (1 << 31) - 1), (0, 1, 10, 10, 5, (1 << 31) - 1)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_relative_bias_gradient(N, H, Q, K, R, B, dtype, launches):
    got = launches(f"bias_grad({N}, {H}, {Q}, {K}, {R}, {B}, {dtype})")
    if any("bias_fold" in g[0] for g in got):
        return
    assert blocks(got, "bias_buckets") == -(-B // 4)  # a wave per bucket, four in a workgroup
    if N:
        places = min(R, K - 1) + min(R, Q - 1) + 1
        assert blocks(got, "bias_places") == -(-places // 64)
