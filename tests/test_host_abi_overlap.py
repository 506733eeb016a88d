"""Host only: outputs that lie over inputs they may not lie over are refused, and only those, before a pointer is read.  The addresses here are not memory:
what is not refused goes as far as the CUDA runtime, which has no device to run it on, and nothing of this is called where there is one."""
import ctypes
import random

import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are accepted would run")

A = 1 << 20
OVER, ACCEPTED = -1, -5               # invalid argument; CUDA error: no device


@pytest.fixture(scope="module")
def lib():
    from paper_2405_14917_b200 import binding
    return binding.lib()


def _product(lib, y, M=4, ldx=256, ldy=128, yt=1, N=128, K=256):
    return lib.slim_fp8_linear(A, 1, ldx, 1 << 30, 1 << 29, y, yt, ldy, M, N, K, 1 << 31, 1 << 20, None)


def test_product(lib):
    lin = lambda *a, **k: _product(lib, *a, **k)
    assert lin(A) == OVER and lin(A, M=1) == OVER
    assert lin(A, M=17) == ACCEPTED                                   # x is quantised first
    assert lin(A + 16) == OVER                                            # within x's first row
    assert lin(A - 128 * 2 * 4 + 16) == OVER                              # y's last elements over x's first
    assert lin(A + 2 * 256 * 3 + 512 - 16) == OVER                        # y's first over x's last
    assert lin(A + 512, ldx=1024, ldy=1024) == ACCEPTED               # side by side in one buffer
    assert lin(A + 496, ldx=1024, ldy=1024) == OVER                       # by 16 bytes
    assert lin(A - 512, ldx=1024, ldy=512, yt=0) == ACCEPTED          # fp32 rows beside
    assert lin(A - 496, ldx=1024, ldy=512, yt=0) == OVER
    assert lin(A - 512, ldx=1024, ldy=1024, yt=0) == ACCEPTED         # another stride, and between the rows all the same
    assert lin(A + 4 * 512) == ACCEPTED and lin(A - 4 * 256) == ACCEPTED      # behind, before


def test_product_at_random_places(lib):
    rng = random.Random(1)
    seen = set()
    for _ in range(3000):
        M, K, N, yt = rng.randint(1, 6), 16 * rng.randint(1, 4), rng.randint(1, 60), rng.choice([0, 1])
        es = 4 if yt == 0 else 2
        ldx, ldy = K + 8 * rng.randint(0, 12), N + rng.randint(0, 90)
        if rng.random() < 0.5:
            ldy = max(N, ldx * 2 // es)
        y = A + 16 * rng.randint(-60, 60)
        bytes_x = {A + 2 * ldx * m + i for m in range(M) for i in range(2 * K)}
        over = any(y + es * ldy * m + i in bytes_x for m in range(M) for i in range(es * N))
        assert _product(lib, y, M, ldx, ldy, yt, N, K) == (OVER if over else ACCEPTED), (M, K, N, yt, ldx, ldy, y - A)
        seen.add((over, 2 * ldx == es * ldy))
    assert len(seen) == 4


@pytest.mark.parametrize("call", ["grad", "step"])
def test_gradient(lib, call):
    def run(grad, ld=100, ldg=100, M=3, V=100):
        a = (A, 1, ld, 1 << 30, 8, 1 << 29, 0, None, ctypes.c_double(1.0), M, V, 4)
        if call == "grad":
            return lib.slim_distill_grad(*a, 1 << 28, 1 << 27, grad, ldg, None)
        return lib.slim_distill_step(*a, 1 << 27, 1 << 26, grad, ldg, None)
    fine = ACCEPTED
    assert run(A) == fine                                                 # in place
    assert run(A, ld=104, ldg=104) == fine
    assert run(A, ldg=104) == OVER
    assert run(A, ldg=104, M=1) == fine                                   # of one row no stride is used
    assert run(A + 2) == OVER and run(A - 2) == OVER and run(A + 2, M=1) == OVER
    assert run(A + 200, ld=200, ldg=200) == fine and run(A + 198, ld=200, ldg=200) == OVER
    assert run(A + 600) == fine and run(A + 598) == OVER
    assert run(A - 600) == fine and run(A - 598) == OVER
