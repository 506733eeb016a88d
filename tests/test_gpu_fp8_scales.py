"""GPU: scales of the 8-bit layer that are not powers of two are not taken for the power of two below them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _slim():
    from paper_2405_14917_b200 import binding
    return binding


# every kernel form: x quantised inside (to 16 tokens), by a launch of its own (tiles of 32, 64 and 128 tokens), CTA pairs
@pytest.mark.parametrize("bad", [1.5, 3.0 * 2.0 ** -100, -1.0, 0.0, -0.0, 2.0 ** -127, 2.0 ** -149, float("inf"), -float("inf"), float("nan"),
                                 1.0 + 2.0 ** -23])
@pytest.mark.parametrize("M", [1, 2, 16, 20, 50, 100, 300, 600])
def test_outputs_under_a_scale_that_is_no_power_of_two_are_nan(M, bad):
    slim = _slim()
    N, K = 9000 if M == 600 else 400, 1296
    g = torch.Generator().manual_seed(M)
    codes, scales = slim.fp8_quantize((torch.randn(N, K, generator=g) * 0.02).half().cuda())
    x = torch.randn(M, K, generator=g).half().cuda()
    ws = torch.empty(slim.fp8_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    slim.workspace_init(ws)
    clean = slim.fp8_linear(x, codes, scales, ws)
    scales[1, 7] = bad                               # rows 128 .. 255 of W
    y = slim.fp8_linear(x, codes, scales, ws)
    slim.workspace_status(ws)
    assert torch.isnan(y[:, 128:256]).all()
    assert torch.equal(y[:, :128], clean[:, :128]) and torch.equal(y[:, 256:], clean[:, 256:])


@pytest.mark.parametrize("M", [1, 20, 100, 600])
def test_the_smallest_and_the_largest_scale_are_taken(M):
    """2^-126 and 2^127, in fp32: exact products with x = 2^-10 and 2^-100, one term per output."""
    slim = _slim()
    N, K = 256, 272
    codes = torch.zeros(N, K, device="cuda")
    codes[:, 5] = 2.0
    codes = codes.to(torch.float8_e4m3fn)
    for exponent, e in ((-126, 20), (127, -100)):
        scales = torch.full((2, 3), 2.0 ** exponent, device="cuda")
        x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
        x[:, 5] = 2.0 ** e
        layer = slim.Fp8Linear(codes, scales)
        y = layer.forward(x, layer.new_workspace(M), out_dtype=torch.float32)
        assert (y == 2.0 ** (exponent + e + 1)).all()
