"""GPU: products of the 8-bit layer that an fp32 sum holds exactly are exact, at every number of tokens."""
import pytest
import torch

pytestmark = pytest.mark.gpu


# each kernel form: x quantised inside (to 16 tokens), by a launch of its own (tiles of 32, 64 and 128 tokens), CTA pairs; K cut over a cluster and not
@pytest.mark.parametrize("M", [1, 7, 16, 30, 60, 128, 200, 600])
@pytest.mark.parametrize("N,K", [(300, 13824), (9000, 1040)])
@pytest.mark.parametrize("low", [0, -8])
def test_sums_of_integers(M, N, K, low):
    """Whole numbers up to 8 in x and W: every code is exact, every product a whole number up to 64 and every partial sum one below 2^20, so fp32 sums
    round nothing.  An accumulator of fewer than 20 bits would (with low = 0 the sums are of 16 K = 221000 at K = 13824)."""
    from paper_2405_14917_b200 import binding as slim
    g = torch.Generator(device="cuda").manual_seed(M + N)
    W = torch.randint(low, 9, (N, K), generator=g, device="cuda")
    x = torch.randint(low, 9, (M, K), generator=g, device="cuda")
    layer = slim.Fp8Linear(W.float().to(torch.float8_e4m3fn), torch.ones((N + 127) // 128, (K + 127) // 128, device="cuda"))
    ws = layer.new_workspace(M)
    y = layer.forward(x.half(), ws, out_dtype=torch.float32)
    slim.workspace_status(ws)
    assert torch.equal(y.double(), x.double() @ W.double().t())
