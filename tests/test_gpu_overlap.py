"""GPU: outputs of the 8-bit layer and of the distillation calls that lie over their inputs are right or refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _slim():
    from paper_2405_14917_b200 import binding
    return binding


@pytest.mark.parametrize("M", [1, 5, 16, 17, 40, 100, 300])
def test_product_over_its_input(M):
    """Up to 16 tokens x is read while y is written: refused.  Beyond, x has been quantised by then."""
    slim = _slim()
    n = 2048
    g = torch.Generator().manual_seed(M)
    layer = slim.Fp8Linear.from_weight((torch.randn(n, n, generator=g) * 0.02).half().cuda())
    x = torch.randn(M, n, generator=g).half().cuda()
    ws = layer.new_workspace(M)
    want = layer.forward(x, ws)
    if M > 16:
        assert layer.forward(x, ws, out=x) is x and torch.equal(x, want)
        return
    keep = x.clone()
    with pytest.raises(slim.SlimError) as e:
        layer.forward(x, ws, out=x)
    assert e.value.status == -1 and torch.equal(x, keep)
    # columns of one buffer, side by side: no overlap
    both = torch.zeros(M, 2 * n, dtype=torch.float16, device="cuda")
    both[:, :n] = keep
    layer.forward(both[:, :n], ws, out=both[:, n:])
    assert torch.equal(both[:, n:], want) and torch.equal(both[:, :n], keep)


@pytest.mark.parametrize("M", [3, 700])
def test_gradient_partly_over_the_logits(M):
    slim = _slim()
    V, k = 1000, 5
    buf = torch.randn(M, V + 8, device="cuda")
    s, shifted = buf[:, :V], buf[:, 8:]
    value, index = torch.topk(s, k, dim=1)
    d = torch.ones(M, device="cuda")
    loss, saved = slim.distill_loss(s, index, value)
    keep = buf.clone()
    for call in (lambda out: slim.distill_step(s, index, value, d, out=out), lambda out: slim.distill_grad(s, index, value, saved, d, out=out)):
        for out in (shifted, torch.as_strided(buf, (M, V), (V, 1))):     # another first column; the same start with another stride
            with pytest.raises(slim.SlimError) as e:
                call(out)
            assert e.value.status == -1 and torch.equal(buf, keep)
