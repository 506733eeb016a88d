"""A tuning step through an 8-bit output head: a full-precision teacher's top logits (slim_dense_linear), the head's logits, the loss with its
gradient, the gradient of the head's input; each stage against its fp64 oracle on what the stage before gave, and the step as a whole captured and replayed.
And the two ways a call takes into the library (host module; general path) agree."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle
from tests.test_gpu_distill import _check as check_loss
from tests.test_gpu_fp8 import _check as check_product

pytestmark = pytest.mark.gpu


def _slim():
    from paper_2405_14917_b200 import binding
    return binding


def _setup(M, V, K, k, T, rest, seed=3):
    slim = _slim()
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn(V, K, generator=g) * 0.05).to(torch.bfloat16)
    head = slim.Fp8Linear.from_weight(W.cuda())
    head.prepare_input_grad()
    h = torch.randn(M, K, generator=g).to(torch.bfloat16).cuda()
    teacher = slim.dense_linear(h.half() * 1.1, W.half().cuda())            # fp32 [M][V], another model's opinion
    value, index = torch.topk(teacher, k, dim=1)
    index[1] = -1                                                            # a padded token
    lse = torch.logsumexp(teacher / T, 1) if rest else None
    dloss = torch.full((M,), 1.0 / M, device="cuda")
    return head, h, index, value, lse, dloss


def _step(head, h, index, value, lse, dloss, T, ws, ws_grad):
    slim = _slim()
    logits = head.forward(h, ws)
    loss, dlogits = slim.distill_step(logits, index, value, dloss, temperature=T, teacher_lse=lse)
    return logits, loss, dlogits, head.input_grad(dlogits, ws_grad)


@pytest.mark.parametrize("M,V,K,k,T,rest", [(3, 1008, 288, 5, 1.0, False), (40, 2000, 512, 16, 2.0, True), (300, 4096, 416, 32, 1.0, True)])
def test_each_stage_of_a_step(M, V, K, k, T, rest):
    slim = _slim()
    head, h, index, value, lse, dloss = _setup(M, V, K, k, T, rest)
    ws, ws_grad = head.new_workspace(M), head.new_workspace(M, input_grad=True)
    logits, loss, dlogits, dh = _step(head, h, index, value, lse, dloss, T, ws, ws_grad)
    slim.workspace_status(ws), slim.workspace_status(ws_grad)
    check_product(logits, h, head.codes, head.scales)
    check_loss(logits.cpu(), index.cpu(), value.cpu(), None if lse is None else lse.cpu(), dloss.cpu(), T, "bf16", loss, dlogits)
    codes_t = head.codes.view(torch.uint8).t().contiguous().view(torch.float8_e4m3fn)
    check_product(dh, dlogits, codes_t, head.scales.t())
    assert (dh[1] == 0).all() and loss[1] == 0
    # in place: the gradient over the logits, the same step
    again = logits.clone()
    loss2, same = slim.distill_step(again, index, value, dloss, temperature=T, teacher_lse=lse, out=again)
    assert same is again and torch.equal(again, dlogits) and torch.equal(loss2, loss)


def test_the_loss_falls_along_the_gradient_of_the_input():
    """<gradient of the input, v> against the difference of the summed loss along v, through the dequantised head in fp64; the 8-bit rounding of x and
    of the logits' gradient is what keeps them apart (2^-4 an element at most, of either sign)."""
    M, V, K, k, T = 6, 512, 256, 512, 1.0
    head, h, index, value, _, dloss = _setup(M, V, K, k, T, False)
    ws, ws_grad = head.new_workspace(M), head.new_workspace(M, input_grad=True)
    _, _, dlogits, dh = _step(head, h, index, value, None, dloss, T, ws, ws_grad)
    w = fp8_oracle.decode(head.codes.view(torch.uint8).cpu().numpy()) * fp8_oracle._spread(head.scales.cpu().numpy(), V, K)
    from oracle.distill_oracle import distill
    xc, xs = fp8_oracle.quantize(h.double().cpu().numpy(), rows=1)
    x = fp8_oracle.decode(xc) * np.repeat(xs, 128, 1)[:, :K]                 # where the head's product was taken
    v = np.random.default_rng(0).normal(size=x.shape)
    at = lambda e: (distill((x + e * v) @ w.T, index.cpu().numpy(), value.double().cpu().numpy(), T)[0] * dloss.double().cpu().numpy()).sum()
    slope = (at(1e-5) - at(-1e-5)) / 2e-5
    dl = dlogits.double().cpu().numpy()
    big = np.repeat(np.abs(dl).reshape(M, -1, 128).max(2), 128, 1)
    # dlogits as the product sees them: 2^-4 of an element, or 2^-10 of the block's largest; the logits they were taken at are rounded to bf16 (2^-8
    # relative: at most that much of p (1 - p) and of q each, doubled)
    y = np.abs(x @ w.T).max()
    slack = (np.abs(v @ w.T) * (np.maximum(np.abs(dl) * 2.0 ** -4, big * 2.0 ** -10) + 2 * 2.0 ** -8 * y * (np.abs(dl) + big))).sum()
    slack += 2.0 ** -8 * (np.abs(dh.double().cpu().numpy()) * np.abs(v)).sum()
    assert abs((dh.double().cpu().numpy() * v).sum() - slope) <= slack


def test_captured_step_and_two_streams():
    slim = _slim()
    M, V, K, k, T = 33, 3008, 544, 20, 1.5
    head, h, index, value, lse, dloss = _setup(M, V, K, k, T, True)
    ws, ws_grad = head.new_workspace(M), head.new_workspace(M, input_grad=True)
    want = _step(head, h, index, value, lse, dloss, T, ws, ws_grad)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(head, h, index, value, lse, dloss, T, ws, ws_grad)
    keep = h.clone()
    h.zero_()
    graph.replay()
    h.copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    # two streams at once, each with workspaces of its own
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    spaces = [(head.new_workspace(M), head.new_workspace(M, input_grad=True)) for _ in streams]
    torch.cuda.synchronize()
    results = []
    for _ in range(5):
        for s, (a, b) in zip(streams, spaces):
            with torch.cuda.stream(s):
                results.append(_step(head, h, index, value, lse, dloss, T, a, b))
    torch.cuda.synchronize()
    for r in results:
        for a, b in zip(want, r):
            assert torch.equal(a, b)


def test_the_general_path_gives_the_same(monkeypatch):
    slim = _slim()
    M, V, K, k, T = 20, 1040, 288, 7, 1.0
    head, h, index, value, lse, dloss = _setup(M, V, K, k, T, True)
    ws, ws_grad = head.new_workspace(M), head.new_workspace(M, input_grad=True)
    want = _step(head, h, index, value, lse, dloss, T, ws, ws_grad)
    loss, saved = slim.distill_loss(want[0], index, value, temperature=T, teacher_lse=lse)
    grad = slim.distill_grad(want[0], index, value, saved, dloss, temperature=T, teacher_lse=lse)
    out = torch.empty(M, V, device="cuda")
    y32 = head.forward(h, ws, out=out)
    assert y32 is out and torch.equal(head.forward(h, ws, out_dtype=torch.float32), out)
    monkeypatch.setattr(slim, "_host", slim._NoHost)
    for a, b in zip(want, _step(head, h, index, value, lse, dloss, T, ws, ws_grad)):
        assert torch.equal(a, b)
    loss2, saved2 = slim.distill_loss(want[0], index, value, temperature=T, teacher_lse=lse)
    assert torch.equal(loss, loss2) and torch.equal(saved, saved2)
    assert torch.equal(grad, slim.distill_grad(want[0], index, value, saved, dloss, temperature=T, teacher_lse=lse))
    assert torch.equal(out, head.forward(h, ws, out_dtype=torch.float32))
    # what neither path takes
    p = torch.nn.Parameter(want[0].float(), requires_grad=True)
    assert torch.equal(slim.distill_loss(p, index, value)[0], slim.distill_loss(p.detach(), index, value)[0])
    with pytest.raises(TypeError):
        slim.fp8_linear(h, head.codes.view(torch.uint8), head.scales, ws)
