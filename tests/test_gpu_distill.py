"""GPU parity: the distillation loss over a teacher's top logits, its gradient and the one-pass step against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle.distill_oracle import distill

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _slim():
    from paper_2405_14917_b200 import binding
    return binding


def _case(M, V, k, kind, T, rest, seed, index_type=torch.int64, value_type=torch.float32):
    g = torch.Generator().manual_seed(seed)
    teacher = torch.randn(M, V, generator=g) * 3
    student = (teacher + torch.randn(M, V, generator=g)).to(TYPES[kind])
    value, index = torch.topk(teacher, min(k, V), dim=1)
    lse = torch.logsumexp(teacher.double() / T, 1).float() if rest else None
    dloss = torch.rand(M, generator=g) + 0.5
    return student, index.to(index_type), value.to(value_type), lse, dloss


def _bounds(student, parts, grad_ref, dloss, T, kind):
    """Error bounds of the loss and of every gradient element.

    A log-probability carries, in units of 1: the rounding of log2(e)/T, of s - m and of their product (2^-24 each of D =
    (m - s) log2(e)/T, at the column and, weighted, in the sum), ex2 (2^-22, and again where a partial sum is brought to the row's maximum: three
    times at most), and fp32 sums of positive terms: chains of at most 32 + 1 additions in a thread per pass, 5 in its warp, 4 over the warps, 3 over a
    cluster and 32 + 5 over the entries, 2^-24 each; 1/Z within 2^-23.  The rest is fp64.  D is cut at 150: beyond, p is 0 in fp32."""
    s = student.double().numpy()
    finite = np.where(np.isfinite(s), s, -np.inf)
    with np.errstate(invalid="ignore"):
        D = np.minimum(np.nan_to_num((finite.max(1, keepdims=True) - finite) * 1.4427 / T, nan=150.0, posinf=150.0), 150.0)
    passes = 1 + s.shape[1] // (512 * 8 * (4 if kind == "fp32" else 8))
    # in the sum an element of distance D weighs 2^-D, and D 2^-D < 0.54: the columns of a row add up to less than 0.54 V / Z of it, and Z >= 1
    p = parts["p"]
    in_sum = (p * D).sum(1)
    d_sum = (33 * passes + 49) * 2.0 ** -24 + 3 * 2.0 ** -22 + 2.0 ** -23 + 4 * 2.0 ** -24 * in_sum
    d_col = d_sum[:, None] + 4 * 2.0 ** -24 * D + 2.0 ** -22
    q, q_rest, p_rest = parts["q"], parts["q_rest"], parts["p_rest"]
    ratio = np.divide(q_rest, p_rest, out=np.zeros_like(q_rest), where=p_rest > 0)
    p_listed_err = (p * d_col * (q > 0)).sum(1)
    loss_tol = (q * d_col).sum(1) + ratio * p_listed_err + q_rest * d_sum
    half = torch.finfo(TYPES[kind]).eps / 2
    scale = np.abs(dloss.double().numpy())[:, None] / T
    mass = q.sum(1) + q_rest
    grad_tol = half * np.abs(grad_ref) + scale * (p * (mass + ratio)[:, None] * (2 * d_col + 2 * d_sum[:, None]) + 1e-12 * q)
    grad_tol += {"fp16": 2.0 ** -25, "bf16": 1e-38, "fp32": 1e-37}[kind]      # half of fp16's smallest step; what ex2 flushes
    return loss_tol + 2.0 ** -24 * 1e-6, grad_tol


def _check(student, index, value, lse, dloss, T, kind, got_loss, got_grad):
    loss, grad, parts = distill(student.double().numpy(), index.numpy(), value.double().numpy(), T,
                                None if lse is None else lse.double().numpy(), dloss.double().numpy())
    loss_tol, grad_tol = _bounds(student, parts, grad, dloss, T, kind)
    loss_tol += 2.0 ** -24 * np.abs(np.where(np.isfinite(loss), loss, 0))
    if got_loss is not None:
        got = got_loss.cpu().double().numpy()
        ok = np.isfinite(loss)
        assert (got[~ok] == loss[~ok]).all() or np.isnan(loss[~ok]).any()
        err = np.abs(got[ok] - loss[ok])
        assert (err <= loss_tol[ok]).all(), (err / loss_tol[ok]).max()
    if got_grad is not None:
        err = np.abs(got_grad.cpu().double().numpy() - grad)
        assert (err <= grad_tol).all(), (err / grad_tol).max()


def _run_all(student, index, value, lse, dloss, T, kind, dev="cuda"):
    slim = _slim()
    s, i, v, d = student.to(dev), index.to(dev), value.to(dev), dloss.to(dev)
    z = None if lse is None else lse.to(dev)
    loss, saved = slim.distill_loss(s, i, v, temperature=T, teacher_lse=z)
    grad = slim.distill_grad(s, i, v, saved, d, temperature=T, teacher_lse=z)
    _check(student, index, value, lse, dloss, T, kind, loss, grad)
    loss1, grad1 = slim.distill_step(s, i, v, d, temperature=T, teacher_lse=z)
    _check(student, index, value, lse, dloss, T, kind, loss1, grad1)
    return loss1, grad1


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("M,V,k,T", [(1, 1, 1, 1.0), (2, 2, 1, 1.0), (3, 7, 5, 2.0), (5, 33, 40, 0.5), (4, 1000, 128, 1.5), (3, 4099, 8, 1.0),
                                     (300, 515, 20, 4.0), (1, 32000, 64, 1.0), (40, 32001, 3, 2.0)])
def test_loss_gradient_and_step(M, V, k, T, kind, rest):
    _run_all(*_case(M, V, k, kind, T, rest, seed=M + V + k), T, kind)


@pytest.mark.parametrize("M,V,kind,rest", [(2, 152064, "bf16", True), (1, 262145, "fp16", True), (1, 131073, "fp32", False), (300, 40001, "fp16", True),
                                           (1, 600003, "fp32", True), (2, 2097152, "fp32", True), (1, 2097152, "fp16", True),
                                           (1, 2097151, "fp32", False), (2, 1048577, "bf16", True)])
def test_rows_longer_than_a_cta_or_a_cluster_holds(M, V, kind, rest):
    _run_all(*_case(M, V, 33, kind, 1.0, rest, seed=V), 1.0, kind)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("M,V,k", [(297, 1000, 5), (900, 333, 1), (450, 8191, 70), (310, 20003, 300), (200, 70001, 33)])
def test_many_rows(M, V, k, kind, rest):
    """More rows than CTAs, or clusters, at once; rows off 16 bytes; among them every kind of row that is not the ordinary one."""
    student, index, value, lse, dloss = _case(M, V, k, kind, 1.0, rest, M + V)
    index[3, :] = -1
    student[3, :] = float("nan")
    index[M - 1, :] = V
    index[5, k // 2] = -1
    if k > 2:
        index[7, 2] = index[7, 0]
        index[M - 2, :] = index[M - 2, 0]
        if rest:
            value[M - 2, :] -= 7.0
    student[11, ::2] = -float("inf")
    student[12, :] = -float("inf")
    value[13, :] = -float("inf")
    loss, grad = _run_all(student, index, value, lse, dloss, 1.0, kind)
    assert (loss[[3, M - 1]] == 0).all() and (grad[[3, M - 1]] == 0).all()


def test_not_finite_rows_among_many_stay_alone():
    student, index, value, lse, dloss = _case(400, 5001, 6, "bf16", 1.0, True, 8)
    student[1, 77] = float("nan")
    student[399, 4001] = float("inf")
    loss, grad = _slim().distill_step(student.cuda(), index.cuda(), value.cuda(), dloss.cuda(), teacher_lse=lse.cuda())
    assert torch.isnan(loss[[1, 399]]).all() and torch.isnan(grad[[1, 399]]).all()
    keep = [i for i in range(400) if i not in (1, 399)]
    _check(student[keep], index[keep], value[keep], lse[keep], dloss[keep], 1.0, "bf16", loss[keep], grad[keep])


@pytest.mark.parametrize("index_type", [torch.int32, torch.int64])
@pytest.mark.parametrize("value_type", [torch.float16, torch.bfloat16, torch.float32])
def test_types_of_the_entries(index_type, value_type):
    _run_all(*_case(6, 700, 12, "fp32", 1.0, True, 5, index_type, value_type), 1.0, "fp32")


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("k", [513, 1024])
def test_many_entries(k, rest):
    _run_all(*_case(3, 5000, k, "bf16", 1.0, rest, k), 1.0, "bf16")


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
def test_absent_and_repeated_entries(kind, rest):
    student, index, value, lse, dloss = _case(6, 300, 7, kind, 1.0, rest, 11)
    index[0, 2] = -1
    index[1, :] = -1                       # nothing present
    index[2, 5] = 300                      # past the end: absent
    index[3, 4] = index[3, 1]              # one column twice
    index[4, :] = index[4, 0]              # and seven times
    value[5, 3] = -np.inf
    if rest:
        value[4, :] -= 3.0                 # seven entries of one column that stay below 1 together
    loss, grad = _run_all(student, index, value, lse, dloss, 1.0, kind)
    assert loss[1] == 0 and (grad[1] == 0).all()


def test_rows_whose_values_leave_nothing():
    student, index, value, _, dloss = _case(4, 100, 5, "fp32", 1.0, False, 3)
    value[1, :] = -np.inf
    index[2, :] = -1
    student[2, :] = float("nan")           # a padded row may hold anything
    student[1, 5] = float("inf")
    loss, grad = _slim().distill_step(student.cuda(), index.cuda(), value.cuda(), dloss.cuda())
    assert (loss[1:3] == 0).all() and (grad[1:3] == 0).all()
    keep = [0, 3]
    _check(student[keep], index[keep], value[keep], None, dloss[keep], 1.0, "fp32", loss[keep], grad[keep])


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
def test_masked_logits(kind, rest):
    """Columns at minus infinity or at the type's lowest value, outside the entries, inside them, and all of a row."""
    T = 1.0
    student, index, value, lse, dloss = _case(7, 1000, 6, kind, T, rest, 21)
    low = torch.finfo(TYPES[kind]).min
    listed = torch.zeros(7, 1000, dtype=torch.bool).scatter_(1, index, True)
    student[0, 500:][~listed[0, 500:]] = -float("inf")
    student[1, 300:][~listed[1, 300:]] = low
    student[2, index[2, 1]] = -float("inf")       # p = 0 where the teacher has mass
    student[3, :] = -float("inf")
    student[4, :] = low                           # uniform
    student[5][~listed[5]] = -float("inf")        # nothing outside the entries
    loss, grad = _run_all(student, index, value, lse, dloss, T, kind)
    assert loss[2] == float("inf") and loss[3] == float("inf")
    assert torch.isfinite(grad).all()


def test_not_finite_rows_stay_alone():
    student, index, value, lse, dloss = _case(5, 5000, 6, "bf16", 1.0, True, 8)
    student[1, 77] = float("nan")
    student[3, 4001] = float("inf")
    loss, grad = _slim().distill_step(student.cuda(), index.cuda(), value.cuda(), dloss.cuda(), teacher_lse=lse.cuda())
    assert torch.isnan(loss[[1, 3]]).all() and torch.isnan(grad[[1, 3]]).all()
    keep = [0, 2, 4]
    _check(student[keep], index[keep], value[keep], lse[keep], dloss[keep], 1.0, "bf16", loss[keep], grad[keep])


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
@pytest.mark.parametrize("V,ld,off,ldg,offg", [(1000, 1003, 1, 1000, 0), (1000, 1008, 8, 1016, 8), (997, 1200, 3, 1005, 2), (40000, 40001, 5, 40001, 5)])
def test_strided_rows(V, ld, off, ldg, offg, kind):
    student, index, value, lse, dloss = _case(5, V, 9, kind, 1.0, True, ld)
    wide = torch.full((5, ld + off), 7.0, dtype=TYPES[kind], device="cuda")
    wide[:, off:off + V] = student.cuda()
    s = torch.as_strided(wide, (5, V), (ld + off, 1), off)
    out_wide = torch.full((5, ldg + offg + 4), 3.0, dtype=TYPES[kind], device="cuda")
    out = torch.as_strided(out_wide, (5, V), (ldg + offg + 4, 1), offg)
    before = out_wide.clone()
    loss, grad = _slim().distill_step(s, index.cuda(), value.cuda(), dloss.cuda(), teacher_lse=lse.cuda(), out=out)
    assert grad is out
    _check(student, index, value, lse, dloss, 1.0, kind, loss, out)
    torch.as_strided(before, out.shape, out.stride(), offg).copy_(out)
    assert torch.equal(before, out_wide)                       # nothing beside the rows was written


@pytest.mark.parametrize("M,V", [(3, 1001), (2, 40000), (1, 150001), (300, 600), (700, 4001), (200, 70001)])
@pytest.mark.parametrize("step", [False, True])
def test_gradient_in_place_of_the_logits(M, V, step):
    slim = _slim()
    student, index, value, lse, dloss = _case(M, V, 16, "bf16", 1.0, True, V)
    s, i, v, z, d = student.cuda(), index.cuda(), value.cuda(), lse.cuda(), dloss.cuda()
    want = slim.distill_step(s, i, v, d, teacher_lse=z)[1]
    if step:
        slim.distill_step(s, i, v, d, teacher_lse=z, out=s)
    else:
        _, saved = slim.distill_loss(s, i, v, teacher_lse=z)
        want = slim.distill_grad(s, i, v, saved, d, teacher_lse=z)
        slim.distill_grad(s, i, v, saved, d, teacher_lse=z, out=s)
    assert torch.equal(s, want)


def test_repeatable_captured_and_on_another_stream():
    slim = _slim()
    student, index, value, lse, dloss = _case(9, 33000, 32, "bf16", 2.0, True, 1)
    s, i, v, z, d = student.cuda(), index.cuda(), value.cuda(), lse.cuda(), dloss.cuda()
    out = torch.empty_like(s)
    loss, _ = slim.distill_step(s, i, v, d, temperature=2.0, teacher_lse=z, out=out)
    for _ in range(3):
        again, grad = slim.distill_step(s, i, v, d, temperature=2.0, teacher_lse=z)
        assert torch.equal(again, loss) and torch.equal(grad, out)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            l2, g2 = slim.distill_step(s, i, v, d, temperature=2.0, teacher_lse=z)
    other = _case(9, 33000, 32, "bf16", 2.0, True, 2)
    for new, buf in zip(other, (s, i, v, z, d)):
        buf.copy_(new)
    graph.replay()
    torch.cuda.synchronize()
    _check(*other, 2.0, "bf16", l2, g2)


def test_refusals():
    slim = _slim()
    student, index, value, lse, dloss = _case(3, 50, 4, "fp16", 1.0, True, 1)
    s, i, v, z, d = student.cuda(), index.cuda(), value.cuda(), lse.cuda(), dloss.cuda()
    for T in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(slim.SlimError):
            slim.distill_loss(s, i, v, temperature=T)
    with pytest.raises(TypeError):
        slim.distill_loss(student, i, v)                       # on the host
    with pytest.raises(TypeError):
        slim.distill_loss(s.double(), i, v)
    with pytest.raises(TypeError):
        slim.distill_loss(s, i.float(), v)
    with pytest.raises(ValueError):
        slim.distill_loss(s, i[:2], v)
    with pytest.raises(ValueError):
        slim.distill_loss(s.t(), i, v)                         # columns, not rows, are contiguous
    with pytest.raises(ValueError):
        slim.distill_loss(s[:1].expand(3, 50), i, v)
    with pytest.raises(ValueError):
        slim.distill_loss(s, i, v, teacher_lse=z[:2])
    with pytest.raises(ValueError):
        slim.distill_step(s, i, v, d[:2])
    with pytest.raises((TypeError, ValueError)):
        slim.distill_step(s, i, v, d, out=torch.empty(3, 50, device="cuda"))
    with pytest.raises(slim.SlimError):
        slim.distill_loss(torch.zeros(1, 50, device="cuda").half(), torch.zeros(1, 1025, dtype=torch.int64, device="cuda"), torch.zeros(1, 1025, device="cuda"))
    loss, saved = slim.distill_loss(s[:0], i[:0], v[:0])       # no row: nothing to do
    assert loss.shape == (0,) and slim.distill_grad(s[:0], i[:0], v[:0], saved, d[:0]).shape == (0, 50)


def test_rows_farther_apart_than_32_bits_count():
    """Row strides whose offsets pass 2^31 elements, in a buffer that is never read beside the rows."""
    V, ld = 4003, 1_150_000_001
    student, index, value, lse, dloss = _case(3, V, 9, "fp16", 1.0, True, 4)
    buf = torch.empty(2 * ld + V, dtype=torch.float16, device="cuda")
    s = torch.as_strided(buf, (3, V), (ld, 1), 0)
    s.copy_(student)
    loss, saved = _slim().distill_loss(s, index.cuda(), value.cuda(), teacher_lse=lse.cuda())
    grad = _slim().distill_grad(s, index.cuda(), value.cuda(), saved, dloss.cuda(), teacher_lse=lse.cuda(), out=s)
    assert grad is s
    _check(student, index, value, lse, dloss, 1.0, "fp16", loss, grad)


def test_a_batch_of_more_than_32_bits_of_logits():
    """The many-rows kernel on 70000 x 32000 logits, the gradient in their place: rows from the far end against the oracle."""
    M, V, k = 70000, 32000, 4
    g = torch.Generator(device="cuda").manual_seed(5)
    s = torch.empty(M, V, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    index = torch.randint(0, V, (M, k), generator=g, device="cuda", dtype=torch.int32)
    value = torch.randn(M, k, generator=g, device="cuda") + 3
    dloss = torch.ones(M, device="cuda")
    rows = [0, 1, 67107, 67108, 67109, 69998, 69999]          # 67108 x 32000 is where 2^31 lies
    student = s[rows].cpu()
    loss, grad = _slim().distill_step(s, index, value, dloss, out=s)
    _check(student, index[rows].cpu(), value[rows].cpu(), None, dloss[rows].cpu(), 1.0, "bf16", loss[rows], grad[rows])
