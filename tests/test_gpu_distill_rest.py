"""GPU parity: the distillation loss with the rest class where the columns outside the entries have next to nothing of the student's mass (sharp
students, low temperatures, masks), or logits that are not finite, against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle.distill_oracle import distill

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _slim():
    from paper_2405_14917_b200 import binding
    return binding


def _far(M, V, k, kind, T, seed):
    """Rows whose unlisted logits lie below the listed ones by 2 T to 900 T (what the type holds of it), the first by 84 to 92 T; the last row's at a
    mask's value (fp16's lowest, a 64th of the others').  The teacher has 0.1 to 50 % of its mass outside the entries."""
    g = torch.Generator().manual_seed(seed)
    index = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(M)])
    gap = T * torch.exp(torch.rand(M, 1, generator=g) * np.log(450.0)) * 2
    near = min(M, 9)
    gap[:near, 0] = T * torch.linspace(84.0, 92.0, 9)[:near]
    s = torch.randn(M, V, generator=g) * T - gap + 4 * T
    s.scatter_(1, index, 4 * T + torch.randn(M, k, generator=g) * T)
    student = s.to(TYPES[kind])
    if M > 1:
        student[-1] = torch.finfo(TYPES[kind]).min / (1 if kind == "fp16" else 64)
        student[-1, index[-1]] = (torch.randn(k, generator=g) * T).to(TYPES[kind])
    value = torch.randn(M, k, generator=g) * T * 2
    kept = 1.0 - 10.0 ** (-0.3 - 2.7 * torch.rand(M, generator=g, dtype=torch.float64))
    lse = (torch.logsumexp(value.double() / T, 1) - torch.log(kept)).float()
    dloss = 1.0 + torch.rand(M, generator=g)
    return student, index, value, lse, dloss


def _check(student, index, value, lse, dloss, T, kind, got_loss, got_grad):
    """Bounds in the relative error of every factor, u = 2^-24.  D: distance from the maximum that an exponential is taken from, in units of 1: it carries
    the roundings of log2(e) / T, of the difference and of the product, 3 u D; ex2 is within 4 u, the reciprocal within 2 u, and a value flushed by it is less than
    2^-126.  A sum over the columns: those of each term, one addition of u per step of a chain (at most 33 per pass of a thread, 49 across threads), and
    three times an ex2 where partial sums come to one maximum (a further one for Z, the sum of two parts).
    p' is A R / Z (A = 2^((m' - m) c): m' the largest logit outside, R the sum relative to it), or 1 less the set's mass where that is under a half."""
    s, ix, z = student.double().numpy(), index.numpy(), lse.double().numpy()
    loss, grad, parts = distill(s, ix, value.double().numpy(), T, z, dloss.double().numpy())
    u = 2.0 ** -24
    M, V = s.shape
    p, q, q_rest = parts["p"], parts["q"], parts["q_rest"]
    listed = np.zeros((M, V), bool)
    for t in range(M):
        listed[t, ix[t][(ix[t] >= 0) & (ix[t] < V)]] = True
    with np.errstate(all="ignore"):
        top, top_out = s.max(1), np.where(listed, -np.inf, s).max(1)
        D_in, D_out, A_D = (top[:, None] - s) / T, (top_out[:, None] - s) / T, (top - top_out) / T
        w = np.where(listed, 0.0, np.exp(-D_out))
        R = w.sum(1)
        w /= R[:, None]
    passes = 1 + V // (512 * 8 * (4 if kind == "fp32" else 8))
    chain = (33 * passes + 49) * u + 3 * 4 * u
    in_R = chain + (w * np.where(listed, 0.0, np.minimum(D_out, 1e4))).sum(1) * 3 * u
    in_Z = chain + 4 * u + (p * np.minimum(D_in, 1e4)).sum(1) * 3 * u
    in_set = (p * listed).sum(1)
    p_rest = 1.0 - in_set
    p_rest = np.where(in_set < 0.5, p_rest, np.exp(np.minimum(np.log(np.maximum(p_rest, 1e-300)), -A_D + np.log(R) + 1e-3)))
    d_listed = np.minimum(D_in, 1e300) * 3 * u + in_Z[:, None]                       # of log p at an entry
    set_err = (p * listed * (d_listed + 4 * u)).sum(1)
    log_rest = np.where(in_set < 0.5, set_err / np.maximum(1 - in_set, 0.5), A_D * 3 * u + in_R + in_Z)
    loss_tol = (q * np.where(q > 0, d_listed, 0)).sum(1) + q_rest * log_rest + u * np.abs(loss)
    half = torch.finfo(TYPES[kind]).eps / 2
    scale = (np.abs(dloss.double().numpy()) / T)[:, None]
    # outside: (p' - q') w, all of it; in the set: p - q
    A_rel = np.minimum(A_D, 150) * 3 * u + 4 * u
    diff_err = np.where(in_set < 0.5, set_err + 2 * u, p_rest * (A_rel + in_R + in_Z + 6 * u) + q_rest * 2 * u + 2.0 ** -125)
    w_err = w * (np.where(listed, 0.0, np.minimum(D_out, 150)) * 3 * u + 4 * u + in_R[:, None] + 5 * u) + 2.0 ** -126
    outside = w * diff_err[:, None] + np.abs(p_rest - q_rest)[:, None] * w_err
    inside = p * (np.minimum(D_in, 150) * 3 * u + in_Z[:, None] + 8 * u) + 2.0 ** -125 + 1e-12 * q
    grad_tol = half * np.abs(grad) * 1.01 + scale * np.where(listed, inside, outside)
    grad_tol += {"fp16": 2.0 ** -25, "bf16": 2.0 ** -134, "fp32": 2.0 ** -149}[kind]
    if got_loss is not None:
        err = np.abs(got_loss.cpu().double().numpy() - loss)
        assert (err <= loss_tol).all(), (err / loss_tol).max()
    if got_grad is not None:
        err = np.abs(got_grad.cpu().double().numpy() - grad)
        assert (err <= grad_tol).all(), (err / grad_tol).max()


def _calls(student, index, value, lse, dloss, T):
    slim = _slim()
    s, i, v, z, d = student.cuda(), index.cuda(), value.cuda(), lse.cuda(), dloss.cuda()
    loss, saved = slim.distill_loss(s, i, v, temperature=T, teacher_lse=z)
    grad = slim.distill_grad(s, i, v, saved, d, temperature=T, teacher_lse=z)
    return loss, grad, *slim.distill_step(s, i, v, d, temperature=T, teacher_lse=z)


# a CTA per row, a cluster per row, longer rows than either holds; and more rows than CTAs (pairs of CTAs) at once
SHAPES = [(12, 700, 5), (3, 40001, 64), (2, 300007, 33), (400, 1001, 70), (300, 40001, 9)]


@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("T", [0.1, 0.25, 1.0])
@pytest.mark.parametrize("M,V,k", SHAPES)
def test_loss_where_the_student_leaves_the_rest_next_to_nothing(M, V, k, T, kind):
    case = _far(M, V, k, kind, T, V)
    loss, _, loss1, _ = _calls(*case, T)
    assert torch.isfinite(loss).all() and torch.isfinite(loss1).all()
    _check(*case, T, kind, loss, None)
    _check(*case, T, kind, loss1, None)


@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("T", [0.1, 0.25, 1.0])
@pytest.mark.parametrize("M,V,k", SHAPES)
def test_gradient_where_the_student_leaves_the_rest_next_to_nothing(M, V, k, T, kind):
    case = _far(M, V, k, kind, T, V + 1)
    _, grad, _, grad1 = _calls(*case, T)
    _check(*case, T, kind, None, grad)
    _check(*case, T, kind, None, grad1)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("M,V,k", SHAPES)
def test_gradient_there_under_a_large_weight(M, V, k, kind):
    """dloss / T of 1e6 (a loss scale; a low temperature): finite, as the definition's."""
    T = 0.1
    student, index, value, lse, dloss = _far(M, V, k, kind, T, V + 2)
    case = (student, index, value, lse, dloss * 65536)
    _, grad, _, grad1 = _calls(*case, T)
    assert torch.isfinite(grad).all() and torch.isfinite(grad1).all()
    _check(*case, T, kind, None, grad)
    _check(*case, T, kind, None, grad1)


@pytest.mark.parametrize("M,V,k,kind", [(200, 32000, 160, "fp32"), (200, 32000, 161, "fp32"), (200, 60000, 300, "bf16"), (160, 65001, 321, "fp16"),
                                        (300, 30001, 330, "bf16"), (320, 4001, 770, "fp32")])
def test_many_entries_in_many_rows(M, V, k, kind):
    """Rows of one CTA and of a pair, on both sides of what their shared memory and the choice of kernel take of entries."""
    case = _far(M, V, k, kind, 1.0, k)
    loss, grad, loss1, grad1 = _calls(*case, 1.0)
    _check(*case, 1.0, kind, loss, grad)
    _check(*case, 1.0, kind, loss1, grad1)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("M,V,k", [(4, 700, 5), (2, 40001, 64), (400, 1001, 7)])
def test_plus_infinity_in_a_listed_column(M, V, k, kind, rest):
    """NaN throughout its row (loss, every gradient), whatever the teacher has there, and in no other row."""
    slim = _slim()
    g = torch.Generator().manual_seed(5)
    student, value, dloss = torch.randn(M, V, generator=g).to(TYPES[kind]), torch.randn(M, k, generator=g), torch.rand(M, generator=g) + 0.5
    index = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(M)])
    lse = torch.logsumexp(value, 1) + 0.5
    for row, j in ((0, 0), (M - 1, k - 1)):
        student[row, index[row, j]] = float("inf")
    value[M - 1, :k - 1] = -float("inf")
    if rest:
        value[0] = -float("inf")                     # the entries have nothing: all of the teacher's mass is in the rest
    s, i, v, d = student.cuda(), index.cuda(), value.cuda(), dloss.cuda()
    z = lse.cuda() if rest else None
    loss, saved = slim.distill_loss(s, i, v, teacher_lse=z)
    grad = slim.distill_grad(s, i, v, saved, d, teacher_lse=z)
    loss1, grad1 = slim.distill_step(s, i, v, d, teacher_lse=z)
    for l, g in ((loss, grad), (loss1, grad1)):
        assert torch.isnan(l[[0, M - 1]]).all() and torch.isfinite(l[1:M - 1]).all()
        assert torch.isnan(g[[0, M - 1]]).all() and torch.isfinite(g[1:M - 1]).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("M", [8, 400])
def test_losses_that_are_not_finite_are_the_definitions(M, rest):
    """+infinity where the teacher has mass and the student none; NaN where a logit is NaN or +infinity: row by row as the oracle has them."""
    student, index, value, lse, dloss = _far(M, 1500, 6, "fp32", 1.0, 9)
    listed = torch.zeros(M, 1500, dtype=torch.bool).scatter_(1, index, True)
    student[0][~listed[0]] = -float("inf")           # nothing for the rest
    student[1, index[1, 2]] = -float("inf")          # nothing for an entry
    student[2, :] = -float("inf")
    student[3, index[3, 1]] = float("nan")
    student[4, 700 + int(listed[4, 700])] = float("inf")
    student[5, index[5, 0]] = float("inf")
    s, i, v, d = student.cuda(), index.cuda(), value.cuda(), dloss.cuda()
    z = lse if rest else None
    want, want_grad, _ = distill(student.double().numpy(), index.numpy(), value.double().numpy(), 1.0, None if z is None else z.double().numpy(),
                                 dloss.double().numpy())
    odd = ~np.isfinite(want)
    assert odd.sum() == (6 if rest else 5)
    for loss, grad in (_slim().distill_step(s, i, v, d, teacher_lse=None if z is None else z.cuda()),
                       (_slim().distill_loss(s, i, v, teacher_lse=None if z is None else z.cuda())[0], None)):
        got = loss.cpu().double().numpy()
        np.testing.assert_array_equal(got[odd], want[odd])
        assert np.isfinite(got[~odd]).all()
        if grad is not None:
            np.testing.assert_array_equal(np.isnan(grad.cpu().numpy()), np.isnan(want_grad))


def _masked(M, V, k, T, mask, seed):
    """A vocabulary of which all but the k entries are masked, teacher and student alike; the teacher's log-sum-exp as torch takes it, in fp32."""
    g = torch.Generator().manual_seed(seed)
    index = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(M)])
    value = torch.randn(M, k, generator=g) * 5 + 40 * torch.randn(M, 1, generator=g)
    teacher = torch.full((M, V), mask).scatter_(1, index, value)
    student = torch.full((M, V), mask).scatter_(1, index, value + torch.randn(M, k, generator=g))
    return student, index, value, torch.logsumexp(teacher / T, 1), torch.rand(M, generator=g) + 0.5


@pytest.mark.parametrize("mask", [-float("inf"), torch.finfo(torch.float32).min, -1e4])
@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("M,V,k", [(250, 700, 8), (1000, 1001, 40), (60, 40001, 3)])
def test_a_vocabulary_masked_outside_the_entries(M, V, k, T, mask):
    """All of the teacher's mass is listed: what 1 - sum q is off by is the rounding of its log-sum-exp, and counts as nothing.  So the loss is the KL over
    the entries, in 64 bits here, and outside nothing has a gradient.  A log-sum-exp that is off by at most 2^-22 (1 + |lse|) shifts log q by that much."""
    student, index, value, lse, dloss = _masked(M, V, k, T, mask, V + k)
    lq, s = value.double() / T - lse.double()[:, None], torch.gather(student, 1, index).double() / T
    lp = torch.log_softmax(s, 1)
    q = torch.exp(lq)
    assert (1.0 - q.sum(1) > 0).sum() > M // 5       # the case is there
    want = (q * (lq - lp)).sum(1)
    # log p's error, as in _check: distances of at most some 60 units / T, a chain of few terms of note
    D = (s.max(1, keepdim=True).values - s)
    u = 2.0 ** -24
    tol = (q * (D * 3 * u)).sum(1) + (33 * 2 + 49 + 30) * u + (torch.exp(lp) * D).sum(1) * 3 * u + u * want.abs()
    loss, grad, loss1, grad1 = _calls(student, index, value, lse, dloss, T)
    for l, gr in ((loss, grad), (loss1, grad1)):
        err = (l.cpu().double() - want).abs()
        assert (err <= tol).all(), (err / tol).max()
        assert (gr.cpu().scatter(1, index, 0.0) == 0).all()
        inside = (torch.exp(lp) * q.sum(1, keepdim=True) - q) * dloss.double()[:, None] / T
        err = (torch.gather(gr.cpu(), 1, index).double() - inside).abs()
        bound = (torch.exp(lp) * (D.clamp(max=150) * 3 * u + tol[:, None] + 150 * u) + 1e-12) * dloss.double()[:, None] / T + u * inside.abs() + 2.0 ** -120
        assert (err <= bound).all(), (err / bound).max()


@pytest.mark.parametrize("M", [6, 400])
def test_a_rest_above_the_rounding_of_the_log_sum_exp_counts(M):
    """Just more than 2^-22 (1 + |lse|) outside the entries: the definition's loss, with all of it."""
    student, index, value, lse, dloss = _far(M, 1000, 8, "fp32", 1.0, 3)
    value += 30.0 * torch.randn(M, 1, generator=torch.Generator().manual_seed(1))
    exact = torch.logsumexp(value.double(), 1)
    lse = (exact + 2.0 ** -20 * (1 + exact.abs())).float()
    rest = 1 - torch.exp(value.double() - lse.double()[:, None]).sum(1)
    assert (rest > 2.0 ** -22 * (1 + lse.double().abs())).all() and (rest < 1e-3).all()
    loss, grad, loss1, grad1 = _calls(student, index, value, lse, dloss, 1.0)
    _check(student, index, value, lse, dloss, 1.0, "fp32", loss, grad)
    _check(student, index, value, lse, dloss, 1.0, "fp32", loss1, grad1)
