"""The distillation oracle against closed forms, brute force and differences (CPU)."""
import numpy as np
import pytest

from oracle.distill_oracle import distill
from oracle.slim_oracle import softmax_kl


def _case(M, V, k, seed=0):
    rng = np.random.default_rng(seed)
    teacher = rng.normal(0, 2, (M, V))
    student = teacher + rng.normal(0, 1, (M, V))
    index = np.argsort(-teacher, axis=1)[:, :k]
    return student, teacher, index, np.take_along_axis(teacher, index, 1)


@pytest.mark.parametrize("rest", [False, True])
def test_all_columns_listed_is_the_kl_of_the_search(rest):
    student, teacher, index, value = _case(4, 33, 33)       # with the rest: no column is left to be in it
    T = 1.0
    lse = np.log(np.exp(teacher / T).sum(1)) if rest else None
    loss, _, _ = distill(student, index, value, T, lse)
    np.testing.assert_allclose(loss, softmax_kl(teacher, student), rtol=1e-10)


def test_the_rest_is_one_class():
    student, teacher, index, value = _case(3, 9, 4)
    T = 2.0
    loss, _, _ = distill(student, index, value, T, np.log(np.exp(teacher / T).sum(1)))
    for t in range(3):
        p, q = np.exp(student[t] / T), np.exp(teacher[t] / T)
        p, q = p / p.sum(), q / q.sum()
        pc, qc = np.append(p[index[t]], 1 - p[index[t]].sum()), np.append(q[index[t]], 1 - q[index[t]].sum())
        assert abs(loss[t] - (qc * np.log(qc / pc)).sum()) < 1e-12


@pytest.mark.parametrize("rest,dup,T", [(False, False, 1.0), (True, False, 1.7), (False, True, 2.0), (True, True, 1.0)])
def test_gradient_against_differences(rest, dup, T):
    student, teacher, index, value = _case(3, 17, 5, seed=2)
    lse = np.log(np.exp(teacher / T).sum(1)) if rest else None
    index = index.copy()
    index[0, 3] = -1
    index[2, :] = 99
    if dup:
        index[1, 4] = index[1, 2]
    dloss = np.array([1.0, -0.5, 3.0])
    _, grad, _ = distill(student, index, value, T, lse, dloss)
    h = 1e-5
    for v in range(17):
        up, down = student.copy(), student.copy()
        up[:, v] += h
        down[:, v] -= h
        num = dloss * (distill(up, index, value, T, lse)[0] - distill(down, index, value, T, lse)[0]) / (2 * h)
        np.testing.assert_allclose(grad[:, v], num, atol=1e-9)
    assert (grad[2] == 0).all()
    np.testing.assert_allclose(grad.sum(1), 0, atol=1e-12)


def test_a_log_sum_exp_in_fp32_makes_no_rest():
    """All of the teacher's mass listed: what its rounded log-sum-exp leaves or adds is no class of its own, also where the student has nothing there."""
    student, teacher, index, value = _case(200, 40, 6, seed=4)
    rows = np.arange(200)[:, None]
    masked_teacher, masked_student = np.full_like(teacher, -np.inf), np.full_like(student, -np.inf)
    masked_teacher[rows, index], masked_student[rows, index] = value, student[rows, index]
    lse = np.log(np.exp(masked_teacher).sum(1)).astype(np.float32)
    assert (np.exp(value - lse[:, None].astype(np.float64)).sum(1) < 1).sum() > 50
    loss, grad, parts = distill(masked_student, index, value, 1.0, lse)
    want, _, _ = distill(student[rows, index], np.tile(np.arange(6), (200, 1)), value, 1.0)
    np.testing.assert_allclose(loss, want, atol=1e-5)
    assert (parts["q_rest"] == 0).all() and np.isfinite(grad).all()
    # and a little more than that is one
    loss, _, parts = distill(student, index, value, 1.0, np.log(np.exp(value).sum(1)) + 1e-5)
    np.testing.assert_allclose(parts["q_rest"], 1e-5, rtol=1e-2)
