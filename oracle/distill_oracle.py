"""CPU oracle of the distillation loss over a teacher's top logits and of its gradient, in fp64 from the definition; test infrastructure only."""
import numpy as np


def distill(logits, index, value, temperature, lse=None, dloss=None):
    """loss [M], grad [M][V] (of sum(dloss * loss); dloss = 1 if None) and, per row, what error bounds are made of:
    a dict of p [M][V], q (summed per column) [M][V], q_rest [M], p_rest [M].

    The mass outside the entries, and how it is spread, are taken relative to the largest logit outside them: they are right where its
    exponentials relative to the row's maximum leave fp64's range."""
    s = np.asarray(logits, np.float64) / temperature
    M, V = s.shape
    loss, grad = np.zeros(M), np.zeros((M, V))
    P, Q, q_rests, p_rests = np.zeros((M, V)), np.zeros((M, V)), np.zeros(M), np.ones(M)
    for t in range(M):
        present = [j for j in range(index.shape[1]) if 0 <= index[t, j] < V]
        u = np.array([float(value[t, j]) for j in present]) / temperature
        cols = np.array([int(index[t, j]) for j in present], dtype=np.int64)
        if not present or (lse is None and np.all(u == -np.inf)):
            continue
        top = s[t].max()
        with np.errstate(all="ignore"):
            e = np.zeros(V) if top == -np.inf else np.exp(s[t] - top)
            Z = e.sum()
            p = e / Z if Z != 0 else e
            lp = (s[t] - top) - np.log(Z) if Z != 0 else np.full(V, -np.inf)
            if np.isnan(Z):
                lp = np.full(V, np.nan)
            if lse is None:
                w = np.exp(u - u.max())
                q, lq = w / w.sum(), u - u.max() - np.log(w.sum())
            else:
                lq = u - float(lse[t])
                q = np.exp(lq)
            for j in range(len(cols)):
                if q[j] != 0:
                    loss[t] += q[j] * (lq[j] - lp[cols[j]])
                Q[t, cols[j]] += q[j]
            mass = q.sum()
            factor = np.full(V, mass)
            taken = np.zeros(V)
            if lse is not None:
                outside = np.ones(V, bool)
                outside[cols] = False
                p_rest = p[outside].sum()
                top_out = s[t][outside].max(initial=-np.inf)
                e_out = np.where(outside, np.exp(s[t] - top_out), 0.0) if top_out > -np.inf else np.zeros(V)
                q_rest = 1.0 - mass if outside.any() else 0.0
                if q_rest <= min(2.0 ** -22 * (1.0 + abs(float(lse[t]))), 0.5):       # what an fp32 log-sum-exp is off by
                    q_rest = 0.0
                factor += q_rest
                if q_rest > 0:
                    lp_rest = (top_out - top) + np.log(e_out.sum()) - np.log(Z) if top_out > -np.inf else -np.inf
                    loss[t] += q_rest * (np.log(q_rest) - (np.nan if np.isnan(Z) else lp_rest))
                    if top_out > -np.inf:
                        taken = q_rest * e_out / e_out.sum()
                    else:
                        factor[outside] = 0.0
                q_rests[t], p_rests[t] = q_rest, p_rest
            grad[t] = (p * factor - taken - Q[t]) * (1.0 if dloss is None else float(dloss[t])) / temperature
        P[t] = p
    return loss, grad, dict(p=P, q=Q, q_rest=q_rests, p_rest=p_rests)
