"""CPU oracle of the distillation loss over a teacher's top logits and of its gradient, in fp64 from the definition; test infrastructure only."""
import numpy as np


def distill(logits, index, value, temperature, lse=None, dloss=None):
    """loss [M], grad [M][V] (of sum(dloss * loss); dloss = 1 if None) and, per row, what error bounds are made of:
    a dict of p [M][V], q (summed per column) [M][V], q_rest [M], p_rest [M]."""
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
            e = np.exp(s[t] - top) if top > -np.inf else np.zeros(V)
            Z = e.sum()
            p = e / Z if Z != 0 else e
            lp = np.where(p > 0, (s[t] - top) - np.log(Z), -np.inf) if Z != 0 else np.full(V, -np.inf)
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
            if lse is not None:
                outside = np.ones(V, bool)
                outside[cols] = False
                p_rest = p[outside].sum()
                q_rest = max(0.0, 1.0 - mass) if outside.any() else 0.0
                factor += q_rest
                if q_rest > 0:
                    loss[t] += q_rest * (np.log(q_rest) - np.log(p_rest))
                    factor[outside] = factor[outside] - q_rest / p_rest if p_rest > 0 else 0.0
                q_rests[t], p_rests[t] = q_rest, p_rest
            grad[t] = (p * factor - Q[t]) * (1.0 if dloss is None else float(dloss[t])) / temperature
        P[t] = p
    return loss, grad, dict(p=P, q=Q, q_rest=q_rests, p_rest=p_rests)
