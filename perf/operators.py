"""The 8-bit linear layer with a scale per block of 128 and the distillation loss over a teacher's top logits, as cases
whose speed and accuracy are compared between a plain form in torch and this library's kernels.

The 8-bit layer: a weight [N][K] in e4m3 with one scale per 128 x 128 block; activations are quantised inside the call with
one scale per token and 128 columns.  Forward, the gradient of its input through the frozen weight, and the quantizer that makes the weight.
The loss: KL between a teacher's top logits and the student's softmax, its gradient, and both in one pass.
"""
import math

import torch

DEVICE = "cuda"
own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"fp16": 2, "bf16": 2, "fp32": 4}


def listed():
    return [
        # decoding one token through one projection, the smallest call of an 8-bit layer: latency counts
        {"name": "fp8 1 token 4096x4096", "path": "linear", "M": 1, "N": 4096, "K": 4096, "type": "fp16", "out": "fp16"},
        # a decode batch on a wide layer
        {"name": "fp8 16 tokens 11008x4096", "path": "linear", "M": 16, "N": 11008, "K": 4096, "type": "bf16", "out": "bf16"},
        # an output head over an odd vocabulary, hidden size not a multiple of the block, logits in fp32 for a loss
        {"name": "fp8 77 tokens head 32003x4112", "path": "linear", "M": 77, "N": 32003, "K": 4112, "type": "fp16", "out": "fp32"},
        # a short prompt
        {"name": "fp8 512 tokens 5120x13824", "path": "linear", "M": 512, "N": 5120, "K": 13824, "type": "fp16", "out": "fp16"},
        # prefill of a long prompt
        {"name": "fp8 2048 tokens 13824x5120", "path": "linear", "M": 2048, "N": 13824, "K": 5120, "type": "bf16", "out": "bf16"},
        # the gradient of a head's input for a training batch, and of a projection's for a ragged few tokens
        {"name": "fp8 input grad 1000 tokens 32000x4096", "path": "grad", "M": 1000, "N": 32000, "K": 4096, "type": "bf16", "out": "bf16"},
        {"name": "fp8 input grad 33 tokens 4096x11008", "path": "grad", "M": 33, "N": 4096, "K": 11008, "type": "fp16", "out": "fp16"},
        # making the 8-bit layer from a checkpoint's weight
        {"name": "fp8 quantise 11008x4096", "path": "quantise", "N": 11008, "K": 4096, "type": "bf16"},
        # scoring a few tokens: the loss alone
        {"name": "distill loss 16 x 32000", "path": "loss", "M": 16, "V": 32000, "k": 8, "type": "fp16", "T": 1.0, "rest": False},
        # a training batch over a large vocabulary, loss and gradient as two calls
        {"name": "distill loss and grad 512 x 152064", "path": "loss-grad", "M": 512, "V": 152064, "k": 32, "type": "bf16", "T": 2.0, "rest": True},
        # a training batch, loss and gradient in one pass
        {"name": "distill step 4096 x 32000", "path": "step", "M": 4096, "V": 32000, "k": 64, "type": "bf16", "T": 1.0, "rest": True},
        # an odd vocabulary in fp32
        {"name": "distill step 777 x 50257 fp32", "path": "step", "M": 777, "V": 50257, "k": 20, "type": "fp32", "T": 1.5, "rest": False},
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread evenly over its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999 * step)))
    return max(lo, min(hi, int(v) // step * step))


def draw(rng):
    path = rng.choice(["linear", "linear", "linear", "grad", "grad", "quantise", "loss", "loss-grad", "step", "step"])
    if path == "quantise":
        return {"path": path, "N": _log(rng, 500, 14000), "K": _log(rng, 512, 14000, 16), "type": rng.choice(["fp16", "bf16", "fp32"])}
    if path in ("linear", "grad"):
        M = _log(rng, 1, 2048)
        # any number of output features forward; the gradient takes them as its K
        N, K = _log(rng, 512, 32768, 16 if path == "grad" else 1), _log(rng, 512, 13824, 16)
        while M * N * K > 2048 * 13824 * 5120:
            N = max(512, N // 2 // 16 * 16)
        kind = rng.choice(["fp16", "bf16"])
        return {"path": path, "M": M, "N": N, "K": K, "type": kind, "out": rng.choice([kind, kind, "fp32"])}
    V = _log(rng, 1000, 152064)
    M = _log(rng, 1, max(1, min(4096, 4096 * 32000 // V)))
    kind = rng.choice(["fp16", "bf16", "fp32"])
    if kind == "fp32":
        M = max(1, M // 2)
    return {"path": path, "M": M, "V": V, "k": _log(rng, 1, 128), "type": kind, "T": rng.choice([1.0, 1.0, 1.5, 2.0, 4.0]), "rest": rng.random() < 0.5}


# ------------------------------------------------------------------------------------------------ inputs

def _generator(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 1000003 + sum(ord(c) for c in case["path"]))
    return g


def _weight(case, g):
    """N(0, 0.02^2) with one input channel in a hundred ten times as large (the outlier channels of the paper's Theorem 1)."""
    N, K = case["N"], case["K"]
    W = torch.randn(N, K, generator=g, device=DEVICE) * 0.02
    W *= 1.0 + 9.0 * (torch.rand(K, generator=g, device=DEVICE) < 0.01).float()
    return W.to(TYPES[case["type"]])


def _block_scales(amax):
    """The smallest power of two >= amax / 448 (1 where amax is 0): 448 = 0.875 * 2^9 is e4m3's largest value."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126).int()
    return torch.where(amax > 0, ((e + 127) << 23).view(torch.float32), torch.ones_like(amax))


def _spread(scales, rows, cols):
    """One scale per 128 x 128 block as one per element."""
    return scales.repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def _plain_quantise(W):
    N, K = W.shape
    w = W.float()
    padded = torch.zeros((N + 127) // 128 * 128, (K + 127) // 128 * 128, device=W.device)
    padded[:N, :K] = w
    amax = padded.view(padded.shape[0] // 128, 128, padded.shape[1] // 128, 128).abs().amax((1, 3))
    scales = _block_scales(amax)
    return (w / _spread(scales, N, K)).to(torch.float8_e4m3fn), scales


def prepare(case, seed):
    g = _generator(case, seed)
    if case["path"] == "quantise":
        return {"case": case, "W": _weight(case, g)}
    kind = TYPES[case["type"]]
    M = case["M"]
    if case["path"] in ("linear", "grad"):
        N, K = case["N"], case["K"]
        codes, scales = _plain_quantise(_weight(case, g))
        state = {"case": case, "codes": codes, "scales": scales}
        if case["path"] == "linear":
            # channels of different sizes, a few of them large
            x = torch.randn(M, K, generator=g, device=DEVICE) * torch.exp(0.5 * torch.randn(K, generator=g, device=DEVICE))
        else:
            # the gradient of a mean loss: small, and rows of different sizes
            x = torch.randn(M, N, generator=g, device=DEVICE) * torch.exp(torch.randn(M, 1, generator=g, device=DEVICE)) * 0.01
        state["x"] = x.to(kind)
        if own:
            from paper_2405_14917_b200 import binding as slim
            layer = slim.Fp8Linear(codes, scales)
            state["layer"] = layer
            if case["path"] == "linear":
                state["ws"] = layer.new_workspace(M)
            else:
                layer.prepare_input_grad()
                state["ws"] = layer.new_workspace(M, input_grad=True)
        return state
    V, k, T = case["V"], case["k"], case["T"]
    # a student that has learnt part of what the teacher knows
    base = torch.randn(M, V, generator=g, device=DEVICE) * 2.0
    base += 6.0 * (torch.rand(M, V, generator=g, device=DEVICE) < 4.0 / V).float()
    teacher = base + torch.randn(M, V, generator=g, device=DEVICE) * 0.5
    student = (base + torch.randn(M, V, generator=g, device=DEVICE)).to(kind)
    value, index = torch.topk(teacher, k, dim=1)
    # one row in eight is padding: no entry is present
    empty = torch.rand(M, generator=g, device=DEVICE) < 0.125
    index = torch.where(empty[:, None], torch.full_like(index, -1), index)
    state = {"case": case, "logits": student, "index": index, "value": value,
             "lse": torch.logsumexp(teacher / T, 1) if case["rest"] else None}
    if case["path"] != "loss":
        # the weight of a token in the mean; with fp16 gradients under a loss scale, as their small values ask for
        state["dloss"] = (16.0 if case["type"] == "fp16" else 1.0 / M) * (0.5 + torch.rand(M, generator=g, device=DEVICE))
    return state


# ------------------------------------------------------------------------------------------------ the plain form

def _plain_product(x, codes, scales):
    """x in blocks of 128 of its columns, times the dequantised weight."""
    M, K = x.shape
    xf = x.float()
    padded = torch.zeros(M, (K + 127) // 128 * 128, device=x.device)
    padded[:, :K] = xf
    s = _block_scales(padded.view(M, -1, 128).abs().amax(2)).repeat_interleave(128, 1)[:, :K]
    xq = (xf / s).to(torch.float8_e4m3fn).float() * s
    return xq @ (codes.float() * _spread(scales, codes.shape[0], codes.shape[1])).t()


def _plain_distill(state, with_grad):
    """Exponentials over the vocabulary in 32 bits.  In 64: their sums, the few listed entries and what is left of a sum, the
    masses outside them, since a small loss is the difference of large terms."""
    index, value, lse, T = state["index"], state["value"].double(), state["lse"], state["case"]["T"]
    logits = state["logits"].float()
    V = logits.shape[1]
    present = (index >= 0) & (index < V)
    at = torch.where(present, index, torch.zeros_like(index))
    u = torch.where(present, value / T, torch.full_like(value, -math.inf))
    some = present.any(1)
    top = logits.amax(1, keepdim=True)
    e = torch.exp((logits - top) / T)
    Z = e.sum(1, keepdim=True, dtype=torch.float64)
    logp = (torch.gather(logits, 1, at).double() - top) / T - torch.log(Z)
    if lse is None:
        u = u - torch.where(some, u.amax(1), torch.zeros_like(u[:, 0]))[:, None]
        q = torch.exp(u)
        total = q.sum(1, keepdim=True).clamp(min=1e-30)
        logq, q = u - torch.log(total), q / total
    else:
        logq = u - lse.double()[:, None]
        q = torch.exp(logq)
    loss = torch.where(present, q * (logq - logp), torch.zeros_like(q)).sum(1)
    if lse is not None:
        outside = e.clone()
        outside.scatter_(1, torch.where(present, at, at[:, :1]), 0.0)
        p_listed = torch.where(present, torch.exp(logp), torch.zeros_like(logp)).sum(1)
        p_rest = torch.where(p_listed < 0.5, 1.0 - p_listed, outside.sum(1, dtype=torch.float64) / Z[:, 0])
        q_rest = (1.0 - q.sum(1)).clamp(min=0.0)
        loss = loss + torch.where(q_rest > 0, q_rest * (torch.log(q_rest) - torch.log(p_rest)), torch.zeros_like(q_rest))
    loss = torch.where(some, loss, torch.zeros_like(loss)).float()
    if not with_grad:
        return loss
    scale = torch.where(some, state["dloss"] / T, torch.zeros_like(loss))
    p = (e / Z).float()
    if lse is None:
        grad = p * q.sum(1, keepdim=True).float()
        grad.scatter_add_(1, at, torch.where(present, -q, torch.zeros_like(q)).float())
    else:
        mass = q.sum(1) + q_rest
        grad = p * (mass - torch.where(q_rest > 0, q_rest / p_rest, torch.zeros_like(q_rest))).float()[:, None]
        listed_p = (torch.exp(logp) * mass[:, None] - q).float()
        grad.scatter_(1, torch.where(present, at, at[:, :1]), torch.where(present, listed_p, listed_p[:, :1]))
    return loss, (grad * scale[:, None]).to(state["logits"].dtype)


def run(state):
    case = state["case"]
    path = case["path"]
    if own:
        from paper_2405_14917_b200 import binding as slim
        if path == "quantise":
            return slim.fp8_quantize(state["W"])
        if path == "linear":
            return state["layer"].forward(state["x"], state["ws"], out_dtype=TYPES[case["out"]])
        if path == "grad":
            return state["layer"].input_grad(state["x"], state["ws"], out_dtype=TYPES[case["out"]])
        top = (state["index"], state["value"])
        if path == "loss":
            return slim.distill_loss(state["logits"], *top, temperature=case["T"], teacher_lse=state["lse"])[0]
        if path == "loss-grad":
            loss, saved = slim.distill_loss(state["logits"], *top, temperature=case["T"], teacher_lse=state["lse"])
            return loss, slim.distill_grad(state["logits"], *top, saved, state["dloss"], temperature=case["T"], teacher_lse=state["lse"])
        return slim.distill_step(state["logits"], *top, state["dloss"], temperature=case["T"], teacher_lse=state["lse"])
    if path == "quantise":
        return _plain_quantise(state["W"])
    if path == "linear":
        return _plain_product(state["x"], state["codes"], state["scales"]).to(TYPES[case["out"]])
    if path == "grad":
        return _plain_product(state["x"], state["codes"].t(), state["scales"].t()).to(TYPES[case["out"]])
    return _plain_distill(state, path != "loss")


def work(case):
    path = case["path"]
    if path == "quantise":
        N, K = case["N"], case["K"]
        return {"bytes": N * K * (BYTES[case["type"]] + 1) + 4 * ((N + 127) // 128) * ((K + 127) // 128), "flops": 2 * N * K}
    M = case["M"]
    if path in ("linear", "grad"):
        N, K = case["N"], case["K"]
        i, o = (K, N) if path == "linear" else (N, K)
        return {"bytes": N * K + 4 * ((N + 127) // 128) * ((K + 127) // 128) + M * i * BYTES[case["type"]] + M * o * BYTES[case["out"]],
                "flops": 2 * M * N * K}
    V, k, b = case["V"], case["k"], BYTES[case["type"]]
    small = M * k * 12 + M * 4 * (1 + int(case["rest"]))
    if path == "loss":
        return {"bytes": M * V * b + small, "flops": 4 * M * V}
    # the loss has to be known as a whole before the first gradient, but one pass can hold a row; two calls read it twice
    return {"bytes": M * V * b * (3 if path == "loss-grad" else 2) + small + 4 * M, "flops": 8 * M * V}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits

def _e4m3(v):
    """Nearest e4m3 value (three mantissa bits, exponents from -6 on, ties to even) of |v| <= 448, in 64 bits."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    # log2 may err by an ulp next to a power of two: a value at or above it has the step of its binade
    step = torch.where(v.abs() >= 16.0 * step, 2.0 * step, step)
    step = torch.where((v.abs() < 8.0 * step) & (step > 2.0 ** -9), 0.5 * step, step)
    return torch.round(v / step) * step


def _exact_scales(amax):
    e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -140) / 448.0))
    e = torch.where(448.0 * torch.exp2(e - 1.0) >= amax, e - 1.0, e)
    e = torch.where(448.0 * torch.exp2(e) < amax, e + 1.0, e).clamp(min=-126.0)
    return torch.where(amax > 0, torch.exp2(e), torch.ones_like(amax))


def exact(case, seed):
    state = prepare(case, seed)
    path = case["path"]
    if path == "quantise":
        W = state["W"].double()
        N, K = W.shape
        codes, rows = torch.empty_like(W), []
        for r in range(0, N, 128):
            line = []
            for c in range(0, K, 128):
                line.append(W[r:r + 128, c:c + 128].abs().max())
            s = _exact_scales(torch.stack(line))
            codes[r:r + 128] = _e4m3(W[r:r + 128] / s.repeat_interleave(128)[:K])
            rows.append(s)
        return codes, torch.stack(rows)
    if path in ("linear", "grad"):
        x, codes, scales = state["x"].double(), state["codes"].double(), state["scales"].double()
        if path == "grad":
            codes, scales = codes.t(), scales.t()
        N, K = codes.shape
        y = torch.zeros(x.shape[0], N, dtype=torch.float64, device=x.device)
        for j in range(0, K, 128):
            xb = x[:, j:j + 128]
            s = _exact_scales(xb.abs().amax(1, keepdim=True))
            y += (_e4m3(xb / s) * s) @ (codes[:, j:j + 128] * scales[:, j // 128].repeat_interleave(128)[:N, None]).t()
        return y
    s, T = state["logits"].double() / case["T"], case["T"]
    M, V = s.shape
    logp = torch.log_softmax(s, 1)
    index, value = state["index"], state["value"].double() / T
    present = (index >= 0) & (index < V)
    some = present.any(1)
    q = torch.zeros(M, index.shape[1], dtype=torch.float64, device=s.device)
    if state["lse"] is None:
        q[some] = torch.softmax(value.masked_fill(~present, -math.inf)[some], 1)
    else:
        q = torch.exp(value - state["lse"].double()[:, None]) * present
    target = torch.zeros(M, V, dtype=torch.float64, device=s.device)
    target.scatter_add_(1, index.clamp(0, V - 1), q)
    in_set = torch.zeros(M, V, dtype=torch.bool, device=s.device)
    in_set.scatter_(1, index.clamp(0, V - 1), present)
    loss = (torch.xlogy(target, target) - target * logp).sum(1)
    p = torch.exp(logp)
    grad = p * target.sum(1, keepdim=True) - target
    if state["lse"] is not None:
        q_rest = (1.0 - q.sum(1)).clamp(min=0.0) * some
        p_rest = (p * ~in_set).sum(1)
        loss += torch.xlogy(q_rest, q_rest / p_rest)
        grad += p * q_rest[:, None] - torch.where(in_set, torch.zeros_like(p), p * (q_rest / p_rest)[:, None])
    loss = torch.where(some, loss, torch.zeros_like(loss))
    if path == "loss":
        return loss
    return loss, grad * (state["dloss"].double() * some / T)[:, None]
