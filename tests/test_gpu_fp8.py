"""GPU parity: the 8-bit layer (block quantizer, product at any number of tokens, gradient of the input) against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as orc

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _slim():
    from paper_2405_14917_b200 import binding
    return binding


def _weight(N, K, seed, kind="fp16"):
    g = torch.Generator().manual_seed(seed)
    W = torch.randn(N, K, generator=g) * 0.02
    W[:, torch.rand(K, generator=g) < 0.02] *= 10
    return W.to(TYPES[kind])


def _x(M, K, seed, kind="fp16"):
    g = torch.Generator().manual_seed(seed + 1)
    return (torch.randn(M, K, generator=g) * torch.exp(0.5 * torch.randn(K, generator=g))).to(TYPES[kind])


def _check(y, x, codes, scales):
    """Products of two e4m3 values, and their products with powers of two, are exact in fp32.  The tensor cores add 32 of them to the
    accumulator at a time; over K columns that is K / 32 roundings of at most 2^-23 of what the terms add up to in magnitude (128 of them are allowed
    beside, for what is lost when 33 terms are lined up), then one rounding to y."""
    want, mag = orc.linear(x.double().cpu().numpy(), codes.view(torch.uint8).cpu().numpy(), scales.double().cpu().numpy())
    half = torch.finfo(y.dtype).eps / 2
    tol = (128 + codes.shape[1] / 32) * 2.0 ** -23 * mag + half * np.abs(want) + (2.0 ** -25 if y.dtype == torch.float16 else 0.0)
    err = np.abs(y.double().cpu().numpy() - want)
    assert np.isfinite(err).all()
    assert (err <= tol).all(), (err / np.maximum(tol, 1e-300)).max()


@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("N,K", [(128, 128), (1, 16), (130, 272), (300, 1008), (16, 4096)])
def test_quantizer_is_exact(N, K, kind):
    slim = _slim()
    W = _weight(N, K, N + K, kind)
    if N > 128 and K > 128:
        W[128:, 128:256] = 0                              # a block of zeros
        W[:3, 0] = torch.tensor([448.0, -3.5, 2.0 ** -12])
    codes, scales = slim.fp8_quantize(W.cuda())
    want_c, want_s = orc.quantize(W.double().numpy())
    np.testing.assert_array_equal(scales.cpu().numpy(), want_s)
    np.testing.assert_array_equal(codes.view(torch.uint8).cpu().numpy(), want_c)


def test_quantizer_of_extreme_blocks():
    slim = _slim()
    W = torch.zeros(640, 128)
    W[0, :3] = torch.tensor([3.0e38, -1.0e38, 1.0])       # near fp32's end
    W[128, :3] = torch.tensor([2.0 ** -140, 2.0 ** -149, 0.0])
    W[256, :4] = torch.tensor([float("inf"), float("nan"), 5.0, -float("inf")])
    W[384] = torch.linspace(-448, 448, 128)
    W[512, 0] = 448.0001
    codes, scales = slim.fp8_quantize(W.cuda())
    want_c, want_s = orc.quantize(W.double().numpy())
    np.testing.assert_array_equal(scales.cpu().numpy(), want_s)
    got = codes.view(torch.uint8).cpu().numpy()
    nan = (want_c & 0x7f) == 0x7f
    assert ((got & 0x7f)[nan] == 0x7f).all()
    np.testing.assert_array_equal(got[~nan], want_c[~nan])


@pytest.mark.parametrize("kind,out", [("fp16", "fp16"), ("bf16", "bf16"), ("fp16", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("M,N,K", [(1, 128, 128), (1, 16, 16), (1, 4096, 4096), (2, 1, 48), (5, 1000, 1040), (16, 11008, 256), (17, 513, 4112),
                                   (32, 256, 2048), (33, 130, 272), (64, 777, 1024), (65, 1024, 4096), (100, 3001, 528), (128, 128, 13824),
                                   (129, 300, 272), (256, 256, 128), (257, 1000, 1040), (300, 1, 16), (512, 2000, 2064), (1000, 4111, 144)])
def test_linear(M, N, K, kind, out):
    slim = _slim()
    layer = slim.Fp8Linear.from_weight(_weight(N, K, M + N + K, kind).cuda())
    x = _x(M, K, M, kind).cuda()
    ws = layer.new_workspace(M)
    y = layer.forward(x, ws, out_dtype=TYPES[out])
    slim.workspace_status(ws)
    assert y.dtype == TYPES[out]
    _check(y, x, layer.codes, layer.scales)


@pytest.mark.parametrize("M,N,K", [(1000, 9000, 272), (1024, 11008, 528), (700, 9000, 1040), (600, 7001, 2064), (300, 11600, 1040),
                                   (600, 500, 4112), (200, 4096, 11008), (130, 1023, 8192)])
def test_several_tiles(M, N, K):
    """More tiles than CTA pairs, at each width that a tile may have (256 features, with one accumulator, 224, 192, 160), ragged last ones; and narrow
    and deep layers of more tokens than one tile of the kernel that cuts K."""
    slim = _slim()
    layer = slim.Fp8Linear.from_weight(_weight(N, K, N, "bf16").cuda())
    x = _x(M, K, M, "bf16").cuda()
    ws = layer.new_workspace(M)
    y = layer.forward(x, ws)
    slim.workspace_status(ws)
    _check(y, x, layer.codes, layer.scales)


@pytest.mark.parametrize("M", [3, 40, 200])
def test_scales_of_every_block_count(M):
    """Scales that differ by many powers of two from block to block, and others than the quantizer would give: each block under its own."""
    slim = _slim()
    N, K = 400, 1296
    codes, scales = slim.fp8_quantize(_weight(N, K, 5).cuda())
    g = torch.Generator().manual_seed(9)
    scales = torch.exp2(torch.randint(-12, 4, scales.shape, generator=g).float()).cuda()
    layer = slim.Fp8Linear(codes, scales)
    x = _x(M, K, 3)
    x *= torch.exp2(torch.arange(K) // 128 % 5 - 2.0).half()
    x = (x.float() * torch.exp2(torch.randint(-3, 4, (M, 1), generator=g).float())).half().cuda()
    _check(layer.forward(x, layer.new_workspace(M), out_dtype=torch.float32), x, codes, scales)
    with pytest.raises(ValueError):
        slim.Fp8Linear(codes, scales * 1.5)
    with pytest.raises(ValueError):
        slim.Fp8Linear(codes, -scales)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 512), (33, 1008, 272), (70, 32000, 256), (300, 2000, 1040)])
def test_input_gradient(M, N, K, kind):
    """dx = dy W: against the oracle, and along a direction against the differences of the forward's exact form."""
    slim = _slim()
    layer = slim.Fp8Linear.from_weight(_weight(N, K, K, kind).cuda())
    g = torch.Generator().manual_seed(M)
    dy = (torch.randn(M, N, generator=g) * torch.exp(torch.randn(M, 1, generator=g)) * 0.01).to(TYPES[kind]).cuda()
    ws = layer.new_workspace(M, input_grad=True)
    dx = layer.input_grad(dy, ws, out_dtype=torch.float32)
    slim.workspace_status(ws)
    _check(dx, dy, layer.codes.view(torch.uint8).t().contiguous().view(torch.float8_e4m3fn), layer.scales.t())
    # y(x) = x W-hat^T is linear in x for a fixed W-hat: <dy, y(x + v) - y(x)> = <dx, v>, up to the 8-bit rounding of dy (2^-4
    # relative an element, 2^-10 of its block's largest where that is more)
    v = torch.randn(M, K, generator=g).double().numpy()
    w = orc.decode(layer.codes.view(torch.uint8).cpu().numpy()) * orc._spread(layer.scales.cpu().numpy(), N, K)
    d = dy.double().cpu().numpy()
    diff = ((v @ w.T) * d).sum()
    big = np.repeat(np.abs(np.pad(d, ((0, 0), (0, -N % 128)))).reshape(M, -1, 128).max(2), 128, 1)[:, :N]
    bound = (np.abs(v @ w.T) * np.maximum(np.abs(d) * 2.0 ** -4, big * 2.0 ** -10)).sum() + 1e-4 * (np.abs(v) * np.abs(dx.double().cpu().numpy())).sum()
    assert abs((dx.double().cpu().numpy() * v).sum() - diff) <= bound


@pytest.mark.parametrize("M", [1, 16, 30, 60, 100, 300])
def test_strides_and_what_lies_beside(M):
    slim = _slim()
    N, K = 333, 400
    layer = slim.Fp8Linear.from_weight(_weight(N, K, 1).cuda())
    wide = torch.full((M, K + 24), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, 8:8 + K] = _x(M, K, 2).cuda()
    x = wide[:, 8:8 + K]
    out = torch.full((M + 2, N + 13), 7.0, dtype=torch.float16, device="cuda")
    y = out[:M, :N]
    ws = layer.new_workspace(M)
    assert layer.forward(x, ws, out=y) is y
    _check(y, x, layer.codes, layer.scales)
    assert (out[:, N:] == 7).all() and (out[M:] == 7).all()


@pytest.mark.parametrize("M", [4, 20, 50, 90, 200])
def test_not_finite_tokens_stay_alone(M):
    slim = _slim()
    N, K = 260, 1040
    layer = slim.Fp8Linear.from_weight(_weight(N, K, 4).cuda())
    x = _x(M, K, 6).cuda()
    clean = layer.forward(x, layer.new_workspace(M))
    x[1, 700] = float("inf")
    x[2, 3] = float("nan")
    y = layer.forward(x, layer.new_workspace(M))
    assert torch.isnan(y[1:3]).all()
    keep = [i for i in range(M) if i not in (1, 2)]
    assert torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("M", [1, 16, 32, 48, 128, 400])
def test_repeatable_captured_and_on_a_side_stream(M):
    slim = _slim()
    N, K = 1100, 2064
    layer = slim.Fp8Linear.from_weight(_weight(N, K, 8).cuda())
    x = _x(M, K, 1).cuda()
    ws = layer.new_workspace(M)
    y = layer.forward(x, ws)
    for _ in range(3):
        assert torch.equal(layer.forward(x, ws), y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        z = layer.forward(x, ws)
    x.copy_(_x(M, K, 2))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    slim.workspace_status(ws)
    _check(z, x, layer.codes, layer.scales)


def test_a_workspace_shared_with_the_group_wise_layers():
    """One workspace of the larger size, the two kinds of layer in turn on one stream."""
    slim = _slim()
    from paper_2405_14917_b200 import workloads as wl
    N, K, M = 5120, 13824, 512                            # a group-wise layer that is cut across CTAs and uses the flags
    W, a = wl.make_weight_and_norms_device((1, N, K), N, K, "cuda")
    low = slim.QuantLinear.from_weight(W, a, 3)
    high = slim.Fp8Linear.from_weight(W)
    ws = torch.empty(max(low.workspace_bytes(M), slim.fp8_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
    slim.workspace_init(ws)
    x = _x(M, K, 3).cuda()
    first = low.forward(x, ws)
    second = high.forward(x, ws)
    for _ in range(3):
        assert torch.equal(low.forward(x, ws), first)
        assert torch.equal(high.forward(x, ws), second)
    slim.workspace_status(ws)


def test_empty_calls_and_refusals():
    slim = _slim()
    layer = slim.Fp8Linear.from_weight(_weight(256, 272, 1).cuda())
    ws = layer.new_workspace(64)
    assert layer.forward(torch.zeros(0, 272, dtype=torch.float16, device="cuda"), ws).shape == (0, 256)
    x = _x(40, 272, 1).cuda()
    with pytest.raises(slim.SlimError) as e:
        layer.forward(x, torch.zeros(1280, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -4
    with pytest.raises(TypeError):
        layer.forward(x.float(), ws)
    with pytest.raises(TypeError):
        layer.forward(x.cpu(), ws)
    with pytest.raises(ValueError):
        layer.forward(x[:, :256], ws)                      # another K
    with pytest.raises(slim.SlimError):
        layer.forward(torch.as_strided(torch.zeros(40 * 276, dtype=torch.float16, device="cuda"), (40, 272), (276, 1)), ws)   # rows off 16 bytes
    with pytest.raises((TypeError, ValueError)):
        layer.forward(x, ws, out_dtype=torch.bfloat16)
    with pytest.raises(slim.SlimError):
        slim.fp8_quantize(torch.zeros(128, 100, dtype=torch.float16, device="cuda"))       # K not a multiple of 16
    with pytest.raises(ValueError):
        slim.Fp8Linear(layer.codes, layer.scales[:1])
    odd = slim.Fp8Linear.from_weight(_weight(250, 272, 1).cuda())
    with pytest.raises(ValueError):
        odd.input_grad(torch.zeros(4, 250, dtype=torch.float16, device="cuda"), ws)


@pytest.mark.parametrize("M", [2, 40, 200])
def test_a_weight_of_more_than_32_bits_of_codes(M):
    """262400 x 8208 codes: the last rows, beyond 2^31 bytes, against the oracle."""
    slim = _slim()
    N, K, tail = 262400, 8208, 300
    W = torch.empty(N, K, dtype=torch.bfloat16, device="cuda")
    W[:] = torch.randn(1, K, device="cuda").bfloat16()
    W[-tail:] = _weight(tail, K, 3, "bf16").cuda()
    codes, scales = slim.fp8_quantize(W)
    first = (N - tail) // 128 * 128
    want_c, want_s = orc.quantize(W[first:].double().cpu().numpy())
    np.testing.assert_array_equal(codes[first:].view(torch.uint8).cpu().numpy(), want_c)
    np.testing.assert_array_equal(scales[first // 128:].cpu().numpy(), want_s)
    x = _x(M, K, 1, "bf16").cuda()
    layer = slim.Fp8Linear(codes, scales)
    ws = layer.new_workspace(M)
    y = layer.forward(x, ws)
    slim.workspace_status(ws)
    _check(y[:, first:], x, codes[first:], scales[first // 128:])


@pytest.mark.parametrize("M", [3, 20, 50, 150])
def test_rows_farther_apart_than_32_bits_count(M):
    slim = _slim()
    N, K = 130, 272
    layer = slim.Fp8Linear.from_weight(_weight(N, K, 1).cuda())
    ld = (2 ** 31 + 2 ** 20) // (M - 1) // 8 * 8 + 8
    buf = torch.empty((M - 1) * ld + 512, dtype=torch.float16, device="cuda")
    x, y = torch.as_strided(buf, (M, K), (ld, 1), 0), torch.as_strided(buf, (M, N), (ld, 1), 272)
    x.copy_(_x(M, K, 2))
    assert layer.forward(x, layer.new_workspace(M), out=y) is y
    _check(y, x, layer.codes, layer.scales)


def test_a_sum_of_nothing():
    slim = _slim()
    codes, scales = slim.fp8_quantize(torch.zeros(200, 0, dtype=torch.float16, device="cuda"))
    layer = slim.Fp8Linear(codes, scales)
    y = layer.forward(torch.zeros(3, 0, dtype=torch.float16, device="cuda"), layer.new_workspace(3), out=torch.full((3, 200), 5.0, device="cuda"))
    assert (y == 0).all()
