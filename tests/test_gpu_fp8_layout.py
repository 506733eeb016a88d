"""GPU: the transposed codes that the gradient of an 8-bit layer's input reads are complete wherever they are read."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def _slim():
    from paper_2405_14917_b200 import binding
    return binding


def _layer(N, K, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return _slim().Fp8Linear.from_weight(torch.randn(N, K, generator=g, device="cuda").bfloat16() * 0.02)


def _dy(M, N, seed=2):
    return torch.randn(M, N, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def test_first_call_on_one_stream_second_on_another():
    """The layout is made on a stream that is busy; a call on another stream right behind it."""
    N, K, M = 4096, 4096, 8
    layer, dy = _layer(N, K), _dy(M, N)
    other = _slim().Fp8Linear(layer.codes, layer.scales)
    other.prepare_input_grad()
    ws, ws2 = other.new_workspace(M, input_grad=True), layer.new_workspace(M, input_grad=True)
    want = other.input_grad(dy, ws)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    big = torch.randn(8192, 8192, device="cuda")
    big @ big
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        for _ in range(20):
            big @ big                                # a few hundred milliseconds
        layer.prepare_input_grad()
    with torch.cuda.stream(b):
        got = layer.input_grad(dy, ws2)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_first_call_under_capture_is_refused_and_leaves_nothing_behind():
    N, K, M = 512, 272, 8
    layer, dy = _layer(N, K), _dy(M, N)
    ws = layer.new_workspace(M, input_grad=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dy + 1                                       # a capture of nothing is warned about
        with pytest.raises(RuntimeError, match="prepare_input_grad"):
            layer.input_grad(dy, ws)
        with pytest.raises(RuntimeError, match="captur"):
            layer.prepare_input_grad()
    # an eager call then makes the layout, and a capture of it is taken
    want = layer.input_grad(dy, ws)
    other = _slim().Fp8Linear(layer.codes, layer.scales)
    other.prepare_input_grad()
    assert torch.equal(want, other.input_grad(dy, ws))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer.input_grad(dy, ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_threads_that_make_the_first_call_together():
    N, K, M = 2048, 1040, 4
    dy = _dy(M, N)
    for seed in range(5):
        layer = _layer(N, K, seed)
        other = _slim().Fp8Linear(layer.codes, layer.scales)
        want = other.input_grad(dy, other.new_workspace(M, input_grad=True))
        spaces = [layer.new_workspace(M, input_grad=True) for _ in range(6)]
        torch.cuda.synchronize()
        got, gate = [None] * 6, threading.Barrier(6)

        def call(i):
            gate.wait()
            with torch.cuda.stream(torch.cuda.Stream()):
                got[i] = layer.input_grad(dy, spaces[i])

        threads = [threading.Thread(target=call, args=(i,)) for i in range(6)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        assert all(g is not None and torch.equal(g, want) for g in got)


def test_a_layer_is_copied_with_and_without_its_layout():
    import copy
    N, K, M = 256, 272, 3
    layer, dy = _layer(N, K), _dy(M, N)
    ws = layer.new_workspace(M, input_grad=True)
    early = copy.deepcopy(layer)
    want = layer.input_grad(dy, ws)
    assert torch.equal(early.input_grad(dy, ws), want) and torch.equal(copy.deepcopy(layer).input_grad(dy, ws), want)
