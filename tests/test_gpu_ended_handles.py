"""Handles whose last reference goes while a graph is captured: on the capturing thread, on a stream that is not captured, on another thread.  The capture is not broken by it, and their
memory comes back."""
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1906_03707_amd import binding
    binding.lib()
    return binding


def make(B, seq=False):
    from paper_1906_03707_amd import synth
    rowptr, col = synth.sbm(6, 40, 0.3, 0.01, seed=11)
    return (B.SeqHag(rowptr, col, 60) if seq else B.hag_search(rowptr, col, 60)).upload()


@pytest.mark.parametrize("seq", [False, True])
@pytest.mark.parametrize("where", ["here", "stream", "thread"])
def test_handles_that_end_during_a_capture(B, where, seq):
    h, ends = make(B), [make(B, seq) for _ in range(3)]
    x = torch.randn(240, 64, device="cuda")
    want = h.forward(x, "gcn")
    side, failed = torch.cuda.Stream(), []
    torch.cuda.synchronize()

    def end():
        try:
            ends.pop()
        except BaseException as error:
            failed.append(error)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        if where == "thread":
            thread = threading.Thread(target=end)
            thread.start()
            thread.join()
        elif where == "stream":
            with torch.cuda.stream(side):
                end()
        else:
            end()
        y = h.forward(x, "gcn")
    assert not failed
    for _ in range(3):
        y.zero_()
        graph.replay()
        assert torch.equal(y, want)
        torch.cuda.synchronize()
    h.forward(x, "gcn")                                    # whatever waited is freed by the next call
    assert not B._ended
    ends.clear()
    assert not B._ended


def test_what_waits_is_freed_by_other_calls(B):
    freed = []
    h, s = make(B), make(B, True)
    x = torch.randn(240, 32, device="cuda")
    w_ih, w_hh, b = (torch.randn(*shape, device="cuda") for shape in ((128, 32), (128, 32), (128,)))
    for n, call in enumerate((lambda: h.upload(), lambda: s.upload(), lambda: h.forward(x), lambda: h.backward(x), lambda: h.naive_forward(x), lambda: s.lstm_forward(x, w_ih, w_hh, b))):
        B._ended.append((freed.append, n))
        call()
        assert not B._ended and freed == list(range(n + 1))


@pytest.mark.parametrize("where", ["stream", "thread"])
def test_their_memory_comes_back(B, where):
    import numpy as np
    n, degree = 20000, 250
    rng = np.random.default_rng(3)
    col = np.sort(rng.integers(0, n // degree, (n, degree)) + np.arange(degree) * (n // degree), 1).astype(np.int32).ravel()
    x = torch.randn(240, 64, device="cuda")
    h = make(B)
    h.forward(x)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    ends = [B.hag_search(np.arange(n + 1, dtype=np.int64) * degree, col, 0).upload()]
    torch.cuda.synchronize()
    held = before - torch.cuda.mem_get_info()[0]
    assert held >= 4 * n * degree
    with torch.cuda.graph(graph):
        if where == "thread":
            thread = threading.Thread(target=ends.clear)
            thread.start()
            thread.join()
        else:
            with torch.cuda.stream(side):
                ends.clear()
        assert not B._ended and before - torch.cuda.mem_get_info()[0] <= held // 2
        y = h.forward(x)
    graph.replay()
    assert torch.equal(y, h.forward(x))
