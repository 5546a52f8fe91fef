"""The workspace that ``paged_attention`` brings itself, over streams, graphs and threads."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_block import DEV, aq, attend_case  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.fixture
def made(aq, monkeypatch):
    """(stream, whether it was capturing) of each workspace that calls make."""
    from paper_2401_06118_amd import block

    seen, make = [], block.attention_workspace

    def noted(*args, **kw):
        seen.append((torch.cuda.current_stream().cuda_stream, torch.cuda.is_current_stream_capturing()))
        return make(*args, **kw)

    monkeypatch.setattr(block, "attention_workspace", noted)
    monkeypatch.setattr(block, "_workspaces", {})
    return seen


def split_case():
    """One sequence whose pieces many workgroups join."""
    bt, q = attend_case([9000], [1], 8, 1, 128, 16, torch.float16)
    return q.to(DEV), bt.gpu()


def test_workspace_of_a_forked_stream_in_a_graph(aq, made):
    """A side stream of a capture gets a workspace that is zeroed on it, in the graph."""
    q, gpu = split_case()
    want = aq.paged_attention(q, *gpu)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):  # (modules are loaded before the capture)
        aq.paged_attention(q, *gpu)
    torch.cuda.synchronize()
    made.clear()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        a = aq.paged_attention(q, *gpu, stream=side)
        b = aq.paged_attention(q, *gpu)
        main.wait_stream(side)
    assert made == [(side.cuda_stream, True), (main.cuda_stream, True)]
    for _ in range(5):
        a.zero_()
        b.zero_()
        aq.paged_attention(q, *gpu, stream=side)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want)


def test_workspace_of_a_capturing_stream_that_is_not_current(aq, made):
    """A stream that captures while another one is current gets a workspace of the graph's own."""
    q, gpu = split_case()
    want = aq.paged_attention(q, *gpu)
    s, out = torch.cuda.Stream(), torch.empty_like(q)
    with torch.cuda.stream(s):
        aq.paged_attention(q, *gpu)
    torch.cuda.synchronize()
    made.clear()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        with torch.cuda.stream(other):
            aq.paged_attention(q, *gpu, out=out, stream=s)
    assert made == [(s.cuda_stream, True)]
    for _ in range(5):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_workspace_of_another_stream(aq, made):
    """Eager calls with an explicit stream: made on it once, then kept."""
    q, gpu = split_case()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [aq.paged_attention(q, *gpu, stream=s) for _ in range(3)]
    s.synchronize()
    assert made == [(s.cuda_stream, False)]
    assert all(torch.equal(o, aq.paged_attention(q, *gpu)) for o in outs)


def test_workspace_of_threads(aq, made, monkeypatch):
    """Threads that make the first calls on one stream together share one workspace."""
    import threading
    import time

    from paper_2401_06118_amd import block

    make = block.attention_workspace
    monkeypatch.setattr(block, "attention_workspace", lambda *a, **k: (time.sleep(0.2), make(*a, **k))[1])
    device, s = torch.device("cuda", torch.cuda.current_device()), torch.cuda.Stream()
    got, start = [], threading.Barrier(4)

    def first():
        start.wait()
        got.append(block._workspace(device, 128, s, s.cuda_stream))

    threads = [threading.Thread(target=first) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(made) == 1 and all(w is got[0] for w in got) and len(got) == 4


def test_gradients_of_no_tokens_on_another_stream(aq):
    """The zeros that rope_backward returns for no tokens are there for the stream that it was given."""
    z = lambda *s: torch.zeros(*s, dtype=torch.float16, device=DEV)  # noqa: E731
    q, k, w = z(0, 4, 64), z(0, 2, 64), torch.ones(64, dtype=torch.float16, device=DEV)
    table, pos = aq.rotary_table(4, 64), torch.zeros(0, dtype=torch.int32, device=DEV)
    s = torch.cuda.Stream()
    junk = [torch.full((64,), 7.0, device=DEV) for _ in range(8)]
    torch.cuda.synchronize()
    del junk
    torch.cuda._sleep(200_000_000)  # the current stream has something to do
    got = aq.rope_backward(q, k, table, pos, q=q, k=k, q_weight=w, k_weight=w, stream=s)
    with torch.cuda.stream(s):
        seen = [g.cpu() for g in got[2:]]
    assert all((g == 0).all() for g in seen)
