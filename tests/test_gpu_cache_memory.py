"""The default workspace of a cache attention is the call's: it goes back to the
allocator, whatever the stream and the thread."""
import threading

import pytest

from test_gpu_cache import World, _torch, av, run_attention  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def test_workspace_is_given_back(av):
    t = _torch()
    w = World(av, "bf16", [6000, 500], 16, 2, 64, 16, seed=1, max_len=1 << 20)
    assert av.avits_cache_attention_workspace(w.cache, 16, True) > 1 << 26
    o, lse = w.outputs()
    side = t.cuda.Stream()

    def call(**kw):
        av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse, weight=1.0, accumulate=False,
                                 **kw)

    t.cuda.synchronize()
    before = t.cuda.memory_allocated()
    call()
    call(stream=side)
    with t.cuda.stream(side):
        call()
    threads = [threading.Thread(target=call) for _ in range(3)]
    [x.start() for x in threads]
    [x.join() for x in threads]
    t.cuda.synchronize()
    assert t.cuda.memory_allocated() == before
    w.check(o, lse, w.acc.cpu().numpy(), 1.0, accumulate=False)


def test_workspace_is_used_again(av):
    """Calls in a row on one stream take the same memory: no more is reserved."""
    t = _torch()
    w = World(av, "bf16", [6000, 500], 16, 2, 64, 16, seed=2)
    run_attention(w, weight=1.0)
    t.cuda.synchronize()
    before = t.cuda.memory_reserved()
    outs = [w.outputs() for _ in range(20)]
    for o, lse in outs:
        av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse)
    t.cuda.synchronize()
    assert t.cuda.memory_reserved() <= before + (2 << 20)      # the outputs' own, if any
    for o, lse in outs:
        assert t.equal(o, outs[0][0]) and t.equal(lse, outs[0][1])


def test_captured_on_a_forked_stream(av):
    """stream= a stream that joined a capture: its workspace is the graph's, which
    eager calls afterwards do not get."""
    t = _torch()
    w = World(av, "bf16", [6000, 500], 16, 2, 64, 16, seed=3)
    other = World(av, "bf16", [5000, 700], 16, 2, 64, 16, seed=4)
    o, lse = w.outputs()
    acc0 = w.acc.cpu().numpy()
    side = t.cuda.Stream()
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        side.wait_stream(t.cuda.current_stream())
        av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse, weight=1.0, accumulate=False,
                                 stream=side)
        t.cuda.current_stream().wait_stream(side)
    eager = [(other.outputs(), other.outputs()) for _ in range(4)]
    main = t.cuda.Stream()
    t.cuda.synchronize()
    for (oa, la), (ob, lb) in eager:
        graph.replay()
        with t.cuda.stream(main):
            av.avits_cache_attention(other.cache, other.q, other.scale, oa, lse=la)
        av.avits_cache_attention(other.cache, other.q, other.scale, ob, lse=lb, stream=side)
        graph.replay()
    t.cuda.synchronize()
    w.check(o, lse, acc0, 1.0, accumulate=False)
    for pair in eager:
        for oe, le in pair:
            other.check(oe, le)
