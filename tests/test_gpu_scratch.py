"""GPU tests of the binding's scratch and of tensors on other streams: graphs beside eager calls and beside each other."""
import numpy as np
import pytest

from test_gpu_attend import Case

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

LONG = [([(3000, 1), (50, 1), (700, 1)], 1), ([(3000, 60), (50, 1)], 60)]


def _captured(cache, c, t, new, stream=None):
    """(graph, out, lse) of one attention call, warmed up on the stream that it is captured on."""
    out = torch.empty_like(c.q)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    side = stream or torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.attend(c.q, *t, max_new=new, out=out, lse=lse)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        cache.attend(c.q, *t, max_new=new, out=out, lse=lse)
    return g, out, lse


@pytest.mark.parametrize("requests,new", LONG)
def test_a_graph_beside_a_larger_eager_call_on_its_stream(requests, new):
    """The call after the capture needs more scratch; a replay then writes to none of the tensors made since."""
    rng = np.random.default_rng(new)
    c = Case(rng, requests, D=64)
    big = Case(rng, [(2600, 90)] * 4 + [(600, 1)] * 300, D=64)
    s = torch.cuda.Stream()
    cache, t = c.cache(), c.tensors()
    print(f"[gpu] graph beside a larger eager call {requests}", flush=True)
    want = cache.attend(c.q, *t, max_new=new)
    torch.cuda.synchronize()
    g, out, lse = _captured(cache, c, t, new, s)
    other = big.cache()
    other._ws = cache._ws                                    # the scratch that the graph's stream has
    with torch.cuda.stream(s):
        before = {k: v[2] for k, v in cache._ws.by_stream.items()}
        other.attend(big.q, *big.tensors(), max_new=90)
        assert cache._ws.by_stream[s.cuda_stream][2] > before[s.cuda_stream]
        fresh = [torch.full((n,), 90, dtype=torch.uint8, device="cuda") for n in sorted(set(before.values())) for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(3):
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert all(bool((x == 90).all()) for x in fresh)


@pytest.mark.parametrize("requests,new", LONG)
def test_two_graphs_replayed_on_two_streams(requests, new):
    rng = np.random.default_rng(new + 1)
    c = Case(rng, requests, D=64)
    cache, t = c.cache(), c.tensors()
    d = Case(rng, requests, D=64)                            # other queries over the same cache
    print(f"[gpu] two graphs at once {requests}", flush=True)
    want = [cache.attend(x.q, *t, max_new=new) for x in (c, d)]
    graphs = [_captured(cache, x, t, new) for x in (c, d)]
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(3):
        for _, out, lse in graphs:
            out.fill_(float("nan"))
            lse.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(20):
            for (g, _, _), s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for (_, out, lse), w in zip(graphs, want):
            assert torch.equal(out, w[0]) and torch.equal(lse, w[1])


def test_block_plans_captured_twice_have_scratch_of_their_own():
    from paper_2606_30391_amd import festina as F
    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32)).cuda()
    R = 3000
    b = F.DeviceBlocks(i32(np.zeros(R)), i32(np.full(R, 3)), i32(np.full((R, 1), -1)), i32(np.arange(R)), i32([R]), 16, 3 * R)
    print("[gpu] two graphs of a block plan", flush=True)
    b.extend()
    torch.cuda.synchronize()
    want = b.slot.clone()
    kept = dict(b._ws.by_stream)
    graphs = []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            b.extend()
    assert b._ws.by_stream.keys() == kept.keys()             # neither is a stream's
    for g in graphs:
        b.slot.fill_(-7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.slot, want)


def _busy(stream):
    """Work of some milliseconds on `stream`."""
    with torch.cuda.stream(stream):
        x = torch.randn((8192, 8192), device="cuda").bfloat16()
        for _ in range(20):
            x = x @ x


def _dropped(stream, make, call):
    """`call` gets tensors that are dropped right after it, while `stream` has not come to it; others are made since."""
    kept = make()
    again = [x.clone() for x in kept]
    sizes = [x.numel() * x.element_size() for x in again]
    old = [x.untyped_storage().data_ptr() for x in again]
    torch.cuda.synchronize()
    _busy(stream)
    call(*again)
    done = torch.cuda.Event()
    done.record(stream)
    del again
    fresh = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
    assert not done.query(), "the stream had nothing to do"
    assert not {x.data_ptr() for x in fresh} & set(old)
    torch.cuda.synchronize()
    return kept


def test_tensors_dropped_after_a_call_on_another_stream():
    """A call's inputs keep their memory until the other stream has read them."""
    from paper_2606_30391_amd import festina as F
    rng = np.random.default_rng(41)
    c = Case(rng, [(700, 1), (3000, 1)] + [(40, 1)] * 300, D=64)
    cache, t = c.cache(), c.tensors()
    s = torch.cuda.Stream()
    print("[gpu] tensors dropped after calls on another stream", flush=True)
    want = cache.attend(c.q, *t, max_new=1)
    got = []
    _dropped(s, lambda: (c.q, *t), lambda q, a, b, f: got.extend(cache.attend(q, a, b, f, max_new=1, stream=s)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

    H, D, bt, T = 2, 64, 32, 2000
    new = F.DeviceCache.empty(64, bt, H, D)
    k, v = (torch.randn((T, H, D), device="cuda") for _ in range(2))
    slot = torch.arange(T, dtype=torch.int32, device="cuda")
    new.store(k, v, slot)
    torch.cuda.synchronize()
    want = [x.clone() for x in (new.k, new.v, new.k_scale, new.v_scale)]
    for x in (new.k, new.v, new.k_scale, new.v_scale):
        x.zero_()
    _dropped(s, lambda: (k, v, slot), lambda *x: new.store(*x, stream=s))
    blocks = T // bt                                         # (whole ones: what lies behind the last token was left alone)
    for x, y in zip((new.k, new.v, new.k_scale, new.v_scale), want):
        assert torch.equal(x[:blocks], y[:blocks])

    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32)).cuda()
    R = 3000
    b = F.DeviceBlocks(i32(np.full(R, 5)), i32(np.zeros(R)), i32(np.arange(R)[:, None]), i32(np.full(R, -1)), i32([0]), 16, 0)
    _dropped(s, lambda: (torch.ones(R, dtype=torch.uint8, device="cuda"),), lambda d: b.release(d, stream=s))
    assert int(b.n_free_out) == R and torch.equal(b.free_ids, torch.arange(R, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("bad", [{"window": -1}, {"scale": float("nan")}])
def test_a_refused_call_leaves_nothing_behind(bad):
    """The first call of its sizes on a cache is refused; the same call without the fault is answered."""
    from paper_2606_30391_amd import festina as F
    rng = np.random.default_rng(51)
    c = Case(rng, [(20, 2), (30, 1)], D=64)
    cache, t = c.cache(), c.tensors()
    print(f"[gpu] a call after a refused one {bad}", flush=True)
    with pytest.raises(F.FestinaError):
        cache.attend(c.q, *t, max_new=2, **bad)
    out, lse = cache.attend(c.q, *t, max_new=2)
    torch.cuda.synchronize()
    c.compare(out, lse, c.want())


def test_windows_and_bounds_past_32_bits():
    """2^32 + 5 is no window of 5, and neither is a negative one."""
    from paper_2606_30391_amd import festina as F
    rng = np.random.default_rng(52)
    c = Case(rng, [(200, 2), (30, 1)], D=64)
    cache, t = c.cache(), c.tensors()
    print("[gpu] windows past 32 bits", flush=True)
    for new, window in ((2, 2 ** 32 + 5), (2 ** 32 + 1, 0), (2 ** 31, 2 ** 31), (2, 2 ** 31 - 1)):
        out, lse = cache.attend(c.q, *t, max_new=new, window=window)
        torch.cuda.synchronize()
        c.compare(out, lse, c.want())
    for kw in ({"max_new": 2, "window": 5 - 2 ** 32}, {"max_new": 2 - 2 ** 32}):
        with pytest.raises(F.FestinaError):
            cache.attend(c.q, *t, **kw)


def test_queries_that_ask_for_a_gradient_are_refused():
    rng = np.random.default_rng(53)
    c = Case(rng, [(200, 2), (30, 1)], D=64)
    cache, t = c.cache(), c.tensors()
    print("[gpu] queries that ask for a gradient", flush=True)
    want = cache.attend(c.q, *t, max_new=2)
    q = c.q.clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        cache.attend(q, *t, max_new=2)
    with torch.no_grad():
        out, lse = cache.attend(q, *t, max_new=2)
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
