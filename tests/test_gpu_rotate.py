"""GPU tests of the norm and rotation of queries and keys against the definition in 64 bits (drafts_reference.rotate, which
also says what float32 arithmetic may be off by); half a unit in the last place of the outputs comes on top."""
import numpy as np
import pytest

import drafts_reference as D

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -134), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -25),
         "f32": (torch.float32, 2.0 ** -24, 2.0 ** -150)}


def _near(got, want, bound, dtype):
    _, half, least = TYPES[dtype]
    off = np.abs(got.double().cpu().numpy() - want)
    return bool((off <= bound * (1 + half) + half * np.abs(want) + least).all())


def _freq(half):
    return 1e4 ** (-np.arange(half) / max(half, 1))


CASES = [  # tokens, heads, kv heads, dim, rotated, interleaved, norm
    (1, 32, 8, 128, 128, False, True), (33, 14, 7, 64, 64, True, True), (17, 3, 1, 96, 96, False, True),
    (5, 8, 8, 256, 128, True, False), (40, 5, 5, 96, 48, True, True), (300, 9, 2, 128, 64, False, False),
    (7, 1, 1, 64, 0, False, True), (2049, 4, 4, 64, 32, False, True), (2300, 3, 3, 256, 256, True, True),
    (6, 0, 2, 128, 128, False, True), (6, 2, 0, 128, 128, True, True), (11, 70, 1, 64, 16, False, True)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(int(x)) for x in c))
def test_heads(case, dtype):
    from paper_2606_30391_amd import festina
    T, heads, kv, dim, rotated, inter, norm = case
    rng = np.random.default_rng(T)
    t = TYPES[dtype][0]
    make = lambda *s: torch.from_numpy(rng.normal(size=s)).cuda().to(t)
    q, k = make(T, heads, dim), make(T, kv, dim)
    w = [torch.from_numpy(1 + 0.2 * rng.normal(size=dim)).cuda().to(t) if norm else None for _ in range(2)]
    position = rng.integers(0, 9000, T)
    position[::3] = rng.integers(-2 ** 31, 2 ** 31, len(position[::3]))
    print(f"[gpu] {case} {dtype}", flush=True)
    r = festina.DeviceRotary(_freq(rotated // 2), dim, *w, 1e-6, inter)
    got = r.apply(q, k, torch.tensor(position, dtype=torch.int32, device="cuda"))
    for x, y, g in ((q, got[0], w[0]), (k, got[1], w[1])):
        want, bound = D.rotate(x.double().cpu().numpy(), position, _freq(rotated // 2),
                               None if g is None else g.double().cpu().numpy(), 1e-6, inter)
        assert _near(y, want, bound, dtype)
        if not norm:                                         # what is not rotated stays as it is
            assert torch.equal(y[..., rotated:], x[..., rotated:])


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_places(dtype):
    """Slices of one projection's output, rows that leave no alignment, outputs in the inputs' own memory, and one weight only."""
    from paper_2606_30391_amd import festina
    rng = np.random.default_rng(4)
    t = TYPES[dtype][0]
    position = torch.arange(9, dtype=torch.int32, device="cuda") * 1000
    w = torch.from_numpy(rng.normal(size=64)).cuda().to(t)
    r = festina.DeviceRotary(_freq(32), 64, None, w)
    for pad in (0, 1, 8):
        both = torch.from_numpy(rng.normal(size=(9, 8 * 64 + pad))).cuda().to(t)
        was = both.clone()
        heads = both[:, pad:].reshape(9, 8, 64) if pad == 0 else both[:, pad:].unflatten(1, (8, 64))
        q, k, v = heads[:, :5], heads[:, 5:7], heads[:, 7:]
        assert q.data_ptr() == both.data_ptr() + pad * both.element_size()
        host = [x.double().cpu().numpy() for x in (q, k)]
        print(f"[gpu] {dtype} {pad} elements before the heads", flush=True)
        apart = r.apply(q, k, position)
        assert torch.equal(both, was)
        assert r.apply(q, k, position, q_out=q, k_out=k)[0] is q
        assert torch.equal(q, apart[0]) and torch.equal(k, apart[1])
        assert torch.equal(v, was[:, pad:].unflatten(1, (8, 64))[:, 7:]) and torch.equal(both[:, :pad], was[:, :pad])
        for x, y, g in ((host[0], q, None), (host[1], k, w)):
            want, bound = D.rotate(x, position.cpu().numpy(), _freq(32), None if g is None else g.double().cpu().numpy())
            assert _near(y, want, bound, dtype)
        turned = torch.from_numpy(rng.normal(size=(8, 9, 64))).cuda().to(t).transpose(0, 1)       # heads before tokens
        a, b = r.apply(turned[:, :6], turned[:, 6:], position)
        c, d = r.apply(turned[:, :6].contiguous(), turned[:, 6:].contiguous(), position)
        assert torch.equal(a, c) and torch.equal(b, d)


def test_zeros_large_values_and_what_is_not_finite():
    from paper_2606_30391_amd import festina
    r = festina.DeviceRotary(_freq(16), 64, torch.ones(64), torch.ones(64))
    x = torch.zeros((4, 1, 64), dtype=torch.float32, device="cuda")
    x[1, 0, 3], x[2, 0, 5], x[3] = 1e15, float("nan"), 1e-30
    position = torch.zeros(4, dtype=torch.int32, device="cuda")
    y, _ = r.apply(x, x.clone(), position)
    want, bound = D.rotate(x.double().cpu().numpy(), [0] * 4, _freq(16), np.ones(64))
    assert torch.equal(y[0], x[0]) and y[2].isnan().all()
    assert _near(y[[1, 3]], want[[1, 3]], bound[[1, 3]], "f32")
    plain = festina.DeviceRotary(_freq(16), 64)              # without a norm, an infinity stays among the elements of its pair
    x = torch.ones((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 0, 40], x[0, 0, 2] = float("inf"), float("nan")
    y, _ = plain.apply(x, x.clone(), position[:1] + 3)
    assert y[0, 0, 40] == float("inf") and y.isnan().nonzero()[:, 2].tolist() == [2, 18]
    assert torch.equal(y[0, 0, 32:], x[0, 0, 32:])


def test_refusals():
    from paper_2606_30391_amd import festina
    r = festina.DeviceRotary(_freq(32), 64)
    q, k = (torch.zeros((3, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    p = torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad in (lambda: r.apply(q[:2], k, p), lambda: r.apply(q, k.float(), p), lambda: r.apply(q, k, p.long()),
                lambda: r.apply(q, k, p[:2]), lambda: r.apply(q[..., :32], k, p), lambda: r.apply(q.cpu(), k, p),
                lambda: r.apply(q.double(), k.double(), p), lambda: r.apply(q, k, p, q_out=q[:, :3]),
                lambda: r.apply(q, k, p, k_out=k[:1].expand(3, 2, 64)), lambda: r.apply(q.requires_grad_(), k, p)):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            bad()
    with torch.no_grad():
        r.apply(q, k, p)
    with pytest.raises(ValueError):
        festina.DeviceRotary(_freq(32), 64, torch.ones(32))
    for freq, dim in ((_freq(20), 64), (_freq(64), 64), (_freq(8), 80)):
        with pytest.raises(festina.FestinaError):
            x = torch.zeros((1, 1, dim), dtype=torch.bfloat16, device="cuda")
            festina.DeviceRotary(freq, dim).apply(x, x.clone(), p[:1])


def test_graph_stream_and_no_tokens():
    from paper_2606_30391_amd import festina
    g = torch.Generator("cuda").manual_seed(2)
    r = festina.DeviceRotary(_freq(64), 128, torch.ones(128))
    q, k = (torch.randn((50, h, 128), generator=g, device="cuda").bfloat16() for h in (6, 2))
    p = torch.arange(50, dtype=torch.int32, device="cuda")
    want = r.apply(q, k, p)
    out = [torch.zeros_like(x) for x in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.apply(q, k, p, *out)
    for _ in range(3):
        for x in out:
            x.zero_()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(out, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = r.apply(q, k, p, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    none = r.apply(q[:0], k[:0], p[:0])
    assert none[0].shape == (0, 6, 128)


def test_outputs_that_share_memory_are_refused():
    from paper_2606_30391_amd import festina
    r = festina.DeviceRotary(_freq(32), 64)
    p = torch.arange(6, dtype=torch.int32, device="cuda")
    buf = torch.randn((6, 12, 64), device="cuda").bfloat16()
    was = buf.clone()
    q, k = buf[:, 1:9], buf[:, 10:12]
    fresh = torch.zeros((6, 8, 64), dtype=torch.bfloat16, device="cuda")
    for name, out in (("a head further", dict(q_out=buf[:, 0:8])), ("over the keys", dict(q_out=buf[:, 3:11])),
                      ("over the queries", dict(k_out=buf[:, 7:9])), ("each other", dict(q_out=fresh, k_out=fresh[:, :2])),
                      ("in place beside its input's", dict(q_out=q, k_out=q[:, 6:])),
                      ("half a head further", dict(q_out=buf.flatten(1)[:, 32:32 + 512].unflatten(1, (8, 64)))),
                      ("itself", dict(q_out=torch.zeros(9000, dtype=torch.bfloat16, device="cuda").as_strided((6, 8, 64), (512, 32, 1)))),
                      ("itself in another token", dict(k_out=torch.zeros(9000, dtype=torch.bfloat16, device="cuda").as_strided((6, 2, 64), (64, 64, 1))))):
        print(f"[gpu] {name}", flush=True)
        with pytest.raises(ValueError):
            r.apply(q, k, p, **out)
    assert torch.equal(buf, was)


def test_outputs_beside_their_inputs():
    from paper_2606_30391_amd import festina
    r = festina.DeviceRotary(_freq(32), 64, torch.ones(64), torch.ones(64))
    for T in (1, 6):
        p = torch.arange(T, dtype=torch.int32, device="cuda") + 5
        q, k = (torch.randn((T, h, 64), device="cuda").bfloat16() for h in (4, 2))
        want = r.apply(q, k, p)
        pairs = torch.zeros((T, 6, 2, 64), dtype=torch.bfloat16, device="cuda")      # a head's output behind its input
        pairs[:, :4, 0], pairs[:, 4:, 0] = q, k
        print(f"[gpu] {T} tokens", flush=True)
        r.apply(pairs[:, :4, 0], pairs[:, 4:, 0], p, pairs[:, :4, 1], pairs[:, 4:, 1])
        assert torch.equal(pairs[:, :4, 1], want[0]) and torch.equal(pairs[:, 4:, 1], want[1])
        assert torch.equal(pairs[:, :4, 0], q) and torch.equal(pairs[:, 4:, 0], k)
        packed = torch.cat([q, k, torch.zeros_like(q), torch.zeros_like(k)], 1)      # all four of a token side by side
        r.apply(packed[:, :4], packed[:, 4:6], p, packed[:, 6:10], packed[:, 10:])
        assert torch.equal(packed[:, 6:], torch.cat(want, 1)) and torch.equal(packed[:, :6], torch.cat([q, k], 1))
        r.apply(packed[:, :4], packed[:, 4:6], p, packed[:, :4], packed[:, 4:6])     # and in place
        assert torch.equal(packed[:, :6], torch.cat(want, 1))
