"""GPU tests of attention over draft trees against the definition in 64 bits; the bounds come from the arithmetic
(kv_reference.attend_bounds): float32 logits and sums, weights in half precision, one rounding of the output."""
import numpy as np
import pytest

import drafts_reference as D
import kv_reference as K

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -11)}


class Case:
    """Requests of (length, new tokens) over a shuffled pool; what no request holds is NaN codes."""

    def __init__(self, rng, requests, dim=128, H=2, G=4, bt=32, dtype="bf16", spread=3, columns=None, words=False, extra=2):
        self.dim, self.H, self.G, self.bt, self.dtype = dim, H, G, bt, dtype
        self.length = np.array([x for x, _ in requests], np.int64)
        self.new = np.array([x for _, x in requests], np.int64)
        self.first = np.concatenate([[0], np.cumsum(self.new)])
        cols = -(-self.length // bt)
        MB = columns or int(max(1, cols.max(initial=1)))
        n = int(cols.sum()) + 2
        ids = rng.permutation(n)
        self.table = np.full((len(requests), MB), -1, np.int64)
        at = 0
        for r, c in enumerate(cols):
            self.table[r, :c] = ids[at:at + c]
            at += c
        self.k = K.encode(rng.normal(0, 112, (n, H, bt, dim)).clip(-448, 448))
        self.v = K.encode(rng.normal(0, 112, (n, H, dim, bt)).clip(-448, 448))
        self.ks = (2.0 ** rng.integers(-8, -5, (n, H))).astype(np.float32)
        self.vs = (2.0 ** rng.integers(-10, -3, (n, H))).astype(np.float32)
        held = np.zeros((n, bt), bool)
        for r, L in enumerate(self.length):
            for p in range(L):
                held[self.table[r, p // bt], p % bt] = True
        self.k[~held[:, None, :].repeat(H, 1)] = 0xFF
        np.swapaxes(self.v, 2, 3)[~held[:, None, :].repeat(H, 1)] = 0x7F
        self.T = int(self.first[-1]) + extra
        self.seen = [0] * self.T
        for r, m in enumerate(self.new):
            f = int(self.first[r])
            parent = D.tree(rng, m, spread) if m <= 64 else []
            for i, line in enumerate(D.paths(parent, m) if m <= 64 else []):
                self.seen[f + i] = sum(1 << x for x in line)
            if words:
                for i in range(m):
                    self.seen[f + i] = int(rng.integers(0, 2 ** 63)) * 2 + int(rng.integers(0, 2)) if rng.random() < 0.8 else 0
        q = torch.from_numpy(rng.normal(size=(self.T, H * G, dim))).to(TYPES[dtype][0])
        self.q = q.cuda()

    def cache(self):
        from paper_2606_30391_amd import festina
        return festina.DeviceCache(*(torch.from_numpy(x).cuda() for x in (self.k, self.v, self.ks, self.vs)))

    def device(self):
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
        signed = [x - 2 ** 64 if x >= 2 ** 63 else x for x in self.seen]
        return i32(self.table), i32(self.length), i32(self.first), torch.tensor(signed, dtype=torch.int64, device="cuda")

    def run(self, window=0, max_new=None, **k):
        table, length, first, seen = self.device()
        out = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device="cuda")
        lse = torch.full(self.q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
        return self.cache().attend(self.q, table, length, first, max_new or int(max(1, self.new.max(initial=1))), window=window,
                                   seen=seen, out=out, lse=lse, **k)

    def check(self, got, window=0):
        out, lse = (x.double().cpu().numpy() for x in got)
        want, wlse, mag = D.attend(self.q.double().cpu().numpy(), self.k, self.v, self.ks, self.vs, self.table, self.length,
                                   self.first, self.seen, self.dim ** -0.5, window)
        to, tl = K.attend_bounds(want, wlse, mag, self.dim, TYPES[self.dtype][1])
        n = int(self.first[-1])
        assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()                       # rows of no request
        w, x = want[:n], out[:n]
        assert np.array_equal(np.isnan(w), np.isnan(x))
        assert (np.abs(x - w) <= to[:n])[~np.isnan(w)].all()
        wl, xl = wlse[:n], lse[:n]
        assert np.array_equal(np.isneginf(wl), np.isneginf(xl)) and np.array_equal(np.isnan(wl), np.isnan(xl))
        fine = np.isfinite(wl)
        assert (np.abs(xl - wl) <= tl[:n])[fine].all()


SHAPES = [  # requests, dim, kv heads, group, block, type
    ([(403, 8)], 128, 8, 4, 64, "bf16"), ([(1, 1)], 64, 1, 1, 16, "f16"), ([(64, 64), (70, 64), (63, 1)], 64, 2, 2, 32, "bf16"),
    ([(300, 16), (5, 5), (0, 0), (1000, 33), (129, 64), (64, 3)], 128, 2, 4, 64, "bf16"),
    ([(300, 16), (5, 5), (0, 0), (1000, 33), (129, 64), (64, 3)], 96, 1, 8, 16, "f16"),
    ([(700, 20), (131, 1), (66, 2), (600, 64)], 256, 2, 2, 128, "bf16"), ([(700, 20), (131, 1), (66, 2)], 256, 1, 16, 256, "f16"),
    ([(2000, 64), (100, 1), (130, 2)], 64, 7, 2, 32, "f16"), ([(900, 5)] * 12, 96, 2, 1, 64, "bf16"),
    ([(1500, 70), (900, 31), (64, 64), (12, 2)], 64, 2, 2, 16, "bf16"),                # beside a run
    ([(1500, 170), (900, 31), (64, 64), (12, 2)], 128, 1, 4, 64, "f16"),
    ([(100, 90), (300, 31), (64, 64), (12, 2)], 64, 2, 1, 64, "bf16"), ([(65, 65), (300, 64)], 128, 1, 1, 16, "f16"),   # and in a short table
    ([(500, 32), (77, 20), (64, 30), (512, 32)], 128, 1, 4, 64, "bf16"), ([(500, 8), (77, 3)], 256, 1, 16, 64, "f16"),     # eight row tiles of one launch
    ([(9, 2), (65, 1)] * 300, 64, 1, 2, 16, "bf16")]                                   # more than a workgroup sums


@pytest.mark.parametrize("n", range(len(SHAPES)))
@pytest.mark.parametrize("window", [0, 40, 300])
def test_trees(n, window):
    requests, dim, H, G, bt, dtype = SHAPES[n]
    c = Case(np.random.default_rng(n), requests, dim, H, G, bt, dtype)
    print(f"[gpu] {SHAPES[n][1:]} window {window} requests {requests[:6]}", flush=True)
    c.check(c.run(window), window)


@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_words_that_are_no_trees_and_windows_shorter_than_a_path(dim):
    for n, window in enumerate((0, 1, 5, 64)):
        c = Case(np.random.default_rng(n), [(500, 60), (64, 64), (20, 7), (1000, 12)], dim, 1, 4, 32, "f16", words=True)
        print(f"[gpu] dim {dim} window {window}", flush=True)
        c.check(c.run(window), window)


def test_chains_equal_runs():
    """A tree whose every node follows the one before is what attend() without it computes, bit for bit where it takes the same
    kernel, else within the bounds."""
    c = Case(np.random.default_rng(3), [(400, 4), (200, 64), (70, 20)], 64, 2, 2, 32, "f16", spread=1)
    table, length, first, seen = c.device()
    for window in (0, 100):
        a = c.cache().attend(c.q, table, length, first, 64, window=window, seen=seen)
        b = c.cache().attend(c.q, table, length, first, 64, window=window)
        n = int(c.first[-1])
        c.check([torch.cat([x[:n], torch.full_like(x[n:], 7.0)]) for x in a], window)
        assert (a[0][:n].double() - b[0][:n].double()).abs().max() < 0.01


def test_nan_at_a_node_reaches_only_the_rows_that_see_it():
    for dim, G, requests in ((128, 4, [(300, 30), (64, 8)]), (64, 1, [(500, 12), (33, 33)]), (96, 8, [(700, 64)]), (256, 1, [(90, 40)])):
        c = Case(np.random.default_rng(dim), requests, dim, 2, G, 32, "bf16")
        for r, (L, n) in enumerate(requests):
            for node, which in ((n - 1, 0), (n // 2, 1), (n - 2, 1)):
                p = L - n + node
                b, o = c.table[r, p // 32], p % 32
                if which:
                    c.v[b, 1, 5, o] = 0xFF
                else:
                    c.k[b, 0, o, 3] = 0x7F
        print(f"[gpu] dim {dim} group {G}", flush=True)
        c.check(c.run())


def test_blocks_that_are_not_there_and_fewer_held_than_new():
    c = Case(np.random.default_rng(4), [(300, 20), (40, 33), (600, 64)], 64, 1, 4, 16, "bf16")
    c.table[0, 2], c.table[1, 2], c.table[2, 37] = -1, 10 ** 6, -5
    c.check(c.run())
    c = Case(np.random.default_rng(5), [(300, 20), (40, 33), (600, 64)], 128, 1, 4, 16, "bf16")
    c.length[1] = 20                                         # nodes 0 .. 12 have no key
    c.check(c.run())


def test_positions_past_what_the_table_holds_are_cut():
    c = Case(np.random.default_rng(6), [(300, 20), (70, 33)], 64, 2, 2, 32, "f16")
    want = c.run()
    c.length[0] = 10 ** 6
    got = c.run()
    n = slice(20, 53)
    assert torch.equal(got[0][n], want[0][n]) and torch.isfinite(got[0][:20].float()).logical_not().any()   # (reads NaN slots)


def test_a_long_cache_split_over_the_keys():
    """One request of 40,000 tokens: compared row by row with attend() of the node's path alone."""
    from paper_2606_30391_amd import festina
    g = torch.Generator("cuda").manual_seed(1)
    L, n, bt, H, G, dim = 40000, 24, 64, 2, 4, 128
    blocks = -(-L // bt)
    k, v = (torch.randn((blocks, H, *s), generator=g, device="cuda").mul_(100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            for s in ((bt, dim), (dim, bt)))
    sc = torch.full((blocks, H), 2.0 ** -7, device="cuda")
    cache = festina.DeviceCache(k, v, sc, sc.clone())
    table = torch.randperm(blocks, generator=g, device="cuda").int()[None].contiguous()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    parent = D.tree(np.random.default_rng(2), n, 3)
    q = torch.randn((n, H * G, dim), generator=g, device="cuda").half()
    seen = torch.tensor([sum(1 << x for x in line) for line in D.paths(parent, n)], device="cuda")
    out, lse = cache.attend(q, table, i32([L]), i32([0, n]), n, seen=seen)
    # every node's path put together behind the cached tokens, in its own last blocks
    f8 = lambda x: x.view(torch.float8_e4m3fn).float()
    ks = f8(k[table[0].long()]).permute(1, 0, 2, 3).reshape(H, -1, dim)[:, :L] * 2.0 ** -7
    vs = f8(v[table[0].long()]).permute(1, 0, 3, 2).reshape(H, -1, dim)[:, :L] * 2.0 ** -7
    for i, line in enumerate(D.paths(parent, n)):
        at = torch.tensor(list(range(L - n)) + [L - n + x for x in line], device="cuda")
        for h in (0, H * G - 1):
            x = ks[h // G][at].double() @ q[i, h].double() * dim ** -0.5
            w = torch.softmax(x, 0)
            want = w @ vs[h // G][at].double()
            size = w @ vs[h // G][at].double().abs()
            assert ((out[i, h].double() - want).abs() <= 2.0 ** -11 * want.abs() + size * 2.0 ** -10).all()
            assert abs(float(lse[i, h]) - float(torch.logsumexp(x, 0))) < 1e-4


def test_queries_out_of_a_projection_streams_and_graphs():
    c = Case(np.random.default_rng(7), [(300, 16), (40, 9), (700, 33)], 128, 2, 2, 64, "bf16")
    table, length, first, seen = c.device()
    cache = c.cache()
    wide = torch.randn((c.T, 8, 128), device="cuda").bfloat16()
    wide[:, 2:6] = c.q
    out = torch.full_like(wide, 7.0)
    got = cache.attend(wide[:, 2:6], table, length, first, 33, seen=seen, out=out[:, 1:5])
    want = cache.attend(c.q, table, length, first, 33, seen=seen)
    n = int(c.first[-1])
    assert torch.equal(out[:n, 1:5], want[0][:n]) and (out[:, 0] == 7).all() and (out[:, 5:] == 7).all()
    assert torch.equal(got[1][:n], want[1][:n])
    res = [torch.zeros_like(x) for x in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(c.q, table, length, first, 33, seen=seen, out=res[0], lse=res[1])
    for _ in range(3):
        for x in res:
            x.zero_()
        graph.replay()
        cache.attend(c.q, table, length, first, 33, seen=seen)           # the eager call has scratch of its own
        assert all(torch.equal(x[:n], y[:n]) for x, y in zip(res, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = cache.attend(c.q, table, length, first, 33, seen=seen, stream=side)
    side.synchronize()
    assert all(torch.equal(x[:n], y[:n]) for x, y in zip(a, want))
    for bad in (seen[:-1], seen.int(), seen.cpu(), seen[::2]):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            cache.attend(c.q, table, length, first, 33, seen=bad)


def _against_64_bits(dim, H, G, bt, dtype, lengths, new, window=0, seed=0):
    """Many or long requests: the same definition on the device in 64 bits, request by request."""
    from paper_2606_30391_amd import festina
    rng = np.random.default_rng(seed)
    g = torch.Generator("cuda").manual_seed(seed)
    R, T, cols = len(lengths), int(sum(new)), [-(-x // bt) for x in lengths]
    n = sum(cols) + 1
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")
    k, v = (randn(n, H, *s).mul_(112).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for s in ((bt, dim), (dim, bt)))
    ks, vs = (torch.exp2(torch.randint(lo, hi, (n, H), generator=g, device="cuda").float()) for lo, hi in ((-8, -5), (-10, -3)))
    ids = torch.randperm(n, generator=g, device="cuda").int()
    table = torch.full((R, max(cols)), -1, dtype=torch.int32, device="cuda")
    first, at = np.concatenate([[0], np.cumsum(new)]), 0
    words, sees = [], []
    for r, c in enumerate(cols):
        table[r, :c] = ids[at:at + c]
        at += c
        lines = D.paths(D.tree(rng, new[r], 3), new[r]) if new[r] <= 64 else []
        words += [sum(1 << x for x in line) for line in lines] or [0] * new[r]
        sees.append(lines)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
    q = randn(T, H * G, dim).to(TYPES[dtype][0])
    seen = torch.tensor([w - 2 ** 64 if w >= 2 ** 63 else w for w in words], dtype=torch.int64, device="cuda")
    out, lse = festina.DeviceCache(k, v, ks, vs).attend(q, table, i32(lengths), i32(first), max(new), window=window, seen=seen)
    worst = []
    f64 = lambda x: x.view(torch.float8_e4m3fn).double()
    for r in range(R):
        a, L, m = int(first[r]), lengths[r], new[r]
        before, mine = L - m, table[r, :cols[r]].long()
        mask = torch.zeros((m, L), dtype=torch.bool, device="cuda")
        j = torch.arange(L, device="cuda")
        for i in range(m):
            line = sees[r][i] if m <= 64 else list(range(i + 1))
            mask[i, :before] = True
            mask[i, before + torch.tensor(line, device="cuda")] = True
            if window:
                far = j <= before + len(line) - 1 - window
                mask[i] &= ~(far & (j < before))
        if m > 64 and window:
            mask &= j > before + torch.arange(m, device="cuda")[:, None] - window
        for h in range(H):
            K_ = (f64(k[mine, h]) * ks[mine, h].double()[:, None, None]).reshape(-1, dim)[:L]
            V_ = (f64(v[mine, h]) * vs[mine, h].double()[:, None, None]).transpose(1, 2).reshape(-1, dim)[:L]
            sc = vs[mine, h].double().repeat_interleave(bt)[:L]
            Q = q[a:a + m, h * G:(h + 1) * G].double().reshape(m * G, dim)
            x = (Q @ K_.T * dim ** -0.5).masked_fill(~mask.repeat_interleave(G, 0), -torch.inf)
            w = torch.softmax(x, 1)
            want = w @ V_
            keys = mask.sum(1).repeat_interleave(G).double()
            logit = (Q.abs() @ K_.T.abs()).amax(1) * dim ** -0.5
            vmax = ((V_ / sc[:, None]).abs().amax(0) * sc.max())[None].expand_as(want)
            to, tl = K.attend_bounds(want.cpu().numpy(), torch.logsumexp(x, 1).cpu().numpy(),
                                     ((w @ V_.abs()).cpu().numpy(), vmax.cpu().numpy(), logit.cpu().numpy(), keys.cpu().numpy()),
                                     dim, TYPES[dtype][1])
            o = out[a:a + m, h * G:(h + 1) * G].double().reshape(m * G, dim)
            l = lse[a:a + m, h * G:(h + 1) * G].double().reshape(-1)
            worst.append(float(((o - want).abs().cpu() / torch.from_numpy(to)).max()))
            worst.append(float(((l - torch.logsumexp(x, 1)).abs().cpu() / torch.from_numpy(tl)).max()))
    print(f"[gpu] of the bound at most {max(worst):.3f}", flush=True)
    assert max(worst) <= 1


@pytest.mark.parametrize("dim,H,G,bt,dtype,longest,new,window", [
    (128, 2, 4, 64, "bf16", 2500, 9, 0), (64, 1, 2, 16, "f16", 900, 40, 0), (96, 1, 8, 32, "bf16", 700, 5, 300)])
@pytest.mark.parametrize("R", [70, 530])
def test_many_requests(R, dim, H, G, bt, dtype, longest, new, window):
    """More requests than a wave has lanes, and than a workgroup sums; few and many units of keys for each workgroup."""
    rng = np.random.default_rng(R)
    lengths = [int(x) for x in rng.integers(1, longest if R == 70 else longest // 4, R)]
    count = [min(x, 1 + int(rng.integers(0, new))) for x in lengths]
    count[3] = min(lengths[3], new)
    print(f"[gpu] {R} requests, dim {dim}", flush=True)
    _against_64_bits(dim, H, G, bt, dtype, lengths, count, window, R)


@pytest.mark.parametrize("dim,H,G,bt,dtype,new", [(128, 4, 4, 64, "bf16", 16), (128, 4, 4, 128, "f16", 33), (64, 8, 2, 32, "bf16", 24),
                                                  (64, 6, 4, 64, "f16", 64), (96, 4, 4, 64, "bf16", 12), (256, 4, 2, 64, "bf16", 12)])
def test_long_requests_in_pieces(dim, H, G, bt, dtype, new):
    """So many keys that the workgroups take pieces of all tiles' line, short requests among the long ones."""
    lengths = [40000, 70, 25000, 130, 33333, 64, 21000, 16001]
    _against_64_bits(dim, H, G, bt, dtype, lengths, [new, 3, new, new, 1, min(new, 64), new // 2, new], 0, dim)


@pytest.mark.parametrize("requests,dim,G,max_new", [
    ([(300, 90)], 64, 1, None), ([(700, 70), (900, 65)], 128, 4, None), ([(300, 0), (40, 0)], 64, 1, 80),
    ([(30, 0)] * 20 + [(600, 0)], 96, 2, 70)])
def test_steps_without_trees(requests, dim, G, max_new):
    c = Case(np.random.default_rng(8), requests, dim, 2, G, 16, "bf16", extra=4)
    print(f"[gpu] dim {dim} group {G} requests {requests[:3]}", flush=True)
    for window in (0, 50):
        c.check(c.run(window, max_new), window)


@pytest.mark.parametrize("requests,dim,G", [([(300, 20), (40, 33), (600, 64)], 64, 4), ([(200, 4), (70, 9), (0, 2)], 128, 1),
                                            ([(700, 70), (90, 80), (300, 12)], 64, 2)])
def test_windows_past_all_positions_with_fewer_held_than_new(requests, dim, G):
    c = Case(np.random.default_rng(9), requests, dim, 2, G, 16, "bf16")
    c.length[1] = c.new[1] * 2 // 3
    print(f"[gpu] dim {dim} group {G} {requests}", flush=True)
    for window in (2 ** 31 - 1, 2 ** 31 - 64, 2 ** 40):
        c.check(c.run(window), window)
        table, length, first, _ = c.device()
        far, none = (c.cache().attend(c.q, table, length, first, int(c.new.max()), window=w) for w in (window, 0))
        n = int(c.first[-1])
        assert all(torch.equal(x[:n].nan_to_num(9e9), y[:n].nan_to_num(9e9)) for x, y in zip(far, none))
