"""GPU tests of draft trees, their acceptance, the move of the kept tokens and the blocks behind them, against
tests/drafts_reference.py.  Whole numbers and codes: everything is equal."""
import numpy as np
import pytest

import drafts_reference as D
import kv_reference as K

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

i32 = lambda x: torch.tensor(np.asarray(x, np.int64), dtype=torch.int32, device="cuda")


class Step:
    """Requests with `counts` new tokens each and what lies before them; tokens of a small vocabulary."""

    def __init__(self, rng, counts, before, spread=4, extra=3, words=3):
        self.counts, self.before = np.array(counts, np.int64), np.array(before, np.int64)
        self.length = self.counts + self.before
        self.first = np.concatenate([[0], np.cumsum(self.counts)]).astype(np.int64)
        self.T = int(self.first[-1]) + extra
        self.parent = np.full(self.T, -1)
        for r, n in enumerate(counts):
            self.parent[self.first[r]:self.first[r] + n] = D.tree(rng, n, spread) if n <= 64 else np.arange(n) - 1
        self.token, self.choice = rng.integers(0, words, (2, self.T))

    def device(self):
        from paper_2606_30391_amd import festina
        d = festina.DeviceDrafts(i32(self.parent), i32(self.token), len(self.counts))
        for x in (d.seen, d.position, d.path, d.kept, d.next, d.length):
            x.fill_(77)
        return d, i32(self.first), i32(self.length), i32(self.choice)

    def check(self, d, parent=None):
        parent = self.parent if parent is None else parent
        seen, position = D.plan(self.first, self.length, parent)
        path, kept, after, left = D.accept(self.first, self.length, parent, self.token, self.choice)
        word = lambda x: [v % 2 ** 64 for v in x.cpu().tolist()]
        keep77 = lambda x: [77 if v is None else v for v in x]
        assert word(d.seen) == keep77(seen) and d.position.cpu().tolist() == keep77(position)
        assert d.path.cpu().tolist() == keep77(path)
        assert (d.kept.cpu().tolist(), d.next.cpu().tolist(), d.length.cpu().tolist()) == (kept, after, left)


COUNTS = {"one": [1], "none": [0, 0, 0], "few": [8, 1, 0, 64, 63, 2], "run": [65, 3, 300, 0, 17], "chain": [64, 64],
          "many": list(range(65)) * 5}


@pytest.mark.parametrize("spread", [1, 2, 6, 64])
@pytest.mark.parametrize("name", COUNTS)
def test_plan_and_acceptance(name, spread):
    rng = np.random.default_rng(spread)
    counts = COUNTS[name]
    s = Step(rng, counts, rng.integers(0, 500, len(counts)), spread)
    print(f"[gpu] {name}, parents {spread} back", flush=True)
    d, first, length, choice = s.device()
    d.plan(first, length)
    d.accept(first, length, choice)
    s.check(d)


def test_parents_that_are_none_and_no_parents_at_all():
    from paper_2606_30391_amd import festina
    rng = np.random.default_rng(5)
    s = Step(rng, [30, 64, 5], [7, 0, 3])
    bad = rng.random(s.T) < 0.2
    s.parent[bad] = rng.choice([-9, 64, 2 ** 31 - 1, -2 ** 31], int(bad.sum()))
    d, first, length, choice = s.device()
    d.plan(first, length)
    d.accept(first, length, choice)
    s.check(d)
    lone = festina.DeviceDrafts(None, i32(s.token), 3)
    for x in (lone.seen, lone.position, lone.path):
        x.fill_(77)
    lone.plan(first, length)
    lone.accept(first, length, choice)
    s.check(lone, np.concatenate([np.arange(n) - 1 for n in (30, 64, 5)] + [np.full(3, -1)]))


def test_lengths_may_be_updated_in_place_and_numbers_past_the_tokens_are_bounded():
    """accept() into the lengths' own array; `first` entries past the tokens are cut off there."""
    import ctypes as C
    from paper_2606_30391_amd import festina
    s = Step(np.random.default_rng(6), [8, 20], [100, 3], extra=0)
    d, first, length, choice = s.device()
    d.accepted.length = C.c_void_p(length.data_ptr())
    d.accept(first, length, choice)
    assert length.cpu().tolist() == D.accept(s.first, s.length, s.parent, s.token, s.choice)[3]
    first = i32([0, 8, 10 ** 6])
    d, _, length, choice = s.device()
    d.plan(first, length)
    s.check_first = D.plan(s.first, s.length, s.parent)[0]
    assert [v % 2 ** 64 for v in d.seen.cpu().tolist()] == s.check_first
    assert festina.DeviceDrafts(None, None, 0, 0, "cuda").plan(i32([0]), i32([])) is None


class Caches:
    def __init__(self, rng, s, H, dim, bt, layers, odd=False):
        self.bt, cols = bt, -(-s.length // bt)
        self.MB = int(max(1, cols.max(initial=1)))
        n = int(cols.sum()) + 2
        ids = rng.permutation(n)
        self.table = np.full((len(s.counts), self.MB), -1, np.int64)
        at = 0
        for r, c in enumerate(cols):
            self.table[r, :c] = ids[at:at + c]
            at += c
        self.used, self.free = at, ids[at:]
        self.host = [(rng.integers(0, 256, (n, H, bt, dim)).astype(np.uint8), rng.integers(0, 256, (n, H, dim, bt)).astype(np.uint8),
                      (2.0 ** rng.integers(-8, -3, (n, H))).astype(np.float32), (2.0 ** rng.integers(-8, 2, (n, H))).astype(np.float32))
                     for _ in range(layers)]

    def device(self):
        from paper_2606_30391_amd import festina
        return [festina.DeviceCache(*(torch.from_numpy(x).cuda() for x in layer)) for layer in self.host]

    def check(self, caches, s, path, kept):
        for i, (c, host) in enumerate(zip(caches, self.host)):
            want = D.keep(*host, self.table, s.length, s.first, path, kept)
            assert K.same_codes(c.k.cpu().numpy(), want[0]), f"keys of layer {i}"
            assert K.same_codes(c.v.cpu().numpy(), want[1]), f"values of layer {i}"
            assert np.array_equal(c.k_scale.cpu().numpy(), want[2]) and np.array_equal(c.v_scale.cpu().numpy(), want[3])


def _paths(rng, s, share):
    path, kept = np.full(s.T, -1), np.zeros(len(s.counts), np.int64)
    for r, n in enumerate(s.counts):
        p = np.arange(n) if n > 64 else np.flatnonzero(rng.random(n) < share)
        path[s.first[r]:s.first[r] + len(p)] = p
        kept[r] = len(p)
    return path, kept


@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("bt", [16, 32, 64, 128, 256])
def test_kept_tokens(dim, bt):
    rng = np.random.default_rng(dim + bt)
    counts = [64, 1, 0, 17, 70, 40, 33, 64, 8]
    for share, layers, H in ((0.3, 2, 2), (0.9, 1, 1), (1.0, 1, 3)):
        s = Step(rng, counts, rng.integers(0, 2 * bt, len(counts)))
        c = Caches(rng, s, H, dim, bt, layers)
        path, kept = _paths(rng, s, share)
        print(f"[gpu] dim {dim} blocks of {bt} share {share}", flush=True)
        caches = c.device()
        caches[0].keep(i32(c.table), i32(s.length), i32(s.first), i32(path), i32(kept), also=caches[1:])
        c.check(caches, s, path, kept)


def test_more_layers_than_one_launch_takes():
    rng = np.random.default_rng(1)
    s = Step(rng, [20, 9], [5, 30])
    c = Caches(rng, s, 1, 64, 16, 66)
    path, kept = _paths(rng, s, 0.5)
    caches = c.device()
    caches[0].keep(i32(c.table), i32(s.length), i32(s.first), i32(path), i32(kept), also=caches[1:])
    c.check(caches, s, path, kept)
    with pytest.raises(ValueError, match="once"):
        caches[0].keep(i32(c.table), i32(s.length), i32(s.first), i32(path), i32(kept), also=caches)


def test_what_is_no_path_is_left_alone():
    """Paths that do not ascend or leave the request, counts past it, blocks that are not there, fewer tokens than new ones."""
    rng = np.random.default_rng(2)
    counts = [12] * 9
    s = Step(rng, counts, [5, 20, 20, 20, 20, 20, 20, 20, 20])
    c = Caches(rng, s, 2, 64, 16, 1)
    path, kept = _paths(rng, s, 0.5)
    at = lambda r: slice(s.first[r], s.first[r] + 4)
    kept[:] = 4
    for r in range(9):
        path[at(r)] = [0, 3, 5, 9]
    path[at(1)] = [0, 5, 3, 9]
    path[at(2)] = [0, 3, 3, 9]
    path[at(3)] = [0, 3, 5, 12]
    path[at(4)] = [-1, 3, 5, 9]
    kept[5] = 100                                            # cut to the request's 12, whose entries are no path
    path[s.first[5] + 4:s.first[5] + 12] = -1
    kept[6] = -3
    c.table[7, 1] = 10 ** 6
    s.length[8] = 10 ** 5                                    # more than the table holds
    caches = c.device()
    caches[0].keep(i32(c.table), i32(s.length), i32(s.first), i32(path), i32(kept))
    c.check(caches, s, path, kept)
    s.length[0] = 7                                          # fewer tokens than new ones
    caches = c.device()
    caches[0].keep(i32(c.table), i32(s.length), i32(s.first), i32(path), i32(kept))
    c.check(caches, s, path, kept)


@pytest.mark.parametrize("R", [1, 64, 65, 700, 33000])
@pytest.mark.parametrize("place", ["apart", "held", "keep"])
def test_blocks_behind_the_kept_tokens(R, place):
    from paper_2606_30391_amd import festina
    rng = np.random.default_rng(R)
    bt, MB = 16, 6
    held = rng.integers(0, MB * bt + 1, R)
    keep = np.maximum(held - rng.integers(0, 70, R), 0)
    odd = rng.random(R) < 0.1
    keep[odd] = rng.choice([-1, 10 ** 6, -2 ** 31], int(odd.sum()))
    held[::17] = -3
    keep[5::19], held[5::19] = 3, MB * bt + 40
    table = rng.permutation(R * MB).reshape(R, MB)
    n_blocks = R * MB
    free = np.full(n_blocks, -1)
    free[:2] = [4, 9]
    full = n_blocks - 5 if R == 700 else 2                   # the list ends inside
    want = D.trim(held, keep, table, free, full, bt)
    b = festina.DeviceBlocks(i32(held), i32(np.zeros(R)), i32(table), i32(free), i32([full]), bt, 0)
    k = i32(keep)
    if place == "held":
        b.length, b.n_free_out = b.held, b.n_free
    elif place == "keep":
        b.length = k
    b._structs()
    print(f"[gpu] {R} requests, lengths {place}", flush=True)
    b.trim(k)
    got = b.free_ids.cpu().numpy(), b.length.cpu().numpy(), int(b.n_free_out.item())
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]) and got[2] == want[2]


def test_a_graph_of_a_step_and_another_stream():
    """Plan, accept, keep and trim captured together and replayed, the caches restored in between; and on a side stream."""
    from paper_2606_30391_amd import festina
    rng = np.random.default_rng(8)
    counts = [30, 64, 0, 9, 70, 1]
    s = Step(rng, counts, rng.integers(0, 90, len(counts)), words=2)
    c = Caches(rng, s, 2, 64, 16, 2)
    d, first, length, choice = s.device()
    caches, table = c.device(), i32(c.table)
    path, kept, _, left = D.accept(s.first, s.length, s.parent, s.token, s.choice)
    path = np.array([-1 if x is None else x for x in path])
    n_blocks = len(c.host[0][0])
    free = torch.full((n_blocks,), -1, dtype=torch.int32, device="cuda")
    blocks = festina.DeviceBlocks(length, torch.zeros_like(length), table, free, i32([0]), 16, 0)
    want = D.trim(s.length, left, c.table, [-1] * n_blocks, 0, 16)

    def step(stream=None):
        d.plan(first, length, stream)
        d.accept(first, length, choice, stream)
        caches[0].keep(table, length, first, d.path, d.kept, also=caches[1:], stream=stream)
        blocks.trim(d.length, stream)

    def restore():
        for cache, host in zip(caches, c.host):
            for x, y in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), host):
                x.copy_(torch.from_numpy(y))
        for x in (d.seen, d.position, d.path, d.kept, d.next, d.length):
            x.fill_(77)
        free.fill_(-1)

    def check():
        torch.cuda.synchronize()
        s.check(d)
        c.check(caches, s, path, kept)
        assert np.array_equal(free.cpu().numpy(), want[0]) and int(blocks.n_free_out.item()) == want[2]

    step()                                                   # loads the kernels
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(3):
        restore()
        print(f"[gpu] replay {n}", flush=True)
        graph.replay()
        check()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        restore()
        torch.cuda.synchronize()
        step(stream)
        check()


def test_tensors_that_do_not_fit_are_refused():
    from paper_2606_30391_amd import festina
    s = Step(np.random.default_rng(9), [4, 4], [3, 3])
    d, first, length, choice = s.device()
    for bad in (lambda: d.plan(first[:-1], length), lambda: d.plan(first, length.long()), lambda: d.accept(first, length, choice[1:]),
                lambda: d.accept(first, length, choice.cpu()), lambda: festina.DeviceDrafts(None, None, 3),
                lambda: festina.DeviceDrafts(i32([1, 2]), i32([1]), 1),
                lambda: festina.DeviceDrafts(i32([-1]), None, 1).accept(i32([0, 1]), i32([1]), i32([1]))):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            bad()


def test_trees_on_another_device_than_the_results_are_refused():
    from paper_2606_30391_amd import festina
    for trees in ((i32([-1, 0]), None), (None, i32([1, 2]))):
        with pytest.raises(ValueError, match="on device 0, not on device -1"):
            festina.DeviceDrafts(*trees, 1, device="cpu")
