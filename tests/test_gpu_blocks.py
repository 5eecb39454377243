"""GPU tests of block tables, slot maps and releases against the sequential definition: every integer equal."""
import numpy as np
import pytest

import kv_reference as K

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def _gpu(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(x, dtype)).cuda()


def _state(rng, R, bt, longest, decoding=0.5, spare=3, columns=None):
    """Requests holding tokens in a shuffled pool: (held, add, table, free_ids, n_free)."""
    held = np.where(rng.random(R) < decoding, rng.integers(0, longest + 1, R), 0)
    add = np.where(held > 0, rng.integers(0, 3, R), rng.integers(0, longest + 1, R))
    MB = columns or int(max(1, (-(-(held + add) // bt)).max(initial=1)))
    have = -(-held // bt)
    need = int((-(-(held + add) // bt) - have).sum())
    ids = rng.permutation(int(have.sum()) + need + spare)
    table = np.full((R, MB), -1)
    at = 0
    for r in range(R):
        table[r, :have[r]] = ids[at:at + have[r]]
        at += have[r]
    free = np.full(len(ids), -5)
    free[:len(ids) - at] = ids[at:]
    return held, add, table, free, len(ids) - at


def _check_extend(held, add, table, free, n_free, bt, max_tokens, alias=False):
    from paper_2606_30391_amd import festina as F
    want = K.extend(held, add, table, free, n_free, bt, max_tokens)
    b = F.DeviceBlocks(_gpu(held), _gpu(add), _gpu(table), _gpu(free), _gpu([n_free]), bt, max_tokens)
    b.slot.fill_(-77)
    if alias:                                               # updated in place
        b.length, b.n_free_out = b.held, b.n_free
        b._structs()
    b.extend()
    torch.cuda.synchronize()
    got = [x.cpu().numpy() for x in (b.table, b.slot, b.first, b.length, b.served, b.n_free_out)]
    for name, x, y in zip(("table", "slot", "first", "length", "served", "n_free"), got, want):
        assert np.array_equal(x, np.asarray(y).reshape(x.shape)), name
    return b, want


# one workgroup, the three launches, odd counts, more than one chunk of 256 requests, tokens past one fill stretch
CASES = [(1, 16, 1, 0.0), (1, 256, 700, 0.0), (7, 64, 300, 0.5), (255, 32, 40, 0.9), (1024, 16, 7, 0.9),
         (1025, 16, 7, 0.9), (300, 128, 3000, 0.3), (4097, 32, 90, 0.5), (2500, 16, 0, 1.0), (70, 16, 8192, 0.0)]


@pytest.mark.parametrize("R,bt,longest,decoding", CASES)
@pytest.mark.parametrize("budget", ["all", "blocks", "tokens"])
def test_extend_matches_the_definition(R, bt, longest, decoding, budget):
    rng = np.random.default_rng(R * 1000 + bt)
    held, add, table, free, n_free = _state(rng, R, bt, longest, decoding)
    tokens = int(add.sum()) + (13 if budget == "all" else 0)
    if budget == "blocks":
        n_free = n_free * 2 // 3
    if budget == "tokens":
        tokens = tokens * 2 // 3
    print(f"[gpu] extend R={R} bt={bt} tokens={tokens} budget={budget}", flush=True)
    _check_extend(held, add, table, free, n_free, bt, tokens)


@pytest.mark.parametrize("R", [40, 3000])
def test_extend_in_place_with_bad_requests_and_bad_ids(R):
    rng = np.random.default_rng(R)
    held, add, table, free, n_free = _state(rng, R, 32, 100)
    held[3], add[5], add[8] = -4, -1, 32 * table.shape[1] + 1     # never served, take nothing
    held[11], add[11] = 2 ** 31 - 1, 2 ** 31 - 1
    free[n_free // 2] = 10 ** 9                                   # no such block: its tokens have no slot
    if n_free > 3:
        free[n_free - 3] = -2
    table[table >= 0] = np.where(rng.random((table >= 0).sum()) < 0.1, -9, table[table >= 0])
    good = (held >= 0) & (add >= 0) & (held.astype(np.int64) + add <= 32 * table.shape[1])
    tokens = int(add[good].sum())
    print(f"[gpu] extend in place, bad requests R={R}", flush=True)
    _check_extend(held, add, table, free, n_free, 32, tokens, alias=True)


@pytest.mark.parametrize("n_free", [-3, 10 ** 6])
def test_extend_takes_a_free_count_outside_the_pool_at_the_nearer_end(n_free):
    rng = np.random.default_rng(5)
    held, add, table, free, _ = _state(rng, 30, 16, 60)
    free[:] = rng.permutation(len(free))
    print(f"[gpu] extend n_free={n_free}", flush=True)
    _check_extend(held, add, table, free, n_free, 16, int(add.sum()))


def test_extend_without_requests_or_tokens():
    none = np.zeros(0, np.int64)
    print("[gpu] extend nothing", flush=True)
    _check_extend(none, none, np.zeros((0, 4)), np.arange(9), 4, 16, 40)
    _check_extend(none, none, np.zeros((0, 4)), np.arange(9), 4, 16, 9000)
    _check_extend(np.array([5, 0]), np.array([0, 0]), np.array([[1], [-1]]), np.arange(9), 4, 16, 0)
    _check_extend(np.array([5, 0]), np.array([1, 1]), np.array([[1], [-1]]), np.arange(9), 4, 16, 0)


def test_many_idle_requests_between_two_busy_ones():
    """Stretches of requests without tokens longer than a workgroup's list."""
    R = 9000
    held, add = np.zeros(R, int), np.zeros(R, int)
    add[0] = add[4500] = add[R - 1] = 1500
    print("[gpu] extend idle requests", flush=True)
    _check_extend(held, add, np.full((R, 100), -1), np.arange(400)[::-1], 400, 16, 6000)


@pytest.mark.parametrize("R", [1, 200, 256, 257, 5000])
def test_release_then_extend_again(R):
    from paper_2606_30391_amd import festina as F
    rng = np.random.default_rng(R)
    bt = 32
    held, add, table, free, n_free = _state(rng, R, bt, 300, 0.8, spare=40)
    tokens = int(add.sum())
    print(f"[gpu] release R={R}", flush=True)
    b, want = _check_extend(held, add, table, free, n_free, bt, tokens)
    table, _, _, length, _, n = want
    b.advance()                                              # length and the count are the next step's
    done = rng.random(R) < 0.4
    b.release(_gpu(done, np.uint8))
    torch.cuda.synchronize()
    free2, length2, n2 = K.release(length, done, table, free, n, bt)
    assert np.array_equal(b.free_ids.cpu().numpy(), free2)
    assert np.array_equal(b.length.cpu().numpy(), length2) and int(b.n_free_out) == n2
    b.advance()
    add2 = rng.integers(0, 5, R)
    b.add.copy_(_gpu(np.where(length2 + add2 <= table.shape[1] * bt, add2, 0)))
    add2 = b.add.cpu().numpy()
    b.extend()
    torch.cuda.synchronize()
    want = K.extend(length2, add2, table, free2, n2, bt, tokens)
    for name, x, y in zip(("table", "slot", "first", "length", "served", "n_free"),
                          (b.table, b.slot, b.first, b.length, b.served, b.n_free_out), want):
        assert np.array_equal(x.cpu().numpy(), np.asarray(y).reshape(x.shape)), name


def test_release_of_more_ids_than_the_list_holds_and_of_bad_lengths():
    from paper_2606_30391_amd import festina as F
    held = np.array([64, 200, -1, 64, 32])
    table = np.arange(20).reshape(5, 4) % 6
    free = np.arange(6)
    done = np.array([1, 1, 1, 1, 0])
    print("[gpu] release overfull", flush=True)
    b = F.DeviceBlocks(_gpu(held), _gpu(held * 0), _gpu(table), _gpu(free), _gpu([3]), 32, 0)
    b.release(_gpu(done, np.uint8))
    torch.cuda.synchronize()
    want = K.release(held, done, table, free, 3, 32)
    assert np.array_equal(b.free_ids.cpu().numpy(), want[0]) and int(b.n_free_out) == want[2] == 6
    assert np.array_equal(b.length.cpu().numpy(), want[1])


def test_a_step_on_another_stream_and_in_a_graph():
    from paper_2606_30391_amd import festina as F
    rng = np.random.default_rng(9)
    for R in (50, 2000):
        held, add, table, free, n_free = _state(rng, R, 16, 100)
        tokens = int(add.sum())
        want = K.extend(held, add, table, free, n_free, 16, tokens)
        b = F.DeviceBlocks(_gpu(held), _gpu(add), _gpu(table), _gpu(free), _gpu([n_free]), 16, tokens)
        done = _gpu(np.ones(R), np.uint8)
        print(f"[gpu] extend on a stream, in a graph R={R}", flush=True)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        b.extend(stream=s)
        s.synchronize()
        assert np.array_equal(b.slot.cpu().numpy(), want[1])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b.extend()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.extend()
        for _ in range(3):
            for x in (b.slot, b.first, b.length, b.n_free_out):
                x.fill_(-7)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for name, x, y in zip(("table", "slot", "first", "length", "served", "n_free"),
                                  (b.table, b.slot, b.first, b.length, b.served, b.n_free_out), want):
                assert np.array_equal(x.cpu().numpy(), np.asarray(y).reshape(x.shape)), name


def test_binding_checks_its_tensors():
    from paper_2606_30391_amd import festina as F
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    good = dict(held=i(4), add=i(4), table=i(4, 2), free_ids=i(8), n_free=i(1), block_tokens=16, max_tokens=8)
    F.DeviceBlocks(**good)
    for key, bad in [("held", i(5)), ("add", i(4).long()), ("table", i(4, 4)[:, ::2]), ("n_free", i(2)),
                     ("free_ids", torch.zeros(8, dtype=torch.int32))]:
        with pytest.raises(ValueError):
            F.DeviceBlocks(**{**good, key: bad})
    b = F.DeviceBlocks(**good)
    with pytest.raises(ValueError):
        b.release(i(4))
    with pytest.raises(F.FestinaError):
        F.DeviceBlocks(**{**good, "block_tokens": 24}).extend()


@pytest.mark.parametrize("busy", [[0, -1], [0, 1, -2, -1], [5, -1]])
def test_a_million_idle_requests_cost_no_walk(busy):
    """Requests without tokens between two with some, all in one stretch of the fill: right, and found by few reads."""
    from paper_2606_30391_amd import festina as F
    R, bt = 1 << 20, 16
    held, add = np.full(R, 16), np.zeros(R, int)
    add[busy] = 37
    table = np.full((R, 4), -1)
    table[:, 0] = np.arange(R) % 64
    free = np.arange(64)
    print(f"[gpu] extend a million idle requests {busy}", flush=True)
    b, _ = _check_extend(held, add, table, free, 64, bt, 200)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    b.extend()
    end.record()
    torch.cuda.synchronize()
    print(f"{begin.elapsed_time(end):.3f} ms")
    assert begin.elapsed_time(end) < 10                     # all launches take 0.06; a read after the other 120
