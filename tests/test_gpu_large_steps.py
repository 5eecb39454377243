"""GPU tests around the sizes at which the serving step's calls take other kernels: many runs a workgroup in the store, sums in
a launch of their own and long fills in the block plans, releases in chunks and in place."""
import numpy as np
import pytest

import kv_reference as K
from test_gpu_blocks import _gpu, _state
from test_gpu_cache import _cache, _slots

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def _extend(held, add, table, free, n_free, bt, max_tokens):
    """kv_reference.extend over arrays."""
    held, add, (R, columns) = held.astype(np.int64), add.astype(np.int64), table.shape
    fits = (held >= 0) & (add >= 0) & (held + add <= columns * bt)
    have = np.where(fits, -(-held // bt), 0)
    need, takes = np.where(fits, -(-(held + add) // bt) - have, 0), np.where(fits, add, 0)
    served = fits & (np.cumsum(need) <= n_free) & (np.cumsum(takes) <= max_tokens)
    need, takes = np.where(served, need, 0), np.where(served, takes, 0)
    first = np.concatenate([[0], np.cumsum(takes)])
    used = np.cumsum(need) - need
    table = table.copy()
    r = np.repeat(np.arange(R), need)
    i = np.arange(need.sum()) - used[r]
    table[r, have[r] + i] = free[n_free - 1 - (used[r] + i)]
    r = np.repeat(np.arange(R), takes)
    p = held[r] + np.arange(takes.sum()) - first[r]
    ids = table[r, p // bt].astype(np.int64)
    slot = np.full(max_tokens, -1, np.int32)
    slot[:len(r)] = np.where((ids >= 0) & (ids < len(free)), ids * bt + p % bt, -1)
    return table, slot, first, held + takes, served, n_free - need.sum()


def test_the_reference_over_arrays_agrees_with_the_one_over_requests():
    rng = np.random.default_rng(1)
    for budget in (1.0, 0.6):
        held, add, table, free, n_free = _state(rng, 200, 16, 90)
        held[3], add[5], add[8] = -4, -1, 16 * table.shape[1] + 1
        args = (held, add, table, free, int(n_free * budget), 16, int(add.clip(0).sum()))
        for x, y in zip(_extend(*args), K.extend(*args)):
            assert np.array_equal(np.asarray(x).reshape(-1), np.asarray(y).reshape(-1))


def _check_extend(held, add, table, free, n_free, bt, tokens, in_place):
    from paper_2606_30391_amd import festina as F
    want = _extend(held, add, table, free, n_free, bt, tokens)
    b = F.DeviceBlocks(_gpu(held), _gpu(add), _gpu(table), _gpu(free), _gpu([n_free]), bt, tokens)
    b.slot.fill_(-77)
    if in_place:
        b.length, b.n_free_out = b.held, b.n_free
        b._structs()
    b.extend()
    torch.cuda.synchronize()
    for name, x, y in zip(("table", "slot", "first", "length", "served", "n_free"),
                          (b.table, b.slot, b.first, b.length, b.served, b.n_free_out), want):
        assert np.array_equal(x.cpu().numpy().reshape(-1), np.asarray(y).reshape(-1)), name


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("R", [16384, 16385, 40000])
@pytest.mark.parametrize("budget", ["all", "blocks", "tokens"])
def test_extends_of_many_requests(R, budget, in_place):
    rng = np.random.default_rng(R)
    held, add, table, free, n_free = _state(rng, R, 32, 70, 0.7)
    held[100], add[200] = -1, -5
    tokens = int(add.clip(0).sum()) + 13
    if budget == "blocks":
        n_free = n_free * 2 // 3
    if budget == "tokens":
        tokens = tokens * 2 // 3
    print(f"[gpu] extend R={R} budget={budget} in place {in_place}", flush=True)
    _check_extend(held, add, table, free, n_free, 32, tokens, in_place)


@pytest.mark.parametrize("R,longest,spare", [(300, 100000, 0), (20000, 1500, 777), (300, 100001, -12345)])
def test_extends_of_millions_of_slots(R, longest, spare):
    """From 8 Mi slots on a wave fills stretches of 1,024; an odd number of them, and a budget that ends inside a request."""
    rng = np.random.default_rng(R + longest)
    held, add, table, free, n_free = _state(rng, R, 256, longest, 0.3)
    add[::7] = np.where(held[::7] > 0, 0, add[::7])
    tokens = int(add.sum()) + spare
    tokens += 1 - tokens % 2
    assert tokens > 8 << 20
    print(f"[gpu] extend of {tokens} slots, R={R}", flush=True)
    _check_extend(held, add, table, free, n_free, 256, tokens, False)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("R", [64, 65, 5000, 32768, 32769, 40001])
def test_releases(R, in_place):
    """In place, and beyond 32,768 requests, whole chunks of 256 after sums in a launch of their own."""
    from paper_2606_30391_amd import festina as F
    rng = np.random.default_rng(R)
    bt = 16
    held, _, table, free, n_free = _state(rng, R, bt, 60, 0.9, spare=11)
    held[7] = -2
    done = rng.random(R) < 0.4
    print(f"[gpu] release R={R} in place {in_place}", flush=True)
    b = F.DeviceBlocks(_gpu(held), _gpu(held * 0), _gpu(table), _gpu(free), _gpu([n_free]), bt, 0)
    if in_place:
        b.length, b.n_free_out = b.held, b.n_free
        b._structs()
    want = K.release(held, done, table, free, n_free, bt)
    b.release(_gpu(done, np.uint8))
    torch.cuda.synchronize()
    assert np.array_equal(b.free_ids.cpu().numpy(), want[0])
    assert np.array_equal(b.length.cpu().numpy(), want[1]) and int(b.n_free_out) == want[2]


@pytest.mark.parametrize("T,H,D,bt,dtype", [(8191, 1, 64, 16, "f16"), (8192, 1, 64, 16, "f16"), (20000, 1, 64, 32, "bf16"),
                                            (4097, 4, 64, 64, "f32"), (2600, 7, 96, 16, "bf16"), (2050, 8, 128, 32, "f16"),
                                            (4500, 60, 64, 16, "bf16"), (900, 300, 64, 32, "bf16")])
def test_stores_of_several_runs_a_workgroup(T, H, D, bt, dtype):
    """A workgroup looks for runs among T H / 4,096 tokens, up to 64: ragged runs, some of one token, some of many blocks."""
    rng = np.random.default_rng(T + H)
    runs, left = [], T
    while left:
        n = min(left, int(rng.integers(1, 4) if rng.random() < 0.6 else rng.integers(1, 120)))
        runs.append((int(rng.integers(0, bt)), n))
        left -= n
    blocks = sum((o + n + bt - 1) // bt for o, n in runs)
    slot = _slots(rng, runs, blocks + 5, bt)
    cache, before = _cache(rng, blocks + 5, bt, H, D)
    t = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]
    spread = torch.from_numpy(2.0 ** rng.integers(-3, 4, (T, 1, 1))).cuda()
    k, v = ((torch.randn((T, H, D), device="cuda", generator=torch.Generator("cuda").manual_seed(i)) * spread).to(t)
            for i in (1, 2))
    print(f"[gpu] store T={T} H={H} D={D} bt={bt} {dtype}, {len(runs)} runs", flush=True)
    cache.store(k, v, torch.from_numpy(slot.astype(np.int32)).cuda())
    torch.cuda.synchronize()
    got = [x.cpu().numpy() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    # heads are independent: of many, the first, the last and every seventh are compared
    heads = sorted({0, H - 1, *range(0, H, 7 if H < 50 else 41)})
    want = K.store(*(x[:, heads] for x in before), *(x[:, heads].float().cpu().numpy() for x in (k, v)), slot, bt)
    assert np.array_equal(got[2][:, heads], want[2]) and np.array_equal(got[3][:, heads], want[3])
    assert K.same_codes(got[0][:, heads], want[0])
    assert K.same_codes(got[1][:, heads], want[1])
