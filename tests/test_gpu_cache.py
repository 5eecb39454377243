"""GPU tests of the write into the 8-bit key/value cache: codes and scales equal to the 64-bit definition's (every
product with a power of two is exact, so there is one right code), and nothing else touched."""
import numpy as np
import pytest

import kv_reference as K

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _cache(rng, n_blocks, bt, H, D):
    from paper_2606_30391_amd import festina as F
    k = rng.integers(0, 256, (n_blocks, H, bt, D), dtype=np.uint8)
    v = rng.integers(0, 256, (n_blocks, H, D, bt), dtype=np.uint8)
    ks, vs = (2.0 ** rng.integers(-9, -4, (n_blocks, H)) for _ in range(2))
    up = lambda x: torch.from_numpy(x).cuda()
    return F.DeviceCache(up(k), up(v), up(ks.astype(np.float32)), up(vs.astype(np.float32))), (k, v, ks, vs)


def _check(cache, before, k, v, slot, bt, stream=None):
    want = K.store(*before, k.float().cpu().numpy(), v.float().cpu().numpy(), slot, bt)
    cache.store(k, v, torch.from_numpy(np.asarray(slot, np.int32)).cuda(), stream=stream)
    torch.cuda.synchronize()
    got = [x.cpu().numpy() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    assert np.array_equal(got[2], want[2]) and np.array_equal(got[3], want[3])
    assert K.same_codes(got[0], want[0])
    assert K.same_codes(got[1], want[1])
    return got


def _slots(rng, runs, n_blocks, bt):
    """Slots of runs of (offset, tokens): consecutive blocks of a shuffled order, a run per block."""
    ids = rng.permutation(n_blocks)
    slot, at = [], 0
    for off, n in runs:
        p = off
        while n > 0:
            m = min(n, bt - p)
            slot += list(range(int(ids[at]) * bt + p, int(ids[at]) * bt + p + m))
            at, n, p = at + 1, n - m, 0
    return np.array(slot, np.int64)


RUNS = [[(0, 1)], [(5, 1), (0, 1), (15, 1)], [(3, 40), (0, 16), (9, 2), (0, 5)], [(1, 100), (0, 257), (13, 3)]]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bt", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("D,H", [(64, 3), (96, 1), (128, 2), (256, 1)])
def test_store_matches_the_definition(dtype, bt, D, H):
    rng = np.random.default_rng(bt * D + H)
    for runs in RUNS:
        slot = _slots(rng, runs, 64, bt)
        cache, before = _cache(rng, 64, bt, H, D)
        spread = 2.0 ** rng.integers(-3, 4, (len(slot), H, 1))
        k, v = (torch.from_numpy(rng.normal(0, 1, (len(slot), H, D)) * spread).to(TYPES[dtype]).cuda() for _ in range(2))
        print(f"[gpu] store {dtype} bt={bt} D={D} H={H} runs={runs}", flush=True)
        _check(cache, before, k, v, slot, bt)


def test_token_by_token_grows_the_scale():
    """A block filled one token a call, magnitudes rising: the older codes follow every change of scale."""
    rng = np.random.default_rng(3)
    bt, H, D = 32, 2, 64
    cache, state = _cache(rng, 4, bt, H, D)
    for i in range(bt):
        x = rng.normal(0, 1.5 ** (i % 11), (2, 1, H, D))
        k, v = (torch.from_numpy(y).to(torch.bfloat16).cuda() for y in x)
        print(f"[gpu] store token {i}", flush=True)
        state = _check(cache, state, k, v, [2 * bt + i], bt)


@pytest.mark.parametrize("T", [2048, 2049, 5000])
def test_many_tokens_of_ragged_runs(T):
    """Around the size from which a workgroup looks for runs among several tokens."""
    rng = np.random.default_rng(T)
    bt, H, D = 32, 1, 64
    runs, left = [], T
    while left:
        off = int(rng.integers(0, bt))
        n = min(left, int(rng.integers(1, 90)))
        runs.append((off, n))
        left -= n
    blocks = sum((o + n + bt - 1) // bt for o, n in runs)
    slot = _slots(rng, runs, blocks + 5, bt)
    cache, before = _cache(rng, blocks + 5, bt, H, D)
    k, v = (torch.from_numpy(rng.normal(0, 1, (T, H, D))).to(torch.float16).cuda() for _ in range(2))
    print(f"[gpu] store ragged T={T}", flush=True)
    _check(cache, before, k, v, slot, bt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extremes(dtype):
    """Zeros, subnormals, ties, the format's ends, infinities and NaN; a token of nothing but NaN."""
    rng = np.random.default_rng(11)
    bt, H, D = 16, 1, 64
    rows = [np.zeros(D), np.full(D, np.nan), np.full(D, np.inf), np.full(D, 1e-38), np.full(D, 3e38), -np.full(D, 1e30),
            np.where(np.arange(D) == 7, np.inf, rng.normal(0, 1, D)), np.where(np.arange(D) == 9, -np.nan, 448.0),
            np.where(np.arange(D) == 0, 448.0, np.arange(D) * 2.0 ** -10), np.where(np.arange(D) == 0, 449.0, 1.0),
            np.where(np.arange(D) == 0, -256.0, (np.arange(D) + 0.5) * 2), np.full(D, -0.0)]
    for off in (0, 3):
        for i, row in enumerate(rows):
            cache, before = _cache(rng, 3, bt, H, D)
            x = torch.from_numpy(np.asarray(row)[None, None]).to(TYPES[dtype]).cuda()
            print(f"[gpu] store extreme {i} offset {off} {dtype}", flush=True)
            _check(cache, before, x, -x, [bt + off], bt)


def test_slots_that_are_nowhere_store_nothing():
    rng = np.random.default_rng(12)
    bt, H, D, n = 16, 2, 64, 6
    cache, before = _cache(rng, n, bt, H, D)
    slot = [-1, 5, 6, n * bt, 2 ** 31 - 1, -2 ** 31, 17, 40, 39, -1]
    x = torch.from_numpy(rng.normal(0, 1, (len(slot), H, D))).to(torch.bfloat16).cuda()
    slot[8] = 4 * bt                                              # (a block of its own)
    print("[gpu] store nowhere", flush=True)
    _check(cache, before, x, x, slot, bt)
    cache.store(x[:0], x[:0], torch.zeros(0, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["packed", "heads first", "odd", "broadcast"])
def test_strides(dtype, layout):
    rng = np.random.default_rng(13)
    bt, H, D, T = 32, 3, 96, 75
    t = TYPES[dtype]
    make = lambda *s: torch.from_numpy(rng.normal(0, 1, s)).to(t).cuda()
    if layout == "packed":
        both = make(T, 4 * H, D)
        k, v = both[:, 2 * H:3 * H], both[:, 3 * H:]
    elif layout == "heads first":
        k, v = make(H, T, D).transpose(0, 1), make(H, T, D).transpose(0, 1)
    elif layout == "odd":                                          # rows at any element
        k, v = make(T, H, D + 3)[:, :, 1:D + 1], make(T, H, D + 5)[:, :, 3:D + 3]
    else:                                                          # one head's keys for all heads
        k, v = make(T, 1, D).expand(T, H, D), make(1, H, D).expand(T, H, D)
    cache, before = _cache(rng, 8, bt, H, D)
    print(f"[gpu] store strides {layout} {dtype}", flush=True)
    _check(cache, before, k, v, _slots(rng, [(7, T)], 8, bt), bt)


def test_a_cache_past_32_bit_offsets():
    """Blocks whose codes lie beyond 2^32 bytes: 70,000 blocks of 64 tokens x 1,024 elements (4.6 GB each)."""
    from paper_2606_30391_amd import festina as F
    bt, H, D, n = 64, 4, 256, 70_000
    rng = np.random.default_rng(14)
    print("[gpu] store past 32 bits", flush=True)
    cache = F.DeviceCache.empty(n, bt, H, D)
    ids = [n - 1, 66_000, 2]
    slot = np.concatenate([np.arange(i * bt, i * bt + m) for i, m in zip(ids, (64, 20, 1))])
    k, v = (torch.from_numpy(rng.normal(0, 1, (len(slot), H, D))).to(torch.bfloat16).cuda() for _ in range(2))
    cache.k[ids] = 0
    cache.v[ids] = 0
    cache.store(k, v, torch.from_numpy(slot.astype(np.int32)).cuda())
    torch.cuda.synchronize()
    small = np.concatenate([np.arange(i * bt, i * bt + m) for i, m in zip(range(3), (64, 20, 1))])
    zeros = np.zeros((3, H, bt, D), np.uint8)
    want = K.store(zeros, zeros.transpose(0, 1, 3, 2), np.zeros((3, H)), np.zeros((3, H)), k.float().cpu().numpy(),
                   v.float().cpu().numpy(), small, bt)
    for got, w in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), want):
        g = got[ids].cpu().numpy()
        assert K.same_codes(g, w) if g.dtype == np.uint8 else np.array_equal(g, w)


def test_a_stream_and_a_graph():
    rng = np.random.default_rng(15)
    bt, H, D = 16, 2, 128
    cache, before = _cache(rng, 9, bt, H, D)
    slot = _slots(rng, [(3, 20), (0, 40)], 9, bt)
    k, v = (torch.from_numpy(rng.normal(0, 1, (len(slot), H, D))).to(torch.bfloat16).cuda() for _ in range(2))
    print("[gpu] store on a stream, in a graph", flush=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    want = _check(cache, before, k, v, slot, bt, stream=s)
    st = torch.from_numpy(slot.astype(np.int32)).cuda()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.store(k, v, st)
    for _ in range(3):
        for t, x in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), before):
            t.copy_(torch.from_numpy(np.asarray(x)).to(t.dtype))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), want):
            assert np.array_equal(t.cpu().numpy(), w)


def test_binding_checks_its_tensors():
    from paper_2606_30391_amd import festina as F
    cache = F.DeviceCache.empty(4, 16, 2, 64)
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    slot = torch.zeros(3, dtype=torch.int32, device="cuda")
    for k, v, s in [(x[:, :1], x, slot), (x, x[:2], slot), (x.float(), x, slot), (x.double(), x.double(), slot),
                    (x, x, slot[:2]), (x, x, slot.long()), (x.transpose(1, 2), x, slot), (x.cpu(), x, slot)]:
        with pytest.raises(ValueError):
            cache.store(k, v, s)
    with pytest.raises(F.FestinaError):
        F.DeviceCache.empty(4, 16, 2, 80).store(x.new_zeros((3, 2, 80)), x.new_zeros((3, 2, 80)), slot)
