"""What the calls of a step of drafted tokens refuse, before anything is launched (no GPU needed): the C ABI with addresses
that are never followed, and the definitions of tests/drafts_reference.py against each other."""
import ctypes as C
import math

import numpy as np
import pytest

import drafts_reference as D
from paper_2606_30391_amd import festina as F
from test_abi_cpu import lib, no_gpu  # noqa: F401

FAKE = 0x100000
INVALID, UNSUPPORTED, OK, DEVICE = F.FESTINA_ERR_INVALID, F.FESTINA_ERR_UNSUPPORTED, F.FESTINA_OK, F.FESTINA_ERR_DEVICE


def _drafts(**k):
    a = dict(n_requests=4, n_tokens=40, first=FAKE, length=FAKE, parent=FAKE)
    return F.festina_drafts(**{**a, **k})


@no_gpu
@pytest.mark.parametrize("change,status", [
    (dict(), DEVICE), (dict(parent=None), DEVICE), (dict(n_requests=-1), INVALID), (dict(n_tokens=-1), INVALID),
    (dict(first=None), INVALID), (dict(length=None), INVALID), (dict(n_requests=(1 << 20) + 1), UNSUPPORTED),
    (dict(n_requests=0, first=None, length=None), OK)])
def test_plan_and_accept(lib, change, status):  # noqa: F811
    d = _drafts(**change)
    assert lib.festina_plan_drafts(C.byref(d), FAKE, FAKE, None) == status
    out = F.festina_accepted(FAKE, FAKE, FAKE, FAKE)
    assert lib.festina_accept_drafts(C.byref(d), FAKE, FAKE, C.byref(out), None) == status


@no_gpu
def test_plan_and_accept_refuse_missing_arrays(lib):  # noqa: F811
    d = _drafts()
    plan = lambda *a: lib.festina_plan_drafts(C.byref(d), *a, None)
    assert plan(None, None) == INVALID and plan(FAKE + 4, FAKE) == INVALID
    assert plan(None, FAKE) == DEVICE and plan(FAKE, None) == DEVICE
    assert lib.festina_plan_drafts(None, FAKE, FAKE, None) == INVALID
    for i in range(4):
        out = F.festina_accepted(*(None if j == i else FAKE for j in range(4)))
        assert lib.festina_accept_drafts(C.byref(d), FAKE, FAKE, C.byref(out), None) == INVALID
    out = F.festina_accepted(FAKE, FAKE, FAKE, FAKE)
    assert lib.festina_accept_drafts(C.byref(d), None, FAKE, C.byref(out), None) == INVALID
    assert lib.festina_accept_drafts(C.byref(d), FAKE, None, C.byref(out), None) == INVALID
    assert lib.festina_accept_drafts(C.byref(d), FAKE, FAKE, None, None) == INVALID


def _cache(**k):
    a = dict(n_blocks=8, block_tokens=32, n_kv_heads=2, head_dim=64, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE)
    return F.festina_kv_cache(**{**a, **k})


@no_gpu
def test_keep(lib):  # noqa: F811
    base = dict(n_requests=4, max_blocks=5, n_tokens=40, block_table=FAKE, length=FAKE, first=FAKE, path=FAKE, kept=FAKE)

    def call(caches=None, **k):
        caches = [_cache(), _cache()] if caches is None else caches
        q = F.festina_kept(**{**base, **k})
        return lib.festina_keep_tokens((F.festina_kv_cache * max(len(caches), 1))(*caches), len(caches), C.byref(q), None)

    assert call() == DEVICE and call([_cache()] * 65) == DEVICE
    assert call([]) == OK and call(n_requests=0) == OK and call(n_tokens=0) == OK
    for name in ("block_table", "length", "first", "path", "kept"):
        assert call(**{name: None}) == INVALID, name
    for name, value in (("n_requests", -1), ("max_blocks", 0), ("n_tokens", -1)):
        assert call(**{name: value}) == INVALID, name
    assert call(n_requests=(1 << 20) + 1) == UNSUPPORTED and call(max_blocks=1 << 27) == UNSUPPORTED
    for change in (dict(n_blocks=9), dict(block_tokens=64), dict(n_kv_heads=1), dict(head_dim=128), dict(k=None), dict(v=FAKE + 8)):
        assert call([_cache(), _cache(**change)]) == INVALID, change
    assert call([_cache(head_dim=80)]) == UNSUPPORTED and call([_cache(block_tokens=8)]) == UNSUPPORTED
    q = F.festina_kept(**base)
    assert lib.festina_keep_tokens(None, 1, C.byref(q), None) == INVALID
    assert lib.festina_keep_tokens(None, -1, C.byref(q), None) == INVALID
    assert lib.festina_keep_tokens(C.byref(_cache()), 1, None, None) == INVALID


@no_gpu
def test_trim(lib):  # noqa: F811
    ws = F.festina_blocks_workspace_bytes(100, 0)

    def call(keep=FAKE, bytes_=ws, **k):
        a = dict(n_requests=100, max_blocks=8, block_tokens=16, n_blocks=64, held=FAKE, add=None, block_table=FAKE,
                 free_ids=FAKE, n_free=FAKE)
        q = F.festina_kv_requests(**{**a, **k})
        out = F.festina_kv_step(max_tokens=0, first=None, slot=None, length=FAKE, served=None, n_free_out=FAKE)
        return lib.festina_trim_blocks(C.byref(q), keep, C.byref(out), FAKE, bytes_, None)

    assert call() == DEVICE
    assert call(keep=None) == INVALID and call(held=None) == INVALID and call(bytes_=ws - 1) == INVALID
    assert call(block_tokens=24) == UNSUPPORTED and call(n_requests=0, keep=None) == DEVICE


@no_gpu
def test_attention_over_drafts(lib):  # noqa: F811
    c = _cache(n_blocks=64)

    def att(**k):
        a = dict(n_requests=4, max_blocks=8, n_tokens=40, n_heads=8, max_new=16, dtype=F.FESTINA_BF16, window=0, scale=0.1,
                 block_table=FAKE, length=FAKE, first=FAKE, q=FAKE, q_token_stride=512, q_head_stride=64, out=FAKE,
                 out_token_stride=512, out_head_stride=64, lse=FAKE)
        return F.festina_attention(**{**a, **k})

    def call(seen=FAKE, less=0, **k):
        a = att(**k)
        n = F.festina_attend_drafts_workspace_bytes(c, a)
        return lib.festina_attend_drafts(C.byref(c), C.byref(a), seen, FAKE, max(n - less, 0), None)

    assert call() == DEVICE
    assert call(seen=None) == INVALID and call(seen=FAKE + 4) == INVALID and call(less=1) == INVALID
    assert call(n_heads=7) == INVALID and call(window=-1) == INVALID and call(q=None) == INVALID and call(max_new=0) == INVALID
    assert call(dtype=F.FESTINA_F32) == UNSUPPORTED and call(q_head_stride=60) == INVALID
    assert call(n_tokens=0, seen=None) == OK and call(n_requests=0) == OK


@no_gpu
def test_rotation(lib):  # noqa: F811
    def call(rot=None, **k):
        r = F.festina_rotary(**{**dict(head_dim=128, rotated=128, interleaved=0, eps=1e-6, turn=FAKE, q_weight=FAKE,
                                       k_weight=FAKE), **(rot or {})})
        a = dict(n_tokens=5, n_heads=8, n_kv_heads=2, dtype=F.FESTINA_BF16, position=FAKE, q=FAKE, k=FAKE,
                 q_token_stride=1024, q_head_stride=128, k_token_stride=256, k_head_stride=128, q_out=FAKE, k_out=FAKE,
                 q_out_token_stride=1024, q_out_head_stride=128, k_out_token_stride=256, k_out_head_stride=128)
        h = F.festina_heads(**{**a, **k})
        return lib.festina_rotate_heads(C.byref(r), C.byref(h), None)

    assert call() == DEVICE and call(dict(q_weight=None, k_weight=None)) == DEVICE
    assert call(dict(rotated=0, turn=None)) == DEVICE and call(q=FAKE + 2) == DEVICE        # narrower loads
    for rot in (dict(head_dim=0), dict(rotated=-16), dict(rotated=144), dict(eps=-1.0), dict(eps=math.nan), dict(turn=None),
                dict(turn=FAKE + 4)):
        assert call(rot) == INVALID, rot
    assert call(dict(head_dim=80, rotated=64)) == UNSUPPORTED and call(dict(rotated=40)) == UNSUPPORTED
    for k in (dict(n_tokens=-1), dict(n_heads=-1), dict(dtype=7), dict(position=None), dict(q=None), dict(k_out=None),
              dict(q_token_stride=-8), dict(k_out_head_stride=-1), dict(q=FAKE + 1)):
        assert call(**k) == INVALID, k
    assert call(n_heads=70000) == UNSUPPORTED and call(n_tokens=2 ** 31 - 1) == UNSUPPORTED
    assert call(n_tokens=0, position=None) == OK and call(n_heads=0, n_kv_heads=0) == OK
    assert call(n_heads=0, q=None, q_out=None) == DEVICE
    assert lib.festina_rotate_heads(None, None, None) == INVALID


def test_turns_are_exact():
    assert F._turn(2 * math.pi) in (0, 2 ** 64 - 1, 2 ** 64 - 2 ** 10) or abs(F._turn(2 * math.pi) - 2 ** 64) < 2 ** 13
    assert abs(F._turn(1.0) - 2 ** 64 / (2 * math.pi)) < 2 ** 12 and F._turn(0.0) == 0
    assert F._turn(-1.0) == 2 ** 64 - F._turn(1.0)
    for bad in (math.nan, math.inf):
        with pytest.raises(ValueError):
            F._turn(bad)


def test_the_reference_against_small_examples():
    first, length = [0, 4, 4, 5], [14, 7, 3]
    parent, token, choice = [-1, 0, 0, 2, -1], [9, 5, 6, 7, 9], [6, 1, 7, 3, 2]
    seen, position = D.plan(first, length, parent)
    assert seen == [1, 3, 5, 13, 1] and position == [10, 11, 11, 12, 2]
    path, kept, after, left = D.accept(first, length, parent, token, choice)
    assert path == [0, 2, 3, -1, 0] and kept == [3, 0, 1] and after == [3, -1, 2] and left == [13, 7, 3]
    free, n, count = D.trim([14, 7, 3], left, np.array([[3, 4], [5, 6], [7, 8]]), [9] * 10, 2, 8)
    assert list(n) == [13, 7, 3] and count == 2
    free, n, count = D.trim([14, 7, 3], [8, 0, 4], np.array([[3, 4], [5, 6], [7, 8]]), [9] * 10, 2, 8)
    assert list(n) == [8, 0, 3] and count == 4 and list(free[:4]) == [9, 9, 4, 5]


def test_the_reference_rotation_keeps_lengths_and_differences():
    rng = np.random.default_rng(3)
    x, freq = rng.normal(size=(6, 2, 32)), 1e4 ** (-np.arange(8) / 8)
    for inter in (False, True):
        y, _ = D.rotate(x, np.arange(6), freq, None, 0.0, inter)
        assert np.allclose((y * y).sum(-1), (x * x).sum(-1)) and np.array_equal(y[..., 16:], x[..., 16:])
        a, b = (D.rotate(np.stack([x[0], x[1]]), [p, p + 5], freq, None, 0.0, inter)[0] for p in (0, 2 ** 30))
        assert np.allclose((a[0] * a[1]).sum(-1), (b[0] * b[1]).sum(-1), atol=1e-6)      # by the distance alone
