"""Pins of the 64-bit reference of the serving step's operators, and what can be checked of the operators without a
GPU: the header's refusals and the binding's argument checks."""
import ctypes as C
import os

import numpy as np
import pytest

import kv_reference as K
from paper_2606_30391_amd import festina as F

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(F.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return F.lib()


def _no_gpu_visible():
    return torch.cuda.device_count() == 0


no_gpu = pytest.mark.skipif(not _no_gpu_visible(), reason="fake-pointer error paths run only without a GPU")


# ------------------------------------------------------------------ the reference itself

def test_e4m3_values_and_rounding_agree_with_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(K.decode(codes), want, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 20001), np.random.default_rng(1).normal(0, 1, 5000) * 2.0 ** -7,
                        [0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 464.0, -1e9]])
    got = K.decode(K.encode(x))
    want = torch.from_numpy(np.clip(x, -448, 448)).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(got, want)
    assert np.all(np.isnan(K.decode(K.encode([np.nan, np.inf, -np.inf]))))


def test_extend_worked_example():
    # blocks of 16; request 0 holds 15 tokens in block 9 and adds 2, request 1 starts with 17, request 2 waits
    table = np.full((3, 2), -1, np.int32)
    table[0, 0] = 9
    t, slot, first, length, served, n = K.extend([15, 0, 0], [2, 17, 1], table, np.arange(12), 3, 16, 32)
    assert t.tolist() == [[9, 2], [1, 0], [-1, -1]]
    assert slot[:2].tolist() == [9 * 16 + 15, 2 * 16]
    assert slot[2:19].tolist() == list(range(16, 32)) + [0] and slot[19:].tolist() == [-1] * 13
    assert first.tolist() == [0, 2, 19, 19] and length.tolist() == [17, 17, 0]
    assert served.tolist() == [1, 1, 0] and n == 0
    ids, length, n = K.release([17, 17, 0], [1, 0, 1], t, [7] * 12, n, 16)
    assert ids[:2].tolist() == [9, 2] and n == 2 and length.tolist() == [0, 17, 0]


def test_scales():
    assert K.scale_of(448.0) == 1.0 and K.scale_of(448.1) == 2.0 and K.scale_of(0.0) == 2.0 ** -32
    assert K.scale_of(1e30) == 2.0 ** 32


def test_attention_worked_example():
    # one block, two keys with logits 0 and ln 3: weights 1/4 and 3/4
    kc = np.zeros((1, 1, 16, 64), np.uint8)
    vc = np.zeros((1, 1, 64, 16), np.uint8)
    kc[0, 0, 1, 0] = K.encode(1.0)
    vc[0, 0, :, 0], vc[0, 0, :, 1] = K.encode(4.0), K.encode(8.0)
    q = np.zeros((1, 1, 64))
    q[0, 0, 0] = np.log(3.0)
    one = np.ones((1, 1))
    o, lse, _ = K.attend(q, kc, vc, one, one, [[0]], [2], [0, 1], 1.0)
    assert np.allclose(o, 7.0, atol=1e-12) and np.allclose(lse, np.log(4.0))
    o, lse, _ = K.attend(q, kc, vc, one, one, [[0]], [2], [0, 1], 1.0, window=1)
    assert np.allclose(o, 8.0) and np.allclose(lse, np.log(3.0))


# ------------------------------------------------------------------ refusals

FAKE = C.c_void_p(0x1000)        # never dereferenced: the calls below fail validation first
WS = C.c_void_p(0x100000)


def _blocks(R=8, MB=4, BT=16, NB=32, tokens=64):
    return (F.festina_kv_requests(R, MB, BT, NB, *([FAKE] * 5)),
            F.festina_kv_step(tokens, *([FAKE] * 5)))


def _extend(q, o, ws=WS, n=1 << 30):
    return F.lib().festina_extend_blocks(C.byref(q), C.byref(o), ws, n, None)


def _release(q, o, done=FAKE, ws=WS, n=1 << 30):
    return F.lib().festina_release_blocks(C.byref(q), done, C.byref(o), ws, n, None)


@no_gpu
def test_blocks_reject_bad_arguments_before_launch(lib):
    need = F.festina_blocks_workspace_bytes(8, 64)
    assert need > 0 and need % 256 == 0
    assert F.festina_blocks_workspace_bytes(-1, 64) == F.festina_blocks_workspace_bytes(8, -1) == 0
    assert F.festina_blocks_workspace_bytes(4096, 1 << 20) <= F.festina_blocks_workspace_bytes(8192, 1 << 21)
    q, o = _blocks()
    for call in (_extend, _release):
        assert call(q, o, ws=None) == F.FESTINA_ERR_INVALID
        assert call(q, o, ws=C.c_void_p(0x100008)) == F.FESTINA_ERR_INVALID
        assert call(q, o, n=F.festina_blocks_workspace_bytes(8, 0) - 1) == F.FESTINA_ERR_INVALID
        assert call(q, o) == F.FESTINA_ERR_DEVICE                            # accepted, and nothing to launch on
        for kw, want in [(dict(R=-1), 1), (dict(MB=0), 1), (dict(BT=0), 1), (dict(NB=0), 1), (dict(BT=24), 3),
                         (dict(BT=8), 3), (dict(BT=512), 3), (dict(NB=1 << 27), 3), (dict(MB=1 << 27), 3),
                         (dict(R=(1 << 20) + 1), 3)]:
            assert call(*_blocks(**kw)) == want, kw
        for i, field in [(0, "held"), (0, "block_table"), (0, "free_ids"), (0, "n_free"), (1, "length"), (1, "n_free_out")]:
            s = _blocks()
            setattr(s[i], field, None)
            assert call(*s) == F.FESTINA_ERR_INVALID, field
    for i, field in [(0, "add"), (1, "first"), (1, "slot"), (1, "served")]:
        s = _blocks()
        setattr(s[i], field, None)
        assert _extend(*s) == F.FESTINA_ERR_INVALID, field
    assert _extend(*_blocks(tokens=-1)) == F.FESTINA_ERR_INVALID
    assert _extend(*_blocks(tokens=2 ** 31 - 4096), n=1 << 40) == F.FESTINA_ERR_UNSUPPORTED
    assert _extend(*_blocks(tokens=2 ** 31 - 4097), n=1 << 40) == F.FESTINA_ERR_DEVICE
    assert F.festina_blocks_workspace_bytes(8, 2 ** 31 - 4096) == 0 < F.festina_blocks_workspace_bytes(8, 2 ** 31 - 4097)
    assert _release(q, o, done=None) == F.FESTINA_ERR_INVALID
    assert F.lib().festina_extend_blocks(None, C.byref(o), WS, need, None) == F.FESTINA_ERR_INVALID
    assert F.lib().festina_release_blocks(C.byref(q), FAKE, None, WS, need, None) == F.FESTINA_ERR_INVALID


def _cache(NB=32, BT=16, H=2, D=64):
    return F.festina_kv_cache(NB, BT, H, D, *([FAKE] * 4))


BAD_CACHES = [(dict(NB=0), 1), (dict(BT=0), 1), (dict(H=0), 1), (dict(D=0), 1), (dict(BT=8), 3), (dict(BT=48), 3),
              (dict(BT=512), 3), (dict(D=80), 3), (dict(D=512), 3), (dict(NB=1 << 27), 3), (dict(H=1025), 3)]


@no_gpu
def test_store_rejects_bad_arguments_before_launch(lib):
    def tokens(T=8, dtype=F.FESTINA_BF16):
        return F.festina_kv_tokens(T, dtype, FAKE, FAKE, 128, 64, 128, 64, FAKE)

    call = lambda c, t: F.lib().festina_store_kv(C.byref(c), C.byref(t), None)
    assert call(_cache(), tokens()) == F.FESTINA_ERR_DEVICE
    for kw, want in BAD_CACHES:
        assert call(_cache(**kw), tokens()) == want, kw
    for field in ("k", "v", "k_scale", "v_scale"):
        c = _cache()
        setattr(c, field, None)
        assert call(c, tokens()) == F.FESTINA_ERR_INVALID, field
    c = _cache()
    c.v = C.c_void_p(0x1008)                                                 # not 16-byte aligned
    assert call(c, tokens()) == F.FESTINA_ERR_INVALID
    for field, value in [("n_tokens", -1), ("dtype", 3), ("dtype", -1), ("k", None), ("v", None), ("slot", None),
                         ("k_token_stride", -1), ("v_head_stride", -64), ("k", C.c_void_p(0x1001))]:
        t = tokens()
        setattr(t, field, value)
        assert call(_cache(), t) == F.FESTINA_ERR_INVALID, field
    assert call(_cache(H=1024), tokens(T=2 ** 31 - 1)) == F.FESTINA_ERR_UNSUPPORTED    # more workgroups than a launch has
    t = tokens(T=0)
    t.k = t.v = t.slot = None
    assert call(_cache(), t) == F.FESTINA_OK                                 # no tokens: nothing launched
    assert F.lib().festina_store_kv(None, C.byref(tokens()), None) == F.FESTINA_ERR_INVALID
    assert F.lib().festina_store_kv(C.byref(_cache()), None, None) == F.FESTINA_ERR_INVALID


@no_gpu
def test_attend_rejects_bad_arguments_before_launch(lib):
    def att(R=4, MB=8, T=4, heads=4, new=1, dtype=F.FESTINA_BF16, window=0):
        return F.festina_attention(R, MB, T, heads, new, dtype, window, 0.125, FAKE, FAKE, FAKE, FAKE, heads * 64, 64,
                                   FAKE, heads * 64, 64, None)

    def call(c, t, ws=WS, n=1 << 40):
        return F.lib().festina_attend(C.byref(c), C.byref(t), ws, n, None)

    need = F.festina_attend_workspace_bytes(_cache(), att())
    assert need > 0 and need % 256 == 0
    assert call(_cache(), att(), n=need - 1) == F.FESTINA_ERR_INVALID
    assert call(_cache(), att(), ws=None) == F.FESTINA_ERR_INVALID
    assert call(_cache(), att(), ws=C.c_void_p(0x100010)) == F.FESTINA_ERR_INVALID
    assert call(_cache(), att()) == F.FESTINA_ERR_DEVICE
    for kw, want in BAD_CACHES:
        assert call(_cache(**kw), att()) == want, kw
        assert F.festina_attend_workspace_bytes(_cache(**kw), att()) == 0
    for kw, want in [(dict(R=-1), 1), (dict(MB=0), 1), (dict(T=-1), 1), (dict(heads=0), 1), (dict(heads=5), 1),
                     (dict(new=0), 1), (dict(window=-1), 1), (dict(dtype=F.FESTINA_F32), 3), (dict(dtype=7), 3),
                     (dict(R=(1 << 20) + 1), 3), (dict(MB=1 << 26), 3), (dict(T=1 << 29), 3)]:
        assert call(_cache(), att(**kw)) == want, kw
        assert F.festina_attend_workspace_bytes(_cache(), att(**kw)) == 0
    wide = _cache(H=32)                                                      # more workgroups than a launch has
    for new in (1, 64):
        assert call(wide, att(R=1 << 20, T=1 << 20, heads=32, new=new)) == F.FESTINA_ERR_UNSUPPORTED
        assert call(wide, att(R=1 << 18, T=1 << 18, heads=32, new=new)) == F.FESTINA_ERR_DEVICE
    for field, value in [("block_table", None), ("length", None), ("first", None), ("q", None), ("out", None),
                         ("q", C.c_void_p(0x1008)), ("out", C.c_void_p(0x1004)), ("q_token_stride", 12),
                         ("q_head_stride", -64), ("out_head_stride", 68), ("scale", float("nan"))]:
        t = att()
        setattr(t, field, value)
        assert call(_cache(), t) == F.FESTINA_ERR_INVALID, field
    for kw in (dict(R=0), dict(T=0)):                                        # nothing to do, nothing launched
        t = att(**kw)
        t.q = t.out = t.block_table = None
        assert call(_cache(), t, ws=None, n=0) == F.FESTINA_OK
    assert F.lib().festina_attend(None, C.byref(att()), WS, need, None) == F.FESTINA_ERR_INVALID
    assert F.lib().festina_attend(C.byref(_cache()), None, WS, need, None) == F.FESTINA_ERR_INVALID


def test_binding_refuses_tensors_of_host_memory_and_wrong_types(lib):
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device memory"):
        F.DeviceBlocks(i, i, torch.zeros((4, 2), dtype=torch.int32), i, i[:1], 16, 8)
    with pytest.raises(ValueError, match="device memory"):
        F.DeviceCache(torch.zeros((2, 1, 16, 64), dtype=torch.uint8), None, None, None)
    with pytest.raises(ValueError, match="two dimensions"):
        F.DeviceBlocks(i, i, i, i, i[:1], 16, 8)


def test_a_captured_call_has_scratch_of_its_own(monkeypatch):
    """What a graph captured must neither be replaced by a larger call nor shared with another graph."""
    import contextlib
    import torch.cuda
    capturing = [False]
    monkeypatch.setattr(F, "_on", lambda stream, device: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    w = F._Workspaces()
    eager = w.get(1000, 5, "cpu")
    assert w.get(900, 5, "cpu")[1] == eager[1] and eager[2] == 5
    capturing[0] = True
    graphs = [w.get(1000, 5, "cpu") for _ in range(2)]
    assert len({eager[1], graphs[0][1], graphs[1][1]}) == 3
    assert all(g[0].data_ptr() == g[1] and g[0].numel() >= 1000 for g in graphs)
    capturing[0] = False
    assert w.get(1000, 5, "cpu")[1] == eager[1]              # the stream's own is as it was
    assert w.get(2000, 5, "cpu")[1] not in (graphs[0][1], graphs[1][1])
