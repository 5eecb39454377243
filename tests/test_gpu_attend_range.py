"""GPU tests of attention where the rows' weights span more than half precision does: blocks whose value scales lie far
apart, and one key of far more weight than all others.  The bound takes each step of 64 keys for itself."""
import numpy as np
import pytest

import kv_reference as K
from test_gpu_attend import TYPES, Case

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

STEP = 64


def _tolerance(c, out, magnitude):
    """As kv_reference.attend_bounds, but a weight's rounding is 2^-11 of it or 2^-19 of the largest weight (times its value
    scale) among its step's keys: the kernels keep the largest of a step above 2^-6, where the format's error is 2^-25."""
    mag, _, logit, keys = magnitude
    dx = (c.D + 4) * 2.0 ** -24 * logit
    rel = 2.0 ** -11 + 2 * dx + 2.0 ** -20 + keys * 2.0 ** -24
    tol = TYPES[c.dtype][1] * np.abs(out) + 1.01 * mag * rel[..., None] + 1e-30
    scale = float(np.float32(c.D ** -0.5))
    for r in range(len(c.length)):
        L, n, bt = int(c.length[r]), int(c.new[r]), c.bt
        ids = c.table[r][:-(-L // bt)]
        for h in range(c.H):
            k = (K.decode(c.k[ids, h]) * c.ks[ids, h].astype(np.float64)[:, None, None]).reshape(-1, c.D)[:L]
            v = np.abs(np.swapaxes(K.decode(c.v[ids, h]), 1, 2)).reshape(-1, c.D)[:L]
            sc = np.repeat(c.vs[ids, h].astype(np.float64), bt)[:L]
            for i in range(n):
                p, t = L - n + i, int(c.first[r]) + i
                for y in range(h * c.G, (h + 1) * c.G):
                    x = scale * (k[:p + 1] @ c.q[t, y].double().cpu().numpy())
                    w = np.exp(x - x.max())
                    w = w / w.sum() * sc[:p + 1]
                    for s in range(0, p + 1, STEP):
                        tol[t, y] += 2.0 ** -19 * w[s:s + STEP].max() * v[s:min(s + STEP, p + 1)].sum(0)
    return tol


def _check(c, label):
    print(f"[gpu] attend {label} D={c.D} bt={c.bt} {c.dtype} {list(zip(c.length.tolist(), c.new.tolist()))}", flush=True)
    out, lse = c.cache().attend(c.q, *c.tensors(), max_new=max(1, int(c.new.max())))
    torch.cuda.synchronize()
    o, l, magnitude = c.want()
    tol = _tolerance(c, o, magnitude)
    far = np.abs(out.double().cpu().numpy() - o)
    assert (far <= tol).all(), f"{(far / tol).max():.3g} of the bound"
    assert np.all(np.abs(lse.double().cpu().numpy() - l) <= K.attend_bounds(o, l, magnitude, c.D, 0.0)[1])


@pytest.mark.parametrize("requests", [[(640, 1)], [(500, 3)], [(640, 40)], [(2500, 1), (900, 1)], [(3000, 2)], [(2500, 33)]])
@pytest.mark.parametrize("D,G,bt,dtype", [(64, 2, 64, "bf16"), (96, 1, 128, "f16"), (128, 4, 64, "f16"), (256, 1, 64, "bf16")])
@pytest.mark.parametrize("blocks", [(2,), (0, 5)])
def test_one_large_element_leaves_the_others_exact(requests, D, G, bt, dtype, blocks):
    """A block that holds values 2^18 or 2^22 times the others in one element, and small ones elsewhere (which its scale rounds
    to zero): the sums of the other elements are those of the other blocks."""
    rng = np.random.default_rng(D + blocks[0] + requests[0][0])
    c = Case(rng, requests, D=D, H=1, G=G, bt=bt, dtype=dtype)
    c.vs = np.where(np.isnan(c.vs), c.vs, np.float32(2.0 ** -12 if dtype == "f16" else 2.0 ** -10))
    for r in range(len(requests)):
        for b in blocks:
            if b < c.length[r] // bt:
                i = c.table[r, b]
                c.vs[i] *= 2.0 ** (18 if dtype == "f16" else 22)
                c.v[i, :, 1:] = 0
    _check(c, "one large element")


@pytest.mark.parametrize("requests", [[(65536, 1)], [(40000, 3)], [(20000, 33)]])
@pytest.mark.parametrize("sink", [0, 10000])
@pytest.mark.parametrize("logit", [17.0, 19.0])
def test_many_keys_of_little_weight_beside_one_of_much(requests, sink, logit):
    """One key whose value is zero takes nearly all the weight; what the others add is the result."""
    rng = np.random.default_rng(sink + requests[0][1])
    c = Case(rng, requests, D=64, H=1, G=1, bt=64)
    c.k[:], c.ks[:] = 0, 1.0
    c.q = torch.zeros_like(c.q)
    c.q[:, :, 0] = 8.0
    b, o = c.table[0, sink // 64], sink % 64
    c.k[b, 0, o, 0] = K.encode(16.0)
    c.ks[b] = logit / 16.0                                   # times 8 and 64^-1/2
    c.v = np.where(c.v >= 0x80, c.v - 0x80, c.v)             # values that do not cancel
    c.v[b, 0, :, o] = 0
    c.vs[:] = 2.0 ** -7
    _check(c, f"a key of logit {logit} at {sink}")
