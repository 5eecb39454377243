"""GPU test: inputs with a forward-mode tangent are refused where a gradient would be, instead of losing it without a word."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def _calls():
    from paper_2606_30391_amd import festina
    r = festina.DeviceRotary(1e3 ** (-np.arange(32) / 32), 64)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    p = i32([0, 1, 2])
    cache = festina.DeviceCache.empty(4, 16, 2, 64)
    q, k = (torch.randn((3, h, 64), device="cuda").bfloat16() for h in (4, 2))
    cache.store(k, k, p)
    seen = torch.tensor([1, 3, 5], device="cuda")
    table, length, first = i32([[0]]), i32([3]), i32([0, 3])
    return q, k, {"rotate": lambda q, k: r.apply(q, k, p)[0],
                  "rotate in place": lambda q, k: r.apply(q, k, p, q, k)[0],
                  "rotate into": lambda q, k: r.apply(q.detach().clone(), k.detach().clone(), p, q, k)[0],
                  "drafts": lambda q, k: cache.attend(q, table, length, first, 3, seen=seen)[0],
                  "attend": lambda q, k: cache.attend(q, table, length, first, 3)[0]}


@pytest.mark.parametrize("name", ["rotate", "rotate in place", "rotate into", "drafts", "attend"])
def test_tangents_are_refused(name):
    from torch.autograd import forward_ad
    q, k, calls = _calls()
    call = calls[name]
    want = call(q.clone(), k.clone())
    with forward_ad.dual_level():
        assert torch.equal(call(q.clone(), k.clone()), want)                         # (nothing has a tangent)
        dual = lambda x: forward_ad.make_dual(x.clone(), torch.ones_like(x))
        print(f"[gpu] {name}", flush=True)
        with pytest.raises(ValueError):
            call(dual(q), k.clone())
        if name.startswith("rotate"):
            with pytest.raises(ValueError):
                call(q.clone(), dual(k))
        with torch.no_grad(), pytest.raises(ValueError):                             # (which leaves tangents as they are)
            call(dual(q), k.clone())
        if name != "rotate into":
            assert torch.equal(call(forward_ad.unpack_dual(dual(q)).primal, k.clone()), want)
    assert torch.equal(call(q.clone(), k.clone()), want)
