"""Which outputs the rotation takes: whether two tensors [tokens][heads][dim] share memory, and whether one's elements do, against
sets of addresses (no GPU)."""
import random

import pytest

torch = pytest.importorskip("torch")
from paper_2606_30391_amd import festina as F  # noqa: E402


def _places(t):
    s, p, _ = t.stride()
    return [t.storage_offset() + i * s + h * p + d for i in range(t.shape[0]) for h in range(t.shape[1]) for d in range(t.shape[2])]


def _view(rng, memory, dim):
    shape = (rng.choice([1, 2, 3, 5, 0, 7]), rng.choice([1, 2, 3, 4, 0]), dim)
    stride = (rng.choice([0, 1, dim, 2 * dim, 3 * dim, 4 * dim, 4 * dim + 1, 9 * dim, 40]),
              rng.choice([0, dim, 2 * dim, 3 * dim, dim + 3, 7 * dim, dim - 1]), 1)
    return memory.as_strided(shape, stride, rng.choice([0, 1, dim, dim - 1, 3 * dim, 5 * dim, 60, 100]))


@pytest.mark.parametrize("seed", range(4))
def test_shared_memory_is_found(seed):
    rng, memory, found = random.Random(seed), torch.zeros(4000, dtype=torch.float16), [0, 0, 0, 0]
    for _ in range(1500):
        x, y = (_view(rng, memory, 8) for _ in range(2))
        want = bool(set(_places(x)) & set(_places(y)))
        at = F._place(x, 8), F._place(y, 8)
        assert F._meet(*at, 8) == want == F._meet(*at[::-1], 8), (x.shape, x.stride(), x.storage_offset(), y.shape, y.stride(), y.storage_offset())
        own = len(set(_places(x))) == len(_places(x))
        assert F._once(at[0], 8) == own, (x.shape, x.stride())
        found[want] += 1
        found[2 + own] += 1
    assert min(found) > 100


def test_large_views_need_no_list_of_their_rows(monkeypatch):
    """The layouts that programs have are told apart by their strides alone."""
    monkeypatch.setattr(F.np, "arange", lambda *a: pytest.fail("a list of rows"))
    at = lambda T, H, stride, a: (a, a + (T - 1) * stride[0] + (H - 1) * stride[1] + 128, T, H, *stride)
    q, k = at(40000, 32, (48 * 128, 128), 0), at(40000, 8, (48 * 128, 128), 32 * 128)          # a packed projection
    assert not F._meet(q, k, 128) and F._once(q, 128) and F._once(k, 128)
    x, y = at(40000, 16, (16 * 256, 256), 0), at(40000, 16, (16 * 256, 256), 128)              # pairs of heads
    assert not F._meet(x, y, 128) and F._once(y, 128)
    x, y = at(40000, 32, (128, 40000 * 128), 0), at(40000, 16, (128, 40000 * 128), 32 * 40000 * 128)       # heads before tokens
    assert not F._meet(x, y, 128) and F._once(x, 128)
    assert not F._meet(q, at(40000, 8, (1024, 128), 40000 * 48 * 128), 128)
