"""GPU test of known tokens beside draft trees (Server.verify): the rest of a prompt, of 1 to 64 tokens, stays in the cache whatever
the model would have chosen, as a step of its own would have left it."""
import numpy as np
import pytest

import drafts_reference as D
import kv_reference as K

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

BT, H, G, DIM, BLOCKS, CONTEXT, TOKENS = 16, 2, 2, 64, 60, 256, 260
i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _server(layers=2):
    from paper_2606_30391_amd.serve import Server
    return Server(4, CONTEXT, BLOCKS, TOKENS, layers, H, DIM, BT)


def _data(n, gen):
    return [torch.randn((n, h, DIM), generator=gen, device="cuda").bfloat16() for h in (H * G, H, H)]


@pytest.mark.parametrize("add,known", [
    ([8, 30, 1, 5], [1, 30, 1, 0]),                          # the last 30 tokens of a prompt, a single token
    ([64, 64, 2, 0], [64, 1, 2, 0]), ([20, 40, 70, 64], [5, 33, 70, 2]),             # trees behind known tokens, a run
    ([1, 1, 1, 1], [1, 1, 1, 1])])
def test_known_tokens_stay(add, known):
    rng, gen = np.random.default_rng(sum(add)), torch.Generator("cuda").manual_seed(3)
    srv = _server()
    prompts = [33, 1, 16, 40]
    data = _data(sum(prompts), gen)
    srv.step(prompts, lambda layer: data)
    parent = np.concatenate([D.tree(rng, n, 3) if n <= 64 else np.full(n, 7) for n in add]).astype(np.int64)
    token, choice = rng.integers(0, 3, len(parent)), rng.integers(0, 3, len(parent))
    given = [x.copy() for x in (parent, token, choice)]
    first = np.concatenate([[0], np.cumsum(add)])
    length = np.array(prompts) + add
    data = _data(len(parent), gen)
    print(f"[gpu] new {add} known {known}", flush=True)
    device = [i32(x) for x in given]
    srv.verify(add, device[0], device[1], lambda layer: data, lambda out: device[2], known=known)
    assert all(np.array_equal(x.cpu().numpy(), y) for x, y in zip(device, given))     # the caller's own are left as they are
    for r in range(4):
        for i in range(known[r] - 1 if add[r] <= 64 else 0):
            parent[first[r] + i + 1], choice[first[r] + i] = i, token[first[r] + i + 1]
    path, kept, after, left = D.accept(first, length, parent, token, choice)
    assert srv.drafts.kept.tolist() == kept and srv.drafts.next.tolist() == after and srv.blocks.held.tolist() == left
    assert all(k >= n for k, n in zip(kept, known))
    # the next step has the model's own choices again
    data = _data(4, gen)
    srv.verify([1] * 4, i32([-1] * 4), i32([1] * 4), lambda layer: data, lambda out: i32([2, 0, 1, 7]))
    assert srv.drafts.kept.tolist() == [1] * 4 and srv.drafts.next.tolist() == [2, 0, 1, 7]
    # and trees whose parents are as given
    data = _data(12, gen)
    srv.verify([3] * 4, i32([-1, 0, 0] * 4), i32([1, 2, 3] * 4), lambda layer: data, lambda out: i32([3, 0, 9] * 4))
    assert srv.drafts.kept.tolist() == [2] * 4 and srv.drafts.next.tolist() == [9] * 4


@pytest.mark.parametrize("rest", [1, 17, 64])
def test_the_rest_of_a_prompt_beside_trees_is_what_a_step_of_its_own_makes(rest):
    """The codes equal bit for bit (the same tokens at the same places), the outputs those of the definition in 64 bits."""
    from paper_2606_30391_amd import festina
    gen = torch.Generator("cuda").manual_seed(rest)
    rotary = festina.DeviceRotary(1e3 ** (-np.arange(16) / 16), DIM)
    both, alone = _server(1), _server(1)
    begin = _data(100 + 20, gen)
    for srv in (both, alone):
        srv.step([100, 20, 0, 0], lambda layer: begin, rotary=rotary)
    chunk, tree = _data(rest, gen), _data(8, gen)
    mixed = [torch.cat(x) for x in zip(chunk, tree)]
    n = rest + 8
    got = both.verify([rest, 8, 0, 0], i32([-1] * rest + [-1, 0, 0, 1, 1, 2, 2, 3]), i32(np.arange(n) % 5),
                      lambda layer: mixed, lambda out: i32([-3] * n), rotary=rotary, known=[rest, 1, 0, 0])[0]
    want = alone.step([rest, 0, 0, 0], lambda layer: chunk, rotary=rotary)[0]
    assert both.drafts.kept.tolist() == [rest, 1, 0, 0] and both.blocks.held.tolist() == [100 + rest, 21, 0, 0]
    assert alone.blocks.held.tolist() == [100 + rest, 20, 0, 0]
    q, _ = rotary.apply(chunk[0], chunk[1], i32(np.arange(100, 100 + rest)))
    for srv, out in ((both, got[:rest]), (alone, want)):
        cache = [x.cpu().numpy() for x in (srv.caches[0].k, srv.caches[0].v, srv.caches[0].k_scale, srv.caches[0].v_scale)]
        o, lse, mag = D.attend(q.double().cpu().numpy(), *cache, srv.blocks.table[:1].cpu().numpy(), [100 + rest], [0, rest],
                               [2 ** (i + 1) - 1 for i in range(rest)], DIM ** -0.5)
        assert (np.abs(out.double().cpu().numpy() - o) <= K.attend_bounds(o, lse, mag, DIM, 2.0 ** -8)[0]).all()
    for c in range(-(-(100 + rest) // BT)):
        a, b = int(both.blocks.table[0, c]), int(alone.blocks.table[0, c])
        m = min(BT, 100 + rest - c * BT)
        x, y = both.caches[0], alone.caches[0]
        assert torch.equal(x.k[a, :, :m], y.k[b, :, :m]) and torch.equal(x.v[a, :, :, :m], y.v[b, :, :, :m])
        assert torch.equal(x.k_scale[a], y.k_scale[b]) and torch.equal(x.v_scale[a], y.v_scale[b])


def test_refused_counts_leave_nothing_behind():
    srv = _server(1)
    data = _data(5, torch.Generator("cuda").manual_seed(1))
    step = lambda known: srv.verify([3, 2, 0, 0], i32([-1, 0, 0, -1, 0]), i32([7, 8, 9, 7, 8]), lambda layer: data,
                                    lambda out: i32([9, 0, 5, 1, 1]), known=known)
    for known in ([4, 0, 0, 0], [3, 2], [-1, 0, 0, 0], [0, 0, 1, 0]):
        with pytest.raises(ValueError):
            step(known)
        assert srv.blocks.held.tolist() == [0] * 4 and srv.blocks.n_free.tolist() == [BLOCKS]
    step(torch.tensor([0, 2, 0, 0]))
    assert srv.drafts.kept.tolist() == [2, 2, 0, 0] and srv.drafts.next.tolist() == [5, 1, -1, -1]
