"""GPU test of steps of drafted tokens run together (paper_2606_30391_amd.serve.Server.verify): prompts, then trees whose
tokens are partly accepted, each step's books, codes, positions and attention against the definitions in 64 bits."""
import numpy as np
import pytest

import drafts_reference as D
import kv_reference as K

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

BT, H, G, DIM, LAYERS, BLOCKS, CONTEXT, TOKENS = 16, 2, 3, 64, 2, 40, 192, 200


@pytest.mark.parametrize("window", [0, 50])
def test_prompts_then_trees(window):
    from paper_2606_30391_amd import festina
    from paper_2606_30391_amd.serve import Server
    rng = np.random.default_rng(window)
    gen = torch.Generator("cuda").manual_seed(5)
    srv = Server(4, CONTEXT, BLOCKS, TOKENS, LAYERS, H, DIM, BT)
    freq = 1e3 ** (-np.arange(24) / 24)
    weight = torch.from_numpy(1 + 0.1 * rng.normal(size=(2, DIM)))
    rotary = festina.DeviceRotary(freq, DIM, *weight)
    held, table, free, n_free = np.zeros(4, np.int64), np.zeros((4, CONTEXT // BT), np.int32), np.arange(BLOCKS - 1, -1, -1), BLOCKS
    layers = [(np.zeros((BLOCKS, H, BT, DIM), np.uint8), np.zeros((BLOCKS, H, DIM, BT), np.uint8),
               np.zeros((BLOCKS, H), np.float32), np.zeros((BLOCKS, H), np.float32)) for _ in range(LAYERS)]
    for n, add in enumerate([[33, 1, 16, 100], [8, 20, 1, 40], [31, 64, 0, 5], [12, 70, 30, 0], [3, 3, 3, 3], [60, 50, 40, 30],
                            [64, 64, 64, 8], [20, 20, 20, 90]]):
        T = sum(add)
        parent = np.concatenate([D.tree(rng, a, 3) if a <= 64 else np.arange(a) - 1 for a in add]).astype(np.int64)
        token, choice = rng.integers(0, 2, (2, T))
        data = [[torch.randn((T, h, DIM), generator=gen, device="cuda").bfloat16() for h in (H * G, H, H)]
                for _ in range(LAYERS)]
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        print(f"[gpu] window {window}, step {n}: {add}", flush=True)
        drafted = n > 0
        if drafted:
            got = srv.verify(add, i32(parent), i32(token), lambda layer: data[layer], lambda out: i32(choice), window, rotary)
        else:
            got = srv.step(add, lambda layer: data[layer], window, rotary)
        table, slot, first, length, served, n_free = K.extend(held, add, table, free, n_free, BT, TOKENS)
        filled = int(first[-1])
        seen, position = D.plan(first, length, parent if drafted else np.arange(T) * 0 + 10 ** 6)
        if not drafted:                                      # (runs, short ones among them)
            seen = [0] * T
            for r in range(4):
                for i in range(add[r]):
                    position[first[r] + i] = i
                    seen[first[r] + i] = 2 ** (i + 1) - 1
        position = np.array([0 if p is None else p for p in position])
        for i in range(LAYERS):
            x = [y.double().cpu().numpy() for y in data[i]]
            q, _ = rotary.apply(data[i][0], data[i][1], i32(position))
            _, k = rotary.apply(data[i][0], data[i][1], i32(position))
            for a, b, w in ((x[0], q, weight[0]), (x[1], k, weight[1])):             # the rotation itself
                want, bound = D.rotate(a, position, freq, w.numpy())
                assert (np.abs(b.double().cpu().numpy() - want) <= bound * 1.01 + 2.0 ** -8 * np.abs(want)).all()
            layers[i] = K.store(*layers[i], k.double().cpu().numpy(), x[2], slot[:T], BT)
            o, lse, mag = D.attend(q.double().cpu().numpy(), *layers[i], table, length, first,
                                   [0 if s is None else s for s in seen], DIM ** -0.5, window)
            tol = K.attend_bounds(o, lse, mag, DIM, 2.0 ** -8)[0]
            assert (np.abs(got[i].double().cpu().numpy() - o) <= tol)[:filled].all()
        if drafted:
            path, kept, after, left = D.accept(first, length, parent, token, choice)
            assert srv.drafts.kept.cpu().tolist() == kept and srv.drafts.next.cpu().tolist() == after
            path = np.array([-1 if p is None else p for p in path])
            layers = [D.keep(*x, table, length, first, path, kept) for x in layers]
            free, length, n_free = D.trim(length, left, table, free, n_free, BT)
        held = length
        assert srv.blocks.held.cpu().tolist() == list(held) and int(srv.blocks.n_free.item()) == n_free
        for i, cache in enumerate(srv.caches):
            for r in range(4):
                for c in range(-(-int(held[r]) // BT)):
                    b, m = int(table[r, c]), min(BT, int(held[r]) - c * BT)
                    assert int(srv.blocks.table[r, c].item()) == b
                    assert K.same_codes(cache.k[b, :, :m].cpu().numpy(), layers[i][0][b, :, :m])
                    assert K.same_codes(cache.v[b, :, :, :m].cpu().numpy(), layers[i][1][b, :, :, :m])
                    assert np.array_equal(cache.k_scale[b].cpu().numpy(), layers[i][2][b])
                    assert np.array_equal(cache.v_scale[b].cpu().numpy(), layers[i][3][b])
    assert served.tolist() == [1, 1, 1, 0]                   # the last one's chunk does not fit its row of the table


@pytest.mark.parametrize("draft", ["1", "7", "64"])
def test_the_command_verifies_drafts(capsys, draft):
    from paper_2606_30391_amd import serve
    serve.main(["--gpus", "8", "--requests", "64", "--most", "6", "--steps", "20", "--layers", "2", "--heads", "4",
                "--kv-heads", "2", "--dim", "64", "--block", "32", "--draft", draft])
    said = capsys.readouterr().out
    print(said, flush=True)
    assert "drafts:" in said and "decode:" in said
    free = said.split("us a layer; ")[1].split(" blocks free")[0].split(" of ")
    assert free[0] == free[1]                                # every block came back


def test_trees_and_choices_of_other_sizes_than_the_step_are_refused():
    from paper_2606_30391_amd.serve import Server
    srv = Server(2, CONTEXT, BLOCKS, TOKENS, 1, H, DIM, BT)
    data = [torch.randn((5, h, DIM), device="cuda").bfloat16() for h in (H * G, H, H)]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    parent, token, choice = i32(-1, 0, 0, -1, 0), i32(7, 8, 9, 7, 8), i32(9, 0, 5, 1, 1)
    step = lambda p, t, c: srv.verify([3, 2], p, t, lambda layer: data, lambda out: c)
    for change in ((i32(-1), token, choice), (parent, i32(7), choice), (parent, token, i32(9)), (parent[:4], token, choice),
                   (parent, token[None], choice), (parent, token, choice.cpu()), (parent.long(), token, choice)):
        with pytest.raises(ValueError):
            step(*change)
        assert srv.blocks.held.tolist() == [0, 0] and srv.blocks.n_free.tolist() == [BLOCKS]
    step(parent, token, choice)                              # none of them left anything behind
    assert srv.drafts.kept.tolist() == [2, 1] and srv.drafts.next.tolist() == [5, 1]
    assert srv.blocks.held.tolist() == [2, 1] and srv.blocks.n_free.tolist() == [BLOCKS - 2]


def test_counts_as_a_tensor_on_the_host():
    from paper_2606_30391_amd.serve import Server
    srv = Server(2, CONTEXT, BLOCKS, TOKENS, 1, H, DIM, BT)
    data = [torch.randn((5, h, DIM), device="cuda").bfloat16() for h in (H * G, H, H)]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    add = torch.tensor([3, 2])
    srv.step(add, lambda layer: data)
    assert srv.blocks.held.tolist() == [3, 2]
    srv.verify(add, i32(-1, 0, 0, -1, 0), i32(7, 8, 9, 7, 8), lambda layer: data, lambda out: i32(9, 0, 5, 1, 1))
    assert srv.blocks.held.tolist() == [5, 3] and srv.drafts.kept.tolist() == [2, 1]
