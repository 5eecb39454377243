"""GPU test of the serving steps run together (paper_2606_30391_amd.serve): prompts, decode steps, a request that
leaves and one that takes its place, each step's books, codes and attention against the definitions in 64 bits."""
import numpy as np
import pytest

import kv_reference as K

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

BT, H, G, D, LAYERS, BLOCKS, CONTEXT, TOKENS = 16, 2, 3, 64, 2, 24, 128, 160


class Reference:
    """The same steps written out on the CPU."""

    def __init__(self, n):
        self.held, self.table = np.zeros(n, np.int64), np.zeros((n, CONTEXT // BT), np.int32)
        self.free, self.n_free = np.arange(BLOCKS - 1, -1, -1), BLOCKS
        self.layers = [(np.zeros((BLOCKS, H, BT, D), np.uint8), np.zeros((BLOCKS, H, D, BT), np.uint8),
                        np.zeros((BLOCKS, H)), np.zeros((BLOCKS, H))) for _ in range(LAYERS)]

    def step(self, add, qkv, window):
        self.table, slot, first, length, served, self.n_free = K.extend(self.held, add, self.table, self.free,
                                                                        self.n_free, BT, TOKENS)
        out = []
        for i in range(LAYERS):
            q, k, v = (x.double().cpu().numpy() for x in qkv(i))
            self.layers[i] = K.store(*self.layers[i], k, v, slot[:len(k)], BT)
            o, lse, mag = K.attend(q, *self.layers[i], self.table, length, first, D ** -0.5, window)
            out.append((o, K.attend_bounds(o, lse, mag, D, 2.0 ** -8)[0]))
        self.held = length
        return out, served, int(first[-1])

    def finish(self, done):
        self.free, self.held, self.n_free = K.release(self.held, done, self.table, self.free, self.n_free, BT)


@pytest.mark.parametrize("window", [0, 20])
def test_prompts_decode_leave_and_join(window):
    from paper_2606_30391_amd.serve import Server
    gen = torch.Generator("cuda").manual_seed(5)
    srv, ref = Server(4, CONTEXT, BLOCKS, TOKENS, LAYERS, H, D, BT), Reference(4)
    none, third = np.zeros(4, np.uint8), np.array([0, 0, 1, 0], np.uint8)
    steps = [([33, 1, 16, 100], none), ([1, 1, 1, 1], none), ([1, 15, 1, 0], third), ([1, 1, 47, 1], none),
             ([0, 0, 0, 0], none), ([1, 1, 1, 1], none),
             ([80, 1, 90, 1], none)]                       # the pool ends inside this one
    for n, (add, done) in enumerate(steps):
        print(f"[gpu] window {window}, step {n}: {add}", flush=True)
        T = min(sum(add), TOKENS)
        if sum(add) > TOKENS:
            with pytest.raises(ValueError):
                srv.step(add, None)
            add = [80, 1, 70, 1]
            T = sum(add)
        data = [[torch.randn((T, h, D), generator=gen, device="cuda").bfloat16() for h in (H * G, H, H)]
                for _ in range(LAYERS)]
        got = srv.step(add, lambda layer: data[layer], window)
        want, served, filled = ref.step(add, lambda layer: data[layer], window)
        assert np.array_equal(srv.blocks.served.cpu().numpy(), served)
        assert np.array_equal(srv.blocks.held.cpu().numpy(), ref.held)
        assert int(srv.blocks.n_free.item()) == ref.n_free
        for i, cache in enumerate(srv.caches):
            for r in range(4):
                for c in range(-(-int(ref.held[r]) // BT)):
                    b = ref.table[r, c]
                    assert int(srv.blocks.table[r, c].item()) == b
                    m = min(BT, int(ref.held[r]) - c * BT)
                    assert K.same_codes(cache.k[b, :, :m].cpu().numpy(), ref.layers[i][0][b, :, :m])
                    assert K.same_codes(cache.v[b, :, :, :m].cpu().numpy(), ref.layers[i][1][b, :, :, :m])
                    assert np.array_equal(cache.k_scale[b].cpu().numpy(), ref.layers[i][2][b])
                    assert np.array_equal(cache.v_scale[b].cpu().numpy(), ref.layers[i][3][b])
            o, tol = want[i]
            assert (np.abs(got[i].double().cpu().numpy() - o) <= tol)[:filled].all()
        if done.any():
            srv.finish(torch.from_numpy(done).cuda())
            ref.finish(done)
            assert int(srv.blocks.n_free.item()) == ref.n_free
    assert served.tolist() != [1, 1, 1, 1] and ref.n_free < 6


def test_the_command_serves_the_busiest_gpu(capsys):
    from paper_2606_30391_amd import serve
    serve.main(["--gpus", "8", "--requests", "64", "--most", "6", "--steps", "3", "--layers", "1", "--heads", "4",
                "--kv-heads", "2", "--dim", "64", "--block", "32"])
    said = capsys.readouterr().out
    print(said, flush=True)
    assert "prompts:" in said and "decode: 3 steps" in said


def test_the_layers_share_one_scratch():
    from paper_2606_30391_amd.serve import Server
    gen = torch.Generator("cuda").manual_seed(6)
    layers = 12
    srv = Server(8, 4096, 600, 400, layers, 2, 64, 64)
    add = [40] * 7 + [100]
    data = [[torch.randn((sum(add), h, 64), generator=gen, device="cuda").bfloat16() for h in (8, 2, 2)]
            for _ in range(layers)]
    print("[gpu] twelve layers, one scratch", flush=True)
    got = srv.step(add, lambda i: data[i])
    torch.cuda.synchronize()
    kept = [ws for c in srv.caches for ws, _, _ in c._ws.by_stream.values()]
    assert len({ws.data_ptr() for ws in kept}) == 1
    alone = Server(8, 4096, 600, 400, 1, 2, 64, 64)
    for i in (0, 5, 11):                                     # each layer's rows as if it were alone
        want = alone.step(add, lambda _: data[i])
        assert torch.equal(got[i], want[0])
        alone.finish(torch.ones(8, dtype=torch.uint8, device="cuda"))
