"""One GPU's serving steps over an 8-bit paged cache: what the GPU that the dispatcher chose then runs.

``Server`` holds the cache blocks of its requests and one cache a layer.  step() gives every request blocks and
slots for its new tokens (festina_extend_blocks), then in each layer stores their keys and values through the slot
map (festina_store_kv) and attends over the cache (festina_attend); finish() returns the blocks of finished requests
(festina_release_blocks).  The block tables, slots and lengths stay on the device: a step has no wait for it.

    python -m paper_2606_30391_amd.serve [--gpus 64] [--requests 1024] [--steps 64] [--layers 4] ...

draws a dispatcher workload, lets festina_dispatch_requests place it, and serves the requests of the GPU that got
most of them: their prompts in units of at most 2,048 tokens, then decode steps with a request leaving as its
predicted output is made.  Queries, keys and values are random (no model is involved).  It prints what a step's
cache and attention take, the part of a decode or prefill table's entry that grows with the tokens held.
"""
from __future__ import annotations

import argparse

import numpy as np

from . import festina, workloads

UNIT = 2048                # most prompt tokens of one request in a step (the sweep workload's prefill unit)


class Server:
    """Cache blocks and caches of up to n_requests requests of at most max_context tokens, n_blocks blocks of
    block_tokens in each of n_layers layers; step_tokens bounds the new tokens of a step."""

    def __init__(self, n_requests: int, max_context: int, n_blocks: int, step_tokens: int, n_layers: int,
                 n_kv_heads: int, head_dim: int, block_tokens: int = 64, device="cuda"):
        import torch
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)
        columns = -(-int(max_context) // int(block_tokens))
        free = torch.arange(n_blocks - 1, -1, -1, dtype=torch.int32, device=device)
        self.blocks = festina.DeviceBlocks(z(n_requests), z(n_requests), z(n_requests, columns), free,
                                           torch.full((1,), n_blocks, dtype=torch.int32, device=device),
                                           block_tokens, step_tokens)
        self.caches = []
        for _ in range(n_layers):                            # a step's layers follow one another: one scratch for all
            self.caches.append(festina.DeviceCache.empty(n_blocks, block_tokens, n_kv_heads, head_dim, device,
                                                         self.caches[0] if self.caches else None))

    def step(self, add, qkv, window: int = 0):
        """One step with add[r] new tokens of request r (host integers): each layer's attention, a list.

        qkv(layer) returns that layer's queries [tokens][heads][dim], keys and values [tokens][kv heads][dim] of the
        step's tokens, request after request; tokens is sum(add).  blocks.served says afterwards whose tokens were
        in the step: where blocks or step_tokens run out, those of the requests from there on are not, and their
        rows of the output hold nothing."""
        import torch
        add = np.ascontiguousarray(add, np.int32)
        tokens, b = int(add.sum()), self.blocks
        if add.shape != tuple(b.add.shape) or add.min(initial=0) < 0 or tokens > b.max_tokens:
            raise ValueError(f"add: {b.add.shape[0]} counts, none negative, of at most {b.max_tokens} tokens in all")
        host = torch.empty(b.add.shape, dtype=torch.int32, pin_memory=True)      # pageable memory would wait for the stream
        host.numpy()[:] = add
        b.add.copy_(host, non_blocking=True)
        b.extend()
        out = []
        for layer, cache in enumerate(self.caches):
            q, k, v = qkv(layer)
            cache.store(k, v, b.slot[:tokens])
            out.append(cache.attend(q, b.table, b.length, b.first, int(add.max(initial=1)), window=window)[0])
        b.advance()
        return out

    def finish(self, done):
        """Return the blocks of the requests whose done (device, uint8 or bool) is not 0; they hold no token then."""
        self.blocks.release(done)
        self.blocks.advance()


def busiest(n_requests: int, n_gpus: int, most: int, device="cuda"):
    """(GPU, prompt lengths, predicted outputs) of the GPU that the dispatcher gives most of a drawn workload."""
    import torch
    inp = workloads.make_dispatch(n_requests=n_requests, n_gpus=n_gpus)
    d = festina.DeviceDispatch(inp, device)
    d.run()
    torch.cuda.synchronize(device)
    gpu = d.results()[0]
    if not (gpu >= 0).any():
        raise SystemExit("the dispatcher placed no request")
    g = int(np.bincount(gpu[gpu >= 0]).argmax())
    mine = np.flatnonzero(gpu == g)[:most]
    return g, inp["requests"]["prompt_tokens"][mine], inp["requests"]["pred_out_tokens"][mine]


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(prog="python -m paper_2606_30391_amd.serve", description=__doc__.split("\n")[0])
    for name, value, what in (("--gpus", 64, "GPUs of the drawn fleet"), ("--requests", 1024, "requests drawn"),
                              ("--most", 32, "requests served at once"), ("--steps", 64, "decode steps"),
                              ("--layers", 4, "layers"), ("--heads", 32, "query heads"),
                              ("--kv-heads", 8, "key and value heads"), ("--dim", 128, "head dimension"),
                              ("--block", 64, "tokens of a block")):
        ap.add_argument(name, type=int, default=value, help=f"{what} ({value})")
    a = ap.parse_args(argv)
    g, prompt, output = busiest(a.requests, a.gpus, a.most)
    R = len(prompt)
    total = prompt + np.minimum(output, a.steps)
    n_blocks = int((-(-total // a.block)).sum())
    units = int(-(-prompt.max() // UNIT))
    tokens = max(int(np.minimum(prompt, UNIT).sum()), R)
    srv = Server(R, int(total.max()), n_blocks, tokens, a.layers, a.kv_heads, a.dim, a.block)
    gen = torch.Generator("cuda").manual_seed(1)
    new = lambda h: torch.randn((tokens, h, a.dim), generator=gen, device="cuda").bfloat16()
    q, k, v = new(a.heads), new(a.kv_heads), new(a.kv_heads)
    print(f"GPU {g}: {R} requests, {int(prompt.sum())} prompt tokens, {n_blocks} blocks of {a.block} tokens in {a.layers} "
          f"layers ({2 * n_blocks * a.block * a.kv_heads * a.dim * a.layers / 2**20:.0f} MiB)", flush=True)

    def timed(add):
        n = int(add.sum())
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        srv.step(add, lambda layer: (q[:n], k[:n], v[:n]))
        end.record()
        return begin, end

    timed(np.minimum(prompt, UNIT))                        # untimed: the first call loads the kernels
    srv.finish(torch.ones(R, dtype=torch.uint8, device="cuda"))
    left, marks = prompt.astype(np.int64), []
    for _ in range(units):
        add = np.minimum(left, UNIT)
        left = left - add
        marks.append(timed(add))
    torch.cuda.synchronize()
    print("prompts:", ", ".join(f"{b.elapsed_time(e):.2f}" for b, e in marks), "ms a step", flush=True)

    todo, marks = np.minimum(output, a.steps).astype(np.int64), []
    for _ in range(int(todo.max())):
        marks.append(timed((todo > 0).astype(np.int64)))
        todo -= todo > 0
        over = todo == 0
        if over.any():
            srv.finish(torch.from_numpy(over).cuda())
            todo[over] = -1
    torch.cuda.synchronize()
    ms = np.array([b.elapsed_time(e) for b, e in marks])
    print(f"decode: {len(ms)} steps, median {1e3 * np.median(ms):.0f} us a step, {1e3 * np.median(ms) / a.layers:.0f} us a "
          f"layer; {int(srv.blocks.n_free.item())} of {n_blocks} blocks free at the end")


if __name__ == "__main__":
    main()
