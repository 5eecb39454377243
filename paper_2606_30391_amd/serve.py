"""One GPU's serving steps over an 8-bit paged cache: what the GPU that the dispatcher chose then runs.

``Server`` holds the cache blocks of its requests and one cache a layer.  step() gives every request blocks and
slots for its new tokens (festina_extend_blocks), then in each layer stores their keys and values through the slot
map (festina_store_kv) and attends over the cache (festina_attend); finish() returns the blocks of finished requests
(festina_release_blocks).  verify() is a step whose new tokens are trees of drafted ones: each sees its own path
(festina_plan_drafts, festina_attend_drafts), and what the model does not accept leaves the cache again
(festina_accept_drafts, festina_keep_tokens, festina_trim_blocks).  Either normalises and rotates queries and keys when given a
DeviceRotary (festina_rotate_heads).  The block tables, slots and lengths stay on the device: a step has no wait for it.

    python -m paper_2606_30391_amd.serve [--gpus 64] [--requests 1024] [--steps 64] [--layers 4] ...

draws a dispatcher workload, lets festina_dispatch_requests place it, and serves the requests of the GPU that got
most of them: their prompts in units of at most 2,048 tokens, then decode steps with a request leaving as its
predicted output is made; with --draft N each decode step verifies a tree of N drafted tokens a request.  Queries, keys,
values and choices are random (no model is involved).  It prints what a step's cache and attention take, the part of a decode or
prefill table's entry that grows with the tokens held.
"""
from __future__ import annotations

import argparse

import numpy as np

from . import festina, workloads

UNIT = 2048                # most prompt tokens of one request in a step (the sweep workload's prefill unit)
NODES = 64                 # most tokens of a draft tree (festina_drafts): more of one request are a run


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
        i32 = lambda: torch.zeros(max(step_tokens, 0), dtype=torch.int32, device=device)
        self.runs = festina.DeviceDrafts(None, None, n_requests, step_tokens, self.blocks.table.device)
        self.drafts, self.choice = festina.DeviceDrafts(i32(), i32(), n_requests), i32()

    def step(self, add, qkv, window: int = 0, rotary=None):
        """One step with add[r] new tokens of request r (host integers): each layer's attention, a list.

        qkv(layer) returns that layer's queries [tokens][heads][dim], keys and values [tokens][kv heads][dim] of the
        step's tokens, request after request; tokens is sum(add).  blocks.served says afterwards whose tokens were
        in the step: where blocks or step_tokens run out, those of the requests from there on are not, and their
        rows of the output hold nothing.  rotary (a DeviceRotary) is applied to the queries and keys at their positions."""
        add = np.ascontiguousarray(add, np.int32)
        out = self._layers(self._begin(add), int(add.max(initial=1)), qkv, window, rotary)
        self.blocks.advance()
        return out

    def verify(self, add, parent, token, qkv, choose, window: int = 0, rotary=None, known=None):
        """One step of drafted tokens: add[r] nodes of request r's tree (host integers; 0: none), parent and token [tokens] theirs,
        request after request (device int32; festina_drafts).  qkv as for step(); choose(outputs of the layers) returns the
        tokens [tokens] (device int32) that the model chooses behind the nodes.  Returns the layers' outputs; drafts.next [requests]
        is the token behind each request's accepted ones, drafts.kept their number, drafts.path which they were.

        known[r] (host integers, of which 0 is as 1) says how many of request r's tokens are no guesses, such as the rest of a prompt: from
        the first on they follow one another, whatever parent says, and all are kept, whatever the model chooses; the tree goes on
        behind the last of them.  Without it the first alone is known, and what the model would not have chosen leaves the cache.
        More than 64 new tokens of a request are no tree but a run, all of them known: parent is not read for them."""
        import torch
        b, d, add = self.blocks, self.drafts, np.ascontiguousarray(add, np.int32)
        chain = None if known is None else self._chain(add, known)
        each, int32 = (int(add.sum()),), (torch.int32,)      # (copies would repeat what is shorter)
        festina._check(parent, "parent", int32, each)
        festina._check(token, "token", int32, each)
        tokens = self._begin(add)
        d.parent[:tokens].copy_(parent)
        d.token[:tokens].copy_(token)
        if chain is not None:
            at, then, node = self._indexes(chain)
            d.parent.index_copy_(0, then, node.int())
        d.plan(b.first, b.length)
        out = self._layers(tokens, int(add.max(initial=1)), qkv, window, rotary, d)
        choice = choose(out)
        festina._check(choice, "choose()", int32, each)
        self.choice[:tokens].copy_(choice)
        if chain is not None:
            # the first child with the chosen token is the next known one
            self.choice.index_copy_(0, at, d.token.index_select(0, then))
        d.accept(b.first, b.length, self.choice)
        if self.caches:
            self.caches[0].keep(b.table, b.length, b.first, d.path, d.kept, also=self.caches[1:])
        b.advance()
        b.trim(d.length)
        b.advance()
        return out

    @staticmethod
    def _chain(add, known):
        """Known tokens that another known one follows: their index in the step, that one's, and their index in their request."""
        known = np.ascontiguousarray(known, np.int64)
        if add.ndim != 1 or known.shape != add.shape or (known < 0).any() or (known > add).any() or ((add > NODES) & (known < add)).any():
            raise ValueError(f"known: a count for each request, of at most its new tokens; all of more than {NODES}")
        n = np.where(add > NODES, 0, np.maximum(known - 1, 0))
        if not n.any():
            return None
        node = np.concatenate([np.arange(x) for x in n])
        at = np.repeat(np.cumsum(add, dtype=np.int64) - add, n) + node
        return np.stack([at, at + 1, node])

    def _indexes(self, chain):
        import torch
        host = torch.empty(chain.shape, dtype=torch.int64, pin_memory=True)      # as in _begin()
        host.numpy()[:] = chain
        return host.to(self.choice.device, non_blocking=True).unbind(0)

    def _begin(self, add):
        """Blocks and slots of a step with add (an int32 array) new tokens; how many they are."""
        import torch
        tokens, b = int(add.sum()), self.blocks
        if add.shape != tuple(b.add.shape) or add.min(initial=0) < 0 or tokens > b.max_tokens:
            raise ValueError(f"add: {b.add.shape[0]} counts, none negative, of at most {b.max_tokens} tokens in all")
        host = torch.empty(b.add.shape, dtype=torch.int32, pin_memory=True)      # pageable memory would wait for the stream
        host.numpy()[:] = add
        b.add.copy_(host, non_blocking=True)
        b.extend()
        return tokens

    def _layers(self, tokens, longest, qkv, window, rotary, drafts=None):
        b, out = self.blocks, []
        seen = None if drafts is None else drafts.seen[:tokens]
        if rotary is not None and drafts is None:
            drafts = self.runs
            drafts.plan(b.first, b.length)
        for layer, cache in enumerate(self.caches):
            q, k, v = qkv(layer)
            if rotary is not None:
                q, k = rotary.apply(q, k, drafts.position[:tokens])
            cache.store(k, v, b.slot[:tokens])
            out.append(cache.attend(q, b.table, b.length, b.first, max(longest, 1), window=window, seen=seen)[0])
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
                              ("--block", 64, "tokens of a block"), ("--draft", 0, "drafted tokens of a request and step, up to 64")):
        ap.add_argument(name, type=int, default=value, help=f"{what} ({value})")
    a = ap.parse_args(argv)
    if not 0 <= a.draft <= 64:
        ap.error("--draft: 0 to 64")
    g, prompt, output = busiest(a.requests, a.gpus, a.most)
    R = len(prompt)
    total = prompt + np.minimum(output, a.steps) + 2 * a.draft
    n_blocks = int((-(-total // a.block)).sum())
    units = int(-(-prompt.max() // UNIT))
    tokens = max(int(np.minimum(prompt, UNIT).sum()), R * max(a.draft, 1))
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
    chosen = torch.randint(0, 2, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    drafted = torch.randint(0, 2, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    parent = torch.from_numpy(np.tile(np.maximum(np.arange(max(a.draft, 1)) - 2, -1) + (np.arange(max(a.draft, 1)) == 1),
                                      R).astype(np.int32)).cuda()        # two guesses a node, side by side
    made = 0

    def verified(add):
        n = int(add.sum())
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        srv.verify(add, parent[:n], drafted[:n], lambda layer: (q[:n], k[:n], v[:n]), lambda out: chosen[:n])
        end.record()
        return begin, end

    if a.draft:
        verified(np.zeros(R, np.int64))                      # untimed
    for _ in range(int(todo.max())):
        if not (todo > 0).any():
            break
        alive = (todo > 0).astype(np.int64)
        if a.draft:
            marks.append(verified(alive * a.draft))
            kept = np.minimum(srv.drafts.kept.cpu().numpy(), np.maximum(todo, 0))
            made += int(kept.sum())
            todo -= kept
        else:
            marks.append(timed(alive))
            todo -= todo > 0
        over = todo == 0
        if over.any():
            srv.finish(torch.from_numpy(over).cuda())
            todo[over] = -1
    torch.cuda.synchronize()
    ms = np.array([b.elapsed_time(e) for b, e in marks])
    if a.draft:
        print(f"drafts: {made} tokens in {len(ms)} steps of up to {R} trees of {a.draft}")
    print(f"decode: {len(ms)} steps, median {1e3 * np.median(ms):.0f} us a step, {1e3 * np.median(ms) / a.layers:.0f} us a "
          f"layer; {int(srv.blocks.n_free.item())} of {n_blocks} blocks free at the end")


if __name__ == "__main__":
    main()
