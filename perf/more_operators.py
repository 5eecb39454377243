"""Timed cases of a step of drafted tokens: rotation, draft trees, attention over them, acceptance, compaction.

A serving step may bring several drafted tokens a request, which form a tree: node 0 is the request's last
token, every other node a guess at what follows its parent.  The step's calls in the order in which they are made:
``plan`` turns the parents into the nodes' ancestors (a word a node) and positions, once for all layers;
``rotate`` normalises the queries and keys of each head and rotates them by those positions; ``attend`` lets every
node see the cached tokens and its ancestors; ``accept`` follows the tokens that the model chose down the trees; and
``keep`` moves the accepted nodes' keys and values of all layers together and gives the blocks behind them back.

Request lengths are those of the placement workloads, as in the serving operators' cases: "fleet" is
lognormal(6, 1) clipped to 16-8192, "bursty" 70% lognormal(5, 1) and 30% lognormal(8, 1), "even" spreads lengths
evenly over 1..longest and "same" gives every request the longest.  Lengths and trees follow from the case, so that its
work is known; the seed draws the requests' order, the tokens, the choices and all values.

``exact`` evaluates the same definitions (include/festina.h) in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn
DEV = "cuda"
MOST = 64                    # nodes of a tree; a request with more new tokens is a run, each the next one's parent


def listed():
    return [
        # --- ancestors and positions
        # a step of one GPU at the largest batch of the profile tables: 32 requests, trees of 8
        {"name": "plan-step", "op": "plan", "requests": 32, "law": "fleet", "longest": 8192, "nodes": 8, "spread": 2,
         "ragged": False, "prompt": 0},
        # a rack's requests at once, trees of 1 to 64, beside a prompt's chunk
        {"name": "plan-rack", "op": "plan", "requests": 4096, "law": "fleet", "longest": 8192, "nodes": 64, "spread": 5,
         "ragged": True, "prompt": 2048},
        # --- norms and rotation of queries and keys
        # the 256 nodes of such a step, heads side by side in one projection's output
        {"name": "rotate-step", "op": "rotate", "requests": 32, "law": "fleet", "longest": 8192, "nodes": 8, "spread": 2,
         "ragged": False, "prompt": 0, "heads": 32, "kv_heads": 8, "dim": 128, "rotated": 128, "interleaved": False,
         "norm": True, "dtype": "bf16", "packed": True, "far": 0},
        # a large prefill: prompts of the bursty law in one pass
        {"name": "rotate-prompts", "op": "rotate", "requests": 32, "law": "bursty", "longest": 8192, "nodes": 8192,
         "spread": 1, "ragged": False, "prompt": 0, "heads": 32, "kv_heads": 8, "dim": 128, "rotated": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "packed": False, "far": 0},
        # --- attention over the cache and the trees
        # one request alone, the latency of a tree of 8
        {"name": "drafts-one", "op": "attend", "requests": 1, "law": "fleet", "longest": 8192, "nodes": 8, "spread": 2,
         "ragged": False, "prompt": 0, "heads": 32, "kv_heads": 8, "dim": 128, "block": 64, "dtype": "bf16", "window": 0},
        # a step at the tables' largest batch
        {"name": "drafts-step", "op": "attend", "requests": 32, "law": "fleet", "longest": 8192, "nodes": 16, "spread": 3,
         "ragged": False, "prompt": 0, "heads": 32, "kv_heads": 8, "dim": 128, "block": 64, "dtype": "bf16", "window": 0},
        # trees of 1 to 61 nodes over half-precision heads of 64 with a window, beside a prompt's chunk
        {"name": "drafts-odd", "op": "attend", "requests": 41, "law": "bursty", "longest": 8191, "nodes": 61, "spread": 4,
         "ragged": True, "prompt": 777, "heads": 14, "kv_heads": 7, "dim": 64, "block": 32, "dtype": "f16", "window": 1000},
        # long contexts of every length: 64 requests up to 32,768 tokens, trees of 32
        {"name": "drafts-long", "op": "attend", "requests": 64, "law": "even", "longest": 32768, "nodes": 32, "spread": 3,
         "ragged": False, "prompt": 0, "heads": 32, "kv_heads": 8, "dim": 128, "block": 128, "dtype": "bf16", "window": 0},
        # --- what the model accepts
        {"name": "accept-step", "op": "accept", "requests": 32, "law": "fleet", "longest": 8192, "nodes": 8, "spread": 2,
         "ragged": False, "prompt": 0},
        {"name": "accept-rack", "op": "accept", "requests": 4096, "law": "fleet", "longest": 8192, "nodes": 64, "spread": 5,
         "ragged": True, "prompt": 2048},
        # --- the accepted nodes' keys and values moved together, the blocks behind them given back
        {"name": "keep-step", "op": "keep", "requests": 32, "law": "fleet", "longest": 1023, "nodes": 8, "spread": 2,
         "ragged": False, "prompt": 0, "layers": 4, "kv_heads": 8, "dim": 128, "block": 64},
        # wide trees over blocks of 16, which they span several of
        {"name": "keep-wide", "op": "keep", "requests": 160, "law": "even", "longest": 255, "nodes": 63, "spread": 5,
         "ragged": True, "prompt": 0, "layers": 4, "kv_heads": 8, "dim": 128, "block": 16},
    ]


def _log_int(rng, lo, hi):
    """Whole number, log-uniform over [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges, costing no more than the largest listed one."""
    op = rng.choice(["plan", "rotate", "rotate", "attend", "attend", "attend", "accept", "keep", "keep"])
    case = {"op": op, "law": rng.choice(["fleet", "bursty", "even"]), "nodes": _log_int(rng, 1, MOST),
            "spread": rng.randint(1, 6), "ragged": rng.random() < 0.5, "prompt": rng.choice([0, 0, 65, _log_int(rng, 66, 2048)])}
    if op in ("plan", "accept"):
        return {**case, "requests": _log_int(rng, 1, 4095), "longest": _log_int(rng, 64, 8191)}
    dim = rng.choice([64, 96, 128, 256])
    if op == "rotate":
        kv_heads = rng.randint(1, 12)
        case.update(longest=_log_int(rng, 16, 8191), heads=kv_heads * rng.choice([1, 2, 4, 7]), kv_heads=kv_heads, dim=dim,
                    rotated=rng.choice([dim, dim, dim // 2]), interleaved=rng.random() < 0.4, norm=rng.random() < 0.7,
                    dtype=rng.choice(["bf16", "f16", "f32"]), packed=rng.random() < 0.5, far=rng.choice([0, 0, 1 << 16, 1 << 24]))
        if rng.random() < 0.5:
            case["nodes"] = _log_int(rng, 65, 4096)
        tokens = max(case["nodes"], case["prompt"])
        most = max(1, 100_000_000 // ((case["heads"] + kv_heads) * dim * tokens))
        return {**case, "requests": _log_int(rng, 1, min(512, most))}
    block = rng.choice([16, 32, 64, 128])
    if op == "keep":
        layers, kv_heads, longest = rng.randint(1, 8), rng.randint(1, 12), _log_int(rng, 16, 511)
        most = max(1, 60_000_000 // (layers * kv_heads * dim * (max(longest, case["prompt"], 16) + block)))
        return {**case, "requests": _log_int(rng, 1, min(512, most)), "longest": longest, "layers": layers,
                "kv_heads": kv_heads, "dim": dim, "block": block}
    kv_heads = rng.choice([1, 2, 4, 7, 8])
    heads = kv_heads * rng.choice([1, 2, 4, 7, 8, 16])
    longest = max(case["nodes"], _log_int(rng, 16, 65536))
    wide = max(case["nodes"], case["prompt"])                      # (the plain form pads every request to the widest)
    most = min(1_000_000_000 // (longest * kv_heads * dim), 130_000_000_000 // (longest * heads * wide * dim))
    if most < 1:
        case["prompt"], most = 0, 1
        longest = max(case["nodes"], min(longest, 130_000_000_000 // (heads * case["nodes"] * dim)))
    return {**case, "requests": _log_int(rng, 1, max(1, min(256, most))), "longest": longest, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "block": block, "dtype": rng.choice(["bf16", "f16"]),
            "window": rng.choice([0, 0, 0, 1000])}


# ------------------------------------------------------------------------------ the cases' sizes

def lengths(case):
    """The law's quantiles over the requests, ascending."""
    n, longest = case["requests"], case["longest"]
    u = (torch.arange(n, dtype=torch.float64) + 0.5) / n
    if case["law"] == "same":
        x = torch.full((n,), float(longest), dtype=torch.float64)
    elif case["law"] == "even":
        x = 1 + u * (longest - 1)
    else:
        z = lambda p: math.sqrt(2.0) * torch.erfinv(2 * p - 1)  # noqa: E731
        if case["law"] == "fleet":
            x = torch.exp(6.0 + z(u))
        else:
            x = torch.where(u < 0.7, torch.exp(5.0 + z(u.clamp(max=0.6999) / 0.7)),
                            torch.exp(8.0 + z(((u - 0.7) / 0.3).clamp(1e-4, 1 - 1e-9))))
        x = x.clamp(min(16, longest), longest)
    return x.round().to(torch.int64)


def step(case):
    """(before, new): tokens cached before the step, and the step's new ones.  Request 0 brings a prompt's chunk
    where the case has one; where nodes pass what a tree may have, every request brings its whole prompt."""
    n = lengths(case)
    r = torch.arange(n.numel())
    if case["nodes"] > MOST:
        new = n.clamp(max=case["nodes"])
    else:
        new = 1 + (37 * r + 11) % case["nodes"] if case["ragged"] else torch.full_like(n, case["nodes"])
    if case["prompt"]:
        new[0] = case["prompt"]
    return (n - new).clamp(min=0), new


def trees(case):
    """Parents [R][64] of the requests' nodes, -1 for node 0; node i's parent is one of the `spread` nodes before it."""
    r, i = torch.arange(case["requests"])[:, None], torch.arange(MOST)[None, :]
    back = (7919 * i + 104729 * r) % i.clamp(min=1, max=case["spread"])
    return torch.where(i > 0, i - 1 - back, -1)


def depths(parent):
    depth = torch.zeros_like(parent)
    for i in range(1, MOST):
        depth[:, i] = depth.gather(1, parent[:, i:i + 1]).flatten() + 1
    return depth


def cdiv(a, b):
    return (a + b - 1) // b


def work(case):
    before, new = step(case)
    tokens, R = int(new.sum()), case["requests"]
    if case["op"] == "plan":
        return {"bytes": 8 * R + 16 * tokens, "flops": 0}
    if case["op"] == "accept":
        return {"bytes": 20 * R + 16 * tokens, "flops": 0}
    if case["op"] == "rotate":
        size = 4 if case["dtype"] == "f32" else 2
        elements = tokens * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * size * elements + 4 * tokens, "flops": 0}
    hd = case["kv_heads"] * case["dim"]
    if case["op"] == "keep":
        # half of the deepest path of each tree, a byte read and one written for each element of the keys and the values
        depth = torch.where(torch.arange(MOST) < new[:, None], depths(trees(case)), 0).amax(1)
        moved = int(torch.where(new <= MOST, depth, 0).sum()) // 2
        return {"bytes": 4 * case["layers"] * hd * moved + 12 * R + 4 * tokens, "flops": 0}
    w = case["window"] or (1 << 40)
    run = (new > MOST)[:, None]
    i = torch.arange(int(new.max()))
    depth = torch.zeros((R, max(MOST, i.numel())), dtype=torch.int64)
    depth[:, :MOST] = depths(trees(case))
    depth = torch.where(run, i, depth[:, :i.numel()])
    pairs = (before[:, None] + depth + 1).clamp(max=w)
    pairs = int(torch.where(i < new[:, None], pairs, 0).sum())
    seen = int(torch.minimum(before, torch.tensor(w)).sum()) + tokens
    return {"bytes": 2 * hd * seen + 4 * tokens * case["heads"] * case["dim"] + 8 * tokens,
            "flops": 4 * case["heads"] * case["dim"] * pairs}


# ------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _i32(x):
    return x.to(device=DEV, dtype=torch.int32)


def _codes(shape, g):
    """A cache's worth of e4m3 codes of normally distributed values (the scale is a power of two)."""
    out = torch.empty(shape, dtype=torch.uint8, device=DEV)
    for part in out.split(max(1, (1 << 28) // max(1, out[0].numel()))):
        x = torch.randn(part.shape, generator=g, device=DEV, dtype=torch.float32)
        part.copy_(x.mul_(112.0).clamp_(-448.0, 448.0).to(E4M3).view(torch.uint8))
    return out


def _scales(n_blocks, heads, g):
    e = torch.randint(-8, -5, (n_blocks, heads), generator=g, device=DEV)
    return torch.exp2(e.float())


def _flat(rows, new):
    """The entries [r, i < new[r]] of `rows`, request after request."""
    return rows[torch.arange(rows.shape[1], device=rows.device) < new[:, None]]


def prepare(case, seed):
    g = _gen(seed)
    R = case["requests"]
    order = torch.randperm(R, generator=g, device=DEV)
    before, new = (x.to(DEV)[order] for x in step(case))
    length, tokens = before + new, int(new.sum())
    first = torch.zeros(R + 1, dtype=torch.int64, device=DEV)
    first[1:] = torch.cumsum(new, 0)
    state = {"case": case, "tokens": tokens, "new": int(new.max()), "length": _i32(length), "first": _i32(first)}
    # the trees, one row of nodes a request; runs continue past what a tree may have
    tree = trees(case).to(DEV)[order]
    wide = max(MOST, int(new.max()))
    i = torch.arange(wide, device=DEV)
    parent = (i - 1).repeat(R, 1)
    parent[:, :MOST] = torch.where((new > MOST)[:, None], parent[:, :MOST], tree)
    state["parent"] = _i32(_flat(parent, new))
    if case["op"] in ("accept", "keep"):
        # tokens of a small vocabulary; three nodes of four were guessed right by some child
        token = torch.randint(0, 1000, (R, wide), generator=g, device=DEV)
        choice = torch.randint(0, 1000, (R, wide), generator=g, device=DEV)
        lucky = torch.rand((R, wide), generator=g, device=DEV) < 0.75
        lucky &= (i < new[:, None]) & (parent >= 0)
        child = torch.full((R, wide), -1, dtype=torch.int64, device=DEV)
        child.scatter_reduce_(1, parent.clamp(min=0), torch.where(lucky, i.expand(R, wide), -1), "amax")
        choice = torch.where(child >= 0, token.gather(1, child.clamp(min=0)), choice)
        state["token"], state["choice"] = _i32(_flat(token, new)), _i32(_flat(choice, new))
    if case["op"] in ("plan", "accept"):
        if own:
            from paper_2606_30391_amd import festina
            state["drafts"] = festina.DeviceDrafts(state["parent"], state.get("token"), R)
        return state
    d = case["dim"]
    depth = torch.zeros((R, wide), dtype=torch.int64, device=DEV)
    depth[:, :MOST] = depths(tree)
    depth = torch.where((new > MOST)[:, None], i, depth)
    if case["op"] == "rotate":
        heads, h, dtype, half = case["heads"], case["kv_heads"], DTYPES[case["dtype"]], case["rotated"] // 2
        state["position"] = _i32(_flat(before[:, None] + depth, new) + case["far"])
        state["freq"] = (1e4 ** (-torch.arange(half, dtype=torch.float64) / half))       # radians a position, host
        # the projections' outputs: queries, keys and values side by side in one buffer, or each on its own
        if case["packed"]:
            both = torch.randn((tokens, heads + 2 * h, d), generator=g, device=DEV).to(dtype)
            state["q"], state["k"] = both[:, :heads], both[:, heads:heads + h]
        else:
            state["q"] = torch.randn((tokens, heads, d), generator=g, device=DEV).to(dtype)
            state["k"] = torch.randn((tokens, h, d), generator=g, device=DEV).to(dtype)
        state["eps"] = 1e-6
        state["qw"] = state["kw"] = None
        if case["norm"]:
            state["qw"], state["kw"] = (1 + 0.2 * torch.randn((2, d), generator=g, device=DEV)).to(dtype).unbind(0)
        if own:
            from paper_2606_30391_amd import festina
            state["rotary"] = festina.DeviceRotary(state["freq"], d, state["qw"], state["kw"], state["eps"],
                                                   case["interleaved"], device=DEV)
        return state
    h, bt = case["kv_heads"], case["block"]
    have = cdiv(length, bt)
    used = int(have.sum())
    n_blocks = used + 3
    ids = torch.randperm(n_blocks, generator=g, device=DEV)
    c = torch.arange(int(have.max()), device=DEV)
    start = torch.cumsum(have, 0) - have
    state["table"] = _i32(torch.where(c < have[:, None], ids[(start[:, None] + c).clamp(max=n_blocks - 1)], -1))
    state["n_blocks"] = n_blocks
    layers = []
    for _ in range(case.get("layers", 1)):
        layers.append((_codes((n_blocks, h, bt, d), g), _codes((n_blocks, h, d, bt), g),
                       _scales(n_blocks, h, g), _scales(n_blocks, h, g)))
    # what lies past a request's last token in its last block is whatever was there
    last = state["table"].gather(1, (have - 1)[:, None]).flatten().long()
    past = torch.arange(bt, device=DEV) >= ((length - 1) % bt + 1)[:, None]
    for k, v, _, _ in layers:
        k[last] = torch.where(past[:, None, :, None], 0x7F, k[last].int()).to(torch.uint8)
        v[last] = torch.where(past[:, None, None, :], 0x7F, v[last].int()).to(torch.uint8)
    state["layers"] = layers
    if case["op"] == "attend":
        seen = torch.zeros((R, wide), dtype=torch.int64, device=DEV)
        for j in range(MOST):
            up = seen.gather(1, tree[:, j:j + 1].clamp(min=0)).flatten() if j else 0
            seen[:, j] = up | (1 << j if j < 63 else -(1 << 63))
        state["seen"] = _flat(torch.where((new > MOST)[:, None], 0, seen), new)
        state["depth"] = _flat(depth, new)
        state["q"] = torch.randn((tokens, case["heads"], d), generator=g, device=DEV).to(DTYPES[case["dtype"]])
    else:
        free = torch.full((n_blocks,), -1, dtype=torch.int32, device=DEV)
        free[:3] = _i32(ids[used:])
        state.update(free_ids=free, n_free=torch.tensor([3], dtype=torch.int32, device=DEV))
        state["path"], state["kept"], _, state["left"] = _accept(state)
    if own:
        from paper_2606_30391_amd import festina
        state["caches"] = [festina.DeviceCache(*x) for x in layers]
        if case["op"] == "keep":
            state["blocks"] = festina.DeviceBlocks(held=state["length"], add=torch.zeros_like(state["length"]),
                                                   table=state["table"], free_ids=state["free_ids"],
                                                   n_free=state["n_free"], block_tokens=bt, max_tokens=0)
    return state


# ------------------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    if not own:
        return {"plan": _plan, "rotate": _rotate, "attend": _attend, "accept": _accept, "keep": _keep}[case["op"]](state)
    if case["op"] == "plan":
        d = state["drafts"]
        d.plan(state["first"], state["length"])
        return d.seen, d.position
    if case["op"] == "accept":
        d = state["drafts"]
        d.accept(state["first"], state["length"], state["choice"])
        return d.path, d.kept, d.next, d.length
    if case["op"] == "rotate":
        return state["rotary"].apply(state["q"], state["k"], state["position"])
    cache = state["caches"][0]
    if case["op"] == "attend":
        return cache.attend(state["q"], state["table"], state["length"], state["first"], max_new=state["new"],
                            window=case["window"], seen=state["seen"])
    cache.keep(state["table"], state["length"], state["first"], state["path"], state["kept"], also=state["caches"][1:])
    b = state["blocks"]
    b.trim(state["left"])
    return [(c.k.view(E4M3), c.v.view(E4M3), c.k_scale, c.v_scale) for c in state["caches"]], b.free_ids, b.length, b.n_free_out


def _owner(s):
    """Of every token: its request, its index there, and its request's new tokens."""
    first = s["first"].long()
    t = torch.arange(s["tokens"], device=first.device)
    r = torch.searchsorted(first[1:], t, right=True)
    return r, t - first[r], (first[1:] - first[:-1])[r]


def _plan(s):
    r, i, n = _owner(s)
    first, before = s["first"].long(), (s["length"].long() - (s["first"][1:] - s["first"][:-1]).long())[r]
    parent, tree = s["parent"].long(), n <= MOST
    up = torch.where(tree & (parent >= 0) & (parent < i), parent, -1)
    bit = torch.bitwise_left_shift(torch.ones_like(i), i.clamp(max=63))
    seen, at, depth = torch.where(tree, bit, 0), up, torch.zeros_like(i)
    for _ in range(MOST - 1):                                # an ancestor a time
        there = at >= 0
        t = first[r] + at.clamp(min=0)
        seen = torch.where(there, seen | bit[t], seen)
        depth = depth + there
        at = torch.where(there, up[t], -1)
    return seen, (before + torch.where(tree, depth, i)).int()


def _rotate(s):
    case, half = s["case"], s["case"]["rotated"] // 2
    angle = s["position"].double()[:, None] * s["freq"].to(s["position"].device)
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    out = []
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        dtype, x = x.dtype, x.float()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * w.float()
        y = x.clone()
        if case["interleaved"]:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = x[..., :half], x[..., half:2 * half]
            y[..., :half], y[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
        out.append(y.to(dtype))
    return out[0], out[1]


def _accept(s):
    r, i, n = _owner(s)
    first, parent, R = s["first"].long(), s["parent"].long(), s["case"]["requests"]
    t = torch.arange(s["tokens"], device=r.device)
    tree = n <= MOST
    up = torch.where(tree & (parent >= 0) & (parent < i), parent, 0)
    # of every node, the first child whose token was chosen there
    right = tree & (i > 0) & (parent >= 0) & (parent < i) & (s["token"] == s["choice"][first[r] + up])
    child = torch.full((s["tokens"],), MOST, dtype=torch.int64, device=r.device)
    child.scatter_reduce_(0, first[r] + up, torch.where(right, i, MOST), "amin")
    new = first[1:] - first[:-1]
    run = new > MOST
    path = torch.where(tree, -1, i)
    kept = torch.where(run, new, (new > 0).long())
    node = torch.zeros(R, dtype=torch.int64, device=r.device)
    alive = (new > 0) & ~run
    last = torch.where(run, new - 1, 0)
    for k in range(min(MOST, s["new"])):                     # one node deeper a time
        at = (first[:-1] + k).clamp(max=s["tokens"] - 1)
        path = torch.where((i == k) & alive[r], node[r], path)
        kept = torch.where(alive, k + 1, kept)
        last = torch.where(alive, node, last)
        then = child[(first[:-1] + node).clamp(max=s["tokens"] - 1)]
        alive = alive & (then < MOST)
        node = torch.where(alive, then, node)
    chosen = s["choice"][(first[:-1] + last).clamp(max=s["tokens"] - 1)]
    left = s["length"].long() - new + kept
    return path.int(), kept.int(), torch.where(new > 0, chosen.long(), -1).int(), left.int()


def _attend(s):
    case, table, q = s["case"], s["table"].long(), s["q"]
    bt, h, d, new = case["block"], case["kv_heads"], case["dim"], s["new"]
    length, first = s["length"].long(), s["first"].long()
    n, columns = table.shape
    groups, keys = case["heads"] // h, columns * bt
    at = table.clamp(min=0)
    ck, cv, ks, vs = s["layers"][0]
    k = (ck.view(E4M3)[at].float() * ks[at][..., None, None]).permute(0, 2, 1, 3, 4).reshape(n, h, keys, d)
    v = (cv.view(E4M3)[at].float() * vs[at][..., None, None]).permute(0, 2, 1, 4, 3).reshape(n, h, keys, d)
    j = torch.arange(keys, device=q.device)
    v = torch.where((j < length[:, None])[:, None, :, None], v, 0.0)
    i = torch.arange(new, device=q.device)
    count = first[1:] - first[:-1]
    row = (first[:-1, None] + i).clamp(max=q.shape[0] - 1)
    qs = q[row].float().reshape(n, new, h, groups, d).permute(0, 2, 1, 3, 4).reshape(n, h, new * groups, d)
    x = torch.matmul(qs, k.transpose(-1, -2).contiguous()) / math.sqrt(d)
    before = length - count
    pos = before[:, None] + s["depth"][row]                  # of a node: the tokens before it on its path
    node = (j - before[:, None])[:, None, :]                 # which of the new tokens a key is
    word = s["seen"][row][..., None]
    tree = (node >= 0) & ((word >> node.clamp(0, 63)) & 1).bool() & (node < MOST)
    tree &= (node < count[:, None, None])
    run = (node >= 0) & (node <= i[:, None])
    sees = torch.where((count > MOST)[:, None, None], run, tree) | (node < 0)
    if case["window"]:                                       # ancestors are no more than a tree's nodes away
        sees &= (node >= 0) & (count <= MOST)[:, None, None] | (j > pos[..., None] - case["window"])
    sees = sees[:, None, :, None, :]
    x = torch.where(sees, x.view(n, h, new, groups, keys), -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, h, new * groups, keys), v).view(n, h, new, groups, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(n * new, h * groups, d)
    lse = (top + torch.log(total)).permute(0, 2, 1, 3, 4).reshape(n * new, h * groups)
    r, i, _ = _owner(s)
    return o[r * new + i].to(q.dtype), lse[r * new + i]


def _keep(s):
    case, table = s["case"], s["table"].long()
    bt, R = case["block"], case["requests"]
    r, i, n = _owner(s)
    first, length, kept = s["first"].long(), s["length"].long(), s["kept"].long()
    before = length - (first[1:] - first[:-1])
    path = s["path"].long()
    moved = (path >= 0) & (n <= MOST)                        # tokens i of the kept ones, from path[i]
    to, since = before[r] + i, before[r] + path.clamp(min=0)
    block, offset = table[r, (to // bt).clamp(max=table.shape[1] - 1)], to % bt
    source, place = table[r, since // bt], since % bt
    block, offset, source, place = block[moved], offset[moved], source[moved], place[moved]
    # the block of the first new token may hold older ones
    older = (kept > 0) & (before % bt > 0) & (first[1:] - first[:-1] <= MOST)
    part = table.gather(1, (before // bt).clamp(max=table.shape[1] - 1)[:, None]).flatten()[older]
    held = torch.arange(bt, device=r.device) < (before % bt)[older][:, None]
    out = []
    for layer in s["layers"]:
        for codes, scale, tokens_last in ((layer[0], layer[2], False), (layer[1], layer[3], True)):
            now = scale.clone()
            now[block] = 0.0
            now[part] = scale[part]
            now.index_reduce_(0, block, scale[source], "amax")
            x = codes[source, :, :, place] if tokens_last else codes[source, :, place]
            x = (x.view(E4M3).float() * (scale[source] / now[block])[..., None]).to(E4M3).view(torch.uint8)
            y = codes[part].view(E4M3).float() * (scale / now)[part][:, :, None, None]
            mask = held[:, None, None, :] if tokens_last else held[:, None, :, None]
            codes[part] = torch.where(mask, y.to(E4M3).view(torch.uint8).int(), codes[part].int()).to(torch.uint8)
            if tokens_last:
                codes[block, :, :, offset] = x
            else:
                codes[block, :, offset] = x
            scale.copy_(now)
        out.append((layer[0].view(E4M3), layer[1].view(E4M3), layer[2], layer[3]))
    # the blocks behind the kept tokens
    left, free = s["left"].long(), s["free_ids"]
    gives = (cdiv(length, bt) - cdiv(left, bt)).clamp(min=0)
    ends = torch.cumsum(gives, 0)
    e = torch.arange(free.numel(), device=r.device) - s["n_free"]
    who = torch.searchsorted(ends, e, right=True).clamp(max=R - 1)
    at = (cdiv(left, bt)[who] + e - (ends - gives)[who]).clamp(0, table.shape[1] - 1)
    free.copy_(torch.where((e >= 0) & (e < ends[-1]), table[who, at].int(), free))
    return out, free, left.int(), (s["n_free"] + ends[-1]).int()


# ------------------------------------------------------------------------------ 64 bits

def _e4m3_64(x):
    """x rounded to the nearest e4m3 value (ties to even), from the format's definition."""
    e = torch.frexp(x.abs())[1].to(torch.float64) - 1
    step_ = torch.exp2(e.clamp(min=-6) - 3)
    return torch.round(x / step_) * step_


def exact(case, seed):
    if case["op"] in ("plan", "accept"):
        return None                                          # whole numbers only
    f64 = torch.float64
    s = prepare(case, seed)
    if case["op"] == "rotate":
        n = case["rotated"]
        f = s["freq"].to(DEV)
        out = []
        for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
            y = x.to(f64)
            if w is not None:
                y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + s["eps"]) * w.to(f64)
            z = torch.view_as_complex((y[..., :n].unflatten(-1, (n // 2, 2)) if case["interleaved"] else
                                       y[..., :n].unflatten(-1, (2, n // 2)).transpose(-1, -2)).contiguous())
            z = z * torch.polar(torch.ones((), dtype=f64, device=DEV), s["position"].to(f64)[:, None, None] * f)
            z = torch.view_as_real(z)
            y[..., :n] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            out.append(y)
        return out[0], out[1]
    first, length = s["first"].tolist(), s["length"].tolist()
    if case["op"] == "keep":
        bt, path, kept = case["block"], s["path"].tolist(), s["kept"].tolist()
        out = []
        for k, v, ks, vs in s["layers"]:
            done = []
            for codes, scale in ((k.view(E4M3).to(f64), ks.to(f64)),
                                 (v.view(E4M3).to(f64).transpose(-1, -2).contiguous(), vs.to(f64))):
                values, was, now = codes * scale[:, :, None, None], scale, scale.clone()
                result = codes.clone()
                for r in range(case["requests"]):
                    n = first[r + 1] - first[r]
                    if n > MOST or n == 0:
                        continue
                    b = length[r] - n
                    table = s["table"][r].tolist()
                    p = [b + j for j in path[first[r]:first[r] + kept[r]]]       # where the kept tokens were
                    for c in range(b // bt, (b + kept[r] - 1) // bt + 1):
                        lo, hi = max(b, c * bt), min(b + kept[r], (c + 1) * bt)
                        came = [table[p[y - b] // bt] for y in range(lo, hi)]
                        if lo > c * bt:
                            came.append(table[c])
                        at = table[c]
                        now[at] = was[came].amax(0)
                        old = values[at, :, :lo - c * bt] / now[at][:, None, None]
                        result[at, :, :lo - c * bt] = _e4m3_64(old)
                        src = torch.tensor(p[lo - b:hi - b], device=DEV)
                        blk = torch.tensor([table[y // bt] for y in p[lo - b:hi - b]], device=DEV)
                        x = values[blk, :, src % bt].transpose(0, 1)
                        result[at, :, lo - c * bt:hi - c * bt] = _e4m3_64(x / now[at][:, None, None])
                done += [result, now]
            out.append((done[0], done[2].transpose(-1, -2).contiguous(), done[1], done[3]))
        return out, None, None, None
    q, heads, h, d, bt = s["q"].to(f64), case["heads"], case["kv_heads"], case["dim"], case["block"]
    out = torch.zeros((q.shape[0], heads, d), dtype=f64, device=DEV)
    lse = torch.full((q.shape[0], heads), -math.inf, dtype=f64, device=DEV)
    parent = s["parent"].tolist()
    ck, cv, ks, vs = s["layers"][0]
    for r in range(case["requests"]):
        a, b, n = first[r], first[r + 1], length[r]
        m, before = b - a, n - (b - a)
        if m > MOST:
            among = torch.ones((m, m), dtype=torch.bool, device=DEV).tril()
            depth = torch.arange(m, device=DEV)
        else:
            line = []                                        # each node's path from the root, itself included
            for i in range(m):
                line.append((line[parent[a + i]] if parent[a + i] >= 0 else []) + [i])
            among = torch.zeros((m, m), dtype=torch.bool)
            for i, x in enumerate(line):
                among[i, x] = True
            among = among.to(DEV)
            depth = torch.tensor([len(x) - 1 for x in line], device=DEV)
        place = torch.cat([torch.arange(before, device=DEV), before + depth])    # positions of the keys
        hidden = torch.cat([torch.zeros((m, before), dtype=torch.bool, device=DEV), ~among], 1)
        if case["window"]:
            hidden |= place <= (before + depth)[:, None] - case["window"]
        ids = s["table"][r, :cdiv(n, bt)].long()
        for g in range(h):
            k = (ck[ids, g].view(E4M3).to(f64) * ks[ids, g].to(f64)[:, None, None]).reshape(-1, d)[:n]
            v = (cv[ids, g].view(E4M3).to(f64) * vs[ids, g].to(f64)[:, None, None]).transpose(1, 2).reshape(-1, d)[:n]
            for y in range(g * (heads // h), (g + 1) * (heads // h)):
                x = (q[a:b, y] @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                lse[a:b, y] = torch.logsumexp(x, 1)
                out[a:b, y] = torch.exp(x - lse[a:b, y, None]) @ v
    return out, lse
