"""What the speed of the operators around a bounded KV cache is measured on, through the calls of ``binding``:

``rope``    ``mlora_rope_append``: rotates a pass's queries and keys (half-split or interleaved pairs, part of a head, any
            frequencies) and appends its K/V rows to the streams' own segments.
``scored``  ``mlora_attention_scored``: attention over shared prefix, own segments and draft tree that also adds every key's
            softmax weight, summed over the rows and query heads that share its KV head, to a running total.
``evict``   ``mlora_kv_evict``: keeps the ``budget`` rows of an own segment with the largest totals (the newest in any case) and
            moves the kept rows that lie behind the budget into the places of the dropped ones.

With ``own`` false the operators run in a plain form of elementary torch operations; with it true, as the framework's calls.
Heads, streams, prompts and trees are those of ``gen.configs``; values are synthetic and made on the GPU from the seed alone."""
import math

import numpy as np
import torch

own = False

# query heads, KV heads, features of a head
HEADS = {"1b": (32, 8, 64), "3b": (24, 8, 128)}
_TYPES = {"fp16": torch.float16, "fp32": torch.float32}


# ----------------------------------------------------------------------------- the cases
def listed():
    return [
        # one stream's decode step: the smallest call, all latency.  q, k, v as the fused projection writes them
        {"name": "rope_step_1", "kind": "rope", "heads": "1b", "streams": 1, "nodes": 1, "dtype": "fp32", "rotary": 64,
         "interleaved": False, "scaling": "plain", "suffix": 64, "spread": 0.0, "capacity": 320, "base": 512},
        # a tree pass of eight streams behind a long prompt, context stretched by a ramp over the frequencies
        {"name": "rope_tree_8x32", "kind": "rope", "heads": "3b", "streams": 8, "nodes": 32, "dtype": "fp32", "rotary": 128,
         "interleaved": False, "scaling": "ramp", "suffix": 777, "spread": 0.9, "capacity": 1056, "base": 60000},
        # a long prompt into one segment: interleaved pairs in half of every head
        {"name": "rope_prompt_16384", "kind": "rope", "heads": "1b", "streams": 1, "nodes": 16384, "dtype": "fp16", "rotary": 32,
         "interleaved": True, "scaling": "plain", "suffix": 0, "spread": 0.0, "capacity": 16384, "base": 0},
        # the rest of a prompt of odd length behind what is cached, three quarters of every head, scaled by wavelength
        {"name": "rope_prompt_5003", "kind": "rope", "heads": "3b", "streams": 1, "nodes": 5003, "dtype": "fp32", "rotary": 96,
         "interleaved": False, "scaling": "waves", "suffix": 1021, "spread": 0.0, "capacity": 6144, "base": 100000},
        # one stream's decode step, short context
        {"name": "scored_step_1", "kind": "scored", "heads": "1b", "streams": 1, "nodes": 1, "prefix": 512, "suffix": 64,
         "spread": 0.0, "capacity": 320},
        # eight streams of very different lengths behind the benchmark's prompt
        {"name": "scored_step_8", "kind": "scored", "heads": "1b", "streams": 8, "nodes": 1, "prefix": 512, "suffix": 2048,
         "spread": 0.95, "capacity": 2304},
        # eight long streams of the larger heads: every byte of the cache is read
        {"name": "scored_long_8", "kind": "scored", "heads": "3b", "streams": 8, "nodes": 1, "prefix": 2048, "suffix": 16384,
         "spread": 0.1, "capacity": 16640},
        # tree passes: 16 nodes behind the benchmark's prompt, 32 nodes of the larger heads
        {"name": "scored_tree_8x16", "kind": "scored", "heads": "1b", "streams": 8, "nodes": 16, "prefix": 512, "suffix": 256,
         "spread": 0.5, "capacity": 320},
        {"name": "scored_tree_8x32", "kind": "scored", "heads": "3b", "streams": 8, "nodes": 32, "prefix": 2048, "suffix": 1024,
         "spread": 0.3, "capacity": 1056},
        # one row too many, the steady state of a bounded stream that decodes
        {"name": "evict_1_of_257", "kind": "evict", "heads": "1b", "streams": 1, "suffix": 257, "spread": 0.0, "capacity": 320,
         "budget": 256, "recent": 32},
        # eight streams after tree rounds that accepted different numbers of rows
        {"name": "evict_8_to_2048", "kind": "evict", "heads": "1b", "streams": 8, "suffix": 2066, "spread": 0.01, "capacity": 2304,
         "budget": 2048, "recent": 128},
        # long prompts of 16 streams cut to half
        {"name": "evict_16_to_4096", "kind": "evict", "heads": "3b", "streams": 16, "suffix": 8192, "spread": 0.4, "capacity": 8320,
         "budget": 4096, "recent": 512},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "scored", "scored", "evict"])
    heads = rng.choice(sorted(HEADS))
    hd = HEADS[heads][2]
    spread = round(rng.uniform(0.0, 1.0), 2)
    if kind == "rope":
        streams = _log(rng, 1, 64)
        nodes = rng.choice([1, _log(rng, 1, 64), _log(rng, 1, 16384 // streams)])
        suffix = _log(rng, 1, 2048) - 1
        return {"kind": kind, "heads": heads, "streams": streams, "nodes": nodes, "dtype": rng.choice(sorted(_TYPES)),
                "rotary": 16 * rng.randint(1, hd // 16), "interleaved": rng.random() < 0.5,
                "scaling": rng.choice(["plain", "linear", "base", "waves", "ramp"]), "suffix": suffix, "spread": spread,
                "capacity": suffix + nodes + rng.randint(0, 64), "base": _log(rng, 1, 1 << 20) - 1}
    if kind == "scored":
        if rng.random() < 0.5:
            streams, nodes = _log(rng, 1, 32), 1
            suffix = _log(rng, 1, min(32768, 131072 // streams)) - 1
            prefix = rng.choice([0, _log(rng, 1, 4096)])
        else:
            nodes = rng.randint(2, 64)
            streams = _log(rng, 1, max(1, 256 // nodes))
            suffix, prefix = _log(rng, 1, 1024) - 1, rng.choice([0, _log(rng, 1, 2048)])
        return {"kind": kind, "heads": heads, "streams": streams, "nodes": nodes, "prefix": prefix, "suffix": suffix,
                "spread": spread, "capacity": suffix + nodes + rng.randint(0, 64)}
    streams = _log(rng, 1, 32)
    suffix = _log(rng, 2, min(32768, 131072 // streams))
    budget = max(1, min(suffix, int(suffix * rng.choice([rng.uniform(0.1, 1.0), 0.99]))))
    return {"kind": kind, "heads": heads, "streams": streams, "suffix": suffix, "spread": spread, "capacity": suffix + rng.randint(0, 64),
            "budget": budget, "recent": rng.choice([0, rng.randint(0, budget)])}


def _lengths(c):
    """rows in the streams' own segments: from `suffix` down to `suffix` * (1 - `spread`)"""
    n = c["streams"]
    return [c["suffix"] - int(c["suffix"] * c["spread"] * s / max(1, n - 1)) for s in range(n)]


# ----------------------------------------------------------------------------- inputs
def _frequencies(rotary, scaling):
    """radians per position of every pair, and the factor on cos and sin: contexts of 8192 stretched by 8"""
    theta, length, factor = 1e4, 8192.0, 8.0
    i = np.arange(rotary // 2, dtype=np.float64)
    if scaling == "base" and rotary > 2:
        theta *= factor ** (rotary / (rotary - 2.0))
    f = theta ** (-2.0 * i / rotary)
    if scaling == "linear":
        f = f / factor
    elif scaling == "waves":                       # long waves / factor, short ones as they are, a slope between
        s = np.clip((length * f / (2 * math.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = (1 - s) * f / factor + s * f
    elif scaling == "ramp":                        # pairs of 32 turns and more as they are, of one and less / factor
        dim = lambda turns: rotary * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
        lo, hi = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), rotary - 1)
        ramp = np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        f = f / factor * ramp + f * (1 - ramp)
    return f, (0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0)


def _parents(n, T, branch=3):
    """the same tree for every stream: node i hangs off node (i - 1) // branch"""
    p = [-1] + [(i - 1) // branch for i in range(1, T)]
    return p, torch.tensor([p] * n, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = case
    Hq, Hkv, hd = HEADS[c["heads"]]
    n, cap = c["streams"], c["capacity"]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *s, dtype=torch.float16: torch.randn(*s, generator=g, device="cuda", dtype=dtype)  # noqa: E731
    lens = _lengths(c)
    st = {"case": c, "lens": lens, "suffix_len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
          "status": torch.zeros(1, dtype=torch.int32, device="cuda"),
          "own_k": rand(n, Hkv, cap, hd), "own_v": rand(n, Hkv, cap, hd)}
    # (what keys have gathered so far: a few much, most little)
    st["own_weight"] = torch.empty(n, Hkv, cap, device="cuda").exponential_(generator=g) ** 2
    if c["kind"] == "rope":
        T = c["nodes"]
        rows = n * T
        qkv = rand(rows, (Hq + 2 * Hkv) * hd, dtype=_TYPES[c["dtype"]])
        st["q"], st["k"], st["v"] = qkv.split([Hq * hd, Hkv * hd, Hkv * hd], dim=1)
        if T <= 64:                                # a tree: a node's position is its depth
            p, _ = _parents(n, T)
            depth = [0] * T
            for i in range(1, T):
                depth[i] = depth[p[i]] + 1
        else:
            depth = range(T)
        st["positions"] = (c["base"] + st["suffix_len"].view(n, 1) + torch.tensor(list(depth), dtype=torch.int32, device="cuda")).view(-1)
        f, st["gain"] = _frequencies(c["rotary"], c["scaling"])
        st["freq"] = torch.from_numpy(f).cuda()
        st["q_out"] = torch.empty(rows, Hq, hd, dtype=torch.float16, device="cuda")
        st["own_position"] = torch.randint(0, 1 << 20, (n, Hkv, cap), generator=g, device="cuda", dtype=torch.int32)
    elif c["kind"] == "scored":
        T, P = c["nodes"], c["prefix"]
        st["q"] = rand(n * T, Hq, hd)
        st["prefix_k"], st["prefix_v"] = (rand(Hkv, P, hd), rand(Hkv, P, hd)) if P else (None, None)
        st["prefix_weight"] = torch.empty(Hkv, P, device="cuda").exponential_(generator=g) if P else None
        st["parent"], st["tree"] = _parents(n, T)
        st["out"] = torch.empty(n * T, Hq, hd, dtype=torch.float16, device="cuda")
    else:
        # positions: the rows that earlier calls kept in no order, then those appended since; every 16th total is a tie
        pos = torch.arange(cap, device="cuda", dtype=torch.int32).repeat(n, Hkv, 1)
        B = c["budget"]
        order = torch.rand(n, Hkv, B, generator=g, device="cuda").argsort(dim=2).to(torch.int32)
        pos[:, :, :B] = order
        st["own_position"] = pos
        tie = torch.rand(n, Hkv, cap, generator=g, device="cuda") < 1 / 16
        st["own_weight"] = torch.where(tie, torch.tensor(0.25, device="cuda"), st["own_weight"])
        st["newest"] = st["suffix_len"] - 1
        # the totals and positions are written beside the ones that were read: a program that steps swaps the two
        st["out_weight"], st["out_position"] = torch.zeros_like(st["own_weight"]), torch.zeros_like(pos)
        st["out_len"] = torch.zeros_like(st["suffix_len"])
    return st


# ----------------------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own_rope(state) if kind == "rope" else _own_scored(state) if kind == "scored" else _own_evict(state)
    return _plain_rope(state) if kind == "rope" else _plain_scored(state) if kind == "scored" else _plain_evict(state)


def _out_rope(st):
    return {"q": st["q_out"], "k": st["own_k"], "v": st["own_v"], "weight": st["own_weight"], "position": st["own_position"]}


def _out_scored(st):
    return {"out": st["out"], "weight": st["own_weight"], "prefix_weight": st["prefix_weight"]}


def _out_evict(st):
    return {"k": st["own_k"], "v": st["own_v"], "weight": st["out_weight"], "position": st["out_position"], "len": st["out_len"]}


def _own_rope(st):
    from paper_2604_18655_b200 import binding as mb
    mb.mlora_rope_append(st["q"], st["k"], st["v"], st["positions"], st["freq"], st["q_out"], st["own_k"], st["own_v"],
                         st["suffix_len"], st["status"], gain=st["gain"], interleaved=st["case"]["interleaved"],
                         own_weight=st["own_weight"], own_position=st["own_position"])
    return _out_rope(st)


def _own_scored(st):
    from paper_2604_18655_b200 import binding as mb
    c = st["case"]
    if "workspace" not in st:                      # (once: a program keeps it)
        Hq, Hkv, hd = HEADS[c["heads"]]
        st["workspace"] = torch.empty(mb.mlora_attention_scored_workspace_bytes(c["streams"], c["nodes"], Hq, Hkv, hd, c["prefix"],
                                                                                c["suffix"]), dtype=torch.uint8, device="cuda")
    mb.mlora_attention_scored(st["q"], st["prefix_k"], st["prefix_v"], st["own_k"], st["own_v"], st["suffix_len"], c["suffix"],
                              st["tree"], st["out"], st["own_weight"], st["prefix_weight"], st["workspace"], st["status"])
    return _out_scored(st)


def _own_evict(st):
    from paper_2604_18655_b200 import binding as mb
    c = st["case"]
    if "workspace" not in st:
        st["workspace"] = torch.empty(mb.mlora_kv_evict_workspace_bytes(c["streams"], HEADS[c["heads"]][1], c["suffix"], c["budget"]),
                                      dtype=torch.uint8, device="cuda")
    mb.mlora_kv_evict(st["own_k"], st["own_v"], st["own_weight"], st["own_position"], st["suffix_len"], c["suffix"], st["newest"],
                      c["budget"], c["recent"], st["out_weight"], st["out_position"], st["out_len"], st["workspace"], st["status"])
    return _out_evict(st)


# ----------------------------------------------------------------------------- plain forms
def _plain_rotate(x, positions, freq, gain, rotary, interleaved):
    """x [rows, heads, hd], 32 bits"""
    angle = positions.double()[:, None] * freq[None]                       # far positions: 64 bits
    angle = angle - torch.round(angle / (2 * math.pi)) * (2 * math.pi)
    cos, sin = (torch.cos(angle) * gain).float()[:, None], (torch.sin(angle) * gain).float()[:, None]
    r, h = x[..., :rotary], rotary // 2
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :h], r[..., h:])
    u, w = a * cos - b * sin, b * cos + a * sin
    r = torch.stack((u, w), dim=-1).flatten(-2) if interleaved else torch.cat((u, w), dim=-1)
    return torch.cat((r, x[..., rotary:]), dim=-1)


def _plain_rope(st):
    c = st["case"]
    Hq, Hkv, hd = HEADS[c["heads"]]
    n, T = c["streams"], c["nodes"]
    args = (st["positions"], st["freq"], st["gain"], c["rotary"], c["interleaved"])
    st["q_out"].copy_(_plain_rotate(st["q"].float().view(-1, Hq, hd), *args))
    k = _plain_rotate(st["k"].float().view(-1, Hkv, hd), *args).half().view(n, T, Hkv, hd).transpose(1, 2)
    v = st["v"].half().view(n, T, Hkv, hd).transpose(1, 2)
    at = (st["suffix_len"].long()[:, None] + torch.arange(T, device="cuda"))[:, None, :].expand(n, Hkv, T)
    full = at[..., None].expand(n, Hkv, T, hd)
    st["own_k"].scatter_(2, full, k)
    st["own_v"].scatter_(2, full, v)
    st["own_weight"].scatter_(2, at, 0.0)
    st["own_position"].scatter_(2, at, st["positions"].view(n, 1, T).expand(n, Hkv, T))
    return _out_rope(st)


def _plain_scored(st):
    c = st["case"]
    Hq, Hkv, hd = HEADS[c["heads"]]
    n, T, P = c["streams"], c["nodes"], c["prefix"]
    G, L = Hq // Hkv, c["suffix"] + c["nodes"]
    q = st["q"].float().view(n, T, Hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(n, Hkv, T * G, hd) / math.sqrt(hd)
    k, v = st["own_k"][:, :, :L].float(), st["own_v"][:, :, :L]
    s = torch.matmul(q, k.transpose(2, 3)).view(n, Hkv, T, G, L)
    # which own rows a node sees: the cached ones, and those of its path to the root
    sees = torch.zeros(T, T, dtype=torch.bool, device="cuda")
    up = torch.arange(T, device="cuda")
    par = st["tree"][0].long()
    for _ in range(1 + int(math.log(max(T, 1), 3)) + 1):                   # (the trees are three wide: no path is longer)
        sees[torch.arange(T, device="cuda"), up] = True
        up = torch.clamp(par[up], min=0)
    j = torch.arange(L, device="cuda")[None] - st["suffix_len"].long()[:, None]           # [n, L] place among the pass's rows
    tree = sees[:, torch.clamp(j, 0, T - 1)].permute(1, 0, 2) & (j < T)[:, None]          # [n, T, L]
    s = s.masked_fill(~((j < 0)[:, None] | tree)[:, None, :, None, :], -math.inf)
    top = s.amax(dim=-1)
    if P:
        sp = torch.matmul(q.transpose(0, 1).reshape(Hkv, n * T * G, hd), st["prefix_k"].float().transpose(1, 2))
        sp = sp.view(Hkv, n, T, G, P).transpose(0, 1)
        top = torch.maximum(top, sp.amax(dim=-1))
        sp = torch.exp(sp - top[..., None])
    s = torch.exp(s - top[..., None])
    total = s.sum(dim=-1) + (sp.sum(dim=-1) if P else 0)
    s = s / total[..., None]
    # rows behind the pass are not read: what they hold is not part of the sum
    out = torch.matmul(s.view(n, Hkv, T * G, L), v.float().masked_fill((j >= T)[:, None, :, None], 0.0))
    if P:
        sp = sp / total[..., None]
        op = torch.matmul(sp.transpose(0, 1).reshape(Hkv, n * T * G, P), st["prefix_v"].float())
        out = out + op.view(Hkv, n, T * G, hd).transpose(0, 1)
        st["prefix_weight"] += sp.sum(dim=(0, 2, 3))
    st["own_weight"][:, :, :L] += s.sum(dim=(2, 3))
    st["out"].copy_(out.view(n, Hkv, T, G, hd).transpose(1, 2).reshape(n * T, Hq, hd))
    return _out_scored(st)


def _plain_evict(st):
    c = st["case"]
    n, S, B = c["streams"], c["suffix"], c["budget"]
    Hkv, hd = st["own_k"].shape[1], st["own_k"].shape[3]
    w, pos, lens = st["own_weight"][:, :, :S], st["own_position"][:, :, :S], st["suffix_len"].long()
    i = torch.arange(S, device="cuda").expand(n, Hkv, S)
    there = i < lens[:, None, None]
    newest = pos > (st["newest"].long() - c["recent"])[:, None, None]
    # the order of keeping: rows that are there, the newest, falling total, rising index
    order = torch.sort(w, dim=2, descending=True, stable=True).indices
    rank = (there.long() * 2 + (there & newest).long()).gather(2, order)
    order = order.gather(2, torch.sort(rank, dim=2, descending=True, stable=True).indices)
    keep = torch.zeros(n, Hkv, S, dtype=torch.bool, device="cuda").scatter_(2, order[:, :, :B], True) & there
    # the kept rows behind the budget go to the dropped places before it, both in rising order
    hole, mover = ~keep & (i < B) & there, keep & (i >= B)
    holes = torch.sort(hole.to(torch.uint8), dim=2, descending=True, stable=True).indices[:, :, :B]
    movers = torch.sort(mover.to(torch.uint8), dim=2, descending=True, stable=True).indices[:, :, :B]
    moves = torch.arange(min(B, S), device="cuda") < mover.sum(dim=2, keepdim=True)
    src = i[:, :, :B].scatter(2, holes, torch.where(moves, movers, holes))
    full = src[..., None].expand(n, Hkv, src.shape[2], hd)
    alive = src < lens[:, None, None]
    st["own_k"][:, :, :B] = st["own_k"].gather(2, full)
    st["own_v"][:, :, :B] = st["own_v"].gather(2, full)
    st["out_weight"][:, :, :B] = torch.where(alive, w.gather(2, src), st["out_weight"][:, :, :B])
    st["out_position"][:, :, :B] = torch.where(alive, pos.gather(2, src), st["out_position"][:, :, :B])
    st["out_len"].copy_(torch.clamp(lens, max=B))
    return _out_evict(st)


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    Hq, Hkv, hd = HEADS[c["heads"]]
    lens, n = _lengths(c), c["streams"]
    row = hd * 2
    if c["kind"] == "rope":
        rows, size = n * c["nodes"], 2 if c["dtype"] == "fp16" else 4
        feats = (Hq + 2 * Hkv) * hd
        return {"bytes": rows * (feats * (size + 2) + 4 + Hkv * 8) + c["rotary"] // 2 * 8 + 4 * n,
                "flops": rows * (Hq + Hkv) * c["rotary"] * 3}
    if c["kind"] == "scored":
        T, P, R = c["nodes"], c["prefix"], c["nodes"] * Hq
        keys = sum(lens) + n * T
        return {"bytes": 2 * n * R * row + Hkv * (P + keys) * (2 * row + 8) + 4 * n * (T + 1),
                "flops": 4 * hd * R * (n * P + keys)}
    total = 0.0
    for s in lens:                                 # rows that move: the newest among those behind the budget, and their share
        tail = max(0, s - c["budget"])
        new = min(tail, c["recent"])
        moved = new + (tail - new) * (c["budget"] - c["recent"]) / max(1, s - c["recent"]) if tail else 0
        total += Hkv * (s * 8 + min(s, c["budget"]) * 8 + moved * 4 * row)
    return {"bytes": total + 12 * n, "flops": Hkv * sum(lens)}


# ----------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    c, st = case, prepare(case, seed)
    return _exact_rope(c, st) if c["kind"] == "rope" else _exact_scored(c, st) if c["kind"] == "scored" else _exact_evict(c, st)


def _exact_rope(c, st):
    """pairs as complex numbers, turned by exp(i * position * frequency)"""
    Hq, Hkv, hd = HEADS[c["heads"]]
    T, m = c["nodes"], c["rotary"] // 2
    turn = torch.polar(torch.full((), st["gain"], dtype=torch.float64, device="cuda"), st["positions"].double()[:, None, None] * st["freq"])
    first = torch.arange(m, device="cuda") * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else m)

    def turned(x, heads):
        x = x.double().reshape(-1, heads, hd)
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    k, v = turned(st["k"], Hkv), st["v"].double().reshape(-1, Hkv, hd)
    own_k, own_v = st["own_k"].double(), st["own_v"].double()
    weight, position = st["own_weight"].double(), st["own_position"].clone()
    for s, at in enumerate(st["lens"]):
        mine = slice(s * T, (s + 1) * T)
        own_k[s, :, at:at + T], own_v[s, :, at:at + T] = k[mine].transpose(0, 1), v[mine].transpose(0, 1)
        weight[s, :, at:at + T] = 0
        position[s, :, at:at + T] = st["positions"][mine]
    return {"q": turned(st["q"], Hq), "k": own_k, "v": own_v, "weight": weight, "position": position}


def _exact_scored(c, st):
    """stream by stream and KV head by KV head: an ordinary softmax over the keys one row after the other sees"""
    Hq, Hkv, hd = HEADS[c["heads"]]
    n, T, P, G = c["streams"], c["nodes"], c["prefix"], Hq // Hkv
    q = st["q"].double().view(n, T, Hkv, G, hd)
    out = torch.empty(n, T, Hkv, G, hd, dtype=torch.float64, device="cuda")
    weight = st["own_weight"].double()
    pw = st["prefix_weight"].double() if P else None
    sees = np.zeros((T, T), dtype=bool)
    for t in range(T):
        a = t
        while a >= 0:
            sees[t, a] = True
            a = st["parent"][a]
    for s in range(n):
        S = st["lens"][s]
        allowed = torch.from_numpy(np.concatenate([np.ones((T, P + S), dtype=bool), sees], axis=1)).cuda()[:, None]
        for h in range(Hkv):
            k, v = st["own_k"][s, h, :S + T].double(), st["own_v"][s, h, :S + T].double()
            if P:
                k, v = torch.cat([st["prefix_k"][h].double(), k]), torch.cat([st["prefix_v"][h].double(), v])
            e = torch.einsum("tgd,kd->tgk", q[s, :, h], k) / math.sqrt(hd)
            p = torch.softmax(torch.where(allowed, e, torch.full_like(e, -math.inf)), dim=-1)
            out[s, :, h] = torch.einsum("tgk,kd->tgd", p, v)
            p = p.sum(dim=(0, 1))
            weight[s, h, :S + T] += p[P:]
            if P:
                pw[h] += p[:P]
    return {"out": out.view(n * T, Hq, hd), "weight": weight, "prefix_weight": pw}


def _exact_evict(c, st):
    """one segment after the other, on the host"""
    B, R = c["budget"], c["recent"]
    k, v = st["own_k"].double(), st["own_v"].double()
    ow, op = st["out_weight"].double().cpu().numpy(), st["out_position"].cpu().numpy()
    w, pos = st["own_weight"].double().cpu().numpy(), st["own_position"].cpu().numpy()
    for s, S in enumerate(st["lens"]):
        for h in range(w.shape[1]):
            a, p = w[s, h, :S], pos[s, h, :S]
            kept = np.zeros(S, dtype=bool)
            kept[np.lexsort((np.arange(S), -a, ~(p > int(S - 1) - R)))[:B]] = True
            src = np.arange(min(S, B))
            src[~kept[:B]] = np.flatnonzero(kept[B:]) + B
            at = torch.from_numpy(src).cuda()
            k[s, h, :len(src)], v[s, h, :len(src)] = k[s, h][at], v[s, h][at]
            ow[s, h, :len(src)], op[s, h, :len(src)] = a[src], p[src]
    return {"k": k, "v": v, "weight": torch.from_numpy(ow), "position": torch.from_numpy(op),
            "len": torch.tensor([min(S, B) for S in st["lens"]], dtype=torch.int32)}
