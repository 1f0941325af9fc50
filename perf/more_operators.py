"""Cases for the operators of one decoding step with a tree of drafted tokens, and their plain forms.

The step: the drafted tokens' keys and values go to the pages of a cache (``cache_write``), the verifier attends
from every node of the tree to the cached context and to the node's own ancestors (``tree_attention``), its head
gives a row of logits for each node (``head_logits_int8``, whose weights ``quantize_rows`` has laid out), the tree is
verified against them (``tree_verify``) and the accepted path's entries move together in the cache
(``cache_compact``).

A case is a dict of plain values with a "kind":

  attn    tree_attention of one layer
  cache   cache_write in each of a stack of layers, and where "commit" is set cache_compact of all of them
  verify  tree_verify, with or without the draft's distributions
  int8    head_logits_int8 on bf16 or float32 hidden states
  quant   quantize_rows

Where ``own`` is false, ``run`` computes them from elementary torch operations; where it is true, it calls the
framework.
"""

import math

import torch

own = False

DEV = "cuda:0"
ABSENT = -2  # the parent of a node that a shorter tree does not have


def listed():
    return [
        # one token of one sequence on the 500M sub-model: the smallest call, launch latency
        {"name": "attn_single", "kind": "attn", "B": 1, "n": 1, "heads": 16, "kv_heads": 16, "D": 64, "ctx": 700,
         "page": 16, "dtype": "bf16"},
        # the middle sub-model's heads, the paper's batch and lengths (1,024-token prompts, up to 512 new tokens),
        # trees of up to 16 nodes
        {"name": "attn_tree_b102", "kind": "attn", "B": 102, "n": 16, "heads": 24, "kv_heads": 24, "D": 96,
         "ctx": 1536, "page": 16, "dtype": "bf16"},
        # a few long documents on the 3B sub-model's heads, trees of up to 32 nodes
        {"name": "attn_long", "kind": "attn", "B": 4, "n": 32, "heads": 34, "kv_heads": 34, "D": 128, "ctx": 65536,
         "page": 64, "dtype": "bf16"},
        # a small float32 model with shared heads (the development setting), odd batch and tree
        {"name": "attn_shared_f32", "kind": "attn", "B": 7, "n": 9, "heads": 12, "kv_heads": 3, "D": 64, "ctx": 900,
         "page": 32, "dtype": "f32"},
        # prompts of different lengths go to the pages of one layer
        {"name": "cache_prompts", "kind": "cache", "B": 8, "n": 1536, "layers": 1, "kv_heads": 24, "D": 96,
         "ctx": 0, "page": 16, "dtype": "bf16", "commit": False},
        # one step's trees in the 3B sub-model's last five layers, and the accepted paths moved together
        {"name": "cache_step_b102", "kind": "cache", "B": 102, "n": 16, "layers": 5, "kv_heads": 34, "D": 128,
         "ctx": 192, "page": 16, "dtype": "bf16", "commit": True},
        # one sequence, a tree of eight nodes: latency
        {"name": "verify_single", "kind": "verify", "B": 1, "n": 8, "V": 49152, "temperature": 0.4, "top_p": 0.9,
         "greedy": False, "draft": True},
        # the paper's batch and sampling settings, trees of up to 16 nodes
        {"name": "verify_b102", "kind": "verify", "B": 102, "n": 16, "V": 49152, "temperature": 0.4, "top_p": 0.9,
         "greedy": False, "draft": True},
        # one token on the 3B head: bound by the weights' bytes
        {"name": "int8_single", "kind": "int8", "T": 1, "d": 4352, "V": 49152, "dtype": "bf16"},
        # the verifier's rows of 102 trees of 16 nodes
        {"name": "int8_tree_b102", "kind": "int8", "T": 1632, "d": 4352, "V": 49152, "dtype": "bf16"},
        # the 3B head's weights, once when a server loads them
        {"name": "quant_head", "kind": "quant", "T": 49152, "d": 4352, "dtype": "bf16"},
        # odd float32 rows
        {"name": "quant_odd_f32", "kind": "quant", "T": 1531, "d": 1001, "dtype": "f32"},
    ]


# ---------------------------------------------------------------------------
# more cases of the same ranges
# ---------------------------------------------------------------------------

def _log(rng, lo, hi, step=1):
    """A whole number in [lo, hi], even over its logarithm, a multiple of step."""
    x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(x / step)) * step))


def _cache_bytes(c):
    return c["B"] * (c["ctx"] + c["n"]) * c["kv_heads"] * c["D"] * (2 if c["dtype"] == "bf16" else 4) * 2


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "cache", "verify", "verify", "int8", "int8", "quant"])
    if kind == "attn":
        c = {"kind": kind, "B": _log(rng, 1, 128), "n": _log(rng, 1, 64), "kv_heads": _log(rng, 1, 34),
             "D": rng.choice([32, 64, 96, 128, 192, 256]), "ctx": _log(rng, 1, 100000),
             "page": rng.choice([16, 32, 64, 256]), "dtype": rng.choice(["bf16", "bf16", "f32"])}
        c["heads"] = c["kv_heads"] * rng.choice([1, 1, 2, 4, 8])
        # both the cache's bytes and the rows that read it stay below the largest listed case's
        while _cache_bytes(c) * max(1, c["n"] * (c["heads"] // c["kv_heads"]) // 32) > (1 << 32) or \
                _cache_bytes(c) > (1 << 32):
            c["ctx"] = max(1, c["ctx"] // 2)
            c["B"] = max(1, c["B"] * 3 // 4)
        return c
    if kind == "cache":
        commit = rng.random() < 0.6
        c = {"kind": kind, "B": _log(rng, 1, 102), "n": _log(rng, 1, 64) if commit else _log(rng, 1, 4096),
             "layers": rng.randint(1, 6), "kv_heads": _log(rng, 1, 34), "D": rng.choice([32, 64, 96, 128, 256]),
             "ctx": _log(rng, 1, 1024), "page": rng.choice([16, 32, 64, 256]),
             "dtype": rng.choice(["bf16", "bf16", "f32"]), "commit": commit}
        while c["B"] * c["n"] > 16384 or c["layers"] * _cache_bytes(c) > (1 << 30):
            c["B"], c["ctx"] = max(1, c["B"] // 2), max(1, c["ctx"] // 2)
        return c
    if kind == "verify":
        greedy = rng.random() < 0.2
        c = {"kind": kind, "B": _log(rng, 1, 102), "n": _log(rng, 1, 64), "V": _log(rng, 1000, 65536),
             "temperature": rng.choice([0.4, 0.7, 1.0]), "top_p": rng.choice([0.9, 0.95, 1.0]), "greedy": greedy,
             "draft": not greedy and rng.random() < 0.7}
        while c["B"] * c["n"] * c["V"] > 102 * 16 * 49152:
            c["B"] = max(1, c["B"] // 2)
        return c
    if kind == "int8":
        c = {"kind": kind, "T": _log(rng, 1, 2048), "d": _log(rng, 256, 4352, rng.choice([16, 64, 128])),
             "V": _log(rng, 8000, 128256), "dtype": rng.choice(["bf16", "bf16", "f32"])}
        while c["T"] * c["d"] * c["V"] > 1632 * 4352 * 49152:
            c["T"] = max(1, c["T"] // 2)
        return c
    c = {"kind": kind, "T": _log(rng, 1, 65536), "d": _log(rng, 64, 8192), "dtype": rng.choice(["bf16", "f32"])}
    while c["T"] * c["d"] > 49152 * 4352 // 2:
        c["T"] //= 2
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _lengths(case, g):
    """Context lengths from two thirds of the largest up to it."""
    lo = case["ctx"] * 2 // 3
    x = lo + (torch.rand(case["B"], generator=g, device=DEV) * (case["ctx"] - lo + 1)).to(torch.int32)
    x[torch.randint(0, case["B"], (1,), generator=g, device=DEV)] = case["ctx"]
    return x.clamp_(max=case["ctx"]).to(torch.int32)


def _tree(B, n, g):
    """Parents of random trees (every earlier node is as likely), some with fewer nodes than n; node 0 is the last
    token that has been decided."""
    i = torch.arange(n, device=DEV)
    parents = (torch.rand(B, n, generator=g, device=DEV) * i).to(torch.int32)
    parents = torch.minimum(parents, (i - 1).clamp_(min=0).to(torch.int32))
    parents[:, 0] = -1
    nodes = n - (torch.rand(B, 1, generator=g, device=DEV) * torch.rand(B, 1, generator=g, device=DEV)
                 * (n // 2 + 1)).to(torch.int64)
    parents[i >= nodes] = ABSENT
    return parents.contiguous()


def _table(case, g):
    """Pages in no order, as a server that has run for a while hands them out, and a few that nobody has."""
    per = -(-(case["ctx"] + case["n"]) // case["page"])
    total = case["B"] * per + 3
    table = torch.randperm(total, generator=g, device=DEV)[:case["B"] * per].view(case["B"], per)
    return table.to(torch.int32).contiguous(), total


def _attn_inputs(case, seed):
    g, dt = _gen(seed), _dt(case["dtype"])
    table, total = _table(case, g)
    shape = (total, case["kv_heads"], case["page"], case["D"])
    kp = torch.randn(shape, generator=g, device=DEV, dtype=dt)
    vp = torch.randn(shape, generator=g, device=DEV, dtype=dt)
    # scores of a standard deviation near 2: a few entries carry a good part of a row
    q = (torch.randn(case["B"], case["n"], case["heads"], case["D"], generator=g, device=DEV) * 2.0).to(dt)
    return q, kp, vp, table, _lengths(case, g), _tree(case["B"], case["n"], g)


def _path(parents, g):
    """A path from the root down, as a verification gives it: (nodes [B, n], accepted [B])."""
    B, n = parents.shape
    path = torch.full((B, n), -1, dtype=torch.int32, device=DEV)
    at = torch.zeros(B, dtype=torch.int64, device=DEV)
    cur = torch.zeros(B, dtype=torch.int32, device=DEV)
    path[:, 0] = 0
    for i in range(1, n):
        take = (parents[:, i] == cur) & (torch.rand(B, generator=g, device=DEV) < 0.5)
        at += take
        cur = torch.where(take, torch.full_like(cur, i), cur)
        path.scatter_(1, at[:, None], cur[:, None])
    return path, at.to(torch.int32)


def _cache_inputs(case, seed):
    g, dt, L = _gen(seed), _dt(case["dtype"]), case["layers"]
    table, total = _table(case, g)
    shape = (L, total, case["kv_heads"], case["page"], case["D"])
    kp = torch.randn(shape, generator=g, device=DEV, dtype=dt)
    vp = torch.randn(shape, generator=g, device=DEV, dtype=dt)
    new = (L, case["B"], case["n"], case["kv_heads"], case["D"])
    k = torch.randn(new, generator=g, device=DEV, dtype=dt)
    v = torch.randn(new, generator=g, device=DEV, dtype=dt)
    lengths = _lengths(case, g)
    if case["commit"]:
        parents = _tree(case["B"], case["n"], g)
        counts = (parents != ABSENT).sum(1).to(torch.int32)
        path, accepted = _path(parents, g)
    else:
        # prompts from half of the longest up to it
        counts = (case["n"] - torch.rand(case["B"], generator=g, device=DEV) * (case["n"] // 2)).to(torch.int32)
        path = accepted = None
    return k, v, kp, vp, table, lengths, counts, path, accepted


def _verify_inputs(case, seed):
    g, B, n, V = _gen(seed), case["B"], case["n"], case["V"]
    parents = _tree(B, n, g)
    target = torch.randn(B, n, V, generator=g, device=DEV) * 2.0
    draft = target + 0.4 * torch.randn(B, n, V, generator=g, device=DEV)
    tokens = torch.randint(0, V, (B, n), generator=g, device=DEV)
    rows = torch.arange(B, device=DEV)
    for i in range(1, n):
        row = draft[rows, parents[:, i].clamp(min=0).long()] / case["temperature"]
        if case["draft"]:
            # a draw from the draft's softmax at the node's parent
            u = torch.rand(B, V, generator=g, device=DEV).clamp_(1e-9, 1.0 - 1e-7)
            tokens[:, i] = (row - torch.log(-torch.log(u))).argmax(1)
        else:
            # the draft's most likely tokens, the next one for each further child
            seen = ((parents[:, :i] == parents[:, i:i + 1]).sum(1) % min(4, V))[:, None]
            tokens[:, i] = row.topk(min(4, V), dim=1).indices.gather(1, seen)[:, 0]
    ua = torch.rand(B, n, generator=g, device=DEV)
    us = torch.rand(B, generator=g, device=DEV)
    return target, tokens.to(torch.int32), parents, ua, us, draft if case["draft"] else None


def _rows(case, g):
    """Hidden states with a few channels far above the others."""
    d = case["d"]
    channel = torch.ones(d, device=DEV)
    channel[torch.randperm(d, generator=g, device=DEV)[:max(1, d // 256)]] = 8.0
    return (torch.randn(case["T"], d, generator=g, device=DEV) * channel).to(_dt(case["dtype"]))


def _int8_inputs(case, seed):
    g = _gen(seed)
    o = _rows(case, g)
    W = torch.randint(-127, 128, (case["V"], case["d"]), generator=g, device=DEV, dtype=torch.int8)
    s = (0.5 + torch.rand(case["V"], generator=g, device=DEV)) * (3.0 * 0.02 / 127.0)
    return o, W, s


def _quant_inputs(case, seed):
    return _rows(case, _gen(seed))


def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case}
    if kind == "attn":
        s["q"], s["kp"], s["vp"], s["table"], s["len"], s["parents"] = _attn_inputs(case, seed)
    elif kind == "cache":
        (s["k"], s["v"], s["kp"], s["vp"], s["table"], s["len"], s["counts"], s["path"],
         s["accepted"]) = _cache_inputs(case, seed)
    elif kind == "verify":
        s["target"], s["tokens"], s["parents"], s["ua"], s["us"], s["draft"] = _verify_inputs(case, seed)
    elif kind == "int8":
        s["o"], s["W"], s["s"] = _int8_inputs(case, seed)
    else:
        s["x"] = _quant_inputs(case, seed)
    return s


# ---------------------------------------------------------------------------
# one pass: the framework's operators
# ---------------------------------------------------------------------------

def _run_own(s):
    from paper_2608_09703_amd import api

    c, kind = s["case"], s["case"]["kind"]
    if kind == "attn":
        return api.tree_attention(s["q"], s["kp"], s["vp"], s["table"], s["len"], s["parents"])
    if kind == "cache":
        for layer in range(c["layers"]):
            api.cache_write(s["k"][layer], s["v"][layer], s["kp"][layer], s["vp"][layer], s["table"], s["len"],
                            counts=s["counts"])
        if not c["commit"]:
            return [s["kp"], s["vp"]]
        new = api.cache_compact(s["kp"], s["vp"], s["table"], s["len"], s["path"], s["accepted"])
        return [s["kp"], s["vp"], new]
    if kind == "verify":
        return list(api.tree_verify(s["target"], s["tokens"], s["parents"], s["ua"], s["us"],
                                    draft_logits=s["draft"], temperature=c["temperature"], top_p=c["top_p"],
                                    greedy=c["greedy"]))
    if kind == "int8":
        return api.head_logits_int8(s["o"], s["W"], s["s"])
    q, scale = api.quantize_rows(s["x"])
    return [q * scale[:, None], scale]


# ---------------------------------------------------------------------------
# one pass: the plain forms
# ---------------------------------------------------------------------------

def _ancestors(parents):
    """[B, n, n]: whether node j is node i or above it, in a tree that has node i."""
    B, n = parents.shape
    anc = torch.zeros(B, n, n, dtype=torch.bool, device=DEV)
    rows = torch.arange(B, device=DEV)
    for i in range(n):
        p = parents[:, i]
        has = (p >= -1) & (p < i)
        above = anc[rows, p.clamp(min=0, max=max(i - 1, 0)).long()]
        linked = above.any(1)  # the parent is there
        up = (p >= 0)[:, None] & above
        anc[:, i] = up
        anc[:, i, i] = has & ((p == -1) | linked)
    return anc


def _plain_attn(s):
    c = s["case"]
    B, n, H, D, Hk = c["B"], c["n"], c["heads"], c["D"], c["kv_heads"]
    g = H // Hk
    per = s["table"].shape[1]
    S = per * c["page"]
    out = torch.zeros(B, n, H, D, device=DEV)
    anc = _ancestors(s["parents"])
    t = torch.arange(S, device=DEV)
    step = max(1, (1 << 30) // (S * Hk * D))
    for b in range(0, B, step):
        e = min(B, b + step)
        idx = s["table"][b:e].long()
        k = s["kp"][idx].float().permute(0, 2, 1, 3, 4).reshape((e - b) * Hk, S, D)
        v = s["vp"][idx].float().permute(0, 2, 1, 3, 4).reshape((e - b) * Hk, S, D)
        q = s["q"][b:e].float().view(e - b, n, Hk, g, D).permute(0, 2, 1, 3, 4).reshape((e - b) * Hk, n * g, D)
        ctx = s["len"][b:e].long()[:, None, None]
        node = t[None, None, :] - ctx
        see = (node < 0).expand(e - b, n, S) | \
            (anc[b:e].gather(2, node.clamp(0, n - 1).expand(e - b, n, S)) & (node >= 0) & (node < n))
        see = see & anc[b:e].any(2)[:, :, None]
        see = see[:, None, :, None, :].expand(e - b, Hk, n, g, S).reshape((e - b) * Hk, n * g, S)
        z = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(D))
        z = torch.where(see, z, torch.full((), -math.inf, device=DEV))
        m = z.max(2, keepdim=True).values
        m = torch.where(m > -math.inf, m, torch.zeros_like(m))
        p = torch.exp(z - m)
        tot = p.sum(2, keepdim=True)
        o = torch.matmul(p, v) / torch.where(tot > 0, tot, torch.ones_like(tot))
        out[b:e] = o.view(e - b, Hk, n, g, D).permute(0, 2, 1, 3, 4).reshape(e - b, n, H, D)
    return out.to(s["q"].dtype)


def _slots(s, position):
    """(page, entry in it) of positions [B, m]."""
    page = s["case"]["page"]
    return s["table"].gather(1, (position // page)).long(), position % page


def _plain_cache(s):
    c = s["case"]
    n = c["n"]
    i = torch.arange(n, device=DEV)[None, :].expand(c["B"], n)
    page, entry = _slots(s, s["len"].long()[:, None] + i)
    keep = i < s["counts"][:, None]
    for layer in range(c["layers"]):
        s["kp"][layer].permute(0, 2, 1, 3)[page[keep], entry[keep]] = s["k"][layer][keep]
        s["vp"][layer].permute(0, 2, 1, 3)[page[keep], entry[keep]] = s["v"][layer][keep]
    if not c["commit"]:
        return [s["kp"], s["vp"]]
    taken = i <= s["accepted"][:, None]
    src, src_at = _slots(s, s["len"].long()[:, None] + s["path"].clamp(min=0).long())
    for pool in (s["kp"], s["vp"]):
        rows = pool.permute(0, 1, 3, 2, 4)
        moved = rows[:, src[taken], src_at[taken]]
        rows[:, page[taken], entry[taken]] = moved
    return [s["kp"], s["vp"], s["len"] + s["accepted"] + 1]


def _single(x):
    """A sampling setting as the float32 number that a sampler's settings hold."""
    return float(torch.tensor(x, dtype=torch.float32))


def _plain_probs(rows, temperature, top_p):
    """Sampling distributions in 64 bits: a draw must not depend on a rounding."""
    temperature, top_p = _single(temperature), _single(top_p)
    z = rows.double() / temperature
    e = torch.exp(z - z.max(1, keepdim=True).values)
    p = e / e.sum(1, keepdim=True)
    if top_p >= 1.0:
        return p
    val, at = torch.sort(p, dim=1, descending=True, stable=True)
    before = torch.cumsum(val, 1) - val
    kept = torch.zeros_like(p).scatter_(1, at, torch.where(before < top_p, val, torch.zeros_like(val)))
    return kept / kept.sum(1, keepdim=True)


def _plain_verify(s):
    c = s["case"]
    B, n, V = c["B"], c["n"], c["V"]
    rows = torch.arange(B, device=DEV)
    tokens, parents = s["tokens"].long(), s["parents"].long()
    cur = torch.zeros(B, dtype=torch.int64, device=DEV)
    depth = torch.zeros_like(cur)
    path = torch.full((B, n), -1, dtype=torch.int64, device=DEV)
    path[:, 0] = 0
    temperature, top_p = c["temperature"], c["top_p"]

    def dist(logits, node):
        return _plain_probs(logits[rows, node], temperature, top_p)

    best = r = q = None
    if c["greedy"]:
        best = s["target"].max(2).values[:, :, None] == s["target"]
        best = torch.where(best, torch.arange(V, device=DEV), torch.full((), V, device=DEV)).min(2).values
    else:
        r = dist(s["target"], cur)
        q = dist(s["draft"], cur) if c["draft"] else None
    for i in range(1, n):
        here = parents[:, i] == cur
        x = tokens[:, i]
        if c["greedy"]:
            ok = here & (best[rows, cur] == x)
        else:
            qx = q[rows, x] if c["draft"] else torch.ones(B, dtype=torch.float64, device=DEV)
            ok = here & (s["ua"][:, i].double() * qx < r[rows, x])
            left = (r - q).clamp(min=0.0) if c["draft"] else r.scatter(1, x[:, None], 0.0)
            tot = left.sum(1, keepdim=True)
            left = torch.where(tot > 0, left / torch.where(tot > 0, tot, torch.ones_like(tot)), r)
            r = torch.where((here & ~ok)[:, None], left, r)
        depth += ok
        cur = torch.where(ok, torch.full_like(cur, i), cur)
        path.scatter_(1, depth[:, None], cur[:, None])
        if not c["greedy"]:
            r = torch.where(ok[:, None], dist(s["target"], cur), r)
            q = torch.where(ok[:, None], dist(s["draft"], cur), q) if c["draft"] else None
    if c["greedy"]:
        nxt = best[rows, cur]
    else:
        cum = torch.cumsum(r, 1)
        nxt = (cum <= s["us"].double()[:, None] * cum[:, -1:]).sum(1)
    return [depth.to(torch.int32), path.to(torch.int32), nxt.to(torch.int32)]


def _plain_quantize(x):
    x = x.float()
    # in 64 bits: values next to the middle between two numbers
    scale = (x.abs().max(1, keepdim=True).values.double() / 127.0).float()
    q = torch.round(x.double() / torch.where(scale > 0, scale, torch.ones_like(scale)).double())
    return q.clamp(-127.0, 127.0).float(), scale


def _plain_int8(s):
    q, scale = _plain_quantize(s["o"])
    # sums of whole numbers past 2^24: in parts that 32 bits hold exactly
    z = torch.zeros(s["case"]["T"], s["case"]["V"], device=DEV)
    for k in range(0, s["case"]["d"], 1024):
        z += torch.matmul(q[:, k:k + 1024], s["W"][:, k:k + 1024].float().t())
    return z * scale * s["s"][None, :]


def _plain_quant(s):
    q, scale = _plain_quantize(s["x"])
    return [q * scale, scale[:, 0]]


def run(state):
    if own:
        return _run_own(state)
    return {"attn": _plain_attn, "cache": _plain_cache, "verify": _plain_verify, "int8": _plain_int8,
            "quant": _plain_quant}[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind, es = case["kind"], 2 if case.get("dtype") == "bf16" else 4
    if kind == "attn":
        # lengths lie between two thirds of the largest and the largest
        entries = case["B"] * (case["ctx"] * 5 // 6 + case["n"])
        q = case["B"] * case["n"] * case["heads"] * case["D"]
        return {"bytes": 2 * entries * case["kv_heads"] * case["D"] * es + 2 * q * es,
                "flops": 4 * entries * case["n"] * case["heads"] * case["D"]}
    if kind == "cache":
        entry = 2 * case["kv_heads"] * case["D"] * es * case["layers"]
        if not case["commit"]:
            return {"bytes": 2 * case["B"] * (case["n"] * 3 // 4) * entry, "flops": 0}
        # written once, and an accepted node or two moved
        return {"bytes": 2 * case["B"] * (case["n"] * 7 // 8 + 2) * entry, "flops": 0}
    if kind == "verify":
        # the distributions at the root and at one accepted node
        rows = case["B"] * min(2, case["n"]) * (2 if case["draft"] else 1)
        return {"bytes": rows * case["V"] * 4, "flops": rows * case["V"] * 8}
    if kind == "int8":
        T, d, V = case["T"], case["d"], case["V"]
        return {"bytes": T * d * es + V * d + 4 * V + 4 * T * V, "flops": 2 * T * d * V}
    n = case["T"] * case["d"]
    return {"bytes": n * es + n + 4 * case["T"], "flops": 4 * n}


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------

def _exact_attn(case, seed):
    q, kp, vp, table, lengths, parents = _attn_inputs(case, seed)
    B, n, H, D, Hk, page = case["B"], case["n"], case["heads"], case["D"], case["kv_heads"], case["page"]
    g = H // Hk
    out = torch.zeros(B, n, H, D, dtype=torch.float64, device=DEV)
    par, lens = parents.tolist(), lengths.tolist()
    for b in range(B):
        ctx = lens[b]
        sees = torch.zeros(n, ctx + n, dtype=torch.bool)
        for i in range(n):
            up, chain = i, []
            while up >= 0:
                chain.append(up)
                nxt = par[b][up]
                if nxt < -1 or nxt >= up:
                    chain = None
                    break
                up = nxt
            if chain is not None:
                sees[i, :ctx] = True
                sees[i, [ctx + x for x in chain]] = True
        sees = sees.to(DEV)
        pages = table[b, :-(-(ctx + n) // page)].long()
        for h in range(Hk):
            k = kp[pages, h].reshape(-1, D)[:ctx + n].double()
            v = vp[pages, h].reshape(-1, D)[:ctx + n].double()
            z = q[b, :, h * g:(h + 1) * g].double().reshape(n * g, D).mm(k.t()) / math.sqrt(D)
            z = z.view(n, g, -1).masked_fill(~sees[:, None, :], -math.inf)
            p = torch.softmax(z, dim=2).masked_fill(~sees.any(1)[:, None, None], 0.0)
            out[b, :, h * g:(h + 1) * g] = p.view(n * g, -1).mm(v).view(n, g, D)
    return out


def _exact_cache(case, seed):
    k, v, kp, vp, table, lengths, counts, path, accepted = _cache_inputs(case, seed)
    if case["B"] * case["n"] > 20000:
        return None
    lens, cnt, tab, page = lengths.tolist(), counts.tolist(), table.tolist(), case["page"]
    for new, pool in ((k, kp), (v, vp)):
        for b in range(case["B"]):
            at = [lens[b] + i for i in range(cnt[b])]
            pg = torch.tensor([tab[b][p // page] for p in at], device=DEV)
            en = torch.tensor([p % page for p in at], device=DEV)
            pool[:, pg, :, en] = new[:, b, :cnt[b]].transpose(0, 1)
            if path is not None:
                for j, node in enumerate(path[b, :int(accepted[b]) + 1].tolist()):
                    src, dst = lens[b] + node, lens[b] + j
                    pool[:, tab[b][dst // page], :, dst % page] = pool[:, tab[b][src // page], :, src % page]
    if path is None:
        return [kp.double(), vp.double()]
    return [kp.double(), vp.double(), lengths + accepted + 1]


def _exact_probs(row, temperature, top_p):
    temperature, top_p = _single(temperature), _single(top_p)
    p = torch.softmax(row.double() / temperature, 0)
    if top_p < 1.0:
        val, at = torch.sort(-p, stable=True)
        reached = torch.cumsum(-val, 0) >= top_p
        last = int(torch.nonzero(reached)[0]) if bool(reached.any()) else p.numel() - 1
        drop = at[last + 1:]
        p[drop] = 0.0
        p = p / p.sum()
    return p


def _exact_verify(case, seed):
    target, tokens, parents, ua, us, draft = _verify_inputs(case, seed)
    B, n = case["B"], case["n"]
    tok, par, ua, us = tokens.tolist(), parents.tolist(), ua.tolist(), us.tolist()
    depth, paths, nxt = [], [], []
    for b in range(B):
        path = [0]
        while True:
            node = path[-1]
            children = [i for i in range(node + 1, n) if par[b][i] == node]
            if case["greedy"]:
                y = int(torch.nonzero(target[b, node] == target[b, node].max())[0])
                taken = next((i for i in children if tok[b][i] == y), None)
            else:
                p = _exact_probs(target[b, node], case["temperature"], case["top_p"])
                q = None
                taken = None
                for i in children:
                    x = tok[b][i]
                    if q is None:
                        q = _exact_probs(draft[b, node], case["temperature"], case["top_p"]) if case["draft"] else 0
                    qx = float(q[x]) if case["draft"] else 1.0
                    if ua[b][i] * qx < float(p[x]):
                        taken = i
                        break
                    if case["draft"]:
                        left = torch.relu(p - q)
                    else:
                        left = p.clone()
                        left[x] = 0.0
                    if float(left.sum()) > 0.0:
                        p = left / left.sum()
                if taken is None:
                    cum = torch.cumsum(p, 0)
                    y = int(torch.searchsorted(cum, us[b] * cum[-1], right=True))
            if taken is None:
                break
            path.append(taken)
        depth.append(len(path) - 1)
        paths.append(path + [-1] * (n - len(path)))
        nxt.append(y)
    return [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (depth, paths, nxt)]


def _exact_quantize(x):
    # the scale is the float32 number next to the largest magnitude over 127
    scale = (x.abs().amax(1).double() / 127.0).float().double()[:, None]
    steps = x.double() / scale.masked_fill(scale == 0.0, 1.0)
    return steps.round().clamp(-127.0, 127.0), scale


def _exact_int8(case, seed):
    o, W, s = _int8_inputs(case, seed)
    q, scale = _exact_quantize(o)
    out = torch.empty(case["T"], case["V"], dtype=torch.float64, device=DEV)
    for v in range(0, case["V"], 16384):
        out[:, v:v + 16384] = q.mm(W[v:v + 16384].double().t()) * scale * s[v:v + 16384].double()
    return out


def _exact_quant(case, seed):
    q, scale = _exact_quantize(_quant_inputs(case, seed))
    return [q * scale, scale[:, 0]]


def exact(case, seed):
    return {"attn": _exact_attn, "cache": _exact_cache, "verify": _exact_verify, "int8": _exact_int8,
            "quant": _exact_quant}[case["kind"]](case, seed)
