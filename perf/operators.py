"""The operators around a verification, as measured workloads with their plain forms.

Between one verification and the next, a server of tree speculative decoding attends from every tree
node to the request's paged cache and to the node's ancestors (``attention``), applies penalties,
biases and grammar masks to the LM head's logits and renews their row statistics (``logits``), grows
the requests by the accepted tokens (``extend``: pages, block tables, slots) and writes those tokens'
keys and values into the cache (``commit``).

``run`` computes each in elementary torch operations, or with ``own`` through the framework.
"""

import math

import numpy as np
import torch

own = False


def _attention(name, batch, nodes, depth, heads, kv_heads, head_dim, ctx_lo, ctx_hi, page,
               dtype="bf16", prefix=0):
    return {"name": name, "kind": "attention", "batch": batch, "nodes": nodes, "depth": depth,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "page": page, "dtype": dtype, "prefix": prefix}


def _logits(name, batch, nodes, depth, vocab, hist_lo, hist_hi, bias, masks, dtype="bf16",
            temperature=1.0):
    return {"name": name, "kind": "logits", "batch": batch, "nodes": nodes, "depth": depth,
            "vocab": vocab, "hist_lo": hist_lo, "hist_hi": hist_hi, "bias": bias, "masks": masks,
            "dtype": dtype, "temperature": temperature}


def _extend(name, batch, seq_lo, seq_hi, max_new, page):
    return {"name": name, "kind": "extend", "batch": batch, "seq_lo": seq_lo, "seq_hi": seq_hi,
            "max_new": max_new, "page": page}


def _commit(name, batch, nodes, depth, layers, kv_heads, head_dim, page, dtype="bf16"):
    return {"name": name, "kind": "commit", "batch": batch, "nodes": nodes, "depth": depth,
            "layers": layers, "kv_heads": kv_heads, "head_dim": head_dim, "page": page,
            "dtype": dtype}


def listed():
    """``nodes`` counts the drafted nodes: a tree has one more, its root."""
    return [
        # one user: a tree of 64 draft nodes on a short conversation, where latency counts
        _attention("attention-tree-1", 1, 64, 7, 32, 8, 128, 1000, 1000, 16),
        # a full server batch of such trees with contexts of 1000 to 2900 tokens
        _attention("attention-tree-256", 256, 64, 7, 32, 8, 128, 1000, 2900, 64),
        # plain decoding, a token a request: one pass over long caches
        _attention("attention-token-64", 64, 0, 0, 32, 8, 128, 2000, 10000, 32),
        # plain decoding behind a system prompt that all requests share
        _attention("attention-prefix-256", 256, 0, 0, 32, 8, 128, 8242, 8800, 64, prefix=8192),
        # two very long documents, single-chain drafting, a key head per query head, fp16
        _attention("attention-chain-f16-2", 2, 5, 5, 16, 16, 64, 60001, 99999, 128, dtype="f16"),
        # the target's logits of a full batch: penalties over the history and the drafted path
        _logits("logits-256", 256, 64, 7, 128256, 500, 4000, 0, 0),
        # one user's tree
        _logits("logits-1", 1, 64, 7, 128256, 1000, 1000, 16, 0),
        # structured output: a grammar mask at every node, fp32 logits, an odd vocabulary
        _logits("logits-mask-f32-16", 16, 40, 6, 32003, 100, 1000, 16, 64, dtype="f32",
                temperature=0.7),
        # a decoding cycle's growth of a full batch
        _extend("extend-256", 256, 100, 8000, 8, 16),
        # prompts that enter the cache together
        _extend("extend-prompts-32", 32, 0, 0, 8000, 16),
        # the accepted nodes of a full batch, all layers
        _commit("commit-256", 256, 64, 7, 32, 8, 128, 16),
        # those of one tree
        _commit("commit-1", 1, 64, 7, 32, 8, 128, 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attention", "attention", "attention", "logits", "logits", "extend",
                       "commit"))
    if kind == "attention":
        heads, kv_heads = rng.choice(((32, 8), (32, 32), (16, 2), (8, 1), (40, 8), (64, 8)))
        shape = rng.choice(("token", "chain", "tree", "tree"))
        depth = {"token": 0, "chain": rng.randint(2, 8), "tree": rng.randint(6, 8)}[shape]
        nodes = {"token": 0, "chain": depth, "tree": _log_int(rng, 12, 200)}[shape]
        ctx = _log_int(rng, 32, 40000)
        hi = ctx + rng.randint(0, ctx // 2)
        # at most the keys, the scores and the heads' keys of the largest listed cases
        most = min(500000 // hi, 17_000_000 * 64 // (heads * hi * (nodes + 1)),
                   4_000_000 // (kv_heads * hi))
        batch = _log_int(rng, 1, max(1, min(256, most)))
        page = rng.choice((16, 32, 64, 128))
        prefix = ctx // page // 2 * page if rng.random() < 0.3 else 0
        c = _attention("", batch, nodes, depth, heads, kv_heads, rng.choice((64, 80, 96, 128, 128)),
                       ctx, hi, page, rng.choice(("bf16", "bf16", "f16")), prefix)
    elif kind == "logits":
        vocab = rng.choice((32000, 32003, 50257, 128256, 151936))
        nodes = rng.choice((0, rng.randint(2, 8), rng.randint(12, 100)))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        batch = _log_int(rng, 1, max(1, min(256, 1_000_000_000 // ((nodes + 1) * vocab))))
        hist = _log_int(rng, 8, 8000)
        c = _logits("", batch, nodes, min(nodes, rng.randint(5, 8)), vocab, hist // 2, hist,
                    rng.choice((0, 7, 100)), rng.choice((0, 1, 32)), dtype,
                    rng.choice((1.0, 0.7, 1.3)))
    elif kind == "extend":
        hi = _log_int(rng, 1, 4000)
        c = _extend("", _log_int(rng, 1, 500), 0, _log_int(rng, 1, 8000), hi,
                    rng.choice((16, 32, 64, 128)))
    else:
        nodes = rng.randint(4, 80)
        c = _commit("", _log_int(rng, 1, 256), nodes, min(nodes, rng.randint(4, 8)),
                    rng.randint(1, 32), rng.choice((1, 2, 8)), rng.choice((64, 96, 128)),
                    rng.choice((16, 32, 64)), rng.choice(("bf16", "f16")))
    return {k: v for k, v in c.items() if k != "name"}


# --- inputs ------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_DEV = "cuda"


def _parents(case, seed):
    """Random trees, breadth first: a chain where the depth takes all nodes, else each node under
    one of the nodes of the level before."""
    rng = np.random.default_rng([seed & 0x7FFFFFFF, 1])
    B, n, depth = case["batch"], case["nodes"], case["depth"]
    par = np.full((B, n + 1), -1, np.int32)
    for b in range(B):
        if depth >= n:
            par[b, 1:] = np.arange(n)
            continue
        # one node at least on each level, the rest spread at random
        extra = rng.multinomial(n - depth, np.full(depth, 1.0 / depth))
        before, at = np.zeros(1, np.int64), 1
        for width in (1 + extra).tolist():
            par[b, at:at + width] = np.sort(rng.choice(before, width))
            before, at = np.arange(at, at + width), at + width
    return par


def _prepare_attention(c, seed, g):
    B, n1, H, KH, D, ps = (c["batch"], c["nodes"] + 1, c["heads"], c["kv_heads"], c["head_dim"],
                           c["page"])
    dt = _TYPES[c["dtype"]]
    rng = np.random.default_rng([seed & 0x7FFFFFFF, 2])
    ctx = rng.integers(c["ctx_lo"], c["ctx_hi"] + 1, B)
    ctx[0] = c["ctx_hi"]
    width = -(-int(c["ctx_hi"]) // ps) + 2
    shared = c["prefix"] // ps
    need = -(-ctx // ps) - shared
    pages = shared + int(need.sum()) + 8
    order = rng.permutation(pages)
    table = np.full((B, width), -1, np.int32)
    table[:, :shared] = order[:shared]
    at = shared
    for b in range(B):
        table[b, shared:shared + need[b]] = order[at:at + need[b]]
        at += need[b]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device=_DEV) * scale).to(dt)

    k_cache, v_cache = (torch.empty((pages, KH, ps, D), dtype=dt, device=_DEV) for _ in range(2))
    step = max(1, (1 << 28) // (KH * ps * D))
    for t in (k_cache, v_cache):
        for p in range(0, pages, step):
            t[p:p + step] = torch.randn(t[p:p + step].shape, generator=g, device=_DEV)
    # the projection's output, queries, keys and values of a node in one row
    qkv = normal(B, n1, H + 2 * KH, D)
    qkv[:, :, :H] *= 2
    return {"q": qkv[:, :, :H], "k_new": qkv[:, :, H:H + KH], "v_new": qkv[:, :, H + KH:],
            "parents": torch.as_tensor(_parents(c, seed), device=_DEV), "k_cache": k_cache,
            "v_cache": v_cache, "block_table": torch.as_tensor(table, device=_DEV),
            "ctx_len": torch.as_tensor(ctx.astype(np.int32), device=_DEV),
            "scale": 1.0 / math.sqrt(D)}


def _prepare_logits(c, seed, g):
    B, n1, V = c["batch"], c["nodes"] + 1, c["vocab"]
    dt = _TYPES[c["dtype"]]
    z = torch.empty((B, n1, V), dtype=dt, device=_DEV)
    step = max(1, (1 << 28) // (n1 * V))
    for b in range(0, B, step):
        x = torch.randn(z[b:b + step].shape, generator=g, device=_DEV).mul_(3.0)
        x += 6.0 * (torch.rand(x.shape, generator=g, device=_DEV) < 0.01)
        z[b:b + step] = x
        del x

    def rand(*shape):
        return torch.rand(shape, generator=g, device=_DEV)

    # token ids that repeat as words do: low ids often, high ones rarely
    def ids(*shape):
        return (V * rand(*shape) ** 3).to(torch.int32).clamp_(max=V - 1)

    hist = torch.randint(c["hist_lo"], c["hist_hi"] + 1, (B,), generator=g, device=_DEV)
    s = {"logits": z, "out": torch.empty_like(z), "temperature": c["temperature"],
         "parents": torch.as_tensor(_parents(c, seed), device=_DEV), "tokens": ids(B, n1),
         "history": ids(B, c["hist_hi"]), "history_len": hist.to(torch.int32),
         "prompt_len": (hist * rand(B)).to(torch.int32), "repetition": 1.0 + 0.3 * rand(B),
         "presence": 0.5 * rand(B), "frequency": 0.5 * rand(B), "bias_tokens": None,
         "bias_values": None, "masks": None, "mask_index": None}
    if c["bias"]:
        # distinct tokens, a few of them banned
        first = torch.randint(0, V, (B, 1), generator=g, device=_DEV)
        s["bias_tokens"] = ((first + 211 * torch.arange(c["bias"], device=_DEV)) % V).to(torch.int32)
        x = 4.0 * torch.randn((B, c["bias"]), generator=g, device=_DEV)
        s["bias_values"] = torch.where(rand(B, c["bias"]) < 0.2, -math.inf, x)
    if c["masks"]:
        words = (V + 31) // 32
        m = torch.randint(-2 ** 31, 2 ** 31, (c["masks"], words), generator=g, device=_DEV)
        m &= torch.randint(-2 ** 31, 2 ** 31, (c["masks"], words), generator=g, device=_DEV)
        s["masks"] = m.to(torch.int32)
        s["mask_index"] = torch.randint(-1, c["masks"], (B, n1), generator=g,
                                        device=_DEV).to(torch.int32)
    return s


def _prepare_extend(c, seed, g):
    B, ps, most = c["batch"], c["page"], c["max_new"]
    rng = np.random.default_rng([seed & 0x7FFFFFFF, 3])
    seq = rng.integers(c["seq_lo"], c["seq_hi"] + 1, B)
    new = rng.integers(min(1, most), most + 1, B)
    held = -(-seq // ps)
    need = -(-(seq + new) // ps) - held
    width = -(-(c["seq_hi"] + most) // ps)
    pages = int(held.sum() + need.sum()) + 64
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((B, width), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    free = np.full(pages, -1, np.int32)
    free[:pages - at] = order[at:]
    i32 = [torch.as_tensor(np.asarray(x, np.int32), device=_DEV)
           for x in (new, seq, table, free, [pages - at])]
    return dict(zip(("new_len", "seq_len", "block_table", "free_pages", "free_count"), i32),
                page_size=ps, max_new=most)


def _prepare_commit(c, seed, g):
    B, n1, L, KH, D, ps = (c["batch"], c["nodes"] + 1, c["layers"], c["kv_heads"], c["head_dim"],
                           c["page"])
    dt = _TYPES[c["dtype"]]
    rng = np.random.default_rng([seed & 0x7FFFFFFF, 4])
    par = _parents(c, seed)
    pages = 32768 // ps
    k, v = (torch.empty((L, B, n1, KH, D), dtype=dt, device=_DEV) for _ in range(2))
    kc, vc = (torch.empty((L, pages, KH, ps, D), dtype=dt, device=_DEV) for _ in range(2))
    for t in (k, v, kc, vc):
        for i in range(L):
            t[i] = torch.randn(t[i].shape, generator=g, device=_DEV)
    path = np.full((B, c["depth"]), -1, np.int32)
    length = np.zeros(B, np.int32)
    slots = np.full((B, c["depth"] + 1), -1, np.int32)
    room = 32768 // B
    for b in range(B):
        x, chain = int(rng.integers(0, n1)), []
        while x > 0:
            chain.append(x)
            x = int(par[b, x])
        path[b, :len(chain)] = chain[::-1]
        length[b] = len(chain) + 1
        first = b * room + int(rng.integers(0, room - length[b] + 1))
        slots[b, :length[b]] = np.arange(first, first + length[b])
    i32 = [torch.as_tensor(x, device=_DEV) for x in (path, length, slots)]
    return dict(zip(("path_nodes", "new_len", "slots"), i32), k_new=k, v_new=v, k_cache=kc,
                v_cache=vc)


def prepare(case, seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(seed)
    make = {"attention": _prepare_attention, "logits": _prepare_logits, "extend": _prepare_extend,
            "commit": _prepare_commit}[case["kind"]]
    return dict(make(case, seed, g), case=case)


# --- plain forms -------------------------------------------------------------


def _reach(parents):
    """[B, i, j]: whether node j is i or an ancestor of i (the links' matrix summed over all its
    powers; every sum is 0 or 1)."""
    n1 = parents.shape[1]
    node = torch.arange(n1, device=parents.device)
    link = (parents.unsqueeze(-1) == node).to(torch.float32)
    eye = torch.eye(n1, device=parents.device).expand_as(link)
    return torch.linalg.solve_triangular(eye - link, eye, upper=False, unitriangular=True) > 0.5


def _plain_attention(s):
    q, kn, vn, kc, vc = s["q"], s["k_new"], s["v_new"], s["k_cache"], s["v_cache"]
    B, n1, H, D = q.shape
    KH, ps = kc.shape[1], kc.shape[2]
    table = s["block_table"].clamp(min=0).long()
    L = table.shape[1] * ps
    at = torch.arange(L, device=q.device)
    cached = at < s["ctx_len"].unsqueeze(-1)                          # [B, L]
    see = torch.cat([cached.unsqueeze(1).expand(B, n1, L), _reach(s["parents"])], dim=-1)

    def keys(cache, new):
        old = cache[table].to(torch.float32).transpose(1, 2).reshape(B, KH, L, D)
        old = old.masked_fill_(~cached[:, None, :, None], 0.0)
        return torch.cat([old, new.to(torch.float32).transpose(1, 2)], dim=2)

    qf = q.to(torch.float32).reshape(B, n1, KH, H // KH, D).permute(0, 2, 3, 1, 4)
    qf = qf.reshape(B, KH, H // KH * n1, D)
    p = torch.matmul(qf, keys(kc, kn).transpose(-1, -2)).mul_(s["scale"])
    p = p.view(B, KH, H // KH, n1, L + n1).masked_fill_(~see[:, None, None], -math.inf)
    p = p.sub_(p.amax(dim=-1, keepdim=True)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(B, KH, H // KH * n1, L + n1), keys(vc, vn))
    o = o.view(B, KH, H // KH, n1, D) / total
    return o.permute(0, 3, 1, 2, 4).reshape(B, n1, H, D).to(q.dtype)


def _counts(ids, valid, V):
    """[..., V]: how often each token occurs among the valid ones of the last dimension."""
    n = torch.zeros(ids.shape[:-1] + (V,), dtype=torch.float32, device=ids.device)
    return n.scatter_add_(-1, ids.long(), valid.to(torch.float32))


def _plain_logits(s):
    z, hist, T = s["logits"], s["history"], s["temperature"]
    B, n1, V = z.shape
    at = torch.arange(hist.shape[1], device=z.device)
    past = at < s["history_len"].unsqueeze(-1)
    prompt = at < s["prompt_len"].unsqueeze(-1)
    told = _counts(hist, prompt & past, V) > 0                         # [B, V]
    made = _counts(hist, past & ~prompt, V)
    path = _reach(s["parents"])
    path[:, :, 0] = False                                              # the root is in the history
    n = _counts(s["tokens"].unsqueeze(1).expand(B, n1, n1), path, V) + made.unsqueeze(1)
    x = z.to(torch.float32)
    rho, alpha, beta = (s[k].view(B, 1, 1) for k in ("repetition", "presence", "frequency"))
    x = torch.where(told.unsqueeze(1) | (n > 0), torch.where(x > 0, x / rho, x * rho), x)
    less = alpha * (n > 0) + beta * n
    del n
    if s["bias_tokens"] is not None:
        bias = torch.zeros((B, V), device=z.device)
        bias.scatter_(-1, s["bias_tokens"].long(), s["bias_values"])
        less -= bias.unsqueeze(1)
    x = x - less
    del less
    if s["masks"] is not None:
        bit = torch.arange(32, device=z.device, dtype=torch.int32)
        allowed = (s["masks"].unsqueeze(-1) >> bit & 1).flatten(1)[:, :V] > 0
        which = s["mask_index"].long()
        x = torch.where(allowed[which.clamp(min=0)] | (which < 0).unsqueeze(-1), x, -math.inf)
    out = s["out"].copy_(x)
    del x
    top = out.amax(dim=-1).to(torch.float32)
    # terms of a value less than its row's maximum: 32 bits hold each, a row's sum is kept in 64
    e = (out.to(torch.float32) - top.unsqueeze(-1)).mul_(1.0 / T).exp_()
    return {"logits": out, "row_max": top,
            "row_sum": e.sum(dim=-1, dtype=torch.float64).to(torch.float32)}


def _plain_extend(s):
    new, seq, ps, most = s["new_len"].long(), s["seq_len"].long(), s["page_size"], s["max_new"]
    table, free = s["block_table"], s["free_pages"]
    B, width = table.shape
    held, want = (seq + ps - 1) // ps, (seq + new + ps - 1) // ps
    need = want - held
    upto = need.cumsum(0)
    total = s["free_count"].long()
    fine = upto <= total
    # page j of request b: its own, or from the top of the free pages
    j = torch.arange(width, device=new.device)
    from_top = total - 1 - (upto - need).unsqueeze(-1) - (j - held.unsqueeze(-1))
    fresh = (j >= held.unsqueeze(-1)) & (j < want.unsqueeze(-1)) & fine.unsqueeze(-1)
    table.copy_(torch.where(fresh, free[from_top.clamp(0, free.shape[0] - 1)], table))
    k = torch.arange(most, device=new.device)
    at = seq.unsqueeze(-1) + k
    page = table.gather(1, (at // ps).clamp(max=width - 1)).long()
    slots = torch.where((k < new.unsqueeze(-1)) & fine.unsqueeze(-1), page * ps + at % ps, -1)
    return {"slots": slots.to(torch.int32), "block_table": table,
            "seq_len": torch.where(fine, seq + new, seq).to(torch.int32),
            "free_count": (total - torch.where(fine, need, 0).sum()).to(torch.int32),
            "status": (~fine).to(torch.int32)}


def _plain_commit(s):
    B, most = s["slots"].shape
    ps = s["k_cache"].shape[3]
    rows = torch.cat([torch.zeros_like(s["new_len"]).unsqueeze(-1), s["path_nodes"]], dim=-1)
    b, k = torch.nonzero(torch.arange(most, device=rows.device) < s["new_len"].unsqueeze(-1),
                         as_tuple=True)
    slot, node = s["slots"][b, k].long(), rows[b, k].long()
    for_k, for_v = (c.transpose(2, 3) for c in (s["k_cache"], s["v_cache"]))
    for_k[:, slot // ps, slot % ps] = s["k_new"][:, b, node]
    for_v[:, slot // ps, slot % ps] = s["v_new"][:, b, node]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_attention(s):
    import paper_2505_12398_amd as tv
    return tv.tree_attention(s["q"], s["k_new"], s["v_new"], s["parents"], s["k_cache"],
                             s["v_cache"], s["block_table"], s["ctx_len"], s["scale"],
                             prefix_len=s["case"]["prefix"])


def _own_logits(s):
    import paper_2505_12398_amd as tv
    out, row_max, row_sum = tv.process_logits(
        s["logits"], s["temperature"], s["parents"], s["tokens"], history=s["history"],
        history_len=s["history_len"], prompt_len=s["prompt_len"], repetition=s["repetition"],
        presence=s["presence"], frequency=s["frequency"], bias_tokens=s["bias_tokens"],
        bias_values=s["bias_values"], masks=s["masks"], mask_index=s["mask_index"], out=s["out"])
    # the verifier takes the sums in 64 bits; their terms have 32, and so many are compared
    return {"logits": out, "row_max": row_max, "row_sum": row_sum.to(torch.float32)}


def _own_extend(s):
    import paper_2505_12398_amd as tv
    e = tv.cache_extend(s["new_len"], s["seq_len"], s["block_table"], s["free_pages"],
                        s["free_count"], s["page_size"], s["max_new"])
    return {"slots": e.slots, "block_table": s["block_table"], "seq_len": e.seq_len,
            "free_count": e.free_count, "status": e.status}


def _own_commit(s):
    import paper_2505_12398_amd as tv
    tv.cache_commit(s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["new_len"], s["slots"],
                    path_nodes=s["path_nodes"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"attention": _own_attention, "logits": _own_logits, "extend": _own_extend,
                "commit": _own_commit}[kind](s)
    return {"attention": _plain_attention, "logits": _plain_logits, "extend": _plain_extend,
            "commit": _plain_commit}[kind](s)


# --- work --------------------------------------------------------------------


def work(case):
    c, B = case, case["batch"]
    n1 = c.get("nodes", 0) + 1
    size = {"bf16": 2, "f16": 2, "f32": 4}.get(c.get("dtype"), 4)
    if c["kind"] == "attention":
        H, KH, D = c["heads"], c["kv_heads"], c["head_dim"]
        ctx = (c["ctx_lo"] + c["ctx_hi"]) / 2
        # a tree's nodes see the path to the root, half the depth on average
        seen = ctx + 1 + c["depth"] / 2
        cached = c["prefix"] + B * (ctx - c["prefix"])
        return {"bytes": size * D * (2 * KH * cached + B * n1 * (2 * H + 2 * KH)),
                "flops": 4.0 * D * H * B * n1 * seen}
    if c["kind"] == "logits":
        V = c["vocab"]
        # read and written once, with the rows' masks and the histories; an exponential counts 8
        return {"bytes": B * n1 * (2 * size * V + 12) + min(c["masks"], B * n1) * V / 8 +
                B * 4 * (c["hist_lo"] + c["hist_hi"]) / 2, "flops": 12.0 * B * n1 * V}
    if c["kind"] == "extend":
        new = (1 + c["max_new"]) / 2
        # lengths in and out, the slots' rows, the fresh pages from the stack into the tables
        return {"bytes": B * 4 * (4 + c["max_new"] + 2 * new / c["page"]), "flops": 0}
    rows = B * (2 + c["depth"] / 2)
    return {"bytes": 2 * 2 * size * c["layers"] * c["kv_heads"] * c["head_dim"] * rows, "flops": 0}


# --- 64 bits -----------------------------------------------------------------


def _paths(parents):
    """For every node of a tree, itself and its ancestors but the root."""
    got = []
    for i, p in enumerate(parents):
        got.append([] if i == 0 else got[p] + [i])
    return got


def _exact_attention(c, s):
    B, n1, H, D = s["q"].shape
    KH, ps = s["k_cache"].shape[1:3]
    out = torch.empty((B, n1, H, D), dtype=torch.float64, device=_DEV)
    for b, par in enumerate(s["parents"].tolist()):
        n = int(s["ctx_len"][b])
        hidden = torch.full((n1, n1), -math.inf, dtype=torch.float64)
        for i, p in enumerate(_paths(par)):
            hidden[i, [0] + p] = 0.0
        hidden = torch.cat([torch.zeros((n1, n), dtype=torch.float64), hidden], dim=1).to(_DEV)
        pages = s["block_table"][b, :-(-n // ps)].long()
        k, v = (torch.cat([cache[pages].double().permute(1, 0, 2, 3).reshape(KH, -1, D)[:, :n],
                           new[b].double().transpose(0, 1)], dim=1)
                for cache, new in ((s["k_cache"], s["k_new"]), (s["v_cache"], s["v_new"])))
        for h in range(H):
            kv = h // (H // KH)
            w = s["q"][b, :, h].double() @ k[kv].T * s["scale"] + hidden
            out[b, :, h] = torch.exp(w - w.logsumexp(dim=1, keepdim=True)) @ v[kv]
    return out


def _exact_logits(c, s):
    B, n1, V = s["logits"].shape
    z = torch.empty((B, n1, V), dtype=torch.float64, device=_DEV)
    top = torch.empty((B, n1), dtype=torch.float64, device=_DEV)
    total = torch.empty_like(top)
    tokens, parents = s["tokens"].tolist(), s["parents"].tolist()
    for b in range(B):
        n, p = int(s["history_len"][b]), int(s["prompt_len"][b])
        told = torch.bincount(s["history"][b, :min(n, p)], minlength=V)
        made = torch.bincount(s["history"][b, min(n, p):n], minlength=V)
        rho, alpha, beta = (float(s[k][b]) for k in ("repetition", "presence", "frequency"))
        extra = torch.zeros((n1, V), dtype=torch.int64)
        for i, path in enumerate(_paths(parents[b])):
            for j in path:
                extra[i, tokens[b][j]] += 1
        n = (extra.to(_DEV) + made).double()
        x = s["logits"][b].double()
        x = torch.where((n > 0) | (told > 0), torch.where(x > 0, x / rho, x * rho), x)
        x = x - (n > 0) * alpha - beta * n
        if s["bias_tokens"] is not None:
            x[:, s["bias_tokens"][b].long()] += s["bias_values"][b].double()
        if s["masks"] is not None:
            for i in range(n1):
                m = int(s["mask_index"][b, i])
                if m >= 0:
                    words = s["masks"][m].cpu().numpy().view(np.uint8)
                    bits = np.unpackbits(words, bitorder="little")[:V]
                    x[i, torch.as_tensor(bits == 0, device=_DEV)] = -math.inf
        z[b] = x
        # the statistics are those of the values as they are stored
        r = x.to(s["logits"].dtype).double()
        top[b] = r.amax(dim=1)
        total[b] = ((r - top[b].unsqueeze(1)) / s["temperature"]).exp().sum(dim=1)
    return {"logits": z, "row_max": top, "row_sum": total}


def _exact_commit(c, s):
    ps = c["page"]
    for b, n in enumerate(s["new_len"].tolist()):
        for k in range(n):
            node = int(s["path_nodes"][b, k - 1]) if k else 0
            page, at = divmod(int(s["slots"][b, k]), ps)
            s["k_cache"][:, page, :, at] = s["k_new"][:, b, node]
            s["v_cache"][:, page, :, at] = s["v_new"][:, b, node]
    return {"k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double()}


def exact(case, seed):
    """What ``run`` returns in 64 bits (the growth of the tables is whole numbers: None)."""
    if case["kind"] == "extend":
        return None
    return {"attention": _exact_attention, "logits": _exact_logits,
            "commit": _exact_commit}[case["kind"]](case, prepare(case, seed))
