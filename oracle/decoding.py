"""Plain 64-bit forms of the operators around a verification: attention of tree
nodes over a paged cache, penalties, biases and masks on logits, growth of block
tables, commit of accepted keys and values. Written from their definitions, one
tree, node and token at a time; no code of the library."""

import numpy as np

RELEASE = -(1 << 31)
OK, FULL, OVERFLOW, BAD_LENGTH = range(4)


def path(parents, i):
    """Node i and its ancestors, up to the first link that does not point back."""
    got = [int(i)]
    while got[-1] > 0:
        p = int(parents[got[-1]])
        if p < 0 or p >= got[-1]:
            break
        got.append(p)
    return got


def cached(cache, table, n):
    """[n, kv_heads, D]: positions 0 .. n - 1 of a request; None if a page is none."""
    P, KH, ps, D = cache.shape
    if n > len(table) * ps:
        return None
    got = np.zeros((n, KH, D))
    for x in range(0, n, ps):
        page = int(table[x // ps])
        if not 0 <= page < P:
            return None
        m = min(ps, n - x)
        got[x:x + m] = cache[page, :, :m].transpose(1, 0, 2)
    return got


def tree_attention(q, k_new, v_new, parents, k_cache, v_cache, table, ctx, scale):
    """Outputs of one tree [N+1, heads, D], with sum_x p_x |v_x| and the largest
    scale * sum_d |q_d k_d| of its visible keys (what rounding errors scale with);
    NaN for a table that names a page that is none."""
    n1, H, D = q.shape
    KH = k_new.shape[1]
    out, mass, big = np.full((n1, H, D), np.nan), np.zeros((n1, H, D)), np.zeros((n1, H))
    old_k, old_v = cached(k_cache, table, ctx), cached(v_cache, table, ctx)
    if old_k is None or old_v is None:
        return out, mass, big
    for i in range(n1):
        see = sorted(path(parents, i))
        k = np.concatenate([old_k, k_new[see]])
        v = np.concatenate([old_v, v_new[see]])
        for h in range(H):
            kh, vh = k[:, h // (H // KH)], v[:, h // (H // KH)]
            s = scale * (kh @ q[i, h])
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ vh
            mass[i, h] = w @ np.abs(vh)
            big[i, h] = scale * (np.abs(kh) @ np.abs(q[i, h])).max()
    return out, mass, big


def process_logits(z, parents, tokens, history, prompt_len, rho, alpha, beta, biases, allowed):
    """One tree's logits [N+1, V] after penalties, biases (a list of (token, value), the
    last of a token's counts) and masks (per node an array of truth values or None);
    parents None: the paths count nothing."""
    n1, V = z.shape
    out = np.array(z, dtype=np.float64)
    told = set(int(t) for t in history[:prompt_len])
    made = {}
    for t in history[prompt_len:]:
        made[int(t)] = made.get(int(t), 0) + 1
    last = {int(t): float(x) for t, x in biases}
    for i in range(n1):
        n = dict(made)
        if parents is not None:
            for x in path(parents, i):
                if x > 0:
                    t = int(tokens[x])
                    n[t] = n.get(t, 0) + 1
        for t in told | set(n) | set(last):
            if not 0 <= t < V:
                continue
            x = float(z[i, t])
            if t in told or t in n:
                x = x / rho if x > 0 else x * rho
            out[i, t] = x - (alpha * (t in n) + beta * n.get(t, 0) - last.get(t, 0.0))
        if allowed is not None and allowed[i] is not None:
            out[i, ~allowed[i]] = -np.inf
    return out


def cache_extend(new_len, seq_len, table, free, count, ps, max_new, prefix_len=0):
    """(slots, seq_len, table, free, count, status) after a call, one request after the
    other."""
    B, width = table.shape
    table, free, seq = table.copy(), free.copy(), seq_len.copy()
    slots, status = np.full((B, max_new), -1, np.int32), np.zeros(B, np.int32)
    stack = list(free[:min(max(count, 0), len(free))])
    for b in range(B):
        if not 0 <= seq[b] <= width * ps:
            status[b] = BAD_LENGTH
        elif new_len[b] == RELEASE:
            first = prefix_len // ps if seq[b] >= prefix_len else 0
            for j in range(first, -(-int(seq[b]) // ps)):
                if len(stack) < len(free):
                    stack.append(table[b, j])
                    free[len(stack) - 1] = table[b, j]
                table[b, j] = -1
    wanted, avail, used = 0, len(stack), 0
    for b in range(B):
        if status[b] != OK:
            continue
        if new_len[b] == RELEASE:
            seq[b] = 0
            continue
        n = max(int(new_len[b]), 0)
        if n > max_new or int(seq[b]) + n > width * ps:
            status[b] = OVERFLOW
            continue
        held = -(-int(seq[b]) // ps)
        need = -(-(int(seq[b]) + n) // ps) - held
        wanted += need
        if need and wanted > avail:
            status[b] = FULL
            continue
        for j in range(need):
            table[b, held + j] = stack.pop()
        used += need
        for k in range(n):
            x = int(seq[b]) + k
            page = int(table[b, x // ps])
            slots[b, k] = page * ps + x % ps if 0 <= page < len(free) else -1
        seq[b] += n
    return slots, seq, table, free, avail - used, status


def cache_commit(k_new, k_cache, new_len, slots, path_nodes):
    """The cache [layers, pages, kv_heads, page_size, D] after a call (keys or values)."""
    L, B, n1 = k_new.shape[:3]
    P, ps = k_cache.shape[1], k_cache.shape[3]
    cache = k_cache.copy()
    for b in range(B):
        for k in range(min(int(new_len[b]), slots.shape[1])):
            node = k
            if path_nodes is not None and k > 0:
                node = int(path_nodes[b, k - 1]) if k <= path_nodes.shape[1] else -1
            s = int(slots[b, k])
            if 0 <= s < P * ps and 0 <= node < n1:
                cache[:, s // ps, :, s % ps] = k_new[:, b, node]
    return cache
