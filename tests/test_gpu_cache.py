"""tv_cache_extend and tv_cache_commit against the plain forms, bit for bit, and a
run of decoding cycles with all the operators (needs an MI355X)."""

import numpy as np
import pytest
import torch

import paper_2505_12398_amd as tv
from oracle import decoding as D

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    tv.load_library()
    yield


def state(batch, ps, width, most, rng, spare=20, release=0.0, prefix=0):
    cap = width * ps
    seq = rng.integers(0, max(1, cap - most) + 1, batch)
    seq[rng.random(batch) < 0.1] = 0
    new = rng.integers(-2, most + 1, batch)
    new[rng.random(batch) < release] = D.RELEASE
    held = -(-seq // ps)
    pages = int(held.sum()) + spare
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((batch, width), -1, np.int32)
    at = 0
    for b in range(batch):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    free = np.full(pages, -1, np.int32)
    free[:spare] = order[at:]
    return new.astype(np.int32), seq.astype(np.int32), table, free, spare


def check(new, seq, table, free, count, ps, most, prefix=0, in_place=False):
    want = D.cache_extend(new, seq, table, free, count, ps, most, prefix)
    dev = [torch.as_tensor(x, device=DEV).contiguous() for x in (new, seq, table, free)]
    n = torch.tensor([count], dtype=torch.int32, device=DEV)
    out = None
    if in_place:
        out = tv.CacheGrowth(torch.empty((len(new), most), dtype=torch.int32, device=DEV), dev[1],
                             n, torch.empty(len(new), dtype=torch.int32, device=DEV))
    e = tv.cache_extend(dev[0], dev[1], dev[2], dev[3], n, ps, most, prefix_len=prefix, out=out)
    got = (e.slots, e.seq_len, dev[2], dev[3], e.free_count, e.status)
    for g, w, name in zip(got, want, ("slots", "seq_len", "table", "free", "count", "status")):
        np.testing.assert_array_equal(g.cpu().numpy().reshape(np.shape(w)), w, err_msg=name)
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,ps,width,most", [
    (1, 16, 1, 1), (5, 16, 4, 0), (7, 32, 3, 20), (64, 16, 8, 8), (1023, 16, 5, 9),
    (1024, 64, 2, 5), (1025, 16, 3, 3), (3000, 16, 4, 7), (3, 16, 700, 9000), (40, 128, 20, 2000)])
def test_extend(batch, ps, width, most, in_place):
    """Enough pages and too few; one workgroup's slots and many; with requests that end."""
    rng = np.random.default_rng(batch)
    for spare, release in ((batch * (most // ps + 1) + 3, 0.0), (batch // 3, 0.0),
                           (batch // 4 + 1, 0.2)):
        s = state(batch, ps, width, most, rng, spare, release)
        check(*s, ps, most, in_place=in_place)


def test_extend_bad_lengths():
    rng = np.random.default_rng(3)
    new, seq, table, free, count = state(12, 16, 4, 10, rng)
    seq[:4] = (-1, 65, -2147483648, 2147483647)
    new[4:9] = (11, 2147483647, -2147483647, 10, 0)
    seq[7] = 64
    check(new, seq, table, free, count, 16, 10)


@pytest.mark.parametrize("count", [-5, 0, 1000])
def test_extend_counts_out_of_range(count):
    rng = np.random.default_rng(4)
    new, seq, table, free, _ = state(12, 16, 4, 10, rng, spare=12)
    free[:] = np.arange(len(free))
    check(new, seq, table, free, count, 16, 10)


def test_extend_pages_that_are_none():
    """A request on a bad page gets no slot there; pages pushed past the stack are dropped."""
    rng = np.random.default_rng(5)
    new, seq, table, free, count = state(6, 16, 4, 20, rng, spare=12)
    table[0, 0], table[1, 0] = -1, 99999
    seq[:2], new[:2] = 5, 20
    check(new, seq, table, free, count, 16, 20)
    new[:] = D.RELEASE
    check(new, seq, table, free, len(free) - 2, 16, 20)


@pytest.mark.parametrize("prefix", [16, 48])
def test_extend_releases_keep_the_common_prefix(prefix):
    rng = np.random.default_rng(prefix)
    for _ in range(3):
        s = state(50, 16, 6, 12, rng, 9, 0.4, prefix)
        check(*s, 16, 12, prefix)


@pytest.mark.parametrize("layers,batch,n1,kv_heads,dim,ps,dtype", [
    (1, 1, 1, 1, 8, 16, torch.bfloat16), (3, 5, 9, 2, 64, 16, torch.float16),
    (2, 33, 20, 8, 128, 32, torch.bfloat16), (4, 3, 40, 3, 48, 64, torch.float32),
    (2, 4, 6, 2, 32, 16, torch.uint8)])
@pytest.mark.parametrize("path", [True, False])
def test_commit(layers, batch, n1, kv_heads, dim, ps, dtype, path):
    """Slots and nodes that are none, lengths of commit_paths' codes, rows left as they were."""
    rng = np.random.default_rng([batch, n1])
    P, most = 12 + batch * n1 // ps, n1 + 2
    bits = torch.randint(0, 256, (2, layers, batch, n1, kv_heads, dim * dtype.itemsize),
                         dtype=torch.uint8)
    k, v = (x.view(dtype) for x in bits)
    kc, vc = (torch.randint(0, 256, (layers, P, kv_heads, ps, dim * dtype.itemsize),
                            dtype=torch.uint8).view(dtype) for _ in range(2))
    slots = rng.permutation(P * ps)[:batch * most].reshape(batch, most).astype(np.int32) \
        if batch * most <= P * ps else None
    if slots is None:
        P = -(-batch * most // ps)
        kc, vc = (torch.randint(0, 256, (layers, P, kv_heads, ps, dim * dtype.itemsize),
                                dtype=torch.uint8).view(dtype) for _ in range(2))
        slots = rng.permutation(P * ps)[:batch * most].reshape(batch, most).astype(np.int32)
    slots[rng.random(slots.shape) < 0.1] = -1
    slots[0, 0] = P * ps + 3
    new = rng.integers(-2, most + 3, batch).astype(np.int32)
    new[0] = most
    nodes = rng.integers(-1, n1 + 1, (batch, most - 2)).astype(np.int32) if path else None

    def i8(t):
        return t.contiguous().view(torch.uint8).numpy()
    want = [D.cache_commit(i8(n), i8(c), new, slots, nodes) for n, c in ((k, kc), (v, vc))]
    dev = [t.to(DEV) for t in (k, v, kc, vc)]
    tv.cache_commit(*dev, torch.as_tensor(new, device=DEV), torch.as_tensor(slots, device=DEV),
                    path_nodes=torch.as_tensor(nodes, device=DEV) if path else None)
    for c, w in zip(dev[2:], want):
        np.testing.assert_array_equal(i8(c.cpu()), w)


def test_commit_from_a_projection_into_side_by_side_caches():
    """Keys and values as slices of the layers' projections, pages that hold both."""
    L, B, n1, KH, D_, ps, P = 3, 4, 7, 2, 64, 16, 9
    qkv = torch.randn((L, B, n1, 8 + 2 * KH, D_), device=DEV).to(torch.bfloat16)
    both = torch.zeros((L, P, 2, KH, ps, D_), dtype=torch.bfloat16, device=DEV)
    k, v = qkv[:, :, :, 8:8 + KH], qkv[:, :, :, 8 + KH:]
    slots = torch.arange(B * 3, dtype=torch.int32, device=DEV).view(B, 3) * 11
    path = torch.tensor([[2, 5]] * B, dtype=torch.int32, device=DEV)
    n = torch.tensor([3, 1, 0, 2], dtype=torch.int32, device=DEV)
    tv.cache_commit(k, v, both[:, :, 0], both[:, :, 1], n, slots, path_nodes=path)
    want = torch.zeros_like(both)
    for b, m in enumerate(n.tolist()):
        for j in range(m):
            s, node = int(slots[b, j]), (0, 2, 5)[j]
            want[:, s // ps, 0, :, s % ps], want[:, s // ps, 1, :, s % ps] = k[:, b, node], v[:, b, node]
    assert torch.equal(both, want)


def test_commit_of_a_long_prompt():
    """More rows than the launch's workgroups take in one step each."""
    n1, ps, KH = 20011, 1024, 2
    P = -(-n1 // ps) + 1
    k, v = (torch.randint(0, 256, (1, 1, n1, KH, 16), dtype=torch.uint8, device=DEV)
            for _ in range(2))
    caches = torch.zeros((2, 1, P, KH, ps, 16), dtype=torch.uint8, device=DEV)
    slots = torch.randperm(P * ps, device=DEV)[:n1].int().view(1, n1)
    n = torch.tensor([n1 - 3], dtype=torch.int32, device=DEV)
    tv.cache_commit(k, v, caches[0], caches[1], n, slots)
    want = torch.zeros_like(caches)
    at = slots[0, :n1 - 3].long()
    for c, t in ((0, k), (1, v)):
        want[c, 0, at // ps, :, at % ps] = t[0, 0, :n1 - 3]
    assert torch.equal(caches, want)


def test_pages_beyond_32_bits():
    """Pages 2^28 bytes apart: what is committed to far pages is what attention reads there."""
    n1, KH, D_, ps, P, apart = 40, 2, 64, 16, 20, 1 << 27
    far = [torch.empty((P - 1) * apart + KH * ps * D_, dtype=torch.bfloat16, device=DEV)
           .as_strided((P, KH, ps, D_), (apart, ps * D_, D_, 1)) for _ in range(2)]
    near = torch.zeros((2, P, KH, ps, D_), dtype=torch.bfloat16, device=DEV)
    k, v = (torch.randn((1, 1, n1, KH, D_), device=DEV).bfloat16() for _ in range(2))
    pages = torch.tensor([[19, 17, 8]], dtype=torch.int32, device=DEV)
    at = torch.arange(n1, device=DEV)
    slots = (pages[:, at // ps] * ps + at % ps).int()
    n = torch.tensor([n1], dtype=torch.int32, device=DEV)
    for caches in (far, near):
        tv.cache_commit(k, v, caches[0][None], caches[1][None], n, slots)
    out = []
    for caches in (far, near):
        q = torch.arange(5 * 4 * D_, device=DEV).view(1, 5, 4, D_).sin().bfloat16()
        new = torch.arange(5 * KH * D_, device=DEV).view(1, 5, KH, D_).cos().bfloat16()
        parents = torch.tensor([[-1, 0, 0, 2, 1]], dtype=torch.int32, device=DEV)
        out.append(tv.tree_attention(q, new, new, parents, caches[0], caches[1], pages, n, 0.1))
    for p in pages[0].tolist():
        for c in range(2):
            m = n1 - 32 if p == 8 else ps
            assert torch.equal(far[c][p, :, :m], near[c][p, :, :m])
    assert torch.equal(*out) and bool(out[0].isfinite().all())


def test_calls_on_a_given_stream():
    """Everything that a call allocates belongs to the stream that it is given: work that the
    current stream starts meanwhile, on memory of the same sizes, changes no result."""
    s = torch.cuda.Stream()
    B, n1, H, KH, D_, ps, width = 3, 9, 8, 2, 64, 16, 12
    gen = torch.Generator(DEV).manual_seed(5)
    q = torch.randn((B, n1, H, D_), device=DEV, generator=gen).bfloat16()
    kv = torch.randn((B, n1, KH, D_), device=DEV, generator=gen).bfloat16()
    cache = torch.randn((B * width, KH, ps, D_), device=DEV, generator=gen).bfloat16()
    table = torch.arange(B * width, dtype=torch.int32, device=DEV).view(B, width)
    ctx = torch.tensor([0, 17, 150], dtype=torch.int32, device=DEV)
    parents = torch.arange(-1, n1 - 1, dtype=torch.int32, device=DEV).repeat(B, 1)
    logits = torch.randn((B, n1, 5000), device=DEV, generator=gen)
    new = torch.tensor([3, 0, 2], dtype=torch.int32, device=DEV)
    path = torch.tensor([[1, 2, 0], [4, 0, 0], [5, 0, 0]], dtype=torch.int32, device=DEV)[:, :2]

    def calls(stream):
        free = torch.arange(B * width, dtype=torch.int32, device=DEV)
        count = torch.tensor([B * width], dtype=torch.int32, device=DEV)
        grown, caches = table.clone(), torch.zeros((2, 1, *cache.shape), device=DEV).bfloat16()
        torch.cuda.synchronize()
        out = tv.tree_attention(q, kv, kv, parents, cache, cache, table, ctx, 0.1, stream=stream)
        rows = tv.process_logits(logits, 0.7, stream=stream)
        g = tv.cache_extend(new, ctx, grown, free, count, ps, 4, stream=stream)
        tv.cache_commit(kv[None], kv[None], *caches, new, g.slots, path_nodes=path, stream=stream)
        for t in (out, *rows, torch.empty(1 << 22, dtype=torch.uint8, device=DEV)):
            torch.empty_like(t).fill_(7)
        torch.cuda.synchronize()
        return out, *rows, g.slots, g.seq_len, g.free_count, g.status, grown, caches

    for a, b in zip(calls(None), calls(s.cuda_stream)):
        assert torch.equal(a, b)


def test_captured_growth():
    """A captured cycle's growth in place, replayed: every replay grows the requests again."""
    rng = np.random.default_rng(8)
    new, seq, table, free, count = state(30, 16, 12, 6, rng, spare=400)
    seq //= 4
    dev = [torch.as_tensor(x, device=DEV).contiguous() for x in (new, seq, table, free)]
    n = torch.tensor([count], dtype=torch.int32, device=DEV)
    out = tv.CacheGrowth(torch.empty((30, 6), dtype=torch.int32, device=DEV), dev[1], n,
                         torch.empty(30, dtype=torch.int32, device=DEV))
    graph = torch.cuda.CUDAGraph()
    tv.cache_extend(*(torch.zeros_like(dev[0]), dev[1], dev[2], dev[3], n), 16, 6, out=out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        tv.cache_extend(dev[0], dev[1], dev[2], dev[3], n, 16, 6, out=out)
    for k in range(5):
        slots, seq, table, free, count, status = D.cache_extend(new, seq, table, free, count, 16, 6)
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip((out.slots, dev[1], dev[2], dev[3], n, out.status),
                        (slots, seq, table, free, count, status)):
            np.testing.assert_array_equal(g.cpu().numpy().reshape(np.shape(w)), w, err_msg=str(k))
        new = rng.integers(-2, 7, 30).astype(np.int32)
        dev[0].copy_(torch.as_tensor(new))


def test_decoding_cycles():
    """Three cycles of everything together, as a server runs them: draft trees, attention over
    the cache and the tree, an LM head, penalties, the verification with the processed rows'
    statistics, the commit of paths, pages and keys. The attention of every cycle over the paged
    cache equals that over a plain copy of the committed keys and values."""
    B, n1, H, KH, Dh, ps, V, K = 6, 13, 8, 2, 64, 16, 4099, 512
    g = torch.Generator(device=DEV).manual_seed(4)
    bf = torch.bfloat16

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV)
    w_t, w_d = (randn(V, K) * 0.2).to(bf), (randn(V, K) * 0.2).to(bf)
    w_qkv = (randn(K, (H + 2 * KH) * Dh) * K ** -0.5).to(bf)
    embed = randn(V, K).to(bf)
    kc = torch.full((1, 64, KH, ps, Dh), float("nan"), dtype=bf, device=DEV)
    vc = kc.clone()
    table = torch.full((B, 10), -1, dtype=torch.int32, device=DEV)
    free = torch.randperm(64, generator=g, device=DEV).to(torch.int32)
    count = torch.tensor([64], dtype=torch.int32, device=DEV)
    seq = torch.zeros(B, dtype=torch.int32, device=DEV)
    # prompts of 1 to 40 tokens
    plen = torch.randint(1, 41, (B,), generator=g, device=DEV).to(torch.int32)
    prompt = torch.randint(0, V, (B, 40), generator=g, device=DEV).to(torch.int32)
    pk, pv = randn(1, B, 40, KH, Dh).to(bf), randn(1, B, 40, KH, Dh).to(bf)
    e = tv.cache_extend(plen, seq, table, free, count, ps, 40)
    tv.cache_commit(pk, pv, kc, vc, plen, e.slots)
    assert e.status.tolist() == [tv.TV_CACHE_OK] * B
    plain = [([pk[0, b, i] for i in range(int(plen[b]))], [pv[0, b, i] for i in range(int(plen[b]))])
             for b in range(B)]
    seq, count = e.seq_len, e.free_count
    text = [prompt[b, :int(plen[b])].tolist() + [int(b)] for b in range(B)]
    T = 1.0
    for cycle in range(3):
        par = np.full((B, n1), -1, np.int32)
        rng = np.random.default_rng(cycle)
        for i in range(1, n1):
            par[:, i] = rng.integers(max(0, i - 4), i, B)
        parents = torch.as_tensor(par, device=DEV)
        hist = torch.zeros((B, 80), dtype=torch.int32, device=DEV)
        for b in range(B):
            hist[b, :len(text[b])] = torch.tensor(text[b], dtype=torch.int32)
        told = dict(history=hist, prompt_len=plen, repetition=torch.full((B,), 1.1, device=DEV),
                    presence=torch.full((B,), 0.2, device=DEV),
                    history_len=torch.tensor([len(t) for t in text], dtype=torch.int32, device=DEV))
        # draft logits level by level need a draft model; here each node's are given
        zd, _, _ = tv.lmhead_stats(randn(B, n1, K).to(bf), w_d, T)
        u = (torch.rand((B, n1), generator=g, device=DEV) * 2 ** 24).floor() / 2 ** 24
        tokens, st = tv.draft_tokens(parents, zd, T, u, tv.TV_SIBLINGS_WITHOUT_REPLACEMENT)
        assert not st.any()
        root = torch.tensor([t[-1] for t in text], device=DEV)
        ids = tokens.clone().long()
        ids[:, 0] = root
        x = embed[ids]
        qkv = (x.reshape(B * n1, K) @ w_qkv).view(B, n1, H + 2 * KH, Dh)
        q, k, v = qkv[:, :, :H], qkv[:, :, H:H + KH], qkv[:, :, H + KH:]
        o = tv.tree_attention(q, k, v, parents, kc[0], vc[0], table, seq, Dh ** -0.5)
        for b in range(B):
            n = len(plain[b][0])
            assert int(seq[b]) == n
            ck = torch.stack(plain[b][0]).double().cpu().numpy()
            cv = torch.stack(plain[b][1]).double().cpu().numpy()
            pages = [np.zeros((-(-n // ps), KH, ps, Dh)) for _ in range(2)]
            for i in range(n):
                pages[0][i // ps, :, i % ps], pages[1][i // ps, :, i % ps] = ck[i], cv[i]
            want, mass, _ = D.tree_attention(
                q[b].double().cpu().numpy(), k[b].double().cpu().numpy(),
                v[b].double().cpu().numpy(), par[b], *pages, np.arange(len(pages[0])), n, Dh ** -0.5)
            err = np.abs(o[b].double().cpu().numpy() - want)
            assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -7 * mass).all(), (cycle, b)
        zt, _, _ = tv.lmhead_stats(o.reshape(B, n1, K).contiguous(), w_t, T)
        zt, tm, ts = tv.process_logits(zt, T, parents, tokens, out=zt, **told)
        # the draft was drawn from its own logits: these pass through, with their statistics
        _, dm, ds = tv.process_logits(zd, T)
        uv = (torch.rand((B, n1), generator=g, device=DEV) * 2 ** 24).floor() / 2 ** 24
        out = tv.verify_batch(parents, tokens, zt, zd, T, uv, tv.TV_SIBLINGS_WITHOUT_REPLACEMENT,
                              stats=(tm, ts, dm, ds))
        assert not out.status.any()
        nodes, path, length = tv.commit_paths(parents, tokens, out, max_len=n1)
        e = tv.cache_extend(length, seq, table, free, count, ps, n1 + 1)
        tv.cache_commit(k[None], v[None], kc, vc, length, e.slots, path_nodes=nodes)
        assert e.status.tolist() == [tv.TV_CACHE_OK] * B
        for b in range(B):
            n = int(length[b])
            text[b] += path[b, :n].tolist()
            for node in [0] + nodes[b, :n - 1].tolist():
                plain[b][0].append(k[b, node])
                plain[b][1].append(v[b, node])
        seq, count = e.seq_len, e.free_count
    # every request ends: all pages are free again
    e = tv.cache_extend(torch.full_like(seq, tv.TV_CACHE_RELEASE), seq, table, free, count, ps, 1)
    assert int(e.free_count) == 64 and sorted(free.tolist()) == list(range(64))


@pytest.mark.parametrize("count,want", [(5, 5), (0, 0), (-3, 0), (99, 8)])
def test_extend_of_an_empty_batch(count, want):
    """The count of free pages is passed on, also where the caller has a place for it."""
    def i32(*shape):
        return torch.zeros(shape, dtype=torch.int32, device=DEV)
    n = torch.tensor([count], dtype=torch.int32, device=DEV)
    out = tv.CacheGrowth(i32(0, 4), i32(0), i32(1) - 7, i32(0))
    args = (i32(0), i32(0), i32(0, 3), i32(8), n, 16, 4)
    assert tv.cache_extend(*args, out=out) is out
    assert out.free_count.tolist() == [want] and n.tolist() == [count]
    assert tv.cache_extend(*args).free_count.tolist() == [want]


def test_the_given_stream_is_the_current_one_meanwhile():
    """Whatever stream is current, the default one given by its handle 0 among them; a cycle's
    calls then equal those on the current stream."""
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    dev = torch.device(DEV)
    for now in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(now):
            for given in (None, 0, side.cuda_stream, other.cuda_stream):
                with tv._lib._On(dev, given) as at:
                    assert at == (now.cuda_stream if given is None else given)
                    assert torch.cuda.current_stream().cuda_stream == at
                assert torch.cuda.current_stream() == now
    z = torch.randn((3, 5, 4001), device=DEV)
    n = torch.tensor([2, 0, 4], dtype=torch.int32, device=DEV)
    path = torch.tensor([[1, 0, 9, 0, 2, 0]] * 3, dtype=torch.int32, device=DEV)[:, ::2]
    k = torch.randn((1, 3, 5, 2, 8), device=DEV)
    slots = torch.arange(12, dtype=torch.int32, device=DEV).view(3, 4)

    def calls(stream):
        cache = torch.zeros((2, 1, 4, 2, 16, 8), device=DEV)
        torch.cuda.synchronize()
        rows = tv.process_logits(z, 0.7, stream=stream)
        tv.cache_commit(k, k, cache[0], cache[1], n, slots, path_nodes=path, stream=stream)
        torch.cuda.synchronize()
        return *rows, cache
    want = calls(None)
    with torch.cuda.stream(side):
        for stream in (0, other.cuda_stream):
            for a, b in zip(calls(stream), want):
                assert torch.equal(a, b)
