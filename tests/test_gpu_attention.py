"""tv_tree_attention against the plain 64-bit form, on small cases where it can go
wrong: trees and single tokens, ragged and empty contexts, pages that end inside a
tile, odd sizes, both types, common prefixes, garbage in masked places (needs an
MI355X)."""

import numpy as np
import pytest
import torch

import paper_2505_12398_amd as tv
from oracle import decoding as D

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    tv.load_library()
    yield


def trees(kind, batch, n1, rng):
    par = np.full((batch, n1), -1, np.int32)
    i = np.arange(1, n1)
    for b in range(batch):
        par[b, 1:] = {"chain": i - 1, "star": 0 * i, "tree": rng.integers((i - 1) // 3, i)}[kind]
    return par


def inputs(batch, n1, heads, kv_heads, dim, ps, ctx, dtype="bf16", kind="tree", prefix=0, seed=0,
           spare=3, scale_q=1.0):
    """Host inputs (the values the device holds, in 64 bits) and their device tensors: q, k and
    v as slices of one projection, every page in a random place, garbage in all unused rows."""
    rng = np.random.default_rng([seed, batch, n1, heads, dim, ps])
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(seed)
    ctx = np.asarray(ctx, np.int32)
    shared = prefix // ps
    need = [max(0, -(-int(c) // ps) - (shared if prefix and c >= prefix else 0)) for c in ctx]
    pages = shared + sum(need) + spare
    order = rng.permutation(pages)
    width = max([1] + [-(-int(c) // ps) for c in ctx])
    table = np.full((batch, width), -7, np.int32)
    at = shared
    for b in range(batch):
        first = shared if prefix and ctx[b] >= prefix else 0
        if first:
            table[b, :first] = order[:first]
        table[b, first:first + need[b]] = order[at:at + need[b]]
        at += need[b]

    def normal(*shape):
        return torch.randn(shape, generator=g, dtype=torch.float32)
    qkv = normal(batch, n1, heads + 2 * kv_heads, dim)
    qkv[:, :, :heads] *= scale_q
    qkv = qkv.to(dt)
    kc, vc = (normal(pages, kv_heads, ps, dim).to(dt) for _ in range(2))
    # what no position holds is garbage
    used = np.zeros((pages, ps), bool)
    for b in range(batch):
        for x in range(max(int(ctx[b]), 0)):
            used[table[b, x // ps], x % ps] = True
    hole = torch.as_tensor(~used)[:, None, :, None]
    kc = torch.where(hole, torch.tensor(float("nan"), dtype=dt), kc)
    vc = torch.where(hole, torch.tensor(float("inf"), dtype=dt), vc)
    par = trees(kind, batch, n1, rng)
    host = dict(q=qkv[:, :, :heads], k_new=qkv[:, :, heads:heads + kv_heads],
                v_new=qkv[:, :, heads + kv_heads:], k_cache=kc, v_cache=vc)
    dev = qkv.to(DEV)
    call = dict(q=dev[:, :, :heads], k_new=dev[:, :, heads:heads + kv_heads],
                v_new=dev[:, :, heads + kv_heads:], parents=torch.as_tensor(par, device=DEV),
                k_cache=kc.to(DEV), v_cache=vc.to(DEV),
                block_table=torch.as_tensor(table, device=DEV),
                ctx_len=torch.as_tensor(ctx, device=DEV), scale=float(np.float32(dim ** -0.5)),
                prefix_len=prefix)
    host = {k: v.double().numpy() for k, v in host.items()}
    return dict(host, parents=par, table=table, ctx=ctx), call


def tolerance(exact, mass, big, dtype, dim, keys):
    """A rounding of the output; of every weight to the same type, which moves the numerator by
    at most that share of sum p |v|; fp32: the score's dot product ((dim + 4) roundings of
    sum |q k|, twice, for exp(x + d) = exp(x) (1 + d), d < 1e-3 here), the exponent and the
    frame in powers of two (4 roundings of it), and sums over the keys."""
    half = torch.finfo(TYPES[dtype]).eps / 2
    fp = 2.0 ** -24
    score = 2 * (dim + 8) * fp * big[..., None] + 8 * fp
    # fp16 weights below its smallest normal number lose up to half its spacing there
    low = keys * 2.0 ** -25 if dtype == "f16" else 0.0
    peak = np.abs(mass)
    return half * np.abs(exact) + (1.1 * half + 2 * score + 2 * keys * fp) * peak + low * 8 + \
        (2.0 ** -25 if dtype == "f16" else 1e-38)


def check(host, call, dtype="bf16", out=None, **kw):
    got = tv.tree_attention(**call, **kw) if out is None else out
    got = got.double().cpu().numpy()
    dim = got.shape[-1]
    for b in range(got.shape[0]):
        if host["ctx"][b] < 0:
            continue
        exact, mass, big = D.tree_attention(
            host["q"][b], host["k_new"][b], host["v_new"][b], host["parents"][b], host["k_cache"],
            host["v_cache"], host["table"][b], int(host["ctx"][b]), call["scale"])
        tol = tolerance(exact, mass, big, dtype, dim, int(host["ctx"][b]) + got.shape[1])
        err = np.abs(got[b] - exact)
        assert (err <= tol).all(), (b, float(np.nanmax(err / tol)),
                                    np.argwhere(~(err <= tol))[:3].tolist())
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n1,kind", [(1, "chain"), (2, "chain"), (6, "star"), (17, "tree"),
                                     (65, "tree")])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2), (8, 1)])
def test_trees_and_heads(dtype, n1, kind, heads, kv_heads):
    """Contexts around the sizes of tiles and pages, none and one token among them."""
    ctx = [0, 1, 15, 16, 17, 31, 33, 64, 129, 300]
    host, call = inputs(len(ctx), n1, heads, kv_heads, 128, 16, ctx, dtype, kind)
    check(host, call, dtype)


@pytest.mark.parametrize("dim", [8, 16, 40, 64, 72, 80, 96, 104, 120, 128])
@pytest.mark.parametrize("n1", [1, 9])
def test_head_sizes(dim, n1):
    host, call = inputs(3, n1, 6, 2, dim, 32, [70, 3, 257], "f16" if dim % 16 else "bf16")
    check(host, call, "f16" if dim % 16 else "bf16")


@pytest.mark.parametrize("ps", [16, 32, 64, 256, 1024])
def test_page_sizes(ps):
    host, call = inputs(4, 5, 4, 2, 64, ps, [ps - 1, ps, 2 * ps + 7, 5])
    check(host, call)


@pytest.mark.parametrize("n1,kind,heads,kv_heads", [
    (128, "tree", 4, 2), (129, "chain", 8, 2), (200, "tree", 3, 1), (1024, "tree", 2, 1),
    (1024, "chain", 1, 1), (33, "tree", 64, 8), (11, "tree", 16, 1)])
def test_many_rows(n1, kind, heads, kv_heads):
    """Many query rows of one key head: several row tiles, all of a tree's words of the mask."""
    host, call = inputs(2, n1, heads, kv_heads, 32, 16, [45, 0], kind=kind)
    check(host, call)


@pytest.mark.parametrize("batch,n1,ctx", [
    (1, 1, [5000]), (1, 65, [2500]), (3, 3, [4000, 7, 1111]), (40, 1, None), (37, 9, None)])
def test_long_and_ragged(batch, n1, ctx):
    """Few long contexts, divided over many workgroups, and many ragged ones."""
    rng = np.random.default_rng(batch)
    ctx = ctx or rng.integers(0, 700, batch)
    host, call = inputs(batch, n1, 8, 2, 128, 64, ctx)
    check(host, call)


@pytest.mark.parametrize("n1", [1, 7, 65])
@pytest.mark.parametrize("prefix", [16, 64, 208, 1040])
def test_common_prefix(n1, prefix):
    """Trees that have the prefix, exactly it, less, none and no part at all; the entries that
    the call must not read are no pages."""
    ctx = [prefix + 50, prefix, prefix - 1, prefix + 1, -1, 0, prefix + 333, prefix + 16]
    host, call = inputs(8, n1, 8, 2, 64, 16, ctx, prefix=prefix)
    table = call["block_table"].clone()
    pages = table[0, :prefix // 16].clone()
    for b in (0, 1, 3, 6, 7):
        table[b, :prefix // 16] = -1
    out = torch.full((8, n1, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    got = tv.tree_attention(**dict(call, block_table=table), prefix_pages=pages, out=out)
    assert (got[4] == 7.0).all()
    check(host, call, out=got)
    # pages by default: those of tree 0
    again = tv.tree_attention(**call)
    assert torch.equal(again[[0, 1, 2, 3, 5, 6, 7]], got[[0, 1, 2, 3, 5, 6, 7]])


def test_prefix_of_many_single_tokens():
    rng = np.random.default_rng(1)
    host, call = inputs(300, 1, 8, 2, 128, 64, 512 + rng.integers(0, 100, 300), prefix=512)
    check(host, call)


@pytest.mark.parametrize("prefix", [0, 48])
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 128), ("bf16", 64), ("f16", 40)])
@pytest.mark.parametrize("n1,kind", [(24, "tree"), (48, "chain"), (65, "tree"), (300, "tree")])
def test_rows_of_many_trees(n1, kind, dtype, dim, prefix):
    """Enough trees that workgroups take 96 or 192 rows at a time."""
    batch = 130 if n1 < 300 else 24
    rng = np.random.default_rng(n1)
    ctx = rng.integers(-3, 200, batch)
    ctx[:4] = 200, 0, 48, 47
    host, call = inputs(batch, n1, 8, 2, dim, 16, ctx, dtype, kind, prefix=prefix)
    check(host, call, dtype)


@pytest.mark.parametrize("heads", [4, 8])
def test_garbage_and_pages_that_are_none_in_many_trees(heads):
    """As above for one tree: no other node and no other tree sees any of it."""
    batch, n1 = 130, 40
    rng = np.random.default_rng(3)
    host, call = inputs(batch, n1, heads, 2, 64, 16, rng.integers(17, 150, batch))
    par = np.full((batch, n1), -1, np.int32)
    par[:, 1], par[:, 2] = 0, 0
    par[:, 3:] = np.arange(1, n1 - 2)
    call["parents"] = torch.as_tensor(par, device=DEV)
    host["parents"] = par
    clean = check(host, call)
    k, v, table = call["k_new"].clone(), call["v_new"].clone(), call["block_table"].clone()
    k[::3, 8::2] = float("nan")
    v[::3, 8::2, 0] = float("inf")
    v[1::3, 20, :, 3] = float("inf")
    table[5, 1], table[127, 0] = -1, call["k_cache"].shape[0]
    got = tv.tree_attention(**dict(call, k_new=k, v_new=v, block_table=table)).double().cpu().numpy()
    assert np.isnan(got[[5, 127]]).all()
    keep = np.ones((batch, n1, heads, 64), bool)
    keep[[5, 127]] = False
    keep[::3, 8::2] = False
    keep[1::3, 20::2, :, 3] = False
    np.testing.assert_array_equal(got[keep], clean[keep])
    others = [b for b in range(batch) if b not in (5, 127)]
    assert np.isnan(got[[b for b in others if b % 3 == 0], 8::2]).all()
    assert (got[[b for b in others if b % 3 == 1], 20::2, :, 3] == np.inf).all()


def test_peaked_and_large_scores():
    """Scores of several hundred: one key holds nearly all of a row's weight."""
    host, call = inputs(3, 9, 4, 2, 64, 16, [100, 33, 5], scale_q=40.0)
    check(host, call)


def test_values_far_above_the_scores_grow_along_the_row():
    """Every later key scores higher: the running maximum moves at each tile."""
    host, call = inputs(1, 3, 2, 1, 32, 16, [900], "f16")
    ramp = np.linspace(0.0, 60.0, 900)
    kc = host["k_cache"]
    q = np.zeros_like(host["q"])
    q[..., 0] = 1.0 / call["scale"]
    q = torch.tensor(q, dtype=torch.float16)
    for x in range(900):
        kc[host["table"][0, x // 16], :, x % 16, 0] = ramp[x]
    call["k_cache"] = torch.tensor(kc, dtype=torch.float16, device=DEV)
    call["q"] = q.to(DEV)
    host["k_cache"], host["q"] = call["k_cache"].double().cpu().numpy(), q.double().numpy()
    check(host, call, "f16")


def test_garbage_in_nodes_that_are_not_ancestors():
    """NaN and infinities in one branch's keys and values reach no node of the other."""
    host, call = inputs(2, 40, 4, 2, 64, 16, [37, 0])
    par = np.full((2, 40), -1, np.int32)
    par[:, 1], par[:, 2] = 0, 0
    par[:, 3:] = np.arange(1, 38)                       # two chains, odd and even nodes
    call["parents"] = torch.as_tensor(par, device=DEV)
    host["parents"] = par
    clean = tv.tree_attention(**call)
    bad = call["k_new"].clone(), call["v_new"].clone()
    bad[0][:, 8::2] = float("nan")
    bad[1][:, 8::2, 0] = float("inf")
    bad[1][:, 8::2, 1] = float("nan")
    got = tv.tree_attention(**dict(call, k_new=bad[0], v_new=bad[1]))
    fine = [i for i in range(40) if i % 2 or i < 8]
    assert torch.equal(got[:, fine], clean[:, fine])
    assert torch.isnan(got[:, 8::2]).all()
    # values alone: infinities stay infinities of their own dimension
    v = call["v_new"].clone()
    v[:, 20, :, 3] = float("inf")
    got = tv.tree_attention(**dict(call, v_new=v, k_new=call["k_new"].clone()))
    below = [i for i in range(40) if 20 in D.path(par[0], i)]
    others = [i for i in range(40) if i not in below]
    assert torch.equal(got[:, others], clean[:, others])
    assert (got[:, below][..., 3] == float("inf")).all()
    rest = [d for d in range(64) if d != 3]
    assert torch.equal(got[:, below][..., rest], clean[:, below][..., rest])


def test_links_that_do_not_point_back_end_a_path():
    host, call = inputs(1, 6, 2, 2, 32, 16, [20])
    par = np.array([[-1, 0, 9, 2, -3, 4]], np.int32)
    call["parents"], host["parents"] = torch.as_tensor(par, device=DEV), par
    check(host, call)


@pytest.mark.parametrize("n1", [1, 65])
def test_pages_that_are_none(n1):
    """A tree with a bad page or a context beyond its table gets NaN everywhere, the others
    theirs (other lengths cut the work elsewhere, so to the bounds and not to the bit); entries
    behind the context are not looked at."""
    ctx = [200, 100, 300, 64, 30]
    host, call = inputs(5, n1, 8, 2, 64, 16, ctx)
    table = call["block_table"].clone()
    table[1, 3], table[2, 18] = -1, call["k_cache"].shape[0]
    table[3, 4:] = 1 << 30
    lens = call["ctx_len"].clone()
    lens[0] = table.shape[1] * 16 + 1
    got = tv.tree_attention(**dict(call, block_table=table, ctx_len=lens))
    assert torch.isnan(got[:3]).all()
    host["ctx"][:3] = -1
    check(host, call, out=got)


def test_inactive_trees_are_left_as_they_were():
    host, call = inputs(6, 9, 4, 2, 64, 16, [-1, 33, -5, 0, 700, -2147483648])
    out = torch.full((6, 9, 4, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    check(host, call, out=tv.tree_attention(**call, out=out))
    assert (out[[0, 2, 5]] == 3.0).all()
    none = tv.tree_attention(**dict(call, ctx_len=torch.full_like(call["ctx_len"], -1)), out=out)
    assert torch.equal(none, out)


def test_no_pages_at_all():
    """A table without columns and a cache without pages: the trees alone."""
    host, call = inputs(2, 5, 4, 2, 64, 16, [0, 0])
    call["block_table"] = call["block_table"][:, :0].contiguous()
    call["k_cache"], call["v_cache"] = call["k_cache"][:0], call["v_cache"][:0]
    host["table"] = host["table"][:, :0]
    check(host, call)


def test_strided_pages_and_nodes():
    """Keys and values of a page side by side, q apart from k and v."""
    host, call = inputs(3, 5, 4, 2, 64, 16, [50, 16, 0])
    both = torch.stack([call["k_cache"], call["v_cache"]], dim=1)
    call["k_cache"], call["v_cache"] = both[:, 0], both[:, 1]
    call["q"] = call["q"].contiguous()
    check(host, call)


def test_repeated_calls_streams_and_workspaces():
    """The same bits on every call, on another stream, and on a workspace full of garbage that
    another call has used."""
    host, call = inputs(5, 17, 8, 2, 128, 16, [900, 40, 0, 333, 2000])
    want = check(host, call)
    need = tv.tv_tree_attention_workspace_size(5, 17, 8, 2, 128, 0)
    ws = torch.full((max(need, 1 << 20),), 0xff, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        got = tv.tree_attention(**call, workspace=ws)
        assert np.array_equal(got.double().cpu().numpy(), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = tv.tree_attention(**call)
    s.synchronize()
    assert np.array_equal(got.double().cpu().numpy(), want)


def test_captured_and_replayed():
    """One capture serves other lengths and tables: replays equal eager calls."""
    host, call = inputs(4, 9, 8, 2, 64, 16, [100, 7, 250, 31])
    _, other = inputs(4, 9, 8, 2, 64, 16, [3, 250, 16, 0], seed=5)
    need = tv.tv_tree_attention_workspace_size(4, 9, 8, 2, 64, 0)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    out = torch.zeros((4, 9, 8, 64), dtype=torch.bfloat16, device=DEV)
    tv.tree_attention(**call, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tv.tree_attention(**call, out=out, workspace=ws)
    for k in range(4):
        src = call if k % 2 == 0 else other
        lens = src["ctx_len"].clone()
        if k % 2:
            lens = lens.clamp(max=int(call["ctx_len"].min()))
        want = tv.tree_attention(**dict(call, ctx_len=lens))
        keep = call["ctx_len"].clone()
        call["ctx_len"].copy_(lens)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), k
        call["ctx_len"].copy_(keep)


def test_offsets_beyond_32_bits():
    """A cache of more than 4 GiB, the tree's pages at its far end."""
    ps, KH, D_, pages = 64, 8, 128, 36000                # 4.7 GB of keys
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GB")
    g = torch.Generator(device=DEV).manual_seed(2)
    kc = torch.empty((pages, KH, ps, D_), dtype=torch.bfloat16, device=DEV)
    vc = torch.empty_like(kc)
    table = torch.tensor([[35999, 5, 35998, 20000]], dtype=torch.int32, device=DEV)
    for p in table[0].tolist():
        kc[p] = torch.randn(kc[p].shape, generator=g, device=DEV)
        vc[p] = torch.randn(kc[p].shape, generator=g, device=DEV)
    qkv = torch.randn((1, 3, 48, D_), generator=g, device=DEV).to(torch.bfloat16)
    par = torch.tensor([[-1, 0, 1]], dtype=torch.int32, device=DEV)
    ctx = torch.tensor([250], dtype=torch.int32, device=DEV)
    args = (qkv[:, :, :32], qkv[:, :, 32:40], qkv[:, :, 40:], par)
    far = tv.tree_attention(*args, kc, vc, table, ctx, 0.088)
    near_k, near_v = kc[table[0].long()].contiguous(), vc[table[0].long()].contiguous()
    near = tv.tree_attention(*args, near_k, near_v,
                             torch.arange(4, dtype=torch.int32, device=DEV)[None], ctx, 0.088)
    assert torch.equal(far, near) and not torch.isnan(far).any()


def rounded_weights_tolerance(host, call, b, i, h, dtype, extra=0.0):
    """Where the sum of the weights is that of the rounded ones, sum w (1 + d) v / sum w (1 + d)
    differs from the exact out by at most half a step of sum p |v - out|; the output's own
    rounding; fp32 as in ``tolerance``; fp16 weights below 2^-21 of the largest are rounded to
    multiples of 2^-31 of it at worst: half of that a key, of |v - out|."""
    see = sorted(D.path(host["parents"][b], i))
    ctx = int(host["ctx"][b])
    kh = h // (host["q"].shape[2] // host["k_new"].shape[2])
    k = np.concatenate([D.cached(host["k_cache"], host["table"][b], ctx), host["k_new"][b][see]])[:, kh]
    v = np.concatenate([D.cached(host["v_cache"], host["table"][b], ctx), host["v_new"][b][see]])[:, kh]
    s = call["scale"] * (k @ host["q"][b, i, h])
    p = np.exp(s - s.max())
    p /= p.sum()
    out = p @ v
    half, fp = torch.finfo(TYPES[dtype]).eps / 2, 2.0 ** -24
    big = call["scale"] * (np.abs(k) @ np.abs(host["q"][b, i, h])).max()
    far = np.abs(v - out)
    tol = half * np.abs(out) + 1.1 * half * (p @ far) + \
        (4 * (k.shape[1] + 8) * fp * big + 16 * fp + 2 * len(s) * fp) * (p @ np.abs(v))
    if dtype == "f16":
        tol = tol + 1.1 * 2.0 ** -32 * far.sum(0) * p.max() + 2.0 ** -25
    return out, tol + extra


def one_request(ctx, scores, values, dtype, dim=64, heads=2, seed=0):
    """A single token on a context whose keys have these scores (natural) and values [ctx, dim];
    its own key's score is that of the lowest."""
    host, call = inputs(1, 1, heads, 1, dim, 64, [ctx], dtype, seed=seed)
    dt = TYPES[dtype]
    # two dimensions hold a score: what one rounds away is in the other
    q = torch.zeros((1, 1, heads, dim), dtype=dt)
    q[..., 0] = q[..., 1] = 8.0
    s = torch.tensor(np.append(scores, min(scores))) / (8.0 * call["scale"])
    k = torch.zeros((ctx + 1, dim), dtype=dt)
    k[:, 0] = s.to(dt)
    k[:, 1] = (s - k[:, 0].double()).to(dt)
    kc, vc = call["k_cache"].cpu(), call["v_cache"].cpu()
    for x in range(ctx):
        page = int(host["table"][0, x // 64])
        kc[page, :, x % 64] = k[x]
        vc[page, :, x % 64] = torch.as_tensor(values[x]).to(dt)
    call.update(q=q.to(DEV), k_cache=kc.to(DEV), v_cache=vc.to(DEV),
                k_new=k[None, None, None, ctx].to(DEV),
                v_new=torch.zeros((1, 1, 1, dim), dtype=dt, device=DEV))
    host.update(q=q.double().numpy(), **{n: call[n].double().cpu().numpy()
                                         for n in ("k_cache", "v_cache", "k_new", "v_new")})
    return host, call


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("above", [3.1, 4.3, 5.4])
def test_a_key_that_holds_nearly_all_weight(dtype, above):
    """Its weight in the frame of a smaller, earlier maximum is no power of two; the output is its
    value all the same, to the output's own rounding and the others' share."""
    rng = np.random.default_rng(2)
    scores = rng.uniform(-20.0, -15.0, 200)
    scores[0], scores[150] = -above, 0.0
    host, call = one_request(200, scores + 12.0, rng.normal(0, 1, (200, 64)), dtype)
    got = tv.tree_attention(**call).double().cpu().numpy()
    for h in range(2):
        want, tol = rounded_weights_tolerance(host, call, 0, 0, h, dtype)
        err = np.abs(got[0, 0, h] - want)
        assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("rows", [1, 65])
@pytest.mark.parametrize("gap", [12.0, 16.0, 18.0])
def test_a_key_far_above_many_others_in_fp16(gap, rows):
    """30000 keys at e^-gap of the first one's weight: together they count, though each of them
    is below the smallest fp16 number next to 1. The requests have the same context, and there
    are so many of them that one workgroup takes all of a context."""
    rng = np.random.default_rng(1)
    n, batch = 30000, 600 if rows == 1 else 260
    scores = np.append([gap], rng.uniform(-1.0, 0.0, n - 1))
    values = np.concatenate([np.zeros((1, 64)), rng.uniform(0.5, 1.5, (n - 1, 64))])
    host, call = one_request(n, scores, values, "f16")
    for name in ("q", "k_new", "v_new"):
        call[name] = call[name].repeat(batch, rows, 1, 1)
    call["parents"] = torch.zeros((batch, rows), dtype=torch.int32, device=DEV) - 1
    call["block_table"] = call["block_table"].repeat(batch, 1)
    call["ctx_len"] = call["ctx_len"].repeat(batch)
    got = tv.tree_attention(**call).double().cpu().numpy()
    for h in range(2):
        want, tol = rounded_weights_tolerance(host, call, 0, 0, h, "f16")
        err = np.abs(got[:, :, h] - want)
        assert (err <= tol).all(), (float(err.max()), float(tol.min()), float(want.min()))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_other_rows_scores_change_no_bits(dtype):
    """A request's bits do not depend on what other requests of the call, or other nodes of its
    tree, ask for: with and without a common prefix, at the same lengths."""
    for n1, prefix in ((1, 0), (1, 256), (9, 0), (9, 256)):
        host, call = inputs(6, n1, 8, 2, 64, 16, [prefix + 300] * 6, dtype, "star", prefix=prefix)
        want = tv.tree_attention(**call)
        q = call["q"].clone()
        q[1::2] *= 30
        assert torch.equal(tv.tree_attention(**dict(call, q=q))[::2], want[::2]), (n1, prefix)
        q = call["q"].clone()
        q[:, 1::2] *= 30
        q[:, :, 1::2] *= 30
        assert torch.equal(tv.tree_attention(**dict(call, q=q))[:, ::2, ::2], want[:, ::2, ::2])


@pytest.mark.parametrize("n1", [1, 3, 65])
@pytest.mark.parametrize("ctx", [1, 5, 31, 33, 48, 79])
def test_infinite_last_value_of_a_context(n1, ctx):
    """A value that is infinite at the last cached position is infinite in the output and in its
    own dimension alone, wherever the context ends in a tile."""
    host, call = inputs(2, n1, 4, 2, 64, 16, [ctx, ctx + 200])
    clean = check(host, call)
    v = call["v_cache"].clone()
    for b in range(2):
        x = int(host["ctx"][b]) - 1
        v[int(host["table"][b, x // 16]), :, x % 16, 3] = float("inf")
    got = tv.tree_attention(**dict(call, v_cache=v)).double().cpu().numpy()
    assert (got[..., 3] == np.inf).all()
    rest = [d for d in range(64) if d != 3]
    assert np.array_equal(got[..., rest], clean[..., rest])


def test_default_prefix_pages_are_those_of_a_tree_that_has_the_prefix():
    """The first trees of a batch may take no part or have shorter contexts."""
    for first in (1, 3, 70):
        ctx = [-1, 20, 0] + [63] * 67
        ctx = ctx[:first] + [64 + 30, 64, 64 + 5, 10, 64 + 77]
        host, call = inputs(len(ctx), 3, 4, 2, 64, 16, ctx, prefix=64)
        check(host, call)
    none = dict(call, ctx_len=call["ctx_len"].clamp(max=63))
    host["ctx"] = np.minimum(host["ctx"], 63)
    check(host, none)


def test_prefix_longer_than_the_table():
    """No tree can have it: contexts the table holds are computed, longer ones have bad pages."""
    host, call = inputs(3, 3, 4, 2, 64, 16, [40, 64, 5])
    width = call["block_table"].shape[1]
    lens = call["ctx_len"].clone()
    lens[1] = (width + 2) * 16
    far = torch.zeros(width + 1, dtype=torch.int32, device=DEV)
    for pages in (None, far):
        got = tv.tree_attention(**dict(call, ctx_len=lens, prefix_len=(width + 1) * 16),
                                prefix_pages=pages)
        assert torch.isnan(got[1]).all()
        host["ctx"][1] = -1
        check(host, call, out=got)


@pytest.mark.parametrize("prefix", [0, 1024])
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("n1,kind,batch", [(24, "tree", 80), (65, "tree", 50), (48, "chain", 40),
                                           (384, "tree", 6), (384, "chain", 6)])
def test_wide_blocks_on_long_contexts(n1, kind, batch, dtype, dim, prefix):
    """Workgroups of 96 and 192 rows over 60 tiles and more, in the common prefix too, with nodes
    kept as words and walked; contexts that end around a tile's end. Some of the trees are
    compared (all row tiles and heads of them), and the others' outputs are finite."""
    rng = np.random.default_rng(n1)
    ctx = rng.integers(1800, 2100, batch)
    ctx[:6] = 2000, 2016, 2015, 2033, 1024, 3
    host, call = inputs(batch, n1, 8, 2, dim, 16, ctx, dtype, kind, prefix=prefix)
    got = tv.tree_attention(**call)
    assert bool(got.isfinite().all())
    host["ctx"][2:4] = -1
    host["ctx"][6:-1] = -1
    check(host, call, dtype, out=got)
