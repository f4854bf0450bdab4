"""The cache of 4 bits against the plain 64-bit forms: rows written and read back bit by bit,
attention over it, and a request's life from its prompt on (needs an MI355X)."""

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


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(x, np.int32), device=DEV)


# --- writing and reading -----------------------------------------------------


def commit_inputs(layers, batch, n1, heads, dim, ps, pages, dtype, seed=0):
    rng = np.random.default_rng([seed, layers, batch, dim])
    g = torch.Generator().manual_seed(seed)
    scale = torch.exp2(torch.randint(-12, 12, (2, layers, batch, n1, heads, dim // 32, 1), generator=g).float())
    x = torch.randn((2, layers, batch, n1, heads, dim // 32, 32), generator=g) * scale
    new = x.flatten(-2).to(TYPES[dtype])
    cache = rng.integers(0, 255, (2, layers) + tv.fp4_cache_shape(pages, heads, ps, dim)).astype(np.uint8)
    return new, cache, rng


def largest(dtype):
    """The exponent up to which 6 2^(e - 127) is a finite number of the type (of both types' grids the
    next value, 8 2^(e - 127), is none)."""
    return 140 if dtype == "f16" else 252


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layers,batch,n1,heads,dim,ps", [
    (1, 1, 1, 1, 32, 16), (2, 3, 7, 2, 64, 16), (3, 2, 5, 3, 96, 32), (1, 4, 9, 2, 128, 64),
    (2, 1, 40, 1, 128, 16)])
def test_commit(layers, batch, n1, heads, dim, ps, dtype):
    """Accepted nodes in any order, nodes and slots that are none among them; all other bytes stay."""
    pages, most = 6, n1 + 2
    new, cache, rng = commit_inputs(layers, batch, n1, heads, dim, ps, pages, dtype)
    path = rng.integers(-2, n1 + 2, (batch, most - 1))
    slots = np.stack(np.array_split(rng.permutation(pages * ps)[:batch * most], batch))
    slots[rng.random(slots.shape) < 0.15] = -1
    slots[0, -1] = pages * ps + 3
    n = rng.integers(0, most + 1, batch)
    n[0] = most + 5
    for p in (path, None):
        kc, vc = (torch.as_tensor(c, device=DEV) for c in cache)
        k, v = new.to(DEV)
        tv.cache_commit_fp4(k, v, kc, vc, ps, i32(n), i32(slots),
                            path_nodes=None if p is None else i32(p))
        for got, x, before in ((kc, new[0], cache[0]), (vc, new[1], cache[1])):
            want = D.cache_commit_fp4(x.double().numpy(), before, ps, n, slots, p, largest(dtype))
            np.testing.assert_array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("heads,dim,dtype", [(16, 128, "bf16"), (16, 128, "f16"), (32, 128, "bf16"),
                                             (24, 96, "f16"), (24, 96, "bf16"), (5, 96, "f16"), (40, 64, "bf16")])
def test_wide_rows(heads, dim, dtype):
    """Rows of 256 pieces of eight and more, of which threads have several, numbers of pieces that 256 is
    no multiple of, and more rows than a workgroup takes at a time: written, with nodes, slots and pages
    that are none, and read back from any place."""
    ps, pages, B, n1, most = 16, 4, 2, 13, 15
    new, cache, rng = commit_inputs(1, B, n1, heads, dim, ps, pages, dtype, seed=3)
    path = rng.integers(-1, n1 + 1, (B, most - 1))
    slots = np.stack(np.array_split(rng.permutation(pages * ps)[:B * most], B))
    slots[0, 4], slots[1, 9], slots[1, 2] = -1, pages * ps, -2 ** 31
    n = [most + 3, 11]
    kc, vc = (torch.as_tensor(c, device=DEV) for c in cache)
    tv.cache_commit_fp4(new[0].to(DEV), new[1].to(DEV), kc, vc, ps, i32(n), i32(slots), path_nodes=i32(path))
    held = [D.cache_commit_fp4(x.double().numpy(), c, ps, n, slots, path, largest(dtype))
            for x, c in zip(new, cache)]
    for got, want in zip((kc, vc), held):
        np.testing.assert_array_equal(got.cpu().numpy(), want)
    table, first, length, start = np.array([[2, -1, 0], [3, 1, pages]]), [5, 0], [30, 41], [3, 40]
    rows = 79                                # (of the second the last two are behind it)
    at = cache.shape[-1] // 17 * 16
    if dtype == "f16":                       # exponents around those fp16 holds, where others were
        held = [c.copy() for c in held]
        for c in held:
            c[..., at:] = np.where(c[..., at:] == 255, 255, 100 + c[..., at:] % 41)
        kc, vc = (torch.as_tensor(c, device=DEV) for c in held)
    out = tuple(torch.full((1, rows, heads, dim), 7.0, dtype=TYPES[dtype], device=DEV) for _ in range(2))
    tv.cache_read_fp4(kc, vc, ps, i32(table), i32(length), i32(start), rows, first=i32(first), out=out)
    for got, c in zip(out, held):
        want = D.cache_read_fp4(c, ps, dim, table, first, length, start, np.full((1, rows, heads, dim), 7.0))
        want = torch.tensor(want).to(TYPES[dtype]).double().numpy()
        np.testing.assert_array_equal(got.double().cpu().numpy(), want)


def special_blocks(dtype):
    """Ties, zeros of both signs, numbers below the normal ones, the largest ones, blocks around the
    borders of their exponent, and blocks with a number that is not finite."""
    t = TYPES[dtype]
    tiny, top = torch.finfo(t).smallest_normal, torch.finfo(t).max
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]
    rows = [ties + [-x for x in ties] + [0.0, -0.0] * 8]
    rows += [[x * 2.0 ** k for x in rows[0]] for k in (-14, -9, 5, 12)]
    for x in (7.0, 7.0 * (1 + torch.finfo(t).eps), 7.0 * (1 - torch.finfo(t).eps / 2), 6.0, 4.0, 1.75):
        for k in (-8, 0, 9):
            rows.append([x * 2.0 ** k, -1.0, 0.1] + [0.3 * 2.0 ** k] * 29)
    rows += [[0.0] * 32, [-0.0] * 32, [tiny] + [tiny / 2] * 31, [tiny / 4, -tiny / 8] * 16,
             [7 * tiny, tiny / 4] * 16, [top, -top] + [top / 7] * 30, [top / 2] + [1.0] * 31,
             [49152.0] * 16 + [57344.0, -57345.0] * 8, [float("inf")] + [1.0] * 31,
             [2.0] * 31 + [float("nan")], [1.0] * 16 + [-float("inf")] * 16]
    return torch.tensor(rows).to(t)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_special_numbers(dtype):
    x = special_blocks(dtype)
    n = x.shape[0]
    k = x.view(1, 1, n, 1, 32)
    ps = 16
    pages = -(-n // ps)
    cache = np.zeros((1,) + tv.fp4_cache_shape(pages, 1, ps, 32), np.uint8)
    kc, vc = (torch.as_tensor(cache, device=DEV) for _ in range(2))
    kd = k.to(DEV)
    slots = np.arange(n)[None]
    tv.cache_commit_fp4(kd, -kd, kc, vc, ps, i32([n]), i32(slots))
    want = D.cache_commit_fp4(k.double().numpy(), cache, ps, [n], slots, None, largest(dtype))
    np.testing.assert_array_equal(kc.cpu().numpy(), want)
    gk, gv = tv.cache_read_fp4(kc, vc, ps, i32(np.arange(pages)[None]), i32([n]), i32([0]), n,
                               dtype=TYPES[dtype])
    back = D.cache_read_fp4(want, ps, 32, np.arange(pages)[None], [0], [n], [0], np.zeros((1, n, 1, 32)))
    np.testing.assert_array_equal(gk.double().cpu().numpy(), back)
    np.testing.assert_array_equal(gv.double().cpu().numpy(), -back)
    finite = x.isfinite().all(-1)
    assert bool(gk[0, finite.to(DEV)].isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layers,heads,dim,ps", [(1, 1, 32, 16), (2, 3, 64, 16), (2, 2, 96, 64),
                                                 (1, 8, 128, 32)])
def test_read(layers, heads, dim, ps, dtype):
    """Any bytes at all; ranges that begin inside a page, empty ones, ones that leave the table,
    pages that are none; rows of no request and beyond the outputs."""
    rng = np.random.default_rng(dim)
    pages, B, width, rows = 9, 6, 4, 260
    cache = rng.integers(0, 256, (2, layers) + tv.fp4_cache_shape(pages, heads, ps, dim)).astype(np.uint8)
    at = cache.shape[-1] // 17 * 16
    if dtype == "f16":                       # exponents around those fp16 holds
        cache[..., at:] = 100 + cache[..., at:] % 44
    table = rng.integers(0, pages, (B, width))
    table[1, 1], table[2, 0], table[5, 2] = -1, pages, 1 << 30
    first = np.array([0, 5, ps - 1, -3, width * ps - 2, 2 * ps])
    length = np.array([2 * ps + 3, 30, 0, 9, 7, -4])
    start = np.array([0, 2 * ps + 9, 0, 200, 252, 5])
    g = torch.Generator().manual_seed(1)
    before = torch.randn((2, layers, rows, heads, dim), generator=g).to(TYPES[dtype])
    out = tuple(b.clone().to(DEV) for b in before)
    kc, vc = (torch.as_tensor(c, device=DEV) for c in cache)
    got = tv.cache_read_fp4(kc, vc, ps, i32(table), i32(length), i32(start), rows, first=i32(first),
                            out=out)
    assert got is out
    for x, b, c in zip(out, before, cache):
        want = D.cache_read_fp4(c, ps, dim, table, first, length, start, b.double().numpy())
        with np.errstate(over="ignore"):
            if dtype == "f16":               # one rounding, to the nearest
                want = want.astype(np.float16).astype(np.float64)
            else:                            # 6 2^127 alone is too large
                want = torch.tensor(want).to(torch.bfloat16).double().numpy()
        np.testing.assert_array_equal(x.double().cpu().numpy(), want)
    # without first, and into rows that lie apart (a buffer that new rows follow)
    buf = torch.zeros((layers, rows, 2 * heads, dim), dtype=TYPES[dtype], device=DEV)
    k, v = buf[:, :, :heads], buf[:, :, heads:]
    tv.cache_read_fp4(kc, vc, ps, i32(table), i32(length), i32(start), rows, out=(k, v))
    k2, v2 = tv.cache_read_fp4(kc, vc, ps, i32(table), i32(length), i32(start), rows, first=i32(0 * first),
                               dtype=TYPES[dtype])
    told = np.zeros(rows, bool)
    for s, n in zip(start, length):
        told[s:s + max(n, 0)] = True
    told = torch.as_tensor(told, device=DEV)
    for a, b in ((k, k2), (v, v2)):
        a, b = a[:, told], b[:, told]
        assert bool(((a == b) | (a.isnan() & b.isnan())).all())
        assert not buf[:, ~told].any()


def test_many_rows_of_long_requests():
    """Rows that a launch takes in several steps, against a table lookup of all bytes."""
    ps, KH, dim, n = 64, 2, 128, [70001, 3, 40000]
    g = torch.Generator(device=DEV).manual_seed(3)
    need = [-(-x // ps) for x in n]
    pages = sum(need)
    cache = torch.randint(0, 256, (2, 1) + tv.fp4_cache_shape(pages, KH, ps, dim), dtype=torch.uint8,
                          generator=g, device=DEV)
    at = cache.shape[-1] // 17 * 16
    cache[..., at:] = 120 + cache[..., at:] % 16
    order = torch.randperm(pages, generator=g, device=DEV).int()
    table = torch.zeros((3, max(need)), dtype=torch.int32, device=DEV)
    done = 0
    for b in range(3):
        table[b, :need[b]] = order[done:done + need[b]]
        done += need[b]
    start = np.cumsum(n) - n
    k, v = tv.cache_read_fp4(cache[0], cache[1], ps, table, i32(n), i32(start), sum(n))
    values = torch.tensor(D.FP4_VALUES + tuple(-x for x in D.FP4_VALUES), device=DEV)
    for x, c in ((k, cache[0, 0]), (v, cache[1, 0])):
        code = torch.stack([c[..., :at] & 15, c[..., :at] >> 4], -1).flatten(-2).int()
        all_rows = values[code].view(pages, KH, ps, dim // 32, 32) * \
            torch.exp2(c[..., at:].float() - 127).view(pages, KH, ps, dim // 32, 1)
        all_rows = all_rows.flatten(-2).to(torch.bfloat16)
        for b in range(3):
            want = all_rows[table[b, :need[b]].long()].transpose(1, 2).reshape(-1, KH, dim)[:n[b]]
            assert torch.equal(x[0, start[b]:start[b] + n[b]], want)
    # and back into another cache: values of the grid keep theirs
    other = torch.zeros_like(cache)
    slots = torch.full((3, max(n)), -1, dtype=torch.int32, device=DEV)
    k_new, v_new = (torch.zeros((1, 3, max(n), KH, dim), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for b in range(3):
        x = torch.arange(n[b], device=DEV)
        slots[b, :n[b]] = table[b, x // ps] * ps + x.int() % ps
        k_new[0, b, :n[b]], v_new[0, b, :n[b]] = k[0, start[b]:start[b] + n[b]], v[0, start[b]:start[b] + n[b]]
    tv.cache_commit_fp4(k_new, v_new, other[0], other[1], ps, i32(n), slots)
    k2, v2 = tv.cache_read_fp4(other[0], other[1], ps, table, i32(n), i32(start), sum(n))
    assert torch.equal(k2, k) and torch.equal(v2, v)


@pytest.mark.parametrize("order", ["kv first", "layers in a row", "rows first, layers backwards", "one"])
def test_outputs_between_each_other(order):
    """Rows of all layers, of keys and values, in one buffer; one buffer as both for one cache as both."""
    ps, KH, dim, L, rows = 16, 2, 64, 3, 21
    rng = np.random.default_rng(6)
    cache = rng.integers(0, 250, (2, L) + tv.fp4_cache_shape(3, KH, ps, dim)).astype(np.uint8)
    kc, vc = (torch.as_tensor(c, device=DEV) for c in cache)
    args = (ps, i32([[2, 0]]), i32([rows]), i32([0]), rows)
    want = tv.cache_read_fp4(kc, vc, *args)
    if order == "one":
        got = tv.cache_read_fp4(kc, kc, *args, out=(want[1], want[1]))
        assert torch.equal(got[0], want[0])
        return
    if order == "kv first":
        k, v = torch.zeros((2, L, rows, KH, dim), dtype=torch.bfloat16, device=DEV)
    elif order == "layers in a row":
        buf = torch.zeros((rows, 2, L, KH, dim), dtype=torch.bfloat16, device=DEV)
        k, v = buf[:, 0].transpose(0, 1), buf[:, 1].transpose(0, 1)
    else:
        buf = torch.zeros((L, rows, 2, KH, dim), dtype=torch.bfloat16, device=DEV)
        k, v = buf[:, :, 1], buf[:, :, 0]
    if "backwards" in order:                 # (torch has no negative strides: through the C-ABI)
        st = tv.tv_cache_read_fp4(L, 1, KH, dim, tv.TV_DTYPE_BF16, kc, vc, kc.stride(0), kc.stride(1), 3, *args[:2],
                                  2, None, args[2], args[3], rows, k[L - 1].data_ptr(), v[L - 1].data_ptr(),
                                  -k.stride(0), k.stride(1), torch.cuda.current_stream().cuda_stream)
        assert st == tv.TV_OK
        k, v = k.flip(0), v.flip(0)
    else:
        tv.cache_read_fp4(kc, vc, *args, out=(k, v))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_widest_rows():
    """512 heads of 128, the most there are, against a table lookup of all bytes, and back again."""
    ps, KH, dim, n = 16, 512, 128, 20
    g = torch.Generator(device=DEV).manual_seed(5)
    cache = torch.randint(0, 256, (2, 1) + tv.fp4_cache_shape(2, KH, ps, dim), dtype=torch.uint8, generator=g,
                          device=DEV)
    at = cache.shape[-1] // 17 * 16
    cache[..., at:] = 120 + cache[..., at:] % 16
    table = i32([[1, 0]])
    k, v = tv.cache_read_fp4(cache[0], cache[1], ps, table, i32([n]), i32([0]), n)
    values = torch.tensor(D.FP4_VALUES + tuple(-x for x in D.FP4_VALUES), device=DEV)
    for x, c in ((k, cache[0, 0]), (v, cache[1, 0])):
        code = torch.stack([c[..., :at] & 15, c[..., :at] >> 4], -1).flatten(-2).int()
        rows = values[code].view(2, KH, ps, dim // 32, 32) * \
            torch.exp2(c[..., at:].float() - 127).view(2, KH, ps, dim // 32, 1)
        want = rows.flatten(-2).to(torch.bfloat16)[[1, 0]].transpose(1, 2).reshape(-1, KH, dim)[:n]
        assert torch.equal(x[0], want)
    # values of the grid keep theirs, though not always their exponent
    other = torch.zeros_like(cache)
    slots = (16 * (1 - torch.arange(n, device=DEV) // 16) + torch.arange(n, device=DEV) % 16).int()[None]
    tv.cache_commit_fp4(k[:, None], v[:, None], other[0], other[1], ps, i32([n]), slots)
    k2, v2 = tv.cache_read_fp4(other[0], other[1], ps, table, i32([n]), i32([0]), n)
    assert torch.equal(k2, k) and torch.equal(v2, v)


def test_lengths_far_beyond_the_outputs():
    """Positions whose rows the outputs do not have cost nothing, however many: the rows there are hold
    theirs, NaN behind the table."""
    ps, KH, dim, rows, most = 16, 2, 64, 100, 2 ** 31 - 1
    rng = np.random.default_rng(8)
    cache = rng.integers(0, 255, (2, 2) + tv.fp4_cache_shape(5, KH, ps, dim)).astype(np.uint8)
    kc, vc = (torch.as_tensor(c, device=DEV) for c in cache)
    table = np.array([[3, 1, 4]])
    # (and the call without what the outputs do not have)
    for first, start, as_first, as_start in ((0, 0, 0, 0), (7, 40, 7, 40), (5, -20, 25, 0),
                                             (0, -2 ** 30, 2 ** 30, 0), (-3, 99, -3, 99),
                                             (most, 90, most, 90), (0, 100, 0, 100), (0, most, 0, 100),
                                             (0, -2 ** 31, 0, 100)):
        out = tuple(torch.full((2, rows, KH, dim), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        tv.cache_read_fp4(kc, vc, ps, i32(table), i32([most]), i32([start]), rows, first=i32([first]), out=out)
        for got, c in zip(out, cache):
            want = D.cache_read_fp4(c, ps, dim, table, [as_first], [rows - as_start], [as_start],
                                    np.full((2, rows, KH, dim), 5.0))
            want = torch.tensor(want).to(torch.bfloat16).double().numpy()
            np.testing.assert_array_equal(got.double().cpu().numpy(), want, err_msg=f"{first} {start}")


def test_write_and_read_captured_and_replayed():
    ps, KH, dim = 16, 2, 64
    g = torch.Generator(device=DEV).manual_seed(4)
    new = torch.randn((2, 1, 3, 8, KH, dim), generator=g, device=DEV).to(torch.bfloat16)
    cache = torch.zeros((2, 1) + tv.fp4_cache_shape(4, KH, ps, dim), dtype=torch.uint8, device=DEV)
    table, start = i32([[0, 3], [1, 0], [2, 0]]), i32([0, 8, 16])
    slots, n = i32([[x * ps + y for y in range(8)] for x in (0, 1, 2)]), i32([8, 8, 8])
    out = tuple(torch.zeros((1, 24, KH, dim), dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def go():
        tv.cache_commit_fp4(new[0], new[1], cache[0], cache[1], ps, n, slots)
        tv.cache_read_fp4(cache[0], cache[1], ps, table, n, start, 24, out=out)
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for lens in ([8, 8, 8], [0, 5, 8], [3, 0, 1]):
        new.copy_(torch.randn(new.shape, generator=g, device=DEV))
        n.copy_(torch.tensor(lens, dtype=torch.int32))
        cache.zero_()
        for t in out:
            t.zero_()
        go()
        torch.cuda.synchronize()
        want = [t.clone() for t in out] + [cache.clone()]
        cache.zero_()
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip([*out, cache], want):
            assert torch.equal(a, b), lens


# --- attention ---------------------------------------------------------------


def trees(kind, batch, n1, rng):
    par = np.full((batch, n1), -1, np.int32)
    i = np.arange(1, n1)
    for b in range(batch):
        par[b, 1:] = {"chain": i - 1, "star": 0 * i, "tree": rng.integers((i - 1) // 3, i)}[kind]
    return par


def decoded(cache, ps, dim):
    """[pages, kv_heads, page_size, D] in 64 bits of bytes [pages, kv_heads, bytes] (as
    ``oracle.decoding.fp4_cache``, whole arrays at a time)."""
    at = cache.shape[-1] // 17 * 16
    raw = cache[..., :at]
    code = np.stack([raw & 15, raw >> 4], -1).reshape(cache.shape[:2] + (ps, dim // 32, 32))
    table = np.array(D.FP4_VALUES + tuple(-x for x in D.FP4_VALUES))
    e = cache[..., at:].reshape(cache.shape[:2] + (ps, dim // 32, 1)).astype(np.float64)
    x = np.where(e == 255, np.nan, table[code] * np.exp2(e - 127))
    return x.reshape(cache.shape[:2] + (ps, dim))


def test_decoded_is_the_oracles():
    rng = np.random.default_rng(0)
    cache = rng.integers(0, 256, tv.fp4_cache_shape(2, 3, 16, 96)).astype(np.uint8)
    np.testing.assert_array_equal(decoded(cache, 16, 96), D.fp4_cache(cache, 16, 96))


def inputs(batch, n1, heads, kv_heads, dim, ps, ctx, dtype="bf16", kind="tree", prefix=0, seed=0,
           spare=3, scale_q=1.0):
    """Host inputs (the values the device holds, in 64 bits) and the call: q, k and v as slices of one
    projection, every page in a random place, NaN in all unused rows."""
    rng = np.random.default_rng([seed, batch, n1, heads, dim, ps])
    g = torch.Generator().manual_seed(seed)
    ctx = np.asarray(ctx, np.int32)
    shared = prefix // ps
    need = [max(0, -(-int(c) // ps) - (shared if prefix and c >= prefix else 0)) for c in ctx]
    pages = shared + sum(need) + spare
    order = rng.permutation(pages)
    table = np.full((batch, max([1] + [-(-int(c) // ps) for c in ctx])), -7, np.int32)
    at = shared
    for b in range(batch):
        first = shared if prefix and ctx[b] >= prefix else 0
        if first:
            table[b, :first] = order[:first]
        table[b, first:first + need[b]] = order[at:at + need[b]]
        at += need[b]
    used = np.zeros((pages, ps), bool)
    for b in range(batch):
        x = np.arange(max(int(ctx[b]), 0))
        used[table[b, x // ps], x % ps] = True
    caches = []
    for _ in range(2):
        c = rng.integers(0, 256, tv.fp4_cache_shape(pages, kv_heads, ps, dim)).astype(np.uint8)
        e = c[..., c.shape[-1] // 17 * 16:].reshape(pages, kv_heads, ps, dim // 32)
        e[:] = np.where(used[:, None, :, None], 123 + e % 5, 255)
        caches.append(c)
    qkv = torch.randn((batch, n1, heads + 2 * kv_heads, dim), generator=g)
    qkv[:, :, :heads] *= scale_q
    qkv = qkv.to(TYPES[dtype])
    par = trees(kind, batch, n1, rng)
    dev = qkv.to(DEV)
    call = dict(q=dev[:, :, :heads], k_new=dev[:, :, heads:heads + kv_heads],
                v_new=dev[:, :, heads + kv_heads:], parents=i32(par),
                k_cache=torch.as_tensor(caches[0], device=DEV),
                v_cache=torch.as_tensor(caches[1], device=DEV), page_size=ps, block_table=i32(table),
                ctx_len=i32(ctx), scale=float(np.float32(dim ** -0.5)), prefix_len=prefix)
    host = dict(q=qkv[:, :, :heads].double().numpy(),
                k_new=qkv[:, :, heads:heads + kv_heads].double().numpy(),
                v_new=qkv[:, :, heads + kv_heads:].double().numpy(), parents=par, table=table, ctx=ctx,
                k_cache=decoded(caches[0], ps, dim), v_cache=decoded(caches[1], ps, dim))
    return host, call


def tolerance(exact, mass, big, dtype, dim, keys, most):
    """The output's rounding; that of every weight (half a step of sum p |v - out| <= 2 sum p |v|); fp32:
    the score's dot product, the exponent and the frame, sums over the keys; fp16 weights below 2^-21
    of the largest are multiples of 2^-31 of it (half of that a key, of |v - out| <= 2 max |v|), and
    outputs below its normal range multiples of 2^-24. (The cache's values are exact in both types.)"""
    half, fp = torch.finfo(TYPES[dtype]).eps / 2, 2.0 ** -24
    tol = half * np.abs(exact) + \
        (2.2 * half + 4 * (dim + 8) * fp * big[..., None] + 16 * fp + 2 * keys * fp) * mass
    if dtype == "f16":
        tol = tol + 2.0 ** -31 * keys * most + 2.0 ** -25
    return tol + 1e-30


def check(host, call, dtype="bf16", out=None, **kw):
    got = tv.tree_attention_fp4(**call, **kw) if out is None else out
    got = got.double().cpu().numpy()
    most = max(float(np.nanmax(np.abs(host["v_cache"]), initial=0.0)), float(np.abs(host["v_new"]).max()))
    for b in range(got.shape[0]):
        if host["ctx"][b] < 0:
            continue
        exact, mass, big = D.tree_attention(
            host["q"][b], host["k_new"][b], host["v_new"][b], host["parents"][b], host["k_cache"],
            host["v_cache"], host["table"][b], int(host["ctx"][b]), call["scale"])
        tol = tolerance(exact, mass, big, dtype, got.shape[-1], int(host["ctx"][b]) + got.shape[1], most)
        err = np.abs(got[b] - exact)
        assert (err <= tol).all(), (b, float(np.nanmax(err / tol)), np.argwhere(~(err <= tol))[:3].tolist())
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n1,kind", [(1, "chain"), (2, "chain"), (6, "star"), (17, "tree"), (65, "tree")])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2), (8, 1)])
def test_trees_and_heads(dtype, n1, kind, heads, kv_heads):
    ctx = [0, 1, 15, 16, 17, 31, 33, 64, 129, 300]
    host, call = inputs(len(ctx), n1, heads, kv_heads, 128, 16, ctx, dtype, kind)
    check(host, call, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("n1", [1, 9, 40])
def test_head_sizes(dim, n1, dtype):
    host, call = inputs(3, n1, 6, 2, dim, 32, [70, 3, 257], dtype)
    check(host, call, dtype)


@pytest.mark.parametrize("ps", [16, 32, 64, 256, 1024])
def test_page_sizes(ps):
    host, call = inputs(4, 5, 4, 2, 64, ps, [ps - 1, ps, 2 * ps + 7, 5])
    check(host, call)


@pytest.mark.parametrize("n1,kind,heads,kv_heads", [
    (128, "tree", 4, 2), (129, "chain", 8, 2), (200, "tree", 3, 1), (1024, "tree", 2, 1),
    (1024, "chain", 1, 1), (33, "tree", 64, 8), (11, "tree", 16, 1)])
def test_many_rows(n1, kind, heads, kv_heads):
    host, call = inputs(2, n1, heads, kv_heads, 32, 16, [45, 0], kind=kind)
    check(host, call)


@pytest.mark.parametrize("batch,n1,ctx", [
    (1, 1, [5000]), (1, 65, [2500]), (3, 3, [4000, 7, 1111]), (40, 1, None), (37, 9, None)])
def test_long_and_ragged(batch, n1, ctx):
    rng = np.random.default_rng(batch)
    ctx = ctx or rng.integers(0, 700, batch)
    host, call = inputs(batch, n1, 8, 2, 128, 64, ctx)
    check(host, call)


@pytest.mark.parametrize("n1", [1, 7, 65])
@pytest.mark.parametrize("prefix", [16, 208, 1040])
def test_common_prefix(n1, prefix):
    ctx = [prefix + 50, prefix, prefix - 1, prefix + 1, -1, 0, prefix + 333, prefix + 16]
    host, call = inputs(8, n1, 8, 2, 64, 16, ctx, prefix=prefix)
    table = call["block_table"].clone()
    pages = table[0, :prefix // 16].clone()
    for b in (0, 1, 3, 6, 7):
        table[b, :prefix // 16] = -1
    out = torch.full((8, n1, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    got = tv.tree_attention_fp4(**dict(call, block_table=table), prefix_pages=pages, out=out)
    assert (got[4] == 7.0).all()
    check(host, call, out=got)
    again = tv.tree_attention_fp4(**call)
    assert torch.equal(again[[0, 1, 2, 3, 5, 6, 7]], got[[0, 1, 2, 3, 5, 6, 7]])


@pytest.mark.parametrize("prefix", [0, 48])
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 128), ("bf16", 64), ("f16", 32)])
@pytest.mark.parametrize("n1,kind", [(24, "tree"), (48, "chain"), (65, "tree"), (300, "tree")])
def test_rows_of_many_trees(n1, kind, dtype, dim, prefix):
    """Enough trees that workgroups take 96 or 192 rows at a time."""
    batch = 130 if n1 < 300 else 24
    rng = np.random.default_rng(n1)
    ctx = rng.integers(-3, 200, batch)
    ctx[:4] = 200, 0, 48, 47
    host, call = inputs(batch, n1, 8, 2, dim, 16, ctx, dtype, kind, prefix=prefix)
    got = tv.tree_attention_fp4(**call)
    active = torch.as_tensor(ctx >= 0, device=DEV)
    assert bool(got[active].isfinite().all())
    host["ctx"][30:-2] = -1
    check(host, call, dtype, out=got)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64), ("bf16", 96)])
@pytest.mark.parametrize("n1,kind,batch,prefix", [(24, "tree", 80, 0), (65, "tree", 50, 1024),
                                                  (384, "chain", 6, 0)])
def test_wide_blocks_on_long_contexts(n1, kind, batch, prefix, dtype, dim):
    rng = np.random.default_rng(n1)
    ctx = rng.integers(1800, 2100, batch)
    ctx[:6] = 2000, 2016, 2015, 2033, 1024, 3
    host, call = inputs(batch, n1, 8, 2, dim, 16, ctx, dtype, kind, prefix=prefix)
    got = tv.tree_attention_fp4(**call)
    assert bool(got.isfinite().all())
    host["ctx"][2:4] = -1
    host["ctx"][6:-1] = -1
    check(host, call, dtype, out=got)


@pytest.mark.parametrize("n1", [1, 65])
def test_blocks_and_nodes_that_are_not_finite(n1):
    """A key's NaN block makes its request NaN; a value's, its own 32 dimensions; a node's infinity
    reaches those that see it alone."""
    host, call = inputs(3, n1, 4, 2, 64, 16, [100, 300, 40], kind="star")
    clean = tv.tree_attention_fp4(**call)
    at = 16 * 32
    kc, vc = call["k_cache"].clone(), call["v_cache"].clone()
    kc[int(host["table"][0, 3]), :, at + 2 * 5] = 255
    vc[int(host["table"][1, 7]), :, at + 2 * 9 + 1] = 255
    got = tv.tree_attention_fp4(**dict(call, k_cache=kc, v_cache=vc))
    assert bool(got[0].isnan().all()) and bool(got[1, ..., 32:].isnan().all())
    assert torch.equal(got[1, ..., :32], clean[1, ..., :32]) and torch.equal(got[2], clean[2])
    if n1 > 1:
        v = call["v_new"].clone()
        v[:, 7, :, 3] = float("inf")
        got = tv.tree_attention_fp4(**dict(call, v_new=v, k_new=call["k_new"].clone()))
        others = [i for i in range(n1) if i != 7]
        rest = [d for d in range(64) if d != 3]
        assert torch.equal(got[:, others], clean[:, others]) and (got[:, 7, :, 3] == float("inf")).all()
        assert torch.equal(got[:, 7][..., rest], clean[:, 7][..., rest])


@pytest.mark.parametrize("n1", [1, 65])
def test_pages_that_are_none_and_inactive_trees(n1):
    ctx = [200, 100, 300, 64, 30, -1]
    host, call = inputs(6, n1, 8, 2, 64, 16, ctx)
    table = call["block_table"].clone()
    table[1, 3], table[2, 18] = -1, call["k_cache"].shape[0]
    table[3, 4:] = 1 << 30
    lens = call["ctx_len"].clone()
    lens[0] = table.shape[1] * 16 + 1
    out = torch.full((6, n1, 8, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    got = tv.tree_attention_fp4(**dict(call, block_table=table, ctx_len=lens), out=out)
    assert torch.isnan(got[:3]).all() and (got[5] == 3.0).all()
    host["ctx"][:3] = -1
    check(host, call, out=got)


def test_no_pages_at_all():
    host, call = inputs(2, 5, 4, 2, 64, 16, [0, 0])
    call["block_table"] = call["block_table"][:, :0].contiguous()
    call["k_cache"], call["v_cache"] = call["k_cache"][:0], call["v_cache"][:0]
    host["table"] = host["table"][:, :0]
    host["k_cache"] = host["v_cache"] = np.zeros((0, 2, 16, 64))
    check(host, call)


def test_strided_pages_large_scores_streams_and_workspaces():
    host, call = inputs(3, 5, 4, 2, 64, 16, [50, 16, 0], scale_q=40.0)
    both = torch.stack([call["k_cache"], call["v_cache"]], dim=1)
    call["k_cache"], call["v_cache"] = both[:, 0], both[:, 1]
    want = check(host, call)
    need = tv.tv_tree_attention_workspace_size(3, 5, 4, 2, 64, 0)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        assert np.array_equal(tv.tree_attention_fp4(**call, workspace=ws).double().cpu().numpy(), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = tv.tree_attention_fp4(**call)
    s.synchronize()
    assert np.array_equal(got.double().cpu().numpy(), want)


def test_attention_captured_and_replayed():
    host, call = inputs(4, 9, 8, 2, 64, 16, [100, 7, 250, 31])
    ws = torch.empty(tv.tv_tree_attention_workspace_size(4, 9, 8, 2, 64, 0), dtype=torch.uint8, device=DEV)
    out = torch.zeros((4, 9, 8, 64), dtype=torch.bfloat16, device=DEV)
    tv.tree_attention_fp4(**call, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tv.tree_attention_fp4(**call, out=out, workspace=ws)
    for lens in ([100, 7, 250, 31], [3, 7, 0, 16], [99, 0, 64, 30], [100, 7, 250, 31]):
        call["ctx_len"].copy_(torch.tensor(lens, dtype=torch.int32))
        want = tv.tree_attention_fp4(**call)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), lens


def test_offsets_beyond_32_bits():
    """Pages up to 5 GB into a cache, for reading, writing and attention."""
    ps, KH, dim = 64, 8, 128
    size = tv.fp4_cache_shape(1, KH, ps, dim)[2]
    pages = (5 << 30) // (KH * size)
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GB")
    kc, vc = (torch.zeros((1, pages, KH, size), dtype=torch.uint8, device=DEV) for _ in range(2))
    table = i32([[pages - 1, 5, pages - 2, 20000]])
    g = torch.Generator(device=DEV).manual_seed(2)
    qkv = torch.randn((1, 250, 48, dim), generator=g, device=DEV).to(torch.bfloat16)
    k, v = qkv[:, :, 32:40], qkv[:, :, 40:]
    x = torch.arange(250, device=DEV)
    slots = (table[0, x // ps] * ps + x.int() % ps)[None]
    tv.cache_commit_fp4(k[None], v[None], kc, vc, ps, i32([250]), slots)
    near = torch.arange(4, dtype=torch.int32, device=DEV)[None]
    nk, nv = (torch.zeros((1, 4, KH, size), dtype=torch.uint8, device=DEV) for _ in range(2))
    tv.cache_commit_fp4(k[None], v[None], nk, nv, ps, i32([250]), x.int()[None])
    for far, own in ((kc, nk), (vc, nv)):
        assert torch.equal(far[:, table[0].long()], own)
    a = tv.cache_read_fp4(kc, vc, ps, table, i32([250]), i32([0]), 250)
    b = tv.cache_read_fp4(nk, nv, ps, near, i32([250]), i32([0]), 250)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    args = (qkv[:, :3, :32].contiguous(), k[:, :3].contiguous(), v[:, :3].contiguous(), i32([[-1, 0, 1]]))
    ctx = i32([250])
    far = tv.tree_attention_fp4(*args, kc[0], vc[0], ps, table, ctx, 0.088)
    want = tv.tree_attention_fp4(*args, nk[0], nv[0], ps, near, ctx, 0.088)
    assert torch.equal(far, want) and bool(far.isfinite().all())


# --- a prompt's packed rows ---------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_packed_prompts_without_a_copy(dtype):
    """Prompts as tv_prompt_attention takes them, packed one behind the other in a projection's output, are
    one request of the commit: its nodes the rows, their slots those of all prompts in that order. The
    same cache as that of one request a prompt, rows of no prompt written nowhere."""
    H, KH, dim, ps, pages, n, before = 4, 2, 64, 16, 12, [40, 1, 0, 33, 17], 3
    B, T = len(n), sum(n)
    g = torch.Generator(device=DEV).manual_seed(2)
    qkv = torch.randn((before + T + 4, H + 2 * KH, dim), generator=g, device=DEV).to(TYPES[dtype])
    k, v = qkv[:, H:H + KH], qkv[:, H + KH:]
    q_start = before + np.concatenate([[0], np.cumsum(n)])
    out = tv.prompt_attention(qkv[:, :H], k, v, i32(q_start), 0.125)
    assert bool(out[before:before + T].isfinite().all())
    table = torch.full((B, 3), -1, dtype=torch.int32, device=DEV)
    free = i32(np.random.default_rng(1).permutation(pages))
    grown = tv.cache_extend(i32(n), i32([0] * B), table, free, i32([pages]), ps, max(n))
    assert not grown.status.any()
    prompt = torch.as_tensor(np.repeat(np.arange(B), n), device=DEV)        # of every row, and which of it
    row = torch.as_tensor(np.concatenate([np.arange(x) for x in n]), device=DEV)
    empty = torch.zeros((2, 1) + tv.fp4_cache_shape(pages, KH, ps, dim), dtype=torch.uint8, device=DEV)
    packed, apart = empty.clone(), empty.clone()
    slots = grown.slots[prompt, row][None]
    rows = slice(before, before + T)
    tv.cache_commit_fp4(k[rows][None, None], v[rows][None, None], packed[0], packed[1], ps, i32([T]), slots)
    k_pad, v_pad = (torch.zeros((1, B, max(n), KH, dim), dtype=TYPES[dtype], device=DEV) for _ in range(2))
    k_pad[0, prompt, row], v_pad[0, prompt, row] = k[rows], v[rows]
    tv.cache_commit_fp4(k_pad, v_pad, apart[0], apart[1], ps, i32(n), grown.slots)
    assert torch.equal(packed, apart) and int((packed != 0).flatten(2).any(-1).sum()) > 0
    back = tv.cache_read_fp4(packed[0], packed[1], ps, table, grown.seq_len, i32(q_start[:-1] - before), T,
                             dtype=TYPES[dtype])
    for got, x in zip(back, (k[rows], v[rows])):
        want = np.empty((T, KH, dim))
        for at in np.ndindex(T, KH):
            for i in range(0, dim, 32):
                want[at][i:i + 32] = D.fp4_values(*D.fp4_encode(x[at][i:i + 32].double().cpu().numpy(), largest(dtype)))
        np.testing.assert_array_equal(got[0].double().cpu().numpy(), want)


# --- a request's life --------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_prompt_pieces_then_cycles(dtype):
    """Prompts in two pieces: the first attended and written in 4 bits, the second attended behind what
    is read back; then cycles of trees whose accepted nodes follow. Every attention against the plain
    form on the values that the cache has to hold."""
    rng = np.random.default_rng(9)
    g = torch.Generator(device=DEV).manual_seed(9)
    B, H, KH, dim, ps, pages, width = 3, 8, 2, 64, 16, 40, 12
    t, scale = TYPES[dtype], 0.125
    kc, vc = (torch.zeros((1,) + tv.fp4_cache_shape(pages, KH, ps, dim), dtype=torch.uint8, device=DEV)
              for _ in range(2))
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    free, count, seq = i32(rng.permutation(pages)), i32([pages]), i32([0] * B)
    held = [[np.zeros((0, KH, dim)) for _ in range(2)] for _ in range(B)]    # keys, values as cached

    def rounded(x):
        out = np.empty(x.shape)
        for at in np.ndindex(x.shape[:2]):
            for i in range(0, dim, 32):
                codes, e = D.fp4_encode(x[at][i:i + 32], largest(dtype))
                out[at][i:i + 32] = D.fp4_values(codes, e)
        return out

    def close(got, want, mass):
        # the roundings of weights and output, and fp32's, generously: 4 half steps of sum p |v|
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= 4 * torch.finfo(t).eps / 2 * mass + 1e-6).all(), float(err.max())

    for piece in range(2):
        n = [[40, 1, 33], [25, 60, 1]][piece]
        at = np.concatenate([[0], np.cumsum(n)])
        qkv = torch.randn((at[-1], H + 2 * KH, dim), generator=g, device=DEV).to(t)
        q, k, v = qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:]
        ctx = [x[0].shape[0] for x in held]
        k_at = np.concatenate([[0], np.cumsum([c + m for c, m in zip(ctx, n)])])
        keys, values = (torch.zeros((k_at[-1], KH, dim), dtype=t, device=DEV) for _ in range(2))
        tv.cache_read_fp4(kc, vc, ps, table, seq, i32(k_at[:-1]), int(k_at[-1]),
                          out=(keys[None], values[None]))
        for b in range(B):
            keys[k_at[b] + ctx[b]:k_at[b + 1]] = k[at[b]:at[b + 1]]
            values[k_at[b] + ctx[b]:k_at[b + 1]] = v[at[b]:at[b + 1]]
        out = tv.prompt_attention(q, keys, values, i32(at), scale, k_start=i32(k_at))
        for b in range(B):
            mine = [x[at[b]:at[b + 1]].double().cpu().numpy() for x in (q, k, v)]
            want, mass, _ = D.prompt_attention(mine[0], np.concatenate([held[b][0], mine[1]]),
                                               np.concatenate([held[b][1], mine[2]]), scale)
            close(out[at[b]:at[b + 1]], want, mass)
            for i in range(2):
                held[b][i] = np.concatenate([held[b][i], rounded(mine[1 + i])])
        most = max(n)
        grown = tv.cache_extend(i32(n), seq, table, free, count, ps, most)
        assert not grown.status.any()
        # one request a row, as the commit takes them
        rows = torch.as_tensor(at[:-1, None] + np.minimum(np.arange(most), np.array(n)[:, None] - 1), device=DEV)
        tv.cache_commit_fp4(k[rows][None], v[rows][None], kc, vc, ps, i32(n), grown.slots)
        seq, count = grown.seq_len, grown.free_count
    for cycle in range(3):
        n1 = 7
        par = trees("tree", B, n1, rng)
        qkv = torch.randn((B, n1, H + 2 * KH, dim), generator=g, device=DEV).to(t)
        q, k, v = qkv[:, :, :H], qkv[:, :, H:H + KH], qkv[:, :, H + KH:]
        out = tv.tree_attention_fp4(q, k, v, i32(par), kc[0], vc[0], ps, table, seq, scale)
        new, path = [], np.full((B, n1 - 1), -1)
        for b in range(B):
            mine = [x[b].double().cpu().numpy() for x in (q, k, v)]
            m = held[b][0].shape[0]
            assert int(seq[b]) == m
            pad = [np.zeros((-(-m // ps), KH, ps, dim)) for _ in range(2)]
            for x in range(m):
                for i in range(2):
                    pad[i][x // ps, :, x % ps] = held[b][i][x]
            want, mass, _ = D.tree_attention(*mine, par[b], *pad, np.arange(len(pad[0])), m, scale)
            close(out[b], want, mass)
            nodes = sorted(D.path(par[b], int(rng.integers(0, n1))))
            path[b, :len(nodes) - 1] = nodes[1:]
            new.append(len(nodes))
            for i in range(2):
                held[b][i] = np.concatenate([held[b][i], rounded(mine[1 + i][nodes])])
        grown = tv.cache_extend(i32(new), seq, table, free, count, ps, n1)
        tv.cache_commit_fp4(k[None], v[None], kc, vc, ps, i32(new), grown.slots, path_nodes=i32(path))
        seq, count = grown.seq_len, grown.free_count
    total = int(seq.sum())
    start = np.cumsum([x[0].shape[0] for x in held]) - [x[0].shape[0] for x in held]
    gk, gv = tv.cache_read_fp4(kc, vc, ps, table, seq, i32(start), total, dtype=t)
    for got, i in ((gk, 0), (gv, 1)):
        np.testing.assert_array_equal(got[0].double().cpu().numpy(), np.concatenate([x[i] for x in held]))
