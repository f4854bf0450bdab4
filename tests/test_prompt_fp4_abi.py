"""Refusals of prompt attention and of the operators of a cache of 4 bits, through the C-ABI
with fake addresses and through the binding with CPU tensors: nothing reaches the GPU."""

import os
import re

import pytest
import torch

import paper_2505_12398_amd as tv

A, WS = 0x10000, 0x40000000
BAD, UNS, WSP = tv.TV_ERR_INVALID_ARG, tv.TV_ERR_UNSUPPORTED, tv.TV_ERR_WORKSPACE


def call_prompt(**kw):
    args = dict(batch=2, num_queries=50, num_keys=70, heads=8, kv_heads=2, head_dim=64,
                dtype=tv.TV_DTYPE_BF16, q=A, q_stride=512, k=A, v=A, kv_stride=128, q_start=A,
                k_start=A, scale=0.125, out=A, workspace=WS,
                workspace_bytes=tv.tv_prompt_attention_workspace_size(2, 50, 70, 8, 2, 64))
    args.update(kw)
    return tv.tv_prompt_attention(**args)


@pytest.mark.parametrize("kw,want", [
    (dict(batch=-1), BAD), (dict(num_queries=-1), BAD), (dict(num_keys=-1), BAD),
    (dict(heads=0), BAD), (dict(kv_heads=0), BAD), (dict(heads=9), BAD), (dict(head_dim=0), BAD),
    (dict(dtype=tv.TV_DTYPE_F32), BAD), (dict(dtype=9), BAD), (dict(scale=0.0), BAD),
    (dict(scale=-1.0), BAD), (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD),
    (dict(q_stride=504), BAD), (dict(kv_stride=120), BAD), (dict(q=None), BAD), (dict(k=None), BAD),
    (dict(v=None), BAD), (dict(q_start=None), BAD), (dict(out=None), BAD), (dict(q=A + 8), BAD),
    (dict(k=A + 2), BAD), (dict(v=A + 8), BAD), (dict(out=A + 8), BAD), (dict(q_start=A + 2), BAD),
    (dict(k_start=A + 1), BAD), (dict(batch=tv.TV_MAX_BATCH + 1), UNS),
    (dict(head_dim=tv.TV_MAX_HEAD_DIM + 8, q_stride=2048, kv_stride=2048), UNS),
    (dict(head_dim=60), UNS), (dict(heads=2048, kv_heads=2048), UNS), (dict(q_stride=516), UNS),
    (dict(kv_stride=132), UNS), (dict(kv_stride=(1 << 24) + 8), UNS), (dict(scale=2.4e38), UNS),
    (dict(num_queries=1 << 26), UNS), (dict(batch=1 << 20, heads=32, kv_heads=8, q_stride=2048,
                                            kv_stride=512), UNS),
    (dict(workspace=None), WSP), (dict(workspace=WS + 128), WSP), (dict(workspace_bytes=0), WSP),
])
def test_prompt_refusals(kw, want):
    assert call_prompt(**kw) == want


def test_prompt_empty_calls_and_workspace_size():
    none = dict(q=None, k=None, v=None, q_start=None, out=None, workspace=None, workspace_bytes=0)
    assert call_prompt(batch=0, **none) == tv.TV_OK
    assert call_prompt(num_queries=0, **none) == tv.TV_OK
    size = tv.tv_prompt_attention_workspace_size
    for args in ((0, 5, 5, 8, 2, 64), (1, 0, 5, 8, 2, 64), (1, 5, -1, 8, 2, 64),
                 (1, 5, 5, 9, 2, 64), (1, 5, 5, 8, 2, 60), (1, 5, 5, 8, 2, 136)):
        assert size(*args) == 0, args
    assert size(1, 5, 5, 8, 2, 64) > 0 and size(300, 100000, 100000, 32, 8, 128) % 256 == 0


def test_prompt_keys_that_32_bits_cannot_count():
    """The kernel rounds a sequence's keys up to whole tiles of 32, and counts on for the key groups
    that have none: of 2^31 - 31 keys and more the count was negative, and the outputs NaN."""
    size = tv.tv_prompt_attention_workspace_size
    most = 2 ** 31 - 1024
    for dim in (8, 64, 128):
        assert size(2, 50, most, 8, 2, dim) == size(2, 50, 70, 8, 2, dim) > 0
        for n in (most + 1, 2 ** 31 - 31, 2 ** 31 - 1):
            assert size(2, 50, n, 8, 2, dim) == 0
            assert call_prompt(num_keys=n, head_dim=dim, q_stride=8 * dim, kv_stride=2 * dim) == UNS
    # the tiles counted of the most keys, of four key groups, and as many again that are loaded ahead
    assert (-(-most // 32) + 4 + 4 * 5) * 32 + 64 <= 2 ** 31 - 1


def call_commit(**kw):
    args = dict(layers=2, batch=2, num_nodes=5, kv_heads=2, head_dim=64, dtype=tv.TV_DTYPE_BF16,
                k_new=A, v_new=A, new_layer_stride=1 << 16, node_stride=128, k_cache=A, v_cache=A,
                cache_layer_stride=1 << 16, page_stride=1088, num_pages=8, page_size=16, new_len=A,
                max_new=4, slots=A, path_nodes=A, path_width=3)
    args.update(kw)
    return tv.tv_cache_commit_fp4(**args)


@pytest.mark.parametrize("kw,want", [
    (dict(layers=-1), BAD), (dict(batch=-1), BAD), (dict(num_nodes=0), BAD),
    (dict(kv_heads=0), BAD), (dict(head_dim=0), BAD), (dict(num_pages=-1), BAD),
    (dict(max_new=-1), BAD), (dict(path_width=-1), BAD), (dict(dtype=tv.TV_DTYPE_F32), BAD),
    (dict(node_stride=120), BAD), (dict(page_stride=1072), BAD), (dict(k_new=None), BAD),
    (dict(v_new=None), BAD), (dict(k_cache=None), BAD), (dict(v_cache=None), BAD),
    (dict(new_len=None), BAD), (dict(slots=None), BAD), (dict(k_new=A + 8), BAD),
    (dict(v_cache=A + 4), BAD), (dict(path_nodes=A + 2), BAD), (dict(head_dim=72), UNS),
    (dict(head_dim=160, node_stride=320, page_stride=1 << 14), UNS), (dict(page_size=20), UNS),
    (dict(page_size=8), UNS), (dict(page_size=2048, page_stride=1 << 20), UNS),
    (dict(node_stride=132), UNS), (dict(page_stride=1096), UNS), (dict(new_layer_stride=12), UNS),
    (dict(cache_layer_stride=(1 << 16) + 8), UNS), (dict(layers=tv.TV_MAX_LAYERS + 1), UNS),
    (dict(max_new=tv.TV_MAX_NEW + 1), UNS), (dict(num_pages=1 << 27), UNS),
    (dict(kv_heads=1 << 11, node_stride=1 << 17, page_stride=1 << 24), UNS),
    (dict(cache_layer_stride=0), BAD), (dict(cache_layer_stride=1072), BAD),
    (dict(cache_layer_stride=-544), BAD),
])
def test_commit_refusals(kw, want):
    assert call_commit(**kw) == want


def test_commit_refuses_one_cache_for_keys_and_values():
    """Every row would be written twice, in any order."""
    assert call_commit(v_new=A + (1 << 20)) == BAD
    for none in (dict(layers=0), dict(batch=0), dict(max_new=0), dict(num_pages=0)):
        assert call_commit(v_new=A + (1 << 20), **none) == tv.TV_OK


@pytest.mark.parametrize("kw", [dict(layers=0), dict(batch=0), dict(max_new=0), dict(num_pages=0)])
def test_commit_empty_calls(kw):
    assert call_commit(**kw, k_new=None, new_len=None, slots=None) == tv.TV_OK


def call_read(**kw):
    args = dict(layers=2, batch=2, kv_heads=2, head_dim=64, dtype=tv.TV_DTYPE_F16, k_cache=A,
                v_cache=A, cache_layer_stride=1 << 16, page_stride=1088, num_pages=8, page_size=16,
                block_table=A, table_width=4, first=A, length=A, row_start=A, num_rows=100, k_out=A,
                v_out=A, out_layer_stride=1 << 16, row_stride=128)
    args.update(kw)
    return tv.tv_cache_read_fp4(**args)


@pytest.mark.parametrize("kw,want", [
    (dict(layers=-1), BAD), (dict(batch=-1), BAD), (dict(kv_heads=0), BAD), (dict(head_dim=0), BAD),
    (dict(num_pages=-1), BAD), (dict(table_width=-1), BAD), (dict(num_rows=-1), BAD),
    (dict(dtype=tv.TV_DTYPE_F32), BAD), (dict(row_stride=120), BAD), (dict(page_stride=1072), BAD),
    (dict(k_cache=None), BAD), (dict(v_cache=None), BAD), (dict(block_table=None), BAD),
    (dict(length=None), BAD), (dict(row_start=None), BAD), (dict(k_out=None), BAD),
    (dict(v_out=None), BAD), (dict(k_out=A + 8), BAD), (dict(k_cache=A + 4), BAD),
    (dict(length=A + 2), BAD), (dict(first=A + 1), BAD), (dict(head_dim=48), UNS),
    (dict(page_size=48), UNS), (dict(row_stride=132), UNS), (dict(out_layer_stride=12), UNS),
    (dict(page_stride=1096), UNS), (dict(cache_layer_stride=8), UNS),
    (dict(layers=tv.TV_MAX_LAYERS + 1), UNS), (dict(batch=tv.TV_MAX_BATCH + 1), UNS),
    (dict(table_width=1 << 27), UNS), (dict(num_pages=1 << 27), UNS),
])
def test_read_refusals(kw, want):
    assert call_read(**kw) == want


@pytest.mark.parametrize("kw", [dict(layers=0), dict(batch=0), dict(num_rows=0)])
def test_read_empty_calls(kw):
    assert call_read(**kw, length=None, k_out=None, block_table=None) == tv.TV_OK


def rows_meet(layers, layer, rows, row, size, at):
    """Whether two rows of ``size`` bytes of k_out at 0 and v_out at ``at`` share bytes."""
    begins = sorted(a + x * layer + r * row for a in (0, at) for x in range(layers) for r in range(rows))
    return any(b - a < size for a, b in zip(begins, begins[1:]))


# (strides in elements, ``at`` the bytes from k_out to v_out)
OVERLAPS = [dict(out_layer_stride=0), dict(out_layer_stride=8), dict(out_layer_stride=99 * 128),
            dict(out_layer_stride=-1024), dict(out_layer_stride=120, row_stride=256),
            dict(out_layer_stride=136, row_stride=256),
            dict(out_layer_stride=128, row_stride=256, layers=3),
            dict(at=16), dict(at=240), dict(at=-240), dict(at=99 * 256), dict(at=128, layers=1, num_rows=3),
            dict(at=(1 << 17) + 99 * 256), dict(at=-(1 << 17)),
            dict(at=512, out_layer_stride=128, row_stride=512, layers=3),
            dict(at=240, out_layer_stride=512 * 100, row_stride=256)]


@pytest.mark.parametrize("kw", OVERLAPS)
def test_read_refuses_outputs_that_overlap(kw):
    """Layers, or keys and values, whose rows share bytes were written in any order."""
    kw = dict(kw)
    at = kw.pop("at", 1 << 22)
    size = 2 * 2 * 64
    full = dict(layers=2, out_layer_stride=1 << 16, row_stride=128, num_rows=100)
    full.update(kw)
    assert rows_meet(full["layers"], 2 * full["out_layer_stride"], full["num_rows"], 2 * full["row_stride"],
                     size, at)
    assert call_read(**kw, k_out=WS, v_out=WS + at) == BAD


def test_read_refuses_one_output_for_two_caches():
    assert call_read(k_cache=A, v_cache=A + 16) == BAD


def call_attention(**kw):
    args = dict(batch=2, num_nodes=5, heads=8, kv_heads=2, head_dim=64, dtype=tv.TV_DTYPE_BF16,
                parents=A, q=A, q_stride=512, k_new=A, v_new=A, kv_stride=128, k_cache=A,
                v_cache=A, page_stride=1088, num_pages=10, page_size=16, block_table=A,
                table_width=4, ctx_len=A, prefix_pages=A, prefix_len=0, scale=0.125, out=A,
                workspace=WS,
                workspace_bytes=tv.tv_tree_attention_workspace_size(2, 5, 8, 2, 64, 0))
    args.update(kw)
    return tv.tv_tree_attention_fp4(**args)


@pytest.mark.parametrize("kw,want", [
    (dict(batch=-1), BAD), (dict(heads=9), BAD), (dict(dtype=tv.TV_DTYPE_F32), BAD),
    (dict(scale=0.0), BAD), (dict(prefix_len=8), BAD), (dict(q_stride=504), BAD),
    (dict(kv_stride=120), BAD), (dict(page_stride=1072), BAD), (dict(parents=None), BAD),
    (dict(k_cache=None), BAD), (dict(v_cache=A + 8), BAD), (dict(ctx_len=A + 2), BAD),
    (dict(head_dim=40), UNS), (dict(head_dim=72, q_stride=576, kv_stride=144, page_stride=2048), UNS),
    (dict(page_size=24), UNS), (dict(page_stride=1096), UNS),
    (dict(page_stride=(1 << 29) + 16), UNS), (dict(q_stride=1 << 28), UNS),
    (dict(workspace=None), WSP), (dict(workspace_bytes=0), WSP),
])
def test_attention_refusals(kw, want):
    assert call_attention(**kw) == want


def test_rows_that_32_bits_cannot_count():
    """Over a prefix the rows of all trees are one item's: of nearly 2^31 of them, the indexes of the
    last team's rows overflowed, and queries were read before their tensor."""
    size = tv.tv_tree_attention_workspace_size
    assert size(16384 * 64 - 8, 1024, 2, 1, 8, 16) > 0             # 2^31 - 2^14 rows
    for batch, nodes, heads in ((2 ** 20 - 7, 1024, 2), (2 ** 20 - 1, 1024, 2), (46340, 46, 1007)):
        assert batch * nodes * heads <= 2 ** 31 - 1
        few = batch * nodes * heads <= 2 ** 31 - 2 ** 14
        assert (size(batch, nodes, heads, 1, 8, 16) > 0) == few
        if not few:
            assert call_attention(batch=batch, num_nodes=nodes, heads=heads, kv_heads=1, head_dim=32, q_stride=64,
                                  kv_stride=32, prefix_len=16) == UNS


@pytest.mark.parametrize("page_size", [16, 64, 512])
def test_tables_whose_positions_32_bits_cannot_count(page_size):
    """A context within 32 of 2^31 overflowed the count of its tiles, and was read before the table."""
    most, stride = (2 ** 31 - 1024) // page_size, tv.tv_fp4_page_bytes(page_size, 64) * 2
    for width in (most + 1, (2 ** 31 - 1) // page_size):
        assert call_attention(page_size=page_size, page_stride=stride, table_width=width) == UNS
        # (of 16 bits)
        assert tv.tv_tree_attention(
            2, 5, 8, 2, 64, tv.TV_DTYPE_BF16, A, A, 512, A, A, 128, A, A, 128 * page_size, 10, page_size, A,
            width, A, A, 0, 0.125, A, WS, tv.tv_tree_attention_workspace_size(2, 5, 8, 2, 64, 0)) == UNS
    # the widest table is taken (as far as its missing workspace)
    assert call_attention(page_size=page_size, page_stride=stride, table_width=most, workspace=None) == WSP


def test_page_bytes():
    for ps in (16, 64, 1024):
        for dim in (32, 64, 96, 128):
            assert tv.tv_fp4_page_bytes(ps, dim) == ps * dim // 32 * 17
            assert tv.fp4_cache_shape(5, 3, ps, dim) == (5, 3, ps * dim // 32 * 17)
    for ps, dim in ((8, 64), (24, 64), (2048, 64), (0, 64), (16, 0), (16, 48), (16, 160), (16, -32)):
        assert tv.tv_fp4_page_bytes(ps, dim) == 0
        with pytest.raises(tv.TvError):
            tv.fp4_cache_shape(5, 3, ps, dim)


# --- the binding ---------------------------------------------------------------

I32 = dict(dtype=torch.int32)
BF = torch.bfloat16


def prompt_tensors(dtype=BF):
    qkv = torch.zeros(9, 8, 32, dtype=dtype)
    return dict(q=qkv[:, :4], k=qkv[:, 4:6], v=qkv[:, 6:], q_start=torch.tensor([0, 4, 9], **I32),
                scale=1.0)


@pytest.mark.parametrize("name,change,error", [
    ("q", lambda t: t.float(), TypeError), ("k", lambda t: t.half(), TypeError),
    ("k", lambda t: t[..., :16], ValueError), ("v", lambda t: t[:8], ValueError),
    ("k", lambda t: t[:8], ValueError), ("q", lambda t: t[:, ::2], ValueError),
    ("v", lambda t: t.contiguous(), ValueError), ("q", lambda t: t[0], ValueError),
    ("q", lambda t: t.transpose(1, 2).contiguous().transpose(1, 2), ValueError),
    ("q_start", lambda t: t.long(), TypeError), ("q_start", lambda t: t[:0], ValueError),
    ("k_start", lambda t: torch.zeros(2, **I32), ValueError),
    ("k_start", lambda t: torch.zeros(3), TypeError),
    ("out", lambda t: torch.zeros(9, 4, 32), TypeError),
    ("out", lambda t: torch.zeros(8, 4, 32, dtype=BF), ValueError),
    ("scale", lambda t: -1.0, tv.TvError), ("q", lambda t: t, tv.TvError),
])
def test_prompt_binding_checks(name, change, error):
    args = prompt_tensors()
    args[name] = change(args.get(name))
    with pytest.raises(error):
        tv.prompt_attention(**args)


def fp4_tensors():
    B, n1, H, KH, D, ps = 2, 3, 4, 2, 32, 16
    shape = tv.fp4_cache_shape(5, KH, ps, D)
    return dict(q=torch.zeros(B, n1, H, D, dtype=BF), k_new=torch.zeros(B, n1, KH, D, dtype=BF),
                v_new=torch.zeros(B, n1, KH, D, dtype=BF),
                parents=torch.tensor([[-1, 0, 1]] * B, **I32),
                k_cache=torch.zeros(shape, dtype=torch.uint8),
                v_cache=torch.zeros(shape, dtype=torch.uint8), page_size=ps,
                block_table=torch.zeros(B, 4, **I32), ctx_len=torch.zeros(B, **I32), scale=1.0)


@pytest.mark.parametrize("name,change,error", [
    ("q", lambda t: t.float(), TypeError), ("k_new", lambda t: t.half(), TypeError),
    ("k_cache", lambda t: t.to(BF), TypeError), ("v_cache", lambda t: t[:4], ValueError),
    ("k_cache", lambda t: t[..., :-16], ValueError), ("k_cache", lambda t: t[0], ValueError),
    ("v_cache", lambda t: torch.cat([t, t], dim=2)[:, :, :t.shape[2]], ValueError),
    ("page_size", lambda t: 32, ValueError), ("page_size", lambda t: 24, tv.TvError),
    ("block_table", lambda t: t[:, ::2], ValueError), ("ctx_len", lambda t: t[:1], ValueError),
    ("scale", lambda t: -1.0, tv.TvError), ("q", lambda t: t, tv.TvError),
])
def test_attention_binding_checks(name, change, error):
    args = fp4_tensors()
    args[name] = change(args[name])
    with pytest.raises(error):
        tv.tree_attention_fp4(**args)


def test_cache_binding_checks():
    k = torch.zeros(2, 3, 4, 2, 32, dtype=BF)
    c = torch.zeros((2,) + tv.fp4_cache_shape(5, 2, 16, 32), dtype=torch.uint8)
    n, s = torch.ones(3, **I32), torch.zeros(3, 2, **I32)
    args = dict(k_new=k, v_new=k, k_cache=c, v_cache=c.clone(), page_size=16, new_len=n, slots=s)
    for bad, error in ((dict(v_new=k[:1]), ValueError), (dict(k_cache=c[0]), ValueError),
                       (dict(v_cache=c[:, :4]), ValueError), (dict(k_new=k.half()), TypeError),
                       (dict(k_new=k.float(), v_new=k.float()), TypeError),
                       (dict(k_cache=c.to(BF)), TypeError), (dict(page_size=32), ValueError),
                       (dict(page_size=20), tv.TvError), (dict(new_len=n.long()), TypeError),
                       (dict(slots=s[:2]), ValueError), (dict(path_nodes=s.long()), TypeError),
                       (dict(k_new=k[:, :, :, :1], v_new=k[:, :, :, :1]), ValueError),
                       (dict(k_cache=c[..., ::2]), ValueError), ({}, tv.TvError)):
        with pytest.raises(error):
            tv.cache_commit_fp4(**dict(args, **bad))
    tv.cache_commit_fp4(**dict(args, slots=s[:, :0].contiguous()))
    tv.cache_commit_fp4(**dict(args, k_new=k[:, :0], v_new=k[:, :0], new_len=n[:0], slots=s[:0]))
    args = dict(k_cache=c, v_cache=c.clone(), page_size=16, block_table=s, length=n, row_start=n,
                rows=7)
    out = torch.zeros(2, 7, 2, 32, dtype=BF)
    for bad, error in ((dict(v_cache=c[:1]), ValueError), (dict(k_cache=c[0]), ValueError),
                       (dict(length=n.long()), TypeError), (dict(row_start=n[:2]), ValueError),
                       (dict(first=n[:2]), ValueError), (dict(block_table=n), ValueError),
                       (dict(dtype=torch.float32), TypeError), (dict(page_size=0), tv.TvError),
                       (dict(out=(out, out.half())), TypeError), (dict(out=(out, out[:1])), ValueError),
                       (dict(out=(out[:, :6], out[:, :6])), ValueError), ({}, tv.TvError)):
        with pytest.raises(error):
            tv.cache_read_fp4(**dict(args, **bad))
    assert tv.cache_read_fp4(**dict(args, rows=0))[0].shape == (2, 0, 2, 32)


def test_read_into_outputs_of_another_type():
    c = torch.zeros((2,) + tv.fp4_cache_shape(5, 2, 16, 32), dtype=torch.uint8)
    n = torch.ones(3, **I32)
    for dt, other in ((BF, torch.float16), (torch.float16, BF)):
        out = tuple(torch.zeros(2, 0, 2, 32, dtype=dt) for _ in range(2))
        args = (c, c.clone(), 16, torch.zeros(3, 2, **I32), n, n, 0)
        assert tv.cache_read_fp4(*args, out=out) is out and tv.cache_read_fp4(*args, dtype=dt, out=out) is out
        with pytest.raises(TypeError):
            tv.cache_read_fp4(*args, dtype=other, out=out)


def test_empty_calls_on_tensors_that_are_not_on_a_gpu():
    a = prompt_tensors()
    assert tv.prompt_attention(**dict(a, q_start=a["q_start"][:1])).shape == (9, 4, 32)
    assert tv.prompt_attention(**dict(a, q=a["q"][:0], k=a["k"][:0], v=a["v"][:0])).shape == (0, 4, 32)
    a = fp4_tensors()
    none = {x: t[:0] if x in ("q", "k_new", "v_new", "parents", "block_table", "ctx_len") else t
            for x, t in a.items()}
    assert tv.tree_attention_fp4(**none).shape == (0, 3, 4, 32)


def test_constants_match_header():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "include", "tv.h")) as f:
        text = f.read()
    for name in ("TV_FP4_BLOCK", "TV_FP4_BLOCK_BYTES"):
        assert int(re.search(rf"#define {name}\s+(\d+)", text).group(1)) == getattr(tv, name), name
