"""Refusals of the operators around a verification, through the C-ABI with fake
addresses and through the binding with CPU tensors: nothing reaches the GPU."""

import contextlib

import numpy as np
import pytest
import torch

import paper_2505_12398_amd as tv

A, WS = 0x10000, 0x40000000
BAD, UNS, WSP = tv.TV_ERR_INVALID_ARG, tv.TV_ERR_UNSUPPORTED, tv.TV_ERR_WORKSPACE


def call_attention(**kw):
    args = dict(batch=2, num_nodes=5, heads=8, kv_heads=2, head_dim=64, dtype=tv.TV_DTYPE_BF16,
                parents=A, q=A, q_stride=512, k_new=A, v_new=A, kv_stride=128, k_cache=A,
                v_cache=A, page_stride=2 * 16 * 64, num_pages=10, page_size=16, block_table=A,
                table_width=4, ctx_len=A, prefix_pages=A, prefix_len=0, scale=0.125, out=A,
                workspace=WS,
                workspace_bytes=tv.tv_tree_attention_workspace_size(2, 5, 8, 2, 64, 0))
    args.update(kw)
    return tv.tv_tree_attention(**args)


@pytest.mark.parametrize("kw,want", [
    (dict(batch=-1), BAD), (dict(num_nodes=0), BAD), (dict(heads=0), BAD), (dict(kv_heads=0), BAD),
    (dict(heads=9), BAD), (dict(head_dim=0), BAD), (dict(dtype=tv.TV_DTYPE_F32), BAD),
    (dict(dtype=7), BAD), (dict(scale=0.0), BAD), (dict(scale=float("nan")), BAD),
    (dict(scale=float("inf")), BAD), (dict(scale=-1.0), BAD), (dict(prefix_len=8), BAD),
    (dict(prefix_len=-16), BAD), (dict(q_stride=504), BAD), (dict(kv_stride=120), BAD),
    (dict(page_stride=2 * 16 * 64 - 8), BAD), (dict(num_pages=-1), BAD),
    (dict(table_width=-1), BAD), (dict(parents=None), BAD), (dict(q=None), BAD),
    (dict(k_new=None), BAD), (dict(v_new=None), BAD), (dict(k_cache=None), BAD),
    (dict(v_cache=None), BAD), (dict(block_table=None), BAD), (dict(ctx_len=None), BAD),
    (dict(out=None), BAD), (dict(prefix_len=16, prefix_pages=None), BAD), (dict(q=A + 8), BAD),
    (dict(v_cache=A + 2), BAD), (dict(out=A + 8), BAD), (dict(ctx_len=A + 2), BAD),
    (dict(batch=tv.TV_MAX_BATCH + 1), UNS), (dict(num_nodes=tv.TV_MAX_NODES + 1), UNS),
    (dict(head_dim=tv.TV_MAX_HEAD_DIM + 8, q_stride=2048, kv_stride=2048, page_stride=1 << 20), UNS),
    (dict(head_dim=60), UNS), (dict(heads=2048, kv_heads=2048), UNS), (dict(page_size=24), UNS),
    (dict(page_size=8), UNS), (dict(page_size=2048), UNS), (dict(q_stride=516), UNS),
    (dict(kv_stride=132), UNS), (dict(page_stride=2 * 16 * 64 + 4), UNS),
    (dict(q_stride=1 << 28), UNS), (dict(table_width=1 << 27), UNS), (dict(workspace=None), WSP),
    (dict(workspace=WS + 128), WSP), (dict(workspace_bytes=0), WSP),
])
def test_attention_refusals(kw, want):
    assert call_attention(**kw) == want


def test_attention_empty_batch_and_workspace_size():
    assert call_attention(batch=0, q=None, k_new=None, v_new=None, parents=None, ctx_len=None,
                          out=None, workspace=None, workspace_bytes=0) == tv.TV_OK
    size = tv.tv_tree_attention_workspace_size
    for args in ((0, 5, 8, 2, 64, 0), (1, 0, 8, 2, 64, 0), (1, 5, 9, 2, 64, 0),
                 (1, 5, 8, 2, 60, 0), (1, 5, 8, 2, 136, 0), (1, 5, 8, 2, 64, -16)):
        assert size(*args) == 0, args
    assert size(1, 5, 8, 2, 64, 0) > 0 and size(256, 65, 32, 8, 128, 64) % 256 == 0


def test_attention_scale_whose_exponents_are_not_finite():
    for scale in (3.4e38, 2.4e38, 1.8e38):
        assert call_attention(scale=scale) == UNS
    assert call_attention(scale=2.0 ** 127, workspace=None) == WSP


def call_logits(**kw):
    args = dict(batch=2, num_nodes=5, vocab=1000, first_node=0, num_rows=5, logits=A,
                dtype=tv.TV_DTYPE_BF16, temperature=1.0, parents=A, tokens=A, history=A,
                max_history=10, history_len=A, prompt_len=A, repetition=A, presence=A, frequency=A,
                bias_tokens=A, bias_values=A, max_bias=3, masks=A, num_masks=2, mask_index=A,
                out=A, row_max=A, row_sum=A, workspace=WS,
                workspace_bytes=tv.tv_process_logits_workspace_size(2, 5, 1000))
    args.update(kw)
    return tv.tv_process_logits(**args)


@pytest.mark.parametrize("kw,want", [
    (dict(batch=-1), BAD), (dict(num_nodes=0), BAD), (dict(vocab=1), BAD),
    (dict(first_node=-1), BAD), (dict(num_rows=-1), BAD), (dict(first_node=1), BAD),
    (dict(num_rows=6), BAD), (dict(first_node=6, num_rows=0), BAD), (dict(max_history=-1), BAD),
    (dict(max_bias=-1), BAD), (dict(num_masks=-1), BAD), (dict(dtype=tv.TV_DTYPE_F16), BAD),
    (dict(temperature=0.0), BAD), (dict(temperature=float("nan")), BAD), (dict(logits=None), BAD),
    (dict(out=None), BAD), (dict(parents=None), BAD), (dict(tokens=None), BAD),
    (dict(history_len=None), BAD), (dict(bias_values=None), BAD), (dict(bias_tokens=None), BAD),
    (dict(masks=None), BAD), (dict(row_max=None), BAD), (dict(row_sum=None), BAD),
    (dict(logits=A + 1), BAD), (dict(dtype=tv.TV_DTYPE_F32, out=A + 2), BAD),
    (dict(row_sum=A + 4), BAD), (dict(history=A + 2), BAD), (dict(mask_index=A + 1), BAD),
    (dict(temperature=1e-5), UNS), (dict(vocab=tv.TV_MAX_VOCAB + 1), UNS),
    (dict(dtype=tv.TV_DTYPE_F32, vocab=tv.TV_MAX_VOCAB_F32 + 1), UNS),
    (dict(num_nodes=tv.TV_MAX_NODES + 1), UNS), (dict(batch=tv.TV_MAX_BATCH + 1), UNS),
    (dict(max_history=tv.TV_MAX_HISTORY + 1), UNS), (dict(max_bias=tv.TV_MAX_BIAS + 1), UNS),
    (dict(workspace=None), WSP), (dict(workspace=WS + 64), WSP), (dict(workspace_bytes=8), WSP),
])
def test_logits_refusals(kw, want):
    assert call_logits(**kw) == want


def test_logits_empty_calls_and_workspace_size():
    assert call_logits(batch=0, logits=None, out=None) == tv.TV_OK
    assert call_logits(first_node=5, num_rows=0, logits=None, out=None) == tv.TV_OK
    assert tv.tv_process_logits_workspace_size(0, 5, 1000) == 0
    assert tv.tv_process_logits_workspace_size(1, 5, 1) == 0
    # a maximum and a sum per row, chunk of the vocabulary and wavefront
    assert tv.tv_process_logits_workspace_size(256, 65, 128256) >= 256 * 65 * 16 * 4 * 8


def test_logits_of_more_workgroups_than_a_launch_has():
    assert call_logits(batch=1 << 20, num_nodes=1, num_rows=1, vocab=17 * 8192,
                       workspace_bytes=1 << 60) == UNS


def call_extend(**kw):
    args = dict(batch=2, new_len=A, max_new=4, seq_len=A, new_seq_len=A, block_table=A,
                table_width=8, page_size=16, prefix_len=0, free_pages=A, num_pages=32,
                free_count=A, new_free_count=A, slots=A, status=A)
    args.update(kw)
    return tv.tv_cache_extend(**args)


@pytest.mark.parametrize("kw,want", [
    (dict(batch=-1), BAD), (dict(max_new=-1), BAD), (dict(table_width=-1), BAD),
    (dict(page_size=0), BAD), (dict(prefix_len=-16), BAD), (dict(prefix_len=8), BAD),
    (dict(num_pages=-1), BAD), (dict(new_len=None), BAD), (dict(seq_len=None), BAD),
    (dict(new_seq_len=None), BAD), (dict(block_table=None), BAD), (dict(free_pages=None), BAD),
    (dict(free_count=None), BAD), (dict(new_free_count=None), BAD), (dict(slots=None), BAD),
    (dict(status=None), BAD), (dict(slots=A + 2), BAD), (dict(batch=tv.TV_MAX_BATCH + 1), UNS),
    (dict(page_size=48), UNS), (dict(page_size=8), UNS), (dict(num_pages=1 << 27), UNS),
    (dict(table_width=1 << 27), UNS), (dict(max_new=tv.TV_MAX_NEW + 1), UNS),
])
def test_extend_refusals(kw, want):
    assert call_extend(**kw) == want


def test_extend_empty_batch():
    assert call_extend(batch=0, new_len=None, seq_len=None, status=None) == tv.TV_OK


def test_extend_empty_batch_checks_the_counts():
    assert call_extend(batch=0, free_count=A + 2) == BAD
    assert call_extend(batch=0, new_free_count=A + 2) == BAD
    assert call_extend(batch=0, new_free_count=None) == tv.TV_OK


def call_commit(**kw):
    args = dict(layers=2, batch=2, num_nodes=5, kv_heads=2, head_bytes=128, k_new=A, v_new=A,
                new_layer_stride=1 << 16, node_stride=256, k_cache=A, v_cache=A,
                cache_layer_stride=1 << 16, page_stride=4096, num_pages=8, page_size=16, new_len=A,
                max_new=4, slots=A, path_nodes=A, path_width=3)
    args.update(kw)
    return tv.tv_cache_commit(**args)


@pytest.mark.parametrize("kw,want", [
    (dict(layers=-1), BAD), (dict(batch=-1), BAD), (dict(num_nodes=0), BAD),
    (dict(kv_heads=0), BAD), (dict(head_bytes=0), BAD), (dict(num_pages=-1), BAD),
    (dict(max_new=-1), BAD), (dict(path_width=-1), BAD), (dict(node_stride=240), BAD),
    (dict(page_stride=4080), BAD), (dict(k_new=None), BAD), (dict(v_new=None), BAD),
    (dict(k_cache=None), BAD), (dict(v_cache=None), BAD), (dict(new_len=None), BAD),
    (dict(slots=None), BAD), (dict(k_new=A + 8), BAD), (dict(v_cache=A + 4), BAD),
    (dict(path_nodes=A + 2), BAD), (dict(head_bytes=120), UNS), (dict(page_size=20), UNS),
    (dict(node_stride=264), UNS), (dict(page_stride=4104), UNS), (dict(new_layer_stride=24), UNS),
    (dict(layers=tv.TV_MAX_LAYERS + 1), UNS), (dict(max_new=tv.TV_MAX_NEW + 1), UNS),
    (dict(num_pages=1 << 27), UNS),
    (dict(cache_layer_stride=0), BAD), (dict(cache_layer_stride=4080), BAD),
    (dict(cache_layer_stride=-2048), BAD),
])
def test_commit_refusals(kw, want):
    assert call_commit(**kw) == want


def test_commit_refuses_layers_that_share_bytes():
    """Every small layout against all pairs of pages (an empty batch: nothing is launched)."""
    page, refused = 256, 0
    for layers in (1, 2, 3, 5):
        for pages in (1, 2, 3, 7):
            for step in (256, 272, 512, 768, 1280):
                for apart in list(range(-3840, 3841, 80)) + [256 * k for k in range(-9, 10)]:
                    starts = np.array([[i * apart + p * step for p in range(pages)]
                                       for i in range(layers)])
                    shared = any((np.abs(starts[i][:, None] - starts[j]) < page).any()
                                 for i in range(layers) for j in range(i))
                    got = call_commit(layers=layers, batch=0, kv_heads=1, head_bytes=16,
                                      page_size=16, num_pages=pages, page_stride=step,
                                      cache_layer_stride=apart)
                    assert got == (BAD if shared else tv.TV_OK), (layers, pages, step, apart)
                    refused += shared
    assert refused > 100
    far = dict(batch=0, layers=tv.TV_MAX_LAYERS, page_stride=1 << 62, num_pages=(1 << 27) - 1)
    assert call_commit(cache_layer_stride=(1 << 62) + 4096, **far) == tv.TV_OK
    assert call_commit(cache_layer_stride=(1 << 62) + 2048, **far) == BAD


@pytest.mark.parametrize("kw", [dict(layers=0), dict(batch=0), dict(max_new=0), dict(num_pages=0)])
def test_commit_empty_calls(kw):
    assert call_commit(**kw, k_new=None, new_len=None, slots=None) == tv.TV_OK


# --- the binding ---------------------------------------------------------------


class Streams:
    """The parts of torch.cuda that the binding asks, with streams that are numbers; wrapping the
    handle 0 makes a stream of its own, as torch does."""

    def __init__(self, monkeypatch, device, now):
        self.device, self.now, self.default = device, dict(now), 0
        patch = monkeypatch.setattr
        patch(torch.cuda, "current_device", lambda: self.device)
        patch(torch.cuda, "set_device", lambda d: setattr(self, "device", d))
        patch(torch._C, "_cuda_getCurrentRawStream", lambda d: self.now[d], raising=False)
        patch(torch.cuda, "ExternalStream", lambda h, device=None: (h or 77, self.index(device)))
        patch(torch.cuda, "default_stream", lambda device=None: (0, self.index(device)))
        patch(torch.cuda, "stream", self.stream)

    def index(self, device):
        index = device.index if isinstance(device, torch.device) else device
        return self.device if index is None else index

    @contextlib.contextmanager
    def stream(self, s):
        before = self.device, dict(self.now)
        self.device, self.now[s[1]] = s[1], s[0]
        yield
        self.device, self.now = before


@pytest.mark.parametrize("device", ["cuda", "cuda:0", "cuda:1"])
@pytest.mark.parametrize("current", [0, 5])
@pytest.mark.parametrize("given", [None, 0, 5, 9])
def test_the_stream_of_a_call_is_current_meanwhile(monkeypatch, device, current, given):
    """What a call allocates belongs to the stream that it enqueues on, the default one (handle 0)
    too; afterwards device and streams are those of before."""
    s = Streams(monkeypatch, 0, {0: current, 1: 3})
    dev = torch.device(device)
    index = dev.index or 0
    want = s.now[index] if given is None else given
    with tv._lib._On(dev, given) as at:
        assert at == want and s.device == index and s.now[index] == want
    assert s.device == 0 and s.now == {0: current, 1: 3}


def attention_tensors(dtype=torch.bfloat16):
    B, n1, H, KH, D, ps = 2, 3, 4, 2, 32, 16
    i32 = torch.int32
    return dict(q=torch.zeros(B, n1, H, D, dtype=dtype),
                k_new=torch.zeros(B, n1, KH, D, dtype=dtype),
                v_new=torch.zeros(B, n1, KH, D, dtype=dtype),
                parents=torch.tensor([[-1, 0, 1]] * B, dtype=i32),
                k_cache=torch.zeros(5, KH, ps, D, dtype=dtype),
                v_cache=torch.zeros(5, KH, ps, D, dtype=dtype),
                block_table=torch.zeros(B, 4, dtype=i32), ctx_len=torch.zeros(B, dtype=i32),
                scale=1.0)


@pytest.mark.parametrize("name,change,error", [
    ("q", lambda t: t.float(), TypeError), ("k_new", lambda t: t.half(), TypeError),
    ("v_cache", lambda t: t.float(), TypeError), ("k_new", lambda t: t[:, :2], ValueError),
    ("v_new", lambda t: t[..., :16], ValueError), ("v_cache", lambda t: t[:4], ValueError),
    ("q", lambda t: t.transpose(2, 3).contiguous().transpose(2, 3), ValueError),
    ("k_cache", lambda t: t.transpose(1, 2).contiguous().transpose(1, 2), ValueError),
    ("v_new", lambda t: torch.zeros(2, 3, 4, 32, dtype=t.dtype)[:, :, :2], ValueError),
    ("parents", lambda t: t.long(), TypeError), ("parents", lambda t: t[:1], ValueError),
    ("block_table", lambda t: t[:, ::2], ValueError), ("ctx_len", lambda t: t[:1], ValueError),
    ("k_cache", lambda t: t[0], ValueError),
])
def test_attention_binding_checks(name, change, error):
    args = attention_tensors()
    args[name] = change(args[name])
    with pytest.raises(error):
        tv.tree_attention(**args)


def test_attention_binding_reports_the_status():
    with pytest.raises(tv.TvError) as e:
        tv.tree_attention(**dict(attention_tensors(), scale=-1.0))
    assert e.value.code == BAD


@pytest.mark.parametrize("kw,error", [
    (dict(logits=torch.zeros(2, 3, 10, dtype=torch.float16)), TypeError),
    (dict(logits=torch.zeros(2, 3, 20)[..., ::2]), ValueError),
    (dict(history=torch.zeros(2, 4, dtype=torch.int64)), TypeError),
    (dict(history=torch.zeros(3, 4, dtype=torch.int32)), ValueError),
    (dict(repetition=torch.zeros(2, dtype=torch.float64)), TypeError),
    (dict(masks=torch.zeros(1, 2, dtype=torch.int32)), ValueError),
    (dict(bias_tokens=torch.zeros(2, 4, dtype=torch.int32),
          bias_values=torch.zeros(2, 3)), ValueError),
    (dict(out=torch.zeros(2, 3, 9)), ValueError),
    (dict(parents=torch.zeros(2, 3, dtype=torch.int32)), tv.TvError),
    (dict(nodes=(2, 2)), tv.TvError),
])
def test_logits_binding_checks(kw, error):
    with pytest.raises(error):
        tv.process_logits(**dict(dict(logits=torch.zeros(2, 3, 10), temperature=1.0), **kw))


def test_cache_binding_checks():
    i32 = dict(dtype=torch.int32)
    args = dict(new_len=torch.ones(2, **i32), seq_len=torch.zeros(2, **i32),
                block_table=torch.zeros(2, 4, **i32), free_pages=torch.zeros(8, **i32),
                free_count=torch.zeros(1, **i32), page_size=16, max_new=4)
    for name, value, error in (("new_len", torch.ones(2, dtype=torch.int64), TypeError),
                               ("seq_len", torch.zeros(3, **i32), ValueError),
                               ("free_count", torch.zeros(2, **i32), ValueError),
                               ("page_size", 24, tv.TvError), ("prefix_len", 8, tv.TvError)):
        with pytest.raises(error):
            tv.cache_extend(**dict(args, **{name: value}))
    grown = tv.cache_extend(**dict(args, new_len=torch.zeros(0, **i32),
                                   seq_len=torch.zeros(0, **i32),
                                   block_table=torch.zeros(0, 4, **i32)))
    assert grown.slots.shape == (0, 4) and grown.free_count.tolist() == [0]
    k, c = torch.zeros(2, 3, 4, 2, 16), torch.zeros(2, 5, 2, 16, 16)
    n, s = torch.ones(3, **i32), torch.zeros(3, 2, **i32)
    for bad, error in ((dict(v_new=k[:1]), ValueError), (dict(k_cache=c[0]), ValueError),
                       (dict(v_cache=c[:, :4]), ValueError), (dict(k_new=k.half()), TypeError),
                       (dict(new_len=n.long()), TypeError), (dict(slots=s[:2]), ValueError),
                       (dict(path_nodes=s.long()), TypeError),
                       (dict(k_cache=c.transpose(2, 3)), ValueError)):
        with pytest.raises(error):
            tv.cache_commit(**dict(dict(k_new=k, v_new=k, k_cache=c, v_cache=c.clone(), new_len=n,
                                        slots=s), **bad))


def test_tensors_that_are_not_on_a_gpu_are_refused():
    """Valid calls, whose addresses would be the host's; empty ones start nothing and pass."""
    i32 = dict(dtype=torch.int32)
    a = attention_tensors()
    z = torch.zeros(2, 3, 10)
    n, s = torch.ones(2, **i32), torch.zeros(2, 2, **i32)
    k, c = torch.zeros(1, 2, 4, 2, 16), torch.zeros(1, 5, 2, 16, 16)
    growth = (n, n * 0, torch.zeros(2, 4, **i32), torch.zeros(8, **i32), torch.zeros(1, **i32), 16, 4)
    for call in (lambda: tv.tree_attention(**a), lambda: tv.process_logits(z, 1.0),
                 lambda: tv.process_logits(z, 1.0, want_stats=False),
                 lambda: tv.cache_extend(*growth),
                 lambda: tv.cache_commit(k, k, c, c.clone(), n, s)):
        with pytest.raises(tv.TvError) as e:
            call()
        assert e.value.code == BAD
    none = {name: t[:0] if name in ("q", "k_new", "v_new", "parents", "block_table", "ctx_len")
            else t for name, t in a.items()}
    assert tv.tree_attention(**none).shape == (0, 3, 4, 32)
    assert tv.process_logits(z, 1.0, nodes=(3, 0))[0].shape == z.shape
    assert tv.process_logits(z[:0], 1.0)[0].shape == (0, 3, 10)
    tv.cache_commit(k, k, c, c.clone(), n, s[:, :0].contiguous())
    tv.cache_commit(k[:, :0], k[:, :0], c, c.clone(), n[:0], s[:0])


def test_constants_match_header():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "include", "tv.h")) as f:
        text = f.read()
    for name in ("TV_MAX_HEAD_DIM", "TV_MIN_PAGE", "TV_MAX_PAGE", "TV_MAX_HISTORY", "TV_MAX_BIAS",
                 "TV_MAX_NEW", "TV_MAX_LAYERS"):
        value = re.search(rf"#define {name}\s+([^\n/]+)", text).group(1)
        assert eval(value) == getattr(tv, name), name
    for name in ("TV_CACHE_OK", "TV_CACHE_FULL", "TV_CACHE_OVERFLOW", "TV_CACHE_BAD_LENGTH",
                 "TV_DTYPE_F16"):
        assert int(re.search(rf"\b{name}\s*=\s*(\d+)", text).group(1)) == getattr(tv, name), name
    assert tv.TV_CACHE_RELEASE == np.iinfo(np.int32).min
