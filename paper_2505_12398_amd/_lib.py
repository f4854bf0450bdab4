"""ctypes binding of libtv (include/tv.h). Argument marshalling only."""

from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtv.so")

TV_OK, TV_ERR_INVALID_ARG, TV_ERR_UNSUPPORTED, TV_ERR_WORKSPACE, TV_ERR_HIP = range(5)
TV_DTYPE_BF16, TV_DTYPE_F32, TV_DTYPE_F16 = 0, 1, 2
TV_SIBLINGS_WITHOUT_REPLACEMENT, TV_SIBLINGS_WITH_REPLACEMENT = 0, 1
(TV_TREE_OK, TV_TREE_BAD_PARENT, TV_TREE_BAD_TOKEN, TV_TREE_DUP_SIBLING, TV_TREE_NONFINITE,
 TV_TREE_DEGENERATE, TV_TREE_ABORTED) = range(7)
TV_NODE_UNTESTED, TV_NODE_ACCEPTED, TV_NODE_REJECTED, TV_NODE_PRUNED = range(4)
TV_MAX_BATCH = 1 << 20
TV_MAX_NODES = 1024
TV_MAX_VOCAB = 1 << 20
TV_MAX_VOCAB_F32 = 1 << 19
TV_NUM_COUNTERS = 4
TV_MAX_LMHEAD_ROWS = 1 << 18
TV_MAX_HIDDEN = 1 << 16
TV_MAX_HEAD_DIM = 128
TV_MIN_PAGE, TV_MAX_PAGE = 16, 1024
TV_MAX_HISTORY = 1 << 24
TV_MAX_BIAS = 1 << 16
TV_MAX_NEW = 1 << 20
TV_MAX_LAYERS = 4096
TV_FP4_BLOCK, TV_FP4_BLOCK_BYTES = 32, 17
TV_CACHE_RELEASE = -(1 << 31)
TV_CACHE_OK, TV_CACHE_FULL, TV_CACHE_OVERFLOW, TV_CACHE_BAD_LENGTH = range(4)


class TvError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {tv_status_string(code)} (status {code})")
        self.code = code


_lib = None

_VERIFY_ARGTYPES = [
    ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,            # batch, num_nodes, vocab
    ctypes.c_void_p, ctypes.c_void_p,                          # parents, tokens
    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,          # target, draft, dtype
    ctypes.c_float, ctypes.c_void_p, ctypes.c_int32,           # temperature, uniforms, mode
    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,         # accept_len, node, bonus
    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,         # status, node_state, theta
    ctypes.c_void_p, ctypes.c_void_p,                          # p_init, counters
    ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,         # workspace, bytes, stream
]


_SAMPLE_ARGTYPES = [
    ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,            # batch, num_nodes, vocab
    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,          # parents, draft, dtype
    ctypes.c_float, ctypes.c_void_p, ctypes.c_int32,           # temperature, uniforms, mode
    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,         # tokens, status, stream
]


def load_library(path: str = LIB_PATH):
    """Load libtv.so once. Raises if it is not built."""
    global _lib
    if _lib is None:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing; build it with __graft_entry__.build()")
        lib = ctypes.CDLL(path)
        lib.tv_workspace_size.argtypes = [ctypes.c_int32] * 3
        lib.tv_workspace_size.restype = ctypes.c_size_t
        for name in ("tv_verify", "tv_verify_tokenlevel"):
            fn = getattr(lib, name)
            fn.argtypes = _VERIFY_ARGTYPES
            fn.restype = ctypes.c_int
        lib.tv_verify_noalloc.argtypes = _VERIFY_ARGTYPES[:19] + [ctypes.c_void_p]
        lib.tv_verify_noalloc.restype = ctypes.c_int
        lib.tv_verify_stats.argtypes = (_VERIFY_ARGTYPES[:11] + [ctypes.c_void_p] * 4 +
                                        _VERIFY_ARGTYPES[11:])
        lib.tv_verify_stats.restype = ctypes.c_int
        lib.tv_lmhead_workspace_size.argtypes = [ctypes.c_int32, ctypes.c_int32]
        lib.tv_lmhead_workspace_size.restype = ctypes.c_size_t
        lib.tv_lmhead_stats.argtypes = [ctypes.c_int32] * 3 + [ctypes.c_void_p] * 2 + \
            [ctypes.c_float] + [ctypes.c_void_p] * 4 + [ctypes.c_size_t, ctypes.c_void_p]
        lib.tv_lmhead_stats.restype = ctypes.c_int
        lib.tv_draft_tokens.argtypes = _SAMPLE_ARGTYPES
        lib.tv_draft_tokens.restype = ctypes.c_int
        lib.tv_commit_paths.argtypes = [ctypes.c_int32, ctypes.c_int32] + \
            [ctypes.c_void_p] * 5 + [ctypes.c_int32] + [ctypes.c_void_p] * 4
        lib.tv_commit_paths.restype = ctypes.c_int
        i32, i64, ptr, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
        lib.tv_tree_attention_workspace_size.argtypes = [i32] * 6
        lib.tv_tree_attention_workspace_size.restype = size
        lib.tv_tree_attention.argtypes = (
            [i32] * 6 + [ptr, ptr, i64, ptr, ptr, i64, ptr, ptr, i64, i32, i32, ptr, i32, ptr, ptr,
                         i32, ctypes.c_float, ptr, ptr, size, ptr])
        lib.tv_tree_attention.restype = ctypes.c_int
        lib.tv_process_logits_workspace_size.argtypes = [i32] * 3
        lib.tv_process_logits_workspace_size.restype = size
        lib.tv_process_logits.argtypes = (
            [i32] * 5 + [ptr, i32, ctypes.c_float, ptr, ptr, ptr, i32] + [ptr] * 7 +
            [i32, ptr, i32] + [ptr] * 5 + [size, ptr])
        lib.tv_process_logits.restype = ctypes.c_int
        lib.tv_cache_extend.argtypes = [i32, ptr, i32, ptr, ptr, ptr, i32, i32, i32, ptr, i32] + \
            [ptr] * 5
        lib.tv_cache_extend.restype = ctypes.c_int
        lib.tv_cache_commit.argtypes = ([i32] * 5 + [ptr, ptr, i64, i64, ptr, ptr, i64, i64, i32,
                                                     i32, ptr, i32, ptr, ptr, i32, ptr])
        lib.tv_cache_commit.restype = ctypes.c_int
        lib.tv_prompt_attention_workspace_size.argtypes = [i32] * 6
        lib.tv_prompt_attention_workspace_size.restype = size
        lib.tv_prompt_attention.argtypes = (
            [i32] * 7 + [ptr, i64, ptr, ptr, i64, ptr, ptr, ctypes.c_float, ptr, ptr, size, ptr])
        lib.tv_prompt_attention.restype = ctypes.c_int
        lib.tv_fp4_page_bytes.argtypes = [i32, i32]
        lib.tv_fp4_page_bytes.restype = size
        lib.tv_cache_commit_fp4.argtypes = [i32] + lib.tv_cache_commit.argtypes
        lib.tv_cache_commit_fp4.restype = ctypes.c_int
        lib.tv_cache_read_fp4.argtypes = (
            [i32] * 5 + [ptr, ptr, i64, i64, i32, i32, ptr, i32, ptr, ptr, ptr, i32, ptr, ptr, i64,
                         i64, ptr])
        lib.tv_cache_read_fp4.restype = ctypes.c_int
        lib.tv_tree_attention_fp4.argtypes = lib.tv_tree_attention.argtypes
        lib.tv_tree_attention_fp4.restype = ctypes.c_int
        lib.tv_status_string.argtypes = [ctypes.c_int]
        lib.tv_status_string.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def tv_status_string(code: int) -> str:
    return load_library().tv_status_string(int(code)).decode()


def tv_workspace_size(batch: int, num_nodes: int, vocab: int) -> int:
    return int(load_library().tv_workspace_size(batch, num_nodes, vocab))


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _dtype_code(t):
    import torch
    if t.dtype == torch.bfloat16:
        return TV_DTYPE_BF16
    if t.dtype == torch.float32:
        return TV_DTYPE_F32
    raise TypeError(f"logits must be bfloat16 or float32, got {t.dtype}")


def _call(name, batch, num_nodes, vocab, parents, tokens, target_logits, draft_logits, dtype,
          temperature, uniforms, mode, accept_len, accepted_node, bonus_token, status,
          node_state, node_theta, p_init, counters, workspace, workspace_bytes, stream):
    fn = getattr(load_library(), name)
    return int(fn(batch, num_nodes, vocab, _ptr(parents), _ptr(tokens), _ptr(target_logits),
                  _ptr(draft_logits), dtype, float(temperature), _ptr(uniforms), mode,
                  _ptr(accept_len), _ptr(accepted_node), _ptr(bonus_token), _ptr(status),
                  _ptr(node_state), _ptr(node_theta), _ptr(p_init), _ptr(counters),
                  _ptr(workspace), int(workspace_bytes), stream))


def tv_verify(batch, num_nodes, vocab, parents, tokens, target_logits, draft_logits, dtype,
              temperature, uniforms, mode, accept_len, accepted_node, bonus_token, status,
              node_state=None, node_theta=None, p_init=None, counters=None, workspace=None,
              workspace_bytes=0, stream=None) -> int:
    """C-ABI ``tv_verify``: pointers may be torch tensors or raw ints; returns the status."""
    return _call("tv_verify", batch, num_nodes, vocab, parents, tokens, target_logits,
                 draft_logits, dtype, temperature, uniforms, mode, accept_len, accepted_node,
                 bonus_token, status, node_state, node_theta, p_init, counters, workspace,
                 workspace_bytes, stream)


def tv_verify_noalloc(batch, num_nodes, vocab, parents, tokens, target_logits, draft_logits,
                      dtype, temperature, uniforms, mode, accept_len, accepted_node, bonus_token,
                      status, node_state=None, node_theta=None, p_init=None, counters=None,
                      stream=None) -> int:
    """C-ABI ``tv_verify_noalloc``: ``tv_verify`` on the library's own device
    scratch (no workspace argument); returns the status."""
    fn = load_library().tv_verify_noalloc
    return int(fn(batch, num_nodes, vocab, _ptr(parents), _ptr(tokens), _ptr(target_logits),
                  _ptr(draft_logits), dtype, float(temperature), _ptr(uniforms), mode,
                  _ptr(accept_len), _ptr(accepted_node), _ptr(bonus_token), _ptr(status),
                  _ptr(node_state), _ptr(node_theta), _ptr(p_init), _ptr(counters), stream))


def tv_verify_stats(batch, num_nodes, vocab, parents, tokens, target_logits, draft_logits,
                    dtype, temperature, uniforms, mode, target_max, target_sum, draft_max,
                    draft_sum, accept_len, accepted_node, bonus_token, status, node_state=None,
                    node_theta=None, p_init=None, counters=None, workspace=None,
                    workspace_bytes=0, stream=None) -> int:
    """C-ABI ``tv_verify_stats``: ``tv_verify`` with the row statistics given."""
    fn = load_library().tv_verify_stats
    return int(fn(batch, num_nodes, vocab, _ptr(parents), _ptr(tokens), _ptr(target_logits),
                  _ptr(draft_logits), dtype, float(temperature), _ptr(uniforms), mode,
                  _ptr(target_max), _ptr(target_sum), _ptr(draft_max), _ptr(draft_sum),
                  _ptr(accept_len), _ptr(accepted_node), _ptr(bonus_token), _ptr(status),
                  _ptr(node_state), _ptr(node_theta), _ptr(p_init), _ptr(counters),
                  _ptr(workspace), int(workspace_bytes), stream))


def tv_lmhead_workspace_size(rows: int, vocab: int) -> int:
    return int(load_library().tv_lmhead_workspace_size(rows, vocab))


def tv_lmhead_stats(rows, hidden_size, vocab, hidden, weight, temperature, logits, row_max,
                    row_sum, workspace, workspace_bytes, stream=None) -> int:
    """C-ABI ``tv_lmhead_stats``: pointers may be torch tensors or raw ints."""
    return int(load_library().tv_lmhead_stats(
        int(rows), int(hidden_size), int(vocab), _ptr(hidden), _ptr(weight), float(temperature),
        _ptr(logits), _ptr(row_max), _ptr(row_sum), _ptr(workspace), int(workspace_bytes),
        _ptr(stream)))


def lmhead_stats(hidden, weight, temperature, stream=None, out=None):
    """Logits and their row statistics for bf16 hidden states [..., K] and a bf16
    weight [N, K] (torch tensors on one device); returns (logits [..., N] bf16,
    row_max [...] float32, row_sum [...] float64). Raises on a non-OK return."""
    import torch
    K = hidden.shape[-1]
    N = weight.shape[0]
    lead = tuple(hidden.shape[:-1])
    M = 1
    for d in lead:
        M *= d
    dev = hidden.device
    if hidden.dtype != torch.bfloat16 or weight.dtype != torch.bfloat16:
        raise TypeError("hidden and weight must be bfloat16")
    if tuple(weight.shape) != (N, K) or not hidden.is_contiguous() or not weight.is_contiguous():
        raise ValueError("weight must be [vocab, hidden] and both tensors contiguous")
    if out is None:
        out = (torch.empty(lead + (N,), dtype=torch.bfloat16, device=dev),
               torch.empty(lead, dtype=torch.float32, device=dev),
               torch.empty(lead, dtype=torch.float64, device=dev))
    nbytes = tv_lmhead_workspace_size(M, N)
    ws = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
    if stream is None:
        stream = torch.cuda.current_stream(dev).cuda_stream if dev.type == "cuda" else None
    st = tv_lmhead_stats(M, K, N, hidden, weight, temperature, out[0], out[1], out[2], ws, nbytes,
                         stream)
    if st != TV_OK:
        raise TvError(st, "tv_lmhead_stats")
    return out


def tv_verify_tokenlevel(batch, num_nodes, vocab, parents, tokens, target_logits, draft_logits,
                         dtype, temperature, uniforms, mode, accept_len, accepted_node,
                         bonus_token, status, node_state=None, node_theta=None, p_init=None,
                         counters=None, workspace=None, workspace_bytes=0, stream=None) -> int:
    """C-ABI ``tv_verify_tokenlevel``; same arguments as :func:`tv_verify`."""
    return _call("tv_verify_tokenlevel", batch, num_nodes, vocab, parents, tokens,
                 target_logits, draft_logits, dtype, temperature, uniforms, mode, accept_len,
                 accepted_node, bonus_token, status, node_state, node_theta, p_init, counters,
                 workspace, workspace_bytes, stream)


def tv_draft_tokens(batch, num_nodes, vocab, parents, draft_logits, dtype, temperature,
                    uniforms, mode, tokens, status, stream=None) -> int:
    """C-ABI ``tv_draft_tokens``: pointers may be torch tensors or raw ints;
    returns the status."""
    return int(load_library().tv_draft_tokens(
        int(batch), int(num_nodes), int(vocab), _ptr(parents), _ptr(draft_logits), int(dtype),
        float(temperature), _ptr(uniforms), int(mode), _ptr(tokens), _ptr(status),
        _ptr(stream)))


def draft_tokens(parents, draft_logits, temperature, uniforms, mode, stream=None):
    """Draws the tokens of a batch of draft trees on the device (torch tensors
    in, (tokens, status) int32 tensors out); raises on a non-OK return."""
    import torch
    B, n1 = parents.shape
    V = draft_logits.shape[-1]
    dev = draft_logits.device
    for name, t, shape in (("parents", parents, (B, n1)), ("uniforms", uniforms, (B, n1)),
                           ("draft_logits", draft_logits, (B, n1, V))):
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
        if t.device != dev or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous on {dev}")
    if parents.dtype != torch.int32 or uniforms.dtype != torch.float32:
        raise TypeError("parents must be int32 and uniforms float32")
    tokens = torch.empty((B, n1), dtype=torch.int32, device=dev)
    status = torch.empty(B, dtype=torch.int32, device=dev)
    if stream is None:
        stream = torch.cuda.current_stream(dev).cuda_stream if dev.type == "cuda" else None
    st = tv_draft_tokens(B, n1, V, parents, draft_logits, _dtype_code(draft_logits), temperature,
                         uniforms, mode, tokens, status, stream)
    if st != TV_OK:
        raise TvError(st, "tv_draft_tokens")
    return tokens, status


TV_COMMIT_OVERFLOW, TV_COMMIT_INCONSISTENT = -1, -2


def tv_commit_paths(batch, num_nodes, parents, tokens, accepted_node, bonus_token, status,
                    max_len, path_nodes, path_tokens, path_len, stream=None) -> int:
    """C-ABI ``tv_commit_paths``: pointers may be torch tensors or raw ints;
    returns the status."""
    return int(load_library().tv_commit_paths(
        int(batch), int(num_nodes), _ptr(parents), _ptr(tokens), _ptr(accepted_node),
        _ptr(bonus_token), _ptr(status), int(max_len), _ptr(path_nodes), _ptr(path_tokens),
        _ptr(path_len), _ptr(stream)))


def commit_paths(parents, tokens, out: "VerifyOutputs", max_len: int, stream=None):
    """The committed chain of every tree after a verification (torch tensors
    in; (path_nodes, path_tokens, path_len) int32 tensors out); raises on a
    non-OK return."""
    import torch
    B, n1 = parents.shape
    dev = parents.device
    pn = torch.empty((B, max(max_len, 1)), dtype=torch.int32, device=dev)
    pt = torch.empty((B, max_len + 1), dtype=torch.int32, device=dev)
    pl = torch.empty(B, dtype=torch.int32, device=dev)
    if stream is None:
        stream = torch.cuda.current_stream(dev).cuda_stream if dev.type == "cuda" else None
    st = tv_commit_paths(B, n1, parents, tokens, out.accepted_node, out.bonus_token, out.status,
                         max_len, pn, pt, pl, stream)
    if st != TV_OK:
        raise TvError(st, "tv_commit_paths")
    return pn[:, :max_len], pt, pl


def tv_tree_attention_workspace_size(batch, num_nodes, heads, kv_heads, head_dim,
                                     prefix_len=0) -> int:
    return int(load_library().tv_tree_attention_workspace_size(
        batch, num_nodes, heads, kv_heads, head_dim, prefix_len))


def tv_tree_attention(batch, num_nodes, heads, kv_heads, head_dim, dtype, parents, q, q_stride,
                      k_new, v_new, kv_stride, k_cache, v_cache, page_stride, num_pages, page_size,
                      block_table, table_width, ctx_len, prefix_pages, prefix_len, scale, out,
                      workspace, workspace_bytes, stream=None) -> int:
    """C-ABI ``tv_tree_attention``: pointers may be torch tensors or raw ints;
    returns the status."""
    return int(load_library().tv_tree_attention(
        int(batch), int(num_nodes), int(heads), int(kv_heads), int(head_dim), int(dtype),
        _ptr(parents), _ptr(q), int(q_stride), _ptr(k_new), _ptr(v_new), int(kv_stride),
        _ptr(k_cache), _ptr(v_cache), int(page_stride), int(num_pages), int(page_size),
        _ptr(block_table), int(table_width), _ptr(ctx_len), _ptr(prefix_pages), int(prefix_len),
        float(scale), _ptr(out), _ptr(workspace), int(workspace_bytes), _ptr(stream)))


def tv_process_logits_workspace_size(batch, num_nodes, vocab) -> int:
    return int(load_library().tv_process_logits_workspace_size(batch, num_nodes, vocab))


def tv_process_logits(batch, num_nodes, vocab, first_node, num_rows, logits, dtype, temperature,
                      parents, tokens, history, max_history, history_len, prompt_len, repetition,
                      presence, frequency, bias_tokens, bias_values, max_bias, masks, num_masks,
                      mask_index, out, row_max, row_sum, workspace, workspace_bytes,
                      stream=None) -> int:
    """C-ABI ``tv_process_logits``: pointers may be torch tensors or raw ints;
    returns the status."""
    return int(load_library().tv_process_logits(
        int(batch), int(num_nodes), int(vocab), int(first_node), int(num_rows), _ptr(logits),
        int(dtype), float(temperature), _ptr(parents), _ptr(tokens), _ptr(history),
        int(max_history), _ptr(history_len), _ptr(prompt_len), _ptr(repetition), _ptr(presence),
        _ptr(frequency), _ptr(bias_tokens), _ptr(bias_values), int(max_bias), _ptr(masks),
        int(num_masks), _ptr(mask_index), _ptr(out), _ptr(row_max), _ptr(row_sum),
        _ptr(workspace), int(workspace_bytes), _ptr(stream)))


def tv_cache_extend(batch, new_len, max_new, seq_len, new_seq_len, block_table, table_width,
                    page_size, prefix_len, free_pages, num_pages, free_count, new_free_count,
                    slots, status, stream=None) -> int:
    """C-ABI ``tv_cache_extend``: pointers may be torch tensors or raw ints;
    returns the status."""
    return int(load_library().tv_cache_extend(
        int(batch), _ptr(new_len), int(max_new), _ptr(seq_len), _ptr(new_seq_len),
        _ptr(block_table), int(table_width), int(page_size), int(prefix_len), _ptr(free_pages),
        int(num_pages), _ptr(free_count), _ptr(new_free_count), _ptr(slots), _ptr(status),
        _ptr(stream)))


def tv_cache_commit(layers, batch, num_nodes, kv_heads, head_bytes, k_new, v_new,
                    new_layer_stride, node_stride, k_cache, v_cache, cache_layer_stride,
                    page_stride, num_pages, page_size, new_len, max_new, slots, path_nodes,
                    path_width, stream=None) -> int:
    """C-ABI ``tv_cache_commit`` (sizes and strides in bytes): pointers may be
    torch tensors or raw ints; returns the status."""
    return int(load_library().tv_cache_commit(
        int(layers), int(batch), int(num_nodes), int(kv_heads), int(head_bytes), _ptr(k_new),
        _ptr(v_new), int(new_layer_stride), int(node_stride), _ptr(k_cache), _ptr(v_cache),
        int(cache_layer_stride), int(page_stride), int(num_pages), int(page_size), _ptr(new_len),
        int(max_new), _ptr(slots), _ptr(path_nodes), int(path_width), _ptr(stream)))


def tv_prompt_attention_workspace_size(batch, num_queries, num_keys, heads, kv_heads,
                                       head_dim) -> int:
    return int(load_library().tv_prompt_attention_workspace_size(
        batch, num_queries, num_keys, heads, kv_heads, head_dim))


def tv_prompt_attention(batch, num_queries, num_keys, heads, kv_heads, head_dim, dtype, q, q_stride,
                        k, v, kv_stride, q_start, k_start, scale, out, workspace, workspace_bytes,
                        stream=None) -> int:
    """C-ABI ``tv_prompt_attention``: pointers may be torch tensors or raw ints;
    returns the status."""
    return int(load_library().tv_prompt_attention(
        int(batch), int(num_queries), int(num_keys), int(heads), int(kv_heads), int(head_dim),
        int(dtype), _ptr(q), int(q_stride), _ptr(k), _ptr(v), int(kv_stride), _ptr(q_start),
        _ptr(k_start), float(scale), _ptr(out), _ptr(workspace), int(workspace_bytes),
        _ptr(stream)))


def tv_fp4_page_bytes(page_size, head_dim) -> int:
    return int(load_library().tv_fp4_page_bytes(page_size, head_dim))


def tv_cache_commit_fp4(layers, batch, num_nodes, kv_heads, head_dim, dtype, k_new, v_new,
                        new_layer_stride, node_stride, k_cache, v_cache, cache_layer_stride,
                        page_stride, num_pages, page_size, new_len, max_new, slots, path_nodes,
                        path_width, stream=None) -> int:
    """C-ABI ``tv_cache_commit_fp4`` (the caches' strides in bytes): pointers may be
    torch tensors or raw ints; returns the status."""
    return int(load_library().tv_cache_commit_fp4(
        int(layers), int(batch), int(num_nodes), int(kv_heads), int(head_dim), int(dtype),
        _ptr(k_new), _ptr(v_new), int(new_layer_stride), int(node_stride), _ptr(k_cache),
        _ptr(v_cache), int(cache_layer_stride), int(page_stride), int(num_pages), int(page_size),
        _ptr(new_len), int(max_new), _ptr(slots), _ptr(path_nodes), int(path_width),
        _ptr(stream)))


def tv_cache_read_fp4(layers, batch, kv_heads, head_dim, dtype, k_cache, v_cache,
                      cache_layer_stride, page_stride, num_pages, page_size, block_table,
                      table_width, first, length, row_start, num_rows, k_out, v_out,
                      out_layer_stride, row_stride, stream=None) -> int:
    """C-ABI ``tv_cache_read_fp4`` (the caches' strides in bytes): pointers may be
    torch tensors or raw ints; returns the status."""
    return int(load_library().tv_cache_read_fp4(
        int(layers), int(batch), int(kv_heads), int(head_dim), int(dtype), _ptr(k_cache),
        _ptr(v_cache), int(cache_layer_stride), int(page_stride), int(num_pages), int(page_size),
        _ptr(block_table), int(table_width), _ptr(first), _ptr(length), _ptr(row_start),
        int(num_rows), _ptr(k_out), _ptr(v_out), int(out_layer_stride), int(row_stride),
        _ptr(stream)))


def tv_tree_attention_fp4(batch, num_nodes, heads, kv_heads, head_dim, dtype, parents, q, q_stride,
                          k_new, v_new, kv_stride, k_cache, v_cache, page_stride, num_pages,
                          page_size, block_table, table_width, ctx_len, prefix_pages, prefix_len,
                          scale, out, workspace, workspace_bytes, stream=None) -> int:
    """C-ABI ``tv_tree_attention_fp4`` (page_stride in bytes): pointers may be torch
    tensors or raw ints; returns the status."""
    return int(load_library().tv_tree_attention_fp4(
        int(batch), int(num_nodes), int(heads), int(kv_heads), int(head_dim), int(dtype),
        _ptr(parents), _ptr(q), int(q_stride), _ptr(k_new), _ptr(v_new), int(kv_stride),
        _ptr(k_cache), _ptr(v_cache), int(page_stride), int(num_pages), int(page_size),
        _ptr(block_table), int(table_width), _ptr(ctx_len), _ptr(prefix_pages), int(prefix_len),
        float(scale), _ptr(out), _ptr(workspace), int(workspace_bytes), _ptr(stream)))


def _check(name, t, shape, dtype, dev):
    """``t`` contiguous on ``dev`` with that shape and type (None passes); its address."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous on {dev}")
    return t.data_ptr()


class _On:
    """The device of a call as the current one, and the stream to enqueue on (the given one or
    that device's current stream). A given stream is the current one meanwhile: tensors made
    for the call belong to it, and are not given to another stream's work before it is done."""

    __slots__ = ("index", "before", "stream", "current")

    def __init__(self, dev, stream):
        self.index = self.current = None
        self.stream = stream
        if dev.type == "cuda":
            import torch
            index = torch.cuda.current_device() if dev.index is None else dev.index
            if index != torch.cuda.current_device():
                self.index = index
            now = torch._C._cuda_getCurrentRawStream(index)
            if stream is None:
                self.stream = now
            elif stream != now:
                # (wrapped, the default stream's handle 0 would give a new stream)
                self.current = torch.cuda.stream(torch.cuda.ExternalStream(stream, device=dev)
                                                 if stream else torch.cuda.default_stream(dev))

    def __enter__(self):
        if self.index is not None:
            import torch
            self.before = torch.cuda.current_device()
            torch.cuda.set_device(self.index)
        if self.current is not None:
            self.current.__enter__()
        return self.stream

    def __exit__(self, *_):
        if self.current is not None:
            self.current.__exit__(None, None, None)
        if self.index is not None:
            import torch
            torch.cuda.set_device(self.before)
        return False


def _on_gpu(dev, what):
    """Refuses a call that would start on tensors elsewhere, whose addresses no kernel may use."""
    if dev.type != "cuda":
        raise TvError(TV_ERR_INVALID_ARG, f"{what} on tensors of {dev}")


def _workspace(need, workspace, dev):
    import torch
    if workspace is None:
        return torch.empty(max(need, 1), dtype=torch.uint8, device=dev), need
    if workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous on {dev}")
    return workspace, workspace.numel() * workspace.element_size()


def _rows(name, t, dev, dtype, shape):
    """Stride between the nodes of a [B, N+1, heads, head_dim] tensor whose nodes follow each
    other evenly, each node's heads together (a slice of a projection's output)."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    B, n1, H, D = shape
    sb, sn, sh, sd = t.stride()
    stride = sn if n1 > 1 else sb if B > 1 else H * D
    if t.device != dev or sd != 1 and D > 1 or sh != D and H > 1 or sb != n1 * stride and B > 1:
        raise ValueError(f"{name}: nodes must lie evenly spaced on {dev}, their heads contiguous")
    return stride


def _pages(name, t, dev, dtype, shape):
    """Stride between the pages of a [pages, kv_heads, page_size, head_dim] cache."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    P, KH, ps, D = shape
    sp, sh, sr, sd = t.stride()
    if t.device != dev or (sd != 1 and D > 1) or sr != D or (sh != ps * D and KH > 1):
        raise ValueError(f"{name}: pages must be contiguous on {dev}")
    return sp if P > 1 else KH * ps * D


def tree_attention(q, k_new, v_new, parents, k_cache, v_cache, block_table, ctx_len, scale,
                   prefix_len=0, prefix_pages=None, out=None, stream=None, workspace=None):
    """Attention of all tree nodes over the paged cache and their ancestors
    (``tv_tree_attention``): q [B, N+1, heads, D], k_new and v_new
    [B, N+1, kv_heads, D] (bfloat16 or float16; views of one projection's output
    will do), k_cache and v_cache [pages, kv_heads, page_size, D], block_table
    [B, width] and ctx_len [B] int32. ``prefix_pages`` [prefix_len / page_size]
    int32 are the pages of the common prefix (default: those of the first tree that
    has it). Returns out [B, N+1, heads, D]; raises on a non-OK return."""
    import torch
    if q.dim() != 4 or k_new.dim() != 4 or k_cache.dim() != 4:
        raise ValueError("q, k_new, v_new and the caches have four dimensions")
    B, n1, H, D = q.shape
    P, KH, ps, _ = k_cache.shape
    dev, dt, i32 = q.device, q.dtype, torch.int32
    if dt != torch.bfloat16 and dt != torch.float16:
        raise TypeError(f"q must be bfloat16 or float16, got {dt}")
    q_stride = _rows("q", q, dev, dt, (B, n1, H, D))
    kv_stride = _rows("k_new", k_new, dev, dt, (B, n1, KH, D))
    if _rows("v_new", v_new, dev, dt, (B, n1, KH, D)) != kv_stride:
        raise ValueError("k_new and v_new must have the same strides")
    page_stride = _pages("k_cache", k_cache, dev, dt, (P, KH, ps, D))
    if _pages("v_cache", v_cache, dev, dt, (P, KH, ps, D)) != page_stride:
        raise ValueError("k_cache and v_cache must have the same strides")
    width = block_table.shape[-1]
    parents = _check("parents", parents, (B, n1), i32, dev)
    table = _check("block_table", block_table, (B, width), i32, dev)
    ctx = _check("ctx_len", ctx_len, (B,), i32, dev)
    prefix = _check("prefix_pages", prefix_pages, (prefix_len // ps,), i32, dev)
    if prefix_len and prefix_pages is None:
        prefix = table
    lib = load_library()
    with _On(dev, stream) as at:
        if out is None:
            out = torch.empty((B, n1, H, D), dtype=dt, device=dev)
        to = _check("out", out, (B, n1, H, D), dt, dev)
        ws, nbytes = _workspace(
            lib.tv_tree_attention_workspace_size(B, n1, H, KH, D, prefix_len), workspace, dev)
        if B:
            _on_gpu(dev, "tv_tree_attention")
        st = lib.tv_tree_attention(
            B, n1, H, KH, D, TV_DTYPE_BF16 if dt == torch.bfloat16 else TV_DTYPE_F16, parents,
            q.data_ptr(), q_stride, k_new.data_ptr(), v_new.data_ptr(), kv_stride,
            k_cache.data_ptr(), v_cache.data_ptr(), page_stride, P, ps, table, width, ctx, prefix,
            prefix_len, scale, to, ws.data_ptr(), nbytes, at)
    if st != TV_OK:
        raise TvError(st, "tv_tree_attention")
    return out


def _packed(name, t, dev, dtype, shape):
    """Stride between the rows of a [rows, heads, head_dim] tensor, each row's heads together (a
    slice of a projection's output)."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    n, H, D = shape
    sn, sh, sd = t.stride()
    if t.device != dev or sd != 1 and D > 1 or sh != D and H > 1:
        raise ValueError(f"{name}: rows must lie on {dev}, their heads contiguous")
    return sn if n > 1 else H * D


def _pages4(name, t, dev, shape):
    """Stride between the pages of a [pages, kv_heads, bytes of a head's page] cache of 4 bits."""
    if t.dtype != _uint8():
        raise TypeError(f"{name} must be torch.uint8, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    P, KH, size = shape
    sp, sh, sb = t.stride()
    if t.device != dev or sb != 1 or sh != size and KH > 1:
        raise ValueError(f"{name}: pages must be contiguous on {dev}")
    return sp if P > 1 else KH * size


def _uint8():
    import torch
    return torch.uint8


def _code16(what, dtype):
    import torch
    if dtype == torch.bfloat16:
        return TV_DTYPE_BF16
    if dtype != torch.float16:
        raise TypeError(f"{what} must be bfloat16 or float16, got {dtype}")
    return TV_DTYPE_F16


def fp4_cache_shape(pages, kv_heads, page_size, head_dim):
    """Shape of one layer's uint8 tensor of a cache of 4 bits, for keys or for values."""
    size = tv_fp4_page_bytes(page_size, head_dim)
    if not size:
        raise TvError(TV_ERR_UNSUPPORTED, f"a cache of 4 bits of pages of {page_size} rows of {head_dim}")
    return pages, kv_heads, size


def prompt_attention(q, k, v, q_start, scale, k_start=None, out=None, stream=None, workspace=None):
    """Causal attention of packed prompts (``tv_prompt_attention``): q [queries, heads, D], k and v
    [keys, kv_heads, D] (bfloat16 or float16; views of one projection's output will do); sequence b
    has the rows q_start[b] .. q_start[b + 1] - 1 of q and k_start[b] .. k_start[b + 1] - 1 of k and v
    (int32 [B + 1]; ``k_start`` None: the same), its queries being the last positions of its keys.
    Returns out [queries, heads, D] (rows of no sequence are left as they were; new tensors hold
    nothing there); raises on a non-OK return."""
    import torch
    if q.dim() != 3 or k.dim() != 3 or q_start.dim() != 1 or not len(q_start):
        raise ValueError("q, k and v have three dimensions, q_start one and at least one entry")
    (nq, H, D), (nk, KH, _), B = q.shape, k.shape, q_start.shape[0] - 1
    dev, dt, i32 = q.device, q.dtype, torch.int32
    code = _code16("q", dt)
    q_stride = _packed("q", q, dev, dt, (nq, H, D))
    kv_stride = _packed("k", k, dev, dt, (nk, KH, D))
    if _packed("v", v, dev, dt, (nk, KH, D)) != kv_stride:
        raise ValueError("k and v must have the same strides")
    if k_start is None and nk != nq:
        raise ValueError(f"{nk} keys for {nq} queries need a k_start")
    qs = _check("q_start", q_start, (B + 1,), i32, dev)
    ks = _check("k_start", k_start, (B + 1,), i32, dev)
    lib = load_library()
    with _On(dev, stream) as at:
        if out is None:
            out = torch.empty((nq, H, D), dtype=dt, device=dev)
        to = _check("out", out, (nq, H, D), dt, dev)
        ws, nbytes = _workspace(
            lib.tv_prompt_attention_workspace_size(B, nq, nk, H, KH, D), workspace, dev)
        if B and nq:
            _on_gpu(dev, "tv_prompt_attention")
        st = lib.tv_prompt_attention(B, nq, nk, H, KH, D, code, q.data_ptr(), q_stride, k.data_ptr(),
                                     v.data_ptr(), kv_stride, qs, ks, scale, to, ws.data_ptr(),
                                     nbytes, at)
    if st != TV_OK:
        raise TvError(st, "tv_prompt_attention")
    return out


def tree_attention_fp4(q, k_new, v_new, parents, k_cache, v_cache, page_size, block_table, ctx_len,
                       scale, prefix_len=0, prefix_pages=None, out=None, stream=None,
                       workspace=None):
    """``tree_attention`` over a cache of 4 bits (``tv_tree_attention_fp4``): k_cache and v_cache
    uint8 [pages, kv_heads, bytes] (``fp4_cache_shape``) of ``page_size`` rows a page."""
    import torch
    if q.dim() != 4 or k_new.dim() != 4 or k_cache.dim() != 3:
        raise ValueError("q, k_new and v_new have four dimensions, the caches three")
    B, n1, H, D = q.shape
    P, KH, _ = k_cache.shape
    dev, dt, i32 = q.device, q.dtype, torch.int32
    code = _code16("q", dt)
    q_stride = _rows("q", q, dev, dt, (B, n1, H, D))
    kv_stride = _rows("k_new", k_new, dev, dt, (B, n1, KH, D))
    if _rows("v_new", v_new, dev, dt, (B, n1, KH, D)) != kv_stride:
        raise ValueError("k_new and v_new must have the same strides")
    shape = fp4_cache_shape(P, KH, page_size, D)
    page_stride = _pages4("k_cache", k_cache, dev, shape)
    if _pages4("v_cache", v_cache, dev, shape) != page_stride:
        raise ValueError("k_cache and v_cache must have the same strides")
    width = block_table.shape[-1]
    parents = _check("parents", parents, (B, n1), i32, dev)
    table = _check("block_table", block_table, (B, width), i32, dev)
    ctx = _check("ctx_len", ctx_len, (B,), i32, dev)
    prefix = _check("prefix_pages", prefix_pages, (prefix_len // page_size,), i32, dev)
    if prefix_len and prefix_pages is None:
        prefix = table
    lib = load_library()
    with _On(dev, stream) as at:
        if out is None:
            out = torch.empty((B, n1, H, D), dtype=dt, device=dev)
        to = _check("out", out, (B, n1, H, D), dt, dev)
        ws, nbytes = _workspace(
            lib.tv_tree_attention_workspace_size(B, n1, H, KH, D, prefix_len), workspace, dev)
        if B:
            _on_gpu(dev, "tv_tree_attention_fp4")
        st = lib.tv_tree_attention_fp4(
            B, n1, H, KH, D, code, parents, q.data_ptr(), q_stride, k_new.data_ptr(),
            v_new.data_ptr(), kv_stride, k_cache.data_ptr(), v_cache.data_ptr(), page_stride, P,
            page_size, table, width, ctx, prefix, prefix_len, scale, to, ws.data_ptr(), nbytes, at)
    if st != TV_OK:
        raise TvError(st, "tv_tree_attention_fp4")
    return out


def process_logits(logits, temperature, parents=None, tokens=None, history=None, history_len=None,
                   prompt_len=None, repetition=None, presence=None, frequency=None,
                   bias_tokens=None, bias_values=None, masks=None, mask_index=None, nodes=None,
                   out=None, want_stats=True, stream=None, workspace=None):
    """Penalties, biases and masks on the logits [B, N+1, V] of tree nodes
    (``tv_process_logits``; bfloat16 or float32), into ``out`` (which may be
    ``logits``). ``nodes`` = (first, count) restricts the call to those nodes of
    every tree. Returns (out, row_max [B, N+1] float32, row_sum [B, N+1] float64),
    the statistics ``verify_batch`` takes (None without ``want_stats``); rows of
    other nodes are left as they were (new tensors hold nothing there). Raises on a
    non-OK return."""
    import torch
    B, n1, V = logits.shape
    dev, i32, f32 = logits.device, torch.int32, torch.float32
    first, count = (0, n1) if nodes is None else nodes
    dtype = _dtype_code(logits)
    H = history.shape[-1] if history is not None else 0
    nb = bias_tokens.shape[-1] if bias_tokens is not None else 0
    nm = masks.shape[0] if masks is not None else 0
    per_row, per_tree = (B, n1), (B,)
    z = _check("logits", logits, (B, n1, V), logits.dtype, dev)
    ins = (_check("parents", parents, per_row, i32, dev),
           _check("tokens", tokens, per_row, i32, dev),
           _check("history", history, (B, H), i32, dev), H,
           _check("history_len", history_len, per_tree, i32, dev),
           _check("prompt_len", prompt_len, per_tree, i32, dev),
           _check("repetition", repetition, per_tree, f32, dev),
           _check("presence", presence, per_tree, f32, dev),
           _check("frequency", frequency, per_tree, f32, dev),
           _check("bias_tokens", bias_tokens, (B, nb), i32, dev),
           _check("bias_values", bias_values, (B, nb), f32, dev), nb,
           _check("masks", masks, (nm, (V + 31) // 32), i32, dev), nm,
           _check("mask_index", mask_index, per_row, i32, dev))
    row_max = row_sum = ws = None
    nbytes = 0
    lib = load_library()
    with _On(dev, stream) as at:
        if out is None:
            out = torch.empty_like(logits)
        to = _check("out", out, (B, n1, V), logits.dtype, dev)
        if want_stats:
            row_max = torch.empty(per_row, dtype=f32, device=dev)
            row_sum = torch.empty(per_row, dtype=torch.float64, device=dev)
            ws, nbytes = _workspace(lib.tv_process_logits_workspace_size(B, n1, V), workspace, dev)
        if B and count:
            _on_gpu(dev, "tv_process_logits")
        st = lib.tv_process_logits(B, n1, V, first, count, z, dtype, temperature, *ins, to,
                                   _ptr(row_max), _ptr(row_sum), _ptr(ws), nbytes, at)
    if st != TV_OK:
        raise TvError(st, "tv_process_logits")
    return out, row_max, row_sum


@dataclass
class CacheGrowth:
    slots: object        # [B, max_new] int32
    seq_len: object      # [B] int32
    free_count: object   # [1] int32
    status: object       # [B] int32, TV_CACHE_*


def cache_extend(new_len, seq_len, block_table, free_pages, free_count, page_size, max_new,
                 prefix_len=0, out: CacheGrowth | None = None, stream=None) -> CacheGrowth:
    """Growth of all requests by ``new_len`` positions (``tv_cache_extend``; int32
    tensors): writes the block table's new entries in place and returns slots,
    new lengths, the new count of free pages and the requests' statuses (``out``
    may hold ``seq_len`` and ``free_count`` themselves). Raises on a non-OK
    return."""
    import torch
    B, dev, i32 = new_len.shape[0], block_table.device, torch.int32
    if out is None and B == 0:
        return CacheGrowth(new_len.new_empty((0, max_new)), seq_len.clone(),
                           free_count.clamp(0, free_pages.shape[0]), new_len.new_empty(0))
    width, pages, per = block_table.shape[-1], free_pages.shape[0], (B,)
    new = _check("new_len", new_len, per, i32, dev)
    seq = _check("seq_len", seq_len, per, i32, dev)
    table = _check("block_table", block_table, (B, width), i32, dev)
    free = _check("free_pages", free_pages, (pages,), i32, dev)
    count = _check("free_count", free_count, (1,), i32, dev)
    with _On(dev, stream) as at:
        if out is None:
            out = CacheGrowth(torch.empty((B, max_new), dtype=i32, device=dev),
                              torch.empty(B, dtype=i32, device=dev),
                              torch.empty(1, dtype=i32, device=dev),
                              torch.empty(B, dtype=i32, device=dev))
        slots = _check("slots", out.slots, (B, max_new), i32, dev)
        out_seq = _check("out.seq_len", out.seq_len, per, i32, dev)
        out_count = _check("out.free_count", out.free_count, (1,), i32, dev)
        status = _check("status", out.status, per, i32, dev)
        _on_gpu(dev, "tv_cache_extend")
        st = load_library().tv_cache_extend(B, new, max_new, seq, out_seq, table, width, page_size,
                                            prefix_len, free, pages, count, out_count, slots,
                                            status, at)
    if st != TV_OK:
        raise TvError(st, "tv_cache_extend")
    return out


def cache_commit(k_new, v_new, k_cache, v_cache, new_len, slots, path_nodes=None, stream=None):
    """Writes the committed nodes' keys and values of all layers into the cache
    (``tv_cache_commit``): k_new and v_new [layers, B, N+1, kv_heads, D], k_cache
    and v_cache [layers, pages, kv_heads, page_size, D] of any one type, new_len
    [B] and slots [B, max_new] as ``cache_extend`` took and gave them, path_nodes
    [B, width] from ``commit_paths`` (None: node k goes to slot k). Raises on a
    non-OK return."""
    import torch
    if k_new.dim() != 5 or k_cache.dim() != 5:
        raise ValueError("k_new, v_new and the caches have five dimensions")
    L, B, n1, KH, D = k_new.shape
    _, P, _, ps, _ = k_cache.shape
    dev, dt, i32 = k_cache.device, k_cache.dtype, torch.int32
    for name, t, lead in (("k_cache", k_cache, L), ("v_cache", v_cache, L), ("v_new", v_new, L)):
        if t.dim() != 5 or t.shape[0] != lead:
            raise ValueError(f"{name} must have five dimensions and {lead} layers")
    if L == 0:
        return
    nodes, pages = (B, n1, KH, D), (P, KH, ps, D)
    node = _rows("k_new", k_new[0], dev, dt, nodes)
    page = _pages("k_cache", k_cache[0], dev, dt, pages)
    same = _rows("v_new", v_new[0], dev, dt, nodes) == node and \
        _pages("v_cache", v_cache[0], dev, dt, pages) == page
    new_layer, layer = (k_new.stride(0), k_cache.stride(0)) if L > 1 else (0, 0)
    if not same or L > 1 and (v_new.stride(0) != new_layer or v_cache.stride(0) != layer):
        raise ValueError("keys and values must have the same strides")
    most, width, path = slots.shape[-1], 0, None
    new = _check("new_len", new_len, (B,), i32, dev)
    at_slots = _check("slots", slots, (B, most), i32, dev)
    e = k_new.element_size()
    with _On(dev, stream) as at:
        if path_nodes is not None:
            width = path_nodes.shape[-1]
            path_nodes = path_nodes.contiguous()
            path = _check("path_nodes", path_nodes, (B, width), i32, dev)
        if B and most and P:
            _on_gpu(dev, "tv_cache_commit")
        st = load_library().tv_cache_commit(
            L, B, n1, KH, D * e, k_new.data_ptr(), v_new.data_ptr(), new_layer * e, node * e,
            k_cache.data_ptr(), v_cache.data_ptr(), layer * e, page * e, P, ps, new, most,
            at_slots, path, width, at)
    if st != TV_OK:
        raise TvError(st, "tv_cache_commit")


def _layers4(k_cache, v_cache, page_size, head_dim, dev):
    """Layers, pages, key heads and strides between layers and pages of the caches of 4 bits
    [layers, pages, kv_heads, bytes]."""
    if k_cache.dim() != 4 or v_cache.dim() != 4 or v_cache.shape[0] != k_cache.shape[0]:
        raise ValueError("the caches have four dimensions and as many layers")
    L, P, KH, _ = k_cache.shape
    shape = fp4_cache_shape(P, KH, page_size, head_dim)
    if L == 0:
        return L, P, KH, 0, 0
    page = _pages4("k_cache", k_cache[0], dev, shape)
    layer = k_cache.stride(0) if L > 1 else 0
    if _pages4("v_cache", v_cache[0], dev, shape) != page or L > 1 and v_cache.stride(0) != layer:
        raise ValueError("k_cache and v_cache must have the same strides")
    return L, P, KH, layer, page


def cache_commit_fp4(k_new, v_new, k_cache, v_cache, page_size, new_len, slots, path_nodes=None,
                     stream=None):
    """``cache_commit`` into a cache of 4 bits (``tv_cache_commit_fp4``): k_new and v_new
    [layers, B, N+1, kv_heads, D] bfloat16 or float16, k_cache and v_cache uint8
    [layers, pages, kv_heads, bytes] (``fp4_cache_shape``) of ``page_size`` rows a page."""
    if k_new.dim() != 5 or v_new.dim() != 5 or v_new.shape[0] != k_new.shape[0]:
        raise ValueError("k_new and v_new have five dimensions and as many layers")
    _, B, n1, KH, D = k_new.shape
    dev, dt = k_cache.device, k_new.dtype
    code = _code16("k_new", dt)
    L, P, heads, layer, page = _layers4(k_cache, v_cache, page_size, D, dev)
    if k_new.shape[0] != L or heads != KH:
        raise ValueError(f"k_new has {k_new.shape[0]} layers of {KH} heads, the caches {L} of {heads}")
    if L == 0:
        return
    node = _rows("k_new", k_new[0], dev, dt, (B, n1, KH, D))
    new_layer = k_new.stride(0) if L > 1 else 0
    if _rows("v_new", v_new[0], dev, dt, (B, n1, KH, D)) != node or \
            L > 1 and v_new.stride(0) != new_layer:
        raise ValueError("k_new and v_new must have the same strides")
    import torch
    i32, most, width, path = torch.int32, slots.shape[-1], 0, None
    new = _check("new_len", new_len, (B,), i32, dev)
    at_slots = _check("slots", slots, (B, most), i32, dev)
    with _On(dev, stream) as at:
        if path_nodes is not None:
            width = path_nodes.shape[-1]
            path_nodes = path_nodes.contiguous()
            path = _check("path_nodes", path_nodes, (B, width), i32, dev)
        if B and most and P:
            _on_gpu(dev, "tv_cache_commit_fp4")
        st = load_library().tv_cache_commit_fp4(
            L, B, n1, KH, D, code, k_new.data_ptr(), v_new.data_ptr(), new_layer, node,
            k_cache.data_ptr(), v_cache.data_ptr(), layer, page, P, page_size, new, most, at_slots,
            path, width, at)
    if st != TV_OK:
        raise TvError(st, "tv_cache_commit_fp4")


def cache_read_fp4(k_cache, v_cache, page_size, block_table, length, row_start, rows, first=None,
                   dtype=None, out=None, stream=None):
    """Positions first[b] .. first[b] + length[b] - 1 of every request (``first`` None: from 0) out of
    a cache of 4 bits [layers, pages, kv_heads, bytes] into rows row_start[b] .. of two tensors
    [layers, ``rows``, kv_heads, D] (``tv_cache_read_fp4``; int32 tensors [B], block_table
    [B, width]): new ones of ``dtype`` (bfloat16 by default), or ``out`` = (k, v) (of ``dtype`` if
    that is given), whose rows may lie apart. Returns them; rows that no request names are left as
    they were (new tensors hold nothing there). Raises on a non-OK return."""
    import torch
    dev, i32 = k_cache.device, torch.int32
    if k_cache.dim() != 4 or block_table.dim() != 2:
        raise ValueError("the caches have four dimensions, block_table two")
    D = k_cache.shape[-1] * TV_FP4_BLOCK // (page_size * TV_FP4_BLOCK_BYTES) if page_size > 0 else 0
    L, P, KH, layer, page = _layers4(k_cache, v_cache, page_size, D, dev)
    B, width = block_table.shape
    table = _check("block_table", block_table, (B, width), i32, dev)
    n = _check("length", length, (B,), i32, dev)
    to = _check("row_start", row_start, (B,), i32, dev)
    begin = _check("first", first, (B,), i32, dev)
    with _On(dev, stream) as at:
        if out is None:
            dtype = torch.bfloat16 if dtype is None else dtype
            out = tuple(torch.empty((L, rows, KH, D), dtype=dtype, device=dev) for _ in range(2))
        k, v = out
        dt = k.dtype
        if dtype is not None and dtype != dt:
            raise TypeError(f"out is of {dt}, not of {dtype}")
        code = _code16("k", dt)
        if k.dim() != 4 or v.dim() != 4 or k.shape[0] != L or v.shape[0] != L:
            raise ValueError(f"the outputs have four dimensions and {L} layers")
        if L == 0:
            return out
        row = _packed("k", k[0], dev, dt, (rows, KH, D))
        out_layer = k.stride(0) if L > 1 else 0
        if _packed("v", v[0], dev, dt, (rows, KH, D)) != row or L > 1 and v.stride(0) != out_layer:
            raise ValueError("k and v must have the same strides")
        if B and rows:
            _on_gpu(dev, "tv_cache_read_fp4")
        st = load_library().tv_cache_read_fp4(
            L, B, KH, D, code, k_cache.data_ptr(), v_cache.data_ptr(), layer, page, P, page_size,
            table, width, begin, n, to, rows, k.data_ptr(), v.data_ptr(), out_layer, row, at)
    if st != TV_OK:
        raise TvError(st, "tv_cache_read_fp4")
    return out


def workspace_tensor(batch: int, num_nodes: int, vocab: int, device):
    """A device buffer of tv_workspace_size() bytes (torch allocations are
    256-byte aligned)."""
    import torch
    n = tv_workspace_size(batch, num_nodes, vocab)
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device), n


@dataclass
class VerifyOutputs:
    accept_len: object
    accepted_node: object
    bonus_token: object
    status: object
    node_state: object = None
    node_theta: object = None
    p_init: object = None
    counters: object = None


def verify_batch(parents, tokens, target_logits, draft_logits, temperature, uniforms, mode,
                 tokenlevel=False, want_nodes=True, want_p_init=False, want_counters=True,
                 out: VerifyOutputs | None = None, stream=None,
                 workspace=None, want_theta=None, stats=None) -> VerifyOutputs:
    """Allocate outputs and the workspace (torch, same device) unless given,
    check shapes, call the C entry point on the current stream and raise on a
    non-OK return. ``want_nodes`` asks for node states and (unless
    ``want_theta`` is False) the tested probabilities; without the latter,
    tv_verify skips the residual updates that decide nothing. ``stats`` =
    (target_max, target_sum, draft_max, draft_sum) [B, N+1] tensors calls
    tv_verify_stats (Traversal Verification with the row statistics given)."""
    import torch
    B, n1 = parents.shape
    V = target_logits.shape[-1]
    dev = target_logits.device
    for name, t, shape in (("parents", parents, (B, n1)), ("tokens", tokens, (B, n1)),
                           ("uniforms", uniforms, (B, n1)),
                           ("target_logits", target_logits, (B, n1, V)),
                           ("draft_logits", draft_logits, (B, n1, V))):
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
        if t.device != dev or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous on {dev}")
    if parents.dtype != torch.int32 or tokens.dtype != torch.int32:
        raise TypeError("parents and tokens must be int32")
    if uniforms.dtype != torch.float32:
        raise TypeError("uniforms must be float32")
    if draft_logits.dtype != target_logits.dtype:
        raise TypeError("target and draft logits must share a dtype")
    dtype = _dtype_code(target_logits)
    if out is None:
        i32 = dict(dtype=torch.int32, device=dev)
        out = VerifyOutputs(
            accept_len=torch.empty(B, **i32), accepted_node=torch.empty(B, **i32),
            bonus_token=torch.empty(B, **i32), status=torch.empty(B, **i32),
            node_state=torch.empty((B, n1), dtype=torch.int8, device=dev) if want_nodes else None,
            node_theta=torch.empty((B, n1), dtype=torch.float32, device=dev)
            if (want_nodes if want_theta is None else want_theta) else None,
            p_init=torch.empty((B, n1), dtype=torch.float32, device=dev) if want_p_init else None,
            counters=torch.empty((B, TV_NUM_COUNTERS), **i32) if want_counters else None)
    if stream is None:
        stream = torch.cuda.current_stream(dev).cuda_stream if dev.type == "cuda" else None
    if workspace is None:
        workspace, ws_bytes = workspace_tensor(B, n1, V, dev)
    else:
        ws_bytes = workspace.numel() * workspace.element_size()
    if stats is not None:
        if tokenlevel:
            raise ValueError("row statistics are taken by Traversal Verification only")
        tm, ts, dm, ds = stats
        for name, t, dt in (("target_max", tm, torch.float32), ("target_sum", ts, torch.float64),
                            ("draft_max", dm, torch.float32), ("draft_sum", ds, torch.float64)):
            if tuple(t.shape) != (B, n1) or t.dtype != dt or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {dt} tensor of shape {(B, n1)}")
        st = tv_verify_stats(B, n1, V, parents, tokens, target_logits, draft_logits, dtype,
                             temperature, uniforms, mode, tm, ts, dm, ds, out.accept_len,
                             out.accepted_node, out.bonus_token, out.status, out.node_state,
                             out.node_theta, out.p_init, out.counters, workspace, ws_bytes,
                             stream)
        if st != TV_OK:
            raise TvError(st, "tv_verify_stats")
        return out
    fn = tv_verify_tokenlevel if tokenlevel else tv_verify
    st = fn(B, n1, V, parents, tokens, target_logits, draft_logits, dtype, temperature,
            uniforms, mode, out.accept_len, out.accepted_node, out.bonus_token, out.status,
            out.node_state, out.node_theta, out.p_init, out.counters, workspace, ws_bytes,
            stream)
    if st != TV_OK:
        raise TvError(st, fn.__name__)
    return out
