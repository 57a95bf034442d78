"""ctypes binding of the C ABI in include/domino.h (argument marshalling only).

Every function here has the name of the C entry point it calls.  Tensor arguments may be
torch tensors (their data_ptr() is passed) or raw integer addresses; the library itself
does all the work.  Loading fails loudly when libdomino.so has not been built: there is no
fallback implementation.
"""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdomino.so")

DOMINO_OK = 0
DOMINO_ERR_INVALID_ARG = -1
DOMINO_ERR_UNSUPPORTED = -2
DOMINO_ERR_CUDA = -3
DOMINO_ERR_TIMEOUT = -4
DOMINO_ERR_BAD_TOKEN = -5
DOMINO_ERR_BAD_PAGE = -6

# every entry point declared in include/domino.h
SYMBOLS = ("domino_workspace_bytes", "domino_draft_step", "domino_workspace_bytes_host",
           "domino_draft_step_host", "domino_check_status", "domino_status_string",
           "domino_abi_version", "domino_launches_per_step", "domino_timing_begin", "domino_timing_end",
           "domino_draft_step_static_scratch", "domino_verify_tree_greedy", "domino_rollout_workspace_bytes",
           "domino_rollout_greedy", "domino_rollout_sample", "domino_input_table_bytes",
           "domino_build_input_table", "domino_launches_per_step_table", "domino_debug_hold",
           "domino_verify_tree_sample", "domino_rollout_sample_gumbel", "domino_sample_filtered",
           "domino_verify_tree_filtered", "domino_distill_loss", "domino_distill_grad", "domino_distill_loss_grad",
           "domino_rope", "domino_rope_append", "domino_attend_workspace_bytes", "domino_attend_paged",
           "domino_cache_commit")

DOMINO_STATIC_SCRATCH_BYTES = 16 << 20

# element types of logits (domino_sample_filtered, domino_verify_tree_filtered, domino_distill_*) and of caches
DOMINO_F32 = 0
DOMINO_BF16 = 1
DOMINO_F16 = 2

# domino_distill_*: what stands for the ids outside the teacher's list
DOMINO_DISTILL_RENORM = 0
DOMINO_DISTILL_TAIL = 1

# domino_rope, domino_rope_append: which elements of a head form a pair
DOMINO_ROPE_HALF = 0
DOMINO_ROPE_PAIRS = 1

# domino_attend_paged: which of its sequence's keys a new token sees
DOMINO_MASK_CAUSAL = 0
DOMINO_MASK_FULL = 1
DOMINO_MASK_TREE = 2

# domino_debug_hold: what a GRU CTA withholds (a failure-detection test hook)
DOMINO_HOLD_OFF = 0
DOMINO_HOLD_STATE = 1
DOMINO_HOLD_CLEAR_BARRIER = 2
DOMINO_HOLD_ROW_COPY = 3
DOMINO_HOLD_KEY_TILE = 4

KERNEL_KINDS = ("gather", "gru_input_proj", "w1_hidden_proj", "gru", "vocab_gemm_softmax_topk", "merge_tree",
                "rollout_base_gemm", "rollout_steps", "tree_verify", "sample_filtered", "distill",
                "rope", "attend", "cache_commit")


class domino_head_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("emb", "w_ih", "w_hh", "b_ih", "b_hh", "w1", "b1", "w2", "b2")] + \
               [("Ds", ctypes.c_int), ("R", ctypes.c_int), ("x_table", ctypes.c_void_p)]


class domino_kv_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("page_stride", "token_stride", "head_stride")] + \
               [(n, ctypes.c_int) for n in ("pages", "page", "heads", "head_dim", "dtype")]


class domino_kv_batch(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("table_width", ctypes.c_int),
                ("kv_len", ctypes.c_void_p), ("start", ctypes.c_void_p), ("B", ctypes.c_int)]


class DominoError(RuntimeError):
    def __init__(self, code: int, what: str = ""):
        super().__init__(f"{what}: {domino_status_string(code)} ({code})" if what else domino_status_string(code))
        self.code = code


_lib = None


def load():
    """Load libdomino.so (raises if it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                           "(there is no non-CUDA implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.domino_workspace_bytes.argtypes = [I] * 8
    lib.domino_workspace_bytes.restype = S
    lib.domino_workspace_bytes_host.argtypes = [I] * 8
    lib.domino_workspace_bytes_host.restype = S
    step_args = [P, P, P, ctypes.POINTER(domino_head_weights)] + [I] * 6 + [P] * 6 + [P, S, P]
    lib.domino_draft_step.argtypes = step_args
    lib.domino_draft_step.restype = I
    lib.domino_draft_step_host.argtypes = step_args
    lib.domino_draft_step_host.restype = I
    lib.domino_check_status.argtypes = [P, P]
    lib.domino_check_status.restype = I
    lib.domino_status_string.argtypes = [I]
    lib.domino_status_string.restype = ctypes.c_char_p
    lib.domino_abi_version.argtypes = []
    lib.domino_abi_version.restype = I
    lib.domino_launches_per_step.argtypes = [I] * 8
    lib.domino_launches_per_step.restype = I
    lib.domino_launches_per_step_table.argtypes = [I] * 8
    lib.domino_launches_per_step_table.restype = I
    lib.domino_timing_begin.argtypes = [I]
    lib.domino_timing_begin.restype = I
    lib.domino_timing_end.argtypes = [P, P, I]
    lib.domino_timing_end.restype = I
    lib.domino_draft_step_static_scratch.argtypes = [P, P, P, ctypes.POINTER(domino_head_weights)] + [I] * 6 + \
        [P] * 6 + [P, P]
    lib.domino_draft_step_static_scratch.restype = I
    lib.domino_verify_tree_greedy.argtypes = [P, P, P, I, I, I, P, P, P, P, P]
    lib.domino_verify_tree_greedy.restype = I
    lib.domino_verify_tree_sample.argtypes = [P, P, P, P, ctypes.c_float, I, I, I, P, P, P, P, P]
    lib.domino_verify_tree_sample.restype = I
    lib.domino_rollout_workspace_bytes.argtypes = [I] * 6
    lib.domino_rollout_workspace_bytes.restype = ctypes.c_size_t
    lib.domino_rollout_greedy.argtypes = [P, P, P, ctypes.POINTER(domino_head_weights)] + [I] * 4 + [P, P, P,
                                                                                               ctypes.c_size_t, P]
    lib.domino_rollout_greedy.restype = I
    lib.domino_rollout_sample.argtypes = [P, P, P, P, ctypes.POINTER(domino_head_weights)] + [I] * 4 + [
        P, P, P, ctypes.c_size_t, P]
    lib.domino_rollout_sample.restype = I
    lib.domino_rollout_sample_gumbel.argtypes = [P, P, ctypes.c_uint64, P, ctypes.POINTER(domino_head_weights)] + [
        I] * 4 + [P, P, P, ctypes.c_size_t, P]
    lib.domino_rollout_sample_gumbel.restype = I
    lib.domino_input_table_bytes.argtypes = [I, I]
    lib.domino_input_table_bytes.restype = S
    lib.domino_build_input_table.argtypes = [P, P, I, I, I, P, P]
    lib.domino_build_input_table.restype = I
    lib.domino_debug_hold.argtypes = [I, I, I]
    lib.domino_debug_hold.restype = I
    L, F = ctypes.c_int64, ctypes.c_float
    lib.domino_sample_filtered.argtypes = [P, I, L, P, P, P, P, P, I, I, P, P, P]
    lib.domino_sample_filtered.restype = I
    lib.domino_verify_tree_filtered.argtypes = [P, I, L, P, P, P, P, P, P, P, I, I, I, P, P, P, P, P, P]
    lib.domino_verify_tree_filtered.restype = I
    lib.domino_distill_loss.argtypes = [P, I, L, P, P, P, F, I, I, I, I, P, P, P]
    lib.domino_distill_loss.restype = I
    lib.domino_distill_grad.argtypes = [P, I, L, P, P, P, P, F, I, I, I, I, P, P, L, P]
    lib.domino_distill_grad.restype = I
    lib.domino_distill_loss_grad.argtypes = [P, I, L, P, P, P, P, F, I, I, I, I, P, P, P, L, P]
    lib.domino_distill_loss_grad.restype = I
    cache, batch = ctypes.POINTER(domino_kv_cache), ctypes.POINTER(domino_kv_batch)
    lib.domino_rope.argtypes = [P, I, L, L, P, P, F, I, I, I, I, I, I, P, L, L, P]
    lib.domino_rope.restype = I
    lib.domino_rope_append.argtypes = [P, L, P, L, P, L, P, P, I, P, F, I, I, I, I, P, L, cache, batch, P]
    lib.domino_rope_append.restype = I
    lib.domino_attend_workspace_bytes.argtypes = [I, I, cache]
    lib.domino_attend_workspace_bytes.restype = S
    lib.domino_attend_paged.argtypes = [P, L, I, I, cache, batch, F, I, P, I, P, L, P, P, S, P]
    lib.domino_attend_paged.restype = I
    lib.domino_cache_commit.argtypes = [cache, batch, I, L, P, P, I, P, P]
    lib.domino_cache_commit.restype = I
    _lib = lib
    return lib


def _addr(x):
    if x is None or type(x) is int:
        return x
    try:
        return x.data_ptr()
    except AttributeError:
        pass
    if isinstance(x, int):
        return x
    if hasattr(x, "ctypes"):  # numpy array
        return x.ctypes.data
    raise TypeError(f"cannot take the address of {type(x)}")


def _stream(s):
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return s.cuda_stream  # torch.cuda.Stream


def make_head(emb=None, w_ih=None, w_hh=None, b_ih=None, b_hh=None, w1=None, b1=None, w2=None, b2=None,
              Ds=0, R=0, x_table=None) -> domino_head_weights:
    return domino_head_weights(_addr(emb), _addr(w_ih), _addr(w_hh), _addr(b_ih), _addr(b_hh), _addr(w1),
                               _addr(b1), _addr(w2), _addr(b2), int(Ds), int(R), _addr(x_table))


def domino_input_table_bytes(V, Ds) -> int:
    return int(load().domino_input_table_bytes(V, Ds))


def domino_build_input_table(emb, w_ih, V, H, Ds, table, stream=None) -> int:
    """table [V, 3 Ds] fp32 = emb . W_ih^T (device); synchronises the stream."""
    return int(load().domino_build_input_table(_addr(emb), _addr(w_ih), V, H, Ds, _addr(table), _stream(stream)))


def domino_workspace_bytes(B, K, H, V, Ds, R, k, N) -> int:
    return int(load().domino_workspace_bytes(B, K, H, V, Ds, R, k, N))


def domino_workspace_bytes_host(B, K, H, V, Ds, R, k, N) -> int:
    return int(load().domino_workspace_bytes_host(B, K, H, V, Ds, R, k, N))


def domino_draft_step(hidden, prefix_ids, w_lm, head, B, K, H, V, k, N, topk_ids, topk_logp, tree_parent,
                      tree_token, tree_depth, tree_score, workspace, workspace_bytes, stream=None) -> int:
    h = ctypes.byref(head) if head is not None else None
    return int(load().domino_draft_step(_addr(hidden), _addr(prefix_ids), _addr(w_lm), h, B, K, H, V, k, N,
                                        _addr(topk_ids), _addr(topk_logp), _addr(tree_parent),
                                        _addr(tree_token), _addr(tree_depth), _addr(tree_score),
                                        _addr(workspace), int(workspace_bytes), _stream(stream)))


def domino_draft_step_host(hidden_host, prefix_ids_host, w_lm, head, B, K, H, V, k, N, topk_ids_host,
                           topk_logp_host, tree_parent_host, tree_token_host, tree_depth_host, tree_score_host,
                           workspace, workspace_bytes, stream=None) -> int:
    h = ctypes.byref(head) if head is not None else None
    return int(load().domino_draft_step_host(
        _addr(hidden_host), _addr(prefix_ids_host), _addr(w_lm), h, B, K, H, V, k, N, _addr(topk_ids_host),
        _addr(topk_logp_host), _addr(tree_parent_host), _addr(tree_token_host), _addr(tree_depth_host),
        _addr(tree_score_host), _addr(workspace), int(workspace_bytes), _stream(stream)))


def domino_check_status(workspace, stream=None) -> int:
    return int(load().domino_check_status(_addr(workspace), _stream(stream)))


def domino_status_string(code: int) -> str:
    return load().domino_status_string(int(code)).decode()


def domino_abi_version() -> int:
    return int(load().domino_abi_version())


def domino_launches_per_step(B, K, H, V, Ds, R, k, N) -> int:
    return int(load().domino_launches_per_step(B, K, H, V, Ds, R, k, N))


def domino_launches_per_step_table(B, K, H, V, Ds, R, k, N) -> int:
    return int(load().domino_launches_per_step_table(B, K, H, V, Ds, R, k, N))


def domino_timing_begin(max_launches: int) -> int:
    return int(load().domino_timing_begin(int(max_launches)))


def domino_timing_end() -> dict:
    """Stops per-kernel timing; returns {kind name: (total ms, launches)}."""
    n = len(KERNEL_KINDS)
    ms = (ctypes.c_float * n)()
    cnt = (ctypes.c_int * n)()
    rc = int(load().domino_timing_end(ctypes.cast(ms, ctypes.c_void_p), ctypes.cast(cnt, ctypes.c_void_p), n))
    if rc != 0:
        raise DominoError(rc, "domino_timing_end")
    return {KERNEL_KINDS[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}


def domino_draft_step_static_scratch(hidden, prefix_ids, w_lm, head, B, K, H, V, k, N, topk_ids, topk_logp,
                                     tree_parent, tree_token, tree_depth, tree_score, device_status=None,
                                     stream=None) -> int:
    """The draft step for callers that cannot allocate device memory: no workspace argument;
    the library's own static 16 MiB device array serves as scratch (see include/domino.h)."""
    h = ctypes.byref(head) if head is not None else None
    return int(load().domino_draft_step_static_scratch(
        _addr(hidden), _addr(prefix_ids), _addr(w_lm), h, B, K, H, V, k, N, _addr(topk_ids), _addr(topk_logp),
        _addr(tree_parent), _addr(tree_token), _addr(tree_depth), _addr(tree_score), _addr(device_status),
        _stream(stream)))


def domino_verify_tree_greedy(target_logits, tree_parent, tree_token, B, N, V, row_argmax, accepted_nodes,
                              accepted_count, bonus_token, stream=None) -> int:
    """Greedy verification of B draft trees against the target's fp32 logits [B, N+1, V] (device)."""
    return int(load().domino_verify_tree_greedy(_addr(target_logits), _addr(tree_parent), _addr(tree_token), B, N, V,
                                                _addr(row_argmax), _addr(accepted_nodes), _addr(accepted_count),
                                                _addr(bonus_token), _stream(stream)))


def domino_verify_tree_sample(target_logits, tree_parent, tree_token, uniforms, temperature, B, N, V, row_sample,
                              accepted_nodes, accepted_count, bonus_token, stream=None) -> int:
    """Verification at temperature T > 0 of B draft trees against the target's fp32 logits
    [B, N+1, V] with one uniform per row [B, N+1] (device)."""
    return int(load().domino_verify_tree_sample(_addr(target_logits), _addr(tree_parent), _addr(tree_token),
                                                _addr(uniforms), float(temperature), B, N, V, _addr(row_sample),
                                                _addr(accepted_nodes), _addr(accepted_count), _addr(bonus_token),
                                                _stream(stream)))


def domino_sample_filtered(logits, dtype, row_stride, temperature, top_k, top_p, min_p, uniforms, rows, V, tokens,
                           logp=None, stream=None) -> int:
    """One token per row of ``logits`` [rows, row_stride] after temperature, top-k, top-p and min-p (device
    arrays [rows] or None), drawn with ``uniforms`` fp32 [rows]; logp: its log-probability among the kept ids."""
    return int(load().domino_sample_filtered(_addr(logits), int(dtype), int(row_stride), _addr(temperature),
                                             _addr(top_k), _addr(top_p), _addr(min_p), _addr(uniforms), rows, V,
                                             _addr(tokens), _addr(logp), _stream(stream)))


def domino_verify_tree_filtered(target_logits, dtype, row_stride, tree_parent, tree_token, temperature, top_k, top_p,
                                min_p, uniforms, B, N, V, row_sample, row_logp, accepted_nodes, accepted_count,
                                bonus_token, stream=None) -> int:
    """Verification of B draft trees against a target that decodes with the filters of domino_sample_filtered
    (settings [B] per sequence or None): logits [B (N + 1), row_stride], one uniform per row."""
    return int(load().domino_verify_tree_filtered(_addr(target_logits), int(dtype), int(row_stride),
                                                  _addr(tree_parent), _addr(tree_token), _addr(temperature),
                                                  _addr(top_k), _addr(top_p), _addr(min_p), _addr(uniforms), B, N, V,
                                                  _addr(row_sample), _addr(row_logp), _addr(accepted_nodes),
                                                  _addr(accepted_count), _addr(bonus_token), _stream(stream)))


def domino_distill_loss(logits, dtype, row_stride, teacher_ids, teacher_scores, weights, temperature, mode, rows, V,
                        kt, loss, lse=None, stream=None) -> int:
    """Loss of every row of student logits against the teacher's list of kt ids and scores, and the two
    log-sum-exps [rows, 2] that domino_distill_grad takes."""
    return int(load().domino_distill_loss(_addr(logits), int(dtype), int(row_stride), _addr(teacher_ids),
                                          _addr(teacher_scores), _addr(weights), float(temperature), int(mode), rows,
                                          V, kt, _addr(loss), _addr(lse), _stream(stream)))


def domino_distill_grad(logits, dtype, row_stride, teacher_ids, teacher_scores, weights, grad_loss, temperature, mode,
                        rows, V, kt, lse, dlogits, grad_stride, stream=None) -> int:
    """Gradient of domino_distill_loss by the logits, times ``grad_loss`` [rows] (None: 1)."""
    return int(load().domino_distill_grad(_addr(logits), int(dtype), int(row_stride), _addr(teacher_ids),
                                          _addr(teacher_scores), _addr(weights), _addr(grad_loss), float(temperature),
                                          int(mode), rows, V, kt, _addr(lse), _addr(dlogits), int(grad_stride),
                                          _stream(stream)))


def domino_distill_loss_grad(logits, dtype, row_stride, teacher_ids, teacher_scores, weights, grad_loss, temperature,
                             mode, rows, V, kt, loss, lse, dlogits, grad_stride, stream=None) -> int:
    """domino_distill_loss and domino_distill_grad in one pass over the logits."""
    return int(load().domino_distill_loss_grad(_addr(logits), int(dtype), int(row_stride), _addr(teacher_ids),
                                               _addr(teacher_scores), _addr(weights), _addr(grad_loss),
                                               float(temperature), int(mode), rows, V, kt, _addr(loss), _addr(lse),
                                               _addr(dlogits), int(grad_stride), _stream(stream)))


def make_cache(k, v, page_stride, token_stride, head_stride, pages, page, heads, head_dim, dtype) -> domino_kv_cache:
    """A paged cache of keys and values (strides in elements).  The structure holds addresses: keep the tensors."""
    return domino_kv_cache(_addr(k), _addr(v), int(page_stride), int(token_stride), int(head_stride), int(pages),
                           int(page), int(heads), int(head_dim), int(dtype))


def make_batch(table, table_stride, table_width, kv_len, start, B) -> domino_kv_batch:
    """New tokens of B sequences on a paged cache.  The structure holds addresses: keep the tensors."""
    return domino_kv_batch(_addr(table), int(table_stride), int(table_width), _addr(kv_len), _addr(start), int(B))


def _ref(x):
    return ctypes.byref(x) if x is not None else None


def domino_rope(x, dtype, x_token_stride, x_head_stride, positions, freq, amplitude, layout, gradient, tokens, heads,
                head_dim, rot, y, y_token_stride, y_head_stride, stream=None) -> int:
    """y = rotary positions applied to x [tokens][heads][head_dim]; gradient: turned back (device)."""
    return int(load().domino_rope(_addr(x), int(dtype), int(x_token_stride), int(x_head_stride), _addr(positions),
                                  _addr(freq), float(amplitude), int(layout), int(gradient), tokens, heads, head_dim,
                                  rot, _addr(y), int(y_token_stride), int(y_head_stride), _stream(stream)))


def domino_rope_append(q, q_stride, k, k_stride, v, v_stride, positions, tree_depth, N, freq, amplitude, layout, rot,
                       q_heads, tokens, q_out, q_out_stride, cache, batch, stream=None) -> int:
    """New tokens' queries turned into q_out; their keys, turned, and values written to the paged cache (device)."""
    return int(load().domino_rope_append(_addr(q), int(q_stride), _addr(k), int(k_stride), _addr(v), int(v_stride),
                                         _addr(positions), _addr(tree_depth), int(N), _addr(freq), float(amplitude),
                                         int(layout), rot, q_heads, tokens, _addr(q_out), int(q_out_stride),
                                         _ref(cache), _ref(batch), _stream(stream)))


def domino_attend_workspace_bytes(tokens, q_heads, cache) -> int:
    return int(load().domino_attend_workspace_bytes(tokens, q_heads, _ref(cache)))


def domino_attend_paged(q, q_stride, tokens, q_heads, cache, batch, scale, mask, tree_parent, N, out, out_stride, lse,
                        workspace, workspace_bytes, stream=None) -> int:
    """Attention of a batch's new tokens over the paged cache: out, and lse fp32 [tokens][q_heads] or None (device)."""
    return int(load().domino_attend_paged(_addr(q), int(q_stride), tokens, q_heads, _ref(cache), _ref(batch),
                                          float(scale), int(mask), _addr(tree_parent), int(N), _addr(out),
                                          int(out_stride), _addr(lse), _addr(workspace), int(workspace_bytes),
                                          _stream(stream)))


def domino_cache_commit(cache, batch, layers, layer_stride, accepted_nodes, accepted_count, N, new_len,
                        stream=None) -> int:
    """The accepted nodes' keys and values moved behind the anchor in all layers; new_len [B] (device)."""
    return int(load().domino_cache_commit(_ref(cache), _ref(batch), int(layers), int(layer_stride),
                                          _addr(accepted_nodes), _addr(accepted_count), int(N), _addr(new_len),
                                          _stream(stream)))


def domino_rollout_workspace_bytes(B, K, H, V, Ds, R) -> int:
    return int(load().domino_rollout_workspace_bytes(B, K, H, V, Ds, R))


def domino_rollout_greedy(hidden, anchors, w_lm, head, B, K, H, V, tokens, logp, workspace, workspace_bytes,
                          stream=None) -> int:
    """Greedy sequential draft loop: tokens t_1..t_K [B, K] and their log-probabilities (device)."""
    h = ctypes.byref(head) if head is not None else None
    return int(load().domino_rollout_greedy(_addr(hidden), _addr(anchors), _addr(w_lm), h, B, K, H, V,
                                            _addr(tokens), _addr(logp), _addr(workspace), int(workspace_bytes),
                                            _stream(stream)))


def domino_rollout_sample(hidden, anchors, uniforms, w_lm, head, B, K, H, V, tokens, logp, workspace,
                          workspace_bytes, stream=None) -> int:
    """Sampled sequential draft loop: ``uniforms`` device float32 [B, K] in [0, 1)."""
    h = ctypes.byref(head) if head is not None else None
    return int(load().domino_rollout_sample(_addr(hidden), _addr(anchors), _addr(uniforms), _addr(w_lm), h, B, K, H,
                                            V, _addr(tokens), _addr(logp), _addr(workspace), int(workspace_bytes),
                                            _stream(stream)))


def domino_rollout_sample_gumbel(hidden, anchors, seed, w_lm, head, B, K, H, V, tokens, logp, workspace,
                                 workspace_bytes, stream=None) -> int:
    """Sampled sequential draft loop by the exponential race under a 64-bit ``seed``."""
    h = ctypes.byref(head) if head is not None else None
    return int(load().domino_rollout_sample_gumbel(_addr(hidden), _addr(anchors), int(seed) & ((1 << 64) - 1),
                                                   _addr(w_lm), h, B, K, H, V, _addr(tokens), _addr(logp),
                                                   _addr(workspace), int(workspace_bytes), _stream(stream)))


def domino_debug_hold(what, gru_cta=-1, step=-1) -> int:
    """Test hook: the next GRU launch's CTA ``gru_cta`` withholds its states of position ``step``
    (DOMINO_HOLD_STATE) or its clear-barrier arrival (DOMINO_HOLD_CLEAR_BARRIER); DOMINO_HOLD_OFF
    disarms.  The step then reports DOMINO_ERR_TIMEOUT through its device status.
    DOMINO_HOLD_ROW_COPY: the next sampled verification does not stage part of row ``gru_cta``.
    DOMINO_HOLD_KEY_TILE: CTA ``gru_cta`` of the next attention on the tensor cores lacks its first tile of keys."""
    return int(load().domino_debug_hold(int(what), int(gru_cta), int(step)))
