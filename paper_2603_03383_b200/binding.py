"""ctypes binding of ``libmtv.so`` — argument marshalling only.

Every function has the name and argument order of its C declaration in
``include/mtv.h``; tensors are passed as device pointers, the current torch
stream is used unless one is given.  There is no fallback: if the CUDA library
is missing, loading fails with an error.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# MTV_LIB names another build of the same library (a variant of build.py, e.g. the bounds-checking one).
LIB_PATH = os.environ.get("MTV_LIB") or os.path.join(_HERE, "libmtv.so")

MTV_OK = 0
MTV_ERR_BOUNDS = -7
ERR = {-7: "MTV_ERR_BOUNDS", -1: "MTV_ERR_INVALID_ARG", -2: "MTV_ERR_UNSUPPORTED_SHAPE", -3: "MTV_ERR_WORKSPACE",
       -4: "MTV_ERR_CUDA", -5: "MTV_ERR_TIMEOUT", -6: "MTV_ERR_CAPACITY"}
MTV_ERR_TIMEOUT = -5
MTV_ERR_CAPACITY = -6
MAX_K = 8

EXPORTS = ["tree_build_static", "tree_gen_cartesian", "tree_gen_rank_prior", "tree_query", "tree_destroy",
           "mtv_workspace_bytes", "medusa_heads_topk", "tree_verify_attention", "tree_accept",
           "kv_compact_accepted", "mtv_verify_step", "mtv_verify_step_host", "mtv_last_error",
           "mtv_set_kernel_taps", "mtv_kernel_taps_used", "mtv_device_error",
           "tree_accept_static_scratch", "tree_accept_static_scratch_capacity", "tree_kv_append_rope",
           "lm_head_argmax", "tree_accept_keys", "mtv_selftest_wait_timeout", "tree_kv_append_rope_layers",
           "mtv_verify_steps", "mtv_debug_bounds_enabled", "heads_merge_shards", "attn_interleave_shards",
           "keys_merge_shards", "node_argmax_keys", "tree_kv_append_rope_paged", "kv_append_rope_paged",
           "kv_compact_accepted_paged", "tree_attention_paged_workspace_bytes", "tree_verify_attention_paged",
           "logits_constrain", "constrained_argmax_keys", "token_counts_add", "tree_kv_append_rope_paged_fp8",
           "kv_append_rope_paged_fp8", "kv_read_paged_fp8", "kv_compact_accepted_paged_fp8", "tree_verify_attention_paged_fp8"]


class MtvError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        detail = ""
        if code == -4:
            detail = ": " + lib().mtv_last_error().decode()
        super().__init__("%s failed with %s%s" % (where, ERR.get(code, code), detail))


class TreeInfo(C.Structure):
    _fields_ = [("T", C.c_int32), ("K", C.c_int32), ("P", C.c_int32), ("C", C.c_int32),
                ("anc_words", C.c_int32), ("on_device", C.c_int32),
                ("k_d", C.c_int32 * MAX_K), ("cand_offset", C.c_int32 * MAX_K),
                ("node_ranks", C.POINTER(C.c_int32)), ("parent", C.POINTER(C.c_int32)),
                ("depth", C.POINTER(C.c_int32)), ("rank", C.POINTER(C.c_int32)),
                ("tree_indices", C.POINTER(C.c_int32)), ("retrieve_indices", C.POINTER(C.c_int32)),
                ("anc", C.POINTER(C.c_uint64)), ("medusa_attn_mask", C.POINTER(C.c_uint8))]


class StepArgs(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("V", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32),
                ("D", C.c_int32), ("n_layers", C.c_int32), ("Lcap", C.c_int32),
                ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_t", C.c_int64),
                ("scale", C.c_float),
                ("hidden", C.c_void_p), ("W1", C.c_void_p), ("b1", C.c_void_p), ("W2", C.c_void_p),
                ("root_tok", C.c_void_p), ("q_layers", C.c_void_p),
                ("k_caches", C.c_void_p), ("v_caches", C.c_void_p),
                ("k_caches_host", C.c_void_p), ("v_caches_host", C.c_void_p),
                ("logits", C.c_void_p), ("seq_lens", C.c_void_p),
                ("cand", C.c_void_p), ("cand_logit", C.c_void_p), ("tree_tok", C.c_void_p),
                ("out_layers", C.c_void_p),
                ("accept_len", C.c_void_p), ("best_path", C.c_void_p), ("acc_nodes", C.c_void_p),
                ("acc_tok", C.c_void_p), ("next_root", C.c_void_p), ("status", C.c_void_p),
                ("ws", C.c_void_p), ("ws_bytes", C.c_size_t),
                ("x_final", C.c_void_p), ("W_lm", C.c_void_p)]


class AppendArgs(C.Structure):
    _fields_ = [("k_new_layers", C.c_void_p), ("v_new_layers", C.c_void_p), ("rope_theta", C.c_float)]


class PoolLayout(C.Structure):
    _fields_ = [("stride_page", C.c_int64), ("stride_h", C.c_int64), ("stride_t", C.c_int64),
                ("page_size", C.c_int32), ("n_pages", C.c_int32)]


class LogitRules(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("counts", "seen", "repetition", "presence", "frequency", "bias_ids", "bias",
                                          "mask", "mask_of")] + [("n_bias", C.c_int32), ("n_masks", C.c_int32)]


_lib = None


def lib():
    """Load the CUDA library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("CUDA library %s is missing: run paper_2603_03383_b200/build.py "
                               "(there is no CPU fallback)" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
        L.tree_build_static.argtypes = [i32, i32, vp, i32, C.POINTER(vp)]
        L.tree_gen_cartesian.argtypes = [i32, vp, i32, vp, C.POINTER(C.c_int)]
        L.tree_gen_rank_prior.argtypes = [i32, i32, i32, vp, C.POINTER(C.c_int)]
        L.tree_query.argtypes = [vp, C.POINTER(TreeInfo)]
        L.tree_destroy.argtypes = [vp]
        L.tree_destroy.restype = None
        L.mtv_workspace_bytes.argtypes = [vp] + [i32] * 7
        L.mtv_workspace_bytes.restype = sz
        L.medusa_heads_topk.argtypes = [vp, i32, i32, i32] + [vp] * 8 + [vp, sz, vp]
        L.tree_verify_attention.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, i64, i64, i64, i32, vp,
                                            C.c_float, vp, vp, vp, sz, vp]
        L.tree_accept.argtypes = [vp, i32, i32] + [vp] * 7 + [vp, sz, vp]
        L.kv_compact_accepted.argtypes = [vp, i32, i32, i32, i32, vp, vp, i64, i64, i64, i32, vp, vp, vp, vp, vp]
        L.mtv_verify_step.argtypes = [vp, C.POINTER(StepArgs), vp]
        L.mtv_verify_step_host.argtypes = [vp, C.POINTER(StepArgs), C.POINTER(StepArgs), vp]
        L.mtv_last_error.restype = C.c_char_p
        L.mtv_set_kernel_taps.argtypes = [i32, vp, vp, i32]
        L.mtv_kernel_taps_used.argtypes = [i32]
        L.mtv_device_error.argtypes = [vp, i32, C.POINTER(C.c_int32)]
        L.tree_accept_static_scratch.argtypes = [vp, i32, i32] + [vp] * 7 + [vp]
        L.tree_accept_static_scratch_capacity.restype = sz
        L.tree_kv_append_rope.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, C.c_float,
                                          vp, vp]
        L.lm_head_argmax.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
        L.tree_accept_keys.argtypes = [vp, i32] + [vp] * 7 + [vp]
        L.mtv_selftest_wait_timeout.argtypes = [vp, vp]
        L.tree_kv_append_rope_layers.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, i64, i64, i64, i32, vp,
                                                 C.c_float, vp, vp]
        L.heads_merge_shards.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.attn_interleave_shards.argtypes = [i32, i32, i32, i32, vp, vp, vp]
        L.keys_merge_shards.argtypes = [i32, i32, i32, vp, vp, vp]
        L.node_argmax_keys.argtypes = [vp, i32, i32, vp, vp, vp, sz, vp]
        pool = C.POINTER(PoolLayout)
        L.tree_kv_append_rope_paged.argtypes = [vp, i32, i32, i32, i32, i32] + [vp] * 6 + [pool, vp, i32, vp, C.c_float, vp, vp]
        L.kv_append_rope_paged.argtypes = [i32] * 6 + [vp] * 6 + [pool, vp, i32, vp, vp, C.c_float, vp, vp]
        L.kv_compact_accepted_paged.argtypes = [vp, i32, i32, i32, i32, vp, vp, pool, vp, i32] + [vp] * 6
        L.tree_attention_paged_workspace_bytes.argtypes = [vp] + [i32] * 5
        L.tree_attention_paged_workspace_bytes.restype = sz
        L.tree_verify_attention_paged.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, pool, vp, i32, i32, vp, C.c_float, vp, vp,
                                                  vp, sz, vp]
        L.tree_kv_append_rope_paged_fp8.argtypes = [vp, i32, i32, i32, i32, i32] + [vp] * 6 + [pool, vp, i32, vp, vp, vp, C.c_float, vp, vp]
        L.kv_append_rope_paged_fp8.argtypes = [i32] * 6 + [vp] * 6 + [pool, vp, i32] + [vp] * 4 + [C.c_float, vp, vp]
        L.kv_read_paged_fp8.argtypes = [i32] * 5 + [vp, vp, pool, vp, i32] + [vp] * 8
        L.kv_compact_accepted_paged_fp8.argtypes = L.kv_compact_accepted_paged.argtypes
        L.tree_verify_attention_paged_fp8.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, pool, vp, i32, i32, vp, vp, vp, C.c_float, vp, vp,
                                                      vp, sz, vp]
        rules = C.POINTER(LogitRules)
        L.logits_constrain.argtypes = [vp, i32, i32, i32, vp, i64, vp, i64, rules, vp, vp]
        L.constrained_argmax_keys.argtypes = [vp, i32, i32, i32, vp, i64, rules, vp, vp, vp]
        L.token_counts_add.argtypes = [i32, i32, i32, vp, vp, i32, vp, vp, vp]
        L.mtv_verify_steps.argtypes = [vp, C.POINTER(StepArgs), C.POINTER(AppendArgs), i32, vp]
        _lib = L
    return _lib


def _check(rc, where):
    if rc != MTV_OK:
        raise MtvError(rc, where)


# Addresses and streams go over as plain integers (every function has its argument types declared): a decode loop makes
# one attention call per layer, and wrapping each pointer and building a Stream object cost more than the kernel's launch.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def tree_gen_cartesian(topk: Sequence[int]):
    K = len(topk)
    tk = (C.c_int32 * K)(*topk)
    n = C.c_int(0)
    lib().tree_gen_cartesian(K, tk, 0, None, C.byref(n))
    buf = (C.c_int32 * (max(n.value, 1) * K))()
    _check(lib().tree_gen_cartesian(K, tk, n.value, buf, C.byref(n)), "tree_gen_cartesian")
    return [list(buf[i * K:(i + 1) * K]) for i in range(n.value)]


def tree_gen_rank_prior(K: int, T_total: int, R_max: int = 10):
    n = C.c_int(0)
    buf = (C.c_int32 * (max(T_total - 1, 1) * K))()
    _check(lib().tree_gen_rank_prior(K, T_total, R_max, buf, C.byref(n)), "tree_gen_rank_prior")
    return [list(buf[i * K:(i + 1) * K]) for i in range(n.value)]


class Tree:
    """Owner of one ``mtv_tree_t`` (built by ``tree_build_static``)."""

    def __init__(self, K: int, node_ranks, upload: bool = True):
        flat = []
        for row in node_ranks:
            row = list(row)
            flat += row + [-1] * (K - len(row))
        n = len(flat) // K
        arr = (C.c_int32 * max(len(flat), 1))(*flat)
        h = C.c_void_p()
        _check(lib().tree_build_static(K, n, arr, 1 if upload else 0, C.byref(h)), "tree_build_static")
        self.handle = h
        info = TreeInfo()
        _check(lib().tree_query(h, C.byref(info)), "tree_query")
        self.info = info
        self.T, self.K, self.P, self.C = info.T, info.K, info.P, info.C
        self.k_d = list(info.k_d[:self.K])
        self.cand_offset = list(info.cand_offset[:self.K])
        T, K1 = self.T, self.K + 1
        self.node_ranks = [list(info.node_ranks[i * K:(i + 1) * K]) for i in range(T)]
        self.parent = list(info.parent[:T])
        self.depth = list(info.depth[:T])
        self.rank = list(info.rank[:T])
        self.tree_indices = list(info.tree_indices[:T])
        self.retrieve_indices = [list(info.retrieve_indices[p * K1:(p + 1) * K1]) for p in range(self.P)]
        self.anc = [[info.anc[i * info.anc_words + w] for w in range(info.anc_words)] for i in range(T)]
        self.medusa_attn_mask = [[info.medusa_attn_mask[i * T + j] for j in range(T)] for i in range(T)]

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.tree_destroy(self.handle)
            self.handle = None


def tree_build_static(K, node_ranks, upload=True) -> Tree:
    return Tree(K, node_ranks, upload)


def mtv_device_error(tree: Tree, clear: bool = True) -> int:
    code = C.c_int32(0)
    _check(lib().mtv_device_error(tree.handle, 1 if clear else 0, C.byref(code)), "mtv_device_error")
    return code.value


def mtv_debug_bounds_enabled() -> bool:
    return bool(lib().mtv_debug_bounds_enabled())


def mtv_selftest_wait_timeout(tree: Tree, stream=None):
    """Enqueue a kernel whose bounded wait must run out (about a second); see include/mtv.h."""
    _check(lib().mtv_selftest_wait_timeout(tree.handle, _stream(stream)), "mtv_selftest_wait_timeout")


def mtv_workspace_bytes(tree: Tree, B, H, V, Hq, Hkv, D, Lcap) -> int:
    return lib().mtv_workspace_bytes(tree.handle, B, H, V, Hq, Hkv, D, Lcap)


def _ws(ws):
    return ws.data_ptr(), ws.nbytes


def medusa_heads_topk(tree, hidden, W1, b1, W2, root_tok, cand, cand_logit, tree_tok, ws, stream=None):
    B, H = hidden.shape
    V = W2.shape[1]
    p, n = _ws(ws)
    _check(lib().medusa_heads_topk(tree.handle, B, H, V, _ptr(hidden), _ptr(W1), _ptr(b1), _ptr(W2),
                                   _ptr(root_tok), _ptr(cand), _ptr(cand_logit), _ptr(tree_tok), p, n,
                                   _stream(stream)), "medusa_heads_topk")


def tree_verify_attention(tree, q, k_cache, v_cache, seq_lens, out, ws, scale=0.0, status=None, stream=None,
                          Lcap=None):
    B, T, Hq, D = q.shape
    Hkv = k_cache.shape[1]
    Lcap = k_cache.shape[2] if Lcap is None else Lcap
    sb, sh, st = strides = k_cache.stride()[:3]
    assert v_cache.stride()[:3] == strides
    p, n = _ws(ws)
    _check(lib().tree_verify_attention(tree.handle, B, Hq, Hkv, D, _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                       sb, sh, st, Lcap, _ptr(seq_lens), scale, _ptr(out), _ptr(status), p, n,
                                       _stream(stream)), "tree_verify_attention")


def tree_kv_append_rope(tree, q, k_new, v_new, k_cache, v_cache, seq_lens, rope_theta=0.0, status=None, stream=None,
                        Lcap=None):
    B, T, Hq, D = q.shape
    Hkv = k_new.shape[2]
    Lcap = k_cache.shape[2] if Lcap is None else Lcap
    sb, sh, st = k_cache.stride(0), k_cache.stride(1), k_cache.stride(2)
    assert (v_cache.stride(0), v_cache.stride(1), v_cache.stride(2)) == (sb, sh, st)
    _check(lib().tree_kv_append_rope(tree.handle, B, Hq, Hkv, D, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache),
                                     _ptr(v_cache), sb, sh, st, Lcap, _ptr(seq_lens), rope_theta, _ptr(status),
                                     _stream(stream)), "tree_kv_append_rope")


def tree_kv_append_rope_layers(tree, q_layers, k_new_layers, v_new_layers, k_ptrs, v_ptrs, strides, Lcap, seq_lens,
                               rope_theta=0.0, status=None, stream=None):
    """q_layers [n_layers][B][T][Hq][D], k_new_layers / v_new_layers [n_layers][B][T][Hkv][D]; k_ptrs / v_ptrs as for
    kv_compact_accepted."""
    n_layers, B, T, Hq, D = q_layers.shape
    Hkv = k_new_layers.shape[3]
    sb, sh, st = strides
    _check(lib().tree_kv_append_rope_layers(tree.handle, B, Hq, Hkv, D, n_layers, _ptr(q_layers), _ptr(k_new_layers),
                                            _ptr(v_new_layers), _ptr(k_ptrs), _ptr(v_ptrs), sb, sh, st, Lcap,
                                            _ptr(seq_lens), rope_theta, _ptr(status), _stream(stream)),
           "tree_kv_append_rope_layers")


def tree_accept(tree, logits, tree_tok, accept_len, best_path, acc_nodes, acc_tok, next_root, ws, stream=None):
    B, T, V = logits.shape
    p, n = _ws(ws)
    _check(lib().tree_accept(tree.handle, B, V, _ptr(logits), _ptr(tree_tok), _ptr(accept_len), _ptr(best_path),
                             _ptr(acc_nodes), _ptr(acc_tok), _ptr(next_root), p, n, _stream(stream)),
           "tree_accept")


def lm_head_argmax(tree, x, W, keys, am=None, am_val=None, stream=None):
    """x [B][T][H], W [V][H] bf16; keys [B*T] int64 storage for the uint64 keys (see include/mtv.h)."""
    B, T, H = x.shape
    _check(lib().lm_head_argmax(tree.handle, B, H, W.shape[0], _ptr(x), _ptr(W),
                                _ptr(am), _ptr(am_val), _ptr(keys), _stream(stream)), "lm_head_argmax")


def tree_accept_keys(tree, B, keys, tree_tok, accept_len, best_path, acc_nodes, acc_tok, next_root, stream=None):
    _check(lib().tree_accept_keys(tree.handle, B, _ptr(keys), _ptr(tree_tok), _ptr(accept_len), _ptr(best_path),
                                  _ptr(acc_nodes), _ptr(acc_tok), _ptr(next_root), _stream(stream)),
           "tree_accept_keys")


def tree_accept_static_scratch(tree, logits, tree_tok, accept_len, best_path, acc_nodes, acc_tok, next_root,
                               stream=None):
    """tree_accept for callers that may not allocate: no workspace argument (see include/mtv.h)."""
    B, T, V = logits.shape
    rc = lib().tree_accept_static_scratch(tree.handle, B, V, _ptr(logits), _ptr(tree_tok), _ptr(accept_len),
                                          _ptr(best_path), _ptr(acc_nodes), _ptr(acc_tok), _ptr(next_root),
                                          _stream(stream))
    if rc == -3:    # too large for the built-in array: the library says by how much
        raise MtvError(rc, "tree_accept_static_scratch [%s]" % lib().mtv_last_error().decode())
    _check(rc, "tree_accept_static_scratch")


def tree_accept_static_scratch_capacity() -> int:
    return lib().tree_accept_static_scratch_capacity()


def cache_pointer_array(caches, device=None):
    """int64 tensor holding the device addresses of a list of cache tensors."""
    t = torch.tensor([c.data_ptr() for c in caches], dtype=torch.int64)
    return t.to(device) if device is not None else t


def kv_compact_accepted(tree, k_ptrs, v_ptrs, n_layers, B, Hkv, D, strides, Lcap, seq_lens, accept_len, acc_nodes,
                        status=None, stream=None):
    sb, sh, st = strides
    _check(lib().kv_compact_accepted(tree.handle, B, Hkv, D, n_layers, _ptr(k_ptrs), _ptr(v_ptrs), sb, sh, st,
                                     Lcap, _ptr(seq_lens), _ptr(accept_len), _ptr(acc_nodes), _ptr(status),
                                     _stream(stream)), "kv_compact_accepted")


def mtv_verify_step(tree, args: StepArgs, stream=None):
    _check(lib().mtv_verify_step(tree.handle, C.byref(args), _stream(stream)), "mtv_verify_step")


def heads_merge_shards(tree, v_slab, cand_shards, logit_shards, root_tok, cand, cand_logit, tree_tok, ws, stream=None):
    """cand_shards [n][B][C], logit_shards [n][B][C-1] (every rank's medusa_heads_topk results, gathered)."""
    n, B, _ = cand_shards.shape
    p, nbytes = _ws(ws)
    _check(lib().heads_merge_shards(tree.handle, B, n, v_slab, _ptr(cand_shards), _ptr(logit_shards), _ptr(root_tok),
                                    _ptr(cand), _ptr(cand_logit), _ptr(tree_tok), p, nbytes, _stream(stream)),
           "heads_merge_shards")


def attn_interleave_shards(gathered, out, stream=None):
    """gathered [n][B][T][Hq_local][D] -> out [B][T][n * Hq_local][D]."""
    n, B, T, Hl, D = gathered.shape
    _check(lib().attn_interleave_shards(B * T, n, Hl, D, _ptr(gathered), _ptr(out), _stream(stream)),
           "attn_interleave_shards")


def node_argmax_keys(tree, logits, keys, ws, stream=None):
    """logits [B][T][V] bf16 -> keys [B*T] (int64 storage of the uint64 keys)."""
    B, T, V = logits.shape
    p, n = _ws(ws)
    _check(lib().node_argmax_keys(tree.handle, B, V, _ptr(logits), _ptr(keys), p, n, _stream(stream)), "node_argmax_keys")


def keys_merge_shards(v_slab, key_shards, keys, stream=None):
    """key_shards [n][B*T] (int64 storage of the uint64 keys) -> keys [B*T]."""
    n, m = key_shards.shape
    _check(lib().keys_merge_shards(m, n, v_slab, _ptr(key_shards), _ptr(keys), _stream(stream)), "keys_merge_shards")


def mtv_verify_steps(tree, steps: Sequence[StepArgs], appends: Optional[Sequence[AppendArgs]] = None, stream=None):
    """A chain of steps on one stream (see include/mtv.h); `steps` and `appends` are sequences of the structs."""
    n = len(steps)
    arr = (StepArgs * n)(*steps)
    app = None
    if appends is not None:
        assert len(appends) == n
        app = (AppendArgs * n)(*appends)
    _check(lib().mtv_verify_steps(tree.handle, arr, app, n, _stream(stream)), "mtv_verify_steps")


def mtv_verify_step_host(tree, dev: StepArgs, host: StepArgs, stream=None):
    _check(lib().mtv_verify_step_host(tree.handle, C.byref(dev), C.byref(host), _stream(stream)),
           "mtv_verify_step_host")


# ------------------------------------------------------------------------------------- caches in pages
# What these calls and those of the next section are given is looked at before its address goes over: a kernel that reads int64 as int32, or
# past the end of a tensor, reports nothing.  A refusal names the argument.  (pysrc/tensors.cpp looks at all tensors of a call in one step; a set of
# rules is looked at when it is made.)
_BF16, _I32, _I64, _F32, _ANY, _FP8, _OPTIONAL, _STRIDED, _LIKE_PREVIOUS = 0, 1, 2, 3, 4, 5, 16, 32, 64
_MAYBE_I32 = _I32 | _OPTIONAL
_tensors = None


def _refuse(where, name):
    raise MtvError(-1, "%s: %s" % (where, name))


def _look(where, names, *args):
    """args: (tensor, kind, elements at least) one after another, see pysrc/tensors.cpp -> (device, address, address, ...)."""
    global _tensors
    if _tensors is None:
        from . import _tensors as loaded        # (missing: run build.py)
        _tensors = loaded
    found = _tensors.addresses(*args)
    if type(found) is int:
        _refuse(where, names[found])
    # the library launches on the current device
    if found[0] < 0 or found[0] != torch._C._cuda_getDevice():
        _refuse(where, "tensors that are not on the current CUDA device")
    return found


def pool_layout(pool: torch.Tensor) -> PoolLayout:
    """Layout of a pool tensor [n_pages][Hkv][page_size][D] of any strides with the columns innermost (a pool whose pages hold
    [page_size][Hkv][D] is passed as its transposed view): bf16, or the codes of the calls with the suffix _fp8 (float8_e4m3fn)."""
    if pool.dim() != 4 or pool.stride(3) != 1 or pool.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
        _refuse("pool_layout", "pool")
    sp, sh, st = pool.stride()[:3]
    layout = PoolLayout(sp, sh, st, pool.shape[2], pool.shape[0])
    layout.dtype = pool.dtype
    return layout


def _layout_of(pool, dtype, where):
    """Strides are counted in elements: a layout that was made of another type's pool is refused."""
    if getattr(pool, "dtype", dtype) is not dtype:
        _refuse(where, "pool")


_APPEND = ("q_layers", "q_out_layers", "k_new_layers", "v_new_layers", "k_ptrs", "v_ptrs", "page_table", "seq_lens", "status")
_SCALES = ("k_scale", "v_scale")
_APPEND_FP8, _APPEND_ROWS, _APPEND_ROWS_FP8 = _APPEND + _SCALES, _APPEND + ("row_starts",), _APPEND + _SCALES + ("row_starts",)


def _scales(scales, n):
    """The two scales' part of a look, for calls that have them."""
    return (scales[0], _F32, n, scales[1], _F32, n) if scales else ()


def _append_tree(where, call, dtype, scales, tree, q_layers, q_out_layers, k_new_layers, v_new_layers, k_ptrs, v_ptrs, pool, page_table, seq_lens,
                 rope_theta, status, stream):
    shape = q_layers.shape
    if len(shape) != 5 or shape[2] != tree.T:
        _refuse(where, "q_layers")
    n_layers, B, T, Hq, D = shape
    if k_new_layers.dim() != 5 or page_table.dim() != 2:
        _refuse(where, "k_new_layers" if page_table.dim() == 2 else "page_table")
    Hkv, max_pages = k_new_layers.shape[3], page_table.shape[1]
    if k_new_layers.shape != (n_layers, B, T, Hkv, D):
        _refuse(where, "k_new_layers")
    _layout_of(pool, dtype, where)
    rows = n_layers * B * T * D
    _, q, q_out, k, v, kp, vp, table, lens, st, *sc = _look(
        where, _APPEND_FP8, q_layers, _BF16, rows * Hq, q_out_layers, _BF16 | _LIKE_PREVIOUS, -1, k_new_layers, _BF16, -1,
        v_new_layers, _BF16 | _LIKE_PREVIOUS, -1, k_ptrs, _I64, n_layers, v_ptrs, _I64, n_layers, page_table, _I32, B * max_pages, seq_lens, _I32, B,
        status, _MAYBE_I32, B, *_scales(scales, n_layers * Hkv))
    _check(call(tree.handle, B, Hq, Hkv, D, n_layers, q, q_out, k, v, kp, vp, pool, table, max_pages, lens, *sc, rope_theta, st, _stream(stream)), where)


def _append_rows(where, call, dtype, scales, q_layers, q_out_layers, k_new_layers, v_new_layers, k_ptrs, v_ptrs, pool, page_table, seq_lens, row_starts,
                 rope_theta, status, stream):
    for t, dim, name in ((q_layers, 4, "q_layers"), (k_new_layers, 4, "k_new_layers"), (page_table, 2, "page_table")):
        if t.dim() != dim:
            _refuse(where, name)
    (n_layers, n_rows, Hq, D), (B, max_pages), Hkv = q_layers.shape, page_table.shape, k_new_layers.shape[2]
    if k_new_layers.shape != (n_layers, n_rows, Hkv, D):
        _refuse(where, "k_new_layers")
    _layout_of(pool, dtype, where)
    _, q, q_out, k, v, kp, vp, table, lens, st, *sc, starts = _look(
        where, _APPEND_ROWS_FP8 if scales else _APPEND_ROWS, q_layers, _BF16, -1, q_out_layers, _BF16 | _LIKE_PREVIOUS, -1, k_new_layers, _BF16, -1,
        v_new_layers, _BF16 | _LIKE_PREVIOUS, -1, k_ptrs, _I64, n_layers, v_ptrs, _I64, n_layers, page_table, _I32, -1, seq_lens, _I32, B,
        status, _MAYBE_I32, B, *_scales(scales, n_layers * Hkv), row_starts, _I32, B + 1)
    _check(call(B, n_rows, Hq, Hkv, D, n_layers, q, q_out, k, v, kp, vp, pool, table, max_pages, lens, starts, *sc, rope_theta, st, _stream(stream)), where)


def tree_kv_append_rope_paged(tree, q_layers, q_out_layers, k_new_layers, v_new_layers, k_ptrs, v_ptrs, pool: PoolLayout, page_table,
                              seq_lens, rope_theta=0.0, status=None, stream=None):
    """q_layers, q_out_layers [n_layers][B][T][Hq][D], k_new_layers / v_new_layers [n_layers][B][T][Hkv][D]; k_ptrs / v_ptrs: device
    arrays of the layers' pools (cache_pointer_array); page_table [B][max_pages]."""
    _append_tree("tree_kv_append_rope_paged", lib().tree_kv_append_rope_paged, torch.bfloat16, (), tree, q_layers, q_out_layers, k_new_layers,
                 v_new_layers, k_ptrs, v_ptrs, pool, page_table, seq_lens, rope_theta, status, stream)


def kv_append_rope_paged(q_layers, q_out_layers, k_new_layers, v_new_layers, k_ptrs, v_ptrs, pool: PoolLayout, page_table, seq_lens,
                         row_starts, rope_theta=0.0, status=None, stream=None):
    """q_layers, q_out_layers [n_layers][n_rows][Hq][D], k_new_layers / v_new_layers [n_layers][n_rows][Hkv][D]; row_starts [B+1]."""
    _append_rows("kv_append_rope_paged", lib().kv_append_rope_paged, torch.bfloat16, (), q_layers, q_out_layers, k_new_layers, v_new_layers, k_ptrs,
                 v_ptrs, pool, page_table, seq_lens, row_starts, rope_theta, status, stream)


def tree_kv_append_rope_paged_fp8(tree, q_layers, q_out_layers, k_new_layers, v_new_layers, k_ptrs, v_ptrs, pool: PoolLayout, page_table,
                                  seq_lens, k_scale, v_scale, rope_theta=0.0, status=None, stream=None):
    """tree_kv_append_rope_paged into pools of e4m3 codes; k_scale, v_scale [n_layers][Hkv] fp32."""
    _append_tree("tree_kv_append_rope_paged_fp8", lib().tree_kv_append_rope_paged_fp8, torch.float8_e4m3fn, (k_scale, v_scale), tree, q_layers,
                 q_out_layers, k_new_layers, v_new_layers, k_ptrs, v_ptrs, pool, page_table, seq_lens, rope_theta, status, stream)


def kv_append_rope_paged_fp8(q_layers, q_out_layers, k_new_layers, v_new_layers, k_ptrs, v_ptrs, pool: PoolLayout, page_table, seq_lens,
                             row_starts, k_scale, v_scale, rope_theta=0.0, status=None, stream=None):
    """kv_append_rope_paged into pools of e4m3 codes; k_scale, v_scale [n_layers][Hkv] fp32."""
    _append_rows("kv_append_rope_paged_fp8", lib().kv_append_rope_paged_fp8, torch.float8_e4m3fn, (k_scale, v_scale), q_layers, q_out_layers,
                 k_new_layers, v_new_layers, k_ptrs, v_ptrs, pool, page_table, seq_lens, row_starts, rope_theta, status, stream)


_READ = ("k_ptrs", "v_ptrs", "page_table", "first", "row_starts", "k_scale", "v_scale", "k_out_layers", "v_out_layers", "status")


def kv_read_paged_fp8(k_ptrs, v_ptrs, pool: PoolLayout, page_table, row_starts, k_scale, v_scale, k_out_layers, v_out_layers, first=None,
                      status=None, stream=None):
    """k_out_layers, v_out_layers [n_layers][n_rows][Hkv][D] bf16; row_starts [B+1], first [B] (None: from slot 0)."""
    where = "kv_read_paged_fp8"
    if k_out_layers.dim() != 4:
        _refuse(where, "k_out_layers")
    if page_table.dim() != 2:
        _refuse(where, "page_table")
    (n_layers, n_rows, Hkv, D), (B, max_pages) = k_out_layers.shape, page_table.shape
    _layout_of(pool, torch.float8_e4m3fn, where)
    _, kp, vp, table, at, starts, ks, vs, k, v, st = _look(
        where, _READ, k_ptrs, _I64, n_layers, v_ptrs, _I64, n_layers, page_table, _I32, -1, first, _MAYBE_I32, B, row_starts, _I32, B + 1,
        k_scale, _F32, n_layers * Hkv, v_scale, _F32, n_layers * Hkv, k_out_layers, _BF16, -1, v_out_layers, _BF16 | _LIKE_PREVIOUS, -1,
        status, _MAYBE_I32, B)
    _check(lib().kv_read_paged_fp8(B, n_rows, Hkv, D, n_layers, kp, vp, pool, table, max_pages, at, starts, ks, vs, k, v, st, _stream(stream)), where)


_COMPACT = ("k_ptrs", "v_ptrs", "page_table", "seq_lens", "new_lens", "accept_len", "acc_nodes", "status")


def _compact(where, call, dtype, tree, k_ptrs, v_ptrs, n_layers, Hkv, D, pool, page_table, seq_lens, new_lens, accept_len, acc_nodes, status, stream):
    if page_table.dim() != 2:
        _refuse(where, "page_table")
    B, max_pages = page_table.shape
    _layout_of(pool, dtype, where)
    _, kp, vp, table, lens, new, n, nodes, st = _look(
        where, _COMPACT, k_ptrs, _I64, n_layers, v_ptrs, _I64, n_layers, page_table, _I32, -1, seq_lens, _I32, B, new_lens, _I32, B, accept_len, _I32, B,
        acc_nodes, _I32, B * (tree.K + 1), status, _MAYBE_I32, B)
    _check(call(tree.handle, B, Hkv, D, n_layers, kp, vp, pool, table, max_pages, lens, new, n, nodes, st, _stream(stream)), where)


def kv_compact_accepted_paged(tree, k_ptrs, v_ptrs, n_layers, Hkv, D, pool: PoolLayout, page_table, seq_lens, new_lens, accept_len,
                              acc_nodes, status=None, stream=None):
    """new_lens may be seq_lens itself; accept_len [B], acc_nodes [B][K + 1]."""
    _compact("kv_compact_accepted_paged", lib().kv_compact_accepted_paged, torch.bfloat16, tree, k_ptrs, v_ptrs, n_layers, Hkv, D, pool, page_table,
             seq_lens, new_lens, accept_len, acc_nodes, status, stream)


def kv_compact_accepted_paged_fp8(tree, k_ptrs, v_ptrs, n_layers, Hkv, D, pool: PoolLayout, page_table, seq_lens, new_lens, accept_len,
                                  acc_nodes, status=None, stream=None):
    """kv_compact_accepted_paged of pools of e4m3 codes."""
    _compact("kv_compact_accepted_paged_fp8", lib().kv_compact_accepted_paged_fp8, torch.float8_e4m3fn, tree, k_ptrs, v_ptrs, n_layers, Hkv, D, pool,
             page_table, seq_lens, new_lens, accept_len, acc_nodes, status, stream)


def paged_workspace_bytes(tree, B, Hq, Hkv, D, shared_len=0) -> int:
    """Bytes of device scratch of tree_verify_attention_paged (0: sizes that it refuses)."""
    return lib().tree_attention_paged_workspace_bytes(tree.handle, B, Hq, Hkv, D, shared_len)


_ATTENTION = ("q", "out", "k_pool", "v_pool", "page_table", "seq_lens", "status", "ws") + _SCALES
_layout_of_sizes = functools.lru_cache(maxsize=256)(PoolLayout)      # (numbers alone; making one costs as much as looking at three tensors)


def _attention(where, call, kind, scales, tree, q, k_pool, v_pool, page_table, seq_lens, out, ws, shared_len, scale, status, stream):
    shape, pools, strides = q.shape, k_pool.shape, k_pool.stride()
    if len(shape) != 4 or shape[1] != tree.T:
        _refuse(where, "q")
    B, T, Hq, D = shape
    if len(pools) != 4 or pools[3] != D or strides[3] != 1:
        _refuse(where, "k_pool")
    if v_pool.stride() != strides:
        _refuse(where, "v_pool")
    if page_table.dim() != 2:
        _refuse(where, "page_table")
    max_pages = page_table.shape[1]
    _, q_at, out_at, k, v, table, lens, st, ws_at, *sc = _look(
        where, _ATTENTION, q, _BF16, -1, out, _BF16 | _LIKE_PREVIOUS, -1, k_pool, kind | _STRIDED, -1,
        v_pool, kind | _STRIDED | _LIKE_PREVIOUS, -1, page_table, _I32, B * max_pages, seq_lens, _I32, B, status, _MAYBE_I32, B, ws, _ANY, -1,
        *_scales(scales, pools[1]))
    _check(call(tree.handle, B, Hq, pools[1], D, q_at, k, v, _layout_of_sizes(strides[0], strides[1], strides[2], pools[2], pools[0]), table, max_pages,
                shared_len, lens, *sc, scale, out_at, st, ws_at, ws.nbytes, _stream(stream)), where)


def tree_verify_attention_paged(tree, q, k_pool, v_pool, page_table, seq_lens, out, ws, shared_len=0, scale=0.0, status=None,
                                stream=None):
    """q, out [B][T][Hq][D]; k_pool, v_pool [n_pages][Hkv][page_size][D] (see pool_layout), the same strides."""
    _attention("tree_verify_attention_paged", lib().tree_verify_attention_paged, _BF16, (), tree, q, k_pool, v_pool, page_table, seq_lens, out, ws,
               shared_len, scale, status, stream)


def tree_verify_attention_paged_fp8(tree, q, k_pool, v_pool, page_table, seq_lens, out, ws, k_scale, v_scale, shared_len=0, scale=0.0,
                                    status=None, stream=None):
    """tree_verify_attention_paged over pools of e4m3 codes (float8_e4m3fn); k_scale, v_scale [Hkv] fp32, the layer's."""
    _attention("tree_verify_attention_paged_fp8", lib().tree_verify_attention_paged_fp8, _FP8, (k_scale, v_scale), tree, q, k_pool, v_pool, page_table,
               seq_lens, out, ws, shared_len, scale, status, stream)


# ------------------------------------------------------------------------------------- constrained decoding
def logit_rules(counts=None, seen=None, repetition=None, presence=None, frequency=None, bias_ids=None, bias=None, mask=None,
                mask_of=None) -> LogitRules:
    """counts [B][V], seen [B][words], repetition / presence / frequency [B] fp32, bias_ids / bias [B][n], mask [n_masks][words],
    mask_of [B][T]; words of 32 tokens in int32 storage (see include/mtv.h).  The tensors have to outlive the rules' use."""
    tensors = (counts, seen, repetition, presence, frequency, bias_ids, bias, mask, mask_of)
    names = [n for n, _ in LogitRules._fields_]
    i32, f32 = (torch.int32, torch.uint32), (torch.float32,)
    # what the rules ask of a call: at most B sequences, V tokens in W words, T nodes, one device
    asks, devs = {}, set()
    for t, name, types, dims in zip(tensors, names, (i32, i32, f32, f32, f32, i32, f32, i32, i32), ("BV", "BW", "B", "B", "B", "Bn", "Bn", "mW", "BT")):
        if t is None:
            continue
        if t.dtype not in types or t.dim() != len(dims) or not t.is_contiguous():
            _refuse("logit_rules", name)
        for d, size in zip(dims, t.shape):
            if asks.setdefault(d, size) != size and d != "B":
                _refuse("logit_rules", name)
            asks[d] = min(asks[d], size)
        devs.add(t.get_device())
    if (bias_ids is None) != (bias is None):
        _refuse("logit_rules", "bias_ids" if bias_ids is None else "bias")
    if "V" in asks and asks.get("W", (asks["V"] + 31) // 32) != (asks["V"] + 31) // 32:
        _refuse("logit_rules", "mask" if seen is None else "seen")
    if len(devs) > 1:
        _refuse("logit_rules", "tensors of several devices")
    r = LogitRules(*[_ptr(t) for t in tensors])
    r.n_bias = 0 if bias_ids is None else bias_ids.shape[-1]
    r.n_masks = 0 if mask is None else mask.shape[0]
    r.tensors = tensors
    r.asks = tuple(asks.get(d) for d in "BVWT") + (devs.pop() if devs else None,)
    return r


_LOGIT_TYPES = {torch.bfloat16: 0, torch.float32: 1}


def _logit_rows(x, where):
    """(type, row stride) of logits [B][T][V] with rows at even distances; anything else is refused."""
    if x.dim() != 3:
        raise MtvError(-1, where)
    B, T, V = x.shape
    sb, st, sv = x.stride()
    if (V > 1 and sv != 1) or (B > 1 and T > 1 and sb != T * st) or x.dtype not in _LOGIT_TYPES:
        raise MtvError(-1, where)
    return _LOGIT_TYPES[x.dtype], st if T > 1 else sb if B > 1 else V


def _constrained_rows(tree, logits, rules, where):
    """(B, V, type, row stride) of a constrained call; rules of other sizes or of another device are refused."""
    dtype, stride = _logit_rows(logits, where)
    B, T, V = logits.shape
    if T != tree.T:
        _refuse(where, "logits")
    b, v, w, t, device = getattr(rules, "asks", (None,) * 5)
    if ((b is not None and b < B) or (v is not None and v != V) or (w is not None and w != (V + 31) // 32) or (t is not None and t != T) or
            (device is not None and device != logits.get_device())):
        _refuse(where, "rules")
    return B, V, dtype, stride


def logits_constrain(tree, logits, out, rules: LogitRules, tree_tok=None, stream=None):
    """logits, out [B][T][V], bf16 or fp32, rows evenly spaced; out may be logits."""
    where = "logits_constrain"
    B, V, dtype, stride = _constrained_rows(tree, logits, rules, where)
    dtype_out, stride_out = _logit_rows(out, where)
    kind = _F32 if dtype else _BF16
    _, x, y, tok = _look(where, ("logits", "out", "tree_tok"), logits, kind | _STRIDED, -1, out, kind | _STRIDED | _LIKE_PREVIOUS, -1,
                         tree_tok, _MAYBE_I32, B * tree.T)
    _check(lib().logits_constrain(tree.handle, B, V, dtype, x, stride, y, stride_out, rules, tok, _stream(stream)), where)


def constrained_argmax_keys(tree, logits, keys, rules: LogitRules, tree_tok=None, stream=None):
    """logits [B][T][V], bf16 or fp32, rows evenly spaced -> keys [B*T] (int64 storage of the uint64 keys)."""
    where = "constrained_argmax_keys"
    B, V, dtype, stride = _constrained_rows(tree, logits, rules, where)
    _, x, tok, keys_at = _look(where, ("logits", "tree_tok", "keys"), logits, (_F32 if dtype else _BF16) | _STRIDED, -1,
                               tree_tok, _MAYBE_I32, B * tree.T, keys, _I64, B * tree.T)
    _check(lib().constrained_argmax_keys(tree.handle, B, V, dtype, x, stride, rules, tok, keys_at, _stream(stream)), where)


def token_counts_add(tokens, counts, seen, lens=None, prompt=False, stream=None):
    """tokens [B][n] -> counts [B][V], seen [B][words]."""
    where = "token_counts_add"
    if tokens.dim() != 2 or counts.dim() != 2:
        _refuse(where, "tokens" if tokens.dim() != 2 else "counts")
    (B, n), V = tokens.shape, counts.shape[1]
    _, tok, ls, c, s = _look(where, ("tokens", "lens", "counts", "seen"), tokens, _I32, -1, lens, _MAYBE_I32, B, counts, _I32, B * V,
                             seen, _I32, B * ((V + 31) // 32))
    _check(lib().token_counts_add(B, V, n, tok, ls, 1 if prompt else 0, c, s, _stream(stream)), where)


KERNELS = ["heads_resblock", "heads_vocab_topk", "heads_merge", "attn_partial", "attn_combine",
           "argmax_partial", "accept_finish", "kv_compact", "seq_advance"]


class KernelTaps:
    """Per-kernel device timing through ``mtv_set_kernel_taps`` (CUDA events on the launch stream)."""

    def __init__(self, capacity_per_kernel: int):
        self.cap = capacity_per_kernel
        self.ev = {}
        for kid, name in enumerate(KERNELS):
            st = [torch.cuda.Event(enable_timing=True) for _ in range(self.cap)]
            sp = [torch.cuda.Event(enable_timing=True) for _ in range(self.cap)]
            for e in st + sp:
                e.record()          # torch creates the CUDA event lazily: force it now
            a = (C.c_void_p * self.cap)(*[e.cuda_event for e in st])
            b = (C.c_void_p * self.cap)(*[e.cuda_event for e in sp])
            self.ev[kid] = (st, sp, a, b)

    def __enter__(self):
        for kid, (_, _, a, b) in self.ev.items():
            _check(lib().mtv_set_kernel_taps(kid, a, b, self.cap), "mtv_set_kernel_taps")
        return self

    def __exit__(self, *exc):
        self.used = {kid: lib().mtv_kernel_taps_used(kid) for kid in self.ev}
        for kid in self.ev:
            lib().mtv_set_kernel_taps(kid, None, None, 0)

    def times_ms(self):
        """{kernel name: [ms per recorded launch]} — call after a device synchronize."""
        out = {}
        for kid, (st, sp, _, _) in self.ev.items():
            n = self.used[kid]
            out[KERNELS[kid]] = [st[i].elapsed_time(sp[i]) for i in range(n)]
        return out
