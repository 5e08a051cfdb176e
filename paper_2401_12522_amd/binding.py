"""ctypes binding of include/bita.h.  Argument marshalling only: every step of the
path runs in the HIP kernels of libbita.so.  torch supplies device memory and the
current stream."""
import ctypes as C
import functools
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.environ.get("BITA_LIBRARY") or os.path.join(_PKG, "libbita.so")   # override: another build of the same ABI
_lib = None

EXPORTS = [
    "bita_packed_bytes", "bita_pack_weight", "bita_model_create", "bita_model_destroy",
    "bita_workspace_bytes", "bita_tree_template_create", "bita_tree_template_destroy",
    "bita_tree_template_info", "bita_build_tree", "bita_verify_step", "bita_accept",
    "bita_compact_kv", "bita_decode_step", "bita_prefill_workspace_bytes", "bita_prefill_prepare", "bita_prefill", "bita_attention_workspace_bytes", "bita_attention_plan_info", "bita_attention_launch_info", "bita_tree_attention",
    "bita_gemm_workspace_bytes", "bita_gemm", "bita_gemm_noalloc_max_scratch_bytes", "bita_gemm_noalloc_scratch_bytes",
    "bita_gemm_noalloc", "bita_select", "bita_tune_gemm", "bita_gemm_plan_info", "bita_gemm_plan_detail", "bita_profile_enable",
    "bita_profile_disable", "bita_profile_read", "bita_last_error",
    "bita_quantize_rows", "bita_norm_q8", "bita_silu_mul_q8", "bita_packed_q8_bytes", "bita_pack_weight_q8",
    "bita_model_create_q8", "bita_gemm_q8_workspace_bytes", "bita_gemm_q8_plan_info", "bita_gemm_q8",
    "bita_kv_write_mx", "bita_kv_read_mx", "bita_qk_norm_rope", "bita_tree_attention_mx_workspace_bytes", "bita_tree_attention_mx_plan_info",
    "bita_tree_attention_mx", "bita_prompt_attention",
]


class BitaError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libbita error {code}: {msg}")
        self.code = code


class _Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim",
                                           "d_ffn", "vocab", "n_prompt", "n_mask", "max_pos")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float)]


class _Weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("tok_emb", "mask_emb", "final_norm", "lm_head")] + \
               [(n, C.POINTER(C.c_void_p)) for n in ("attn_norm", "ffn_norm", "wqkv", "wo", "w_gate_up",
                                                     "w_down", "prompt_k", "prompt_v")]


class _ScalesQ8(C.Structure):
    _fields_ = [(n, C.POINTER(C.c_void_p)) for n in ("wqkv", "wo", "w_gate_up", "w_down")]


class _KV(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_cache", "v_cache", "k_tree", "v_tree")] + \
               [(n, C.c_int32) for n in ("smax", "rows", "batch", "ctx_hint")] + \
               [("block_table", C.c_void_p)] + [(n, C.c_int32) for n in ("page_size", "n_pages", "max_pages")]


class _KVMX(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale")] + \
               [(n, C.c_int32) for n in ("bits", "batch", "n_kv_heads", "head_dim", "smax")] + \
               [("block_table", C.c_void_p)] + [(n, C.c_int32) for n in ("page_size", "n_pages", "max_pages")]


class _StepOut(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("token", "argmax", "topk_ids", "topk_val", "logits", "path", "n_acc", "bonus", "emitted",
                                           "next_group", "next_shift")]


def lib():
    """Load libbita.so (once).  Raises if it is missing: the product has no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} not built; run `python __graft_entry__.py` (or "
                           "paper_2401_12522_amd/build.py) first")
    L = C.CDLL(_LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    L.bita_packed_bytes.restype, L.bita_packed_bytes.argtypes = sz, [i64, i64]
    L.bita_pack_weight.restype, L.bita_pack_weight.argtypes = C.c_int, [vp, i64, i64, vp, i64, i64, i64, vp]
    L.bita_model_create.restype = C.c_int
    L.bita_model_create.argtypes = [C.POINTER(_Config), C.POINTER(_Weights), C.POINTER(vp)]
    L.bita_model_destroy.restype, L.bita_model_destroy.argtypes = None, [vp]
    L.bita_workspace_bytes.restype, L.bita_workspace_bytes.argtypes = sz, [vp, i32, i32]
    L.bita_tree_template_create.restype = C.c_int
    L.bita_tree_template_create.argtypes = [vp, vp, i32, i32, i32, C.POINTER(vp)]
    L.bita_tree_template_destroy.restype, L.bita_tree_template_destroy.argtypes = None, [vp]
    L.bita_tree_template_info.restype, L.bita_tree_template_info.argtypes = i32, [vp, i32]
    L.bita_build_tree.restype = C.c_int
    L.bita_build_tree.argtypes = [vp, vp, vp, i32, i32, vp, vp, i32, vp, vp]
    L.bita_verify_step.restype = C.c_int
    L.bita_verify_step.argtypes = [vp, C.POINTER(_KV), vp, vp, vp, i32, vp, sz, i32, vp, vp, vp, vp, vp]
    L.bita_accept.restype = C.c_int
    L.bita_accept.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    L.bita_compact_kv.restype = C.c_int
    L.bita_compact_kv.argtypes = [vp, C.POINTER(_KV), vp, i32, vp, vp, i32, vp]
    L.bita_decode_step.restype = C.c_int
    L.bita_decode_step.argtypes = [vp, C.POINTER(_KV), vp, vp, vp, i32, i32, vp, vp, vp, i32, vp, sz, i32, C.POINTER(_StepOut), vp]
    L.bita_prefill_workspace_bytes.restype, L.bita_prefill_workspace_bytes.argtypes = sz, [vp, i32, i32]
    L.bita_prefill_prepare.restype, L.bita_prefill_prepare.argtypes = C.c_int, [vp, i32, i32]
    L.bita_prefill.restype = C.c_int
    L.bita_prefill.argtypes = [vp, C.POINTER(_KV), vp, i32, vp, vp, i32, i32, vp, sz, vp, vp]
    L.bita_attention_workspace_bytes.restype = sz
    L.bita_attention_workspace_bytes.argtypes = [i32] * 6
    L.bita_tree_attention.restype = C.c_int
    L.bita_tree_attention.argtypes = [vp] * 12 + [i32] * 7 + [vp, sz, vp, vp, vp]
    L.bita_gemm_workspace_bytes.restype, L.bita_gemm_workspace_bytes.argtypes = sz, [i32, i64, i64]
    L.bita_gemm.restype, L.bita_gemm.argtypes = C.c_int, [vp, vp, i32, i64, i64, vp, i64, vp, sz, vp, vp]
    L.bita_gemm_noalloc_max_scratch_bytes.restype, L.bita_gemm_noalloc_max_scratch_bytes.argtypes = sz, []
    L.bita_gemm_noalloc_scratch_bytes.restype, L.bita_gemm_noalloc_scratch_bytes.argtypes = sz, [i32, i64, i64]
    L.bita_gemm_noalloc.restype, L.bita_gemm_noalloc.argtypes = C.c_int, [vp, vp, i32, i64, i64, vp, i64, vp, vp]
    L.bita_select.restype, L.bita_select.argtypes = C.c_int, [vp, vp, i32, i32, i32, vp, vp, vp, vp]
    L.bita_tune_gemm.restype, L.bita_tune_gemm.argtypes = None, [i32, i32]
    L.bita_gemm_plan_info.restype, L.bita_gemm_plan_info.argtypes = C.c_int, [i32, i64, i64, vp]
    L.bita_gemm_plan_detail.restype, L.bita_gemm_plan_detail.argtypes = C.c_int, [i32, i64, i64, i32, vp]
    L.bita_attention_plan_info.restype, L.bita_attention_plan_info.argtypes = C.c_int, [i32] * 8 + [vp]
    L.bita_attention_launch_info.restype, L.bita_attention_launch_info.argtypes = C.c_int, [i32] * 8 + [vp]
    L.bita_profile_enable.restype, L.bita_profile_enable.argtypes = C.c_int, [i32]
    L.bita_profile_disable.restype, L.bita_profile_disable.argtypes = None, []
    L.bita_profile_read.restype, L.bita_profile_read.argtypes = C.c_int, [i32, vp, vp, vp]
    L.bita_last_error.restype, L.bita_last_error.argtypes = C.c_char_p, []
    L.bita_quantize_rows.restype, L.bita_quantize_rows.argtypes = C.c_int, [vp, i32, i32, i64, i64, vp, i64, vp, vp]
    L.bita_norm_q8.restype = C.c_int
    L.bita_norm_q8.argtypes = [vp, i32, i32, i64, i64, vp, i32, i64, vp, C.c_float, vp, i64, vp, i64, vp, vp]
    L.bita_silu_mul_q8.restype, L.bita_silu_mul_q8.argtypes = C.c_int, [vp, i32, i32, i64, i64, i32, vp, i64, vp, vp]
    L.bita_packed_q8_bytes.restype, L.bita_packed_q8_bytes.argtypes = sz, [i64, i64]
    L.bita_pack_weight_q8.restype, L.bita_pack_weight_q8.argtypes = C.c_int, [vp, i64, i64, i64, vp, i64, i64, i64, vp]
    L.bita_model_create_q8.restype = C.c_int
    L.bita_model_create_q8.argtypes = [C.POINTER(_Config), C.POINTER(_Weights), C.POINTER(_ScalesQ8), C.POINTER(vp)]
    L.bita_gemm_q8_workspace_bytes.restype, L.bita_gemm_q8_workspace_bytes.argtypes = sz, [i32, i64, i64]
    L.bita_gemm_q8_plan_info.restype, L.bita_gemm_q8_plan_info.argtypes = C.c_int, [i32, i64, i64, vp]
    L.bita_gemm_q8.restype, L.bita_gemm_q8.argtypes = C.c_int, [vp, i64, vp, i32, i64, vp, vp, i64, vp, sz, vp, i32, i64, vp]
    kvp = C.POINTER(_KVMX)
    L.bita_kv_write_mx.restype = C.c_int
    L.bita_kv_write_mx.argtypes = [kvp, vp, i64, i64, i64, vp, i64, i64, i64, i32, i32, vp, vp, vp, i32, vp, vp]
    L.bita_kv_read_mx.restype = C.c_int
    L.bita_kv_read_mx.argtypes = [kvp, vp, i64, i64, i64, vp, i64, i64, i64, i32, i32, vp, vp, vp]
    L.bita_qk_norm_rope.restype = C.c_int
    L.bita_qk_norm_rope.argtypes = [vp, i32, i32, i64, i32, i32, i32, vp, vp, C.c_float, vp, vp, vp, i32, vp, i64, i64, vp, i64, i64, vp, i64, i64, vp]
    L.bita_tree_attention_mx_workspace_bytes.restype, L.bita_tree_attention_mx_workspace_bytes.argtypes = sz, [i32] * 8
    L.bita_tree_attention_mx_plan_info.restype, L.bita_tree_attention_mx_plan_info.argtypes = C.c_int, [i32] * 8 + [vp]
    L.bita_tree_attention_mx.restype = C.c_int
    L.bita_tree_attention_mx.argtypes = [vp, vp, kvp, vp, i64, i64, i64, vp, i64, i64, i64, vp, vp, i32, vp, vp, i32, i32, vp, sz, vp, vp]
    L.bita_prompt_attention.restype = C.c_int
    L.bita_prompt_attention.argtypes = [vp, i64, i64, vp, i64, i64, vp, i64, i64, vp, i32, i32, i32, i32, i32, vp, i64, vp]
    _lib = L
    return L


def _check(rc):
    if rc != 0:
        raise BitaError(rc, lib().bita_last_error().decode())


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(0)


def _stream():
    # the current stream's handle without building a Stream object around it (3.2 -> 0.4 us, and a step
    # asks four times); a null handle is the default stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # not a public name: a torch may come without it
    return C.c_void_p(raw(torch.cuda.current_device()) if raw else torch.cuda.current_stream().cuda_stream)


def packed_bytes(n_rows, k):
    return lib().bita_packed_bytes(n_rows, k)


def pack_weight(src, dst=None, tile0=0, tile_stride=1, total_rows=None):
    """src: bf16 cuda tensor [N][K].  Returns the packed uint8 buffer (allocated here
    when dst is None, sized for total_rows rows)."""
    n, k = src.shape
    assert src.dtype == torch.bfloat16 and src.is_cuda and src.is_contiguous()
    total_rows = total_rows or n
    if dst is None:
        dst = torch.empty(packed_bytes(total_rows, k), dtype=torch.uint8, device=src.device)
    _check(lib().bita_pack_weight(_ptr(src), n, k, _ptr(dst), total_rows, tile0, tile_stride, _stream()))
    return dst


class TreeTemplate:
    def __init__(self, parent, is_mask, n_tree, n_mask):
        parent = np.ascontiguousarray(parent, np.int32)
        is_mask = np.ascontiguousarray(is_mask, np.uint8)
        self.handle = C.c_void_p()
        _check(lib().bita_tree_template_create(parent.ctypes.data_as(C.c_void_p), is_mask.ctypes.data_as(C.c_void_p),
                                               int(n_tree), int(parent.shape[0]), int(n_mask), C.byref(self.handle)))
        info = lambda w: lib().bita_tree_template_info(self.handle, w)   # noqa: E731
        self.rows, self.n_tree, self.n_groups = info(0), info(1), info(2)
        self.depth, self.kmax, self.words = info(3), info(4), info(5)
        self.n_mask = int(n_mask)

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.bita_tree_template_destroy(self.handle)
            self.handle = None


class Model:
    """Packs the matrices of a weight source (anything with .torch(name, layer) giving bf16
    cuda tensors [out][in]) and creates the library handle.  The packed buffers and the
    small row-major tensors are kept alive here; the library only borrows them.
    int8: the layers' matrices as 8-bit integers, one scale for each of their rows (the LM head stays bfloat16)."""

    def __init__(self, cfg, weights, max_pos, n_layers=None, free_source=False, int8=False):
        self.cfg, self.int8 = cfg, bool(int8)
        L = cfg.n_layers if n_layers is None else n_layers
        self.n_layers = L
        dev = torch.device("cuda")
        keep = self._keep = []
        hd = cfg.head_dim

        def pack_many(parts, k, interleave=False):
            total = sum(p.shape[0] for p in parts)
            dst = torch.empty(packed_bytes(total, k), dtype=torch.uint8, device=dev)
            if interleave:
                for i, p in enumerate(parts):
                    pack_weight(p.contiguous(), dst, i, len(parts), total_rows=total)
            else:
                row = 0
                for p in parts:
                    pack_weight(p.contiguous(), dst, row // 16, 1, total_rows=total)
                    row += p.shape[0]
            keep.append(dst)
            return dst

        def pack_many_q8(parts, k, interleave=False):
            total = sum(p.shape[0] for p in parts)
            dst = torch.empty(packed_q8_bytes(total, k), dtype=torch.uint8, device=dev)
            scales, row = [], 0
            for i, p in enumerate(parts):
                q, s = quantize_rows(p.contiguous())
                pack_weight_q8(q, dst, i if interleave else row // 16, len(parts) if interleave else 1, total_rows=total)
                scales.append(s.view(-1, 16) if interleave else s)
                row += p.shape[0]
            scale = torch.stack(scales, 1).reshape(-1) if interleave else torch.cat(scales)
            keep.extend((dst, scale))
            return dst, scale

        def small(name, layer=None):
            t = weights.torch(name, layer).to(dev).contiguous()
            keep.append(t)
            return t

        def arr(ts):
            a = (C.c_void_p * len(ts))(*[t.data_ptr() for t in ts])
            keep.append(a)
            return a
        cols = {n: [] for n in ("attn_norm", "ffn_norm", "wqkv", "wo", "w_gate_up", "w_down", "prompt_k", "prompt_v")}
        scales = {n: [] for n in ("wqkv", "wo", "w_gate_up", "w_down")}
        for l in range(L):
            g = lambda n: weights.torch(n, l).to(dev)     # noqa: E731
            for name, parts, k, interleave in (("wqkv", ("wq", "wk", "wv"), cfg.d_model, False), ("wo", ("wo",), cfg.n_heads * hd, False),
                                               ("w_gate_up", ("w_gate", "w_up"), cfg.d_model, True), ("w_down", ("w_down",), cfg.d_ffn, False)):
                parts = [g(p) for p in parts]
                if int8:
                    packed, scale = pack_many_q8(parts, k, interleave)
                    scales[name].append(scale)
                else:
                    packed = pack_many(parts, k, interleave)
                cols[name].append(packed)
            cols["attn_norm"].append(small("attn_norm", l))
            cols["ffn_norm"].append(small("ffn_norm", l))
            if cfg.n_prompt > 0:
                cols["prompt_k"].append(small("prompt_k", l))
                cols["prompt_v"].append(small("prompt_v", l))
            if free_source:
                torch.cuda.synchronize()
                for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down"):
                    weights._store.pop((n, l), None)
        w = _Weights()
        w.tok_emb = small("tok_emb").data_ptr()
        w.mask_emb = small("mask_emb").data_ptr() if cfg.n_mask > 0 else None
        w.final_norm = small("final_norm").data_ptr()
        w.lm_head = pack_many([weights.torch("lm_head").to(dev)], cfg.d_model).data_ptr()
        for n, ts in cols.items():
            if ts:
                setattr(w, n, arr(ts))
        c = _Config(L, cfg.d_model, cfg.n_heads, cfg.n_kv_heads, hd, cfg.d_ffn, cfg.vocab, cfg.n_prompt,
                    cfg.n_mask, int(max_pos), cfg.rms_eps, cfg.rope_theta)
        torch.cuda.synchronize()
        self.max_pos = int(max_pos)
        self.handle = C.c_void_p()
        if int8:
            sq = _ScalesQ8(**{n: arr(ts) for n, ts in scales.items()})
            _check(lib().bita_model_create_q8(C.byref(c), C.byref(w), C.byref(sq), C.byref(self.handle)))
        else:
            _check(lib().bita_model_create(C.byref(c), C.byref(w), C.byref(self.handle)))

    def workspace_bytes(self, batch, rows):
        return lib().bita_workspace_bytes(self.handle, batch, rows)

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.bita_model_destroy(self.handle)
            self.handle = None


class KVState:
    """Caller-owned KV cache, per-pass tree scratch and ctx_len for `batch` sequences."""

    def __init__(self, cfg, n_layers, batch, smax, rows):
        dev = torch.device("cuda")
        shape_c = (n_layers, batch, cfg.n_kv_heads, smax, cfg.head_dim)
        shape_t = (n_layers, batch, cfg.n_kv_heads, rows, cfg.head_dim)
        self.k_cache = torch.zeros(shape_c, dtype=torch.bfloat16, device=dev)
        self.v_cache = torch.zeros(shape_c, dtype=torch.bfloat16, device=dev)
        self.k_tree = torch.zeros(shape_t, dtype=torch.bfloat16, device=dev)
        self.v_tree = torch.zeros(shape_t, dtype=torch.bfloat16, device=dev)
        self.ctx_len = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.smax, self.rows, self.batch = smax, rows, batch

    def resize_rows(self, n_layers, cfg, rows):
        """Lay the per-pass scratch out for a template of `rows` rows (the template may change from
        step to step).  The memory is kept when it is large enough; the contents are undefined."""
        shape_t = (n_layers, self.batch, cfg.n_kv_heads, rows, cfg.head_dim)
        n = n_layers * self.batch * cfg.n_kv_heads * rows * cfg.head_dim
        for name in ("k_tree", "v_tree"):
            flat = getattr(self, "_" + name + "_flat", None)
            if flat is None:
                flat = getattr(self, name).reshape(-1)
            if flat.numel() < n:
                flat = torch.zeros(n, dtype=torch.bfloat16, device=self.k_cache.device)
            setattr(self, "_" + name + "_flat", flat)
            setattr(self, name, flat[:n].view(shape_t))
        self.rows = rows

    def desc(self, ctx_hint):
        return _KV(self.k_cache.data_ptr(), self.v_cache.data_ptr(), self.k_tree.data_ptr(),
                   self.v_tree.data_ptr(), self.smax, self.rows, self.batch, int(ctx_hint), None, 0, 0, 0)


class PagedKVState(KVState):
    """KV state whose caches are page pools [n_layers][n_pages][n_kv_heads][page_size][head_dim];
    block_table [batch][max_pages] names the pages of every sequence (here: a seeded shuffle of
    the pool, so that neighbouring slots of a sequence are not neighbours in memory)."""

    def __init__(self, cfg, n_layers, batch, smax, rows, page_size, n_pages=None, seed=0):
        dev = torch.device("cuda")
        self.page_size = int(page_size)
        self.max_pages = (smax + page_size - 1) // page_size
        self.n_pages = int(n_pages or batch * self.max_pages)
        assert self.n_pages >= batch * self.max_pages
        shape_c = (n_layers, self.n_pages, cfg.n_kv_heads, page_size, cfg.head_dim)
        shape_t = (n_layers, batch, cfg.n_kv_heads, rows, cfg.head_dim)
        self.k_cache = torch.zeros(shape_c, dtype=torch.bfloat16, device=dev)
        self.v_cache = torch.zeros(shape_c, dtype=torch.bfloat16, device=dev)
        self.k_tree = torch.zeros(shape_t, dtype=torch.bfloat16, device=dev)
        self.v_tree = torch.zeros(shape_t, dtype=torch.bfloat16, device=dev)
        self.ctx_len = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.smax, self.rows, self.batch = smax, rows, batch
        perm = np.random.default_rng(seed).permutation(self.n_pages)[: batch * self.max_pages]
        self.block_table = torch.tensor(perm.reshape(batch, self.max_pages), dtype=torch.int32, device=dev)

    def desc(self, ctx_hint):
        return _KV(self.k_cache.data_ptr(), self.v_cache.data_ptr(), self.k_tree.data_ptr(),
                   self.v_tree.data_ptr(), self.smax, self.rows, self.batch, int(ctx_hint),
                   self.block_table.data_ptr(), self.page_size, self.n_pages, self.max_pages)

    def contiguous(self, b):
        """(k, v) of sequence b as [n_layers][n_kv_heads][max_pages * page_size][head_dim] copies."""
        pages = self.block_table[b].long()
        def one(pool):
            x = pool[:, pages]                                      # [L][max_pages][Hkv][page][hd]
            return x.permute(0, 2, 1, 3, 4).reshape(x.shape[0], x.shape[2], -1, x.shape[4])
        return one(self.k_cache), one(self.v_cache)

    def load_contiguous(self, b, k, v, n):
        """Write slots 0..n-1 of sequence b from k, v [n_layers][n_kv_heads][>= n][head_dim]; sets ctx_len[b] = n."""
        for i in range((n + self.page_size - 1) // self.page_size):
            lo, hi = i * self.page_size, min((i + 1) * self.page_size, n)
            page = int(self.block_table[b, i])
            self.k_cache[:, page, :, : hi - lo] = k[:, :, lo:hi]
            self.v_cache[:, page, :, : hi - lo] = v[:, :, lo:hi]
        self.ctx_len[b] = n


class StepBuffers:
    """Device outputs of one step for a given template and batch."""

    def __init__(self, model, tmpl, batch, kmax, want_logits=False):
        dev = torch.device("cuda")
        i32 = dict(dtype=torch.int32, device=dev)
        self.kmax = int(kmax)
        self.token = torch.zeros((batch, tmpl.rows), **i32)
        self.argmax = torch.zeros((batch, tmpl.n_tree), **i32)
        nm = max(tmpl.n_groups * tmpl.n_mask, 1)
        self.topk_ids = torch.zeros((batch, nm, self.kmax), **i32)
        self.topk_val = torch.zeros((batch, nm, self.kmax), dtype=torch.float32, device=dev)
        self.logits = torch.zeros((batch, tmpl.rows, model.cfg.vocab), dtype=torch.float32, device=dev) if want_logits else None
        self.path = torch.zeros((batch, tmpl.depth + 1), **i32)
        self.n_acc = torch.zeros(batch, **i32)
        self.bonus = torch.zeros(batch, **i32)
        self.emitted = torch.zeros((batch, tmpl.depth + 1), **i32)
        self.next_group = torch.zeros(batch, **i32)
        self.next_shift = torch.zeros(batch, **i32)
        self.workspace = torch.empty(model.workspace_bytes(batch, tmpl.rows), dtype=torch.uint8, device=dev)


def build_tree(tmpl, root_token, cand, group, shift, batch, token_out):
    cand_rows, kmax = (cand.shape[1], cand.shape[2]) if cand is not None else (0, 0)
    _check(lib().bita_build_tree(tmpl.handle, _ptr(root_token), _ptr(cand), cand_rows, kmax, _ptr(group),
                                 _ptr(shift), batch, _ptr(token_out), _stream()))


def verify_step(model, kv, ctx_hint, tmpl, buf, batch):
    d = kv.desc(ctx_hint)
    has_masks = tmpl.n_groups > 0
    _check(lib().bita_verify_step(model.handle, C.byref(d), tmpl.handle, _ptr(buf.token), _ptr(kv.ctx_len), batch,
                                  _ptr(buf.workspace), buf.workspace.numel(), buf.kmax, _ptr(buf.argmax),
                                  _ptr(buf.topk_ids if has_masks else None),
                                  _ptr(buf.topk_val if has_masks else None), _ptr(buf.logits), _stream()))


def accept(tmpl, buf, batch):
    _check(lib().bita_accept(tmpl.handle, _ptr(buf.token), _ptr(buf.argmax), batch, _ptr(buf.path),
                             _ptr(buf.n_acc), _ptr(buf.bonus), _ptr(buf.emitted), _ptr(buf.next_group),
                             _ptr(buf.next_shift), _stream()))


def compact_kv(model, kv, ctx_hint, buf, batch, path=None, n_acc=None):
    d = kv.desc(ctx_hint)
    path = buf.path if path is None else path
    n_acc = buf.n_acc if n_acc is None else n_acc
    _check(lib().bita_compact_kv(model.handle, C.byref(d), _ptr(path), path.shape[1], _ptr(n_acc),
                                 _ptr(kv.ctx_len), batch, _stream()))


def prefill_workspace(model, batch, chunk_rows):
    """A workspace tensor for prefill() with these sizes."""
    need = lib().bita_prefill_workspace_bytes(model.handle, batch, chunk_rows)
    return torch.empty(need, dtype=torch.uint8, device="cuda")


def prefill_prepare(model, n_tokens, chunk_rows):
    """Create the model's chain templates for this chunking ahead of time (needed before a
    prefill is captured into a graph)."""
    _check(lib().bita_prefill_prepare(model.handle, int(n_tokens), int(chunk_rows)))


def prefill(model, kv, ctx_hint, tokens, chunk_rows, seq_len=None, workspace=None, next_token=None):
    """tokens int32 cuda [B][n]; appends them (row b up to seq_len[b]) to the cache by chunked causal
    passes.  Returns the greedy token after each sequence's last one, int32 cuda [B] (written into
    next_token when given; with workspace and next_token supplied nothing is allocated here)."""
    batch, n = tokens.shape
    assert tokens.dtype == torch.int32 and tokens.is_contiguous()
    need = lib().bita_prefill_workspace_bytes(model.handle, batch, chunk_rows)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=tokens.device)
    if next_token is None:
        next_token = torch.full((batch,), -1, dtype=torch.int32, device=tokens.device)
    d = kv.desc(ctx_hint)
    _check(lib().bita_prefill(model.handle, C.byref(d), _ptr(tokens), n, _ptr(seq_len), _ptr(kv.ctx_len), batch,
                              int(chunk_rows), _ptr(workspace), workspace.numel(), _ptr(next_token), _stream()))
    return next_token


def decode_step(model, kv, ctx_hint, tmpl, buf, batch, root_token, cand, group=None, shift=None):
    """The four calls of one step on the current stream (no host sync), by the library's own call for all of them."""
    if buf.path.shape[1] == tmpl.depth + 1:
        d = kv.desc(ctx_hint)
        ptr = lambda t: t.data_ptr() if t is not None else None                     # noqa: E731
        has_masks = tmpl.n_groups > 0
        out = _StepOut(ptr(buf.token), ptr(buf.argmax), ptr(buf.topk_ids) if has_masks else None, ptr(buf.topk_val) if has_masks else None,
                       ptr(buf.logits), ptr(buf.path), ptr(buf.n_acc), ptr(buf.bonus), ptr(buf.emitted), ptr(buf.next_group), ptr(buf.next_shift))
        cand_rows, kmax = (cand.shape[1], cand.shape[2]) if cand is not None else (0, 0)
        _check(lib().bita_decode_step(model.handle, C.byref(d), tmpl.handle, _ptr(root_token), _ptr(cand), cand_rows, kmax, _ptr(group),
                                      _ptr(shift), _ptr(kv.ctx_len), batch, _ptr(buf.workspace), buf.workspace.numel(), buf.kmax,
                                      C.byref(out), _stream()))
        return
    build_tree(tmpl, root_token, cand, group, shift, batch, buf.token)
    verify_step(model, kv, ctx_hint, tmpl, buf, batch)
    accept(tmpl, buf, batch)
    compact_kv(model, kv, ctx_hint, buf, batch)


def profile_enable(max_records):
    _check(lib().bita_profile_enable(int(max_records)))


def profile_read(capacity):
    """Returns (ms[n], weight_bytes[n]) of the GEMM launches recorded since profile_enable."""
    n = C.c_int32(0)
    ms = np.zeros(capacity, np.float32)
    wb = np.zeros(capacity, np.int64)
    _check(lib().bita_profile_read(capacity, C.byref(n), ms.ctypes.data_as(C.c_void_p), wb.ctypes.data_as(C.c_void_p)))
    lib().bita_profile_disable()
    return ms[: n.value], wb[: n.value]


def gemm(a, w_packed, n_rows, k=None, a_lo=None):
    """a (and optionally a_lo, the residual plane): bf16 cuda [M][lda]; returns fp32 [M][n_rows]."""
    m, lda = a.shape
    k = lda if k is None else k
    ws = torch.empty(lib().bita_gemm_workspace_bytes(m, n_rows, k), dtype=torch.uint8, device=a.device)
    out = torch.empty((m, n_rows), dtype=torch.float32, device=a.device)
    _check(lib().bita_gemm(_ptr(a), _ptr(a_lo), m, k, lda, _ptr(w_packed), n_rows, _ptr(ws), ws.numel(), _ptr(out), _stream()))
    return out


def gemm_noalloc(a, w_packed, n_rows, out, k=None, a_lo=None):
    """bita_gemm_noalloc: as gemm(), but the library's static scratch replaces the workspace and the
    caller brings the output (fp32 cuda [M][n_rows]); nothing is allocated by the call."""
    m, lda = a.shape
    k = lda if k is None else k
    assert out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == (m, n_rows)
    _check(lib().bita_gemm_noalloc(_ptr(a), _ptr(a_lo), m, k, lda, _ptr(w_packed), n_rows, _ptr(out), _stream()))
    return out


def gemm_plan_info(m_rows, n_rows, k, planes=2):
    """{splits, variant, mt_pass, ksteps_per_split, tall_tiles} the launch heuristic picks for this GEMM shape
    with `planes` activation planes."""
    out = (C.c_int32 * 5)()
    _check(lib().bita_gemm_plan_detail(int(m_rows), int(n_rows), int(k), int(planes), out))
    return dict(splits=out[0], variant=out[1], mt_pass=out[2], ksteps_per_split=out[3], tall_tiles=out[4])


def attention_plan_info(batch, rows, heads, kv_heads, head_dim, ctx_hint, n_prompt=0, page_size=0):
    """{splits, heads, rows, waves (of a workgroup), workgroups} that tree attention over these sizes is cut into, before
    neighbouring row tiles of a head are joined to workgroups that share chunks (attention_launch_info)."""
    out = (C.c_int32 * 5)()
    _check(lib().bita_attention_plan_info(batch, rows, heads, kv_heads, head_dim, int(ctx_hint), n_prompt, page_size, out))
    return dict(splits=out[0], heads=out[1], rows=out[2], waves=out[3], workgroups=out[4])


def attention_launch_info(batch, rows, heads, kv_heads, head_dim, ctx_hint, n_prompt=0, page_size=0):
    """{splits, heads, rows, waves (of a workgroup), workgroups, share (row tiles that share chunks in one), ranked
    (sequences start longest first)} that tree attention over these sizes launches."""
    out = (C.c_int32 * 7)()
    _check(lib().bita_attention_launch_info(batch, rows, heads, kv_heads, head_dim, int(ctx_hint), n_prompt, page_size, out))
    return dict(splits=out[0], heads=out[1], rows=out[2], waves=out[3], workgroups=out[4], share=out[5], ranked=bool(out[6]))


def select(tmpl, logits, kmax):
    """logits fp32 cuda [B][R][vocab] -> (argmax int32 [B][T], topk_ids int32 [B][G*n][kmax], topk_val fp32)."""
    B, R, V = logits.shape
    assert R == tmpl.rows and logits.dtype == torch.float32 and logits.is_contiguous()
    argmax = torch.empty((B, tmpl.n_tree), dtype=torch.int32, device=logits.device)
    n_sel = tmpl.n_groups * tmpl.n_mask
    ids = torch.empty((B, n_sel, kmax), dtype=torch.int32, device=logits.device)
    val = torch.empty((B, n_sel, kmax), dtype=torch.float32, device=logits.device)
    _check(lib().bita_select(tmpl.handle, _ptr(logits), B, V, kmax, _ptr(argmax), _ptr(ids), _ptr(val), _stream()))
    return argmax, ids, val


def tree_attention(tmpl, q, k_cache, v_cache, k_tree, v_tree, prompt_k, prompt_v, ctx_len, ctx_hint, q_lo=None,
                   k_tree_lo=None, v_tree_lo=None, two_plane_out=False):
    """q [B][R][Hq][hd]; k/v_cache [B][Hkv][smax][hd]; k/v_tree [B][Hkv][R][hd];
    prompt_k/v [Hkv][P][hd] or None; q_lo, k_tree_lo, v_tree_lo: optional low bf16 planes.  Returns bf16
    [B][R][Hq*hd], or the pair (hi, lo) of bf16 planes when two_plane_out."""
    B, R, Hq, hd = q.shape
    Hkv, smax = k_cache.shape[1], k_cache.shape[2]
    P = 0 if prompt_k is None else prompt_k.shape[1]
    ws = torch.empty(lib().bita_attention_workspace_bytes(B, R, Hq, hd, int(ctx_hint), P), dtype=torch.uint8, device=q.device)
    out = torch.empty((B, R, Hq * hd), dtype=torch.bfloat16, device=q.device)
    out_lo = torch.empty_like(out) if two_plane_out else None
    _check(lib().bita_tree_attention(tmpl.handle, _ptr(q), _ptr(q_lo), _ptr(k_cache), _ptr(v_cache), _ptr(k_tree), _ptr(v_tree),
                                     _ptr(k_tree_lo), _ptr(v_tree_lo), _ptr(prompt_k), _ptr(prompt_v), _ptr(ctx_len), B, Hq, Hkv, hd, P, smax,
                                     int(ctx_hint), _ptr(ws), ws.numel(), _ptr(out), _ptr(out_lo), _stream()))
    return (out, out_lo) if two_plane_out else out


# ---- 8-bit linear layers ---------------------------------------------------------------------------------------------
# (Called for every layer of a pass: arguments are looked at once each, pointers go over as integers.)
_F32_BF16 = {torch.float32: 0, torch.bfloat16: 1}
_I8 = {torch.int8: 2}


# the current stream's handle (as in _stream)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


@functools.lru_cache(4096)
def _gemm_q8_scratch(m, n, k):
    return lib().bita_gemm_q8_workspace_bytes(m, n, k)


def _matrix(name, t, types, dev, rows=None, cols=None):
    """Rows, columns and row stride of t, a matrix of one of these types (and this size) on the current device whose rows have
    neighbouring elements and do not overlap."""
    if t.dtype in types and t.dim() == 2 and t.get_device() == dev:
        r, c = t.shape
        ld, step = t.stride()
        if r > 0 and c > 0 and (rows is None or r == rows) and (cols is None or c == cols) and (step == 1 or c == 1) and (ld >= c or r == 1):
            return r, c, ld if r > 1 else c
    raise ValueError(f"{name}: wanted {rows or 'any'} x {cols or 'any'} of {' or '.join(str(x) for x in types)} on cuda:{dev}, rows of neighbouring elements "
                     f"that do not overlap; got {tuple(t.shape)} of {t.dtype} on {t.device}, strides {tuple(t.stride())}")


def _vector(name, t, n, dtype, dev):
    if not (t.dtype is dtype and t.get_device() == dev and t.dim() == 1 and t.numel() == n and (n < 2 or t.stride(0) == 1)):
        raise ValueError(f"{name}: wanted {n} neighbouring {dtype} on cuda:{dev}; got {tuple(t.shape)} of {t.dtype} on {t.device}, strides {tuple(t.stride())}")


def _bytes(name, t, n, dev):
    if not (t.dtype is torch.uint8 and t.get_device() == dev and t.is_contiguous() and t.numel() >= n):
        raise ValueError(f"{name}: wanted a contiguous buffer of {n} uint8 on cuda:{dev}; got {tuple(t.shape)} of {t.dtype} on {t.device}")


def empty_q8(rows, cols, device="cuda"):
    """An int8 matrix whose rows are a multiple of 16 bytes apart, as gemm_q8 reads them."""
    return torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device=device)[:, :cols]


def _q8_out(x, rows, cols, q, scale, dev):
    if q is None:
        q = empty_q8(rows, cols, x.device)
    if scale is None:
        scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    else:
        _vector("scale", scale, rows, torch.float32, dev)
    return q, scale, _matrix("q", q, _I8, dev, rows, cols)[2]


def quantize_rows(x, q=None, scale=None):
    """x: cuda [M][K], float32 or bfloat16.  Every row as 8-bit integers and a scale: (q int8 [M][K], scale fp32 [M]), written into
    q and scale where they are given."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    m, k, ldx = _matrix("x", x, _F32_BF16, dev)
    q, scale, ldq = _q8_out(x, m, k, q, scale, dev)
    rc = L.bita_quantize_rows(x.data_ptr(), _F32_BF16[x.dtype], m, k, ldx, q.data_ptr(), ldq, scale.data_ptr(), _raw_stream(dev))
    if rc:
        _check(rc)
    return q, scale


def norm_q8(x, gain, eps, delta=None, total=None, q=None, scale=None):
    """RMSNorm of x + delta times gain (bfloat16 [D]), rows as 8-bit integers: (q, scale).  x, delta: cuda [M][D], float32 or
    bfloat16.  With delta, x + delta is stored in total (x's type and size); total None: in x itself."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    m, d, ldx = _matrix("x", x, _F32_BF16, dev)
    _vector("gain", gain, d, torch.bfloat16, dev)
    pd = td = ldd = pt = ldt = 0
    if delta is not None:
        ldd = _matrix("delta", delta, _F32_BF16, dev, m, d)[2]
        pd, td = delta.data_ptr(), _F32_BF16[delta.dtype]
        total = x if total is None else total
        ldt = _matrix("total", total, {x.dtype: 0}, dev, m, d)[2]
        pt = total.data_ptr()
    elif total is not None:
        raise ValueError("total: there is nothing to store without delta")
    q, scale, ldq = _q8_out(x, m, d, q, scale, dev)
    rc = L.bita_norm_q8(x.data_ptr(), _F32_BF16[x.dtype], m, d, ldx, pd, td, ldd, gain.data_ptr(), eps, pt, ldt, q.data_ptr(), ldq, scale.data_ptr(),
                        _raw_stream(dev))
    if rc:
        _check(rc)
    return q, scale


def silu_mul_q8(gate_up, tile=0, q=None, scale=None):
    """silu(gate) * up of gate_up, cuda [M][2F], float32 or bfloat16, rows as 8-bit integers: (q int8 [M][F], scale).  tile 16: tiles of
    16 gate columns, each followed by its 16 up columns, as a product with an interleaved weight leaves them; tile 0: all gate columns first."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    m, f2, ldx = _matrix("gate_up", gate_up, _F32_BF16, dev)
    if f2 % 2:
        raise ValueError(f"gate_up: {f2} columns are not two halves")
    q, scale, ldq = _q8_out(gate_up, m, f2 // 2, q, scale, dev)
    rc = L.bita_silu_mul_q8(gate_up.data_ptr(), _F32_BF16[gate_up.dtype], m, f2 // 2, ldx, tile, q.data_ptr(), ldq, scale.data_ptr(), _raw_stream(dev))
    if rc:
        _check(rc)
    return q, scale


def packed_q8_bytes(n_rows, k):
    return lib().bita_packed_q8_bytes(n_rows, k)


def pack_weight_q8(src, dst=None, tile0=0, tile_stride=1, total_rows=None):
    """src: int8 cuda [N][K] (quantize_rows of a weight).  Returns the packed uint8 buffer (allocated here when dst is None,
    sized for total_rows rows)."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    n, k, ld = _matrix("src", src, _I8, dev)
    total_rows = total_rows or n
    need = packed_q8_bytes(total_rows, k)
    if dst is None:
        dst = torch.empty(need, dtype=torch.uint8, device=src.device)
    _bytes("dst", dst, need, dev)
    _check(L.bita_pack_weight_q8(src.data_ptr(), n, k, ld, dst.data_ptr(), total_rows, tile0, tile_stride, _raw_stream(dev)))
    return dst


def gemm_q8_plan_info(m_rows, n_rows, k):
    """{rows, cols (of a workgroup), splits (of k), skinny} that gemm_q8 of these sizes launches."""
    out = (C.c_int32 * 4)()
    _check(lib().bita_gemm_q8_plan_info(int(m_rows), int(n_rows), int(k), out))
    return dict(rows=out[0], cols=out[1], splits=out[2], skinny=bool(out[3]))


def gemm_q8(a, a_scale, w_packed, w_scale, n_rows, out=None, out_dtype=torch.float32, workspace=None):
    """a: int8 cuda [M][K] with its rows' scales (quantize_rows, norm_q8, silu_mul_q8); w_packed: pack_weight_q8 of an int8 [n_rows][K],
    w_scale its rows' scales in packed order.  Returns [M][n_rows] in float32 or bfloat16, written into out where it is given.
    workspace: a uint8 cuda tensor of bita_gemm_q8_workspace_bytes (allocated here when it is None and one is needed)."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    m, k, lda = _matrix("a", a, _I8, dev)
    k16, pa = (k + 15) & ~15, a.data_ptr()
    if m == 1:
        lda = k16
    if lda & 15 or pa & 15 or a.untyped_storage().nbytes() - a.storage_offset() < (m - 1) * lda + k16:
        raise ValueError("a: rows have to start at multiples of 16 bytes and to be readable to the next one behind their end (empty_q8)")
    _vector("a_scale", a_scale, m, torch.float32, dev)
    _vector("w_scale", w_scale, n_rows, torch.float32, dev)
    _bytes("w_packed", w_packed, (n_rows + 15 >> 4) * (k + 127 >> 7) * 2048, dev)
    if out is None:
        out = torch.empty((m, n_rows), dtype=out_dtype, device=a.device)
    ldo = _matrix("out", out, _F32_BF16, dev, m, n_rows)[2]
    pw = nw = 0
    if workspace is None:
        nw = _gemm_q8_scratch(m, n_rows, k)
        if nw:
            workspace = torch.empty(nw, dtype=torch.uint8, device=a.device)
    else:
        _bytes("workspace", workspace, 0, dev)
        nw = workspace.numel()
    if nw:
        pw = workspace.data_ptr()
    rc = L.bita_gemm_q8(pa, lda, a_scale.data_ptr(), m, k, w_packed.data_ptr(), w_scale.data_ptr(), n_rows, pw, nw, out.data_ptr(), _F32_BF16[out.dtype],
                        ldo, _raw_stream(dev))
    if rc:
        _check(rc)
    return out


# ---- a K/V cache in 4 or 8 bits, and the attention block around it ------------------------------------------------------------
# (Called for every layer of a pass: a tensor is asked for each thing once, messages are made up only for what is refused.)
_BF16, _I32, _U8, _F32 = {torch.bfloat16: 1}, {torch.int32: 0}, {torch.uint8: 0}, {torch.float32: 0}


def _refuse(name, t, types, dev, shape, what="last dimension contiguous"):
    raise ValueError(f"{name}: wanted {' x '.join('any' if n is None else str(n) for n in shape)} of {' or '.join(str(x) for x in types)} on cuda:{dev}, {what}; "
                     f"got {tuple(t.shape)} of {t.dtype} on {t.device}, strides {tuple(t.stride())}")


def _strides(name, t, types, dev, shape):
    """Strides of t, a tensor of one of these types and of this shape on the current device, neighbouring elements last."""
    if t.dtype in types and t.shape == shape and t.get_device() == dev:
        s = t.stride()
        if s[-1] == 1:
            return s
    _refuse(name, t, types, dev, shape)


def _dense(name, t, types, dev, shape):
    """The same of a contiguous tensor; its address."""
    if t.dtype in types and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    _refuse(name, t, types, dev, shape, "contiguous")


def _shape(name, t, n):
    """Extents of a tensor of n dimensions."""
    shape = t.shape
    if len(shape) != n:
        raise ValueError(f"{name}: wanted {n} dimensions; got {tuple(shape)}")
    return shape


class KVCacheMX:
    """One layer's K/V cache as microscaled blocks of 32 values in 4 or 8 bits (head_dim 64 or 128): 68 or 132 bytes a row of 128 values instead
    of 256.  Contiguous [batch][n_kv_heads][smax], or with a block_table (int32 cuda [batch][max_pages]) pools of
    [n_pages][n_kv_heads][page_size].  k, v (codes, uint8) and k_scale, v_scale (uint8) are allocated here where they are not given.  The
    caller keeps the sequences' lengths, as KVState.ctx_len does."""

    def __init__(self, n_kv_heads, head_dim, batch, smax, bits=4, block_table=None, page_size=0, n_pages=None, k=None, v=None, k_scale=None, v_scale=None):
        dev = torch.cuda.current_device()
        self.n_kv_heads, self.head_dim, self.batch, self.smax, self.bits = int(n_kv_heads), int(head_dim), int(batch), int(smax), int(bits)
        if self.bits not in (4, 8) or self.head_dim not in (64, 128) or min(self.n_kv_heads, self.batch, self.smax) < 1:
            raise ValueError(f"KVCacheMX: bits 4 or 8, head_dim 64 or 128 and positive sizes wanted; got {bits}, {head_dim}, {(n_kv_heads, batch, smax)}")
        self.block_table, self.page_size, self.max_pages, self.n_pages = block_table, 0, 0, 0
        if block_table is not None:
            self.page_size, self.max_pages = int(page_size), _shape("block_table", block_table, 2)[1]
            _dense("block_table", block_table, _I32, dev, (self.batch, self.max_pages))
            if self.page_size < 16 or self.page_size & (self.page_size - 1) or self.smax > self.max_pages * self.page_size:
                raise ValueError(f"KVCacheMX: page_size a power of two >= 16 and smax <= {self.max_pages} pages of it wanted; got {page_size}, {smax}")
            self.n_pages = int(n_pages) if n_pages is not None else k.shape[0] if k is not None else self.batch * self.max_pages
        rows = (self.n_pages, self.n_kv_heads, self.page_size) if block_table is not None else (self.batch, self.n_kv_heads, self.smax)
        for name, t, width in (("k", k, self.head_dim * self.bits // 8), ("v", v, self.head_dim * self.bits // 8), ("k_scale", k_scale, self.head_dim // 32),
                               ("v_scale", v_scale, self.head_dim // 32)):
            if t is None:
                t = torch.zeros(rows + (width,), dtype=torch.uint8, device="cuda") if width > 4 else torch.full(rows + (width,), 127, dtype=torch.uint8, device="cuda")
            _dense(name, t, _U8, dev, rows + (width,))
            setattr(self, name, t)
        self._device = dev
        self._desc = _KVMX(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(), self.bits, self.batch, self.n_kv_heads,
                           self.head_dim, self.smax, block_table.data_ptr() if block_table is not None else None, self.page_size, self.n_pages, self.max_pages)
        self._ref = C.byref(self._desc)

    def on(self, dev):
        """The descriptor, for a call on device dev."""
        if dev != self._device:
            raise ValueError(f"the cache is on cuda:{self._device}, the current device is cuda:{dev}")
        return self._ref


def kv_write_mx(cache, k, v, start, count=None, path=None, cu_rows=None):
    """Rounds rows to blocks as they are written to the cache: row i of sequence b to slot start[b] + i (rows that would lie outside the cache are
    dropped).  k, v: cuda float32 or bfloat16, [B][Hkv][n][hd] as tree_attention's pass rows, or with cu_rows
    (int32 [B+1]) packed [T][Hkv][hd].  start, count: int32 [B]; count None: all rows.  path int32 [B][m]: row i is k[b, :, path[b, i]]
    (accept's path, with count its n_acc).  No length is changed."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    ref, B, H, D, dtype = cache.on(dev), cache.batch, cache.n_kv_heads, cache.head_dim, k.dtype
    seq = vseq = pcount = ppath = m = pcu = 0
    if cu_rows is not None:
        n = _shape("k", k, 3)[0]
        row, head, _ = _strides("k", k, _F32_BF16, dev, (n, H, D))
        vrow, vhead, _ = _strides("v", v, {dtype}, dev, (n, H, D))
        pcu = _dense("cu_rows", cu_rows, _I32, dev, (B + 1,))
    else:
        n = _shape("k", k, 4)[2]
        seq, head, row, _ = _strides("k", k, _F32_BF16, dev, (B, H, n, D))
        vseq, vhead, vrow, _ = _strides("v", v, {dtype}, dev, (B, H, n, D))
    if count is not None:
        pcount = _dense("count", count, _I32, dev, (B,))
    if path is not None:
        m = _shape("path", path, 2)[1]
        ppath = _dense("path", path, _I32, dev, (B, m))
    rc = L.bita_kv_write_mx(ref, k.data_ptr(), seq, head, row, v.data_ptr(), vseq, vhead, vrow, _F32_BF16[dtype], n, _dense("start", start, _I32, dev, (B,)), pcount, ppath, m,
                            pcu, _raw_stream(dev))
    if rc:
        _check(rc)


def kv_read_mx(cache, k, v, length, start=None):
    """The way back: slot start[b] + i of the cache, i < min(length[b], n), to k[b, :, i] and v[b, :, i] (cuda bfloat16 or float32 [B][Hkv][n][hd];
    exact in either; one of them may be None).  start, length: int32 [B]; start None: 0.  What lies behind a length is left as it is."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    ref, one = cache.on(dev), k if k is not None else v
    B, dtype, n = cache.batch, one.dtype, _shape("k" if k is not None else "v", one, 4)[2]
    shape = (B, cache.n_kv_heads, n, cache.head_dim)
    seq = head = row = vseq = vhead = vrow = pk = pv = pstart = 0
    if k is not None:
        seq, head, row, _ = _strides("k", k, _F32_BF16, dev, shape)
        pk = k.data_ptr()
    if v is not None:
        vseq, vhead, vrow, _ = _strides("v", v, {dtype} if k is not None else _F32_BF16, dev, shape)
        pv = v.data_ptr()
    if start is not None:
        pstart = _dense("start", start, _I32, dev, (B,))
    rc = L.bita_kv_read_mx(ref, pk, seq, head, row, pv, vseq, vhead, vrow, _F32_BF16[dtype], n, pstart, _dense("length", length, _I32, dev, (B,)), _raw_stream(dev))
    if rc:
        _check(rc)


def qk_norm_rope(x, pos, cos, sin, n_heads, n_kv_heads, q_gain=None, k_gain=None, eps=1e-5, q=None, k=None, v=None):
    """Queries and keys of a QKV product x (cuda [M][(n_heads + 2 n_kv_heads) * hd], float32 or bfloat16) ready for attention: RMSNorm of every head with a gain
    (bfloat16 [hd]; None: no norm), rotation of its pairs (i, i + hd/2) by the angles of pos[m] (cos, sin: float32 [max_pos][hd/2]).
    Returns (q [M][n_heads][hd], k [M][n_kv_heads][hd], v) in bfloat16, written into q, k, v where they are given (they may be views of a
    bfloat16 x's own columns).  v: x's rounded to bfloat16; where x is bfloat16 and no v is given, a view of x."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    max_pos, half = table = _shape("cos", cos, 2)
    hd, bf16 = 2 * half, torch.bfloat16
    m = _shape("x", x, 2)[0]
    ldx = _strides("x", x, _F32_BF16, dev, (m, (n_heads + 2 * n_kv_heads) * hd))[0]
    dtype, pqg, pkg, pv, ldv, hv = x.dtype, 0, 0, 0, 0, 0
    if q_gain is not None:
        pqg = _dense("q_gain", q_gain, _BF16, dev, (hd,))
    if k_gain is not None:
        pkg = _dense("k_gain", k_gain, _BF16, dev, (hd,))
    if q is None:
        q = x.new_empty((m, n_heads, hd), dtype=bf16)
    if k is None:
        k = x.new_empty((m, n_kv_heads, hd), dtype=bf16)
    (ldq, hq, _), (ldk, hk, _) = _strides("q", q, _BF16, dev, (m, n_heads, hd)), _strides("k", k, _BF16, dev, (m, n_kv_heads, hd))
    if v is None and dtype is bf16:
        v = x[:, (n_heads + n_kv_heads) * hd:].unflatten(1, (n_kv_heads, hd))
    else:
        if v is None:
            v = x.new_empty((m, n_kv_heads, hd), dtype=bf16)
        ldv, hv, _ = _strides("v", v, _BF16, dev, (m, n_kv_heads, hd))
        pv = v.data_ptr()
    rc = L.bita_qk_norm_rope(x.data_ptr(), _F32_BF16[dtype], m, ldx, n_heads, n_kv_heads, hd, pqg, pkg, eps, _dense("pos", pos, _I32, dev, (m,)),
                             _dense("cos", cos, _F32, dev, table), _dense("sin", sin, _F32, dev, table), max_pos, q.data_ptr(), ldq, hq, k.data_ptr(), ldk, hk, pv, ldv, hv,
                             _raw_stream(dev))
    if rc:
        _check(rc)
    return q, k, v


@functools.lru_cache(4096)
def _attention_mx_scratch(*sizes):
    return lib().bita_tree_attention_mx_workspace_bytes(*sizes)


def tree_attention_mx_plan_info(batch, rows, heads, kv_heads, head_dim, bits, ctx_hint, n_prompt=0):
    """{splits (of a sequence's keys, on average), queries, waves (of a workgroup), workgroups} that tree_attention_mx of these sizes launches."""
    out = (C.c_int32 * 4)()
    _check(lib().bita_tree_attention_mx_plan_info(batch, rows, heads, kv_heads, head_dim, bits, int(ctx_hint), n_prompt, out))
    return dict(splits=out[0], queries=out[1], waves=out[2], workgroups=out[3])


def tree_attention_mx(tmpl, q, cache, k_rows, v_rows, ctx_len, ctx_hint, prompt_k=None, prompt_v=None, token=None, out=None, workspace=None):
    """tree_attention over a KVCacheMX: q bfloat16 [B][R][Hq][hd]; k_rows, v_rows bfloat16 [B][Hkv][R][hd] (any strides): the pass' rows, not in
    the cache yet; ctx_len int32 [B], at most ctx_hint; prompt_k/v bfloat16 [Hkv][P][hd] or None; token int32 [B][R] or None (tree rows with
    a negative token are absent, their output zero).  Returns bfloat16 [B][R][Hq*hd], written into out where it is given.
    workspace: uint8 cuda of bita_tree_attention_mx_workspace_bytes (allocated here when it is None and one is needed)."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    ref, B, H, D, R = cache.on(dev), cache.batch, cache.n_kv_heads, cache.head_dim, tmpl.rows
    Hq, ctx_hint = _shape("q", q, 4)[2], int(ctx_hint)
    seq, head, row, _ = _strides("k_rows", k_rows, _BF16, dev, (B, H, R, D))
    vseq, vhead, vrow, _ = _strides("v_rows", v_rows, _BF16, dev, (B, H, R, D))
    P = pk = pv = pt = pw = nw = 0
    if prompt_k is not None:
        P = _shape("prompt_k", prompt_k, 3)[1]
        pk, pv = _dense("prompt_k", prompt_k, _BF16, dev, (H, P, D)), _dense("prompt_v", prompt_v, _BF16, dev, (H, P, D))
    if token is not None:
        pt = _dense("token", token, _I32, dev, (B, R))
    pq = _dense("q", q, _BF16, dev, (B, R, Hq, D))
    if out is None:
        out = q.new_empty((B, R, Hq * D))
        po = out.data_ptr()
    else:
        po = _dense("out", out, _BF16, dev, (B, R, Hq * D))
    if workspace is None:
        nw = _attention_mx_scratch(B, R, Hq, H, D, cache.bits, ctx_hint, P)
        if nw:
            workspace = q.new_empty(nw, dtype=torch.uint8)
    else:
        _bytes("workspace", workspace, 0, dev)
        nw = workspace.numel()
    if nw:
        pw = workspace.data_ptr()
    rc = L.bita_tree_attention_mx(tmpl.handle, pq, ref, k_rows.data_ptr(), seq, head, row, v_rows.data_ptr(), vseq, vhead, vrow, pk, pv, P,
                                  _dense("ctx_len", ctx_len, _I32, dev, (B,)), pt, Hq, ctx_hint, pw, nw, po, _raw_stream(dev))
    if rc:
        _check(rc)
    return out


def prompt_attention(q, k, v, cu_seqlens, out=None):
    """Causal attention over packed prompts: q bfloat16 [T][Hq][hd], k, v bfloat16 [T][Hkv][hd] (any strides: columns of one QKV product, or tensors of their
    own); sequence b is rows cu_seqlens[b] .. cu_seqlens[b+1]-1 (int32 cuda [B+1]).  Returns bfloat16 [T][Hq*hd], written into out where it is
    given; rows outside the sequences are left as they are (undefined where out is allocated here)."""
    L, dev = _lib or lib(), torch.cuda.current_device()
    T, Hq, D = shape = _shape("q", q, 3)
    H = _shape("k", k, 3)[1]
    ldq, hq, _ = _strides("q", q, _BF16, dev, shape)
    ldk, hk, _ = _strides("k", k, _BF16, dev, (T, H, D))
    ldv, hv, _ = _strides("v", v, _BF16, dev, (T, H, D))
    n = cu_seqlens.numel()
    if out is None:
        out, ldo = q.new_empty((T, Hq * D)), Hq * D
    else:
        ldo = _strides("out", out, _BF16, dev, (T, Hq * D))[0]
    rc = L.bita_prompt_attention(q.data_ptr(), ldq, hq, k.data_ptr(), ldk, hk, v.data_ptr(), ldv, hv, _dense("cu_seqlens", cu_seqlens, _I32, dev, (n,)), n - 1, T, Hq, H, D,
                                 out.data_ptr(), ldo, _raw_stream(dev))
    if rc:
        _check(rc)
    return out
