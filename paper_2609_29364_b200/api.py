"""ctypes binding of include/nsd.h.  Same names as the C ABI, argument
marshalling only: tensors are torch CUDA tensors (device memory and streams are
torch's), every step runs inside libnsd.so."""
from __future__ import annotations

import ctypes
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libnsd.so")
_lib = None

STATUS = {
    0: "NSD_OK", 1: "NSD_ERR_INVALID_ARG", 2: "NSD_ERR_OUT_OF_RANGE", 3: "NSD_ERR_CAPACITY",
    4: "NSD_ERR_UNSUPPORTED", 5: "NSD_ERR_CUDA", 6: "NSD_ERR_DEVICE_FAULT", 7: "NSD_ERR_NOT_PLANNED",
    8: "NSD_ERR_TIMEOUT",
}


class NsdError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        super().__init__(f"{where}: {STATUS.get(code, code)}" + (f" ({detail})" if detail else ""))


class NsdConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "num_layers", "num_slabs", "num_q_heads", "num_kv_heads", "head_dim", "block_size", "num_blocks",
        "region_b_begin", "max_batch", "max_gamma", "vocab_size", "flags")] + [
        ("max_table_entries", ctypes.c_int64), ("wait_budget", ctypes.c_int32), ("reserved", ctypes.c_int32)]


# nsd_config.flags (include/nsd.h)
NSD_FLAG_ATTN_CP_ASYNC = 1 << 0
NSD_FLAG_ATTN_TCGEN05 = 1 << 1
NSD_FLAG_ATTN_NO_TCGEN05 = 1 << 2
NSD_FLAG_LOGITS_DIRECT = 1 << 3
NSD_FLAG_ROUND_SPLIT_ALWAYS = 1 << 4
NSD_FLAG_ROUND_SPLIT_NEVER = 1 << 5
NSD_FLAG_NO_DEPENDENT_LAUNCH = 1 << 6
NSD_FLAG_TEST_STARVE_GATHER = 1 << 30


_vp = ctypes.c_void_p


class SchedParams(ctypes.Structure):
    _fields_ = [("worker_avail", ctypes.c_double), ("target_interval", ctypes.c_double), ("slack", ctypes.c_double),
                ("max_batch", ctypes.c_int32), ("row_capacity", ctypes.c_int32), ("block_capacity", ctypes.c_int64),
                ("token_limit", ctypes.c_int64)]


class RoundArgs(ctypes.Structure):
    _fields_ = [
        ("kv_pool", _vp), ("n_mig_blocks", ctypes.c_int64), ("mig_src", _vp), ("mig_dst", _vp),
        ("batch", ctypes.c_int32), ("gamma", ctypes.c_int32), ("ctx_len", _vp), ("kv_indptr", _vp),
        ("kv_indices", _vp), ("is_migrated", _vp), ("k_new", _vp), ("v_new", _vp), ("q", _vp), ("o", _vp),
        ("p", _vp), ("q_draft", _vp), ("draft_tok", _vp), ("u_acc", _vp), ("u_smp", _vp), ("acc_len", _vp),
        ("out_tok", _vp), ("new_ctx_len", _vp), ("fuse_gather", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("q_indptr", _vp),
    ]


class ChunkMasks(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("reserved", ctypes.c_int32), ("prefix_len", _vp), ("row_first", _vp)]


# nsd_rope_append flags (include/nsd.h)
NSD_ROPE_ADJACENT = 1 << 0
NSD_ROPE_CYCLED = 1 << 1


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libnsd.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: run `python -m paper_2609_29364_b200.build` "
                          "(or __graft_entry__.build()); there is no non-CUDA path")
    lib = ctypes.CDLL(_LIB_PATH)
    i32, i64, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    cfgp = ctypes.POINTER(NsdConfig)
    rap = ctypes.POINTER(RoundArgs)
    lib.nsd_status_string.restype = ctypes.c_char_p
    lib.nsd_status_string.argtypes = [i32]
    lib.nsd_last_error.restype = ctypes.c_char_p
    lib.nsd_last_error.argtypes = [_vp]
    lib.nsd_workspace_bytes.restype = sz
    lib.nsd_workspace_bytes.argtypes = [cfgp]
    lib.nsd_kv_pool_bytes.restype = sz
    lib.nsd_kv_pool_bytes.argtypes = [cfgp]
    lib.nsd_create.restype = i32
    lib.nsd_create.argtypes = [cfgp, _vp, sz, ctypes.POINTER(_vp)]
    lib.nsd_destroy.restype = i32
    lib.nsd_destroy.argtypes = [_vp]
    lib.nsd_verify_plan.restype = i32
    lib.nsd_verify_plan.argtypes = [_vp, i32, i32, _vp, _vp, _vp, _vp, i32, _vp]
    lib.nsd_kv_prepare.restype = i32
    lib.nsd_kv_prepare.argtypes = [_vp, _vp, i64, _vp, _vp, i32, i32, _vp, _vp, _vp, _vp, _vp, _vp, i32, i32, i32, _vp, i64, _vp]
    lib.nsd_kv_commit.restype = i32
    lib.nsd_kv_commit.argtypes = [_vp, _vp, i32, i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, i32, i32, _vp, _vp]
    lib.nsd_verify_attn.restype = i32
    lib.nsd_verify_attn.argtypes = [_vp, _vp, _vp, _vp, _vp, i32, i32, _vp, _vp, _vp, i32, i32, _vp]
    lib.nsd_spec_accept.restype = i32
    lib.nsd_spec_accept.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, i32, i32, i32, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.nsd_spec_accept_logits.restype = i32
    lib.nsd_spec_accept_logits.argtypes = [_vp, _vp, i32, ctypes.c_float, _vp, _vp, _vp, _vp, i32, i32, i32, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.nsd_verify_round.restype = i32
    lib.nsd_verify_round.argtypes = [_vp, rap, _vp]
    lib.nsd_verify_round_host.restype = i32
    lib.nsd_verify_round_host.argtypes = [_vp, rap, rap, i64, _vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.nsd_verify_attn_static.restype = i32
    lib.nsd_verify_attn_static.argtypes = [_vp, i32, i32, i32, i32, i32, _vp, _vp, i32, i32, _vp, _vp, _vp, _vp, _vp]
    lib.nsd_schedule_batch.restype = i32
    lib.nsd_schedule_batch.argtypes = [ctypes.POINTER(SchedParams), i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                       ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_double)]
    lib.nsd_block_tables.restype = i32
    lib.nsd_block_tables.argtypes = [_vp, i32, _vp, _vp, _vp, i64, _vp, _vp, i64, _vp, i64, i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.nsd_rope_append.restype = i32
    lib.nsd_rope_append.argtypes = [_vp, _vp, i32, i64, i32, _vp, i64, _vp, i64, _vp, i64, _vp, i64, _vp, i32, _vp, _vp, i32, _vp, _vp]
    lib.nsd_chunk_plan_bytes.restype = sz
    lib.nsd_chunk_plan_bytes.argtypes = [_vp, i64]
    lib.nsd_chunk_plan.restype = i32
    lib.nsd_chunk_plan.argtypes = [_vp, _vp, sz, i32, i64, _vp, _vp, _vp, ctypes.POINTER(ChunkMasks), _vp]
    lib.nsd_chunk_attn.restype = i32
    lib.nsd_chunk_attn.argtypes = [_vp, _vp, sz, _vp, _vp, i64, _vp, _vp, i64, _vp, i32, ctypes.c_float, ctypes.c_float, _vp, _vp]
    lib.nsd_launch_count.restype = i64
    lib.nsd_launch_count.argtypes = [_vp]
    lib.nsd_get_status.restype = i32
    lib.nsd_get_status.argtypes = [_vp, _vp, ctypes.POINTER(i32)]
    _lib = lib
    return lib


def _ptr(t) -> Optional[int]:
    """Address of a torch tensor (CUDA or pinned host), numpy array, int or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if hasattr(t, "data_ptr"):
        assert t.is_contiguous()
        return t.data_ptr()
    if hasattr(t, "ctypes"):
        assert t.flags["C_CONTIGUOUS"]
        return t.ctypes.data
    raise TypeError(type(t))


def _tensor(t, dtype, what, n=0):
    """Address of a contiguous torch tensor of the given dtype with at least n elements (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        if t.dtype is not dtype:
            raise TypeError(f"{what}: {dtype} is wanted, got {t.dtype}")
        raise ValueError(f"{what}: {n} contiguous elements are wanted, got {t.numel()} with strides {t.stride()}")
    return t.data_ptr()


def _rows(t, width, what):
    """Address and row stride of a tensor [rows][...] whose rows are `width` contiguous elements."""
    shape, stride = t.shape, t.stride()
    if len(shape) == 2:
        inner = shape[1] == width and (stride[1] == 1 or width == 1)
    else:
        inner = len(shape) == 3 and shape[1] * shape[2] == width and stride[2] == 1 and stride[1] == shape[2]
    if not inner:
        raise ValueError(f"{what}: rows of {width} contiguous elements are wanted, got shape {tuple(shape)}, strides {stride}")
    return t.data_ptr(), (stride[0] if shape[0] > 1 else width)


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        import torch

        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def nsd_verify_attn_static(kv_slab, num_blocks, num_q_heads, num_kv_heads, head_dim, block_size, q, o, batch, gamma,
                           h_ctx_len, ctx_len, kv_indptr, kv_indices, stream=None):
    """Attention without any device allocation: the scratch is a fixed array inside
    libnsd.so (see include/nsd.h for who needs this, the size limits and the rule
    that calls must not overlap on the GPU).  Needs no VerifyContext."""
    rc = load_library().nsd_verify_attn_static(_ptr(kv_slab), num_blocks, num_q_heads, num_kv_heads, head_dim,
                                               block_size, _ptr(q), _ptr(o), batch, gamma, _ptr(h_ctx_len),
                                               _ptr(ctx_len), _ptr(kv_indptr), _ptr(kv_indices),
                                               _stream_handle(stream))
    if rc != 0:
        raise NsdError(rc, "nsd_verify_attn_static")


def nsd_schedule_batch(*, worker_avail, target_interval, slack, max_batch, pred_done, kv_ready, eligible=None,
                       rows=None, blocks=None, tokens=None, row_capacity=2 ** 31 - 1, block_capacity=2 ** 62,
                       token_limit=2 ** 62):
    """Algorithm 1 on the host (numpy arrays in, list of admitted indices and predicted start out)."""
    import numpy as np

    n = len(pred_done)
    prm = SchedParams(worker_avail, target_interval, slack, max_batch, row_capacity, block_capacity, token_limit)
    out = np.empty(max(1, min(n, max(max_batch, 0))), dtype=np.int32)
    m, start = ctypes.c_int32(0), ctypes.c_double(0.0)
    f64 = lambda a: None if a is None else np.ascontiguousarray(a, dtype=np.float64)
    i32a = lambda a: None if a is None else np.ascontiguousarray(a, dtype=np.int32)
    keep = [f64(pred_done), f64(kv_ready), None if eligible is None else np.ascontiguousarray(eligible, dtype=np.uint8),
            i32a(rows), i32a(blocks), i32a(tokens)]
    rc = load_library().nsd_schedule_batch(ctypes.byref(prm), n, _ptr(keep[2]), _ptr(keep[0]), _ptr(keep[1]),
                                           _ptr(keep[3]), _ptr(keep[4]), _ptr(keep[5]), _ptr(out), ctypes.byref(m),
                                           ctypes.byref(start))
    if rc != 0:
        raise NsdError(rc, "nsd_schedule_batch")
    return out[:m.value].tolist(), start.value


class VerifyContext:
    """Owns an nsd_ctx and the torch-allocated workspace it lives on."""

    def __init__(self, *, num_layers, num_q_heads, num_kv_heads, head_dim, block_size, num_blocks, region_b_begin,
                 max_batch, max_gamma, vocab_size, max_table_entries, num_slabs=None, flags=0, wait_budget=0,
                 device="cuda:0"):
        import torch

        self.lib = load_library()
        self.cfg = NsdConfig(num_layers=num_layers, num_slabs=num_slabs or num_layers, num_q_heads=num_q_heads,
                             num_kv_heads=num_kv_heads, head_dim=head_dim, block_size=block_size,
                             num_blocks=num_blocks, region_b_begin=region_b_begin, max_batch=max_batch,
                             max_gamma=max_gamma, vocab_size=vocab_size, flags=flags,
                             max_table_entries=max_table_entries, wait_budget=wait_budget, reserved=0)
        self.device = torch.device(device)
        self._device_index = self.device.index if self.device.index is not None else torch.cuda.current_device()
        # the same handle as torch.cuda.current_stream(device).cuda_stream, without making a stream object for every call
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
        self._i32, self._i64, self._f32, self._bf16 = torch.int32, torch.int64, torch.float32, torch.bfloat16
        self._h = _vp()
        nbytes = self.lib.nsd_workspace_bytes(ctypes.byref(self.cfg))
        if nbytes == 0:
            raise NsdError(4, "nsd_workspace_bytes", "invalid or unsupported configuration")
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            rc = self.lib.nsd_create(ctypes.byref(self.cfg), self.workspace.data_ptr(), nbytes, ctypes.byref(self._h))
        if rc != 0:
            raise NsdError(rc, "nsd_create")

    # -- helpers
    def _check(self, rc: int, where: str):
        if rc != 0:
            detail = self.lib.nsd_last_error(self._h).decode() if rc == 5 else ""
            raise NsdError(rc, where, detail)

    def pool_bytes(self) -> int:
        return self.lib.nsd_kv_pool_bytes(ctypes.byref(self.cfg))

    def close(self):
        if self._h:
            self.lib.nsd_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the C ABI, one method per entry point
    def nsd_verify_plan(self, h_ctx_len, h_kv_indptr, h_is_migrated, gamma, chunk_blocks=0, stream=None, h_q_indptr=None):
        batch = len(h_ctx_len)
        self._check(self.lib.nsd_verify_plan(self._h, batch, gamma, _ptr(h_ctx_len), _ptr(h_kv_indptr),
                                             _ptr(h_is_migrated), _ptr(h_q_indptr), chunk_blocks, _stream_handle(stream)),
                    "nsd_verify_plan")

    def nsd_kv_prepare(self, kv_pool, n_mig_blocks, mig_src, mig_dst, batch, gamma, ctx_len, kv_indptr, kv_indices,
                       k_new, v_new, is_migrated=None, append_subset=0, layer_begin=0, layer_count=None, stream=None,
                       q_indptr=None, total_rows=0):
        if layer_count is None:
            layer_count = self.cfg.num_layers - layer_begin
        self._check(self.lib.nsd_kv_prepare(self._h, _ptr(kv_pool), n_mig_blocks, _ptr(mig_src), _ptr(mig_dst), batch,
                                            gamma, _ptr(ctx_len), _ptr(kv_indptr), _ptr(kv_indices), _ptr(k_new),
                                            _ptr(v_new), _ptr(is_migrated), append_subset, layer_begin, layer_count,
                                            _ptr(q_indptr), int(total_rows), _stream_handle(stream)), "nsd_kv_prepare")

    def nsd_kv_commit(self, kv_pool, batch, gamma, ctx_len, acc_len, kv_indptr, kv_indices, exp_indptr, exp_indices,
                      new_ctx_len=None, layer_begin=0, layer_count=None, stream=None, q_indptr=None):
        if layer_count is None:
            layer_count = self.cfg.num_layers - layer_begin
        self._check(self.lib.nsd_kv_commit(self._h, _ptr(kv_pool), batch, gamma, _ptr(ctx_len), _ptr(acc_len),
                                           _ptr(kv_indptr), _ptr(kv_indices), _ptr(exp_indptr), _ptr(exp_indices),
                                           _ptr(new_ctx_len), layer_begin, layer_count, _ptr(q_indptr),
                                           _stream_handle(stream)), "nsd_kv_commit")

    def nsd_verify_attn(self, kv_pool, q, o, lse, batch, gamma, ctx_len, kv_indptr, kv_indices, layer=0, subset=0,
                        stream=None):
        self._check(self.lib.nsd_verify_attn(self._h, _ptr(kv_pool), _ptr(q), _ptr(o), _ptr(lse), batch, gamma,
                                             _ptr(ctx_len), _ptr(kv_indptr), _ptr(kv_indices), layer, subset,
                                             _stream_handle(stream)), "nsd_verify_attn")

    def nsd_spec_accept(self, p, q, draft_tok, u_acc, u_smp, batch, gamma, vocab, ctx_len, acc_len, out_tok,
                        new_ctx_len=None, stream=None, q_indptr=None):
        self._check(self.lib.nsd_spec_accept(self._h, _ptr(p), _ptr(q), _ptr(draft_tok), _ptr(u_acc), _ptr(u_smp),
                                             batch, gamma, vocab, _ptr(ctx_len), _ptr(acc_len), _ptr(out_tok),
                                             _ptr(new_ctx_len), _ptr(q_indptr), _stream_handle(stream)), "nsd_spec_accept")

    def nsd_spec_accept_logits(self, logits, logits_dtype, temperature, q, draft_tok, u_acc, u_smp, batch, gamma, vocab,
                               gamma_r, ctx_len, acc_len, out_tok, new_ctx_len=None, stream=None):
        self._check(self.lib.nsd_spec_accept_logits(self._h, _ptr(logits), logits_dtype, float(temperature), _ptr(q),
                                                    _ptr(draft_tok), _ptr(u_acc), _ptr(u_smp), batch, gamma, vocab,
                                                    _ptr(gamma_r), _ptr(ctx_len), _ptr(acc_len), _ptr(out_tok),
                                                    _ptr(new_ctx_len), _stream_handle(stream)), "nsd_spec_accept_logits")

    # -- chunks of new tokens
    def _stream(self, stream, *tensors):
        """The given stream, or the current one of the context's device (whichever device is current).  The last argument
        to be formed, when types and shapes are known to be right: the kernels read the tensors' addresses as they are, so
        one that lies in pageable memory or on another device is refused here."""
        device = self._device_index
        for t in tensors:
            if t is not None and t.get_device() != device and not (t.get_device() < 0 and t.is_pinned()):
                raise ValueError(f"tensors on cuda:{device} (or in pinned memory) are wanted, got one of shape {tuple(t.shape)} on {t.device}")
        if stream is None:
            return self._raw_stream(self._device_index)
        return stream if isinstance(stream, int) else stream.cuda_stream

    def nsd_block_tables(self, ctx_len, new_len, held, n_held, free_blocks, free_begin, kv_indptr, kv_indices, q_indptr,
                         slot_map, positions, row_req, n_held_new, free_end, stream=None):
        """Sizes come from the tensors: batch = len(ctx_len), held [batch][stride], capacities of kv_indices and of the
        row outputs (slot_map, positions, row_req: nullable, of one length)."""
        batch, i32, i64 = ctx_len.numel(), self._i32, self._i64
        max_rows = None
        for t in (slot_map, positions, row_req):
            if t is not None:
                if max_rows is not None and t.numel() != max_rows:
                    raise ValueError("slot_map, positions and row_req have to have one length")
                max_rows = t.numel()
        if held.dim() != 2 or held.shape[0] < batch:
            raise ValueError("held: [batch][stride] is wanted")
        rc = self.lib.nsd_block_tables(
            self._h, batch, _tensor(ctx_len, i32, "ctx_len"), _tensor(new_len, i32, "new_len", batch), _tensor(held, i32, "held"),
            held.shape[1], _tensor(n_held, i32, "n_held", batch), _tensor(free_blocks, i32, "free_blocks"), free_blocks.numel(),
            _tensor(free_begin, i64, "free_begin", 1), kv_indices.numel(), max_rows or 0, _tensor(kv_indptr, i64, "kv_indptr", batch + 1),
            _tensor(kv_indices, i32, "kv_indices"), _tensor(q_indptr, i64, "q_indptr", batch + 1), _tensor(slot_map, i64, "slot_map"),
            _tensor(positions, i32, "positions"), _tensor(row_req, i32, "row_req"), _tensor(n_held_new, i32, "n_held_new", batch),
            _tensor(free_end, i64, "free_end", 1),
            self._stream(stream, ctx_len, new_len, held, n_held, free_blocks, free_begin, kv_indptr, kv_indices, q_indptr, slot_map,
                         positions, row_req, n_held_new, free_end))
        if rc:
            self._check(rc, "nsd_block_tables")

    def nsd_rope_append(self, kv_pool, layer, q, k, v, q_out, positions, sections, inv_freq, slot_map=None, adjacent=False,
                        cycled=False, stream=None):
        """q, k, v: [rows][heads * head_dim] or [rows][heads][head_dim], rows any stride apart (slices of one projection),
        fp32 or bf16; q_out bf16; positions int32 [axes][rows]; sections: pairs of each axis."""
        some = q if q is not None else k
        if some is None or (k is None) != (v is None):
            raise ValueError("q, or k and v, or all three are wanted")
        n, dtype = some.shape[0], some.dtype
        wq, wk = self.cfg.num_q_heads * self.cfg.head_dim, self.cfg.num_kv_heads * self.cfg.head_dim
        qp = kp = vp = op = None
        qs = ks = vs = os_ = 0
        if q is not None:
            qp, qs = _rows(q, wq, "q")
            if q_out is None or q_out.dtype is not self._bf16 or q_out.shape[0] < n:
                raise TypeError("q_out: bfloat16 with q's rows is wanted")
            op, os_ = _rows(q_out, wq, "q_out")
        if k is not None:
            if k.shape[0] != n or v.shape[0] != n or k.dtype is not dtype or v.dtype is not dtype:
                raise ValueError("q, k and v have to have the same rows and dtype")
            kp, ks = _rows(k, wk, "k")
            vp, vs = _rows(v, wk, "v")
        axes = len(sections)
        if positions.dim() != 2 or positions.shape[1] != n or positions.shape[0] != axes:
            raise ValueError("positions: [axes][rows] is wanted, and sections: one number per axis")
        rc = self.lib.nsd_rope_append(
            self._h, _ptr(kv_pool), layer, n, 0 if dtype is self._f32 else (1 if dtype is self._bf16 else -1), qp, qs, kp, ks, vp, vs,
            op, os_, _tensor(positions, self._i32, "positions"), axes, (ctypes.c_int32 * axes)(*sections),
            _tensor(inv_freq, self._f32, "inv_freq", sum(sections)),
            (NSD_ROPE_ADJACENT if adjacent else 0) | (NSD_ROPE_CYCLED if cycled else 0), _tensor(slot_map, self._i64, "slot_map", n),
            self._stream(stream, None if type(kv_pool) is int else kv_pool, q, k, v, q_out if q is not None else None, positions, inv_freq, slot_map))
        if rc:
            self._check(rc, "nsd_rope_append")

    def nsd_chunk_plan_bytes(self, max_rows: int) -> int:
        return int(self.lib.nsd_chunk_plan_bytes(self._h, max_rows))

    def nsd_chunk_plan(self, plan, max_rows, q_indptr, ctx_len, kv_indptr, window=0, prefix_len=None, row_first=None, stream=None):
        batch, i32, i64 = ctx_len.numel(), self._i32, self._i64
        masks = ChunkMasks(window, 0, _tensor(prefix_len, i32, "prefix_len", batch), _tensor(row_first, i32, "row_first", max_rows))
        rc = self.lib.nsd_chunk_plan(
            self._h, plan.data_ptr(), plan.numel() * plan.element_size(), batch, max_rows, _tensor(q_indptr, i64, "q_indptr", batch + 1),
            _tensor(ctx_len, i32, "ctx_len"), _tensor(kv_indptr, i64, "kv_indptr", batch + 1), ctypes.byref(masks),
            self._stream(stream, plan, q_indptr, ctx_len, kv_indptr, prefix_len, row_first))
        if rc:
            self._check(rc, "nsd_chunk_plan")

    def nsd_chunk_attn(self, plan, max_rows, kv_pool, q, o, lse, kv_indices, layer=0, scale=0.0, softcap=0.0, alibi_slopes=None,
                       stream=None):
        """q: [rows][q heads * head_dim] or [rows][q heads][head_dim], rows any multiple of 8 elements apart; o contiguous."""
        heads, f32 = self.cfg.num_q_heads, self._f32
        width = heads * self.cfg.head_dim
        if q.dtype is not self._bf16 or q.shape[0] < max_rows:
            raise TypeError("q: bfloat16 with max_rows rows is wanted")
        qp, qs = _rows(q, width, "q")
        rc = self.lib.nsd_chunk_attn(
            self._h, plan.data_ptr(), plan.numel() * plan.element_size(), _ptr(kv_pool), qp, qs, _tensor(o, self._bf16, "o", max_rows * width),
            _tensor(lse, f32, "lse", max_rows * heads), max_rows, _tensor(kv_indices, self._i32, "kv_indices"), layer, scale, softcap,
            _tensor(alibi_slopes, f32, "alibi_slopes", heads), self._stream(stream, plan, None if type(kv_pool) is int else kv_pool, q, o, lse, kv_indices, alibi_slopes))
        if rc:
            self._check(rc, "nsd_chunk_attn")

    @staticmethod
    def round_args(**kw) -> RoundArgs:
        a = RoundArgs()
        a._keepalive = [v for v in kw.values() if hasattr(v, "data_ptr")]    # the struct holds raw addresses only
        for name, _ in RoundArgs._fields_:
            v = kw.pop(name, None)
            if name in ("n_mig_blocks", "batch", "gamma", "fuse_gather", "reserved"):
                setattr(a, name, int(v or 0))
            else:
                setattr(a, name, _ptr(v))
        assert not kw, f"unknown round arguments: {list(kw)}"
        return a

    def nsd_verify_round(self, args: RoundArgs, stream=None):
        self._check(self.lib.nsd_verify_round(self._h, ctypes.byref(args), _stream_handle(stream)), "nsd_verify_round")

    def nsd_verify_round_host(self, h_args: RoundArgs, d_args: RoundArgs, total_table_entries: int, stream=None):
        up, down = ctypes.c_int64(0), ctypes.c_int64(0)
        self._check(self.lib.nsd_verify_round_host(self._h, ctypes.byref(h_args), ctypes.byref(d_args),
                                                   total_table_entries, _stream_handle(stream), ctypes.byref(up),
                                                   ctypes.byref(down)), "nsd_verify_round_host")
        return up.value, down.value

    def nsd_launch_count(self) -> int:
        return int(self.lib.nsd_launch_count(self._h))

    def nsd_get_status(self, stream=None):
        bad = ctypes.c_int32(-1)
        rc = self.lib.nsd_get_status(self._h, _stream_handle(stream), ctypes.byref(bad))
        return rc, bad.value
