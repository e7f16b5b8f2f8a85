"""Python binding of librgd (refusal-gated decoding on MI355X / gfx950).

Argument marshalling only: every step of the decode path runs in the HIP
library.  Tensors are PyTorch tensors on the GPU; their data pointers and the
current HIP stream are passed through the C ABI declared in include/rgd.h.
Importing this module loads the library and raises if it has not been built.
"""
from __future__ import annotations

import ctypes as C
import os

__all__ = [
    "RGDError", "lib", "ModelConfig", "Model", "KV", "Table", "prefill_kv", "probe", "probe_fixed", "gate",
    "sample_continuations", "sample_continuations_pless", "check_status", "kernel_attention", "kernel_lm_head", "kernel_argmax",
    "kernel_sample", "kernel_sample_noalloc", "kernel_sample_pless", "sampler_workspace_bytes", "timing_enable", "timing_read", "TIMERS", "PagedCache", "paged_workspace_bytes", "paged_select",
    "paged_reserve", "paged_compact", "paged_append", "paged_attention_workspace_bytes", "paged_attention",
    "RotaryScaling", "Rotary", "paged_append_rotated", "paged_share_bytes", "paged_share",
    "paged_attention_shared_workspace_bytes", "paged_attention_shared",
    "verify_workspace_bytes", "verify_drafts", "sample_truncated_workspace_bytes", "sample_truncated", "EVENT_INCOMPAT", "EVENT_STOP", "EVENT_MAXLEN",
    "DTYPE_F32", "DTYPE_BF16",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librgd.so")
EXPORTS = (
    "rgd_version", "rgd_last_error", "rgd_model_create", "rgd_model_destroy", "rgd_kv_create",
    "rgd_kv_destroy", "rgd_kv_set_prefix_len", "rgd_table_create", "rgd_table_destroy",
    "rgd_prefill_kv", "rgd_prefill_kv_scored", "rgd_probe", "rgd_probe_fixed", "rgd_probe_soft", "rgd_probe_adaptive", "rgd_gate", "rgd_sample_continuations", "rgd_sample_continuations_pless", "rgd_check_status",
    "rgd_kernel_attention", "rgd_kernel_lm_head", "rgd_sampler_workspace_bytes",
    "rgd_kernel_argmax", "rgd_kernel_sample", "rgd_kernel_sample_noalloc", "rgd_kernel_sample_pless", "rgd_kernel_probe_step", "rgd_timing_enable", "rgd_timing_read",
    "rgd_paged_workspace_bytes", "rgd_paged_select", "rgd_paged_reserve", "rgd_paged_reserve_granted", "rgd_paged_compact", "rgd_paged_append",
    "rgd_paged_attention_workspace_bytes", "rgd_paged_attention", "rgd_verify_workspace_bytes", "rgd_verify_drafts",
    "rgd_rotary_frequencies", "rgd_paged_append_rotated", "rgd_paged_share_bytes", "rgd_paged_share",
    "rgd_paged_attention_shared_workspace_bytes", "rgd_paged_attention_shared",
    "rgd_sample_truncated_workspace_bytes", "rgd_sample_truncated",
)

DTYPE_F32, DTYPE_BF16 = 0, 1
EVENT_INCOMPAT, EVENT_STOP, EVENT_MAXLEN, EVENT_SKIPPED = 0, 1, 2, 3
STATUS = {0: "OK", 1: "INVALID_ARG", 2: "OOM", 3: "HIP", 4: "UNSUPPORTED", 5: "NONFINITE", 6: "STATE"}

# PyTorch ships its own HIP runtime (same soname as the system one).  Loading it
# first makes librgd bind to that instance; loading librgd first would bring in
# the system runtime and leave the process with two HIP/HSA runtimes, of which
# the second sees no device.
try:
    import torch  # noqa: F401
except ImportError:  # CPU-only use of the binding (export checks) needs no torch
    pass

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with paper_2607_20791_amd/build.py "
                      "(there is no fallback path)")
lib = C.CDLL(LIB_PATH)

VP, I32, U32, F32, U64 = C.c_void_p, C.c_int32, C.c_uint32, C.c_float, C.c_uint64
I64 = C.c_int64
I32P = C.POINTER(C.c_int32)


class ModelConfig(C.Structure):
    _fields_ = [("n_layers", I32), ("d_model", I32), ("n_heads", I32), ("n_kv_heads", I32),
                ("head_dim", I32), ("ffn_dim", I32), ("vocab", I32), ("dtype", I32),
                ("rms_eps", F32), ("rope_theta", F32), ("max_pos", I32)]


class LayerWeights(C.Structure):
    _fields_ = [(n, VP) for n in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate",
                                  "w_up", "w_down")]


class Weights(C.Structure):
    _fields_ = [("embed", VP), ("final_norm", VP), ("lm_head", VP),
                ("layers", C.POINTER(LayerWeights))]


class PagedCacheDesc(C.Structure):
    _fields_ = [(n, I32) for n in ("n_layers", "n_pages", "n_kv_heads", "page_size", "head_dim", "dtype", "max_seqs",
                                   "max_pages")] + \
               [(n, VP) for n in ("pool_k", "pool_v", "pages", "lens", "refs", "status")]


class RotaryScalingDesc(C.Structure):
    _fields_ = [("kind", I32), ("factor", C.c_double), ("context", C.c_double), ("low", C.c_double), ("high", C.c_double)]


class RotaryDesc(C.Structure):
    _fields_ = [("dim", I32), ("interleaved", I32), ("scale", F32), ("freq", C.POINTER(C.c_double))]


def _sig(name, res, *args):
    f = getattr(lib, name)
    f.restype = res
    f.argtypes = list(args)
    return f


_sig("rgd_version", C.c_char_p)
_sig("rgd_last_error", C.c_char_p)
_sig("rgd_model_create", I32, C.POINTER(ModelConfig), C.POINTER(Weights), I32, C.POINTER(VP))
_sig("rgd_model_destroy", None, VP)
_sig("rgd_kv_create", I32, VP, I32, I32, I32, I32, VP, VP, VP, VP, C.POINTER(VP))
_sig("rgd_kv_destroy", None, VP)
_sig("rgd_kv_set_prefix_len", I32, VP, I32, I32)
_sig("rgd_table_create", I32, I32P, I32P, I32, I32P, I32, C.POINTER(VP))
_sig("rgd_table_destroy", None, VP)
_sig("rgd_prefill_kv", I32, VP, VP, VP, I32, I32, I32, VP, VP)
_sig("rgd_probe", I32, VP, VP, VP, VP, I32, I32, I32, I32, VP, VP, VP, VP)
_sig("rgd_probe_fixed", I32, VP, VP, VP, VP, I32, I32, I32, I32, VP, VP, VP, VP)
_sig("rgd_probe_soft", I32, VP, VP, VP, VP, I32, I32, I32, I32, I32, C.c_float, VP, VP, VP, VP)
_sig("rgd_probe_adaptive", I32, VP, VP, VP, VP, I32, I32, I32, I32, I32, C.c_float, VP, C.c_float, VP, VP, VP, VP)
_sig("rgd_prefill_kv_scored", I32, VP, VP, VP, I32, I32, I32, VP, I32, VP, C.c_float, VP, VP)
_sig("rgd_kernel_probe_step", I32, VP, VP, I32, VP, I32, I32, I32, I32, C.c_float, VP, VP, VP, VP)
_sig("rgd_gate", I32, VP, VP, I32, I32P, I32P, I32P, VP)
_sig("rgd_sample_continuations", I32, VP, VP, VP, I32P, I32, I32, I32, F32, F32, VP, VP, VP, VP, VP)
_sig("rgd_sample_continuations_pless", I32, VP, VP, VP, I32P, I32, I32, I32, F32, VP, VP, VP, VP, VP)
_sig("rgd_check_status", I32, VP, VP)
_sig("rgd_kernel_attention", I32, VP, VP, I32, I32P, I32P, VP, VP, I32, I32, VP, VP, I32, VP, I32,
     I32, I32, VP, VP)
_sig("rgd_kernel_lm_head", I32, VP, VP, I32, VP, VP)
_sig("rgd_sampler_workspace_bytes", U64, I32, I32)
_sig("rgd_kernel_argmax", I32, VP, I32, I32, VP, VP, VP)
_sig("rgd_kernel_sample", I32, VP, I32, I32, F32, F32, VP, U32, U32, I32, VP, VP, VP)
_sig("rgd_kernel_sample_noalloc", I32, VP, I32, I32, F32, F32, VP, U32, U32, I32, VP, VP)
_sig("rgd_kernel_sample_pless", I32, VP, I32, I32, F32, VP, U32, U32, I32, VP, VP, VP)
_CACHE = C.POINTER(PagedCacheDesc)
_sig("rgd_paged_workspace_bytes", U64, _CACHE)
_sig("rgd_paged_select", I32, _CACHE, VP, VP, VP, VP)
_sig("rgd_paged_reserve", I32, _CACHE, VP, VP, VP)
_sig("rgd_paged_reserve_granted", I32, _CACHE, VP, VP, VP, VP)
_sig("rgd_paged_compact", I32, _CACHE, VP, VP, VP)
_sig("rgd_paged_append", I32, _CACHE, I32, VP, VP, I64, I64, I32, VP, VP)
_sig("rgd_paged_attention_workspace_bytes", U64, _CACHE, I32, I32)
_sig("rgd_paged_attention", I32, _CACHE, I32, VP, I64, I32, VP, I32, VP, VP, VP, VP)
_sig("rgd_verify_workspace_bytes", U64, I32, I32, I32)
_sig("rgd_verify_drafts", I32, VP, VP, VP, VP, I32, I32, I32, F32, F32, VP, VP, VP, VP, VP)
_sig("rgd_rotary_frequencies", I32, I32, C.c_double, C.POINTER(RotaryScalingDesc), C.POINTER(C.c_double), C.POINTER(F32))
_sig("rgd_paged_append_rotated", I32, _CACHE, I32, VP, VP, VP, I64, I64, I64, I32, VP, I32, VP, C.POINTER(RotaryDesc), VP, VP,
     F32, VP, I64, VP)
_sig("rgd_paged_share_bytes", U64, _CACHE, I32, I32)
_sig("rgd_paged_share", I32, _CACHE, I32, VP, I32, VP, VP, VP, VP)
_sig("rgd_paged_attention_shared_workspace_bytes", U64, _CACHE, I32, I32)
_sig("rgd_paged_attention_shared", I32, _CACHE, I32, VP, I64, I32, I32, VP, VP, VP, VP, VP)
_sig("rgd_sample_truncated_workspace_bytes", U64, I32, I32)
_sig("rgd_sample_truncated", I32, VP, I64, I32, I32, VP, VP, VP, VP, VP, VP, VP, VP, VP)
_sig("rgd_timing_enable", I32, VP, I32)
_sig("rgd_timing_read", I32, VP, C.POINTER(C.c_double), C.POINTER(C.c_int64))

TIMERS = ("lm_head", "attention", "attn_prefix", "sampler", "step")


class RGDError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"rgd error {STATUS.get(code, code)}: {msg}")
        self.code = code


def _check(rc):
    if rc != 0:
        raise RGDError(rc, lib.rgd_last_error().decode())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _host_i32(seq):
    import numpy as np
    a = np.ascontiguousarray(np.asarray(seq, dtype=np.int32))
    return a, a.ctypes.data_as(I32P)


class Model:
    """A model handle over caller-owned device weights (kept alive here)."""

    def __init__(self, cfg: ModelConfig, tensors: dict, layers: list, max_rows: int):
        self.cfg = cfg
        self._keep = (tensors, layers)
        lw = (LayerWeights * len(layers))()
        for i, L in enumerate(layers):
            for n in LayerWeights._fields_:
                setattr(lw[i], n[0], L[n[0]].data_ptr())
        self._lw = lw
        w = Weights(tensors["embed"].data_ptr(), tensors["final_norm"].data_ptr(),
                    tensors["lm_head"].data_ptr(), lw)
        h = VP()
        _check(lib.rgd_model_create(C.byref(cfg), C.byref(w), max_rows, C.byref(h)))
        self.h = h

    def close(self):
        if self.h:
            lib.rgd_model_destroy(self.h)
            self.h = VP()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KV:
    """Prompt-KV and tail-page state over caller-owned device buffers."""

    def __init__(self, model: Model, max_prompts, max_prefix, n_pages, page_size, prefix_k,
                 prefix_v, pool_k, pool_v):
        self.model = model
        self._keep = (prefix_k, prefix_v, pool_k, pool_v)
        self.prefix_k, self.prefix_v, self.pool_k, self.pool_v = prefix_k, prefix_v, pool_k, pool_v
        h = VP()
        _check(lib.rgd_kv_create(model.h, max_prompts, max_prefix, n_pages, page_size,
                                 _ptr(prefix_k), _ptr(prefix_v), _ptr(pool_k), _ptr(pool_v),
                                 C.byref(h)))
        self.h = h

    def set_prefix_len(self, prompt, length):
        _check(lib.rgd_kv_set_prefix_len(self.h, prompt, length))

    def close(self):
        if self.h:
            lib.rgd_kv_destroy(self.h)
            self.h = VP()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Table:
    """Refusal-prefix table (CSR host arrays, copied to the device)."""

    def __init__(self, offsets, tokens, owner=None, min_match=2):
        import numpy as np
        off, offp = _host_i32(offsets)
        tok, tokp = _host_i32(tokens if len(tokens) else np.zeros(1, np.int32))
        n = len(off) - 1
        ownp = None
        if owner is not None:
            own, ownp = _host_i32(owner)
        h = VP()
        _check(lib.rgd_table_create(offp, tokp, n, ownp, min_match, C.byref(h)))
        self.h = h

    def close(self):
        if self.h:
            lib.rgd_table_destroy(self.h)
            self.h = VP()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def prefill_kv(model, kv, tokens, start_pos, last_logits):
    B, n = tokens.shape
    _check(lib.rgd_prefill_kv(model.h, kv.h, _ptr(tokens), B, n, start_pos, _ptr(last_logits),
                              _stream()))


def probe(model, kv, last_logits, table, B, k, c, eos, probe_tokens, probe_len, event):
    """table None: fixed-length probe (no refusal set)."""
    _check(lib.rgd_probe(model.h, kv.h, _ptr(last_logits), table.h if table is not None else None, B, k, c,
                         eos, _ptr(probe_tokens), _ptr(probe_len), _ptr(event), _stream()))


def probe_fixed(model, kv, last_logits, table, B, k, c, eos, probe_tokens, probe_len, event):
    """Probe with no early exit: k greedy tokens (or up to eos), then the table
    judges the finished probe (table None: every probe is a hit)."""
    _check(lib.rgd_probe_fixed(model.h, kv.h, _ptr(last_logits), table.h if table is not None else None, B, k,
                               c, eos, _ptr(probe_tokens), _ptr(probe_len), _ptr(event), _stream()))


def kernel_probe_step(model, logits, table, k, c, eos, topk, rho, probe_tokens, probe_len, event):
    """One probe step for prompts 0..R-1 (R = logits rows) on given logits."""
    _check(lib.rgd_kernel_probe_step(model.h, _ptr(logits), logits.shape[0],
                                     table.h if table is not None else None, k, c, eos, topk, float(rho),
                                     _ptr(probe_tokens), _ptr(probe_len), _ptr(event), _stream()))


def prefill_kv_scored(model, kv, tokens, start_pos, last_logits, cls_layer, cls_w, cls_b, scores):
    """Prefill plus the residual-stream pre-check score of each prompt."""
    B, n = tokens.shape
    _check(lib.rgd_prefill_kv_scored(model.h, kv.h, _ptr(tokens), B, n, start_pos, _ptr(last_logits), cls_layer,
                                     _ptr(cls_w), float(cls_b), _ptr(scores), _stream()))


def probe_adaptive(model, kv, last_logits, table, B, k, c, eos, topk, rho, scores, theta, probe_tokens,
                   probe_len, event):
    """Adaptive gate: prompts scored <= theta are SKIPPED, the others probed."""
    _check(lib.rgd_probe_adaptive(model.h, kv.h, _ptr(last_logits), table.h if table is not None else None, B,
                                  k, c, eos, topk, float(rho), _ptr(scores), float(theta), _ptr(probe_tokens),
                                  _ptr(probe_len), _ptr(event), _stream()))


def probe_soft(model, kv, last_logits, table, B, k, c, eos, topk, rho, probe_tokens, probe_len, event):
    """Probe with the soft compatibility gate: tokens 1..c are soft steps."""
    _check(lib.rgd_probe_soft(model.h, kv.h, _ptr(last_logits), table.h if table is not None else None, B, k,
                              c, eos, topk, float(rho), _ptr(probe_tokens), _ptr(probe_len), _ptr(event),
                              _stream()))


def gate(kv, event, B):
    """Returns (decision list, miss index list)."""
    import numpy as np
    dec = np.zeros(B, np.int32)
    miss = np.zeros(B, np.int32)
    nm = C.c_int32(0)
    _check(lib.rgd_gate(kv.h, _ptr(event), B, dec.ctypes.data_as(I32P), C.byref(nm),
                        miss.ctypes.data_as(I32P), _stream()))
    return dec, miss[:nm.value]


def sample_continuations(model, kv, last_logits, prompt_idx, N, steps, T, min_p, seeds, out,
                         forced=None, logits_tap=None):
    pi, pip = _host_i32(prompt_idx)
    _check(lib.rgd_sample_continuations(model.h, kv.h, _ptr(last_logits), pip, len(pi), N, steps,
                                        T, min_p, _ptr(seeds), _ptr(forced), _ptr(logits_tap),
                                        _ptr(out), _stream()))


def sample_continuations_pless(model, kv, last_logits, prompt_idx, N, steps, T, seeds, out,
                               forced=None, logits_tap=None):
    pi, pip = _host_i32(prompt_idx)
    _check(lib.rgd_sample_continuations_pless(model.h, kv.h, _ptr(last_logits), pip, len(pi), N, steps,
                                              T, _ptr(seeds), _ptr(forced), _ptr(logits_tap),
                                              _ptr(out), _stream()))


def check_status(model):
    _check(lib.rgd_check_status(model.h, _stream()))


def kernel_attention(model, q, row_prompt, plen, prefix_k, prefix_v, max_prompts, max_prefix,
                     pool_k, pool_v, page_size, pages, max_pages, tail_len, out, splits=0):
    rp, rpp = _host_i32(row_prompt)
    pl, plp = _host_i32(plen)
    _check(lib.rgd_kernel_attention(model.h, _ptr(q), len(rp), rpp, plp, _ptr(prefix_k),
                                    _ptr(prefix_v), max_prompts, max_prefix, _ptr(pool_k),
                                    _ptr(pool_v), page_size, _ptr(pages), max_pages, tail_len,
                                    splits, _ptr(out), _stream()))


def kernel_lm_head(model, h, logits):
    _check(lib.rgd_kernel_lm_head(model.h, _ptr(h), h.shape[0], _ptr(logits), _stream()))


def timing_enable(model, period=1):
    """period >= 1 times every period-th launch of each unit; 0 (or False) stops."""
    _check(lib.rgd_timing_enable(model.h, int(period)))


def timing_read(model):
    """{unit: (total ms, launches)} since the last read."""
    ms = (C.c_double * len(TIMERS))()
    n = (C.c_int64 * len(TIMERS))()
    _check(lib.rgd_timing_read(model.h, ms, n))
    return {k: (ms[i], n[i]) for i, k in enumerate(TIMERS)}


def sampler_workspace_bytes(R, V):
    return int(lib.rgd_sampler_workspace_bytes(R, V))


def kernel_argmax(z, workspace, out):
    R, V = z.shape
    _check(lib.rgd_kernel_argmax(_ptr(z), R, V, _ptr(workspace), _ptr(out), _stream()))


def kernel_sample(z, T, min_p, seeds, ctr, stream0, draws, workspace, out):
    R, V = z.shape
    _check(lib.rgd_kernel_sample(_ptr(z), R, V, T, min_p, _ptr(seeds), ctr, stream0, draws,
                                 _ptr(workspace), _ptr(out), _stream()))


NOALLOC_SCRATCH_BYTES = 1 << 20


def kernel_sample_noalloc(z, T, min_p, seeds, ctr, stream0, draws, out):
    """rgd_kernel_sample without a workspace: the library's fixed device scratch
    (RGD_NOALLOC_SCRATCH_BYTES) is used; nothing is allocated."""
    R, V = z.shape
    _check(lib.rgd_kernel_sample_noalloc(_ptr(z), R, V, T, min_p, _ptr(seeds), ctr, stream0, draws, _ptr(out),
                                         _stream()))


def kernel_sample_pless(z, T, seeds, ctr, stream0, draws, workspace, out):
    R, V = z.shape
    _check(lib.rgd_kernel_sample_pless(_ptr(z), R, V, T, _ptr(seeds), ctr, stream0, draws,
                                       _ptr(workspace), _ptr(out), _stream()))


# ------------------------------------------------------------ paged sequences --
def _refuse(msg):
    raise RGDError(1, msg)


def _tensor(device, name, t, dtype, shape):
    """The address of a contiguous tensor of this type, shape (None: any) and device (its index); anything else is
    refused."""
    if t is None:
        _refuse(f"{name} is None")
    if t.dtype is not dtype or t.get_device() != device:
        _refuse(f"{name} must be a {dtype} tensor on GPU {device}, got {t.dtype} on {t.device}")
    if shape is not None and t.shape != shape:
        _refuse(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        _refuse(f"{name} must be contiguous")
    return t.data_ptr()


def _int32(*numbers):
    """Refuses what ctypes would pass on as its lowest 32 bits."""
    if max(numbers) > 0x7FFFFFFF or min(numbers) < -0x80000000:
        _refuse(f"{max(numbers, key=abs)} is out of range")


def _optional(device, name, t, dtype, shape):
    return None if t is None else _tensor(device, name, t, dtype, shape)


def _sized(device, name, t, need):
    p = _tensor(device, name, t, torch.uint8, None)
    if t.numel() < need:
        _refuse(f"{name} holds {t.numel()} of {need} bytes")
    return p


def _workspace(device, ws, need):
    return _sized(device, "workspace", ws, need)


def _rows(device, name, t, dtype, shape):
    """Address and row stride of a tensor [rows][heads][D] whose rows may lie apart (a slice of a fused projection)."""
    if t is None:
        _refuse(f"{name} is None")
    if t.dtype is not dtype or t.get_device() != device or t.shape != shape:
        _refuse(f"{name} must be a {dtype} tensor {tuple(shape)} on GPU {device}, got {t.dtype} {tuple(t.shape)} on "
                f"{t.device}")
    row, head, one = t.stride()
    if (shape[2] > 1 and one != 1) or (shape[1] > 1 and head != shape[2]):
        _refuse(f"{name}: the heads of a row must be contiguous")
    return t.data_ptr(), row if shape[0] > 1 else shape[1] * shape[2]


def _launch(device, fn, *args):
    """fn(*args, stream) on the operands' device and its current stream."""
    if torch._C._cuda_getDevice() == device:  # (there are tensors on it, so it is initialised)
        _check(fn(*args, torch._C._cuda_getCurrentRawStream(device)))
        return
    with torch.cuda.device(device):
        _check(fn(*args, torch._C._cuda_getCurrentRawStream(device)))


class PagedCache:
    """Paged sequences over caller-owned device tensors (kept alive here):
    pool_k [L][pages][Hkv][page_size][D], pool_v [L][pages][Hkv][D][page_size]
    (bf16 or fp32), and int32 pages [S][max_pages], lens [S], refs [pages],
    status [1].  The operators below change the tensors in place."""

    def __init__(self, pool_k, pool_v, pages, lens, refs, status):
        types = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}
        if pool_k.dim() != 5 or pool_k.dtype not in types or not pool_k.is_cuda:
            _refuse("pool_k must be a 5-dimensional bf16 or fp32 tensor on a GPU")
        L, P, H, ps, D = pool_k.shape
        if pages.dim() != 2:
            _refuse("pages must have two dimensions")
        S, width = pages.shape
        dev, i32 = pool_k.get_device(), torch.int32
        _int32(*pool_k.shape, *pages.shape)
        self.desc = PagedCacheDesc(L, P, H, ps, D, types[pool_k.dtype], S, width,
                                   _tensor(dev, "pool_k", pool_k, pool_k.dtype, None),
                                   _tensor(dev, "pool_v", pool_v, pool_k.dtype, (L, P, H, D, ps)),
                                   _tensor(dev, "pages", pages, i32, None), _tensor(dev, "lens", lens, i32, (S,)),
                                   _tensor(dev, "refs", refs, i32, (P,)), _tensor(dev, "status", status, i32, (1,)))
        self.ref = C.byref(self.desc)
        self.device, self.gpu, self.dtype = pool_k.device, dev, pool_k.dtype
        self.pool_k, self.pool_v, self.pages, self.lens, self.refs, self.status = pool_k, pool_v, pages, lens, refs, status
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = L, P, H, ps, D
        self.max_seqs, self.max_pages = S, width
        self._needs = {}  # workspace bytes by what they are for

    def need(self, what, fn, *args):
        n = self._needs.get(what)
        if n is None:
            _int32(0, *args)
            n = self._needs[what] = _bytes(fn(self.ref, *args))
        return n


def _bytes(n):
    if n == 0:
        raise RGDError(1, lib.rgd_last_error().decode())
    return int(n)


def paged_workspace_bytes(cache):
    return cache.need("pages", lib.rgd_paged_workspace_bytes)


def paged_select(cache, parent, keep, workspace=None):
    """Sequence s becomes the first keep[s] positions (None or negative: all) of
    sequence parent[s] (None or outside the cache: itself), all at once.  Without parent it needs no workspace."""
    dev, shape = cache.gpu, (cache.max_seqs,)
    ws = None
    if parent is not None or workspace is not None:
        ws = _workspace(dev, workspace, paged_workspace_bytes(cache))
    _launch(dev, lib.rgd_paged_select, cache.ref, _optional(dev, "parent", parent, torch.int32, shape),
            _optional(dev, "keep", keep, torch.int32, shape), ws)


def paged_reserve(cache, grow, workspace, granted=None):
    """Makes room for grow[s] more positions of each sequence and adds them to lens;
    cache.status becomes 1, and nothing else changes, where there is none.  granted (int32 [S], may be grow)
    receives what each sequence got, 0 then: the n_new of what is queued without a look at the status."""
    dev, shape = cache.gpu, (cache.max_seqs,)
    pg = _tensor(dev, "grow", grow, torch.int32, shape)
    ws = _workspace(dev, workspace, paged_workspace_bytes(cache))
    if granted is None:
        _launch(dev, lib.rgd_paged_reserve, cache.ref, pg, ws)
    else:
        _launch(dev, lib.rgd_paged_reserve_granted, cache.ref, pg, _tensor(dev, "granted", granted, torch.int32, shape), ws)


def paged_compact(cache, live, workspace):
    """Moves the live pages to [0, live[0])."""
    dev = cache.gpu
    _launch(dev, lib.rgd_paged_compact, cache.ref, _tensor(dev, "live", live, torch.int32, (1,)),
            _workspace(dev, workspace, paged_workspace_bytes(cache)))


def paged_append(cache, layer, k, v, n, n_new=None):
    """K and V rows [S * n][Hkv][D] (rows may lie apart) of each sequence's last n_new[s]
    (None: n) positions into the pages of one layer."""
    _int32(layer, n)
    dev, S = cache.gpu, cache.max_seqs
    shape = (S * n, cache.n_kv_heads, cache.head_dim)
    pk, ldk = _rows(dev, "k", k, cache.dtype, shape)
    pv, ldv = _rows(dev, "v", v, cache.dtype, shape)
    _launch(dev, lib.rgd_paged_append, cache.ref, layer, pk, pv, ldk, ldv, n,
            _optional(dev, "n_new", n_new, torch.int32, (S,)))


def paged_attention_workspace_bytes(cache, n, n_heads):
    return cache.need((n, n_heads), lib.rgd_paged_attention_workspace_bytes, n, n_heads)


def paged_attention(cache, layer, q, n, n_new, workspace, out, lse=None):
    """Causal attention of each sequence's last n_new[s] (None: n) positions, q
    [S * n][heads][D] (rows may lie apart), into out [S * n][heads * D] and lse [S * n][heads]."""
    _int32(layer, n)
    dev, S, D = cache.gpu, cache.max_seqs, cache.head_dim
    if q is None or q.dim() != 3:
        _refuse("q must be a tensor of three dimensions")
    heads = q.shape[1]
    pq, ldq = _rows(dev, "q", q, cache.dtype, (S * n, heads, D))
    _launch(dev, lib.rgd_paged_attention, cache.ref, layer, pq, ldq, n,
            _optional(dev, "n_new", n_new, torch.int32, (S,)), heads,
            _workspace(dev, workspace, paged_attention_workspace_bytes(cache, n, heads)),
            _tensor(dev, "out", out, cache.dtype, (S * n, heads * D)),
            _optional(dev, "lse", lse, torch.float32, (S * n, heads)))


# ------------------------------------------------- rotary positions, head norms --
class RotaryScaling:
    """How a rotation's frequencies are changed by `factor` for positions beyond the trained `context`: kind "linear",
    "base", "by_rotations" or "by_index" (the last two between `low` and `high` turns over the context; high None: 4 turns by
    rotations, 32 by index, as models trained with these have them)."""

    KINDS = ("linear", "base", "by_rotations", "by_index")

    def __init__(self, kind, factor, context=0.0, low=1.0, high=None):
        if kind not in self.KINDS:
            _refuse(f"kind must be one of {', '.join(self.KINDS)}")
        if high is None:
            high = 32.0 if kind == "by_index" else 4.0
        self.desc = RotaryScalingDesc(1 + self.KINDS.index(kind), factor, context, low, high)


class Rotary:
    """A rotation of the first `dim` dimensions of a head, in pairs (j, j + dim / 2) or, interleaved, (2 j, 2 j + 1), by
    position * freq[j] radians, cosine and sine times `scale`.  Give theta (and scaling), or frequencies of your own."""

    def __init__(self, dim, theta=None, interleaved=False, scaling=None, freq=None, scale=1.0):
        _int32(dim)
        if (theta is None) == (freq is None):
            _refuse("one of theta and freq is wanted")
        if freq is None:
            factor = F32(1.0)
            self.freq = (C.c_double * max(1, min(dim, 128) // 2))()
            _check(lib.rgd_rotary_frequencies(dim, theta, C.byref(scaling.desc) if scaling else None, self.freq,
                                              C.byref(factor)))
            scale *= factor.value
        else:
            if scaling is not None:
                _refuse("scaling goes with theta")
            if len(freq) * 2 != dim:
                _refuse(f"{dim} dimensions have {dim // 2} frequencies, got {len(freq)}")
            self.freq = (C.c_double * max(1, len(freq)))(*freq)
        self.dim, self.interleaved, self.scale = dim, bool(interleaved), scale
        self.desc = RotaryDesc(dim, self.interleaved, scale, self.freq)
        self.ref = C.byref(self.desc)


def paged_append_rotated(cache, layer, q, k, v, n, rotary, q_out, n_new=None, positions=None, q_norm=None, k_norm=None,
                         eps=1e-5):
    """paged_append of q [S * n][heads][D], k and v [S * n][Hkv][D] (rows may lie apart) as a projection leaves them: the
    heads of q and k are normed (gains q_norm, k_norm [D] fp32, None: not), rotated by their positions (positions int32 [S * n],
    None: those in the cache; rotary None: not), k and v appended to the pages of one layer and q written to q_out (q itself, or apart)."""
    _int32(layer, n)
    dev, S, D, i32, f32 = cache.gpu, cache.max_seqs, cache.head_dim, torch.int32, torch.float32
    if q is None or q.dim() != 3:
        _refuse("q must be a tensor of three dimensions")
    heads, kv = q.shape[1], (S * n, cache.n_kv_heads, D)
    shape = (S * n, heads, D)
    pq, ldq = _rows(dev, "q", q, cache.dtype, shape)
    pk, ldk = _rows(dev, "k", k, cache.dtype, kv)
    pv, ldv = _rows(dev, "v", v, cache.dtype, kv)
    po, ldo = _rows(dev, "q_out", q_out, cache.dtype, shape)
    _launch(dev, lib.rgd_paged_append_rotated, cache.ref, layer, pq, pk, pv, ldq, ldk, ldv, n,
            _optional(dev, "n_new", n_new, i32, (S,)), heads, _optional(dev, "positions", positions, i32, (S * n,)),
            None if rotary is None else rotary.ref, _optional(dev, "q_norm", q_norm, f32, (D,)),
            _optional(dev, "k_norm", k_norm, f32, (D,)), eps, po, ldo)


# ------------------------------------------- attention over pages that are shared --
def paged_share_bytes(cache, n, n_heads):
    return cache.need(("share", n, n_heads), lib.rgd_paged_share_bytes, n, n_heads)


def paged_share(cache, n, n_new, n_heads, group, plan, shared=None):
    """Finds which leading pages the sequences of each group (labels int32 [S]; None: all are one) share, for up to n new
    tokens each (n_new int32 [S], None: n), once for all layers: plan (uint8, paged_share_bytes) receives it for
    paged_attention_shared, shared (int32 [S]) the positions."""
    _int32(n, n_heads)
    dev, i32, shape = cache.gpu, torch.int32, (cache.max_seqs,)
    _launch(dev, lib.rgd_paged_share, cache.ref, n, _optional(dev, "n_new", n_new, i32, shape), n_heads,
            _optional(dev, "group", group, i32, shape), _sized(dev, "plan", plan, paged_share_bytes(cache, n, n_heads)),
            _optional(dev, "shared", shared, i32, shape))


def paged_attention_shared_workspace_bytes(cache, n, n_heads):
    return cache.need(("shared", n, n_heads), lib.rgd_paged_attention_shared_workspace_bytes, n, n_heads)


def paged_attention_shared(cache, layer, q, n, plan, workspace, out, lse=None):
    """paged_attention with the counts of a plan, whose shared positions are read once for each group: q
    [S * n][heads][D] (rows may lie apart) into out [S * n][heads * D] and lse [S * n][heads]."""
    _int32(layer, n)
    dev, S, D = cache.gpu, cache.max_seqs, cache.head_dim
    if q is None or q.dim() != 3:
        _refuse("q must be a tensor of three dimensions")
    heads = q.shape[1]
    pq, ldq = _rows(dev, "q", q, cache.dtype, (S * n, heads, D))
    _launch(dev, lib.rgd_paged_attention_shared, cache.ref, layer, pq, ldq, n, heads,
            _sized(dev, "plan", plan, paged_share_bytes(cache, n, heads)),
            _workspace(dev, workspace, paged_attention_shared_workspace_bytes(cache, n, heads)),
            _tensor(dev, "out", out, cache.dtype, (S * n, heads * D)),
            _optional(dev, "lse", lse, torch.float32, (S * n, heads)))


# ------------------------------------------------------- verification of drafts --
def verify_workspace_bytes(S, K, V):
    _int32(S, K, V)
    n = lib.rgd_verify_workspace_bytes(S, K, V)
    if n == 0:
        _refuse("S, K or V out of range")
    return int(n)


def verify_drafts(target, draft, draft_tokens, n_draft, T, min_p, u, workspace, out, n_accepted):
    """Accepts a prefix of each sequence's drafts and draws the token after it, from target
    logits [S][K+1][V], the drafts' logits [S][K][V] (None: certain drafts) and uniforms u [S][K+1]."""
    if target is None or target.dim() != 3 or not target.is_cuda:
        _refuse("target must be a 3-dimensional tensor on a GPU")
    S, K1, V = target.shape
    K, dev, f32, i32 = K1 - 1, target.get_device(), torch.float32, torch.int32
    _launch(dev, lib.rgd_verify_drafts, _tensor(dev, "target", target, f32, None),
            _optional(dev, "draft", draft, f32, (S, K, V)), _tensor(dev, "draft_tokens", draft_tokens, i32, (S, K)),
            _optional(dev, "n_draft", n_draft, i32, (S,)), S, K, V, T, min_p, _tensor(dev, "u", u, f32, (S, K1)),
            _workspace(dev, workspace, verify_workspace_bytes(S, K, V)), _tensor(dev, "out", out, i32, (S, K1)),
            _tensor(dev, "n_accepted", n_accepted, i32, (S,)))


# ------------------------------------------------- sampling with limits for each row --
def sample_truncated_workspace_bytes(R, V):
    _int32(R, V)
    n = lib.rgd_sample_truncated_workspace_bytes(R, V)
    if n == 0:
        _refuse("R or V out of range")
    return int(n)


def sample_truncated(z, u, workspace, out, T=None, top_k=None, top_p=None, min_p=None, logp=None):
    """Draws one id from each row of logits z [R][V] (rows may lie apart) by the uniforms u [R], under limits for each row:
    temperature T, then top_k (int32), top_p and min_p (each [R]; None: without); logp [R] receives the id's log probability."""
    if z is None or z.dim() != 2 or not z.is_cuda:
        _refuse("z must be a 2-dimensional tensor on a GPU")
    R, V = z.shape
    dev, f32, i32, shape = z.get_device(), torch.float32, torch.int32, (R,)
    if z.dtype is not f32 or (V > 1 and z.stride(1) != 1):
        _refuse(f"z must be fp32 with contiguous rows, got {z.dtype} of strides {z.stride()}")
    _launch(dev, lib.rgd_sample_truncated, z.data_ptr(), z.stride(0) if R > 1 else V, R, V, _optional(dev, "T", T, f32, shape),
            _optional(dev, "top_k", top_k, i32, shape), _optional(dev, "top_p", top_p, f32, shape),
            _optional(dev, "min_p", min_p, f32, shape), _tensor(dev, "u", u, f32, shape),
            _workspace(dev, workspace, sample_truncated_workspace_bytes(R, V)), _tensor(dev, "out", out, i32, shape),
            _optional(dev, "logp", logp, f32, shape))
