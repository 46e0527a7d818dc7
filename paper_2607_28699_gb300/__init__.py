"""Python binding of the WitCert GB300 library (ctypes over ``include/witcert.h``).

Argument marshalling only: every function passes device pointers, sizes and
the current CUDA stream to the C ABI, where all work runs in the library's
CUDA kernels.  PyTorch supplies device memory and streams.  There is no CPU
fallback: importing this package without the compiled library raises.

    import paper_2607_28699_gb300 as wc
    desc = wc.CacheDesc(num_q_heads=28, num_kv_heads=4, num_pages=n)
    cache = wc.LayerCache.empty(desc, device="cuda")
    wc.kv_quantize_witness(desc, layer, k, v, slot_mapping, cache)
    ws = wc.Workspace(desc, batch, max_pages)
    out, meter, meter_raw = wc.metered_decode_attention(desc, layer, q, block_table,
                                                        ctx_lens, cache, ws)
    keep_q, keep_kv, n_kept = wc.gate(meter_raw, group, tau)

and for the unmetered 8-bit cache with one scale per page and head (rotation, append and
attention, of one token or of many):

    desc = wc.BlockDesc(num_q_heads=28, num_kv_heads=4, num_pages=n)
    cache = wc.BlockCache.empty(desc, device="cuda")
    q = wc.block_append(desc, k, v, ctx_lens, block_table, cache, cu_new=cu, cos=cos, sin=sin, q=q)
    ws = wc.BlockWorkspace(desc, batch, n_tok, max_pages)
    out = wc.block_extend_attention(desc, q, cu, block_table, ctx_lens, cache, ws)
    out = wc.block_decode_attention(desc, q, block_table, ctx_lens, cache, ws)

Layers that norm their queries and keys and see a window of the last tokens give ``block_append`` the weights (k_norm, q_norm)
and the attention calls ``window`` and ``sinks``; ``qk_norm_rotate`` norms and rotates ahead of the metered caches.
"""

import ctypes
import math
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libwitcert.so")

SCHEME_DITHER_INT8 = 0
SCHEME_FP8_E4M3 = 1
SCHEME_DITHER_INT8_G32 = 2
ROPE_HALF = 0
ROPE_INTERLEAVED = 1
CODE_INT8 = 0
CODE_E4M3 = 1
ACT_FP16 = 0
ACT_BF16 = 1
DEV_BAD_SLOT, DEV_BAD_PAGE, DEV_BAD_CTX, DEV_TIMEOUT, DEV_BAD_PAIR, DEV_BAD_APPEND = 1, 2, 4, 8, 16, 32
DEV_BAD_POSITION, DEV_BAD_ROWS = 64, 128
EXPORTS = ("wc_kv_quantize_witness", "wc_workspace_size", "wc_metered_decode_attention",
           "wc_metered_decode_attention_tier_b", "wc_metered_decode_attention_noalloc",
           "wc_kv_quantize_witness_v", "wc_metered_decode_attention_v", "wc_gate_joint",
           "wc_metered_decode_attention_repair", "wc_repair_select",
           "wc_kv_quantize_witness_g32", "wc_metered_decode_attention_g32", "wc_select_bypass_pairs",
           "wc_metered_decode_attention_append", "wc_testing_decode_stalled_page",
           "wc_block_append", "wc_block_append_norm", "wc_qk_norm_rotate", "wc_block_workspace_size", "wc_block_decode_attention", "wc_block_extend_attention",
           "wc_block_decode_attention_window", "wc_block_extend_attention_window",
           "wc_gate", "wc_read_status", "wc_last_error", "wc_version")


class WitCertError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"witcert status {status}: {message}")
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64
    lib.wc_kv_quantize_witness.argtypes = [vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.wc_kv_quantize_witness.restype = ctypes.c_int
    lib.wc_workspace_size.argtypes = [vp, i32, i32]
    lib.wc_workspace_size.restype = ctypes.c_size_t
    lib.wc_metered_decode_attention.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp,
                                                vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.wc_metered_decode_attention.restype = ctypes.c_int
    lib.wc_metered_decode_attention_tier_b.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp,
                                                       ctypes.c_double, vp, vp, vp, vp, vp, vp, ctypes.c_size_t,
                                                       vp]
    lib.wc_metered_decode_attention_tier_b.restype = ctypes.c_int
    lib.wc_testing_decode_stalled_page.argtypes = [vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                                   vp, ctypes.c_size_t, i32, vp]
    lib.wc_testing_decode_stalled_page.restype = ctypes.c_int
    lib.wc_gate.argtypes = [vp, i32, i32, ctypes.c_float, vp, vp, vp, vp]
    lib.wc_gate.restype = ctypes.c_int
    lib.wc_gate_joint.argtypes = [vp, vp, vp, i32, i32, ctypes.c_float, ctypes.c_float, vp, vp, vp, vp]
    lib.wc_gate_joint.restype = ctypes.c_int
    lib.wc_kv_quantize_witness_v.argtypes = [vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.wc_kv_quantize_witness_v.restype = ctypes.c_int
    lib.wc_metered_decode_attention_v.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp,
                                                  vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.wc_metered_decode_attention_v.restype = ctypes.c_int
    lib.wc_metered_decode_attention_repair.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp,
                                                       vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.wc_metered_decode_attention_repair.restype = ctypes.c_int
    lib.wc_repair_select.argtypes = [vp, vp, vp, i32, i32, i32, vp, ctypes.c_float, vp, vp, vp, vp, vp, vp]
    lib.wc_repair_select.restype = ctypes.c_int
    lib.wc_kv_quantize_witness_g32.argtypes = [vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.wc_kv_quantize_witness_g32.restype = ctypes.c_int
    lib.wc_metered_decode_attention_g32.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, i32,
                                                    ctypes.c_double, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.wc_metered_decode_attention_g32.restype = ctypes.c_int
    lib.wc_select_bypass_pairs.argtypes = [vp, i32, i32, i32, i32, vp, vp]
    lib.wc_select_bypass_pairs.restype = ctypes.c_int
    lib.wc_metered_decode_attention_append.argtypes = [vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp,
                                                       vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.wc_metered_decode_attention_append.restype = ctypes.c_int
    i64, f32 = ctypes.c_int64, ctypes.c_float
    lib.wc_block_append.argtypes = [vp, i32, vp, i64, vp, i64, vp, i64, vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, i32,
                                    vp, vp, vp, vp, vp, vp]
    lib.wc_block_append.restype = ctypes.c_int
    lib.wc_block_append_norm.argtypes = [vp, i32, vp, i64, vp, i64, vp, i64, vp, i32, vp, vp, i32, vp, i32, vp, vp, vp, i32,
                                         vp, vp, f32, vp, vp, vp, vp, vp, vp]
    lib.wc_block_append_norm.restype = ctypes.c_int
    lib.wc_qk_norm_rotate.argtypes = [i32, i32, vp, i64, vp, i64, i32, vp, i64, vp, i64, i32, i32, vp, vp, f32, i32, i32, vp,
                                      vp, vp, i32, vp, vp]
    lib.wc_qk_norm_rotate.restype = ctypes.c_int
    lib.wc_block_workspace_size.argtypes = [vp, i32, i32, i32]
    lib.wc_block_workspace_size.restype = ctypes.c_size_t
    lib.wc_block_decode_attention.argtypes = [vp, i32, vp, i64, vp, i32, vp, i32, vp, vp, vp, vp, f32, vp, vp, vp,
                                              ctypes.c_size_t, vp]
    lib.wc_block_decode_attention.restype = ctypes.c_int
    lib.wc_block_extend_attention.argtypes = [vp, i32, vp, i64, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp, f32, i32,
                                              vp, vp, vp, ctypes.c_size_t, vp]
    lib.wc_block_extend_attention.restype = ctypes.c_int
    lib.wc_block_decode_attention_window.argtypes = [vp, i32, vp, i64, vp, i32, vp, i32, vp, vp, vp, vp, f32, i32, i32, vp, vp, vp,
                                                     ctypes.c_size_t, vp]
    lib.wc_block_decode_attention_window.restype = ctypes.c_int
    lib.wc_block_extend_attention_window.argtypes = [vp, i32, vp, i64, i32, vp, vp, i32, vp, i32, vp, vp, vp, vp, f32, i32, i32,
                                                     vp, vp, vp, ctypes.c_size_t, vp]
    lib.wc_block_extend_attention_window.restype = ctypes.c_int
    lib.wc_read_status.argtypes = [vp, i32, vp, vp]
    lib.wc_read_status.restype = ctypes.c_int
    lib.wc_last_error.argtypes = []
    lib.wc_last_error.restype = ctypes.c_char_p
    lib.wc_version.restype = ctypes.c_int32
    del u64
    return lib


lib = _load()


class _Desc(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("num_bands", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("scheme", ctypes.c_int32), ("rope_layout", ctypes.c_int32),
                ("dither_bits", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("seed", ctypes.c_uint64)]


@dataclass
class CacheDesc:
    """Mirror of ``wc_cache_desc``."""
    num_q_heads: int
    num_kv_heads: int
    num_pages: int
    scheme: int = SCHEME_DITHER_INT8
    rope_layout: int = ROPE_HALF
    dither_bits: int = 8
    seed: int = 0
    head_dim: int = 128
    num_bands: int = 8
    page_size: int = 16

    @property
    def group(self):
        return self.num_q_heads // self.num_kv_heads

    def c(self):
        return _Desc(self.head_dim, self.num_q_heads, self.num_kv_heads, self.num_bands,
                     self.page_size, self.num_pages, self.scheme, self.rope_layout,
                     self.dither_bits, 0, self.seed & (2 ** 64 - 1))


def _check(status):
    if status != 0:
        raise WitCertError(status, lib.wc_last_error().decode())


# A call of one layer on a short context is bound by this marshalling: the pointers go to
# ctypes as plain integers, and the current stream's handle is taken without the Stream
# object around it (3.0 us of a call, 0.3 so).  Decode of 4096 tokens, 8 heads, outputs
# given: 18.1 -> 10.4 us on the host; gate 8.6 -> 4.0; a 33-token write 11.4 -> 6.8.
def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous")
    return t.data_ptr()


# Not part of torch's public interface: a build without them takes the Stream object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


@dataclass
class LayerCache:
    """One layer's paged cache tensors (layout in ``include/witcert.h``)."""
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    k_scale: Optional[torch.Tensor]
    v_scale: Optional[torch.Tensor]
    k_witness: torch.Tensor
    v_witness: Optional[torch.Tensor] = None   # (||v^ - v||, ||v||) per slot, value side only
    k_bypass: Optional[torch.Tensor] = None    # grouped scheme: exact bypassed key values [.., 16, 2m]
    bypass_pairs: Optional[torch.Tensor] = None   # grouped scheme: int32 [Hkv, m] RoPE pair set

    @staticmethod
    def empty(desc: CacheDesc, device="cuda", value_witness=False, num_bypass_pairs=0):
        shp = (desc.num_pages, desc.num_kv_heads, desc.page_size)
        code_t = torch.uint8 if desc.scheme == SCHEME_FP8_E4M3 else torch.int8
        grouped = desc.scheme == SCHEME_DITHER_INT8_G32
        sshp = shp + (desc.head_dim // 32,) if grouped else shp
        dither = desc.scheme != SCHEME_FP8_E4M3
        m = num_bypass_pairs if grouped else 0
        return LayerCache(
            torch.zeros(shp + (desc.head_dim,), dtype=code_t, device=device),
            torch.zeros(shp + (desc.head_dim,), dtype=code_t, device=device),
            torch.zeros(sshp, dtype=torch.float16, device=device) if dither else None,
            torch.zeros(sshp, dtype=torch.float16, device=device) if dither else None,
            torch.zeros(shp + (desc.num_bands,), dtype=torch.float16, device=device),
            torch.zeros(shp + (2,), dtype=torch.float16, device=device) if value_witness else None,
            torch.zeros(shp + (2 * m,), dtype=torch.float16, device=device) if m else None,
            torch.zeros(desc.num_kv_heads, m, dtype=torch.int32, device=device) if grouped else None)

    @property
    def num_bypass_pairs(self):
        return 0 if self.bypass_pairs is None else int(self.bypass_pairs.shape[1])

    def nbytes(self):
        return sum(t.numel() * t.element_size() for t in
                   (self.k_codes, self.v_codes, self.k_scale, self.v_scale, self.k_witness, self.v_witness,
                    self.k_bypass)
                   if t is not None)


def kv_quantize_witness(desc: CacheDesc, layer: int, k: torch.Tensor, v: torch.Tensor,
                        slot_mapping: torch.Tensor, cache: LayerCache,
                        dev_status: Optional[torch.Tensor] = None, stream=None):
    """``wc_kv_quantize_witness`` (``_v`` when the cache holds a value witness):
    k, v fp16 [n_tok, Hkv, 128]; slots int32 [n_tok]."""
    d = desc.c()
    if desc.scheme == SCHEME_DITHER_INT8_G32:
        _check(lib.wc_kv_quantize_witness_g32(
            ctypes.byref(d), layer, _ptr(k), _ptr(v), _ptr(slot_mapping), int(slot_mapping.numel()),
            _ptr(cache.k_codes), _ptr(cache.v_codes), _ptr(cache.k_scale), _ptr(cache.v_scale),
            _ptr(cache.k_witness), _ptr(cache.k_bypass), _ptr(cache.bypass_pairs), cache.num_bypass_pairs,
            _ptr(dev_status), _stream(stream)))
    elif cache.v_witness is None:
        _check(lib.wc_kv_quantize_witness(
            ctypes.byref(d), layer, _ptr(k), _ptr(v), _ptr(slot_mapping), int(slot_mapping.numel()),
            _ptr(cache.k_codes), _ptr(cache.v_codes), _ptr(cache.k_scale), _ptr(cache.v_scale),
            _ptr(cache.k_witness), _ptr(dev_status), _stream(stream)))
    else:
        _check(lib.wc_kv_quantize_witness_v(
            ctypes.byref(d), layer, _ptr(k), _ptr(v), _ptr(slot_mapping), int(slot_mapping.numel()),
            _ptr(cache.k_codes), _ptr(cache.v_codes), _ptr(cache.k_scale), _ptr(cache.v_scale),
            _ptr(cache.k_witness), _ptr(cache.v_witness), _ptr(dev_status), _stream(stream)))


def workspace_size(desc: CacheDesc, batch: int, max_pages: int) -> int:
    d = desc.c()
    n = lib.wc_workspace_size(ctypes.byref(d), batch, max_pages)
    if n == 0:
        raise WitCertError(1, lib.wc_last_error().decode())
    return n


class Workspace:
    """Zero-filled device workspace for ``metered_decode_attention``."""

    def __init__(self, desc: CacheDesc, batch: int, max_pages: int, device="cuda"):
        self.nbytes = workspace_size(desc, batch, max_pages)
        self.buf = torch.zeros(self.nbytes + 256, dtype=torch.uint8, device=device)
        off = (-self.buf.data_ptr()) % 256
        self.view = self.buf[off:off + self.nbytes]

    def ptr(self):
        return ctypes.c_void_p(self.view.data_ptr())


def metered_decode_attention(desc: CacheDesc, layer: int, q: torch.Tensor, block_table: torch.Tensor,
                             ctx_lens: torch.Tensor, cache: LayerCache, ws: Workspace,
                             out=None, meter=None, meter_raw=None, stream=None):
    """``wc_metered_decode_attention``; returns (out [B,Hq,128], meter [B,Hq], meter_raw [B,Hq]) fp32."""
    batch, max_pages = block_table.shape
    dev = q.device
    if out is None:
        out = torch.empty(batch, desc.num_q_heads, desc.head_dim, dtype=torch.float32, device=dev)
    if meter is None:
        meter = torch.empty(batch, desc.num_q_heads, dtype=torch.float32, device=dev)
    if meter_raw is None:
        meter_raw = torch.empty(batch, desc.num_q_heads, dtype=torch.float32, device=dev)
    d = desc.c()
    if desc.scheme == SCHEME_DITHER_INT8_G32:
        _decode_g32(d, layer, q, block_table, ctx_lens, cache, ws, 0.0, out, meter, meter_raw, None, None, stream)
        return out, meter, meter_raw
    _check(lib.wc_metered_decode_attention(
        ctypes.byref(d), layer, _ptr(q), _ptr(block_table), max_pages, _ptr(ctx_lens), batch,
        _ptr(cache.k_codes), _ptr(cache.v_codes), _ptr(cache.k_scale), _ptr(cache.v_scale),
        _ptr(cache.k_witness), _ptr(out), _ptr(meter), _ptr(meter_raw), ws.view.data_ptr(), ws.nbytes,
        _stream(stream)))
    return out, meter, meter_raw


def metered_decode_attention_append(desc: CacheDesc, layer: int, q: torch.Tensor, block_table: torch.Tensor,
                                    ctx_lens: torch.Tensor, cache: LayerCache, ws: Workspace, k_new: torch.Tensor,
                                    v_new: torch.Tensor, slot_new: torch.Tensor, out=None, meter=None,
                                    meter_raw=None, stream=None):
    """``wc_metered_decode_attention_append``: writes each sequence's new token (k_new, v_new fp16
    [B, Hkv, 128] at slot_new int32 [B], the last of its context) and decodes, in one step;
    returns (out, meter, meter_raw)."""
    batch, max_pages = block_table.shape
    dev = q.device
    cells = (batch, desc.num_q_heads)
    out = torch.empty(batch, desc.num_q_heads, desc.head_dim, dtype=torch.float32, device=dev) if out is None else out
    meter = torch.empty(cells, dtype=torch.float32, device=dev) if meter is None else meter
    meter_raw = torch.empty(cells, dtype=torch.float32, device=dev) if meter_raw is None else meter_raw
    d = desc.c()
    _check(lib.wc_metered_decode_attention_append(
        ctypes.byref(d), layer, _ptr(q), _ptr(block_table), max_pages, _ptr(ctx_lens), batch,
        _ptr(cache.k_codes), _ptr(cache.v_codes), _ptr(cache.k_scale), _ptr(cache.v_scale),
        _ptr(cache.k_witness), _ptr(k_new), _ptr(v_new), _ptr(slot_new), _ptr(out), _ptr(meter), _ptr(meter_raw),
        ws.view.data_ptr(), ws.nbytes, _stream(stream)))
    return out, meter, meter_raw


def _decode_g32(d, layer, q, block_table, ctx_lens, cache, ws, delta_loc, out, meter, meter_raw, meter_b,
                meter_b_raw, stream):
    """``wc_metered_decode_attention_g32`` (grouped-scale cache with the outlier bypass)."""
    batch, max_pages = block_table.shape
    _check(lib.wc_metered_decode_attention_g32(
        ctypes.byref(d), layer, _ptr(q), _ptr(block_table), max_pages, _ptr(ctx_lens), batch,
        _ptr(cache.k_codes), _ptr(cache.v_codes), _ptr(cache.k_scale), _ptr(cache.v_scale),
        _ptr(cache.k_witness), _ptr(cache.k_bypass), _ptr(cache.bypass_pairs), cache.num_bypass_pairs,
        float(delta_loc), _ptr(out), _ptr(meter), _ptr(meter_raw), _ptr(meter_b), _ptr(meter_b_raw),
        ws.view.data_ptr(), ws.nbytes, _stream(stream)))


def select_bypass_pairs(k: torch.Tensor, m: int, rope_layout: int = ROPE_HALF, pairs=None, stream=None):
    """``wc_select_bypass_pairs``: k fp16 [n_tok, Hkv, 128] -> int32 [Hkv, m], the m RoPE pairs of
    largest energy per KV head in increasing order."""
    n_tok, hkv = k.shape[0], k.shape[1]
    pairs = torch.empty(hkv, m, dtype=torch.int32, device=k.device) if pairs is None else pairs
    _check(lib.wc_select_bypass_pairs(_ptr(k), n_tok, hkv, rope_layout, m, _ptr(pairs), _stream(stream)))
    return pairs


def metered_decode_attention_tier_b(desc: CacheDesc, layer: int, q: torch.Tensor, block_table: torch.Tensor,
                                    ctx_lens: torch.Tensor, cache: LayerCache, ws: Workspace, delta_loc: float,
                                    out=None, meter=None, meter_raw=None, meter_b=None, meter_b_raw=None,
                                    stream=None):
    """``wc_metered_decode_attention_tier_b``; returns (out, meter, meter_raw, meter_b, meter_b_raw)."""
    batch, max_pages = block_table.shape
    dev = q.device
    cells = (batch, desc.num_q_heads)
    out = torch.empty(batch, desc.num_q_heads, desc.head_dim, dtype=torch.float32, device=dev) if out is None else out
    meter = torch.empty(cells, dtype=torch.float32, device=dev) if meter is None else meter
    meter_raw = torch.empty(cells, dtype=torch.float32, device=dev) if meter_raw is None else meter_raw
    meter_b = torch.empty(cells, dtype=torch.float32, device=dev) if meter_b is None else meter_b
    meter_b_raw = torch.empty(cells, dtype=torch.float32, device=dev) if meter_b_raw is None else meter_b_raw
    d = desc.c()
    if desc.scheme == SCHEME_DITHER_INT8_G32:
        _decode_g32(d, layer, q, block_table, ctx_lens, cache, ws, delta_loc, out, meter, meter_raw, meter_b,
                    meter_b_raw, stream)
        return out, meter, meter_raw, meter_b, meter_b_raw
    _check(lib.wc_metered_decode_attention_tier_b(
        ctypes.byref(d), layer, _ptr(q), _ptr(block_table), max_pages, _ptr(ctx_lens), batch,
        _ptr(cache.k_codes), _ptr(cache.v_codes), _ptr(cache.k_scale), _ptr(cache.v_scale),
        _ptr(cache.k_witness), float(delta_loc), _ptr(out), _ptr(meter), _ptr(meter_raw), _ptr(meter_b),
        _ptr(meter_b_raw), ws.view.data_ptr(), ws.nbytes, _stream(stream)))
    return out, meter, meter_raw, meter_b, meter_b_raw


def metered_decode_attention_v(desc: CacheDesc, layer: int, q: torch.Tensor, block_table: torch.Tensor,
                               ctx_lens: torch.Tensor, cache: LayerCache, ws: Workspace, out=None, meter=None,
                               meter_raw=None, value_term=None, v_max=None, out_bound=None, stream=None):
    """``wc_metered_decode_attention_v``; returns (out, meter, meter_raw, value_term, v_max, out_bound)."""
    if cache.v_witness is None:
        raise ValueError("the cache holds no value witness (LayerCache.empty(..., value_witness=True))")
    batch, max_pages = block_table.shape
    dev = q.device
    cells = (batch, desc.num_q_heads)
    new = lambda t: torch.empty(cells, dtype=torch.float32, device=dev) if t is None else t
    out = torch.empty(batch, desc.num_q_heads, desc.head_dim, dtype=torch.float32, device=dev) if out is None else out
    meter, meter_raw, value_term, v_max, out_bound = map(new, (meter, meter_raw, value_term, v_max, out_bound))
    d = desc.c()
    _check(lib.wc_metered_decode_attention_v(
        ctypes.byref(d), layer, _ptr(q), _ptr(block_table), max_pages, _ptr(ctx_lens), batch,
        _ptr(cache.k_codes), _ptr(cache.v_codes), _ptr(cache.k_scale), _ptr(cache.v_scale),
        _ptr(cache.k_witness), _ptr(cache.v_witness), _ptr(out), _ptr(meter), _ptr(meter_raw),
        _ptr(value_term), _ptr(v_max), _ptr(out_bound), ws.view.data_ptr(), ws.nbytes, _stream(stream)))
    return out, meter, meter_raw, value_term, v_max, out_bound


def metered_decode_attention_repair(desc: CacheDesc, layer: int, q: torch.Tensor, block_table: torch.Tensor,
                                    ctx_lens: torch.Tensor, cache: LayerCache, ws: Workspace, out=None, meter=None,
                                    meter_raw=None, page_terms=None, softmax_norm=None, stream=None):
    """``wc_metered_decode_attention_repair``; returns (out, meter, meter_raw, page_terms [B,Hq,max_pages,2],
    softmax_norm [B,Hq,2])."""
    batch, max_pages = block_table.shape
    dev = q.device
    cells = (batch, desc.num_q_heads)
    out = torch.empty(batch, desc.num_q_heads, desc.head_dim, dtype=torch.float32, device=dev) if out is None else out
    meter = torch.empty(cells, dtype=torch.float32, device=dev) if meter is None else meter
    meter_raw = torch.empty(cells, dtype=torch.float32, device=dev) if meter_raw is None else meter_raw
    if page_terms is None:
        page_terms = torch.empty(batch, desc.num_q_heads, max_pages, 2, dtype=torch.float32, device=dev)
    if softmax_norm is None:
        softmax_norm = torch.empty(batch, desc.num_q_heads, 2, dtype=torch.float32, device=dev)
    d = desc.c()
    _check(lib.wc_metered_decode_attention_repair(
        ctypes.byref(d), layer, _ptr(q), _ptr(block_table), max_pages, _ptr(ctx_lens), batch,
        _ptr(cache.k_codes), _ptr(cache.v_codes), _ptr(cache.k_scale), _ptr(cache.v_scale),
        _ptr(cache.k_witness), _ptr(out), _ptr(meter), _ptr(meter_raw), _ptr(page_terms), _ptr(softmax_norm),
        ws.view.data_ptr(), ws.nbytes, _stream(stream)))
    return out, meter, meter_raw, page_terms, softmax_norm


def repair_select(page_terms: torch.Tensor, softmax_norm: torch.Tensor, ctx_lens: torch.Tensor, tau: float,
                  keep_q=None, contrib=True, repair_pages=None, n_repair=None, d_after=None, dev_status=None,
                  stream=None):
    """``wc_repair_select``; returns (contrib [B,Hq,max_pages] fp32 or None, repair_pages int32
    [B,Hq,max_pages] (the first n_repair entries of a row are meaningful), n_repair int32 [B,Hq],
    d_after fp32 [B,Hq]).  ``contrib=False`` skips storing the contributions."""
    batch, num_q_heads, max_pages = page_terms.shape[:3]
    dev = page_terms.device
    if contrib is True:
        contrib = torch.zeros(batch, num_q_heads, max_pages, dtype=torch.float32, device=dev)
    elif contrib is False:
        contrib = None
    if repair_pages is None:
        repair_pages = torch.full((batch, num_q_heads, max_pages), -1, dtype=torch.int32, device=dev)
    n_repair = torch.empty(batch, num_q_heads, dtype=torch.int32, device=dev) if n_repair is None else n_repair
    d_after = torch.empty(batch, num_q_heads, dtype=torch.float32, device=dev) if d_after is None else d_after
    _check(lib.wc_repair_select(_ptr(page_terms), _ptr(softmax_norm), _ptr(ctx_lens), batch, num_q_heads, max_pages,
                                _ptr(keep_q), float(tau), _ptr(contrib), _ptr(repair_pages), _ptr(n_repair),
                                _ptr(d_after), _ptr(dev_status), _stream(stream)))
    return contrib, repair_pages, n_repair, d_after


def gate_joint(meter_raw: torch.Tensor, value_term: torch.Tensor, v_max: torch.Tensor, group: int, tau_k: float,
               tau_v: float, keep_q=None, keep_kv=None, n_kept=None, stream=None):
    """``wc_gate_joint``: returns (keep_q uint8 [n], keep_kv uint8 [n/group], n_kept int32 [2])."""
    n = meter_raw.numel()
    dev = meter_raw.device
    keep_q = torch.empty(n, dtype=torch.uint8, device=dev) if keep_q is None else keep_q
    keep_kv = torch.empty(n // group, dtype=torch.uint8, device=dev) if keep_kv is None else keep_kv
    n_kept = torch.empty(2, dtype=torch.int32, device=dev) if n_kept is None else n_kept
    _check(lib.wc_gate_joint(_ptr(meter_raw), _ptr(value_term), _ptr(v_max), n, group, float(tau_k), float(tau_v),
                             _ptr(keep_q), _ptr(keep_kv), _ptr(n_kept), _stream(stream)))
    return keep_q, keep_kv, n_kept


def gate(meter_raw: torch.Tensor, group: int, tau: float, keep_q=None, keep_kv=None, n_kept=None,
         stream=None):
    """``wc_gate``: returns (keep_q uint8 [n], keep_kv uint8 [n/group], n_kept int32 [2])."""
    n = meter_raw.numel()
    dev = meter_raw.device
    keep_q = torch.empty(n, dtype=torch.uint8, device=dev) if keep_q is None else keep_q
    keep_kv = torch.empty(n // group, dtype=torch.uint8, device=dev) if keep_kv is None else keep_kv
    n_kept = torch.empty(2, dtype=torch.int32, device=dev) if n_kept is None else n_kept
    _check(lib.wc_gate(_ptr(meter_raw), n, group, float(tau), _ptr(keep_q), _ptr(keep_kv),
                       _ptr(n_kept), _stream(stream)))
    return keep_q, keep_kv, n_kept


# ---- block-scaled 8-bit cache -------------------------------------------------------------------


class _BlockDesc(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("code", ctypes.c_int32),
                ("rope_layout", ctypes.c_int32), ("rotary_dim", ctypes.c_int32)]


@dataclass(frozen=True)
class BlockDesc:
    """Mirror of ``wc_block_desc``."""
    num_q_heads: int
    num_kv_heads: int
    num_pages: int
    code: int = CODE_INT8
    rope_layout: int = ROPE_HALF
    rotary_dim: int = 128
    head_dim: int = 128
    page_size: int = 16

    @property
    def group(self):
        return self.num_q_heads // self.num_kv_heads

    def __post_init__(self):
        object.__setattr__(self, "_c", _BlockDesc(self.head_dim, self.num_q_heads, self.num_kv_heads, self.page_size,
                                                  self.num_pages, self.code, self.rope_layout, self.rotary_dim))

    def c(self):
        return self._c


_CODE_TYPE = {torch.int8: CODE_INT8, torch.uint8: CODE_E4M3, torch.float8_e4m3fn: CODE_E4M3}


@dataclass(frozen=True)
class BlockCache:
    """One layer's block-scaled cache tensors (layout in ``include/witcert.h``): codes int8, or uint8 or float8_e4m3fn for
    ``CODE_E4M3``; without scales (None) a cache of raw fp8 codes, such as a ``LayerCache``'s of the fp8 scheme."""
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    k_scale: Optional[torch.Tensor]
    v_scale: Optional[torch.Tensor]

    def __post_init__(self):
        blocks = self.k_codes.numel() // (16 * 128)      # pages x KV heads
        for t in (self.k_codes, self.v_codes):
            if t.element_size() != 1 or t.numel() != blocks * 16 * 128 or not t.is_contiguous():
                raise ValueError("the cache's codes must be contiguous bytes [num_pages, num_kv_heads, 16, 128]")
        for t in (self.k_scale, self.v_scale):
            if t is not None and (t.dtype != torch.float32 or t.numel() != blocks or not t.is_contiguous()):
                raise ValueError("the cache's scales must be contiguous float32 [num_pages, num_kv_heads]")
        object.__setattr__(self, "blocks", blocks)
        k, v = (_CODE_TYPE.get(t.dtype) for t in (self.k_codes, self.v_codes))
        object.__setattr__(self, "code", k if k == v else None)

    @staticmethod
    def empty(desc: BlockDesc, device="cuda"):
        shp = (desc.num_pages, desc.num_kv_heads)
        codes = shp + (desc.page_size, desc.head_dim)
        code_t = torch.uint8 if desc.code == CODE_E4M3 else torch.int8
        return BlockCache(torch.zeros(codes, dtype=code_t, device=device), torch.zeros(codes, dtype=code_t, device=device),
                          torch.zeros(shp, dtype=torch.float32, device=device),
                          torch.zeros(shp, dtype=torch.float32, device=device))

    def nbytes(self):
        return sum(t.numel() * t.element_size() for t in (self.k_codes, self.v_codes, self.k_scale, self.v_scale)
                   if t is not None)


class BlockWorkspace:
    """Zero-filled device workspace for the block attention calls of up to ``n_tok`` query tokens."""

    def __init__(self, desc: BlockDesc, batch: int, n_tok: int, max_pages: int, device="cuda"):
        self.nbytes = lib.wc_block_workspace_size(ctypes.byref(desc._c), batch, n_tok, max_pages)
        if self.nbytes == 0:
            raise WitCertError(1, lib.wc_last_error().decode())
        self.buf = torch.zeros(self.nbytes + 256, dtype=torch.uint8, device=device)
        off = (-self.buf.data_ptr()) % 256
        self.view = self.buf[off:off + self.nbytes]

    def ptr(self):
        return ctypes.c_void_p(self.view.data_ptr())


_ACT = {torch.float16: ACT_FP16, torch.bfloat16: ACT_BF16}


# As above, a short call is bound by this marshalling (an append of one token: 5 us on the GPU), so the checks
# are few and in line.
def _rows(t: torch.Tensor, heads: int, act, name: str):
    """Token stride of [n, heads, 128] rows whose heads are contiguous (a view of a packed projection, for
    instance)."""
    n, h, d = t.shape
    if h != heads or d != 128 or _ACT.get(t.dtype) != act or act is None:
        raise ValueError(f"{name} must be float16 or bfloat16 [n, {heads}, 128] like the others, got {t.dtype} {list(t.shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1 or (s1 != 128 and heads > 1):
        raise ValueError(f"{name}'s heads must be contiguous")
    return s0 if n > 1 else heads * 128


def _ints(t: torch.Tensor, n: int, name: str):
    if t.dtype != torch.int32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and hold {n} int32 values, got {t.numel()} {t.dtype}")
    return t.data_ptr()


def _weights(t: Optional[torch.Tensor], name: str):
    """Norm weights of a head."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != 128 or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous float32 [128], got {t.dtype} {list(t.shape)}")
    return t.data_ptr()


def _block_cache(desc: BlockDesc, c: BlockCache):
    if c.blocks != desc.num_pages * desc.num_kv_heads:
        raise ValueError("the cache does not have the descriptor's shape")
    if c.code != desc.code:
        raise ValueError(f"the cache's codes ({c.k_codes.dtype}, {c.v_codes.dtype}) are not the descriptor's (code {desc.code})")
    ks, vs = c.k_scale, c.v_scale
    return (c.k_codes.data_ptr(), c.v_codes.data_ptr(), None if ks is None else ks.data_ptr(),
            None if vs is None else vs.data_ptr())


def block_append(desc: BlockDesc, k: torch.Tensor, v: torch.Tensor, ctx_lens: torch.Tensor, block_table: torch.Tensor,
                 cache: BlockCache, cu_new: Optional[torch.Tensor] = None, cos: Optional[torch.Tensor] = None,
                 sin: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                 q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 dev_status: Optional[torch.Tensor] = None, stream=None, k_norm: Optional[torch.Tensor] = None,
                 q_norm: Optional[torch.Tensor] = None, norm_eps: float = 1e-6):
    """``wc_block_append``: k, v fp16 or bf16 [n_tok, Hkv, 128] (views with a token stride too), the last tokens of
    contexts of ctx_lens int32 [B]; cu_new int32 [B + 1], None: one token per sequence; cos, sin fp32
    [positions, rotary_dim / 2].  Returns the rotated queries (``q_out``) if ``q`` [n_tok, Hq, 128] is given.
    ``wc_block_append_norm`` with k_norm or q_norm, fp32 [128]: the heads' rows are normed before they are rotated."""
    batch, max_pages = block_table.shape
    act, n_tok, hkv = _ACT.get(k.dtype), k.shape[0], desc.num_kv_heads
    ks, vs = _rows(k, hkv, act, "k"), _rows(v, hkv, act, "v")
    if v.shape[0] != n_tok:
        raise ValueError("k and v must have the same number of tokens")
    qp = op = None
    qs = num_positions = 0
    if q is not None:
        qs = _rows(q, desc.num_q_heads, act, "q")
        if q.shape[0] != n_tok:
            raise ValueError("k and q must have the same number of tokens")
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif q_out.shape != q.shape or q_out.dtype != q.dtype or not q_out.is_contiguous():
            raise ValueError("q_out must be contiguous and have q's shape and type")
        qp, op = q.data_ptr(), q_out.data_ptr()
    cp = sp = None
    if cos is not None:
        shape = cos.shape
        if (sin is None or sin.shape != shape or len(shape) != 2 or shape[1] * 2 != desc.rotary_dim or cos.dtype != torch.float32
                or sin.dtype != torch.float32 or not cos.is_contiguous() or not sin.is_contiguous()):
            raise ValueError(f"cos and sin must be contiguous float32 [positions, {desc.rotary_dim // 2}]")
        num_positions, cp, sp = shape[0], cos.data_ptr(), sin.data_ptr()
    call, norms = lib.wc_block_append, ()
    if k_norm is not None or q_norm is not None:
        call, norms = lib.wc_block_append_norm, (_weights(k_norm, "k_norm"), _weights(q_norm, "q_norm"), norm_eps)
    st = call(
        ctypes.byref(desc._c), act, k.data_ptr(), ks, v.data_ptr(), vs, qp, qs, op, n_tok,
        None if cu_new is None else _ints(cu_new, batch + 1, "cu_new"), _ints(block_table, batch * max_pages, "block_table"),
        max_pages, _ints(ctx_lens, batch, "ctx_lens"), batch,
        None if positions is None else _ints(positions, n_tok, "positions"), cp, sp, num_positions, *norms,
        *_block_cache(desc, cache), _ptr(dev_status), _stream(stream))
    if st:
        _check(st)
    return q_out


def _rows_in_out(t: Optional[torch.Tensor], out: Optional[torch.Tensor], act, dtype, out_act, name: str):
    """(pointer and stride of the rows and of their output, heads), the output."""
    if t is None:
        if out is not None:
            raise ValueError(f"{name}_out needs {name}")
        return (None, 0, None, 0, 0), None
    shape = t.shape
    heads = shape[1] if len(shape) == 3 else 0
    stride = _rows(t, heads, act, name)
    if out is None:
        if out_act is None:
            raise ValueError(f"dtype must be float16 or bfloat16, got {dtype}")
        out = t.new_empty(shape, dtype=dtype)
        return (t.data_ptr(), stride, out.data_ptr(), heads * 128, heads), out
    if out.shape != shape:
        raise ValueError(f"{name}_out must have {name}'s shape")
    return (t.data_ptr(), stride, out.data_ptr(), _rows(out, heads, out_act, name + "_out"), heads), out


def qk_norm_rotate(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None,
                   cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None,
                   q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None, norm_eps: float = 1e-6,
                   rope_layout: int = ROPE_HALF, dtype: Optional[torch.dtype] = None, q_out: Optional[torch.Tensor] = None,
                   k_out: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None, stream=None):
    """``wc_qk_norm_rotate``: q [n_tok, Hq, 128] and k [n_tok, Hkv, 128] (fp16 or bf16, views with a token stride too; None: none)
    normed by q_norm, k_norm (fp32 [128]; None: not) and rotated to positions int32 [n_tok] by cos, sin fp32
    [positions, rotary_dim / 2] (None: not).  Returns (q_out, k_out): new dense tensors of ``dtype`` (the inputs' unless given),
    or the ones given, which may be the inputs."""
    if q is None and k is None:
        raise ValueError("q or k must be given")
    x = k if q is None else q
    act, n_tok = _ACT.get(x.dtype), x.shape[0]
    if k is not None and k.shape[0] != n_tok:
        raise ValueError("q and k must have the same number of tokens")
    if dtype is None:
        dtype = x.dtype if q_out is k_out is None else (k_out if q_out is None else q_out).dtype
    out_act = _ACT.get(dtype)
    q_rows, q_out = _rows_in_out(q, q_out, act, dtype, out_act, "q")
    k_rows, k_out = _rows_in_out(k, k_out, act, dtype, out_act, "k")
    rotary_dim, tables = 0, (None, None, None, 0)
    if cos is not None:
        shape = cos.shape
        if (sin is None or sin.shape != shape or len(shape) != 2 or cos.dtype != torch.float32 or sin.dtype != torch.float32
                or not cos.is_contiguous() or not sin.is_contiguous()):
            raise ValueError("cos and sin must be contiguous float32 [positions, rotary_dim / 2]")
        if positions is None:
            raise ValueError("cos and sin need positions")
        rotary_dim, tables = 2 * shape[1], (_ints(positions, n_tok, "positions"), cos.data_ptr(), sin.data_ptr(), shape[0])
    elif sin is not None or positions is not None:
        raise ValueError("sin and positions need cos")
    st = lib.wc_qk_norm_rotate(act, out_act, *q_rows, *k_rows, n_tok, _weights(q_norm, "q_norm"), _weights(k_norm, "k_norm"), norm_eps, rope_layout,
                               rotary_dim, *tables, _ptr(dev_status), _stream(stream))
    if st:
        _check(st)
    return q_out, k_out


def _attention_out(desc, q, out, lse, return_lse):
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise ValueError("out must be contiguous and have q's shape and type")
    if lse is None:
        if return_lse:
            lse = torch.empty(q.shape[0], desc.num_q_heads, dtype=torch.float32, device=q.device)
    elif lse.dtype != torch.float32 or lse.numel() != q.shape[0] * desc.num_q_heads or not lse.is_contiguous():
        raise ValueError("lse must be contiguous float32 [n_tok, num_q_heads]")
    return out, lse


_SCALE_128 = 1.0 / math.sqrt(128)


def _window(window, sinks):
    """As int32 values that mean the same (the library refuses those below its limits)."""
    return max(0, min(window, 0x7FFFFFFF)), max(-1, min(sinks, 0x7FFFFFFF))


def block_decode_attention(desc: BlockDesc, q: torch.Tensor, block_table: torch.Tensor, ctx_lens: torch.Tensor,
                           cache: BlockCache, ws: BlockWorkspace, softmax_scale: Optional[float] = None, out=None,
                           lse=None, return_lse=False, stream=None, window: Optional[int] = None, sinks: int = 0):
    """``wc_block_decode_attention``: q [B, Hq, 128], one token per sequence; softmax_scale 1 / sqrt(128) unless given.
    ``wc_block_decode_attention_window`` with a ``window``: each token sees the last ``window`` positions of its context and the
    first ``sinks``.  Returns out, or (out, lse) with ``return_lse`` or an ``lse`` to fill."""
    batch, max_pages = block_table.shape
    act = _ACT.get(q.dtype)
    qs = _rows(q, desc.num_q_heads, act, "q")
    if q.shape[0] != batch:
        raise ValueError(f"q must have one token per sequence ({batch}), got {q.shape[0]}")
    out, lse = _attention_out(desc, q, out, lse, return_lse)
    call, part = lib.wc_block_decode_attention, ()
    if window is not None:
        call, part = lib.wc_block_decode_attention_window, _window(window, sinks)
    elif sinks:
        raise ValueError("sinks need a window")
    st = call(
        ctypes.byref(desc._c), act, q.data_ptr(), qs, _ints(block_table, batch * max_pages, "block_table"), max_pages,
        _ints(ctx_lens, batch, "ctx_lens"), batch, *_block_cache(desc, cache),
        _SCALE_128 if softmax_scale is None else softmax_scale, *part, out.data_ptr(), None if lse is None else lse.data_ptr(),
        ws.view.data_ptr(), ws.nbytes, _stream(stream))
    if st:
        _check(st)
    return out if lse is None else (out, lse)


def block_extend_attention(desc: BlockDesc, q: torch.Tensor, cu_q: torch.Tensor, block_table: torch.Tensor,
                           ctx_lens: torch.Tensor, cache: BlockCache, ws: BlockWorkspace,
                           softmax_scale: Optional[float] = None, causal=True, out=None, lse=None, return_lse=False,
                           stream=None, window: Optional[int] = None, sinks: int = 0):
    """``wc_block_extend_attention``: q [n_tok, Hq, 128], rows cu_q[b] .. cu_q[b + 1] - 1 the last tokens of sequence
    b's context.  ``wc_block_extend_attention_window`` with a ``window`` (causal only): each row sees the last ``window`` positions
    up to its own and the first ``sinks``.  Returns out, or (out, lse) with ``return_lse`` or an ``lse`` to fill."""
    batch, max_pages = block_table.shape
    act = _ACT.get(q.dtype)
    qs = _rows(q, desc.num_q_heads, act, "q")
    out, lse = _attention_out(desc, q, out, lse, return_lse)
    call, part = lib.wc_block_extend_attention, (int(causal),)
    if window is not None:
        if not causal:
            raise ValueError("a window is causal")
        call, part = lib.wc_block_extend_attention_window, _window(window, sinks)
    elif sinks:
        raise ValueError("sinks need a window")
    st = call(
        ctypes.byref(desc._c), act, q.data_ptr(), qs, q.shape[0], _ints(cu_q, batch + 1, "cu_q"),
        _ints(block_table, batch * max_pages, "block_table"), max_pages, _ints(ctx_lens, batch, "ctx_lens"), batch,
        *_block_cache(desc, cache), _SCALE_128 if softmax_scale is None else softmax_scale, *part,
        out.data_ptr(), None if lse is None else lse.data_ptr(), ws.view.data_ptr(), ws.nbytes, _stream(stream))
    if st:
        _check(st)
    return out if lse is None else (out, lse)


def read_status(ws_or_word, stream=None) -> int:
    """Synchronising read-and-clear of the device status word; returns the bits."""
    if isinstance(ws_or_word, (Workspace, BlockWorkspace)):
        p, is_word = ws_or_word.ptr(), 0
    else:
        p, is_word = _ptr(ws_or_word), 1
    bits = ctypes.c_uint32(0)
    st = lib.wc_read_status(p, is_word, ctypes.byref(bits), _stream(stream))
    if st not in (0, 5):
        _check(st)
    return bits.value


def version():
    v = lib.wc_version()
    return (v >> 16, v & 0xFFFF)
