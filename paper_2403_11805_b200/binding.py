"""ctypes binding of libllms.so: the same names as include/llms.h, argument marshalling only.

Tensors may be torch tensors (device or pinned host), numpy arrays (host) or raw integer addresses;
nothing here computes anything.  A missing library is an error: there is no fallback path.
"""
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# LLMS_LIBRARY names another build of the library to load instead of the in-tree one (the checked build's test uses it)
LIB_PATH = os.environ.get("LLMS_LIBRARY") or os.path.join(_HERE, "libllms.so")
_lib = None

OK = 0
ERR_INVALID_ARG, ERR_BAD_BITS, ERR_MISALIGNED, ERR_BUF_TOO_SMALL = -1, -2, -3, -4
ERR_CUDA, ERR_TIMEOUT, ERR_CORRUPT, ERR_UNSUPPORTED = -5, -6, -7, -8


class LlmsError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        msg = lib().llms_strerror(status).decode()
        if status == ERR_CUDA:
            msg += ": " + lib().llms_last_cuda_error().decode()
        super().__init__(f"{what}: {msg} ({status})")


class KVDesc(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32), ("head_dim", C.c_int32),
        ("n_tokens", C.c_int32), ("chunk_len", C.c_int32), ("group_size", C.c_int32), ("quant_mode", C.c_int32),
        ("stride_l", C.c_int64), ("stride_s", C.c_int64), ("stride_h", C.c_int64),
    ]


META_DTYPE = np.dtype([("chunk_id", "<u4"), ("bits", "<u4"), ("offset", "<u8"), ("nbytes", "<u8"),
                       ("n_groups", "<u4"), ("checksum", "<u4")])
STATE_DTYPE = np.dtype([("ctx_id", "<u4"), ("chunk_id", "<u4"), ("bits", "<u4"), ("resident", "<u4"),
                        ("locked", "<u4"), ("pad_", "<u4"), ("last_access_step", "<u8")])

_SIGNATURES = {
    "llms_strerror": (C.c_char_p, [C.c_int]),
    "llms_last_cuda_error": (C.c_char_p, []),
    "llms_record_layout": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]),
    "llms_record_bytes": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p]),
    "llms_compressed_size": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]),
    "llms_codec_workspace_bytes": (C.c_int, [C.c_int, C.c_void_p]),
    "llms_compress_chunks": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                       C.c_uint64, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]),
    "llms_compress_chunks_static": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                              C.c_uint64, C.c_void_p, C.c_void_p]),
    "llms_decompress_chunks": (C.c_int, [C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                         C.c_void_p, C.c_uint64, C.c_void_p]),
    "llms_decompress_chunks_ordered": (C.c_int, [C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p, C.c_int,
                                                 C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]),
    "llms_codec_corrupt_count": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "llms_tolerance_workspace_bytes": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p]),
    "llms_chunk_tolerance": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                                       C.c_uint64, C.c_void_p]),
    "llms_chunk_tolerance_from_probs": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                                                  C.c_uint64, C.c_void_p]),
    "llms_assign_bits": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]),
    "llms_assign_levels": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "llms_optimize_thresholds": (C.c_int, [C.c_void_p, C.c_int, C.c_float, C.c_void_p]),
    "llms_optimize_thresholds_levels": (C.c_int, [C.c_void_p, C.c_int, C.c_float, C.c_void_p, C.c_void_p]),
    "llms_compress_context": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p, C.c_uint64,
                                        C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p]),
    "llms_decode_workspace_bytes": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p]),
    "llms_decode_attention": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                        C.c_int64, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_float,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_uint64,
                                        C.c_void_p]),
    "llms_evict_tokens": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int, C.c_void_p, C.c_int,
                                    C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p]),
    "llms_lctru_order": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p]),
    "llms_swap_out": (C.c_int, [C.c_void_p, C.c_uint64, C.c_void_p, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p,
                                C.c_void_p, C.c_void_p, C.c_void_p]),
    "llms_swap_in": (C.c_int, [C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_uint64,
                               C.c_void_p, C.c_void_p, C.c_void_p]),
    "llms_wait": (C.c_int, [C.c_void_p, C.c_uint32]),
    "llms_stream_probe": (C.c_int, [C.c_void_p, C.c_uint64, C.c_void_p, C.c_uint64, C.c_uint64, C.c_int, C.c_int, C.c_void_p]),
    "llms_debug_bounds": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "llms_stream_probe_split": (C.c_int, [C.c_void_p, C.c_uint64, C.c_void_p, C.c_uint64, C.c_uint64, C.c_int, C.c_int, C.c_int,
                                          C.c_void_p]),
}


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2403_11805_b200.build` "
                               "(there is no CPU or PyTorch fallback)")
        _lib = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(_lib, name)
            fn.restype, fn.argtypes = res, args
    return _lib


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        assert x.flags.c_contiguous
        return x.ctypes.data
    if hasattr(x, "data_ptr"):          # torch tensor
        assert x.is_contiguous()
        return x.data_ptr()
    if isinstance(x, C.Structure):
        return C.addressof(x)
    raise TypeError(type(x))


def _nbytes(x):
    if isinstance(x, np.ndarray):
        return x.nbytes
    return x.numel() * x.element_size()


def _stream(s):
    if s is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _event(e):
    if e is None:
        return None
    if isinstance(e, int):
        return e
    h = e.cuda_event
    return h.value if hasattr(h, "value") else int(h)


def _check(rc, what):
    if rc < 0:
        raise LlmsError(rc, what)
    return rc


def make_desc(n_layers, n_kv_heads, n_q_heads, head_dim, n_tokens, chunk_len, group_size, quant_mode=0):
    """Descriptor of a contiguous kv[l][s][h][t][c] tensor."""
    d = KVDesc()
    d.n_layers, d.n_kv_heads, d.n_q_heads, d.head_dim = n_layers, n_kv_heads, n_q_heads, head_dim
    d.n_tokens, d.chunk_len, d.group_size, d.quant_mode = n_tokens, chunk_len, group_size, quant_mode
    d.stride_h = n_tokens * head_dim
    d.stride_s = n_kv_heads * d.stride_h
    d.stride_l = 2 * d.stride_s
    return d


def desc_of(shape, quant_mode=0, n_tokens=None):
    """Descriptor for a synth.KVShape (n_tokens overrides the token count, e.g. for a slot pool)."""
    return make_desc(shape.n_layers, shape.n_kv_heads, shape.n_q_heads, shape.head_dim,
                     shape.n_tokens if n_tokens is None else n_tokens, shape.chunk_len, shape.group_size, quant_mode)


def new_meta(n, pinned=False):
    """n zeroed llms_chunk_meta entries as a numpy structured array (optionally over pinned memory)."""
    if not pinned:
        return np.zeros(n, dtype=META_DTYPE)
    import torch
    t = torch.zeros(max(n, 1) * META_DTYPE.itemsize, dtype=torch.uint8).pin_memory()
    return t.numpy()[:n * META_DTYPE.itemsize].view(META_DTYPE)   # the view keeps the pinned storage alive


def new_pinned(n, dtype=np.uint8):
    """n zeroed elements as a numpy array over page-locked memory (e.g. the level array of compress_context)."""
    import torch
    dt = np.dtype(dtype)
    t = torch.zeros(max(n, 1) * dt.itemsize, dtype=torch.uint8).pin_memory()
    return t.numpy()[:n * dt.itemsize].view(dt)                  # the view keeps the pinned storage alive


def new_event(stream=None):
    """A created cudaEvent_t wrapped by torch (recorded once so that the handle exists)."""
    import torch
    ev = torch.cuda.Event()
    ev.record(torch.cuda.current_stream() if stream is None else stream)
    return ev


# ----------------------------------------------------------------------------- sizes

def record_layout(desc, bits):
    co, nb = C.c_uint64(), C.c_uint64()
    _check(lib().llms_record_layout(C.addressof(desc), int(bits), C.addressof(co), C.addressof(nb)), "llms_record_layout")
    return co.value, nb.value


def record_bytes(desc, bits):
    nb = C.c_uint64()
    _check(lib().llms_record_bytes(C.addressof(desc), int(bits), C.addressof(nb)), "llms_record_bytes")
    return nb.value


def compressed_size(desc, bits):
    bits = np.ascontiguousarray(bits, dtype=np.uint8)
    nb = C.c_uint64()
    _check(lib().llms_compressed_size(C.addressof(desc), _ptr(bits), len(bits), C.addressof(nb)), "llms_compressed_size")
    return nb.value


def codec_workspace_bytes(n):
    nb = C.c_uint64()
    _check(lib().llms_codec_workspace_bytes(int(n), C.addressof(nb)), "llms_codec_workspace_bytes")
    return nb.value


def tolerance_workspace_bytes(desc, W):
    nb = C.c_uint64()
    _check(lib().llms_tolerance_workspace_bytes(C.addressof(desc), int(W), C.addressof(nb)), "llms_tolerance_workspace_bytes")
    return nb.value


# ----------------------------------------------------------------------------- codec

def codec_launches(desc, bits):
    """Kernels one compress or decompress call launches.  Groups of channels of a token: one codec kernel for the whole
    call (the bit-widths are phases of it, and its last CTA stores or checks the sums; a pageable meta array gets the
    sums by a copy).  Channel-wise mode: one kernel per bit-width present and one small kernel for the sums."""
    return len(set(int(b) for b in bits)) + 1 if desc.quant_mode == 1 else 1


def compress_chunks(desc, kv, chunk_ids, bits, out_buf, meta, workspace, stream=None, out_bytes=None, workspace_bytes=None):
    chunk_ids = np.ascontiguousarray(chunk_ids, dtype=np.uint32)
    bits = np.ascontiguousarray(bits, dtype=np.uint8)
    assert len(chunk_ids) == len(bits) and len(meta) >= len(bits)
    _check(lib().llms_compress_chunks(
        C.addressof(desc), _ptr(kv), _ptr(chunk_ids), _ptr(bits), len(bits), _ptr(out_buf),
        _nbytes(out_buf) if out_bytes is None else out_bytes, _ptr(meta), _ptr(workspace),
        _nbytes(workspace) if workspace_bytes is None else workspace_bytes, _stream(stream)), "llms_compress_chunks")


STATIC_MAX_CHUNKS = 1024


def compress_chunks_static(desc, kv, chunk_ids, bits, out_buf, meta, stream=None, out_bytes=None):
    """llms_compress_chunks_static: same as compress_chunks, scratch built into the library (<= 1024 chunks)."""
    chunk_ids = np.ascontiguousarray(chunk_ids, dtype=np.uint32)
    bits = np.ascontiguousarray(bits, dtype=np.uint8)
    assert len(chunk_ids) == len(bits) and len(meta) >= len(bits)
    _check(lib().llms_compress_chunks_static(
        C.addressof(desc), _ptr(kv), _ptr(chunk_ids), _ptr(bits), len(bits), _ptr(out_buf),
        _nbytes(out_buf) if out_bytes is None else out_bytes, _ptr(meta), _stream(stream)), "llms_compress_chunks_static")


def decompress_chunks(desc, buf, meta, dst_chunk_ids, kv_out, workspace, stream=None, n=None, workspace_bytes=None,
                      buf_bytes=None):
    ids = None if dst_chunk_ids is None else np.ascontiguousarray(dst_chunk_ids, dtype=np.uint32)
    n = len(meta) if n is None else n
    _check(lib().llms_decompress_chunks(
        C.addressof(desc), _ptr(buf), _nbytes(buf) if buf_bytes is None else buf_bytes, _ptr(meta), _ptr(ids), n, _ptr(kv_out), _ptr(workspace),
        _nbytes(workspace) if workspace_bytes is None else workspace_bytes, _stream(stream)), "llms_decompress_chunks")


def decompress_chunks_ordered(desc, buf, meta, dst_chunk_ids, kv_out, workspace, stream=None, n=None, workspace_bytes=None,
                              buf_bytes=None):
    """llms_decompress_chunks_ordered: meta pinned; its checksums are read by the device in stream order."""
    ids = None if dst_chunk_ids is None else np.ascontiguousarray(dst_chunk_ids, dtype=np.uint32)
    n = len(meta) if n is None else n
    _check(lib().llms_decompress_chunks_ordered(
        C.addressof(desc), _ptr(buf), _nbytes(buf) if buf_bytes is None else buf_bytes, _ptr(meta), _ptr(ids), n, _ptr(kv_out), _ptr(workspace),
        _nbytes(workspace) if workspace_bytes is None else workspace_bytes, _stream(stream)), "llms_decompress_chunks_ordered")


def codec_corrupt_count(workspace, stream=None):
    """Synchronises the stream; returns the number of records whose checksum did not match."""
    bad = C.c_uint32()
    rc = lib().llms_codec_corrupt_count(_ptr(workspace), C.addressof(bad), _stream(stream))
    if rc not in (OK, ERR_CORRUPT):
        _check(rc, "llms_codec_corrupt_count")
    return bad.value


# ----------------------------------------------------------------------------- tolerance score

def chunk_tolerance(desc, kv, q_win, W, scores, workspace, stream=None):
    _check(lib().llms_chunk_tolerance(C.addressof(desc), _ptr(kv), _ptr(q_win), int(W), _ptr(scores), _ptr(workspace),
                                      _nbytes(workspace), _stream(stream)), "llms_chunk_tolerance")


def chunk_tolerance_from_probs(desc, probs, W, scores, workspace, stream=None):
    _check(lib().llms_chunk_tolerance_from_probs(C.addressof(desc), _ptr(probs), int(W), _ptr(scores), _ptr(workspace),
                                                 _nbytes(workspace), _stream(stream)), "llms_chunk_tolerance_from_probs")


# ----------------------------------------------------------------------------- policy (host)

def assign_bits(scores, frac):
    s = np.ascontiguousarray(scores, dtype=np.float32)
    f = np.asarray(frac, dtype=np.float32)
    bits = np.empty(s.size, dtype=np.uint8)
    order = np.empty(s.size, dtype=np.uint32)
    _check(lib().llms_assign_bits(_ptr(s), int(s.size), _ptr(f), _ptr(bits), _ptr(order)), "llms_assign_bits")
    return bits, order


def assign_levels(scores, frac, levels):
    """Eq. 2 for a level set {top, middle, low}, e.g. (4, 2, 1)."""
    s = np.ascontiguousarray(scores, dtype=np.float32)
    f = np.asarray(frac, dtype=np.float32)
    lv = np.asarray(levels, dtype=np.uint8)
    assert f.size == 3 and lv.size == 3
    bits = np.empty(s.size, dtype=np.uint8)
    order = np.empty(s.size, dtype=np.uint32)
    _check(lib().llms_assign_levels(_ptr(s), int(s.size), _ptr(f), _ptr(lv), _ptr(bits), _ptr(order)), "llms_assign_levels")
    return bits, order


def level_counts(n, frac, levels=(8, 4, 2)):
    """How many of n chunks each level gets under llms_assign_levels (the counts depend on n and frac alone):
    asked of the library itself, on n distinct scores."""
    bits, _ = assign_levels(np.arange(n, 0, -1, dtype=np.float32), frac, levels)
    return tuple(int((bits == b).sum()) for b in levels)


def optimize_thresholds(scores, ratio_global):
    s = np.ascontiguousarray(scores, dtype=np.float32)
    frac = np.zeros(3, dtype=np.float32)
    _check(lib().llms_optimize_thresholds(_ptr(s), int(s.size), float(ratio_global), _ptr(frac)), "llms_optimize_thresholds")
    return frac


def optimize_thresholds_levels(scores, ratio_global, levels):
    s = np.ascontiguousarray(scores, dtype=np.float32)
    lv = np.asarray(levels, dtype=np.uint8)
    assert lv.size == 3
    frac = np.zeros(3, dtype=np.float32)
    _check(lib().llms_optimize_thresholds_levels(_ptr(s), int(s.size), float(ratio_global), _ptr(lv), _ptr(frac)),
           "llms_optimize_thresholds_levels")
    return frac


def lctru_order(table):
    t = np.ascontiguousarray(table, dtype=STATE_DTYPE)
    order = np.empty(max(len(t), 1), dtype=np.uint32)
    m = _check(lib().llms_lctru_order(_ptr(t), len(t), _ptr(order)), "llms_lctru_order")
    return order[:m].copy()


# ----------------------------------------------------------------------------- a whole context

def compress_context(desc, kv, q_win, W, frac, levels, scores_dev, scores_host, bits_out, out_buf, meta,
                     tolerance_workspace, codec_workspace, after_scores=None, stream=None):
    """llms_compress_context: scores, levels and records of every chunk in one call.
    frac: float32[3], levels: uint8[3], bits_out: uint8[n_chunks] numpy arrays; scores_host: fp32 tensor.
    With scores_host, bits_out and meta all in page-locked memory nothing synchronises: the three arrays are valid
    once after_scores has completed.  Otherwise the stream is synchronised once inside the call."""
    assert frac.dtype == np.float32 and levels.dtype == np.uint8 and bits_out.dtype == np.uint8
    _check(lib().llms_compress_context(
        C.addressof(desc), _ptr(kv), _ptr(q_win), int(W), _ptr(frac), _ptr(levels), _ptr(scores_dev), _ptr(scores_host),
        _ptr(bits_out), _ptr(out_buf), _nbytes(out_buf), _ptr(meta), _ptr(tolerance_workspace), _nbytes(tolerance_workspace),
        _ptr(codec_workspace), _nbytes(codec_workspace), _event(after_scores), _stream(stream)), "llms_compress_context")


# ----------------------------------------------------------------------------- the resident cache in use

DTYPE_F16, DTYPE_BF16 = 0, 1


def _refuse(what):
    raise LlmsError(ERR_INVALID_ARG, what)


def _dtype_of(x):
    name = str(x.dtype)
    if name == "torch.float16":
        return DTYPE_F16
    if name == "torch.bfloat16":
        return DTYPE_BF16
    raise LlmsError(ERR_UNSUPPORTED, f"a cache of {name} (float16 and bfloat16 are taken)")


def _on_device(what, *tensors):
    """The library works on the current device: a tensor of another one, or of the host, is refused."""
    import torch
    here = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            _refuse(f"{what}: a tensor on {t.device} in a call on cuda:{here}")


def _rows_of(x, n, width, dtype, what):
    """(address, elements from one sequence to the next) of a [n, heads, head_dim] tensor: a sequence's heads lie side by side,
    the sequences any number of elements apart (q, k and v may be views of one projection's output)."""
    if x.dim() != 3 or x.shape[0] != n or x.shape[1] * x.shape[2] != width or x.dtype != dtype:
        _refuse(f"{what}: {tuple(x.shape)} of {x.dtype}, [{n}, heads, head_dim] with {width} elements of {dtype} each wanted")
    st = x.stride()
    if (x.shape[2] > 1 and st[2] != 1) or (x.shape[1] > 1 and st[1] != x.shape[2]):
        _refuse(f"{what}: a sequence's heads must lie side by side")
    return x.data_ptr(), (st[0] if n > 1 else width)


def _whole(x, shape, name, what):
    """Address of a contiguous tensor that must have this shape and type."""
    if tuple(x.shape) != shape or not str(x.dtype).endswith(name) or not x.is_contiguous():
        _refuse(f"{what}: {tuple(x.shape)} of {x.dtype}, a contiguous {shape} of {name} wanted")
    return x.data_ptr()


def _batch(chunk_table, lens, what):
    """(address, row stride) of an int32 chunk table [n_seqs, chunks], address of the lengths."""
    n = lens.shape[0]
    if chunk_table.dim() != 2 or chunk_table.shape[0] != n or not str(chunk_table.dtype).endswith(".int32") or not (
            chunk_table.shape[1] == 1 or chunk_table.stride(1) == 1):
        _refuse(f"{what}: chunk_table must be int32 [n_seqs, chunks] with its rows' entries side by side")
    return chunk_table.data_ptr(), (chunk_table.stride(0) if n > 1 else chunk_table.shape[1]), _whole(lens, (n,), ".int32", f"{what}: lens")


def decode_workspace_bytes(desc, n_seqs, max_len, with_mass=False):
    nb = C.c_uint64()
    _check(lib().llms_decode_workspace_bytes(C.addressof(desc), int(n_seqs), int(max_len), int(with_mass), C.addressof(nb)),
           "llms_decode_workspace_bytes")
    return nb.value


def decode_attention(desc, layer, kv, q, chunk_table, lens, max_len, out, workspace, k_new=None, v_new=None, window=0, scale=None,
                     lse=None, mass_in=None, mass_out=None, stream=None):
    """llms_decode_attention: one new token per sequence attends to its cached tokens, in one layer of the pool.
    kv: the pool (fp16 or bf16, device); q, out: [n_seqs, n_q_heads, head_dim]; k_new, v_new: [n_seqs, n_kv_heads, head_dim],
    stored at position lens - 1; chunk_table: int32 [n_seqs, chunks]; lens: int32 [n_seqs]; scale: 1/sqrt(head_dim) if None;
    lse: fp32 [n_seqs, n_q_heads]; mass_in, mass_out: fp32 [n_seqs, n_kv_heads, >= max_len]."""
    what = "llms_decode_attention"
    n, d = lens.shape[0], desc.head_dim
    _on_device(what, kv, q, chunk_table, lens, out, workspace, k_new, v_new, lse, mass_in, mass_out)
    dtype = _dtype_of(kv)
    q_ptr, q_stride = _rows_of(q, n, desc.n_q_heads * d, kv.dtype, f"{what}: q")
    k_ptr = v_ptr = None
    new_stride = 0
    if k_new is not None or v_new is not None:
        if k_new is None or v_new is None:
            _refuse(f"{what}: k_new and v_new come together")
        k_ptr, new_stride = _rows_of(k_new, n, desc.n_kv_heads * d, kv.dtype, f"{what}: k_new")
        v_ptr, v_stride = _rows_of(v_new, n, desc.n_kv_heads * d, kv.dtype, f"{what}: v_new")
        if v_stride != new_stride:
            _refuse(f"{what}: k_new and v_new must have the same stride")
    table_ptr, table_stride, lens_ptr = _batch(chunk_table, lens, what)
    if table_stride < chunk_table.shape[1] or chunk_table.shape[1] * desc.chunk_len < max_len:
        _refuse(f"{what}: max_len {max_len} is more than {chunk_table.shape[1]} chunks of a table row hold")
    if out.dtype != kv.dtype or out.numel() != n * desc.n_q_heads * d or not out.is_contiguous():
        _refuse(f"{what}: out must be a contiguous [{n}, {desc.n_q_heads}, {d}] of {kv.dtype}")
    in_ptr = out_mass = None
    mass_stride = 0
    if mass_out is not None:
        mass_stride = mass_out.shape[-1]
        out_mass = _whole(mass_out, (n, desc.n_kv_heads, mass_stride), ".float32", f"{what}: mass_out")
    if mass_in is not None:
        in_ptr = _whole(mass_in, (n, desc.n_kv_heads, mass_stride), ".float32", f"{what}: mass_in")
    _check(lib().llms_decode_attention(
        C.addressof(desc), dtype, layer, kv.data_ptr(), q_ptr, q_stride, k_ptr, v_ptr, new_stride, table_ptr, table_stride, lens_ptr,
        n, max_len, window, d ** -0.5 if scale is None else scale, out.data_ptr(),
        None if lse is None else _whole(lse, (n, desc.n_q_heads), ".float32", f"{what}: lse"), in_ptr, out_mass, mass_stride,
        workspace.data_ptr(), _nbytes(workspace), _stream(stream)), what)


def evict_tokens(desc, kv, mass, chunk_table, lens, max_len, budget, recent, kept, new_lens, mass_out=None, dst_table=None,
                 stream=None):
    """llms_evict_tokens: per layer and KV head the `budget` heaviest tokens stay (the last `recent` in any case).
    mass, mass_out: fp32 [n_layers, n_seqs, n_kv_heads, >= max_len] (mass_out None: in place); kept: int32 [n_layers, n_seqs,
    n_kv_heads, budget]; new_lens: int32 [n_seqs]; dst_table: int32 [n_seqs, chunks] or None (rows stay in their chunks)."""
    what = "llms_evict_tokens"
    n = lens.shape[0]
    _on_device(what, kv, mass, chunk_table, lens, kept, new_lens, mass_out, dst_table)
    if kv.element_size() != 2:
        _refuse(f"{what}: elements of 2 bytes are moved, not {kv.dtype}")
    shape = (desc.n_layers, n, desc.n_kv_heads, mass.shape[-1])
    table_ptr, table_stride, lens_ptr = _batch(chunk_table, lens, what)
    if table_stride < chunk_table.shape[1] or chunk_table.shape[1] * desc.chunk_len < max_len:
        _refuse(f"{what}: max_len {max_len} is more than {chunk_table.shape[1]} chunks of a table row hold")
    dst_ptr, dst_stride = None, 0
    if dst_table is not None:
        dst_ptr, dst_stride, _ = _batch(dst_table, lens, f"{what}: dst_table")
        if dst_stride < dst_table.shape[1] or dst_table.shape[1] * desc.chunk_len < min(budget, max_len):
            _refuse(f"{what}: {dst_table.shape[1]} chunks of a dst_table row do not hold {min(budget, max_len)} tokens")
    mass_ptr = _whole(mass, shape, ".float32", f"{what}: mass")
    _check(lib().llms_evict_tokens(
        C.addressof(desc), kv.data_ptr(), mass_ptr, shape[3], table_ptr, table_stride, lens_ptr, n, max_len, budget, recent,
        dst_ptr, dst_stride, mass_ptr if mass_out is None else _whole(mass_out, shape, ".float32", f"{what}: mass_out"),
        _whole(kept, shape[:3] + (budget,), ".int32", f"{what}: kept"), _whole(new_lens, (n,), ".int32", f"{what}: new_lens"),
        _stream(stream)), what)


# ----------------------------------------------------------------------------- swap

def swap_out(dev_buf, meta, pinned_dst, host_offsets=None, side_stream=None, after=None, done=None, n=None,
             dev_bytes=None, host_bytes=None):
    ho = None if host_offsets is None else np.ascontiguousarray(host_offsets, dtype=np.uint64)
    _check(lib().llms_swap_out(_ptr(dev_buf), _nbytes(dev_buf) if dev_bytes is None else dev_bytes, _ptr(meta),
                               len(meta) if n is None else n, _ptr(pinned_dst),
                               _nbytes(pinned_dst) if host_bytes is None else host_bytes, _ptr(ho),
                               _stream(side_stream), _event(after), _event(done)), "llms_swap_out")


def swap_in(pinned_src, meta, dev_buf, host_offsets=None, side_stream=None, after=None, done=None, n=None,
            dev_bytes=None, host_bytes=None):
    ho = None if host_offsets is None else np.ascontiguousarray(host_offsets, dtype=np.uint64)
    _check(lib().llms_swap_in(_ptr(pinned_src), _nbytes(pinned_src) if host_bytes is None else host_bytes, _ptr(ho),
                              _ptr(meta), len(meta) if n is None else n, _ptr(dev_buf),
                              _nbytes(dev_buf) if dev_bytes is None else dev_bytes,
                              _stream(side_stream), _event(after), _event(done)), "llms_swap_in")


def wait(event, timeout_ms=10000):
    _check(lib().llms_wait(_event(event), int(timeout_ms)), "llms_wait")


# ----------------------------------------------------------------------------- checked build

def debug_bounds():
    """llms_debug_bounds: (compiled_in, violations, first_address) of the loaded library."""
    c, v, a = C.c_uint32(0), C.c_uint32(0), C.c_uint64(0)
    _check(lib().llms_debug_bounds(C.byref(c), C.byref(v), C.byref(a)), "llms_debug_bounds")
    return int(c.value), int(v.value), int(a.value)


# ----------------------------------------------------------------------------- measurement aid

def stream_probe(src, dst, iters, read_kib, write_kib, stream=None, split=None):
    """llms_stream_probe: a plain stream of the given read:write mix (KiB per warp iteration) over src / dst.
    split (llms_stream_probe_split): 0 a warp per iteration, 1 resident CTAs with a fixed split, 2 resident CTAs that
    draw their iterations from counters."""
    if split is None:
        _check(lib().llms_stream_probe(_ptr(src), _nbytes(src), _ptr(dst), _nbytes(dst), int(iters), int(read_kib),
                                       int(write_kib), _stream(stream)), "llms_stream_probe")
    else:
        _check(lib().llms_stream_probe_split(_ptr(src), _nbytes(src), _ptr(dst), _nbytes(dst), int(iters), int(read_kib),
                                             int(write_kib), int(split), _stream(stream)), "llms_stream_probe_split")
