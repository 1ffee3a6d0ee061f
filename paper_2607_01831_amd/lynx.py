"""Python binding of liblynx.so (include/lynx.h): argument marshalling only.

Every function has the name and argument order of its C entry point.  Tensors
are torch CUDA tensors; their device pointers and the current HIP stream are
passed through ctypes.  Nothing here computes any part of the method: if the
library is missing the binding raises instead of falling back to anything.
"""
from __future__ import annotations

import ctypes
import functools
import struct
import warnings
from dataclasses import dataclass
from pathlib import Path

import torch

LIBRARY = Path(__file__).resolve().parent / "liblynx.so"
ARGS = LIBRARY.with_name("_args.so")  # host code of the binding

LYNX_OK, LYNX_EINVAL, LYNX_ENOTSUP, LYNX_EWORKSPACE, LYNX_EHIP = 0, -1, -2, -3, -4
HEAD_DIM = 128
K_GROUP = 128
MAX_DRAFTS = 64


class LynxError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {lynx_strerror(status)} ({status})")


class lynx_layout(ctypes.Structure):
    _fields_ = [("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("k_group_tokens", ctypes.c_int32), ("block_tokens", ctypes.c_int32),
                ("max_blocks_per_seq", ctypes.c_int32), ("num_blocks", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32)]


class lynx_meta(ctypes.Structure):
    _fields_ = [("k_scale", ctypes.c_void_p), ("k_zero", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("v_zero", ctypes.c_void_p)]


_lib = None


_HMETA_NAMES = ("k_gmin", "k_gscale", "k_mu", "k_sigma", "v_gmin", "v_gscale", "v_mu", "v_sigma")


class lynx_hmeta(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in _HMETA_NAMES]


def load():
    """Load liblynx.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not LIBRARY.exists():
        raise RuntimeError(f"{LIBRARY} is not built: run `python -m paper_2607_01831_amd.build` "
                           "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(str(LIBRARY))
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    LP, MP = ctypes.POINTER(lynx_layout), ctypes.POINTER(lynx_meta)
    sigs = {
        "lynx_kv_encode": ([LP, I32, I32, P, P, P, P, P, P, P, MP, P], ctypes.c_int),
        "lynx_kv_merge": ([P, P, P, SZ, P], ctypes.c_int),
        "lynx_attn_workspace_bytes": ([LP, I32, I32, I32, I32], SZ),
        "lynx_attn_anchor_decode": ([LP, I32, I32, I32, P, P, P, P, MP, P, P, P, P, SZ, P],
                                    ctypes.c_int),
        "lynx_attn_anchor_decode_split": ([I32, LP, I32, I32, I32, P, P, P, P, MP, P, P, P, P, SZ, P],
                                          ctypes.c_int),
        "lynx_attn_anchor_decode_noalloc": ([LP, I32, I32, I32, P, P, P, P, MP, P, P, P, P],
                                            ctypes.c_int),
        "lynx_attn_verify": ([LP, I32, I32, I32, I32, P, P, P, P, MP, P, P, P, P, P, SZ, P],
                             ctypes.c_int),
        "lynx_attn_anchor_decode_tail": ([LP, I32, I32, I32, P, P, P, P, MP, P, I32, P, P, P, P, P,
                                          SZ, P], ctypes.c_int),
        "lynx_spec_accept_workspace_bytes": ([I32, I32, I32], SZ),
        "lynx_spec_accept_greedy": ([I32, I32, I32, P, P, P, P, P, SZ, P], ctypes.c_int),
        "lynx_spec_accept_sample": ([I32, I32, I32, P, P, P, P, P, P, P, SZ, P], ctypes.c_int),
        "lynx_serialized_bytes": ([I32, I32, ctypes.POINTER(SZ), ctypes.POINTER(SZ)], ctypes.c_int),
        "lynx_kv_serialize": ([I32, I32, P, P, P, P, P], ctypes.c_int),
        "lynx_kv_deserialize_anchor": ([LP, I32, I32, I32, P, P, P, P, MP, P], ctypes.c_int),
        "lynx_kv_deserialize_residual": ([LP, I32, I32, I32, P, P, P, P, P, P, P], ctypes.c_int),
        "lynx_hkv_encode": ([LP, I32, I32, P, P, P, ctypes.c_float, I32, P, P, P, P,
                             ctypes.POINTER(lynx_hmeta), P], ctypes.c_int),
        "lynx_hkv_dequant": ([LP, I32, I32, P, I32, P, P, ctypes.c_float, I32,
                              ctypes.POINTER(lynx_hmeta), P, P, P], ctypes.c_int),
        "lynx_kv_encode_split": ([LP, I32, I32, I32, P, P, P, P, P, P, P, MP, P], ctypes.c_int),
        "lynx_kv_merge_split": ([I32, SZ, P, P, P, P], ctypes.c_int),
        "lynx_kv_dequant_anchor_split": ([LP, I32, I32, I32, P, P, P, MP, P, P, P], ctypes.c_int),
        "lynx_attn_tree_workspace_bytes": ([LP, I32, I32, I32, I32], SZ),
        "lynx_attn_verify_tree": ([P, I32, I32, I32, I32, P, P, P, P, P, P, P, P, P, P, P, SZ, P], ctypes.c_int),
        "lynx_spec_tree_workspace_bytes": ([I32, I32, I32], SZ),
        "lynx_spec_accept_tree_greedy": ([I32, I32, I32, P, P, P, P, P, P, P, SZ, P], ctypes.c_int),
        "lynx_spec_accept_tree_sample": ([I32, I32, I32, P, P, P, P, P, P, P, P, SZ, P], ctypes.c_int),
        "lynx_kv_append": ([P, I32, I32, I32, P, P, P, P, P, P, P, P, P, P, P, P, P, P, P], ctypes.c_int),
        "lynx_kv_append_begin": ([P, I32, P, P, P, P, P, P], ctypes.c_int),
        "lynx_kv_dequant": ([P, I32, I32, P, P, P, P, P, P, P, P, P], ctypes.c_int),
        "lynx_attn_hier": ([P, I32, I32, I32, I32, P, P, I32, P, P, ctypes.c_float, I32, P, P, I32, P, P, P, P, P, SZ, P],
                           ctypes.c_int),
        "lynx_qk_norm_rope": ([I32, I32, I32, I32, P, I64, P, I64, P, I64, P, P, I32, P, P, ctypes.c_float, P, I32, I32,
                               ctypes.c_float, P, P, P, P], ctypes.c_int),
        "lynx_blocks_extend": ([P, I32, I32, I32, P, P, P, P, P, P, P, P, P, P, P, P], ctypes.c_int),
        "lynx_blocks_release": ([P, I32, P, P, P, P, P, P], ctypes.c_int),
        "lynx_strerror": ([ctypes.c_int], ctypes.c_char_p),
    }
    for name, (args, res) in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _lib = lib
    return lib


def lynx_strerror(status: int) -> str:
    return load().lynx_strerror(status).decode()


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("liblynx takes device tensors")
    if not t.is_contiguous():
        raise ValueError("liblynx takes contiguous tensors")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        if torch.cuda.is_initialized():
            # the same handle without a Stream object around it (1.4 us a call)
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return stream


def _check(fn: str, status: int):
    if status != LYNX_OK:
        raise LynxError(fn, status)


# Size checks of the tensors a call reads or writes.  The C ABI sees only
# pointers, so a short tensor would become an out-of-bounds device access:
# the binding rejects it first.  A call makes a dozen of these, and a short
# kernel waits for them (the checks and the pointers in one function each,
# sizes computed once a call: an anchor decode 14.2 -> 10.5 us on the host).
def _arg(fn: str, what: str, t, nbytes: int):
    """The device pointer of tensor `t`, which holds at least nbytes bytes; an
    int is a pointer already, None is NULL."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if t.nbytes < nbytes:
        raise ValueError(f"{fn}: {what} holds {t.nbytes} bytes; the call uses {nbytes}")
    if not t.is_cuda:
        raise ValueError("liblynx takes device tensors")
    if not t.is_contiguous():
        raise ValueError("liblynx takes contiguous tensors")
    return t.data_ptr()


def _meta_arg(fn: str, L: "Layout", meta: "Meta", rows: int) -> lynx_meta:
    """fp32 metadata rows 0 .. rows - 1 (sequences) of the layout."""
    heads = rows * L.num_kv_heads
    k = heads * -(-L.max_tokens // K_GROUP) * HEAD_DIM * 4
    v = heads * L.max_tokens * 4
    return lynx_meta(_arg(fn, "meta.k_scale", meta.k_scale, k), _arg(fn, "meta.k_zero", meta.k_zero, k),
                     _arg(fn, "meta.v_scale", meta.v_scale, v), _arg(fn, "meta.v_zero", meta.v_zero, v))


def _hmeta_arg(fn: str, L: "Layout", hmeta: "HMeta", rows: int) -> lynx_hmeta:
    heads = rows * L.num_kv_heads
    page = heads * -(-L.max_tokens // 256) * HEAD_DIM * 4
    chunk = heads * -(-L.max_tokens // 32) * HEAD_DIM * 4
    return lynx_hmeta(*(_arg(fn, f"hmeta.{name}", getattr(hmeta, name), page if name[2] == "g" else chunk)
                        for name in _HMETA_NAMES))


def _attn_args(fn: str, L: "Layout", B: int, Hq: int, seq_lens, block_table, k_plane, v_plane, row_bytes: int,
               meta: "Meta", q, nq: int = 1):
    """The arguments every attention call starts with, up to q."""
    if B <= 0:
        return (ctypes.byref(L.c()),), (_ptr(seq_lens), _ptr(block_table), _ptr(k_plane), _ptr(v_plane),
                                        ctypes.byref(meta.c()), _ptr(q))
    plane = L.plane_bytes(row_bytes)
    return (ctypes.byref(L.c()),), (
        _arg(fn, "seq_lens", seq_lens, B * 4),
        _arg(fn, "block_table", block_table, B * L.max_blocks_per_seq * 4),
        _arg(fn, "plane 0", k_plane, plane), _arg(fn, "plane 1", v_plane, plane),
        ctypes.byref(_meta_arg(fn, L, meta, B)), _arg(fn, "q", q, B * nq * Hq * HEAD_DIM * 2))


def _here(stream):
    """The current device and the stream of a call, one of that device (without a
    CUDA context yet there is no tensor to launch on)."""
    if not torch.cuda.is_initialized():
        return 0, stream
    dev = torch._C._cuda_getDevice()
    if stream is None:
        return dev, torch._C._cuda_getCurrentRawStream(dev)
    if not isinstance(stream, torch.cuda.Stream):
        return dev, stream
    if stream.device_index != dev:
        raise ValueError(f"the stream is one of device {stream.device_index}, not of the current one ({dev})")
    return dev, stream.cuda_stream


def _typed_form(fn: str, what: str, t, nbytes: int, dtype, dev: int):
    """_arg for a contiguous tensor of one type on the call's device (planes are
    uint8, counts and tables int32, metadata and scores fp32, K, V and q BF16).
    A call makes up to 21 of these: one test where nothing is wrong."""
    if t is None or t.__class__ is int:
        return t
    if t.dtype is not dtype or t.nbytes < nbytes or t.get_device() != dev or not t.is_contiguous():
        if t.dtype is not dtype:
            raise ValueError(f"{fn}: {what} is {t.dtype}; the call uses {dtype}")
        if t.is_cuda and t.get_device() != dev:
            raise ValueError(f"{fn}: {what} is on device {t.get_device()}, not on the current one ({dev})")
        _arg(fn, what, t, nbytes)  # raises for what is left
    return t.data_ptr()


def _fastest_typed():
    """The same in C++, which leaves to the form above what does not pass (an append
    9.5 -> 5.7 us on the host), or that form where it is not built."""
    global _args
    if not ARGS.exists():
        return _typed_form
    try:
        from . import _args
    except ImportError as e:
        warnings.warn(f"{ARGS} does not load ({e}): build it again for this Python and torch "
                      "(python -m paper_2607_01831_amd.build)", RuntimeWarning)
        return _typed_form
    _args.otherwise(_typed_form)
    return _args.typed


_typed = _fastest_typed()


def _whole(name: str, dev: int, stream, *args):
    """A whole call in C++: its status, or None where an argument does not pass or
    that code is not built: the form behind it then makes the call, or says what is
    wrong (norms and rotation of one token 8.6 -> 4.6 us on the host)."""
    f = _whole_calls.get(name)
    if f is None:
        f = _whole_calls[name] = _whole_call(name)
    return f(dev, stream, *args)


_whole_calls: dict = {}


def _whole_call(name: str):
    call = None if _typed is _typed_form else getattr(_args, name[len("lynx_"):], None)
    if call is None:
        return lambda *args: None
    return functools.partial(call, ctypes.cast(getattr(load(), name), ctypes.c_void_p).value)


_BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
_pack_layout, _pack_meta = struct.Struct("7i").pack, struct.Struct("4P").pack


def _packed(L: "Layout") -> bytes:
    """The lynx_layout as bytes (a quarter of the time of the ctypes structure)."""
    return _pack_layout(L.num_kv_heads, L.head_dim, L.k_group_tokens, L.block_tokens, L.max_blocks_per_seq,
                        L.num_blocks, L.max_tokens)


def _typed_meta(fn: str, L: "Layout", meta: "Meta", rows: int, dev: int) -> bytes:
    heads = rows * L.num_kv_heads
    k, v = heads * -(-L.max_tokens // K_GROUP) * HEAD_DIM * 4, heads * L.max_tokens * 4
    return _pack_meta(_typed(fn, "meta.k_scale", meta.k_scale, k, _F32, dev) or 0,
                      _typed(fn, "meta.k_zero", meta.k_zero, k, _F32, dev) or 0,
                      _typed(fn, "meta.v_scale", meta.v_scale, v, _F32, dev) or 0,
                      _typed(fn, "meta.v_zero", meta.v_zero, v, _F32, dev) or 0)


@dataclass
class Layout:
    """Cache geometry (see lynx_layout in include/lynx.h)."""
    num_kv_heads: int
    block_tokens: int
    max_blocks_per_seq: int
    num_blocks: int
    max_tokens: int
    head_dim: int = HEAD_DIM
    k_group_tokens: int = K_GROUP

    def c(self) -> lynx_layout:
        return lynx_layout(self.num_kv_heads, self.head_dim, self.k_group_tokens,
                           self.block_tokens, self.max_blocks_per_seq, self.num_blocks,
                           self.max_tokens)

    @property
    def n_groups(self) -> int:
        return -(-self.max_tokens // K_GROUP)

    def plane_bytes(self, row_bytes: int = 64) -> int:
        return self.num_blocks * self.num_kv_heads * self.block_tokens * row_bytes


@dataclass
class Meta:
    """fp32 metadata tensors of a batch (device)."""
    k_scale: torch.Tensor  # [B][Hkv][n_groups][128]
    k_zero: torch.Tensor
    v_scale: torch.Tensor  # [B][Hkv][max_tokens]
    v_zero: torch.Tensor

    @staticmethod
    def empty(L: Layout, B: int, device="cuda") -> "Meta":
        ks = (B, L.num_kv_heads, L.n_groups, HEAD_DIM)
        vs = (B, L.num_kv_heads, L.max_tokens)
        f = dict(dtype=torch.float32, device=device)
        return Meta(torch.zeros(ks, **f), torch.zeros(ks, **f), torch.zeros(vs, **f),
                    torch.zeros(vs, **f))

    def c(self) -> lynx_meta:
        return lynx_meta(_ptr(self.k_scale), _ptr(self.k_zero), _ptr(self.v_scale),
                         _ptr(self.v_zero))


def lynx_kv_encode(L: Layout, b: int, T: int, block_table, k, v, k_anc, v_anc, k_res, v_res,
                   meta: Meta, stream=None) -> None:
    fn = "lynx_kv_encode"
    n, plane = T * L.num_kv_heads * HEAD_DIM * 2, L.plane_bytes(64)
    _check(fn, load().lynx_kv_encode(
        ctypes.byref(L.c()), b, T, _arg(fn, "block_table", block_table, (b + 1) * L.max_blocks_per_seq * 4),
        _arg(fn, "k", k, n), _arg(fn, "v", v, n), _arg(fn, "k_anc", k_anc, plane), _arg(fn, "v_anc", v_anc, plane),
        _arg(fn, "k_res", k_res, plane), _arg(fn, "v_res", v_res, plane),
        ctypes.byref(_meta_arg(fn, L, meta, b + 1)), _stream(stream)))


def lynx_kv_merge(anc, res, codes, n_packed_bytes: int | None = None, stream=None) -> None:
    n = anc.numel() if n_packed_bytes is None else n_packed_bytes
    if n > anc.numel() or n > res.numel() or 2 * n > codes.numel():
        raise ValueError("lynx_kv_merge: the planes hold fewer bytes than asked for")
    _check("lynx_kv_merge", load().lynx_kv_merge(_ptr(anc), _ptr(res), _ptr(codes), n,
                                                 _stream(stream)))


def lynx_attn_workspace_bytes(L: Layout, B: int, Hq: int, num_queries: int,
                              max_seq_len: int) -> int:
    lay = L.c()
    return int(load().lynx_attn_workspace_bytes(ctypes.byref(lay), B, Hq, num_queries,
                                                 max_seq_len))


# Arrival counters at the head of every attention workspace (lynx.h).
ATTN_COUNTER_BYTES = 262144


def lynx_attn_tree_workspace_bytes(L: Layout, B: int, Hq: int, n: int, max_seq_len: int) -> int:
    return int(load().lynx_attn_tree_workspace_bytes(ctypes.byref(L.c()), B, Hq, n, max_seq_len))


def workspace(L: Layout, B: int, Hq: int, num_queries: int, max_seq_len: int,
              device="cuda", tree: bool = True) -> torch.Tensor:
    """A device buffer (allocated by torch) for any attention call of as many
    queries, of lynx_attn_tree_workspace_bytes() bytes, or with tree=False of
    lynx_attn_workspace_bytes(); zero-filled: the arrival counters at its head
    must start at zero."""
    size = lynx_attn_tree_workspace_bytes if tree else lynx_attn_workspace_bytes
    n = size(L, B, Hq, num_queries, max_seq_len)
    return torch.zeros(max(n, ATTN_COUNTER_BYTES), dtype=torch.uint8, device=device)


def lynx_attn_anchor_decode(L: Layout, B: int, Hq: int, max_seq_len: int, seq_lens,
                            block_table, k_anc, v_anc, meta: Meta, q, out, lse=None,
                            workspace_buf=None, stream=None) -> None:
    fn = "lynx_attn_anchor_decode"
    lay, args = _attn_args(fn, L, B, Hq, seq_lens, block_table, k_anc, v_anc, 64, meta, q)
    ws = workspace_buf
    _check(fn, load().lynx_attn_anchor_decode(
        *lay, B, Hq, max_seq_len, *args, _arg(fn, "out", out, B * Hq * HEAD_DIM * 2), _arg(fn, "lse", lse, B * Hq * 4),
        _ptr(ws), 0 if ws is None else ws.nbytes, _stream(stream)))


def lynx_attn_anchor_decode_split(anchor_bits: int, L: Layout, B: int, Hq: int, max_seq_len: int,
                                  seq_lens, block_table, k_anc, v_anc, meta: Meta, q, out, lse=None,
                                  workspace_buf=None, stream=None) -> None:
    """Decode over the A-bit anchor planes of a split width (rows of 16 A bytes)."""
    fn = "lynx_attn_anchor_decode_split"
    if anchor_bits not in (2, 4, 6):
        raise LynxError(fn, LYNX_EINVAL)
    lay, args = _attn_args(fn, L, B, Hq, seq_lens, block_table, k_anc, v_anc, 16 * anchor_bits, meta, q)
    ws = workspace_buf
    _check(fn, load().lynx_attn_anchor_decode_split(
        anchor_bits, *lay, B, Hq, max_seq_len, *args, _arg(fn, "out", out, B * Hq * HEAD_DIM * 2),
        _arg(fn, "lse", lse, B * Hq * 4), _ptr(ws), 0 if ws is None else ws.nbytes, _stream(stream)))


# Scratch held by the library for lynx_attn_anchor_decode_noalloc (lynx.h).
NOALLOC_SCRATCH_BYTES = 16 << 20


def lynx_attn_anchor_decode_noalloc(L: Layout, B: int, Hq: int, max_seq_len: int, seq_lens,
                                    block_table, k_anc, v_anc, meta: Meta, q, out, lse=None,
                                    stream=None) -> None:
    """lynx_attn_anchor_decode without a workspace: the library's own static
    scratch (calls that overlap on one GPU race)."""
    fn = "lynx_attn_anchor_decode_noalloc"
    lay, args = _attn_args(fn, L, B, Hq, seq_lens, block_table, k_anc, v_anc, 64, meta, q)
    _check(fn, load().lynx_attn_anchor_decode_noalloc(
        *lay, B, Hq, max_seq_len, *args, _arg(fn, "out", out, B * Hq * HEAD_DIM * 2),
        _arg(fn, "lse", lse, B * Hq * 4), _stream(stream)))


def lynx_attn_anchor_decode_tail(L: Layout, B: int, Hq: int, max_seq_len: int, seq_lens,
                                 block_table, k_anc, v_anc, meta: Meta, q, k_tail, v_tail, out,
                                 lse=None, workspace_buf=None, stream=None) -> None:
    """Anchor decode that also attends the BF16 tail k_tail / v_tail
    ([B][n_tail][Hkv][128], or None for n_tail = 0)."""
    fn = "lynx_attn_anchor_decode_tail"
    lay, args = _attn_args(fn, L, B, Hq, seq_lens, block_table, k_anc, v_anc, 64, meta, q)
    n_tail = 0 if k_tail is None else int(k_tail.shape[1])
    n = B * n_tail * L.num_kv_heads * HEAD_DIM * 2
    ws = workspace_buf
    _check(fn, load().lynx_attn_anchor_decode_tail(
        *lay, B, Hq, max_seq_len, *args, n_tail, _arg(fn, "k_tail", k_tail, n),
        _ptr(v_tail) if k_tail is None else _arg(fn, "v_tail", v_tail, n), _arg(fn, "out", out, B * Hq * HEAD_DIM * 2),
        _arg(fn, "lse", lse, B * Hq * 4), _ptr(ws), 0 if ws is None else ws.nbytes, _stream(stream)))


def _scratch(make, nbytes: int, device, stream) -> torch.Tensor:
    """A call's own workspace, made (torch.empty, torch.zeros) on the stream that the
    call runs on: cleared before it, and free again behind it."""
    if stream is None:
        return make(nbytes, dtype=torch.uint8, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        return make(nbytes, dtype=torch.uint8, device=device)


def lynx_spec_accept_workspace_bytes(B: int, k: int, vocab: int) -> int:
    return int(load().lynx_spec_accept_workspace_bytes(B, k, vocab))


def lynx_spec_accept_greedy(target_logits, draft_tokens, accepted, next_token,
                            workspace_buf=None, stream=None) -> None:
    """target_logits fp32 [B][k+1][V], draft_tokens int32 [B][k]; writes
    accepted and next_token (int32 [B]).  workspace_buf: None allocates
    lynx_spec_accept_workspace_bytes() bytes with torch, on the call's stream."""
    B, k1, V = (int(x) for x in target_logits.shape)
    ws = workspace_buf
    if ws is None:
        n = lynx_spec_accept_workspace_bytes(B, k1 - 1, V)
        ws = _scratch(torch.empty, max(n, 16), target_logits.device, stream)
    _check("lynx_spec_accept_greedy", load().lynx_spec_accept_greedy(
        B, k1 - 1, V, _ptr(target_logits), _ptr(draft_tokens), _ptr(accepted), _ptr(next_token),
        _ptr(ws), ws.nbytes, _stream(stream)))


def lynx_spec_accept_sample(target_probs, draft_probs, draft_tokens, uniforms, accepted,
                            next_token, workspace_buf=None, stream=None) -> None:
    """target_probs fp32 [B][k+1][V], draft_probs fp32 [B][k][V], draft_tokens
    int32 [B][k], uniforms fp32 [B][k+1]; writes accepted and next_token
    (int32 [B]).  workspace_buf: None allocates
    lynx_spec_accept_workspace_bytes() bytes with torch, on the call's stream."""
    B, k1, V = (int(x) for x in target_probs.shape)
    ws = workspace_buf
    if ws is None:
        n = lynx_spec_accept_workspace_bytes(B, k1 - 1, V)
        ws = _scratch(torch.empty, max(n, 16), target_probs.device, stream)
    _check("lynx_spec_accept_sample", load().lynx_spec_accept_sample(
        B, k1 - 1, V, _ptr(target_probs), _ptr(draft_probs), _ptr(draft_tokens), _ptr(uniforms),
        _ptr(accepted), _ptr(next_token), _ptr(ws), ws.nbytes, _stream(stream)))


def lynx_attn_verify(L: Layout, B: int, Hq: int, k: int, max_seq_len: int, seq_lens,
                     block_table, k_codes, v_codes, meta: Meta, q, k_new, v_new, out,
                     workspace_buf=None, stream=None) -> None:
    fn = "lynx_attn_verify"
    lay, args = _attn_args(fn, L, B, Hq, seq_lens, block_table, k_codes, v_codes, 128, meta, q, k)
    n = B * k * L.num_kv_heads * HEAD_DIM * 2
    ws = workspace_buf
    _check(fn, load().lynx_attn_verify(
        *lay, B, Hq, k, max_seq_len, *args, _arg(fn, "k_new", k_new, n), _arg(fn, "v_new", v_new, n),
        _arg(fn, "out", out, B * k * Hq * HEAD_DIM * 2), _ptr(ws), 0 if ws is None else ws.nbytes, _stream(stream)))


def lynx_attn_verify_tree(L: Layout, B: int, Hq: int, n: int, max_seq_len: int, seq_lens, block_table,
                          k_codes, v_codes, meta: Meta, q, k_new, v_new, parents, out,
                          workspace_buf=None, stream=None) -> None:
    """Verification of a tree: q [B][n][Hq][128], k_new and v_new
    [B][n][Hkv][128], parents int32 [B][n]; workspace() of n queries."""
    fn, (dev, stream) = "lynx_attn_verify_tree", _here(stream)
    ws, nb, nn = workspace_buf, max(B, 0), max(n, 0)
    plane, kv = L.plane_bytes(128), nb * nn * L.num_kv_heads * HEAD_DIM * 2
    io = nb * nn * Hq * HEAD_DIM * 2
    _check(fn, load().lynx_attn_verify_tree(
        _packed(L), B, Hq, n, max_seq_len, _typed(fn, "seq_lens", seq_lens, nb * 4, _I32, dev),
        _typed(fn, "block_table", block_table, nb * L.max_blocks_per_seq * 4, _I32, dev),
        _typed(fn, "k_codes", k_codes, plane, _U8, dev), _typed(fn, "v_codes", v_codes, plane, _U8, dev),
        _typed_meta(fn, L, meta, nb, dev), _typed(fn, "q", q, io, _BF16, dev),
        _typed(fn, "k_new", k_new, kv, _BF16, dev), _typed(fn, "v_new", v_new, kv, _BF16, dev),
        _typed(fn, "parents", parents, nb * nn * 4, _I32, dev), _typed(fn, "out", out, io, _BF16, dev),
        _typed(fn, "workspace_buf", ws, 0, _U8, dev), 0 if ws is None else ws.nbytes, stream))


def lynx_spec_tree_workspace_bytes(B: int, n: int, vocab: int) -> int:
    return int(load().lynx_spec_tree_workspace_bytes(B, n, vocab))


def spec_tree_workspace(B: int, n: int, vocab: int, device="cuda") -> torch.Tensor:
    """A device buffer of lynx_spec_tree_workspace_bytes() bytes, zero-filled:
    every call finds it zero and leaves it zero."""
    return _tree_scratch(B, n, vocab, device, None)


def _tree_scratch(B: int, n: int, vocab: int, device, stream) -> torch.Tensor:
    return _scratch(torch.zeros, max(lynx_spec_tree_workspace_bytes(B, n, vocab), 16), device, stream)


def _tree_args(fn: str, dev: int, scores, tokens, parents, accepted, path, next_token, uniforms=None):
    if scores.dim() != 3:
        raise ValueError(f"{fn}: the scores are [B][n + 1][vocab]")
    B, n1, V = (int(x) for x in scores.shape)
    rows = B * (n1 - 1) * 4
    return B, n1 - 1, V, [
        _typed(fn, "scores", scores, B * n1 * V * 4, _F32, dev), _typed(fn, "tokens", tokens, rows, _I32, dev),
        _typed(fn, "parents", parents, rows, _I32, dev),
        *([] if uniforms is None else [_typed(fn, "uniforms", uniforms, B * n1 * 4, _F32, dev)]),
        _typed(fn, "accepted", accepted, B * 4, _I32, dev), _typed(fn, "path", path, rows, _I32, dev),
        _typed(fn, "next_token", next_token, B * 4, _I32, dev)]


def lynx_spec_accept_tree_greedy(target_logits, tokens, parents, accepted, path, next_token,
                                 workspace_buf=None, stream=None) -> None:
    """target_logits fp32 [B][n+1][V], tokens and parents int32 [B][n]; writes
    accepted, next_token (int32 [B]) and path (int32 [B][n]).  workspace_buf:
    spec_tree_workspace(); None makes one for this call, on its stream."""
    fn, on, (dev, stream) = "lynx_spec_accept_tree_greedy", stream, _here(stream)
    B, n, V, args = _tree_args(fn, dev, target_logits, tokens, parents, accepted, path, next_token)
    ws = workspace_buf if workspace_buf is not None else _tree_scratch(B, n, V, target_logits.device, on)
    _check(fn, load().lynx_spec_accept_tree_greedy(B, n, V, *args, _typed(fn, "workspace_buf", ws, 0, _U8, dev), ws.nbytes,
                                                   stream))


def lynx_spec_accept_tree_sample(target_probs, tokens, parents, uniforms, accepted, path, next_token,
                                 workspace_buf=None, stream=None) -> None:
    """target_probs fp32 [B][n+1][V], uniforms fp32 [B][n+1]; the rest as
    lynx_spec_accept_tree_greedy."""
    fn, on, (dev, stream) = "lynx_spec_accept_tree_sample", stream, _here(stream)
    if uniforms is None:
        raise LynxError(fn, LYNX_EINVAL)
    B, n, V, args = _tree_args(fn, dev, target_probs, tokens, parents, accepted, path, next_token, uniforms)
    ws = workspace_buf if workspace_buf is not None else _tree_scratch(B, n, V, target_probs.device, on)
    _check(fn, load().lynx_spec_accept_tree_sample(B, n, V, *args, _typed(fn, "workspace_buf", ws, 0, _U8, dev), ws.nbytes,
                                                   stream))


# BF16 K rows kept per sequence for its open group (lynx.h).
OPEN_ROWS = 256


def lynx_kv_append(L: Layout, B: int, max_new: int, seq_lens, counts, path, block_table, k_new, v_new, k_open,
                   k_codes, v_codes, k_anc, v_anc, k_res, v_res, meta: Meta, stream=None) -> None:
    """k_new, v_new: BF16 [B][n_src][Hkv][128]; path int32 [B][max_new] or None;
    k_open BF16 [B][OPEN_ROWS][Hkv][128]; pairs of planes that are not kept are
    None."""
    fn, (dev, stream) = "lynx_kv_append", _here(stream)
    nb, row = max(B, 0), L.num_kv_heads * HEAD_DIM * 2
    if k_new.dim() != 4:
        raise ValueError(f"{fn}: k_new is [B][n_src][Hkv][128]")
    n_src = int(k_new.shape[1])
    codes, nibbles = L.plane_bytes(128), L.plane_bytes(64)
    _check(fn, load().lynx_kv_append(
        _packed(L), B, max_new, n_src, _typed(fn, "seq_lens", seq_lens, nb * 4, _I32, dev),
        _typed(fn, "counts", counts, nb * 4, _I32, dev), _typed(fn, "path", path, nb * max(max_new, 0) * 4, _I32, dev),
        _typed(fn, "block_table", block_table, nb * L.max_blocks_per_seq * 4, _I32, dev),
        _typed(fn, "k_new", k_new, nb * n_src * row, _BF16, dev), _typed(fn, "v_new", v_new, nb * n_src * row, _BF16, dev),
        _typed(fn, "k_open", k_open, nb * OPEN_ROWS * row, _BF16, dev),
        _typed(fn, "k_codes", k_codes, codes, _U8, dev), _typed(fn, "v_codes", v_codes, codes, _U8, dev),
        _typed(fn, "k_anc", k_anc, nibbles, _U8, dev), _typed(fn, "v_anc", v_anc, nibbles, _U8, dev),
        _typed(fn, "k_res", k_res, nibbles, _U8, dev), _typed(fn, "v_res", v_res, nibbles, _U8, dev),
        _typed_meta(fn, L, meta, nb, dev), stream))


def lynx_kv_append_begin(L: Layout, B: int, seq_lens, block_table, k_codes, meta: Meta, k_open,
                         stream=None) -> None:
    fn, (dev, stream) = "lynx_kv_append_begin", _here(stream)
    nb = max(B, 0)
    _check(fn, load().lynx_kv_append_begin(
        _packed(L), B, _typed(fn, "seq_lens", seq_lens, nb * 4, _I32, dev),
        _typed(fn, "block_table", block_table, nb * L.max_blocks_per_seq * 4, _I32, dev),
        _typed(fn, "k_codes", k_codes, L.plane_bytes(128), _U8, dev), _typed_meta(fn, L, meta, nb, dev),
        _typed(fn, "k_open", k_open, nb * OPEN_ROWS * L.num_kv_heads * HEAD_DIM * 2, _BF16, dev), stream))


def lynx_kv_dequant(L: Layout, B: int, max_n: int, starts, counts, block_table, k_codes, v_codes, meta: Meta,
                    k_out, v_out, stream=None) -> None:
    """k_out, v_out: BF16 [B][max_n][Hkv][128] (device, written)."""
    fn, (dev, stream) = "lynx_kv_dequant", _here(stream)
    nb = max(B, 0)
    n = nb * max(max_n, 0) * L.num_kv_heads * HEAD_DIM * 2
    _check(fn, load().lynx_kv_dequant(
        _packed(L), B, max_n, _typed(fn, "starts", starts, nb * 4, _I32, dev),
        _typed(fn, "counts", counts, nb * 4, _I32, dev),
        _typed(fn, "block_table", block_table, nb * L.max_blocks_per_seq * 4, _I32, dev),
        _typed(fn, "k_codes", k_codes, L.plane_bytes(128), _U8, dev), _typed(fn, "v_codes", v_codes, L.plane_bytes(128), _U8, dev),
        _typed_meta(fn, L, meta, nb, dev), _typed(fn, "k_out", k_out, n, _BF16, dev),
        _typed(fn, "v_out", v_out, n, _BF16, dev), stream))


# ----------------------------------------------------------------------------
# Allocation helpers (torch device memory only)
# ----------------------------------------------------------------------------

@dataclass
class HMeta:
    """fp32 metadata of the hierarchical codec (device): page minimum and
    range [B][Hkv][ceil(max_tokens/256)][128], chunk mean and scale
    [B][Hkv][ceil(max_tokens/32)][128], for K and V."""
    k_gmin: torch.Tensor
    k_gscale: torch.Tensor
    k_mu: torch.Tensor
    k_sigma: torch.Tensor
    v_gmin: torch.Tensor
    v_gscale: torch.Tensor
    v_mu: torch.Tensor
    v_sigma: torch.Tensor

    @staticmethod
    def empty(L: Layout, B: int, device="cuda") -> "HMeta":
        pg = (B, L.num_kv_heads, -(-L.max_tokens // 256), HEAD_DIM)
        ch = (B, L.num_kv_heads, -(-L.max_tokens // 32), HEAD_DIM)
        z = lambda shape: torch.zeros(shape, dtype=torch.float32, device=device)
        return HMeta(z(pg), z(pg), z(ch), z(ch), z(pg), z(pg), z(ch), z(ch))

    def c(self) -> lynx_hmeta:
        return lynx_hmeta(*(_ptr(getattr(self, f)) for f, _ in lynx_hmeta._fields_))


def lynx_kv_encode_split(L: Layout, anchor_bits: int, b: int, T: int, block_table, k, v, k_anc, v_anc,
                         k_res, v_res, meta: Meta, stream=None) -> None:
    """k, v: BF16 [T][Hkv][128]; planes: uint8 device tensors of rows of
    16 anchor_bits (anchor) and 16 (8 - anchor_bits) (residual) bytes."""
    fn = "lynx_kv_encode_split"
    n = T * L.num_kv_heads * HEAD_DIM * 2
    # (a width that the library rejects needs no plane)
    wa, wr = (anchor_bits, 8 - anchor_bits) if 0 < anchor_bits < 8 else (0, 0)
    anc, res = L.plane_bytes(16 * wa), L.plane_bytes(16 * wr)
    _check(fn, load().lynx_kv_encode_split(
        ctypes.byref(L.c()), anchor_bits, b, T,
        _arg(fn, "block_table", block_table, (b + 1) * L.max_blocks_per_seq * 4), _arg(fn, "k", k, n),
        _arg(fn, "v", v, n), _arg(fn, "k_anc", k_anc, anc), _arg(fn, "v_anc", v_anc, anc),
        _arg(fn, "k_res", k_res, res), _arg(fn, "v_res", v_res, res),
        ctypes.byref(_meta_arg(fn, L, meta, b + 1)), _stream(stream)))


def lynx_kv_merge_split(anchor_bits: int, anc, res, codes, stream=None) -> None:
    """Rows of A-bit anchors and (8 - A)-bit residuals -> rows of 128 codes."""
    n_rows = anc.numel() // (16 * anchor_bits)
    if (anc.numel() != n_rows * 16 * anchor_bits or res.numel() != n_rows * 16 * (8 - anchor_bits)
            or codes.numel() < n_rows * 128):
        raise ValueError("lynx_kv_merge_split: plane sizes do not match one another")
    _check("lynx_kv_merge_split", load().lynx_kv_merge_split(
        anchor_bits, n_rows, _ptr(anc), _ptr(res), _ptr(codes), _stream(stream)))


def lynx_kv_dequant_anchor_split(L: Layout, anchor_bits: int, b: int, T: int, block_table, k_anc, v_anc,
                                 meta: Meta, k_out, v_out, stream=None) -> None:
    """k_out, v_out: BF16 [T][Hkv][128] (device, written)."""
    fn = "lynx_kv_dequant_anchor_split"
    n = T * L.num_kv_heads * HEAD_DIM * 2
    anc = L.plane_bytes(16 * anchor_bits) if 0 < anchor_bits < 8 else 0
    _check(fn, load().lynx_kv_dequant_anchor_split(
        ctypes.byref(L.c()), anchor_bits, b, T,
        _arg(fn, "block_table", block_table, (b + 1) * L.max_blocks_per_seq * 4), _arg(fn, "k_anc", k_anc, anc),
        _arg(fn, "v_anc", v_anc, anc), ctypes.byref(_meta_arg(fn, L, meta, b + 1)), _arg(fn, "k_out", k_out, n),
        _arg(fn, "v_out", v_out, n), _stream(stream)))


# codec variants of the hierarchical codec (lynx.h LYNX_HQ_*)
LYNX_HQ_BIASED, LYNX_HQ_CENTRED, LYNX_HQ_INT4 = 0, 1, 2


def lynx_hkv_encode(L: Layout, b: int, T: int, block_table, k, v, alpha: float, variant: int,
                    k_anc, v_anc, k_res, v_res, hmeta: HMeta, stream=None) -> None:
    """k_res, v_res may be None for LYNX_HQ_INT4."""
    fn = "lynx_hkv_encode"
    n, plane = T * L.num_kv_heads * HEAD_DIM * 2, L.plane_bytes(64)
    _check(fn, load().lynx_hkv_encode(
        ctypes.byref(L.c()), b, T, _arg(fn, "block_table", block_table, (b + 1) * L.max_blocks_per_seq * 4),
        _arg(fn, "k", k, n), _arg(fn, "v", v, n), alpha, variant, _arg(fn, "k_anc", k_anc, plane),
        _arg(fn, "v_anc", v_anc, plane), _arg(fn, "k_res", k_res, plane), _arg(fn, "v_res", v_res, plane),
        ctypes.byref(_hmeta_arg(fn, L, hmeta, b + 1)), _stream(stream)))


def lynx_hkv_dequant(L: Layout, b: int, T: int, block_table, full: bool, k_plane, v_plane,
                     alpha: float, variant: int, hmeta: HMeta, k_out, v_out, stream=None) -> None:
    """k_out, v_out: BF16 [T][Hkv][128] (device, written)."""
    fn = "lynx_hkv_dequant"
    n, plane = T * L.num_kv_heads * HEAD_DIM * 2, L.plane_bytes(128 if full else 64)
    _check(fn, load().lynx_hkv_dequant(
        ctypes.byref(L.c()), b, T, _arg(fn, "block_table", block_table, (b + 1) * L.max_blocks_per_seq * 4),
        1 if full else 0, _arg(fn, "k_plane", k_plane, plane), _arg(fn, "v_plane", v_plane, plane), alpha, variant,
        ctypes.byref(_hmeta_arg(fn, L, hmeta, b + 1)), _arg(fn, "k_out", k_out, n), _arg(fn, "v_out", v_out, n),
        _stream(stream)))


_pack_hmeta = struct.Struct("8P").pack


def _typed_hmeta(fn: str, L: "Layout", hmeta: "HMeta", rows: int, dev: int) -> bytes:
    heads = rows * L.num_kv_heads
    page, chunk = (heads * -(-L.max_tokens // n) * HEAD_DIM * 4 for n in (256, 32))
    return _pack_hmeta(*(_typed(fn, "hmeta." + name, getattr(hmeta, name), page if name[2] == "g" else chunk, _F32, dev) or 0
                         for name in _HMETA_NAMES))


def lynx_attn_hier(L: Layout, B: int, Hq: int, k: int, max_seq_len: int, seq_lens, block_table, full: bool, k_plane,
                   v_plane, alpha: float, variant: int, hmeta: HMeta, q, k_tail, v_tail, out, lse=None,
                   workspace_buf=None, stream=None) -> None:
    """Attention over the hierarchical codec's 4-bit planes, or its merged codes
    (full): q [B][k][Hq][128], k_tail and v_tail [B][n_tail][Hkv][128] or None,
    lse fp32 [B][k][Hq] or None; workspace() of k queries."""
    fn, (dev, stream) = "lynx_attn_hier", _here(stream)
    status = _whole(fn, dev, stream, L, B, Hq, k, max_seq_len, seq_lens, block_table, full, k_plane, v_plane, alpha, variant,
                    hmeta, q, k_tail, v_tail, out, lse, workspace_buf)
    if status is not None:
        return _check(fn, status)
    ws, nb, nk = workspace_buf, max(B, 0), max(k, 0)
    if (k_tail is None) != (v_tail is None):
        raise LynxError(fn, LYNX_EINVAL)
    if k_tail is not None and k_tail.dim() != 4:
        raise ValueError(f"{fn}: k_tail is [B][n_tail][Hkv][128]")
    n_tail = 0 if k_tail is None else int(k_tail.shape[1])
    plane, tail = L.plane_bytes(128 if full else 64), nb * n_tail * L.num_kv_heads * HEAD_DIM * 2
    io = nb * nk * Hq * HEAD_DIM * 2
    _check(fn, load().lynx_attn_hier(
        _packed(L), B, Hq, k, max_seq_len, _typed(fn, "seq_lens", seq_lens, nb * 4, _I32, dev),
        _typed(fn, "block_table", block_table, nb * L.max_blocks_per_seq * 4, _I32, dev), 1 if full else 0,
        _typed(fn, "k_plane", k_plane, plane, _U8, dev), _typed(fn, "v_plane", v_plane, plane, _U8, dev), alpha, variant,
        _typed_hmeta(fn, L, hmeta, nb, dev), _typed(fn, "q", q, io, _BF16, dev), n_tail,
        _typed(fn, "k_tail", k_tail, tail, _BF16, dev), _typed(fn, "v_tail", v_tail, tail, _BF16, dev),
        _typed(fn, "out", out, io, _BF16, dev), _typed(fn, "lse", lse, nb * nk * Hq * 4, _F32, dev),
        _typed(fn, "workspace_buf", ws, 0, _U8, dev), 0 if ws is None else ws.nbytes, stream))


def _heads(fn: str, what: str, t, tokens: int, dev: int):
    """Pointer, heads and token stride of BF16 heads [tokens][heads][128], which may
    be part of a wider row."""
    if t is None:
        return None, 0, 0
    if t.dim() != 3 or t.shape[0] != tokens or t.shape[2] != HEAD_DIM:
        raise ValueError(f"{fn}: {what} is [tokens][heads][128]")
    heads, (step, head, one) = int(t.shape[1]), t.stride()
    if t.dtype is not _BF16:
        raise ValueError(f"{fn}: {what} is {t.dtype}; the call uses {_BF16}")
    if t.get_device() != dev:
        raise ValueError("liblynx takes device tensors" if not t.is_cuda else
                         f"{fn}: {what} is on device {t.get_device()}, not on the current one ({dev})")
    if one != 1 or (head != HEAD_DIM and heads > 1):
        raise ValueError(f"{fn}: the heads of {what} do not follow one another")
    return t.data_ptr(), heads, step if tokens > 1 else max(step, heads * HEAD_DIM) // 8 * 8


def lynx_qk_norm_rope(q, k, v, positions, rows, q_weight, k_weight, eps: float, inv_freq, pairs: bool, scale: float,
                      q_out, k_out, v_out, stream=None) -> None:
    """q [tokens][Hq][128], k and v [tokens][Hkv][128] BF16, contiguous or views of
    a fused row; positions, rows (or None) int32 [tokens]; weights BF16 [128] or
    None; inv_freq fp32 [rotary_dim / 2] or None; q_out [rows..][Hq][128], k_out and
    v_out [rows..][Hkv][128] (the leading dims are rows in order).  v and v_out may
    be None."""
    fn, (dev, stream) = "lynx_qk_norm_rope", _here(stream)
    status = _whole(fn, dev, stream, q, k, v, positions, rows, q_weight, k_weight, eps, inv_freq, pairs, scale, q_out, k_out,
                    v_out)
    if status is not None:
        return _check(fn, status)
    n = int(q.shape[0])
    qp, Hq, qs = _heads(fn, "q", q, n, dev)
    kp, Hkv, ks = _heads(fn, "k", k, n, dev)
    vp, Hv, vs = _heads(fn, "v", v, n, dev)
    if (v is None) != (v_out is None):
        raise LynxError(fn, LYNX_EINVAL)
    if v is not None and Hv != Hkv:
        raise ValueError(f"{fn}: v has {Hv} heads, k {Hkv}")
    n_rows = q_out.numel() // (Hq * HEAD_DIM) if Hq else 0
    out = n_rows * Hkv * HEAD_DIM * 2
    _check(fn, load().lynx_qk_norm_rope(
        n, Hq, Hkv, HEAD_DIM, qp, qs, kp, ks, vp, vs, _typed(fn, "positions", positions, n * 4, _I32, dev),
        _typed(fn, "rows", rows, n * 4, _I32, dev), n_rows, _typed(fn, "q_weight", q_weight, HEAD_DIM * 2, _BF16, dev),
        _typed(fn, "k_weight", k_weight, HEAD_DIM * 2, _BF16, dev), eps, _typed(fn, "inv_freq", inv_freq, 0, _F32, dev),
        0 if inv_freq is None else 2 * inv_freq.numel(), 1 if pairs else 0, scale,
        _typed(fn, "q_out", q_out, 0, _BF16, dev), _typed(fn, "k_out", k_out, out, _BF16, dev),
        _typed(fn, "v_out", v_out, out, _BF16, dev), stream))


def _blocks_args(fn: str, L: Layout, B: int, dev: int, block_table, free_blocks, free_state):
    return (_typed(fn, "block_table", block_table, max(B, 0) * L.max_blocks_per_seq * 4, _I32, dev),
            _typed(fn, "free_blocks", free_blocks, L.num_blocks * 4, _I32, dev),
            _typed(fn, "free_state", free_state, 8, _I32, dev))


def lynx_blocks_extend(L: Layout, B: int, n_src: int, seq_lens, counts, block_table, free_blocks, free_state, granted,
                       starts, seq_of=None, positions=None, slots=None, rows=None, stream=None) -> None:
    """Room for counts[b] <= n_src new tokens behind every sequence; max_rows is
    the length of the token arrays seq_of, positions, slots and rows that are given
    (B * n_src where none is)."""
    fn, (dev, stream) = "lynx_blocks_extend", _here(stream)
    status = _whole(fn, dev, stream, L, B, n_src, seq_lens, counts, block_table, free_blocks, free_state, granted, starts,
                    seq_of, positions, slots, rows)
    if status is not None:
        return _check(fn, status)
    nb = max(B, 0)
    given = [t.numel() for t in (seq_of, positions, slots, rows) if t is not None]
    max_rows = min(given) if given else min(nb * max(n_src, 0), 1 << 30)
    _check(fn, load().lynx_blocks_extend(
        _packed(L), B, n_src, max_rows, _typed(fn, "seq_lens", seq_lens, nb * 4, _I32, dev),
        _typed(fn, "counts", counts, nb * 4, _I32, dev), *_blocks_args(fn, L, B, dev, block_table, free_blocks, free_state),
        _typed(fn, "granted", granted, nb * 4, _I32, dev), _typed(fn, "starts", starts, (nb + 1) * 4, _I32, dev),
        *(_typed(fn, what, t, max_rows * 4, _I32, dev)
          for what, t in (("seq_of", seq_of), ("positions", positions), ("slots", slots), ("rows", rows))), stream))


def lynx_blocks_release(L: Layout, B: int, seq_lens, keep, block_table, free_blocks, free_state, stream=None) -> None:
    fn, (dev, stream) = "lynx_blocks_release", _here(stream)
    status = _whole(fn, dev, stream, L, B, seq_lens, keep, block_table, free_blocks, free_state)
    if status is not None:
        return _check(fn, status)
    nb = max(B, 0)
    _check(fn, load().lynx_blocks_release(
        _packed(L), B, _typed(fn, "seq_lens", seq_lens, nb * 4, _I32, dev), _typed(fn, "keep", keep, nb * 4, _I32, dev),
        *_blocks_args(fn, L, B, dev, block_table, free_blocks, free_state), stream))


def lynx_serialized_bytes(num_kv_heads: int, n_tokens: int) -> tuple[int, int]:
    """(anchor_bytes, residual_bytes) of an object of n_tokens tokens."""
    a, r = ctypes.c_size_t(), ctypes.c_size_t()
    _check("lynx_serialized_bytes", load().lynx_serialized_bytes(num_kv_heads, n_tokens,
                                                                 ctypes.byref(a), ctypes.byref(r)))
    return int(a.value), int(r.value)


def lynx_kv_serialize(num_kv_heads: int, n_tokens: int, k, v, anchor_buf, residual_buf,
                      stream=None) -> None:
    """k, v: BF16 [n_tokens][Hkv][128] (an object's tokens); the buffers are
    uint8 device tensors of lynx_serialized_bytes() bytes."""
    fn = "lynx_kv_serialize"
    n, na, nr = n_tokens * num_kv_heads * HEAD_DIM * 2, 0, 0
    if num_kv_heads > 0 and n_tokens > 0:
        na, nr = lynx_serialized_bytes(num_kv_heads, n_tokens)
    _check(fn, load().lynx_kv_serialize(
        num_kv_heads, n_tokens, _arg(fn, "k", k, n), _arg(fn, "v", v, n), _arg(fn, "anchor_buf", anchor_buf, na),
        _arg(fn, "residual_buf", residual_buf, nr), _stream(stream)))


def lynx_kv_deserialize_anchor(L: Layout, b: int, t0: int, n_tokens: int, block_table, anchor_buf,
                               k_anc, v_anc, meta: Meta, stream=None) -> None:
    fn = "lynx_kv_deserialize_anchor"
    na = lynx_serialized_bytes(L.num_kv_heads, n_tokens)[0] if n_tokens > 0 else 0
    plane = L.plane_bytes(64)
    _check(fn, load().lynx_kv_deserialize_anchor(
        ctypes.byref(L.c()), b, t0, n_tokens,
        _arg(fn, "block_table", block_table, (b + 1) * L.max_blocks_per_seq * 4),
        _arg(fn, "anchor_buf", anchor_buf, na), _arg(fn, "k_anc", k_anc, plane), _arg(fn, "v_anc", v_anc, plane),
        ctypes.byref(_meta_arg(fn, L, meta, b + 1)), _stream(stream)))


def lynx_kv_deserialize_residual(L: Layout, b: int, t0: int, n_tokens: int, block_table,
                                 residual_buf, k_anc, v_anc, k_codes, v_codes,
                                 stream=None) -> None:
    fn = "lynx_kv_deserialize_residual"
    nr = lynx_serialized_bytes(L.num_kv_heads, n_tokens)[1] if n_tokens > 0 else 0
    plane = L.plane_bytes(64)
    _check(fn, load().lynx_kv_deserialize_residual(
        ctypes.byref(L.c()), b, t0, n_tokens,
        _arg(fn, "block_table", block_table, (b + 1) * L.max_blocks_per_seq * 4),
        _arg(fn, "residual_buf", residual_buf, nr), _arg(fn, "k_anc", k_anc, plane), _arg(fn, "v_anc", v_anc, plane),
        _arg(fn, "k_codes", k_codes, 2 * plane), _arg(fn, "v_codes", v_codes, 2 * plane), _stream(stream)))


@dataclass
class KVPool:
    """Nibble planes, metadata and (after merge) code planes of one layer."""
    layout: Layout
    B: int
    k_anc: torch.Tensor
    v_anc: torch.Tensor
    k_res: torch.Tensor
    v_res: torch.Tensor
    meta: Meta
    k_codes: torch.Tensor | None = None
    v_codes: torch.Tensor | None = None

    @staticmethod
    def allocate(L: Layout, B: int, device="cuda", codes: bool = True) -> "KVPool":
        n = L.plane_bytes(64)
        u8 = dict(dtype=torch.uint8, device=device)
        pool = KVPool(L, B, torch.zeros(n, **u8), torch.zeros(n, **u8), torch.zeros(n, **u8),
                      torch.zeros(n, **u8), Meta.empty(L, B, device))
        if codes:
            pool.k_codes = torch.zeros(2 * n, **u8)
            pool.v_codes = torch.zeros(2 * n, **u8)
        return pool

    @staticmethod
    def allocate_layers(L: Layout, B: int, layers: int, device="cuda", codes: bool = True):
        """Pools for `layers` layers whose planes are consecutive slices of one
        allocation per plane kind, so that a whole cache's residual planes can
        be transported and merged in one call each.  Returns (pools, whole),
        whole being a KVPool-like record of the full-length planes (its meta
        is that of layer 0 and is not used)."""
        n = L.plane_bytes(64)
        u8 = dict(dtype=torch.uint8, device=device)
        big = {name: torch.zeros(layers * n, **u8) for name in ("k_anc", "v_anc", "k_res", "v_res")}
        if codes:
            big["k_codes"] = torch.zeros(layers * 2 * n, **u8)
            big["v_codes"] = torch.zeros(layers * 2 * n, **u8)
        pools = []
        for l in range(layers):
            pool = KVPool(L, B, *(big[name][l * n:(l + 1) * n] for name in ("k_anc", "v_anc", "k_res", "v_res")),
                          Meta.empty(L, B, device))
            if codes:
                pool.k_codes = big["k_codes"][l * 2 * n:(l + 1) * 2 * n]
                pool.v_codes = big["v_codes"][l * 2 * n:(l + 1) * 2 * n]
            pools.append(pool)
        whole = KVPool(L, B, big["k_anc"], big["v_anc"], big["k_res"], big["v_res"], pools[0].meta,
                       big.get("k_codes"), big.get("v_codes"))
        return pools, whole

    def encode(self, b: int, T: int, block_table, k, v, stream=None) -> None:
        lynx_kv_encode(self.layout, b, T, block_table, k, v, self.k_anc, self.v_anc, self.k_res,
                       self.v_res, self.meta, stream)

    def merge(self, stream=None) -> None:
        lynx_kv_merge(self.k_anc, self.k_res, self.k_codes, stream=stream)
        lynx_kv_merge(self.v_anc, self.v_res, self.v_codes, stream=stream)

    def open_rows(self) -> torch.Tensor:
        """The BF16 K rows of the sequences' open groups, for append()."""
        return torch.zeros(self.B, OPEN_ROWS, self.layout.num_kv_heads, HEAD_DIM, dtype=torch.bfloat16,
                           device=self.k_anc.device)

    def append(self, max_new: int, seq_lens, counts, path, block_table, k_new, v_new, k_open, stream=None) -> None:
        """lynx_kv_append into the nibble planes, and the codes where there are any."""
        lynx_kv_append(self.layout, self.B, max_new, seq_lens, counts, path, block_table, k_new, v_new, k_open,
                       self.k_codes, self.v_codes, self.k_anc, self.v_anc, self.k_res, self.v_res, self.meta, stream)


@dataclass
class FreeBlocks:
    """The blocks of a paged cache that no sequence has, and the sequences' table
    (device): what lynx_blocks_extend and lynx_blocks_release keep."""
    table: torch.Tensor  # int32 [B][max_blocks_per_seq], -1 where there is no block
    stack: torch.Tensor  # int32 [num_blocks]
    state: torch.Tensor  # int32 [2]: ids on the stack, 0

    @staticmethod
    def allocate(L: Layout, B: int, device="cuda") -> "FreeBlocks":
        """Empty sequences, every block free, block 0 on top."""
        i32 = dict(dtype=torch.int32, device=device)
        return FreeBlocks(torch.full((B, L.max_blocks_per_seq), -1, **i32),
                          torch.arange(L.num_blocks - 1, -1, -1, **i32), torch.tensor([L.num_blocks, 0], **i32))


def contiguous_layout(Hkv: int, B: int, T: int) -> Layout:
    """One block of T tokens per sequence; block_table[b] = [b]."""
    return Layout(num_kv_heads=Hkv, block_tokens=T, max_blocks_per_seq=1, num_blocks=B,
                  max_tokens=T)
