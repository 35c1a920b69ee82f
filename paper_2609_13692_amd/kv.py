"""The paged key/value cache of include/mpt.h, in 16 bits or in 4: pages that the
sequences of a layout share, appends (with the rotation to positions on the
way, if asked), attention of new tokens over the pages, tokens read back, and
the join of attention over parts of a context.

As :mod:`.mpt` this only marshals arguments: every step runs in the HIP kernels
of ``libmpt.so``. Calls enqueue on the current stream (or ``stream``) and
synchronise only where ``check=True`` asks for a host result. Lists of slots,
lengths and pages are int32 device tensors.
"""
from __future__ import annotations

import ctypes
import math
import struct

import torch

from .mpt import KvDescriptor, KvDescriptorMx4, MptError, _check, load

BF16, F16, F32, MX4 = 0, 1, 2, 3                # MX4: added to a 16-bit type
_KIND = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}
MAX_PARTS = 16
_ROTATION = struct.Struct("PPiif").pack         # mpt_kv_rotation
_POINTERS = [struct.Struct(f"{n}P").pack for n in range(MAX_PARTS + 1)]      # host arrays of device pointers
STATUS_BITS = {1: "slot", 2: "length", 4: "page", 8: "duplicate", 16: "not empty", 32: "no pages", 64: "shared page"}


def _list(t, n, name, index):
    """Address of a contiguous int32 tensor of at least n elements on GPU `index`."""
    if t.dtype is not torch.int32:
        raise TypeError(f"{name} must be torch.int32, got {t.dtype}")
    if t.get_device() != index:
        raise ValueError(f"{name} must be on GPU {index}, got {t.device}")
    if not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{name} must be contiguous, of at least {n} elements; got {tuple(t.shape)}")
    return t.data_ptr()


def _on(stream, index):
    """Address of a stream of GPU index (None: its current one), and what new
    tensors that its work uses are made under."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(index) or None, None
    if stream.device_index != index:
        raise ValueError(f"stream must be on GPU {index}, is on GPU {stream.device_index}")
    return stream.cuda_stream or None, torch.cuda.stream(stream)


def _run(index, call, *args):
    """The call with GPU index as the current one, where launches go: the
    address of a default stream does not say whose it is."""
    if torch._C._cuda_getDevice() == index:
        return call(*args)
    with torch.cuda.device(index):
        return call(*args)


def _new(shape, dtype, device, under):
    if under is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with under:                    # the allocator then orders reuse by that stream
        return torch.empty(shape, dtype=dtype, device=device)


def _like(t, dtype, under):
    if under is None:
        return torch.empty_like(t, dtype=dtype)
    with under:
        return torch.empty_like(t, dtype=dtype)


class KvCache:
    """Keys and values of many sequences in pages that they may share.

    ``k`` and ``v`` are [layers, pages, slots per page, heads, dim] tensors
    (bfloat16 or float16) of any strides that are multiples of 8 elements, the
    last one 1; ``table`` [slots, pages of a sequence], ``length`` [slots],
    ``ref`` [pages] and ``status`` [1] are int32, ``free_bits`` int64, one bit
    per page: together the state described at ``mpt_kv_cache``.
    :meth:`create` allocates and empties one.

    In 4 bits (``mpt_kv_cache_mx4``) ``k`` and ``v`` are uint8 [layers, pages,
    slots per page, heads, dim / 2], of strides that are multiples of 16, with
    ``k_scale`` and ``v_scale`` uint8 [layers, pages, slots per page, heads,
    dim / 32], and ``dtype`` (bfloat16 or float16) is the type that tokens come
    in and are read as.

    The cache holds the workspaces of its calls: of attention one for each size
    that its calls need (at most three), all of them for as long as the cache
    lives, so that graphs captured earlier stay valid. Calls on one cache must
    be ordered (one stream, or events between streams).
    """

    def __init__(self, k, v, table, length, ref, free_bits, status, k_scale=None, v_scale=None, dtype=None):
        if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v must be [layers, pages, slots, heads, dim] of one shape and type")
        four = k_scale is not None or v_scale is not None
        if four:
            if k.dtype is not torch.uint8:
                raise TypeError(f"k and v with scales must be uint8, got {k.dtype}")
            if dtype not in (torch.bfloat16, torch.float16):
                raise TypeError(f"a cache in 4 bits needs dtype bfloat16 or float16, got {dtype}")
            for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
                if t is None or t.dtype is not torch.uint8 or t.device != k.device or \
                        t.shape != (*k.shape[:4], k.shape[4] // 16) or k.shape[4] % 16 or t.stride(4) != 1:
                    raise ValueError(f"{name} must be uint8 [layers, pages, slots, heads, dim / 32] on {k.device}, with contiguous rows")
        elif k.dtype not in (torch.bfloat16, torch.float16) or dtype not in (None, k.dtype):
            raise TypeError(f"k and v must be bfloat16 or float16, got {k.dtype}")
        if not k.is_cuda:
            raise ValueError("k must be a device tensor")
        if k.stride(4) != 1 or v.stride(4) != 1:
            raise ValueError("the elements of a row must be contiguous")
        layers, pages, size, heads, dim = k.shape
        dim, kind = (2 * dim, _KIND[dtype] + MX4) if four else (dim, _KIND[k.dtype])
        for name, t, want, n in (("ref", ref, torch.int32, pages), ("free_bits", free_bits, torch.int64, -(-pages // 64)),
                                  ("status", status, torch.int32, 1), ("length", length, torch.int32, 1),
                                  ("table", table, torch.int32, 1), ("v", v, v.dtype, 0)):
            if t.dtype != want or t.device != k.device or t.numel() < n or (name != "v" and not t.is_contiguous()):
                raise ValueError(f"{name} must be a contiguous {want} tensor of at least {n} elements on {k.device}")
        if table.dim() != 2 or table.shape[0] != length.numel():
            raise ValueError("table must be [slots, pages of a sequence], length [slots]")
        self.k, self.v, self.table, self.length, self.ref = k, v, table, length, ref
        self.free_bits, self.status = free_bits, status
        self.k_scale, self.v_scale = k_scale, v_scale
        self.device, self.dtype = k.device, dtype if four else k.dtype
        self.page_size, self.n_heads, self.head_dim = size, heads, dim
        self.max_seqs, self._index = table.shape[0], k.get_device()
        whole = KvDescriptorMx4()
        d = whole.c
        d.k, d.v = k.data_ptr(), v.data_ptr()
        d.k_stride[:], d.v_stride[:] = k.stride()[:4], v.stride()[:4]
        d.table, d.length, d.ref = table.data_ptr(), length.data_ptr(), ref.data_ptr()
        d.free_bits, d.status = free_bits.data_ptr(), status.data_ptr()
        d.dtype, d.n_layers, d.n_pages, d.page_size = kind, layers, pages, size
        d.n_heads, d.head_dim, d.max_seqs, d.max_pages = heads, dim, table.shape[0], table.shape[1]
        if four:
            whole.k_scale, whole.v_scale = k_scale.data_ptr(), v_scale.data_ptr()
            whole.k_scale_stride[:], whole.v_scale_stride[:] = k_scale.stride()[:4], v_scale.stride()[:4]
        self._whole, self._d = whole, d
        self._p = ctypes.addressof(d)
        self._lib = load()
        n = self._lib.mpt_kv_workspace_bytes(self._p)
        if n == 0:
            raise MptError(-1, "mpt_kv_workspace_bytes", self._lib.mpt_last_error().decode())
        self._ws = torch.empty(n, dtype=torch.uint8, device=self.device)
        self._ws_at, self._ws_bytes = self._ws.data_ptr(), n
        self._ws_stream = torch._C._cuda_getCurrentRawStream(self._index) or None
        self._at_ws, self._at_sizes, self._scale = {}, {}, 1.0 / math.sqrt(dim)

    @classmethod
    def create(cls, n_layers, n_pages, page_size, n_heads, head_dim, max_seqs, max_len, dtype=torch.bfloat16,
               device="cuda", heads_first=None, bits=16):
        """An empty cache of 16 or 4 bits; ``heads_first`` puts a page's heads
        outside its slots (None: in 4 bits, where a head's row alone is a part
        of what memory hands out at a time)."""
        if bits not in (16, 4):
            raise ValueError(f"a cache has 16 bits or 4, got {bits}")
        if bits == 4 and head_dim % 32:
            raise ValueError(f"head_dim in 4 bits must be a multiple of 32, got {head_dim}")
        if heads_first is None:
            heads_first = bits == 4
        shape = (n_layers, n_pages) + ((n_heads, page_size) if heads_first else (page_size, n_heads))

        def pool(row, dtype):
            # zeros: a page is copied whole, tokens that were never written included
            x = torch.zeros((*shape, row), dtype=dtype, device=device)
            return x.transpose(2, 3) if heads_first else x
        how = {}
        if bits == 4:
            k, v = (pool(head_dim // 2, torch.uint8) for _ in range(2))
            how = dict(k_scale=pool(head_dim // 32, torch.uint8), v_scale=pool(head_dim // 32, torch.uint8), dtype=dtype)
        else:
            k, v = (pool(head_dim, dtype) for _ in range(2))
        i32 = dict(dtype=torch.int32, device=device)
        c = cls(k, v, torch.full((max_seqs, max(1, -(-max_len // page_size))), -1, **i32), torch.zeros(max_seqs, **i32),
                torch.zeros(n_pages, **i32), torch.zeros(-(-n_pages // 64), dtype=torch.int64, device=device),
                torch.zeros(1, **i32), **how)
        c.reset()
        return c

    def reset(self, stream=None):
        _check(_run(self._index, self._lib.mpt_kv_reset, self._p, _on(stream, self._index)[0]), "mpt_kv_reset")

    def take_status(self, stream=None) -> list[str]:
        """What calls have found wrong in device data since the last look."""
        bits = ctypes.c_uint32(0)
        at = _on(stream, self._index)[0]
        _check(_run(self._index, self._lib.mpt_kv_status, self._p, ctypes.addressof(bits), at), "mpt_kv_status")
        return [name for bit, name in STATUS_BITS.items() if bits.value & bit]

    def _on(self, stream):
        """As the function _on. The allocator learns of a stream that the
        workspaces were not used on before."""
        at, under = _on(stream, self._index)
        if at != self._ws_stream:
            self._ws_stream = at
            for ws in (self._ws, *self._at_ws.values()):
                ws.record_stream(stream or torch.cuda.current_stream(self._index))
        return at, under

    def _pages(self, name, lists, check, stream):
        out = ctypes.c_int64(0) if check else None
        args = []
        if lists:
            n = lists[0].numel()
            args = [n] + [None if t is None else _list(t, n, name, self._index) for t in lists]
        rc = _run(self._index, getattr(self._lib, name), self._p, *args, ctypes.addressof(out) if check else None,
                  self._ws_at, self._ws_bytes, self._on(stream)[0])
        if rc:
            _check(rc, name)
        return out.value if check else None

    def fork(self, src, dst, keep, new_len, check=False, stream=None):
        """Empty slots dst become sequences of new_len tokens sharing the first
        keep with src (-1: none). With check, waits and returns the number of
        free pages left, or raises."""
        return self._pages("mpt_kv_fork", (src, dst, keep, new_len), check, stream)

    def extend(self, seqs, new_len, check=False, stream=None):
        """Grows sequences to new_len tokens."""
        return self._pages("mpt_kv_extend", (seqs, new_len), check, stream)

    def free(self, seqs, keep=None, check=False, stream=None):
        """Cuts sequences to keep tokens (None: to none)."""
        return self._pages("mpt_kv_free", (seqs, keep), check, stream)

    def compact(self, check=False, stream=None):
        """Moves the pages in use to the lowest numbers; with check returns
        how many they are."""
        return self._pages("mpt_kv_compact", (), check, stream)

    def copy(self, src, dst, check=False, stream=None):
        """Copies page contents (all layers)."""
        return self._pages("mpt_kv_copy", (src, dst), check, stream)

    def _rows(self, t, heads, name, dtype):
        shape = t.shape
        if len(shape) != 3 or shape[1] != heads or shape[2] != self.head_dim or t.dtype is not dtype:
            raise ValueError(f"{name} must be [tokens, {heads}, {self.head_dim}] of {dtype}, got {tuple(shape)} of {t.dtype}")
        by_token, by_head, by_element = t.stride()
        if by_element != 1 or t.get_device() != self._index:
            raise ValueError(f"{name} must be on {self.device}, with contiguous rows")
        return t.data_ptr(), by_token, by_head

    def append(self, layer, k_new, v_new, q_off, seqs, stream=None):
        """Writes the newest tokens' keys and values of one layer; q_off [n + 1]
        cuts the tokens into the sequences in seqs [n]."""
        n, tokens, index = seqs.numel(), k_new.shape[0], self._index
        if v_new.shape[0] != tokens:
            raise ValueError("k_new and v_new must have one row per token")
        rc = _run(index, self._lib.mpt_kv_append, self._p, layer, n, _list(seqs, n, "seqs", index),
                  _list(q_off, n + 1, "q_off", index), tokens, *self._rows(k_new, self.n_heads, "k_new", self.dtype),
                  *self._rows(v_new, self.n_heads, "v_new", self.dtype), _on(stream, index)[0])
        if rc:
            _check(rc, "mpt_kv_append")

    def append_rotated(self, layer, k_new, v_new, q_off, seqs, freq, q=None, q_out=None, interleaved=False, positions=None,
                       factor=1.0, stream=None):
        """As append, with the keys (and the queries q [tokens, heads, dim])
        rotated to their positions: pair i of a row by position * freq[i], its
        first 2 len(freq) elements in all (see mpt_kv_append_rotated). Returns
        the rotated queries, in q_out (which may be q) or a new tensor; None
        without any. Queries without a place (of bad slots, no positions given)
        are not written: their rows of a new tensor hold anything. positions
        [tokens] int32 in the place of the tokens' own in their sequences; with
        k_new and v_new None nothing is written, and then, with positions, q_off
        and seqs may be None."""
        index = self._index
        at, under = _on(stream, index)
        if freq.dtype is not torch.float32 or freq.get_device() != index or freq.dim() != 1 or not freq.is_contiguous():
            raise ValueError(f"freq must be a contiguous float32 vector on GPU {index}")
        if (k_new is None) != (v_new is None) or (k_new is None and q is None):
            raise ValueError("needs k_new and v_new, or q, or all three")
        tokens = (q if k_new is None else k_new).shape[0]
        k = v = q_in = out = (None, 0, 0)
        heads = 1
        if k_new is not None:
            if v_new.shape[0] != tokens:
                raise ValueError("v_new must have one row per token")
            k, v = self._rows(k_new, self.n_heads, "k_new", self.dtype), self._rows(v_new, self.n_heads, "v_new", self.dtype)
        if q is not None:
            heads = q.shape[1]
            q_in = self._rows(q, heads, "q", self.dtype)
            if q_out is None:
                q_out = _like(q, self.dtype, under)
                by_token, by_head, by_element = q_out.stride()
                if by_element != 1:                        # q's rows overlap, or are a column each
                    q_out = _new(q.shape, self.dtype, self.device, under)
                    by_token, by_head, _ = q_out.stride()
                out = q_out.data_ptr(), by_token, by_head
            elif q_out.shape[0] != tokens:
                raise ValueError("q_out must have one row per token")
            else:
                out = q_in if q_out is q else self._rows(q_out, heads, "q_out", self.dtype)
            if q.shape[0] != tokens:
                raise ValueError("q must have one row per token")
        elif q_out is not None:
            raise ValueError("q_out without q")
        n, lists = 0, (None, None)
        if seqs is not None:
            n = seqs.numel()
            lists = _list(seqs, n, "seqs", index), _list(q_off, n + 1, "q_off", index)
        elif k_new is not None or positions is None or q_off is not None:
            raise ValueError("needs q_off and seqs, but for queries alone with positions")
        rotation = _ROTATION(freq.data_ptr(), 0 if positions is None else _list(positions, tokens, "positions", index),
                             2 * freq.numel(), bool(interleaved), factor)
        rc = _run(index, self._lib.mpt_kv_append_rotated, self._p, layer, n, *lists, tokens, *k, *v, rotation, heads, *q_in, *out, at)
        if rc:
            _check(rc, "mpt_kv_append_rotated")
        return q_out

    def read(self, layer, off, seqs, tokens, first=None, k_out=None, v_out=None, stream=None):
        """(keys, values) [tokens, heads, dim] of one layer in the cache's 16-bit
        type: of entry i those from first[i] on (None: the newest) of the
        sequence in slot seqs[i], off[i + 1] - off[i] of them, in rows off[i] on.
        Tokens that are not there are zeros (see mpt_kv_read)."""
        n, index, heads = seqs.numel(), self._index, self.n_heads
        at, under = _on(stream, index)
        if k_out is None:
            k_out = _new((tokens, heads, self.head_dim), self.dtype, self.device, under)
            if v_out is None:
                v_out = _like(k_out, self.dtype, under)
        elif v_out is None:
            v_out = _new((tokens, heads, self.head_dim), self.dtype, self.device, under)
        if k_out.shape[0] != tokens or v_out.shape[0] != tokens:
            raise ValueError("k_out and v_out must have one row per token")
        rc = _run(index, self._lib.mpt_kv_read, self._p, layer, n, _list(seqs, n, "seqs", index),
                  _list(off, n + 1, "off", index), None if first is None else _list(first, n, "first", index), tokens,
                  *self._rows(k_out, heads, "k_out", self.dtype), *self._rows(v_out, heads, "v_out", self.dtype), at)
        if rc:
            _check(rc, "mpt_kv_read")
        return k_out, v_out

    def attend(self, layer, q, q_off, seqs, causal=True, window=0, softcap=0.0, scale=None, kv_begin=None, out=None,
               lse=None, out_dtype=None, stream=None):
        """(out, lse) of the newest tokens' queries over their sequences (see
        mpt_kv_attention). scale defaults to 1 / sqrt(dim)."""
        tokens, heads, dim = q.shape
        n, index = seqs.numel(), self._index
        at, under = self._on(stream)
        if out is None:
            out = _new((tokens, heads, dim), out_dtype or self.dtype, self.device, under)
        elif out.shape[0] != tokens or (out_dtype or out.dtype) != out.dtype:
            raise ValueError("out must have one row per token, of out_dtype")
        if lse is None:
            lse = _new((tokens, heads), torch.float32, self.device, under)
        elif lse.dtype is not torch.float32 or lse.get_device() != index or lse.shape != (tokens, heads) or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32 [tokens, heads] device tensor")
        key = (n, tokens, heads)
        need = self._at_sizes.get(key)
        if need is None:
            need = self._lib.mpt_kv_attention_workspace_bytes(self._p, n, tokens, heads)
            if len(self._at_sizes) < 4096:
                self._at_sizes[key] = need
        ws = self._at_ws.get(need)
        if ws is None:
            ws = self._at_ws[need] = _new(need, torch.uint8, self.device, under)
        rc = _run(
            index, self._lib.mpt_kv_attention, self._p, layer, n, _list(seqs, n, "seqs", index),
            _list(q_off, n + 1, "q_off", index), tokens, heads,
            *self._rows(q, heads, "q", self.dtype), *self._rows(out, heads, "out", out.dtype), _KIND.get(out.dtype, -1),
            lse.data_ptr(), None if kv_begin is None else _list(kv_begin, n, "kv_begin", index), 1 if causal else 0,
            min(window, 1 << 30), softcap, self._scale if scale is None else scale, ws.data_ptr(), need, at)
        if rc:
            _check(rc, "mpt_kv_attention")
        return out, lse


def merge(parts, lses, out_dtype=None, out=None, lse=None, stream=None):
    """(out, lse) of attention over disjoint parts of a context: parts are
    [..., dim] tensors of one shape and type, lses float32 [...] (see
    mpt_kv_merge)."""
    if len(parts) != len(lses) or not 1 <= len(parts) <= MAX_PARTS:
        raise ValueError(f"needs 1 .. {MAX_PARTS} parts, each with its lse")
    first, first_lse = parts[0], lses[0]
    kind, index = _KIND.get(first.dtype), first.get_device()
    if kind is None or index < 0:
        raise TypeError(f"parts must be bfloat16, float16 or float32 device tensors, got {first.dtype} on {first.device}")
    shape, dtype = first.shape, first.dtype
    rows = shape[:-1]
    for p, l in zip(parts, lses):
        if p.dtype is not dtype or p.get_device() != index or not p.is_contiguous() or p.shape != shape:
            raise ValueError("parts must be contiguous device tensors of one shape and type")
        if l.dtype is not torch.float32 or l.get_device() != index or not l.is_contiguous() or l.shape != rows:
            raise ValueError("lses must be contiguous float32 device tensors of the parts' shape without the last dimension")
    at, under = _on(stream, index)
    if out is None:
        out = _like(first, out_dtype or dtype, under)
    elif out.shape != shape or out.get_device() != index or not out.is_contiguous() or (out_dtype or out.dtype) != out.dtype:
        raise ValueError("out must be a contiguous device tensor of the parts' shape and out_dtype")
    if lse is None:
        lse = _like(first_lse, torch.float32, under)
    elif lse.shape != rows or lse.dtype is not torch.float32 or lse.get_device() != index or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 device tensor")
    n = len(parts)
    pack = _POINTERS[n]
    rc = _run(index, load().mpt_kv_merge, n, first_lse.numel(), shape[-1], pack(*[p.data_ptr() for p in parts]),
              pack(*[l.data_ptr() for l in lses]), kind, out.data_ptr(), _KIND.get(out.dtype, -1), lse.data_ptr(), at)
    if rc:
        _check(rc, "mpt_kv_merge")
    return out, lse
