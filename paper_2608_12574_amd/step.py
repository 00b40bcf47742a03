"""What a decode step does beside the mask: edits of logits, the best tokens, trees of drafted tokens, and a paged K/V cache.

As in ``tam``, this module marshals arguments only; every step runs in
``libtam.so`` on the stream given, or torch's current stream.  The tensors and the stream of a call
are of the current device, or it is refused.  Scratch comes from torch's caching allocator.
"""
from __future__ import annotations

import ctypes

from . import tam as _tam
from .tam import DTYPE_BF16, DTYPE_FP16, TAM_OK, Chunk, Edits, Pages, Rotation, TamError, _calls, _check


def _bad(where, what):
    return TamError(-1, where, what)


def _int32(where, name, t, n, gpu):
    """The pointer of a contiguous int32 tensor of n elements on GPU number `gpu`."""
    if t.dtype is not _int or t.get_device() != gpu or t.numel() != n or not t.is_contiguous():
        raise _bad(where, f"{name} must be a contiguous int32 tensor of {n} elements on cuda:{gpu}")
    return t.data_ptr()


def _rows_of(where, name, t, B, dtype, gpu):
    """(pointer, row stride, columns) of a [B, n] tensor on GPU number `gpu` whose rows are contiguous."""
    if t.dtype is not dtype or t.get_device() != gpu or t.dim() != 2:
        raise _bad(where, f"{name} must be a [{B}, n] {dtype} tensor on cuda:{gpu}")
    rows, n = t.shape
    stride, step = t.stride()
    if rows != B or (n > 1 and step != 1):
        raise _bad(where, f"{name} must be a [{B}, n] {dtype} tensor on cuda:{gpu} with contiguous rows")
    return t.data_ptr(), stride if rows > 1 else n, n


_int = _float = _long = _byte = None  # torch's types, once torch is there


def _ready():
    global _int, _float, _long, _byte
    import torch
    c = _calls()
    c.adjust = _tam.lib().tam_adjust_logits
    _int, _float, _long, _byte = torch.int32, torch.float32, torch.int64, torch.uint8
    return c


def _stream(where, c, stream, gpu):
    """The HIP stream of a call on GPU number `gpu`, which has to be the current one, as the launch goes there."""
    if c.device() != gpu:
        raise _bad(where, f"the tensors lie on cuda:{gpu}, the current device is cuda:{c.device()}")
    if stream is None:
        return c.stream_of(gpu)
    if getattr(stream, "device_index", gpu) != gpu:
        raise _bad(where, f"the stream is of cuda:{stream.device_index}, the tensors lie on cuda:{gpu}")
    return stream.cuda_stream


def _adjust(logits, stream, handle=None, rows=None, ids=None, tokens=None, length=None, prompt=None, repetition=None,
            frequency=None, presence=None, bias_ids=None, bias=None):
    where = "tam_adjust_logits"
    c = _tam._calls_made if _int is not None else _ready()
    dtype = c.dtypes.get(logits.dtype)
    if dtype is None or not logits.is_cuda or logits.dim() != 2:
        raise _bad(where, "logits must be a [B, V] fp32 or bf16 tensor on the GPU")
    gpu = logits.get_device()
    hip_stream = _stream(where, c, stream, gpu)
    B, V = logits.shape
    row_stride, step = logits.stride()
    if V > 1 and step != 1:
        raise _bad(where, "logits must have contiguous rows")
    row_stride = row_stride if B > 1 else max(row_stride, V)
    raw = rows_p = ids_p = None
    num_rows = stride = 0
    if handle is not None:
        if rows is not None or handle._raw is None:
            raise _bad(where, "a handle and mask rows" if handle._raw else "the handle is closed")
        if not handle.host_only and handle.device.index != gpu:
            raise _bad(where, f"the handle lies on {handle.device}, the logits on cuda:{gpu}")
        if V < handle.vocab_size:
            raise _bad(where, f"logits have {V} columns, the vocabulary {handle.vocab_size} tokens")
        V, raw = handle.vocab_size, handle._raw
        ids_p = _int32(where, "node_ids", ids, B, gpu)
    elif rows is not None:
        if ids is None or rows.dim() != 2:
            raise _bad(where, "rows must be [R, words] and come with row_ids")
        rows_p, stride, width = _rows_of(where, "rows", rows, rows.shape[0], _long, gpu)
        num_rows = rows.shape[0]
        if width < (V + 63) // 64:
            raise _bad(where, f"rows must have {(V + 63) // 64} words")
        ids_p = _int32(where, "row_ids", ids, B, gpu)
        rows_p = rows_p or ids_p and ids_p & -8  # no rows at all have no memory, and none of it is read: nothing is valid
    elif ids is not None:
        raise _bad(where, "row_ids without rows")
    text_p, text_stride, history = (None, 0, 0) if tokens is None else _rows_of(where, "tokens", tokens, B, _int, gpu)
    floats = []
    for t in (repetition, frequency, presence):
        if t is None:
            floats.append(None)
            continue
        if t.dtype is not _float or t.get_device() != gpu or t.numel() != B or not t.is_contiguous():
            raise _bad(where, f"repetition, frequency and presence must be contiguous [{B}] fp32 tensors on cuda:{gpu}")
        floats.append(t.data_ptr())
    named_p, named_stride, named = (None, 0, 0) if bias_ids is None else _rows_of(where, "bias_ids", bias_ids, B, _int, gpu)
    bias_p, other, n = (None, 0, 0) if bias is None else _rows_of(where, "bias", bias, B, _float, gpu)
    if named_stride != other or named != n:
        raise _bad(where, "bias_ids and bias must have the same shape and strides")
    e = Edits(text_p, text_stride, history, None if length is None else _int32(where, "length", length, B, gpu),
              None if prompt is None else _int32(where, "prompt", prompt, B, gpu), *floats, named_p, bias_p, named_stride, named)
    rc = c.adjust(raw, rows_p, num_rows, stride, ids_p, ctypes.byref(e), B, V, logits.data_ptr(), dtype, row_stride, hip_stream)
    if rc != TAM_OK:
        _check(rc, where)
    return logits


def adjust_logits(logits, tokens=None, length=None, prompt=None, repetition=None, frequency=None, presence=None,
                  bias_ids=None, bias=None, rows=None, row_ids=None, stream=None):
    """Penalties for repeated tokens, biases and a mask on ``logits`` [B, V] (fp32 or
    bf16), in place.  A token ``v`` of row ``b`` that occurs in
    ``tokens[b, :length[b]]`` has its logit divided (multiplied where it is not
    positive) by ``repetition[b]``; ``frequency[b]`` is subtracted for each time it occurs
    after the first ``prompt[b]`` tokens, ``presence[b]`` once if it does; then the
    ``bias`` of the last entry of ``bias_ids[b]`` that names it is added.  Ids outside
    the vocabulary (-1 fills up rows) name no token.  ``rows`` [R, ceil(V/64)]: mask
    rows as ``export_rows`` gives them (int64); row ``b`` keeps the tokens of mask
    row ``row_ids[b]``, none when that is outside [0, R), and the others become -inf.
    Everything but ``logits`` is optional; ``Handle.adjust_logits`` takes the mask from
    a handle's nodes instead."""
    return _adjust(logits, stream, rows=rows, ids=row_ids, tokens=tokens, length=length, prompt=prompt,
                   repetition=repetition, frequency=frequency, presence=presence, bias_ids=bias_ids, bias=bias)


def _scratch(dtype, device, stream, *shape):
    """Memory for a call on ``stream``: from that stream's share of torch's allocator, so that
    nothing still running on another stream holds it."""
    import torch
    if stream is None:
        return torch.empty(*shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(*shape, dtype=dtype, device=device)


def top_tokens(logits, k, return_lse=False, stream=None):
    """The ``k`` (1 to 64) largest of each row of ``logits`` [B, V] (fp32 or bf16), as ``adjust_logits`` or ``apply_mask``
    leave them: (int32 [B, k] tokens, fp32 [B, k] log probabilities) in descending order, of equal logits the lowest token
    first, and with ``return_lse`` the fp32 [B] logarithms of the sums.  Where fewer than ``k`` logits are left (-inf is
    none), the rest is token -1 at -inf.  A NaN is larger than every number, and its row's log probabilities are NaN."""
    where = "tam_top_tokens"
    c = _tam._calls_made if _int is not None else _ready()
    dtype = c.dtypes.get(logits.dtype)
    if dtype is None or not logits.is_cuda or logits.dim() != 2:
        raise _bad(where, "logits must be a [B, V] fp32 or bf16 tensor on the GPU")
    gpu = logits.get_device()
    on = _stream(where, c, stream, gpu)
    B, V = logits.shape
    row_stride, step = logits.stride()
    if V > 1 and step != 1:
        raise _bad(where, "logits must have contiguous rows")
    row_stride = row_stride if B > 1 else V
    lib = _tam.lib()
    size = lib.tam_top_tokens_work(B, V, k, dtype)
    if size < 0:
        _check(-1, where)
    device = logits.device
    tokens, logprobs = _scratch(_int, device, stream, B, k), _scratch(_float, device, stream, B, k)
    lse = _scratch(_float, device, stream, B) if return_lse else None
    work = _scratch(_byte, device, stream, size) if size else None
    rc = lib.tam_top_tokens(logits.data_ptr(), dtype, B, V, row_stride, k, tokens.data_ptr(), logprobs.data_ptr(),
                            lse.data_ptr() if return_lse else None, work.data_ptr() if size else None, on)
    if rc != TAM_OK:
        _check(rc, where)
    return (tokens, logprobs, lse) if return_lse else (tokens, logprobs)


def tree_masks(parents, offsets=None, longest=None, stream=None):
    """Which tokens of its row each drafted token sees.  ``parents`` int32 [tokens]: the number, in its row, of the
    token that each one follows; -1 (or whatever is no earlier token of the row): the text before the row.  Row i is
    ``offsets[i]:offsets[i + 1]`` (one token per row without ``offsets``).  ``longest``: tokens of the longest row, or more, if the
    host knows (else all of them, and masks that grow with the square of the call's tokens): the width of the masks.  Returns (int64 [tokens, ceil(longest / 64)]: bit j % 64 of word
    j // 64 is set for the token itself and its ancestors, as ``PageCache.attend`` takes it; int32 [tokens]: how many ancestors,
    as ``PageCache.append`` takes it).  Tokens of no row are not written."""
    where = "tam_tree_masks"
    c = _tam._calls_made if _int is not None else _ready()
    if not parents.is_cuda:
        raise _bad(where, "parents must lie on the GPU")
    gpu = parents.get_device()
    on = _stream(where, c, stream, gpu)
    T = parents.numel()
    up = _int32(where, "parents", parents, T, gpu)
    rows, off = T, None
    if offsets is not None:
        rows = offsets.numel() - 1
        if rows < 0:
            raise _bad(where, "offsets must be [rows + 1]")
        off = _int32(where, "offsets", offsets, rows + 1, gpu)
    if longest is None:
        longest = T if offsets is not None else 1
    words = max(1, (longest + 63) // 64)
    device = parents.device
    seen, depth = _scratch(_long, device, stream, T, words), _scratch(_int, device, stream, T)
    rc = _tam.lib().tam_tree_masks(up, off, rows, T, seen.data_ptr(), words, depth.data_ptr(), on)
    if rc != TAM_OK:
        _check(rc, where)
    return seen, depth


class PageCache:
    """A paged K/V cache.

    ``data`` [2 * layers, pages, kv_heads, page_tokens, head_dim] (bf16 or fp16): plane
    2 l is layer l's K, plane 2 l + 1 its V.  ``table`` [slots, max_pages] int32, ``length``
    [slots] int32 and ``refs`` [pages] int32 are the sequences: token t of slot s lies in
    page ``table[s, t // page_tokens]``; ``refs`` counts the table entries that name a
    page, and a page at 0 is free.  The tensors are the caller's and change in
    place; the tables change on the device, and nothing here waits for it.
    """

    def __init__(self, data, table, length, refs):
        import torch
        where = "PageCache"
        if data.dim() != 5 or not data.is_cuda or data.dtype not in (torch.bfloat16, torch.float16):
            raise _bad(where, "data must be a [2 * layers, pages, kv_heads, page_tokens, head_dim] bf16 or fp16 "
                              "tensor on the GPU")
        planes, pages, kv, page, dim = data.shape
        if planes < 2 or planes % 2 or pages < 1 or not data[0, 0].is_contiguous():
            raise _bad(where, "data needs a K and a V plane per layer and contiguous pages")
        self._gpu = gpu = data.get_device()
        if table.dim() != 2 or table.dtype is not torch.int32 or table.get_device() != gpu or (
                table.shape[1] > 1 and table.stride(1) != 1):
            raise _bad(where, f"table must be a [slots, max_pages] int32 tensor on cuda:{gpu} with contiguous rows")
        slots, width = table.shape
        stride = table.stride(0) if slots > 1 else width
        self._calls = _tam._calls_made if _int is not None else _ready()
        length_p = _int32(where, "length", length, slots, gpu)
        refs_p = _int32(where, "refs", refs, pages, gpu)
        self.data, self.table, self.length, self.refs = data, table, length, refs
        self.layers, self.kv_heads, self.page_tokens, self.head_dim = planes // 2, kv, page, dim
        self._torch, self._device, self._dtype = torch, data.device, data.dtype
        size = data.element_size()
        self._pages = Pages(data.data_ptr(), planes, data.stride(0) * size, data.stride(1) * size, kv * page * dim * size,
                            pages, page, table.data_ptr(), slots, width, stride, length_p, refs_p)
        self._pages_ref = ctypes.byref(self._pages)
        dtype = DTYPE_FP16 if data.dtype is torch.float16 else DTYPE_BF16
        self._chunk = Chunk(None, None, data.stride(1), data.stride(2), data.stride(3), pages, page, kv, dim, dtype,
                            table.data_ptr(), slots, width, stride, length_p)
        self._lib = _tam.lib()
        self._work_bytes = self._lib.tam_pages_work(self._pages_ref, slots)  # enough for any call
        if self._work_bytes < 0:
            _check(-1, where)

    @classmethod
    def empty(cls, layers, kv_heads, head_dim, pages, slots, max_pages, page_tokens=16, dtype=None, device="cuda"):
        """A cache of ``pages`` free pages and ``slots`` empty sequences of at most ``max_pages`` pages."""
        import torch
        data = torch.empty((2 * layers, pages, kv_heads, page_tokens, head_dim), dtype=dtype or torch.bfloat16,
                           device=device)
        return cls(data, torch.full((slots, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(slots, dtype=torch.int32, device=device),
                   torch.zeros(pages, dtype=torch.int32, device=device))

    # -- pages -----------------------------------------------------------------
    def _empty(self, shape, dtype, stream):
        if stream is None:
            return self._torch.empty(shape, dtype=dtype, device=self._device)
        return _scratch(dtype, self._device, stream, shape)

    def _work(self, stream):
        return self._empty(self._work_bytes, self._torch.uint8, stream)

    def _on(self, where, stream):
        return _stream(where, self._calls, stream, self._gpu)

    def fork(self, slots, parents, lengths=None, stream=None):
        """Slot ``slots[i]`` becomes a copy of the first ``lengths[i]`` tokens (all of them without
        ``lengths``) of slot ``parents[i]`` as it was before the call; a parent outside the
        slots (-1) frees the slot.  Pages are shared, not copied."""
        where = "tam_pages_fork"
        n, gpu, on = slots.numel(), self._gpu, self._on(where, stream)
        s, p = _int32(where, "slots", slots, n, gpu), _int32(where, "parents", parents, n, gpu)
        keep = None if lengths is None else _int32(where, "lengths", lengths, n, gpu)
        work = self._work(stream)
        rc = self._lib.tam_pages_fork(self._pages_ref, s, p, keep, n, work.data_ptr(), on)
        if rc != TAM_OK:
            _check(rc, where)

    def free(self, slots, stream=None):
        """The slots' sequences end; pages that no other slot names are free."""
        self._on("tam_pages_fork", stream)
        parents = self._empty(slots.shape, slots.dtype, stream)
        if stream is None:
            parents.fill_(-1)
        else:
            with self._torch.cuda.stream(stream):
                parents.fill_(-1)
        self.fork(slots, parents, stream=stream)

    def extend(self, slots, counts, stream=None):
        """Room for ``counts[i]`` more tokens in slot ``slots[i]``, for all of them or for none;
        a shared, partly filled last page is copied first.  Returns int32 [4] on the GPU: 1 if done
        (else 0, and nothing has changed: ``store``, ``append``, ``attend`` and ``accept`` would take the sequences' last tokens
        for the new ones), pages needed, pages that were free, slots that ``max_pages`` is too small for."""
        where = "tam_pages_extend"
        n, gpu, on = slots.numel(), self._gpu, self._on(where, stream)
        s, c = _int32(where, "slots", slots, n, gpu), _int32(where, "counts", counts, n, gpu)
        work = self._work(stream)
        info = self._empty(4, self._torch.int32, stream)
        rc = self._lib.tam_pages_extend(self._pages_ref, s, c, n, info.data_ptr(), work.data_ptr(), on)
        if rc != TAM_OK:
            _check(rc, where)
        return info

    def compact(self, stream=None):
        """The pages in use move to the front of the pool.  Returns int32 [2] (pages in use,
        pages moved) and int32 [pages] (each page's new number, -1 of a free one), both on the GPU."""
        where = "tam_pages_compact"
        on = self._on(where, stream)
        work = self._work(stream)
        info = self._empty(2, self._torch.int32, stream)
        moved = self._empty(self.refs.shape, self._torch.int32, stream)
        rc = self._lib.tam_pages_compact(self._pages_ref, info.data_ptr(), moved.data_ptr(), work.data_ptr(), on)
        if rc != TAM_OK:
            _check(rc, where)
        return info, moved

    # -- a layer's new tokens ------------------------------------------------------
    def _new(self, where, layer, tokens, offsets, slots, longest):
        if not 0 <= layer < self.layers:
            raise _bad(where, f"layer {layer} of {self.layers}")
        c = Chunk.from_buffer_copy(self._chunk)  # a call's own: threads may share the cache
        if offsets is not None:
            rows = offsets.numel() - 1
            if rows < 0:
                raise _bad(where, "offsets must be [rows + 1]")
            c.offsets = _int32(where, "offsets", offsets, rows + 1, self._gpu)
        else:
            rows, c.offsets = tokens, None
        c.slot_ids = None if slots is None else _int32(where, "slots", slots, rows, self._gpu)
        plane = self._pages.plane_stride
        c.k = self._pages.data + 2 * layer * plane
        c.v = c.k + plane
        c.rows, c.tokens, c.longest = rows, tokens, (1 if offsets is None else 0) if longest is None else longest
        return ctypes.byref(c)

    def _vectors(self, where, name, t, heads=None):
        """(pointer, token stride, head stride) of a [tokens, heads, head_dim] tensor."""
        shape, strides = t.shape, t.stride()
        if (len(shape) != 3 or t.get_device() != self._gpu or t.dtype is not self._dtype or shape[2] != self.head_dim
                or strides[2] != 1 or (heads is not None and shape[1] != heads)):
            raise _bad(where, f"{name} must be a [tokens, {heads or 'heads'}, {self.head_dim}] {self.data.dtype} tensor "
                              f"on cuda:{self._gpu} with contiguous vectors")
        # of a single token or head any stride will do
        return t.data_ptr(), strides[0] if shape[0] > 1 else 0, strides[1] if shape[1] > 1 else 0

    def store(self, layer, k, v, offsets=None, slots=None, longest=None, stream=None):
        """K and V [tokens, kv_heads, head_dim] of the new tokens into their pages.  Row i's tokens are
        ``offsets[i]:offsets[i + 1]`` (one token per row without ``offsets``), the last ones of slot ``slots[i]``
        (slot i without ``slots``), whose length counts them already (``extend``)."""
        where = "tam_pages_store"
        on = self._on(where, stream)
        kp, vp = self._vectors(where, "k", k, self.kv_heads), self._vectors(where, "v", v, self.kv_heads)
        if k.shape[0] != v.shape[0]:
            raise _bad(where, "k and v have different numbers of tokens")
        rc = self._lib.tam_pages_store(self._new(where, layer, k.shape[0], offsets, slots, longest), *kp, *vp, on)
        if rc != TAM_OK:
            _check(rc, where)

    def append(self, layer, q, k, v, frequencies, depth=None, adjacent=False, offsets=None, slots=None, longest=None,
               out=None, stream=None):
        """``store`` of ``k`` and ``v`` with K turned by its tokens' positions; returns ``q`` [tokens, heads, head_dim] turned
        alike (into ``out``, which may be ``q``; ``q`` None: no queries).  ``frequencies`` fp32 [pairs]: pair i of a vector, its
        elements i and pairs + i, or with ``adjacent`` 2 i and 2 i + 1, turns by position * frequencies[i]; what follows the
        pairs (a multiple of 4) stays.  A token's position is its place in its sequence, or with ``depth`` int32 [tokens] that
        many after the place of its row's first token (``tree_masks``).  Tokens of no row are not written."""
        where = "tam_pages_append"
        on = self._on(where, stream)
        kp, vp = self._vectors(where, "k", k, self.kv_heads), self._vectors(where, "v", v, self.kv_heads)
        T = k.shape[0]
        qp = op = (None, 0, 0)
        heads = 0
        if v.shape[0] != T or (q is not None and q.shape[0] != T):
            raise _bad(where, "q, k and v have different numbers of tokens")
        if q is not None:
            qp, heads = self._vectors(where, "q", q), q.shape[1]
            if out is None:
                out = _scratch(self._dtype, self._device, stream, T, heads, self.head_dim)
                op = out.data_ptr(), heads * self.head_dim, self.head_dim
            elif out.shape != q.shape:
                raise _bad(where, "out must have q's shape")
            else:
                op = self._vectors(where, "out", out)
        elif out is not None:
            raise _bad(where, "out without q")
        if frequencies.dtype is not _float or frequencies.get_device() != self._gpu or frequencies.dim() != 1 or (
                not frequencies.is_contiguous()):
            raise _bad(where, f"frequencies must be a contiguous [pairs] fp32 tensor on cuda:{self._gpu}")
        turn = Rotation(frequencies.data_ptr(), frequencies.numel(), bool(adjacent),
                        None if depth is None else _int32(where, "depth", depth, T, self._gpu))
        rc = self._lib.tam_pages_append(self._new(where, layer, T, offsets, slots, longest), ctypes.byref(turn), *kp, *vp,
                                        *qp, heads, *op, on)
        if rc != TAM_OK:
            _check(rc, where)
        return out

    def attend(self, layer, q, offsets=None, slots=None, longest=None, scale=None, out=None, return_lse=False,
               stream=None, seen=None):
        """Attention of the new tokens' queries ``q`` [tokens, heads, head_dim] over their sequences, each over the
        tokens up to its own; ``heads`` is a multiple of ``kv_heads``.  Rows as for ``store``, whose tokens
        have been stored.  ``scale``: of the products (1 / sqrt(head_dim)).  ``longest``: the tokens of the longest
        row, or more, if the host knows (a hint that chooses the launch: give it with ``offsets`` where rows are short).
        ``seen`` int64 [tokens, words]: a token sees, of its row's tokens, those j whose bit j % 64 of word j // 64 is set
        (``tree_masks``; any will do), instead of those up to itself, and all that lies before the row's first one.
        The softmax and its sums are fp32; its weights are rounded to the cache's type before they meet V.
        Returns ``out`` (like ``q``; tokens of no row and the memory between are not written) and with ``return_lse``
        the fp32 [tokens, heads] logarithms of the sums."""
        where = "tam_attend" if seen is None else "tam_attend_seen"
        on = self._on(where, stream)
        qp = self._vectors(where, "q", q)
        T, heads = q.shape[0], q.shape[1]
        if out is None:
            out = _scratch(self._dtype, self._device, stream, T, heads, self.head_dim)
            op = out.data_ptr(), heads * self.head_dim, self.head_dim
        elif out.shape != q.shape:
            raise _bad(where, "out must have q's shape")
        else:
            op = self._vectors(where, "out", out)
        lse = _scratch(_float, self._device, stream, T, heads) if return_lse else None
        chunk = self._new(where, layer, T, offsets, slots, longest)
        lib = self._lib
        size = lib.tam_attend_work(chunk, heads)
        if size < 0:
            _check(-1, where)
        work = _scratch(_byte, self._device, stream, size) if size else None
        scale = self.head_dim ** -0.5 if scale is None else scale
        rest = *op, lse.data_ptr() if return_lse else None, work.data_ptr() if size else None, on
        if seen is None:
            rc = lib.tam_attend(chunk, *qp, heads, scale, *rest)
        else:
            bits, stride, words = _rows_of(where, "seen", seen, T, _long, self._gpu)
            rc = lib.tam_attend_seen(chunk, *qp, heads, scale, bits, words, stride, *rest)
        if rc != TAM_OK:
            _check(rc, where)
        return (out, lse) if return_lse else out

    # -- a tree of drafted tokens ----------------------------------------------------
    def accept(self, tokens, picks, parents, offsets=None, slots=None, longest=None, stream=None):
        """Of the new tokens' trees the path that the model's choices follow stays in the cache, in every layer.  Rows as for
        ``store``; ``tokens``, ``picks`` and ``parents`` int32 [tokens]: the drafted tokens, the choice after each, and their
        parents (as for ``tree_masks``).  A row's token 0 stays; after a token that stays, the first one that follows it and
        is its choice (below 0, as ``top_tokens`` gives where nothing is valid: none).  They move to the places behind the text before the row, the slot ends there, and pages past its
        end are given back.  Returns, on the GPU, int32 [tokens]: the numbers in the row of its tokens that stay, then -1
        (tokens of no row are not written); int32 [rows]: how many; int32 [rows]: the choice after the last one (-1 for an
        empty row)."""
        where = "tam_pages_accept"
        on = self._on(where, stream)
        T, gpu = tokens.numel(), self._gpu
        lists = [_int32(where, name, t, T, gpu) for name, t in (("tokens", tokens), ("picks", picks), ("parents", parents))]
        chunk = self._new(where, 0, T, offsets, slots, longest)
        rows = T if offsets is None else offsets.numel() - 1
        size = self._lib.tam_pages_accept_work(chunk)
        if size < 0:
            _check(-1, where)
        # one piece of memory, which costs the host less than four: the scratch, the path, the two lists
        words = (size + 15) // 16 * 4
        both = _scratch(_int, self._device, stream, words + T + 2 * rows)
        at = both.data_ptr()
        rc = self._lib.tam_pages_accept(self._pages_ref, chunk, *lists, at + 4 * words, at + 4 * (words + T),
                                        at + 4 * (words + T + rows), at, on)
        if rc != TAM_OK:
            _check(rc, where)
        return both.split((words, T, rows, rows))[1:]
