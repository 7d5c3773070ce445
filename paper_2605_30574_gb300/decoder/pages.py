"""A key/value cache of pages, held in 4 bits: rows into it and out of it,
attention over it, and its pages copied.

A ``PageCache`` holds, for every layer, pages of ``page`` tokens with all their kv
heads.  A row (one token's key or value of one head, of d elements) is kept as
whole numbers c between -7 and 7, with a scale for each 32 elements:

    A = max |x|,  E = floor(log2 A),  r = max(2^-14, (max of the 32 |x|) 2^(2 - E) / 7),
    s = r 2^(E - 2),  c = x / s,

r rounded to four significant bits and c to whole numbers (ties to even), so a value
is off by half of s at most.  Rows with A below 2^-100 are held as zeros; those with A
of 2^100 or more, an infinity or a NaN are NaN.  At 128 dims that is 69 bytes for the
256 of bf16.  c s is exact in bf16.

The calls take ``table`` [B][W], ``starts`` [B + 1] and ``lengths`` [B], int32 on the
cache's device: sequence b has ``lengths[b]`` tokens in the pages ``table[b]`` (behind
its last one the table may hold anything), and its newest tokens are the rows
``starts[b]`` to ``starts[b + 1]`` of what is stored, loaded or attends; one token
each is ``starts`` = 0 .. B.  The kernels read the three on the device, so a captured
graph goes by what they hold when it is replayed.  Rows before ``starts[0]`` and behind
``starts[B]`` are left as they are.  ``PageTables`` keeps them for sequences that share
pages.

Tensors are bf16, d 64, 128 or 256, pages of 16, 32, 64, 128 or 256 tokens; k, v and q
may have any strides (those that the kernels cannot read are copied).  Kernels go to
torch's current stream; tracers, which would not record them, are refused.  No
gradients: tensors that require one, where they are recorded, or that have a tangent are
refused.  The same inputs give the same bits.
"""
from __future__ import annotations

import ctypes
from array import array
from typing import Dict, Iterable, List, Optional, Sequence, Tuple, Union

import torch
import torch.autograd.forward_ad as _fwad

from . import BF16, _current_device, _launch, lib, there, untraced

_PAGES = {16: 4, 32: 5, 64: 6, 128: 7, 256: 8}
_U8, _I32 = torch.uint8, torch.int32


class _Described(ctypes.Structure):
    """A cache as the kernels' launches take it."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("codes", "ratios", "exponents")] + [
        (n, ctypes.c_int) for n in ("layers", "pages", "heads", "head_dim", "log_page")]


class PageCache:
    """The cache's tensors, uint8 and contiguous, on one CUDA device:

    * ``codes`` [layers][pages][2][heads][page][d / 2]: c + 8 in a nibble, the low one
      first; keys, then values.  In a key the 8 elements 32 i + 8 t come at place
      t d / 32 + i, in a value the 4 elements 32 i + 4 g at place g d / 32 + i;
    * ``ratios`` [layers][pages][2][heads][page][d / 32]: bits 14 to 7 of r in fp16;
    * ``exponents`` [layers][pages][heads][page][2]: E + 127 of key and value, 255 for
      a row of NaN.
    """

    def __init__(self, codes: torch.Tensor, ratios: torch.Tensor, exponents: torch.Tensor):
        what = "PageCache"
        for name, t, dims in (("codes", codes, 6), ("ratios", ratios, 6), ("exponents", exponents, 5)):
            if not isinstance(t, torch.Tensor) or t.dtype is not _U8:
                raise TypeError(f"{what}: {name} must be a uint8 tensor")
            if t.device.type != "cuda" or t.device != codes.device:
                raise ValueError(f"{what}: the tensors must be on one CUDA device")
            if t.dim() != dims or not t.is_contiguous() or there(what, name, t).data_ptr() & 15:
                raise ValueError(f"{what}: {name} must be contiguous, at a 16-byte boundary, of {dims} dimensions")
        layers, pages, two, heads, page, half = codes.shape
        if half not in (32, 64, 128) or page not in _PAGES or two != 2:
            raise ValueError(f"{what}: heads of 64, 128 or 256, and pages of {', '.join(map(str, _PAGES))} tokens")
        if not 1 <= heads <= 1024 or not 1 <= layers <= 65535 or not 1 <= pages < 1 << 31:
            raise ValueError(f"{what}: between 1 and 1024 heads, 1 and 65535 layers, and a page at least")
        if ratios.shape != (layers, pages, 2, heads, page, half // 16) or exponents.shape != (layers, pages, heads, page, 2):
            raise ValueError(f"{what}: ratios and exponents must be of the codes' sizes")
        self._hold(codes, ratios, exponents)
        with torch.cuda.device(codes.device):
            self._scratch = lib().decoder_page_attention_scratch(2 * half)
        if self._scratch < 0:
            raise RuntimeError(f"{what}: CUDA error {-self._scratch}")

    def _hold(self, codes, ratios, exponents):
        self.codes, self.ratios, self.exponents, self.device = codes, ratios, exponents, codes.device
        self.layers, self.pages, _, self.kv_heads, self.page, half = codes.shape
        self.head_dim = 2 * half
        self._places = codes.data_ptr(), ratios.data_ptr(), exponents.data_ptr()
        self._described = _Described(*self._places, self.layers, self.pages, self.kv_heads, self.head_dim, _PAGES[self.page])
        self._at = ctypes.addressof(self._described)

    @classmethod
    def empty(cls, layers: int, pages: int, kv_heads: int, head_dim: int, page: int = 64, device="cuda") -> "PageCache":
        """A cache whose pages hold anything."""
        if head_dim not in (64, 128, 256) or page not in _PAGES:
            raise ValueError(f"PageCache: heads of 64, 128 or 256, and pages of {', '.join(map(str, _PAGES))} tokens")
        one = (layers, pages, 2, kv_heads, page)
        return cls(*(torch.empty(s, dtype=_U8, device=device)
                     for s in ((*one, head_dim // 2), (*one, head_dim // 32), (layers, pages, kv_heads, page, 2))))

    @property
    def nbytes(self) -> int:
        return sum(t.numel() for t in (self.codes, self.ratios, self.exponents))

    def _layer(self, what: str, layer: int) -> int:
        """The address of the cache's description, for a layer that there is."""
        if not isinstance(layer, int) or not 0 <= layer < self.layers:
            raise ValueError(f"{what}: the cache has layers 0 to {self.layers - 1}")
        places = self.codes.data_ptr(), self.ratios.data_ptr(), self.exponents.data_ptr()
        if places != self._places:
            raise ValueError(f"{what}: the cache has {'other' if all(places) else 'no'} memory than it was made with")
        return self._at


def _where(what, cache, table, starts, lengths):
    """The three, as addresses, with the table's width and the sequences."""
    if not isinstance(cache, PageCache):
        raise TypeError(f"{what}: cache must be a PageCache")
    try:
        device, (B, W) = cache.device, table.shape
        if (table.dtype is starts.dtype is lengths.dtype is _I32 and table.device == device == starts.device and lengths.device == device
                and starts.shape == (B + 1,) and lengths.shape == (B,) and table.is_contiguous() and starts.is_contiguous()
                and lengths.is_contiguous() and not (table.is_neg() or starts.is_neg() or lengths.is_neg())):
            at = (table.data_ptr(), starts.data_ptr(), lengths.data_ptr(), W, B)
            if at[0] and at[1] and at[2] and W and not W >> 31 and not B >> 30:
                return at
    except (AttributeError, ValueError):
        pass
    for name, t, dims in (("table", table, 2), ("starts", starts, 1), ("lengths", lengths, 1)):
        if not isinstance(t, torch.Tensor) or t.dtype is not _I32:
            raise TypeError(f"{what}: {name} must be an int32 tensor")
        if t.device != cache.device:
            raise ValueError(f"{what}: {name} must be on the cache's device")
        if t.dim() != dims or not t.is_contiguous() or t.is_neg():
            raise ValueError(f"{what}: {name} must be contiguous, of {dims} dimension{'s' * (dims > 1)}")
        there(what, name, t)
    B, W = table.shape
    if starts.shape[0] != B + 1 or lengths.shape[0] != B:
        raise ValueError(f"{what}: of B sequences, table must be [B][W], starts [B + 1] and lengths [B]")
    if B and not W:
        raise ValueError(f"{what}: the table has no pages")
    if W >> 31 or B >> 30:
        raise ValueError(f"{what}: fewer than 2^31 pages to a sequence and 2^30 sequences")
    return (table.data_ptr(), starts.data_ptr(), lengths.data_ptr(), W, B)


def _bf16(what, name, t, cache, shape):
    """Where the kernels can read and write the tensor as it is: its address and its strides
    of token and head; else None."""
    if isinstance(t, torch.Tensor) and t.dtype is BF16 and t.shape == shape and t.device == cache.device:
        at = t.data_ptr()
        if at:
            token, head, one = t.stride()
            kernels = one == 1 and not (token | head | at >> 1) & 7 and not t.is_neg() and token < 1 << 38 and head < 1 << 38
            return (at, token, head) if kernels else None
    if not isinstance(t, torch.Tensor) or t.dtype is not BF16:
        raise TypeError(f"{what}: {name} must be a bf16 tensor")
    if t.device != cache.device:
        raise ValueError(f"{what}: {name} must be on the cache's device")
    if t.dim() != 3 or t.shape[-1] != cache.head_dim or (shape is not None and t.shape != shape):
        raise ValueError(f"{what}: {name} must be [tokens][heads][{cache.head_dim}]" + (f", here {tuple(shape)}" if shape else ""))
    there(what, name, t)


def _copied(t):
    """A copy that the kernels can read and write, and where it is."""
    t = t.resolve_neg().clone(memory_format=torch.contiguous_format)
    return t, (t.data_ptr(), *t.stride()[:2])


_increment = torch.autograd.graph.increment_version


def _written(*ts):
    # (inference tensors have no versions, and are passed over there)
    _increment(ts)


def _overlaps(t):
    """Whether two of its rows may lie in the same place."""
    sizes = sorted((s, n) for s, n in zip(t.stride(), t.shape) if n > 1)
    return any(s < (sizes[i - 1][0] * sizes[i - 1][1] if i else 1) for i, (s, _) in enumerate(sizes))


def _meet(a, b):
    """Whether the places from the first to the last of both have any in common."""
    (a0, a1), (b0, b1) = ((t.data_ptr(), t.data_ptr() + 2 * sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 2) for t in (a, b))
    return a.numel() > 0 and b.numel() > 0 and a0 < b1 and b0 < a1


def _apart(a, b):
    """Whether two tensors [tokens][heads][d] of one shape, each without places that overlap,
    have none in common: by their strides, if those are the same, else by their first and last
    places."""
    x, y = a.data_ptr(), b.data_ptr()
    if x > y:
        a, b, x, y = b, a, y, x
    shape, strides, gap = a.shape, a.stride(), (y - x) // 2
    (n, heads, d), (token, head, one) = shape, strides
    row = (heads - 1) * head + (d - 1) * one + 1
    if gap >= (n - 1) * token + row or (row <= gap <= token - row and b.stride() == strides):
        return True
    dims = sorted([(s, n) for s, n in zip(strides, shape) if n > 1])
    if dims != sorted([(s, n) for s, n in zip(b.stride(), shape) if n > 1]):
        return False

    def met(gap, i):
        # (what the smaller strides reach is less than this one)
        if i < 0:
            return gap == 0
        s, n = dims[i]
        return any(-n < j < n and met(gap - j * s, i - 1) for j in (gap // s, gap // s + 1))
    return not met(gap, len(dims) - 1)


def _underived(what, names, *ts):
    """Only tensors' values are read or written: those whose gradient or tangent would be lost
    are refused."""
    for name, t in zip(names, ts):
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{what}: {name} requires a gradient, and the call has none (detached, or under torch.no_grad())")
        if _fwad._current_level >= 0 and _fwad.unpack_dual(t).tangent is not None:
            raise ValueError(f"{what}: {name} has a tangent, and the call makes none")


def _target(what, name, t):
    if t.requires_grad or _fwad._current_level >= 0:
        _underived(what, [name], t)
    if t.is_inference() and not torch.is_inference_mode_enabled():
        raise ValueError(f"{what}: {name} is an inference tensor and is written to")
    if not t.is_contiguous() and t.numel() and _overlaps(t):
        raise ValueError(f"{what}: rows of {name} overlap")


def store_pages(cache: PageCache, layer: int, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, starts: torch.Tensor,
                lengths: torch.Tensor) -> None:
    """Rounds the newest tokens' keys and values, k and v [tokens][heads][d], to 4 bits
    into the layer's pages: those of sequence b take its last places below ``lengths[b]``.
    A token without a place (before position 0, behind the table's pages, or in a page
    that is none of the cache's) is left out.  Pages that are written to belong to one
    sequence each."""
    what = "store_pages"
    untraced(what)
    where = _where(what, cache, table, starts, lengths)
    rows = k.shape[0] if isinstance(k, torch.Tensor) and k.dim() else 0
    shape = (rows, cache.kv_heads, cache.head_dim)
    at_k, at_v = _bf16(what, "k", k, cache, shape), _bf16(what, "v", v, cache, shape)
    if k.requires_grad or v.requires_grad or _fwad._current_level >= 0:
        _underived(what, "kv", k, v)
    at = cache._layer(what, layer)
    if rows >= 1 << 31:
        raise ValueError(f"{what}: fewer than 2^31 tokens")
    if not rows or not where[-1]:
        return
    if cache.device.index != _current_device():
        with torch.cuda.device(cache.device):
            return store_pages(cache, layer, k, v, table, starts, lengths)
    if at_k is None:
        k, at_k = _copied(k)
    if at_v is None:
        v, at_v = _copied(v)
    _launch("decoder_page_rows", 0, at, layer, *at_k, *at_v, *where, rows)
    _written(cache.codes, cache.ratios, cache.exponents)


def load_pages(cache: PageCache, layer: int, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, starts: torch.Tensor,
               lengths: torch.Tensor) -> None:
    """Writes the values that the newest tokens are held as to k and v [tokens][heads][d]; with
    ``starts`` that go by the lengths, those of whole sequences.  A token before position 0 is
    zeros, one in a page that is none of the cache's, or behind the table's, NaN.  k and v have
    no place in common (with strides of their own, neither lies between the other's)."""
    what = "load_pages"
    untraced(what)
    where = _where(what, cache, table, starts, lengths)
    rows = k.shape[0] if isinstance(k, torch.Tensor) and k.dim() else 0
    shape = (rows, cache.kv_heads, cache.head_dim)
    at_k, at_v = _bf16(what, "k", k, cache, shape), _bf16(what, "v", v, cache, shape)
    _target(what, "k", k)
    _target(what, "v", v)
    at = cache._layer(what, layer)
    if rows >= 1 << 31:
        raise ValueError(f"{what}: fewer than 2^31 tokens")
    # (mostly one lies behind the other, which is seen from their places and strides)
    if rows and not (at_k and at_v and at_k[1:] == at_v[1:]
                     and abs(at_k[0] - at_v[0]) >= 2 * ((rows - 1) * at_k[1] + (cache.kv_heads - 1) * at_k[2] + cache.head_dim)) \
            and not _apart(k, v):
        raise ValueError(f"{what}: rows of k and v are in the same place")
    if not rows or not where[-1]:
        return
    if cache.device.index != _current_device():
        with torch.cuda.device(cache.device):
            return load_pages(cache, layer, k, v, table, starts, lengths)
    # (what the kernels cannot write to gets its rows by way of a copy)
    to, tv = k, v
    if at_k is None:
        to, at_k = _copied(k)
    if at_v is None:
        tv, at_v = _copied(v)
    _launch("decoder_page_rows", 1, at, layer, *at_k, *at_v, *where, rows)
    if k is to and v is tv:
        return _written(k, v)
    with torch.no_grad():
        for a, b in ((k, to), (v, tv)):
            _written(a) if a is b else a.copy_(b)


def page_attention(cache: PageCache, layer: int, q: torch.Tensor, table: torch.Tensor, starts: torch.Tensor,
                   lengths: torch.Tensor, *, scale: Optional[float] = None, window: int = 0,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the newest tokens' queries, q [tokens][Hq][d], over their sequences'
    keys and values, the newest tokens' own included (which are stored before): token i
    of the n newest of a sequence is at position p = length - n + i and sees those up to
    p, with ``window`` above 0 only those above p - window.  Query head h reads kv head
    h // (Hq / heads).  A token that sees nothing gives 0; one whose keys or values hold NaN,
    NaN.  A page that a row looks into and that is none of the cache's makes its tile's rows
    NaN, and a sequence longer than the table is wide all its rows.  ``scale`` is
    1 / sqrt(d) by default; scores, and ``scale`` times q, have to be below 2^127.

    Returns [tokens][Hq][d], bf16: ``out`` (contiguous) if given, else a new tensor whose
    rows outside of all sequences hold anything.  Scores and sums are in fp32, q to the
    bits of fp16 below 2^15 times its row's largest, weights in fp16."""
    what = "page_attention"
    untraced(what)
    where = _where(what, cache, table, starts, lengths)
    shape = q.shape if isinstance(q, torch.Tensor) else ()
    at_q = _bf16(what, "q", q, cache, shape if len(shape) == 3 and shape[2] == cache.head_dim else None)
    if q.requires_grad or _fwad._current_level >= 0:
        _underived(what, "q", q)
    rows, hq, d = shape
    if rows * hq >= 1 << 26:
        raise ValueError(f"{what}: fewer than 2^26 rows (tokens times heads)")
    if hq == 0 or hq % cache.kv_heads:
        raise ValueError(f"{what}: the query heads must be a multiple of the cache's {cache.kv_heads}")
    if not isinstance(window, int) or not 0 <= window < 1 << 31:
        raise ValueError(f"{what}: window must be a whole number, 0 (none) to 2^31 - 1")
    scale = d ** -0.5 if scale is None else float(scale)
    at = cache._layer(what, layer)
    if out is not None:
        _bf16(what, "out", out, cache, q.shape)
        _target(what, "out", out)
        if not out.is_contiguous() or out.is_neg() or out.data_ptr() & 15:
            raise ValueError(f"{what}: out must be contiguous, at a 16-byte boundary")
        if _meet(out, q):
            raise ValueError(f"{what}: out and q overlap")
    if cache.device.index != _current_device():
        with torch.cuda.device(cache.device):
            return page_attention(cache, layer, q, table, starts, lengths, scale=scale, window=window, out=out)
    y = torch.empty_like(q, memory_format=torch.contiguous_format) if out is None else out
    if not rows or not where[-1]:
        return y
    if at_q is None:
        q, at_q = _copied(q)
    args = at, layer, *at_q, *where, rows, hq, scale, window, y.data_ptr()
    # Short sequences take no scratch, whose allocation is 3 us of a call of 29, so that is
    # tried first where it is likely (in vain, it costs 2.5).
    most, short = where[3] * cache.page, False
    if most <= 512 or (most <= 2048 and where[4] * cache.kv_heads >= 128):
        short = _launch("decoder_page_attention", *args, None) is not False
    if not short:
        scratch = torch.empty(cache._scratch, dtype=_U8, device=q.device)
        _launch("decoder_page_attention", *args, scratch.data_ptr())
    if out is not None:
        _written(out)
    return y


def copy_pages(cache: PageCache, src: Sequence[int], dst: Sequence[int]) -> None:
    """Copies pages ``src[i]`` to ``dst[i]`` in all layers.  No page may be written twice,
    or written and read."""
    what = "copy_pages"
    untraced(what)
    if not isinstance(cache, PageCache):
        raise TypeError(f"{what}: cache must be a PageCache")
    n = len(src)
    if len(dst) != n:
        raise ValueError(f"{what}: as many pages to copy to as from")
    if n == 0:
        return
    ints = ctypes.c_int * n
    try:
        # (2000 pages: 68 us, 590 with ctypes' own conversion and Python's min, max and set)
        pages = ints.from_buffer(array("i", src)), ints.from_buffer(array("i", dst))
        refused = lib().decoder_page_copy_refused(*pages, n, cache.pages)
    except TypeError:
        raise TypeError(f"{what}: pages must be whole numbers") from None
    except OverflowError:
        refused = 1
    if refused == 1:
        raise ValueError(f"{what}: the cache has pages 0 to {cache.pages - 1}")
    if refused == 2:
        raise ValueError(f"{what}: a page is written twice, or written and read")
    if refused:
        raise MemoryError(f"{what}: {n} pages")
    at = cache._layer(what, 0)
    if cache.device.index != _current_device():
        with torch.cuda.device(cache.device):
            return copy_pages(cache, src, dst)
    _launch("decoder_page_copy", at, *pages, n)
    _written(cache.codes, cache.ratios, cache.exponents)


class PageTables:
    """Which pages of a cache hold which sequences, and how many tokens: kept on the host,
    by numbers that sequences are given.  Sequences may share pages.  A page that others hold
    too must not be written to: ``extend`` copies one that is begun, so that the tokens it
    gives may be stored, and ``tensors`` for a store refuses what lies in any other.

    The calls that copy pages do so on torch's current stream, in that order with the
    calls that read and write them; ``tensors`` gives what those take, as of then."""

    def __init__(self, cache: PageCache):
        if not isinstance(cache, PageCache):
            raise TypeError("PageTables: cache must be a PageCache")
        self.cache = cache
        self._users = [0] * cache.pages
        self._free = list(range(cache.pages - 1, -1, -1))
        self._pages: Dict[int, List[int]] = {}
        self._lengths: Dict[int, int] = {}
        self._next = 0

    def _known(self, what: str, ids) -> List[int]:
        ids = list(ids)
        for i in ids:
            if i not in self._pages:
                raise ValueError(f"PageTables.{what}: there is no sequence {i!r}")
        return ids

    @property
    def free(self) -> int:
        """Pages that no sequence holds."""
        return len(self._free)

    def length(self, sequence: int) -> int:
        return self._lengths[self._known("length", [sequence])[0]]

    def pages(self, sequence: int) -> Tuple[int, ...]:
        return tuple(self._pages[self._known("pages", [sequence])[0]])

    def _new(self, pages: List[int], length: int) -> int:
        self._next += 1
        self._pages[self._next], self._lengths[self._next] = pages, length
        for p in pages:
            self._users[p] += 1
        return self._next

    def _release(self, page: int) -> None:
        self._users[page] -= 1
        if not self._users[page]:
            self._free.append(page)

    def add(self, length: int = 0) -> int:
        """A new sequence with room for its first ``length`` tokens."""
        _whole("add", "length", length)
        n = -(-length // self.cache.page)
        if n > len(self._free):
            raise RuntimeError(f"PageTables.add: {n} pages, and {len(self._free)} are free")
        return self._new([self._free.pop() for _ in range(n)], length)

    def extend(self, sequences: Iterable[int], tokens: Union[int, Iterable[int]] = 1) -> None:
        """Makes the sequences longer, by as many tokens (one number, or one for each), which
        ``store_pages`` may then write.  A begun page that another sequence holds too is
        copied first.  With too few free pages nothing is done."""
        ids = self._known("extend", sequences)
        more = [tokens] * len(ids) if isinstance(tokens, int) else list(tokens)
        if len(set(ids)) != len(ids) or len(more) != len(ids):
            raise ValueError("PageTables.extend: each sequence once, and as many numbers of tokens as sequences")
        for n in more:
            _whole("extend", "tokens", n)
        page, left, copied, added = self.cache.page, {}, [], []
        for i, n in zip(ids, more):
            held, length = self._pages[i], self._lengths[i]
            if n and length % page:
                last = held[-1]
                users = left.get(last, self._users[last])
                if users > 1:                        # (the last of them keeps it)
                    copied.append((i, last))
                    left[last] = users - 1
            added.append(-(-(length + n) // page) - len(held))
        if len(copied) + sum(added) > len(self._free):
            raise RuntimeError(f"PageTables.extend: {len(copied) + sum(added)} pages, and {len(self._free)} are free")
        # (a copy that fails changes nothing either)
        dst = self._free[len(self._free) - len(copied):]
        copy_pages(self.cache, [last for _, last in copied], dst)
        del self._free[len(self._free) - len(copied):]
        for (i, last), to in zip(copied, dst):
            self._users[last] -= 1
            self._users[to] = 1
            self._pages[i][-1] = to
        for i, n, new in zip(ids, more, added):
            for _ in range(new):
                self._pages[i].append(self._free.pop())
                self._users[self._pages[i][-1]] = 1
            self._lengths[i] += n

    def fork(self, sequence: int, n: int = 1) -> List[int]:
        """``n`` sequences that hold what this one does; nothing is copied yet."""
        self._known("fork", [sequence])
        _whole("fork", "n", n)
        return [self._new(list(self._pages[sequence]), self._lengths[sequence]) for _ in range(n)]

    def splice(self, sequence: int, donor: int, tokens: int) -> None:
        """The sequence's first ``tokens`` become the donor's, by reference: whole pages
        that both have."""
        self._known("splice", [sequence, donor])
        _whole("splice", "tokens", tokens)
        n, odd = divmod(tokens, self.cache.page)
        if odd or tokens > min(self._lengths[sequence], self._lengths[donor]):
            raise ValueError(f"PageTables.splice: whole pages of {self.cache.page} tokens that both sequences have")
        if sequence == donor:
            return
        held, given = self._pages[sequence], self._pages[donor]
        for i in range(n):
            self._users[given[i]] += 1
            self._release(held[i])
            held[i] = given[i]

    def drop(self, sequences: Iterable[int]) -> None:
        """Gives the sequences up, and pages that no other holds."""
        ids = self._known("drop", sequences)
        if len(set(ids)) != len(ids):
            raise ValueError("PageTables.drop: each sequence once")
        for i in ids:
            for p in self._pages.pop(i):
                self._release(p)
            del self._lengths[i]

    def compact(self) -> int:
        """Moves the pages in use to the cache's first, and returns their number.  Tables
        that ``tensors`` gave before are of no use then."""
        used = [p for p, n in enumerate(self._users) if n]
        k = len(used)
        src = [p for p in used if p >= k]
        dst = [p for p in range(k) if not self._users[p]]
        to = dict(zip(src, dst))
        copy_pages(self.cache, src, dst)
        for p, q in to.items():
            self._users[q], self._users[p] = self._users[p], 0
        for i, held in self._pages.items():
            self._pages[i] = [to.get(p, p) for p in held]
        self._free = list(range(self.cache.pages - 1, k - 1, -1))
        return k

    def tensors(self, sequences: Iterable[int], new: Union[None, int, Iterable[int]] = 1,
                width: int = 0, store: bool = False) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """``table``, ``starts`` and ``lengths`` of the sequences on the cache's device, of
        which the ``new`` last tokens are stored, loaded or attend (one number, or one for
        each; None: all).  The table has ``width`` columns, or as many more as it needs.
        With ``store`` new tokens whose page another sequence holds too are refused, and a
        sequence that is named twice: tables that a call stores by are to be asked for so."""
        ids = self._known("tensors", sequences)
        lengths = [self._lengths[i] for i in ids]
        new = lengths if new is None else [new] * len(ids) if isinstance(new, int) else list(new)
        if len(new) != len(ids) or any(not isinstance(n, int) or not 0 <= n <= m for n, m in zip(new, lengths)):
            raise ValueError("PageTables.tensors: as many new tokens as each sequence has, at most")
        if store:
            if len(set(ids)) != len(ids):
                raise ValueError("PageTables.tensors: each sequence once, for a store")
            for i, n, length in zip(ids, new, lengths):
                if n and max([self._users[p] for p in self._pages[i][(length - n) // self.cache.page:]]) > 1:
                    raise ValueError(f"PageTables.tensors: sequence {i}'s last {n} tokens lie in a page that another sequence holds too")
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        width = max([1, width] + [len(self._pages[i]) for i in ids])
        flat, none, B = array("i"), array("i", [-1]), len(ids)
        for i in ids:
            flat.extend(self._pages[i])
            flat += none * (width - len(self._pages[i]))
        flat.extend(starts + lengths)
        t = torch.frombuffer(flat, dtype=_I32).to(self.cache.device)
        return t[:B * width].view(B, width), t[B * width:B * width + B + 1], t[B * width + B + 1:]


def _whole(what, name, n):
    if not isinstance(n, int) or n < 0:
        raise ValueError(f"PageTables.{what}: {name} must be a whole number, 0 or more")
