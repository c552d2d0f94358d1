"""Operators on a filled pool: new tokens, attention over cached sequences, accepted drafts, and eviction.

:class:`CacheSession` keeps the C handles of one batch of cached sequences together, as
:class:`~paper_2408_08147_b200.session.TransferSession` does for a transfer.  It marshals
arguments and allocates outputs and scratch with torch; every number is computed by the
library's kernels.

    seqs = Sequences(seq_len, tbl_off, tbl)                       # the decode side's tables
    with CacheSession(geom, pool_t, seqs, num_q_heads=32) as s:
        out, lse = s.attend(layer, q, scores_t=scores)            # scores accumulate in place
        kept, _, new_len = s.evict(s, scores_all, budget=1024, sink=4, recent=256,
                                   kept_scores_t=scores_all)      # compacts the pool in place

A step that drafts a tree of tokens (``lens_t`` counts them):

        q = s.append(layer, k, v, q, rotary=Rotary(128), position_t=positions, seq_len_t=lens_t)
        out, lse = s.attend(layer, q, mask_t=pack_mask(sees), seq_len_t=lens_t)
        lens_t = s.accept(path, seq_len_t=lens_t)                 # behind the last layer
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional, Sequence, Tuple

import numpy as np
import torch

from . import binding as B

# the handle of torch's current stream, without the Stream object around it where this torch has that call
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)

_NO_STRIDE, _NO_ROTARY = (0, 0, 0), (0, 0, 1, 0, 0, 1.0)
_DTYPES = {torch.bfloat16: B.PDKV_DTYPE_BF16, torch.float16: B.PDKV_DTYPE_FP16}


@dataclass
class Sequences:
    """Cached sequences of a batch (see ``pdkv_seqs_desc``): own tokens in CSR block tables,
    optionally behind shared prefixes (``seq_prefix[r]``: index of the prefix, -1 for none)."""

    seq_len: Sequence[int]
    tbl_off: np.ndarray
    tbl: np.ndarray
    prefix_len: Optional[Sequence[int]] = None
    prefix_tbl_off: Optional[np.ndarray] = None
    prefix_tbl: Optional[np.ndarray] = None
    seq_prefix: Optional[Sequence[int]] = None

    def __post_init__(self):
        def arr(a, dt):
            return None if a is None else np.ascontiguousarray(a, dt)

        self.seq_len, self.tbl_off, self.tbl = arr(self.seq_len, np.int32), arr(self.tbl_off, np.int64), arr(self.tbl, np.int32)
        self.prefix_len, self.seq_prefix = arr(self.prefix_len, np.int32), arr(self.seq_prefix, np.int32)
        self.prefix_tbl_off, self.prefix_tbl = arr(self.prefix_tbl_off, np.int64), arr(self.prefix_tbl, np.int32)
        n = int(self.seq_len.shape[0])
        if self.tbl_off.shape != (n + 1,):
            raise ValueError("tbl_off needs one entry more than seq_len")
        if n and self.tbl_off[-1] > self.tbl.shape[0]:
            raise ValueError("tbl is shorter than tbl_off says")
        if self.prefix_len is not None and self.prefix_len.size:
            if self.prefix_tbl_off is None or self.prefix_tbl is None or self.seq_prefix is None:
                raise ValueError("prefixes need prefix_tbl_off, prefix_tbl and seq_prefix")
            if self.prefix_tbl_off.shape != (self.prefix_len.shape[0] + 1,) or self.seq_prefix.shape != (n,):
                raise ValueError("prefix_tbl_off / seq_prefix do not match the lengths")
            if self.prefix_tbl_off[-1] > self.prefix_tbl.shape[0]:
                raise ValueError("prefix_tbl is shorter than prefix_tbl_off says")

    @property
    def n_seq(self) -> int:
        return int(self.seq_len.shape[0])

    @property
    def max_len(self) -> int:
        return int(self.seq_len.max()) if self.n_seq else 0


def pack_mask(see_t):
    """Words for ``mask_t`` of :meth:`CacheSession.attend` from truth values ``[..., query, newest token]``: bit ``j % 32`` of int32 word ``j // 32``."""
    *lead, n = see_t.shape
    words = (n + 31) // 32
    bits = torch.zeros((*lead, words * 32), dtype=torch.int64, device=see_t.device)
    bits[..., :n] = see_t
    weights = torch.ones(32, dtype=torch.int64, device=see_t.device) << torch.arange(32, device=see_t.device)
    return (bits.unflatten(-1, (words, 32)) * weights).sum(-1).to(torch.int32)


class Rotary:
    """Rotation of heads by position (see ``pdkv_rotary``), laid out once on the device.

    ``dims`` of a head turn, from the first; ``frequencies`` are radians per position, one for each pair of dims (default:
    ``base ** (-2 i / dims)``).  ``adjacent``: pairs ``(2i, 2i + 1)`` instead of ``(i, i + dims / 2)``.  ``axes``: the axis whose position
    turns each pair, for positions in time, height and width (``np.repeat(range(3), (16, 24, 24))``).  ``scale``: factor of the dims that turn.
    """

    def __init__(self, dims: int, *, base: float = 10000.0, frequencies=None, adjacent: bool = False, axes=None, scale: float = 1.0, device="cuda"):
        if dims < 2 or dims % 2:
            raise ValueError(f"dims: expected an even number of at least 2, got {dims}")
        pairs = dims // 2
        if frequencies is None:
            frequencies = float(base) ** (-np.arange(pairs, dtype=np.float64) / pairs)
        frequencies = np.asarray(frequencies, np.float64)
        if frequencies.shape != (pairs,):
            raise ValueError(f"frequencies: expected {pairs}, got the shape {frequencies.shape}")
        self.dims, self.adjacent, self.scale, self.n_axes = dims, bool(adjacent), float(scale), 1
        self.turns_t = torch.from_numpy(B.pdkv_rotary_turns(frequencies).view(np.int64)).to(device)
        self.axis_t = None
        if axes is not None:
            axes = np.asarray(axes, np.int64)
            if axes.shape != (pairs,) or axes.min() < 0 or axes.max() > 255:
                raise ValueError(f"axes: expected {pairs} axes from 0 to 255")
            self.n_axes = int(axes.max()) + 1
            self.axis_t = torch.from_numpy(axes.astype(np.uint8)).to(device)
        # of pdkv_rotary, in order
        self.fields = (dims, int(self.adjacent), self.n_axes, self.turns_t.data_ptr(), self.axis_t.data_ptr() if self.n_axes > 1 else 0, B.float32(self.scale))
        self.device = self.turns_t.device


class CacheSession:
    """Pool handle + sequence handle of one batch.

    ``pool_t`` is the torch CUDA tensor that holds the pool described by ``geom``.  With
    ``num_q_heads`` the session attends; ``dtype`` (torch.bfloat16 or torch.float16) is the type
    of K, V, q and out and defaults to the pool's own; it is needed for a pool that is held as bytes or words.  Scratch is allocated once and kept: calls
    of one session are meant for one stream at a time (pass ``scratch_t`` for others).
    ``stream`` None means torch's current stream of the pool's device at each call.  What a call
    allocates comes from torch's current stream and is recorded on the stream that it runs on, so its
    memory is not given away before the call has run; that stream has to live as long as the tensors.
    """

    def __init__(self, geom, pool_t, seqs: Sequences, *, num_q_heads: int = 0, q_tokens: int = 1, dtype=None,
                 stream: Optional[int] = None, workspace_t=None):
        self.geom, self.pool_t, self.seqs = geom, pool_t, seqs
        self.num_q_heads, self.q_tokens, self.stream = num_q_heads, q_tokens, stream
        self.pool = self.handle = None
        self._scratch = [None, None]   # without and with scores; never replaced, recorded graphs may hold them
        self._scratch_stream = [0, 0]  # torch's current stream when they were allocated
        if dtype is None:
            dtype = pool_t.dtype if pool_t.dtype in _DTYPES else torch.bfloat16
        if dtype not in _DTYPES:
            raise ValueError("attention takes bfloat16 or float16")
        self._kv_heads = geom.num_kv_heads
        self._other_type = pool_t.dtype in _DTYPES and dtype != pool_t.dtype
        if num_q_heads and self._other_type:
            raise ValueError(f"the pool holds {pool_t.dtype}, not {dtype}")
        if not pool_t.is_contiguous():
            raise ValueError("the pool tensor has to be contiguous")
        self.dtype = dtype
        self._device, self._index = pool_t.device, pool_t.device.index or 0
        try:
            self.pool = B.pdkv_pool_create(B.desc_of(geom), pool_t.data_ptr(), pool_t.numel() * pool_t.element_size(),
                                           pool_t.device.index or 0)
            self.handle, self.workspace_bytes = B.pdkv_seqs_create(
                self.pool, seqs.seq_len, seqs.tbl_off, seqs.tbl, seqs.prefix_len, seqs.prefix_tbl_off, seqs.prefix_tbl,
                seqs.seq_prefix, num_q_heads, q_tokens if num_q_heads else 0,
                _DTYPES[dtype],
                workspace_t.data_ptr() if workspace_t is not None else 0,
                workspace_t.numel() * workspace_t.element_size() if workspace_t is not None else 0,
                self._on(None))
            self.workspace_t = workspace_t
            self._need = [B.pdkv_attend_scratch(self.handle, w) if num_q_heads else 0 for w in (False, True)]
            self._shape = (seqs.n_seq, q_tokens, num_q_heads, geom.head_dim)
            self._max_len = seqs.max_len
            self._scale = geom.head_dim ** -0.5
            n, t, h, d = self._shape
            dense = [t * h * d, h * d, d]
            self._lse_stride = (t * h, h, 1)
            # argument block of the plain call: dense q and out, the default scale
            self._plain = B.pdkv_attend_args(q_stride=(*dense,), out_stride=(*dense,), scale=self._scale)
        except Exception:
            self.close()
            raise

    def _on(self, stream: Optional[int]) -> int:
        if stream is not None:
            return stream
        if self.stream is not None:
            return self.stream
        return self._on_current()

    def _on_current(self) -> int:
        return _current_stream(self._index) if self.pool_t.is_cuda else 0

    def _record(self, stream: int, *tensors) -> None:
        """The caching allocator hands a freed block to the next request on the stream it was allocated for: tell it of
        the other stream that uses these."""
        if self.pool_t.is_cuda:
            user = torch.cuda.ExternalStream(stream, self._device)
            for t in tensors:
                t.record_stream(user)

    def _check(self, name, t, dtype, shape):
        if t.dtype != dtype or t.shape != shape or t.device != self._device:
            raise ValueError(f"{name}: expected {dtype} {tuple(shape)} on {self._device}, "
                             f"got {t.dtype} {tuple(t.shape)} on {t.device}")

    def _lens(self, seq_len_t):
        if seq_len_t is None:
            return 0
        self._check("seq_len_t", seq_len_t, torch.int32, (self.seqs.n_seq,))
        if not seq_len_t.is_contiguous():
            raise ValueError("seq_len_t has to be contiguous")
        return seq_len_t.data_ptr()

    def _rows(self, name, t, lead, least):
        """fp32 rows over tokens: shape (*lead, width) with adjacent tokens."""
        shape = t.shape
        if t.dtype != torch.float32 or t.device != self._device or shape[:-1] != lead or shape[-1] < least:
            raise ValueError(f"{name}: expected float32 {lead} x at least {least} tokens on {self._device}, "
                             f"got {t.dtype} {tuple(shape)} on {t.device}")
        if shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: tokens have to be adjacent")

    def scratch_bytes(self, with_scores: bool = False) -> int:
        return self._need[bool(with_scores)]

    def attend(self, layer: int, q_t, *, scale: Optional[float] = None, out_t=None, lse_t=None, scores_t=None,
               scores_in_t=None, seq_len_t=None, scratch_t=None, stream: Optional[int] = None, cap: Optional[float] = None, slopes_t=None,
               mask_t=None, n_new_t=None, offset_t=None):
        """Attention of one layer; ``q_t`` is ``[n_seq, q_tokens, num_q_heads, head_dim]`` (any strides with
        adjacent dims).  Returns ``(out, lse)``.  With ``scores_t`` (float32 ``[n_seq, num_kv_heads, >= longest]``)
        the attention weights of the own tokens are added to it, or to ``scores_in_t`` and the sums
        stored in ``scores_t``.  ``seq_len_t``: current own lengths (int32, device).  There is no backward pass: a
        ``q_t`` that asks for a gradient is refused.

        Other forms than plain causal (``pdkv_attend_form``): ``cap`` turns logits into ``cap * tanh(logit / cap)``; ``slopes_t`` (float32
        ``[num_q_heads]``) adds slope times the position of the key minus that of the query; ``mask_t`` (int32 ``[n_seq, q_tokens, words]``, see
        :func:`pack_mask`; expanded along the batch where all share it) says which of the newest tokens a query token sees: a drafted tree,
        documents in a chunk, a prefix seen both ways; only ``n_new_t[r]`` (int32 ``[n_seq]``) of the ``q_tokens`` are there; ``offset_t`` (int32
        ``[n_seq, q_tokens]``): positions of the newest tokens counted from their first, where they are not 0, 1, 2 ... (with ``slopes_t``)."""
        shape = self._shape
        made = []
        self._check("q_t", q_t, self.dtype, shape)
        if q_t.requires_grad and torch.is_grad_enabled():
            raise ValueError("q_t: attention over a cache has no gradient; detach it or call under torch.no_grad()")
        a = B.pdkv_attend_args.from_buffer_copy(self._plain)
        dense = q_t.is_contiguous()
        if not dense:
            stride = q_t.stride()
            if shape[3] > 1 and stride[3] != 1:
                raise ValueError("q_t: the dims of a head have to be adjacent")
            a.q_stride = stride[:3]
        if out_t is None:
            out_t = torch.empty_like(q_t) if dense else torch.empty(shape, dtype=self.dtype, device=self._device)
            made.append(out_t)
        else:
            self._check("out_t", out_t, self.dtype, shape)
            stride = out_t.stride()
            if shape[3] > 1 and stride[3] != 1:
                raise ValueError("out_t: the dims of a head have to be adjacent")
            a.out_stride = stride[:3]
        if lse_t is None:
            lse_t = torch.empty_strided(shape[:3], self._lse_stride, dtype=torch.float32, device=self._device)   # (quicker than empty)
            made.append(lse_t)
        else:
            self._check("lse_t", lse_t, torch.float32, shape[:3])
            if not lse_t.is_contiguous():
                raise ValueError("lse_t has to be contiguous")
        a.q, a.out, a.lse = q_t.data_ptr(), out_t.data_ptr(), lse_t.data_ptr()
        if scale is not None:
            a.scale = scale
        if seq_len_t is not None:
            a.seq_len = self._lens(seq_len_t)
        if scores_t is not None:
            lead = (shape[0], self.geom.num_kv_heads)
            scores_in_t = scores_t if scores_in_t is None else scores_in_t
            self._rows("scores_t", scores_t, lead, self._max_len)
            self._rows("scores_in_t", scores_in_t, lead, self._max_len)
            a.scores_in, a.scores_out = scores_in_t.data_ptr(), scores_t.data_ptr()
            a.scores_in_stride, a.scores_out_stride = scores_in_t.stride()[:2], scores_t.stride()[:2]
        elif scores_in_t is not None:
            raise ValueError("scores_in_t needs scores_t to receive the sums")
        home = self._on_current()
        stream = home if stream is None and self.stream is None else self._on(stream)
        if scratch_t is None:
            which = scores_t is not None
            scratch_t = self._scratch[which]
            if scratch_t is None:
                scratch_t = self._scratch[which] = torch.empty(max(self._need[which], 16), dtype=torch.uint8, device=self._device)
                self._scratch_stream[which] = home
            if stream != self._scratch_stream[which]:
                self._record(stream, scratch_t)
            size = scratch_t.numel()
        else:
            size = scratch_t.numel() * scratch_t.element_size()
        if stream != home:
            self._record(stream, *made)
        if cap is None and slopes_t is None and mask_t is None and n_new_t is None and offset_t is None:
            B.pdkv_attend(self.handle, layer, a, scratch_t.data_ptr(), size, stream)
        else:
            B.pdkv_attend_formed(self.handle, layer, a, self._form(cap, slopes_t, mask_t, n_new_t, offset_t), scratch_t.data_ptr(), size, stream)
        return out_t, lse_t

    def _form(self, cap, slopes_t, mask_t, n_new_t, offset_t):
        n, T, Hq, _ = self._shape
        slopes = mask = n_new = offset = row = 0
        stride = (0, 0)
        if cap is None:
            cap = 0.0
        elif not cap > 0:
            raise ValueError(f"cap: expected a positive number, got {cap}")
        else:
            cap = B.float32(cap)
        if slopes_t is not None:
            slopes = self._weights("slopes_t", slopes_t, Hq)
        if mask_t is not None:
            self._check("mask_t", mask_t, torch.int32, (n, T, (T + 31) // 32))
            stride = mask_t.stride()
            if T > 32 and stride[2] != 1:
                raise ValueError("mask_t: the words of a query token have to be adjacent")
            mask = mask_t.data_ptr()
        if n_new_t is not None:
            n_new = self._ints("n_new_t", n_new_t, (n,))
        if offset_t is not None:
            if slopes_t is None:
                raise ValueError("offset_t needs slopes_t")
            self._check("offset_t", offset_t, torch.int32, (n, T))
            if T > 1 and offset_t.stride(1) != 1:
                raise ValueError("offset_t: the tokens of a sequence have to be adjacent")
            offset, row = offset_t.data_ptr(), offset_t.stride(0)
        return B.attend_form(cap, slopes, mask, stride[0], stride[1], n_new, offset, row)

    def _heads(self, name, t, shape):
        """Strides between sequences, rows and heads of a tensor [sequences, rows, heads, head_dim] or [rows, heads, head_dim]."""
        if t.shape != shape or t.dtype is not self.dtype or t.device != self._device:
            raise ValueError(f"{name}: expected {self.dtype} {shape} on {self._device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        stride = t.stride()
        if stride[-1] != 1 and shape[-1] > 1 and t.numel():
            raise ValueError(f"{name}: the dims of a head have to be adjacent")
        return stride[:3] if len(shape) == 4 else (0, stride[0], stride[1])

    def _weights(self, name, t, n):
        """Device address of n float32 numbers."""
        self._check(name, t, torch.float32, (n,))
        if n > 1 and t.stride(0) != 1:
            raise ValueError(f"{name} has to be contiguous")
        return t.data_ptr()

    def _ints(self, name, t, shape):
        """Device address of a dense int32 tensor."""
        if t.dtype is not torch.int32 or t.shape != shape or t.device != self._device or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous int32 {shape} on {self._device}, got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")
        return t.data_ptr()

    def append(self, layer: int, k_t, v_t, q_t=None, *, q_out_t=None, rotary: Optional[Rotary] = None, position_t=None, q_norm_t=None,
               k_norm_t=None, eps: float = 1e-6, seq_len_t=None, n_new_t=None, row_begin_t=None, stream: Optional[int] = None):
        """New tokens enter the cache of one layer.  ``k_t`` and ``v_t`` are ``[n_seq, new, num_kv_heads, head_dim]`` (of which the first
        ``n_new_t[r]`` count), or ``[rows, num_kv_heads, head_dim]`` with the sequences' rows one after the other at ``row_begin_t``
        (int32 ``[n_seq + 1]``); any strides with adjacent dims.  The lengths (the session's, or ``seq_len_t``) count the new tokens, which become
        the last ones; behind the session's lengths there is no place: where ``seq_len_t`` is above them, the new tokens replace the last cached
        ones, and :meth:`status` raises.  ``q_t`` (as ``k_t``, with the query heads) is returned normalised and rotated, in ``q_out_t`` (which may be ``q_t``).
        Keys and queries are divided by their root mean square and multiplied by ``k_norm_t`` / ``q_norm_t`` (float32 ``[head_dim]``) where
        given, then turned by ``rotary`` at ``position_t`` (int32, one for each row, ``[axes, rows]`` for several axes; default: where the token
        stands in the cache behind its prefix, which an eviction changes).  There is no backward pass.  (:meth:`attend` takes ``[n_seq, q_tokens, ...]``: rows
        that came one after the other are spread out by the caller.)"""
        n_seq, _, _, D = self._shape
        if self._other_type:
            raise ValueError(f"the pool holds {self.pool_t.dtype}, not {self.dtype}")
        packed = row_begin_t is not None
        if packed:
            rows = k_t.shape[0]
            lead = (rows,)
        else:
            lead = (n_seq, k_t.shape[1] if len(k_t.shape) == 4 else 0)
            rows = n_seq * lead[1]
        shape = (*lead, self._kv_heads, D)
        k_stride, v_stride = self._heads("k_t", k_t, shape), self._heads("v_t", v_t, shape)
        if (k_t.requires_grad or v_t.requires_grad or (q_t is not None and q_t.requires_grad)) and torch.is_grad_enabled():
            raise ValueError("entering a cache has no gradient; detach the tensors or call under torch.no_grad()")
        home = self._on_current()
        stream = home if stream is None and self.stream is None else self._on(stream)
        q = q_out = 0
        q_stride = q_out_stride = _NO_STRIDE
        if q_t is not None:
            if not self.num_q_heads:
                raise ValueError("q_t: the session has no query heads")
            shape = (*lead, self.num_q_heads, D)
            q_stride = self._heads("q_t", q_t, shape)
            if q_out_t is None:
                q_out_t = torch.empty_like(q_t)
                q_out_stride = q_out_t.stride()
                q_out_stride = (0, q_out_stride[0], q_out_stride[1]) if packed else q_out_stride[:3]
                if stream != home:
                    self._record(stream, q_out_t)
            else:
                q_out_stride = self._heads("q_out_t", q_out_t, shape)
            q, q_out = q_t.data_ptr(), q_out_t.data_ptr()
        elif q_out_t is not None:
            raise ValueError("q_out_t needs q_t")
        row_begin = n_new = seq_len = position = q_norm = k_norm = 0
        if packed:
            row_begin = self._ints("row_begin_t", row_begin_t, (n_seq + 1,))
            if n_new_t is not None:
                raise ValueError("n_new_t does not go with row_begin_t")
        elif n_new_t is not None:
            n_new = self._ints("n_new_t", n_new_t, (n_seq,))
        if seq_len_t is not None:
            seq_len = self._ints("seq_len_t", seq_len_t, (n_seq,))
        if q_norm_t is not None:
            q_norm = self._weights("q_norm_t", q_norm_t, D)
        if k_norm_t is not None:
            k_norm = self._weights("k_norm_t", k_norm_t, D)
        turn = _NO_ROTARY
        if rotary is not None:
            if rotary.device != self._device:
                raise ValueError(f"rotary: laid out on {rotary.device}, the pool is on {self._device}")
            turn = rotary.fields
            if position_t is not None:
                position = self._ints("position_t", position_t, (rotary.n_axes, rows) if rotary.n_axes > 1 else (rows,))
            elif rotary.n_axes > 1:
                raise ValueError("rotary: several axes need position_t")
        elif position_t is not None:
            raise ValueError("position_t needs rotary")
        a = B.append_args(rows, row_begin, n_new, seq_len, q, k_t.data_ptr(), v_t.data_ptr(), q_out, *q_stride, *k_stride, *v_stride, *q_out_stride, q_norm, k_norm, B.float32(eps),
                          position, rows, *turn)
        B.pdkv_append(self.handle, layer, a, stream)
        return q_out_t

    def accept(self, path_t, *, n_new_t=None, new_tokens: Optional[int] = None, seq_len_t=None, new_len_t=None,
               layers: Optional[Tuple[int, int]] = None, stream: Optional[int] = None):
        """Of the newest tokens of each sequence (``new_tokens``, default: the session's ``q_tokens``; ``n_new_t[r]`` of them are there) those named by
        ``path_t`` (int32 ``[n_seq, path]``, ascending, -1 behind the last) stay: their keys and values move to the place behind the tokens
        before the newest, in all layers.  Returns the new lengths (``new_len_t`` may be ``seq_len_t``).  Accumulated weights do not move: of the
        ``scores_t`` of :meth:`attend`, entry ``len - new + path[j]`` of each row has to go to ``len - new + j``, and zeros behind, before an eviction
        goes by them."""
        l0, l1 = (0, self.geom.num_layers) if layers is None else layers
        if not 0 <= l0 < l1 <= self.geom.num_layers:
            raise ValueError(f"layers: expected a range within [0, {self.geom.num_layers}), got {layers}")
        n_seq = self._shape[0]
        shape, stride = path_t.shape, path_t.stride()
        if path_t.dtype is not torch.int32 or len(shape) != 2 or shape[0] != n_seq or path_t.device != self._device:
            raise ValueError(f"path_t: expected int32 [{n_seq}, path] on {self._device}, got {path_t.dtype} {tuple(shape)} on {path_t.device}")
        if shape[1] > 1 and stride[1] != 1:
            raise ValueError("path_t: the entries of a path have to be adjacent")
        home = self._on_current()
        stream = home if stream is None and self.stream is None else self._on(stream)
        lens = (n_seq,)
        n_new = 0 if n_new_t is None else self._ints("n_new_t", n_new_t, lens)
        seq_len = 0 if seq_len_t is None else self._ints("seq_len_t", seq_len_t, lens)
        if new_len_t is None:
            new_len_t = torch.empty_like(n_new_t) if n_new_t is not None else path_t.new_empty(lens)
            new_len = new_len_t.data_ptr()
            if stream != home:
                self._record(stream, new_len_t)
        else:
            new_len = self._ints("new_len_t", new_len_t, lens)
        a = B.accept_args(path_t.data_ptr(), stride[0], shape[1], self.q_tokens if new_tokens is None else new_tokens, n_new, seq_len, new_len)
        B.pdkv_accept(self.handle, l0, l1, a, stream)
        return new_len_t

    def evict(self, dst: "CacheSession", scores_t, budget: int, *, sink: int = 0, recent: int = 0,
              layers: Optional[Tuple[int, int]] = None, kept_t=None, kept_scores_t=None, new_len_t=None, seq_len_t=None,
              stream: Optional[int] = None):
        """Keep the ``budget`` heaviest tokens per (layer, sequence, KV head) and move them, in order, to the
        front of the same sequences in ``dst`` (this session itself: in place).  ``scores_t`` is float32
        ``[layers, n_seq, num_kv_heads, >= longest]``.  Returns ``(kept, kept_scores, new_len)``."""
        l0, l1 = (0, self.geom.num_layers) if layers is None else layers
        if not 0 <= l0 < l1 <= self.geom.num_layers:
            raise ValueError(f"layers: expected a range within [0, {self.geom.num_layers}), got {layers}")
        n_seq = self._shape[0]
        lead = (l1 - l0, n_seq, self.geom.num_kv_heads)
        self._rows("scores_t", scores_t, lead, self._max_len)
        made = []
        if kept_t is None:
            kept_t = scores_t.new_empty((*lead, budget), dtype=torch.int32)
            made.append(kept_t)
        else:
            self._check("kept_t", kept_t, torch.int32, (*lead, budget))
            if not kept_t.is_contiguous():
                raise ValueError("kept_t has to be contiguous")
        if kept_scores_t is None:
            kept_scores_t = scores_t.new_empty((*lead, budget))
            made.append(kept_scores_t)
        else:
            self._rows("kept_scores_t", kept_scores_t, lead, min(budget, self._max_len))
        if new_len_t is None:
            new_len_t = scores_t.new_empty((n_seq,), dtype=torch.int32)
            made.append(new_len_t)
        a = B.pdkv_evict_args(budget=budget, sink=sink, recent=recent, seq_len=self._lens(seq_len_t), scores=scores_t.data_ptr(),
                              scores_stride=scores_t.stride()[:3], kept=kept_t.data_ptr(), kept_scores=kept_scores_t.data_ptr(),
                              kept_scores_stride=kept_scores_t.stride()[:3], kept_scores_len=kept_scores_t.shape[-1],
                              new_len=self._lens(new_len_t))
        stream = self._on(stream)
        if stream != self._on_current():
            self._record(stream, *made)
        B.pdkv_evict(self.handle, dst.handle, l0, l1, a, stream)
        return kept_t, kept_scores_t, new_len_t

    def items(self) -> np.ndarray:
        """The attention work list (``pdkv_attend_item``)."""
        return B.pdkv_seqs_items(self.handle)

    def status(self, stream: Optional[int] = None) -> None:
        """Wait for the session's stream and raise if a kernel reported an error since the last call of this: a wait that gave up, or lengths above
        the session's in an append or accept."""
        B.pdkv_seqs_status(self.handle, self._on(stream))

    def close(self) -> None:
        if self.handle:
            B.pdkv_seqs_destroy(self.handle)
            self.handle = None
        if self.pool:
            B.pdkv_pool_destroy(self.pool)
            self.pool = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()
