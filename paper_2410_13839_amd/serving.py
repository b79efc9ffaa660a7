"""Paged serving on torch tensors: block tables and slots from request
lengths, cache writes, attention of new tokens over the cache, beam selection
and the page copies of beams (include/mtp.h's mtp_pages_* and mtp_beam_*).

Each function checks its tensors, allocates its outputs and workspace with
torch and enqueues one library call on torch's current stream of the tensors'
device; nothing is copied to the host and nothing waits, so the calls can be
captured into a graph.  What a call writes into a caller's tensor counts as an
in-place change of it (its version moves on).  Tensors made on another stream
must be ordered before the call by the caller, as for any torch operation.  A
refused call raises ValueError (a tensor of the wrong kind, or a call inside
torch.jit.trace, whose graph cannot hold it) or MTPError (the library's own
checks) with nothing launched.

A step of a served batch:

    plan = plan_pages(length, add, table, num_pages, max_tokens, parent=parents)
    copy_pages(pools, plan.copies)                      # beams only
    for l in range(layers):
        write_pages(pools[l], plan.slots, k, v)
        o = attend_pages(pools[l], plan.table, plan.row_start, plan.kv_len, q)
    step = select_beams(logits, score, length, done, eos_id)

A pool is [pages, 2, kv heads, 16 * head dim] in float32 or bfloat16 (pools of
several layers: one more leading dimension), the page format of include/mtp.h.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad as _forward
from torch.autograd.graph import increment_version as _changed

from . import binding as _b

PAGE = 16
_DTYPE = {torch.float32: _b.MTP_DTYPE_F32, torch.bfloat16: _b.MTP_DTYPE_BF16}


class PagePlan(NamedTuple):
    """int32 tensors; the fields of mtp_plan_args (views of one allocation)."""
    table: torch.Tensor       # [rows, max_pages]
    row_start: torch.Tensor   # [rows + 1]
    kv_len: torch.Tensor      # [rows]
    slots: torch.Tensor       # [max_tokens]
    positions: torch.Tensor   # [max_tokens]
    copies: torch.Tensor      # [rows, 2]
    status: torch.Tensor      # [4]: pages missing, bad rows, bad table entries, tokens without a slot


class BeamStep(NamedTuple):
    """[requests, beams] each; parent counts rows over all requests."""
    score: torch.Tensor
    length: torch.Tensor
    done: torch.Tensor
    parent: torch.Tensor
    token: torch.Tensor


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _i32(x: int, name: str) -> int:
    if not -(1 << 31) <= x < 1 << 31:            # (ctypes would drop the upper bits)
        raise ValueError(f"{name}: {x} does not fit 32 bits")
    return x


def _ints(t: torch.Tensor, name: str, shape, device) -> int:
    if t.dtype is not torch.int32 or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous int32 tensor of shape {tuple(shape)} on {device}, "
                         f"not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


# the current stream's handle without the Stream object around it (3 us of a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(fn, args, device) -> None:
    """fn on torch's current stream of `device` (made the current device for the call)."""
    index = device.index
    if torch.cuda.current_device() == index:
        fn(args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            fn(args, _raw_stream(index))


def _workspace(size, args, device):
    """Scratch of the size that `size` reports, in args; the caller holds it until the launch."""
    need = size(args)
    if not need:
        return None
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    args.workspace, args.workspace_bytes = ws.data_ptr(), need
    return ws


_is_tracing = getattr(torch._C, "_is_tracing", None) or torch.jit.is_tracing


def _device(t: torch.Tensor, name: str) -> torch.device:
    """The device that a call's tensors have to share; every call asks for it before it allocates or launches."""
    if _is_tracing():                            # (a trace would hold the output's allocation and not what fills it)
        raise ValueError("the serving operators cannot be traced")
    if not t.is_cuda:
        raise ValueError(f"{name}: a tensor on a GPU, not on {t.device}")
    return t.device


def _no_gradient(t: torch.Tensor, name: str) -> None:
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name}: the serving operators have no backward pass (call them under torch.no_grad)")
    # (the level, -1 outside dual_level, spares a call 0.25 us a tensor)
    if _forward._current_level >= 0 and _forward.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name}: the serving operators have no forward-mode derivative (unpack_dual gives the primal)")


def _cache(pool: torch.Tensor) -> _b.mtp_cache:
    if pool.dim() != 4 or pool.dtype not in _DTYPE or not pool.is_contiguous():
        raise ValueError("pool: a contiguous float32 or bfloat16 tensor [pages, 2, kv heads, 16 * head dim]")
    pages, two, heads, block = pool.shape
    _no_gradient(pool, "pool")
    if two != 2 or block not in (PAGE * 64, PAGE * 128):
        raise ValueError(f"pool: [pages, 2, kv heads, 16 * 64 or 16 * 128], not {tuple(pool.shape)}")
    return _b.mtp_cache(pool.data_ptr(), _DTYPE[pool.dtype], pages, heads, block // PAGE)


def _rows(t: torch.Tensor, name: str, pool: torch.Tensor, dim: int, heads: Optional[int] = None) -> int:
    """Token stride of [tokens, heads, head dim] rows in the pool's type."""
    shape = t.shape
    if t.dtype != pool.dtype or t.device != pool.device or len(shape) != 3 or shape[2] != dim or \
            (heads is not None and shape[1] != heads):
        raise ValueError(f"{name}: {pool.dtype} [tokens, {'heads' if heads is None else heads}, {dim}] on {pool.device}, "
                         f"not {t.dtype} {tuple(shape)} on {t.device}")
    s0, s1, s2 = t.stride()
    if shape[0] and (s2 != 1 or (s1 != dim and shape[1] > 1)):
        raise ValueError(f"{name}: a token's heads must be contiguous")
    _no_gradient(t, name)
    return s0 if shape[0] > 1 else shape[1] * dim


def plan_pages(length: torch.Tensor, add: torch.Tensor, table: torch.Tensor, num_pages: int, max_tokens: int,
               parent: Optional[torch.Tensor] = None, out_table: Optional[torch.Tensor] = None) -> PagePlan:
    """Block tables, slots and positions of the next tokens (mtp_pages_plan).
    length, add: int32 [rows]; table: int32 [rows, max_pages]; max_tokens: the
    size of slots and positions (at least the new tokens' number).  out_table
    receives the new table (a new tensor by default; `table` itself is allowed
    without parents).  The status counts stay on the device."""
    dev = _device(length, "length")
    _need(table.dim() == 2 and length.dim() == 1, "length: [rows]; table: [rows, max_pages]")
    n, m = table.shape
    _need(0 <= max_tokens < 1 << 31 and 0 < num_pages < 1 << 27 and m < 1 << 31,
          "max_tokens in [0, 2^31), num_pages in [1, 2^27), max_pages in 32 bits")
    p_len, p_add = _ints(length, "length", (n,), dev), _ints(add, "add", (n,), dev)
    p_in = _ints(table, "table", (n, m), dev)
    p_par = None if parent is None else _ints(parent, "parent", (n,), dev)
    # one allocation for the outputs, cut once (views cost the call more than its checks); the table first
    own = n * m if out_table is None else 0
    cut = (own, 2 * n, n, n + 1, 4, max_tokens, max_tokens)
    new, copies, kv_len, row_start, status, slots, positions = torch.split_with_sizes(
        torch.empty(sum(cut), dtype=torch.int32, device=dev), cut)
    new = new.view(n, m) if out_table is None else out_table
    p_new = new.data_ptr() if out_table is None else _ints(new, "out_table", (n, m), dev)
    _need(p_par is None or p_new != p_in or n == 0, "out_table: not the table itself where rows have parents")
    base, tok = status.data_ptr() - 4 * (4 * n + 1), slots.data_ptr()
    args = _b.mtp_plan_args(n, m, num_pages, max_tokens, p_par, p_len, p_add, p_in, p_new,
                            base + 4 * 3 * n, base + 4 * 2 * n, tok, tok + 4 * max_tokens, base, base + 4 * (4 * n + 1), None, 0)
    ws = _workspace(_b.mtp_pages_plan_workspace_size, args, dev)
    if n == 0:
        row_start.zero_()
        status.zero_()
        slots.fill_(-1)
        positions.fill_(-1)
    else:
        _launch(_b.mtp_pages_plan, args, dev)
        if out_table is not None:
            _changed(out_table)
    return PagePlan(new, row_start, kv_len, slots, positions, copies.view(n, 2), status)


def write_pages(pool: torch.Tensor, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> None:
    """Stores k, v [tokens, kv heads, head dim] at `slots` int32 [tokens] of
    one layer's pool (mtp_pages_write); slots outside the pool are skipped."""
    dev = _device(pool, "pool")
    cache = _cache(pool)
    heads, dim = cache.n_kv_heads, cache.head_dim
    ks, vs = _rows(k, "k", pool, dim, heads), _rows(v, "v", pool, dim, heads)
    _need(k.shape[0] == v.shape[0], "k and v: the same number of tokens")
    p = _ints(slots, "slots", (k.shape[0],), dev)
    _launch(_b.mtp_pages_write, _b.mtp_write_args(cache, k.shape[0], p, k.data_ptr(), v.data_ptr(), ks, vs), dev)
    _changed(pool)


def copy_pages(pools: torch.Tensor, copies: torch.Tensor) -> None:
    """Copies the pages that a plan's `copies` names, in one layer's pool or,
    with a leading dimension, in every layer's (mtp_pages_copy)."""
    _need(pools.dim() in (4, 5) and pools.dtype in _DTYPE and pools.is_contiguous(),
          "pools: a contiguous float32 or bfloat16 tensor [layers,] [pages, 2, kv heads, 16 * head dim]")
    _no_gradient(pools, "pools")
    dev = _device(pools, "pools")
    layers = pools.shape[0] if pools.dim() == 5 else 1
    pages = pools.shape[-4]
    page_bytes = pools.shape[-3] * pools.shape[-2] * pools.shape[-1] * pools.element_size()
    _need(copies.dim() == 2, "copies: [n, 2]")
    p = _ints(copies, "copies", (copies.shape[0], 2), dev)
    _launch(_b.mtp_pages_copy, _b.mtp_copy_args(pools.data_ptr(), page_bytes, pages * page_bytes, _i32(layers, "layers"), pages,
                                                _i32(copies.shape[0], "copies"), p), dev)
    _changed(pools)


def attend_pages(pool: torch.Tensor, table: torch.Tensor, row_start: torch.Tensor, kv_len: torch.Tensor,
                 q: torch.Tensor, causal: bool = True, window: int = 0, scale: Optional[float] = None, max_kv: int = 0,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of q [tokens, heads, head dim] over one layer's pool
    (mtp_pages_attention): causal chunks (the queries are their rows' last
    positions, `window` > 0 of them visible), or full attention with causal =
    False.  scale defaults to head dim ** -0.5.  Tokens outside every row keep
    what `out` holds (a new `out` starts undefined there); out shares no element
    with q or the pool."""
    dev = _device(pool, "pool")
    cache = _cache(pool)
    dim = cache.head_dim
    qs = _rows(q, "q", pool, dim)
    _need(table.dim() == 2, "table: [rows, max_pages]")
    n, m = table.shape
    own = out is None
    if own:
        out = torch.empty_like(q)                # (contiguous, as a token's heads are)
        os = q.shape[1] * dim
    else:
        _need(out.shape == q.shape, "out: q's shape")
        os = _rows(out, "out", pool, dim)
    args = _b.mtp_attention_args(cache, n, _i32(m, "max_pages"), _i32(q.shape[0], "tokens"), q.shape[1],
                                 _b.MTP_ATTN_CAUSAL if causal else _b.MTP_ATTN_FULL, _i32(window, "window"),
                                 _i32(max_kv, "max_kv"), dim ** -0.5 if scale is None else scale,
                                 _ints(table, "table", (n, m), dev), _ints(row_start, "row_start", (n + 1,), dev),
                                 _ints(kv_len, "kv_len", (n,), dev), q.data_ptr(), out.data_ptr(), qs, os, None, 0)
    ws = _workspace(_b.mtp_pages_attention_workspace_size, args, dev)
    _launch(_b.mtp_pages_attention, args, dev)
    if not own:
        _changed(out)
    return out


def select_beams(logits: torch.Tensor, score: torch.Tensor, length: torch.Tensor, done: torch.Tensor, eos_id: int,
                 eos_min: int = 0, alpha: float = 0.0) -> BeamStep:
    """The next beams of [requests, beams, vocab] float32 logits
    (mtp_beam_select); score float32, length and done int32 [requests, beams].
    Beams of one request that are still alike (at its start) are told apart by
    a score of -infinity for all but the first."""
    dev = _device(logits, "logits")
    _need(logits.dim() == 3 and logits.dtype == torch.float32, "logits: float32 [requests, beams, vocab]")
    r, w, v = logits.shape
    ld = logits.stride(1) if w > 1 else (logits.stride(0) if r > 1 else v)
    _no_gradient(logits, "logits")
    _no_gradient(score, "score")
    _need(v == 0 or logits.stride(2) == 1 or v == 1, "logits: a row's logits must be contiguous")
    _need(r <= 1 or w <= 1 or logits.stride(0) == w * ld, "logits: the rows must be evenly spaced")
    _need(score.dtype == torch.float32 and tuple(score.shape) == (r, w) and score.device == dev and score.is_contiguous(),
          "score: contiguous float32 [requests, beams] on the logits' device")
    new = torch.empty((5, r, w), dtype=torch.int32, device=dev)
    base, step = new.data_ptr(), 4 * r * w
    args = _b.mtp_beam_args(_i32(r, "requests"), _i32(w, "beams"), _i32(v, "vocab"), _i32(eos_id, "eos_id"),
                            _i32(eos_min, "eos_min"), alpha, logits.data_ptr(), ld, score.data_ptr(),
                            _ints(length, "length", (r, w), dev), _ints(done, "done", (r, w), dev), base, base + step,
                            base + 2 * step, base + 3 * step, base + 4 * step, None, 0)
    ws = _workspace(_b.mtp_beam_select_workspace_size, args, dev)
    _launch(_b.mtp_beam_select, args, dev)
    del ws
    new = new.unbind(0)
    return BeamStep(new[0].view(torch.float32), *new[1:])
