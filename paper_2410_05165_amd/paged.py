"""Verifying drafted trees on a caller's own target: the step plan, the cache append,
tree attention over pages and the logit rules of include/atspeed.h on PyTorch tensors,
and ``PagedKV``, the caches and page tables of one target.

The functions have the library's names, check their tensors, allocate outputs that are
not given and enqueue on the current stream of the tensors' GPU.  Everything computed
is computed by the library's kernels.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import NamedTuple, Optional

import torch

from .binding import (BF16, FP32, AtspeedError, KvAppendArgs, LogitRulesArgs, PagePlanArgs, TreeAttentionArgs,
                      load_library)

DTYPES = {torch.float32: FP32, torch.bfloat16: BF16}
_lib = None


def _library():
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


def _call(fn, args, device, *more):
    """fn(args, *more, stream) on the current stream of GPU `device` (its index)."""
    if device == torch._C._cuda_getDevice():
        status = fn(args, *more, torch._C._cuda_getCurrentRawStream(device))
    else:
        with torch.cuda.device(device):
            status = fn(args, *more, torch._C._cuda_getCurrentRawStream(device))
    if status != 0:
        raise AtspeedError(status, _lib.atspeed_last_error().decode())


def _want(t, name, dtype, shape, device):
    """The address of a contiguous tensor of this type and shape on GPU `device` (None: null)."""
    if t is None:
        return 0
    if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name}: want a contiguous {dtype} {tuple(shape)} on GPU {device}, got {t.dtype} "
                     f"{tuple(t.shape)} on {t.device}")


def _gpu(t, name):
    """The index of the tensor's GPU."""
    if not t.is_cuda:
        raise ValueError(f"{name} is on {t.device}: the operators run on the GPU alone")
    return t.get_device()


def _rows(t, name, shape, dtype, device):
    """(address, row stride, head stride) of [rows, heads, d_head] with any row and head strides."""
    if t.shape == shape and t.dtype is dtype and t.get_device() == device:
        row, head, one = t.stride()
        if one == 1:   # the stride of a dimension of one element says nothing
            return t.data_ptr(), row if shape[0] > 1 else 0, head if shape[1] > 1 else 0
    raise ValueError(f"{name}: want {dtype} {tuple(shape)} on GPU {device}, the last dimension contiguous")


def _caches(k_cache, v_cache):
    """(GPU, address and strides of the keys, address and strides of the values)."""
    device, shape, dtype = _gpu(k_cache, "k_cache"), k_cache.shape, k_cache.dtype
    if len(shape) != 4 or dtype not in DTYPES:
        raise ValueError("k_cache: want float32 or bfloat16 [pages, page_size, kv_heads, d_head]")
    *ks, k1 = k_cache.stride()
    *vs, v1 = v_cache.stride()
    for i in range(3):
        if shape[i] == 1:   # the stride of a dimension of one element says nothing
            ks[i] = vs[i] = 0
    if v_cache.shape != shape or v_cache.dtype is not dtype or v_cache.get_device() != device or k1 != 1 or v1 != 1:
        raise ValueError("the caches want one type, shape and device, the last dimension contiguous")
    return device, (k_cache.data_ptr(), *ks), (v_cache.data_ptr(), *vs)


class StepPlan(NamedTuple):
    """What atspeed_page_plan writes (int32 tensors; ``mask`` int64 bit words, None for chains)."""
    n_free: torch.Tensor
    length: torch.Tensor
    ctx: torch.Tensor
    refused: torch.Tensor
    row_off: torch.Tensor
    row_user: torch.Tensor
    row_pos: torch.Tensor
    slot: torch.Tensor
    tree_slot: torch.Tensor
    mask: Optional[torch.Tensor]


def atspeed_page_plan(held, keep, add, block_table, free_pages, n_free, page_size: int, max_rows: int,
                      parent=None) -> StepPlan:
    """Plans one step; ``block_table`` [B, max_pages] and ``free_pages`` [pool] change in place.

    held, keep, add [B], n_free [1]: int32; parent [B, max_nodes] int32 or None (chains).
    The returned n_free and length are the next step's n_free and held.
    """
    dev, where, i32 = _gpu(block_table, "block_table"), block_table.device, torch.int32
    if block_table.dim() != 2:
        raise ValueError("block_table: want [B, max_pages]")
    B, most = block_table.shape
    if max_rows < 0:
        raise ValueError("max_rows must be >= 0")
    nodes = 0
    if parent is not None:
        if parent.dim() != 2:
            raise ValueError("parent: want [B, max_nodes]")
        nodes = parent.shape[1]
    buf = torch.empty(4 * (B + max_rows) + 2, dtype=i32, device=where)
    out = buf.unsafe_split_with_sizes([1, B, B, B, B + 1, max_rows, max_rows, max_rows, max_rows])   # no autograd here
    mask = torch.empty((max_rows, (nodes + 63) // 64), dtype=torch.int64, device=where) if parent is not None else None
    at = buf.data_ptr()
    row = at + 4 * (4 * B + 2)
    args = PagePlanArgs.pack(B, page_size, most, free_pages.numel(), max_rows, nodes,
                        _want(held, "held", i32, (B,), dev), _want(keep, "keep", i32, (B,), dev),
                        _want(add, "add", i32, (B,), dev), _want(parent, "parent", i32, (B, nodes), dev),
                        _want(block_table, "block_table", i32, (B, most), dev),
                        _want(free_pages, "free_pages", i32, (free_pages.numel(),), dev),
                        _want(n_free, "n_free", i32, (1,), dev),
                        at, at + 4, at + 4 * (B + 1), at + 4 * (2 * B + 1), at + 4 * (3 * B + 1),
                        row, row + 4 * max_rows, row + 8 * max_rows, row + 12 * max_rows,
                        mask.data_ptr() if mask is not None else 0)
    _call(_library().atspeed_page_plan, args, dev)
    return StepPlan(*out, mask)


def atspeed_kv_append(k, v, k_cache, v_cache, slot):
    """Writes rows k, v [rows, kv_heads, d_head] to their cache slots [rows] (int32; outside the cache: skipped).

    Caches [pages, page_size, kv_heads, d_head]; all four may be strided, the last dimension contiguous.
    """
    dev, kc, vc = _caches(k_cache, v_cache)
    pool, page, heads, dh = k_cache.shape
    dtype, n = k_cache.dtype, slot.numel()
    shape = (n, heads, dh)
    k_at, k_row, k_head = _rows(k, "k", shape, dtype, dev)
    v_at, v_row, v_head = _rows(v, "v", shape, dtype, dev)
    args = KvAppendArgs.pack(DTYPES[dtype], n, heads, dh, page, pool, k_at, v_at, k_row, k_head, v_row, v_head, *kc, *vc,
                        _want(slot, "slot", torch.int32, (n,), dev))
    _call(_library().atspeed_kv_append, args, dev)


def atspeed_tree_attention(q, k_cache, v_cache, block_table, row_off, ctx, max_ctx: int, max_new: int, mask=None,
                           scale: Optional[float] = None, out=None, return_lse: bool = False):
    """Attention of q [rows, heads, d_head] over the paged caches, which hold the rows' own keys already.

    block_table [B, max_pages], row_off [B + 1], ctx [B], mask [rows, words] as atspeed_page_plan gives them;
    mask None: each row sees its context and its request's rows up to itself.  max_ctx and max_new: what ctx and
    a request's row count stay within.  scale: 1 / sqrt(d_head) by default.  Returns out (given or new, of q's
    type), or (out, lse [rows, heads] fp32).
    """
    dev, kc, vc = _caches(k_cache, v_cache)
    pool, page, kv_heads, dh = k_cache.shape
    if q.dim() != 3 or block_table.dim() != 2:
        raise ValueError("want q [rows, heads, d_head] and block_table [B, max_pages]")
    dtype, i32 = k_cache.dtype, torch.int32
    rows, heads, _ = q.shape
    shape = (rows, heads, dh)
    q_at = _rows(q, "q", shape, dtype, dev)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=q.device)
    o_at = _rows(out, "out", shape, dtype, dev)
    lse = torch.empty((rows, heads), dtype=torch.float32, device=q.device) if return_lse else None
    B, most = block_table.shape
    words = 0 if mask is None else mask.shape[-1]
    args = TreeAttentionArgs.pack(DTYPES[dtype], B, rows, heads, kv_heads, dh, page, most, pool, max_ctx, max_new, words,
                             1.0 / math.sqrt(dh) if scale is None else scale, *q_at, *kc, *vc,
                             _want(block_table, "block_table", i32, (B, most), dev),
                             _want(row_off, "row_off", i32, (B + 1,), dev), _want(ctx, "ctx", i32, (B,), dev),
                             _want(mask, "mask", torch.int64, (rows, words), dev), *o_at,
                             lse.data_ptr() if return_lse else 0)
    lib, need = _library(), C.c_size_t(0)
    status = lib.atspeed_tree_attention_workspace_bytes(args, need)
    if status != 0:
        raise AtspeedError(status, lib.atspeed_last_error().decode())
    ws = torch.empty(need.value, dtype=torch.uint8, device=q.device) if need.value else None
    _call(lib.atspeed_tree_attention, args, dev, ws.data_ptr() if ws is not None else None, need.value)
    return (out, lse) if return_lse else out


def _rule_counts(history, bias, allowed, cols, device):
    """(max_hist, n_bias, n_states, address and stride of the biases) of the rules."""
    n_bias = 0 if bias is None else bias.shape[0]
    if bias is not None and (bias.dtype is not torch.float32 or bias.get_device() != device or
                             bias.shape != (n_bias, cols) or (cols > 1 and bias.stride(1) != 1)):
        raise ValueError(f"bias: want float32 [n, {cols}] on GPU {device}, rows contiguous")
    return (0 if history is None else history.shape[-1], n_bias, 0 if allowed is None else allowed.shape[0],
            (0, 0) if bias is None else (bias.data_ptr(), bias.stride(0) if n_bias > 1 else cols))


def pack_rules(cols: int, token_base: int, B: int, device, history=None, hist_len=None, repetition=None, frequency=None,
               presence=None, temperature=None, bias=None, bias_index=None, allowed=None, state=None,
               mask_value: float = -1.0e4):
    """The arguments of Engine.atspeed_set_logit_rules: rules without logits, rows or trees, state [B]."""
    dev, f32, i32, vec = device.index or 0, torch.float32, torch.int32, (B,)
    hist, n_bias, states, biases = _rule_counts(history, bias, allowed, cols, dev)
    return LogitRulesArgs.pack(FP32, B, 0, cols, token_base, hist, 0, 0, n_bias, states, 0, 1, mask_value, 0, 0, 0, 0, 0, 0,
                               _want(history, "history", i32, (B, hist), dev), _want(hist_len, "hist_len", i32, vec, dev),
                               0, 0, _want(repetition, "repetition", f32, vec, dev),
                               _want(frequency, "frequency", f32, vec, dev), _want(presence, "presence", f32, vec, dev),
                               _want(temperature, "temperature", f32, vec, dev), *biases,
                               _want(bias_index, "bias_index", i32, vec, dev),
                               _want(allowed, "allowed", i32, (states, (cols + 31) // 32), dev),
                               _want(state, "state", i32, vec, dev))


def atspeed_logit_rules(logits, row_off, token_base: int = 0, history=None, hist_len=None, repetition=None,
                        frequency=None, presence=None, temperature=None, bias=None, bias_index=None, allowed=None,
                        state=None, mask=None, node_token=None, mask_value: float = -math.inf, out=None, out_row=None,
                        state_by_request: bool = False):
    """Penalties, biases, temperature and grammar masks on logits [rows, cols] (fp32 or bf16), as fp32.

    row_off [B + 1]; history [B, max_hist] and hist_len [B]; repetition, frequency, presence, temperature [B] fp32;
    bias [n, cols] fp32 with bias_index [B]; allowed [states, ceil(cols / 32)] int32 bit words with state [rows]
    (state_by_request: [B]); node_token [B, max_nodes] with mask [rows, words] (None: chains).  out: fp32 [rows, cols],
    or with out_row [rows] any [.., cols] that its rows are scattered to; may be ``logits`` itself.  Parts that are
    None are left out.
    """
    if logits.dim() != 2 or logits.dtype not in DTYPES or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits: want float32 or bfloat16 [rows, cols], rows contiguous")
    dev, where = _gpu(logits, "logits"), logits.device
    rows, cols = logits.shape
    f32, i32 = torch.float32, torch.int32
    if out is None:
        if out_row is not None:
            raise ValueError("out_row scatters to a given out")
        out = torch.empty((rows, cols), dtype=f32, device=where)
    elif out.dtype is not f32 or out.get_device() != dev or out.shape[-1] != cols or (cols > 1 and out.stride(-1) != 1):
        raise ValueError("out: want float32 [.., cols] on the logits' device, rows contiguous")
    flat = out if out.dim() == 2 else out.view(-1, cols)
    n_out = flat.shape[0]
    if out_row is None and n_out != rows:
        raise ValueError("out: want as many rows as logits")
    B = row_off.numel() - 1
    vec = (B,)
    nodes = 0 if node_token is None else node_token.shape[-1]
    words = 0 if mask is None else mask.shape[-1]
    hist, n_bias, states, biases = _rule_counts(history, bias, allowed, cols, dev)
    args = LogitRulesArgs.pack(
        DTYPES[logits.dtype], B, rows, cols, token_base, hist, nodes, words, n_bias, states, n_out,
        1 if state_by_request else 0, mask_value, logits.data_ptr(), logits.stride(0) if rows > 1 else cols,
        flat.data_ptr(), flat.stride(0) if n_out > 1 else cols, _want(out_row, "out_row", i32, (rows,), dev),
        _want(row_off, "row_off", i32, (B + 1,), dev), _want(history, "history", i32, (B, hist), dev),
        _want(hist_len, "hist_len", i32, vec, dev), _want(node_token, "node_token", i32, (B, nodes), dev),
        _want(mask, "mask", torch.int64, (rows, words), dev), _want(repetition, "repetition", f32, vec, dev),
        _want(frequency, "frequency", f32, vec, dev), _want(presence, "presence", f32, vec, dev),
        _want(temperature, "temperature", f32, vec, dev), *biases, _want(bias_index, "bias_index", i32, vec, dev),
        _want(allowed, "allowed", i32, (states, (cols + 31) // 32), dev),
        _want(state, "state", i32, vec if state_by_request else (rows,), dev))
    _call(_library().atspeed_logit_rules, args, dev)
    return out


class PagedKV:
    """Key and value caches of one target in pages, with the requests' page tables and the free list.

    One page table serves every layer.  ``plan`` starts a step, ``append`` and ``attention`` run per layer.
    A request is a row of the tables; add rows to an ended request's row to start another in its place
    (keep 0 gives its pages back first).
    """

    def __init__(self, n_layers: int, n_pages: int, page_size: int, n_kv_heads: int, d_head: int, max_batch: int,
                 max_len: int, dtype=torch.bfloat16, device="cuda:0"):
        dev = torch.device(device)
        shape = (n_layers, n_pages, page_size, n_kv_heads, d_head)
        i32 = dict(dtype=torch.int32, device=dev)
        self.page_size, self.max_len = page_size, max_len
        self.k, self.v = torch.zeros(shape, dtype=dtype, device=dev), torch.zeros(shape, dtype=dtype, device=dev)
        self.block_table = torch.full((max_batch, -(-max_len // page_size)), -1, **i32)
        self.free_pages = torch.arange(n_pages, **i32)
        self.n_free = torch.full((1,), n_pages, **i32)
        self.length = torch.zeros(max_batch, **i32)      # tokens whose pages each request holds

    def plan(self, keep, add, max_rows: int, parent=None) -> StepPlan:
        """Keeps keep[b] of each request's tokens and makes room for add[b] rows (atspeed_page_plan)."""
        p = atspeed_page_plan(self.length, keep, add, self.block_table, self.free_pages, self.n_free, self.page_size,
                              max_rows, parent)
        self.length, self.n_free = p.length, p.n_free
        return p

    def append(self, layer: int, plan: StepPlan, k, v):
        """Keys and values [rows, kv_heads, d_head] of the plan's rows (of its first k.shape[0] rows)."""
        atspeed_kv_append(k, v, self.k[layer], self.v[layer], plan.slot[:k.shape[0]])

    def attention(self, layer: int, plan: StepPlan, q, max_new: int, max_ctx: Optional[int] = None, **kw):
        """Attention of the plan's rows (of its first q.shape[0] rows) over one layer's pages."""
        return atspeed_tree_attention(q, self.k[layer], self.v[layer], self.block_table, plan.row_off, plan.ctx,
                                      self.max_len if max_ctx is None else max_ctx, max_new,
                                      mask=None if plan.mask is None else plan.mask[:q.shape[0]], **kw)
