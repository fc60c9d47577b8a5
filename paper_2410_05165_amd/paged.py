"""Verifying drafted trees on a caller's own target: the step plan, the cache append,
tree attention over pages and the logit rules of include/atspeed.h on PyTorch tensors,
and ``PagedKV``, the caches and page tables of one target.

The functions have the library's names, check their tensors, allocate outputs that are
not given (_marshal.so, csrc/marshal.cpp) and enqueue on the current stream of the
tensors' GPU.  Everything computed is computed by the library's kernels; no gradients flow
through it, and what it writes in place counts as changed in place for a backward pass
that saved it.
"""
from __future__ import annotations

import math
from typing import NamedTuple, Optional

import torch

from .binding import AtspeedError, pack_rules  # noqa: F401

try:
    from . import _marshal
except ImportError as e:
    raise ImportError(f"_marshal.so or libatspeed.so is not built (run __graft_entry__.build()): {e}") from e

_marshal.set_error(AtspeedError)


def _run(fn, at, *args):
    """fn(*args, stream) on the current stream of the GPU of tensor `at` (a CPU tensor is refused by fn)."""
    device = at.get_device()
    if device < 0:
        return fn(*args, 0)
    if device == torch._C._cuda_getDevice():
        return fn(*args, torch._C._cuda_getCurrentRawStream(device))
    with torch.cuda.device(device):
        return fn(*args, torch._C._cuda_getCurrentRawStream(device))


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
    return StepPlan._make(_run(_marshal.page_plan, block_table, held, keep, add, block_table, free_pages, n_free, page_size,
                               max_rows, parent))


def atspeed_kv_append(k, v, k_cache, v_cache, slot):
    """Writes rows k, v [rows, kv_heads, d_head] to their cache slots [rows] (int32; outside the cache: skipped).

    Caches [pages, page_size, kv_heads, d_head]; all four may be strided, the last dimension contiguous.
    """
    _run(_marshal.kv_append, k_cache, k, v, k_cache, v_cache, slot)


def atspeed_tree_attention(q, k_cache, v_cache, block_table, row_off, ctx, max_ctx: int, max_new: int, mask=None,
                           scale: Optional[float] = None, out=None, return_lse: bool = False):
    """Attention of q [rows, heads, d_head] over the paged caches, which hold the rows' own keys already.

    block_table [B, max_pages], row_off [B + 1], ctx [B], mask [rows, words] as atspeed_page_plan gives them;
    mask None: each row sees its context and its request's rows up to itself.  max_ctx and max_new: what ctx and
    a request's row count stay within.  scale: 1 / sqrt(d_head) by default.  Returns out (given or new, of q's
    type), or (out, lse [rows, heads] fp32).
    """
    return _run(_marshal.tree_attention, k_cache, q, k_cache, v_cache, block_table, row_off, ctx, max_ctx, max_new, mask,
                scale, out, return_lse)


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
    return _run(_marshal.logit_rules, logits, logits, row_off, token_base, history, hist_len, repetition, frequency,
                presence, temperature, bias, bias_index, allowed, state, mask, node_token, mask_value, out, out_row,
                state_by_request)


class PagedKV:
    """Key and value caches of one target in pages, with the requests' page tables and the free list.

    One page table serves every layer.  ``plan`` starts a step, ``append`` and ``attention`` run per layer.
    A request is a row of the tables; add rows to an ended request's row to start another in its place
    (keep 0 gives its pages back first).  The tables, ``length`` and ``n_free`` change in place, so a step can be
    captured into a graph: each replay goes on from the step before, captured or not.
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
        with torch.inference_mode():                     # caches made under it are written outside it, too
            torch._foreach_copy_([self.length, self.n_free], [p.length, p.n_free])   # in place, for captured steps
        return p

    def append(self, layer: int, plan: StepPlan, k, v):
        """Keys and values [rows, kv_heads, d_head] of the plan's rows (of its first k.shape[0] rows)."""
        atspeed_kv_append(k, v, self.k[layer], self.v[layer], plan.slot[:k.shape[0]])

    def attention(self, layer: int, plan: StepPlan, q, max_new: int, max_ctx: Optional[int] = None, **kw):
        """Attention of the plan's rows (of its first q.shape[0] rows) over one layer's pages."""
        return atspeed_tree_attention(q, self.k[layer], self.v[layer], self.block_table, plan.row_off, plan.ctx,
                                      self.max_len if max_ctx is None else max_ctx, max_new,
                                      mask=None if plan.mask is None else plan.mask[:q.shape[0]], **kw)
