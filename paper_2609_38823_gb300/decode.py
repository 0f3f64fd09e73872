"""A decode step of several requests on a paged cache, layer after layer: the
norms, the projections in 4 bits, the attention over the pages and the MoE layer
under its expert prefix, every step a library call.

    h1 = h + Wo attention(Wqkv rmsnorm(h))      (8-bit rows, 4-bit weights)
    h  = h1 + MoE_l(rmsnorm(h1))                (prefix [0, K_l))

``PagedCache`` owns the pools of all layers, the block tables and the lengths;
``plan`` gives a step's rows their pages and slots, on the device. A request's
visual block stays in its pages and is left out of the attention from the layer at
which the request's exit was taken (``hide``), so the cache is not copied.
``DecodeStep`` sequences the calls; it makes no host synchronisation, so that a
step can be captured in a CUDA graph and replayed while the requests grow. No
position encoding is applied: ``rotate`` is called on the queries and keys of every
layer, with the rows' positions, where a model has one.
"""
from __future__ import annotations

from typing import Callable, Optional, Sequence

import torch

from . import (DECOMOE_BF16, decomoe_add_rmsnorm_q8, decomoe_moe_layer, decomoe_moe_layer_workspace_bytes,
               decomoe_paged_advance, decomoe_paged_append, decomoe_paged_attention,
               decomoe_paged_attention_workspace_bytes, decomoe_paged_plan, decomoe_paged_plan_step, decomoe_w4_linear,
               workspace)


def quantize_w4(w: torch.Tensor, group: int = 128):
    """(bytes [N, K / 2], bf16 scales [N, K / group]) of a weight matrix [N, K], as
    decomoe_w4_linear takes them: per group the scale that maps its largest
    magnitude onto 7, values rounded to the nearest code. Once, when a model is
    loaded."""
    N, K = w.shape
    g = w.float().view(N, K // group, group)
    scale = (g.abs().amax(-1) / 7).clamp(min=2.0 ** -60).to(torch.bfloat16)
    q = (torch.round(g / scale.float()[..., None]).clamp(-8, 7) + 8).to(torch.uint8).view(N, K)
    return (q[:, 0::2] | q[:, 1::2] << 4).contiguous(), scale.contiguous()


class PagedCache:
    """Keys and values of `layers` layers for up to `requests` requests in
    `pages` pages of `page_size` rows, bf16. `max_pages` bounds a request.

    `active` [requests] says which slots a decode step adds a row to (1) and which it
    leaves alone (0: no request, or one that waits). All do at the start; a released slot
    does not until rows are planned for it again."""

    def __init__(self, layers: int, requests: int, pages: int, page_size: int, max_pages: int, hkv: int, d: int,
                 device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        # keys and values of a page side by side: the two pools are slices of one buffer
        self.pool = torch.zeros(layers, pages, 2, page_size, hkv, d, dtype=torch.bfloat16, device=device)
        self.page_size = page_size
        self.table = torch.full((requests, max_pages), -1, **i32)
        self.free = torch.arange(pages, **i32)       # given out from free[head] on
        self.head, self.head_next = torch.zeros(1, **i32), torch.zeros(1, **i32)
        self.cached, self.seq_len = torch.zeros(requests, **i32), torch.zeros(requests, **i32)
        self.row_start = torch.zeros(requests + 1, **i32)
        self.active = torch.ones(requests, **i32)
        self.hide_begin = torch.zeros(requests, **i32)
        self.hide_count = torch.zeros(layers, requests, **i32)
        self.status = torch.zeros(1, **i32)

    def k(self, layer: int) -> torch.Tensor:
        return self.pool[layer, :, 0]

    def v(self, layer: int) -> torch.Tensor:
        return self.pool[layer, :, 1]

    def plan(self, fresh: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None) -> None:
        """Pages, slots [N] and positions [N] of the rows that this step adds
        (fresh [requests]); seq_len then counts them. Rows are numbered request after
        request, over those that add some. Repeating it before ``advance`` changes
        nothing."""
        self.active.logical_or_(fresh > 0)
        decomoe_paged_plan(self.cached, fresh, self.page_size, self.free, self.table, self.seq_len, self.row_start, slots,
                           positions, free_head=self.head, free_head_out=self.head_next, status=self.status)

    def plan_step(self, fresh: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None) -> None:
        """``plan`` for a decode step: one row where fresh [requests] is 1, none where it
        is 0; slots and positions [requests] by request, -1 where none is added."""
        decomoe_paged_plan_step(self.cached, fresh, self.page_size, self.free, self.table, self.seq_len, slots, positions,
                                free_head=self.head, free_head_out=self.head_next, status=self.status)

    def advance(self) -> None:
        """The step's rows are in the cache: those that got a page. Where the list of free
        pages ran out (the status word then says DECOMOE_ERR_BAD_INPUT, and the step's
        results of such a request lack its own row: look at it before using them), a
        request ends in front of the first page that it did not get, and the next plan
        tries again."""
        decomoe_paged_advance(self.cached, self.seq_len, self.table, self.page_size, free_head=self.head,
                              free_head_out=self.head_next)

    def release(self, request: int) -> None:
        """The request is over: its pages go back to the list (those of a hidden block
        that were given back before must be -1 in the table). Reads its length on the
        host, between steps."""
        n = -(-int(self.cached[request]) // self.page_size)
        pages = self.table[request, :n]
        pages = pages[pages >= 0]
        head = int(self.head) - pages.numel()
        if head < 0:
            raise ValueError("more pages released than were given out")
        self.free[head:head + pages.numel()] = pages
        self.head.fill_(head)
        self.table[request] = -1
        self.cached[request] = 0
        self.seq_len[request] = 0
        self.active[request] = 0
        self.hide_begin[request] = 0
        self.hide_count[:, request] = 0

    def hide(self, request: int, begin: int, count: int, from_layer: int) -> None:
        """Leave rows [begin, begin + count) of a request out of the attention of
        every layer from `from_layer` on (its visual block after the exit)."""
        self.hide_begin[request] = begin
        self.hide_count[:from_layer, request] = 0
        self.hide_count[from_layer:, request] = count


class DecodeLayer:
    """Device weights of one layer: norm weights [d] bf16 or None, the fused query,
    key and value projection [(Hq + 2 Hkv) D, d] and the output projection
    [d, Hq D] as (bytes, scales) pairs, and the MoE layer with its prefix K."""

    def __init__(self, norm_attn, w_qkv, w_out, norm_moe, w_r, bias, w_gate_up, w_down, K: int):
        self.norm_attn, self.w_qkv, self.w_out, self.norm_moe = norm_attn, w_qkv, w_out, norm_moe
        self.w_r, self.bias, self.w_gate_up, self.w_down, self.K = w_r, bias, w_gate_up, w_down, K


class DecodeStep:
    """One new token for each of B requests through all layers. `fresh` [B] (the
    cache's `active`) says which of them have one: a slot of 0 adds no row and takes no
    page, its slot and position are -1, and what its row of the hidden states holds is carried
    through the layers without a meaning."""

    def __init__(self, layers: Sequence[DecodeLayer], cache: PagedCache, B: int, hq: int, k: int, eps: float = 1e-6,
                 rotate: Optional[Callable[[torch.Tensor, torch.Tensor, torch.Tensor], None]] = None):
        self.layers, self.cache, self.B, self.hq, self.topk, self.eps = list(layers), cache, B, hq, k, eps
        self.rotate = rotate
        hkv, D = cache.pool.shape[4:]
        E, d = layers[0].w_r.shape
        m = layers[0].w_down.shape[2]
        dev = cache.pool.device
        bf = dict(dtype=torch.bfloat16, device=dev)
        self.fresh = cache.active
        self.slots, self.positions = (torch.empty(B, dtype=torch.int32, device=dev) for _ in range(2))
        self.x8 = torch.empty(B, d, dtype=torch.float8_e4m3fn, device=dev)
        self.x8_scale = torch.empty(B, dtype=torch.float32, device=dev)
        self.qkv = torch.empty(B, hq + 2 * hkv, D, **bf)
        self.q, self.k_new, self.v_new = self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:]
        self.heads = torch.empty(B, hq, D, **bf)
        self.proj, self.h1, self.xn = (torch.empty(B, d, **bf) for _ in range(3))
        self.h = [torch.empty(B, d, **bf) for _ in range(2)]
        self.attn_ws = workspace(decomoe_paged_attention_workspace_bytes(B, hq, hkv, D), dev)
        self.moe_ws = workspace(decomoe_moe_layer_workspace_bytes(B, d, E, k, m, DECOMOE_BF16), dev)

    def __call__(self, h0: torch.Tensor, trace=None) -> torch.Tensor:
        """Hidden states [B, d] of the requests' newest tokens to those after the
        last layer. trace(l, step, h_in, h_out), if given, is called after each
        layer's launches are queued (the buffers are reused by later layers)."""
        c = self.cache
        c.plan_step(self.fresh, self.slots, self.positions)
        h = h0
        for l, w in enumerate(self.layers):
            out = self.h[l & 1]
            decomoe_add_rmsnorm_q8(h, None, w.norm_attn, y8=self.x8, y8_scale=self.x8_scale, eps=self.eps)
            decomoe_w4_linear(self.x8, *w.w_qkv, self.qkv.view(self.B, -1), x_scale=self.x8_scale)
            if self.rotate is not None:
                self.rotate(self.q, self.k_new, self.positions)
            decomoe_paged_append(self.k_new, self.v_new, self.slots, c.k(l), c.v(l), status=c.status)
            decomoe_paged_attention(self.q, c.k(l), c.v(l), c.table, c.seq_len, self.heads, self.attn_ws,
                                    hide_begin=c.hide_begin, hide_count=c.hide_count[l], status=c.status)
            decomoe_w4_linear(self.heads.view(self.B, -1), *w.w_out, self.proj)
            decomoe_add_rmsnorm_q8(self.proj, h, w.norm_moe, self.h1, self.xn, eps=self.eps)
            decomoe_moe_layer(self.xn, w.w_r, w.bias, w.w_gate_up, w.w_down, self.topk, out, self.moe_ws, K_fixed=w.K,
                              residual=self.h1, status=c.status)
            if trace is not None:
                trace(l, self, h, out)
            h = out
        return h
