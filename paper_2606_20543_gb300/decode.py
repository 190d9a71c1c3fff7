"""Device buffers of a batch that decodes over the paged 8-bit cache, and the
calls of a pass: plan, append and attention for every layer, sampling.

Marshalling only.  Everything runs on torch's current stream and nothing waits
for the device, so a pass can be captured in a CUDA graph; what went wrong on
the device is in ``status`` (include/ssd.h).
"""
from __future__ import annotations

import torch

from . import (Grid, Rng, Sampling, cache as make_cache, rotary as make_rotary,
               ssd_cache_append, ssd_cache_attention, ssd_cache_attention_workspace,
               ssd_cache_plan, ssd_rotary_table, ssd_sample)


def _row_stride(x):
    """Elements from row to row; of a single row, whose stride may be anything, its width."""
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


class PagedDecode:
    """B sequences over a pool of ``num_blocks`` blocks of ``block`` tokens for
    each of ``layers`` layers; all layers share the block tables.

    A pass over up to N_max new tokens of every sequence (a prompt, one token
    each, or the drafts of a frontier):

        plan(n_new)              blocks, slots and positions of the new tokens
        attend(layer, q, k, v)   once per layer: rotate, cache, attend
        sample(logits, ...)      the next tokens
        advance(n)               n of the new tokens of every sequence stay

    Tokens that do not stay (rejected drafts) are overwritten by the next pass.  A sequence that
    plan() cannot serve (the pool has no block for it, or its lengths are out of range: ``status``
    says so) is left out of the pass, on the device: n_new is 0, it attends to nothing, its rows of
    o hold what they held and it does not advance.
    ``release(mask)`` gives the blocks of finished sequences back; their next
    pass starts at length 0."""

    def __init__(self, grid: Grid, B, Hq, Hkv, d, num_blocks, block, max_blocks, N_max, freq,
                 sections, interleaved=False, layers=1, device="cuda"):
        self.g, self.B, self.Hq, self.Hkv, self.d = grid, B, Hq, Hkv, d
        self.num_blocks, self.block, self.max_blocks = num_blocks, block, max_blocks
        self.N_max, self.N, self.device = N_max, N_max, device

        def new(shape, dtype, fill=0):
            return torch.full(shape, fill, dtype=dtype, device=device)

        pool = (layers, num_blocks, Hkv, block, d)
        self.k, self.v = (torch.empty(pool, dtype=torch.float8_e4m3fn, device=device)
                          for _ in range(2))
        self.k_scale, self.v_scale = (new(pool[:3], torch.float32) for _ in range(2))
        self.caches = [make_cache(self.k[i], self.v[i], self.k_scale[i], self.v_scale[i])
                       for i in range(layers)]
        # positions go up to the prefix and the longer side (or a flat index within the prefix)
        n_pos = grid.prefix_len + max(grid.grid_h, grid.row_stride) + 1
        self.table = new((n_pos, d // 2, 2), torch.float32)
        ssd_rotary_table(n_pos, d // 2, freq, self.table)
        self.rotary = make_rotary(self.table, sections, interleaved)
        # positions of the grid's tokens on the axes; before and behind them one that is refused
        P, W, cells = grid.prefix_len, grid.grid_w, grid.grid_h * grid.grid_w
        i = torch.arange(cells, device=device)
        self._grid_pos = new((cells + 2, 3), torch.int32, -1)
        self._grid_pos[1:-1] = torch.stack([torch.full_like(i, P), P + i // W, P + i % W], 1)
        # every block is free; the ring's last place takes what release() does not move
        self.ring = torch.arange(num_blocks + 1, dtype=torch.int32, device=device)
        self.head, self.next_head = new((1,), torch.int64), new((1,), torch.int64)
        self.tail = new((1,), torch.int64, num_blocks)
        self.cache_len, self.held, self.n_blocks, self.n_new = (new((B,), torch.int32)
                                                                for _ in range(4))
        self.block_table = new((B, max_blocks), torch.int32, -1)
        self._slots = new((B * N_max,), torch.int64, -1)
        self._pos, self._draft_pos = (new((B * N_max, 3), torch.int32) for _ in range(2))
        self._q = new((B * N_max * Hq * d,), torch.bfloat16)
        self._o = new((B * N_max * Hq * d,), torch.bfloat16)
        self.out_tok = new((B * N_max,), torch.int32, -1)
        self.prob, self.kept = new((B * N_max,), torch.float32), new((B * N_max,), torch.int32)
        self.status = new((1,), torch.int32)
        self._ws = {}

    def _workspace(self, N):
        if N not in self._ws:
            n = ssd_cache_attention_workspace(self.B, self.Hq, self.Hkv, self.d, N,
                                              self.max_blocks * self.block)
            self._ws[N] = torch.empty((max(n, 16),), dtype=torch.uint8, device=self.device), n
        return self._ws[N]

    def plan(self, n_new, N=None) -> None:
        """n_new int32 [B] (device), at most N (default N_max) each."""
        self.N = self.N_max if N is None else N
        if not 0 < self.N <= self.N_max:
            raise ValueError("N is between 1 and N_max")
        want = n_new.to(self.n_new).expand(self.B).contiguous()  # (mostly n_new itself)
        rows = self.B * self.N
        self.slots, self.pos = self._slots[:rows], self._pos[:rows]
        ssd_cache_plan(self.g, self.B, self.block, self.max_blocks, self.N, self.cache_len,
                       want, self.held, self.ring, self.num_blocks, self.head, self.tail,
                       self.next_head, self.block_table, self.n_blocks, self.slots, self.pos,
                       self.status)
        torch.mul(want, self.slots.view(self.B, self.N)[:, 0] >= 0, out=self.n_new)  # (if served)
        self._workspace(self.N)  # (allocated here, not in the middle of a pass)

    def attend(self, layer, q, k, v, draft_pos=None, key_start=None, scale=0.0):
        """q bf16 [B * N, Hq * d], k and v bf16 [B * N, Hkv * d]: row b * N + j is new
        token j of sequence b; rows may lie apart (slices of one projection's output).
        draft_pos int32 [B, N]: the new tokens are drafts of these grid indices (y * W + x),
        which give their rotary positions and what they see (without it: the next tokens of the
        flat sequence).  The drafts that advance() keeps become the tokens that follow, so those
        have to be the next ones, in order.  key_start int32 [B]: the first token of a sequence
        that may be seen.  Returns o bf16 [B * N, Hq * d] (valid until the next
        call; rows without a token hold what they held)."""
        rows, width = self.B * self.N, self.Hq * self.d
        for x, heads in ((q, self.Hq), (k, self.Hkv), (v, self.Hkv)):
            if tuple(x.shape) != (rows, heads * self.d) or x.stride(1) != 1 \
                    or x.dtype != torch.bfloat16:
                raise ValueError("q, k, v: bfloat16 [B * N, heads * d], heads side by side")
        for x, n in ((draft_pos, rows), (key_start, self.B)):
            if x is not None and (x.dtype != torch.int32 or x.numel() != n or not x.is_contiguous()):
                raise ValueError("draft_pos: int32 [B, N], key_start: int32 [B], contiguous")
        pos = self.pos
        if draft_pos is not None:
            cells = self.g.grid_h * self.g.grid_w
            pos = self._draft_pos[:rows]
            torch.index_select(self._grid_pos, 0, draft_pos.view(-1).clamp(-1, cells).add_(1), out=pos)
        q_rot, o = self._q[:rows * width], self._o[:rows * width]
        ssd_cache_append(self.caches[layer], self.rotary, self.B, self.N, self.Hq, self.n_new,
                         self.slots, pos, q, _row_stride(q), k, _row_stride(k), v, _row_stride(v),
                         q_rot, self.status)
        ws, n = self._workspace(self.N)
        ssd_cache_attention(self.g, self.caches[layer], self.B, self.Hq, self.cache_len, self.n_new,
                            draft_pos, key_start, self.N, self.block_table, self.max_blocks, q_rot,
                            scale, o, None, ws, n, self.status)
        return o.view(rows, width)

    def sample(self, logits, settings: Sampling, rng: Rng):
        """logits float32 or bf16 [rows, V], rows at most B * N_max.  Returns int32 [rows]."""
        rows, V = logits.shape
        if rows > self.out_tok.shape[0] or logits.stride(1) != 1:
            raise ValueError("logits: at most B * N_max rows, entries side by side")
        tok = self.out_tok[:rows]
        ssd_sample(rows, V, logits, _row_stride(logits), settings, rng, tok, self.prob[:rows],
                   self.kept[:rows], self.status)
        return tok

    def advance(self, n=None) -> None:
        """n int32 [B] (default, and at most: all) of the pass's new tokens stay."""
        self.cache_len.add_(self.n_new if n is None else self.n_new.clamp(max=n))
        self.held.copy_(self.n_blocks)
        self.head.copy_(self.next_head)

    def release(self, mask) -> None:
        """Blocks of the sequences with mask [B] (device, bool) go back to the ring."""
        at = torch.arange(self.max_blocks, device=self.device)
        own = mask[:, None] & (at[None] < self.held[:, None])
        place = (self.tail + torch.cumsum(own.flatten(), 0) - 1) % self.num_blocks
        place = torch.where(own.flatten(), place, self.num_blocks)
        self.ring.scatter_(0, place, self.block_table.flatten())
        self.tail.add_(own.sum())
        self.block_table.masked_fill_(mask[:, None], -1)
        self.cache_len.masked_fill_(mask, 0)
        self.held.masked_fill_(mask, 0)
