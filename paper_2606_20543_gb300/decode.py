"""Device buffers of a batch that decodes over the paged 8-bit cache, and the
calls of a pass: plan, append and attention for every layer, sampling.

Marshalling only.  Everything runs on torch's current stream and nothing waits
for the device, so a pass can be captured in a CUDA graph; what went wrong on
the device is in ``status`` (include/ssd.h).
"""
from __future__ import annotations

import torch

from . import (Grid, Rng, Sampling, cache as make_cache, rotary as make_rotary,
               ssd_cache_append, ssd_cache_append_norm, ssd_cache_attention,
               ssd_cache_attention_shared, ssd_cache_attention_shared_workspace,
               ssd_cache_attention_workspace, ssd_cache_plan, ssd_get_cache_sharing,
               ssd_rotary_table, ssd_sample)


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
    pass starts at length 0.

    Sequences of one prompt hold its blocks once: after the pass that caches the prompt of the first
    of each group, ``share(group_start, blocks)`` gives those blocks to the others, and attend()
    reads them once a group."""

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
        # by N; each workspace is larger than the one before by half, so those outgrown take twice the last
        self._ws, self._outgrown = {}, []
        # groups that share blocks: of every group its blocks and their ids, of every sequence its group;
        # by the number of groups, for the graphs that captured them
        self.groups, self.max_shared, self._groups = 0, 0, {}
        # blocks that a sequence has of its group; -1 for a place whose group goes on without it, else 1
        self._base, self._open = new((B,), torch.int32), new((B,), torch.int32, 1)

    def _workspace(self, N):
        key = N, self.groups, self.max_shared, ssd_get_cache_sharing()
        while self._ws.get(N, (None, None))[1] != key:
            sizes = (self.Hq, self.Hkv, self.d, N, self.max_blocks * self.block)
            n = (ssd_cache_attention_shared_workspace(self.B, self.groups, *sizes, self.max_shared * self.block)
                 if self.groups else ssd_cache_attention_workspace(self.B, *sizes))
            ws = self._ws[N][0] if N in self._ws else None
            if ws is None or ws.numel() < n:
                if ws is not None:
                    self._outgrown.append(ws)  # (graphs may have captured it)
                    n = max(n, ws.numel() * 3 // 2)
                ws = torch.empty((max(n, 16),), dtype=torch.uint8, device=self.device)
            self._ws[N] = ws, key
            key = key[:3] + (ssd_get_cache_sharing(),)  # (set by another thread meanwhile: asked again)
        ws = self._ws[N][0]
        return ws, ws.numel()

    def share(self, group_start, blocks) -> None:
        """Group g, the sequences group_start[g] <= b < group_start[g + 1], shares the first blocks[g]
        blocks of its first sequence, which has cached them whole (0: none); the others, which hold
        nothing, go on behind them, at length blocks[g] * block.  group_start: 0 ... B; host numbers
        both.  Called between passes, not while an earlier group's blocks are held; what of this does not
        hold is refused, for which it waits for the device.  A graph of a pass that was captured before the
        first share() attends without groups, one captured later serves every share() of as many groups
        whose blocks are no more than the most when it was captured; for others it is captured anew.  A
        place that is released can begin anew once all of its group are (their shared blocks go back with
        the last of them); a pass with groups that asks tokens of it before leaves it out, as one that
        plan() cannot serve (status: DEVICE_BOUNDS)."""
        start, blocks = [int(x) for x in group_start], [int(x) for x in blocks]
        if len(start) != len(blocks) + 1 or start[0] != 0 or start[-1] != self.B or not blocks \
                or any(a > b for a, b in zip(start, start[1:])):
            raise ValueError("group_start: 0 ... B, ascending, one more than blocks")
        if min(blocks) < 0 or max(blocks) > self.max_blocks:
            raise ValueError("blocks: between 0 and max_blocks")
        dev = self.device
        sizes = [b - a for a, b in zip(start, start[1:])]
        n = torch.repeat_interleave(torch.tensor(blocks), torch.tensor(sizes)).to(dev)
        is_first = torch.zeros((self.B,), dtype=torch.bool, device=dev)
        is_first[[a for a, size in zip(start, sizes) if size > 0]] = True
        whole = (self.cache_len >= n * self.block) & (self.held >= n)
        bad = torch.stack([(self._base > 0).any(), (is_first & ~whole).any(),
                           (~is_first & (n > 0) & ((self.held > 0) | (self.cache_len > 0))).any()]).tolist()
        for what, is_so in zip(("an earlier group's blocks are held", "the first of a group has not cached its blocks",
                                "another sequence of a group holds blocks"), bad):
            if is_so:
                raise ValueError(what)
        self.groups = len(blocks)
        if self.groups not in self._groups:
            new = lambda *shape, t: torch.zeros(shape, dtype=t, device=dev)  # noqa: E731
            self._groups[self.groups] = dict(
                max_shared=0, group_start=new(self.groups + 1, t=torch.int32), shared=new(self.groups, t=torch.int32),
                _group=new(self.B, t=torch.int64), _shared_ids=new(self.groups, self.max_blocks, t=torch.int32),
                _shared_own=new(self.groups, t=torch.int64))
        kept = self._groups[self.groups]
        kept["max_shared"] = max(kept["max_shared"], *blocks)
        self.__dict__.update(kept)
        self.group_start.copy_(torch.tensor(start, dtype=torch.int32))
        self.shared.copy_(torch.tensor(blocks, dtype=torch.int32))
        self._group.copy_(torch.repeat_interleave(torch.arange(self.groups), torch.tensor(sizes)))
        first = torch.tensor([min(a, self.B - 1) for a in start[:-1]], device=dev)
        self._shared_ids.copy_(self.block_table[first])
        self._shared_own.copy_(self.shared * torch.tensor([int(size > 0) for size in sizes], device=dev))
        base = self.shared[self._group]
        joins = ~is_first & (base > 0)
        take = joins[:, None] & (torch.arange(self.max_blocks, device=dev)[None] < base[:, None])
        self.block_table.copy_(torch.where(take, self._shared_ids[self._group], self.block_table))
        self._base.copy_(base)
        self._open.fill_(1)
        self.cache_len.copy_(torch.where(joins, base * self.block, self.cache_len))
        self.held.copy_(torch.where(joins, base, self.held))

    def plan(self, n_new, N=None) -> None:
        """n_new int32 [B] (device), at most N (default N_max) each."""
        self.N = self.N_max if N is None else N
        if not 0 < self.N <= self.N_max:
            raise ValueError("N is between 1 and N_max")
        want = n_new.to(self.n_new).expand(self.B).contiguous()  # (mostly n_new itself)
        if self.groups:
            want = torch.minimum(want, want * self._open)  # (less than none, if any, of a place that is not open)
        rows = self.B * self.N
        self.slots, self.pos = self._slots[:rows], self._pos[:rows]
        ssd_cache_plan(self.g, self.B, self.block, self.max_blocks, self.N, self.cache_len,
                       want, self.held, self.ring, self.num_blocks, self.head, self.tail,
                       self.next_head, self.block_table, self.n_blocks, self.slots, self.pos,
                       self.status)
        torch.mul(want, self.slots.view(self.B, self.N)[:, 0] >= 0, out=self.n_new)  # (if served)
        self._workspace(self.N)  # (allocated here, not in the middle of a pass)

    def attend(self, layer, q, k, v, draft_pos=None, key_start=None, scale=0.0, norm=None):
        """q bf16 [B * N, Hq * d], k and v bf16 [B * N, Hkv * d]: row b * N + j is new
        token j of sequence b; rows may lie apart (slices of one projection's output).
        draft_pos int32 [B, N]: the new tokens are drafts of these grid indices (y * W + x),
        which give their rotary positions and what they see (without it: the next tokens of the
        flat sequence).  The drafts that advance() keeps become the tokens that follow, so those
        have to be the next ones, in order.  key_start int32 [B]: the first token of a sequence
        that may be seen.  norm: norms of the query and key heads before they are turned
        (paper_2606_20543_gb300.head_norm).  Returns o bf16 [B * N, Hq * d] (valid until the next
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
        new = (self.B, self.N, self.Hq, self.n_new, self.slots, pos, q, _row_stride(q), k, _row_stride(k), v,
               _row_stride(v), q_rot, self.status)
        if norm is None:
            ssd_cache_append(self.caches[layer], self.rotary, *new)
        else:
            ssd_cache_append_norm(self.caches[layer], self.rotary, norm, *new)
        ws, n = self._workspace(self.N)
        rest = (self.Hq, self.cache_len, self.n_new, draft_pos, key_start, self.N, self.block_table,
                self.max_blocks, q_rot, scale, o, None, ws, n, self.status)
        if self.groups:
            ssd_cache_attention_shared(self.g, self.caches[layer], self.B, self.groups, self.group_start,
                                       self.shared, self.max_shared, *rest)
        else:
            ssd_cache_attention(self.g, self.caches[layer], self.B, *rest)
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

    def _give_back(self, ids, own) -> None:
        """Blocks ids[own] to the ring."""
        place = (self.tail + torch.cumsum(own.flatten(), 0) - 1) % self.num_blocks
        place = torch.where(own.flatten(), place, self.num_blocks)
        self.ring.scatter_(0, place, ids.flatten())
        self.tail.add_(own.sum())

    def release(self, mask) -> None:
        """Blocks of the sequences with mask [B] (device, bool) go back to the ring, those that a group
        shares when none of it holds them any more."""
        at = torch.arange(self.max_blocks, device=self.device)
        own = mask[:, None] & (at[None] < self.held[:, None])
        if self.groups:
            own &= at[None] >= self._base[:, None]
        self._give_back(self.block_table, own)
        self.block_table.masked_fill_(mask[:, None], -1)
        self.cache_len.masked_fill_(mask, 0)
        self.held.masked_fill_(mask, 0)
        if self.groups:
            self._base.masked_fill_(mask, 0)
            alive = torch.zeros_like(self.shared).index_add_(0, self._group, (self._base > 0).to(torch.int32))
            done = (alive == 0) & (self._shared_own > 0)
            here = done[:, None] & (at[None] < self._shared_own[:, None])
            self._give_back(self._shared_ids, here)
            self._shared_own.masked_fill_(done, 0)
            self.shared.masked_fill_(done, 0)
            self._open.copy_(1 - 2 * ((self._base == 0) & (self.shared[self._group] > 0)).to(torch.int32))
