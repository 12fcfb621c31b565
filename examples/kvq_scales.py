"""The late scales of an image over a key/value cache held in 4 bits, beside the same scales over a bf16 cache.

    python examples/kvq_scales.py [--model infinity2b_1024_bf16] [--blocks 4] [--batch 1]

A chain of blocks runs scale by scale as a generator does: the early scales unreduced (fvar_block_forward_dense_kvq), the late ones on the
kept rows (fvar_score_select, fvar_block_forward_pruned_kvq, fvar_lowrank_fill); every block appends its keys and values to its cache in
4 bits and attends over what all earlier scales left there.  The same chain over bf16 caches runs next to it on the same inputs.
Prints, per scale, the time of both, the rows held and how far the outputs are apart; then the sizes of the caches, and the first rows
of one cache read back (fvar_kvq_read) against the bf16 rows.  Random weights and inputs: the differences are those of a model without
any training for it."""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2512_16483_amd as fv  # noqa: E402
from workloads import WORKLOADS, Workload  # noqa: E402


class Chain:
    """Blocks with a cache each, in 4 bits or in bf16."""

    def __init__(self, W: Workload, scales, blocks: int, batch: int, four_bits: bool):
        self.W, self.B, self.four = W, batch, four_bits
        d, H, Dh, F = W.hidden, W.heads, W.head_dim, W.ffn_hidden
        self.ctx = fv.Context(hidden=d, heads=H, head_dim=Dh, ffn_hidden=F, scales=scales, dtype="bf16")
        self.capacity, self.len = sum(s * s for s in scales), 0
        g = torch.Generator(device="cuda").manual_seed(1)
        draw = lambda *s: (0.02 * torch.randn(s, generator=g, device="cuda")).to(torch.bfloat16)
        self.weights = [dict(w_qkv=draw(3 * d, d), w_o=draw(d, d), w_fc1=draw(F, d), w_fc2=draw(d, F)) for _ in range(blocks)]
        if four_bits:
            u8 = lambda last: torch.empty((batch, H, self.capacity, last), dtype=torch.uint8, device="cuda")
            self.caches = [fv.KVQ(u8(Dh // 2), u8(Dh // 2), u8(Dh // 32), u8(Dh // 32)) for _ in range(blocks)]
        else:
            rows = lambda: torch.empty((batch, self.capacity, H, Dh), dtype=torch.bfloat16, device="cuda")
            self.caches = [(rows(), rows()) for _ in range(blocks)]
        self.bytes = 2 * blocks * batch * self.capacity * (d // 2 + d // 32 if four_bits else 2 * d)

    def block(self, i: int, x, M: int, keep=None, k: int = 0):
        """Block i on all M rows of x, or on the k rows `keep` of them."""
        B, rows = self.B, k if keep is not None else M
        y = torch.empty((B, rows, self.W.hidden), dtype=torch.bfloat16, device="cuda")
        c, w = self.caches[i], self.weights[i]
        room = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
        if self.four:
            c.len = self.len
            ws = room(fv.fvar_block_kvq_workspace_bytes(self.ctx, c, B, rows))
            if keep is None:
                fv.fvar_block_forward_dense_kvq(self.ctx, w, x, B, M, c, y, ws)
            else:
                fv.fvar_block_forward_pruned_kvq(self.ctx, w, x, B, M, keep, k, c, y, ws)
        else:
            ws = room(fv.fvar_block_workspace_bytes(self.ctx, B, rows))
            if keep is None:
                fv.fvar_block_forward_dense(self.ctx, w, x, B, M, *c, self.capacity, self.len, y, ws)
            else:
                fv.fvar_block_forward_pruned(self.ctx, w, x, B, M, keep, k, *c, self.capacity, self.len, y, ws)
        return y

    def scale(self, x, side: int, factors=None):
        """All blocks of one scale; with factors (W_c, G_c) on the kept rows, the others restored from them."""
        M, B, d = side * side, self.B, self.W.hidden
        rows = M
        for i in range(len(self.weights)):
            if factors is None:
                x = self.block(i, x, M)
                continue
            k = rows = self.W.keep(side)
            keep = torch.empty((B, k), dtype=torch.int32, device="cuda")
            drop = torch.empty((B, M - k), dtype=torch.int32, device="cuda")
            ws = torch.empty(fv.fvar_select_workspace_bytes(self.ctx, B, M), dtype=torch.uint8, device="cuda")
            fv.fvar_score_select(self.ctx, x, B, M, k, keep, drop, ws=ws)
            y_keep, y = self.block(i, x, M, keep, k), torch.empty((B, M, d), dtype=torch.bfloat16, device="cuda")
            fv.fvar_lowrank_fill(self.ctx, y_keep, keep, drop, B, M, k, self.W.rank, *factors, y)
            x = y
        self.len += rows
        return x


def run(W: Workload, scales, blocks: int, batch: int, out=print) -> dict:
    """Both chains over `scales`; {scale: relative 2-norm of the outputs' difference}."""
    four, plain = Chain(W, scales, blocks, batch, True), Chain(W, scales, blocks, batch, False)
    g = torch.Generator(device="cuda").manual_seed(2)
    far = {}
    for side in scales:
        M = side * side
        rows = lambda *s: torch.randn(s, generator=g, device="cuda")
        x = rows(batch, M, W.hidden).to(torch.bfloat16)
        factors = None
        if side in W.late_scales:
            factors = (rows(batch, M, W.rank).to(torch.bfloat16), (rows(batch, W.rank, W.hidden) / W.rank ** 0.5).to(torch.bfloat16))
        ys, us = [], []
        for chain in (four, plain):
            held = chain.len
            chain.scale(x, side, factors)                     # once before it is timed, into the same rows
            chain.len = held
            torch.cuda.synchronize()
            t = time.perf_counter()
            ys.append(chain.scale(x, side, factors))
            torch.cuda.synchronize()
            us.append((time.perf_counter() - t) * 1e6)
        a, b = (y.float() for y in ys)
        far[side] = float((a - b).norm() / b.norm())
        out(f"scale {side:3d}x{side:<3d} rows held {four.len:6d}  4 bits {us[0]:9.0f} us  bf16 {us[1]:9.0f} us  outputs differ by {far[side]:.4f}")
    out(f"caches: 4 bits {four.bytes / 2 ** 20:.1f} MiB, bf16 {plain.bytes / 2 ** 20:.1f} MiB")
    n = min(four.len, 64)
    k = torch.empty((batch, n, W.heads, W.head_dim), dtype=torch.bfloat16, device="cuda")
    four.caches[0].len = four.len
    fv.fvar_kvq_read(four.ctx, four.caches[0], batch, 0, n, k)
    held = plain.caches[0][0][:, :n].float()
    out(f"first {n} keys of block 0, read back: off by {float((k.float() - held).norm() / held.norm()):.4f}")
    return far


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--model", default="infinity2b_1024_bf16", choices=[n for n, w in WORKLOADS.items() if w.dtype == "bf16"])
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--batch", type=int, default=1)
    a = ap.parse_args(argv)
    W = WORKLOADS[a.model]
    run(W, W.scales, a.blocks, a.batch)


if __name__ == "__main__":
    main()
