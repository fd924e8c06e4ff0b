"""One layer served by drafted trees over a paged cache, then evicted by design.

Requests are admitted with their prompts (pages dealt from the pool on the GPU), then
decode in speculative steps: each drafts a small tree of tokens, whose keys and queries
are normalised and rotated to their depths on the way into the cache, attends the tree
over the pages, keeps an accepted path, and goes on from there; at the end a request
leaves and its pages return to the pool.  Lengths, pages, offsets and masks stay on the
GPU throughout.  At last the cache is evicted and decoded over the compact cache.

    python examples/tree_decoding.py [--tokens 500] [--steps 8]
"""
from __future__ import annotations

import argparse
import os
import random
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_21475_gb300 import ebd  # noqa: E402


def draft(rng, n, deep):
    """A tree: a chain of `deep` tokens, the others branch off it."""
    return [i - 1 if i < deep else rng.randrange(-1, i) for i in range(n)]


def main(tokens=500, steps=8, B=3, hq=28, hkv=4, d=128, page=16, drafted=12, deep=5, seed=0):
    dev, dt = "cuda", torch.bfloat16
    rng = random.Random(seed)
    gen = torch.Generator(device=dev).manual_seed(seed)
    longest = tokens + steps * drafted + 1
    blocks = -(-longest // page)
    pc = ebd.alloc_paged(B, hkv, B * blocks, page, d, blocks, dt, dev)
    pool = ebd.alloc_page_pool(B, B * blocks, dev)
    inv_freq, mscale = ebd.rotary_frequencies(d, base=1e6)
    table = ebd.ebd_rotary_table(inv_freq, longest, mscale)
    q_weight, k_weight = (torch.empty(d, device=dev).uniform_(0.8, 1.6, generator=gen).to(dt)
                          for _ in range(2))

    def step(n, parents=None):
        """One forward step of n new tokens per request: its queries, output and offsets."""
        T = B * n
        cu, positions, slots, _ = ebd.ebd_paged_deal(
            pool, pc, torch.full((B,), n, dtype=torch.int32, device=dev), T)
        # stands for the fused projection's output: q, k, v are slices of it
        qkv = torch.empty((T, hq + 2 * hkv, d), dtype=dt, device=dev).normal_(generator=gen)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        q_rot = torch.empty((T, hq, d), dtype=dt, device=dev)
        mask = None  # plain tokens
        if parents is not None:
            mask, positions = ebd.ebd_tree_masks(parents, cu, pc.seq_len, n)
        ebd.ebd_paged_append_norm(pc, k, v, k_weight=k_weight, q=q, q_weight=q_weight, q_out=q_rot,
                                  slots=slots, positions=positions, table=table)
        y, _ = ebd.ebd_paged_tree_attention(q_rot, pc, cu, n, mask)
        return q_rot, y, cu

    step(tokens)  # the prompts
    kept = 0
    for _ in range(steps):
        parents = [p for _ in range(B) for p in draft(rng, drafted, deep)]
        step(drafted, torch.tensor(parents, dtype=torch.int32, device=dev))
        # stands for verification: each request accepts some of its tree's first chain
        accepted = [rng.randint(1, deep) for _ in range(B)]
        cu = torch.arange(B + 1, dtype=torch.int32, device=dev) * drafted
        path = torch.arange(deep, dtype=torch.int32, device=dev).repeat(B, 1)
        pc.seq_len.copy_(ebd.ebd_paged_keep(
            pc, cu, path, torch.tensor(accepted, dtype=torch.int32, device=dev)))
        kept += sum(accepted)
    q_rot, y, cu = step(1)  # a plain token, whose attention the compact cache is compared with
    n_ctx = int(pc.seq_len.min())

    # the last query scores its context; a quarter is kept and decoded over
    dense = ebd.alloc_compact(B, hkv, n_ctx, d, dt, dev)
    dense.idx_c.copy_(torch.arange(n_ctx, device=dev).int().expand(B, hkv, n_ctx))
    dense.n_kept.fill_(n_ctx)
    ebd.ebd_paged_gather(pc, dense)
    obs = ebd.ebd_gather_queries(q_rot.view(B, hq, 1, d), torch.zeros(1, device=dev).int(), hkv)
    scores = torch.empty((B, hkv, n_ctx), device=dev)
    ebd.ebd_score(obs, dense.K_c, scores)
    budget = n_ctx // 4
    cap = (budget + int(8 * budget ** 0.5) + 127) // 64 * 64
    design = ebd.design_for(batch=B, n_kv_heads=hkv, group=hq // hkv, head_dim=d, n_ctx=n_ctx,
                            seed=seed, k_head=budget // 5, budget_tokens=budget)
    cc = ebd.alloc_compact(B, hkv, cap, d, dt, dev)
    ebd.ebd_select(design, scores, cc)
    ebd.ebd_paged_gather(pc, cc)
    f32 = dict(dtype=torch.float32, device=dev)
    y_c, stats = torch.empty((B, hq, d), **f32), [torch.empty((B, hq), **f32) for _ in range(4)]
    ebd.ebd_certified_decode(q_rot, cc.K_c, cc.V_c, cc.logw_c, cc.n_kept, y_c, *stats)

    held = int((pool.held[:, 1] - pool.held[:, 0]).sum())
    ebd.ebd_paged_deal(pool, pc, torch.full((B,), -1, dtype=torch.int32, device=dev), 0)  # all leave
    return dict(kept=kept, n_ctx=n_ctx, held=held, free=int(pool.n_free), pages=B * blocks,
                error=(y_c - y.float()).norm(dim=-1) / y_c.norm(dim=-1), radius=stats[3],
                status=int(pc.dev_status) | int(cc.dev_status))


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=500)
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    r = main(a.tokens, a.steps)
    print(f"{r['kept']} drafted tokens kept, {r['n_ctx']} cached tokens in {r['held']} pages; "
          f"after the requests left {r['free']} of {r['pages']} pages are free")
    print(f"relative error of the compact decode: median {r['error'].median():.3f}; reported "
          f"radius: median {r['radius'].median():.3f}")
