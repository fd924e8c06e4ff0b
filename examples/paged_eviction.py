"""One layer served over a paged cache, then evicted by design.

Two requests' prompts are prefilled in chunks (rotation, append, attention over
the pages), a few tokens are decoded over the full paged cache, and then the cache
is evicted: accumulated-attention scores, the randomized design's kept set, the
kept rows gathered from the pages, and the certified decode over the compact
cache.  The compact decode's output is compared with the paged attention of the
same query, next to the error radius that it reports.

    python examples/paged_eviction.py [--tokens 4000] [--budget 0.25]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_21475_gb300 import ebd  # noqa: E402


def main(tokens=4000, budget=0.25, chunk=512, decode=4, hq=28, hkv=4, d=128, page=64, seed=0):
    dev, dt, B = "cuda", torch.bfloat16, 2
    gen = torch.Generator(device=dev).manual_seed(seed)
    longest = tokens + decode + 1
    blocks = -(-longest // page)
    pc = ebd.alloc_paged(B, hkv, B * blocks, page, d, blocks, dt, dev)
    pc.block_table.copy_(torch.randperm(B * blocks, generator=gen, device=dev).view(B, blocks))
    inv_freq, mscale = ebd.rotary_frequencies(d, base=1e6, scaling="parts", factor=4.0)
    table = ebd.ebd_rotary_table(inv_freq, longest, mscale)

    def step(new):
        """One forward step: `new` tokens of each request through the layer's attention."""
        # stands for the fused projection's output: q, k, v are slices of it
        qkv = torch.empty((sum(new), hq + 2 * hkv, d), dtype=dt, device=dev).normal_(generator=gen)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        q[:, :] *= 1.5
        cu = torch.tensor([0] + new, device=dev).cumsum(0).int()
        pc.seq_len += torch.tensor(new, device=dev).int()
        q_rot = torch.empty((sum(new), hq, d), dtype=dt, device=dev)
        ebd.ebd_paged_append(pc, k, v, cu, table=table, q=q, q_out=q_rot)
        y, lse = ebd.ebd_paged_attention(q_rot, pc, cu, max(new))
        return q_rot, y, lse, cu

    done = [0, 0]
    lengths = [tokens, tokens]
    while done != lengths:  # prompts in chunks, the second request half a chunk ahead
        new = [min(chunk if b == 0 or done[b] else chunk // 2, lengths[b] - done[b]) for b in (0, 1)]
        q_rot, y, lse, cu = step(new)
        done = [a + n for a, n in zip(done, new)]
    q_obs = []
    for _ in range(decode):
        q_rot, y, lse, cu = step([1, 1])
        q_obs.append(q_rot)
    n_ctx = tokens + decode
    assert pc.seq_len.tolist() == [n_ctx, n_ctx]

    # scores: the decoded tokens' queries observe the whole cache, laid out densely
    dense = ebd.alloc_compact(B, hkv, n_ctx, d, dt, dev)
    dense.idx_c.copy_(torch.arange(n_ctx, device=dev).int().expand(B, hkv, n_ctx))
    dense.n_kept.fill_(n_ctx)
    ebd.ebd_paged_gather(pc, dense)
    Q = torch.stack(q_obs, dim=2)  # [B, Hq, decode, d]
    obs = ebd.ebd_gather_queries(Q.contiguous(), torch.arange(decode, device=dev).int(), hkv)
    scores = torch.empty((B, hkv, n_ctx), device=dev)
    ebd.ebd_score(obs, dense.K_c, scores)

    # eviction: kept set and weights by design, kept rows straight from the pages
    kept = int(round(budget * n_ctx))
    cap = (kept + int(8 * kept ** 0.5) + 127) // 64 * 64
    design = ebd.design_for(batch=B, n_kv_heads=hkv, group=hq // hkv, head_dim=d, n_ctx=n_ctx,
                            seed=seed, k_head=kept // 5, budget_tokens=kept)
    cc = ebd.alloc_compact(B, hkv, cap, d, dt, dev)
    ebd.ebd_select(design, scores, cc)
    ebd.ebd_paged_gather(pc, cc)
    f32 = dict(dtype=torch.float32, device=dev)
    y_c, stats = torch.empty((B, hq, d), **f32), [torch.empty((B, hq), **f32) for _ in range(4)]
    ebd.ebd_certified_decode(q_rot, cc.K_c, cc.V_c, cc.logw_c, cc.n_kept, y_c, *stats)
    torch.cuda.synchronize()
    assert pc.dev_status.item() == 0 and cc.dev_status.item() == 0
    err = (y_c - y.float()).norm(dim=-1) / y_c.norm(dim=-1)
    return dict(kept=cc.n_kept.float().mean().item(), n_ctx=n_ctx, error=err, radius=stats[3],
                lse_paged=lse, lse_compact=stats[0], y=y, q=q_rot, pc=pc, cu=cu)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4000)
    ap.add_argument("--budget", type=float, default=0.25)
    a = ap.parse_args()
    r = main(a.tokens, a.budget)
    print(f"{r['n_ctx']} cached tokens per request, {r['kept']:.0f} kept per KV head")
    print(f"relative error of the compact decode: median {r['error'].median():.3f}, "
          f"max {r['error'].max():.3f}; reported radius: median {r['radius'].median():.3f}; "
          f"heads within their radius: {(r['error'] <= r['radius']).float().mean():.3f}")
