"""Plain float64 forms of the paged-cache operators and seeded inputs for their tests."""
import math

import torch


def rotate(x, cs, layout, inverse=False):
    """x [T, H, d] float64 turned by cs [T, R / 2, 2]; layout "half" or "pairs"."""
    x, cs = x.double(), cs.double()
    r = cs.shape[1]
    y = x.clone()
    for i in range(r):
        a, b = (i, i + r) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = cs[:, None, i, 0], cs[:, None, i, 1]
        s = -s if inverse else s
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def row(pool, block_table, b, h, pos):
    """The cached row of one position: [d]."""
    page = pool.shape[2]
    return pool[int(block_table[b, pos // page]), h, pos % page]


def rows(pool, block_table, b, h, n):
    """The first n cached rows of one sequence and head: [n, d] float64."""
    page = pool.shape[2]
    pages = block_table[b, :-(-n // page)].long()
    return pool[pages, h].reshape(-1, pool.shape[3])[:n].double()


def attention(q, K, V, block_table, seq_len, cu, scale, window):
    """y [T, Hq, d], lse [T, Hq] in float64; rows that no mask leaves a key: 0, -inf."""
    T, hq, d = q.shape
    hkv = K.shape[1]
    g = hq // hkv
    y = torch.zeros((T, hq, d), dtype=torch.float64, device=q.device)
    lse = torch.full((T, hq), -math.inf, dtype=torch.float64, device=q.device)
    for b, n in enumerate(seq_len.tolist()):
        lo, hi = int(cu[b]), int(cu[b + 1])
        if hi == lo or n == 0:
            continue
        at = torch.arange(n - (hi - lo), n, device=q.device)[:, None]
        keys = torch.arange(n, device=q.device)
        seen = keys <= at
        if window:
            seen &= keys > at - window
        for h in range(hkv):
            k, v = rows(K, block_table, b, h, n), rows(V, block_table, b, h, n)
            for j in range(h * g, h * g + g):
                s = (q[lo:hi, j].double() @ k.T) * scale
                s = torch.where(seen, s, torch.full_like(s, -math.inf))
                m = s.amax(1, keepdim=True)
                m = torch.where(m == -math.inf, torch.zeros_like(m), m)
                p = torch.where(seen, (s - m).exp(), torch.zeros_like(s))
                l = p.sum(1, keepdim=True)
                # a hidden row of v may hold anything: it takes no part
                for i in range(hi - lo) if not torch.isfinite(v).all() else ():
                    w = p[i][seen[i]]
                    if w.numel():
                        y[lo + i, j] = (w @ v[seen[i]]) / l[i]
                if torch.isfinite(v).all():
                    y[lo:hi, j] = torch.where(l > 0, (p @ v) / l.clamp(min=1e-300), torch.zeros_like(v[:1]))
                lse[lo:hi, j] = torch.where(l[:, 0] > 0, m[:, 0] + l[:, 0].log(),
                                            torch.full_like(m[:, 0], -math.inf))
    return y, lse


def attention_detail(q, K, V, block_table, seq_len, cu, scale, window, absent=()):
    """attention() and, for the size of its rounding errors, sum_j p_j |v_j| and
    (sum_j p_j^2 v_j^2)^1/2 of every output, p the softmax weights.  absent: (sequence,
    block) pairs whose positions no token sees.  Finite inputs."""
    T, hq, d = q.shape
    hkv = K.shape[1]
    page, g = K.shape[2], hq // hkv
    y, mean, root = (torch.zeros((T, hq, d), dtype=torch.float64, device=q.device)
                     for _ in range(3))
    lse = torch.full((T, hq), -math.inf, dtype=torch.float64, device=q.device)
    for b, n in enumerate(torch.as_tensor(seq_len).tolist()):
        lo, hi = int(cu[b]), int(cu[b + 1])
        if hi == lo or n == 0:
            continue
        at = torch.arange(n - (hi - lo), n, device=q.device)[:, None]
        keys = torch.arange(n, device=q.device)
        seen = keys <= at
        if window:
            seen &= keys > at - window
        bt = block_table[b:b + 1].clone()
        for i, block in absent:
            if i == b:
                seen[:, block * page:(block + 1) * page] = False
                bt[0, block] = 0
        for h in range(hkv):
            k, v = rows(K, bt, 0, h, n), rows(V, bt, 0, h, n)
            s = torch.einsum("tgd,nd->tgn", q[lo:hi, h * g:h * g + g].double(), k) * scale
            s.masked_fill_(~seen[:, None], -math.inf)
            z = torch.logsumexp(s, -1)
            p = torch.where(seen[:, None], (s - z[..., None]).exp(), torch.zeros_like(s))
            lse[lo:hi, h * g:h * g + g] = z
            y[lo:hi, h * g:h * g + g] = p @ v
            mean[lo:hi, h * g:h * g + g] = p @ v.abs()
            root[lo:hi, h * g:h * g + g] = ((p * p) @ (v * v)).sqrt()
    return y, lse, mean, root


def attention_bound(y, mean, root, dtype):
    """Bound of each output's error from attention_detail()'s results.

    bfloat16 weights are off by 2^-8 relative at most (8 significant bits, half a unit),
    so the sum is off by 2^-8 sum p |v| at most; with roundings of independent signs it
    exceeds 7 2^-8 (sum p^2 v^2)^1/2 with probability 2 e^(-49 / 2) = 5e-11 (Hoeffding).  The
    result is rounded once, 2^-8 |y|.  Float32: a logit is off by 2e-5 at most (the bound
    of the log-sum-exp), which changes a weight and the sum of weights by 2e-5 each,
    4e-5 sum p |v|; exponentials, sums and joins are far below, 1e-4 sum p |v| is asked."""
    bound = 1e-4 * mean
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (torch.minimum(mean, 7 * root) + y.abs() + bound)
    return bound


def make(new, total, hq, hkv, d, page, dtype, seed, order="head", spare=3, stale=0.0,
         max_blocks=None):
    """Inputs of one call.  new / total: new tokens and lengths per sequence.
    order "head": [page, head, row, d] pools; "row": views of [page, row, head, d]
    pools; "side": K and V side by side in one pool.  stale: what fills every
    slot that no sequence uses (and q, k, v are strided slices of one tensor)."""
    g = torch.Generator().manual_seed(seed)
    blocks = [-(-max(n, 0) // page) for n in total]
    n_pages = sum(blocks) + spare
    deal = torch.randperm(n_pages, generator=g).int()
    width = max_blocks or max(max(blocks), 1)
    bt = torch.full((len(total), width), -1, dtype=torch.int32)
    used = torch.zeros((n_pages, page), dtype=torch.bool)
    at = 0
    for b, n in enumerate(blocks):
        bt[b, :n] = deal[at:at + n]
        for i in range(n):
            used[deal[at + i].long(), :max(0, min(page, total[b] - i * page))] = True
        at += n
    used = used.cuda()
    pools = []
    gg = torch.Generator(device="cuda").manual_seed(seed + 1)
    if order == "side":
        both = torch.randn((n_pages, 2, hkv, page, d), generator=gg, device="cuda").to(dtype)
        pools = [both[:, 0], both[:, 1]]
    else:
        for _ in range(2):
            if order == "row":
                p = torch.randn((n_pages, page, hkv, d), generator=gg, device="cuda").to(dtype)
                pools.append(p.transpose(1, 2))
            else:
                pools.append(torch.randn((n_pages, hkv, page, d), generator=gg,
                                         device="cuda").to(dtype))
    for p in pools:
        p.copy_(torch.where(used[:, None, :, None], p, torch.full_like(p, stale)))
    T = sum(new)
    fused = torch.randn((T, hq + 2 * hkv, d), generator=gg, device="cuda").to(dtype)
    cu = torch.tensor([0] + new).cumsum(0).int().cuda()
    return dict(K=pools[0], V=pools[1], bt=bt.cuda(), seq_len=torch.tensor(total).int().cuda(),
                cu=cu, q=fused[:, :hq], k=fused[:, hq:hq + hkv], v=fused[:, hq + hkv:],
                max_new=max(new), T=T)
