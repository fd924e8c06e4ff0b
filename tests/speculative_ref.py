"""Plain forms of a speculative step's operators: pages dealt one request after another,
norms with the rotation and their gradients in float64, trees, accepted paths."""
import math
import random

import torch

import paged_ref as R


# ---------------------------------------------------------------- pages
def deal(P, n_pages, max_blocks, n_tokens, window, n_new, seq_len, held, free, table):
    """One step, request by request, on Python lists; free is the list of free pages
    (its end is taken first), table the rows of blocks.  Returns the new lengths, holdings,
    packed offsets, who was served, positions and slots; free and table change."""
    B = len(n_new)
    held, length = [list(h) for h in held], list(seq_len)
    for b in range(B):
        lo, hi = held[b]
        keep = lo
        if n_new[b] < 0:
            keep = hi
        elif window:
            while keep < hi and (keep + 1) * P <= length[b] - window + 1:
                keep += 1
        free += table[b][lo:keep]
        held[b][0] = keep
    wanted = tokens = 0
    there = len(free)
    cu, served, pos, slots = [0], [], [], []
    for b in range(B):
        n = n_new[b]
        if n < 0:
            length[b], held[b] = 0, [0, 0]
            served.append(1)
            cu.append(cu[-1])
            continue
        after = -(-(length[b] + n) // P)
        ok = after <= max_blocks
        if ok and n > 0:
            need = max(0, after - held[b][1])
            wanted += need
            tokens += n
            ok = (need == 0 or wanted <= there) and tokens <= n_tokens
            if ok:
                for _ in range(need):
                    table[b][held[b][1]] = free.pop()
                    held[b][1] += 1
                for p in range(length[b], length[b] + n):
                    pos.append(p)
                    slots.append(table[b][p // P] * P + p % P)
                length[b] += n
        served.append(int(ok))
        cu.append(len(pos))
    pad = n_tokens - len(pos)
    return length, held, cu, served, pos + [0] * pad, slots + [-1] * pad


# ---------------------------------------------------------------- norms
def norm(x, w, eps):
    """w x / sqrt(mean x^2 + eps) of the rows of x [T, H, d], float64."""
    x = x.double()
    return w.double() * x / ((x * x).mean(-1, keepdim=True) + eps).sqrt()


def magnitudes(x, cs, layout):
    """|a| |cos| + |b| |sin| of every rotated channel: the size of its terms."""
    m = x.abs().clone()
    r = cs.shape[1]
    for i in range(r):
        a, b = (i, i + r) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = cs[:, None, i, 0].abs().double(), cs[:, None, i, 1].abs().double()
        m[..., a] = x[..., a].abs() * c + x[..., b].abs() * s
        m[..., b] = x[..., b].abs() * c + x[..., a].abs() * s
    return m


def norm_grad(dy, x, w, eps, cs, layout):
    """dx, dweight per row [T, H, d] and, for the size of their errors, the same with every
    term's magnitude."""
    u = dy.double() if cs is None else R.rotate(dy, cs, layout, inverse=True)
    au = dy.double().abs() if cs is None else magnitudes(dy.double(), cs, layout)
    x, w = x.double(), w.double()
    r = 1 / ((x * x).mean(-1, keepdim=True) + eps).sqrt()
    z = x * r
    g, ag = u * w, au * w.abs()
    dx = r * (g - z * (g * z).mean(-1, keepdim=True))
    adx = r * (ag + z.abs() * (ag * z.abs()).mean(-1, keepdim=True))
    return dx, u * z, adx, au * z.abs()


# ---------------------------------------------------------------- trees
def random_parents(new, seed, shape="mixed"):
    rng = random.Random(seed)
    out = []
    for n in new:
        for i in range(n):
            k = rng.random()
            if shape == "chain":
                out.append(i - 1)
            elif shape == "roots":
                out.append(-1)
            else:
                out.append(-1 if i == 0 or k < 0.1 else i - 1 if k < 0.6 else rng.randrange(i))
    return out


def lines(parents, cu):
    """The line of every packed token: its number, its parent's, and so on up."""
    out = []
    for lo, hi in zip(cu, cu[1:]):
        for i in range(hi - lo):
            line = [i]
            while parents[lo + line[-1]] >= 0:
                line.append(parents[lo + line[-1]])
            out.append(line)
    return out


def masks(parents, cu, seq_len, words, window=0):
    """mask [T, words] int32 and positions [T] from the parents."""
    rows, pos = [], []
    b = 0
    for t, line in enumerate(lines(parents, cu)):
        while t >= cu[b + 1]:
            b += 1
        v = 0
        for j in line[:window] if window else line:
            v |= 1 << j
        row = [(v >> 32 * i) & 0xffffffff for i in range(words)]
        rows.append([r - (1 << 32) if r >> 31 else r for r in row])
        pos.append(seq_len[b] - (cu[b + 1] - cu[b]) + len(line) - 1)
    return (torch.tensor(rows, dtype=torch.int32).view(-1, words),
            torch.tensor(pos, dtype=torch.int32))


def tree_seen(mask, positions, cu, seq_len, window=0):
    """Per sequence, [new tokens, length] bool: which positions each new token sees."""
    out = []
    m = mask.cpu().tolist()
    p = positions.cpu().tolist()
    for b, n in enumerate(seq_len):
        lo, hi = cu[b], cu[b + 1]
        base = n - (hi - lo)
        s = torch.zeros((hi - lo, n), dtype=torch.bool)
        for i in range(hi - lo):
            first = max(0, p[lo + i] - window + 1) if window else 0
            s[i, first:max(base, 0)] = True
            for j in range(i + 1):
                if (m[lo + i][j // 32] >> (j % 32)) & 1 and base + j >= 0:
                    s[i, base + j] = True
        out.append(s)
    return out


def attention(q, K, V, block_table, seq_len, cu, scale, seen, absent=()):
    """y, lse, sum_j p_j |v_j| and (sum_j p_j^2 v_j^2)^1/2 of tree attention in float64;
    rows that see nothing: 0, -inf.  Values that a row does not see take no part, whatever
    they are.  absent: (sequence, block) pairs whose positions no token sees."""
    T, hq, d = q.shape
    hkv = K.shape[1]
    page, g = K.shape[2], hq // hkv
    y, mean, root = (torch.zeros((T, hq, d), dtype=torch.float64, device=q.device)
                     for _ in range(3))
    lse = torch.full((T, hq), -math.inf, dtype=torch.float64, device=q.device)
    for b, n in enumerate(seq_len):
        lo, hi = cu[b], cu[b + 1]
        if hi == lo or n == 0:
            continue
        bt = block_table[b:b + 1].clone()
        vis = seen[b].clone().to(q.device)
        for i, block in absent:
            if i == b:
                vis[:, block * page:(block + 1) * page] = False
                bt[0, block] = 0
        for h in range(hkv):
            k, v = R.rows(K, bt, 0, h, n), R.rows(V, bt, 0, h, n)
            s = torch.einsum("tgd,nd->tgn", q[lo:hi, h * g:h * g + g].double(), k) * scale
            s.masked_fill_(~vis[:, None], -math.inf)
            z = torch.logsumexp(s, -1)
            p = torch.where(vis[:, None], (s - z[..., None]).exp(), torch.zeros_like(s))
            p = torch.where(torch.isneginf(z)[..., None], torch.zeros_like(p), p)
            lse[lo:hi, h * g:h * g + g] = z
            at = slice(h * g, h * g + g)
            if torch.isfinite(v).all():
                y[lo:hi, at], mean[lo:hi, at] = p @ v, p @ v.abs()
                root[lo:hi, at] = ((p * p) @ (v * v)).sqrt()
            else:
                for i in range(hi - lo):
                    pi, vi = p[i][:, vis[i]], v[vis[i]]
                    y[lo + i, at], mean[lo + i, at] = pi @ vi, pi @ vi.abs()
                    root[lo + i, at] = ((pi * pi) @ (vi * vi)).sqrt()
    return y, lse, mean, root
