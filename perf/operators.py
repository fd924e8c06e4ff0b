"""Workloads of the paged-cache operators: rotary positions, appending new keys and
values to a paged cache, attention of new tokens over it, and gathering an
eviction's kept rows out of it.

`listed()` names representative calls, `draw()` samples more of the same ranges,
`prepare()` makes a call's inputs on the GPU, and `run()` makes the call: with
`own` true through the library, otherwise as plain torch arithmetic in 32 bits.
`exact()` evaluates the definitions in 64 bits.

Shapes follow the package's workloads: 28/4 and 32/8 heads of 128 or 64
channels, 4/4 heads of 64 in float32, contexts of 512 to 32768 tokens.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # queries of a 16k-token prompt, rotated where the fused projection left them
        dict(name="rotary_prompt_16k", op="rotary", tokens=16384, heads=28, other_heads=8, dim=128,
             rot=128, layout="half", inverse=False, dtype="bf16", past=0),
        # float32 keys of one small layer moved back to position 0 (the gradient's direction),
        # half of each head rotated, neighbouring channels paired
        dict(name="rotary_back_f32", op="rotary", tokens=1021, heads=4, other_heads=0, dim=64,
             rot=32, layout="pairs", inverse=True, dtype="f32", past=5000),
        # one decode step of 32 dialogues: q and k rotated, k and v appended
        dict(name="append_step_b32", op="append", batch=32, new_lo=1, new_hi=1, singles=0.0,
             past_lo=100, past_hi=2047, spread=1, q_heads=32, kv_heads=8, dim=128, page=64,
             rot=128, layout="half", dtype="bf16"),
        # prompt chunks of eight requests, ragged, pages of 16 tokens, half of each head rotated
        dict(name="append_chunks_b8", op="append", batch=8, new_lo=201, new_hi=2048, singles=0.0,
             past_lo=0, past_hi=4001, spread=2, q_heads=28, kv_heads=4, dim=128, page=16,
             rot=64, layout="half", dtype="bf16"),
        # the whole decode batch of the 32k dialogue: the bandwidth-bound extreme
        dict(name="attn_step_dialogue", op="attention", batch=32, new_lo=1, new_hi=1, singles=0.0,
             past_lo=2048, past_hi=32767, spread=3, q_heads=32, kv_heads=8, dim=128, page=64,
             window=0, dtype="bf16"),
        # one request at 6k tokens, one token: latency
        dict(name="attn_step_single", op="attention", batch=1, new_lo=1, new_hi=1, singles=0.0,
             past_lo=6143, past_hi=6143, spread=4, q_heads=28, kv_heads=4, dim=128, page=16,
             window=0, dtype="bf16"),
        # five drafted tokens of eight requests scored in one call
        dict(name="attn_draft_b8", op="attention", batch=8, new_lo=5, new_hi=5, singles=0.0,
             past_lo=6139, past_hi=16379, spread=5, q_heads=32, kv_heads=8, dim=128, page=64,
             window=0, dtype="bf16"),
        # the last 4096-token chunk of a 16k prompt: the arithmetic-bound extreme
        dict(name="attn_chunk_16k", op="attention", batch=1, new_lo=4096, new_hi=4096, singles=0.0,
             past_lo=12288, past_hi=12288, spread=6, q_heads=28, kv_heads=4, dim=128, page=128,
             window=0, dtype="bf16"),
        # a serving batch that mixes decode steps with odd prompt chunks, sliding window, head 64
        dict(name="attn_mixed_window", op="attention", batch=16, new_lo=33, new_hi=1021,
             singles=0.5, past_lo=0, past_hi=4003, spread=7, q_heads=32, kv_heads=8, dim=64,
             page=32, window=1024, dtype="bf16"),
        # short float32 prompts of the small layer
        dict(name="attn_prompt_f32", op="attention", batch=3, new_lo=97, new_hi=512, singles=0.0,
             past_lo=0, past_hi=511, spread=8, q_heads=4, kv_heads=4, dim=64, page=16, window=0,
             dtype="f32"),
        # the kept quarter of 16k-token caches
        dict(name="gather_16k_b25", op="gather", batch=8, past_lo=12001, past_hi=16384, spread=9,
             kv_heads=4, dim=128, page=64, keep=0.25, dtype="bf16"),
        # the kept tenth of one small float32 cache
        dict(name="gather_small_f32", op="gather", batch=1, past_lo=512, past_hi=512, spread=10,
             kv_heads=4, dim=64, page=16, keep=0.1, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    op = rng.choice(["rotary", "append", "attention", "attention", "attention", "gather"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    dim = rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 7, 8])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    layout = rng.choice(["half", "pairs"])
    spread = rng.randrange(1 << 20)
    if op == "rotary":
        return dict(op=op, tokens=_log_int(rng, 1, 16384), heads=rng.randint(1, 28),
                    other_heads=rng.choice([0, 2, 8]), dim=dim,
                    rot=rng.choice([dim // 4, dim // 2, dim]), layout=layout,
                    inverse=rng.random() < 0.5, dtype=dtype, past=_log_int(rng, 1, 100000))
    if op == "gather":
        batch = _log_int(rng, 1, 16)
        hi = _log_int(rng, 16, 16384 if batch <= 8 else 8192)
        return dict(op=op, batch=batch, past_lo=max(1, hi // 2), past_hi=hi, spread=spread,
                    kv_heads=rng.choice([1, 2, 4]), dim=dim, page=page,
                    keep=rng.uniform(0.02, 0.5 if dtype == "bf16" else 0.25), dtype=dtype)
    if op == "append":
        batch = _log_int(rng, 1, 64)
        new_hi = _log_int(rng, 1, max(1, 16384 // batch))
        past_hi = _log_int(rng, 1, 4000)
        return dict(op=op, batch=batch, new_lo=max(1, new_hi // 4), new_hi=new_hi,
                    singles=rng.choice([0.0, 0.5]), past_lo=0, past_hi=past_hi, spread=spread,
                    q_heads=kv_heads * min(group, 4), kv_heads=kv_heads, dim=dim, page=page,
                    rot=rng.choice([dim // 4, dim // 2, dim]), layout=layout, dtype=dtype)
    kind = rng.choice(["step", "step", "few", "chunk", "chunk"])
    window = rng.choice([0, 0, 0, _log_int(rng, 16, 4096)])
    if kind in ("step", "few"):
        new_hi = 1 if kind == "step" else rng.randint(2, 16)
        batch = _log_int(rng, 1, 24 if dtype == "bf16" else 8)
        past_hi = _log_int(rng, 1, 32000 if kind == "step" else 8000)
        singles = 0.0
    else:
        budget = 6.0e7 if dtype == "bf16" else 1.0e6  # query-key pairs of one head, padded
        batch = _log_int(rng, 1, 16)
        new_hi = _log_int(rng, 17, 4096 if dtype == "bf16" else 600)
        while batch > 1 and batch * new_hi * (new_hi + 500) > budget:
            batch = max(1, batch // 2)
        while batch * new_hi * (new_hi + 500) > budget:
            new_hi = max(17, new_hi // 2)
        past_hi = _log_int(rng, 1, max(2, min(16000, int(budget / (batch * new_hi)) - new_hi)))
        kv_heads = min(kv_heads, 4)
        group = min(group, 7)
        singles = rng.choice([0.0, 0.3])
    return dict(op=op, batch=batch, new_lo=max(1, new_hi // 3), new_hi=new_hi, singles=singles,
                past_lo=past_hi // 3, past_hi=past_hi, spread=spread, q_heads=kv_heads * group,
                kv_heads=kv_heads, dim=dim, page=page, window=window, dtype=dtype)


# ---------------------------------------------------------------- sizes
def _lengths(case):
    """New and cached tokens of every sequence: a fixed spread of the case's ranges."""
    rng = random.Random(case["spread"])
    new, past = [], []
    for _ in range(case["batch"]):
        lo, hi = case.get("new_lo", 0), case.get("new_hi", 0)
        new.append(1 if hi and rng.random() < case["singles"] else rng.randint(lo, hi))
        past.append(rng.randint(case["past_lo"], case["past_hi"]))
    if case["op"] != "gather":
        new[rng.randrange(len(new))] = case["new_hi"]
    return new, past


def _visible(case):
    """Query-key pairs that one head's mask leaves, and keys that some query sees."""
    pairs = keys = 0
    w = case["window"]
    for n, p in zip(*_lengths(case)):
        for_each = n * p + n * (n + 1) // 2 if w == 0 else sum(min(p + i + 1, w) for i in range(n))
        pairs += for_each
        keys += p + n if w == 0 else min(p + n, n + w - 1)
    return pairs, keys


def work(case):
    e = DTYPES[case["dtype"]].itemsize
    d = case["dim"]
    if case["op"] == "rotary":
        n = case["tokens"] * case["heads"]
        return {"bytes": 2 * n * d * e + case["tokens"] * (case["rot"] * 4 + 4),
                "flops": n * case["rot"] * 3}
    new, past = _lengths(case)
    t = sum(new)
    if case["op"] == "append":
        rows = case["q_heads"] + 2 * case["kv_heads"]
        return {"bytes": t * (2 * rows * d * e + case["rot"] * 4),
                "flops": t * (case["q_heads"] + case["kv_heads"]) * case["rot"] * 3}
    if case["op"] == "gather":
        kept = sum(_kept(case, p) for p in past) * case["kv_heads"]
        return {"bytes": kept * (4 * d * e + 4), "flops": 0}
    pairs, keys = _visible(case)
    return {"bytes": 2 * t * case["q_heads"] * d * e + 4 * t * case["q_heads"] +
            2 * keys * case["kv_heads"] * d * e,
            "flops": 4 * pairs * case["q_heads"] * d}


def _kept(case, n):
    return max(1, int(round(case["keep"] * n)))


# ---------------------------------------------------------------- inputs
def _table(n_pos, rot):
    """(cos, sin) of each position and pair: base 10000, formed in 64 bits."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * inv.cuda()
    return torch.stack([a.cos(), a.sin()], dim=-1).float()


def _pages(case, lens, gen):
    """A pool whose pages are dealt to the sequences in random order, a few of them to nobody."""
    page, h, d = case["page"], case["kv_heads"], case["dim"]
    blocks = [-(-n // page) for n in lens]
    n_pages, width = sum(blocks) + 3, max(max(blocks), 1)
    order = torch.randperm(n_pages, generator=gen, device="cuda").int()
    table = torch.zeros((len(lens), width), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    dt = DTYPES[case["dtype"]]
    K = torch.empty((n_pages, h, page, d), dtype=dt, device="cuda").normal_(generator=gen)
    V = torch.empty((n_pages, h, page, d), dtype=dt, device="cuda").normal_(generator=gen)
    return K, V, table


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, d = DTYPES[case["dtype"]], case["dim"]
    s = {"case": case}
    if case["op"] == "rotary":
        t, h = case["tokens"], case["heads"]
        fused = torch.empty((t, h + case["other_heads"], d), dtype=dt, device="cuda")
        fused.normal_(generator=gen)
        s["x"] = fused[:, :h]
        s["positions"] = torch.randperm(t, generator=gen, device="cuda").int() + case["past"]
        s["table"] = _table(t + case["past"], case["rot"])
        s["out"] = torch.empty((t, h, d), dtype=dt, device="cuda")
        return s
    new, past = _lengths(case)
    total = [n + p for n, p in zip(new, past)]
    s["K"], s["V"], s["blocks"] = _pages(case, total, gen)
    s["seq_len"] = torch.tensor(total, dtype=torch.int32, device="cuda")
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    s["longest"] = max(total)
    if case["op"] == "gather":
        h = case["kv_heads"]
        kept = [_kept(case, n) for n in total]
        cap = -(-max(kept) // 64) * 64
        s["idx"] = torch.zeros((len(new), h, cap), dtype=torch.int32, device="cuda")
        for b, (n, k) in enumerate(zip(total, kept)):
            pick = torch.rand((h, n), generator=gen, device="cuda").topk(k, dim=1).indices
            s["idx"][b, :, :k] = pick.sort(dim=1).values.int()
        s["n_kept"] = torch.tensor(kept, dtype=torch.int32, device="cuda")[:, None].repeat(1, h)
        s["Kc"] = torch.zeros((len(new), h, cap, d), dtype=dt, device="cuda")
        s["Vc"] = torch.zeros_like(s["Kc"])
        s["logw"] = torch.zeros((len(new), h, cap), dtype=torch.float32, device="cuda")
        return s
    t, hq, hkv = sum(new), case["q_heads"], case["kv_heads"]
    s["cu"] = torch.tensor([0] + new, dtype=torch.int32, device="cuda").cumsum(0).int()
    s["max_new"] = max(new)
    fused = torch.empty((t, hq + 2 * hkv, d), dtype=dt, device="cuda").normal_(generator=gen)
    s["q"], s["k"], s["v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    s["out"] = torch.empty((t, hq, d), dtype=dt, device="cuda")
    if case["op"] == "append":
        s["table"] = _table(max(total), case["rot"])
    else:
        # queries with a few strong matches: logits of standard deviation about 2
        s["q"] = (s["q"] * 2).contiguous()
        s["lse"] = torch.empty((t, hq), dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------- the calls
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2607_21475_gb300 import ebd
    case, op = s["case"], s["case"]["op"]
    layout = ebd.EBD_ROTARY_PAIRS if case.get("layout") == "pairs" else ebd.EBD_ROTARY_HALF
    if op == "rotary":
        return ebd.ebd_rotary(s["x"], s["positions"], s["table"], out=s["out"], layout=layout,
                              inverse=case["inverse"])
    pc = ebd.PagedCache(s["K"], s["V"], s["blocks"], s["seq_len"], s["status"])
    if op == "append":
        ebd.ebd_paged_append(pc, s["k"], s["v"], s["cu"], table=s["table"], layout=layout,
                             q=s["q"], q_out=s["out"])
        return {"K": s["K"], "V": s["V"], "q": s["out"]}
    if op == "gather":
        out = ebd.CompactCache(s["Kc"], s["Vc"], s["logw"], s["idx"], s["n_kept"], s["status"])
        ebd.ebd_paged_gather(pc, out)
        return {"K": s["Kc"], "V": s["Vc"]}
    y, lse = ebd.ebd_paged_attention(s["q"], pc, s["cu"], s["max_new"], window=case["window"],
                                     y=s["out"], lse=s["lse"])
    return {"y": y, "lse": lse}


def _rotated(x, cs, layout, inverse):
    """x [T, H, d] turned by cs [T, rot / 2, 2] (cos, sin), in cs's precision."""
    x = x.to(cs.dtype)
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    if inverse:
        sin = -sin
    half = cs.shape[1]
    head, rest = x[..., :2 * half], x[..., 2 * half:]
    if layout == "pairs":
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = head[..., :half], head[..., half:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, rest], dim=-1)


def _places(s):
    """Sequence, position, page and offset of every new token."""
    cu, n = s["cu"].long(), s["q"].shape[0]
    t = torch.arange(n, device="cuda")
    b = torch.searchsorted(cu[1:], t, right=True)
    pos = s["seq_len"].long()[b] - cu[b + 1] + t
    page = s["blocks"].long()[b, pos // s["case"]["page"]]
    return pos, page, pos % s["case"]["page"]


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    dt = DTYPES[case["dtype"]]
    if op == "rotary":
        cs = s["table"][s["positions"].long()]
        return _rotated(s["x"], cs, case["layout"], case["inverse"]).to(dt)
    page = case["page"]
    if op == "append":
        pos, at, off = _places(s)
        cs = s["table"][pos]
        s["K"][at, :, off] = _rotated(s["k"], cs, case["layout"], False).to(dt)
        s["V"][at, :, off] = s["v"]
        return {"K": s["K"], "V": s["V"], "q": _rotated(s["q"], cs, case["layout"], False).to(dt)}
    if op == "gather":
        idx = s["idx"].long()
        cap, h = idx.shape[2], idx.shape[1]
        live = torch.arange(cap, device="cuda") < s["n_kept"][..., None]
        b = torch.arange(idx.shape[0], device="cuda")[:, None, None]
        at = s["blocks"].long()[b, idx // page]
        heads = torch.arange(h, device="cuda")[None, :, None]
        K, V = s["K"][at, heads, idx % page], s["V"][at, heads, idx % page]
        zero = torch.zeros((), dtype=dt, device="cuda")
        return {"K": torch.where(live[..., None], K, zero),
                "V": torch.where(live[..., None], V, zero)}
    B, hkv, d, n, L = case["batch"], case["kv_heads"], case["dim"], s["max_new"], s["longest"]
    g = case["q_heads"] // hkv
    pos = torch.arange(L, device="cuda")
    at = s["blocks"].long()[:, pos // page]
    K = s["K"][at, :, pos % page].permute(0, 2, 1, 3).float()  # [B, Hkv, L, d]
    V = s["V"][at, :, pos % page].permute(0, 2, 1, 3).float()
    cu, lens = s["cu"].long(), s["seq_len"].long()
    i = torch.arange(n, device="cuda")
    rows = (cu[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    there = i < (cu[1:] - cu[:-1])[:, None]
    q = s["q"][rows].float().view(B, n, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * g, d)
    S = torch.matmul(q * d ** -0.5, K.transpose(2, 3)).view(B, hkv, n, g, L)
    last = (lens - (cu[1:] - cu[:-1]))[:, None] + i  # position of each new token
    seen = pos <= last[..., None]
    if case["window"]:
        seen &= pos > (last - case["window"])[..., None]
    S.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = S.amax(-1, keepdim=True).clamp(min=-1e30)
    S.sub_(top).exp_()
    total = S.sum(-1, keepdim=True)
    y = torch.matmul(S.view(B, hkv, n * g, L), V).view(B, hkv, n, g, d) / total
    y = y.permute(0, 2, 1, 3, 4).reshape(B, n, hkv * g, d)[there]
    lse = (top + total.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, n, hkv * g)[there]
    return {"y": y.to(dt), "lse": lse}


# ---------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op, dev = case["op"], "cuda"
    if op == "gather":
        return None  # rows are copied: nothing is computed
    if op == "rotary":
        cs = torch.view_as_complex(s["table"][s["positions"].long()].double())
        return _turn64(s["x"], cs.conj() if case["inverse"] else cs, case["layout"])
    page, d, hkv = case["page"], case["dim"], case["kv_heads"]
    g = case["q_heads"] // hkv
    cu, lens = s["cu"].tolist(), s["seq_len"].tolist()
    if op == "append":
        K, V = s["K"].double(), s["V"].double()
        q = torch.empty(s["q"].shape, dtype=torch.float64, device=dev)
        for b, n in enumerate(lens):
            lo, hi = cu[b], cu[b + 1]
            pos = torch.arange(n - (hi - lo), n, device=dev)
            cs = torch.view_as_complex(s["table"][pos].double())
            where = s["blocks"][b].long()[torch.div(pos, page, rounding_mode="floor")]
            K[where, :, pos % page] = _turn64(s["k"][lo:hi], cs, case["layout"])
            V[where, :, pos % page] = s["v"][lo:hi].double()
            q[lo:hi] = _turn64(s["q"][lo:hi], cs, case["layout"])
        return {"K": K, "V": V, "q": q}
    if work(case)["flops"] > 6e12:
        return None
    y = torch.empty(s["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=dev)
    for b, n in enumerate(lens):
        lo, hi = cu[b], cu[b + 1]
        mine = s["blocks"][b, :-(-n // page)].long()
        first = n - (hi - lo)
        keys = torch.arange(n, device=dev)
        at = torch.arange(first, n, device=dev)[:, None]
        hide = keys > at
        if case["window"]:
            hide |= keys <= at - case["window"]
        for h in range(hkv):
            k = s["K"][mine, h].reshape(-1, d)[:n].double()
            v = s["V"][mine, h].reshape(-1, d)[:n].double()
            for j in range(h * g, h * g + g):
                z = (s["q"][lo:hi, j].double() @ k.T) / math.sqrt(d)
                z = z.masked_fill(hide, -math.inf)
                lse[lo:hi, j] = torch.logsumexp(z, dim=1)
                y[lo:hi, j] = torch.exp(z - lse[lo:hi, j, None]) @ v
    return {"y": y, "lse": lse}


def _turn64(x, cs, layout):
    """Rotation as a complex product: the pair (a, b) is a + ib, turned by cos + i sin."""
    x = x.double()
    r = 2 * cs.shape[1]
    z = x[..., :r].unflatten(-1, (-1, 2) if layout == "pairs" else (2, -1))
    z = z if layout == "pairs" else z.transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * cs[:, None])
    z = z if layout == "pairs" else z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), x[..., r:]], dim=-1)
