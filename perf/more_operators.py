"""Workloads of a speculative decoding step over a paged cache: pages dealt to the
requests and their tokens mapped to slots, queries and keys normalised per head and
rotated in one pass (with its gradient, and on the way into the pages), a drafted
tree of tokens attended over the cache, and the accepted path kept.

`listed()` names representative calls, `draw()` samples more of the same ranges,
`prepare()` makes a call's inputs on the GPU, and `run()` makes the call: with
`own` true through the library, otherwise as plain torch arithmetic in 32 bits.
`exact()` evaluates the definitions in 64 bits.

Shapes follow the package's workloads: 28/4 and 32/8 heads of 128 or 64 channels, 4
heads of 64 in float32, contexts of up to 32768 tokens, 28 layers.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # the scheduling of one decode step of 256 dialogues, a few of which need a page
        dict(name="deal_step_b256", op="deal", batch=256, past_lo=100, past_hi=8000, steps=0.97,
             prompts=0.0, leave=0.02, new_lo=1, new_hi=1, page=16, window=0, room=1.0, spread=1),
        # a step that admits ragged prompts beside running requests with a sliding window;
        # the pool does not hold all of them
        dict(name="deal_prompts_b64", op="deal", batch=64, past_lo=0, past_hi=16000, steps=0.5,
             prompts=0.4, leave=0.1, new_lo=201, new_hi=8000, page=32, window=4096, room=0.7,
             spread=2),
        # queries of a 16k-token prompt, normalised and rotated where the fused projection
        # left them
        dict(name="norm_prompt_16k", op="norm", tokens=16384, heads=28, other_heads=8, dim=128,
             rot=128, layout="half", per_head=False, dtype="bf16", past=0),
        # the gradient of the same over a training batch of 8k tokens
        dict(name="norm_grad_8k", op="norm_grad", tokens=8192, heads=28, other_heads=8, dim=128,
             rot=128, layout="half", per_head=False, dtype="bf16", past=0),
        # float32 keys of one small layer: weights per head, half of each head rotated,
        # neighbouring channels paired, an odd number of tokens
        dict(name="norm_grad_f32", op="norm_grad", tokens=1021, heads=4, other_heads=0, dim=64,
             rot=32, layout="pairs", per_head=True, dtype="f32", past=5000),
        # one decode step of 32 dialogues, placed by its slot map: q and k normalised and
        # rotated, k and v appended
        dict(name="append_norm_step_b32", op="append", batch=32, new_lo=1, new_hi=1, past_lo=100,
             past_hi=2047, spread=3, q_heads=32, kv_heads=8, dim=128, page=64, rot=128,
             layout="half", slots=True, tree=False, dtype="bf16"),
        # prompt chunks of eight requests, ragged, placed by their offsets
        dict(name="append_norm_chunks_b8", op="append", batch=8, new_lo=201, new_hi=2048,
             past_lo=0, past_hi=4001, spread=4, q_heads=28, kv_heads=4, dim=128, page=16, rot=128,
             layout="half", slots=False, tree=False, dtype="bf16"),
        # one request at 6k tokens, a small drafted tree: masks and attention, latency
        dict(name="tree_single", op="tree", batch=1, new_lo=16, new_hi=16, past_lo=6128,
             past_hi=6128, spread=5, q_heads=28, kv_heads=4, dim=128, page=16, window=0,
             masks=True, dtype="bf16"),
        # trees of up to 64 tokens of the whole 32k dialogue batch: the largest case
        dict(name="tree_dialogue_b32", op="tree", batch=32, new_lo=40, new_hi=64, past_lo=2048,
             past_hi=32700, spread=6, q_heads=32, kv_heads=8, dim=128, page=64, window=0,
             masks=False, dtype="bf16"),
        # float32 trees of a small layer over short contexts, sliding window
        dict(name="tree_f32_window", op="tree", batch=5, new_lo=3, new_hi=33, past_lo=0,
             past_hi=1000, spread=7, q_heads=4, kv_heads=4, dim=64, page=16, window=200,
             masks=True, dtype="f32"),
        # the accepted paths of 32 dialogues, in all 28 layers' caches
        dict(name="keep_b32_l28", op="keep", batch=32, new_lo=64, new_hi=64, past_lo=33,
             past_hi=300, spread=8, layers=28, kv_heads=8, dim=128, page=64, most=8, dtype="bf16"),
        # one request, one small float32 layer
        dict(name="keep_single_f32", op="keep", batch=1, new_lo=16, new_hi=16, past_lo=500,
             past_hi=500, spread=9, layers=1, kv_heads=4, dim=64, page=16, most=5, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    op = rng.choice(["deal", "norm", "norm_grad", "append", "tree", "tree", "tree", "keep"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    dim = rng.choice([64, 128])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    layout = rng.choice(["half", "pairs"])
    spread = rng.randrange(1 << 20)
    if op == "deal":
        batch = _log_int(rng, 1, 1024)
        most = max(2, min(16000, 600000 // batch))
        steps = rng.uniform(0.0, 1.0)
        prompts = rng.uniform(0.0, 1.0 - steps)
        new_hi = _log_int(rng, 1, most)
        return dict(op=op, batch=batch, past_lo=0, past_hi=_log_int(rng, 1, most), steps=steps,
                    prompts=prompts, leave=(1.0 - steps - prompts) / 2, new_lo=max(1, new_hi // 8),
                    new_hi=new_hi, page=page, window=rng.choice([0, 0, _log_int(rng, 16, 4096)]),
                    room=rng.choice([1.0, 1.0, rng.uniform(0.1, 1.0)]), spread=spread)
    if op in ("norm", "norm_grad"):
        dim = rng.choice([64, 80, 96, 128, 128, 256])
        return dict(op=op, tokens=_log_int(rng, 1, 8192), heads=rng.randint(1, 28),
                    other_heads=rng.choice([0, 2, 8]), dim=dim,
                    rot=rng.choice([dim // 4, dim // 2, dim]), layout=layout,
                    per_head=rng.random() < 0.3, dtype=dtype, past=_log_int(rng, 1, 100000))
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 7, 8])
    if op == "append":
        tree = rng.random() < 0.3
        batch = _log_int(rng, 1, 64)
        new_hi = rng.randint(2, 64) if tree else _log_int(rng, 1, max(1, 16384 // batch))
        return dict(op=op, batch=batch, new_lo=max(1, new_hi // 4), new_hi=new_hi, past_lo=0,
                    past_hi=_log_int(rng, 1, 4000), spread=spread,
                    q_heads=kv_heads * min(group, 4), kv_heads=kv_heads, dim=dim, page=page,
                    rot=rng.choice([dim // 4, dim // 2, dim]), layout=layout,
                    slots=rng.random() < 0.5, tree=tree, dtype=dtype)
    if op == "keep":
        new_hi = rng.randint(1, 64)
        return dict(op=op, batch=_log_int(rng, 1, 48), new_lo=max(1, new_hi // 2), new_hi=new_hi,
                    past_lo=0, past_hi=_log_int(rng, 1, 300), spread=spread,
                    layers=_log_int(rng, 1, 28), kv_heads=rng.choice([1, 2, 4, 8]), dim=dim,
                    page=page, most=rng.randint(1, 8), dtype=dtype)
    new_hi = _log_int(rng, 1, 64) if rng.random() < 0.8 else rng.randint(65, 200)
    batch = _log_int(rng, 1, 24 if dtype == "bf16" else 6)
    past_hi = _log_int(rng, 1, (32000 if new_hi <= 64 else 8000) if dtype == "bf16" else 4000)
    budget = 8.0e8 if dtype == "bf16" else 3.0e7  # query-key pairs of all heads, padded
    while batch * (new_hi + 1) * past_hi * kv_heads * group > budget:
        past_hi //= 2
    return dict(op=op, batch=batch, new_lo=max(1, new_hi // 3), new_hi=new_hi,
                past_lo=past_hi // 3, past_hi=past_hi, spread=spread, q_heads=kv_heads * group,
                kv_heads=kv_heads, dim=dim, page=page,
                window=rng.choice([0, 0, 0, _log_int(rng, 4, 4096)]), masks=rng.random() < 0.3,
                dtype=dtype)


# ---------------------------------------------------------------- sizes
def _lengths(case):
    """New and cached tokens of every sequence: a fixed spread of the case's ranges.
    A deal's new tokens may be 0 (idle) or -1 (the request leaves)."""
    rng = random.Random(case["spread"])
    new, past = [], []
    for _ in range(case["batch"]):
        lo, hi, p = case["new_lo"], case["new_hi"], rng.randint(case["past_lo"], case["past_hi"])
        n = rng.randint(lo, hi)
        if case["op"] == "deal":
            kind = rng.random()
            if kind < case["steps"]:
                n = 1
            elif kind < case["steps"] + case["prompts"]:
                p = 0
            else:
                n = -1 if kind < case["steps"] + case["prompts"] + case["leave"] else 0
        new.append(n)
        past.append(p)
    if case["op"] != "deal":
        new[rng.randrange(len(new))] = case["new_hi"]
    return new, past


def _first_kept(case, past):
    """The first block that a request of `past` cached tokens still needs."""
    w = case["window"]
    return max(0, past - w + 1) // case["page"] if w else 0


def _deal_sizes(case):
    """Pages a deal starts with: held first and end block of each request, all pages,
    blocks of a table row, packed tokens there is room for.  Requests with a window hold
    what the last step, two tokens and a page ago, left them."""
    new, past = _lengths(case)
    P = case["page"]
    held = [(max(0, _first_kept(case, max(0, p - 2 - P))), -(-p // P)) for p in past]
    used = sum(hi - lo for lo, hi in held)
    wanted = sum(max(0, -(-(p + max(n, 0)) // P) - -(-p // P)) for n, p in zip(new, past))
    pages = used + max(1, int(wanted * case["room"])) + 3
    width = max(-(-(p + max(n, 0)) // P) for n, p in zip(new, past)) + 1
    return held, pages, width, max(1, sum(max(n, 0) for n in new))


def _pairs(case):
    """Query-key pairs that the prefix leaves to one head, and keys that some query sees;
    of the tree's own pairs (few) each token's own."""
    pairs = keys = 0
    w = case["window"]
    for n, p in zip(*_lengths(case)):
        pairs += n * (min(p, w - 1) if w else p) + n
        keys += (min(p, w - 1) if w else p) + n
    return pairs, keys


def work(case):
    op = case["op"]
    if op == "deal":
        held, pages, width, tokens = _deal_sizes(case)
        new, past = _lengths(case)
        moved = sum(hi - lo for n, (lo, hi) in zip(new, held) if n < 0)
        moved += sum(max(0, -(-(p + n) // case["page"]) - hi)
                     for n, p, (lo, hi) in zip(new, past, held) if n > 0)
        return {"bytes": case["batch"] * 40 + tokens * 12 + moved * 8, "flops": 0}
    e, d = DTYPES[case["dtype"]].itemsize, case["dim"]
    if op in ("norm", "norm_grad"):
        n = case["tokens"] * case["heads"]
        rows = 2 if op == "norm" else 3
        each = 4 * d + 3 * case["rot"] if op == "norm" else 10 * d + 3 * case["rot"]
        return {"bytes": rows * n * d * e + case["tokens"] * (case["rot"] * 4 + 4),
                "flops": n * each}
    new, past = _lengths(case)
    t = sum(new)
    if op == "append":
        rows = case["q_heads"] + 2 * case["kv_heads"]
        return {"bytes": t * (2 * rows * d * e + case["rot"] * 4),
                "flops": t * (case["q_heads"] + case["kv_heads"]) * (4 * d + 3 * case["rot"])}
    if op == "keep":
        moved = sum(max(0, k - c) for k, c in _accepted(case, random.Random(case["spread"] + 1)))
        return {"bytes": case["batch"] * 16 +
                max(1, moved) * case["layers"] * case["kv_heads"] * d * e * 4, "flops": 0}
    pairs, keys = _pairs(case)
    return {"bytes": 2 * t * case["q_heads"] * d * e + 4 * t * case["q_heads"] +
            2 * keys * case["kv_heads"] * d * e + t * 4 * (-(-case["new_hi"] // 32)),
            "flops": 4 * pairs * case["q_heads"] * d}


def _accepted(case, rng):
    """Accepted tokens of every request, and how many of them already lie in order: a path
    follows the tree's first chain, then a branch that was drafted behind that chain."""
    out = []
    for n in _lengths(case)[0]:
        k = rng.randint(0, min(case["most"], n))
        out.append((k, rng.randint(max(0, 2 * k - n), k)))
    return out


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
    shape = (case.get("layers", 1), n_pages, h, page, d)
    dt = DTYPES[case["dtype"]]
    K = torch.empty(shape, dtype=dt, device="cuda").normal_(generator=gen)
    V = torch.empty(shape, dtype=dt, device="cuda").normal_(generator=gen)
    return K, V, table


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _trees(new, rng):
    """Parents of the drafted tokens: half of them continue the token before, some begin at
    the last cached token, the others branch off any earlier one."""
    out = []
    for n in new:
        for i in range(n):
            kind = rng.random()
            out.append(-1 if i == 0 or kind < 0.05 else i - 1 if kind < 0.55 else rng.randrange(i))
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = random.Random(seed)
    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    op = case["op"]
    if op == "deal":
        new, past = _lengths(case)
        held, pages, width, tokens = _deal_sizes(case)
        order = torch.randperm(pages, generator=gen, device="cuda").int()
        s["blocks"] = torch.full((len(new), width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, (lo, hi) in enumerate(held):
            s["blocks"][b, lo:hi] = order[at:at + hi - lo]
            at += hi - lo
        s["free"] = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
        s["free"][:pages - at] = order[at:]
        s["n_free"], s["held"] = _ints([pages - at]), _ints(held)
        s["new"], s["seq_len"], s["tokens"] = _ints(new), _ints(past), tokens
        # what the library's handles hold beside the lists; results
        s["pool"] = torch.zeros((pages, 1, case["page"], 8), dtype=torch.float32, device="cuda")
        s["outs"] = [torch.zeros(n, dtype=t, device="cuda") for n, t in [
            (len(new), torch.int32), ((len(new), 2), torch.int32), (1, torch.int32),
            (len(new) + 1, torch.int32), (len(new), torch.int32), (tokens, torch.int32),
            (tokens, torch.int64)]]
        return s
    dt, d = DTYPES[case["dtype"]], case["dim"]

    def weights(heads):
        shape = (heads, d) if case.get("per_head") else (d,)
        return (torch.empty(shape, device="cuda").normal_(generator=gen) * 0.1 + 1).to(dt)

    if op in ("norm", "norm_grad"):
        t, h = case["tokens"], case["heads"]
        fused = torch.empty((t, h + case["other_heads"], d), device="cuda").normal_(generator=gen)
        # projections: rows of different sizes, a few channels much larger than the others
        fused *= torch.empty((t, 1, 1), device="cuda").uniform_(0.3, 3.0, generator=gen)
        fused[..., ::37] *= 8
        s["x"] = fused.to(dt)[:, :h]
        s["weight"] = weights(h)
        s["positions"] = torch.randperm(t, generator=gen, device="cuda").int() + case["past"]
        s["table"] = _table(t + case["past"], case["rot"])
        s["out"] = torch.empty((t, h, d), dtype=dt, device="cuda")
        if op == "norm_grad":
            s["dy"] = (torch.empty((t, h, d), device="cuda").normal_(generator=gen) * 0.02).to(dt)
            s["dweight"] = torch.empty(s["weight"].shape, device="cuda")
        return s
    new, past = _lengths(case)
    total = [n + p for n, p in zip(new, past)]
    K, V, s["blocks"] = _pages(case, total, gen)
    s["seq_len"] = _ints(total)
    s["cu"] = _ints([0] + new).cumsum(0).int()
    s["max_new"], s["longest"] = max(new), max(total)
    if op == "keep":
        s["K"], s["V"] = K, V
        path = torch.full((len(new), case["most"]), -1, dtype=torch.int32)
        counts = _accepted(case, random.Random(case["spread"] + 1))
        for b, (k, c) in enumerate(counts):
            later = sorted(rng.sample(range(k, new[b]), k - c))
            path[b, :k] = torch.tensor(list(range(c)) + later, dtype=torch.int32)
        s["path"], s["accepted"] = path.cuda(), _ints([k for k, _ in counts])
        s["kept_len"] = torch.zeros_like(s["seq_len"])
        return s
    s["K"], s["V"] = K[0], V[0]
    t, hq, hkv = sum(new), case["q_heads"], case["kv_heads"]
    fused = torch.empty((t, hq + 2 * hkv, d), dtype=dt, device="cuda").normal_(generator=gen)
    s["q"], s["k"], s["v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    s["out"] = torch.empty((t, hq, d), dtype=dt, device="cuda")
    s["parents"] = _ints(_trees(new, rng))
    words = -(-max(new) // 32)
    if op == "append":
        s["q_weight"], s["k_weight"] = weights(hq), weights(hkv)
        s["table"] = _table(max(total), case["rot"])
        pos, at, off = _places(s)
        s["slots"] = at * case["page"] + off
        s["positions"] = pos.int()
        if case["tree"]:
            s["positions"] = _plain_masks(s, words)[1]
        return s
    # queries with a few strong matches: logits of standard deviation about 2
    s["q"] = (s["q"] * 2).contiguous()
    s["lse"] = torch.empty((t, hq), dtype=torch.float32, device="cuda")
    s["mask"], s["positions"] = _plain_masks(s, words)
    s["mask_out"], s["positions_out"] = torch.zeros_like(s["mask"]), torch.zeros_like(s["positions"])
    return s


# ---------------------------------------------------------------- the calls
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2607_21475_gb300 import ebd
    case, op = s["case"], s["case"]["op"]
    layout = ebd.EBD_ROTARY_PAIRS if case.get("layout") == "pairs" else ebd.EBD_ROTARY_HALF
    if op == "deal":
        pc = ebd.PagedCache(s["pool"], s["pool"], s["blocks"], s["seq_len"], s["status"])
        pool = ebd.PagePool(s["free"], s["n_free"], s["held"])
        seq_len, held, n_free, cu, served, pos, slots = s["outs"]
        ebd.ebd_paged_deal(pool, pc, s["new"], s["tokens"], window=case["window"], cu_new=cu,
                           positions=pos, slots=slots, served=served, seq_len_out=seq_len,
                           held_out=held, n_free_out=n_free)
        return {"seq_len": seq_len, "held": held, "n_free": n_free, "cu": cu, "served": served,
                "positions": pos, "slots": slots, "free": s["free"], "blocks": s["blocks"]}
    if op == "norm":
        return ebd.ebd_norm_rotary(s["x"], s["weight"], s["positions"], s["table"], out=s["out"],
                                   layout=layout, eps=EPS)
    if op == "norm_grad":
        dx, dw = ebd.ebd_norm_rotary_backward(s["dy"], s["x"], s["weight"], s["positions"],
                                              s["table"], dx=s["out"], dweight=s["dweight"],
                                              layout=layout, eps=EPS)
        return {"dx": dx, "dweight": dw}
    if op == "keep":
        pc = ebd.PagedCache(s["K"][0], s["V"][0], s["blocks"], s["seq_len"], s["status"])
        ebd.ebd_paged_keep(pc, s["cu"], s["path"], s["accepted"], seq_len_out=s["kept_len"],
                           K_layers=s["K"], V_layers=s["V"])
        return {"K": s["K"], "V": s["V"], "seq_len": s["kept_len"]}
    pc = ebd.PagedCache(s["K"], s["V"], s["blocks"], s["seq_len"], s["status"])
    if op == "append":
        where = {"slots": s["slots"], "positions": s["positions"]} if case["slots"] else (
            {"cu_new": s["cu"], "positions": s["positions"]} if case["tree"] else
            {"cu_new": s["cu"]})
        ebd.ebd_paged_append_norm(pc, s["k"], s["v"], k_weight=s["k_weight"], q=s["q"],
                                  q_weight=s["q_weight"], q_out=s["out"], table=s["table"],
                                  layout=layout, eps=EPS, **where)
        return {"K": s["K"], "V": s["V"], "q": s["out"]}
    mask, positions = s["mask"], s["positions"]
    if case["masks"]:
        mask, positions = ebd.ebd_tree_masks(s["parents"], s["cu"], s["seq_len"], s["max_new"],
                                             window=case["window"], mask=s["mask_out"],
                                             positions=s["positions_out"])
    y, lse = ebd.ebd_paged_tree_attention(s["q"], pc, s["cu"], s["max_new"], mask,
                                          positions=positions, window=case["window"], y=s["out"],
                                          lse=s["lse"])
    return {"y": y, "lse": lse, "mask": mask, "positions": positions}


def _rotated(x, cs, layout):
    """x [T, H, d] turned by cs [T, rot / 2, 2] (cos, sin), in cs's precision."""
    x = x.to(cs.dtype)
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    half = cs.shape[1]
    head, rest = x[..., :2 * half], x[..., 2 * half:]
    if layout == "pairs":
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = head[..., :half], head[..., half:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, rest], dim=-1)


def _normed(x, weight):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()


def _places(s):
    """Position, page and offset of every new token."""
    cu, n = s["cu"].long(), s["q"].shape[0]
    t = torch.arange(n, device="cuda")
    b = torch.searchsorted(cu[1:], t, right=True)
    pos = s["seq_len"].long()[b] - cu[b + 1] + t
    page = s["blocks"].long()[b, pos // s["case"]["page"]]
    return pos, page, pos % s["case"]["page"]


def _plain_masks(s, words):
    """Bit i of a token's row: it descends from the new token i of its sequence (or is it),
    fewer than `window` generations away; and its position."""
    cu, parents = s["cu"].long(), s["parents"].long()
    t = torch.arange(parents.shape[0], device="cuda")
    b = torch.searchsorted(cu[1:], t, right=True)
    window = s["case"].get("window", 0)
    sees = torch.zeros((parents.shape[0], words * 32), dtype=torch.bool, device="cuda")
    at, depth = t - cu[b], torch.zeros_like(t)
    live = torch.ones_like(t, dtype=torch.bool)
    for gen in range(s["max_new"]):
        if not window or gen < window:
            sees[t, at] |= live
        at = torch.where(live, parents[cu[b] + at], at)
        live = live & (at >= 0)
        at = at.clamp(min=0)
        depth += live
    bits = sees.view(-1, words, 32).long() << torch.arange(32, device="cuda")
    mask = bits.sum(-1)
    mask = torch.where(mask >= 1 << 31, mask - (1 << 32), mask).int()
    n_new = cu[1:] - cu[:-1]
    return mask, (s["seq_len"].long()[b] - n_new[b] + depth).int()


def _plain_deal(s):
    case = s["case"]
    P, w = case["page"], case["window"]
    new, length, held = s["new"].long(), s["seq_len"].long(), s["held"].long()
    blocks, free, width = s["blocks"], s["free"], s["blocks"].shape[1]
    B = new.shape[0]
    leaves = new < 0
    lo, hi = held[:, 0], held[:, 1]
    first = torch.zeros_like(lo)
    if w:
        first = (length - w + 1).clamp(min=0) // P
    lo2 = torch.where(leaves, hi, torch.minimum(torch.maximum(lo, first), hi))
    col = torch.arange(width, device="cuda")
    gone = (col >= lo[:, None]) & (col < lo2[:, None])
    released = blocks[gone]
    n = s["n_free"].long()
    at = n + torch.arange(released.shape[0], device="cuda")
    free[at] = released
    n = n + released.shape[0]
    after = (length + new + P - 1) // P
    fits = (new >= 0) & (after <= width)
    grows = fits & (new > 0)
    need = torch.where(grows, (after - hi).clamp(min=0), torch.zeros_like(hi))
    some = torch.where(grows, new, torch.zeros_like(new))
    ok = fits & ((need == 0) | (need.cumsum(0) <= n)) & (some.cumsum(0) <= s["tokens"])
    need, some = need * ok, some * ok
    before = need.cumsum(0) - need
    take = (col >= hi[:, None]) & (col < (hi + need)[:, None])
    which = (n - 1 - before - (col - hi[:, None]).T).T
    blocks[take] = free[which[take]]
    served = (ok | leaves).int()
    zero = torch.zeros_like(hi)
    held2 = torch.stack([torch.where(leaves, zero, lo2),
                         torch.where(leaves, zero, hi + need)], 1).int()
    length2 = torch.where(leaves, zero, length + some).int()
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    cu[1:] = some.cumsum(0)
    t = torch.arange(s["tokens"], device="cuda")
    b = torch.searchsorted(cu[1:].long(), t, right=True).clamp(max=B - 1)
    live = t < cu[-1]
    pos = torch.where(live, length[b] + t - cu[b], torch.zeros_like(t))
    slots = torch.where(live, blocks[b, pos // P].long() * P + pos % P, torch.full_like(t, -1))
    return {"seq_len": length2, "held": held2, "n_free": (n - need.sum()).int(), "cu": cu,
            "served": served, "positions": pos.int(), "slots": slots, "free": free,
            "blocks": blocks}


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "deal":
        return _plain_deal(s)
    dt = DTYPES[case["dtype"]]
    if op == "norm":
        cs = s["table"][s["positions"].long()]
        return _rotated(_normed(s["x"], s["weight"]), cs, case["layout"]).to(dt)
    if op == "norm_grad":
        cs = s["table"][s["positions"].long()] * torch.tensor([1.0, -1.0], device="cuda")
        back = _rotated(s["dy"].float(), cs, case["layout"])
        x = s["x"].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        x = x * r
        g = back * s["weight"].float()
        dx = (g - x * (g * x).mean(-1, keepdim=True)) * r
        dw = (back * x).sum(0) if case["per_head"] else (back * x).sum((0, 1))
        return {"dx": dx.to(dt), "dweight": dw}
    page = case["page"]
    if op == "append":
        pos, at, off = _places(s)
        cs = s["table"][s["positions"].long()]
        s["K"][at, :, off] = _rotated(_normed(s["k"], s["k_weight"]), cs, case["layout"]).to(dt)
        s["V"][at, :, off] = s["v"]
        q = _rotated(_normed(s["q"], s["q_weight"]), cs, case["layout"]).to(dt)
        return {"K": s["K"], "V": s["V"], "q": q}
    cu, lens = s["cu"].long(), s["seq_len"].long()
    n_new = cu[1:] - cu[:-1]
    if op == "keep":
        path, k = s["path"].long(), s["accepted"].long()
        i = torch.arange(path.shape[1], device="cuda")
        b, i = torch.nonzero(i < k[:, None], as_tuple=True)
        base = (lens - n_new)[b]
        src, dst = base + path[b, i], base + i
        at, to = s["blocks"].long()[b, src // page], s["blocks"].long()[b, dst // page]
        for pool in (s["K"], s["V"]):
            pool[:, to, :, dst % page] = pool[:, at, :, src % page]
        return {"K": s["K"], "V": s["V"], "seq_len": (lens - n_new + k).int()}
    mask, positions = s["mask"], s["positions"]
    if case["masks"]:
        mask, positions = _plain_masks(s, s["mask"].shape[1])
    B, hkv, d, n, L = case["batch"], case["kv_heads"], case["dim"], s["max_new"], s["longest"]
    g = case["q_heads"] // hkv
    pos = torch.arange(L, device="cuda")
    at = s["blocks"].long()[:, pos // page]
    K = s["K"][at, :, pos % page].permute(0, 2, 1, 3).float()  # [B, Hkv, L, d]
    V = s["V"][at, :, pos % page].permute(0, 2, 1, 3).float()
    i = torch.arange(n, device="cuda")
    rows = (cu[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    there = i < n_new[:, None]
    q = s["q"][rows].float().view(B, n, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * g, d)
    S = torch.matmul(q * d ** -0.5, K.transpose(2, 3)).view(B, hkv, n, g, L)
    base = lens - n_new
    seen = (pos < base[:, None])[:, None].expand(B, n, L)  # the prefix
    if case["window"]:
        seen = seen & (pos > (positions[rows] - case["window"])[..., None])
    bit = pos - base[:, None]                              # [B, L]: number of the new token
    own_tree = (bit >= 0) & (bit < n_new[:, None])
    bit = bit.clamp(0, 32 * mask.shape[1] - 1)[:, None].expand(B, n, L)
    bits = (mask[rows].long().gather(2, bit // 32) >> (bit % 32)) & 1
    seen = seen | (own_tree[:, None] & (bits == 1))
    S.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = S.amax(-1, keepdim=True).clamp(min=-1e30)
    S.sub_(top).exp_()
    total = S.sum(-1, keepdim=True)
    y = torch.matmul(S.view(B, hkv, n * g, L), V).view(B, hkv, n, g, d) / total
    y = y.permute(0, 2, 1, 3, 4).reshape(B, n, hkv * g, d)[there]
    lse = (top + total.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, n, hkv * g)[there]
    return {"y": y.to(dt), "lse": lse, "mask": mask, "positions": positions}


# ---------------------------------------------------------------- in 64 bits
def exact(case, seed):
    op = case["op"]
    if op in ("deal", "keep"):
        return None  # whole numbers and copied rows: nothing is computed
    if work(case)["flops"] > 6e12:
        return None
    s = prepare(case, seed)
    if op == "norm":
        cs = torch.view_as_complex(s["table"][s["positions"].long()].double())
        return _turn64(_unit64(s["x"]) * s["weight"].double(), cs, case["layout"])
    if op == "norm_grad":
        cs = torch.view_as_complex(s["table"][s["positions"].long()].double())
        u = _turn64(s["dy"], cs.conj(), case["layout"])
        x = s["x"].double()
        size = (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
        along = (u * s["weight"].double() * x).sum(-1, keepdim=True) / x.shape[-1]
        dx = u * s["weight"].double() / size - x * along / size ** 3
        dw = (u * x / size).sum(dim=0)
        return {"dx": dx, "dweight": dw if case["per_head"] else dw.sum(dim=0)}
    page, d, hkv = case["page"], case["dim"], case["kv_heads"]
    g = case["q_heads"] // hkv
    cu, lens = s["cu"].tolist(), s["seq_len"].tolist()
    if op == "append":
        K, V = s["K"].double(), s["V"].double()
        q = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            lo, hi = cu[b], cu[b + 1]
            pos = torch.arange(n - (hi - lo), n, device="cuda")
            cs = torch.view_as_complex(s["table"][s["positions"][lo:hi].long()].double())
            where = s["blocks"][b].long()[torch.div(pos, page, rounding_mode="floor")]
            k = _unit64(s["k"][lo:hi]) * s["k_weight"].double()
            K[where, :, pos % page] = _turn64(k, cs, case["layout"])
            V[where, :, pos % page] = s["v"][lo:hi].double()
            q[lo:hi] = _turn64(_unit64(s["q"][lo:hi]) * s["q_weight"].double(), cs, case["layout"])
        return {"K": K, "V": V, "q": q}
    y = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    parents, w = s["parents"].tolist(), case["window"]
    for b, n in enumerate(lens):
        lo, hi = cu[b], cu[b + 1]
        base = n - (hi - lo)
        seen = torch.zeros((hi - lo, n), dtype=torch.bool)
        for i in range(hi - lo):
            line = [i]
            while parents[lo + line[-1]] >= 0:
                line.append(parents[lo + line[-1]])
            at = base + len(line) - 1
            seen[i, max(0, at - w + 1) if w else 0:base] = True
            seen[i, [base + j for j in (line[:w] if w else line)]] = True
        hide = ~seen.cuda()
        mine = s["blocks"][b, :-(-n // page)].long()
        for h in range(hkv):
            k = s["K"][mine, h].reshape(-1, d)[:n].double()
            v = s["V"][mine, h].reshape(-1, d)[:n].double()
            for j in range(h * g, h * g + g):
                z = (s["q"][lo:hi, j].double() @ k.T) / math.sqrt(d)
                z = z.masked_fill(hide, -math.inf)
                lse[lo:hi, j] = torch.logsumexp(z, dim=1)
                y[lo:hi, j] = torch.exp(z - lse[lo:hi, j, None]) @ v
    return {"y": y, "lse": lse, "mask": None, "positions": None}


def _unit64(x):
    x = x.double()
    return x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()


def _turn64(x, cs, layout):
    """Rotation as a complex product: the pair (a, b) is a + ib, turned by cos + i sin."""
    x = x.double()
    r = 2 * cs.shape[1]
    z = x[..., :r].unflatten(-1, (-1, 2) if layout == "pairs" else (2, -1))
    z = z if layout == "pairs" else z.transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * cs[:, None])
    z = z if layout == "pairs" else z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), x[..., r:]], dim=-1)
