"""A speculative step's operators against plain forms of them.

Bounds, u = 2^-24 (a float32 rounding), one rounding to the type at the end:

* norm and rotation: a row's sum of squares is of non-negative terms added in at most 16
  steps by a lane and 5 across lanes, 21 u relative; the root halves that and with its
  own roundings r is off by 13 u, w r and x (w r) by one more each, the three roundings of
  the turn by 3 u of the terms' size: 18 u (|a cos| + |b sin|).  24 u is asked.
* its gradient: u = R^T dy is off by 3 u of its terms' size, u w by one more; the sum of
  u w x by 21 u of its terms' beside, r by 13 u: dx is off by at most 48 u of
  r (|u| w + |z| mean(|u| w |z|)) with the terms' sizes for |u|.  A weight's gradient adds
  products that are off by 20 u in at most 100 steps for the sizes here: 120 u of the
  sum of the terms' sizes.
* trees: as for causal attention (attention_bound), log-sum-exp 2e-5.
* whole numbers and moved rows: equal.
"""
import math
import random

import pytest
import torch

import paged_ref as R
import speculative_ref as S

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def E():
    from paper_2607_21475_gb300 import ebd
    ebd.lib()
    return ebd


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def cache(E, s):
    return E.PagedCache(s["K"], s["V"], s["bt"], s["seq_len"],
                        torch.zeros(1, dtype=torch.int32, device="cuda"))


def table_of(E, rot, n_pos):
    f, m = E.rotary_frequencies(rot)
    return E.ebd_rotary_table(f, n_pos, m)


def within(got, ref, e, dtype):
    """got lies between the rounded values of ref - e and ref + e."""
    low, high = ((ref - e).to(torch.float32).to(dtype), (ref + e).to(torch.float32).to(dtype))
    if dtype == torch.float32:
        low, high = ref - e - U * ref.abs(), ref + e + U * ref.abs()
    assert ((low <= got) & (got <= high)).all()


# ---------------------------------------------------------------- pages
def fresh_pool(E, B, n_pages, P, max_blocks):
    pc = E.alloc_paged(B, 1, n_pages, P, 8, max_blocks, torch.float32, "cuda")
    return E.alloc_page_pool(B, n_pages, "cuda"), pc


def run_steps(E, B, n_pages, P, max_blocks, n_tokens, window, steps, seed):
    """Steps in place against the plain form, request by request."""
    rng = random.Random(seed)
    pool, pc = fresh_pool(E, B, n_pages, P, max_blocks)
    order = list(range(n_pages))
    rng.shuffle(order)
    pool.free_pages.copy_(ints(order))
    pc.block_table.fill_(-7)
    free, table = list(order), [[-7] * max_blocks for _ in range(B)]
    length, held = [0] * B, [[0, 0]] * B
    short = 0
    for make in steps:
        new = [make(rng, length[b]) for b in range(B)]
        cu, pos, slots, served = E.ebd_paged_deal(pool, pc, ints(new), n_tokens, window=window)
        length, held, cu_r, served_r, pos_r, slots_r = S.deal(
            P, n_pages, max_blocks, n_tokens, window, new, length, held, free, table)
        assert pc.seq_len.tolist() == length and pool.held.tolist() == held
        assert cu.tolist() == cu_r and served.tolist() == served_r
        assert pos.tolist() == pos_r and slots.tolist() == slots_r
        n = pool.n_free.item()
        assert n == len(free) and pool.free_pages[:n].tolist() == free
        assert pc.block_table.tolist() == table
        out = [p for b in range(B) for p in table[b][held[b][0]:held[b][1]]]
        assert sorted(out + free) == list(range(n_pages))  # no page twice, none lost
        want = E.EBD_DEV_CAPACITY if 0 in served_r else 0
        assert pc.dev_status.item() == want
        pc.dev_status.zero_()
        short += 0 in served_r
    return short


def mixed(rng, n):
    k = rng.random()
    return (rng.randint(1, 70) if k < 0.3 else 1) if k < 0.7 or n == 0 else -1 if k < 0.85 else 0


@pytest.mark.parametrize("B,P,window", [(1, 8, 0), (7, 16, 0), (33, 8, 20), (100, 64, 100),
                                        (1000, 16, 0), (1500, 8, 33)])
def test_deal(E, B, P, window):
    blocks = 400 // P
    run_steps(E, B, B * blocks + 1, P, blocks, 70 * B, window, [mixed] * 6, B)


@pytest.mark.parametrize("B,n_pages,n_tokens", [(9, 30, 500), (40, 90, 900), (40, 600, 150),
                                                (1200, 2000, 9000), (3, 1, 5)])
def test_deal_with_too_few_pages_or_places(E, B, n_pages, n_tokens):
    assert run_steps(E, B, n_pages, 8, 40, n_tokens, 0, [mixed] * 6, n_pages) > 0


def test_deal_rows_without_room(E):
    assert run_steps(E, 5, 100, 8, 3, 200, 0, [lambda r, n: r.choice([1, 9, 30])] * 4, 1) > 0


def test_deal_long_prompts_many_requests(E):
    """Large enough for the clustered form, offsets beyond shared memory among them."""
    def prompt(rng, n):
        return rng.choice([0, 1, 700, 3000]) if n == 0 else rng.choice([1, 1, -1])
    run_steps(E, 70, 9000, 16, 200, 80000, 0, [prompt] * 3, 3)
    run_steps(E, 9001, 9100, 8, 4, 9100, 0, [lambda r, n: r.choice([0, 1, 1])] * 2, 4)
    run_steps(E, 65535, 65535, 8, 2, 65535, 8, [lambda r, n: r.choice([0, 1, -1])] * 2, 5)


def test_deal_keeps_given_outputs_apart(E):
    """The same inputs twice, results elsewhere: the same results, inputs unchanged."""
    pool, pc = fresh_pool(E, 3, 20, 8, 5)
    E.ebd_paged_deal(pool, pc, ints([10, 3, 20]), 40)
    before = [pc.seq_len.clone(), pool.held.clone(), pool.n_free.clone()]
    outs = []
    for _ in range(2):
        o = [torch.full_like(t, 77) for t in before]
        cu, pos, slots, _ = E.ebd_paged_deal(pool, pc, ints([1, -1, 6]), 8, seq_len_out=o[0],
                                             held_out=o[1], n_free_out=o[2])
        outs.append([*o, cu, pos, slots, pool.free_pages.clone(), pc.block_table.clone()])
        assert all(torch.equal(a, b) for a, b in zip(before, [pc.seq_len, pool.held, pool.n_free]))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert outs[0][0].tolist() == [11, 0, 26]


def test_deal_clamps_what_is_out_of_range(E):
    pool, pc = fresh_pool(E, 4, 10, 8, 4)
    pool.held.copy_(ints([[0, 9], [3, 1], [-2, 1], [0, 0]]))
    pc.seq_len.copy_(ints([8, -5, 8, 0]))
    pool.n_free.fill_(99)
    cu, pos, slots, served = E.ebd_paged_deal(pool, pc, ints([-1, 1, 0, 5]), 16)
    assert pc.dev_status.item() & E.EBD_DEV_RANGE
    assert 0 <= pool.n_free.item() <= 10 and (pool.held >= 0).all() and (pool.held <= 4).all()
    # a page number outside the pool in the list is dealt, told, and leads nowhere
    pool, pc = fresh_pool(E, 1, 4, 8, 4)
    pool.free_pages.copy_(ints([0, 1, 2, 1000]))
    cu, pos, slots, served = E.ebd_paged_deal(pool, pc, ints([9]), 9)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    assert slots.tolist() == [-1] * 8 + [2 * 8]


def test_deal_in_a_graph_follows_its_inputs(E):
    pool, pc = fresh_pool(E, 5, 200, 8, 30)
    n_new = ints([1, 2, 3, 0, 20])
    outs = dict(cu_new=ints([0] * 6), positions=ints([0] * 40), slots=ints([0] * 40).long(),
                served=ints([0] * 5))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        E.ebd_paged_deal(pool, pc, n_new, 40, **outs)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        E.ebd_paged_deal(pool, pc, n_new, 40, **outs)
    free, table = list(range(200)), [[0] * 30 for _ in range(5)]
    length, held = [0] * 5, [[0, 0]] * 5
    length, held, *_ = S.deal(8, 200, 30, 40, 0, n_new.tolist(), length, held, free, table)
    for new in ([1, 1, 1, 1, 1], [9, -1, 8, 0, 17], [1, 30, 0, -1, 2]):
        n_new.copy_(ints(new))
        g.replay()
        length, held, cu, served, pos, slots = S.deal(8, 200, 30, 40, 0, new, length, held, free,
                                                      table)
        assert pc.seq_len.tolist() == length and outs["slots"].tolist() == slots
        assert outs["cu_new"].tolist() == cu and pc.block_table.tolist() == table


# ---------------------------------------------------------------- norms
NORMS = [  # T, H, d, rot
    (1, 1, 64, 64), (1, 28, 128, 128), (33, 4, 128, 64), (257, 7, 64, 32), (5, 3, 80, 80),
    (19, 2, 96, 12), (3, 2, 10, 6), (700, 5, 128, 128), (7, 1, 64, 2), (9, 33, 128, 128),
    (4, 2, 256, 256), (6, 3, 512, 128), (5, 2, 512, 512), (3, 1, 2, 2), (2, 3, 510, 6), (3, 2, 6, 0),
    (65, 6, 128, 0), (3, 2, 7, 0), (2500, 3, 64, 64),
]


def norm_inputs(T, H, d, dtype, per_head, seed, w_dtype=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((T, H + 2, d), generator=g, device="cuda") * 3
    x *= torch.rand((T, H + 2, 1), generator=g, device="cuda") + 0.1
    dy = torch.randn((T, H, d), generator=g, device="cuda") * 0.1
    w = torch.randn((H, d) if per_head else (d,), generator=g, device="cuda") * 0.2 + 1
    pos = torch.randint(0, 4000, (T,), generator=g, device="cuda").int()
    return x.to(dtype)[:, 1:H + 1], dy.to(dtype), w.to(w_dtype or dtype), pos


def check_normed(got, x, w, pos, tab, layout, dtype, eps=1e-6):
    n = S.norm(x, w, eps)
    if tab is None:
        return within(got, n, 24 * U * n.abs() + 1e-37, dtype)
    cs = tab[pos.long()]
    within(got, R.rotate(n, cs, layout), 24 * U * S.magnitudes(n, cs, layout) + 1e-37, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("T,H,d,rot", NORMS)
@pytest.mark.parametrize("per_head", [False, True])
def test_norm_rotary(E, dtype, layout, T, H, d, rot, per_head):
    x, _, w, pos = norm_inputs(T, H, d, dtype, per_head, T * 7 + d)
    tab = table_of(E, rot, 4000) if rot else None
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    st = ints([0])
    got = E.ebd_norm_rotary(x, w, pos, tab, layout=lay, dev_status=st)
    check_normed(got, x, w, pos, tab, layout, dtype)
    assert st.item() == 0
    z = x.clone(memory_format=torch.contiguous_format)  # (one row of a slice is contiguous itself)
    E.ebd_norm_rotary(z, w, pos, tab, out=z, layout=lay)  # in place
    assert torch.equal(z, got)
    if dtype == torch.bfloat16:  # the same weight in float32
        assert torch.equal(E.ebd_norm_rotary(x, w.float(), pos, tab, layout=lay), got)


def check_grad(dx, dw, dy, x, w, pos, tab, layout, dtype, eps=1e-6):
    cs = None if tab is None else tab[pos.long()]
    rx, rw, ax, aw = S.norm_grad(dy, x, w, eps, cs, layout)
    within(dx, rx, 48 * U * ax + 1e-37, dtype)
    over = (0,) if w.dim() == 2 else (0, 1)
    assert dw.dtype == torch.float32 and dw.shape == w.shape
    assert ((dw.double() - rw.sum(over)).abs() <= 120 * U * aw.sum(over) + 1e-37).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("T,H,d,rot", NORMS)
@pytest.mark.parametrize("per_head", [False, True])
def test_norm_rotary_gradient(E, dtype, layout, T, H, d, rot, per_head):
    x, dy, w, pos = norm_inputs(T, H, d, dtype, per_head, T * 7 + d + 1)
    tab = table_of(E, rot, 4000) if rot else None
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    dx, dw = E.ebd_norm_rotary_backward(dy, x, w, pos, tab, layout=lay)
    check_grad(dx, dw, dy, x, w, pos, tab, layout, dtype)
    again, dw2 = E.ebd_norm_rotary_backward(dy, x, w, pos, tab, layout=lay)
    assert torch.equal(again, dx) and torch.equal(dw2, dw)
    g = dy.clone()
    E.ebd_norm_rotary_backward(g, x, w, pos, tab, dx=g, layout=lay)  # over dy
    assert torch.equal(g, dx)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_norm_gradient_matches_differences(E, layout):
    """dx against central differences of the float64 form (truncation h^2 of third
    derivatives below 10, h = 2^-12: 6e-7), dweight against the forward call's own: y is
    linear in w, a step of 1/2 leaves its roundings only, 2 * 24 u |y| / 1 of every term."""
    T, H, d, rot = 5, 3, 64, 32
    x, dy, w, pos = norm_inputs(T, H, d, torch.float32, False, 3)
    x, dy = x.contiguous() / 3, dy * 10
    tab = table_of(E, rot, 4000)
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    dx, dw = E.ebd_norm_rotary_backward(dy, x, w, pos, tab, layout=lay)

    def loss(x, w):
        return (dy.double() * R.rotate(S.norm(x, w, 1e-6), tab[pos.long()], layout)).sum()

    h = 2.0 ** -12
    for t, head, c in [(0, 0, 0), (1, 2, 17), (4, 1, 33), (2, 0, 63), (3, 1, 31)]:
        e = torch.zeros_like(x, dtype=torch.float64)
        e[t, head, c] = h
        d_ = (loss(x.double() + e, w) - loss(x.double() - e, w)) / (2 * h)
        assert abs(d_.item() - dx[t, head, c].item()) <= 6e-7 + 48 * U * 100
    for c in (0, 5, 31, 32, 63):
        e = torch.zeros_like(w)
        e[c] = 0.5
        y1, y0 = (E.ebd_norm_rotary(x, w + s * e, pos, tab, layout=lay).double() for s in (1, -1))
        slack = (dy.abs().double() * (y1.abs() + y0.abs())).sum() * 50 * U
        assert abs((dy.double() * (y1 - y0)).sum() - dw[c].double()) <= slack


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_norm_rows_off_16_byte_boundaries(E, shift, layout):
    dt = torch.bfloat16
    base = torch.randn(9 * 3 * 64 + 8, device="cuda").to(dt)
    x = base[shift:shift + 9 * 3 * 64].view(9, 3, 64)
    w = torch.randn(72, device="cuda").to(dt)[shift:shift + 64]
    tab, pos = table_of(E, 64, 100), ints(range(9)) * 11
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    if layout == "pairs" and shift % 2:
        for call in (lambda: E.ebd_norm_rotary(x, w, pos, tab, layout=lay),
                     lambda: E.ebd_norm_rotary_backward(x, x, w, pos, tab, layout=lay)):
            with pytest.raises(E.EbdError) as e:
                call()
            assert e.value.code == 4
        return
    check_normed(E.ebd_norm_rotary(x, w, pos, tab, layout=lay), x, w, pos, tab, layout, dt)
    dx, dw = E.ebd_norm_rotary_backward(x, x, w, pos, tab, layout=lay)
    check_grad(dx, dw, x, x, w, pos, tab, layout, dt)


def test_norm_of_extreme_rows(E):
    """Rows of zeros, of values whose squares leave float32, of NaN and infinity: each
    only its own."""
    for dtype in (torch.float32, torch.bfloat16):
        x, dy, w, pos = norm_inputs(6, 2, 64, dtype, False, 9)
        x = x.contiguous()
        x[1] = 0
        x[2] = (x[2].double() * 1e30).to(dtype)
        x[3, 0, 5] = math.nan
        x[4, 1, 7] = math.inf
        tab = table_of(E, 64, 4000)
        y = E.ebd_norm_rotary(x, w, pos, tab)
        rows = torch.ones((6, 2), dtype=torch.bool, device="cuda")
        rows[3, 0] = rows[4, 1] = False
        n = S.norm(x, w, 1e-6)
        cs = tab[pos.long()]
        within(y[rows], R.rotate(n, cs, "half")[rows],
               (24 * U * S.magnitudes(n, cs, "half") + 1e-37)[rows], dtype)
        assert y[3, 0].isnan().all() and (y[1] == 0).all()
        dx, dw = E.ebd_norm_rotary_backward(dy, x, w, pos, tab)
        rx, rw, ax, aw = S.norm_grad(dy, x, w, 1e-6, cs, "half")
        within(dx[rows], rx[rows], (48 * U * ax + 1e-37)[rows], dtype)
        assert dw.isnan().all()
        ok = torch.tensor([0, 1, 2, 5], device="cuda")
        dx, dw = E.ebd_norm_rotary_backward(dy[ok], x[ok], w, pos[ok], tab)
        assert ((dw - rw[ok].sum((0, 1))).abs() <= 120 * U * aw[ok].sum((0, 1)) + 1e-37).all()


def test_norm_without_tokens_and_positions_outside_the_table(E):
    x, dy, w, pos = norm_inputs(3, 2, 64, torch.float32, True, 11)
    tab = table_of(E, 64, 50)
    dw = torch.full((2, 64), 7.0, device="cuda")
    E.ebd_norm_rotary_backward(dy[:0], x[:0], w, pos[:0], tab, dweight=dw)
    assert (dw == 0).all()
    assert E.ebd_norm_rotary(x[:0], w, pos[:0], tab).shape == (0, 2, 64)
    pos = ints([-4, 10, 50])
    for back in (False, True):
        st = ints([0])
        if back:
            dx, dw = E.ebd_norm_rotary_backward(dy, x, w, pos, tab, dev_status=st)
            check_grad(dx, dw, dy, x, w, ints([0, 10, 49]), tab, "half", torch.float32)
        else:
            y = E.ebd_norm_rotary(x, w, pos, tab, dev_status=st)
            check_normed(y, x, w, ints([0, 10, 49]), tab, "half", torch.float32)
        assert st.item() == E.EBD_DEV_RANGE


def test_norm_many_rows_stay_exact(E):
    """Grids of several rounds: every row of a long call, the weight's sum over 3e5 rows
    (its terms' 120 u bound grows with the 200 more steps that a lane adds)."""
    x, dy, w, pos = norm_inputs(40001, 7, 64, torch.bfloat16, False, 12)
    tab = table_of(E, 64, 4000)
    check_normed(E.ebd_norm_rotary(x, w, pos, tab), x, w, pos, tab, "half", torch.bfloat16)
    dx, dw = E.ebd_norm_rotary_backward(dy, x, w, pos, tab)
    rx, rw, ax, aw = S.norm_grad(dy, x, w, 1e-6, tab[pos.long()], "half")
    within(dx, rx, 48 * U * ax + 1e-37, torch.bfloat16)
    assert ((dw - rw.sum((0, 1))).abs() <= 320 * U * aw.sum((0, 1))).all()


# ---------------------------------------------------------------- append
APPENDS = [  # new, total, hq, hkv, d, page, rot
    ([1], [1], 4, 4, 64, 16, 64),
    ([1] * 9, [1, 16, 17, 33, 64, 100, 8, 9, 300], 8, 2, 128, 16, 128),
    ([5, 0, 33, 1], [5, 7, 120, 64], 28, 4, 128, 64, 64),
    ([130, 1, 0, 257], [130, 1, 0, 1000], 4, 1, 64, 8, 16),
    ([3, 40], [3, 41], 6, 3, 80, 32, 80),
    ([3, 40], [30, 41], 2, 1, 10, 32, 6),
    ([1] * 70, list(range(1, 71)), 32, 8, 64, 32, 64),
    ([2, 3], [9, 3], 3, 1, 256, 8, 256),
]


def slots_of(s, new, total, page):
    pos = [p for w, n in zip(new, total) for p in range(n - w, n)]
    seq = [b for b, w in enumerate(new) for _ in range(w)]
    at = s["bt"].long()[torch.tensor(seq).cuda(), torch.tensor(pos).cuda() // page]
    return ints(pos), at, torch.tensor(pos).cuda() % page


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("order", ["head", "row", "side"])
@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append_norm(E, dtype, layout, order, case):
    new, total, hq, hkv, d, page, rot = APPENDS[case]
    s = R.make(new, total, hq, hkv, d, page, dtype, 100 + case, order)
    pc = cache(E, s)
    tab = table_of(E, rot, max(total) + 1)
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    g = torch.Generator(device="cuda").manual_seed(case)
    per_head = case % 2 == 1
    kw, qw = (torch.randn((h, d) if per_head else (d,), generator=g, device="cuda").to(dtype)
              for h in (hkv, hq))
    K0, V0 = s["K"].clone(), s["V"].clone()
    pos, at, off = slots_of(s, new, total, page)
    out = []
    for where in (dict(cu_new=s["cu"]), dict(slots=at * page + off, positions=pos)):
        s["K"].copy_(K0)
        s["V"].copy_(V0)
        q_out = torch.empty((s["T"], hq, d), dtype=dtype, device="cuda")
        E.ebd_paged_append_norm(pc, s["k"], s["v"], k_weight=kw, q=s["q"], q_weight=qw,
                                q_out=q_out, table=tab, layout=lay, **where)
        check_normed(q_out, s["q"], qw, pos, tab, layout, dtype)
        check_normed(s["K"][at, :, off], s["k"], kw, pos, tab, layout, dtype)
        assert torch.equal(s["V"][at, :, off], s["v"])
        untouched = torch.ones(K0.shape[:1] + K0.shape[2:3], dtype=torch.bool, device="cuda")
        untouched[at, off] = False
        keep = untouched[:, None, :, None].expand_as(K0)
        assert torch.equal(s["K"][keep], K0[keep]) and torch.equal(s["V"][keep], V0[keep])
        assert pc.dev_status.item() == 0
        out.append((q_out, s["K"].clone(), s["V"].clone()))
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_append_without_weights_is_the_plain_append(E):
    new, total = [5, 0, 33, 1], [5, 7, 120, 64]
    s = R.make(new, total, 8, 2, 128, 16, torch.bfloat16, 5)
    pc, tab = cache(E, s), table_of(E, 128, 200)
    q1, q2 = (torch.empty((s["T"], 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    E.ebd_paged_append(pc, s["k"], s["v"], s["cu"], table=tab, q=s["q"], q_out=q1)
    K1, V1 = s["K"].clone(), s["V"].clone()
    s["K"].zero_()
    s["V"].zero_()
    E.ebd_paged_append_norm(pc, s["k"], s["v"], cu_new=s["cu"], table=tab, q=s["q"], q_out=q2)
    pos, at, off = slots_of(s, new, total, 16)
    assert torch.equal(q1, q2) and torch.equal(s["K"][at, :, off], K1[at, :, off])
    assert torch.equal(s["V"][at, :, off], V1[at, :, off])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("d,rot", [(128, 32), (128, 128), (64, 32), (80, 40), (96, 20), (10, 6), (256, 64)])
def test_append_without_weights_copies_what_does_not_turn(E, dtype, layout, d, rot):
    """Channels that stay come as they went, whatever they hold; the others turned (three
    float32 roundings of their terms' size and one to the type), and in 16-byte accesses bit
    for bit as the plain append turns them."""
    s = R.make([5, 3], [9, 40], 2, 2, d, 16, dtype, 6)
    pc, tab = cache(E, s), table_of(E, rot, 200)
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    for v in (s["q"], s["k"], s["v"]):
        odd = [-0.0, math.inf, -math.inf, 1e-40, -3e-39, 3e38]
        for i, x in enumerate(odd if rot < d else []):
            v[i % 5, :, rot + i % (d - rot)] = x
    q1, q2 = (torch.empty((8, 2, d), dtype=dtype, device="cuda") for _ in range(2))
    E.ebd_paged_append(pc, s["k"], s["v"], s["cu"], table=tab, layout=lay, q=s["q"], q_out=q1)
    K1, V1 = s["K"].clone(), s["V"].clone()
    E.ebd_paged_append_norm(pc, s["k"], s["v"], cu_new=s["cu"], table=tab, layout=lay, q=s["q"],
                            q_out=q2)
    bits = torch.int32 if dtype == torch.float32 else torch.int16
    wide = 128 // torch.finfo(dtype).bits  # elements of a 16-byte access
    part = wide if layout == "pairs" else 2 * wide
    same = d if rot % part == 0 and d % wide == 0 else d - rot
    for a, b in ((q1, q2), (K1, s["K"]), (V1, s["V"])):
        a, b = a[..., d - same:].contiguous(), b[..., d - same:].contiguous()
        assert torch.equal(a.view(bits), b.view(bits))
    pos, at, off = slots_of(s, [5, 3], [9, 40], 16)
    cs = tab[pos.long()]
    for x, y in ((s["q"], q2), (s["k"], s["K"][at, :, off])):
        x, y = x[..., :rot], y[..., :rot]
        within(y, R.rotate(x, cs, layout), 4 * U * S.magnitudes(x.double(), cs, layout) + 1e-37, dtype)


def test_append_of_a_tree_turns_to_its_positions(E):
    """By offsets and by slots; norms of one of the two only."""
    new, total = [9, 4], [30, 4]
    s = R.make(new, total, 4, 2, 64, 8, torch.float32, 6)
    pc, tab = cache(E, s), table_of(E, 64, 64)
    _, at, off = slots_of(s, new, total, 8)
    parents = S.random_parents(new, 1)
    _, pos = S.masks(parents, s["cu"].tolist(), total, 1)
    pos = pos.cuda()
    w = torch.randn(64, device="cuda")
    q_out = torch.empty((13, 4, 64), device="cuda")
    for where in (dict(cu_new=s["cu"]), dict(slots=at * 8 + off)):
        E.ebd_paged_append_norm(pc, s["k"], s["v"], q=s["q"], q_weight=w, q_out=q_out, table=tab,
                                positions=pos, **where)
        check_normed(q_out, s["q"], w, pos, tab, "half", torch.float32)
        ref = E.ebd_rotary(s["k"], pos, tab)
        assert torch.equal(s["K"][at, :, off], ref)
        E.ebd_paged_append_norm(pc, s["k"], s["v"], k_weight=w, table=tab, positions=pos, **where)
        check_normed(s["K"][at, :, off], s["k"], w, pos, tab, "half", torch.float32)
    # norms without a rotation
    E.ebd_paged_append_norm(pc, s["k"], s["v"], k_weight=w, cu_new=s["cu"], q=s["q"], q_weight=w,
                            q_out=q_out)
    check_normed(s["K"][at, :, off], s["k"], w, None, None, "half", torch.float32)
    check_normed(q_out, s["q"], w, None, None, "half", torch.float32)
    assert pc.dev_status.item() == 0


def test_append_by_slots_leaves_empty_and_bad_places_alone(E):
    s = R.make([6], [6], 2, 1, 64, 8, torch.bfloat16, 7)
    pc, tab = cache(E, s), table_of(E, 64, 64)
    n_slots = s["K"].shape[0] * 8
    K0, V0 = s["K"].clone(), s["V"].clone()
    slots = torch.tensor([-1, n_slots - 1, -1, -1, -1, -1], device="cuda")
    q_out = torch.full((6, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, device="cuda").to(torch.bfloat16)
    pos = ints([1000, 5, -9, 0, 0, 0])  # those of empty places are not looked at
    E.ebd_paged_append_norm(pc, s["k"], s["v"], k_weight=w, q=s["q"], q_weight=w, q_out=q_out,
                            slots=slots, positions=pos, table=tab)
    assert pc.dev_status.item() == 0
    assert (q_out[[0, 2, 3, 4, 5]] == 3).all()
    check_normed(q_out[1:2], s["q"][1:2], w, pos[1:2], tab, "half", torch.bfloat16)
    K0[-1, :, 7], V0[-1, :, 7] = s["K"][-1, :, 7], s["v"][1]
    assert torch.equal(s["K"], K0) and torch.equal(s["V"], V0)
    slots = torch.tensor([n_slots, -2, 1 << 40, -(1 << 40), 0, -1], device="cuda")
    E.ebd_paged_append_norm(pc, s["k"], s["v"], q=s["q"], q_weight=w, q_out=q_out, slots=slots,
                            positions=ints([1] * 6), table=tab)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    assert torch.equal(s["V"][0, :, 0], s["v"][4])
    V0[0, :, 0] = s["v"][4]
    assert torch.equal(s["V"], V0)


def test_append_norm_drops_what_has_no_page(E):
    s = R.make([4, 4, 4], [16, 16, 16], 2, 1, 64, 8, torch.float32, 4)
    s["seq_len"].copy_(ints([18, 16, 2]))   # 2 past the table; 2 before 0
    s["bt"][1, 1] = s["K"].shape[0] + 5     # a page outside the pool
    V0 = s["V"].clone()
    pc = cache(E, s)
    E.ebd_paged_append_norm(pc, s["k"], s["v"], cu_new=s["cu"], k_weight=torch.ones(64, device="cuda"))
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    for t, b, pos in [(0, 0, 14), (1, 0, 15), (10, 2, 0), (11, 2, 1)]:
        assert torch.equal(R.row(s["V"], s["bt"], b, 0, pos), s["v"][t, 0])
        R.row(V0, s["bt"], b, 0, pos).copy_(s["v"][t, 0])
    assert torch.equal(s["V"], V0)


# ---------------------------------------------------------------- masks
@pytest.mark.parametrize("shape", ["mixed", "chain", "roots"])
@pytest.mark.parametrize("new,words", [([1], 1), ([33, 0, 1, 64, 7], 2), ([5] * 40, 3),
                                       ([1024, 3, 1000], 32), ([32, 31], 1)])
@pytest.mark.parametrize("window", [0, 1, 6])
def test_tree_masks(E, shape, new, words, window):
    total = [n + 5 * b for b, n in enumerate(new)]
    parents = S.random_parents(new, len(new), shape)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    st = ints([0])
    mask, pos = E.ebd_tree_masks(ints(parents), ints(cu), ints(total), 32 * words, window=window,
                                 dev_status=st)
    rm, rp = S.masks(parents, cu, total, words, window)
    assert torch.equal(mask.cpu(), rm) and torch.equal(pos.cpu(), rp) and st.item() == 0


def test_tree_masks_bad_parents_and_offsets(E):
    parents = [-1, 1, -5, 2, 99, 3]  # 1: itself, -5 and 99: no token
    st = ints([0])
    mask, pos = E.ebd_tree_masks(ints(parents), ints([0, 6]), ints([10]), 6, dev_status=st)
    rm, rp = S.masks([-1, -1, -1, 2, -1, 3], [0, 6], [10], 1)
    assert torch.equal(mask.cpu(), rm) and torch.equal(pos.cpu(), rp)
    assert st.item() == E.EBD_DEV_RANGE
    # tokens of no sequence, and past max_new, are left alone
    st.zero_()
    mask, pos = torch.full((6, 1), 9, device="cuda").int(), ints([-3] * 6)
    E.ebd_tree_masks(ints([-1] * 6), ints([1, 5]), ints([10]), 3, mask=mask, positions=pos,
                     dev_status=st)
    assert mask[:, 0].tolist() == [9, 1, 2, 4, 9, 9]
    assert pos.tolist() == [-3, 7, 7, 7, -3, -3] and st.item() == E.EBD_DEV_RANGE


# ---------------------------------------------------------------- attention
TREES = [  # new, total, hq, hkv, d, page
    ([1], [1], 4, 4, 64, 16),
    ([7], [7], 4, 1, 64, 8),                          # no prefix
    ([16], [200], 28, 4, 128, 16),
    ([33, 0, 1, 5], [33, 7, 120, 64], 8, 2, 128, 64),
    ([64, 40, 64], [64, 1000, 700], 32, 8, 128, 64),  # 256 rows of one item
    ([100, 31], [130, 95], 14, 2, 64, 32),            # several items of one tree
    ([200], [333], 8, 1, 128, 128),
    ([3, 9], [2000, 5000], 8, 8, 64, 256),            # split over many CTAs
    ([12] * 30, [13 + 17 * i for i in range(30)], 4, 2, 64, 8),
    ([20], [63 + 20], 128, 1, 64, 16),                # a group of 128
    ([65, 2], [129, 66], 5, 1, 128, 8),
    ([300], [420], 2, 2, 64, 1024),
]


def tree_case(E, case, dtype, order="head", window=0, shape="mixed", stale=0.0):
    new, total, hq, hkv, d, page = TREES[case]
    s = R.make(new, total, hq, hkv, d, page, dtype, 300 + case, order, stale=stale)
    s["q"] = s["q"] * 2
    parents = S.random_parents(new, case, shape)
    cu = s["cu"].tolist()
    s["parents"] = ints(parents)
    s["mask"], s["pos"] = (t.cuda() for t in S.masks(parents, cu, total, -(-max(new) // 32), window))
    s["seen"] = S.tree_seen(s["mask"], s["pos"], cu, total, window)
    s["total"], s["new"] = total, new
    return s


def check_tree(E, s, y, lse, dtype, absent=(), rows=None):
    d = s["q"].shape[2]
    ry, rl, mean, root = S.attention(s["q"], s["K"], s["V"], s["bt"], s["total"], s["cu"].tolist(),
                                     d ** -0.5, s["seen"], absent)
    rows = slice(None) if rows is None else rows
    assert ((y.double() - ry).abs() <= R.attention_bound(ry, mean, root, dtype))[rows].all()
    none = torch.isneginf(rl)
    assert torch.equal(torch.isneginf(lse)[rows], none[rows])
    assert (y[none] == 0).all()
    assert ((lse.double() - rl).abs()[rows][~none[rows]] <= 2e-5).all()


def call(E, s, pc, window=0, **kw):
    return E.ebd_paged_tree_attention(s["q"], pc, s["cu"], s["max_new"], s["mask"],
                                      positions=s["pos"], window=window, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", range(len(TREES)))
@pytest.mark.parametrize("window", [0, 1, 9, 150])
def test_tree_attention(E, dtype, case, window):
    s = tree_case(E, case, dtype, ["head", "row", "side"][case % 3], window)
    pc = cache(E, s)
    y, lse = call(E, s, pc, window)
    check_tree(E, s, y, lse, dtype)
    assert pc.dev_status.item() == 0
    y2, lse2 = call(E, s, pc, window)
    assert torch.equal(y, y2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", range(len(TREES)))
def test_chain_is_causal_attention_bit_for_bit(E, dtype, case):
    s = tree_case(E, case, dtype, shape="chain")
    pc = cache(E, s)
    y, lse = call(E, s, pc)
    y2, lse2 = E.ebd_paged_attention(s["q"], pc, s["cu"], s["max_new"])
    assert torch.equal(y, y2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", [1, 3, 5, 8])
@pytest.mark.parametrize("window", [0, 4])
def test_masks_of_any_bits(E, dtype, case, window):
    """Random bits, rows with none, later tokens' bits (hidden all the same), wide rows."""
    s = tree_case(E, case, dtype, window=window)
    g = torch.Generator().manual_seed(case)
    T, words = s["mask"].shape[0], s["mask"].shape[1] + 1
    m = torch.randint(-2 ** 31, 2 ** 31, (T, words), generator=g).int()
    m[::3] = 0
    m[1::5] = -1
    s["mask"] = m.cuda()
    s["seen"] = S.tree_seen(s["mask"], s["pos"], s["cu"].tolist(), s["total"], window)
    pc = cache(E, s)
    y, lse = call(E, s, pc, window)
    check_tree(E, s, y, lse, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("stale", [math.nan, math.inf])
@pytest.mark.parametrize("case", [3, 5, 6, 8])
def test_hidden_values_take_no_part(E, dtype, stale, case):
    """Unused slots, and some tokens of the tree, hold NaN or infinity: who does not see
    them does not meet them."""
    s = tree_case(E, case, dtype, stale=stale)
    cu, total, new = s["cu"].tolist(), s["total"], s["new"]
    bad = []
    for b, n in enumerate(new):
        for i in range(2, n, 11):
            R.row(s["V"], s["bt"], b, 0, total[b] - n + i)[3:40] = stale
            if i % 2:
                R.row(s["K"], s["bt"], b, 0, total[b] - n + i)[1] = math.nan
            bad.append((b, i))
    meets = torch.zeros(sum(new), dtype=torch.bool)
    for b, i in bad:
        n = new[b]
        meets[cu[b]:cu[b] + n] |= s["seen"][b][:, total[b] - n + i]
    pc = cache(E, s)
    y, lse = call(E, s, pc)
    assert pc.dev_status.item() == 0
    ok = (~meets).cuda()
    assert ok.any() and meets.any()
    check_tree(E, s, y, lse, dtype, rows=ok)
    g = s["q"].shape[1] // s["K"].shape[1]
    assert not torch.isfinite(y[meets.cuda()][:, :g, 3:40]).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tree_bad_pages_and_positions(E, dtype):
    s = tree_case(E, 4, dtype)
    s["bt"][1, 2] = s["K"].shape[0] + 3
    pc = cache(E, s)
    y, lse = call(E, s, pc)
    check_tree(E, s, y, lse, dtype, absent=[(1, 2)])
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    # positions outside the tree: clamped
    s = tree_case(E, 2, dtype, window=20)
    s["pos"][3], s["pos"][9] = 0, 100000
    base = 200 - 16
    p = s["pos"].clone()
    p[3], p[9] = base, base + 9
    s["seen"] = S.tree_seen(s["mask"], p, s["cu"].tolist(), s["total"], 20)
    pc = cache(E, s)
    y, lse = call(E, s, pc, 20)
    check_tree(E, s, y, lse, dtype)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tree_longer_than_its_sequence(E, dtype):
    """Tokens before position 0 see nothing; those after it the others that are there."""
    s = tree_case(E, 1, dtype)
    s["seq_len"].fill_(4)  # 7 new tokens
    s["total"] = [4]
    s["mask"].fill_(-1)
    seen = torch.zeros((7, 4), dtype=torch.bool)
    for i in range(3, 7):
        seen[i, :i - 2] = True
    s["seen"] = [seen]
    pc = cache(E, s)
    y, lse = call(E, s, pc)
    check_tree(E, s, y, lse, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_released_pages_behind_the_window_are_not_used(E, dtype):
    s = tree_case(E, 7, dtype, window=300)
    page = 256
    for b, (n, w) in enumerate(zip(s["total"], s["new"])):
        for blk in range(max(0, n - w - 300 + 1) // page):
            s["bt"][b, blk] = -1
    pc = cache(E, s)
    y, lse = call(E, s, pc, 300)
    safe = dict(s, bt=s["bt"].clamp(min=0))
    check_tree(E, safe, y, lse, dtype)
    assert pc.dev_status.item() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_no_sequence_stay(E, dtype):
    s = tree_case(E, 3, dtype)
    T = s["T"]
    y, lse = torch.full_like(s["q"], 5).contiguous(), torch.full(s["q"].shape[:2], 6.0, device="cuda")
    s["cu"].copy_(ints([1, 33, 33, 34, 37]))
    pc = cache(E, s)
    call(E, s, pc, y=y, lse=lse)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    for t in (0, T - 1, T - 2):
        assert (y[t] == 5).all() and (lse[t] == 6).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", [3, 8])
def test_empty_places_behind_the_last_sequence(E, dtype, case):
    """Packed arrays longer than the offsets say: the rest stays, and nothing is reported."""
    s = tree_case(E, case, dtype)
    pc = cache(E, s)
    y, lse = call(E, s, pc)
    T = s["T"]
    q = torch.cat([s["q"], torch.full_like(s["q"][:5], math.nan)])
    mask = torch.cat([s["mask"], torch.full_like(s["mask"][:1], -1).expand(5, -1)])
    y2, lse2 = torch.full_like(q, 3), torch.full(q.shape[:2], 4.0, device="cuda")
    E.ebd_paged_tree_attention(q, pc, s["cu"], s["max_new"], mask, y=y2, lse=lse2)
    assert torch.equal(y2[:T], y) and torch.equal(lse2[:T], lse)
    assert (y2[T:] == 3).all() and (lse2[T:] == 4).all()
    m, p, st = torch.full_like(mask, 7), torch.full((T + 5,), 8, device="cuda").int(), ints([0])
    parents = torch.cat([s["parents"], ints([99] * 5)])
    E.ebd_tree_masks(parents, s["cu"], s["seq_len"], s["max_new"], mask=m, positions=p,
                     dev_status=st)
    assert torch.equal(m[:T], s["mask"]) and torch.equal(p[:T], s["pos"])
    assert (m[T:] == 7).all() and (p[T:] == 8).all()
    assert st.item() == 0 and pc.dev_status.item() == 0


def test_graph_and_stream_of_tree_attention(E):
    """A captured step follows masks, lengths and pages; the other stream's buffers hold."""
    s = tree_case(E, 4, torch.bfloat16)
    pc = cache(E, s)
    want = call(E, s, pc)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(E, s, pc, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    mask, pos = torch.zeros_like(s["mask"]), torch.zeros_like(s["pos"])
    y, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        E.ebd_tree_masks(s["parents"], s["cu"], s["seq_len"], s["max_new"], mask=mask,
                         positions=pos)
        E.ebd_paged_tree_attention(s["q"], pc, s["cu"], s["max_new"], mask, y=y, lse=lse)
    g.replay()
    assert torch.equal(y, want[0]) and torch.equal(lse, want[1])
    parents = S.random_parents(s["new"], 77)
    s["parents"].copy_(ints(parents))
    s["total"] = [64, 900, 650]
    s["seq_len"].copy_(ints(s["total"]))
    g.replay()
    cu = s["cu"].tolist()
    m, p = S.masks(parents, cu, s["total"], 2)
    assert torch.equal(mask.cpu(), m) and torch.equal(pos.cpu(), p)
    s["seen"] = S.tree_seen(m, p, cu, s["total"])
    check_tree(E, s, y, lse, torch.bfloat16)


def test_long_tree_over_a_long_cache(E):
    s = R.make([48, 64], [40000, 33], 8, 2, 128, 64, torch.bfloat16, 9)
    s["q"] = s["q"] * 2
    parents, total = S.random_parents([48, 64], 4), [40000, 64]
    s["seq_len"].copy_(ints(total))
    s["bt"][1, 0] = s["K"].shape[0] - 1
    s["mask"], s["pos"] = (t.cuda() for t in S.masks(parents, [0, 48, 112], total, 2))
    s["total"], s["seen"] = total, S.tree_seen(s["mask"], s["pos"], [0, 48, 112], total)
    pc = cache(E, s)
    y, lse = call(E, s, pc)
    check_tree(E, s, y, lse, torch.bfloat16)


# ---------------------------------------------------------------- accepted paths
def keep_ref(K, V, bt, total, cu, path, k, page):
    """Row by row; K, V [L, ...] clones."""
    K, V = K.clone(), V.clone()
    out = []
    for b, n in enumerate(total):
        base = n - (cu[b + 1] - cu[b])
        for i in range(k[b]):
            p, q = base + path[b][i], base + i
            at, to = int(bt[b, p // page]), int(bt[b, q // page])
            for pool in (K, V):
                pool[:, to, :, q % page] = pool[:, at, :, p % page].clone()
        out.append(base + k[b])
    return K, V, out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layers,order", [(1, "head"), (1, "row"), (1, "side"), (5, "head")])
@pytest.mark.parametrize("new,total,hkv,d,page,most", [
    ([1], [1], 1, 64, 8, 1), ([16], [516], 4, 64, 16, 5), ([7, 0, 64, 30], [7, 9, 90, 31], 2, 128, 8, 64),
    ([40] * 20, [40 + 3 * i for i in range(20)], 8, 128, 64, 9), ([200, 130], [210, 400], 3, 64, 32, 150)])
def test_keep(E, dtype, layers, order, new, total, hkv, d, page, most):
    s = R.make(new, total, hkv, hkv, d, page, dtype, 40, order)
    rng = random.Random(len(new) + most)
    kept = [rng.randint(0, min(most, n)) for n in new]
    path = [sorted(rng.sample(range(n), k)) + [-1] * (most - k) for n, k in zip(new, kept)]
    if layers > 1:
        K, V = (torch.randn((layers, *s["K"].shape), device="cuda").to(dtype) for _ in range(2))
        s["K"], s["V"] = K[0], V[0]
        kw = dict(K_layers=K, V_layers=V)
    else:
        K, V, kw = s["K"][None], s["V"][None], {}
    pc = cache(E, s)
    rk, rv, rl = keep_ref(K, V, s["bt"], total, s["cu"].tolist(), path, kept, page)
    got = E.ebd_paged_keep(pc, s["cu"], ints(path), ints(kept), **kw)
    assert got.tolist() == rl
    assert torch.equal(K, rk) and torch.equal(V, rv) and pc.dev_status.item() == 0
    assert s["seq_len"].tolist() == total


def test_keep_stops_at_a_bad_path(E):
    new, total, page = [10, 10, 10, 10, 40], [30, 30, 30, 30, 60], 8
    s = R.make(new, total, 2, 2, 64, page, torch.float32, 41)
    path = [[1, 3, 3, 5, 6], [0, 2, 1, 4, 5], [2, 4, 10, 11, 12], [-1, 2, 3, 4, 5], [3, 4, 5, 6, 39]]
    pc = cache(E, s)
    rk, rv, rl = keep_ref(s["K"][None], s["V"][None], s["bt"], total, s["cu"].tolist(), path,
                          [2, 2, 2, 0, 5], page)
    got = E.ebd_paged_keep(pc, s["cu"], ints(path), ints([5, 5, 5, 5, 5]))
    assert got.tolist() == rl and torch.equal(s["K"], rk[0]) and torch.equal(s["V"], rv[0])
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    # counts outside their range, lengths below the tree's, a page outside the pool
    s = R.make([4, 4, 4], [12, 2, 12], 1, 1, 64, 8, torch.float32, 42)
    s["bt"][2, 1] = 10 ** 6
    pc = cache(E, s)
    path = [[0, 1, 2, 3], [0, 1, 2, 3], [1, 2, 3, -1]]
    K0 = s["K"].clone()
    got = E.ebd_paged_keep(pc, s["cu"], ints(path), ints([9, 3, 3]))
    assert pc.dev_status.item() == E.EBD_DEV_RANGE and torch.equal(s["K"], K0)
    assert got.tolist() == [12, 2, 11]
    got = E.ebd_paged_keep(pc, s["cu"], ints(path), ints([-3, 0, 0]))
    assert got.tolist() == [8, 0, 8]


def test_keep_long_path_over_a_chain_moves_every_row_down(E):
    """Every source but the last is a later destination."""
    n = 1000
    s = R.make([n], [n + 9], 2, 2, 64, 16, torch.bfloat16, 43)
    path = [list(range(1, n))]
    rk, rv, rl = keep_ref(s["K"][None], s["V"][None], s["bt"], [n + 9], [0, n], path, [n - 1], 16)
    pc = cache(E, s)
    assert E.ebd_paged_keep(pc, s["cu"], ints(path), ints([n - 1])).tolist() == [n + 8]
    assert torch.equal(s["K"], rk[0]) and torch.equal(s["V"], rv[0])


def test_keep_of_one_pool_for_keys_and_values(E):
    """K and V in the same memory: every row moves once, though each is a later source."""
    n = 300
    s = R.make([n], [n + 9], 1, 1, 64, 16, torch.float32, 44)
    path = [list(range(1, n))]
    rk, _, _ = keep_ref(s["K"][None], s["K"][None], s["bt"], [n + 9], [0, n], path, [n - 1], 16)
    s["V"] = s["K"]
    E.ebd_paged_keep(cache(E, s), s["cu"], ints(path), ints([n - 1]))
    assert torch.equal(s["K"], rk[0])


# ---------------------------------------------------------------- the binding
def test_calls_on_another_stream(E):
    """Every call with stream=: after a long piece of work on that stream, into buffers that
    the call makes itself."""
    s = tree_case(E, 3, torch.bfloat16)
    pc, tab = cache(E, s), table_of(E, 128, 200)
    x, dy, w, pos = norm_inputs(33, 4, 128, torch.bfloat16, False, 5)
    T = s["T"]
    qo = torch.empty((T, 8, 128), dtype=torch.bfloat16, device="cuda")
    path, kept = ints([[0, 3], [0, 0], [0, 0], [1, 2]]), ints([2, 0, 1, 2])

    def all_calls(stream):
        pool, pc2 = fresh_pool(E, 3, 20, 8, 5)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                torch.cuda._sleep(2000000)
        out = list(E.ebd_paged_deal(pool, pc2, ints([10, 3, 20]), 40, stream=stream))
        out.append(E.ebd_norm_rotary(x, w, pos, tab_long, stream=stream))
        out += E.ebd_norm_rotary_backward(dy, x, w, pos, tab_long, stream=stream)
        m, p = E.ebd_tree_masks(s["parents"], s["cu"], s["seq_len"], 33, stream=stream)
        E.ebd_paged_append_norm(pc, s["k"], s["v"], k_weight=w, q=s["q"], q_weight=w, q_out=qo,
                                cu_new=s["cu"], positions=p, table=tab, stream=stream)
        out += [m, p, *E.ebd_paged_tree_attention(qo, pc, s["cu"], 33, m, stream=stream)]
        out.append(E.ebd_paged_keep(pc, s["cu"], path, kept, stream=stream))
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        return out

    tab_long = table_of(E, 128, 4000)
    K0 = s["K"].clone()
    want = all_calls(None)
    s["K"].copy_(K0)
    got = all_calls(torch.cuda.Stream())
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and len(want) == len(got)


def test_arguments_are_checked(E):
    s = tree_case(E, 2, torch.bfloat16)
    pc = cache(E, s)
    x, dy, w, pos = norm_inputs(5, 2, 64, torch.bfloat16, False, 1)
    tab = table_of(E, 64, 4000)

    class Elsewhere:
        cuda_stream, device_index = 0, 7

    bad = [
        (TypeError, lambda: E.ebd_norm_rotary(x, w.half(), pos, tab)),
        (ValueError, lambda: E.ebd_norm_rotary(x, w[:32], pos, tab)),
        (ValueError, lambda: E.ebd_norm_rotary(x, w.expand(2, 64), pos, tab)),
        (ValueError, lambda: E.ebd_norm_rotary(x, w, None, tab)),
        (TypeError, lambda: E.ebd_norm_rotary(x, w, pos.long(), tab)),
        (ValueError, lambda: E.ebd_norm_rotary(x, w, pos[:3], tab)),
        (ValueError, lambda: E.ebd_norm_rotary(x, w, pos, tab[:, :, 0])),
        (TypeError, lambda: E.ebd_norm_rotary(x.half(), w, pos, tab)),
        (ValueError, lambda: E.ebd_norm_rotary(x.transpose(1, 2), w, pos, tab)),
        (ValueError, lambda: E.ebd_norm_rotary(x, w, pos, tab, out=x[:4])),
        (ValueError, lambda: E.ebd_norm_rotary(x, w, pos, tab, out=torch.empty_like(x),
                                               stream=Elsewhere())),
        (TypeError, lambda: E.ebd_norm_rotary_backward(dy.float(), x, w, pos, tab)),
        (ValueError, lambda: E.ebd_norm_rotary_backward(dy, x, w, pos, tab, dweight=tab[0])),
        (ValueError, lambda: E.ebd_norm_rotary_backward(
            dy, x, w, pos, tab, workspace=torch.empty(16, device="cuda"))),
        (ValueError, lambda: E.ebd_paged_append_norm(pc, s["k"], s["v"])),
        (ValueError, lambda: E.ebd_paged_append_norm(pc, s["k"], s["v"][:1], cu_new=s["cu"])),
        (ValueError, lambda: E.ebd_paged_append_norm(pc, s["k"], s["v"], cu_new=s["cu"][:1])),
        (ValueError, lambda: E.ebd_paged_append_norm(pc, s["k"], s["v"], cu_new=s["cu"],
                                                     q=s["q"])),
        (TypeError, lambda: E.ebd_paged_append_norm(pc, s["k"], s["v"], slots=s["cu"][:1])),
        (ValueError, lambda: E.ebd_tree_masks(s["parents"], s["cu"], s["cu"], 16)),
        (ValueError, lambda: E.ebd_tree_masks(s["parents"], s["cu"], s["seq_len"], 16,
                                              mask=s["mask"][:3])),
        (ValueError, lambda: E.ebd_paged_tree_attention(s["q"], pc, s["cu"], 16, s["mask"][0])),
        (TypeError, lambda: E.ebd_paged_tree_attention(s["q"], pc, s["cu"], 16,
                                                       s["mask"].long())),
        (ValueError, lambda: E.ebd_paged_tree_attention(s["q"], pc, s["cu"], 16, s["mask"][:2])),
        (ValueError, lambda: E.ebd_paged_keep(pc, s["cu"], s["pos"], s["seq_len"])),
        (ValueError, lambda: E.ebd_paged_keep(pc, s["cu"], s["pos"][None], s["seq_len"],
                                              K_layers=s["K"][None])),
        (ValueError, lambda: E.ebd_paged_keep(pc, s["cu"], s["pos"][None], s["seq_len"],
                                              K_layers=s["K"].clone()[None],
                                              V_layers=s["V"][None])),
        (TypeError, lambda: E.ebd_paged_deal(E.alloc_page_pool(1, s["K"].shape[0], "cuda"), pc,
                                             torch.ones(1, device="cuda"), 4)),
        (ValueError, lambda: E.ebd_paged_deal(E.alloc_page_pool(1, 3, "cuda"), pc, ints([1]), 4)),
        (E.EbdError, lambda: E.ebd_paged_tree_attention(s["q"], pc, s["cu"], 40, s["mask"])),
        (E.EbdError, lambda: E.ebd_norm_rotary(x, w, pos, tab, eps=0.0)),
        (E.EbdError, lambda: E.ebd_paged_keep(pc, s["cu"], s["pos"][None], s["seq_len"],
                                              seq_len_out=s["seq_len"])),
    ]
    for i, (error, f) in enumerate(bad):
        with pytest.raises(error):
            f()
            pytest.fail(f"call {i} was not refused")


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,hq,hkv,d,window", [(torch.bfloat16, 8, 2, 128, 0),
                                                   (torch.float32, 4, 4, 64, 0),
                                                   (torch.bfloat16, 7, 1, 64, 40)])
def test_a_served_run_of_trees(E, dtype, hq, hkv, d, window):
    """Requests come, draft trees, keep paths and leave; every step's attention against a
    plain float64 model that keeps each request's accepted keys and values as a list."""
    P, B, cap, n_pages, eps = 8, 4, 160, 90, 1e-6
    rng = random.Random(5)
    gen = torch.Generator(device="cuda").manual_seed(6)
    pc = E.alloc_paged(B, hkv, n_pages, P, d, 20, dtype, "cuda")
    pc.K_pages.fill_(math.nan)  # whatever the pages held
    pc.V_pages.fill_(math.nan)
    pool = E.alloc_page_pool(B, n_pages, "cuda")
    tab = table_of(E, d, 200)
    kw, qw = (torch.randn(d, generator=gen, device="cuda").to(dtype) for _ in range(2))
    story = [[], [], [], []]  # per request: (key row, value row) of its accepted tokens, float64
    for step in range(6):
        if step == 0:
            new = [30, 17, 0, 1]
        else:
            new = [-1 if b == 1 and step == 3 else 25 if not story[b] else rng.randint(1, 12)
                   for b in range(B)]
        cu, pos, slots, served = E.ebd_paged_deal(pool, pc, ints(new), cap, window=window)
        assert served.tolist() == [1] * B
        for b in range(B):
            if new[b] < 0:
                story[b] = []
        n = [max(v, 0) for v in new]
        parents = [p for b in range(B) for p in S.random_parents(
            [n[b]], 10 * step + b, "mixed" if story[b] else "chain")]
        par = torch.zeros(cap, dtype=torch.int32, device="cuda")
        par[:len(parents)] = ints(parents)
        T = sum(n)
        qkv = torch.randn((cap, hq + 2 * hkv, d), generator=gen, device="cuda").to(dtype)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        mask, tpos = E.ebd_tree_masks(par[:T], cu, pc.seq_len, max(n), window=window)
        at = torch.zeros(cap, dtype=torch.int32, device="cuda")
        at[:T] = tpos
        q_out = torch.empty((cap, hq, d), dtype=dtype, device="cuda")
        E.ebd_paged_append_norm(pc, k, v, k_weight=kw, q=q, q_weight=qw, q_out=q_out, slots=slots,
                                positions=at, table=tab)
        y, lse = E.ebd_paged_tree_attention(q_out[:T], pc, cu, max(n), mask, positions=tpos,
                                            window=window)
        cs = tab[at[:T].long()]
        # the plain model takes the appended rows (rounded once, checked elsewhere) as they are
        kr = R.rotate(S.norm(k[:T], kw, eps), cs, "half")
        lines, cl = S.lines(parents, cu.tolist()), cu.tolist()
        path, kept = [], []
        for b in range(B):
            line = []
            for t in range(cl[b], cl[b + 1]):
                if len(lines[t]) > len(line):
                    line = lines[t]  # the deepest token's path
            order = line[::-1][:max(1, len(line) - 1)] if story[b] else line[::-1]
            path.append(order + [-1] * (32 - len(order)))
            kept.append(len(order))
            for i in range(n[b]):
                t = cl[b] + i
                mine = [cl[b] + j for j in lines[t][::-1]]
                base = len(story[b])
                first = max(0, base + len(mine) - window) if window else 0
                stored = pc.K_pages.view(n_pages, hkv, P, d)
                keys = [x[0] for x in story[b]] + [
                    stored[slots[m] // P, :, slots[m] % P].double() for m in mine]
                vals = [x[1] for x in story[b]] + [v[m].double() for m in mine]
                keys, vals = torch.stack(keys[first:]), torch.stack(vals[first:])
                for h in range(hq):
                    z = (keys[:, h // (hq // hkv)] @ q_out[t, h].double()) * d ** -0.5
                    p = torch.softmax(z, 0)[:, None]
                    vv = vals[:, h // (hq // hkv)]
                    ref, mean = (p * vv).sum(0), (p * vv.abs()).sum(0)
                    root = (p * p * vv * vv).sum(0).sqrt()
                    assert ((y[t, h].double() - ref).abs()
                            <= R.attention_bound(ref, mean, root, dtype)).all()
                    assert abs(lse[t, h].double() - torch.logsumexp(z, 0)) <= 2e-5
        got = pc.K_pages[slots[:T] // P, :, slots[:T] % P]
        within(got, kr, 24 * U * S.magnitudes(S.norm(k[:T], kw, eps), cs, "half") + 1e-37, dtype)
        for b in range(B):
            for j in path[b][:kept[b]]:
                t = cl[b] + j
                story[b].append((got[t].double(), v[t].double()))
        pc.seq_len.copy_(E.ebd_paged_keep(pc, cu, ints(path), ints(kept)))
        assert pc.seq_len.tolist() == [len(x) for x in story]
    assert pc.dev_status.item() == 0


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_a_captured_step_is_the_eager_one(E, dtype, d):
    """A whole step and its norms' gradient in one graph, replayed over changing requests
    and inputs: every kernel waits for the one before it."""
    B, hq, hkv, P, n, cap, eps = 5, 8, 2, 8, 12, 60, 1e-6
    tab = table_of(E, d, 400)
    w = torch.rand(d, device="cuda").to(dtype) + 0.5
    x = {k: torch.zeros(v, dtype=t, device="cuda") for k, v, t in [
        ("n_new", (B,), torch.int32), ("parents", (cap,), torch.int32),
        ("path", (B, 4), torch.int32), ("kept", (B,), torch.int32),
        ("qkv", (cap, hq + 2 * hkv, d), dtype), ("dy", (cap, hq, d), dtype)]}

    def world():
        pc = E.alloc_paged(B, hkv, 150, P, d, 40, dtype, "cuda")
        pc.K_pages.zero_()
        pc.V_pages.zero_()
        o = {k: torch.zeros(v, dtype=t, device="cuda") for k, v, t in [
            ("cu_new", (B + 1,), torch.int32), ("positions", (cap,), torch.int32),
            ("slots", (cap,), torch.int64), ("served", (B,), torch.int32),
            ("mask", (cap, 1), torch.int32), ("tpos", (cap,), torch.int32),
            ("q", (cap, hq, d), dtype), ("y", (cap, hq, d), dtype),
            ("lse", (cap, hq), torch.float32), ("len", (B,), torch.int32),
            ("dx", (cap, hq, d), dtype), ("dw", (d,), torch.float32)]}
        return pc, E.alloc_page_pool(B, 150, "cuda"), o

    def step(pc, pool, o):
        q, k, v = x["qkv"][:, :hq], x["qkv"][:, hq:hq + hkv], x["qkv"][:, hq + hkv:]
        E.ebd_paged_deal(pool, pc, x["n_new"], cap, **{i: o[i] for i in (
            "cu_new", "positions", "slots", "served")})
        E.ebd_tree_masks(x["parents"], o["cu_new"], pc.seq_len, n, mask=o["mask"],
                         positions=o["tpos"])
        E.ebd_paged_append_norm(pc, k, v, k_weight=w, q=q, q_weight=w, q_out=o["q"],
                                slots=o["slots"], positions=o["tpos"], table=tab, eps=eps)
        E.ebd_paged_tree_attention(o["q"], pc, o["cu_new"], n, o["mask"], y=o["y"], lse=o["lse"])
        E.ebd_norm_rotary_backward(x["dy"], q, w, o["tpos"], tab, dx=o["dx"], dweight=o["dw"])
        E.ebd_paged_keep(pc, o["cu_new"], x["path"], x["kept"], seq_len_out=o["len"])
        pc.seq_len.copy_(o["len"])

    eager, other = world(), world()
    first = [t.clone() for t in (other[0].K_pages, other[0].V_pages, other[0].block_table,
                                 other[0].seq_len, other[1].free_pages, other[1].n_free,
                                 other[1].held)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*other)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(*other)
    for t, f in zip((other[0].K_pages, other[0].V_pages, other[0].block_table, other[0].seq_len,
                     other[1].free_pages, other[1].n_free, other[1].held), first):
        t.copy_(f)
    for t in other[2].values():
        t.zero_()
    rng, gen = random.Random(3), torch.Generator(device="cuda").manual_seed(4)
    for i in range(8):
        new = [rng.randint(0, n) if i else n for _ in range(B)]
        if i == 4:
            new[2] = -1
        par = [p for b in range(B) for p in S.random_parents([max(new[b], 0)], 7 * i + b)]
        x["n_new"].copy_(ints(new))
        x["parents"].zero_()
        x["parents"][:len(par)] = ints(par)
        x["kept"].copy_(ints([min(max(v, 0), 1 + b % 4) for b, v in enumerate(new)]))
        x["path"].copy_(ints([[0, 1, 2, 3]] * B))
        for k in ("qkv", "dy"):
            x[k].copy_(torch.randn(x[k].shape, generator=gen, device="cuda"))
        step(*eager)
        g.replay()
        for k in eager[2]:
            assert torch.equal(eager[2][k], other[2][k]), (i, k)
        assert other[0].dev_status.item() == 0  # empty places are no mistake
        for a, b in ((eager[0].K_pages, other[0].K_pages), (eager[0].V_pages, other[0].V_pages),
                     (eager[0].seq_len, other[0].seq_len), (eager[1].held, other[1].held)):
            assert torch.equal(a, b), i


def test_example_runs(E):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "tree_decoding.py")
    spec = importlib.util.spec_from_file_location("tree_decoding", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.main(tokens=200, steps=4)
    assert r["status"] == 0 and r["kept"] >= 4 * 2
