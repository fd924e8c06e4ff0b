"""The paged-cache operators against plain float64 forms of them.

Bounds, with u = 2^-24 (float32) and r = 2^-9 for bfloat16 (half its unit
roundoff), 0 for float32:

* rotation: three float32 roundings of products of size |a| + |b|, e =
  4 u (|a| + |b|), then one rounding to the type: the result lies between the
  rounded values of y - e and y + e;
* table: one float32 rounding of a float64 value: 1.01 u mscale;
* attention: a float32 dot product over d <= 128 channels summed in at most
  d / 4 steps is off by at most 32 u sum |q k| scale <= 32 u 30 (the inputs'
  largest sum of magnitudes is below 30 after scaling), which a softmax turns
  into twice that relative to max |v|, plus the weights' own exponentials and
  sums (4 u each): 1.2e-4 max |v| in the worst case and, errors of random sign,
  far below; 2e-5 max |v| is asked of float32.  bfloat16 adds one rounding of
  the weights and one of the result, each 2 r of the value rounded at most and
  r on average in magnitude: 2 r max |v| is asked of their sum.
* log-sum-exp: 2e-5 absolute (the logits' error).
"""
import math

import pytest
import torch

import paged_ref as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def E():
    from paper_2607_21475_gb300 import ebd
    ebd.lib()
    return ebd


def cache(E, s, status=None):
    if status is None:
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
    return E.PagedCache(s["K"], s["V"], s["bt"], s["seq_len"], status)


def unit(dtype):
    return 2.0 ** -9 if dtype == torch.bfloat16 else 0.0


def table_of(E, rot, n_pos, **kw):
    f, m = E.rotary_frequencies(rot, **kw)
    return E.ebd_rotary_table(f, n_pos, m)


# ---------------------------------------------------------------- rotation
@pytest.mark.parametrize("rot,kw", [(64, {}), (128, dict(base=1e6)), (6, {}), (2, {}),
                                    (128, dict(scaling="linear", factor=4.0)),
                                    (128, dict(scaling="base", factor=8.0)),
                                    (64, dict(scaling="parts", factor=16.0))])
def test_table_matches_float64(E, rot, kw):
    f, m = E.rotary_frequencies(rot, **kw)
    n = 150001
    got = E.ebd_rotary_table(f, n, m).double()
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f.cuda()
    ref = torch.stack([a.cos(), a.sin()], -1) * m
    assert (got - ref).abs().max().item() <= 1.01 * U * m


def check_rotated(got, x, cs, layout, inverse, dtype):
    ref = R.rotate(x, cs, layout, inverse)
    mag = R.rotate(x.abs(), cs.abs() * torch.tensor([1.0, -1.0], device="cuda"), layout)
    mag = torch.maximum(mag.abs(), R.rotate(x.abs(), cs.abs(), layout).abs())
    e = 4 * U * mag + 1e-37
    low, high = (v.to(torch.float32).to(dtype) if dtype == torch.bfloat16 else v
                 for v in (ref - e, ref + e))
    assert ((low <= got) & (got <= high)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("T,H,d,rot", [(1, 1, 64, 64), (1, 28, 128, 128), (33, 4, 128, 64),
                                       (257, 7, 64, 32), (5, 3, 80, 80), (19, 2, 96, 12),
                                       (3, 2, 10, 6), (4000, 5, 128, 128), (7, 1, 64, 2)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(E, dtype, layout, T, H, d, rot, inverse):
    g = torch.Generator(device="cuda").manual_seed(T * 131 + d)
    x = torch.randn((T, H + 2, d), generator=g, device="cuda").to(dtype)[:, 1:H + 1]
    tab = table_of(E, rot, 5000)
    pos = torch.randint(0, 5000, (T,), generator=g, device="cuda").int()
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = E.ebd_rotary(x, pos, tab, layout=lay, inverse=inverse, dev_status=st)
    check_rotated(got, x, tab[pos.long()], layout, inverse, dtype)
    assert torch.equal(got[..., rot:], x[..., rot:])
    assert st.item() == 0
    z = x.contiguous()
    E.ebd_rotary(z, pos, tab, out=z, layout=lay, inverse=inverse)  # in place
    assert torch.equal(z, got)


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rotary_rows_off_16_byte_boundaries(E, shift, layout):
    base = torch.randn(9 * 3 * 64 + 8, device="cuda").to(torch.bfloat16)
    x = base[shift:shift + 9 * 3 * 64].view(9, 3, 64)
    tab = table_of(E, 64, 100)
    pos = torch.arange(9, device="cuda").int() * 11
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    if layout == "pairs" and shift % 2:
        with pytest.raises(E.EbdError) as e:
            E.ebd_rotary(x, pos, tab, layout=lay)
        assert e.value.code == 4
        return
    check_rotated(E.ebd_rotary(x, pos, tab, layout=lay), x, tab[pos.long()], layout, False,
                  torch.bfloat16)


@pytest.mark.parametrize("layout", [0, 1])
def test_rotary_inverse_is_the_gradient(E, layout):
    """<g, R x> = <R' g, x>, and R' g matches central differences of <g, R x>."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, g = (torch.randn((6, 2, 64), generator=gen, device="cuda") for _ in range(2))
    tab = table_of(E, 32, 400)
    pos = torch.tensor([0, 1, 17, 100, 255, 399], device="cuda").int()
    back = E.ebd_rotary(g, pos, tab, layout=layout, inverse=True)
    name = "half" if layout == 0 else "pairs"
    cs = tab[pos.long()]
    assert abs((g.double() * R.rotate(x, cs, name)).sum() - (back.double() * x.double()).sum()) < 1e-3
    h = 0.5  # the map is linear: differences carry rounding only, 2^-24 of |y| / h
    for t, c in [(1, 0), (2, 5), (3, 16), (4, 31), (5, 33)]:
        e = torch.zeros_like(x)
        e[t, 1, c] = h
        d = (E.ebd_rotary(x + e, pos, tab, layout=layout).double()
             - E.ebd_rotary(x - e, pos, tab, layout=layout).double())
        assert abs(((g.double() * d).sum() / (2 * h) - back[t, 1, c].double()).item()) < 2e-5


def test_rotary_position_outside_the_table(E):
    x = torch.randn((3, 2, 64), device="cuda")
    tab = table_of(E, 64, 50)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = E.ebd_rotary(x, torch.tensor([-4, 10, 50], device="cuda").int(), tab, dev_status=st)
    assert st.item() == E.EBD_DEV_RANGE
    check_rotated(got, x, tab[[0, 10, 49]], "half", False, torch.float32)


# ---------------------------------------------------------------- append
APPENDS = [  # new, total, hq, hkv, d, page, rot
    ([1], [1], 4, 4, 64, 16, 64),
    ([1] * 9, [1, 16, 17, 33, 64, 100, 8, 9, 300], 8, 2, 128, 16, 128),
    ([5, 0, 33, 1], [5, 7, 120, 64], 28, 4, 128, 64, 64),
    ([130, 1, 0, 257], [130, 1, 0, 1000], 4, 1, 64, 8, 16),
    ([3, 40], [3, 41], 6, 3, 80, 32, 80),
    ([3, 40], [30, 41], 2, 1, 10, 32, 6),
    ([1] * 70, list(range(1, 71)), 2, 1, 64, 32, 64),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("order", ["head", "row", "side"])
@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append(E, dtype, layout, order, case):
    new, total, hq, hkv, d, page, rot = APPENDS[case]
    s = R.make(new, total, hq, hkv, d, page, dtype, 100 + case, order)
    pc = cache(E, s)
    tab = table_of(E, rot, max(total) + 1)
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    K0, V0 = s["K"].clone(), s["V"].clone()
    q_out = torch.empty((s["T"], hq, d), dtype=dtype, device="cuda")
    E.ebd_paged_append(pc, s["k"], s["v"], s["cu"], table=tab, layout=lay, q=s["q"], q_out=q_out)
    pos = torch.cat([torch.arange(n - w, n) for w, n in zip(new, total)]).cuda()
    seq = torch.cat([torch.full((w,), b) for b, w in enumerate(new)]).cuda()
    cs = tab[pos]
    check_rotated(q_out, s["q"], cs, layout, False, dtype)
    at, off = s["bt"].long()[seq, pos // page], pos % page
    check_rotated(s["K"][at, :, off], s["k"], cs, layout, False, dtype)
    assert torch.equal(s["V"][at, :, off], s["v"])
    untouched = torch.ones(K0.shape[:1] + K0.shape[2:3], dtype=torch.bool, device="cuda")
    untouched[at, off] = False
    keep = untouched[:, None, :, None].expand_as(K0)
    assert torch.equal(s["K"][keep], K0[keep]) and torch.equal(s["V"][keep], V0[keep])
    assert pc.dev_status.item() == 0


def test_append_without_rotation_copies(E):
    s = R.make([3, 9], [20, 9], 2, 2, 64, 16, torch.bfloat16, 3)
    pc = cache(E, s)
    E.ebd_paged_append(pc, s["k"], s["v"], s["cu"])
    for t, (b, pos) in enumerate([(0, 17), (0, 18), (0, 19)] + [(1, i) for i in range(9)]):
        for h in range(2):
            assert torch.equal(R.row(s["K"], s["bt"], b, h, pos), s["k"][t, h])
            assert torch.equal(R.row(s["V"], s["bt"], b, h, pos), s["v"][t, h])


def test_append_drops_what_has_no_page(E):
    """Positions before 0 or past the block table, and pages outside the pool."""
    s = R.make([4, 4, 4], [16, 16, 16], 2, 1, 64, 8, torch.float32, 4)
    s["seq_len"].copy_(torch.tensor([18, 16, 2]).int())   # 2 past the table; 2 before 0
    s["bt"][1, 1] = s["K"].shape[0] + 5                   # sequence 1: a page outside the pool
    K0, V0 = s["K"].clone(), s["V"].clone()
    pc = cache(E, s)
    E.ebd_paged_append(pc, s["k"], s["v"], s["cu"], table=table_of(E, 64, 64), q=s["q"],
                       q_out=torch.empty_like(s["q"].contiguous()))
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    changed = (s["V"] != V0).any(-1).any(1)
    want = torch.zeros_like(changed)
    for b, pos in [(0, 14), (0, 15), (2, 0), (2, 1)]:
        want[s["bt"][b, pos // 8].long(), pos % 8] = True
    assert torch.equal(changed, want) and torch.equal((s["K"] != K0).any(-1).any(1), want)


@pytest.mark.parametrize("cu", [[5, 8, 12], [0, 4, 9], [3, 3, 12], [0, 8, 6], [5, 8, 9], [-2, 6, 12]])
def test_append_skips_tokens_of_no_sequence(E, cu):
    """Packed tokens before the first offset, past the last one or under an offset
    that steps back belong to no sequence: nothing is written for them, not even over
    a sequence's earlier rows, and the status tells."""
    s = R.make([6, 6], [40, 50], 4, 2, 64, 16, torch.bfloat16, 5)
    K0, V0 = s["K"].clone(), s["V"].clone()
    pc, tab = cache(E, s), table_of(E, 64, 64)
    q_out = torch.full((12, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    E.ebd_paged_append(pc, s["k"], s["v"], torch.tensor(cu, device="cuda").int(), table=tab,
                       q=s["q"], q_out=q_out)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    owned = [(b, t) for b in (0, 1) for t in range(max(cu[b], 0), cu[b + 1])]
    changed = torch.zeros(K0.shape[:1] + K0.shape[2:3], dtype=torch.bool, device="cuda")
    q_left = torch.ones(12, dtype=torch.bool)
    for b, t in owned:
        pos = int(s["seq_len"][b]) - (cu[b + 1] - t)
        page, off = int(s["bt"][b, pos // 16]), pos % 16
        changed[page, off] = True
        q_left[t] = False
        assert torch.equal(s["V"][page, :, off], s["v"][t])
        cs = tab[pos][None]
        check_rotated(s["K"][page, :, off][None], s["k"][t][None], cs, "half", False, torch.bfloat16)
        check_rotated(q_out[t][None], s["q"][t][None], cs, "half", False, torch.bfloat16)
    same = ~changed[:, None, :, None].expand_as(K0)
    assert torch.equal(s["K"][same], K0[same]) and torch.equal(s["V"][same], V0[same])
    assert (q_out[q_left] == 7).all()


# ---------------------------------------------------------------- attention
def check_attention(E, s, dtype, scale, window, q=None, stream=None):
    q = s["q"] if q is None else q
    pc = cache(E, s)
    y, lse = E.ebd_paged_attention(q, pc, s["cu"], s["max_new"], scale=scale, window=window,
                                   stream=stream)
    d = q.shape[2]
    ry, rl = R.attention(q, s["K"], s["V"], s["bt"], s["seq_len"], s["cu"],
                         d ** -0.5 if scale is None else scale, window)
    vmax = 5.5  # standard normal values
    tol = 2e-5 * vmax + 2 * unit(dtype) * vmax
    assert y.dtype == dtype and torch.isfinite(y).all()
    assert (y.double() - ry).abs().max().item() <= tol
    empty = rl == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert (y[empty] == 0).all()
    if (~empty).any():
        assert (lse.double() - rl)[~empty].abs().max().item() <= 2e-5
    assert pc.dev_status.item() == 0


ATTN = [  # new, total, hq, hkv, page, window
    ([1], [1], 4, 4, 16, 0),
    ([1], [1000], 28, 4, 16, 0),
    ([1] * 5, [1, 63, 64, 65, 777], 8, 2, 64, 0),
    ([1, 0, 1], [5, 0, 3000], 16, 1, 8, 100),
    ([4, 2, 1], [4, 300, 129], 8, 2, 32, 0),
    ([16, 16], [16, 5000], 2, 2, 128, 0),
    ([37], [37], 7, 1, 16, 0),
    ([128, 129, 1], [128, 129, 1], 4, 4, 256, 0),
    ([300, 1, 0, 77], [300, 513, 12, 1200], 8, 2, 16, 0),
    ([300, 1, 0, 77], [2300, 513, 12, 1200], 8, 2, 1024, 65),
    ([515], [1601], 28, 4, 64, 0),
    ([64, 64], [64, 2000], 3, 1, 32, 1),
    ([200, 3], [200, 3], 128, 1, 32, 128),
    ([1] * 40, [i * 37 % 900 + 1 for i in range(40)], 4, 2, 16, 0),
    ([3] * 33, [i * 91 % 700 + 3 for i in range(33)], 32, 8, 16, 0),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(E, dtype, d, case):
    new, total, hq, hkv, page, window = ATTN[case]
    s = R.make(new, total, hq, hkv, d, page, dtype, 200 + case, stale=math.nan)
    check_attention(E, s, dtype, None, window)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 7, 12, 16, 24, 32, 48, 128])
@pytest.mark.parametrize("new,total", [([1], [5003]), ([2], [4100]), ([1, 150], [2900, 1300])])
def test_items_split_over_many_ctas(E, dtype, d, group, new, total):
    """Few rows over many keys: every CTA has a piece of an item, of 1 to 256 rows
    in slots of 8 to 256; twice, with the same bits."""
    s = R.make(new, total, group, 1, d, 32, dtype, 300 + group, stale=math.nan)
    check_attention(E, s, dtype, None, 0)
    y0, l0 = E.ebd_paged_attention(s["q"], cache(E, s), s["cu"], s["max_new"])
    y1, l1 = E.ebd_paged_attention(s["q"], cache(E, s), s["cu"], s["max_new"])
    assert torch.equal(y0, y1) and torch.equal(l0, l1)


CLOSE = ATTN + [  # as ATTN; long contexts, where a lost tile changes little
    ([1], [5003], 1, 1, 32, 0),
    ([1], [5003], 28, 4, 16, 0),
    ([2], [4100], 16, 1, 32, 0),
    ([1, 150], [2900, 1300], 128, 1, 32, 0),
    ([1, 1, 1], [30000, 20011, 7777], 8, 2, 64, 0),
    ([5, 5], [16379, 6139], 32, 8, 64, 0),
    ([300], [9000], 8, 2, 128, 0),
    ([300, 7], [9000, 12345], 14, 2, 16, 4000),
    ([1] * 300, [i * 53 % 400 + 1 for i in range(300)], 4, 2, 16, 0),
    ([i % 3 for i in range(1025)], [i * 17 % 90 + 2 for i in range(1025)], 4, 1, 8, 0),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(CLOSE)))
def test_attention_to_the_size_of_its_roundings(E, dtype, d, case):
    """Every output within the roundings of its own weights and value, however small it
    is against the largest value."""
    new, total, hq, hkv, page, window = CLOSE[case]
    s = R.make(new, total, hq, hkv, d, page, dtype, 400 + case, stale=math.nan)
    pc = cache(E, s)
    y, lse = E.ebd_paged_attention(s["q"], pc, s["cu"], s["max_new"], window=window)
    K, V = s["K"].nan_to_num(0.0), s["V"].nan_to_num(0.0)
    ry, rl, mean, root = R.attention_detail(s["q"], K, V, s["bt"].clamp(min=0), s["seq_len"],
                                            s["cu"], d ** -0.5, window)
    assert ((y.double() - ry).abs() <= R.attention_bound(ry, mean, root, dtype)).all()
    assert ((lse.double() - rl).abs() <= 2e-5).all()
    assert pc.dev_status.item() == 0


@pytest.mark.parametrize("hq,hkv", [(4, 1), (32, 8)])
@pytest.mark.parametrize("new,total", [(1, 92), (1, 601), (1, 2801), (2, 9002), (1, 30001),
                                       (40, 1240)])
def test_float32_attention_keeps_its_digits(E, hq, hkv, new, total):
    """Relative error of the whole output, logits of standard deviation 2 over 128
    channels.  A logit summed as 8 sums of 16 products (of size 2 each) is off by
    2^-24 / 3^1/2 x 2 x (8 x 16^2 / 2 + 16 x 36)^1/2 x 128^-1/2 = 2.4e-7 (one sum of 128: 5.5e-7),
    and more where the logit is large and its weight counts; the exponential, its
    argument and the sums over keys add about 4e-7.  1e-6 is asked, of every seed."""
    for seed in range(4):
        s = R.make([new], [total], hq, hkv, 128, 64, torch.float32, 500 + seed, stale=math.nan)
        q = (s["q"] * 2).contiguous()
        y, lse = E.ebd_paged_attention(q, cache(E, s), s["cu"], new)
        ry, rl, _, _ = R.attention_detail(q, s["K"].nan_to_num(0.0), s["V"].nan_to_num(0.0),
                                          s["bt"].clamp(min=0), s["seq_len"], s["cu"],
                                          128 ** -0.5, 0)
        assert ((y.double() - ry).norm() / ry.norm()).item() <= 1e-6
        assert ((lse.double() - rl).norm() / rl.norm()).item() <= 3e-7


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("order", ["row", "side"])
@pytest.mark.parametrize("new", [1, 70])
def test_attention_over_other_pool_orders(E, dtype, order, new):
    s = R.make([new] * 3, [new, 200, 333], 8, 2, 128, 32, dtype, 31, order, stale=math.inf)
    check_attention(E, s, dtype, 0.05, 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new,total", [([3, 20, 130], [1, 0, 100]), ([2, 1], [0, 0]),
                                       ([5, 5], [2, 40])])
def test_attention_rows_without_a_key(E, dtype, new, total):
    """Sequences shorter than their new tokens: the first tokens lie before position 0."""
    s = R.make(new, total, 4, 2, 64, 16, dtype, 41, stale=math.nan)
    check_attention(E, s, dtype, None, 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new", [1, 6, 200])
def test_attention_peaked_rows(E, dtype, new):
    """Logits of +-40: one key takes nearly all the weight, and the maximum
    moves from tile to tile (so that every earlier sum is rescaled)."""
    s = R.make([new], [900], 4, 2, 128, 64, dtype, 51)
    s["K"].mul_(torch.linspace(0.2, 3.0, s["K"].shape[0], device="cuda")[:, None, None, None].to(dtype))
    pc = cache(E, s)
    y, lse = E.ebd_paged_attention(s["q"], pc, s["cu"], new, scale=0.4)
    ry, rl = R.attention(s["q"], s["K"], s["V"], s["bt"], s["seq_len"], s["cu"], 0.4, 0)
    # logits up to 160 in magnitude of products: 32 u 0.4 sum |q k| < 32 u 400
    tol = 2 * 32 * U * 400 * 5.5 + 2 * unit(dtype) * 5.5
    assert (y.double() - ry).abs().max().item() <= tol
    assert (lse.double() - rl).abs().max().item() <= 32 * U * 400


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new", [2, 40, 300])
def test_attention_nonfinite_values_of_later_tokens_stay_there(E, dtype, new):
    """A NaN or infinite value is seen by its own token and later ones only."""
    s = R.make([new], [new + 150], 4, 2, 64, 16, dtype, 61)
    bad = {150 + new // 2: math.nan, 150 + new - 1: math.inf}
    for pos, x in bad.items():
        R.row(s["V"], s["bt"], 0, 1, pos)[5] = x
    y, lse = E.ebd_paged_attention(s["q"], cache(E, s), s["cu"], new)
    ry, rl = R.attention(s["q"], s["K"], s["V"], s["bt"], s["seq_len"], s["cu"], 0.125, 0)
    clean = new // 2
    assert torch.isfinite(y[:clean]).all() and torch.isfinite(y[:, :2]).all()
    assert torch.isnan(y[clean:new - 1, 2:, 5]).all()
    fine = torch.isfinite(ry)
    assert ((y.double() - ry)[fine].abs() <= 2e-5 * 5.5 + 2 * unit(dtype) * 5.5).all()
    assert (lse.double() - rl).abs().max().item() <= 2e-5


@pytest.mark.parametrize("dtype,hq,hkv,d,new,total,window", [
    (torch.bfloat16, 32, 8, 128, 1216, 33000, 0),      # whole items: 33k keys in one CTA's piece
    (torch.bfloat16, 32, 8, 64, 1216, 33000, 0),
    (torch.bfloat16, 32, 8, 128, 1216, 60000, 32000),  # hidden at the window's far edge too
    (torch.bfloat16, 28, 4, 128, 5, 100000, 0),        # drafts, pieces of many CTAs
    (torch.float32, 4, 4, 64, 500, 33000, 0),
    (torch.float32, 8, 2, 128, 3, 70000, 0),
])
def test_nonfinite_value_rows_over_long_contexts(E, dtype, hq, hkv, d, new, total, window):
    """Value rows that are NaN in every channel, one in the middle of the new tokens and
    one that leaves the window among them: rows that do not see them are right to the last
    channel, rows that do are NaN, another sequence notices nothing, and no wait runs out."""
    s = R.make([new, 70], [total, 900], hq, hkv, d, 64, dtype, 63)
    V0 = s["V"].clone()
    bad = [total - new + new // 2]
    if window:
        bad.append(total - new + new // 4 - window)  # seen by the first quarter
    for pos in bad:
        for h in range(hkv):
            R.row(s["V"], s["bt"], 0, h, pos).fill_(math.nan)
    pc = cache(E, s)
    y, lse = E.ebd_paged_attention(s["q"], pc, s["cu"], s["max_new"], window=window)
    assert pc.dev_status.item() == 0
    at = torch.arange(total - new, total, device="cuda")
    sees = torch.zeros(new, dtype=torch.bool, device="cuda")
    for pos in bad:
        sees |= (pos <= at) & ((at - pos < window) if window else True)
    assert sees.any() and not sees.all()
    assert torch.isnan(y[:new][sees]).all() and torch.isfinite(y[:new][~sees]).all()
    assert torch.isfinite(y[new:]).all()
    ry, rl, mean, root = R.attention_detail(s["q"][new:], s["K"], s["V"].nan_to_num(0.0),
                                            s["bt"][1:], s["seq_len"][1:], [0, 70], d ** -0.5,
                                            window)
    assert ((y[new:].double() - ry).abs() <= R.attention_bound(ry, mean, root, dtype)).all()
    # tokens around each bad position, as the last ones of a shorter sequence
    for pos in bad:
        mid = pos - (total - new) + (window if pos < total - new else 0)
        lo, hi = max(mid - 64, 0), min(mid + 64, new)
        ry, rl, mean, root = R.attention_detail(s["q"][lo:hi], s["K"], V0, s["bt"][:1],
                                                [total - new + hi], [0, hi - lo], d ** -0.5,
                                                window)
        ok = ~sees[lo:hi]
        assert ok.any()
        bound = R.attention_bound(ry, mean, root, dtype)
        assert ((y[lo:hi].double() - ry).abs() <= bound)[ok].all()
        assert (lse[lo:hi].double() - rl).abs().max().item() <= 2e-5


@pytest.mark.parametrize("new", [2, 40, 300])
def test_attention_window_hides_nonfinite_values(E, new):
    """The same at the window's far edge: a NaN value older than the window."""
    s = R.make([new], [new + 150], 4, 2, 64, 16, torch.bfloat16, 62)
    R.row(s["V"], s["bt"], 0, 0, 101)[7] = math.nan
    y, _ = E.ebd_paged_attention(s["q"], cache(E, s), s["cu"], new, window=50)
    sees = (torch.arange(150, 150 + new) - 101 < 50).cuda()
    assert torch.isnan(y[sees][:, :2, 7]).all()
    assert torch.isfinite(y[~sees]).all() and torch.isfinite(y[:, 2:]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new", [1, 50])
def test_attention_does_not_depend_on_the_launch(E, dtype, new):
    """Same bits twice, and on another stream."""
    s = R.make([new, 1, new], [3000, 700, new], 8, 2, 128, 32, dtype, 71)
    y0, l0 = E.ebd_paged_attention(s["q"], cache(E, s), s["cu"], s["max_new"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y1, l1 = E.ebd_paged_attention(s["q"], cache(E, s), s["cu"], s["max_new"], stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(y0, y1) and torch.equal(l0, l1)


def test_workspace_of_a_call_on_another_stream_is_not_reused(E):
    """The binding's own workspace stays out of the allocator's hands while a call
    on a stream other than the current one still works with it."""
    s = R.make([40] * 4, [3000, 2500, 40, 999], 8, 2, 128, 32, torch.bfloat16, 72)
    ref, _ = E.ebd_paged_attention(s["q"], cache(E, s), s["cu"], 40)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ys = []
    for _ in range(30):
        y, _ = E.ebd_paged_attention(s["q"], cache(E, s), s["cu"], 40, stream=side)
        ys.append(y)
        for n in (1 << 20, 30 << 20, 40 << 20):  # what the allocator would hand out again
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    assert all(torch.equal(y, ref) for y in ys)


def test_buffers_of_a_call_on_another_stream_are_its_own(E):
    """Workspace, outputs and the frequencies' copy of a call on a side stream share no
    memory with tensors freed on the current stream whose writes are still queued,
    nor with tensors made there after a dropped output."""
    s = R.make([40] * 4, [3000, 2500, 40, 999], 8, 2, 128, 32, torch.bfloat16, 73)
    pc = cache(E, s)
    y0, l0 = E.ebd_paged_attention(s["q"], pc, s["cu"], 40)
    f, m = E.rotary_frequencies(128)
    t0 = E.ebd_rotary_table(f, 3000, m)
    pos = torch.arange(s["T"], device="cuda").int()
    r0 = E.ebd_rotary(s["q"], pos, t0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    sizes = [E.ebd_paged_attention_workspace_bytes(pc, 8, 40), t0.numel() * 4, y0.numel() * 2,
             l0.numel() * 4, f.numel() * 8]
    got = []
    for _ in range(4):
        freed = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
        torch.cuda._sleep(20_000_000)  # about 10 ms: what follows here waits that long
        for x in freed:
            x.fill_(255)
        del freed, x
        tab = E.ebd_rotary_table(f, 3000, m, stream=side)
        rot = E.ebd_rotary(s["q"], pos, tab, stream=side)
        y, _ = E.ebd_paged_attention(s["q"], pc, s["cu"], 40, stream=side)  # lse dropped
        got.append((y, rot, tab))
        for n in sizes:
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    for y, rot, tab in got:
        assert torch.equal(y, y0) and torch.equal(rot, r0) and torch.equal(tab, t0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_graph_follows_the_lengths(E, dtype):
    """Append and attention captured once, replayed as the sequences grow."""
    steps = 70
    s = R.make([1, 1], [steps + 30, steps + 200], 8, 2, 64, 16, dtype, 81)
    pc, tab = cache(E, s), table_of(E, 64, 400)
    s["seq_len"].copy_(torch.tensor([30, 200]).int())
    q_out = torch.empty((2, 8, 64), dtype=dtype, device="cuda")
    y = torch.empty((2, 8, 64), dtype=dtype, device="cuda")
    lse = torch.empty((2, 8), device="cuda")
    ws = torch.empty(max(1, E.ebd_paged_attention_workspace_bytes(pc, 8, 1)), dtype=torch.uint8,
                     device="cuda")

    def step():
        s["seq_len"].add_(1)
        E.ebd_paged_append(pc, s["k"], s["v"], s["cu"], table=tab, q=s["q"], q_out=q_out)
        E.ebd_paged_attention(q_out, pc, s["cu"], 1, y=y, lse=lse, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(steps - 1):
        graph.replay()
    torch.cuda.synchronize()
    assert s["seq_len"].tolist() == [30 + steps, 200 + steps]
    ry, rl = R.attention(q_out, s["K"], s["V"], s["bt"], s["seq_len"], s["cu"], 0.125, 0)
    assert (y.double() - ry).abs().max().item() <= (2e-5 + 2 * unit(dtype)) * 5.5
    assert (lse.double() - rl).abs().max().item() <= 2e-5
    assert pc.dev_status.item() == 0


@pytest.mark.parametrize("new", [1, 40])
def test_offsets_past_32_bits(E, new):
    """A pool of more than 2^31 elements, the sequence's pages at its far end."""
    hkv, page, d = 2, 64, 128
    n_pages = (1 << 31) // (hkv * page * d) + 40
    K, V = (torch.empty((n_pages, hkv, page, d), dtype=torch.bfloat16, device="cuda")
            for _ in range(2))
    s = R.make([new], [700], 8, hkv, d, page, torch.bfloat16, 91, spare=0)
    shift = n_pages - s["K"].shape[0]
    K[shift:].copy_(s["K"])
    V[shift:].copy_(s["V"])
    s.update(K=K, V=V, bt=s["bt"] + shift)
    pc, tab = cache(E, s), table_of(E, 128, 1000)
    E.ebd_paged_append(pc, s["k"], s["v"], s["cu"], table=tab)
    for i in (0, new - 1):
        assert torch.equal(R.row(V, s["bt"], 0, 1, 700 - new + i), s["v"][i, 1])
    check_attention(E, s, torch.bfloat16, None, 0)
    out = E.alloc_compact(1, hkv, 64, d, torch.bfloat16, "cuda")
    out.idx_c.copy_((torch.arange(64).int() * 10).cuda().expand(1, hkv, 64))
    out.n_kept.fill_(64)
    E.ebd_paged_gather(pc, out)
    for h in range(hkv):
        assert torch.equal(out.K_c[0, h].double(), R.rows(K, s["bt"], 0, h, 700)[::10][:64])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new", [1, 30, 200])
def test_attention_reports_bad_pages_and_offsets(E, dtype, new):
    """Pages outside the pool and lengths past the block table: a status bit,
    and nothing read outside (other sequences stay right)."""
    s = R.make([new, new], [260, 300], 4, 2, 64, 16, dtype, 95)
    good = dict(s, bt=s["bt"].clone())
    s["bt"][0, 3] = 1 << 20
    s["bt"][0, 5] = -7
    pc = cache(E, s)
    y, lse = E.ebd_paged_attention(s["q"], pc, s["cu"], new)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    y2, lse2 = E.ebd_paged_attention(s["q"], cache(E, good), s["cu"], new)
    assert torch.equal(y[new:], y2[new:]) and torch.equal(lse[new:], lse2[new:])
    far = dict(good, seq_len=good["seq_len"].clone())
    far["seq_len"][1] = 1 << 30
    pc = cache(E, far)
    y, _ = E.ebd_paged_attention(s["q"], pc, s["cu"], new)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    assert torch.equal(y[:new], y2[:new])
    wrong = torch.tensor([0, new, 5 * new], device="cuda").int()  # past the packed tokens
    pc = cache(E, good)
    E.ebd_paged_attention(s["q"], pc, wrong, new)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("most", [1, 7, 31])
def test_attention_more_new_tokens_than_the_bound(E, dtype, most):
    """A sequence with more new tokens than max_new: a status bit, its tokens past
    the bound are left as they were, nothing else is touched."""
    s = R.make([most, 40, 1], [900, 800, 300], 8, 2, 128, 32, dtype, 96)
    pc = cache(E, s)
    y = torch.full((s["T"], 8, 128), 7.0, dtype=dtype, device="cuda")
    need = E.ebd_paged_attention_workspace_bytes(pc, 8, most)
    ws = torch.full((need + 4096,), 9, dtype=torch.uint8, device="cuda")
    E.ebd_paged_attention(s["q"], pc, s["cu"], most, y=y, workspace=ws[:need])
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    assert (ws[need:] == 9).all()
    assert (y[2 * most:most + 40] == 7).all()
    keep = list(range(most)) + [most + 40]
    ry, _ = R.attention(s["q"], s["K"], s["V"], s["bt"], s["seq_len"], s["cu"], 128 ** -0.5, 0)
    assert (y.double() - ry)[keep].abs().max().item() <= 2e-5 * 5.5 + 2 * unit(dtype) * 5.5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cu", [[5, 8, 12], [0, 4, 9], [3, 3, 12], [0, 0, 11], [0, 12, 13]])
def test_attention_reports_tokens_of_no_sequence(E, dtype, cu):
    """Offsets that do not run from 0 to n_tokens: a status bit; the rows of tokens
    of no sequence are left as they were, the others are right."""
    s = R.make([6, 6], [40, 50], 4, 2, 64, 16, dtype, 97)
    pc = cache(E, s)
    y = torch.full((12, 4, 64), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((12, 4), 7.0, device="cuda")
    off = torch.tensor(cu, device="cuda").int()
    E.ebd_paged_attention(s["q"], pc, off, 12, y=y, lse=lse)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    lo, hi = cu[0], min(cu[2], 12)
    held = [min(c, 12) for c in cu]
    ry, rl = R.attention(s["q"], s["K"], s["V"], s["bt"], s["seq_len"],
                         torch.tensor(held, device="cuda").int(), 0.125, 0)
    for t in range(12):
        if lo <= t < hi:
            assert (y[t].double() - ry[t]).abs().max().item() <= (2e-5 + 2 * unit(dtype)) * 5.5
            assert (lse[t].double() - rl[t]).abs().max().item() <= 2e-5
        else:
            assert (y[t] == 7).all() and (lse[t] == 7).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("page", [8, 16, 32])
@pytest.mark.parametrize("new,window", [(1, 50), (1, 1), (40, 50), (300, 129), (7, 1000)])
def test_pages_behind_the_window_may_be_released(E, dtype, page, new, window):
    """Blocks that end before the first position that a new token sees may hold any
    number: no status, the same bits.  The block of that position may not."""
    total = [new + 211, new + 1500, new]
    s = R.make([new] * 3, total, 4, 2, 64, page, dtype, 98, stale=math.nan)
    y0, l0 = E.ebd_paged_attention(s["q"], cache(E, s), s["cu"], new, window=window)
    first = [max(0, n - new - window + 1) for n in total]
    for fill in (-1, 1 << 30):
        bt = s["bt"].clone()
        for b in range(3):
            bt[b, :first[b] // page] = fill
        pc = cache(E, dict(s, bt=bt))
        y, lse = E.ebd_paged_attention(s["q"], pc, s["cu"], new, window=window)
        assert pc.dev_status.item() == 0
        assert torch.equal(y, y0) and torch.equal(lse, l0)
        bt[1, first[1] // page] = fill
        pc = cache(E, dict(s, bt=bt))
        E.ebd_paged_attention(s["q"], pc, s["cu"], new, window=window)
        assert pc.dev_status.item() == E.EBD_DEV_RANGE


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 64, 128])
@pytest.mark.parametrize("new", [1, 30, 200])
def test_attention_leaves_out_keys_on_bad_pages(E, dtype, d, page, new):
    """The positions of a block outside the pool take no part in any row, over long
    runs of tiles and in the last one; a row that sees nothing else is empty."""
    total = [new + 700, new + 1400, new]
    s = R.make([new] * 3, total, 4, 2, d, page, dtype, 99, stale=math.nan)
    absent = [(0, 0), (0, 3), (0, (total[0] - 1) // page), (1, 600 // page), (1, 700 // page),
              (2, 0)]
    bt = s["bt"].clone()
    for i, (b, block) in enumerate(absent):
        bt[b, block] = -1 if i % 2 else s["K"].shape[0] + i
    pc = cache(E, dict(s, bt=bt))
    y, lse = E.ebd_paged_attention(s["q"], pc, s["cu"], new)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    ry, rl, mean, root = R.attention_detail(s["q"], s["K"].nan_to_num(0.0),
                                            s["V"].nan_to_num(0.0), s["bt"], s["seq_len"],
                                            s["cu"], d ** -0.5, 0, absent)
    empty = rl == -math.inf
    assert torch.equal(lse == -math.inf, empty) and (y[empty] == 0).all()
    assert empty.any() and not empty.all()
    bound = R.attention_bound(ry, mean, root, dtype)
    assert ((y.double() - ry).abs() <= bound)[~empty].all()
    assert (lse.double() - rl)[~empty].abs().max().item() <= 2e-5


# ---------------------------------------------------------------- gather
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("order", ["head", "row"])
@pytest.mark.parametrize("d,page,cap", [(64, 8, 1), (128, 64, 300), (80, 16, 77), (8, 32, 64)])
def test_gather(E, dtype, order, d, page, cap):
    total = [1000, 1, 0, 333]
    s = R.make([1] * 4, total, 4, 2, d, page, dtype, 300 + d, order)
    out = E.alloc_compact(4, 2, cap, d, dtype, "cuda")
    out.K_c.fill_(7)
    out.V_c.fill_(7)
    g = torch.Generator().manual_seed(cap)
    out.idx_c.copy_(torch.randint(-3, 1010, (4, 2, cap), generator=g).int())
    out.n_kept.copy_(torch.tensor([[cap, cap + 5], [cap // 2, 0], [cap, cap], [cap, 1]]).int())
    pc = cache(E, s)
    E.ebd_paged_gather(pc, out)
    for b in range(4):
        for h in range(2):
            for p in range(cap):
                i = int(out.idx_c[b, h, p])
                if p < int(out.n_kept[b, h]) and 0 <= i < total[b]:
                    assert torch.equal(out.K_c[b, h, p], R.row(s["K"], s["bt"], b, h, i))
                    assert torch.equal(out.V_c[b, h, p], R.row(s["V"], s["bt"], b, h, i))
                else:
                    assert (out.K_c[b, h, p] == 7).all() and (out.V_c[b, h, p] == 7).all()
    assert pc.dev_status.item() == 0


# ---------------------------------------------------------------- together
def test_example_prefills_evicts_and_decodes():
    """The example's last step against float64 attention over its own pages, and
    a full budget: the compact decode then equals the paged attention."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "paged_eviction.py")
    spec = importlib.util.spec_from_file_location("paged_eviction", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    r = ex.main(tokens=700, budget=0.3, chunk=190, page=32)
    pc = r["pc"]
    ry, rl = R.attention(r["q"], pc.K_pages, pc.V_pages, pc.block_table, pc.seq_len, r["cu"],
                         128 ** -0.5, 0)
    assert (r["y"].double() - ry).abs().max().item() <= (2e-5 + 2 * 2.0 ** -9) * 5.5
    assert (r["lse_paged"].double() - rl).abs().max().item() <= 2e-5
    assert 0.25 * 704 < r["kept"] < 0.35 * 704
    assert torch.isfinite(r["error"]).all() and torch.isfinite(r["radius"]).all()
    full = ex.main(tokens=300, budget=1.0, chunk=128)
    # bfloat16 results of the paged attention against float32 ones: 2^-8 of |y| each
    assert full["error"].max().item() <= 2.0 ** -8
    assert (full["lse_paged"] - full["lse_compact"]).abs().max().item() <= 4e-5
