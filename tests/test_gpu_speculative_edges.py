"""A speculative step's operators at the ends of their ranges, against the plain forms and
with the bounds of test_gpu_speculative.py (u = 2^-24)."""
import math

import pytest
import torch

import paged_ref as R
import speculative_ref as S
from test_gpu_speculative import (cache, check_grad, check_normed, fresh_pool, ints, norm_inputs,
                                  run_steps, slots_of, table_of, tree_case)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    from paper_2607_21475_gb300 import ebd
    ebd.lib()
    return ebd


# ---------------------------------------------------------------- rows of any finite size
# Powers of two only scale a row exactly, so the bounds of ordinary rows hold; what a row of
# such values leaves below 1e-37 is the bounds' own slack.
def sized_rows(x, sizes):
    """Row t of x scaled so that its largest value has the t-th size; signs and the values'
    proportions stay."""
    big = x.double().abs().amax(-1, keepdim=True)
    s = torch.tensor(sizes, dtype=torch.float64, device="cuda")[:, None, None]
    return (x.double() / big * s).to(x.dtype)


LARGE = [(64, 64), (128, 128), (128, 32), (80, 20), (512, 0), (512, 512)]


def large_rows(E, d, rot, dtype, per_head=False):
    top = torch.finfo(dtype).max
    sizes = [2.0 ** 58, 2.0 ** 59.6, 2.0 ** 64, 1e30, 1e38, top, top, top, top, 1.0]
    x, dy, w, pos = norm_inputs(len(sizes), 3, d, dtype, per_head, d + rot)
    x = sized_rows(x, sizes)
    x[6] = torch.where(x[6] < 0, -top, top).to(dtype)  # every value the largest
    x[7] = torch.where(x[7] < 0, -1e38, 1e38).to(dtype)
    x[8] = 1
    x[8, :, d // 2] = -top
    return x, dy * 1e6, w, pos, table_of(E, rot, 4000) if rot else None


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("d,rot", LARGE)
@pytest.mark.parametrize("per_head", [False, True])
def test_norm_of_rows_up_to_the_largest_value(E, dtype, layout, d, rot, per_head):
    x, dy, w, pos, tab = large_rows(E, d, rot, dtype, per_head)
    lay = E.EBD_ROTARY_HALF if layout == "half" else E.EBD_ROTARY_PAIRS
    y = E.ebd_norm_rotary(x, w, pos, tab, layout=lay)
    check_normed(y, x, w, pos, tab, layout, dtype)
    dx, dw = E.ebd_norm_rotary_backward(dy, x, w, pos, tab, layout=lay)
    check_grad(dx, dw, dy, x, w, pos, tab, layout, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128, 512])
def test_append_of_rows_up_to_the_largest_value(E, dtype, d):
    x, _, w, pos, _ = large_rows(E, d, 0, dtype)
    T = x.shape[0]
    s = R.make([T], [T + 5], 3, 3, d, 16, dtype, d)
    pc = cache(E, s)
    q_out = torch.empty((T, 3, d), dtype=dtype, device="cuda")
    E.ebd_paged_append_norm(pc, x, s["v"], k_weight=w, q=x, q_weight=w, q_out=q_out,
                            cu_new=s["cu"])
    _, at, off = slots_of(s, [T], [T + 5], 16)
    check_normed(q_out, x, w, None, None, "half", dtype)
    assert torch.equal(s["K"][at, :, off], q_out) and pc.dev_status.item() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("eps", [2.0 ** -126, 3e-38, 1e-35, 2.0 ** -102 * (1 - 2.0 ** -23), 2.0 ** -102,
                                 1e-30, 1e-20])
@pytest.mark.parametrize("d,rot,per_head", [(64, 64, False), (128, 32, True), (80, 20, False),
                                            (512, 0, False)])
def test_norm_of_small_rows_beside_a_small_eps(E, dtype, eps, d, rot, per_head):
    """Squares below the smallest normal float32 count where eps is as small.  (From 2^-102 on
    what they could add changes r by at most 2^-25, half a u.)"""
    root = eps ** 0.5
    sizes = [0.3 * root, root, 3 * root, 100 * root, 2.0 ** -31, 2.0 ** -29, 1.0, 30 * root]
    if eps < 1e-37:
        sizes += [1e-39, 2e-38]  # (r is so large that these count too)
    x, dy, w, pos = norm_inputs(len(sizes) + 1, 3, d, dtype, per_head, d)
    x[:-1] = sized_rows(x[:-1], sizes)
    x[-1] = 0
    x = x.contiguous()
    tab = table_of(E, rot, 4000) if rot else None
    y = E.ebd_norm_rotary(x, w, pos, tab, eps=eps)
    check_normed(y, x, w, pos, tab, "half", dtype, eps)
    dx, dw = E.ebd_norm_rotary_backward(dy, x, w, pos, tab, eps=eps)
    check_grad(dx, dw, dy, x, w, pos, tab, "half", dtype, eps)
    T = x.shape[0]
    s = R.make([T], [T + 5], 3, 3, d, 16, dtype, d)
    _, at, off = slots_of(s, [T], [T + 5], 16)
    E.ebd_paged_append_norm(cache(E, s), x, s["v"], k_weight=w, cu_new=s["cu"], positions=pos,
                            table=tab, eps=eps)
    assert torch.equal(s["K"][at, :, off], y)


def test_more_rows_than_31_bits_count_are_refused(E):
    """By the marshalling, before anything is launched: a Python error (the tensors here are
    views of one row)."""
    x = torch.zeros((1, 1, 8), device="cuda").to(torch.bfloat16)
    w, dw = torch.ones(8, device="cuda").to(torch.bfloat16), torch.empty(8, device="cuda")
    for shape in ((2 ** 31 + 8, 1, 8), (1, 2 ** 31 + 8, 8)):
        z = x.expand(shape)
        with pytest.raises(ValueError, match="out of range"):
            E.ebd_norm_rotary(z, w, out=z)
        with pytest.raises(ValueError, match="out of range"):
            E.ebd_norm_rotary_backward(z, z, w, dx=z, dweight=dw)


def test_norm_of_more_chunks_than_31_bits_count(E):
    """2^28 heads of one token (69 GB out, from views of a few rows): units of work, offsets and
    heads in 64 bits where they need them."""
    H, d, n = 2 ** 28 + 3, 128, 4
    x, _, w, _ = norm_inputs(1, n, d, torch.bfloat16, False, 31)
    want = E.ebd_norm_rotary(x, w)
    check_normed(want, x, w, None, None, "half", torch.bfloat16)
    got = torch.empty((1, H, d), dtype=torch.bfloat16, device="cuda")
    E.ebd_norm_rotary(x[:, :1].expand(1, H, d), w, out=got)
    for part in got[0].split(1 << 23):
        assert torch.equal(part, want[0, :1].expand(part.shape))
    del got, part
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- causal tokens after a deal
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", [0, 3, 4, 5, 8, 10])
@pytest.mark.parametrize("window", [0, 9])
def test_attention_without_a_mask_is_the_causal_one(E, dtype, case, window):
    """Bit for bit; empty places behind the last sequence stay, and nothing is reported."""
    s = tree_case(E, case, dtype)
    pc, T = cache(E, s), s["T"]
    want = E.ebd_paged_attention(s["q"], pc, s["cu"], s["max_new"], window=window)
    got = E.ebd_paged_tree_attention(s["q"], pc, s["cu"], s["max_new"], None, window=window)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    q = torch.cat([s["q"], torch.full_like(s["q"][:7], math.nan)])
    y, lse = torch.full_like(q, 3), torch.full(q.shape[:2], 4.0, device="cuda")
    E.ebd_paged_tree_attention(q, pc, s["cu"], s["max_new"], None, window=window, y=y, lse=lse)
    assert torch.equal(y[:T], want[0]) and torch.equal(lse[:T], want[1])
    assert (y[T:] == 3).all() and (lse[T:] == 4).all() and pc.dev_status.item() == 0
    # offsets that step back, or past the packed tokens, are still told
    cu = s["cu"].clone()
    cu[-1] = T + 8
    E.ebd_paged_tree_attention(q, pc, cu, s["max_new"] + 8, None, window=window, y=y, lse=lse)
    assert pc.dev_status.item() == E.EBD_DEV_RANGE
    with pytest.raises(ValueError, match="word"):  # an empty mask is none
        E.ebd_paged_tree_attention(s["q"], pc, s["cu"], s["max_new"], s["mask"][:, :0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_dealt_prompts_and_steps_are_attended_without_a_status(E, dtype):
    """Requests that idle, leave or wait for pages leave empty places; prompts longer than any
    tree.  The same tokens packed tightly give the same bits."""
    B, hkv, hq, d, P, cap = 4, 2, 4, 64, 16, 2600
    pc = E.alloc_paged(B, hkv, 160, P, d, 130, dtype, "cuda")
    pc.K_pages.zero_()
    pc.V_pages.zero_()
    pool = E.alloc_page_pool(B, 160, "cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    tab = table_of(E, d, 2100)
    for new, served_want in [([1500, 3, 0, 900], [1, 1, 1, 1]), ([1, 1, 40, 0], [1, 1, 1, 1]),
                             ([0, -1, 1, 1], [1, 1, 1, 1]), ([1, 700, 1, 1], [1, 0, 1, 1])]:
        cu, pos, slots, served = E.ebd_paged_deal(pool, pc, ints(new), cap)
        assert served.tolist() == served_want
        short = 0 in served_want
        assert pc.dev_status.item() == (E.EBD_DEV_CAPACITY if short else 0)
        pc.dev_status.zero_()
        qkv = torch.randn((cap, hq + 2 * hkv, d), generator=gen, device="cuda").to(dtype)
        q_out = torch.full((cap, hq, d), 2.0, dtype=dtype, device="cuda")
        E.ebd_paged_append_norm(pc, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], q=qkv[:, :hq],
                                q_out=q_out, slots=slots, positions=pos, table=tab)
        y, lse = E.ebd_paged_tree_attention(q_out, pc, cu, max(new), None)
        assert pc.dev_status.item() == 0
        n = cu[-1].item()
        want = E.ebd_paged_attention(q_out[:n], pc, cu, max(new))
        assert torch.equal(y[:n], want[0]) and torch.equal(lse[:n], want[1])
        assert pc.dev_status.item() == 0


def test_append_refuses_what_it_would_ignore(E):
    s = R.make([3], [9], 4, 2, 64, 16, torch.bfloat16, 3)
    pc, w = cache(E, s), torch.ones(64, device="cuda").to(torch.bfloat16)
    K0 = s["K"].clone()
    for kw in (dict(q_weight=w), dict(q_out=torch.empty_like(s["q"])),
               dict(q_weight=w, q_out=torch.empty_like(s["q"]))):
        with pytest.raises(ValueError, match="without q"):
            E.ebd_paged_append_norm(pc, s["k"], s["v"], k_weight=w, cu_new=s["cu"], **kw)
    assert torch.equal(s["K"], K0)


def test_a_step_without_tokens(E):
    """Every call of a step in which no request has a token: nothing happens, nothing is
    refused, lengths stay."""
    s = tree_case(E, 3, torch.bfloat16)
    pc = cache(E, s)
    K0, none = s["K"].clone(), ints([0] * 5)
    pool = E.alloc_page_pool(4, s["K"].shape[0], "cuda")
    pool.held.copy_(ints([[0, 1], [0, 1], [0, 2], [0, 1]]))
    cu, pos, slots, served = E.ebd_paged_deal(pool, pc, none[:4], 0)
    assert cu.tolist() == [0] * 5 and served.tolist() == [1] * 4 and pos.shape == (0,)
    mask, tpos = E.ebd_tree_masks(s["parents"][:0], cu, pc.seq_len, 0)
    assert mask.shape == (0, 0) and tpos.shape == (0,)
    w = torch.ones(128, device="cuda").to(torch.bfloat16)
    q = torch.empty_like(s["q"][:0])
    E.ebd_paged_append_norm(pc, s["k"][:0], s["v"][:0], k_weight=w, q=q, q_weight=w, q_out=q,
                            slots=slots, positions=pos)
    for m in (mask, None):
        y, lse = E.ebd_paged_tree_attention(q, pc, cu, 0, m, positions=tpos, window=7)
        assert y.shape == q.shape and lse.shape == q.shape[:2]
    got = E.ebd_paged_keep(pc, cu, ints([[0]] * 4), none[:4])
    assert got.tolist() == s["total"] and pc.dev_status.item() == 0 and torch.equal(s["K"], K0)


# ---------------------------------------------------------------- a deal that cannot serve
def test_unserved_sequences_give_back_what_is_behind_their_window(E):
    """Length, end block and table entries stay; the blocks behind the window are given back,
    and others may be dealt them in the same call."""
    P, window, n_pages = 8, 20, 10
    pool, pc = fresh_pool(E, 2, n_pages, P, 12)
    free, table = list(range(n_pages)), [[0] * 12, [0] * 12]
    length, held = [0, 0], [[0, 0], [0, 0]]
    for new, want in [([48, 0], [1, 1]), ([0, 8], [1, 1]), ([1, 60], [1, 0]), ([3, 9], [1, 1]),
                      ([70, 8], [0, 1]), ([8, 0], [1, 1]), ([36, 0], [0, 1]),
                      ([0, 1], [1, 1])]:
        cu, pos, slots, served = E.ebd_paged_deal(pool, pc, ints(new), 100, window=window)
        length, held, cu_r, served_r, pos_r, slots_r = S.deal(P, n_pages, 12, 100, window, new,
                                                              length, held, free, table)
        assert served.tolist() == served_r == want
        assert pc.seq_len.tolist() == length and pool.held.tolist() == held
        assert pc.block_table.tolist() == table and slots.tolist() == slots_r
        n = pool.n_free.item()
        assert pool.free_pages[:n].tolist() == free and cu.tolist() == cu_r
        out = [p for b in range(2) for p in table[b][held[b][0]:held[b][1]]]
        assert sorted(out + free) == list(range(n_pages))


# ---------------------------------------------------------------- where the forms change
@pytest.mark.parametrize("B,n_tokens", [(1, 4096), (256, 4097), (257, 257), (512, 4096), (513, 600),
                                        (1024, 4096), (1025, 2000)])
def test_deal_at_the_ends_of_its_forms(E, B, n_tokens):
    run_steps(E, B, 6 * B, 8, 30, n_tokens, 0, [lambda r, n: r.choice([0, 1, 2, 5, -1])] * 3, B)


@pytest.mark.parametrize("T,H,d,dtype,per_head", [
    (16, 32, 128, torch.bfloat16, False), (17, 32, 128, torch.bfloat16, False),  # 128, 136 steps
    (512, 4, 64, torch.float32, True), (513, 4, 64, torch.float32, True),        # 128, 129
    (36, 28, 128, torch.bfloat16, False), (1021, 4, 64, torch.float32, True)])   # 252, 256
def test_norm_gradient_at_the_ends_of_its_forms(E, T, H, d, dtype, per_head):
    x, dy, w, pos = norm_inputs(T, H, d, dtype, per_head, T)
    tab = table_of(E, d, 4000)
    dx, dw = E.ebd_norm_rotary_backward(dy, x, w, pos, tab)
    check_grad(dx, dw, dy, x, w, pos, tab, "half", dtype)
    again = E.ebd_norm_rotary_backward(dy, x, w, pos, tab)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
