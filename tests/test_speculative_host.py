"""Host-only checks of a speculative step's entry points: refusals (synchronous, no kernel
is launched) and the plain forms that the GPU tests compare with."""
import ctypes
import math
import random

import pytest
import torch

import speculative_ref as S

FAKE = 0x1000  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def E():
    from paper_2607_21475_gb300.build import build
    build()
    from paper_2607_21475_gb300 import ebd
    return ebd


def good_cache(E, **kw):
    f = dict(dtype=1, batch=2, n_kv_heads=2, head_dim=64, page_size=16, n_pages=10, max_blocks=4,
             reserved=0, page_stride=2048, head_stride=1024, row_stride=64, K_pages=FAKE,
             V_pages=FAKE, block_table=FAKE, seq_len=FAKE)
    f.update(kw)
    return E.EbdPagedCache(*f.values())


def run(good, call, cases):
    for kw, code in cases:
        a = dict(good)
        assert set(kw) <= set(a), kw
        a.update(kw)
        assert call(*a.values()) == code, kw


def test_deal_refusals(E):
    a = dict(B=2, page=16, pages=10, blocks=4, n=5, window=0, new=FAKE, len=FAKE, held=FAKE,
             free=FAKE, list=FAKE, bt=FAKE, len_out=FAKE, held_out=FAKE, free_out=FAKE, cu=FAKE,
             served=None, pos=None, slots=None, st=FAKE, stream=None)
    run(a, E.lib().ebd_paged_deal, [
        (dict(B=0), 1), (dict(pages=0), 1), (dict(blocks=0), 1), (dict(n=-1), 1),
        (dict(window=-1), 1), (dict(page=24), 4), (dict(page=4), 4), (dict(page=2048), 4),
        (dict(blocks=1 << 28), 4), (dict(B=65536), 4), (dict(n=0x7fff0001), 4),
        (dict(pages=0x7fff0001), 4), (dict(len_out=FAKE + 4), 1),
        (dict(held_out=FAKE + 12), 1)] + [(dict([(k, None)]), 1) for k in (
            "new", "len", "held", "free", "list", "bt", "len_out", "held_out", "free_out", "cu",
            "st")])


NORM = dict(dtype=1, T=1, H=2, d=64, x=FAKE, xt=128, xh=64, w=FAKE, wt=1, wh=0, eps=1e-6, pos=FAKE,
            table=FAKE, n_pos=8, rot=64, layout=0, y=FAKE, yt=128, yh=64, st=None, stream=None)
NORM_BAD = [(dict(dtype=2), 1), (dict(T=-1), 1), (dict(T=0x7fffff01), 4), (dict(H=0), 1), (dict(d=0), 1), (dict(d=513), 4),
            (dict(x=None), 1), (dict(w=None), 1), (dict(wt=2), 1), (dict(dtype=0), 1),
            (dict(wh=-1), 1), (dict(eps=0.0), 1), (dict(eps=1e-39), 1), (dict(eps=-1.0), 1), (dict(eps=math.nan), 1),
            (dict(eps=math.inf), 1), (dict(pos=None), 1), (dict(table=FAKE + 4), 1),
            (dict(n_pos=0), 1), (dict(rot=0), 1), (dict(rot=3), 1), (dict(rot=66), 1),
            (dict(layout=2), 1), (dict(layout=1, xt=129), 4)]


def test_norm_refusals(E):
    L = E.lib()
    run(NORM, L.ebd_norm_rotary, NORM_BAD + [(dict(y=None), 1), (dict(T=0), 0)])
    need = 152 * 2 * 64 * 4
    back = {}
    for k, v in NORM.items():
        if k == "x":
            back.update(dy=FAKE, dyt=128, dyh=64)
        back[k] = v
        if k == "yh":
            back["dw"] = FAKE
        if k == "st":
            back.update(ws=FAKE, wsb=max(need, 1 << 20))
    run(back, L.ebd_norm_rotary_backward, NORM_BAD + [
        (dict(y=None), 1), (dict(dy=None), 1), (dict(dw=None), 1), (dict(ws=None), 1),
        (dict(ws=FAKE + 8), 1), (dict(wsb=0), 2), (dict(H=65536), 1),
        (dict(layout=1, dyt=129), 4)])
    assert L.ebd_norm_rotary_backward_workspace_bytes(0, 64, 0) == 0
    a, b = (L.ebd_norm_rotary_backward_workspace_bytes(4, 64, p) for p in (0, 1))
    assert a >= 256 and b >= 4 * 64 * 4


def test_append_norm_refusals(E):
    c = good_cache(E)
    a = dict(c=ctypes.byref(c), T=1, cu=FAKE, slots=None, pos=None, k=FAKE, kt=128, kh=64, v=FAKE,
             vt=128, vh=64, kw=FAKE, kwh=0, qw=FAKE, qwh=0, wt=1, eps=1e-6, table=FAKE, n_pos=8,
             rot=64, layout=0, hq=2, q=FAKE, qt=128, qh=64, o=FAKE, ot=128, oh=64, st=FAKE,
             stream=None)
    call = E.lib().ebd_paged_append_norm
    run(a, call, [
        (dict(T=-1), 1), (dict(cu=None), 1), (dict(slots=FAKE), 1), (dict(cu=None, slots=FAKE), 1),
        (dict(k=None), 1), (dict(v=None), 1), (dict(st=None), 1), (dict(kwh=-1), 1),
        (dict(qwh=-1), 1), (dict(wt=3), 1), (dict(eps=0.0), 1), (dict(table=FAKE + 4), 1),
        (dict(n_pos=0), 1), (dict(rot=66), 1), (dict(layout=7), 1), (dict(hq=-1), 1),
        (dict(q=None), 1), (dict(o=None), 1), (dict(table=None, qw=None), 1),
        (dict(layout=1, kt=129), 4), (dict(T=0), 0)])
    for bad, code in [(dict(dtype=2), 1), (dict(page_size=24), 4), (dict(K_pages=None), 1),
                      (dict(head_dim=520, row_stride=520, head_stride=8320, page_stride=16640), 4)]:
        a["c"] = ctypes.byref(good_cache(E, **bad))
        assert call(*a.values()) == code, bad


def test_tree_refusals(E):
    a = dict(B=2, T=4, most=4, parents=FAKE, cu=FAKE, len=FAKE, window=0, mask=FAKE, words=1,
             pos=FAKE, st=None, stream=None)
    run(a, E.lib().ebd_tree_masks, [
        (dict(B=0), 1), (dict(T=-1), 1), (dict(most=0), 1), (dict(most=33), 1), (dict(words=0), 1),
        (dict(window=-1), 1), (dict(most=1025, words=33), 4), (dict(words=33), 4),
        (dict(B=65536), 4), (dict(parents=None), 1), (dict(cu=None), 1), (dict(len=None), 1),
        (dict(mask=None), 1), (dict(pos=None), 1), (dict(T=0, most=0), 0)])
    c = good_cache(E)
    a = dict(c=ctypes.byref(c), n=1, most=1, hq=2, cu=FAKE, q=FAKE, qt=128, qh=64, scale=0.1,
             window=0, mask=FAKE, words=1, pos=None, y=FAKE, lse=None, st=FAKE, ws=FAKE,
             wsb=1 << 40, stream=None)
    run(a, E.lib().ebd_paged_tree_attention, [
        (dict(c=None), 1), (dict(n=-1), 1), (dict(most=0), 1), (dict(most=33), 1),
        (dict(words=0), 1), (dict(mask=None), 1), (dict(window=5), 1), (dict(window=-1), 1),
        (dict(hq=3), 1), (dict(hq=0), 1), (dict(cu=None), 1), (dict(q=None), 1), (dict(y=None), 1),
        (dict(st=None), 1), (dict(scale=0.0), 1), (dict(q=FAKE + 8), 1), (dict(qt=129), 1),
        (dict(hq=258), 4), (dict(n=0), 0)])
    a = dict(c=ctypes.byref(c), layers=1, stride=0, cu=FAKE, path=FAKE, most=4, n=FAKE,
             len=FAKE + 64, st=FAKE, stream=None)
    call = E.lib().ebd_paged_keep
    run(a, call, [
        (dict(c=None), 1), (dict(layers=0), 1), (dict(layers=2), 1), (dict(layers=2, stride=4), 1),
        (dict(layers=65536, stride=8), 4), (dict(cu=None), 1), (dict(path=None), 1),
        (dict(most=0), 1), (dict(n=None), 1), (dict(len=FAKE), 1), (dict(len=FAKE + 4), 1),
        (dict(st=None), 1)])
    for bad, code in [(dict(head_dim=20, row_stride=24), 4), (dict(row_stride=68), 1),
                      (dict(K_pages=FAKE + 8), 1)]:
        a["c"] = ctypes.byref(good_cache(E, **bad))
        assert call(*a.values()) == code, bad


def test_binding_is_bound_to_every_entry_point(E):
    m = E._call()
    with pytest.raises(RuntimeError, match="address"):
        m.bind({})
    with pytest.raises(TypeError, match="arguments"):
        m.keep(1, 2)


def test_python_refusals(E):
    x, w = torch.zeros(2, 2, 64), torch.zeros(64)
    pc = E.alloc_paged(2, 2, 8, 16, 64, 4, torch.float32, "cpu")
    for call in [lambda: E.ebd_norm_rotary(x[0], w), lambda: E.ebd_norm_rotary(x, w),
                 lambda: E.ebd_norm_rotary_backward(x, x, w),
                 lambda: E.ebd_paged_append_norm(pc, x, x, cu_new=torch.zeros(3).int()),
                 lambda: E.ebd_paged_deal(E.alloc_page_pool(2, 8, "cpu"), pc, torch.zeros(2), 4),
                 lambda: E.ebd_tree_masks(torch.zeros(2, 2), torch.zeros(3).int(),
                                          torch.zeros(2).int(), 4),
                 lambda: E.ebd_paged_tree_attention(x, pc, torch.zeros(3).int(), 1,
                                                    torch.zeros(2, 1).int()),
                 lambda: E.ebd_paged_keep(pc, torch.zeros(3).int(), torch.zeros(2, 1).int(),
                                          torch.zeros(2).int())]:
        with pytest.raises((ValueError, RuntimeError)):
            call()


# ---------------------------------------------------------------- the plain forms
def test_plain_deal_keeps_every_page():
    rng = random.Random(1)
    B, P, pages, blocks = 6, 8, 40, 9
    free, table = list(range(pages)), [[-1] * blocks for _ in range(B)]
    length, held = [0] * B, [[0, 0]] * B
    for _ in range(50):
        new = [rng.choice([0, 1, 1, 9, 20, -1]) for _ in range(B)]
        before = list(length)
        length, held, cu, served, pos, slots = S.deal(P, pages, blocks, 60, 30, new, length, held,
                                                      free, table)
        out = [p for b in range(B) for p in table[b][held[b][0]:held[b][1]]]
        assert sorted(out + free) == list(range(pages))
        for b in range(B):
            want = 0 if new[b] < 0 else before[b] + (new[b] if served[b] else 0)
            assert length[b] == want and cu[b + 1] - cu[b] == max(0, length[b] - before[b])
            for t in range(cu[b], cu[b + 1]):
                assert slots[t] == table[b][pos[t] // P] * P + pos[t] % P
            if length[b]:  # what a next token may see is held
                assert held[b][0] * P <= max(0, before[b] - 29) and held[b][1] * P >= length[b]


def test_plain_norm_gradient_matches_differences():
    g = torch.Generator().manual_seed(2)
    x, dy = (torch.randn((2, 3, 10), generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.randn(10, generator=g, dtype=torch.float64)
    a = torch.rand((2, 3), generator=g, dtype=torch.float64) * 6
    cs = torch.stack([a.cos(), a.sin()], -1) * 1.3
    import paged_ref as R
    for layout in ("half", "pairs"):
        dx, dw, ax, aw = S.norm_grad(dy, x, w, 1e-3, cs, layout)
        x_, w_ = x.clone().requires_grad_(), w.clone().requires_grad_()
        y = R.rotate(S.norm(x_, w_, 1e-3), cs, layout)
        gx, gw = torch.autograd.grad((dy * y).sum(), (x_, w_))
        assert torch.allclose(dx, gx, atol=1e-12) and torch.allclose(dw.sum((0, 1)), gw, atol=1e-12)
        assert (ax >= dx.abs() - 1e-12).all() and (aw >= dw.abs() - 1e-12).all()
        h = 1e-5
        for i in [(0, 0, 0), (1, 2, 7)]:
            e = torch.zeros_like(x)
            e[i] = h
            up, down = ((dy * R.rotate(S.norm(x + s * e, w, 1e-3), cs, layout)).sum()
                        for s in (1, -1))
            assert abs((up - down) / (2 * h) - dx[i]) < 1e-8


def test_plain_masks_of_a_small_tree():
    parents, cu, total = [-1, 0, 0, 2, -1, 4, -1, 0], [0, 6, 8], [16, 2]
    mask, pos = S.masks(parents, cu, total, 1)
    assert mask[:, 0].tolist() == [1, 3, 5, 13, 16, 48, 1, 3]
    assert pos.tolist() == [10, 11, 11, 12, 10, 11, 0, 1]
    mask, _ = S.masks(parents, cu, total, 1, window=2)
    assert mask[:, 0].tolist() == [1, 3, 5, 12, 16, 48, 1, 3]
    seen = S.tree_seen(mask, pos, cu, total, window=4)
    assert seen[0][3].nonzero().flatten().tolist() == [9, 12, 13]
