"""Host-only checks of the paged-cache entry points: refusals (synchronous, no
kernel is launched), the struct's layout, and the frequency scalings."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    from paper_2607_21475_gb300.build import build
    build()
    from paper_2607_21475_gb300 import ebd
    return ebd


def test_struct_layout_matches_c(tmp_path, E):
    names = [n for n, _ in E.EbdPagedCache._fields_]
    prog = tmp_path / "layout.c"
    prog.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ebd.h"\nint main(void){'
                    'printf("%zu", sizeof(ebd_paged_cache));' +
                    "".join(f'printf(" %zu", offsetof(ebd_paged_cache, {n}));' for n in names) +
                    "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)],
                   check=True)
    got = list(map(int, subprocess.run([str(exe)], capture_output=True, text=True,
                                       check=True).stdout.split()))
    assert got == [ctypes.sizeof(E.EbdPagedCache)] + [getattr(E.EbdPagedCache, n).offset
                                                      for n in names]


FAKE = 0x1000  # never dereferenced: validation fails first


def good_cache(E, **kw):
    f = dict(dtype=1, batch=2, n_kv_heads=2, head_dim=64, page_size=16, n_pages=10, max_blocks=4,
             reserved=0, page_stride=2048, head_stride=1024, row_stride=64, K_pages=FAKE,
             V_pages=FAKE, block_table=FAKE, seq_len=FAKE)
    f.update(kw)
    return E.EbdPagedCache(*f.values())


def append(E, c, **kw):
    a = dict(n=1, cu=FAKE, k=FAKE, kt=128, kh=64, v=FAKE, vt=128, vh=64, table=FAKE, n_pos=8,
             rot=64, layout=0, hq=2, q=FAKE, qt=128, qh=64, o=FAKE, ot=128, oh=64, st=FAKE)
    a.update(kw)
    return E.lib().ebd_paged_append(ctypes.byref(c) if c else None, *a.values(), None)


def attention(E, c, **kw):
    a = dict(n=1, max_new=1, hq=2, cu=FAKE, q=FAKE, qt=128, qh=64, scale=0.1, window=0, y=FAKE,
             lse=None, st=FAKE, ws=FAKE, wsb=1 << 40)
    a.update(kw)
    return E.lib().ebd_paged_attention(ctypes.byref(c) if c else None, *a.values(), None)


def gather(E, c, **kw):
    a = dict(idx=FAKE, n=FAKE, cap=4, k=FAKE, v=FAKE, st=FAKE)
    a.update(kw)
    return E.lib().ebd_paged_gather(ctypes.byref(c) if c else None, *a.values(), None)


@pytest.mark.parametrize("call", [append, attention, gather])
def test_bad_caches_are_refused(E, call):
    assert call(E, None) == 1
    for kw, code in [(dict(dtype=2), 1), (dict(batch=0), 1), (dict(n_kv_heads=0), 1),
                     (dict(head_dim=0), 1), (dict(n_pages=0), 1), (dict(max_blocks=0), 1),
                     (dict(page_size=4), 4), (dict(page_size=24), 4), (dict(page_size=2048), 4),
                     (dict(row_stride=63), 1), (dict(page_stride=-1), 1), (dict(page_stride=0), 1),
                     (dict(head_stride=0), 1), (dict(K_pages=None), 1),
                     (dict(V_pages=None), 1), (dict(block_table=None), 1), (dict(seq_len=None), 1),
                     (dict(page_size=1024, max_blocks=1 << 21), 4)]:
        assert call(E, good_cache(E, **kw)) == code, kw


def test_bad_arguments_are_refused(E):
    c = good_cache(E)
    for kw, code in [(dict(n=-1), 1), (dict(cu=None), 1), (dict(k=None), 1), (dict(v=None), 1),
                     (dict(st=None), 1), (dict(layout=2), 1), (dict(rot=3), 1), (dict(rot=66), 1),
                     (dict(rot=0), 1), (dict(n_pos=0), 1), (dict(table=FAKE + 4), 1),
                     (dict(table=None), 1), (dict(q=None), 1), (dict(o=None), 1),
                     (dict(hq=-1), 1), (dict(layout=1, kt=129), 4)]:
        assert append(E, c, **kw) == code, kw
    assert append(E, c, n=0) == 0
    for kw, code in [(dict(n=-1), 1), (dict(max_new=-1), 1), (dict(max_new=0), 1), (dict(hq=3), 1), (dict(hq=0), 1),
                     (dict(cu=None), 1), (dict(q=None), 1), (dict(y=None), 1), (dict(st=None), 1),
                     (dict(scale=0.0), 1), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1),
                     (dict(window=-1), 1), (dict(q=FAKE + 8), 1), (dict(qt=129), 1), (dict(qh=0), 1), (dict(qh=-64), 1),
                     (dict(qh=4), 1), (dict(y=FAKE + 2), 1), (dict(hq=2 * 129), 4)]:
        assert attention(E, c, **kw) == code, kw
    assert attention(E, c, n=0) == 0
    assert attention(E, good_cache(E, head_dim=96, row_stride=96)) == 4
    huge = good_cache(E, batch=60000, max_blocks=1 << 20)  # 16 M positions each
    assert attention(E, huge, n=60000) == 4
    assert attention(E, good_cache(E, row_stride=68)) == 1
    assert attention(E, good_cache(E, K_pages=FAKE + 8)) == 1
    for kw, code in [(dict(idx=None), 1), (dict(n=None), 1), (dict(cap=0), 1), (dict(k=None), 1),
                     (dict(v=None), 1), (dict(st=None), 1), (dict(k=FAKE + 8), 1)]:
        assert gather(E, c, **kw) == code, kw
    assert gather(E, good_cache(E, head_dim=20, row_stride=24)) == 4
    L = E.lib()
    assert L.ebd_rotary_table(None, 2, 2, 1.0, FAKE, None) == 1
    assert L.ebd_rotary_table(FAKE, 0, 2, 1.0, FAKE, None) == 1
    assert L.ebd_rotary_table(FAKE, 2, 2, 1.0, FAKE + 4, None) == 1
    rot = [1, 1, 1, 64, 64, 0, 0, FAKE, 64, 64, FAKE, FAKE, 8, FAKE, 64, 64, None, None]
    for i, bad, code in [(0, 3, 1), (1, -1, 1), (2, 0, 1), (3, 0, 1), (4, 65, 1), (4, 66, 1),
                         (5, 2, 1), (7, None, 1), (10, None, 1), (11, None, 1), (12, 0, 1),
                         (13, None, 1)]:
        x = list(rot)
        x[i] = bad
        assert L.ebd_rotary(*x) == code, (i, bad)
    rot[1] = 0
    assert L.ebd_rotary(*rot) == 0


def test_workspace_is_checked(E):
    c = good_cache(E, batch=4, max_blocks=512)
    need = E.lib().ebd_paged_attention_workspace_bytes(ctypes.byref(c), 4, 1)
    if need:
        assert attention(E, c, wsb=need - 1, hq=4) == 2
        assert attention(E, c, ws=None, hq=4) == 1


def test_python_refusals(E):
    pc = E.alloc_paged(2, 2, 8, 16, 64, 4, torch.float32, "cpu")
    with pytest.raises(ValueError, match="CUDA"):
        E.ebd_paged_append(pc, torch.zeros(1, 2, 64), torch.zeros(1, 2, 64),
                           torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        E.ebd_rotary(torch.zeros(2, 64), None, None)
    with pytest.raises(ValueError):
        E.rotary_frequencies(7)
    with pytest.raises(ValueError):
        E.rotary_frequencies(8, scaling="other")


def test_frequency_scalings(E):
    f, m = E.rotary_frequencies(64)
    assert m == 1.0 and f[0] == 1.0 and abs(f[16].item() - 0.01) < 1e-15
    g, m = E.rotary_frequencies(64, scaling="linear", factor=8.0)
    assert m == 1.0 and torch.equal(g, f / 8)
    g, m = E.rotary_frequencies(64, scaling="base", factor=8.0)
    assert g[0] == 1.0 and abs((f[-1] / g[-1]).item() - 8.0) < 1e-9 and (g <= f).all()
    g, m = E.rotary_frequencies(64, scaling="parts", factor=8.0, original_positions=4096)
    assert abs(m - (0.1 * math.log(8.0) + 1)) < 1e-15
    turns = f * 4096 / (2 * math.pi)
    assert torch.equal(g[turns > 34], f[turns > 34])
    assert torch.allclose(g[turns < 0.9], f[turns < 0.9] / 8, rtol=1e-12)
    mid = (turns < 30) & (turns > 1.2)
    assert (g[mid] < f[mid]).all() and (g[mid] > f[mid] / 8).all()


@pytest.mark.parametrize("rot,base,factor,positions", [
    (128, 1e4, 4.0, 131072),  # the ramp ends past the last pair
    (64, 1e4, 8.0, 131072),
    (64, 1e4, 8.0, 1 << 20),
    (128, 1e4, 4.0, 100),     # the ramp begins before the first pair
    (64, 1e4, 8.0, 4096),
    (2, 1e4, 8.0, 4096),
])
def test_parts_scaling_follows_its_rule_at_both_ends(E, rot, base, factor, positions):
    """A pair of at least fast_turns turns stays, one of at most slow_turns slows by the
    factor, and every pair in between lies on one line from the last index that stays to
    the first that slows in full, wherever these two lie.  Compared in float64 with
    indices found by counting turns one by one."""
    f, _ = E.rotary_frequencies(rot, base=base)
    g, _ = E.rotary_frequencies(rot, base=base, scaling="parts", factor=factor,
                                original_positions=positions)

    def turns(i):
        return base ** (-2.0 * i / rot) * positions / (2 * math.pi)

    lo = next(i for i in range(4 * rot, -4 * rot, -1) if turns(i) >= 32.0)
    hi = next(i for i in range(-4 * rot, 4 * rot) if turns(i) <= 1.0)
    for i in range(rot // 2):
        slow = min(max((i - lo) / (hi - lo), 0.0), 1.0)
        want = f[i].item() * (1 - slow + slow / factor)
        assert abs(g[i].item() - want) <= 1e-12 * f[i].item(), (i, turns(i))
        assert turns(i) < 32.0 or g[i] == f[i]
        assert turns(i) <= 1.0 or g[i] > f[i] / factor * (1 + 1e-9)


# ---------------------------------------------------------------- buffers of the binding
def test_no_entry_point_allocates_outside_its_stream(E):
    """A function that takes a stream makes its buffers and its tensors' copies through
    the helpers that order them on that stream, never with the current stream's pool."""
    import ast
    with open(E.__file__) as fh:
        tree = ast.parse(fh.read())
    makers = {"empty", "zeros", "ones", "full", "empty_like", "zeros_like", "to", "contiguous",
              "clone", "cuda", "float", "double"}
    found = []
    for fn in tree.body:
        if not isinstance(fn, ast.FunctionDef) or fn.name.startswith("_"):
            continue
        if "stream" not in [a.arg for a in fn.args.args]:
            continue
        for node in ast.walk(fn):
            if (isinstance(node, ast.Call) and isinstance(node.func, ast.Attribute)
                    and node.func.attr in makers):
                found.append((fn.name, node.func.attr))
    assert found == []


def test_workspace_is_taken_from_the_streams_pool(E, monkeypatch):
    """Allocation happens while the call's stream is the current one; without a stream
    the current one stays."""
    entered, made = [], []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            entered.append(self.stream)

        def __exit__(self, *exc):
            entered.pop()

    def empty(*shape, **kw):
        made.append(list(entered))
        return real(*shape, **kw)

    real = torch.empty
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch, "empty", empty)
    _, n = E._workspace(256, "cpu", None, "side")
    assert n == 256 and made == [["side"]]
    E._workspace(256, "cpu", None, None)
    assert made == [["side"], []]
    ws = real(300, dtype=torch.uint8)
    assert E._workspace(256, "cpu", ws, "side") == (ws.data_ptr(), 300) and len(made) == 2
    with pytest.raises(ValueError, match="too small"):
        E._workspace(301, "cpu", ws, "side")


# ---------------------------------------------------------------- the tests' own bound
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,hq,n", [(64, 1, 5003), (128, 1, 5003), (128, 8, 30000)])
def test_attention_bound_sees_one_wrong_value_tile(dtype, d, hq, n):
    """A 64-key value tile that is zeros, or another tile's, goes past the bound of the
    attention tests at any place of a long context; exact results with rounded weights
    and outputs do not."""
    import paged_ref as R
    g = torch.Generator().manual_seed(7)
    page = 64
    blocks = -(-n // page)
    K, V = (torch.randn((blocks, 1, page, d), generator=g).to(dtype) for _ in range(2))
    q = torch.randn((1, hq, d), generator=g).to(dtype)
    bt, cu = torch.arange(blocks).int()[None], [0, 1]
    y, lse, mean, root = R.attention_detail(q, K, V, bt, [n], cu, d ** -0.5, 0)
    bound = R.attention_bound(y, mean, root, dtype)
    k, v = R.rows(K, bt, 0, 0, n), R.rows(V, bt, 0, 0, n)
    p = ((q[0].double() @ k.T) * d ** -0.5 - lse[0][:, None]).exp()
    for block in range(blocks - 1):
        at = slice(block * page, (block + 1) * page)
        for wrong in (torch.zeros_like(v[at]), V[(block + 5) % (blocks - 1), 0].double()):
            assert ((p[:, at] @ (wrong - v[at])).abs() > bound[0]).any(), block
    w = p.to(dtype).double()
    assert (((w @ v).to(dtype).double() - y[0]).abs() <= bound[0]).all()
