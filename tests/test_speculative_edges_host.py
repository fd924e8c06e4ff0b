"""Refusals of the speculative calls' marshalling, host only: tensors without memory stand
for those of a GPU."""
import ctypes

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode


@pytest.fixture(scope="module")
def E():
    from paper_2607_21475_gb300.build import build
    build()
    from paper_2607_21475_gb300 import ebd
    return ebd


def on_gpu(*shape, dtype=torch.bfloat16, device="cuda:0"):
    """A tensor that says it is on that GPU; an address is not to be had from it."""
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device=device)


@pytest.mark.parametrize("shape", [(2 ** 31, 1, 1), (1, 2 ** 31, 1), (1, 1, 2 ** 31)])
def test_sizes_past_31_bits_are_refused(E, shape):
    x, w = on_gpu(*shape), on_gpu(shape[2])
    with pytest.raises(ValueError, match="out of range"):
        E.ebd_norm_rotary(x, w, out=x)
    with pytest.raises(ValueError, match="out of range"):
        E.ebd_norm_rotary_backward(x, x, w, dx=x, dweight=on_gpu(shape[2], dtype=torch.float32))


def calls(E):
    """Every call with all its tensors given: (function, arguments by name)."""
    def i32(*shape):
        return on_gpu(*shape, dtype=torch.int32)

    def f32(*shape):
        return on_gpu(*shape, dtype=torch.float32)

    T, B, hq, hkv, d, pages, P = 5, 2, 4, 2, 64, 8, 16
    cache = dict(K_pages=on_gpu(pages, hkv, P, d), V_pages=on_gpu(pages, hkv, P, d),
                 block_table=i32(B, 4), seq_len=i32(B), dev_status=i32(1))
    turn = dict(positions=i32(T), table=f32(50, d // 2, 2))
    pool = dict(free_pages=i32(pages), n_free=i32(1), held=i32(B, 2))

    def on_cache(f):
        return lambda **a: f(pc=E.PagedCache(*(a.pop(k) for k in cache)), **a)

    def deal(**a):
        return E.ebd_paged_deal(E.PagePool(*(a.pop(k) for k in pool)),
                                E.PagedCache(*(a.pop(k) for k in cache)), n_tokens=T, **a)

    return [
        (deal, dict(**pool, **cache, n_new=i32(B), cu_new=i32(B + 1), positions=i32(T),
                    slots=on_gpu(T, dtype=torch.int64), served=i32(B), seq_len_out=i32(B),
                    held_out=i32(B, 2), n_free_out=i32(1))),
        (E.ebd_norm_rotary, dict(x=on_gpu(T, hq, d), weight=on_gpu(d), **turn, out=on_gpu(T, hq, d),
                                 dev_status=i32(1))),
        (E.ebd_norm_rotary_backward, dict(
            dy=on_gpu(T, hq, d), x=on_gpu(T, hq, d), weight=on_gpu(d), **turn, dx=on_gpu(T, hq, d),
            dweight=f32(d), workspace=f32(1 << 20), dev_status=i32(1))),
        (on_cache(E.ebd_paged_append_norm), dict(
            **cache, k_new=on_gpu(T, hkv, d), v_new=on_gpu(T, hkv, d), k_weight=on_gpu(d),
            q=on_gpu(T, hq, d), q_weight=on_gpu(d), q_out=on_gpu(T, hq, d), cu_new=i32(B + 1),
            **turn)),
        (E.ebd_tree_masks, dict(parents=i32(T), cu_new=i32(B + 1), seq_len=i32(B), max_new=T,
                                mask=i32(T, 1), positions=i32(T), dev_status=i32(1))),
        (on_cache(E.ebd_paged_tree_attention), dict(**cache, q=on_gpu(T, hq, d), cu_new=i32(B + 1), max_new=T,
                                                mask=i32(T, 1), positions=i32(T),
                                                y=on_gpu(T, hq, d), lse=f32(T, hq),
                                                workspace=f32(1 << 20))),
        (on_cache(E.ebd_paged_keep), dict(**cache, cu_new=i32(B + 1), path=i32(B, 3), n_accepted=i32(B),
                                 seq_len_out=i32(B))),
    ]


@pytest.mark.skipif(torch.cuda.device_count() == 1,
                    reason="beside one GPU no tensor says that it is on a second")
@pytest.mark.parametrize("which", range(7))
def test_tensors_of_two_gpus_are_refused(E, which):
    """Whichever of them is elsewhere: the kernels would take its address as this GPU's."""
    call, args = calls(E)[which]
    for name, t in args.items():
        if not isinstance(t, torch.Tensor):
            continue
        elsewhere = on_gpu(*t.shape, dtype=t.dtype, device="cuda:1")
        with pytest.raises(ValueError, match="is on cuda:"):
            call(**dict(args, **{name: elsewhere}))


def test_append_refuses_what_it_would_ignore(E):
    """Queries' weight or place without queries: a slip that went unseen."""
    call, args = calls(E)[3]
    for left in ("q_weight", "q_out"):
        a = {k: v for k, v in args.items() if k == left or k not in ("q", "q_weight", "q_out")}
        with pytest.raises(ValueError, match="without q"):
            call(**a)


def test_a_step_without_tokens_needs_no_mask(E):
    """max_new 0, a mask of no words: the largest number of new tokens of no sequence."""
    from test_speculative_host import FAKE, good_cache
    L, c = E.lib(), good_cache(E)
    masks = dict(B=2, T=0, most=0, parents=None, cu=FAKE, len=FAKE, window=0, mask=None, words=0,
                 pos=None, st=None, stream=None)
    attend = dict(c=ctypes.byref(c), n=0, most=0, hq=2, cu=FAKE, q=None, qt=128, qh=64, scale=0.1,
                  window=4, mask=FAKE, words=0, pos=None, y=None, lse=None, st=FAKE, ws=None, wsb=0,
                  stream=None)
    for f, a, some in ((L.ebd_tree_masks, masks, dict(T=1, most=1)),
                       (L.ebd_paged_tree_attention, attend, dict(n=1, most=1))):
        assert f(*a.values()) == E.EBD_OK
        for bad in (dict(words=-1), dict(most=-1), dict(most=1), some):
            assert f(*dict(a, **bad).values()) == 1, bad


def test_more_heads_than_31_bits_count_are_refused(E):
    from test_speculative_host import FAKE, NORM, good_cache
    L, most = E.lib(), 0x3fff0000
    for h in (most + 1, 2 ** 31 - 1):
        assert L.ebd_norm_rotary(*dict(NORM, H=h).values()) == 4
    assert L.ebd_norm_rotary(*dict(NORM, H=most, T=0).values()) == E.EBD_OK
    c = good_cache(E)
    a = dict(c=ctypes.byref(c), T=0, cu=FAKE, slots=None, pos=None, k=FAKE, kt=128, kh=64, v=FAKE,
             vt=128, vh=64, kw=FAKE, kwh=0, qw=FAKE, qwh=0, wt=1, eps=1e-6, table=None, n_pos=0,
             rot=0, layout=0, hq=most - 3, q=FAKE, qt=128, qh=64, o=FAKE, ot=128, oh=64, st=FAKE,
             stream=None)
    assert L.ebd_paged_append_norm(*a.values()) == 4
    assert L.ebd_paged_append_norm(*dict(a, hq=most - 4).values()) == E.EBD_OK


def test_the_library_is_linked_where_the_binding_does_not_compile(monkeypatch, tmp_path):
    """And the binding of other sources does not stay beside it."""
    from paper_2607_21475_gb300 import build as B
    src = tmp_path / "one.cu"
    src.write_text('extern "C" int one() { return 1; }\n')
    binding = tmp_path / "binding.cpp"
    binding.write_text("#error not here\n")
    (tmp_path / "ebd_call.so").write_text("an older one")
    for name, value in dict(BUILD=str(tmp_path), LIB=str(tmp_path / "libebd.so"),
                            CALL=str(tmp_path / "ebd_call.so"), BINDING=str(binding),
                            _sources=lambda: [str(src)]).items():
        monkeypatch.setattr(B, name, value)
    for how in ("sources", "compiler", "torch"):
        if how == "compiler":
            monkeypatch.setenv("CXX", str(tmp_path / "no-such-compiler"))
        if how == "torch":
            monkeypatch.setattr(B, "_torch_root", lambda: None)
        with pytest.raises(RuntimeError, match="is built"):
            B.build()
        assert ctypes.CDLL(B.LIB).one() == 1
        assert not (tmp_path / "ebd_call.so").exists()
        (tmp_path / "libebd.so").unlink()


CLUSTERS = r"""
#include "cluster.h"
static ebd::ClusterMemo memo;
static int asked = 0;
extern "C" int choose(int want, int device, int active) {
  return ebd::cluster_ctas(want, memo, device, [&] { ++asked; return active; });
}
extern "C" int times_asked() { return asked; }
"""


def test_clusters_fall_back_to_eight(tmp_path):
    """A GPU that holds no cluster of sixteen, told by a fake of the question: eight are asked
    for; the question is put once per device."""
    import os
    import subprocess

    from paper_2607_21475_gb300 import build as B
    (tmp_path / "c.cpp").write_text(CLUSTERS)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-fPIC", "-shared", "-I", B.CSRC,
                    str(tmp_path / "c.cpp"), "-o", str(tmp_path / "c.so")], check=True)
    L = ctypes.CDLL(str(tmp_path / "c.so"))
    assert [L.choose(n, 0, 0) for n in (1, 7, 8)] == [1, 7, 8] and L.times_asked() == 0
    assert [L.choose(n, 0, 9) for n in (9, 16)] == [9, 16] and L.times_asked() == 1
    assert [L.choose(n, 1, 0) for n in (9, 16, 8, 3)] == [8, 8, 8, 3] and L.times_asked() == 2
    assert L.choose(16, 0, 0) == 16 and L.choose(16, 1, 9) == 8 and L.times_asked() == 2
    assert [L.choose(16, d, 9) for d in (-1, 64)] == [8, 8] and L.times_asked() == 2
