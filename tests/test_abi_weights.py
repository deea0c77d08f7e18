"""Refusals of the weight, eviction and tree calls: checked on the host before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2412_12706_b200 import build as qp_build
from paper_2412_12706_b200 import qp

A = 0x1000   # aligned, never dereferenced
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    qp_build.build()
    return qp.lib()


def cache(bits=16, n=64, cap=0, D=128, Hq=8, Hkv=2, g=32):
    c = qp.cache_layout_cap(1, Hq, Hkv, D, bits, g, n, cap)
    c.k_codes = c.v_codes = A
    if bits < 16:
        c.k_scale = c.k_zero = c.v_scale = c.v_zero = A
    return c


def strategy(axis, thr=0.0):
    s = qp.qp_strategy()
    s.k_axis, s.outlier_threshold = axis, thr
    for side in (s.k_side, s.v_side):
        side.cap, side.idx, side.val, side.cnt, side.tile_ptr = 8, A, A, A, A
    return s


def test_prompt_weights(lib):
    def call(Q=A, K=A, Bt=1, Hq=8, Hkv=2, D=128, L=256, q0=0, nq=256, w=A, ws=A, size=BIG):
        return lib.qp_prompt_weights(Q, K, Bt, Hq, Hkv, D, L, q0, nq, 0, w, ws, size, None)
    assert call(Q=None) == 1 and call(K=None) == 1 and call(w=None) == 1 and call(ws=None) == 1
    assert call(Hq=7) == 1 and call(L=0, nq=0) == 1 and call(nq=0) == 1 and call(q0=-1) == 1 and call(q0=1) == 1
    assert call(q0=2 ** 31 - 1, nq=256) == 1
    assert call(D=96) == 2 and call(Hq=32) == 2
    assert call(Bt=4096, L=262144, q0=0, nq=1) == 2                      # 32-bit row coordinates
    assert call(Q=A + 2) == 5 and call(K=A + 8) == 5 and call(w=A + 4) == 5 and call(ws=A + 1) == 5
    need = qp.prompt_weights_workspace_bytes(1, 8, 2, 128, 256, 0, 256)
    assert need > 0 and call(size=need - 1) == 4
    assert qp.prompt_weights_workspace_bytes(1, 8, 2, 128, 256, 1, 256) == 0
    assert qp.prompt_weights_workspace_bytes(1, 8, 2, 96, 256, 0, 256) == 0


def test_heavy_select(lib):
    def call(x=A, Bt=1, Hkv=2, L=256, w=32, n=64, cap=64, kept=A):
        return lib.qp_heavy_select(x, Bt, Hkv, L, w, n, cap, kept, A, A, None)
    assert call(x=None) == 1 and call(kept=None) == 1 and call(Bt=0) == 1 and call(w=0) == 1 and call(w=256) == 1
    assert call(n=32) == 3 and call(n=257, cap=257) == 3 and call(cap=63) == 3
    assert call(Bt=65536) == 2


def test_decode_attn_weights(lib):
    def call(c, s=None, q=A, w=A, out=A, ws=A, size=BIG):
        return lib.qp_decode_attn_weights(q, ctypes.byref(c) if c else None, ctypes.byref(s) if s else None, w, out, ws, size, None)
    c = cache()
    assert call(None) == 1 and call(c, q=None) == 1 and call(c, w=None) == 1 and call(c, out=None) == 1 and call(c, ws=None) == 1
    assert call(c, q=A + 2) == 5 and call(c, w=A + 4) == 5 and call(c, out=A + 8) == 5 and call(c, ws=A + 4) == 5
    need = qp.decode_weights_workspace_bytes(c)
    assert need > 0 and call(c, size=need - 1) == 4
    p = cache(bits=4)
    assert call(p) == 2 and call(p, strategy(0)) == 2 and call(p, strategy(1, 6.0)) == 2 and call(p, strategy(7)) == 1
    assert call(p, strategy(1), size=qp.decode_weights_workspace_bytes(p) - 1) == 4
    p.k_zero = None
    assert call(p, strategy(1)) == 1
    p = cache(bits=4)
    p.n_keep = 40
    assert call(p, strategy(1)) == 3
    assert qp.decode_weights_workspace_bytes(p) == 0


def test_evict_kv(lib):
    def call(c, s=None, k=A, v=A, w=A, pos=A, new=100, recent=8):
        return lib.qp_evict_kv(k, v, ctypes.byref(c) if c else None, ctypes.byref(s) if s else None, w, pos, new, recent, None, None)
    c = cache(cap=80)
    assert call(None) == 1 and call(c, k=None) == 1 and call(c, v=None) == 1 and call(c, w=None) == 1 and call(c, pos=None) == 1
    assert call(c, new=-1) == 1 and call(c, recent=-1) == 1
    assert call(c, k=A + 2) == 5 and call(c, v=A + 2) == 5 and call(c, w=A + 4) == 5 and call(c, pos=A + 4) == 5
    assert c.n_keep == 64                                                # nothing changed
    p = cache(bits=2)
    assert call(p) == 2 and call(p, strategy(0)) == 2 and call(p, strategy(1, 6.0)) == 2


def test_decode_attn_tree(lib):
    def call(c, T=8, s=None, t=None, q=A, kd=A, vd=A, m=A, out=A, ws=A, size=BIG):
        return lib.qp_decode_attn_tree(q, T, ctypes.byref(c) if c else None, ctypes.byref(s) if s else None,
                                       ctypes.byref(t) if t else None, kd, vd, m, out, ws, size, None)
    c = cache()
    assert call(None) == 1 and call(c, T=0) == 1 and call(c, T=65) == 2
    for name in ("q", "kd", "vd", "m", "out", "ws"):
        assert call(c, **{name: None}) == 1
        assert call(c, **{name: A + 8}) == 5
    need = qp.decode_tree_workspace_bytes(c, 8)
    assert need > 0 and call(c, size=need - 1) == 4
    p = cache(bits=4)
    assert call(p, s=strategy(0, 6.0)) == 2 and call(p, s=strategy(3)) == 1
    t = qp.qp_tail()
    t.k_tail = t.v_tail = A
    t.n_tail = 32
    assert call(p, t=t) == 1
    t.n_tail, t.k_tail = 3, None
    assert call(p, t=t) == 1
    t.k_tail = A + 2
    assert call(p, t=t) == 5
    assert qp.decode_tree_workspace_bytes(c, 0) == 0 and qp.decode_tree_workspace_bytes(c, 65) == 0


def test_tree_mask_needs_earlier_parents():
    import torch
    assert qp.tree_mask(torch.tensor([[-1, 0, 0, 2]])).tolist() == [[1, 3, 5, 13]]
    assert qp.tree_mask(torch.arange(-1, 63)[None])[0, 63] == -1         # a chain of 64: every bit
    for bad in ([[0]], [[-1, 1]], [[-2]], [[-1, 0, 5]]):
        with pytest.raises(ValueError):
            qp.tree_mask(torch.tensor(bad))
