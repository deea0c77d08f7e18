"""Rotations on the host, and refusals of the rotation and paged-cache calls: checked before anything is launched (no GPU needed)."""
import ctypes
import math

import pytest
import torch

from paper_2412_12706_b200 import build as qp_build
from paper_2412_12706_b200 import qp

A = 0x1000   # aligned, never dereferenced
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    qp_build.build()
    return qp.lib()


def turns(r):
    return [r.turn[i] / 2 ** 64 for i in range(r.rot_dim // 2)]


def wanted(rot, base, kind, s, L):
    """radians a position, by the definition"""
    d = lambda x: rot * math.log(L / (2 * math.pi * x)) / (2 * math.log(base))
    lo, hi = max(math.floor(d(32)), 0), min(math.ceil(d(1)), rot - 1)
    out = []
    for i in range(rot // 2):
        f = (base * s ** (rot / (rot - 2)) if kind == "ntk" else base) ** (-2 * i / rot)
        r = {"plain": 0, "ntk": 0, "linear": 1, "yarn": min(1, max(0, (i - lo) / (hi - lo or 0.001))),
             "bands": 1 - min(1, max(0, (L * f / (2 * math.pi) - 1) / 3))}[kind]
        out.append(f * (1 - r) + f / s * r)
    return out


@pytest.mark.parametrize("rot,base,s,L", [(128, 10000.0, 4.0, 4096), (64, 500000.0, 8.0, 8192), (4, 10000.0, 2.0, 100), (22, 1e6, 32.0, 2048), (128, 10000.0, 1.0, 16)])
@pytest.mark.parametrize("kind", ["plain", "linear", "ntk", "yarn", "bands"])
def test_frequencies(lib, rot, base, s, L, kind):
    r = qp.rope(rot, base, True, kind, s, L)
    assert r.rot_dim == rot and r.interleaved == 1
    # a frequency in 64 bits is off by a few 2^-53 of itself, the turn by 2^-64
    for got, w in zip(turns(r), wanted(rot, base, kind, s, L)):
        assert abs(got - w / (2 * math.pi)) <= 2.0 ** -47 * w / (2 * math.pi) + 2.0 ** -63
    assert r.factor == pytest.approx(0.1 * math.log(s) + 1 if kind == "yarn" else 1.0, rel=2.0 ** -23)
    assert all(r.turn[i] == 0 for i in range(rot // 2, 64))


def test_own_frequencies(lib):
    r = qp.rope(8, freqs=[0.0, math.pi / 2, -math.pi / 2, 2 * math.pi], factor=0.25)
    assert r.factor == 0.25
    got = turns(r)
    assert got[0] == 0 and abs(got[1] - 0.25) < 2 ** -50 and abs(got[2] - 0.75) < 2 ** -50 and min(got[3], 1 - got[3]) < 2 ** -50


def test_refused_rotations(lib):
    def init(rot=64, base=1e4, kind=0, s=2.0, L=100, out=qp.qp_rope()):
        return lib.qp_rope_init(rot, 0, base, kind, s, L, ctypes.byref(out) if out is not None else None)
    assert init() == 0 and init(out=None) == 1
    for bad in (dict(rot=0), dict(rot=3), dict(rot=130), dict(rot=-2), dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(kind=-1), dict(kind=5),
                dict(kind=1, s=0.5), dict(kind=2, s=math.nan), dict(kind=3, s=math.inf), dict(kind=3, L=0), dict(kind=4, L=-1), dict(kind=2, rot=2)):
        assert init(**bad) == 1, bad
    assert init(kind=0, s=math.nan, L=-5) == 0                    # plain looks at neither
    one = (ctypes.c_double * 1)
    f = lambda w, rot=2, m=1.0: lib.qp_rope_freqs(rot, 0, one(w), m, ctypes.byref(qp.qp_rope()))
    assert f(0.5) == 0 and f(math.nan) == 1 and f(6.3) == 1 and f(-6.3) == 1 and f(0.5, m=math.inf) == 1 and f(0.5, rot=1) == 1
    assert lib.qp_rope_freqs(2, 0, None, 1.0, ctypes.byref(qp.qp_rope())) == 1
    r = qp.qp_rope()
    r.rot_dim = 77
    init(rot=5, out=r)
    assert r.rot_dim == 77                                        # refused: left as it was
    with pytest.raises(ValueError):
        qp.rope(8, freqs=[1.0])
    with pytest.raises(KeyError):
        qp.rope(8, scaling="no such")


def test_rotary(lib):
    def call(x=A, xs=(0, 128, 1024), out=2 * A, os=(0, 128, 1024), Bt=1, H=8, L=4, D=128, pos=A, ps=0, rope=None):
        rope = rope or qp.rope(min(D, 128) if D in (64, 128) else 64)
        s3 = lambda s: None if s is None else (ctypes.c_int64 * 3)(*s)
        return lib.qp_rotary(x, s3(xs), out, s3(os), Bt, H, L, D, pos, ps, ctypes.byref(rope), 0, None)
    for bad in (dict(x=None), dict(out=None), dict(pos=None), dict(xs=None), dict(os=None), dict(Bt=0), dict(H=0), dict(L=0), dict(D=0), dict(ps=-1),
                dict(xs=(0, -128, 1024)), dict(out=A, os=(0, 1024, 128))):
        assert call(**bad) == 1, bad
    assert call(D=96) == 2 and call(D=256) == 2 and call(H=1 << 17) == 2
    for bad in (dict(x=A + 2), dict(out=A + 8), dict(pos=A + 2), dict(xs=(0, 132, 1024)), dict(os=(0, 128, 1028))):
        assert call(**bad) == 5, bad
    assert call(D=64, xs=(0, 64, 512), os=(0, 64, 512), rope=qp.rope(128)) == 1          # more channels than the head has
    r = qp.rope(64)
    r.rot_dim = 7
    assert call(rope=r) == 1
    s3 = (ctypes.c_int64 * 3)(0, 128, 1024)
    assert lib.qp_rotary(A, s3, 2 * A, s3, 1, 8, 4, 128, A, 0, None, 0, None) == 1


def paged(n_seqs=3, Hq=8, Hkv=2, D=128, fmt=0, page=64, n_pages=20, max_pages=8):
    c = qp.paged_layout(n_seqs, Hq, Hkv, D, fmt, page, n_pages, max_pages)
    c.k_codes = c.v_codes = c.k_scale = c.v_scale = c.k_tail = c.v_tail = A
    return c


def step(n=5, m=3, start=A, ln=A, pages=A):
    return qp.qp_step(n, m, start, ln, pages)


def test_layout(lib):
    c = qp.paged_layout(3, 8, 2, 128, 0, 64, 20, 8)
    assert (c.codes_bytes, c.scale_bytes, c.tail_bytes) == (20 * 2 * 64 * 128, 20 * 2 * 2, 3 * 2 * 64 * 128 * 2) and c.k_codes is None
    assert ctypes.sizeof(qp.qp_paged) == 8 * 4 + 3 * 8 + 6 * 8 and ctypes.sizeof(qp.qp_step) == 2 * 4 + 3 * 8
    assert ctypes.sizeof(qp.qp_rope) == 16 + 64 * 8
    for bad, code in ((dict(n_seqs=0), 1), (dict(Hq=7), 1), (dict(n_pages=0), 1), (dict(max_pages=0), 1), (dict(D=96), 2), (dict(Hq=32), 2),
                      (dict(fmt=2), 2), (dict(fmt=-1), 2), (dict(page=16), 2), (dict(page=48), 2), (dict(n_seqs=qp.QP_MAX_SEQS + 1), 2), (dict(Hq=65544, Hkv=8193), 2),
                      (dict(n_pages=1 << 25), 2), (dict(max_pages=1 << 25), 2), (dict(Hq=1 << 26, Hkv=1 << 26), 2)):
        with pytest.raises(qp.QpError) as e:
            paged(**bad)
        assert e.value.status == code, bad
    assert lib.qp_paged_layout(1, 8, 2, 128, 0, 64, 20, 8, None) == 1


POINTERS = ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail")


def cache_refusals(call):
    """Refusals that append and attention share."""
    assert call(None) == 1
    for name in POINTERS:
        c = paged()
        setattr(c, name, None)
        assert call(c) == 1
        setattr(c, name, A + 8)
        assert call(c) == 5
    c = paged()
    c.page = 40
    assert call(c) == 2
    c = paged()
    c.n_pages = 1 << 30
    assert call(c) == 2
    for bad in (dict(n=0, m=0), dict(m=0), dict(n=5, m=6), dict(start=None), dict(ln=None), dict(pages=None)):
        assert call(paged(), t=step(**bad)) == 1, bad
    for bad in (dict(start=A + 2), dict(ln=A + 1), dict(pages=A + 2)):
        assert call(paged(), t=step(**bad)) == 5, bad
    assert call(paged(), t=0) == 1


def test_append(lib):
    def call(c, t=None, k=A, ks=256, v=A, vs=256, rope=None, pos=None, q=None, qs=1024, qo=None):
        t = step() if t is None else t
        return lib.qp_paged_append(k, ks, v, vs, ctypes.byref(c) if c else None, ctypes.byref(t) if t else None,
                                   ctypes.byref(rope) if rope else None, pos, q, qs, qo, None)
    cache_refusals(call)
    r = qp.rope(128)
    for bad in (dict(k=None), dict(v=None), dict(ks=248), dict(vs=0), dict(q=A), dict(q=A, qo=A), dict(q=A, qo=2 * A, rope=r, qs=1016),
                dict(q=A, qo=A, rope=r, qs=1032), dict(q=A, rope=r)):
        assert call(paged(), **bad) == 1, bad
    for bad in (dict(k=A + 2), dict(v=A + 8), dict(ks=260), dict(vs=257), dict(pos=A + 2, rope=r), dict(q=A + 4, qo=A, rope=r), dict(q=A, qo=A + 8, rope=r),
                dict(q=A, qo=2 * A, rope=r, qs=1028)):
        assert call(paged(), **bad) == 5, bad
    assert call(paged(D=64), ks=128, vs=128, rope=r) == 1


def test_attention(lib):
    def call(c, t=None, q=A, qs=1024, out=A, ws=A, size=BIG):
        t = step() if t is None else t
        return lib.qp_paged_attn(q, qs, ctypes.byref(c) if c else None, ctypes.byref(t) if t else None, out, ws, size, None)
    cache_refusals(call)
    for bad in (dict(q=None), dict(out=None), dict(ws=None), dict(qs=1016)):
        assert call(paged(), **bad) == 1, bad
    for bad in (dict(q=A + 2), dict(out=A + 8), dict(ws=A + 4), dict(qs=1028)):
        assert call(paged(), **bad) == 5, bad
    need = qp.paged_attn_workspace_bytes(paged(), 5, 3)
    assert need > 0 and call(paged(), size=need - 1) == 4
    for n, m in ((0, 0), (5, 0), (5, 6)):
        assert qp.paged_attn_workspace_bytes(paged(), n, m) == 0
    far = paged(n_seqs=2048, Hq=64, Hkv=8, n_pages=1000, max_pages=1 << 24)              # more work than is numbered in 31 bits
    assert qp.paged_attn_workspace_bytes(far, 4096, 2) == 0 and call(far, t=step(4096, 2), qs=8192) == 2


# ---------------------------------------------------------------------------------------------- the binding

class Tensor:
    """Stand-in that says where it lives."""
    def __init__(self, shape, dtype=torch.bfloat16, device=0, strides=None, address=0x1000):
        self.address, self.shape, self.dtype, self.on = address, torch.Size(shape), dtype, device
        self.is_cuda, self.device = device is not None, "cpu" if device is None else f"cuda:{device}"
        self.strides = tuple(strides) if strides else tuple(math.prod(shape[i + 1:]) for i in range(len(shape)))

    def stride(self, i=None): return self.strides if i is None else self.strides[i]
    def is_contiguous(self): return self.strides == tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))
    def get_device(self): return -1 if self.on is None else self.on
    def data_ptr(self): return self.address
    def numel(self): return math.prod(self.shape)
    def element_size(self): return self.dtype.itemsize
    def dim(self): return len(self.shape)
    def new_empty(self, shape): return Tensor(shape, self.dtype, self.on)


class Library:
    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith("_bytes") or name in ("qp_status_string", "qp_paged_layout", "qp_rope_init", "qp_rope_freqs"):
            return getattr(self.real, name)

        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def library(lib, monkeypatch):
    fake = Library(lib)
    monkeypatch.setattr(qp, "lib", lambda: fake)
    monkeypatch.setattr(qp, "_current_device", lambda: 0)
    monkeypatch.setattr(qp, "_stream", lambda: 0)
    monkeypatch.setattr(qp, "_empty_like", lambda t, memory_format=None: t.new_empty(t.shape))
    return fake


I32 = torch.int32
SEQS, HQ, HKV, D, PAGE, PAGES, MOST, N = 3, 8, 2, 128, 64, 20, 8, 5


def held(device=0, dtype=torch.float8_e4m3fn, **bad):
    a = dict(kc=Tensor((PAGES, HKV, PAGE, D), dtype, device), vc=Tensor((PAGES, HKV, PAGE, D), dtype, device), ks=Tensor((PAGES, HKV), device=device),
             vs=Tensor((PAGES, HKV), device=device), kt=Tensor((SEQS, HKV, PAGE, D), device=device), vt=Tensor((SEQS, HKV, PAGE, D), device=device))
    a.update(bad)
    return qp.paged_cache(HQ, *a.values(), MOST)


def new_step(start=None, ln=None, pages=None, n=N, m=3):
    return qp.PagedStep(start or Tensor((SEQS + 1,), I32), ln or Tensor((SEQS,), I32), pages or Tensor((SEQS, MOST), I32), n, m)


def rows(heads, n=N, **kw):
    return Tensor((n, heads, D), **kw)


@pytest.mark.parametrize("bad", [dict(kc=Tensor((PAGES, HKV, PAGE, D), torch.int8)), dict(vs=Tensor((PAGES, HKV), torch.float32)), dict(ks=Tensor((PAGES, HKV + 1))),
                                 dict(vt=Tensor((SEQS + 1, HKV, PAGE, D))), dict(kt=Tensor((SEQS, HKV, PAGE, D), device=None)),
                                 dict(vc=Tensor((PAGES, HKV, PAGE, D), torch.float8_e4m3fn, 1)),
                                 dict(kc=Tensor((PAGES, HKV, PAGE, D), torch.float8_e4m3fn, strides=(HKV * PAGE * D * 2, PAGE * D, D, 1)))])
def test_arrays_that_are_no_cache_are_refused(library, bad):
    held()
    with pytest.raises(AssertionError):
        held(**bad)


@pytest.mark.parametrize("bad", [dict(start=Tensor((SEQS,), I32)), dict(ln=Tensor((SEQS,), torch.int64)), dict(pages=Tensor((SEQS, MOST), I32, 1)),
                                 dict(start=Tensor((SEQS + 1,), I32, None)), dict(pages=Tensor((SEQS, MOST), I32, strides=(2 * MOST, 1)))])
def test_a_step_of_other_arrays_is_refused(library, bad):
    new_step()
    with pytest.raises(AssertionError):
        new_step(**bad)


def test_strides_reach_the_library(library):
    c, t, r = held(), new_step(), qp.rope(D)
    wide = (HQ + 2 * HKV) * D
    q, k = rows(HQ, strides=(wide, D, 1)), rows(HKV, strides=(wide, D, 1), address=0x8000)
    qp.paged_append(k, rows(HKV), c, t, r, q=q)
    name, a = library.calls.pop()
    assert name == "qp_paged_append" and a[:4] == (0x8000, wide, 0x1000, HKV * D) and a[9] == wide
    one = new_step(n=1, m=1)                                       # one row: its stride says nothing
    qp.paged_append(rows(HKV, 1, strides=(1, D, 1)), rows(HKV, 1), c, one)
    assert library.calls.pop()[1][1] == HKV * D
    qp.paged_attn(q, c, t, out=rows(HQ), workspace=Tensor((1 << 26,), torch.uint8))
    assert library.calls.pop()[1][1] == wide
    x = Tensor((2, 4, 1, D), strides=(4 * D, D, 3, 1))
    qp.rotary(x, Tensor((2, 1), I32), r)
    assert list(library.calls.pop()[1][1]) == [4 * D, D, 0]


@pytest.mark.parametrize("bad", [dict(k=rows(HKV, device=1)), dict(v=rows(HKV + 1)), dict(k=rows(HKV, dtype=torch.float16)), dict(k=rows(HKV, n=N + 1)),
                                 dict(v=rows(HKV, strides=(HKV * D * 2, 2 * D, 1))), dict(k=rows(HKV, strides=(HKV * D, D, 2))), dict(pos=Tensor((N + 1,), I32)),
                                 dict(pos=Tensor((N,), torch.int64)), dict(q=rows(HQ - 1)), dict(q=rows(HQ), q_out=rows(HQ, strides=(HQ * D * 2, D, 1)))])
def test_append_refuses_other_tensors(library, bad):
    a = dict(k=rows(HKV), v=rows(HKV))
    a.update(bad)
    with pytest.raises(AssertionError):
        qp.paged_append(a["k"], a["v"], held(), new_step(), qp.rope(D), a.get("pos"), a.get("q"), a.get("q_out"))
    assert not library.calls


def test_a_step_of_another_cache_is_refused(library):
    other = qp.PagedStep(Tensor((SEQS + 2,), I32), Tensor((SEQS + 1,), I32), Tensor((SEQS + 1, MOST), I32), N, 3)
    wider = qp.PagedStep(Tensor((SEQS + 1,), I32), Tensor((SEQS,), I32), Tensor((SEQS, MOST + 1), I32), N, 3)
    for t in (other, wider):
        with pytest.raises(AssertionError):
            qp.paged_append(rows(HKV), rows(HKV), held(), t)
        with pytest.raises(AssertionError):
            qp.paged_attn(rows(HQ), held(), t)
    assert not library.calls


@pytest.mark.parametrize("bad", [dict(q=rows(HQ + 1)), dict(out=rows(HQ, device=None)), dict(out=rows(HQ, strides=(HQ * D * 2, D, 1))),
                                 dict(ws=Tensor((16,), torch.uint8)), dict(ws=Tensor((1 << 26,), torch.uint8, 1)),
                                 dict(ws=Tensor((1 << 26,), torch.uint8, address=0x1004)), dict(q=rows(HQ, address=0x1002)), dict(out=rows(HQ, address=0x1008)),
                                 dict(q=rows(HQ, strides=(HQ * D + 4, D, 1))), dict(k=rows(HKV, dtype=torch.float32)), dict(m=N + 1)])
@pytest.mark.parametrize("turned", [False, True])
def test_a_refused_layer_step_has_taken_nothing_in(library, bad, turned):
    def run(q=rows(HQ), out=rows(HQ), ws=Tensor((1 << 26,), torch.uint8), k=rows(HKV), m=3):
        return qp.paged_layer_step(q, k, rows(HKV), held(), new_step(m=m), qp.rope(D) if turned else None, None, out, ws)
    run()
    assert [c[0] for c in library.calls] == ["qp_paged_append", "qp_paged_attn"]
    with pytest.raises((AssertionError, qp.QpError)):
        run(**bad)
    assert len(library.calls) == 2


def test_rotary_refuses_other_tensors(library):
    r, x, pos = qp.rope(D), Tensor((2, 4, 7, D)), Tensor((7,), I32)
    qp.rotary(x, pos, r)
    for bad in (dict(x=Tensor((2, 4, 7, D), torch.float16)), dict(x=Tensor((2, 4, 7, D), device=1)), dict(x=Tensor((2, 4, 7, D), strides=(7 * 4 * D, 7 * D, 1, 7))),
                dict(pos=Tensor((8,), I32)), dict(pos=Tensor((1, 7), I32)), dict(pos=Tensor((7,), torch.int64)), dict(out=Tensor((2, 4, 6, D))),
                dict(out=Tensor((2, 4, 7, D), strides=(0, 7 * D, D, 1))), dict(out=Tensor((2, 4, 7, D), device=None))):
        a = dict(x=x, pos=pos, out=None)
        a.update(bad)
        with pytest.raises(AssertionError):
            qp.rotary(a["x"], a["pos"], r, a["out"])
    assert len(library.calls) == 1


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("stride", [0, D, HQ * D - 8])
def test_queries_that_lie_over_one_another_are_refused_before_the_append(lib, library, stride, turned):
    """Rows of queries nearer to one another than they are long: the attention's refusal, made before the tokens are taken in."""
    assert lib.qp_paged_attn(A, stride, ctypes.byref(paged()), ctypes.byref(step()), 2 * A, A, BIG, None) == 1
    with pytest.raises(qp.QpError) as e:
        qp.paged_layer_step(rows(HQ, strides=(stride, D, 1)), rows(HKV), rows(HKV), held(), new_step(), qp.rope(D) if turned else None, None,
                            rows(HQ), Tensor((1 << 26,), torch.uint8))
    assert e.value.status == 1 and not library.calls


@pytest.mark.parametrize("n,m,status", [(N, N + 1, 1), (N, 0, 1), (4096, 2, 2)])
def test_a_refused_layer_step_says_what_the_calls_say(lib, library, n, m, status):
    """A step whose numbers do not belong together, and one of more work than is numbered in 31 bits."""
    far = 1 << 24
    c = held() if status == 1 else qp.paged_cache(64, *(Tensor((PAGES, 8, PAGE, D), torch.float8_e4m3fn) for _ in range(2)),
                                                 *(Tensor((PAGES, 8)) for _ in range(2)), *(Tensor((2048, 8, PAGE, D)) for _ in range(2)), far)
    seqs, most = c.table
    t = qp.PagedStep(Tensor((seqs + 1,), I32), Tensor((seqs,), I32), Tensor((seqs, most), I32), n, m)
    Hq, Hkv, _ = c.heads
    ref = ctypes.byref(c.desc), ctypes.byref(t.desc)
    assert lib.qp_paged_attn(A, Hq * D, *ref, 2 * A, A, BIG, None) == status
    with pytest.raises(qp.QpError) as e:
        qp.paged_layer_step(rows(Hq, n), rows(Hkv, n), rows(Hkv, n), c, t, None, None, rows(Hq, n), Tensor((1 << 26,), torch.uint8))
    assert e.value.status == status and not library.calls
