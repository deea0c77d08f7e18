"""What the binding of the weight, eviction and tree calls refuses before the library is called.  No GPU: the tensors are stand-ins
that say where they live, and the library one that writes down what it was asked for."""
import math

import pytest
import torch

from paper_2412_12706_b200 import qp


class Tensor:
    def __init__(self, shape, dtype=torch.bfloat16, device=0, contiguous=True, address=0x1000):
        self.address = address
        self.shape, self.dtype, self.on, self.contiguous = torch.Size(shape), dtype, device, contiguous
        self.is_cuda, self.device = device is not None, "cpu" if device is None else f"cuda:{device}"

    def is_contiguous(self): return self.contiguous
    def get_device(self): return -1 if self.on is None else self.on
    def data_ptr(self): return self.address
    def numel(self): return math.prod(self.shape)
    def element_size(self): return self.dtype.itemsize


class Library:
    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith("_bytes") or name.startswith("qp_cache_layout") or name in ("qp_status_string", "qp_n_keep"):
            return getattr(self.real, name)

        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


Bt, Hq, Hkv, D, n, T, L = 1, 8, 2, 128, 64, 4, 256


@pytest.fixture
def library(monkeypatch):
    from paper_2412_12706_b200 import build as qp_build
    qp_build.build()
    fake = Library(qp.lib())
    monkeypatch.setattr(qp, "lib", lambda: fake)
    monkeypatch.setattr(qp, "_current_device", lambda: 0)
    monkeypatch.setattr(qp, "_stream", lambda: 0)
    return fake


def cache(bits=16, n_cap=0, device=0):
    d = qp.cache_layout_cap(Bt, Hq, Hkv, D, bits, 32, n, n_cap)
    return qp.Cache(d, Tensor((Bt, Hkv, n_cap or n, D), device=device), None, None, None, None, None)


def tail(device=0, group=32, heads=Hkv):
    t = qp.qp_tail()
    t.n_tail = 3
    return qp.Tail(t, Tensor((Bt, heads, group, D), device=device), Tensor((Bt, heads, group, D), device=device))


def calls(ws_device=0, ws_dtype=torch.uint8, ws_bytes=1 << 26, contiguous=True, tree_tail=None, bits=16):
    ws = Tensor((ws_bytes // ws_dtype.itemsize,), ws_dtype, ws_device, contiguous)
    st = None
    if bits < 16:
        s = qp.qp_strategy()
        s.k_axis = 1
        st = qp.Strategy(s, [])
    f = torch.float32
    return dict(
        prompt=lambda: qp.prompt_weights(Tensor((Bt, Hq, L, D)), Tensor((Bt, Hkv, L, D)), 0, Tensor((Bt, Hkv, L), f), ws),
        decode=lambda: qp.decode_attn_weights(Tensor((Bt, Hq, D)), cache(bits), Tensor((Bt, Hkv, n), f), st, Tensor((Bt, Hq, D)), ws),
        tree=lambda: qp.decode_attn_tree(Tensor((Bt, T, Hq, D)), cache(bits), Tensor((Bt, T, Hkv, D)), Tensor((Bt, T, Hkv, D)),
                                         Tensor((Bt, T), torch.int64), tree_tail, None, Tensor((Bt, T, Hq, D)), ws))


NAMES = ("prompt", "decode", "tree")


@pytest.mark.parametrize("name", NAMES)
def test_a_workspace_of_the_gpu_in_use_is_taken_with_all_its_bytes(library, name):
    for dtype in (torch.uint8, torch.float32):                     # its size is counted in bytes, whatever it holds
        library.calls.clear()
        calls(ws_dtype=dtype)[name]()
        assert len(library.calls) == 1 and 1 << 26 in library.calls[0][1]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("bad", [dict(ws_device=None), dict(ws_device=1), dict(contiguous=False)])
def test_a_workspace_elsewhere_is_refused(library, name, bad):
    with pytest.raises(AssertionError):
        calls(**bad)[name]()
    assert not library.calls


@pytest.mark.parametrize("bad", [dict(device=None), dict(device=1), dict(heads=1), dict(group=64)])
def test_a_tail_of_another_device_or_cache_is_refused(library, bad):
    calls(bits=4, tree_tail=tail())["tree"]()
    assert len(library.calls) == 1
    with pytest.raises(AssertionError):
        calls(bits=4, tree_tail=tail(**bad))["tree"]()
    assert len(library.calls) == 1


def test_an_empty_tail_needs_no_arrays(library):
    calls(bits=4, tree_tail=qp.Tail(qp.qp_tail(), None, None))["tree"]()
    assert len(library.calls) == 1


# ---------------------------------------------------------------------------------------------- the runs of calls

def held(bits=16, n_cap=0):
    f = torch.float32
    cap = n_cap or n
    return qp.HeavyCache(cache(bits, n_cap), None, Tensor((Bt, Hkv, cap), f), Tensor((Bt, Hkv, cap), torch.int32), 300)


def step(hc, q=None, out=None, ws=None, k=None):
    kv = k or Tensor((Bt, Hkv, D))
    pos = hc.pos
    pos.new_empty = lambda shape: Tensor(shape, torch.int32)
    return qp.decode_step_heavy(q or Tensor((Bt, Hq, D)), kv, kv, hc, 8, out or Tensor((Bt, Hq, D)), ws or Tensor((1 << 20,), torch.uint8))


@pytest.mark.parametrize("bad", [dict(q=Tensor((Bt, Hq, D + 1))), dict(q=Tensor((Bt, Hq, D), torch.float16)), dict(q=Tensor((Bt, Hq, D), device=None)),
                                 dict(out=Tensor((Bt, Hq + 1, D))), dict(out=Tensor((Bt, Hq, D), device=1)), dict(ws=Tensor((16,), torch.uint8)),
                                 dict(ws=Tensor((1 << 20,), torch.uint8, None)), dict(k=Tensor((Bt, Hkv, D), torch.float32)),
                                 dict(q=Tensor((Bt, Hq, D), address=0x1008)), dict(out=Tensor((Bt, Hq, D), address=0x1002)),
                                 dict(ws=Tensor((1 << 20,), torch.uint8, address=0x1004))])
@pytest.mark.parametrize("n_cap", [0, 96])
def test_a_refused_step_leaves_the_cache_as_it_was(library, bad, n_cap):
    """A step is two calls: what the second would refuse is refused before the first has taken the token in, so the step can be
    taken again."""
    hc = held(n_cap=n_cap)
    step(hc)
    assert [c[0] for c in library.calls] == ["qp_evict_kv", "qp_decode_attn_weights"] and hc.next_pos == 301
    with pytest.raises((AssertionError, qp.QpError)):
        step(hc, **bad)
    assert len(library.calls) == 2 and hc.next_pos == 301


@pytest.mark.parametrize("K,V,Q", [((Bt, Hkv, L, D), (Bt, Hkv, L - 1, D), (Bt, Hq, L, D)), ((Bt, Hkv, L, D), (Bt, Hkv, L, D), (Bt, Hq, 32, D)),
                                   ((Bt, Hkv, L, D), (Bt, 1, L, D), (Bt, Hq, L, D)), ((Bt, Hkv, L, D), (Bt, Hkv, L, D), (Bt + 1, Hq, L, D)),
                                   ((Bt, Hkv, L, D), (Bt, Hkv, L, 64), (Bt, Hq, L, D)), ((Bt, Hkv, L, D), (Bt, Hkv, L, D), (Bt, Hq, L, 64))])
@pytest.mark.parametrize("bits", [16, 4])
def test_a_prompt_whose_arrays_do_not_belong_together_is_refused(library, monkeypatch, K, V, Q, bits):
    """All queries of the prompt are asked for: a window of them would leave every key without weight that only later rows see."""
    monkeypatch.setattr(qp, "alloc_cache", lambda *a, **k: cache(bits))
    monkeypatch.setattr(qp, "heavy_select", lambda *a: (Tensor((Bt, Hkv, n), torch.int32), None, None))
    monkeypatch.setattr(qp, "prompt_weights", lambda *a: library.calls.append(("qp_prompt_weights", a)))
    with pytest.raises(AssertionError):
        qp.compress_layer_heavy(Tensor(K), Tensor(V), Tensor(Q), n * bits, bits, 32, 8)
    assert not library.calls
