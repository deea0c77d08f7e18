"""Attention of drafted trees over packed caches, against plain 64-bit arithmetic.

Tolerance.  Output: its own rounding to bf16 (2^-8 of the value); the softmax weights rounded to 16 bits (bf16 2^-8 of each
over a 16-bit cache, fp16 2^-11 otherwise, so at most that times sum p|v|); values in fp16 (2^-11 of sum p|v|); keys and
queries in fp16 for B < 16 (2^-11 each of sum|q k|) and 32-bit sums ((D + 8) 2^-23 of it) move a logit by e, a weight by the
factor e^(2 e), the output by at most (e^(2e) - 1) sum p|v| twice (numerator, normaliser).  The reconstruction code * scale + zero
in fp16 is one rounding of a value whose terms are at most three times it; a draft or tail row beyond fp16's 11 bits is exact."""
import math

import pytest
import torch

from paper_2412_12706_b200 import qp

pytestmark = pytest.mark.gpu
DEV = "cuda"


def randn(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(shape, generator=g, device=DEV)).to(torch.bfloat16)


def codes(words, bits):
    sh = bits * torch.arange(32 // bits, device=DEV)
    return ((words.long()[..., None] >> sh) & (2 ** bits - 1)).flatten(-2).double()


def make_cache(Bt, Hq, Hkv, D, n, cap, bits, g, axis, scale=1.5):
    K, V = randn((Bt, Hkv, n, D), 1, scale), randn((Bt, Hkv, n, D), 2)
    kept = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, Hkv, n).contiguous()
    c = qp.alloc_cache(Bt, Hq, Hkv, D, bits, g, n, DEV, cap if cap != n else 0)
    if bits == 16:
        c.k_codes.fill_(float("nan")); c.v_codes.fill_(float("nan"))      # room behind the tokens may hold anything
        qp.gather_quantize(K, V, kept, c)
        return c, None, K.double(), V.double()
    for t in (c.k_scale, c.k_zero, c.v_scale, c.v_zero):
        t.fill_(float("nan"))
    st = qp.make_strategy(c, axis)
    qp.gather_quantize_ex(K, V, kept, c, st)
    v = (codes(c.v_codes, bits) * c.v_scale.double()[..., None] + c.v_zero.double()[..., None]).reshape(Bt, Hkv, cap, D)[:, :, :n]
    k = codes(c.k_codes, bits) if axis == 0 else codes(c.k_codes.view(c.v_codes.shape), bits)
    ks, kz = (c.k_scale, c.k_zero) if axis == 0 else (c.k_scale.view(c.v_scale.shape), c.k_zero.view(c.v_scale.shape))
    k = k * ks.double()[..., None] + kz.double()[..., None]
    k = k.transpose(3, 4).reshape(Bt, Hkv, cap, D) if axis == 0 else k.reshape(Bt, Hkv, cap, D)
    return c, st, k[:, :, :n], v


def reference(q, k, v, kt, vt, kd, vd, sees, bits):
    """sees bool [Bt,T,T]; kt, vt the tail's rows [Bt,Hkv,m,D]"""
    Bt, T, Hq, D = q.shape
    Hkv, n = k.shape[1], k.shape[2] + kt.shape[2]
    k = torch.cat([k, kt.double(), kd.double().transpose(1, 2)], 2)
    v = torch.cat([v, vt.double(), vd.double().transpose(1, 2)], 2)
    x = q.double().view(Bt, T, Hkv, Hq // Hkv, D)
    s = torch.einsum("bthgd,bhnd->bthgn", x, k) / math.sqrt(D)
    hide = torch.cat([torch.zeros((Bt, T, n), dtype=torch.bool, device=DEV), ~sees], -1)[:, :, None, None]
    p = torch.softmax(s.masked_fill(hide, -math.inf), -1)
    v = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    out = torch.einsum("bthgn,bhnd->bthgd", p, v).reshape(Bt, T, Hq, D)
    spread = torch.einsum("bthgn,bhnd->bthgd", p, v.abs()).reshape(Bt, T, Hq, D)
    sum_abs = float(torch.einsum("bthgd,bhnd->bthgn", x.abs(), k.abs().nan_to_num(0, 0, 0)).max())
    e = ((D + 8) * 2.0 ** -23 + (0.0 if bits == 16 else 3 * 2.0 ** -11)) * sum_abs / math.sqrt(D)
    tol = 2.0 ** -8 * out.abs() + ((2.0 ** -8 if bits == 16 else 2.0 ** -11) + 2.0 ** -11 + math.expm1(2 * e)) * spread + 1e-6
    return out, tol


def random_tree(Bt, T, seed):
    g = torch.Generator().manual_seed(seed)
    parents = torch.tensor([[int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(T)] for _ in range(Bt)])
    sees = torch.zeros((Bt, T, T), dtype=torch.bool)
    for b in range(Bt):
        for i in range(T):
            j = i
            while j >= 0:
                sees[b, i, j] = True
                j = int(parents[b, j])
    return parents.to(DEV), sees.to(DEV)


def mask_of(sees):
    return (sees.long() << torch.arange(sees.shape[-1], device=DEV)).sum(-1)


CASES = [  # Bt, Hq, Hkv, D, n, cap, bits, g, axis, T, n_tail
    (1, 1, 1, 64, 1, 1, 16, 32, 0, 1, 0), (1, 32, 8, 128, 100, 130, 16, 32, 0, 5, 0), (2, 8, 1, 128, 127, 127, 16, 64, 0, 16, 0),
    (1, 8, 2, 64, 1000, 1024, 16, 32, 0, 33, 0), (1, 32, 8, 128, 3000, 3000, 16, 32, 0, 64, 0), (1, 64, 8, 128, 513, 513, 16, 32, 0, 64, 0),
    (1, 14, 2, 128, 640, 640, 16, 32, 0, 37, 0),
    (1, 4, 1, 128, 32, 32, 4, 32, 0, 1, 0), (1, 32, 8, 128, 2048, 2048, 4, 32, 0, 8, 5), (2, 8, 2, 128, 640, 704, 4, 64, 0, 64, 63),
    (1, 8, 1, 128, 384, 384, 4, 128, 0, 64, 127), (1, 16, 4, 64, 1024, 1024, 4, 32, 0, 13, 31), (1, 8, 8, 64, 64, 64, 4, 64, 0, 64, 1),
    (1, 32, 8, 128, 1024, 1056, 2, 32, 0, 33, 17), (1, 8, 2, 128, 256, 256, 2, 128, 0, 20, 100), (2, 6, 2, 64, 320, 320, 2, 32, 0, 7, 0),
    (1, 32, 8, 128, 1024, 1024, 8, 32, 0, 24, 30), (1, 8, 2, 128, 512, 512, 8, 64, 0, 63, 2), (1, 8, 4, 64, 96, 96, 8, 32, 0, 2, 9),
    (1, 32, 8, 128, 1024, 1024, 4, 32, 1, 16, 0), (1, 8, 2, 128, 320, 384, 2, 64, 1, 9, 0), (2, 4, 2, 64, 160, 160, 8, 32, 1, 30, 3),
    (1, 8, 1, 128, 256, 256, 4, 128, 1, 41, 0),
]


LONG = [  # several clusters per head, whose results are joined; more heads than the GPU holds at once
    (1, 32, 8, 128, 8192, 8192, 4, 32, 0, 64, 21), (1, 8, 1, 128, 16384, 16384, 16, 32, 0, 5, 0), (1, 8, 1, 64, 20000, 20000, 16, 32, 0, 64, 0),
    (1, 8, 1, 128, 4096, 4224, 2, 64, 1, 33, 0), (1, 8, 2, 64, 6144, 6144, 8, 32, 0, 2, 3), (19, 32, 8, 128, 320, 320, 4, 32, 0, 16, 9),
]


@pytest.mark.parametrize("Bt,Hq,Hkv,D,n,cap,bits,g,axis,T,m", CASES + LONG)
def test_tree(Bt, Hq, Hkv, D, n, cap, bits, g, axis, T, m):
    c, st, k, v = make_cache(Bt, Hq, Hkv, D, n, cap, bits, g, axis)
    parents, sees = random_tree(Bt, T, n + T)
    mask = qp.tree_mask(parents)
    assert torch.equal(mask, mask_of(sees))
    q, kd, vd = randn((Bt, T, Hq, D), 3, 1.5), randn((Bt, T, Hkv, D), 4, 1.5), randn((Bt, T, Hkv, D), 5)
    tail = qp.alloc_tail(c)
    kt = vt = torch.zeros((Bt, Hkv, 0, D), dtype=torch.bfloat16, device=DEV)
    if m:
        tail.k_tail.copy_(randn(tail.k_tail.shape, 6, 1.5)); tail.v_tail.copy_(randn(tail.v_tail.shape, 7))
        tail.k_tail[:, :, m:] = float("nan"); tail.v_tail[:, :, m:] = float("inf")     # rows behind the last are not read
        tail.desc.n_tail = m
        kt, vt = tail.k_tail[:, :, :m], tail.v_tail[:, :, :m]
    strategy = st if axis == 1 else None
    out = qp.decode_attn_tree(q, c, kd, vd, mask if T == 64 else mask | (-1 << T), tail, strategy)   # bits behind T: ignored
    ref, tol = reference(q, k, v, kt, vt, kd, vd, sees, bits)
    worst = float(((out.double() - ref).abs() / tol).max())
    assert worst <= 1, worst
    assert torch.equal(out, qp.decode_attn_tree(q, c, kd, vd, mask, tail, strategy))


@pytest.mark.parametrize("bits", [16, 4])
def test_masks_of_any_shape(bits):
    """Rows that see no draft, rows that see all, bit 63, and what a hidden draft holds does not matter unless it is not finite."""
    Bt, Hq, Hkv, D, n, T = 1, 8, 2, 128, 160, 64
    c, _, k, v = make_cache(Bt, Hq, Hkv, D, n, n, bits, 32, 0)
    g = torch.Generator().manual_seed(9)
    sees = (torch.rand((Bt, T, T), generator=g) < 0.3).to(DEV)
    sees[:, 3], sees[:, 7] = False, True
    sees[:, :, 11] = False
    q, kd, vd = randn((Bt, T, Hq, D), 3), randn((Bt, T, Hkv, D), 4), randn((Bt, T, Hkv, D), 5)
    none = torch.zeros((Bt, Hkv, 0, D), dtype=torch.bfloat16, device=DEV)
    ref, tol = reference(q, k, v, none, none, kd, vd, sees, bits)
    out = qp.decode_attn_tree(q, c, kd, vd, mask_of(sees))
    assert torch.all((out.double() - ref).abs() <= tol)
    kd[:, 11] = float("nan")                                       # a key that no row sees
    again = qp.decode_attn_tree(q, c, kd, vd, mask_of(sees))
    assert torch.equal(again, out)
    # a row of drafts that sees no draft is plain decode attention
    plain = qp.decode_attn(q[:, 3].contiguous(), c)
    assert torch.all((out[:, 3].double() - plain.double()).abs() <= 2 * tol[:, 3])


def test_a_chain_equals_steps_of_the_generation_loop():
    """A drafted chain verified at once gives, up to rounding, what appending its tokens one by one gives."""
    Bt, Hq, Hkv, D, n, T = 2, 8, 2, 128, 256, 6
    c, _, k, v = make_cache(Bt, Hq, Hkv, D, n, n + 32, 4, 32, 0)
    tail = qp.alloc_tail(c)
    q, kd, vd = randn((Bt, T, Hq, D), 3), randn((Bt, T, Hkv, D), 4), randn((Bt, T, Hkv, D), 5)
    parents = (torch.arange(T, device=DEV) - 1).expand(Bt, T)
    out = qp.decode_attn_tree(q, c, kd, vd, qp.tree_mask(parents), tail)
    none = torch.zeros((Bt, Hkv, 0, D), dtype=torch.bfloat16, device=DEV)
    sees = torch.ones((T, T), dtype=torch.bool, device=DEV).tril().expand(Bt, T, T)
    _, tol = reference(q, k, v, none, none, kd, vd, sees, 4)
    for i in range(T):
        qp.append_kv(kd[:, i].contiguous(), vd[:, i].contiguous(), c, tail)
        step = qp.decode_attn_tail(q[:, i].contiguous(), c, tail)
        assert torch.all((step.double() - out[:, i].double()).abs() <= 3 * tol[:, i])
    # the accepted tokens now wait in the tail: the next tree sees them there
    assert tail.desc.n_tail == T
    kt, vt = tail.k_tail[:, :, :T], tail.v_tail[:, :, :T]
    out = qp.decode_attn_tree(q, c, kd, vd, qp.tree_mask(parents), tail)
    ref, tol = reference(q, k, v, kt, vt, kd, vd, sees, 4)
    assert torch.all((out.double() - ref).abs() <= tol)


def test_large_logits_and_values():
    c, _, k, v = make_cache(1, 8, 2, 128, 512, 512, 4, 32, 0, scale=10.0)
    q, kd, vd = randn((1, 9, 8, 128), 3, 20.0), randn((1, 9, 2, 128), 4, 10.0), randn((1, 9, 2, 128), 5, 500.0)
    out = qp.decode_attn_tree(q, c, kd, vd, qp.tree_mask((torch.arange(9, device=DEV) - 1)[None]))
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("bits,n", [(16, 1024), (2, 1024), (4, 9216)])
def test_from_a_graph_on_a_side_stream(bits, n):
    Bt, Hq, Hkv, D, T = 1, 32, 8, 128, 40
    c, _, _, _ = make_cache(Bt, Hq, Hkv, D, n, n, bits, 32, 0)
    q, kd, vd = randn((Bt, T, Hq, D), 3), randn((Bt, T, Hkv, D), 4), randn((Bt, T, Hkv, D), 5)
    mask = qp.tree_mask(random_tree(Bt, T, 5)[0])
    ws = qp.new_decode_workspace(qp.decode_tree_workspace_bytes(c, T), DEV)
    ref = qp.decode_attn_tree(q, c, kd, vd, mask, workspace=ws)
    o = [torch.zeros_like(ref) for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, x in zip(graphs, o):                                    # two graphs, one workspace
        with torch.cuda.graph(g):
            qp.decode_attn_tree(q, c, kd, vd, mask, out=x, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for g in graphs:
            g.replay()
    side.synchronize()
    assert torch.equal(o[0], ref) and torch.equal(o[1], ref)
    assert torch.all(ws[:4 * Bt * Hkv].view(torch.int32) == 0)     # no wait ran out


@pytest.mark.parametrize("bits,n,T,m", [(16, 300, 64, 0), (16, 5000, 20, 0), (4, 2048, 64, 63), (4, 96, 9, 0), (8, 512, 33, 31), (2, 4096, 64, 100), (2, 256, 40, 100)])
def test_drafts_that_are_not_finite(bits, n, T, m):
    """A padded tree: what a draft holds reaches only the rows that see it, channel by channel."""
    Bt, Hq, Hkv, D = 2, 8, 2, 128
    g = 128 if m > 63 else 64 if m > 31 else 32
    n = n // g * g if bits < 16 else n
    c, _, k, v = make_cache(Bt, Hq, Hkv, D, n, n, bits, g, 0)
    tail = qp.alloc_tail(c)
    kt = vt = torch.zeros((Bt, Hkv, 0, D), dtype=torch.bfloat16, device=DEV)
    if m:
        tail.k_tail.copy_(randn(tail.k_tail.shape, 6, 1.5)); tail.v_tail.copy_(randn(tail.v_tail.shape, 7))
        tail.desc.n_tail = m
        kt, vt = tail.k_tail[:, :, :m], tail.v_tail[:, :, :m]
    q, kd, vd = randn((Bt, T, Hq, D), 3, 1.5), randn((Bt, T, Hkv, D), 4, 1.5), randn((Bt, T, Hkv, D), 5)
    sees = random_tree(Bt, T, 7)[1]
    last = T - 3                                                   # the first tree has padding behind its drafts
    sees[0, last:] = False
    sees[0, :, last:] = False
    sees[0, range(last, T), range(last, T)] = True
    ref, tol = reference(q, k, v, kt, vt, kd, vd, sees.to(DEV), bits)
    kd[0, last:], vd[0, last] = float("nan"), float("nan")
    vd[0, last + 1] = float("inf")
    vd[0, last + 2] = -1e30 if bits < 16 else float("-inf")        # beyond fp16
    vd[1, 2, 0, 5] = float("inf"); vd[1, T - 1, 1, 77] = float("-inf")
    out = qp.decode_attn_tree(q, c, kd, vd, mask_of(sees), tail)
    want = ref.clone()
    s = sees.to(DEV)
    want[1, :, :Hq // 2, 5] = torch.where(s[1, :, 2, None], math.inf, want[1, :, :Hq // 2, 5])
    want[1, :, Hq // 2:, 77] = torch.where(s[1, :, T - 1, None], -math.inf, want[1, :, Hq // 2:, 77])
    assert torch.isnan(out[0, last:]).all()                        # their keys are not numbers
    out, want, tol = torch.cat([out[0, :last], out[1]]).double(), torch.cat([want[0, :last], want[1]]), torch.cat([tol[0, :last], tol[1]])
    inf = torch.isinf(want)
    assert inf.any() and torch.equal(out[inf], want[inf])
    assert torch.all((out - want).abs()[~inf] <= tol[~inf])
