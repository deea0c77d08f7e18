"""Accumulated attention weights and the eviction by them, against plain 64-bit arithmetic.

Tolerances.  A logit is a sum of D exact bf16 products: in any order of 32-bit additions (a truncating one costs a whole step)
it is off by at most (D + 8) 2^-23 sum|q k| / sqrt(D), the 8 for the scaling and for what is subtracted before the exponential.
A softmax weight is off by the factor e^(2 e) of the largest such e (numerator and normaliser), and by 2^-20 for the
exponential and the additions of positive terms.  Weights are sums of such terms, so the same relative bound holds for them."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2412_12706_b200 import qp

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rel_bound(sum_abs: float, D: int, terms: int = 1) -> float:
    return math.expm1(2 * (D + 8) * 2.0 ** -23 * sum_abs / math.sqrt(D)) + 2.0 ** -20 + terms * 2.0 ** -23


def randn(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(shape, generator=g, device=DEV)).to(torch.bfloat16)


# ---------------------------------------------------------------------------------------------- prompt

def ref_prompt(Q, K, q0):
    Bt, Hq, nq, D = Q.shape
    Hkv, n = K.shape[1], q0 + nq
    q = Q.double().view(Bt, Hkv, Hq // Hkv, nq, D)
    k = K[:, :, :n].double()
    s = torch.einsum("bhgid,bhjd->bhgij", q, k) / math.sqrt(D)
    hide = torch.arange(n, device=DEV) > (q0 + torch.arange(nq, device=DEV))[:, None]
    p = torch.softmax(s.masked_fill(hide, -math.inf), -1)
    sum_abs = float(torch.einsum("bhgid,bhjd->bhgij", q.abs(), k.abs()).max())
    return p.sum((2, 3)), rel_bound(sum_abs, D, Hq // Hkv * nq)


PROMPTS = [  # Bt, Hq, Hkv, D, L, q_start, n_q
    (1, 1, 1, 64, 1, 0, 1), (1, 4, 2, 128, 2, 0, 2), (2, 8, 2, 64, 33, 0, 33), (1, 8, 1, 128, 127, 0, 127),
    (1, 4, 4, 128, 128, 0, 128), (2, 6, 2, 128, 129, 0, 129), (1, 32, 8, 128, 700, 0, 700), (1, 8, 2, 64, 1024, 0, 1024),
    (1, 7, 1, 128, 513, 0, 513), (1, 16, 2, 64, 1500, 1400, 100), (1, 8, 2, 128, 1000, 333, 1), (2, 4, 1, 128, 900, 100, 515),
    (3, 3, 3, 64, 650, 0, 300), (1, 8, 8, 128, 2049, 0, 2049), (1, 5, 1, 128, 1300, 640, 660),
]


@pytest.mark.parametrize("Bt,Hq,Hkv,D,L,q0,nq", PROMPTS)
def test_prompt_weights(Bt, Hq, Hkv, D, L, q0, nq):
    Q, K = randn((Bt, Hq, nq, D), 1, 1.5), randn((Bt, Hkv, L, D), 2, 1.5)
    n = q0 + nq
    ref, rel = ref_prompt(Q, K, q0)
    K[:, :, n:] = float("nan")                         # keys behind the last query are not looked at
    got = qp.prompt_weights(Q, K, q0)
    assert got.shape == (Bt, Hkv, L)
    err = ((got[:, :, :n].double() - ref).abs() / ref).max()
    assert float(err) <= rel, (float(err), rel)
    assert torch.all(got[:, :, n:] == 0)
    assert torch.equal(got, qp.prompt_weights(Q, K, q0))          # same inputs, same bits


def test_prompt_weights_of_chunks_add_up_to_the_whole():
    Bt, Hq, Hkv, D, L = 2, 8, 2, 128, 1111
    Q, K = randn((Bt, Hq, L, D), 3, 1.5), randn((Bt, Hkv, L, D), 4, 1.5)
    ref, rel = ref_prompt(Q, K, 0)
    w = None
    for lo, hi in ((0, 500), (500, 501), (501, 1024), (1024, 1111)):
        behind = None if w is None else w[:, :, hi:].clone()
        w = qp.prompt_weights(Q[:, :, lo:hi].contiguous(), K, lo, weights=w)
        if behind is not None:
            assert torch.equal(w[:, :, hi:], behind)              # positions behind the chunk are left as they were
    assert float(((w.double() - ref).abs() / ref).max()) <= rel + 4 * 2.0 ** -24


def test_prompt_weights_of_peaked_and_constant_rows():
    Bt, Hq, Hkv, D, L = 1, 4, 1, 128, 640
    Q, K = randn((Bt, Hq, L, D), 5, 12.0), randn((Bt, Hkv, L, D), 6, 12.0)     # logits up to several thousand
    got = qp.prompt_weights(Q, K)
    assert torch.isfinite(got).all()
    sum_abs = float((Q.double().abs() @ K.double().abs().transpose(2, 3)).max())
    assert abs(float(got.double().sum()) - Hq * L) <= Hq * L * rel_bound(sum_abs, D, Hq * L)     # every row gives 1
    got = qp.prompt_weights(torch.zeros_like(Q), K)                            # closed form: row i gives 1 / (i + 1)
    ref = Hq * torch.flip(torch.cumsum(torch.flip(1.0 / torch.arange(1, L + 1, dtype=torch.float64), [0]), 0), [0])
    assert float(((got[0, 0].double().cpu() - ref) / ref).abs().max()) <= rel_bound(0.0, D, Hq * L)
    K[:, :, 600] = float("inf")                                                # only rows from 600 on see this key
    head = qp.prompt_weights(Q[:, :, :600].contiguous(), K)
    assert torch.isfinite(head).all() and torch.all(head[:, :, 600:] == 0)


# ---------------------------------------------------------------------------------------------- decode

def per_token_cache(Bt, Hq, Hkv, D, n, cap, bits, g, seed=0, scale=1.0):
    """(cache, strategy, keys and values that the codes stand for in 64 bits)"""
    K, V = randn((Bt, Hkv, n, D), seed + 11, scale), randn((Bt, Hkv, n, D), seed + 12)
    kept = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, Hkv, n).contiguous()
    cache = qp.alloc_cache(Bt, Hq, Hkv, D, bits, g, n, DEV, cap if cap != n else 0)
    if bits == 16:
        for t in (cache.k_codes, cache.v_codes):
            t.fill_(float("nan"))                                  # room behind the tokens may hold anything
        qp.gather_quantize(K, V, kept, cache)
        return cache, None, K.double(), V.double()
    st = qp.make_strategy(cache, 1)
    qp.gather_quantize_ex(K, V, kept, cache, st)
    both = [unpack(*x, bits).reshape(Bt, Hkv, cap, D)[:, :, :n] for x in
            ((cache.k_codes, cache.k_scale, cache.k_zero), (cache.v_codes, cache.v_scale, cache.v_zero))]
    return cache, st, *both


def unpack(words, scale, zero, bits):
    """what the codes stand for, fp64, in the order of the arrays"""
    sh = bits * torch.arange(32 // bits, device=DEV)
    c = ((words.long()[..., None] >> sh) & (2 ** bits - 1)).flatten(-2).double()
    return (c * scale.double()[..., None] + zero.double()[..., None]).flatten(-2)


def ref_decode(q, k, v):
    Bt, Hq, D = q.shape
    Hkv = k.shape[1]
    x = q.double().view(Bt, Hkv, Hq // Hkv, D)
    p = torch.softmax(torch.einsum("bhgd,bhnd->bhgn", x, k) / math.sqrt(D), -1)
    out = torch.einsum("bhgn,bhnd->bhgd", p, v).view(Bt, Hq, D)
    spread = torch.einsum("bhgn,bhnd->bhgd", p, v.abs()).view(Bt, Hq, D)
    sum_abs = float(torch.einsum("bhgd,bhnd->bhgn", x.abs(), k.abs()).max())
    return out, spread, p.sum(2), sum_abs


def check_decode(q, out, w0, w1, k, v, n):
    ref, spread, p, sum_abs = ref_decode(q, k, v)
    # keys of a packed cache are code * scale + zero with terms up to three times the value: see the factor
    rel = rel_bound(3 * sum_abs, q.shape[-1])
    err = (w1[:, :, :n].double() - w0[:, :, :n].double() - p).abs()
    assert torch.all(err <= rel * p + 2.0 ** -23 * w1[:, :, :n].double()), float((err / p).max())
    assert torch.equal(w1[:, :, n:].view(torch.int32), w0[:, :, n:].view(torch.int32))
    # output: its own rounding (2^-8), the weights rounded to 16 bits (2^-8) and times the scale (2^-11), values in fp16 (2^-11)
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -10 + rel) * spread + 1e-6
    assert torch.all((out.double() - ref).abs() <= tol), float(((out.double() - ref).abs() / tol).max())


DECODES = [  # Bt, Hq, Hkv, D, n, cap, bits, g
    (1, 1, 1, 64, 1, 1, 16, 32), (1, 8, 1, 128, 2, 9, 16, 32), (2, 32, 8, 128, 31, 31, 16, 32), (1, 32, 8, 128, 512, 512, 16, 32),
    (2, 14, 2, 128, 777, 800, 16, 64), (3, 6, 2, 64, 1025, 1025, 16, 32), (1, 64, 8, 128, 5001, 5120, 16, 128),
    (1, 4, 1, 128, 32, 32, 4, 32), (1, 32, 8, 128, 2048, 2048, 4, 32), (2, 8, 1, 128, 640, 768, 4, 64), (1, 8, 2, 128, 896, 896, 4, 128),
    (1, 8, 2, 64, 1024, 1024, 4, 32), (2, 6, 2, 64, 192, 192, 4, 64), (1, 32, 8, 128, 1024, 1024, 8, 32), (1, 7, 1, 128, 320, 320, 8, 64),
    (2, 4, 4, 64, 96, 96, 8, 32), (1, 8, 1, 128, 256, 256, 8, 128), (1, 32, 8, 128, 4096, 4096, 2, 32), (1, 16, 2, 128, 448, 448, 2, 64),
    (1, 3, 3, 64, 320, 320, 2, 32), (1, 8, 2, 128, 384, 384, 2, 128), (8, 32, 8, 128, 1056, 1056, 4, 32),
]


LONG = [  # the logits of a block's run do not fit its shared memory
    (1, 32, 8, 128, 30001, 30016, 16, 32), (1, 8, 1, 64, 20000, 20000, 16, 32), (1, 32, 8, 128, 26656, 26656, 4, 32), (1, 16, 2, 64, 16384, 16384, 8, 64),
    (20, 40, 5, 128, 4100, 4100, 16, 32),
]


@pytest.mark.parametrize("Bt,Hq,Hkv,D,n,cap,bits,g", DECODES + LONG)
def test_decode_attn_weights(Bt, Hq, Hkv, D, n, cap, bits, g):
    cache, st, k, v = per_token_cache(Bt, Hq, Hkv, D, n, cap, bits, g)
    q = randn((Bt, Hq, D), 7, 1.5)
    w = torch.rand((Bt, Hkv, cap), device=DEV) * (torch.rand((Bt, Hkv, cap), device=DEV) < 0.5)
    w[:, :, n:] = float("nan")
    w0 = w.clone()
    out = qp.decode_attn_weights(q, cache, w, st)
    check_decode(q, out, w0, w, k, v, n)
    w2 = w0.clone()
    assert torch.equal(out, qp.decode_attn_weights(q, cache, w2, st)) and torch.equal(w2.view(torch.int32), w.view(torch.int32))


def test_decode_attn_weights_with_large_logits():
    """Logits of several hundred: one token takes everything, nothing overflows."""
    cache, st, k, v = per_token_cache(1, 8, 2, 128, 512, 512, 4, 32, seed=3, scale=8.0)
    q = randn((1, 8, 128), 8, 16.0)
    w = torch.zeros((1, 2, 512), device=DEV)
    out = qp.decode_attn_weights(q, cache, w, st)
    assert torch.isfinite(out).all() and torch.isfinite(w).all()
    assert abs(float(w.double().sum()) - 8) <= 1e-4


# ---------------------------------------------------------------------------------------------- selection

@pytest.mark.parametrize("Bt,Hkv,L,w,n,cap", [(1, 1, 2, 1, 2, 2), (2, 3, 65, 1, 2, 5), (1, 2, 4096, 32, 512, 512), (2, 8, 5000, 8, 4999, 5000),
                                              (1, 8, 33000, 33, 8192, 8200), (8, 8, 9000, 32, 1024, 1100), (1, 1, 140000, 64, 1000, 1000),
                                              (1, 4, 300, 32, 300, 300)])
@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_heavy_select(Bt, Hkv, L, w, n, cap, kind):
    g = torch.Generator().manual_seed(L + n)
    x = torch.rand((Bt, Hkv, L), generator=g) if kind == "spread" else torch.randint(0, 3, (Bt, Hkv, L), generator=g).float()
    order = torch.sort(x[:, :, :L - w], dim=-1, descending=True, stable=True).indices[:, :, :n - w]
    kept = torch.cat([torch.sort(order, -1).values, torch.arange(L - w, L).expand(Bt, Hkv, w)], -1)
    got, kw, kp = qp.heavy_select(x.to(DEV), w, n, cap)
    assert torch.equal(got.cpu().long(), kept)
    assert torch.equal(kw.cpu()[:, :, :n], torch.gather(x, 2, kept)) and torch.all(kw[:, :, n:] == 0)
    assert torch.equal(kp.cpu()[:, :, :n].long(), kept) and torch.all(kp[:, :, n:] == 0)


# ---------------------------------------------------------------------------------------------- replacement

def half_toward(x, up):
    """fp16 next to the fp32 values x, upward or downward, by numpy's neighbours"""
    x = x.cpu().numpy().astype(np.float32)
    h = x.astype(np.float16)
    off = h.astype(np.float32) < x if up else h.astype(np.float32) > x
    return np.where(off, np.nextafter(h, np.float16(np.inf if up else -np.inf)), h)


def ref_row(kn, vn, bits, g):
    """(k codes, v codes, k scale, k zero, v scale, v zero) of one row, groups of g channels, from the definition in 32 bits"""
    def side(x):
        x = x.float().view(*x.shape[:2], -1, g).cpu()
        z = half_toward(x.amin(-1), False)
        zf = torch.from_numpy(z.astype(np.float32))
        top = np.float32(2 ** bits - 1)
        s = half_toward((x.amax(-1) - zf) * torch.tensor(np.float32(1) / top), True)
        sf = torch.from_numpy(s.astype(np.float32))[..., None]
        c = torch.where(sf > 0, torch.round((x - zf[..., None]) / torch.where(sf > 0, sf, torch.ones_like(sf))), torch.zeros_like(x))
        c = c.clamp(0, float(top)).long().view(*x.shape[:3], -1, 32 // bits)
        words = (c << (bits * torch.arange(32 // bits))).sum(-1)
        words = (words - ((words >> 31) << 32)).int()
        return [words.to(DEV)], [torch.from_numpy(s).to(DEV), torch.from_numpy(z).to(DEV)]
    (kc, km), (vc, vm) = side(kn), side(vn)
    return kc + vc + km + vm


def ref_slot(w, pos, new, recent):
    """[Bt,Hkv] slots from the definition, on the host"""
    out = torch.zeros(w.shape[:2], dtype=torch.int32)
    for b in range(w.shape[0]):
        for h in range(w.shape[1]):
            cand = [(float(w[b, h, t]), t) for t in range(w.shape[2]) if int(pos[b, h, t]) <= new - recent]
            out[b, h] = min(cand)[1] if cand else min((int(pos[b, h, t]), t) for t in range(w.shape[2]))[1]
    return out


@pytest.mark.parametrize("Bt,Hq,Hkv,D,n,bits,g,recent", [
    (1, 1, 1, 64, 1, 16, 32, 0), (1, 1, 1, 64, 1, 16, 32, 5), (2, 8, 2, 128, 33, 16, 32, 8), (1, 32, 8, 128, 512, 16, 32, 32),
    (1, 8, 2, 128, 300, 16, 64, 10 ** 6), (2, 4, 4, 128, 64, 4, 32, 16), (1, 8, 2, 64, 96, 4, 32, 1), (2, 8, 1, 128, 128, 2, 64, 40),
    (1, 8, 2, 128, 256, 8, 128, 100), (1, 8, 8, 64, 320, 8, 64, 3), (1, 4, 2, 128, 3008, 2, 32, 300)])
@pytest.mark.parametrize("ties", [False, True])
def test_evict_kv(Bt, Hq, Hkv, D, n, bits, g, recent, ties):
    cache, st, _, _ = per_token_cache(Bt, Hq, Hkv, D, n, n, bits, g)
    gen = torch.Generator().manual_seed(n + bits)
    w = torch.randint(0, 2, (Bt, Hkv, n), generator=gen).float() if ties else torch.rand((Bt, Hkv, n), generator=gen)
    if ties:
        w[w == 0] = -0.0                                            # -0 and +0 are equal
        w[:, :, ::3] = w[:, :, ::3].abs()
    pos = torch.argsort(torch.rand((Bt, Hkv, n), generator=gen), -1).int()
    wd, pd = w.to(DEV), pos.to(DEV)
    before = [None if t is None else t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.k_zero, cache.v_scale, cache.v_zero)]
    kn, vn = randn((Bt, Hkv, D), 21, 3.0), randn((Bt, Hkv, D), 22)
    slots = qp.evict_kv(kn, vn, cache, wd, pd, n, recent, st)
    ref = ref_slot(w, pos, n, recent)
    assert torch.equal(slots.cpu(), ref)
    # the row as the definition stores it, everything else untouched
    b, h = torch.meshgrid(torch.arange(Bt), torch.arange(Hkv), indexing="ij")
    got = (cache.k_codes, cache.v_codes, cache.k_scale, cache.k_zero, cache.v_scale, cache.v_zero)
    rows = (kn, vn) if bits == 16 else ref_row(kn, vn, bits, g)
    for new, old, s in zip(got, before, rows):
        want = old.clone().view(Bt, Hkv, n, -1)                    # per-token arrays: [Bt,Hkv,n, ...] whatever their nominal shape
        want[b, h, ref.long()] = s.view(Bt, Hkv, -1)
        assert torch.equal(new.view(Bt, Hkv, n, -1), want)
    w[b, h, ref.long()], pos[b, h, ref.long()] = 0.0, n
    assert torch.equal(wd.cpu().view(torch.int32), w.view(torch.int32)) and torch.equal(pd.cpu(), pos)


def test_a_16_bit_cache_grows_before_it_evicts():
    Bt, Hq, Hkv, D, n, cap = 2, 8, 2, 128, 30, 32
    cache, _, k, v = per_token_cache(Bt, Hq, Hkv, D, n, cap, 16, 32)
    w, pos = torch.rand((Bt, Hkv, cap), device=DEV), torch.arange(cap, dtype=torch.int32, device=DEV).expand(Bt, Hkv, cap).contiguous()
    for step in range(4):
        kn, vn = randn((Bt, Hkv, D), 30 + step), randn((Bt, Hkv, D), 40 + step)
        s = qp.evict_kv(kn, vn, cache, w, pos, 100 + step, 2)
        if step < 2:
            assert torch.all(s == n + step) and cache.desc.n_keep == n + step + 1
        else:
            # tokens 100 and 101 carry no weight yet and are just outside the two last positions (101, 102 and 102, 103)
            assert cache.desc.n_keep == cap and torch.all(s == n + step - 2)
        b, h = torch.meshgrid(torch.arange(Bt, device=DEV), torch.arange(Hkv, device=DEV), indexing="ij")
        assert torch.equal(cache.k_codes[b, h, s.long()], kn) and torch.all(w[b, h, s.long()] == 0)
        assert torch.all(pos[b, h, s.long()] == 100 + step)


# ---------------------------------------------------------------------------------------------- together

@pytest.mark.parametrize("bits", [16, 4])
def test_generation_at_a_fixed_budget(bits):
    """Prompt, selection, then steps: every stage against the definition on the state that the stage before left."""
    Bt, Hq, Hkv, D, L, n, recent = 2, 8, 2, 128, 700, 128, 32
    K, V, Q = randn((Bt, Hkv, L, D), 51, 1.5), randn((Bt, Hkv, L, D), 52), randn((Bt, Hq, L, D), 53, 1.5)
    hc = qp.compress_layer_heavy(K, V, Q, n * bits, bits, 32, recent)
    ref, rel = ref_prompt(Q, K, 0)
    kept = hc.pos.long()
    assert torch.all(kept[:, :, -recent:] == torch.arange(L - recent, L, device=DEV))
    got = torch.gather(ref, 2, kept)
    assert float(((hc.weights.double() - got).abs() / got).max()) <= rel
    kth = torch.sort(ref[:, :, :L - recent], -1, descending=True).values[:, :, n - recent - 1]
    assert torch.all(got[:, :, :-recent].amin(-1) >= kth * (1 - 2 * rel))
    for step in range(6):
        w0, p0 = hc.weights.clone(), hc.pos.clone()
        kn, vn, q = randn((Bt, Hkv, D), 60 + step, 1.5), randn((Bt, Hkv, D), 70 + step), randn((Bt, Hq, D), 80 + step, 1.5)
        out = qp.decode_step_heavy(q, kn, vn, hc, recent)
        slot = ref_slot(w0.cpu(), p0.cpu(), L + step, recent).to(DEV).long()
        b, h = torch.meshgrid(torch.arange(Bt, device=DEV), torch.arange(Hkv, device=DEV), indexing="ij")
        w0[b, h, slot], p0[b, h, slot] = 0.0, L + step
        assert torch.equal(hc.pos, p0)
        if bits == 16:
            k, v = hc.cache.k_codes.double(), hc.cache.v_codes.double()
            assert torch.equal(hc.cache.k_codes[b, h, slot], kn)
        else:
            c = hc.cache
            k, v = unpack(c.k_codes, c.k_scale, c.k_zero, bits), unpack(c.v_codes, c.v_scale, c.v_zero, bits)
            k, v = k.view(Bt, Hkv, n, D), v.view(Bt, Hkv, n, D)
        check_decode(q, out, w0, hc.weights, k, v, n)
    assert hc.next_pos == L + 6


@pytest.mark.parametrize("bits", [16, 8])
def test_steps_from_a_graph_and_on_another_stream(bits):
    """A captured step replays to the bits of the eager one; two graphs that share a workspace run one after the other."""
    Bt, Hq, Hkv, D, n = 1, 32, 8, 128, 512
    mk = lambda: per_token_cache(Bt, Hq, Hkv, D, n, n, bits, 32, seed=5)
    (c1, s1, _, _), (c2, s2, _, _) = mk(), mk()
    w = torch.rand((Bt, Hkv, n), device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, Hkv, n).contiguous()
    state = [(w.clone(), pos.clone()) for _ in range(2)]
    kn, vn, q = randn((Bt, Hkv, D), 90), randn((Bt, Hkv, D), 91), randn((Bt, Hq, D), 92)
    ws = qp.new_decode_workspace(qp.decode_weights_workspace_bytes(c1), DEV)

    def step(c, s, wp, out, slots):
        qp.evict_kv(kn, vn, c, wp[0], wp[1], n, 32, s, slots)
        qp.decode_attn_weights(q, c, wp[0], s, out, ws)

    o1, o2 = torch.empty_like(q), torch.empty_like(q)
    sl = torch.empty((Bt, Hkv), dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step(c1, s1, state[0], o1, sl)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c2, s2, state[1], o2, sl)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o1, o2) and torch.equal(state[0][0], state[1][0]) and torch.equal(state[0][1], state[1][1])
    assert torch.equal(c1.k_codes, c2.k_codes) and torch.equal(c1.v_codes, c2.v_codes)
    Q, K = randn((1, 8, 300, 128), 93), randn((1, 2, 300, 128), 94)
    ref = qp.prompt_weights(Q, K)
    out = torch.zeros_like(ref)
    pws = torch.empty(qp.prompt_weights_workspace_bytes(1, 8, 2, 128, 300, 0, 300), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qp.prompt_weights(Q, K, weights=out, workspace=pws)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ref + ref)


# ---------------------------------------------------------------------------------------------- long arrays

def spread_out(cache, n_cap):
    """The same tokens in arrays with room for n_cap tokens per head (what lies behind them is not finite)."""
    d = cache.desc
    big = qp.alloc_cache(d.batch, d.n_q_heads, d.n_kv_heads, d.head_dim, d.bits, d.group, d.n_keep, DEV, n_cap)
    n = d.n_keep
    for name in ("k_codes", "v_codes", "k_scale", "k_zero", "v_scale", "v_zero"):
        src, dst = getattr(cache, name), getattr(big, name)
        if src is None:
            continue
        dst = dst.view(d.batch, d.n_kv_heads, n_cap, -1)            # per-token arrays
        dst.view(torch.int16).fill_(0x7fc0 if d.bits == 16 else 0x7e00)
        dst[:, :, :n] = src.view(d.batch, d.n_kv_heads, n, -1)
    return big


@pytest.mark.parametrize("bits,Bt,n_cap", [(16, 20, 131072), (4, 20, 1 << 20)])
def test_strides_past_32_bits(bits, Bt, n_cap):
    """Offsets beyond 2^32 bytes: bit for bit what the same tokens give in short arrays."""
    Hq, Hkv, D, n = 16, 8, 128, 320
    cache, st, _, _ = per_token_cache(Bt, Hq, Hkv, D, n, n, bits, 32)
    big = spread_out(cache, n_cap)
    assert big.k_codes.numel() * big.k_codes.element_size() > 2 ** 32
    q = randn((Bt, Hq, D), 7, 1.5)
    w, wb = torch.zeros((Bt, Hkv, n), device=DEV), torch.zeros((Bt, Hkv, n_cap), device=DEV)
    out = qp.decode_attn_weights(q, cache, w, st)
    assert torch.equal(out, qp.decode_attn_weights(q, big, wb, st)) and torch.equal(w, wb[:, :, :n])
    T = 9
    qt, kd, vd = randn((Bt, T, Hq, D), 8), randn((Bt, T, Hkv, D), 9), randn((Bt, T, Hkv, D), 10)
    mask = qp.tree_mask((torch.arange(T, device=DEV) - 1).expand(Bt, T))
    assert torch.equal(qp.decode_attn_tree(qt, cache, kd, vd, mask, strategy=st), qp.decode_attn_tree(qt, big, kd, vd, mask, strategy=st))
    if bits < 16:                                                  # (a 16-bit cache with room would grow instead)
        pos = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, Hkv, n).contiguous()
        pb = torch.zeros((Bt, Hkv, n_cap), dtype=torch.int32, device=DEV)
        pb[:, :, :n] = pos
        kn, vn = randn((Bt, Hkv, D), 11), randn((Bt, Hkv, D), 12)
        s, sb = qp.evict_kv(kn, vn, cache, w, pos, n, 8, st), qp.evict_kv(kn, vn, big, wb, pb, n, 8, st)
        assert torch.equal(s, sb) and torch.equal(pos, pb[:, :, :n])
        for name in ("k_codes", "v_codes", "k_scale", "v_zero"):
            a, b = getattr(cache, name), getattr(big, name)
            assert torch.equal(a.view(Bt, Hkv, n, -1), b.view(Bt, Hkv, n_cap, -1)[:, :, :n])


def test_prompt_rows_past_32_bits():
    """Keys of the last heads lie beyond 2^32 bytes: the same weights as in an array of their own."""
    Bt, Hq, Hkv, D, L, nq = 34, 4, 4, 128, 131072, 130
    K = torch.zeros((Bt, Hkv, L, D), dtype=torch.bfloat16, device=DEV)
    small = randn((Bt, Hkv, 300, D), 1, 1.5)
    K[:, :, :300] = small
    Q = randn((Bt, Hq, nq, D), 2, 1.5)
    assert K.numel() * 2 > 2 ** 32
    assert torch.equal(qp.prompt_weights(Q, K, 100)[:, :, :300], qp.prompt_weights(Q, small, 100))


def test_prompt_rows_of_other_heads_do_not_matter():
    """A head's last tile of queries reaches into the next head's rows, its last keys into the next head's keys: NaN there stays there."""
    Bt, Hq, Hkv, D, L, q0, nq = 2, 8, 2, 128, 300, 70, 200
    Q, K = randn((Bt, Hq, nq, D), 1, 1.5), randn((Bt, Hkv, L, D), 2, 1.5)
    ref = qp.prompt_weights(Q, K, q0)
    for poison in (float("nan"), float("inf")):
        Q2, K2 = Q.clone(), K.clone()
        Q2[1], K2[1] = poison, poison
        K2[:, :, q0 + nq:] = poison                                     # keys that no query sees
        assert torch.equal(qp.prompt_weights(Q2, K2, q0)[0], ref[0])
        Q2, K2 = Q.clone(), K.clone()
        Q2[0], K2[0] = poison, poison
        assert torch.equal(qp.prompt_weights(Q2, K2, q0)[1], ref[1])


FIRST_CALLS = """
import torch
from paper_2412_12706_b200 import qp
torch.manual_seed(1)
r = lambda *s: torch.randn(s, device="cuda").bfloat16()
Bt, Hq, Hkv, D, L, n, T = 1, 8, 2, 64, 700, 128, 9
c = qp.alloc_cache(Bt, Hq, Hkv, D, 8, 32, n, "cuda")
c16 = qp.alloc_cache(Bt, Hq, Hkv, D, 16, 32, n, "cuda")
for t in (c.k_codes, c.v_codes, c16.k_codes, c16.v_codes, c.k_scale, c.k_zero, c.v_scale, c.v_zero):
    t.zero_()
st = qp.make_strategy(c, 1)
Q, K, q, kd, vd, kn = r(Bt, Hq, L, D), r(Bt, Hkv, L, D), r(Bt, T, Hq, D), r(Bt, T, Hkv, D), r(Bt, T, Hkv, D), r(Bt, Hkv, D)
mask = torch.full((Bt, T), -1, dtype=torch.int64, device="cuda")
q1 = q[:, 0].contiguous()
w = [torch.zeros((Bt, Hkv, n), device="cuda") for _ in range(2)]
pos = torch.arange(n, dtype=torch.int32, device="cuda").expand(Bt, Hkv, n).contiguous()
def calls():
    a = qp.prompt_weights(Q, K)
    s = qp.heavy_select(a, 8, n)
    outs = [a, *s]
    for x, y in ((c, st), (c16, None)):
        outs += [qp.decode_attn_weights(q1, x, w[0], y), qp.decode_attn_tree(q, x, kd, vd, mask, strategy=y)]
    outs.append(qp.evict_kv(kn, kn, c, w[1], pos, n, 4, st))
    return outs
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = calls()
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in got]
for t in (c.k_codes, c.v_codes, c.k_scale, c.k_zero, c.v_scale, c.v_zero, *w):
    t.zero_()
pos.copy_(torch.arange(n, dtype=torch.int32, device="cuda").expand(Bt, Hkv, n))
for a, b in zip(got, calls()):
    assert torch.equal(a, b)
print("same")
"""


def test_first_calls_of_a_process_are_captured():
    """Every operator's first call, with what it sets up once, under capture; the replay gives what eager calls give."""
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=300,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
