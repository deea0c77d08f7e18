"""Accumulated attention weights at the edges of their ranges: small and large values, queries that are not numbers, host threads."""
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2412_12706_b200 import qp
from tests.test_gpu_weights import DEV, randn, rel_bound, unpack

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------- sizes of values

def packed(K, V, Hq, bits, g):
    """(cache, strategy, keys, code * scale of the values, zero points of the values), the last three in 64 bits"""
    Bt, Hkv, n, D = K.shape
    kept = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, Hkv, n).contiguous()
    cache = qp.alloc_cache(Bt, Hq, Hkv, D, bits, g, n, DEV)
    st = qp.make_strategy(cache, 1)
    qp.gather_quantize_ex(K, V, kept, cache, st)
    k = unpack(cache.k_codes, cache.k_scale, cache.k_zero, bits).reshape(Bt, Hkv, n, D)
    cs = unpack(cache.v_codes, cache.v_scale, torch.zeros_like(cache.v_zero), bits).reshape(Bt, Hkv, n, D)
    z = cache.v_zero.double()[..., None].expand(*cache.v_zero.shape, g).reshape(Bt, Hkv, n, D)
    return cache, st, k, cs, z


def heavy_tokens(Bt, Hq, Hkv, D, n, seed):
    """Queries of a KV head that share a direction, and keys of which one in a hundred lies 8 nats along it."""
    along = randn((Bt, Hkv, 1, D), seed).double()
    G = Hq // Hkv
    q = (along + 0.1 * randn((Bt, Hkv, G, D), seed + 1).double()).reshape(Bt, Hq, D).to(torch.bfloat16)
    g = torch.Generator(device=DEV).manual_seed(seed + 2)
    heavy = (torch.rand((Bt, Hkv, n, 1), generator=g, device=DEV) < 0.01).double()
    k = 0.3 * randn((Bt, Hkv, n, D), seed + 3).double() + heavy * along * (8.0 * math.sqrt(D) / along.square().sum(-1, keepdim=True))
    return q, k.to(torch.bfloat16)


def values(kind, shape, seed):
    v = randn(shape, seed).double()
    n = shape[2]
    t = torch.arange(n, device=DEV)[:, None]
    if kind == "rising":                               # later tokens a hundred thousand times larger than the first
        v = v * 10.0 ** (-4 + 5.0 * t / n)
    elif kind == "falling":
        v = v * 10.0 ** (1 - 5.0 * t / n)
    elif kind == "one large token":                    # as large as the interface allows, in the middle of small ones
        v = v * 0.01
        v[:, :, n // 2] = 4000.0 * torch.sign(v[:, :, n // 2])
    elif kind == "constant":                           # every scale is 0
        v = torch.full_like(v, 0.03)
    else:
        v = v * float(kind)
    return v.to(torch.bfloat16)


@pytest.mark.parametrize("bits,g,D,Hq,Hkv", [(8, 32, 128, 32, 8), (8, 128, 128, 8, 1), (8, 64, 64, 8, 2), (4, 32, 128, 32, 8), (4, 64, 64, 6, 2),
                                             (2, 32, 128, 16, 2), (2, 128, 128, 8, 2), (2, 64, 64, 4, 4)])
@pytest.mark.parametrize("kind", ["0.01", "0.03", "0.001", "1", "300", "rising", "falling", "one large token", "constant"])
@pytest.mark.parametrize("n", [256, 8192])
def test_decode_attn_weights_of_small_and_large_values(bits, g, D, Hq, Hkv, kind, n):
    """Tolerance.  Output's own rounding 2^-8; a weight in fp16 is off by 2^-11 of it, its product with a scale by 2^-11 more, so by
    2^-10 (1 + 2^-10) of sum p (|code scale| + |zero|); a logit's error as in check_decode.  Below fp16's normal range errors are
    absolute, 2^-25: weights are held against a reference that leaves the heaviest of them at 2^top with top >= 15 - 5 for scales up
    to 1 (a weight's own 2^-25 is then 2^-35 of the normaliser for each token, the product's the same, times the largest code
    scale), and with top >= 15 - 5 - log2(scale) above, where only the weight's own grows with the scale, relative to it."""
    Bt = 1
    q, K = heavy_tokens(Bt, Hq, Hkv, D, n, 100 + bits)
    V = values(kind, (Bt, Hkv, n, D), 7)
    cache, st, k, cs, z = packed(K, V, Hq, bits, g)
    w = torch.zeros((Bt, Hkv, n), device=DEV)
    out = qp.decode_attn_weights(q, cache, w, st).double().view(Bt, Hkv, Hq // Hkv, D)
    x = q.double().view(Bt, Hkv, Hq // Hkv, D)
    p = torch.softmax(torch.einsum("bhgd,bhnd->bhgn", x, k) / math.sqrt(D), -1)
    sum_abs = float(torch.einsum("bhgd,bhnd->bhgn", x.abs(), k.abs()).max())
    rel = rel_bound(3 * sum_abs, D)
    assert torch.all((w.double() - p.sum(2)).abs() <= (rel + 2.0 ** -23) * p.sum(2))
    ref = torch.einsum("bhgn,bhnd->bhgd", p, cs + z)
    terms = torch.einsum("bhgn,bhnd->bhgd", p, cs.abs() + z.abs())
    top_scale = max(1.0, float(cache.v_scale.max()))
    largest = float(cs.abs().max()) + float(z.abs().max())
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -10 * (1 + 2.0 ** -10) + rel) * terms + 2 * n * 2.0 ** -35 * top_scale * largest + 1e-30
    worst = float(((out - ref).abs() / tol).max())
    assert worst <= 1, worst


@pytest.mark.parametrize("bits,g,D", [(8, 32, 128), (8, 64, 64), (8, 128, 128), (4, 32, 128), (4, 64, 64), (2, 32, 128), (2, 64, 64)])
@pytest.mark.parametrize("kind", ["0.01", "0.03", "0.003", "0.001", "1", "300", "rising", "falling", "one large token"])
def test_output_is_the_mean_of_the_values_under_the_weights_it_adds(bits, g, D, kind):
    """One query head per KV head, accumulators at zero: the weights left there are the output's own, so a logit's error is on both
    sides and what remains are the roundings of the second product (see above) and 2^-19 for two exponentials and the sums."""
    Bt, H, n = 2, 4, 8192
    q, K = heavy_tokens(Bt, H, H, D, n, 200 + bits)
    cache, st, _, cs, z = packed(K, values(kind, (Bt, H, n, D), 8), H, bits, g)
    w = torch.zeros((Bt, H, n), device=DEV)
    out = qp.decode_attn_weights(q, cache, w, st).double()
    p = w.double() / w.double().sum(-1, keepdim=True)
    ref = torch.einsum("bhn,bhnd->bhd", p, cs + z)
    terms = torch.einsum("bhn,bhnd->bhd", p, cs.abs() + z.abs())
    top_scale = max(1.0, float(cache.v_scale.max()))
    largest = float(cs.abs().max()) + float(z.abs().max())
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -10 * (1 + 2.0 ** -10) + 2.0 ** -19) * terms + 2 * n * 2.0 ** -35 * top_scale * largest + 1e-30
    worst = float(((out - ref).abs() / tol).max())
    assert worst <= 1, worst


# ---------------------------------------------------------------------------------------------- queries that are not numbers

@pytest.mark.parametrize("poison", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows", [(1, 130, 259, 388, 517, 646, 775, 896), (640,), (641,), (642,), (643,), (1022,), (1023,)])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (3, 3, 64)])
def test_a_query_that_is_not_finite_shows_in_every_key_it_sees(Hq, Hkv, D, rows, poison):
    """Whatever its row number: its softmax has no value, so neither have the weights up to its position; those behind do not change."""
    Bt, L = 2, 1024
    Q, K = randn((Bt, Hq, L, D), 1, 1.5), randn((Bt, Hkv, L, D), 2, 1.5)
    ref = qp.prompt_weights(Q, K)
    h = Hq - 1                                             # one query head of the last KV head, second batch entry
    Q[1, h, list(rows)] = poison
    got = qp.prompt_weights(Q, K)
    last = max(rows)
    assert torch.isnan(got[1, Hkv - 1, :last + 1]).all()
    assert torch.equal(got[1, Hkv - 1, last + 1:], ref[1, Hkv - 1, last + 1:])
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1, :Hkv - 1], ref[1, :Hkv - 1])


# ---------------------------------------------------------------------------------------------- host threads

THREADS = """
import threading
import torch
from paper_2412_12706_b200 import qp
from tests.test_gpu_tree import make_cache, mask_of, random_tree
from tests.test_gpu_weights import per_token_cache, randn
Bt, Hq, Hkv, D, n, T, N = 1, 8, 2, 128, 2048, 12, 6
caches = [per_token_cache(Bt, Hq, Hkv, D, n, n, bits, 32)[:2] for bits in (2, 4, 8, 16)]
q, qt, kd, vd = randn((Bt, Hq, D), 1), randn((Bt, T, Hq, D), 2), randn((Bt, T, Hkv, D), 3), randn((Bt, T, Hkv, D), 4)
mask = mask_of(random_tree(Bt, T, 5)[1])
Q, K = randn((Bt, Hq, 900, D), 6), randn((Bt, Hkv, 900, D), 7)
torch.cuda.synchronize()
gate, got, failed = threading.Barrier(N), [None] * N, []

def calls():
    out = []
    for c, st in caches:
        w = torch.zeros((Bt, Hkv, n), device="cuda")
        out += [qp.decode_attn_weights(q, c, w, st), w, qp.decode_attn_tree(qt, c, kd, vd, mask, strategy=st)]
    a = qp.prompt_weights(Q, K)
    return out + [a, *qp.heavy_select(a, 8, 128)]

def work(i):
    try:
        with torch.cuda.stream(torch.cuda.Stream()):
            gate.wait()
            got[i] = calls()
            torch.cuda.current_stream().synchronize()
    except Exception as e:
        failed.append(e)

threads = [threading.Thread(target=work, args=(i,)) for i in range(N)]
for t in threads: t.start()
for t in threads: t.join()
assert not failed, failed
ref = calls()
for g in got:
    for a, b in zip(g, ref):
        assert torch.equal(a, b)
print("same")
"""


def test_first_calls_of_several_host_threads_at_once():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for _ in range(3):
        r = subprocess.run([sys.executable, "-c", THREADS], capture_output=True, text=True, timeout=300, cwd=root)
        assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
