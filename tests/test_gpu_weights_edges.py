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


# ---------------------------------------------------------------------------------------------- runs of calls

def overlapping_run(alone, steps=70):
    """Every call of a generation loop reads what the call before it wrote, on a stream whose decode calls may overlap.  alone: the
    GPU is waited for after every call.  (The setting itself stays: a decode call cuts its work by it, so its last bits differ.)"""
    done = torch.cuda.synchronize if alone else lambda: None
    Bt, H, D, n, g = 2, 4, 128, 512, 32
    r = lambda *shape, seed: randn(shape, seed)
    K, V = r(Bt, H, n, D, seed=1), r(Bt, H, n, D, seed=2)
    kept = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, H, n).contiguous()
    X = qp.alloc_cache(Bt, H, H, D, 4, g, n, DEV, n + 3 * g)
    for t in (X.k_codes, X.v_codes, X.k_scale, X.k_zero, X.v_scale, X.v_zero):
        t.zero_()
    qp.gather_quantize(K, V, kept, X)
    tail = qp.alloc_tail(X)
    held = []
    for bits in (8, 16):
        Y = qp.alloc_cache(Bt, H, H, D, bits, g, n, DEV, n + 40 if bits == 16 else 0)
        st = None
        if bits == 16:
            Y.k_codes.zero_(); Y.v_codes.zero_()
            qp.gather_quantize(K, V, kept, Y)
        else:
            st = qp.make_strategy(Y, 1)
            qp.gather_quantize_ex(K, V, kept, Y, st)
        cap = Y.desc.n_cap or n
        pos = torch.arange(cap, dtype=torch.int32, device=DEV).expand(Bt, H, cap).contiguous()
        held.append((Y, st, torch.rand((Bt, H, cap), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV), pos))
    size = max([qp.decode_workspace_bytes(X), qp.decode_tree_workspace_bytes(X, 1)] + [qp.decode_weights_workspace_bytes(Y[0]) for Y in held])
    ws = qp.new_decode_workspace(size, DEV)
    mask = torch.ones((Bt, 1), dtype=torch.int64, device=DEV)
    outs = [torch.empty((Bt, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(5 * steps)]
    slots = torch.empty((Bt, H), dtype=torch.int32, device=DEV)
    q = r(Bt, H, D, seed=4)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        qp.decode_overlap(True)
        for s in range(steps):
            a, b, c, d, e = outs[5 * s:5 * s + 5]
            qp.decode_attn(q, X, a, ws); done()
            for (Y, st, w, pos), kv, o in zip(held, (a, b), (b, c)):
                qp.evict_kv(kv, kv, Y, w, pos, 3 * n + s, 16, st, slots); done()
                qp.decode_attn_weights(kv, Y, w, st, o, ws); done()
            qp.append_kv(c, b, X, tail); done()
            qp.decode_attn_tree(c.view(Bt, 1, H, D), X, b.view(Bt, 1, H, D), a.view(Bt, 1, H, D), mask, tail, None, d.view(Bt, 1, H, D), ws)
            done()
            qp.decode_attn_tail(d, X, tail, e, ws); done()
            q = e
        qp.decode_overlap(False)
    torch.cuda.synchronize()
    state = [t for Y, _, w, pos in held for t in (Y.k_codes, Y.v_codes, w, pos)]
    return outs + state + [X.k_codes, X.v_codes, tail.k_tail, tail.v_tail]


def test_new_calls_among_decode_calls_that_may_overlap():
    ref = overlapping_run(True)
    assert all(torch.isfinite(t.float()).all() for t in ref)
    for _ in range(5):
        for i, (a, b) in enumerate(zip(ref, overlapping_run(False))):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("bits", [16, 4])
def test_steps_at_rising_positions_from_graphs(bits):
    """A captured step stands for the position it was captured at: one graph per step, replayed in order, gives the eager steps'
    bits, through growth (16 bit) and eviction."""
    Bt, Hq, Hkv, D, L, n, recent, steps = 2, 8, 2, 128, 500, 64, 16, 40
    K, V, Q = randn((Bt, Hkv, L, D), 1, 1.5), randn((Bt, Hkv, L, D), 2), randn((Bt, Hq, L, D), 3, 1.5)
    cap = n + 10 if bits == 16 else 0
    news = [(randn((Bt, Hq, D), 10 + s, 1.5), randn((Bt, Hkv, D), 100 + s), randn((Bt, Hkv, D), 200 + s)) for s in range(steps)]

    def state():
        hc = qp.compress_layer_heavy(K, V, Q, n * bits, bits, 32, recent, cap)
        return hc, torch.zeros((steps, Bt, Hq, D), dtype=torch.bfloat16, device=DEV)

    (e, eo), (c, co) = state(), state()
    ws = qp.new_decode_workspace(qp.decode_weights_workspace_bytes(e.cache), DEV)
    for s, (q, k, v) in enumerate(news):
        qp.decode_step_heavy(q, k, v, e, recent, eo[s], ws)
    torch.cuda.synchronize()
    graphs = []
    for s, (q, k, v) in enumerate(news):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            qp.decode_step_heavy(q, k, v, c, recent, co[s], ws)
        graphs.append(g)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    used = e.cache.desc.n_keep
    assert used == c.cache.desc.n_keep == (cap or n) and e.next_pos == c.next_pos == L + steps
    assert torch.equal(eo, co) and torch.equal(e.weights, c.weights) and torch.equal(e.pos, c.pos)
    assert torch.equal(e.cache.k_codes, c.cache.k_codes) and torch.equal(e.cache.v_codes, c.cache.v_codes)


def test_decode_attn_weights_where_one_token_takes_everything():
    """Logits of several hundred, against 64 bits: the token that wins, its weight and the output."""
    for bits in (16, 8, 4, 2):
        Bt, Hq, Hkv, D, n = 1, 8, 2, 128, 512
        K, V = randn((Bt, Hkv, n, D), 3, 8.0), randn((Bt, Hkv, n, D), 4)
        q = randn((Bt, Hq, D), 8, 16.0)
        if bits == 16:
            cache, st = qp.alloc_cache(Bt, Hq, Hkv, D, 16, 32, n, DEV), None
            qp.gather_quantize(K, V, torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, Hkv, n).contiguous(), cache)
            k, v, terms = K.double(), V.double(), V.double().abs()
        else:
            cache, st, k, cs, z = packed(K, V, Hq, bits, 32)
            v, terms = cs + z, cs.abs() + z.abs()
        w = torch.zeros((Bt, Hkv, n), device=DEV)
        out = qp.decode_attn_weights(q, cache, w, st).double().view(Bt, Hkv, Hq // Hkv, D)
        x = q.double().view(Bt, Hkv, Hq // Hkv, D)
        p = torch.softmax(torch.einsum("bhgd,bhnd->bhgn", x, k) / math.sqrt(D), -1)
        assert float(p.max()) > 0.99
        rel = rel_bound(3 * float(torch.einsum("bhgd,bhnd->bhgn", x.abs(), k.abs()).max()), D)
        assert torch.all((w.double() - p.sum(2)).abs() <= rel * p.sum(2) + 2.0 ** -100)      # (a weight below 2^-126 is 0)
        ref, spread = torch.einsum("bhgn,bhnd->bhgd", p, v), torch.einsum("bhgn,bhnd->bhgd", p, terms)
        tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 if bits == 16 else 2.0 ** -9) * spread + rel * spread + 1e-6
        assert torch.all((out - ref).abs() <= tol), (bits, float(((out - ref).abs() / tol).max()))


@pytest.mark.parametrize("bits,g,D", [(4, 32, 128), (4, 64, 64), (4, 128, 128), (8, 32, 128), (8, 64, 64), (2, 32, 128), (2, 64, 64)])
def test_an_evicted_row_beside_the_same_row_of_the_quantizer(bits, g, D):
    """The row that eviction stores and the row that qp_gather_quantize_ex stores of the same numbers.  The zero point is the same.
    The scale is the range times RN(1 / (2^B - 1)), which lies above 1 / (2^B - 1) for B = 2, 4, 8, so never below the quotient's and
    at most one fp16 step above it; codes are rounded against the stored scale, so every number comes back to half of it."""
    Bt, H, n = 4, 8, 256
    n = n // g * g
    K, V = randn((Bt, H, n, D), 5, 3.0), randn((Bt, H, n, D), 6, 0.2)
    kept = torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, H, n).contiguous()
    ref, got = [qp.alloc_cache(Bt, H, H, D, bits, g, n, DEV) for _ in range(2)]
    st = qp.make_strategy(ref, 1)
    qp.gather_quantize_ex(K, V, kept, ref, st)
    qp.gather_quantize_ex(V, K, kept, got, st)
    w, pos = torch.zeros((Bt, H, n), device=DEV), torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, H, n).contiguous()
    for t in range(n):                                             # every row gives its place to the other cache's
        s = qp.evict_kv(K[:, :, t].contiguous(), V[:, :, t].contiguous(), got, w, pos, n + t, n, st)
        assert torch.all(s == t)
    for x, side in ((K, "k"), (V, "v")):
        rows = lambda c, name: getattr(c, f"{side}_{name}").view(Bt, H, n, D // g, -1)
        assert torch.equal(rows(got, "zero"), rows(ref, "zero"))
        step = rows(got, "scale").view(torch.int16).int() - rows(ref, "scale").view(torch.int16).int()
        assert int(step.min()) >= 0 and int(step.max()) <= 1
        same = step[..., 0] == 0
        assert torch.equal(rows(got, "codes")[same], rows(ref, "codes")[same])
        back = unpack(getattr(got, f"{side}_codes"), getattr(got, f"{side}_scale"), getattr(got, f"{side}_zero"), bits).reshape(x.shape)
        half = 0.5 * rows(got, "scale").double().expand(Bt, H, n, D // g, g).reshape(x.shape)
        assert torch.all((back - x.double()).abs() <= half * (1 + 2.0 ** -10) + 2.0 ** -24 * x.double().abs())


@pytest.mark.parametrize("Hq,Hkv,D,L,q0,nq", [(8, 1, 128, 65536, 0, 65536), (4, 2, 64, 131072, 0, 131072), (8, 2, 128, 300001, 299000, 1001)])
def test_prompt_weights_of_long_prompts(Hq, Hkv, D, L, q0, nq):
    """Every row gives 1 in all; the last keys, which only the last rows see, against 64 bits."""
    Q, K = randn((1, Hq, nq, D), 1, 1.5), randn((1, Hkv, L, D), 2, 1.5)
    got = qp.prompt_weights(Q, K, q0).double()
    G, last = Hq // Hkv, 200
    sum_abs, ref = 0.0, []
    hide = torch.arange(L, device=DEV) > (L - last + torch.arange(last, device=DEV))[:, None]
    for h in range(Hkv):
        q, k = Q[0, h * G:(h + 1) * G, -last:].double(), K[0, h].double()
        p = torch.softmax((q @ k.T / math.sqrt(D)).masked_fill(hide, -math.inf), -1)
        ref.append(p.sum((0, 1))[-last:])
        sum_abs = max(sum_abs, float(Q[0, h * G:(h + 1) * G].double().abs().amax((0, 1)) @ k.abs().amax(0)))
    rel = rel_bound(sum_abs, D, G * nq)
    assert torch.all(((got[0, :, -last:] - torch.stack(ref)).abs() / torch.stack(ref)) <= rel)
    assert torch.all((got.sum(-1) - G * nq).abs() <= G * nq * rel)
