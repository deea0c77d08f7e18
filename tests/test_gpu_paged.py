"""The paged cache in 8 bits: appends bit for bit, attention against plain arithmetic in 64 bits over what the cache holds.

Tolerance of the attention.  Codes are exact operands; a query is exact in fp16 but for what lies below 2^-24 of twice its largest
channel.  A logit is a sum of D products in 32 bits, off by (D + 8) 2^-23 sum|q k| / sqrt(D), plus D 2^-24 max|q| max|k| / sqrt(D) for
the small channels; int8 codes enter as c + 128, so there |k| is |k| + 128 scale.  A weight is off by e^(2 e) - 1 of the largest such e,
by 2^-11 for its rounding to fp16 (and by as much in the sum it is divided by), by 2^-20 for the exponential, and by 2^-35 of the
heaviest weight where it is too small for fp16.  The sums over n tokens are in 32 bits, (n / 16 + 64) 2^-23.  All of that counts against
the weighted sum of |v| (int8: |v| + 128 scale); the output is rounded to bf16, 2^-8 of itself, or where it is subnormal half of the
smallest bf16 number, 2^-134 (and the sums then to multiples of 2^-149, together less than as much again).

Waiting values, like queries, are fp16 times the power of two that brings the largest of their block of 32 into [1, 2): a bf16 number has
8 bits, so it is exact from 2^-17 on, and below that rounded to a multiple of 2^-24, so off by at most 2^-25 of the largest; weights sum
to 1, so the output is off by as much."""
import math

import pytest
import torch

from paper_2412_12706_b200 import qp

pytestmark = pytest.mark.gpu
DEV = "cuda"
TOP = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
E4M3, INT8 = torch.float8_e4m3fn, torch.int8


def randn(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(shape, generator=g, device=DEV)).to(torch.bfloat16)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make(seqs, Hq, Hkv, D, page, dtype, longest, spare=3, seed=0):
    """A cache whose pool, scales and tails hold rubbish, and a page table in any order."""
    per = -(-longest // page)
    n_pages = seqs * per + spare
    c = qp.alloc_paged(seqs, Hq, Hkv, D, n_pages, per, page, dtype)
    for t in (c.k_codes, c.v_codes):
        t.view(torch.uint8).fill_(0x7f)                            # e4m3: not a number
    for t in (c.k_scale, c.v_scale, c.k_tail, c.v_tail):
        t.fill_(float("nan"))
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))[:seqs * per]
    return c, order.view(seqs, per).to(torch.int32).to(DEV)


def start_of(new):
    return ints([sum(new[:b]) for b in range(len(new) + 1)])


def stored(x, dtype):
    """(codes as floats, scale bf16) of blocks x [..., page, D] by the definition."""
    top = x.float().abs().amax((-2, -1))
    s = top / torch.full_like(top, TOP[dtype])
    s = ((s.view(torch.int32) + 0xffff) >> 16).to(torch.int16).view(torch.bfloat16)
    f = s.float()[..., None, None]
    y = x.float() * torch.where(f > 0, (torch.ones_like(f) / f).clamp(max=3.4028234663852886e38), torch.zeros_like(f))
    return (y.to(E4M3).float() if dtype is E4M3 else torch.round(y)), s


def check_cache(c, table, k, v, lens, dtype):
    """k, v: per sequence, rows [n, Hkv, D] as the cache takes them (rotated)."""
    page = c.desc.page
    for b, n in enumerate(lens):
        full = n // page
        for codes, scale, tail, x in ((c.k_codes, c.k_scale, c.k_tail, k[b]), (c.v_codes, c.v_scale, c.v_tail, v[b])):
            x = x[:n].transpose(0, 1)
            if full:
                ids = table[b, :full].long()
                want, s = stored(x[:, :full * page].reshape(x.shape[0], full, page, -1).transpose(0, 1), dtype)
                got = codes.view(torch.uint8)[ids].view(dtype).float()
                assert torch.equal(scale[ids], s), (b, "scale")
                assert torch.equal(got, want), (b, "codes", int((got != want).sum()))
            assert torch.equal(tail[b, :, :n - full * page], x[:, full * page:]), (b, "tail")


APPENDS = [  # Hq, Hkv, D, page, dtype, rotation (rot, interleaved) or None, steps of new tokens per sequence
    (8, 2, 128, 32, E4M3, (128, False), [[1, 5, 0], [31, 27, 64], [1, 1, 1], [70, 0, 129], [1, 1, 1]]),
    (4, 4, 64, 64, INT8, None, [[64], [1], [62], [1], [1], [200]]),
    (6, 2, 128, 128, INT8, (64, True), [[127, 128, 1], [1, 1, 126], [1, 1, 1], [300, 1, 5]]),
    (8, 1, 64, 32, E4M3, (22, False), [[33, 1], [30, 31], [1, 1], [1, 1], [100, 31]]),
    (2, 2, 128, 64, E4M3, None, [[0, 3], [63, 0], [1, 61], [0, 1]]),
    (8, 8, 64, 128, E4M3, (64, False), [[1000], [24], [1], [127]]),
]


@pytest.mark.parametrize("Hq,Hkv,D,page,dtype,rot,steps", APPENDS)
def test_append(Hq, Hkv, D, page, dtype, rot, steps):
    seqs = len(steps[0])
    total = [sum(s[b] for s in steps) for b in range(seqs)]
    c, table = make(seqs, Hq, Hkv, D, page, dtype, max(total))
    rope = None if rot is None else qp.rope(rot[0], 500000.0, rot[1], "bands", 8.0)
    wide = [randn((n, Hkv + 3, D), 10 + b) for b, n in enumerate(total)]       # rows of a fused projection
    v = [randn((n, Hkv, D), 20 + b, 3.0) for b, n in enumerate(total)]
    q = [randn((n, Hq, D), 30 + b) for b, n in enumerate(total)]
    turn = lambda x, n0: qp.rotary(x.transpose(0, 1)[None], torch.arange(n0, n0 + x.shape[0], device=DEV, dtype=torch.int32), rope)[0].transpose(0, 1)
    k = [w[:, 1:Hkv + 1] if rope is None else turn(w[:, 1:Hkv + 1], 0) for w in wide]
    lens = [0] * seqs
    used = {int(i) for b in range(seqs) for i in table[b, :total[b] // page]}
    for new in steps:
        rows = lambda x: torch.cat([x[b][lens[b]:lens[b] + new[b]] for b in range(seqs)])
        kw = torch.cat([wide[b][lens[b]:lens[b] + new[b]] for b in range(seqs)])[:, 1:Hkv + 1]
        step = qp.PagedStep(start_of(new), ints(lens), table, sum(new), max(new))
        qr = qp.paged_append(kw, rows(v), c, step, rope, q=rows(q) if rope else None)
        if rope:
            assert torch.equal(qr, torch.cat([turn(q[b][lens[b]:lens[b] + new[b]], lens[b]) for b in range(seqs) if new[b]]))
        lens = [a + n for a, n in zip(lens, new)]
        check_cache(c, table, k, v, lens, dtype)
    for i in range(c.desc.n_pages):                                # pages of nobody are left as they were
        if i not in used:
            assert (c.k_codes[i].view(torch.uint8) == 0x7f).all() and torch.isnan(c.k_scale[i]).all()


def test_a_page_holds_the_same_however_its_tokens_came():
    Hkv, D, page, n = 2, 128, 64, 400
    k, v = randn((n, Hkv, D), 1), randn((n, Hkv, D), 2)
    rope = qp.rope(128)
    seen = []
    for cuts in ([400], [1] * 400, [63, 1, 64, 65, 7, 200], [129, 271]):
        c, table = make(1, 4, Hkv, D, page, E4M3, n, seed=3)
        at = 0
        for m in cuts:
            qp.paged_append(k[at:at + m], v[at:at + m], c, qp.PagedStep(ints([0, m]), ints([at]), table, m, m), rope)
            at += m
        ids = table[0, :n // page].long()
        seen.append([t.view(torch.uint8)[ids] for t in (c.k_codes, c.v_codes)] + [t[ids] for t in (c.k_scale, c.v_scale)] +
                    [t[:, :, :n % page] for t in (c.k_tail, c.v_tail)])
    for other in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], other))


@pytest.mark.parametrize("dtype", [E4M3, INT8])
def test_magnitudes_of_a_page(dtype):
    """Pages of zeros, of the smallest and of the largest numbers, of one number, with numbers that are none."""
    Hkv, D, page = 1, 64, 32
    x = torch.zeros((8 * page, Hkv, D), dtype=torch.bfloat16, device=DEV)
    x[page:2 * page] = randn((page, Hkv, D), 1, 1e-38)
    x[2 * page:3 * page] = randn((page, Hkv, D), 2, 5e37)
    x[3 * page] = 2.0 ** -133                                      # the smallest bf16
    x[4 * page:5 * page] = -7.0
    x[5 * page:6 * page] = randn((page, Hkv, D), 3)
    x[6 * page:7 * page] = randn((page, Hkv, D), 4)
    x[6 * page + 3, 0, 5] = float("nan")
    x[7 * page + 9, 0, 5] = float("-inf")
    c, table = make(1, 1, Hkv, D, page, dtype, 8 * page)
    qp.paged_append(x, x, c, qp.PagedStep(ints([0, 8 * page]), ints([0]), table, 8 * page, 8 * page))
    check_cache(c, table, [x[:6 * page]], [x[:6 * page]], [6 * page], dtype)
    assert torch.isnan(c.k_scale[table[0, 6].long()]).all() and not torch.isfinite(c.v_scale[table[0, 7].long()]).any()


def test_own_positions():
    Hq, Hkv, D, page, n = 4, 2, 64, 32, 50
    k, v, q = randn((n, Hkv, D), 1), randn((n, Hkv, D), 2), randn((n, Hq, D), 3)
    pos = torch.randint(-50, 100000, (n,), device=DEV, dtype=torch.int32)
    rope = qp.rope(64, interleaved=True)
    c, table = make(1, Hq, Hkv, D, page, INT8, n)
    out = torch.empty_like(q)
    qr = qp.paged_append(k, v, c, qp.PagedStep(ints([0, n]), ints([0]), table, n, n), rope, pos=pos, q=q, q_out=out)
    turn = lambda x: qp.rotary(x.transpose(0, 1)[None], pos, rope)[0].transpose(0, 1)
    assert qr is out and torch.equal(qr, turn(q))
    check_cache(c, table, [turn(k)], [v], [n], INT8)
    inplace = q.clone()
    assert torch.equal(qp.paged_append(k, v, c, qp.PagedStep(ints([0, n]), ints([0]), table, n, n), rope, pos=pos, q=inplace, q_out=inplace), qr)


# ---------------------------------------------------------------------------------------------- attention

def fill(c, table, lens, seed, k_scale=1.0, v_scale=1.0, loud=True):
    """Tokens of every sequence straight into the cache; what pages lie behind the last whole one, and slots behind the last token,
    stay rubbish."""
    d = c.desc
    for b, n in enumerate(lens):
        for codes, scale, tail, std, sd in ((c.k_codes, c.k_scale, c.k_tail, k_scale, seed), (c.v_codes, c.v_scale, c.v_tail, v_scale, seed + 1)):
            x = randn((d.n_kv_heads, n, d.head_dim), sd + 7 * b, std)
            full = n // d.page
            if full:
                y = x[:, :full * d.page].reshape(d.n_kv_heads, full, d.page, d.head_dim).transpose(0, 1)
                if loud:                                           # pages of different magnitude
                    y = y * torch.exp2(torch.arange(full, device=DEV) % 5 - 2.0)[:, None, None, None].to(torch.bfloat16)
                got, s = stored(y, codes.dtype)
                ids = table[b, :full].long()
                codes.view(torch.uint8)[ids] = got.to(codes.dtype).view(torch.uint8)
                scale[ids] = s
            tail[b, :, :n - full * d.page] = x[:, full * d.page:]


def ref_attn(q, c, table, lens, new):
    """(out, bound) in 64 bits over what the cache holds."""
    d = c.desc
    G, D, page = d.n_q_heads // d.n_kv_heads, d.head_dim, d.page
    outs, bounds = [], []
    r0 = 0
    for b, (n0, m) in enumerate(zip(lens, new)):
        n = n0 + m
        full = n // page
        ids = table[b, :full].long()
        for i0 in range(0, m, 256):
            i1 = min(m, i0 + 256)
            o = torch.empty((i1 - i0, d.n_q_heads, D), dtype=torch.float64, device=DEV)
            w = torch.empty_like(o)
            for h in range(d.n_kv_heads):
                kv, extra = [], []
                for codes, scale, tail in ((c.k_codes, c.k_scale, c.k_tail), (c.v_codes, c.v_scale, c.v_tail)):
                    s = scale[ids, h].double()[:, None, None].expand(-1, page, 1).reshape(-1, 1)
                    x = codes.view(torch.uint8)[ids, h].view(codes.dtype).double().reshape(-1, D) * s
                    t = tail[b, h, :n - full * page].double()
                    kv.append(torch.cat([x, t]))
                    extra.append(torch.cat([128 * s if codes.dtype is INT8 else 0 * s, torch.zeros((t.shape[0], 1), dtype=torch.float64, device=DEV)]))
                qh = q[r0 + i0:r0 + i1, h * G:(h + 1) * G].double()
                x = torch.einsum("igd,jd->igj", qh, kv[0]) / math.sqrt(D)
                hide = torch.arange(n, device=DEV) > n0 + torch.arange(i0, i1, device=DEV)[:, None, None]
                p = torch.softmax(x.masked_fill(hide, -math.inf), -1)
                o[:, h * G:(h + 1) * G] = torch.einsum("igj,jd->igd", p, kv[1])
                size = torch.einsum("igd,jd->igj", qh.abs(), kv[0].abs() + extra[0]).masked_fill(hide, 0).amax(-1)
                small = qh.abs().amax(-1) * (kv[0].abs() + extra[0]).max()
                e = ((D + 8) * 2.0 ** -23 * size + D * 2.0 ** -24 * small) / math.sqrt(D)
                rel = torch.expm1(2 * e)[..., None] + 2 * 2.0 ** -11 + 2.0 ** -19 + (n / 16 + 64) * 2.0 ** -23
                vv = kv[1].abs() + extra[1]
                w[:, h * G:(h + 1) * G] = rel * torch.einsum("igj,jd->igd", p, vv) + 2.0 ** -35 * p.amax(-1)[..., None] * vv.sum(0)
            outs.append(o)
            bounds.append(w)
        r0 += m
    out, w = torch.cat(outs), torch.cat(bounds)
    waiting = max(float(c.v_tail[b, :, :(n0 + m) % page].abs().nan_to_num(posinf=0).max()) if (n0 + m) % page else 0 for b, (n0, m) in enumerate(zip(lens, new)))
    return out, w + 2.0 ** -8 * out.abs() + 2.0 ** -133 + 2.0 ** -25 * waiting


def check_attn(c, table, lens, new, seed=0, q_scale=1.0, q=None, pad=0):
    d = c.desc
    N = sum(new)
    q = randn((N + pad, d.n_q_heads, d.head_dim), seed + 100, q_scale) if q is None else q
    step = qp.PagedStep(start_of(new), ints(lens), table, N + pad, max(new))
    out = torch.full((N + pad, d.n_q_heads, d.head_dim), 77.0, dtype=torch.bfloat16, device=DEV)
    got = qp.paged_attn(q, c, step, out=out)
    assert (got[N:] == 77.0).all()                                 # rows of no sequence
    ref, bound = ref_attn(q, c, table, lens, new)
    err = (got[:N].double() - ref).abs() - bound
    assert not torch.isnan(got[:N]).any() and float(err.max()) <= 0, (float(err.max()), float((got[:N].double() - ref).norm() / ref.norm()))
    assert torch.equal(got, qp.paged_attn(q, c, step, out=torch.full_like(out, 77.0)))       # same inputs, same bits
    return got


ATTN = [  # Hq, Hkv, D, page, dtype, tokens before, new tokens
    (1, 1, 64, 32, E4M3, [0], [1]), (8, 2, 128, 64, E4M3, [0, 31, 63, 64, 65], [1, 1, 1, 1, 1]),
    (32, 8, 128, 64, E4M3, [2000], [1]), (64, 8, 128, 128, INT8, [1000, 5], [1, 1]), (28, 4, 128, 32, INT8, [333, 0, 777], [1, 0, 1]),
    (6, 2, 64, 32, E4M3, [100, 31, 0, 1000], [2, 1, 2, 2]), (8, 8, 64, 64, INT8, [127, 128], [1, 1]), (4, 4, 128, 32, E4M3, [95, 96, 97], [5, 3, 8]),
    (8, 1, 128, 128, E4M3, [130, 255], [2, 1]), (64, 8, 64, 64, E4M3, [500], [5]), (32, 8, 128, 32, INT8, [40, 700], [16, 3]),
    (7, 1, 128, 64, INT8, [50], [33]), (8, 2, 64, 128, INT8, [0, 300], [100, 1]), (16, 2, 128, 64, E4M3, [0], [260]),
    (32, 8, 128, 64, E4M3, [1, 2000, 0, 64], [200, 1, 64, 63]), (12, 4, 64, 32, E4M3, [513], [301]),
    (64, 8, 128, 64, E4M3, [3000], [129]), (8, 8, 128, 32, INT8, [10, 0], [300, 515]),
]


@pytest.mark.parametrize("Hq,Hkv,D,page,dtype,lens,new", ATTN)
def test_attention(Hq, Hkv, D, page, dtype, lens, new):
    c, table = make(len(lens), Hq, Hkv, D, page, dtype, max(a + b for a, b in zip(lens, new)), seed=len(lens))
    fill(c, table, [a + b for a, b in zip(lens, new)], 3)
    check_attn(c, table, lens, new)
    check_attn(c, table, lens, new, seed=5, q_scale=20.0, pad=3)


def test_many_sequences():
    lens = [(37 * b * b) % 1500 for b in range(300)]
    new = [0 if b % 7 == 3 else 1 for b in range(300)]
    c, table = make(300, 8, 2, 128, 32, E4M3, 1501)
    fill(c, table, [a + b for a, b in zip(lens, new)], 3)
    check_attn(c, table, lens, new)


@pytest.mark.parametrize("Hq,Hkv,D,page,dtype,most", [
    (8, 2, 64, 32, INT8, 1), (8, 1, 128, 64, INT8, 1), (6, 2, 64, 64, E4M3, 3), (32, 8, 128, 32, E4M3, 5), (8, 2, 128, 128, E4M3, 60), (6, 2, 64, 32, INT8, 90)])
def test_many_sequences_of_every_form(Hq, Hkv, D, page, dtype, most):
    lens = [(53 * b * b) % 900 for b in range(90)]
    new = [(b * 7) % (most + 1) for b in range(90)]
    c, table = make(90, Hq, Hkv, D, page, dtype, 900 + most)
    fill(c, table, [a + b for a, b in zip(lens, new)], 3)
    check_attn(c, table, lens, new, pad=5)


@pytest.mark.parametrize("dtype,D", [(E4M3, 64), (INT8, 128)])
def test_short_prompts_between_longer_ones(dtype, D):
    """Runs of sequences that have no whole page yet, which the copies of pages have nothing to wait for in."""
    lens = [90 if b % 11 == 10 else 0 for b in range(1500)]
    new = [10 + b % 13 for b in range(1500)]
    c, table = make(1500, 8, 2, D, 32, dtype, 128)
    fill(c, table, [a + b for a, b in zip(lens, new)], 3)
    check_attn(c, table, lens, new)


@pytest.mark.parametrize("most", [1, 40])
def test_all_the_rows_of_a_table(most):
    seqs = qp.QP_MAX_SEQS
    lens = [(29 * b) % 70 for b in range(seqs)]
    new = [b % (most + 1) if b % 9 == 0 or b == seqs - 1 else 0 for b in range(seqs)]
    c, table = make(seqs, 4, 2, 64, 32, E4M3, 70 + most)
    fill(c, table, [a + b for a, b in zip(lens, new)], 3)
    check_attn(c, table, lens, new)


@pytest.mark.parametrize("new", [[1, 1], [30, 70]])
def test_a_pool_beyond_32_bits(new):
    """Codes of 5 GB: pages whose bytes stand beyond 2^32, appended and attended to."""
    Hq, Hkv, D, page = 16, 8, 128, 128
    lens = [700, 127]
    c, table = make(2, Hq, Hkv, D, page, INT8, 896, spare=40000, seed=2)
    c.k_codes.view(torch.uint8).fill_(1)
    assert int(table.max()) * Hkv * page * D > 2 ** 32
    total = [a + b for a, b in zip(lens, new)]
    k, v = ([randn((n, Hkv, D), 10 * s + b) for b, n in enumerate(total)] for s in (1, 2))
    for at, m in (([0, 0], lens), (lens, new)):
        cut = lambda x: torch.cat([x[b][at[b]:at[b] + m[b]] for b in range(2)])
        qp.paged_append(cut(k), cut(v), c, qp.PagedStep(start_of(m), ints(at), table, sum(m), max(m)))
    check_cache(c, table, k, v, total, INT8)
    check_attn(c, table, lens, new)


def test_two_captured_calls_replayed_together():
    """Without workspaces of the caller's: each graph keeps its own."""
    jobs = []
    for dtype, new, seed in ((E4M3, [1, 1], 1), (INT8, [20, 3], 2), (E4M3, [150, 1], 3)):
        lens = [700, 64]
        c, table = make(2, 8, 2, 128, 64, dtype, 900)
        fill(c, table, [a + b for a, b in zip(lens, new)], seed)
        q = randn((sum(new), 8, 128), seed)
        step = qp.PagedStep(start_of(new), ints(lens), table, sum(new), max(new))
        want = qp.paged_attn(q, c, step)
        out = torch.zeros_like(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            qp.paged_attn(q, c, step, out=out)
        jobs.append((graph, torch.cuda.Stream(), out, want, (q, c, step)))
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, stream, *_ in jobs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, out, want, _ in jobs:
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("ks,vs,qs", [(1e-6, 1e-6, 1e6), (1e6, 1e6, 1e-6), (1.0, 1e-20, 1.0), (30.0, 1e20, 30.0), (1.0, 1.0, 0.0)])
@pytest.mark.parametrize("new", [[1, 1], [40, 9]])
def test_attention_at_any_magnitude(dtype, ks, vs, qs, new):
    lens = [500, 70]
    c, table = make(2, 8, 2, 128, 64, dtype, 540)
    fill(c, table, [a + b for a, b in zip(lens, new)], 11, ks, vs)
    check_attn(c, table, lens, new, q_scale=qs)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("ks,vs,qs", [(1.0, 1e-37, 1.0), (1.0, 1e28, 1.0), (1e-28, 1.0, 1e28), (1e-38, 1e-38, 1.0)])
@pytest.mark.parametrize("new", [[1, 1], [40, 9]])
def test_attention_at_the_ends_of_the_range(dtype, ks, vs, qs, new):
    lens = [500, 70]
    c, table = make(2, 8, 2, 128, 64, dtype, 540)
    fill(c, table, [a + b for a, b in zip(lens, new)], 11, ks, vs)
    check_attn(c, table, lens, new, q_scale=qs)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3e38])
@pytest.mark.parametrize("new", [[3, 2], [20, 9], [70, 1]])
def test_keys_that_earlier_rows_do_not_see(dtype, bad, new):
    lens = [500, 70]
    c, table = make(2, 8, 2, 128, 64, dtype, 600)
    fill(c, table, [a + b for a, b in zip(lens, new)], 11)
    q = randn((sum(new), 8, 128), 3)
    step = qp.PagedStep(start_of(new), ints(lens), table, sum(new), max(new))
    ref, bound = ref_attn(q, c, table, lens, new)
    last = (lens[0] + new[0] - 1) % 64                             # of the first sequence; its key is seen by its own row only
    c.k_tail[0, :, last, 7] = bad
    got = qp.paged_attn(q, c, step)
    if math.isfinite(bad):                                         # the bound counts the largest waiting key
        ref, bound = ref_attn(q, c, table, lens, new)
    rows = [r for r in range(sum(new)) if r != new[0] - 1]
    err = (got.double() - ref).abs() - bound
    assert float(err[rows].max()) <= 0 and not torch.isnan(got[rows]).any()
    if math.isnan(bad):
        assert torch.isnan(got[new[0] - 1]).all()


def test_peaked_rows_and_pages_of_zeros():
    lens, new = [1000], [1]
    c, table = make(1, 8, 1, 128, 32, E4M3, 1001)
    fill(c, table, [1001], 5, 8.0)
    c.v_codes.view(torch.uint8)[table[0, 3].long()] = 0            # a page of zeros has scale 0
    c.v_scale[table[0, 3].long()] = 0
    c.k_codes.view(torch.uint8)[table[0, 7].long()] = 0
    c.k_scale[table[0, 7].long()] = 0
    check_attn(c, table, lens, new, q_scale=12.0)
    check_attn(c, table, [970], [31], q_scale=12.0)


def test_shared_pages_and_strided_queries():
    lens, new, Hq = [300, 200, 256], [1, 4, 2], 8
    c, table = make(3, Hq, 2, 128, 64, E4M3, 400)
    fill(c, table, [a + b for a, b in zip(lens, new)], 5)
    table[1, :3] = table[0, :3]                                    # a common beginning
    table[2, 0] = table[2, 1]                                      # the same page twice
    wide = randn((7, Hq + 4, 128), 9)
    got = check_attn(c, table, lens, new, q=wide[:, 2:Hq + 2])
    assert torch.equal(got, check_attn(c, table, lens, new, q=wide[:, 2:Hq + 2].contiguous()))


def test_numbers_that_do_not_belong_together_are_left_out():
    """Read on the device: such a sequence is not touched, and nothing is addressed by its numbers."""
    Hq, Hkv, D, page = 8, 2, 128, 32
    lens, new = [100, 40, 70], [2, 2, 2]
    c, table = make(3, Hq, Hkv, D, page, E4M3, 128, seed=1)
    fill(c, table, [a + b for a, b in zip(lens, new)], 5)
    q, k = randn((6, Hq, D), 1), randn((6, Hkv, D), 2)
    ref, bound = ref_attn(q, c, table, lens, new)
    for start, ln, most in (([0, 2, 4, 7], lens, 3), ([0, 2, 1, 6], lens, 5), ([-5, 2, 4, 6], lens, 2), ([0, 2, 4, 6], [100, -1, 70], 2),
                            ([0, 2, 4, 6], [100, 40, 127], 2), ([0, 2, 4, 6], [2 ** 31 - 1, 40, 70], 2), ([0, 2, 6, 6], lens, 2),
                            ([6, 0, 6, 0], lens, 6), ([0, 6, 0, 6], lens, 6)):
        step = qp.PagedStep(ints(start), ints(ln), table, 6, most)
        ok = [0 <= start[b] <= start[b + 1] <= 6 and start[b + 1] - start[b] <= most and 0 <= ln[b] and ln[b] + start[b + 1] - start[b] <= 128
              for b in range(3)]
        claims = [sum(ok[b] and start[b] <= r < start[b + 1] for b in range(3)) for r in range(6)]
        out = torch.full_like(q, 77.0)
        qp.paged_attn(q, c, step, out=out)
        for b in range(3):
            if ok[b] and start[b:b + 2] == [2 * b, 2 * b + 2] and ln[b] == lens[b]:
                mine = [r for r in range(start[b], start[b + 1]) if claims[r] == 1]      # (a row that two claim is either's)
                assert float(((out.double() - ref).abs() - bound)[mine].max()) <= 0
        free = [r for r in range(6) if claims[r] == 0]
        assert (out[free] == 77.0).all()
        state = (c.k_tail, c.v_tail, c.k_codes.view(torch.uint8), c.v_codes.view(torch.uint8), c.k_scale, c.v_scale)
        before = [t.clone() for t in state]
        turned = torch.full_like(q, 55.0)
        qp.paged_append(k, k, c, step, qp.rope(128), q=q, q_out=turned)
        for b in range(3):
            if not ok[b]:
                assert torch.equal(c.k_tail[b].view(torch.int16), before[0][b].view(torch.int16))
        if start == sorted(start):                                 # (the owner of a row is searched for in start)
            assert (turned[free] == 55.0).all()
        for t, x in zip(state, before):
            t.copy_(x)


def test_pages_outside_the_pool():
    Hq, Hkv, D, page = 8, 2, 128, 32
    lens, new = [100, 90], [1, 1]
    c, table = make(2, Hq, Hkv, D, page, E4M3, 128, seed=1)
    fill(c, table, [101, 91], 5)
    q = randn((2, Hq, D), 1)
    step = lambda t: qp.PagedStep(ints([0, 1, 2]), ints(lens), t, 2, 1)
    good = qp.paged_attn(q, c, step(table))
    for bad in (-1, c.desc.n_pages, 2 ** 31 - 1, -2 ** 31):
        t = table.clone()
        t[0, 1] = bad
        t[:, 3] = bad                                              # not read: the fourth page is not whole
        got = qp.paged_attn(q, c, step(t))
        assert torch.isnan(got[0]).all() and torch.equal(got[1], good[1])
        state = (c.k_tail, c.v_tail, c.k_codes.view(torch.uint8), c.v_codes.view(torch.uint8), c.k_scale, c.v_scale)
        before = [x.clone() for x in state]
        k = randn((66, Hkv, D), 3)
        # the first completes its fourth page, the second its third, which is in the pool, and its fourth
        qp.paged_append(k, k, c, qp.PagedStep(ints([0, 28, 66]), ints(lens), t, 66, 38))
        keep = torch.ones(c.desc.n_pages, dtype=torch.bool, device=DEV)
        keep[table[1, 2].long()] = False
        for x, y in zip(state[2:], before[2:]):
            assert torch.equal(x[keep].view(torch.uint8), y[keep].view(torch.uint8)) and not torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        for x, y in zip(state, before):
            x.copy_(y)


# ---------------------------------------------------------------------------------------------- the run of calls

def test_generation_steps_from_one_graph():
    """Prompts, then steps: append and attention of a captured step serve every later one, lengths advanced on the device."""
    Hq, Hkv, D, page, seqs = 8, 2, 128, 32, 3
    rope = qp.rope(128, 500000.0, scaling="yarn", factor=4.0)
    c, table = make(seqs, Hq, Hkv, D, page, E4M3, 256)
    ln = ints([0] * seqs)
    first = [50, 1, 130]
    N = sum(first)
    q, k, v = randn((N, Hq, D), 1), randn((N, Hkv, D), 2), randn((N, Hkv, D), 3)
    step = qp.PagedStep(start_of(first), ln, table, N, max(first))
    out = qp.paged_layer_step(q, k, v, c, step, rope)
    ref, bound = ref_attn(qp.paged_append(k, v, c, step, rope, q=q), c, table, [0] * seqs, first)
    assert float(((out.double() - ref).abs() - bound).max()) <= 0
    ln += ints(first)
    start = ints(list(range(seqs + 1)))
    step = qp.PagedStep(start, ln, table, seqs, 1)
    q, k, v = (torch.zeros((seqs, h, D), dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv))
    out = torch.empty_like(q)
    ws = qp.new_decode_workspace(qp.paged_attn_workspace_bytes(c, seqs, 1), DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qp.paged_layer_step(q, k, v, c, step, rope, out=out, workspace=ws)
        ln += 1
    lens = first
    for i in range(70):
        for t, s in ((q, 1), (k, 2), (v, 3)):
            t.copy_(randn(t.shape, 1000 + 10 * i + s))
        graph.replay()
        if i % 9 == 0 or i > 60:
            turned = torch.cat([qp.rotary(q[b:b + 1].transpose(0, 1)[None], ints([lens[b]]), rope)[0].transpose(0, 1) for b in range(seqs)])
            ref, bound = ref_attn(turned, c, table, lens, [1] * seqs)
            assert float(((out.double() - ref).abs() - bound).max()) <= 0, i
        lens = [n + 1 for n in lens]
    assert ln.tolist() == lens


def test_a_prompt_in_chunks_and_drafts_taken_back():
    """Chunks see what came before them; drafted tokens behind the last whole page can be taken back by setting len."""
    Hq, Hkv, D, page, n = 4, 2, 64, 64, 300
    q, k, v = randn((n, Hq, D), 1), randn((n, Hkv, D), 2), randn((n, Hkv, D), 3)
    c, table = make(1, Hq, Hkv, D, page, INT8, 400)
    at = 0
    for m in (100, 1, 150, 49):
        step = qp.PagedStep(ints([0, m]), ints([at]), table, m, m)
        out = qp.paged_layer_step(q[at:at + m], k[at:at + m], v[at:at + m], c, step)
        ref, bound = ref_attn(q[at:at + m], c, table, [at], [m])
        assert float(((out.double() - ref).abs() - bound).max()) <= 0
        at += m
    dq, dk, dv = randn((9, Hq, D), 4), randn((9, Hkv, D), 5), randn((9, Hkv, D), 6)
    step = lambda m: qp.PagedStep(ints([0, m]), ints([n]), table, m, m)
    first = qp.paged_layer_step(dq, dk, dv, c, step(9))            # nine drafts
    before, bound = ref_attn(dq, c, table, [n], [9])
    assert float(((first.double() - before).abs() - bound).max()) <= 0
    dk[2:], dv[2:] = dk[2:] + 1, dv[2:] - 1
    again = qp.paged_layer_step(dq, dk, dv, c, step(9))            # two kept, the others replaced
    ref, bound = ref_attn(dq, c, table, [n], [9])
    assert float(((again.double() - ref).abs() - bound).max()) <= 0
    # the two that were kept see the same (in other bits, perhaps: 32 waiting rows share the power of two that they are scaled by)
    assert torch.equal(ref[:2], before[:2]) and not torch.equal(first[2:], again[2:])


def test_two_streams_and_other_dtypes_at_once():
    lens, new = [700, 64], [1, 1]
    jobs = []
    for dtype, seed in ((E4M3, 1), (INT8, 2)):
        c, table = make(2, 8, 2, 128, 64, dtype, 701)
        fill(c, table, [701, 65], seed)
        q = randn((2, 8, 128), seed)
        step = qp.PagedStep(ints([0, 1, 2]), ints(lens), table, 2, 1)
        ws = qp.new_decode_workspace(qp.paged_attn_workspace_bytes(c, 2, 1), DEV)
        jobs.append((q, c, step, ws, torch.cuda.Stream(), qp.paged_attn(q, c, step), []))
    torch.cuda.synchronize()
    for _ in range(20):
        for q, c, step, ws, stream, _, outs in jobs:
            with torch.cuda.stream(stream):
                outs.append(qp.paged_attn(q, c, step, workspace=ws))
    torch.cuda.synchronize()
    for *_, want, outs in jobs:
        assert all(torch.equal(o, want) for o in outs)
