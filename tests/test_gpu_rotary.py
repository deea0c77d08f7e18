"""Rotation by position against the formula in 64 bits.

Tolerance.  The angle's fraction of a turn is cut to 2^-32 and rounded to 24 bits: off by at most 2^-24 half turns, pi 2^-24; the cosine
and sine of it by 2^-22 more; a product and a sum in 32 bits by 2^-23 of |u| + |v|.  With the factor m that is less than
2^-20 m (|u| + |v|), and the result is rounded to bf16 once: 2^-8 of itself."""
import math

import pytest
import torch

from paper_2412_12706_b200 import qp

pytestmark = pytest.mark.gpu
DEV = "cuda"


def randn(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(shape, generator=g, device=DEV)).to(torch.bfloat16)


def frequencies(rot, base, scaling="plain", factor=1.0, trained=8192):
    """w_i from the definition, pair by pair."""
    w = []
    d = lambda x: rot * math.log(trained / (2 * math.pi * x)) / (2 * math.log(base))
    lo, hi = max(math.floor(d(32)), 0), min(math.ceil(d(1)), rot - 1)
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "ntk" else base
        f = b ** (-2 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "yarn":
            r = min(1, max(0, (i - lo) / (hi - lo if hi != lo else 0.001)))
            f = f * (1 - r) + f / factor * r
        elif scaling == "bands":
            s = min(1, max(0, (trained * f / (2 * math.pi) - 1) / 3))
            f = f / factor * (1 - s) + f * s
        w.append(f)
    return w, (0.1 * math.log(factor) + 1 if scaling == "yarn" else 1.0)


def ref_rotary(x, pos, w, m, inter, sign=1.0):
    """(result, |u| + |v| of every rotated channel) in 64 bits; pos broadcasts over x[..., 0]."""
    rot = 2 * len(w)
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    for i, f in enumerate(w):
        p, q = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        u, v, a = x[..., p].double(), x[..., q].double(), sign * f * pos.double()
        y[..., p], y[..., q] = m * (u * torch.cos(a) - v * torch.sin(a)), m * (v * torch.cos(a) + u * torch.sin(a))
        size[..., p] = size[..., q] = m * (u.abs() + v.abs())
    return y, size


def assert_rotated(got, x, pos, w, m, inter, sign=1.0):
    ref, size = ref_rotary(x, pos, w, m, inter, sign)
    over = (got.double() - ref).abs() - (2.0 ** -8 * ref.abs() + 2.0 ** -20 * size)
    assert float(over.max()) <= 0, float(over.max())
    assert torch.equal(got[..., 2 * len(w):], x[..., 2 * len(w):])


CASES = [  # Bt, H, L, D, rot, interleaved, scaling
    (1, 1, 1, 64, 64, False, "plain"), (1, 32, 1, 128, 128, False, "bands"), (2, 3, 5, 128, 2, True, "plain"),
    (1, 8, 257, 64, 32, True, "yarn"), (3, 7, 33, 128, 128, True, "ntk"), (1, 2, 1000, 128, 64, False, "linear"),
    (2, 5, 31, 64, 22, False, "yarn"), (1, 9, 100, 128, 126, False, "bands"), (1, 64, 40, 128, 96, False, "yarn"),
    (1, 200, 3, 128, 128, False, "plain"), (2, 1, 70, 64, 2, False, "plain"), (1, 300, 2, 64, 50, True, "linear"),
]


@pytest.mark.parametrize("Bt,H,L,D,rot,inter,scaling", CASES)
@pytest.mark.parametrize("transpose", [False, True])
def test_rotary(Bt, H, L, D, rot, inter, scaling, transpose):
    x = randn((Bt, H, L, D), L + rot)
    factor = 1.0 if scaling == "plain" else 8.0
    rope = qp.rope(rot, 500000.0, inter, scaling, factor)
    w, m = frequencies(rot, 500000.0, scaling, factor)
    pos = torch.randint(0, 200000, (Bt, L), device=DEV, dtype=torch.int32)
    got = qp.rotary(x, pos, rope, transpose=transpose)
    assert_rotated(got, x, pos[:, None], w, m, inter, -1.0 if transpose else 1.0)
    assert torch.equal(got, qp.rotary(x, pos, rope, transpose=transpose))
    y = x.clone()                                                  # in place
    assert qp.rotary(y, pos, rope, out=y, transpose=transpose) is y and torch.equal(y, got)
    # rows of a wider projection, read and written where they are
    wide = randn((Bt, L, H + 2, D), 5)
    wide[:, :, 1:H + 1] = x.transpose(1, 2)
    kept = wide.clone()
    part = wide[:, :, 1:H + 1].transpose(1, 2)
    assert torch.equal(qp.rotary(part, pos, rope, transpose=transpose), got)
    qp.rotary(part, pos, rope, out=part, transpose=transpose)
    assert torch.equal(part, got) and torch.equal(wide[:, :, 0], kept[:, :, 0]) and torch.equal(wide[:, :, H + 1], kept[:, :, H + 1])


@pytest.mark.parametrize("inter", [False, True])
def test_far_negative_and_shared_positions(inter):
    pos = torch.tensor([0, 1, -1, -70000, 1048575, 2 ** 24 + 1, 2 ** 30 + 12345, 2 ** 31 - 1, -2 ** 31], device=DEV, dtype=torch.int32)
    x = randn((2, 3, len(pos), 128), 3)
    for rot, base in ((128, 10000.0), (40, 1e6)):
        w, m = frequencies(rot, base)
        got = qp.rotary(x, pos, qp.rope(rot, base, inter))
        # 2^31 times a frequency in 64 bits is off by 2^-22 radians in the reference itself, the turn by 2^-33: within 2^-20
        assert_rotated(got, x, pos, w, m, inter)
        assert torch.equal(got[:, :, 0], x[:, :, 0])               # position 0


def test_own_frequencies_and_factor():
    w = [0.0, 1.0, -0.25, 6.0, 1e-7, 3.0, 0.1, 0.01]
    x, pos = randn((1, 4, 50, 64), 8), torch.arange(1000, 1050, device=DEV, dtype=torch.int32)
    assert_rotated(qp.rotary(x, pos, qp.rope(16, freqs=w, factor=0.5)), x, pos, w, 0.5, False)


def test_transposed_is_the_gradient_and_the_way_back():
    Bt, H, L, D = 1, 2, 40, 64
    rope = qp.rope(48, 10000.0, False, "yarn", 4.0)
    w, m = frequencies(48, 10000.0, "yarn", 4.0)
    pos = torch.arange(3, 3 + L, device=DEV, dtype=torch.int32)
    x, dy = randn((Bt, H, L, D), 1).double().requires_grad_(), randn((Bt, H, L, D), 2)
    y, _ = ref_rotary(x, pos, w, m, False)
    (dx,) = torch.autograd.grad(y, x, dy.double())
    got = qp.rotary(dy, pos, rope, transpose=True)
    _, size = ref_rotary(dy, pos, w, m, False)
    assert float(((got.double() - dx).abs() - (2.0 ** -8 * dx.abs() + 2.0 ** -20 * size)).max()) <= 0
    # by differences: the call is linear, so <dy, R(x + h) - R(x)> is <R^T dy, h>; every rounding to bf16 is off by 2^-8
    h = randn((Bt, H, L, D), 4)
    left = (dy.double() * qp.rotary(h, pos, rope).double()).sum()
    right = (got.double() * h.double()).sum()
    bound = 2.0 ** -8 * ((dy.double() * qp.rotary(h, pos, rope).double()).abs().sum() + (got.double() * h.double()).abs().sum()) * 1.01
    assert abs(float(left - right)) <= float(bound)
    plain = qp.rope(48)
    there = qp.rotary(dy, pos, plain)
    _, size = ref_rotary(there, pos, *frequencies(48, 10000.0), False)
    back = qp.rotary(there, pos, plain, transpose=True)
    # two roundings, the first carried through the second rotation
    assert float(((back.double() - dy.double()).abs() - (2.0 ** -8 * dy.double().abs() + 2.0 ** -8 * 1.01 * size + 2.0 ** -20 * size)).max()) <= 0


def test_a_prompt_compressed_from_unrotated_keys():
    from paper_2412_12706_b200 import synth
    wl = synth.TINY
    k, v = synth.make_kv(wl, 0)
    k, v, qw = k.to(DEV), v.to(DEV), synth.make_q_win(wl, 0).to(DEV)
    rope = qp.rope(wl.head_dim, 10000.0)
    pos = torch.arange(7, 7 + wl.L, dtype=torch.int32, device=DEV)
    cache, kept = qp.compress_layer_rotary(k, v, qw, rope, wl.budget_bits, wl.bits, wl.group, wl.pool, first_pos=7)
    want, kept2 = qp.compress_layer(qp.rotary(k, pos, rope), v, qp.rotary(qw, pos[wl.L - wl.w:], rope), wl.budget_bits, wl.bits, wl.group, wl.pool)
    assert torch.equal(kept, kept2) and torch.equal(cache.k_codes, want.k_codes) and torch.equal(cache.v_codes, want.v_codes)


def test_on_another_stream_and_in_a_graph():
    x, pos = randn((1, 8, 300, 128), 9), torch.arange(300, device=DEV, dtype=torch.int32)
    rope = qp.rope(128)
    want = qp.rotary(x, pos, rope)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(x)
    with torch.cuda.stream(side):
        qp.rotary(x, pos, rope, out=out)
    side.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qp.rotary(x, pos, rope, out=out)
    pos += 5
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, qp.rotary(x, pos, rope))
