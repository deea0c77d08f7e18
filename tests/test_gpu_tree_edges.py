"""Drafted trees at their edges: a block whose wait ran out, every error word, logits and values of any size, long and mixed masks."""
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2412_12706_b200 import qp
from tests.test_gpu_tree import DEV, make_cache, mask_of, random_tree, randn, reference

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Every block in turn reports that a wait ran out, after all its waits have returned (the range-checked build has a call for it).
# What it computed is lost, and with it the rows of its KV head and row group: they are NaN, and its error word is 1; all others are
# as they were.
GIVE_UP = """
import torch
from paper_2412_12706_b200 import qp
from tests.test_gpu_tree import make_cache, mask_of, random_tree, randn
for Bt, Hq, Hkv, D, n, bits, T in ((1, 8, 2, 128, 1000, 16, 5), (1, 8, 1, 128, 8192, 4, 33), (2, 8, 2, 64, 256, 2, 64), (1, 16, 2, 128, 640, 8, 40)):
    c, _, _, _ = make_cache(Bt, Hq, Hkv, D, n, n, bits, 32, 0)
    q, kd, vd = randn((Bt, T, Hq, D), 3), randn((Bt, T, Hkv, D), 4), randn((Bt, T, Hkv, D), 5)
    mask = mask_of(random_tree(Bt, T, 5)[1])
    G = Hq // Hkv
    groups = (T * G + 255) // 256
    W = Bt * Hkv * groups
    words = W * max(1, min(16, 148 // W))
    ws = qp.new_decode_workspace(qp.decode_tree_workspace_bytes(c, T), "cuda")
    err = ws[:4 * words].view(torch.int32)
    good = qp.decode_attn_tree(q, c, kd, vd, mask, workspace=ws)
    assert torch.isfinite(good).all() and not err.any()
    seen, blocks = set(), 0
    for block in range(148 * 2):
        assert qp.debug_give_up(block) == 0
        out = qp.decode_attn_tree(q, c, kd, vd, mask, workspace=ws)
        hit = err.nonzero().flatten().tolist()
        if not hit:                                     # no such block
            assert torch.equal(out, good)
            break
        blocks += 1
        assert len(hit) == 1 and int(err[hit[0]]) == 1
        item = hit[0] // (words // W)
        seen.add(item)
        bh, rg = divmod(item, groups)
        rows = torch.zeros((Bt, Hkv, T * G), dtype=torch.bool, device="cuda")
        rows[bh // Hkv, bh % Hkv, 256 * rg:256 * rg + 256] = True
        rows = rows.view(Bt, Hkv, T, G).transpose(1, 2).reshape(Bt, T, Hq)
        assert torch.isnan(out[rows]).all(), (bits, block, int(torch.isnan(out[rows]).sum()), out[rows].numel())
        assert torch.equal(out[~rows], good[~rows])
    assert seen == set(range(W)) and blocks > W, (seen, blocks)
    assert qp.debug_give_up(-1) == 0
    assert torch.equal(good, qp.decode_attn_tree(q, c, kd, vd, mask, workspace=ws)) and not err.any()
print("poisoned")
"""


def test_what_a_block_lost_whose_wait_ran_out_is_nan():
    env = dict(os.environ, QP_LIBRARY=os.environ.get("QP_CHECKED_LIBRARY") or os.path.join(ROOT, "paper_2412_12706_b200", "libqp_checked.so"))
    r = subprocess.run([sys.executable, "-c", GIVE_UP], env=env, cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "poisoned", r.stdout[-1000:] + r.stderr[-3000:]
    assert qp.debug_give_up(-1) == 2 and qp.debug_give_up(-2) == 1         # the normal build has no such call


def error_words(ws, Bt, Hq, Hkv, T):
    W = Bt * Hkv * ((T * (Hq // Hkv) + 255) // 256)
    return ws[:4 * W * max(1, min(16, 148 // W))].view(torch.int32)


@pytest.mark.parametrize("Bt,Hq,Hkv,D,n,bits,T", [(1, 32, 8, 128, 1024, 16, 40), (1, 32, 8, 128, 9216, 4, 40), (1, 8, 1, 64, 20000, 16, 64),
                                                  (2, 8, 1, 128, 512, 2, 64), (19, 32, 8, 128, 320, 4, 16), (1, 8, 1, 128, 128, 8, 1)])
def test_every_error_word_is_cleared_by_the_call(Bt, Hq, Hkv, D, n, bits, T):
    c, _, _, _ = make_cache(Bt, Hq, Hkv, D, n, n, bits, 32, 0)
    q, kd, vd = randn((Bt, T, Hq, D), 3), randn((Bt, T, Hkv, D), 4), randn((Bt, T, Hkv, D), 5)
    mask = mask_of(random_tree(Bt, T, 5)[1])
    ws = qp.new_decode_workspace(qp.decode_tree_workspace_bytes(c, T), DEV)
    ws.fill_(255)
    out = qp.decode_attn_tree(q, c, kd, vd, mask, workspace=ws)
    assert torch.isfinite(out).all() and torch.all(error_words(ws, Bt, Hq, Hkv, T) == 0)


@pytest.mark.parametrize("bits", [16, 8, 4, 2])
def test_large_logits_and_values_against_64_bits(bits):
    """Logits of several hundred, drafts' values of several hundred: one token takes nearly everything, in cache and drafts."""
    Bt, Hq, Hkv, D, n, T = 1, 8, 2, 128, 512, 9
    c, _, k, v = make_cache(Bt, Hq, Hkv, D, n, n, bits, 32, 0, scale=10.0)
    q, kd, vd = randn((Bt, T, Hq, D), 3, 20.0), randn((Bt, T, Hkv, D), 4, 10.0), randn((Bt, T, Hkv, D), 5, 500.0)
    sees = torch.ones((T, T), dtype=torch.bool, device=DEV).tril().expand(Bt, T, T)
    out = qp.decode_attn_tree(q, c, kd, vd, mask_of(sees)).double()
    if bits < 16:
        # what fp16 makes of the keys and queries is part of the operator: compare with the same factors, so that a logit of
        # several hundred is not moved by 2^-11 of its terms
        half = lambda x: x.double().half().double()
        k, kq, vq, qq = half(k), half(kd), half(vd), half(q)
    else:
        kq, vq, qq = kd, vd, q
    none = torch.zeros((Bt, Hkv, 0, D), dtype=torch.float64, device=DEV)
    ref, _ = reference(qq, k, v, none, none, kq, vq, sees, bits)
    x = qq.double().view(Bt, T, Hkv, Hq // Hkv, D)
    keys, vals = torch.cat([k, kq.double().transpose(1, 2)], 2), torch.cat([v, vq.double().transpose(1, 2)], 2)
    s = torch.einsum("bthgd,bhnd->bthgn", x, keys) / math.sqrt(D)
    hide = torch.cat([torch.zeros((Bt, T, n), dtype=torch.bool, device=DEV), ~sees], -1)[:, :, None, None]
    p = torch.softmax(s.masked_fill(hide, -math.inf), -1)
    assert float(p.max()) > 0.99
    spread = torch.einsum("bthgn,bhnd->bthgd", p, vals.abs()).reshape(out.shape)
    sum_abs = float(torch.einsum("bthgd,bhnd->bthgn", x.abs(), keys.abs()).max())
    e = (D + 8) * 2.0 ** -23 * sum_abs / math.sqrt(D)
    tol = 2.0 ** -8 * ref.abs() + ((2.0 ** -8 if bits == 16 else 2.0 ** -11) + 2.0 ** -11 + math.expm1(2 * e)) * spread + 1e-6
    assert torch.all((out - ref).abs() <= tol), float(((out - ref).abs() / tol).max())


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("Bt,Hq,Hkv,T", [(18, 32, 8, 40), (1, 8, 8, 64)])
def test_a_draft_that_takes_nearly_everything_gives_its_own_value(bits, Bt, Hq, Hkv, T):
    """Two light tokens in the cache (32 for packed ones), and drafts that see themselves 4 to 5.4 nats above them: less than the 2^8
    by which the reference may lag, so the heavy weight is not 1 and its 16 bits round it.  It is in the sum as it is in the product, so that
    a weight's rounding (2^-8 in bf16, 2^-11 in fp16, of it and of the sum) moves the output by twice that of sum p |v - out| only."""
    D, n = 128, 2 if bits == 16 else 32
    c = qp.alloc_cache(Bt, Hq, Hkv, D, bits, 32, n, DEV)
    K, V = torch.zeros((Bt, Hkv, n, D), dtype=torch.bfloat16, device=DEV), randn((Bt, Hkv, n, D), 2)
    qp.gather_quantize(K, V, torch.arange(n, dtype=torch.int32, device=DEV).expand(Bt, Hkv, n).contiguous(), c)
    v = V.double()
    if bits < 16:
        cv = ((c.v_codes.long()[..., None] >> (bits * torch.arange(32 // bits, device=DEV))) & (2 ** bits - 1)).flatten(-2).double()
        v = (cv * c.v_scale.double()[..., None] + c.v_zero.double()[..., None]).reshape(Bt, Hkv, n, D)
    one = randn((Bt, T, Hkv, 1, D), 3)
    q = one.expand(Bt, T, Hkv, Hq // Hkv, D).reshape(Bt, T, Hq, D).contiguous()
    g = torch.Generator(device=DEV).manual_seed(4)
    above = 4.0 + 1.4 * torch.rand((Bt, T, Hkv, 1), generator=g, device=DEV, dtype=torch.float64) + math.log(n / 2)
    above = above.clamp(max=5.4)
    x = one[:, :, :, 0].double()
    kd, vd = (x * above * math.sqrt(D) / x.square().sum(-1, keepdim=True)).to(torch.bfloat16), randn((Bt, T, Hkv, D), 5)
    sees = torch.eye(T, dtype=torch.bool, device=DEV).expand(Bt, T, T)
    out = qp.decode_attn_tree(q, c, kd, vd, mask_of(sees)).double().view(Bt, T, Hkv, -1, D)
    s = (x * kd.double()).sum(-1) / math.sqrt(D)                       # [Bt,T,Hkv]; the cached tokens' logits are 0
    p = torch.exp(s) / (torch.exp(s) + n)
    ref = p[..., None] * vd.double() + ((1 - p)[..., None] / n) * v.sum(2)[:, None]
    away = p[..., None] * (vd.double() - ref).abs() + ((1 - p)[..., None] / n) * (v[:, None] - ref[:, :, :, None]).abs().sum(3)
    spread = p[..., None] * vd.double().abs() + ((1 - p)[..., None] / n) * v.abs().sum(2)[:, None]
    e = ((D + 8) * 2.0 ** -23 + (0.0 if bits == 16 else 3 * 2.0 ** -11)) * float((x * kd.double()).abs().sum(-1).max()) / math.sqrt(D)
    tol = 2.0 ** -8 * ref.abs() + 2 * (2.0 ** -8 if bits == 16 else 2.0 ** -11) * away + (2.0 ** -10 if bits < 16 else 2.0 ** -20) * spread \
        + 2 * math.expm1(2 * e) * away + 1e-6
    worst = float(((out - ref[:, :, :, None]).abs() / tol[:, :, :, None]).max())
    assert worst <= 1, worst
