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
