"""The paged cache at its edges: pages that hold what is no number, or are none, among those a row sees and those it does not.

Outputs of rows that see nothing of it are held to the bound of tests/test_gpu_paged.py; rows that do are not finite, whatever form of the
attention takes them, and however its work is cut."""
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2412_12706_b200 import qp
from tests.test_gpu_paged import DEV, E4M3, INT8, check_attn, check_cache, fill, ints, make, randn, ref_attn, start_of, stored

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FORMS = [  # Hq, Hkv, D, page, dtype, tokens before, new tokens
    (4, 2, 128, 32, E4M3, [500, 70], [100, 33]),                   # rows of both halves of an item
    (2, 2, 64, 32, INT8, [100, 300], [100, 77]),                   # up to 128 rows
    (8, 1, 128, 64, E4M3, [3000, 5], [300, 1]),                    # several items, each cut
    (8, 2, 128, 128, INT8, [0, 130], [700, 260]),
    (1, 1, 128, 128, E4M3, [2800], [160]),                         # a tile a block
    (8, 8, 64, 32, E4M3, [20 * (b % 5) for b in range(40)], [40 + b for b in range(40)]),     # items that are whole in a block
]


def whole_pages(lens, new, page):
    """(sequence, page) of the pages that the step completes."""
    return [(b, i) for b, (n, m) in enumerate(zip(lens, new)) for i in range(n // page, (n + m) // page)]


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("Hq,Hkv,D,page,dtype,lens,new", FORMS)
def test_a_key_in_a_new_page_leaves_the_rows_before_it_alone(Hq, Hkv, D, page, dtype, lens, new, bad):
    """A key that is not finite makes the scale of its page so; rows that stand before the page see none of it."""
    total = [a + b for a, b in zip(lens, new)]
    c, table = make(len(lens), Hq, Hkv, D, page, dtype, max(total))
    fill(c, table, total, 11)
    q = randn((sum(new), Hq, D), 3)
    step = qp.PagedStep(start_of(new), ints(lens), table, sum(new), max(new))
    ref, bound = ref_attn(q, c, table, lens, new)
    pages = whole_pages(lens, new, page)
    pages = pages[:3] + pages[3::max(1, len(pages) // 12)]
    assert pages
    at = start_of(new).tolist()
    behind = 0
    for b, i in pages:
        row = int(table[b, i])
        first = max(0, i * page - lens[b])                         # rows of the sequence before the page
        behind += first
        kept = c.k_scale[row].clone(), c.k_codes[row].clone()
        head = i % Hkv                                             # one head's
        c.k_scale[row, head] = bad
        c.k_codes.view(torch.uint8)[row, head, page - 1, 5] = 0x7f  # as the cache stores it: e4m3 has a code for what is no number
        got = qp.paged_attn(q, c, step)
        sees = torch.zeros((sum(new), Hq), dtype=torch.bool, device=DEV)
        sees[at[b] + first:at[b + 1], head * (Hq // Hkv):(head + 1) * (Hq // Hkv)] = True
        err = (got.double() - ref).abs() - bound
        assert (err[~sees] <= 0).all(), (b, i, int(torch.isnan(got[~sees]).any(-1).sum()))
        if math.isnan(bad):                                        # (an infinite logit of the other sign weighs nothing)
            assert torch.isnan(got[sees]).all(), (b, i)
        c.k_scale[row], c.k_codes[row] = kept
    assert behind > 0


@pytest.mark.parametrize("what", ["outside the pool", "key scale", "value scale", "infinite value scale"])
@pytest.mark.parametrize("Hq,Hkv,D,page,dtype,lens,new", FORMS + [
    (8, 2, 128, 128, E4M3, [1500, 300], [1, 1]), (8, 1, 64, 32, INT8, [900], [3])])              # a few rows
def test_a_page_that_is_no_number_shows_in_every_row_that_sees_it(Hq, Hkv, D, page, dtype, lens, new, what):
    """A page number outside the pool, or a page whose scale is no number: none of its rows comes out as if the page were not there,
    wherever the cuts between blocks fall (a page of 128 tokens is the first of some block's piece, whichever it is)."""
    total = [a + b for a, b in zip(lens, new)]
    c, table = make(len(lens), Hq, Hkv, D, page, dtype, max(total))
    fill(c, table, total, 11)
    q = randn((sum(new), Hq, D), 3)
    at = start_of(new).tolist()
    run = lambda t: qp.paged_attn(q, c, qp.PagedStep(start_of(new), ints(lens), t, sum(new), max(new)))
    good = run(table)
    pages = [(b, i) for b, n in enumerate(total) for i in range(n // page)]
    pages = pages[:30] + pages[30::max(1, len(pages) // 20)]
    for b, i in pages:
        row, head = int(table[b, i]), i % Hkv
        t, kept = table, (c.k_scale[row].clone(), c.v_scale[row].clone())
        heads = slice(head * (Hq // Hkv), (head + 1) * (Hq // Hkv))
        if what == "outside the pool":
            t, heads = table.clone(), slice(0, Hq)
            t[b, i] = (-1, c.desc.n_pages)[i % 2]
        else:
            (c.k_scale if what == "key scale" else c.v_scale)[row, head] = INF if what.startswith("inf") else NAN
        got = run(t)
        rows = slice(at[b] + max(0, i * page - lens[b]), at[b + 1])
        if what.startswith("inf"):                                 # its zeros are no numbers, all else is infinite
            assert not torch.isfinite(got[rows, heads]).any(), (b, i)
        else:
            assert torch.isnan(got[rows, heads]).all(), (b, i, int(torch.isfinite(got[rows, heads]).sum()))
        rest = torch.ones(got.shape[:2], dtype=torch.bool, device=DEV)
        rest[at[b]:at[b + 1], heads] = False                       # (rows before the page, too, may be lost to a value)
        assert torch.equal(got[rest], good[rest]), (b, i)
        c.k_scale[row], c.v_scale[row] = kept


def test_rows_of_nobody_behind_a_sequence_near_the_last_position():
    """Units of the padding's rows, counted on from the sequence's last page, would stand at tokens beyond 2^31."""
    Hkv, D, page, n_tokens, m = 2, 64, 32, 5000, 40
    max_pages = (2 ** 31 - 1025) // page
    n = max_pages * page - m
    assert n % page == 24 and (n + n_tokens) // page * page >= 2 ** 31
    c = qp.alloc_paged(1, 4, Hkv, D, 3, max_pages, page, E4M3)
    for t in (c.k_codes, c.v_codes):
        t.view(torch.uint8).fill_(0x7f)
    for t in (c.k_scale, c.v_scale):
        t.fill_(NAN)
    old = [randn((Hkv, 24, D), s) for s in (1, 2)]
    for t, x in zip((c.k_tail, c.v_tail), old):
        t[0, :, :24] = x
    tails = c.k_tail.clone(), c.v_tail.clone()
    table = torch.zeros((1, max_pages), dtype=torch.int32, device=DEV)
    table[0, -2:] = ints([1, 2])
    k, v, q = randn((n_tokens, Hkv, D), 3), randn((n_tokens, Hkv, D), 4), randn((n_tokens, 4, D), 5)
    rope = qp.rope(D)
    pos = torch.arange(n, n + m, dtype=torch.int32, device=DEV)
    turn = lambda x: qp.rotary(x[:m].transpose(0, 1)[None], pos, rope)[0].transpose(0, 1)
    turned = torch.full_like(q, 55.0)
    qp.paged_append(k, v, c, qp.PagedStep(ints([0, m]), ints([n]), table, n_tokens, m), rope, q=q, q_out=turned)
    for codes, scale, before, x in ((c.k_codes, c.k_scale, old[0], turn(k)), (c.v_codes, c.v_scale, old[1], v[:m])):
        x = torch.cat([before, x.transpose(0, 1)], 1).view(Hkv, 2, page, D).transpose(0, 1)
        want, s = stored(x, E4M3)
        assert torch.equal(scale[1:], s) and torch.equal(codes.view(torch.uint8)[1:].view(E4M3).float(), want)
        assert torch.isnan(scale[0]).all() and (codes.view(torch.uint8)[0] == 0x7f).all()
    assert torch.equal(turned[:m], turn(q)) and (turned[m:] == 55.0).all()
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(tails, (c.k_tail, c.v_tail)))


def arrays(c):
    return [t.view(torch.uint8) if t.dtype != torch.bfloat16 else t.view(torch.int16) for t in (c.k_codes, c.v_codes, c.k_scale, c.v_scale, c.k_tail, c.v_tail)]


def check_left_out(c, table, start, lens, n, most, seed):
    """An append of n rows with these starts: sequences whose numbers belong together are taken in as if each were alone, the others,
    and rows that are nobody's, are left as they are."""
    Hq, Hkv, D, page = c.desc.n_q_heads, c.desc.n_kv_heads, c.desc.head_dim, c.desc.page
    seqs, limit = len(lens), c.desc.max_pages * page
    q, k, v = randn((n, Hq, D), seed), randn((n, Hkv, D), seed + 1), randn((n, Hkv, D), seed + 2)
    rope = qp.rope(D)
    before = [t.clone() for t in arrays(c)]
    good = [b for b in range(seqs) if 0 <= start[b] <= start[b + 1] <= n and start[b + 1] - start[b] <= most and lens[b] >= 0
            and lens[b] + start[b + 1] - start[b] <= limit]
    owners = [[b for b in good if start[b] <= r < start[b + 1]] for r in range(n)]
    alone = []                                                     # the queries, by sequence
    for b in good:                                                 # (each writes its own pages and tails only)
        s = [start[b]] * (b + 1) + [start[b + 1]] * (seqs - b)
        alone.append(qp.paged_append(k, v, c, qp.PagedStep(ints(s), ints(lens), table, n, most), rope, q=q, q_out=torch.full_like(q, 55.0)))
    want = [t.clone() for t in arrays(c)]
    for t, x in zip(arrays(c), before):
        t.copy_(x)
    got = qp.paged_append(k, v, c, qp.PagedStep(ints(start), ints(lens), table, n, most), rope, q=q, q_out=torch.full_like(q, 55.0))
    for name, t, x in zip(("k codes", "v codes", "k scales", "v scales", "k tail", "v tail"), arrays(c), want):
        assert torch.equal(t, x), (name, start[:8])
    by = dict(zip(good, alone))
    for r, mine in enumerate(owners):
        assert any(torch.equal(got[r], by[b][r]) for b in mine) if mine else (got[r] == 55.0).all(), (r, mine, start[:8])
    for t, x in zip(arrays(c), before):
        t.copy_(x)
    return len(good), sum(len(m) > 1 for m in owners)


@pytest.mark.parametrize("D,page,dtype", [(128, 32, E4M3), (64, 64, INT8), (128, 128, E4M3)])
def test_starts_that_do_not_ascend_leave_out_their_own_sequences_only(D, page, dtype):
    lens = [100, 40, 70, 0]
    c, table = make(4, 4, 2, D, page, dtype, 512, seed=1)
    fill(c, table, lens, 5)
    seen = [check_left_out(c, table, start, lens, 400, 400, 7 + i) for i, start in enumerate((
        [0, 999, 2, 300, 400], [0, 250, 1, 200, 90], [-5, 100, 100, 260, 400], [400, 0, 130, 50, 200], [0, 130, 401, 130, 390],
        [10, 300, 20, 310, 30], [2 ** 31 - 1, -2 ** 31, 7, 150, 150], [300, 200, 100, 50, 0], [0, 100, 200, 300, 400]))]
    assert [s[0] for s in seen] == [2, 2, 3, 2, 2, 2, 2, 0, 4] and any(s[1] for s in seen), seen


def test_starts_of_many_sequences_that_do_not_ascend():
    seqs, n = 300, 700
    lens = [(37 * b) % 90 for b in range(seqs)]
    c, table = make(seqs, 2, 1, 64, 32, E4M3, 400, seed=1)
    fill(c, table, lens, 5)
    start = [0] * (seqs + 1)
    for b in range(seqs):
        start[b + 1] = start[b] + (b * b) % 5
    assert start[-1] <= n
    start[7], start[150], start[299] = 5000, 3, -1
    good, twice = check_left_out(c, table, start, lens, n, 700, 3)
    assert 290 < good < 300 and twice > 0


# Every block in turn reports that a wait ran out, after all its waits have returned (the range-checked build has a call for it).  The
# rows that hang on it are NaN, all others as they were: a part that was left out instead would show in other bits.
GIVE_UP = """
import torch
from paper_2412_12706_b200 import qp
from tests.test_gpu_paged import E4M3, INT8, fill, ints, make, randn, start_of
for Hq, Hkv, D, page, dtype, lens, new in (
        (8, 2, 128, 64, E4M3, [3000, 5], [1, 1]), (8, 8, 64, 32, INT8, [700] * 9, [1] * 9), (8, 1, 128, 32, E4M3, [900], [3]),
        (8, 2, 64, 128, E4M3, [1000, 20], [4, 2]),
        (4, 2, 128, 32, E4M3, [500, 70], [100, 33]), (2, 2, 64, 32, INT8, [100, 300], [100, 77]), (8, 1, 128, 64, INT8, [3000, 5], [300, 1]),
        (8, 8, 64, 32, E4M3, [20 * (b % 5) for b in range(40)], [40 + b for b in range(40)])):
    total = [a + b for a, b in zip(lens, new)]
    c, table = make(len(lens), Hq, Hkv, D, page, dtype, max(total))
    fill(c, table, total, 5)
    q = randn((sum(new), Hq, D), 1)
    step = qp.PagedStep(start_of(new), ints(lens), table, sum(new), max(new))
    good = qp.paged_attn(q, c, step)
    assert torch.isfinite(good).all()
    seen, blocks = torch.zeros(good.shape[:2], dtype=torch.bool, device="cuda"), 0
    for block in range(148):
        assert qp.debug_give_up(block) == 0
        out = qp.paged_attn(q, c, step)
        lost = torch.isnan(out).all(-1)
        assert torch.equal(out[~lost], good[~lost]), (Hq, Hkv, D, lens, block)
        seen |= lost
        blocks += bool(lost.any())
    G, work = Hq // Hkv, 0                                         # at least: a block for 32 tiles of 32 tokens, or for one of 128
    for n, m in zip(total, new):
        work += Hkv * (-(-m * G // 256) * -(-(n - m) // 128) if max(new) * G > 32 else n // page * page // 32 // 32)
    assert seen.all() and blocks >= max(1, min(148, work)), (blocks, work)
    assert qp.debug_give_up(-1) == 0 and torch.equal(good, qp.paged_attn(q, c, step))
print("poisoned")
"""


def test_what_a_block_lost_whose_wait_ran_out_is_nan():
    env = dict(os.environ, QP_LIBRARY=os.environ.get("QP_CHECKED_LIBRARY") or os.path.join(ROOT, "paper_2412_12706_b200", "libqp_checked.so"))
    r = subprocess.run([sys.executable, "-c", GIVE_UP], env=env, cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "poisoned", r.stdout[-1000:] + r.stderr[-3000:]


# The range-checked build says which number of a step it left out; what comes out is the normal build's.
CHECKED = """
import torch
from paper_2412_12706_b200 import qp
from tests.test_gpu_paged import E4M3, fill, ints, make, randn, start_of
for new in ([1, 1], [60, 3]):
    lens, n = [100, 40], sum(new)
    c, table = make(2, 8, 2, 128, 32, E4M3, 256)
    fill(c, table, lens, 5)
    q, k = randn((n, 8, 128), 1), randn((n, 2, 128), 2)
    def run(start=start_of(new).tolist(), ln=lens, t=table, attend=True):
        step = qp.PagedStep(ints(start), ints(ln), t, n, max(new))
        turned = qp.paged_append(k, k, c, step, qp.rope(128), q=q)
        out = qp.paged_attn(q, c, step, out=torch.full_like(q, 77.0)) if attend else None
        status, words = qp.debug_check()
        assert status == STATUS, status
        return out, words
    good, words = run()
    assert words == [0, 0, 0, 0] and torch.isfinite(good).all(), words
    bad = table.clone()
    bad[0, 1] = c.desc.n_pages + 5
    for got, site, index, limit in ((run(t=bad), 9, c.desc.n_pages + 5, c.desc.n_pages), (run([0, new[0], n + 1]), 7, new[1] + 1, min(max(new), new[1]) + 1),
                                    (run([-1, new[0], n]), 7, 2 ** 32 - 1, n + 1), (run(ln=[256, 40]), 8, 256, 256 - new[0] + 1)):
        out, words = got
        if STATUS == 0:
            assert words[:3] == [1 + site, index, limit] and words[3] > 0, (words, site, index, limit)
        if site == 9:
            assert torch.isnan(out[:new[0]]).all() and torch.equal(out[new[0]:], good[new[0]:])
        else:
            lost = slice(new[0], n) if site == 7 and index == new[1] + 1 else slice(0, new[0])
            kept = slice(0, new[0]) if lost.start else slice(new[0], n)
            assert (out[lost] == 77.0).all() and torch.equal(out[kept], good[kept])
    assert run()[1] == [0, 0, 0, 0]
print("checked")
"""


@pytest.mark.parametrize("library,status", [("libqp_checked.so", 0), ("libqp.so", 2)])
def test_the_range_checked_build_names_what_was_left_out(library, status):
    env = dict(os.environ, QP_LIBRARY=os.path.join(ROOT, "paper_2412_12706_b200", library))
    r = subprocess.run([sys.executable, "-c", CHECKED.replace("STATUS", str(status))], env=env, cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "checked", r.stdout[-1000:] + r.stderr[-3000:]


def overlapping_run(apart):
    """Decode calls that may overlap one another, each handing its output to rotations, appends and paged attention that write what the
    next reads; apart: with a synchronisation after every call."""
    Bt, H, D, steps, page = 1, 8, 128, 40, 32
    K, V = randn((Bt, H, 600, D), 1), randn((Bt, H, 600, D), 2)
    X, _ = qp.compress_layer(K, V, randn((Bt, H, 32, D), 3), 256 * 8, 8, 32, 7)
    c, table = make(1, H, H, D, page, E4M3, 200)
    rope, ws = qp.rope(D), qp.new_decode_workspace(qp.decode_workspace_bytes(X), DEV)
    paged_ws = qp.new_decode_workspace(qp.paged_attn_workspace_bytes(c, 1, 1), DEV)
    outs = [torch.zeros((Bt, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(5 * steps)]
    done = torch.cuda.synchronize if apart else lambda: None
    start, lens = ints([0, 1]), [ints([s]) for s in range(steps)]
    plan = [qp.PagedStep(start, n, table, 1, 1) for n in lens]
    q = randn((Bt, H, D), 4)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        qp.decode_overlap(True)
        for s in range(steps):
            a, b, t, o, e = outs[5 * s:5 * s + 5]
            qp.decode_attn(q, X, a, ws); done()
            qp.decode_attn(a, X, b, ws); done()
            qp.rotary(b.view(Bt, H, 1, D), lens[s], rope, out=t.view(Bt, H, 1, D)); done()
            qp.decode_attn(t, X, e, ws); done()
            qp.paged_append(t, b, c, plan[s], rope, q=e, q_out=o); done()
            qp.decode_attn(o, X, a, ws); done()
            qp.paged_attn(a, c, plan[s], out=e, workspace=paged_ws); done()
            q = e
        qp.decode_overlap(False)
    torch.cuda.synchronize()
    n = steps // page * page
    ids = table[0, :n // page].long()
    return outs + [c.k_tail[0, :, :steps - n], c.v_tail[0, :, :steps - n]] + [t.view(torch.uint8)[ids] for t in (c.k_codes, c.v_codes)]


def test_paged_calls_among_decode_calls_that_may_overlap():
    want = overlapping_run(True)
    assert all(torch.isfinite(t.float()).all() for t in want)
    for _ in range(5):
        for i, (a, b) in enumerate(zip(want, overlapping_run(False))):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("v_scale", [2.0 ** -60, 1.0, 2.0 ** 34])
@pytest.mark.parametrize("new", [[2, 1], [40, 9], [300, 70]])
def test_values_that_are_zero_beside_small_and_large_ones(dtype, v_scale, new):
    """Whole pages, and 32 waiting rows, of zeros take their share of the weight and leave the others theirs."""
    lens = [500, 70]
    total = [a + b for a, b in zip(lens, new)]
    c, table = make(2, 8, 2, 128, 128, dtype, max(total))
    fill(c, table, total, 11, 1.0, v_scale)
    for b, i in ((0, 0), (0, 2)):                                  # the first of all, and one between others
        row = int(table[b, i])
        c.v_codes.view(torch.uint8)[row] = 0
        c.v_scale[row] = 0
    c.v_tail[1, 0, :32] = 0
    check_attn(c, table, lens, new)


@pytest.mark.parametrize("rot,inter", [(128, False), (80, False), (64, True), (22, False)])
@pytest.mark.parametrize("dtype,page", [(E4M3, 32), (INT8, 128)])
def test_every_call_rounds_a_rotation_alike(rot, inter, dtype, page):
    """Many numbers, so that sums that nearly cancel are among them, where fused and separate products round differently: queries and keys
    of an append are qp_rotary's, and a page holds the same, whatever the calls' sizes, which choose between kernels."""
    n, Hq, Hkv, D = 6000, 32, 8, 128
    k, q = randn((n, Hkv, D), 1), randn((n, Hq, D), 2)
    rope = qp.rope(rot, 500000.0, inter)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    turn = lambda x: qp.rotary(x.transpose(0, 1)[None], pos, rope)[0].transpose(0, 1)
    kr, qr = turn(k), turn(q)
    assert torch.equal(qr[:, :1], torch.cat([qp.rotary(q[i:i + 500, :1].transpose(0, 1)[None], pos[i:i + 500], rope)[0].transpose(0, 1)
                                             for i in range(0, n, 500)]))
    held = []
    for size in (n, 500, 37):
        c, table = make(1, Hq, Hkv, D, page, dtype, n)
        for i in range(0, n, size):
            m = min(size, n - i)
            out = qp.paged_append(k[i:i + m], k[i:i + m], c, qp.PagedStep(ints([0, m]), ints([i]), table, m, m), rope, q=q[i:i + m])
            assert torch.equal(out, qr[i:i + m]), (size, i, int((out != qr[i:i + m]).sum()))
        held.append([t[table[0, :n // page].long()] for t in arrays(c)[:4]] + [c.k_tail[0, :, :n % page]])
        check_cache(c, table, [kr], [k], [n], dtype)
    for other in held[1:]:
        assert all(torch.equal(a, b) for a, b in zip(held[0], other))
