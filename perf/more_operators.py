"""The operators of a paged cache in 8 bits and of the position rotation that goes before it: cases, inputs, plain forms and
64-bit values.

  rotary  queries or keys turned by their positions (interleaved or half layout, part of the head, scaled for long contexts), and back
  append  new tokens of several sequences: keys rotated and both taken into the paged cache, queries rotated on the way
  attn    attention of the new tokens over their sequences' pages and waiting rows, from one token each to a prompt's chunk

A page holds `page` tokens of every KV head in 8 bits with one scale for the keys and one for the values of each page and head;
tokens behind a sequence's last whole page wait in 16 bits.  With `own` false, run() computes elementary torch operations; with
`own` true it makes a user's calls.
"""
import math
import random

import torch

own = False
DEV = "cuda"
TOP = {"e4m3": 448.0, "int8": 127.0}


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # the rotation alone of one new token's queries: latency
        dict(name="rotate 1", op="rotary", batch=1, heads=32, d=128, rot=128, inter=False, scaling="plain", factor=1.0, len=1, far=5000,
             fused=False, back=False),
        # the queries of a whole prompt, read from a fused projection's rows
        dict(name="rotate 8k", op="rotary", batch=1, heads=32, d=128, rot=128, inter=False, scaling="bands", factor=8.0, len=8192, far=0,
             fused=True, back=False),
        # the gradient's way: a quarter-million positions, half of small heads, interleaved, odd length
        dict(name="rotate back 5001 d64", op="rotary", batch=3, heads=8, d=64, rot=32, inter=True, scaling="yarn", factor=16.0, len=5001,
             far=250000, fused=False, back=True),
        # one generation step of one sequence: latency
        dict(name="append 1", op="append", hq=32, hkv=8, d=128, rot=128, inter=False, scaling="plain", factor=1.0, fmt="e4m3", page=64,
             seqs=1, lo=2000, hi=2000, new_lo=1, new_hi=1, fused=True),
        # one generation step of a batch, some of whose pages are completed by it
        dict(name="append 1 x 64", op="append", hq=32, hkv=8, d=128, rot=128, inter=False, scaling="bands", factor=8.0, fmt="e4m3",
             page=32, seqs=64, lo=100, hi=3000, new_lo=1, new_hi=1, fused=True),
        # a prompt
        dict(name="append 8k", op="append", hq=32, hkv=8, d=128, rot=128, inter=False, scaling="bands", factor=8.0, fmt="e4m3", page=64,
             seqs=1, lo=0, hi=0, new_lo=8192, new_hi=8192, fused=True),
        # chunks of several prompts whose keys come rotated, small heads, whole numbers
        dict(name="append chunks int8 d64", op="append", hq=8, hkv=2, d=64, rot=0, inter=False, scaling="plain", factor=1.0, fmt="int8",
             page=128, seqs=7, lo=0, hi=3000, new_lo=1, new_hi=1500, fused=False),
        # a generation step of one sequence: latency
        dict(name="attend 1 on 2k", op="attn", hq=32, hkv=8, d=128, fmt="e4m3", page=64, seqs=1, lo=2000, hi=2000, new_lo=1, new_hi=1),
        # a generation step of a batch of sequences of very different lengths
        dict(name="attend 1 x 64 ragged", op="attn", hq=32, hkv=8, d=128, fmt="e4m3", page=64, seqs=64, lo=1, hi=16000, new_lo=1, new_hi=1),
        # a generation step over long contexts, 70B shapes, whole numbers
        dict(name="attend 1 x 8 on 32k int8", op="attn", hq=64, hkv=8, d=128, fmt="int8", page=128, seqs=8, lo=30000, hi=32700, new_lo=1,
             new_hi=1),
        # a few drafted tokens a sequence
        dict(name="attend 5 x 16 on 4k", op="attn", hq=32, hkv=8, d=128, fmt="e4m3", page=32, seqs=16, lo=3000, hi=4100, new_lo=5, new_hi=5),
        # the last, ragged chunk of a prompt that is taken in by chunks, 70B shapes
        dict(name="attend chunk 1999 of 16k", op="attn", hq=64, hkv=8, d=128, fmt="e4m3", page=64, seqs=1, lo=14301, hi=14301, new_lo=1999,
             new_hi=1999),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    return rng.choice([(32, 8), (64, 8), (8, 2), (8, 8), (4, 4), (28, 4), (6, 2), (8, 1)])


def draw(rng):
    op = rng.choice(["rotary", "append", "append", "attn", "attn", "attn"])
    d = rng.choice([64, 128, 128])
    scaling = rng.choice(["plain", "plain", "linear", "ntk", "yarn", "bands"])
    factor = 1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.0, 16.0])
    rot = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(2, d // 2)])
    if op == "rotary":
        heads = rng.choice([1, 2, 7, 8, 32, 64])
        batch = rng.choice([1, 1, 2, 5])
        n = min(_log(rng, 1, 8192), max(1, 8192 * 32 * 128 // (heads * batch * d)))
        return dict(op=op, batch=batch, heads=heads, d=d, rot=rot, inter=rng.choice([False, True]), scaling=scaling, factor=factor, len=n,
                    far=rng.choice([0, 1000, 100000, 1000000]), fused=rng.choice([False, True]), back=rng.choice([False, False, True]))
    hq, hkv = _heads(rng)
    fmt = rng.choice(["e4m3", "int8"])
    page = rng.choice([32, 64, 128])
    seqs = rng.choice([1, 1, 2, 3, 8, 13, 64])
    hi = _log(rng, 1, 16000)
    lo = rng.choice([0, hi, hi // 2])
    new_hi = rng.choice([1, 1, 1, 2, 5, 16, _log(rng, 17, 4000)])
    if op == "append":
        if fmt == "int8":
            rot = 0                                                # codes are compared as whole numbers
        new_hi = max(1, min(new_hi, 8192 * 40 * 128 // (seqs * (hq + 2 * hkv) * d)))
        return dict(op=op, hq=hq, hkv=hkv, d=d, rot=rot, inter=rng.choice([False, True]), scaling=scaling, factor=factor, fmt=fmt, page=page,
                    seqs=seqs, lo=lo, hi=hi, new_lo=rng.choice([1, new_hi]), new_hi=new_hi, fused=rng.choice([False, True]))
    most = 8 * 32700 * 8 * 128                                     # numbers of a cache, and pairs of query and key
    hi = min(hi, max(1, most // (seqs * hkv * d)))
    new_hi = max(1, min(new_hi, 64 * 1999 * 16300 // (seqs * hq * (hi + new_hi))))
    lo = min(lo, hi)
    return dict(op=op, hq=hq, hkv=hkv, d=d, fmt=fmt, page=page, seqs=seqs, lo=lo, hi=hi, new_lo=rng.choice([1, new_hi]), new_hi=new_hi)


# ------------------------------------------------------------------------------------------------ inputs

def _numbers(case):
    """Tokens before the step and new tokens of every sequence: of the case alone, the same for every seed."""
    r = random.Random(case["seqs"] * 1000003 + case["hi"] * 101 + case["new_hi"])
    old = [r.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    old[0], new[0] = case["hi"], case["new_hi"]
    return old, new


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _rows(g, n, heads, d, fused):
    """bf16 rows [n, heads, d]; fused: a part of a projection's wider rows."""
    wide = torch.randn((n, heads + (4 if fused else 0), d), generator=g, device=DEV)
    wide[:, :, :3] *= 1.5
    return wide.to(torch.bfloat16)[:, :heads]


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _step(case, seed):
    old, new = _numbers(case)
    page, seqs = case["page"], case["seqs"]
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    need = [(o + n + page - 1) // page for o, n in zip(old, new)]
    most = max(need)
    n_pages = sum(need) + 3
    # pages in any order, as a cache that has served for a while gives them out
    order = torch.randperm(n_pages, generator=_gen(seed + 1), device=DEV).to(torch.int32)
    table = torch.zeros((seqs, most), dtype=torch.int32, device=DEV)
    first = 0
    for b, n in enumerate(need):
        table[b, :n] = order[first:first + n]
        first += n
    return dict(start=_int(start), len=_int(old), pages=table, n_tokens=start[-1], n_pages=n_pages, max_pages=most, max_new=max(new),
                longest=max(o + n for o, n in zip(old, new)))


def _scale_of(top, fmt):
    """The stored scale (bf16) of blocks with these largest magnitudes: rounded up, so that nothing is cut off."""
    x = top / torch.full_like(top, TOP[fmt])
    return ((x.view(torch.int32) + 0xffff) >> 16).to(torch.int16).view(torch.bfloat16)


def _codes(x, scale, fmt):
    """x fp32 [..., page, d] -> codes, by the stored scale [...]."""
    s = scale.float()[..., None, None]
    inv = torch.where(s > 0, (torch.ones_like(s) / s).clamp(max=torch.finfo(torch.float32).max), torch.zeros_like(s))
    y = (x * inv).clamp(-TOP[fmt], TOP[fmt])
    return y.to(torch.float8_e4m3fn) if fmt == "e4m3" else torch.round(y).to(torch.int8)


def _pool(g, case, n_pages):
    """Codes and scales of pages in use: noise with a few heavier channels, pages of different loudness."""
    shape = (n_pages, case["hkv"], case["page"], case["d"])
    x = torch.randn(shape, generator=g, device=DEV)
    x[..., :3] *= 3.0
    x *= 0.5 + torch.rand((n_pages, case["hkv"], 1, 1), generator=g, device=DEV)
    s = _scale_of(x.abs().amax((2, 3)), case["fmt"])
    return _codes(x, s, case["fmt"]), s


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "rotary":
        b, h, n, d = case["batch"], case["heads"], case["len"], case["d"]
        if case["fused"]:                                          # [batch, len, wide] rows, seen head by head
            x = torch.randn((b, n, h + 4, d), generator=g, device=DEV).to(torch.bfloat16)[:, :, :h].transpose(1, 2)
        else:
            x = torch.randn((b, h, n, d), generator=g, device=DEV).to(torch.bfloat16)
        first = torch.randint(0, case["far"] + 1, (b, 1), generator=g, device=DEV)
        return dict(case=case, x=x, pos=(first + torch.arange(n, device=DEV)).to(torch.int32))
    s = dict(case=case, **_step(case, seed))
    n, page, d, hkv, seqs = s["n_tokens"], case["page"], case["d"], case["hkv"], case["seqs"]
    (s["kc"], s["ks"]), (s["vc"], s["vs"]) = _pool(g, case, s["n_pages"]), _pool(g, case, s["n_pages"])
    s["kt"] = _rows(g, seqs * hkv, page, d, False).view(seqs, hkv, page, d)
    s["vt"] = _rows(g, seqs * hkv, page, d, False).view(seqs, hkv, page, d)
    if case["op"] == "append":
        s["k"], s["v"] = _rows(g, n, hkv, d, case["fused"]), _rows(g, n, hkv, d, case["fused"])
        s["q"] = _rows(g, n, case["hq"], d, case["fused"]) if case["rot"] else None
    else:
        s["q"] = _rows(g, n, case["hq"], d, False)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

BASE, TRAINED = 500000.0, 8192


def _frequencies(case):
    """Radians a position, one for each rotated pair, and the factor on the rotated channels."""
    rot, kind, s = case["rot"], case["scaling"], case["factor"]
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    base = BASE * s ** (rot / (rot - 2)) if kind == "ntk" else BASE
    f = base ** (-2.0 * i / rot)
    if kind == "linear":
        return f / s, 1.0
    if kind == "yarn":                                             # fast pairs stay, slow ones are stretched, a ramp between
        at = lambda turns: rot * math.log(TRAINED / (turns * 2 * math.pi)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rot - 1)
        ramp = ((i - lo) / (hi - lo if hi != lo else 0.001)).clamp(0, 1)
        return f / s * ramp + f * (1 - ramp), 0.1 * math.log(s) + 1.0
    if kind == "bands":                                            # by the turns a pair makes over the trained length: 1 and 4
        turns = TRAINED * f / (2 * math.pi)
        keep = ((turns - 1.0) / 3.0).clamp(0, 1)
        return f / s * (1 - keep) + f * keep, 1.0
    return f, 1.0


def _turned(x, pos, case, back=False):
    """x [..., d] whose positions broadcast as pos[..., None]: fp32, before the last rounding."""
    f, m = _frequencies(case)
    rot = case["rot"]
    a = pos.double()[..., None] * f                                # in 64 bits: angles of far positions
    c, s = (torch.cos(a) * m).float(), (torch.sin(a) * m).float()
    if back:
        s = -s
    x = x.float()
    y = x.clone()
    if case["inter"]:
        u, v = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = u * c - v * s, v * c + u * s
    else:
        u, v = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = u * c - v * s, v * c + u * s
    return y


def _plain_rotary(s):
    c = s["case"]
    return _turned(s["x"], s["pos"][:, None], c, c["back"]).to(torch.bfloat16)


def _owner(s):
    """Sequence and place in it of every row, and its position."""
    rows = torch.arange(s["n_tokens"], device=DEV)
    seq = torch.searchsorted(s["start"][1:].long(), rows, right=True)
    return seq, s["len"].long()[seq] + rows - s["start"].long()[seq]


def _plain_append(s):
    c = s["case"]
    page, fmt = c["page"], c["fmt"]
    seq, pos = _owner(s)
    k, q = s["k"], s["q"]
    if c["rot"]:
        k = _turned(k, pos[:, None], c).to(torch.bfloat16)
        q = _turned(q, pos[:, None], c).to(torch.bfloat16)
    end = s["len"].long() + (s["start"][1:] - s["start"][:-1]).long()
    # whole pages: those that end in a new token
    at = torch.arange(s["max_pages"], device=DEV)
    whole = ((at[None] + 1) * page <= end[:, None]) & ((at[None] + 1) * page > s["len"].long()[:, None])
    b, p = torch.nonzero(whole, as_tuple=True)
    place = p[:, None] * page + torch.arange(page, device=DEV)     # positions of the page's tokens
    fresh = place >= s["len"].long()[b][:, None]
    row = (s["start"].long()[b][:, None] + place - s["len"].long()[b][:, None]).clamp(min=0)
    ids = s["pages"][b, p].long()
    for new, tail, codes, scale in ((k, s["kt"], s["kc"], s["ks"]), (s["v"], s["vt"], s["vc"], s["vs"])):
        if len(b):
            x = torch.where(fresh[:, :, None, None], new[row], tail[b].transpose(1, 2)).float().transpose(1, 2)
            sc = _scale_of(x.abs().amax((2, 3)), fmt)
            scale[ids] = sc
            codes.view(torch.uint8)[ids] = _codes(x, sc, fmt).view(torch.uint8)
        waits = pos >= (end // page * page)[seq]
        tail[seq[waits], :, pos[waits] % page] = new[waits]
    out = dict(k=s["kc"], v=s["vc"], ks=s["ks"], vs=s["vs"], kt=s["kt"], vt=s["vt"])
    if c["rot"]:
        out["q"] = q
    return out


def _sequences(s, codes, scale, tail, n):
    """fp32 [seqs, hkv, n, d]: what pages and waiting rows hold, in order (anything behind the last token)."""
    c = s["case"]
    page, d = c["page"], c["d"]
    p = -(-n // page)
    x = codes.view(torch.uint8)[s["pages"][:, :p].long()].view(codes.dtype).float() * scale[s["pages"][:, :p].long()].float()[..., None, None]
    x = x.transpose(1, 2).reshape(c["seqs"], c["hkv"], p * page, d)
    at = torch.arange(p * page, device=DEV)
    end = s["len"].long() + (s["start"][1:] - s["start"][:-1]).long()
    waits = at[None] >= (end // page * page)[:, None]
    # (by blocks, so that the rows are not repeated)
    return torch.where(waits[:, None, :, None], tail.float().repeat(1, 1, p, 1), x)[:, :, :n]


def _plain_attn(s):
    c = s["case"]
    hq, hkv, d, seqs, m, n = c["hq"], c["hkv"], c["d"], c["seqs"], s["max_new"], s["longest"]
    G = hq // hkv
    i = torch.arange(m, device=DEV)
    count = (s["start"][1:] - s["start"][:-1]).long()
    row = (s["start"][:-1].long()[:, None] + i).clamp(max=s["n_tokens"] - 1)
    q = s["q"][row].float().view(seqs, m, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, G * m, d)
    k = _sequences(s, s["kc"], s["ks"], s["kt"], n)
    x = (q @ k.transpose(2, 3)).view(seqs, hkv, G, m, n)
    del k
    x *= 1.0 / math.sqrt(d)
    seen = torch.arange(n, device=DEV)[None, None] <= (s["len"].long()[:, None] + i)[:, :, None]
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    x /= x.sum(-1, keepdim=True)
    v = _sequences(s, s["vc"], s["vs"], s["vt"], n)
    v.masked_fill_((torch.arange(n, device=DEV)[None] >= (s["len"].long() + count)[:, None])[:, None, :, None], 0.0)
    o = (x.view(seqs, hkv, G * m, n) @ v).view(seqs, hkv, G, m, d).permute(0, 3, 1, 2, 4).reshape(seqs, m, hq, d)
    return o[i[None] < count[:, None]].to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ the framework's calls

def _handle(s):
    """The rotation, the cache object, the step's numbers and the workspace that a user's program keeps."""
    if "handle" not in s:
        from paper_2412_12706_b200 import qp
        c = s["case"]
        rope = None
        if c.get("rot"):
            rope = qp.rope(c["rot"], BASE, interleaved=c["inter"], scaling=c["scaling"], factor=c["factor"], trained_len=TRAINED)
        if c["op"] == "rotary":
            s["handle"] = rope
            return rope
        cache = qp.paged_cache(c["hq"], s["kc"], s["vc"], s["ks"], s["vs"], s["kt"], s["vt"], s["max_pages"])
        step = qp.PagedStep(s["start"], s["len"], s["pages"], s["n_tokens"], s["max_new"])
        workspace = None
        if c["op"] == "attn":
            workspace = qp.new_decode_workspace(qp.paged_attn_workspace_bytes(cache, s["n_tokens"], s["max_new"]), DEV)
        s["handle"] = rope, cache, step, workspace
    return s["handle"]


def _own(s):
    from paper_2412_12706_b200 import qp
    c = s["case"]
    if c["op"] == "rotary":
        return qp.rotary(s["x"], s["pos"], _handle(s), transpose=c["back"])
    rope, cache, step, workspace = _handle(s)
    if c["op"] == "attn":
        return qp.paged_attn(s["q"], cache, step, workspace=workspace)
    q = qp.paged_append(s["k"], s["v"], cache, step, rope, q=s["q"])
    out = dict(k=s["kc"], v=s["vc"], ks=s["ks"], vs=s["vs"], kt=s["kt"], vt=s["vt"])
    if c["rot"]:
        out["q"] = q
    return out


def run(state):
    if own:
        return _own(state)
    return {"rotary": _plain_rotary, "append": _plain_append, "attn": _plain_attn}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ work and exact values

def work(case):
    if case["op"] == "rotary":
        n = case["batch"] * case["heads"] * case["len"]
        return dict(bytes=4 * n * case["d"] + 4 * case["batch"] * case["len"], flops=3 * n * case["rot"])
    old, new = _numbers(case)
    page, hq, hkv, d = case["page"], case["hq"], case["hkv"], case["d"]
    total = sum(new)
    if case["op"] == "append":
        done = sum((o + n) // page - o // page for o, n in zip(old, new))              # pages completed
        kept = sum(min(o % page, page) for o, n in zip(old, new) if (o + n) // page > o // page)   # waiting rows they take in
        waits = sum(min(n, (o + n) % page) for o, n in zip(old, new))
        rows = 4 * hkv * d * (total + kept + waits) + 2 * hkv * done * (page * d + 2)
        q = 4 * total * hq * d if case["rot"] else 0
        return dict(bytes=rows + q + 4 * (2 * case["seqs"] + done), flops=3 * total * (hq + hkv) * case["rot"])
    held = sum(2 * hkv * d * ((o + n) // page * page + 2 * ((o + n) % page)) + 4 * hkv * ((o + n) // page) for o, n in zip(old, new))
    pairs = sum(n * o + n * (n + 1) // 2 for o, n in zip(old, new))
    return dict(bytes=held + 4 * total * hq * d + 4 * sum((o + n + page - 1) // page for o, n in zip(old, new)), flops=4 * hq * d * pairs)


def _rotated64(x, pos, case, sign):
    """Pair by pair from the definition, in 64 bits: x [..., d], pos broadcasting over x[..., 0]."""
    rot, s = case["rot"], case["factor"]
    y = x.double().clone()
    # the ramp's ends of "yarn": pair numbers at which 32 turns, and one, are made over the trained length
    ends = [rot * math.log(TRAINED / (t * math.tau)) / (2 * math.log(BASE)) for t in (32.0, 1.0)] if case["scaling"] == "yarn" else [0, 0]
    ends = [max(math.floor(ends[0]), 0), min(math.ceil(ends[1]), rot - 1)]
    for i in range(rot // 2):
        w = BASE ** (-2 * i / rot)
        m = 1.0
        if case["scaling"] == "linear":
            w /= s
        elif case["scaling"] == "ntk":
            w = (BASE * s ** (rot / (rot - 2))) ** (-2 * i / rot)
        elif case["scaling"] == "yarn":
            t = min(1.0, max(0.0, (i - ends[0]) / ((ends[1] - ends[0]) or 0.001)))
            w = w * ((1 - t) + t / s)
            m = 1.0 + math.log(s) / 10
        elif case["scaling"] == "bands":
            length = math.tau / w
            if length > TRAINED:
                w /= s
            elif length > TRAINED / 4:
                t = (TRAINED / length - 1) / (4 - 1)
                w = (1 - t) * w / s + t * w
        u, v = (2 * i, 2 * i + 1) if case["inter"] else (i, i + rot // 2)
        z = torch.polar(torch.full((), m, dtype=torch.float64, device=DEV).expand(pos.shape), sign * w * pos.double())
        z = z * torch.complex(x[..., u].double(), x[..., v].double())
        y[..., u], y[..., v] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _rotated64(s["x"], s["pos"][:, None], case, -1.0 if case["back"] else 1.0)
    old, new = _numbers(case)
    page, hkv, hq, d = case["page"], case["hkv"], case["hq"], case["d"]
    first = [sum(new[:b]) for b in range(case["seqs"])]
    if case["op"] == "append":
        pos = torch.cat([torch.arange(o, o + n, device=DEV) for o, n in zip(old, new)])
        k = _rotated64(s["k"], pos[:, None], case, 1.0) if case["rot"] else s["k"].double()
        out = dict(k=None, v=None, ks=None, vs=None, kt=s["kt"].double(), vt=s["vt"].double())
        for b, (o, n) in enumerate(zip(old, new)):
            lo = max(o, (o + n) // page * page)
            for name, x in (("kt", k), ("vt", s["v"].double())):
                if lo < o + n:
                    out[name][b, :, lo % page:lo % page + o + n - lo] = x[first[b] + lo - o:first[b] + n].transpose(0, 1)
        if case["rot"]:
            out["q"] = _rotated64(s["q"], pos[:, None], case, 1.0)
        return out
    got = torch.empty((s["n_tokens"], hq, d), dtype=torch.float64, device=DEV)
    for b, (o, n) in enumerate(zip(old, new)):
        end, full = o + n, (o + n) // page
        ids = s["pages"][b, :full].long()
        for h in range(hkv):
            k, v = (torch.cat([(codes[ids.tolist(), h] if codes.dtype == torch.int8 else codes.view(torch.uint8)[ids, h].view(codes.dtype)).double()
                               .mul(scale[ids, h].double()[:, None, None]).reshape(-1, d), tail[b, h, :end - full * page].double()])
                    for codes, scale, tail in ((s["kc"], s["ks"], s["kt"]), (s["vc"], s["vs"], s["vt"])))
            heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
            for lo in range(0, n, 512):
                hi = min(n, lo + 512)
                x = torch.einsum("igd,jd->gij", s["q"][first[b] + lo:first[b] + hi, heads].double(), k) * d ** -0.5
                hide = torch.arange(end, device=DEV) > o + torch.arange(lo, hi, device=DEV)[:, None]
                p = torch.softmax(x.masked_fill(hide, -math.inf), -1)
                got[first[b] + lo:first[b] + hi, heads] = torch.einsum("gij,jd->igd", p, v)
    return got
