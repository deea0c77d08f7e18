"""The operators that keep a KV cache at a fixed budget by accumulated attention weight, and the attention of a tree of
drafted tokens over the cache: cases, inputs, plain forms and 64-bit values.

  prompt  attention weight every prompt token has received from the queries of the prompt, or of a chunk of it
  decode  one decode step over the cache that also adds its attention weights to the tokens' accumulators
  select  the prompt form of the eviction: the heaviest tokens and the most recent ones, with their weights
  evict   the single-token form: the new token takes the place of the lightest token outside the recent ones
  tree    attention of T drafted tokens, each seeing the cache, the waiting tail and its own ancestors

With `own` false, run() computes elementary torch operations; with `own` true it makes a user's calls.
"""
import math

import torch

own = False
DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # a short prompt of the small configuration (64 channels): launch latency
        dict(name="prompt 1k d64", op="prompt", batch=1, hq=8, hkv=2, d=64, L=1024, q_start=0, nq=1024),
        # a whole 8k prompt of the 8B shapes
        dict(name="prompt 8k", op="prompt", batch=1, hq=32, hkv=8, d=128, L=8192, q_start=0, nq=8192),
        # the last, ragged chunk of a prompt that is taken in by chunks, 70B shapes, added to what earlier chunks gave
        dict(name="prompt chunk 1999 of 16k", op="prompt", batch=1, hq=64, hkv=8, d=128, L=16384, q_start=14301, nq=1999),
        # a generation step at the 1/16 budget in 16 bit, one sequence: latency
        dict(name="decode 512 16bit", op="decode", batch=1, hq=32, hkv=8, d=128, n=512, cap=512, bits=16, group=32),
        # the 4-bit cache of the same memory for a batch of long prompts
        dict(name="decode 8192 4bit b8", op="decode", batch=8, hq=32, hkv=8, d=128, n=8192, cap=8192, bits=4, group=32),
        # 16 bit, 70B shapes, an odd number of tokens in an array with room for more
        dict(name="decode 5001 16bit b4 g8", op="decode", batch=4, hq=64, hkv=8, d=128, n=5001, cap=5120, bits=16, group=32),
        # selection after a 32k prompt for a batch of 8
        dict(name="select 8k of 32k b8", op="select", batch=8, hkv=8, L=32768, w=32, n=8192, cap=8192),
        # one new token into a full 16-bit cache, one sequence: latency
        dict(name="evict 512 16bit", op="evict", batch=1, hq=32, hkv=8, d=128, n=512, bits=16, group=32, recent=32),
        # one new token into a full 4-bit cache of a batch
        dict(name="evict 8192 4bit b8", op="evict", batch=8, hq=32, hkv=8, d=128, n=8192, bits=4, group=32, recent=256),
        # a short chain of drafts, small budget, one sequence: latency
        dict(name="tree 8 on 2k 4bit", op="tree", batch=1, hq=32, hkv=8, d=128, n=2048, bits=4, group=32, axis=0, T=8, tail=5),
        # a full tree over an 8k cache in 16 bit
        dict(name="tree 64 on 8k 16bit", op="tree", batch=1, hq=32, hkv=8, d=128, n=8192, bits=16, group=32, axis=0, T=64, tail=0),
        # an odd tree over 2-bit caches of a batch of long prompts
        dict(name="tree 33 on 8k 2bit b8", op="tree", batch=8, hq=32, hkv=8, d=128, n=8192, bits=2, group=32, axis=0, T=33, tail=17),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    return rng.choice([(32, 8), (64, 8), (8, 2), (8, 8), (4, 4), (28, 4), (6, 2), (8, 1)])


def draw(rng):
    op = rng.choice(["prompt", "decode", "select", "evict", "tree"])
    hq, hkv = _heads(rng)
    d = rng.choice([64, 128, 128])
    batch = rng.choice([1, 1, 2, 3, 4, 8])
    bits = rng.choice([16, 16, 8, 4, 2])
    group = rng.choice([g for g in (32, 64, 128) if g <= d])
    if op == "prompt":
        L = _log(rng, 40, 8192)
        batch = max(1, min(batch, 32 * 8192 * 8192 // (hq * L * L)))
        hi = rng.choice([L, L, rng.randint(1, L)])
        nq = rng.choice([hi, hi, rng.randint(1, hi)])
        return dict(op=op, batch=batch, hq=hq, hkv=hkv, d=d, L=L, q_start=hi - nq, nq=nq)
    if op == "select":
        L = _log(rng, 64, 32768)
        w = rng.choice([1, 8, 32, 33])
        n = rng.randint(w + 1, L)
        return dict(op=op, batch=batch, hkv=hkv, L=L, w=w, n=n, cap=n + rng.choice([0, 0, 1, 100]))
    n = _log(rng, 32, 8192)
    if bits < 16:
        n = max(group, n // group * group)
    if op == "decode":
        cap = n + (rng.choice([0, 0, 1, 77]) if bits == 16 else 0)
        return dict(op=op, batch=batch, hq=hq, hkv=hkv, d=d, n=n, cap=cap, bits=bits, group=group)
    if op == "evict":
        return dict(op=op, batch=batch, hq=hq, hkv=hkv, d=d, n=n, bits=bits, group=group, recent=rng.randint(1, n))
    T = _log(rng, 1, 64)
    tail = rng.randint(0, group - 1) if bits < 16 else 0
    return dict(op=op, batch=batch, hq=hq, hkv=hkv, d=d, n=n, bits=bits, group=group, axis=rng.choice([0, 0, 1]) if bits < 16 else 0,
                T=T, tail=tail)


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _keys(g, batch, hkv, n, d):
    """Keys of a prompt: noise, a few heavier channels, and one token in forty along a direction the queries share."""
    k = torch.randn((batch, hkv, n, d), generator=g, device=DEV)
    k[..., :3] *= 4.0
    along = torch.randn((1, hkv, 1, d), generator=g, device=DEV)
    heavy = torch.rand((batch, hkv, n, 1), generator=g, device=DEV) < 0.025
    return (k + 0.6 * along * heavy).to(torch.bfloat16), along


def _half_down(x):
    """Largest fp16 value that is not above x (finite)."""
    h = x.to(torch.float16)
    b = h.view(torch.int16).to(torch.int32)
    lower = torch.where(h > 0, b - 1, torch.where(h < 0, b + 1, torch.full_like(b, -32767)))
    return torch.where(h.float() > x, lower, b).to(torch.int16).view(torch.float16)


def _quantize(x, bits):
    """x fp32 [..., g]: codes int32 [..., g], scale and zero fp16 [...] (zero rounded down, scale up, ties to even)."""
    top = 2 ** bits - 1
    z = _half_down(x.amin(-1))
    s = -_half_down(-((x.amax(-1) - z.float()) / top))
    sf = s.float()[..., None]
    c = torch.where(sf > 0, torch.round((x - z.float()[..., None]) / torch.where(sf > 0, sf, torch.ones_like(sf))), torch.zeros_like(x))
    return c.clamp(0, top).to(torch.int32), s, z


def _pack(c, bits):
    """codes [..., g] -> int32 words [..., g*bits/32], element e of a group in word e // (32/bits)."""
    per = 32 // bits
    c = c.to(torch.int64).view(*c.shape[:-1], -1, per)
    w = (c << (bits * torch.arange(per, device=c.device))).sum(-1)
    return (w - ((w >> 31) << 32)).to(torch.int32).contiguous()


def _unpack(w, bits):
    sh = bits * torch.arange(32 // bits, device=w.device, dtype=torch.int32)
    return ((w[..., None] >> sh) & (2 ** bits - 1)).flatten(-2)


def _cache(k, v, bits, group, axis, cap):
    """The arrays of a packed cache that holds these tokens (keys per channel with axis 0, per token with axis 1)."""
    b, h, n, d = k.shape
    if bits == 16:
        kc = torch.zeros((b, h, cap, d), dtype=torch.bfloat16, device=DEV)
        vc = torch.zeros_like(kc)
        kc[:, :, :n], vc[:, :, :n] = k, v
        return dict(kc=kc, vc=vc, ks=None, kz=None, vs=None, vz=None)
    grouped = k.float().view(b, h, n // group, group, d).transpose(3, 4) if axis == 0 else k.float().view(b, h, n, d // group, group)
    c, ks, kz = _quantize(grouped, bits)
    kc = _pack(c, bits)
    c, vs, vz = _quantize(v.float().view(b, h, n, d // group, group), bits)
    return dict(kc=kc, vc=_pack(c, bits), ks=ks.contiguous(), kz=kz.contiguous(), vs=vs.contiguous(), vz=vz.contiguous())


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = dict(case=case)
    if op == "select":
        # accumulated weights of a prompt: heavy-tailed, larger for early tokens, never negative
        r = torch.rand((case["batch"], case["hkv"], case["L"]), generator=g, device=DEV)
        age = torch.arange(case["L"], 0, -1, device=DEV) / case["L"]
        s["weights"] = age * (1e-3 - torch.log(r + 1e-6)) ** 2
        return s
    b, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    if op == "prompt":
        k, along = _keys(g, b, hkv, case["L"], d)
        q = torch.randn((b, hq, case["nq"], d), generator=g, device=DEV)
        q = q + 0.6 * along.repeat_interleave(hq // hkv, dim=1)
        # what the chunks before this one have given
        before = torch.rand((b, hkv, case["L"]), generator=g, device=DEV) * (torch.arange(case["L"], device=DEV) < case["q_start"])
        s.update(q=q.to(torch.bfloat16), k=k, weights=before.contiguous())
        return s
    n, bits, group = case["n"], case["bits"], case["group"]
    axis = case.get("axis", 1)
    k, along = _keys(g, b, hkv, n, d)
    v = torch.randn((b, hkv, n, d), generator=g, device=DEV).to(torch.bfloat16)
    cap = case.get("cap", n)
    s["cache"] = _cache(k, v, bits, group, axis, cap)
    along = along.transpose(1, 2)                                           # [1, 1, hkv, d]
    if op == "evict":
        s["k_new"] = _keys(g, b, hkv, 1, d)[0][:, :, 0].contiguous()
        s["v_new"] = torch.randn((b, hkv, d), generator=g, device=DEV).to(torch.bfloat16)
        s["weights"] = torch.log(torch.rand((b, hkv, n), generator=g, device=DEV) + 1e-6) ** 2
        # kept positions: ascending, as the selection leaves them
        s["pos"] = (torch.cumsum(torch.randint(1, 4, (b, hkv, n), generator=g, device=DEV), -1)).to(torch.int32)
        s["new_pos"] = 3 * n + 1
        return s
    if op == "decode":
        q = torch.randn((b, hq, d), generator=g, device=DEV) + 0.6 * along[:, 0].repeat_interleave(hq // hkv, dim=1)
        s["q"] = q.to(torch.bfloat16)
        s["weights"] = torch.rand((b, hkv, cap), generator=g, device=DEV)
        return s
    T = case["T"]
    q = torch.randn((b, T, hq, d), generator=g, device=DEV) + 0.6 * along.repeat_interleave(hq // hkv, dim=2)
    s["q"] = q.to(torch.bfloat16)
    s["kd"] = torch.randn((b, T, hkv, d), generator=g, device=DEV).to(torch.bfloat16)
    s["vd"] = torch.randn((b, T, hkv, d), generator=g, device=DEV).to(torch.bfloat16)
    s["kt"] = torch.randn((b, hkv, group, d), generator=g, device=DEV).to(torch.bfloat16)
    s["vt"] = torch.randn((b, hkv, group, d), generator=g, device=DEV).to(torch.bfloat16)
    # a random tree in which every node hangs on an earlier one (or on the context); a node sees its ancestors and itself
    i = torch.arange(T, device=DEV)
    parent = (torch.rand((b, T), generator=g, device=DEV) * (i + 1)).long() - 1
    sees = torch.zeros((b, T, T), dtype=torch.bool, device=DEV)
    sees[:, i, i] = True
    link = torch.zeros((b, T, T), device=DEV).scatter_(2, parent.clamp(min=0)[..., None], (parent >= 0).float()[..., None])
    reach = link + torch.eye(T, device=DEV)
    for _ in range(6):                                                      # ancestors by doubling: 2^6 >= 64 levels
        reach = (reach @ reach > 0).float()
    s["mask"] = ((reach > 0).long() << i).sum(-1)                           # bit j: node j
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _values(cache, case, axis):
    """Keys and values that the cache stands for, fp32 [b, hkv, n, d]."""
    n, bits, d = case["n"], case["bits"], case["d"]
    if bits == 16:
        return cache["kc"][:, :, :n].float(), cache["vc"][:, :, :n].float()
    ck, cv = _unpack(cache["kc"], bits), _unpack(cache["vc"], bits)
    k = ck.float() * cache["ks"].float()[..., None] + cache["kz"].float()[..., None]
    v = cv.float() * cache["vs"].float()[..., None] + cache["vz"].float()[..., None]
    b, h = k.shape[:2]
    k = k.transpose(3, 4).reshape(b, h, n, d) if axis == 0 else k.reshape(b, h, n, d)
    return k, v.reshape(b, h, n, d)


def _plain_prompt(s):
    c = s["case"]
    b, hq, hkv, d, nq, q0 = c["batch"], c["hq"], c["hkv"], c["d"], c["nq"], c["q_start"]
    G, n = hq // hkv, c["q_start"] + c["nq"]
    q = s["q"].float().view(b, hkv, G * nq, d)
    p = (q @ s["k"][:, :, :n].float().transpose(2, 3)).view(b, hkv, G, nq, n)
    p *= 1.0 / math.sqrt(d)
    rows = q0 + torch.arange(nq, device=p.device)
    p.masked_fill_(torch.arange(n, device=p.device) > rows[:, None], float("-inf"))
    p -= p.amax(-1, keepdim=True)
    p.exp_()
    p /= p.sum(-1, keepdim=True)
    s["weights"][:, :, :n] += p.sum((2, 3))
    return s["weights"]


def _plain_decode(s):
    c = s["case"]
    b, hq, hkv, d, n = c["batch"], c["hq"], c["hkv"], c["d"], c["n"]
    k, v = _values(s["cache"], c, 1)
    q = s["q"].float().view(b, hkv, hq // hkv, d)
    p = (q @ k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    p = (p - p.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    s["weights"][:, :, :n] += p.sum(2)
    return {"out": (p @ v).to(torch.bfloat16).view(b, hq, d), "weights": s["weights"]}


def _plain_select(s):
    c = s["case"]
    L, w, n, cap = c["L"], c["w"], c["n"], c["cap"]
    x = s["weights"]
    order = torch.sort(x[:, :, :L - w], dim=-1, descending=True, stable=True).indices[:, :, :n - w]
    last = torch.arange(L - w, L, device=x.device).expand(x.shape[0], x.shape[1], w)
    kept = torch.cat([torch.sort(order, dim=-1).values, last], -1)
    out = x.new_zeros((x.shape[0], x.shape[1], cap))
    out[:, :, :n] = torch.gather(x, 2, kept)
    pos = torch.zeros(out.shape, dtype=torch.int32, device=x.device)
    pos[:, :, :n] = kept.to(torch.int32)
    return {"kept": kept.to(torch.int32), "weights": out, "pos": pos}


def _plain_evict(s):
    c = s["case"]
    n, bits, group, d = c["n"], c["bits"], c["group"], c["d"]
    w, pos, new = s["weights"], s["pos"], s["new_pos"]
    far = torch.iinfo(torch.int32).max
    slots = torch.arange(n, device=w.device)
    old = pos <= new - c["recent"]
    light = torch.where(old, w, torch.full_like(w, float("inf")))
    pick = old & (light == light.amin(-1, keepdim=True))
    oldest = pos == pos.amin(-1, keepdim=True)                               # where every token is recent
    pick = torch.where(old.any(-1, keepdim=True), pick, oldest)
    slot = torch.where(pick, slots, torch.full_like(slots, far)).amin(-1, keepdim=True)
    a = s["cache"]
    row = slot[..., None]
    if bits == 16:
        a["kc"].scatter_(2, row.expand(-1, -1, 1, d), s["k_new"][:, :, None])
        a["vc"].scatter_(2, row.expand(-1, -1, 1, d), s["v_new"][:, :, None])
        arrays = [a["kc"], a["vc"]]
    else:
        for_k = _quantize(s["k_new"].float().view(*s["k_new"].shape[:2], 1, d // group, group), bits)
        for_v = _quantize(s["v_new"].float().view(*s["v_new"].shape[:2], 1, d // group, group), bits)
        wk, wv = _pack(for_k[0], bits), _pack(for_v[0], bits)
        a["kc"].scatter_(2, row[..., None].expand_as(wk), wk)
        a["vc"].scatter_(2, row[..., None].expand_as(wv), wv)
        a["ks"].scatter_(2, row.expand_as(for_k[1]), for_k[1])
        a["kz"].scatter_(2, row.expand_as(for_k[2]), for_k[2])
        a["vs"].scatter_(2, row.expand_as(for_v[1]), for_v[1])
        a["vz"].scatter_(2, row.expand_as(for_v[2]), for_v[2])
        arrays = [a["kc"], a["vc"], a["ks"], a["kz"], a["vs"], a["vz"]]
    w.scatter_(2, slot, 0.0)
    pos.scatter_(2, slot, new)
    return {"slots": slot[..., 0].to(torch.int32), "weights": w, "pos": pos, "cache": arrays}


def _plain_tree(s):
    c = s["case"]
    b, hq, hkv, d, n, T = c["batch"], c["hq"], c["hkv"], c["d"], c["n"], c["T"]
    G, m = hq // hkv, c["tail"]
    k, v = _values(s["cache"], c, c["axis"])
    k = torch.cat([k, s["kt"][:, :, :m].float(), s["kd"].float().transpose(1, 2)], 2)
    v = torch.cat([v, s["vt"][:, :, :m].float(), s["vd"].float().transpose(1, 2)], 2)
    q = s["q"].float().view(b, T, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, G * T, d)
    p = ((q @ k.transpose(2, 3)) * (1.0 / math.sqrt(d))).view(b, hkv, G, T, n + m + T)
    hidden = ((s["mask"][..., None] >> torch.arange(T, device=p.device)) & 1) == 0
    p[..., n + m:].masked_fill_(hidden[:, None, None], float("-inf"))
    p = (p - p.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    o = (p.view(b, hkv, G * T, -1) @ v).view(b, hkv, G, T, d)
    return o.permute(0, 3, 1, 2, 4).reshape(b, T, hq, d).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ the framework's calls

def _handle(s):
    """The cache object (and strategy, tail, workspace) that a user's program keeps beside its arrays."""
    if "handle" not in s:
        from paper_2412_12706_b200 import qp
        c, a = s["case"], s["cache"]
        desc = qp.cache_layout_cap(c["batch"], c["hq"], c["hkv"], c["d"], c["bits"], c["group"], c["n"], c.get("cap", c["n"]))
        names = (("k_codes", "kc"), ("v_codes", "vc"), ("k_scale", "ks"), ("k_zero", "kz"), ("v_scale", "vs"), ("v_zero", "vz"))
        for name, key in names:
            setattr(desc, name, None if a[key] is None else a[key].data_ptr())
        cache = qp.Cache(desc, *[a[key] for _, key in names])
        per_token = c["bits"] < 16 and c.get("axis", 1) == 1
        strategy = qp.make_strategy(cache, 1) if per_token else None
        tail = workspace = None
        if c["op"] == "tree":
            tail = qp.alloc_tail(cache)
            if tail.k_tail is not None:
                tail.k_tail.copy_(s["kt"])
                tail.v_tail.copy_(s["vt"])
                tail.desc.n_tail = c["tail"]
            workspace = qp.new_decode_workspace(qp.decode_tree_workspace_bytes(cache, c["T"]), DEV)
        elif c["op"] == "decode":
            workspace = qp.new_decode_workspace(qp.decode_weights_workspace_bytes(cache), DEV)
        s["handle"] = cache, strategy, tail, workspace
    return s["handle"]


def _own(s):
    from paper_2412_12706_b200 import qp
    c = s["case"]
    op = c["op"]
    if op == "prompt":
        if "handle" not in s:
            s["handle"] = qp.new_decode_workspace(
                qp.prompt_weights_workspace_bytes(c["batch"], c["hq"], c["hkv"], c["d"], c["L"], c["q_start"], c["nq"]), DEV)
        return qp.prompt_weights(s["q"], s["k"], c["q_start"], weights=s["weights"], workspace=s["handle"])
    if op == "select":
        kept, w, pos = qp.heavy_select(s["weights"], c["w"], c["n"], c["cap"])
        return {"kept": kept, "weights": w, "pos": pos}
    cache, strategy, tail, workspace = _handle(s)
    if op == "decode":
        out = qp.decode_attn_weights(s["q"], cache, s["weights"], strategy=strategy, workspace=workspace)
        return {"out": out, "weights": s["weights"]}
    if op == "evict":
        slots = qp.evict_kv(s["k_new"], s["v_new"], cache, s["weights"], s["pos"], s["new_pos"], c["recent"], strategy=strategy)
        arrays = [t for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.k_zero, cache.v_scale, cache.v_zero) if t is not None]
        return {"slots": slots, "weights": s["weights"], "pos": s["pos"], "cache": arrays}
    return qp.decode_attn_tree(s["q"], cache, s["kd"], s["vd"], s["mask"], tail=tail, strategy=strategy, workspace=workspace)


def run(state):
    if own:
        return _own(state)
    return {"prompt": _plain_prompt, "decode": _plain_decode, "select": _plain_select, "evict": _plain_evict,
            "tree": _plain_tree}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ work and exact values

def work(case):
    op = case["op"]
    if op == "select":
        heads = case["batch"] * case["hkv"]
        return dict(bytes=heads * (4 * case["L"] + 4 * case["n"] + 8 * case["cap"]), flops=0)
    b, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    if op == "prompt":
        nq, q0 = case["nq"], case["q_start"]
        pairs = nq * q0 + nq * (nq + 1) // 2
        return dict(bytes=2 * d * b * (hq * nq + hkv * (q0 + nq)) + 8 * b * hkv * (q0 + nq), flops=2 * d * b * hq * pairs)
    n, bits = case["n"], case["bits"]
    row = 4 * d if bits == 16 else 2 * (d * bits // 8 + 4 * d // case["group"])   # bytes of one token's key and value
    if op == "decode":
        return dict(bytes=b * (hkv * n * (row + 8) + 4 * hq * d), flops=4 * b * hq * n * d)
    if op == "evict":
        return dict(bytes=b * hkv * (8 * n + 4 * d + row + 12), flops=0)
    T, m = case["T"], case["tail"]
    return dict(bytes=b * (hkv * n * row + 4 * hkv * (m + T) * d + 4 * T * hq * d + 8 * T), flops=4 * b * hq * T * d * (n + m + T))


def _wide(cache, case, axis):
    """What the stored codes stand for, in 64 bits, read group by group from the words."""
    n, bits, d, group = case["n"], case["bits"], case["d"], case["group"]
    if bits == 16:
        return cache["kc"].double()[:, :, :n], cache["vc"].double()[:, :, :n]
    per = 32 // bits
    e = torch.arange(group, device=DEV)

    def side(words, scale, zero):
        code = (words.long()[..., e // per] >> ((e % per) * bits)) % (1 << bits)
        return torch.addcmul(zero.double()[..., None], code.double(), scale.double()[..., None])

    k, v = side(cache["kc"], cache["ks"], cache["kz"]), side(cache["vc"], cache["vs"], cache["vz"])
    b, h = v.shape[:2]
    k = torch.einsum("bhudg->bhugd", k).reshape(b, h, n, d) if axis == 0 else k.reshape(b, h, n, d)
    return k, v.reshape(b, h, n, d)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "select":
        r = _plain_select(s)                                                 # nothing is computed: values are moved
        return {"kept": None, "weights": r["weights"].double(), "pos": None}
    if op == "evict":
        w = s["weights"].double()
        r = _plain_evict(s)
        w.scatter_(2, r["slots"].long()[..., None], 0.0)
        return {"slots": None, "weights": w, "pos": None, "cache": [None] * len(r["cache"])}
    b, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    G = hq // hkv
    if op == "prompt":
        nq, q0 = case["nq"], case["q_start"]
        n = q0 + nq
        if b * hq * nq * n > 4e9:
            return None
        keys, got = s["k"].double(), s["weights"].double()
        col = torch.arange(n, device=DEV)
        for h in range(hq):                                                  # one query head at a time, in blocks of rows
            for lo in range(0, nq, 2048):
                rows = torch.arange(lo, min(nq, lo + 2048), device=DEV)
                x = torch.einsum("bid,bjd->bij", s["q"][:, h, rows].double(), keys[:, h // G, :n]) * d ** -0.5
                x = torch.where(col <= (q0 + rows)[:, None], x, torch.full((), -math.inf, dtype=torch.float64, device=DEV))
                got[:, h // G, :n] += torch.softmax(x, -1).sum(1)
        return got
    k, v = _wide(s["cache"], case, case.get("axis", 1))
    if op == "decode":
        x = torch.einsum("bhgd,bhnd->bhgn", s["q"].double().reshape(b, hkv, G, d), k) * d ** -0.5
        p = torch.softmax(x, -1)
        w = s["weights"].double()
        w[:, :, :case["n"]] += p.sum(2)
        return {"out": torch.einsum("bhgn,bhnd->bhgd", p, v).reshape(b, hq, d), "weights": w}
    T, m, n = case["T"], case["tail"], case["n"]
    qd = s["q"].double().reshape(b, T, hkv, G, d)
    x = [torch.einsum("bthgd,bhnd->bthgn", qd, k), torch.einsum("bthgd,bhnd->bthgn", qd, s["kt"][:, :, :m].double()),
         torch.einsum("bthgd,bjhd->bthgj", qd, s["kd"].double())]
    sees = torch.stack([(s["mask"] >> j) % 2 == 1 for j in range(T)], -1)
    x[2] = x[2].masked_fill(~sees[:, :, None, None], -math.inf)
    p = torch.softmax(torch.cat(x, -1) * d ** -0.5, -1)
    o = torch.einsum("bthgn,bhnd->bthgd", p[..., :n], v) + torch.einsum("bthgn,bhnd->bthgd", p[..., n:n + m], s["vt"][:, :, :m].double())
    o = o + torch.einsum("bthgj,bjhd->bthgd", p[..., n + m:], s["vd"].double())
    return o.reshape(b, T, hq, d)
