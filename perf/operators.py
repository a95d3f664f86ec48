"""Timed cases of the rotating and 8-bit cache operators: rotation with the
append, the append into an 8-bit cache, and attention over that cache.

Each case runs through the package's public calls when ``own`` is true, and
through elementary torch operations in 32 bits when it is not.

A case is a dict of plain values:

  kind      "rope" (rotate q and k, append k and v to the bf16 cache), "kv8"
            (the same into the 8-bit cache) or "attn" (attention over the
            8-bit cache)
  hq, hkv, dqk, dv, page    attention geometry; dqk 576 is the latent layout
            (values are part of the key rows: one row a token is appended)
  decodes, dec_lo, dec_hi   decode sequences (one new token) and the range of
            their context lengths
  prompts, new_lo, new_hi, pre_lo, pre_hi   prompts, their new tokens and the
            tokens already cached before them
  lens      seed of the length draw (lengths belong to the case, so that its
            work is fixed; values and page order come from prepare's seed)
  rot_begin, rot_dim, neighbours, axes, dealt   (rope, kv8) the rotated part
            of a head, whether its pairs are neighbours or half a part apart,
            the axes of a position and whether pairs are dealt to them in turn;
            rot_dim 0: no rotation (kv8 alone)
  call      (attn) "decode", "prefill", "serial" or "corun"
  cus_decode   co-run: compute units of the decode share
  lse       whether the log-sum-exp is asked for beside the output

An 8-bit cache holds e4m3 codes [pages, page, hkv, d] and one power-of-two
scale (e8m0) for each 16 tokens, KV head and K / V: [pages, page / 16, hkv, 2].
"""
from __future__ import annotations

import math
import random

import torch

own = False

QWEN = dict(hq=28, hkv=4, dqk=128, dv=128, page=16)
D64 = dict(hq=32, hkv=8, dqk=64, dv=64, page=64)
LATENT = dict(hq=128, hkv=1, dqk=576, dv=512, page=64)
MAX_POSITION = 1 << 15


def _case(kind, geo, name=None, decodes=0, dec=(0, 0), prompts=0, new=(0, 0), pre=(0, 0), lens=1, **more):
    c = dict(kind=kind, decodes=decodes, dec_lo=dec[0], dec_hi=dec[1], prompts=prompts, new_lo=new[0], new_hi=new[1],
             pre_lo=pre[0], pre_hi=pre[1], lens=lens, **geo)
    if kind == "attn":
        c.update(call="decode", cus_decode=0, lse=False)
    else:
        c.update(rot_begin=0, rot_dim=geo["dqk"], neighbours=False, axes=1, dealt=False)
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The new tokens of a decode step, 64 sequences: latency.
        _case("rope", QWEN, "rope-64", 64, (512, 4096)),
        # The new tokens of the benchmark's mixed step: a 2048-token chunk beside 128 decodes.
        _case("rope", QWEN, "rope-mixed", 128, (16, 600), 1, (2048, 2048), (4096, 4096)),
        # Prompts with images: three axes of position, odd lengths, 8 KV heads of 64 in large pages.
        _case("rope", D64, "rope-axes", 5, (100, 900), 6, (500, 1500), (0, 700), axes=3),
        # A 4096-token prompt of the latent layout: the last 64 of 576 columns turn, by neighbouring pairs.
        _case("rope", LATENT, "rope-latent", prompts=1, new=(4096, 4096), rot_begin=512, rot_dim=64, neighbours=True),
        # The decode step's new tokens into the 8-bit cache: blocks that hold rows already.
        _case("kv8", QWEN, "kv8-append-64", 64, (512, 4096)),
        # The mixed step's new tokens into the 8-bit cache.
        _case("kv8", QWEN, "kv8-append-mixed", 128, (16, 600), 1, (2048, 2048), (4096, 4096)),
        # One user's decode step: a single sequence, launch latency and split depth.
        _case("attn", QWEN, "kv8-decode-one", 1, (2000, 2000), lse=True),
        # The decode batch of the package's benchmark.
        _case("attn", QWEN, "kv8-decode-64", 64, (512, 4096)),
        # A large decode batch of a model with 64-wide heads and large pages.
        _case("attn", D64, "kv8-decode-d64", 128, (1000, 8000), lse=True),
        # A few short prompts arriving together, ragged.
        _case("attn", QWEN, "kv8-prefill-short", prompts=5, new=(50, 300), pre=(0, 500), call="prefill", lse=True),
        # The prefill batch of the benchmark.
        _case("attn", QWEN, "kv8-prefill-8x2048", prompts=8, new=(2048, 2048), call="prefill"),
        # The benchmark's mixed step: a 2048-token chunk beside 128 decodes, co-run.
        _case("attn", QWEN, "kv8-mixed-corun", 128, (1024, 8192), 1, (2048, 2048), (4096, 4096), call="corun", cus_decode=96),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(["rope", "kv8", "attn", "attn", "attn"])
    d, page = rng.choice([64, 128]), rng.choice([16, 64])
    hq, hkv = rng.choice([(28, 4), (28, 4), (32, 8), (4, 1), (32, 2), (8, 8), (40, 8), (15, 5)])
    geo = dict(hq=hq, hkv=hkv, dqk=d, dv=d, page=page)
    hi = _log(rng, 1, 16384)
    nhi = _log(rng, 2, 4096)
    phi = rng.choice([0, _log(rng, 1, 8192)])
    c = dict(dec=(max(1, hi // rng.choice([1, 4, 16])), hi), new=(max(2, nhi // rng.choice([1, 3, 8])), nhi),
             pre=(phi // 2, phi), lens=rng.randrange(1, 1 << 20))
    decodes, prompts = _log(rng, 1, 256), _log(rng, 1, 16)
    if kind == "attn":
        call = rng.choice(["decode", "decode", "prefill", "prefill", "serial", "corun"])
        return _case("attn", geo, decodes=0 if call == "prefill" else decodes,
                     prompts=0 if call == "decode" else prompts if call == "prefill" else 1 + prompts // 4,
                     call=call, cus_decode=rng.choice([64, 96, 128]) if call == "corun" else 0, lse=rng.random() < 0.5, **c)
    c["dec"] = (max(1, c["dec"][0] // 8), max(1, c["dec"][1] // 8))
    mix = rng.choice([(decodes, 0), (0, prompts), (decodes, 1 + prompts // 4)])
    axes = rng.choice([1, 1, 2, 3, 4])
    rot = dict(axes=axes, dealt=axes > 1 and rng.random() < 0.5, neighbours=rng.random() < 0.3)
    if kind == "rope" and rng.random() < 0.3:
        geo = dict(LATENT, page=page, hq=rng.choice([64, 128]))
        rot.update(rot_begin=512, rot_dim=64)
    elif rng.random() < 0.3:
        rot.update(rot_dim=geo["dqk"] // 2)
    elif kind == "kv8" and rng.random() < 0.2:
        rot.update(rot_dim=0, axes=1, dealt=False, neighbours=False)
    return _case(kind, geo, decodes=mix[0], prompts=mix[1], **c, **rot)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most and _padded(c) <= 2.5e9:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 250)


def _padded(case):
    """Values that the plain form of attention spreads a batch over, at the most."""
    ns, ls = _lengths(case)
    p = case["prompts"]
    pre = p * max(ns[:p], default=0) * max(ls[:p], default=0) * case["hq"]
    return max(pre, len(ls[p:]) * max(ls[p:], default=0) * case["hkv"] * case["dqk"]) if case["kind"] == "attn" else 0


def _lengths(case):
    """(new tokens, context) of every sequence, decodes after prompts."""
    r = random.Random(case["lens"])
    ns, ls = [], []
    for _ in range(case["prompts"]):
        n = r.randint(case["new_lo"], case["new_hi"])
        ns.append(n)
        ls.append(n + r.randint(case["pre_lo"], case["pre_hi"]))
    for _ in range(case["decodes"]):
        ns.append(1)
        ls.append(r.randint(case["dec_lo"], case["dec_hi"]))
    return ns, ls


def _sections(case):
    """Pairs of each axis: near-equal, the first axes take what is left over."""
    pairs, a = case["rot_dim"] // 2, case["axes"]
    return [pairs // a + (1 if i < pairs % a else 0) for i in range(a)]


def work(case):
    hq, hkv, dqk, dv = case["hq"], case["hkv"], case["dqk"], case["dv"]
    ns, ls = _lengths(case)
    if case["kind"] == "attn":
        b = f = 0
        for n, L in zip(ns, ls):
            b += L * hkv * (dqk + dv) + -(-L // 16) * hkv * 2 + n * hq * (2 * (dqk + dv) + (4 if case["lse"] else 0)) + 4 * -(-L // case["page"])
            f += hq * 2 * (dqk + dv) * (n * (L - n) + n * (n + 1) // 2)
        return {"bytes": b, "flops": f}
    t = sum(ns)
    kv = hkv * (dqk if dqk == 576 else dqk + dv)
    b = t * 4 * case["axes"] + (t * 4 if case["kind"] == "rope" else 4 * (2 * len(ns) + 1))
    if case["rot_dim"]:   # q read and written, a row of the table for a position's share of the pairs
        b += t * hq * dqk * 4 + 4 * min(t, MAX_POSITION) * case["rot_dim"]
    if case["kind"] == "rope":
        return {"bytes": b + t * kv * 4, "flops": 0}
    blocks = sum(-(-L // 16) - (L - n) // 16 for n, L in zip(ns, ls))
    return {"bytes": b + t * kv * 3 + blocks * hkv * 2, "flops": 0}


# ------------------------------------------------------------------ inputs ---

def _generators(seed):
    return torch.Generator(device="cuda").manual_seed(seed), torch.Generator().manual_seed(seed)


def _pages(case, ns, ls, hg):
    """Block table over a pool in random order with one spare page, and the metadata (on the host)."""
    P = case["page"]
    pages = [-(-L // P) for L in ls]
    used = sum(pages)
    perm = torch.randperm(used + 1, generator=hg).to(torch.int32)
    bt = torch.full((len(ls), max(pages)), int(perm[used]), dtype=torch.int32)   # entries past a sequence: the spare page
    at = 0
    for s, n in enumerate(pages):
        bt[s, :n] = perm[at:at + n]
        at += n
    qsl = torch.zeros(len(ls) + 1, dtype=torch.int32)
    qsl[1:] = torch.cumsum(torch.tensor(ns), 0)
    return used + 1, bt, torch.tensor(ls, dtype=torch.int32), qsl


def _cache8(case, pages, g):
    """An 8-bit cache as the append leaves one: codes that fill the type's
    range, scales that differ from block to block by up to 8 times."""
    def codes(d):
        x = torch.empty((pages, case["page"], case["hkv"], d), dtype=torch.float8_e4m3fn, device="cuda")
        for part in x.split(1 << 10):   # (a part at a time: the pool is large)
            part.copy_((torch.randn(part.shape, generator=g, device="cuda") * 112).clamp_(-448, 448))
        return x

    k, v = codes(case["dqk"]), codes(case["dv"])
    e = torch.randint(-8, -5, (pages, case["page"] // 16, case["hkv"], 2), generator=g, device="cuda")
    return k, v, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _table(case):
    """cos and sin of every position's angles, worked out in 64 bits."""
    i = torch.arange(case["rot_dim"] // 2, dtype=torch.float64, device="cuda")
    angle = torch.arange(MAX_POSITION, dtype=torch.float64, device="cuda")[:, None] * (1e6 ** (-2 * i / case["rot_dim"]))[None, :]
    return torch.cat([torch.cos(angle), torch.sin(angle)], 1).float()


def _positions(case, ns, ls):
    """[axes, tokens]: one axis counts the tokens; with more, the first counts
    frames of 32 x 32 patches and the others the patch within a frame."""
    t = torch.cat([torch.arange(L - n, L) for n, L in zip(ns, ls)])
    if case["axes"] == 1:
        return t[None].to(torch.int32)
    i = torch.cat([torch.arange(n) for n in ns])
    start = torch.cat([torch.full((n,), L - n) for n, L in zip(ns, ls)])
    axes = [start + i // 1024, start + i % 1024 // 32, start + i % 32, t]
    return torch.stack(axes[:case["axes"]]).to(torch.int32)


def _inputs(case, seed):
    g, hg = _generators(seed)
    ns, ls = _lengths(case)
    hq, hkv, dqk, dv, T = case["hq"], case["hkv"], case["dqk"], case["dv"], sum(ns)
    pages, bt, sl, qsl = _pages(case, ns, ls, hg)
    x = dict(bt=bt.cuda(), sl=sl.cuda(), qsl=qsl.cuda(), h=(bt, sl, qsl))
    if case["kind"] == "attn":
        x["q"] = torch.randn((T, hq, dqk), generator=g, device="cuda", dtype=torch.bfloat16) * 2
        x["k"], x["v"], x["scales"] = _cache8(case, pages, g)
        return x
    # q, k and v of a token lie in one row, as one projection writes them
    latent = dqk == 576
    widths = [hq * dqk, hkv * dqk] + ([] if latent else [hkv * dv])
    row = torch.randn((T, sum(widths)), generator=g, device="cuda")
    row *= torch.exp(0.7 * torch.randn((T, 1), generator=g, device="cuda"))   # some tokens are larger than others
    q, k, *v = row.to(torch.bfloat16).split(widths, 1)
    x.update(q=q.unflatten(1, (hq, dqk)), k_new=k.unflatten(1, (hkv, dqk)), v_new=None if latent else v[0].unflatten(1, (hkv, dv)))
    if case["rot_dim"]:
        x.update(table=_table(case), pos=_positions(case, ns, ls).cuda())
    if case["kind"] == "kv8":
        x["k"], x["v"], x["scales"] = _cache8(case, pages, g)
        return x
    at = torch.cat([torch.arange(L - n, L) for n, L in zip(ns, ls)])
    seq = torch.repeat_interleave(torch.arange(len(ns)), torch.tensor(ns))
    x["slots"] = (bt[seq, at // case["page"]] * case["page"] + at % case["page"]).to(torch.int32).cuda()
    x["k"] = torch.randn((pages, case["page"], hkv, dqk), generator=g, device="cuda", dtype=torch.bfloat16)
    x["v"] = None if latent else torch.randn((pages, case["page"], hkv, dv), generator=g, device="cuda", dtype=torch.bfloat16)
    return x


def _scale(case):
    return 1.0 / math.sqrt(192.0 if case["dqk"] == 576 else case["dqk"])


_stream = None   # the program's own stream: co-run steps are issued from it
_pair = {}       # the one co-run pair a program keeps, by its split (a state asks for it at each pass:
                 # a state of another split may have replaced it)


def _corun(F, cus_prefill, cus_decode):
    key = (cus_prefill, cus_decode)
    if key not in _pair:
        for old in _pair.values():
            old.close()
        _pair.clear()
        _pair[key] = F.Corun(cus_prefill, cus_decode)
    return _pair[key]


def prepare(case, seed):
    x = _inputs(case, seed)
    state = dict(case=case, x=x)
    if case["kind"] != "attn":   # the attention calls take q with nothing between its rows
        state["q_out"] = torch.empty(x["q"].shape, dtype=torch.bfloat16, device="cuda")
    return _prepare_own(state) if own else state


def _prepare_own(state):
    """What a user's program keeps: the plan, the arguments, the co-run pair."""
    global _stream
    from paper_2606_04415_amd import flexattn as F
    case, x = state["case"], state["x"]
    shape = F.make_shape(case["hq"], case["hkv"], case["dqk"], case["dv"], case["page"], _scale(case), case["dqk"] == 576)
    state.update(F=F, shape=shape)
    if case["kind"] == "attn":
        if _stream is None:
            _stream = torch.cuda.Stream()
        bt, sl, qsl = x["h"]
        pa = F.PagedAttention(shape, F.make_opts(cus_decode=case["cus_decode"], kv_bits=8), qsl, sl, bt.shape[1])
        out, lse = pa.alloc_out(x["q"], with_lse=case["lse"])
        split = pa.plan.info["cus_prefill"], pa.plan.info["cus_decode"]
        if case["call"] == "corun":
            _corun(F, *split)
        args = pa.kv8_args(x["q"], x["k"], x["v"], x["scales"], x["bt"], x["sl"], x["qsl"], out, lse)
        state.update(pa=pa, args=args, split=split, out=out, lse=lse)
        return state
    rope = None
    if case["rot_dim"]:
        rope = F.make_rope(x["table"], x["pos"], rot_begin=case["rot_begin"], neighbours=case["neighbours"],
                           sections=_sections(case) if case["axes"] > 1 else None, dealt=case["dealt"])
    if case["kind"] == "rope":
        args = F.make_rope_append_args(x["q"], state["q_out"], x["k_new"], x["v_new"], x["slots"], x["k"], x["v"])
    else:
        q = (x["q"], state["q_out"]) if rope else (None, None)
        args = F.make_kv8_append_args(x["k_new"], x["v_new"], x["bt"], x["sl"], x["qsl"], x["k"], x["v"], x["scales"], *q)
    state.update(rope=rope, args=args)
    return state


# ------------------------------------------------------------- plain forms ---

def _turn(x, case, table, pos):
    """Rows [tokens, heads, d] with the rotated part turned, in 32 bits."""
    x = x.float()
    if not case["rot_dim"]:
        return x
    half, b = case["rot_dim"] // 2, case["rot_begin"]
    i = torch.arange(half, device=x.device)
    if case["axes"] == 1:
        axis = torch.zeros_like(i)
    elif case["dealt"]:
        axis = i % case["axes"]
        axis = torch.where(i < case["axes"] * torch.tensor(_sections(case), device=x.device)[axis], axis, 0)
    else:
        axis = (i[:, None] >= torch.cumsum(torch.tensor(_sections(case), device=x.device), 0)).sum(1)
    row = pos.long()[axis].T                      # [tokens, pairs]: the position each pair goes by
    c, s = (table[row, i + o][:, None, :] for o in (0, half))
    part = x[..., b:b + case["rot_dim"]]
    u, w = (part[..., 0::2], part[..., 1::2]) if case["neighbours"] else (part[..., :half], part[..., half:])
    u, w = u * c - w * s, w * c + u * s
    turned = torch.stack([u, w], -1).flatten(-2) if case["neighbours"] else torch.cat([u, w], -1)
    return torch.cat([x[..., :b], turned, x[..., b + case["rot_dim"]:]], -1)


def _power(e):
    """2^e of whole numbers, exactly; 0 below the smallest normal number."""
    return torch.where(e < -126, 0, (e.clamp(-126, 127) + 127) << 23).to(torch.int32).view(torch.float32)


def _append8(x, case, kv, new):
    """New rows [tokens, hkv, d] (32 bits) into the codes and scales of K (kv 0) or V (1)."""
    P, hkv = case["page"], case["hkv"]
    pool = x["kv"[kv]].view(torch.uint8).view(-1, 16, hkv, new.shape[-1])         # blocks of 16 rows
    scales = x["scales"].view(torch.uint8).view(-1, hkv, 2)[:, :, kv]
    t = torch.arange(new.shape[0], device=new.device)
    seq = torch.searchsorted(x["qsl"][1:].long(), t, right=True)
    at = x["sl"].long()[seq] - x["qsl"].long()[seq + 1] + t
    block = x["bt"].long()[seq, at // P] * (P // 16) + at % P // 16
    row = at % 16
    first = torch.full((pool.shape[0],), 16, device=new.device).scatter_reduce_(0, block, row, "amin")
    largest = torch.where(new.isfinite(), new.abs(), 0).amax(-1)
    a = torch.zeros((pool.shape[0], hkv), device=new.device).scatter_reduce_(0, block[:, None].expand(-1, hkv), largest, "amax")
    m, e = torch.frexp(a)                          # a <= 448 * 2^k; 448 = 0.875 * 2^9
    e = torch.where(a == 0, -117, torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-117))
    at = (first < 16).nonzero()[:, 0]              # the blocks that get rows
    old, e, head = scales[at].to(torch.int32) - 127, e[at], first[at]
    e = torch.where(head[:, None] > 0, torch.maximum(e, old), e)
    held = pool[at].view(torch.float8_e4m3fn).float() * _power(old - e)[:, None, :, None]
    keep = (torch.arange(16, device=new.device)[None] < head[:, None])[:, :, None, None]
    pool[at] = torch.where(keep, held.to(torch.float8_e4m3fn).view(torch.uint8), pool[at])
    scales[at] = (e + 127).to(torch.uint8)
    whole = torch.zeros((pool.shape[0], hkv), dtype=torch.int32, device=new.device)
    whole[at] = e
    codes = (new * _power(-whole[block])[..., None]).to(torch.float8_e4m3fn)   # at most 448 by the choice of e
    pool[block, row] = codes.view(torch.uint8)


def _attend(case, x, seqs, q):
    """Attention of sequences `seqs` (a slice) with queries [sequences, n, hq, d], zeros behind short ones: out, lse."""
    P, hkv, G = case["page"], case["hkv"], case["hq"] // case["hkv"]
    ns, ls = (v[seqs] for v in _lengths(case))
    n, L = max(ns), max(ls)
    page = x["bt"].long()[seqs, :-(-L // P)]
    e = x["scales"].view(torch.uint8)[page].int() - 127

    def rows(cache, kv):
        z = cache.view(torch.uint8)[page].view(torch.float8_e4m3fn).float()
        z = z.unflatten(2, (P // 16, 16)) * _power(e[..., kv])[:, :, :, None, :, None]
        return z.flatten(1, 3)[:, :L].transpose(1, 2).contiguous()                # [sequences, hkv, L, d]

    k, v = rows(x["k"], 0), rows(x["v"], 1)
    z = q.float().unflatten(2, (hkv, G)).permute(0, 2, 3, 1, 4).flatten(2, 3)      # [sequences, hkv, G * n, d]
    z = torch.matmul(z.contiguous(), k.transpose(2, 3).contiguous()) * _scale(case)
    sl, qsl = x["sl"].long(), x["qsl"].long()
    old = (sl - qsl[1:] + qsl[:-1])[seqs]                                           # tokens before the new ones
    seen = old[:, None] + 1 + torch.arange(n, device=z.device)                      # [sequences, n]
    hidden = torch.arange(L, device=z.device) >= seen.repeat(1, G)[:, :, None]      # [sequences, G * n, L]
    z.masked_fill_(hidden[:, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    z = z.sub_(m).exp_()
    l = z.sum(-1, keepdim=True)
    o = torch.matmul(z, v) / l

    def back(y):
        return y.unflatten(2, (G, n)).permute(0, 3, 1, 2, 4).flatten(2, 3)          # [sequences, n, hq, ...]

    return back(o), back(m + l.log())[..., 0]


def _plain_attention(state):
    case, x = state["case"], state["x"]
    ns, _ = _lengths(case)
    p = case["prompts"]
    outs, lses = [], []
    t = sum(ns[:p])
    if p:
        n = max(ns[:p])
        new = torch.arange(n, device="cuda")[None] < (x["qsl"][1:p + 1] - x["qsl"][:p])[:, None]
        q = torch.zeros((p, n) + x["q"].shape[1:], dtype=x["q"].dtype, device="cuda")
        q[new] = x["q"][:t]
        o, e = _attend(case, x, slice(0, p), q)
        outs.append(o[new])
        lses.append(e[new])
    if case["decodes"]:
        o, e = _attend(case, x, slice(p, None), x["q"][t:][:, None])
        outs.append(o[:, 0])
        lses.append(e[:, 0])
    out = torch.cat(outs).to(torch.bfloat16)
    return {"out": out, "lse": torch.cat(lses)} if case["lse"] else out


def _plain(state):
    case, x = state["case"], state["x"]
    if case["kind"] == "attn":
        return _plain_attention(state)
    table, pos = x.get("table"), x.get("pos")
    k = _turn(x["k_new"], case, table, pos)
    if case["rot_dim"]:
        state["q_out"].copy_(_turn(x["q"], case, table, pos))
    if case["kind"] == "rope":
        at = x["slots"].long()
        x["k"].view(-1, *x["k"].shape[2:])[at] = k.to(torch.bfloat16)
        if x["v"] is not None:
            x["v"].view(-1, *x["v"].shape[2:])[at] = x["v_new"]
        return _outputs(state)
    _append8(x, case, 0, k)
    _append8(x, case, 1, x["v_new"].float())
    return _outputs(state)


def _outputs(state):
    x, y = state["x"], {}
    if state["case"]["rot_dim"]:
        y["q"] = state["q_out"]
    y.update({n: x[n] for n in ("k", "v", "scales") if x.get(n) is not None})
    return y


def run(state):
    if not own:
        return _plain(state)
    F, case = state["F"], state["case"]
    if case["kind"] == "rope":
        F.flex_attn_rope_append(state["shape"], state["rope"], state["args"])
        return _outputs(state)
    if case["kind"] == "kv8":
        F.flex_attn_kv8_append(state["shape"], state["rope"], state["args"])
        return _outputs(state)
    plan, args = state["pa"].plan, state["args"]
    if case["call"] == "decode":
        F.flex_attn_decode_kv8(plan, args)
    elif case["call"] == "prefill":
        F.flex_attn_prefill_kv8(plan, args)
    elif case["call"] == "corun":   # behind what the caller's stream holds, and before what follows there
        caller = torch.cuda.current_stream()
        _stream.wait_stream(caller)
        with torch.cuda.stream(_stream):
            F.flex_attn_mixed_kv8(plan, args, F.FLEX_MODE_CORUN, corun=_corun(F, *state["split"]))
        caller.wait_stream(_stream)
    else:
        F.flex_attn_mixed_kv8(plan, args, F.FLEX_MODE_SERIAL)
    return {"out": state["out"], "lse": state["lse"]} if case["lse"] else state["out"]


# ----------------------------------------------------------------- 64 bits ---

def _exact_turn(rows, case, x):
    """The rotation as a product of complex numbers."""
    rows = rows.double()
    if not case["rot_dim"]:
        return rows
    half, b, A = case["rot_dim"] // 2, case["rot_begin"], case["axes"]
    sec = _sections(case)
    owner = [0] * half
    if case["dealt"]:
        for a in range(1, A):
            for j in range(sec[a]):
                owner[a + A * j] = a
    else:
        owner = [a for a in range(A) for _ in range(sec[a])]
    turn = torch.empty((rows.shape[0], half), dtype=torch.complex128, device="cuda")
    for i, a in enumerate(owner):
        p = x["pos"][a].long()
        turn[:, i] = torch.complex(x["table"][p, i].double(), x["table"][p, half + i].double())
    first = torch.arange(half, device="cuda") * (2 if case["neighbours"] else 1) + b
    second = first + (1 if case["neighbours"] else half)
    z = torch.complex(rows[..., first], rows[..., second]) * turn[:, None]
    rows = rows.clone()
    rows[..., first], rows[..., second] = z.real, z.imag
    return rows


def _exact_code(y):
    """Nearest e4m3 value: steps of 2^-9 below 2^-6, else an eighth of the power of two below."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _exact8(case, x, kv, rows):
    P, hkv = case["page"], case["hkv"]
    codes = x["kv"[kv]].double()
    scale = x["scales"][..., kv].double()
    ns, ls = _lengths(case)
    bt, at = x["h"][0], 0
    for s, (n, L) in enumerate(zip(ns, ls)):
        for b in range((L - n) // 16, -(-L // 16)):
            lo, hi = max(L - n, 16 * b), min(L, 16 * b + 16)
            new = rows[at + lo - (L - n):at + hi - (L - n)]
            page, part = int(bt[s, 16 * b // P]), 16 * b % P
            big = new.abs().amax((0, 2))
            e = torch.ceil(torch.log2(big.clamp(min=1e-300) / 448)).clamp(min=-117)
            e = torch.where(big > 448 * torch.exp2(e), e + 1, e)
            f = torch.exp2(e)
            if lo > 16 * b:
                was = scale[page, part // 16]
                f = torch.maximum(f, was)
                held = codes[page, part:part + lo - 16 * b]
                codes[page, part:part + lo - 16 * b] = _exact_code(held * (was / f)[None, :, None])
            codes[page, part + lo - 16 * b:part + hi - 16 * b] = _exact_code(new / f[None, :, None])
            scale[page, part // 16] = f
        at += n
    return codes, scale


def exact(case, seed):
    x = _inputs(case, seed)
    ns, ls = _lengths(case)
    if case["kind"] != "attn":
        k = _exact_turn(x["k_new"], case, x)
        y = {"q": _exact_turn(x["q"], case, x)} if case["rot_dim"] else {}
        if case["kind"] == "rope":
            at = x["slots"].long()
            y["k"] = x["k"].double()
            y["k"].view(-1, *x["k"].shape[2:])[at] = k
            if x["v"] is not None:
                y["v"] = x["v"].double()
                y["v"].view(-1, *x["v"].shape[2:])[at] = x["v_new"].double()
            return y
        y["k"], ks = _exact8(case, x, 0, k)
        y["v"], vs = _exact8(case, x, 1, x["v_new"].double())
        y["scales"] = torch.stack([ks, vs], -1)
        return y
    hq, hkv, dv, P = case["hq"], case["hkv"], case["dv"], case["page"]
    G, T = hq // hkv, sum(ns)
    out = torch.empty((T, hq, dv), dtype=torch.float64, device="cuda")
    lse = torch.empty((T, hq), dtype=torch.float64, device="cuda")
    at = 0
    for s, (n, L) in enumerate(zip(ns, ls)):
        pages = x["h"][0][s, :-(-L // P)].long().cuda()
        scale = x["scales"].view(torch.uint8)[pages].view(torch.float8_e8m0fnu).double().reshape(-1, hkv, 2).repeat_interleave(16, 0)[:L]
        k, v = ((c.view(torch.uint8)[pages].view(torch.float8_e4m3fn).double().reshape(-1, hkv, c.shape[-1])[:L] * scale[..., i:i + 1])
                .transpose(0, 1).contiguous() for i, c in enumerate((x["k"], x["v"])))
        kt = k.transpose(1, 2).contiguous()
        step = max(1, (1 << 27) // (hq * L))          # rows of queries at a time
        for r0 in range(0, n, step):
            r1 = min(n, r0 + step)
            q = x["q"][at + r0:at + r1].double().reshape(r1 - r0, hkv, G, -1).transpose(0, 1).reshape(hkv, (r1 - r0) * G, -1)
            z = torch.matmul(q.contiguous(), kt) * _scale(case)
            seen = L - n + torch.arange(r0, r1, device="cuda").repeat_interleave(G) + 1
            z.masked_fill_(torch.arange(L, device="cuda")[None, :] >= seen[:, None], -math.inf)
            e = torch.logsumexp(z, -1, keepdim=True)
            o = torch.matmul(torch.exp(z - e), v)
            out[at + r0:at + r1] = o.reshape(hkv, r1 - r0, G, dv).transpose(0, 1).reshape(r1 - r0, hq, dv)
            lse[at + r0:at + r1] = e.reshape(hkv, r1 - r0, G).transpose(0, 1).reshape(r1 - r0, hq)
        at += n
    return {"out": out, "lse": lse} if case["lse"] else out
