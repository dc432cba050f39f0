"""Operators around the prefill, as timed cases with their plain forms.

  rotate  norms of queries and keys for each head and the rotation by position,
          in one pass over the projections (what the prefill's Q and K are made by)
  append  new tokens' queries rotated, their keys rotated and stored in a paged
          cache beside their values, then read back
  read    a cached sequence's keys and values read back from its pages
  attend  attention of the newest tokens over the paged cache

The cache holds the problem's own type, or 4 bits: E2M1 values with one
power-of-two scale for 32 of them.  Pages: [page][KV head][slot][d] values, or
[page][KV head][slot][d / 2] bytes (the even value low) beside
[page][KV head][d / 32][slot] exponents plus 127.
"""
from __future__ import annotations

import math

import torch

own = False   # True: run() makes the framework's calls

DEV = "cuda"


def _case(name, kind, b, hq, hkv, d, lo, hi, new=0, dtype="bf16", cache="same", page=64, rot=0,
          interleaved=False, norm=False, fused=False):
    """b sequences of lo to hi tokens; the newest `new` of each are the call's
    (0: all of them); rot values of a head are rotated."""
    return {"name": name, "kind": kind, "b": b, "hq": hq, "hkv": hkv, "d": d, "lo": lo, "hi": hi,
            "new": new, "dtype": dtype, "cache": cache, "page": page, "rot": rot,
            "interleaved": interleaved, "norm": norm, "fused": fused}


def listed():
    return [
        # the last tokens of a prompt through a small fp32 layer: latency
        _case("rotate_fp32_7", "rotate", 1, 8, 2, 64, 7, 7, dtype="fp32", rot=32,
              interleaved=True),
        # a short prompt of odd length, Q and K as slices of one projection,
        # half of every head rotated
        _case("rotate_4k_fused", "rotate", 1, 32, 8, 128, 4173, 4173, rot=64, norm=True,
              fused=True),
        # the benchmark's layer: 128K tokens
        _case("rotate_128k", "rotate", 1, 32, 8, 128, 131072, 131072, rot=128, norm=True),
        # one token of each of 48 sequences into a 4-bit cache
        _case("append_fp4_b48", "append", 48, 32, 8, 128, 1, 8000, new=1, cache="fp4", rot=128,
              norm=True, fused=True),
        # five prompts of 1K to 50K tokens into a 4-bit cache
        _case("append_fp4_prompts", "append", 5, 32, 8, 128, 1003, 50001, cache="fp4", rot=128),
        # a long cached prompt read back from 4 bits
        _case("read_fp4_128k", "read", 1, 32, 8, 128, 131072, 131072, cache="fp4", page=128),
        # sequences of 64-wide heads read back from bf16, small pages
        _case("read_b8", "read", 8, 16, 4, 64, 100, 12000, page=16),
        # one token of one short sequence, fp32: latency
        _case("attend_fp32_777", "attend", 1, 8, 2, 64, 777, 777, new=1, dtype="fp32"),
        # a decode batch over a bf16 cache, lengths 50 to 64K
        _case("attend_b16", "attend", 16, 32, 8, 128, 50, 65536, new=1),
        # one token after the benchmark's 128K prompt, 4 bits
        _case("attend_fp4_128k", "attend", 1, 32, 8, 128, 131072, 131072, new=1, cache="fp4"),
        # a large decode batch of the Qwen-shaped layer, 4 bits, lengths 1 to 32K
        _case("attend_fp4_b64", "attend", 64, 28, 4, 128, 1, 32768, new=1, cache="fp4", page=128),
        # nine drafted tokens of each of four sequences checked at once
        _case("attend_tokens", "attend", 4, 32, 8, 128, 1500, 24001, new=9),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "append", "read", "attend", "attend", "attend",
                       "attend"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    hq, hkv = rng.choice([(32, 8), (28, 4), (16, 4), (8, 2), (8, 8), (32, 4)])
    d = rng.choice([64, 128, 128])
    rot = rng.choice([d, d, d // 2, 16, 48])
    base = dict(dtype=dtype, interleaved=rng.random() < 0.3, norm=rng.random() < 0.5,
                page=rng.choice([16, 32, 64, 64, 128]),
                cache=rng.choice(["same", "fp4", "fp4"]))
    if kind == "rotate":
        n = _log_int(rng, 1, 20000 if dtype == "fp32" else 60000)
        base["cache"] = "same"
        c = _case("", kind, 1, hq, hkv, d, n, n, rot=rot, fused=rng.random() < 0.5, **base)
    else:
        total = 30000 if dtype == "fp32" else 120000
        b = _log_int(rng, 1, 64)
        hi = _log_int(rng, 20, total // b)
        lo = max(1, min(hi, _log_int(rng, 1, hi)))
        new = 0 if kind in ("append", "read") else rng.choice([1, 1, 1, 2, 5, 16])
        if kind == "append" and rng.random() < 0.5:
            new = rng.choice([1, 1, 3])
        c = _case("", kind, b, hq, hkv, d, lo, hi, new=min(new, lo) if new else 0,
                  rot=rot if kind == "append" else 0, fused=rng.random() < 0.3, **base)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# sizes of a case
# ---------------------------------------------------------------------------
def _lengths(case):
    """Lengths of the sequences: log-spaced from lo to hi, in mixed order."""
    b, lo, hi = case["b"], case["lo"], case["hi"]
    at = [int(round(lo * (hi / lo) ** (i / max(1, b - 1)))) for i in range(b)] if b > 1 else [hi]
    return [at[(i * 5 + 2) % b] if b % 5 else at[(i * 7 + 2) % b] if b % 7 else at[i]
            for i in range(b)]


def _new(case):
    """New tokens of each sequence."""
    return [case["new"] if case["new"] else n for n in _lengths(case)]


def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantise(x):
    """fp32 values [..., d] as 4-bit codes [..., d / 2] and exponents [..., d / 32]."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    m, e = torch.frexp(g.abs().amax(-1))
    # the smallest power of two with no value over 7 of it
    e = torch.where(m <= 0.875, e - 3, e - 2).clamp(-110, 125)
    e = torch.where(m == 0, -110, e)
    a = torch.ldexp(g, -e[..., None]).abs()
    # nearest of the eight magnitudes, ties to the even code
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5)
            + (a > 5))
    code = (code + 8 * torch.signbit(g)).reshape(*x.shape[:-1], -1, 2)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, exps):
    """What codes [..., d / 2] with exponents [..., d / 32] stand for, in fp32."""
    grid = torch.tensor(_GRID + tuple(-x for x in _GRID), device=codes.device)
    nib = torch.stack((codes & 15, codes >> 4), dim=-1).reshape(*codes.shape[:-1], -1, 32)
    return torch.ldexp(grid[nib.long()], (exps.int() - 127)[..., None]).flatten(-2)


def _pages(case, num_pages, gen):
    """Pools as earlier tokens left them."""
    hkv, d, ps, dt = case["hkv"], case["d"], case["page"], _torch_dtype(case)
    loud = 1 + 3 * (torch.rand((hkv, 1, d), generator=gen, device=DEV) < 0.03)
    out = {}
    for x in ("k", "v"):
        step = max(1, (1 << 26) // (hkv * ps * d))
        codes, exps = [], []
        for p0 in range(0, num_pages, step):
            z = torch.randn((min(step, num_pages - p0), hkv, ps, d), generator=gen, device=DEV)
            z = (z * loud if x == "k" else z).to(dt)
            if case["cache"] == "same":
                codes.append(z)
            else:
                c, e = _quantise(z.float())
                codes.append(c)
                exps.append(e.transpose(-1, -2).contiguous())
        out[x] = torch.cat(codes)
        out[x + "_scales"] = torch.cat(exps) if exps else None
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 104729 + 11)
    hq, hkv, d, rot, dt = case["hq"], case["hkv"], case["d"], case["rot"], _torch_dtype(case)
    lens, new = _lengths(case), _new(case)
    tokens = sum(new)
    st = {"case": case, "tokens": tokens}

    def rnd(*shape):
        return torch.randn(shape, generator=gen, device=DEV)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)

    # the projections of the new tokens; fused: slices of one buffer
    if case["kind"] != "read":
        if case["fused"]:
            x = rnd(tokens, hq + 2 * hkv, d).to(dt)
            st["q"], st["k"], st["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        else:
            st["q"], st["k"], st["v"] = (rnd(tokens, h, d).to(dt) for h in (hq, hkv, hkv))
    if rot:
        inv = 500000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
        ang = torch.arange(max(lens), device=DEV, dtype=torch.float64)[:, None] * inv
        st["cos"], st["sin"] = ang.cos().float(), ang.sin().float()
    st["q_weight"] = st["k_weight"] = None
    if case["norm"]:
        st["q_weight"] = (1 + 0.2 * rnd(d)).to(dt)
        st["k_weight"] = (1 + 0.2 * rnd(d)).to(dt)
    st["q_out"] = torch.empty((tokens, hq, d), dtype=dt, device=DEV)
    st["k_out"] = torch.empty((tokens, hkv, d), dtype=dt, device=DEV)
    st["v_out"] = torch.empty((tokens, hkv, d), dtype=dt, device=DEV)
    if case["kind"] == "rotate":
        return st
    # the pages: each sequence's in any order, a few that nobody has
    ps = case["page"]
    per = [-(-n // ps) for n in lens]
    width, num_pages = max(per), sum(per) + 3
    order = torch.randperm(num_pages, generator=gen, device=DEV).int()
    table = torch.zeros((len(lens), width), dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(per):
        table[i, :n] = order[at:at + n]
        at += n
    st["page_table"], st["seq_lens"] = table, ints(lens)
    st["starts"] = ints([sum(new[:i]) for i in range(len(new) + 1)])
    st["new_start"] = None if all(n == 1 for n in new) else st["starts"]
    st["pools"] = _pages(case, num_pages, gen)
    st["max_len"], st["max_new"], st["num_pages"] = max(lens), max(new), num_pages
    st["out"] = torch.empty((tokens, hq, d), dtype=dt, device=DEV)
    st["lse"] = torch.empty((hq, tokens), dtype=torch.float32, device=DEV)
    return st


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _handles(st):
    """The descriptors and the workspace that a user's program keeps: made on
    the state's first pass."""
    from paper_2509_24745_amd import proxyattn as pa
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    rotary = None
    strides = {}
    if case["fused"] and case["kind"] != "read":
        tok = (hq + 2 * hkv) * d
        strides = dict(q_tok_stride=tok, kv_tok_stride=tok)
    if case["rot"] or case["norm"]:
        rotary = pa.Rotary(rotary_dim=case["rot"], interleaved=case["interleaved"], eps=1e-6,
                           cos=st.get("cos"), sin=st.get("sin"), q_weight=st["q_weight"],
                           k_weight=st["k_weight"])
    if case["kind"] == "rotate":
        prob = pa.Problem(seq_len=st["tokens"], num_q_heads=hq, num_kv_heads=hkv, head_dim=d,
                          block_size=128, num_proxy_groups=1, dtype=case["dtype"], **strides)
        return pa, prob, rotary
    sizes = dict(num_seqs=case["b"], num_tokens=st["tokens"], max_new=st["max_new"],
                 max_len=st["max_len"], num_q_heads=hq, num_kv_heads=hkv, head_dim=d,
                 page_size=case["page"], num_pages=st["num_pages"],
                 table_width=st["page_table"].shape[1], dtype=case["dtype"],
                 cache_type=case["cache"])
    cache = pa.Cache(**sizes, **strides)
    packed = pa.Cache(**sizes)   # the arrays that the cache is read back into
    p = st["pools"]
    pages = pa.Pages(p["k"], p["v"], p["k_scales"], p["v_scales"])
    ws = torch.empty(max(16, pa.proxyattn_cache_workspace_size(cache)), dtype=torch.uint8,
                     device=DEV)
    return pa, cache, packed, pages, rotary, ws


def _run_own(st):
    kind = st["case"]["kind"]
    if "handles" not in st:
        st["handles"] = _handles(st)
    if kind == "rotate":
        pa, prob, rotary = st["handles"]
        pa.proxyattn_norm_rotate(prob, rotary, st["q"], st["k"], None, 0, st["q_out"],
                                 st["k_out"])
        return {"q": st["q_out"], "k": st["k_out"]}
    pa, cache, packed, pages, rotary, ws = st["handles"]
    where = (st["page_table"], st["seq_lens"], st["new_start"])
    if kind == "attend":
        pa.proxyattn_cache_attention(cache, st["q"], *where, pages, st["out"], st["lse"], ws)
        return {"out": st["out"], "lse": st["lse"]}
    got = {}
    if kind == "append":
        pa.proxyattn_cache_append(cache, rotary, st["q"], st["k"], st["v"], st["q_out"], *where,
                                  pages)
        got["q"] = st["q_out"]
    pa.proxyattn_cache_read(packed, *where, pages, st["k_out"], st["v_out"])
    return {**got, "k": st["k_out"], "v": st["v_out"]}


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _rotated(case, st, x, weight, pos, ft):
    """x [T][heads][d] normed (with a weight) and rotated, computed in ft."""
    x = x.to(ft)
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.to(ft)
    rot = case["rot"]
    if not rot:
        return x
    c, s = (st[n][pos].to(ft)[:, None, :] for n in ("cos", "sin"))
    y = x[..., :rot]
    if case["interleaved"]:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        y = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
    return torch.cat((y, x[..., rot:]), dim=-1)


def _places(st):
    """Sequence and position of every new token."""
    t = torch.arange(st["tokens"], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(st["starts"], t, right=True) - 1
    behind = st["starts"][seq + 1] - t
    return seq, (st["seq_lens"][seq] - behind).long()


def _slots(st, seq, pos):
    """(page, slot) of positions of sequences."""
    ps = st["case"]["page"]
    return st["page_table"][seq, pos // ps].long(), pos % ps


def _store(st, name, page, slot, x):
    pool = st["pools"][name]
    if st["case"]["cache"] == "same":
        pool[page, :, slot] = x
        return
    codes, exps = _quantise(x.float())
    pool[page, :, slot] = codes
    st["pools"][name + "_scales"][page, :, :, slot] = exps


def _load(st, name, page, slot):
    """Values [..., Hkv, d] of slots, in fp32."""
    x = st["pools"][name][page, :, slot]
    if st["case"]["cache"] == "same":
        return x.float()
    return _values(x, st["pools"][name + "_scales"][page, :, :, slot])


def _run_attend(st):
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    b, n, m = case["b"], st["max_len"], st["max_new"]
    u = torch.arange(n, device=DEV)
    page, slot = _slots(st, torch.arange(b, device=DEV)[:, None], u[None, :].expand(b, n))
    # K and V of every sequence, [b][hkv][n][d]; past a sequence's end any slot, masked
    k = _load(st, "k", page, slot).transpose(1, 2).contiguous()
    v = _load(st, "v", page, slot).transpose(1, 2).contiguous()
    # the new tokens of a sequence in rows of their own, [b][hkv][m * rep][d]
    j = torch.arange(m, device=DEV)
    count = st["starts"][1:] - st["starts"][:-1]
    row = (st["starts"][:-1, None] + torch.minimum(j, count[:, None] - 1)).long()
    q = st["q"].float()[row].reshape(b, m, hkv, hq // hkv, d).transpose(1, 2)
    q = q.reshape(b, hkv, -1, d).contiguous()
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    pos = st["seq_lens"][:, None] - count[:, None] + j
    seen = (u[None, None, :] <= pos[:, :, None]) & (u < st["seq_lens"][:, None])[:, None]
    seen = seen[:, None, :, None].expand(b, 1, m, hq // hkv, n).reshape(b, 1, -1, n)
    x = torch.where(seen, x, float("-inf"))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / total
    lse = top + torch.log(total)
    seq, at = _places(st)
    j = (at - (st["seq_lens"] - count)[seq]).long()
    o = o.reshape(b, hkv, m, hq // hkv, d).transpose(1, 2).reshape(b, m, hq, d)
    lse = lse.reshape(b, hkv, m, hq // hkv).transpose(1, 2).reshape(b, m, hq)
    return {"out": o[seq, j].to(_torch_dtype(case)), "lse": lse[seq, j].t().contiguous()}


def run(st):
    if own:
        return _run_own(st)
    case, dt = st["case"], _torch_dtype(st["case"])
    kind = case["kind"]
    if kind == "attend":
        return _run_attend(st)
    if kind == "rotate":
        pos = torch.arange(st["tokens"], device=DEV)
        return {"q": _rotated(case, st, st["q"], st["q_weight"], pos, torch.float32).to(dt),
                "k": _rotated(case, st, st["k"], st["k_weight"], pos, torch.float32).to(dt)}
    seq, pos = _places(st)
    page, slot = _slots(st, seq, pos)
    got = {}
    if kind == "append":
        got["q"] = _rotated(case, st, st["q"], st["q_weight"], pos, torch.float32).to(dt)
        # keys in 64 bits: many lie next to a border between two 4-bit values
        k = _rotated(case, st, st["k"], st["k_weight"], pos, torch.float64).float().to(dt)
        _store(st, "k", page, slot, k)
        _store(st, "v", page, slot, st["v"])
    return {**got, "k": _load(st, "k", page, slot).to(dt), "v": _load(st, "v", page, slot).to(dt)}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    hq, hkv, d, rot = case["hq"], case["hkv"], case["d"], case["rot"]
    e = 2 if case["dtype"] == "bf16" else 4
    lens, new = _lengths(case), _new(case)
    t = sum(new)
    row = 2 * hkv * (d * e if case["cache"] == "same" else d // 2 + d // 32)   # a cached token
    kv = 2 * hkv * d * e
    table = 4 * rot * max(lens)
    if case["kind"] == "rotate":
        return {"bytes": 2 * t * (hq + hkv) * d * e + table, "flops": 8 * t * (hq + hkv) * d}
    if case["kind"] == "append":   # stored, then read back
        return {"bytes": 2 * t * hq * d * e + t * kv + t * row + t * row + t * kv
                + min(table, 4 * rot * t), "flops": 8 * t * (hq + 2 * hkv) * d}
    if case["kind"] == "read":
        return {"bytes": t * (row + kv), "flops": 2 * t * hkv * d}
    keys = sum(m * n - m * (m - 1) // 2 for n, m in zip(lens, new))
    return {"bytes": sum(lens) * row + 2 * t * hq * d * e + 4 * t * hq,
            "flops": 4 * d * hq * keys}


# ---------------------------------------------------------------------------
# the same in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------
def _exact_rotate(case, st, x, weight, first):
    """Rows of one sequence from position `first`, head dim as complex pairs."""
    z = x.double()
    if weight is not None:
        z = z / torch.sqrt((z ** 2).sum(-1, keepdim=True) / case["d"] + 1e-6) * weight.double()
    r = case["rot"]
    if not r:
        return z
    z = z.clone()
    turn = torch.complex(st["cos"].double(), st["sin"].double())[first:first + z.shape[0], None]
    j = torch.arange(r // 2, device=DEV)
    ia, ib = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + r // 2)
    w = torch.complex(z[..., ia], z[..., ib]) * turn
    z[..., ia], z[..., ib] = w.real, w.imag
    return z


def _exact_store(case, z):
    """What the cache gives back for values z: the type's, or the nearest of the
    15 multiples of each group's power of two."""
    z = z.to(torch.float32).to(_torch_dtype(case)).double()
    if case["cache"] == "same":
        return z
    g = z.reshape(*z.shape[:-1], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 7).clamp(min=-200))
    e = torch.where(7 * 2.0 ** (e - 1) >= top, e - 1, e)
    e = torch.where(7 * 2.0 ** e < top, e + 1, e).clamp(-110, 125)
    a = (g.abs() / 2.0 ** e).clamp(max=6.0)
    # spacing of the values near a: 1/2 below 2, 1 below 4, 2 above
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    return (torch.copysign(torch.round(a / step) * step, g) * 2.0 ** e).flatten(-2)


def _exact_cached(st, name, i, n):
    """Values [n][Hkv][d] that sequence i's pages hold, in 64 bits."""
    case = st["case"]
    pages = st["page_table"][i, :-(-n // case["page"])].long()
    x = st["pools"][name][pages].transpose(1, 2).flatten(0, 1)[:n]
    if case["cache"] == "same":
        return x.double()
    e = st["pools"][name + "_scales"][pages].permute(0, 3, 1, 2).flatten(0, 1)[:n]
    nib = torch.stack((x % 16, x // 16), dim=-1).flatten(-2).double()
    sign, c = 1 - 2 * (nib >= 8).double(), nib % 8
    mag = torch.where(c < 4, c / 2, torch.where(c < 6, c - 2, 2 * c - 8))
    return sign * mag * (2.0 ** (e.double() - 127)).repeat_interleave(32, dim=-1)


def exact(case, seed):
    st = prepare(case, seed)
    lens, new = _lengths(case), _new(case)
    kind = case["kind"]
    if kind == "rotate":
        return {x: _exact_rotate(case, st, st[x], st[x + "_weight"], 0) for x in ("q", "k")}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if kind == "read":
        parts = [[_exact_cached(st, x, i, n)[n - m:] for x in ("k", "v")]
                 for i, (n, m) in enumerate(zip(lens, new))]
        return {x: torch.cat([p[y] for p in parts]) for y, x in enumerate(("k", "v"))}
    at, parts = 0, []
    for i, (n, m) in enumerate(zip(lens, new)):
        q = st["q"][at:at + m]
        if kind == "append":
            k = _exact_rotate(case, st, st["k"][at:at + m], st["k_weight"], n - m)
            parts.append((_exact_rotate(case, st, q, st["q_weight"], n - m),
                          _exact_store(case, k), _exact_store(case, st["v"][at:at + m].double())))
        else:
            k, v = (_exact_cached(st, x, i, n) for x in ("k", "v"))
            o = torch.empty((m, hq, d), dtype=torch.float64, device=DEV)
            lse = torch.empty((m, hq), dtype=torch.float64, device=DEV)
            future = torch.arange(n, device=DEV)[None, :] > (torch.arange(m, device=DEV)
                                                             + n - m)[:, None]
            for h in range(hq):
                kh, vh = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
                x = q[:, h].double() @ kh.t() / math.sqrt(d)
                x.masked_fill_(future, float("-inf"))
                o[:, h] = torch.softmax(x, -1) @ vh
                lse[:, h] = torch.logsumexp(x, -1)
            parts.append((o, lse))
        at += m
    if kind == "append":
        return {x: torch.cat([p[y] for p in parts]) for y, x in enumerate(("q", "k", "v"))}
    return {"out": torch.cat([p[0] for p in parts]),
            "lse": torch.cat([p[1] for p in parts]).t().contiguous()}
