"""The operators around the prefill on the GPU (norm and rotation, appending to
a paged cache, reading it back, attention over it) against plain 64-bit forms
(oracle/cache_oracle.py).

Tolerances count roundings.  Rotated rows are computed in 64 bits and rounded
to fp32 and then to the type: half a step each, eps/2 relative.  Codes, scales
and what is read back are equal.  Attention, with p the probabilities, S the
largest sum |c q k| of a row and n its keys: a score is off by at most
(d + 4) 2^-23 S (d products and sums, the scale, the reference), which moves p
by as much, the exponential by 2^-22 more, sums of n terms by n 2^-24, bf16
probabilities in two terms by 2^-16, in one (more than 16 rows over 4 bits) by half
a step of bf16, 2^-8; so the output by
(2 ((d + 4) 2^-23 S + 2^-22) + 2 n 2^-24 [+ 2^-16 or 2^-8]) sum p |v|, and its own
rounding.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import cache_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pa():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2509_24745_amd import proxyattn
    return proxyattn


HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _np(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _rand(rng, shape, dtype, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(
        DT[dtype]).cuda()


def _ints(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")


def _tables(n, rot):
    if not rot:
        return None, None
    ang = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    return tuple(torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin))


def _rotary(pa, rng, d, rot, interleaved, norm, dtype, table, **kw):
    cos, sin = _tables(table, rot)
    wq, wk = ((_rand(rng, d, dtype, 0.3) + 1) if norm else None for _ in range(2))
    return pa.Rotary(rotary_dim=rot, interleaved=interleaved, eps=1e-5, cos=cos, sin=sin,
                     q_weight=wq, k_weight=wk, **kw)


def _turned(r, x, weight, positions):
    return O.norm_rotate(_np(x), np.asarray(positions), r.rotary_dim, r.interleaved,
                         None if r.cos is None else r.cos.cpu().numpy(),
                         None if r.sin is None else r.sin.cpu().numpy(),
                         None if weight is None else _np(weight), r.eps)


def _close_rows(got, ref, dtype):
    # 64-bit sums of the row's size, then the roundings to fp32 and the type
    tol = np.abs(ref) * (HALF[dtype] + 2.0 ** -23) + 1e-13 * np.abs(ref).max() + 1e-40
    bad = np.abs(_np(got) - ref) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3])


# ---------------------------------------------------------------------------
# norm and rotation of a prompt
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("n,hq,hkv,d,rot,interleaved,norm,dtype", [
    (1, 8, 2, 128, 128, False, True, "bf16"),
    (1, 1, 1, 64, 64, True, False, "fp32"),
    (7, 8, 2, 64, 32, True, True, "fp32"),
    (77, 28, 4, 128, 64, False, True, "bf16"),
    (33, 5, 5, 128, 48, True, False, "bf16"),
    (130, 6, 3, 64, 16, False, False, "bf16"),
    (19, 12, 4, 64, 0, False, True, "bf16"),
    (4100, 4, 1, 128, 128, False, False, "fp32"),   # several tokens to a workgroup
    (9001, 3, 1, 64, 64, False, True, "bf16"),
    (40000, 1, 1, 64, 48, True, True, "bf16"),
])
def test_norm_rotate(pa, n, hq, hkv, d, rot, interleaved, norm, dtype):
    rng = np.random.default_rng(n + d + rot)
    r = _rotary(pa, rng, d, rot, interleaved, norm, dtype, n + 5)
    # slices of one projection buffer
    x = _rand(rng, (n, hq + 2 * hkv, d), dtype, 3.0)
    q, k = x[:, :hq], x[:, hq:hq + hkv]
    tok = (hq + 2 * hkv) * d
    prob = pa.Problem(n, hq, hkv, d, 128, 1, dtype=dtype, q_tok_stride=tok, kv_tok_stride=tok)
    qo, ko = (torch.full((n, h, d), float("nan"), dtype=DT[dtype], device="cuda")
              for h in (hq, hkv))
    before = x.clone()
    pa.proxyattn_norm_rotate(prob, r, q, k, None, 5, qo, ko)
    at = np.arange(n) + 5
    refq, refk = _turned(r, q, r.q_weight, at), _turned(r, k, r.k_weight, at)
    _close_rows(qo, refq, dtype)
    _close_rows(ko, refk, dtype)
    assert torch.equal(x, before)
    # in place, both; positions given one by one, repeated and out of order
    pos = rng.integers(0, n + 5, n)
    pos[: n // 2] = pos[0]
    r2 = pa.Rotary(**{f: getattr(r, f) for f in ("rotary_dim", "interleaved", "eps", "cos", "sin",
                                                "q_weight", "k_weight")},
                   q_out_tok_stride=tok, k_out_tok_stride=tok)
    refq, refk = _turned(r, q, r.q_weight, pos), _turned(r, k, r.k_weight, pos)
    pa.proxyattn_norm_rotate(prob, r2, q, k, _ints(pos.tolist()), 0, q, k)
    _close_rows(q, refq, dtype)
    _close_rows(k, refk, dtype)
    assert torch.equal(x[:, hq + hkv:], before[:, hq + hkv:])


def test_norm_rotate_one_side_and_positions_out_of_the_table(pa):
    rng = np.random.default_rng(4)
    n, hq, d = 9, 4, 64
    r = _rotary(pa, rng, d, 64, False, True, "bf16", 12)
    prob = pa.Problem(n, hq, 2, d, 64, 1)
    q = _rand(rng, (n, hq, d), "bf16")
    qo = torch.empty_like(q)
    pos = [-5, 0, 11, 12, 2 ** 31 - 1, 3, -2 ** 31, 4, 5]
    pa.proxyattn_norm_rotate(prob, r, q, None, _ints(pos), 0, qo, None)
    _close_rows(qo, _turned(r, q, r.q_weight, np.clip(pos, 0, 11)), "bf16")
    # head-major queries
    qh = q.transpose(0, 1).contiguous()
    oh = torch.empty_like(qh)
    ph = pa.Problem(n, hq, 2, d, 64, 1, q_tok_stride=d, q_head_stride=n * d)
    rh = pa.Rotary(rotary_dim=64, eps=r.eps, cos=r.cos, sin=r.sin, q_weight=r.q_weight,
                   q_out_tok_stride=d, q_out_head_stride=n * d)
    pa.proxyattn_norm_rotate(ph, rh, qh, None, _ints(pos), 0, oh, None)
    assert torch.equal(oh.transpose(0, 1), qo)


def test_norm_of_extreme_rows(pa):
    """Rows of zeros (the norm divides by sqrt(eps)), of the largest and of the
    smallest values."""
    d = 128
    x = torch.zeros((4, 1, d), device="cuda")
    x[1], x[2], x[3] = 3e38, 1e-38, 1e-3
    x[1, 0, ::3] = 1.0
    r = pa.Rotary(eps=1e-6, q_weight=torch.ones(d, device="cuda"))
    out = torch.empty_like(x)
    pa.proxyattn_norm_rotate(pa.Problem(4, 1, 1, d, 64, 1, dtype="fp32"), r, x, None, None, 0, out,
                             None)
    _close_rows(out, _turned(r, x, r.q_weight, np.arange(4)), "fp32")


# ---------------------------------------------------------------------------
# the paged cache
# ---------------------------------------------------------------------------
class Batch:
    """A cache with a batch of sequences: their pages in mixed order, some that
    nobody has, every slot NaN or garbage at the start."""

    def __init__(self, pa, rng, lens, new, hq, hkv, d, page, dtype, cache_type, spare_rows=0,
                 null_start=False, spare_pages=3, extra_width=1, **kw):
        self.pa, self.lens, self.new, self.dtype = pa, list(lens), list(new), dtype
        per = [-(-n // page) for n in lens]
        pages = sum(per) + spare_pages
        width = max(per + [1]) + extra_width
        order = rng.permutation(pages)
        table = np.full((len(lens), width), -1, np.int64)
        at = 0
        for b, n in enumerate(per):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = table
        self.start = None if null_start else np.concatenate([[0], np.cumsum(new)]).tolist()
        rows = (len(lens) if null_start else self.start[-1]) + spare_rows
        self.cache = pa.Cache(num_seqs=len(lens), num_tokens=rows, max_new=max(list(new) + [1]),
                              max_len=max(list(lens) + [1]), num_q_heads=hq, num_kv_heads=hkv,
                              head_dim=d, page_size=page, num_pages=pages, table_width=width,
                              dtype=dtype, cache_type=cache_type, **kw)
        self.page_table, self.seq_lens = _ints(table.tolist()), _ints(self.lens)
        self.new_start = _ints(self.start)
        if len(lens) == 0:
            self.page_table = torch.zeros((1, width), dtype=torch.int32, device="cuda")
            self.seq_lens = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.pages = pa.Pages.empty(self.cache)
        for x in (self.pages.k, self.pages.v, self.pages.k_scales, self.pages.v_scales):
            if x is not None:
                x.fill_(float("nan") if x.is_floating_point() else 255)
        self.tokens = O.batch(self.lens, self.start, len(lens))

    @property
    def where(self):
        return self.page_table, self.seq_lens, self.new_start

    def fill(self, rng, loud=1.0):
        """Every token of every sequence, straight into the pages (no kernel):
        returns the keys and values that these then hold, in 64 bits."""
        c, out = self.cache, []
        for name in ("k", "v"):
            pool = getattr(self.pages, name).cpu()
            scales = getattr(self.pages, name + "_scales")
            scales = None if scales is None else scales.cpu()
            seqs = []
            for b, n in enumerate(self.lens):
                x = rng.standard_normal((n, c.num_kv_heads, c.head_dim))
                if name == "k":
                    x[..., :3] *= loud
                x = O.round_to(x, self.dtype)
                if c.cache_type == "fp4":
                    codes, sc = O.quantise(x)
                    x = O.dequantise(codes, sc)
                for j in range(-(-n // c.page_size)):
                    s = slice(j * c.page_size, min(n, (j + 1) * c.page_size))
                    m, p = s.stop - s.start, self.table[b, j]
                    if c.cache_type == "fp4":
                        pool[p, :, :m] = torch.from_numpy(codes[s]).transpose(0, 1)
                        scales[p, :, :, :m] = torch.from_numpy(sc[s]).permute(1, 2, 0)
                    else:
                        pool[p, :, :m] = torch.from_numpy(x[s]).transpose(0, 1).to(pool.dtype)
                seqs.append(x)
            getattr(self.pages, name).copy_(pool)
            if scales is not None:
                getattr(self.pages, name + "_scales").copy_(scales)
            out.append(seqs)
        return out

    def attend(self, q, **kw):
        c, pa = self.cache, self.pa
        t, hq, d = c.num_tokens, c.num_q_heads, c.head_dim
        out = torch.full((t, hq, d), 77.0, dtype=DT[self.dtype], device="cuda")
        lse = torch.full((hq, t), 77.0, device="cuda")
        ws = torch.full((max(16, pa.proxyattn_cache_workspace_size(c)),), 255, dtype=torch.uint8,
                        device="cuda")
        pa.proxyattn_cache_attention(c, q, *self.where, self.pages, out, lse, ws, **kw)
        return out, lse

    def check(self, q, out, lse, keys, values):
        c = self.cache
        scale = c.softmax_scale if c.softmax_scale > 0 else c.head_dim ** -0.5
        ref, rlse, absv, big = O.attention(_np(q), keys, values, self.tokens, scale)
        n = max(self.lens + [1])
        score = (c.head_dim + 4) * 2.0 ** -23 * big
        one_term = c.cache_type == "fp4" and c.num_q_heads // c.num_kv_heads * c.max_new > 16
        prob = 0 if self.dtype == "fp32" else 2.0 ** -8 if one_term else 2.0 ** -16
        a = 2 * (score + 2.0 ** -22) + 2 * n * 2.0 ** -24 + prob
        tol = np.abs(ref) * HALF[self.dtype] * 1.001 + a[..., None] * absv + 1e-30
        got, glse = _np(out), _np(lse)
        rows = [r for r, _, _ in self.tokens]
        rest = sorted(set(range(c.num_tokens)) - set(rows))
        assert (got[rest] == 77).all() and (glse[:, rest] == 77).all(), "rows of no sequence written"
        bad = ~(np.abs(got[rows] - ref[rows]) <= tol[rows])
        assert not bad.any(), (int(bad.sum()), float(np.nanmax(np.abs(got[rows] - ref[rows]))))
        empty = np.isneginf(rlse[:, rows])
        assert (np.isneginf(glse[:, rows]) == empty).all()
        ltol = score.T + n * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(np.where(np.isneginf(rlse), 0, rlse)))
        dl = np.abs(np.where(empty, 0, glse[:, rows]) - np.where(empty, 0, rlse[:, rows]))
        assert (dl <= ltol[:, rows]).all(), float((dl / ltol[:, rows]).max())


APPENDS = [
    # lens, new, hq, hkv, d, page, dtype, cache, rot, interleaved, norm
    ([1], [1], 4, 1, 64, 16, "bf16", "fp4", 64, False, True),
    ([40, 17, 16, 300], [40, 1, 0, 33], 8, 2, 128, 16, "bf16", "fp4", 128, False, True),
    ([40, 17, 16, 300], [40, 1, 0, 33], 8, 2, 128, 32, "bf16", "same", 128, True, False),
    ([100, 0, 65], [64, 0, 65], 28, 4, 64, 64, "fp32", "fp4", 48, True, True),
    ([100, 0, 65], [64, 0, 65], 3, 3, 64, 256, "fp32", "same", 16, False, False),
    ([9] * 70, [2] * 70, 4, 2, 128, 16, "bf16", "fp4", 96, False, True),
    ([3, 1] * 2000, [1, 1] * 2000, 2, 1, 64, 16, "bf16", "fp4", 64, False, False),
    ([5000], [4999], 2, 2, 128, 128, "bf16", "fp4", 128, False, False),
    ([9000], [9000], 1, 1, 64, 64, "bf16", "fp4", 0, False, True),
]


@pytest.mark.parametrize("lens,new,hq,hkv,d,page,dtype,cache,rot,interleaved,norm", APPENDS)
def test_append_and_read(pa, lens, new, hq, hkv, d, page, dtype, cache, rot, interleaved, norm):
    rng = np.random.default_rng(len(lens) + d + page)
    fused = (hq + 2 * hkv) * d
    w = Batch(pa, rng, lens, new, hq, hkv, d, page, dtype, cache, spare_rows=5,
              q_tok_stride=fused, kv_tok_stride=fused)
    c = w.cache
    t = c.num_tokens
    x = _rand(rng, (t, hq + 2 * hkv, d), dtype, 2.0)
    x[:, -1, 5] *= 100   # one loud value in the last head of v
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    r = _rotary(pa, rng, d, rot, interleaved, norm, dtype, max(lens))
    qo = torch.full((t, hq, d), 77.0, dtype=DT[dtype], device="cuda")
    old = [None if p is None else p.clone() for p in (w.pages.k, w.pages.v, w.pages.k_scales,
                                                      w.pages.v_scales)]
    pa.proxyattn_cache_append(c, r, q, k, v, qo, *w.where, w.pages)
    rows = [a for a, _, _ in w.tokens]
    pos = np.zeros(t, np.int64)
    pos[rows] = [p for _, _, p in w.tokens]
    _close_rows(qo[rows], _turned(r, q, r.q_weight, pos)[rows], dtype)
    assert (qo[len(rows):] == 77).all()
    # the pages: the tokens' slots hold the codes, every other slot what it held
    kr = O.round_to(_turned(r, k, r.k_weight, pos), dtype)
    want = [p if p is None else p.cpu() for p in old]
    vals = [kr, _np(v)]
    for i in range(2):
        codes, sc = O.quantise(vals[i]) if cache == "fp4" else (vals[i], None)
        for a, b, p in w.tokens:
            page_, slot = w.table[b, p // page], p % page
            want[i][page_, :, slot] = torch.from_numpy(codes[a]).to(want[i].dtype)
            if sc is not None:
                want[2 + i][page_, :, :, slot] = torch.from_numpy(sc[a])
        if sc is not None:
            vals[i] = O.dequantise(codes, sc)
    for got, ref, name in zip((w.pages.k, w.pages.v, w.pages.k_scales, w.pages.v_scales), want,
                              ("k", "v", "k_scales", "v_scales")):
        if ref is not None:
            same = got.cpu().view(torch.uint8) == ref.contiguous().view(torch.uint8)
            assert same.all(), (name, int((~same).sum()))
    # read back, into head-major arrays
    ko, vo = (torch.full((hkv, t, d), 77.0, dtype=DT[dtype], device="cuda") for _ in range(2))
    ch = pa.Cache(**{f: getattr(c, f) for f in c.__dataclass_fields__
                     if not f.endswith("stride")}, kv_tok_stride=d, kv_head_stride=t * d)
    pa.proxyattn_cache_read(ch, *w.where, w.pages, ko, vo)
    for got, ref in ((ko, vals[0]), (vo, vals[1])):
        got = _np(got).transpose(1, 0, 2)
        assert np.array_equal(got[rows], ref[rows])
        assert (got[len(rows):] == 77).all()


def test_quantisation_borders(pa):
    """Every tie, its neighbours, the clipped top, signs, zeros and the range of
    scales, through the cache and back."""
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    f = mid.astype(np.float32)
    near = np.concatenate([mid, np.nextafter(f, np.float32(9)), np.nextafter(f, np.float32(0)),
                           O.GRID, [6.5, 7.0, -0.0]])
    rows = []
    for e in (-125, -112, -111, -110, -109, -1, 0, 1, 60, 122, 123, 124, 125):
        for top in (7.0, 6.0, 4.0, 3.5, np.nextafter(np.float32(3.5), np.float32(9)), 1.0):
            x = np.concatenate([near, -near])[:60] * 2.0 ** e
            r = np.zeros(64)
            r[:30], r[32:62] = x[:30], x[30:60]
            r[31] = r[63] = top * 2.0 ** e
            r = np.clip(r, -top * 2.0 ** e, top * 2.0 ** e)
            rows.append(r)
    rows += [np.zeros(64), np.full(64, 3.4028234e38), -np.full(64, 3.4028234e38),
             np.full(64, 1e-45)]
    x = np.array(rows).astype(np.float32)
    x = np.clip(x, -3.4028234e38, 3.4028234e38)[:, None, :]
    n = x.shape[0]
    w = Batch(pa, np.random.default_rng(0), [n], [n], 1, 1, 64, 64, "fp32", "fp4")
    k = torch.from_numpy(x).cuda()
    pa.proxyattn_cache_append(w.cache, None, None, k, k, None, *w.where, w.pages)
    codes, sc = O.quantise(x)
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    pa.proxyattn_cache_read(w.cache, *w.where, w.pages, ko, vo)
    got = w.pages.k.cpu()[torch.from_numpy(w.table[0, :-(-n // 64)])].transpose(1, 2).flatten(0, 1)
    bad = np.argwhere(got[:n].numpy() != codes)
    assert not len(bad), (bad[:4], x[tuple(bad[0][:2])], got[tuple(bad[0])], codes[tuple(bad[0])])
    ref = O.dequantise(codes, sc)
    assert np.array_equal(_np(ko), ref) and np.array_equal(_np(vo), ref)


def test_bad_pages_and_lengths_stay_inside(pa):
    """Pages outside the pool take and give nothing; lengths past max_len count
    as max_len; tokens at negative positions are of no sequence; a new_start
    that goes past the rows or backwards reaches no other row."""
    rng = np.random.default_rng(2)
    for cache in ("same", "fp4"):
        w = Batch(pa, rng, [40, 20, 33], [40, 20, 33], 2, 2, 64, 16, "bf16", cache)
        c, t = w.cache, 93
        k, v = _rand(rng, (t, 2, 64), "bf16"), _rand(rng, (t, 2, 64), "bf16")
        pa.proxyattn_cache_append(c, None, None, k, v, None, *w.where, w.pages)
        keep = [p.clone() for p in (w.pages.k, w.pages.v)]
        table = w.page_table.clone()
        table[0, 0], table[1, 1], table[2, 2] = -1, c.num_pages, 2 ** 31 - 1
        ko, vo = (torch.full((t, 2, 64), 77.0, dtype=torch.bfloat16, device="cuda")
                  for _ in range(2))
        pa.proxyattn_cache_read(c, table, w.seq_lens, w.new_start, w.pages, ko, vo)
        lost = torch.zeros(t, dtype=torch.bool)
        lost[:16] = lost[40 + 16:60] = lost[60 + 32:] = True
        assert (ko.cpu()[lost] == 77).all() and (ko.cpu()[~lost] != 77).any(dim=(1, 2)).all()
        k2 = k + 1
        pa.proxyattn_cache_append(c, None, None, k2, v, None, table, w.seq_lens, w.new_start,
                                  w.pages)
        ko2 = torch.full_like(ko, 77.0)
        pa.proxyattn_cache_read(c, *w.where, w.pages, ko2, None)
        first = torch.full_like(ko, 77.0)
        pages2 = pa.Pages(keep[0], keep[1], w.pages.k_scales, w.pages.v_scales)
        if cache == "same":
            pa.proxyattn_cache_read(c, *w.where, pages2, first, None)
            assert torch.equal(ko2[lost.cuda()], first[lost.cuda()])
        q = _rand(rng, (t, 2, 64), "bf16")
        ws = torch.empty(pa.proxyattn_cache_workspace_size(c), dtype=torch.uint8, device="cuda")
        out, lse = torch.empty_like(q), torch.empty((2, t), device="cuda")
        pa.proxyattn_cache_attention(c, q, table, w.seq_lens, w.new_start, w.pages, out, lse, ws)
        big = _ints([2 ** 31 - 1, -5, 10])
        odd = _ints([-7, 200, 10, 95])
        for lens, start in ((big, w.new_start), (w.seq_lens, odd), (big, odd), (big, None)):
            out.fill_(77.0)
            pa.proxyattn_cache_append(c, None, None, k, v, None, w.page_table, lens, start, w.pages)
            pa.proxyattn_cache_read(c, w.page_table, lens, start, w.pages, ko, vo)
            pa.proxyattn_cache_attention(c, q, w.page_table, lens, start, w.pages, out, lse, ws)
        torch.cuda.synchronize()


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
ATTENDS = [
    # lens, new (None: one each, no new_start), hq, hkv, d, page, dtype, cache
    ([1], None, 1, 1, 64, 16, "bf16", "same"),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33], None, 4, 1, 128, 16, "bf16", "same"),
    ([0, 1, 63, 64, 65, 127, 128, 129, 255, 256, 257], None, 8, 2, 128, 64, "bf16", "fp4"),
    ([0, 1, 63, 64, 65, 127, 128, 129, 255, 256, 257], None, 8, 2, 64, 16, "bf16", "fp4"),
    ([0, 5, 64, 100, 131], None, 7, 1, 64, 32, "fp32", "same"),
    ([0, 5, 64, 100, 131, 513], None, 6, 2, 128, 32, "fp32", "same"),
    ([0, 5, 64, 100, 261], None, 16, 4, 128, 128, "fp32", "fp4"),
    ([7, 300, 64], None, 5, 5, 64, 256, "fp32", "fp4"),
    # several new tokens: one row tile, two, four, and more than one of four
    ([300, 40, 9], [4, 0, 3], 8, 2, 128, 64, "bf16", "same"),
    ([300, 40, 9], [7, 1, 8], 8, 2, 128, 64, "bf16", "fp4"),
    ([300, 33, 9], [16, 33, 5], 8, 2, 64, 16, "bf16", "fp4"),
    ([300, 33, 150], [16, 33, 50], 28, 4, 128, 32, "bf16", "same"),
    ([190], [190], 8, 8, 64, 16, "bf16", "same"),
    ([300, 33, 9], [16, 33, 5], 6, 2, 128, 16, "fp32", "same"),
    ([300, 33, 9], [16, 33, 5], 8, 1, 64, 16, "fp32", "fp4"),
    # fewer cached tokens than new ones: rows that see nothing
    ([3, 0, 20], [5, 4, 20], 4, 2, 128, 16, "bf16", "fp4"),
    ([3, 0, 20], [5, 4, 20], 4, 2, 64, 16, "fp32", "same"),
    # long ones among short ones, split over workgroups
    ([20000, 3, 700], None, 4, 1, 128, 64, "bf16", "fp4"),
    ([9000, 3, 700], [3, 2, 1], 4, 2, 64, 64, "bf16", "same"),
    ([6000, 1], None, 2, 1, 128, 32, "fp32", "same"),
    # several row tiles split over workgroups
    ([2100, 5, 900], [9, 1, 20], 8, 2, 128, 64, "bf16", "same"),
    ([1300, 64], [16, 3], 8, 2, 64, 32, "bf16", "same"),
    ([2600, 700], [5, 9], 8, 2, 128, 32, "bf16", "fp4"),
    ([2600, 700], [16, 1], 8, 2, 64, 16, "bf16", "fp4"),
    ([1500, 3, 700], [6, 1, 2], 8, 2, 128, 64, "fp32", "same"),
    ([1500, 3, 700], [6, 1, 2], 8, 2, 64, 16, "fp32", "same"),
    ([2100, 90], [7, 2], 8, 1, 64, 128, "fp32", "fp4"),
    ([2100, 90], [3, 2], 8, 2, 128, 16, "fp32", "fp4"),
]


@pytest.mark.parametrize("lens,new,hq,hkv,d,page,dtype,cache", ATTENDS)
def test_attention(pa, lens, new, hq, hkv, d, page, dtype, cache):
    rng = np.random.default_rng(sum(lens) + hq + d)
    tok = (hq + 1) * d
    w = Batch(pa, rng, lens, new or [1] * len(lens), hq, hkv, d, page, dtype, cache, spare_rows=3,
              null_start=new is None, q_tok_stride=tok)
    keys, values = w.fill(rng, loud=4.0)
    q = _rand(rng, (w.cache.num_tokens, hq + 1, d), dtype, 1.5)[:, :hq]
    out, lse = w.attend(q)
    w.check(q, out, lse, keys, values)
    again, lse2 = w.attend(q)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    ws = torch.empty(pa.proxyattn_cache_workspace_size(w.cache), dtype=torch.uint8, device="cuda")
    third = torch.full_like(out, 77.0)
    pa.proxyattn_cache_attention(w.cache, q, *w.where, w.pages, third, None, ws)
    assert torch.equal(third, out)


@pytest.mark.parametrize("cache", ["same", "fp4"])
def test_attention_of_many_sequences(pa, cache):
    """More sequences than threads look at one by one, some without tokens."""
    rng = np.random.default_rng(8)
    lens = rng.integers(0, 90, 700).tolist()
    new = [int(min(n, rng.integers(0, 3))) for n in lens]
    w = Batch(pa, rng, lens, new, 4, 2, 64, 16, "bf16", cache)
    keys, values = w.fill(rng)
    q = _rand(rng, (w.cache.num_tokens, 4, 64), "bf16")
    w.check(q, *w.attend(q), keys, values)


@pytest.mark.parametrize("b", [2, 63, 64, 65, 256, 257, 700])
def test_runs_dealt_over_any_number_of_sequences(pa, b):
    """A few long sequences among short and empty ones: the runs are cut, and every
    way of finding a workgroup's first one is taken."""
    rng = np.random.default_rng(b)
    lens = rng.integers(0, 40, b)
    lens[[b // 2, b - 1]] = 1500, 2100
    new = np.minimum(lens, rng.integers(0, 3, b))
    new[[b // 2, b - 1]] = 1, 2
    w = Batch(pa, rng, lens.tolist(), new.tolist(), 4, 2, 64, 32, "bf16", "same")
    assert pa.proxyattn_cache_workspace_size(w.cache) > 0
    keys, values = w.fill(rng)
    q = _rand(rng, (w.cache.num_tokens, 4, 64), "bf16")
    w.check(q, *w.attend(q), keys, values)


def test_most_sequences(pa):
    """4096 sequences, most with a token, two long ones: the runs are dealt over
    sequences that nobody keeps at hand."""
    rng = np.random.default_rng(10)
    lens = rng.integers(0, 4, 4096)
    lens[[17, 4000]] = 2500
    new = np.minimum(lens, 1)
    w = Batch(pa, rng, lens.tolist(), new.tolist(), 2, 1, 64, 16, "bf16", "fp4")
    keys, values = w.fill(rng)
    q = _rand(rng, (w.cache.num_tokens, 2, 64), "bf16")
    w.check(q, *w.attend(q), keys, values)


def test_two_calls_at_once(pa):
    """The same step of two batches on two streams, with a workspace each."""
    rng = np.random.default_rng(11)
    both = []
    for i in range(2):
        w = Batch(pa, rng, [3000, 40 + i, 900], [1, 1, 1], 8, 2, 128, 64, "bf16",
                  "same" if i else "fp4", null_start=True)
        keys, values = w.fill(rng)
        q = _rand(rng, (3, 8, 128), "bf16")
        both.append((w, keys, values, q, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for w, _, _, q, st in both:
            with torch.cuda.stream(st):
                got.append(w.attend(q))
    torch.cuda.synchronize()
    for i, (w, keys, values, q, _) in enumerate(both):
        w.check(q, *got[i], keys, values)
        for out, lse in got[i::2]:
            assert torch.equal(out, got[i][0]) and torch.equal(lse, got[i][1])


def test_append_queries_in_place(pa):
    """Queries rotated where they lie, keys alone rotated (no queries), one side of
    norm_rotate: all give what the separate arrays give."""
    rng = np.random.default_rng(12)
    hq, hkv, d, t = 6, 2, 64, 37
    tok = (hq + 2 * hkv) * d
    x = _rand(rng, (t, hq + 2 * hkv, d), "bf16")
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    w = Batch(pa, rng, [50], [t], hq, hkv, d, 16, "bf16", "same", q_tok_stride=tok,
              kv_tok_stride=tok)
    r = _rotary(pa, rng, d, 32, True, True, "bf16", 50)
    qo = torch.empty((t, hq, d), dtype=torch.bfloat16, device="cuda")
    pa.proxyattn_cache_append(w.cache, r, q, k, v, qo, *w.where, w.pages)
    first = (w.pages.k.clone(), w.pages.v.clone())
    ko = torch.empty((t, hkv, d), dtype=torch.bfloat16, device="cuda")
    prob = pa.Problem(t, hq, hkv, d, 64, 1, q_tok_stride=tok, kv_tok_stride=tok)
    pa.proxyattn_norm_rotate(prob, r, None, k, None, 13, None, ko)
    for p in (w.pages.k, w.pages.v):
        p.fill_(float("nan"))
    pa.proxyattn_cache_append(w.cache, r, None, k, v, None, *w.where, w.pages)
    same = [torch.equal(a.view(torch.int16), b.view(torch.int16))
            for a, b in zip(first, (w.pages.k, w.pages.v))]
    assert all(same)
    kr, vr = torch.empty_like(ko), torch.empty_like(ko)
    pa.proxyattn_cache_read(pa.Cache(**{f: getattr(w.cache, f) for f in
                                        w.cache.__dataclass_fields__ if "stride" not in f}),
                            *w.where, w.pages, kr, vr)
    assert torch.equal(kr, ko) and torch.equal(vr, v)
    fields = ("rotary_dim", "interleaved", "eps", "cos", "sin", "q_weight", "k_weight")
    here = pa.Rotary(**{f: getattr(r, f) for f in fields}, q_out_tok_stride=tok)
    pa.proxyattn_cache_append(w.cache, here, q, k, v, q, *w.where, w.pages)
    assert torch.equal(q, qo)


def test_attention_scale_and_output_strides(pa):
    rng = np.random.default_rng(9)
    hq, d, t = 6, 128, 2
    w = Batch(pa, rng, [150, 700], [1, 1], hq, 3, d, 64, "bf16", "fp4", softmax_scale=0.3,
              o_tok_stride=d, o_head_stride=t * d)
    keys, values = w.fill(rng)
    q = _rand(rng, (t, hq, d), "bf16")
    out, lse = w.attend(q)
    w.check(q, out.view(hq, t, d).transpose(0, 1), lse, keys, values)


@pytest.mark.parametrize("dtype,cache", [("bf16", "same"), ("fp32", "fp4")])
def test_scores_of_any_size(pa, dtype, cache):
    """Scores in the hundreds, rising and falling along the keys, so that the
    reference moves late, early or not at all."""
    rng = np.random.default_rng(12)
    w = Batch(pa, rng, [600, 600, 600], [1, 1, 1], 2, 1, 64, 32, dtype, cache, null_start=True)
    keys, values = [], []
    q = torch.ones((3, 2, 64), dtype=DT[dtype], device="cuda")
    k, v = torch.empty((600 * 3, 1, 64)), torch.empty((600 * 3, 1, 64))
    ramp = torch.arange(600.0)
    for b, r in enumerate((ramp / 10, (600 - ramp) / 10, torch.full((600,), 50.0))):
        k[600 * b:600 * (b + 1)] = torch.round(r)[:, None, None] / 2
    v.normal_(generator=torch.Generator().manual_seed(3))
    full = pa.Cache(**{**{f: getattr(w.cache, f) for f in w.cache.__dataclass_fields__},
                       "num_tokens": 1800, "max_new": 600})
    start = _ints([0, 600, 1200, 1800])
    kd, vd = k.to(DT[dtype]).cuda(), v.to(DT[dtype]).cuda()
    pa.proxyattn_cache_append(full, None, None, kd, vd, None, w.page_table, w.seq_lens, start,
                              w.pages)
    pa.proxyattn_cache_read(full, w.page_table, w.seq_lens, start, w.pages, kd, vd)
    for b in range(3):
        keys.append(_np(kd)[600 * b:600 * (b + 1)])
        values.append(_np(vd)[600 * b:600 * (b + 1)])
    w.check(q, *w.attend(q), keys, values)


def test_offsets_past_32_bits(pa):
    """Pools of over 2^32 values: the last pages are the ones in use."""
    rng = np.random.default_rng(13)
    for dtype, cache, pages in (("bf16", "same", 33000), ("bf16", "fp4", 67000)):
        w = Batch(pa, rng, [300, 17], [300, 17], 8, 8, 128, 128, dtype, cache)
        c = pa.Cache(**{**{f: getattr(w.cache, f) for f in w.cache.__dataclass_fields__},
                        "num_pages": pages})
        assert pa.proxyattn_cache_size(c)[0] > 2 ** 32
        table = w.page_table.clone()
        table[table >= 0] += pages - w.cache.num_pages
        pools = pa.Pages.empty(c)
        k, v, q = (_rand(rng, (317, 8, 128), dtype) for _ in range(3))
        pa.proxyattn_cache_append(c, None, None, k, v, None, table, w.seq_lens, w.new_start, pools)
        pa.proxyattn_cache_append(w.cache, None, None, k, v, None, *w.where, w.pages)
        got, ref = [], []
        for cc, tt, pp, to in ((c, table, pools, got), (w.cache, w.page_table, w.pages, ref)):
            ko, vo, out = (torch.empty_like(k) for _ in range(3))
            lse = torch.empty((8, 317), device="cuda")
            ws = torch.empty(pa.proxyattn_cache_workspace_size(cc), dtype=torch.uint8,
                             device="cuda")
            pa.proxyattn_cache_read(cc, tt, w.seq_lens, w.new_start, pp, ko, vo)
            pa.proxyattn_cache_attention(cc, q, tt, w.seq_lens, w.new_start, pp, out, lse, ws)
            to += [ko, vo, out, lse]
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
        del pools


@pytest.mark.parametrize("cache", ["same", "fp4"])
def test_large_passes_equal_small_ones(pa, cache):
    """Passes over more rows than L2 or the MALL hold go about the caches another
    way: the same rows as in parts of 10000 tokens."""
    g = torch.Generator("cuda").manual_seed(5)
    rng = np.random.default_rng(5)
    n, hq, hkv, d, page = 150000, 8, 4, 128, 64
    x = torch.randn((n, hq + 2 * hkv, d), generator=g, device="cuda").bfloat16()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    tok = (hq + 2 * hkv) * d
    r = _rotary(pa, rng, d, 128, False, True, "bf16", n)
    part = 10000

    def strides(m):
        return pa.Problem(m, hq, hkv, d, 128, 1, q_tok_stride=tok, kv_tok_stride=tok)

    for m in (n, 30000):
        qo, ko = torch.empty_like(q[:m].contiguous()), torch.empty_like(k[:m].contiguous())
        pa.proxyattn_norm_rotate(strides(m), r, q[:m], k[:m], None, 0, qo, ko)
        for a in range(0, m, part):
            qp, kp = torch.empty_like(qo[:part]), torch.empty_like(ko[:part])
            pa.proxyattn_norm_rotate(strides(part), r, q[a:a + part], k[a:a + part], None, a, qp, kp)
            assert torch.equal(qp, qo[a:a + part]) and torch.equal(kp, ko[a:a + part])
        pages = -(-m // page)
        table = torch.randperm(pages, generator=g, device="cuda").int()[None].contiguous()
        base = dict(num_seqs=1, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, page_size=page,
                    num_pages=pages, table_width=pages, cache_type=cache, max_len=m)
        one = pa.Cache(num_tokens=m, max_new=m, q_tok_stride=tok, kv_tok_stride=tok, **base)
        big, small = pa.Pages.empty(one), pa.Pages.empty(one)
        qa = torch.empty_like(qo)
        pa.proxyattn_cache_append(one, r, q[:m], k[:m], v[:m], qa, table, _ints([m]),
                                  _ints([0, m]), big)
        assert torch.equal(qa, qo)
        few = pa.Cache(num_tokens=part, max_new=part, q_tok_stride=tok, kv_tok_stride=tok, **base)
        packed = pa.Cache(num_tokens=m, max_new=m, **base)
        packed_few = pa.Cache(num_tokens=part, max_new=part, **base)
        kr, vr = (torch.empty((m, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        pa.proxyattn_cache_read(packed, table, _ints([m]), _ints([0, m]), big, kr, vr)
        if cache == "same":
            assert torch.equal(kr, ko) and torch.equal(vr, v[:m])
        for a in range(0, m, part):
            where = (table, _ints([a + part]), _ints([0, part]))
            s = slice(a, a + part)
            pa.proxyattn_cache_append(few, r, q[s], k[s], v[s], qp, *where, small)
            assert torch.equal(qp, qo[s])
            kp, vp = torch.empty_like(kr[:part]), torch.empty_like(kr[:part])
            pa.proxyattn_cache_read(packed_few, *where, small, kp, vp)
            assert torch.equal(kp, kr[s]) and torch.equal(vp, vr[s])


def test_shared_pages(pa):
    """Two sequences with the same first pages."""
    rng = np.random.default_rng(14)
    w = Batch(pa, rng, [100, 80], [1, 1], 4, 2, 64, 16, "bf16", "fp4", null_start=True)
    keys, values = w.fill(rng)
    table = w.page_table.clone()
    table[1, :4] = table[0, :4]
    w.page_table = table
    for x in (keys, values):
        x[1] = np.concatenate([x[0][:64], x[1][64:]])
    q = _rand(rng, (2, 4, 64), "bf16")
    w.check(q, *w.attend(q), keys, values)


@pytest.mark.parametrize("long", [400, 3000])
def test_step_captured_and_replayed(pa, long):
    """A decode step in a HIP graph, replayed while the lengths grow, each replay
    against the eager step; two captured steps share a workspace.  Runs of a
    workgroup each (the shorter length) and runs that are cut."""
    rng = np.random.default_rng(15)
    hq, hkv, d = 8, 2, 128
    w = Batch(pa, rng, [long, 64, 129], [1, 1, 1], hq, hkv, d, 64, "bf16", "fp4", null_start=True,
              extra_width=2, spare_pages=12)
    w.fill(rng)
    free = sorted(set(range(w.cache.num_pages)) - set(w.table[w.table >= 0].tolist()))
    for b in range(3):   # room to grow
        used = -(-w.lens[b] // 64)
        w.table[b, used] = free.pop()
    c = pa.Cache(**{**{f: getattr(w.cache, f) for f in w.cache.__dataclass_fields__},
                    "max_len": long + 64})
    assert (pa.proxyattn_cache_workspace_size(c) > 0) == (long == 3000)
    table = _ints(w.table.tolist())
    r = _rotary(pa, rng, d, 128, False, True, "bf16", long + 64)
    bufs = pa.CacheBuffers(c)
    eager = pa.CacheBuffers(c)
    bufs2 = pa.CacheBuffers(c)
    bufs2.workspace = bufs.workspace
    q, k, v = (_rand(rng, (3, h, d), "bf16") for h in (hq, hkv, hkv))
    lens = w.seq_lens.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pa.decode(c, r, q, k, v, table, lens, None, w.pages, bufs)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph, graph2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.decode(c, r, q, k, v, table, lens, None, w.pages, bufs)
    with torch.cuda.graph(graph2):
        pa.decode(c, r, q, k, v, table, lens, None, w.pages, bufs2)
    for step in range(5):
        lens += 1
        for x in (q, k, v):
            x.copy_(_rand(rng, tuple(x.shape), "bf16"))
        bufs.out.fill_(77.0)
        bufs2.out.fill_(77.0)
        graph.replay()
        graph2.replay()
        torch.cuda.synchronize()
        pa.decode(c, r, q, k, v, table, lens, None, w.pages, eager)
        torch.cuda.synchronize()
        for got in (bufs, bufs2):
            assert torch.equal(got.out, eager.out) and torch.equal(got.lse, eager.lse), step
            assert torch.equal(got.q, eager.q), step


def test_other_stream(pa):
    """Calls on a stream that is not the current one, behind that stream's work."""
    rng = np.random.default_rng(16)
    w = Batch(pa, rng, [500, 90], [1, 1], 8, 2, 128, 64, "bf16", "same", null_start=True)
    keys, values = w.fill(rng)
    q = _rand(rng, (2, 8, 128), "bf16")
    want, _ = w.attend(q)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    late = torch.zeros_like(q)
    out, lse = torch.empty_like(q), torch.empty((8, 2), device="cuda")
    ws = torch.empty(pa.proxyattn_cache_workspace_size(w.cache), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(2_000_000)
        late.copy_(q)
    pa.proxyattn_cache_attention(w.cache, late, *w.where, w.pages, out, lse, ws, stream=st)
    st.synchronize()
    assert torch.equal(out, want)


def test_prefill_with_rotary(pa):
    """The whole sparse path on projections: the same as on q and k rotated before."""
    rng = np.random.default_rng(19)
    n, hq, hkv, d = 1000, 8, 2, 128
    r = _rotary(pa, rng, d, 128, False, True, "bf16", n)
    q, k, v = (_rand(rng, (n, h, d), "bf16") for h in (hq, hkv, hkv))
    prob = pa.Problem(n, hq, hkv, d, 64, 2)
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    pa.proxyattn_norm_rotate(prob, r, q, k, None, 0, qr, kr)
    want = pa.prefill(prob, qr, kr, v, 0.9)
    got = pa.prefill(prob, q, k, v, 0.9, rotary=r)
    assert torch.equal(q, qr) and torch.equal(k, kr)
    for name in ("out", "lse", "logscore", "mass", "head_count", "block_count", "block_index"):
        assert torch.equal(getattr(got, name), getattr(want, name)), name


@pytest.mark.parametrize("cache", ["same", "fp4"])
def test_prefill_then_decode(pa, cache):
    """A prompt and ten tokens after it as a layer has them: norm and rotation,
    the prefill (dense, so that the whole is one causal attention), the cache
    filled, then single tokens and a pair of drafted ones, all against 64-bit
    causal attention over the same keys and values."""
    rng = np.random.default_rng(17)
    n, more, hq, hkv, d, page = 333, 10, 8, 2, 128, 64
    total = n + more
    fused = (hq + 2 * hkv) * d
    x = _rand(rng, (total, hq + 2 * hkv, d), "bf16", 1.5)
    r = _rotary(pa, rng, d, 128, False, True, "bf16", total)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    qt = O.round_to(_turned(r, q, r.q_weight, np.arange(total)), "bf16")
    kt = O.round_to(_turned(r, k, r.k_weight, np.arange(total)), "bf16")
    # the prompt: rotated in place, so that K and V keep their common strides
    prob = pa.Problem(n, hq, hkv, d, 64, 2, q_tok_stride=fused, kv_tok_stride=fused)
    rin = pa.Rotary(rotary_dim=128, eps=r.eps, cos=r.cos, sin=r.sin, q_weight=r.q_weight,
                    k_weight=r.k_weight, q_out_tok_stride=fused, k_out_tok_stride=fused)
    pa.proxyattn_norm_rotate(prob, rin, q[:n], k[:n], None, 0, q[:n], k[:n])
    bufs = pa.Buffers(prob)
    pa.proxyattn_dense_prefill(prob, q[:n], k[:n], v[:n], bufs.out, bufs.lse, bufs.workspace)
    vt = _np(v)
    ref, _, _, _ = O.attention(qt[:n], [kt[:n]], [vt[:n]], [(i, 0, i) for i in range(n)], d ** -0.5)
    # the prefill's own bars (bf16 probabilities): 2e-2 and 2e-3 on average
    err = np.abs(_np(bufs.out) - ref)
    assert err.max() <= 2e-2 and err.mean() <= 2e-3
    w = Batch(pa, rng, [total], [1], hq, hkv, d, page, "bf16", cache)
    base = {f: getattr(w.cache, f) for f in w.cache.__dataclass_fields__}
    base.update(q_tok_stride=fused, kv_tok_stride=fused)
    fill = pa.Cache(**{**base, "num_tokens": n, "max_new": n})
    pa.proxyattn_cache_append(fill, None, None, k[:n], v[:n], None, w.page_table, _ints([n]),
                              _ints([0, n]), w.pages)
    kc, vc = kt.copy(), vt
    if cache == "fp4":
        kc, vc = (O.dequantise(*O.quantise(y)) for y in (kt, vt))
    at = n
    for m in (1, 1, 2, 1, 5):
        c = pa.Cache(**{**base, "num_tokens": m, "max_new": m})
        s = slice(at, at + m)
        got = pa.decode(c, r, q[s], k[s], v[s], w.page_table, _ints([at + m]), _ints([0, m]),
                        w.pages)
        assert np.array_equal(_np(got.q), qt[s])
        w.cache, w.lens = c, [at + m]
        w.tokens = [(j, 0, at + j) for j in range(m)]
        w.check(got.q, got.out, got.lse, [kc], [vc])
        at += m


def test_empty_batches(pa):
    rng = np.random.default_rng(18)
    w = Batch(pa, rng, [5], [5], 2, 1, 64, 16, "bf16", "fp4")
    for kw in (dict(num_seqs=0), dict(num_tokens=0)):
        c = pa.Cache(**{**{f: getattr(w.cache, f) for f in w.cache.__dataclass_fields__}, **kw})
        assert pa.proxyattn_cache_workspace_size(c) == 0
        pa.proxyattn_cache_append(c, None, None, None, None, None, None, None, None,
                                  pa.Pages(None, None))
        pa.proxyattn_cache_read(c, None, None, None, pa.Pages(None, None), None, None)
        pa.proxyattn_cache_attention(c, None, None, None, None, pa.Pages(None, None), None, None,
                                     None)
    pa.proxyattn_norm_rotate(pa.Problem(0, 2, 1, 64, 64, 1), pa.Rotary(), None, None, None, 0,
                             None, None)
    # a batch whose sequences have no new tokens
    zero = _ints([0, 0])
    out = torch.full((5, 2, 64), 77.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(pa.proxyattn_cache_workspace_size(w.cache), dtype=torch.uint8, device="cuda")
    pa.proxyattn_cache_attention(w.cache, out, w.page_table, w.seq_lens, zero, w.pages, out, None,
                                 ws)
    assert (out == 77).all()
