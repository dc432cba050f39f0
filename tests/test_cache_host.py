"""The norm, rotation and paged-cache entry points on the host: struct layouts,
sizes, every refusal before anything reaches a GPU, and the plain forms'
pins."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import cache_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pa = pytest.importorskip("paper_2509_24745_amd.proxyattn")
torch = pytest.importorskip("torch")

FAKE = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pa.LIB_PATH):
        pytest.skip("libproxyattn.so not built")
    return pa.lib()


@pytest.mark.parametrize("struct", ["proxyattn_rotary", "proxyattn_cache"])
def test_struct_layout_matches_c_compiler(struct, tmp_path):
    cls = getattr(pa, struct)
    fields = [f[0] for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(
        ['#include <stdio.h>', '#include <stddef.h>', '#include "proxyattn.h"', 'int main(void){',
         f'printf("%zu\\n", sizeof({struct}));']
        + [f'printf("%zu\\n", offsetof({struct}, {f}));' for f in fields] + ['return 0;}']))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    vals = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()]
    assert vals == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields]


def _cache(**kw):
    base = dict(num_seqs=4, num_tokens=4, max_new=1, max_len=1000, num_q_heads=32, num_kv_heads=8,
                head_dim=128, page_size=64, num_pages=70, table_width=16)
    base.update(kw)
    return pa.Cache(**base)


@pytest.mark.parametrize("kw,code", [
    ({}, None), (dict(num_seqs=-1), pa.E_INVALID), (dict(num_tokens=-1), pa.E_INVALID),
    (dict(num_seqs=4097), pa.E_UNSUPPORTED), (dict(num_seqs=4096), None),
    (dict(max_new=0), pa.E_INVALID), (dict(max_len=0), pa.E_INVALID),
    (dict(num_pages=0), pa.E_INVALID), (dict(table_width=0), pa.E_INVALID),
    (dict(num_q_heads=30), pa.E_UNSUPPORTED), (dict(num_kv_heads=0), pa.E_INVALID),
    (dict(num_q_heads=4104), pa.E_UNSUPPORTED), (dict(head_dim=96), pa.E_UNSUPPORTED),
    (dict(page_size=8), pa.E_UNSUPPORTED), (dict(page_size=48), pa.E_UNSUPPORTED),
    (dict(page_size=512), pa.E_UNSUPPORTED), (dict(page_size=256), None),
    (dict(max_len=1025), pa.E_INVALID), (dict(max_len=1024), None),
    (dict(table_width=1 << 25), pa.E_UNSUPPORTED), (dict(dtype="fp16"), pa.E_UNSUPPORTED),
    (dict(cache_type="int8"), pa.E_UNSUPPORTED), (dict(cache_type="fp4"), None),
    (dict(softmax_scale=float("nan")), pa.E_INVALID), (dict(q_tok_stride=-8), pa.E_INVALID),
    (dict(q_tok_stride=4100), pa.E_UNSUPPORTED), (dict(kv_head_stride=4), pa.E_UNSUPPORTED),
    (dict(o_tok_stride=4), pa.E_UNSUPPORTED), (dict(dtype="fp32", o_tok_stride=4100), None),
    (dict(softmax_scale=1e-40), pa.E_INVALID), (dict(softmax_scale=1.2e-38), None),
    (dict(softmax_scale=-1.0), None), (dict(softmax_scale=float("inf")), pa.E_INVALID),
    (dict(num_tokens=2 ** 25 + 1), pa.E_UNSUPPORTED), (dict(num_tokens=2 ** 25), None),
    # more units of work than an int counts
    (dict(num_seqs=4096, num_q_heads=4096, num_kv_heads=4096), pa.E_UNSUPPORTED),
    (dict(max_new=2 ** 31 - 1), pa.E_UNSUPPORTED),
])
def test_cache_validation(lib, kw, code):
    c = _cache(**kw)
    if code is None:
        assert pa.proxyattn_cache_workspace_size(c) >= 0
        return
    with pytest.raises(pa.ProxyAttnError) as ei:
        pa.proxyattn_cache_workspace_size(c)
    assert ei.value.code == code


def test_struct_sizes_and_null(lib):
    c = pa.proxyattn_cache.from_buffer_copy(_cache()._c)
    n, m = ctypes.c_size_t(0), ctypes.c_size_t(0)
    c.struct_size = 8
    assert lib.proxyattn_cache_workspace_size(ctypes.byref(c), ctypes.byref(n)) == pa.E_INVALID
    assert lib.proxyattn_cache_workspace_size(None, ctypes.byref(n)) == pa.E_INVALID
    ok = _cache()._c
    assert lib.proxyattn_cache_workspace_size(ctypes.byref(ok), None) == pa.E_INVALID
    assert lib.proxyattn_cache_size(ctypes.byref(ok), ctypes.byref(n), None) == pa.E_INVALID
    assert lib.proxyattn_cache_size(ctypes.byref(ok), ctypes.byref(n), ctypes.byref(m)) == pa.E_OK


@pytest.mark.parametrize("dtype,cache,d,want", [
    ("bf16", "same", 128, (70 * 8 * 64 * 256, 0)), ("fp32", "same", 64, (70 * 8 * 64 * 256, 0)),
    ("bf16", "fp4", 128, (70 * 8 * 64 * 64, 70 * 8 * 64 * 4)),
    ("fp32", "fp4", 64, (70 * 8 * 64 * 32, 70 * 8 * 64 * 2))])
def test_cache_size(lib, dtype, cache, d, want):
    c = _cache(dtype=dtype, cache_type=cache, head_dim=d)
    assert pa.proxyattn_cache_size(c) == want
    p = pa.Pages.empty(c, "cpu")
    assert p.k.numel() * p.k.element_size() == want[0] == p.v.numel() * p.v.element_size()
    assert (p.k_scales.numel() if cache == "fp4" else 0) == want[1]


def _call(lib, name, *args):
    """The call with raw pointers; ints stay, structs go by reference."""
    return getattr(lib, name)(*[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a
                                for a in args])


@pytest.mark.parametrize("kw,rows,groups", [
    # 4 sequences x 8 heads, each 8 units of 128 keys and one for its start
    ({}, 16, 288),
    # 4 bits, 8 new tokens of 4 heads: 8 units of 256 keys and two
    (dict(cache_type="fp4", max_new=8, num_tokens=32, table_width=32, max_len=2000), 32, 320),
    # at most 4 units, or 8 of 64 runs: a workgroup to each run, no workspace
    (dict(cache_type="fp4", max_len=512), 0, 0), (dict(num_seqs=8, num_tokens=8), 0, 0),
    # as many workgroups as two on each of 256 CUs, or one where the rows need the registers
    (dict(num_seqs=64, num_tokens=64, max_len=1025, table_width=17), 16, 512),
    (dict(num_seqs=64, num_tokens=2000, max_new=100, max_len=1025, table_width=17), 64, 256),
    (dict(num_seqs=64, num_tokens=2000, max_new=100, max_len=1025, table_width=17,
          dtype="fp32"), 32, 256),
])
def test_workspace_of_cache_attention(lib, kw, rows, groups):
    """First units of every sequence, then two sets of partial rows to a
    workgroup: reference and sum, and the output, each region rounded up to 256
    bytes."""
    def up(x):
        return -(-x // 256) * 256
    c = _cache(**kw)
    if not groups:
        assert pa.proxyattn_cache_workspace_size(c) == 0
        return
    assert pa.proxyattn_cache_workspace_size(c) == (
        up(4 * (c.num_seqs + 1)) + up(2 * groups * rows * 8) + 2 * groups * rows * 512)


ARGS = {
    "proxyattn_cache_append": dict(c=None, r=None, q=None, k=FAKE, v=FAKE, q_out=None,
                                   table=FAKE, lens=FAKE, start=None, kp=FAKE, vp=FAKE, ks=None,
                                   vs=None, stream=None),
    "proxyattn_cache_read": dict(c=None, table=FAKE, lens=FAKE, start=None, kp=FAKE, vp=FAKE,
                                 ks=None, vs=None, k_out=FAKE, v_out=FAKE, stream=None),
    "proxyattn_cache_attention": dict(c=None, q=FAKE, table=FAKE, lens=FAKE, start=None, kp=FAKE,
                                      vp=FAKE, ks=None, vs=None, out=FAKE, lse=FAKE,
                                      workspace=FAKE, bytes=1 << 40, stream=None),
}
BAD = [
    (dict(table=None), pa.E_INVALID, "page_table is NULL"),
    (dict(lens=None), pa.E_INVALID, "seq_lens is NULL"),
    (dict(lens=FAKE + 2), pa.E_INVALID, "seq_lens not 4-byte"),
    (dict(start=FAKE + 1), pa.E_INVALID, "new_start not 4-byte"),
    (dict(kp=None), pa.E_INVALID, "k_pages is NULL"),
    (dict(vp=FAKE + 8), pa.E_INVALID, "v_pages not 16-byte"),
    (dict(ks=FAKE), pa.E_INVALID, "scales"),
    (dict(vs=FAKE), pa.E_INVALID, "scales"),
]
FP4_BAD = [(dict(), pa.E_INVALID, "k_scales is NULL"),
           (dict(ks=FAKE, vs=FAKE + 4), pa.E_INVALID, "v_scales not 16-byte")]
OWN_BAD = {
    "proxyattn_cache_append": [
        (dict(k=None), pa.E_INVALID, "k is NULL"), (dict(v=FAKE + 4), pa.E_INVALID, "v not"),
        (dict(q=FAKE), pa.E_INVALID, "need a rotary"),
        (dict(q_out=FAKE), pa.E_INVALID, "need a rotary")],
    "proxyattn_cache_read": [(dict(k_out=FAKE + 4), pa.E_INVALID, "k_out not"),
                             (dict(v_out=FAKE + 4), pa.E_INVALID, "v_out not")],
    "proxyattn_cache_attention": [
        (dict(q=None), pa.E_INVALID, "q is NULL"), (dict(out=FAKE + 4), pa.E_INVALID, "out not"),
        (dict(lse=FAKE + 2), pa.E_INVALID, "lse"),
        (dict(workspace=None), pa.E_INVALID, "workspace is NULL"),
        (dict(workspace=FAKE + 8), pa.E_INVALID, "workspace not"),
        (dict(bytes=100), pa.E_WORKSPACE, "workspace 100 bytes")],
}


@pytest.mark.parametrize("name", list(ARGS))
def test_argument_refusals(lib, name):
    for kws, cache in ((BAD + OWN_BAD[name], _cache()), (FP4_BAD, _cache(cache_type="fp4"))):
        for kw, code, text in kws:
            args = {**ARGS[name], "c": cache._c, **kw}
            assert _call(lib, name, *args.values()) == code, (kw, lib.proxyattn_last_error())
            assert text in lib.proxyattn_last_error().decode(), kw
    # fewer rows than sequences without new_start
    args = {**ARGS[name], "c": _cache(num_tokens=3)._c}
    assert _call(lib, name, *args.values()) == pa.E_INVALID
    assert "num_tokens 3" in lib.proxyattn_last_error().decode()
    # nothing to do: no argument is looked at
    for kw in (dict(num_seqs=0), dict(num_tokens=0)):
        args = {k: None for k in ARGS[name]}
        args.update(c=_cache(**kw)._c)
        if "bytes" in args:
            args["bytes"] = 0
        assert _call(lib, name, *args.values()) == pa.E_OK


def _rotary(**kw):
    r = pa.Rotary(rotary_dim=128)._c
    r.cos = r.sin = FAKE
    r.table_len = 5000
    for k, v in kw.items():
        setattr(r, k, v)
    return r


ROTARY_BAD = [
    (dict(struct_size=8), pa.E_INVALID), (dict(rotary_dim=-16), pa.E_INVALID),
    (dict(rotary_dim=144), pa.E_INVALID), (dict(rotary_dim=24), pa.E_UNSUPPORTED),
    (dict(interleaved=2), pa.E_INVALID), (dict(cos=None), pa.E_INVALID),
    (dict(sin=FAKE + 4), pa.E_INVALID), (dict(table_len=0), pa.E_INVALID),
    (dict(q_weight=FAKE + 2), pa.E_INVALID), (dict(k_weight=FAKE, norm_eps=0.0), pa.E_INVALID),
    (dict(k_weight=FAKE, norm_eps=float("nan")), pa.E_INVALID),
    (dict(q_weight=FAKE, norm_eps=-1.0), pa.E_INVALID),
    (dict(q_out_tok_stride=-16), pa.E_INVALID), (dict(k_out_head_stride=4), pa.E_UNSUPPORTED),
]


@pytest.mark.parametrize("kw,code", ROTARY_BAD)
def test_rotary_refusals(lib, kw, code):
    p = pa.Problem(4096, 32, 8, 128, 128, 4).c_struct()
    args = [FAKE, FAKE, None, 0, 2 * FAKE, 2 * FAKE, None]
    assert _call(lib, "proxyattn_norm_rotate", p, _rotary(**kw), *args) == code
    a = {**ARGS["proxyattn_cache_append"], "c": _cache()._c, "r": _rotary(**kw), "q": FAKE,
         "q_out": 2 * FAKE}
    assert _call(lib, "proxyattn_cache_append", *a.values()) == code


def test_norm_rotate_refusals(lib):
    p = pa.Problem(4096, 32, 8, 128, 128, 4).c_struct()

    def call(r, q, k, pos, first, qo, ko, prob=p):
        return _call(lib, "proxyattn_norm_rotate", prob, r, q, k, pos, first, qo, ko, None)

    r = _rotary()
    a, b = FAKE, 2 * FAKE
    assert call(r, a, a, None, 905, b, b) == pa.E_INVALID        # positions up to 5000
    assert "table_len" in lib.proxyattn_last_error().decode()
    assert call(r, a, a, None, 2 ** 31 - 1, b, b) == pa.E_INVALID
    assert call(r, a, a, None, -1, b, b) == pa.E_INVALID
    assert call(r, a, None, None, 0, b, b) == pa.E_INVALID
    assert call(r, None, a, None, 0, b, b) == pa.E_INVALID
    assert call(r, a + 4, a, None, 0, b, b) == pa.E_INVALID
    assert call(r, a, a, None, 0, b, b + 4) == pa.E_INVALID
    assert call(r, a, a, FAKE + 2, 0, b, b) == pa.E_INVALID
    # in place with other strides
    assert call(_rotary(q_out_tok_stride=8192), a, a, None, 0, a, b) == pa.E_INVALID
    assert "in place" in lib.proxyattn_last_error().decode()
    assert call(_rotary(k_out_head_stride=256), a, b, None, 0, 3 * FAKE, b) == pa.E_INVALID
    assert _call(lib, "proxyattn_norm_rotate", p, None, a, a, None, 0, b, b, None) == pa.E_INVALID
    bad = pa.Problem(4096, 32, 8, 96, 128, 4).c_struct()
    assert call(r, a, a, None, 0, b, b, prob=bad) == pa.E_UNSUPPORTED
    # nothing to do
    assert call(r, None, None, None, 0, None, None) == pa.E_OK
    assert call(r, None, None, None, 0, None, None, pa.Problem(0, 32, 8, 128, 128, 4).c_struct()) == pa.E_OK


def test_append_refusals_of_the_rotation(lib):
    base = {**ARGS["proxyattn_cache_append"], "c": _cache()._c}

    def call(**kw):
        return _call(lib, "proxyattn_cache_append", *{**base, **kw}.values())

    assert call(r=_rotary(table_len=999), q=FAKE, q_out=2 * FAKE) == pa.E_INVALID   # max_len 1000
    assert call(r=_rotary(), q=FAKE) == pa.E_INVALID
    assert call(r=_rotary(), q_out=FAKE) == pa.E_INVALID
    assert call(r=_rotary(), q=FAKE, q_out=2 * FAKE + 4) == pa.E_INVALID
    assert call(r=_rotary(q_out_tok_stride=8192), q=FAKE, q_out=FAKE) == pa.E_INVALID


def test_binding_refusals(lib):
    c = _cache()
    bf, i32 = torch.bfloat16, torch.int32
    table = torch.zeros((4, 16), dtype=i32)
    q = torch.zeros((4, 32, 128), dtype=bf)
    fake_pages = pa.Pages(FAKE, FAKE)

    def raises(match, f, *a):
        with pytest.raises(pa.ProxyAttnError, match=match):
            f(*a)

    att = pa.proxyattn_cache_attention
    raises("q: tensor on cpu", att, c, q, FAKE, FAKE, None, fake_pages, FAKE, FAKE, None)
    raises("q: dtype", att, c, q.float(), FAKE, FAKE, None, fake_pages, FAKE, FAKE, None)
    raises("q: .* touches", att, c, q[:3].clone(), FAKE, FAKE, None, fake_pages, FAKE, FAKE, None)
    raises("page_table: dtype", att, c, FAKE, table.long(), FAKE, None, fake_pages, FAKE, FAKE, None)
    raises("page_table: not contiguous", att, c, FAKE, torch.zeros((16, 4), dtype=i32).t(), FAKE,
           None, fake_pages, FAKE, FAKE, None)
    raises("seq_lens: .* touches", att, c, FAKE, FAKE, torch.zeros(3, dtype=i32), None, fake_pages,
           FAKE, FAKE, None)
    raises("new_start: .* touches", att, c, FAKE, FAKE, FAKE, torch.zeros(4, dtype=i32),
           fake_pages, FAKE, FAKE, None)
    raises("k_pages: dtype", att, c, FAKE, FAKE, FAKE, None,
           pa.Pages(torch.zeros(8, dtype=torch.uint8), FAKE), FAKE, FAKE, None)
    raises("v_pages: .* touches", att, c, FAKE, FAKE, FAKE, None,
           pa.Pages(FAKE, torch.zeros(8, dtype=bf)), FAKE, FAKE, None)
    raises("lse: .* touches", att, c, FAKE, FAKE, FAKE, None, fake_pages, FAKE,
           torch.zeros(127), None)
    raises("workspace: tensor on cpu", att, c, FAKE, FAKE, FAKE, None, fake_pages, FAKE, FAKE,
           torch.zeros(1 << 26, dtype=torch.uint8))
    rot = pa.Rotary(rotary_dim=64, cos=torch.zeros((1000, 32)), sin=torch.zeros((999, 32)))
    raises("sin: 999 rows", pa.proxyattn_cache_append, c, rot, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE,
           None, fake_pages)
    rot = pa.Rotary(rotary_dim=64, cos=torch.zeros((1000, 31)), sin=torch.zeros((1000, 31)))
    raises("cos: .* touches", pa.proxyattn_cache_append, c, rot, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE,
           None, fake_pages)
    rot = pa.Rotary(q_weight=torch.zeros(128))
    raises("q_weight: dtype", pa.proxyattn_norm_rotate, pa.Problem(9, 32, 8, 128, 128, 1), rot,
           FAKE, None, None, 0, FAKE, None)
    raises("positions: .* touches", pa.proxyattn_norm_rotate, pa.Problem(9, 32, 8, 128, 128, 1),
           pa.Rotary(), FAKE, None, torch.zeros(8, dtype=i32), 0, FAKE, None)
    raises("k_out: .* touches", pa.proxyattn_cache_read, c, FAKE, FAKE, None, fake_pages,
           torch.zeros((4, 7, 128), dtype=bf), None)


# ---------------------------------------------------------------------------
# pins of the plain forms
# ---------------------------------------------------------------------------
def test_oracle_quantise_pins():
    """Hand-checked groups: ties go to the even code, up to 7 times the scale is
    clipped to 6, above that the scale doubles; zeros take the smallest scale."""
    x = np.zeros((4, 32))
    x[0, :9] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.5]
    x[1, :2] = [7.5, 3.5]
    x[2, 0] = 2.0 ** 127
    codes, scales = O.quantise(x)
    nib = np.stack((codes & 15, codes >> 4), -1).reshape(4, 32)
    assert nib[0, :9].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 9] and scales[0, 0] == 127
    assert nib[1, :2].tolist() == [6, 4] and scales[1, 0] == 128
    assert scales[2, 0] == 252 and nib[2, 0] == 6
    assert scales[3, 0] == 17 and not nib[3].any()
    back = O.dequantise(codes, scales)
    assert back[0, :9].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -0.5] and back[2, 0] == 2.0 ** 127
    again = O.dequantise(*O.quantise(back))
    assert np.array_equal(again, back)


def test_oracle_rotation_pins():
    """Rotations keep the length of every pair and scores depend on the distance
    of positions alone; a quarter turn; rounding to bf16 against torch."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 2, 64))
    ang = np.arange(40)[:, None] * 0.7 ** np.arange(16)
    cos, sin = np.cos(ang), np.sin(ang)
    for inter in (False, True):
        y = O.norm_rotate(x, np.arange(5) + 3, 32, inter, cos, sin)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 32:], x[..., 32:])
        a = [O.norm_rotate(x[:1], np.array([p]), 32, inter, cos, sin)[0, 0] for p in (3, 20)]
        b = [O.norm_rotate(x[1:2], np.array([p]), 32, inter, cos, sin)[0, 0] for p in (8, 25)]
        assert np.isclose(a[0] @ b[0], a[1] @ b[1])
    quarter = O.norm_rotate(np.arange(32.0)[None, None], np.array([0]), 32, False,
                            np.zeros((1, 16)), np.ones((1, 16)))[0, 0]
    assert quarter.tolist() == [-16.0 - i for i in range(16)] + [float(i) for i in range(16)]
    n = O.norm_rotate(np.full((1, 1, 64), 5.0), np.array([0]), weight=np.full(64, 2.0), eps=1e-12)
    assert np.allclose(n, 2.0)
    z = rng.standard_normal(1000)
    assert np.array_equal(O.round_to(z, "bf16"),
                          torch.from_numpy(z.astype(np.float32)).bfloat16().double().numpy())


def test_oracle_attention_pins():
    """One key: its value.  Equal scores: the mean of the keys seen so far.
    Against torch's softmax in 64 bits."""
    rng = np.random.default_rng(1)
    k, v, q = rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64)), rng.standard_normal((3, 4, 64))
    tokens = O.batch([9, 0], [0, 2, 3], 2)
    assert tokens == [(0, 0, 7), (1, 0, 8), (2, 1, -1)]
    out, lse, _, _ = O.attention(q * 0, [k, k[:0]], [v, v[:0]], tokens, 0.125)
    assert np.allclose(out[0, 0], v[:8, 0].mean(0)) and np.isclose(lse[3, 1], np.log(9))
    assert not out[2].any() and np.isneginf(lse[:, 2]).all()
    out, lse, _, _ = O.attention(q, [k], [v], [(0, 0, 8)], 0.3)
    s = torch.from_numpy(0.3 * np.einsum("hd,nhd->hn", q[0], np.repeat(k, 2, 1)))
    assert np.allclose(out[0], np.einsum("hn,nhd->hd", torch.softmax(s, -1).numpy(), np.repeat(v, 2, 1)))
    assert np.allclose(lse[:, 0], torch.logsumexp(s, -1).numpy())
