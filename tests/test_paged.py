"""The paged cache without a GPU: the oracle's closed forms, the frequency rules, host refusals of the C
ABI (fake pointers: every call fails validation, or has no tokens) and of the binding."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2310_17157_amd import binding as B

FAKE = 0x10000000


@pytest.fixture(scope="module")
def lib():
    return B.load()


# ------------------------------------------------------------------ oracle
def test_oracle_rope_closed_forms():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(3, 2, 8))
    f = P.freqs(4)
    assert np.allclose(f, [1.0, 0.01])
    for layout in ("half", "interleaved"):
        y = P.rope(x, [5, 0, -3], f, layout)
        assert np.array_equal(y[1], x[1]) and np.array_equal(y[..., 4:], x[..., 4:])
        back = P.rope(y, [5, 0, -3], f, layout, inverse=True)
        assert np.allclose(back, x, atol=1e-14)
    # a quarter turn of the first pair
    y = P.rope(np.array([[[1.0, 2.0, 3.0, 4.0]]]), [1], [math.pi / 2, 0.0], "half")
    assert np.allclose(y, [[[-3.0, 2.0, 1.0, 4.0]]])
    y = P.rope(np.array([[[1.0, 2.0, 3.0, 4.0]]]), [1], [math.pi / 2, 0.0], "interleaved")
    assert np.allclose(y, [[[-2.0, 1.0, 3.0, 4.0]]])
    # products of rotated queries and keys depend on the distance alone
    q, k = rng.normal(size=(1, 1, 4)), rng.normal(size=(1, 1, 4))
    dot = lambda a, b: float((P.rope(q, [a], f) * P.rope(k, [b], f)).sum())
    assert abs(dot(7, 3) - dot(104, 100)) < 1e-12


def test_oracle_rope_gradient_by_differences():
    """The inverse with its factor is the transpose: the gradient of <w, rope(x)> with respect to x."""
    rng = np.random.default_rng(2)
    f = P.freqs(6, base=50.0)
    for layout in ("half", "interleaved"):
        x, w = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8))
        g = P.rope(w, [9], f, layout, mscale=1.3, inverse=True)
        for i in range(8):
            e = np.zeros_like(x)
            e[0, 0, i] = 1e-6
            d = ((P.rope(x + e, [9], f, layout, 1.3) - P.rope(x - e, [9], f, layout, 1.3)) * w).sum() / 2e-6
            if i < 6:
                assert abs(d - g[0, 0, i]) < 1e-8
            else:
                assert abs(d - w[0, 0, i]) < 1e-8


def test_oracle_attention_on_pages_is_attention_on_rows():
    rng = np.random.default_rng(3)
    K, V = rng.normal(size=(6, 2, 3, 4)), rng.normal(size=(6, 2, 3, 4))
    table = np.array([[4, 1, 5], [4, 0, 2]])
    q = rng.normal(size=(2, 4, 4))
    out, lse, _, _ = P.attn(q, K, V, table, [0, 1], [6, -1], 0.5, 2)
    flat = np.concatenate([K[4, 1], K[1, 1], K[5, 1]])[:7], np.concatenate([V[4, 1], V[1, 1], V[5, 1]])[:7]
    s = np.exp(flat[0] @ q[0, 3] * 0.5)
    assert np.allclose(out[0, 3], s @ flat[1] / s.sum()) and np.isclose(lse[0, 3], math.log(s.sum()))
    assert not out[1].any() and np.isneginf(lse[1]).all()
    x = rng.normal(size=(2, 2, 4))
    new = P.append(K, x, table, [0, 1], [7, 3], heads=[[1], [0]])
    assert np.array_equal(new[5, 1, 1], x[0, 1]) and np.array_equal(new[0, 0, 0], x[1, 0])
    assert (new != K).any(axis=-1).sum() == 2


# ------------------------------------------------------------------ frequencies
@pytest.mark.parametrize("rot", [2, 20, 64, 128, 256])
def test_frequencies(lib, rot):
    """Within a few roundings of pow and the division (1e-14 relative; 2^-53 each)."""
    rules = [("plain", B.DV_ROPE_PLAIN, {}), ("linear", B.DV_ROPE_LINEAR, dict(factor=8.0)),
             ("parts", B.DV_ROPE_PARTS, dict(factor=16.0, orig_len=4096.0, low=1.0, high=32.0)),
             ("parts", B.DV_ROPE_PARTS, dict(factor=8.0, orig_len=8192.0, low=1.0, high=4.0))]
    if rot > 2:
        rules.append(("ntk", B.DV_ROPE_NTK, dict(factor=4.0)))
    for base in (10000.0, 500000.0):
        for name, rule, kw in rules:
            got = B.rotary_freqs(rot, base, rule, **kw).numpy()
            want = P.freqs(rot, base, name, **kw)
            assert got.shape == (rot // 2,) and np.allclose(got, want, rtol=1e-14, atol=0)


def test_frequency_rules_end_points(lib):
    plain = B.rotary_freqs(64).numpy()
    ntk = B.rotary_freqs(64, rule=B.DV_ROPE_NTK, factor=4.0).numpy()
    assert ntk[0] == plain[0] and np.isclose(ntk[-1], plain[-1] / 4.0, rtol=1e-13)
    parts = B.rotary_freqs(64, rule=B.DV_ROPE_PARTS, factor=4.0, orig_len=4096.0).numpy()
    assert parts[0] == plain[0] and np.isclose(parts[-1], plain[-1] / 4.0, rtol=1e-14)


def test_frequency_refusals(lib):
    f = lambda rule=0, rot=8, base=1e4, factor=2.0, orig=100.0, low=1.0, high=2.0, out=(ctypes.c_double * 8)(): \
        lib.dv_rotary_freqs(rule, rot, base, factor, orig, low, high, out)
    assert f() == 0
    assert f(out=None) == B.DV_ERR_NULL
    assert f(rot=7) == f(rot=0) == f(rule=B.DV_ROPE_NTK, rot=2) == B.DV_ERR_SHAPE
    for kw in (dict(rule=4), dict(rule=-1), dict(base=0.0), dict(base=float("nan")), dict(rule=1, factor=0.0),
               dict(rule=1, factor=float("inf")), dict(rule=3, orig=0.0), dict(rule=3, low=2.0, high=2.0)):
        assert f(**kw) == B.DV_ERR_ARG, kw


# ------------------------------------------------------------------ refusals of the C ABI
def _rot(rot=16, layout=0, freq=FAKE, mscale=1.0, reserved=0):
    return B.CRotary(rot, layout, freq, mscale, reserved)


def _kv(H=4, dh=16, page=8, n_pages=10, n_seq=3, max_pages=5, ktype=B.DV_F16, reserved=0, strides=None, K=FAKE, V=FAKE,
        table=FAKE):
    ps, hs, rs = strides or (H * page * dh, page * dh, dh)
    return B.CPagedKV(H, dh, page, n_pages, n_seq, max_pages, ktype, reserved, ps, hs, rs, K, V, table)


def test_rope_refusals(lib):
    def call(r=_rot(), x=FAKE, ldx=64, xt=B.DV_F16, T=3, H=4, dh=16, pos=FAKE, out=FAKE + 4096, ldo=64, flags=0):
        return lib.dv_rope(ctypes.byref(r) if r is not None else None, x, ldx, xt, T, H, dh, pos, out, ldo, flags, None)
    assert call(r=None) == call(x=None) == call(out=None) == call(pos=None) == call(r=_rot(freq=None)) == B.DV_ERR_NULL
    assert call(xt=B.DV_Q4) == B.DV_ERR_DTYPE
    for kw in (dict(r=_rot(rot=18)), dict(r=_rot(rot=7)), dict(r=_rot(rot=0)), dict(T=-1), dict(H=-1), dict(dh=0),
               dict(ldx=63), dict(ldo=63), dict(ldx=-64)):
        assert call(**kw) == B.DV_ERR_SHAPE, kw
    for kw in (dict(r=_rot(layout=2)), dict(r=_rot(mscale=float("inf"))), dict(r=_rot(reserved=1)), dict(flags=2),
               dict(flags=8), dict(out=FAKE, ldx=80)):
        assert call(**kw) == B.DV_ERR_ARG, kw
    assert call(dh=264) == B.DV_ERR_UNSUPPORTED
    assert call(x=FAKE + 1) == call(out=FAKE + 1) == call(r=_rot(freq=FAKE + 4)) == B.DV_ERR_ALIGN
    assert call(T=0, x=None) == call(H=0, out=None) == B.DV_OK           # nothing to do


def test_paged_cache_refusals(lib):
    """Every check of the cache's description, through the append with no tokens."""
    def call(kv):
        return lib.dv_paged_append(ctypes.byref(kv) if kv is not None else None, None, None, 0, None, 0, B.DV_F32, 0, None,
                                   None, None, 0, None, 0, 0, None, 0, None)
    assert call(_kv()) == B.DV_OK
    assert call(None) == call(_kv(K=None)) == call(_kv(V=None)) == call(_kv(table=None)) == B.DV_ERR_NULL
    assert call(_kv(ktype=B.DV_Q4)) == B.DV_ERR_DTYPE
    assert call(_kv(reserved=1)) == B.DV_ERR_ARG
    for k in ("H", "dh", "page", "n_pages", "n_seq", "max_pages"):
        assert call(_kv(**{k: 0})) == B.DV_ERR_SHAPE
    assert call(_kv(dh=20)) == call(_kv(K=FAKE + 8)) == call(_kv(V=FAKE + 2)) == call(_kv(table=FAKE + 2)) == B.DV_ERR_ALIGN
    assert call(_kv(dh=264)) == call(_kv(max_pages=1 << 28)) == B.DV_ERR_UNSUPPORTED
    # strides: row-major pages, gaps, interleaved keys and values; overlapping rows, odd alignment
    for s in ((512, 16, 64), (1024, 128, 16), (4096, 136, 16), (16, 160, 1280 * 4)):
        assert call(_kv(strides=s)) == B.DV_OK, s
    for s in ((504, 128, 16), (512, 120, 16), (512, 128, 8), (512, 16, 56), (-512, 128, 16), (512, 128, 0)):
        assert call(_kv(strides=s)) == B.DV_ERR_SHAPE, s
    for s in ((516, 128, 16), (512, 130, 16), (1024, 256, 20)):
        assert call(_kv(strides=s)) == B.DV_ERR_ALIGN, s
    assert call(_kv(n_pages=1 << 30, strides=(1 << 40, 128, 16))) == B.DV_ERR_SHAPE
    assert call(_kv(page=1, strides=(64, 16, -3))) == B.DV_OK             # one row a page: no row stride


def test_append_refusals(lib):
    def call(kv=_kv(), r=_rot(), k=FAKE, ldk=64, v=FAKE, ldv=64, xt=B.DV_F32, T=3, seq=FAKE, pos=FAKE, heads=None, nh=0,
             q=FAKE, ldq=64, Hq=4, qo=FAKE + 4096, ldqo=64):
        return lib.dv_paged_append(ctypes.byref(kv), ctypes.byref(r) if r is not None else None, k, ldk, v, ldv, xt, T, seq,
                                   pos, heads, nh, q, ldq, Hq, qo, ldqo, None)
    assert call(k=None) == call(v=None) == call(pos=None) == call(q=None) == call(qo=None) == B.DV_ERR_NULL
    assert call(xt=7) == B.DV_ERR_DTYPE
    for kw in (dict(T=-1), dict(Hq=0), dict(heads=FAKE, nh=5), dict(heads=FAKE, nh=-1), dict(seq=None, T=4), dict(ldk=60),
               dict(ldv=60), dict(ldq=60), dict(ldqo=60), dict(r=_rot(rot=18))):
        assert call(**kw) == B.DV_ERR_SHAPE, kw
    assert call(qo=FAKE, ldq=68) == B.DV_ERR_ARG
    assert call(k=FAKE + 2) == call(q=FAKE + 1) == B.DV_ERR_ALIGN


def test_attention_refusals(lib):
    def call(kv=_kv(), q=FAKE, T=3, Hq=8, heads=None, nh=0, seq=FAKE, pos=FAKE, max_len=40, shared=0, scale=1.0, out=FAKE,
             lse=None, ws=FAKE, wb=1 << 30, flags=0):
        return lib.dv_paged_attn(ctypes.byref(kv), q, T, Hq, heads, nh, seq, pos, max_len, shared, scale, out, lse, ws, wb,
                                 flags, None)
    assert call(q=None) == call(pos=None) == call(out=None) == B.DV_ERR_NULL
    for kw in (dict(T=-1), dict(Hq=0), dict(Hq=6), dict(heads=FAKE, nh=9), dict(max_len=0), dict(max_len=41),
               dict(shared=-1), dict(shared=6), dict(max_len=39, shared=5), dict(seq=None, T=4)):
        assert call(**kw) == B.DV_ERR_SHAPE, kw
    assert call(scale=float("nan")) == call(scale=float("inf")) == call(flags=4) == B.DV_ERR_ARG
    assert call(q=FAKE + 4) == call(out=FAKE + 8) == call(lse=FAKE + 1) == B.DV_ERR_ALIGN
    assert call(T=1 << 20) == B.DV_ERR_UNSUPPORTED
    assert call(ws=None) == call(ws=FAKE + 16) == call(wb=128) == B.DV_ERR_WORKSPACE
    assert call(T=0, q=None) == call(heads=FAKE, nh=0, out=None) == B.DV_OK
    size = lambda *a: lib.dv_paged_attn_workspace_bytes(ctypes.byref(_kv(max_pages=5000)), *a)
    assert size(3, 8, 0, 40, 0) > 0 and size(3, 6, 0, 40, 0) == 0 and size(3, 8, 0, 0, 0) == 0
    assert size(3, 8, 0, 40000, 0) > size(3, 8, 0, 40, 0) and size(3, 8, 0, 40000, 2) > 0 and size(3, 8, 9, 40, 0) == 0
    need = size(3, 8, 0, 40000, 100)
    assert call(kv=_kv(max_pages=5000), max_len=40000, shared=100, wb=need - 256) == B.DV_ERR_WORKSPACE


def test_sparse_attn_paged_refusals(lib):
    a = B.CAttn(64, 4, 16, B.DV_F16, FAKE, FAKE, FAKE, None, None, None, FAKE, None)
    def call(a=a, x=FAKE, Bn=2, kv=_kv(), r=None, seq=FAKE, pos=FAKE, max_len=40, shared=0, heads=FAKE, nh=2, scale=1.0,
             out=FAKE, ws=FAKE, wb=1 << 30, flags=0):
        return lib.dv_sparse_attn_paged(ctypes.byref(a), x, Bn, ctypes.byref(kv), ctypes.byref(r) if r is not None else None,
                                        seq, pos, max_len, shared, heads, nh, scale, out, ws, wb, flags, None)
    assert call(x=None) == call(pos=None) == call(heads=None) == call(out=None) == B.DV_ERR_NULL
    for kw in (dict(Bn=0), dict(nh=5), dict(kv=_kv(H=2)), dict(kv=_kv(dh=32)), dict(max_len=41), dict(seq=None, Bn=4),
               dict(r=_rot(rot=18))):
        assert call(**kw) == B.DV_ERR_SHAPE, kw
    assert call(Bn=33) == B.DV_ERR_UNSUPPORTED
    assert call(scale=float("inf")) == call(flags=4) == B.DV_ERR_ARG
    need = lib.dv_sparse_attn_paged_workspace_bytes(ctypes.byref(a), ctypes.byref(_kv()), 2, 2, 40, 0)
    assert need > 0 and call(wb=need - 256) == call(ws=None) == B.DV_ERR_WORKSPACE
    f32 = B.CAttn(64, 4, 16, B.DV_F32, FAKE, FAKE, FAKE, None, None, None, FAKE, None)
    assert call(a=f32) == B.DV_ERR_UNSUPPORTED and call(a=f32, Bn=1, ws=None) == B.DV_ERR_WORKSPACE


# ------------------------------------------------------------------ refusals of the binding
def test_binding_rejects_bad_tensors():
    h16 = lambda *s: torch.zeros(*s, dtype=torch.float16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(TypeError):
        B.PagedKV(h16(4, 2, 8, 16), torch.zeros(4, 2, 8, 16), i32(1, 2)).c()
    with pytest.raises(TypeError):
        B.PagedKV(h16(4, 2, 8, 16).long(), h16(4, 2, 8, 16).long(), i32(1, 2)).c()
    with pytest.raises(ValueError, match="stride"):
        B.PagedKV(h16(4, 2, 8, 16), h16(4, 8, 2, 16).transpose(1, 2), i32(1, 2)).c()
    with pytest.raises(ValueError, match="contiguous"):
        B.PagedKV(h16(4, 2, 16, 8).transpose(2, 3), h16(4, 2, 16, 8).transpose(2, 3), i32(1, 2)).c()
    with pytest.raises(TypeError):
        B.PagedKV(h16(4, 2, 8, 16), h16(4, 2, 8, 16), torch.zeros(1, 2, dtype=torch.int64)).c()
    with pytest.raises(ValueError, match="GPU"):
        B.PagedKV(h16(4, 2, 8, 16), h16(4, 2, 8, 16), i32(1, 2)).c()
    with pytest.raises(TypeError):
        B.Rotary(torch.zeros(8)).c()
    with pytest.raises(ValueError, match="GPU"):
        B.Rotary(torch.zeros(8, dtype=torch.float64)).c()
    with pytest.raises(TypeError):
        B._tokens("x", torch.zeros(2, 3, 4, dtype=torch.int32))
    with pytest.raises(ValueError, match="contiguous"):
        B._tokens("x", torch.zeros(2, 4, 3).transpose(1, 2))
    with pytest.raises(ValueError, match="overlap"):
        B._tokens("x", torch.zeros(3, 4).expand(2, 3, 4))
    with pytest.raises(ValueError, match="shape"):
        B._tokens("x", torch.zeros(2, 3, 4), heads=5)
