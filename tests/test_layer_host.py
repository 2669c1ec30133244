"""Host side of the operators around the matmuls: their refusals (nothing is launched,
no GPU needed), launch plans, and pins of their oracle."""

import ctypes as C
import math
import os

import numpy as np
import pytest

import paper_2608_15531_amd as fq
from oracle import layer as L

FAKE = 1 << 20   # a 16-byte aligned address that is never followed


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fq.LIB_PATH):
        from paper_2608_15531_amd.build import build
        build()
    return fq.load()


def name(status):
    return fq.STATUS_NAMES[status]


def cache(**kw):
    kind = kw.get("kind", fq.FQ_KV_INT8)
    D = kw.get("head_dim", 128)
    row = {fq.FQ_KV_BF16: 2 * D, fq.FQ_KV_INT8: D}.get(kind, D // 2)
    page, heads = kw.get("page_size", 64), kw.get("n_kv_heads", 8)
    d = dict(k=FAKE, v=FAKE, k_meta=FAKE, v_meta=FAKE, page_stride=heads * page * row, head_stride=page * row,
             token_stride=row, meta_page_stride=heads * page, meta_head_stride=page, n_pages=10, page_size=64,
             n_kv_heads=8, head_dim=128, kind=fq.FQ_KV_INT8)
    d.update(kw)
    return fq.fq_kv_cache(**d)


def attn(**kw):
    d = dict(n_seqs=2, n_heads=32, max_q=1, max_kv=500, window=0, sinks=0, total_q=2, q_token_stride=4096,
             q_head_stride=128, o_token_stride=4096, o_head_stride=128, table_stride=10, table_cols=10, scale=0.1)
    d.update(kw)
    return fq.fq_attention(**d)


BAD_CACHES = [
    (dict(k=None), "FQ_ERR_NULL"), (dict(v=None), "FQ_ERR_NULL"), (dict(k_meta=None), "FQ_ERR_NULL"),
    (dict(v_meta=None), "FQ_ERR_NULL"), (dict(n_pages=0), "FQ_ERR_SHAPE"), (dict(n_kv_heads=0), "FQ_ERR_SHAPE"),
    (dict(page_size=0), "FQ_ERR_SHAPE"), (dict(page_size=24), "FQ_ERR_UNSUPPORTED"),
    (dict(page_size=65552), "FQ_ERR_UNSUPPORTED"), (dict(head_dim=96), "FQ_ERR_UNSUPPORTED"),
    (dict(head_dim=0), "FQ_ERR_SHAPE"), (dict(kind=3), "FQ_ERR_UNSUPPORTED"),
    (dict(n_pages=1 << 31), "FQ_ERR_UNSUPPORTED"), (dict(n_kv_heads=65536), "FQ_ERR_UNSUPPORTED"),
    (dict(token_stride=136), "FQ_ERR_ALIGN"), (dict(head_stride=8), "FQ_ERR_ALIGN"),
    (dict(page_stride=-16), "FQ_ERR_SHAPE"), (dict(token_stride=1 << 30), "FQ_ERR_UNSUPPORTED"),
    (dict(meta_head_stride=62), "FQ_ERR_ALIGN"), (dict(meta_page_stride=-4), "FQ_ERR_SHAPE"),
    (dict(k=FAKE + 8), "FQ_ERR_ALIGN"), (dict(v_meta=FAKE + 4), "FQ_ERR_ALIGN"),
]


@pytest.mark.parametrize("kw,want", BAD_CACHES, ids=[f"{list(k)[0]}{i}" for i, (k, _) in enumerate(BAD_CACHES)])
def test_bad_caches_are_refused(lib, kw, want):
    c = cache(**kw)
    assert name(lib.fq_kv_cache_write(C.byref(c), FAKE, FAKE, 1024, 128, 1024, 128, FAKE, 4, None)) == want
    assert name(lib.fq_kv_cache_read(C.byref(c), FAKE, 4, FAKE, FAKE, 0, None)) == want
    a = attn(n_heads=8 if kw.get("n_kv_heads", 8) else 8)
    if "n_kv_heads" not in kw:
        assert name(lib.fq_paged_attention(C.byref(a), FAKE, C.byref(c), FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 30,
                                           None)) == want


def test_cache_calls_refuse(lib):
    c = cache()
    w = lambda *a: name(lib.fq_kv_cache_write(C.byref(c), *a))   # noqa: E731
    assert name(lib.fq_kv_cache_write(None, FAKE, FAKE, 0, 0, 0, 0, FAKE, 1, None)) == "FQ_ERR_NULL"
    assert w(None, FAKE, 1024, 128, 1024, 128, FAKE, 4, None) == "FQ_ERR_NULL"
    assert w(FAKE, FAKE, 1024, 128, 1024, 128, None, 4, None) == "FQ_ERR_NULL"
    assert w(FAKE, FAKE, 1024, 128, 1024, 128, FAKE, -1, None) == "FQ_ERR_SHAPE"
    assert w(FAKE, FAKE, -8, 128, 1024, 128, FAKE, 4, None) == "FQ_ERR_SHAPE"
    assert w(FAKE, FAKE, 1020, 128, 1024, 128, FAKE, 4, None) == "FQ_ERR_ALIGN"
    assert w(FAKE, FAKE + 2, 1024, 128, 1024, 128, FAKE, 4, None) == "FQ_ERR_ALIGN"
    assert w(FAKE, FAKE, 1024, 128, 1024, 128, FAKE + 4, 4, None) == "FQ_ERR_ALIGN"
    assert w(None, None, 0, 0, 0, 0, None, 0, None) == "FQ_OK"            # nothing to store
    r = lambda *a: name(lib.fq_kv_cache_read(C.byref(c), *a))   # noqa: E731
    assert r(FAKE, 4, FAKE, FAKE, 2, None) == "FQ_ERR_UNSUPPORTED"
    assert r(FAKE, -4, FAKE, FAKE, 0, None) == "FQ_ERR_SHAPE"
    assert r(FAKE, 4, FAKE + 8, FAKE, 0, None) == "FQ_ERR_ALIGN"
    assert r(FAKE, 4, None, FAKE, 0, None) == "FQ_ERR_NULL"
    assert r(None, 0, None, None, 1, None) == "FQ_OK"


BAD_CALLS = [
    (dict(n_seqs=0), "FQ_ERR_SHAPE"), (dict(n_heads=12), "FQ_ERR_SHAPE"), (dict(n_heads=0), "FQ_ERR_SHAPE"),
    (dict(max_q=0), "FQ_ERR_SHAPE"), (dict(max_kv=0), "FQ_ERR_SHAPE"), (dict(max_kv=641), "FQ_ERR_SHAPE"),
    (dict(window=-1), "FQ_ERR_SHAPE"), (dict(sinks=-1), "FQ_ERR_SHAPE"), (dict(total_q=-1), "FQ_ERR_SHAPE"),
    (dict(scale=math.inf), "FQ_ERR_SHAPE"), (dict(scale=math.nan), "FQ_ERR_SHAPE"),
    (dict(q_token_stride=-8), "FQ_ERR_SHAPE"), (dict(q_token_stride=4100), "FQ_ERR_ALIGN"),
    (dict(o_head_stride=132), "FQ_ERR_ALIGN"), (dict(table_cols=0), "FQ_ERR_SHAPE"),
    (dict(table_stride=-1), "FQ_ERR_SHAPE"),
    (dict(n_seqs=65536), "FQ_ERR_UNSUPPORTED"), (dict(max_q=1 << 30), "FQ_ERR_UNSUPPORTED"),
]


@pytest.mark.parametrize("kw,want", BAD_CALLS, ids=[f"{list(k)[0]}{i}" for i, (k, _) in enumerate(BAD_CALLS)])
def test_attention_refuses(lib, kw, want):
    c, a = cache(), attn(**kw)
    n = C.c_size_t(7)
    assert name(lib.fq_paged_attention(C.byref(a), FAKE, C.byref(c), FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 40,
                                       None)) == want
    assert name(lib.fq_paged_attention_workspace_bytes(C.byref(a), C.byref(c), C.byref(n))) == want
    assert n.value == 7


def test_attention_refuses_pointers(lib):
    c, a = cache(), attn(max_kv=600)
    good = [FAKE] * 5

    def call(i, p, lse=None, ws=FAKE, size=1 << 30):
        x = list(good)
        if i is not None:
            x[i] = p
        return name(lib.fq_paged_attention(C.byref(a), x[0], C.byref(c), x[1], x[2], x[3], x[4], lse, ws, size, None))

    for i in range(5):
        assert call(i, None) == "FQ_ERR_NULL"
    assert call(0, FAKE + 8) == "FQ_ERR_ALIGN" and call(4, FAKE + 8) == "FQ_ERR_ALIGN"
    assert call(1, FAKE + 2) == "FQ_ERR_ALIGN" and call(None, None, lse=FAKE + 2) == "FQ_ERR_ALIGN"
    assert name(lib.fq_paged_attention(None, FAKE, C.byref(c), FAKE, FAKE, FAKE, FAKE, None, FAKE, 1, None)) == \
        "FQ_ERR_NULL"
    b = attn(total_q=0)
    assert name(lib.fq_paged_attention(C.byref(b), None, C.byref(c), None, None, None, None, None, None, 0,
                                       None)) == "FQ_OK"


def test_attention_workspace_is_checked(lib):
    c, a = cache(), attn(n_seqs=1, total_q=1, max_kv=64000, table_cols=1000)
    n, out = C.c_size_t(0), (C.c_int32 * 8)()
    assert lib.fq_paged_attention_workspace_bytes(C.byref(a), C.byref(c), C.byref(n)) == 0
    assert lib.fq_paged_attention_launch(C.byref(a), C.byref(c), out) == 0
    assert out[3] > 1 and n.value > 256 * 1024

    def call(ws, size):
        return name(lib.fq_paged_attention(C.byref(a), FAKE, C.byref(c), FAKE, FAKE, FAKE, FAKE, None, ws, size, None))

    assert call(None, n.value) == "FQ_ERR_WORKSPACE"
    assert call(FAKE, n.value - 1) == "FQ_ERR_WORKSPACE"
    assert call(FAKE + 16, n.value) == "FQ_ERR_WORKSPACE"


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("heads", [(1, 1), (32, 8), (64, 8), (6, 2), (24, 1)])
def test_attention_plans_cover_the_keys(lib, heads, head_dim):
    """Every plan's ranges cover all tiles that a block of rows can see."""
    for max_q in (1, 5, 16, 100, 2048):
        for max_kv in (1, 31, 33, 1000, 32768, 131072):
            for window, sinks in ((0, 0), (1, 0), (100, 4), (4096, 200)):
                for n_seqs in (1, 7, 64):
                    c = cache(n_kv_heads=heads[1], head_dim=head_dim, kind=fq.FQ_KV_BF16, n_pages=1 << 20)
                    a = attn(n_seqs=n_seqs, n_heads=heads[0], max_q=max_q, max_kv=max_kv, table_cols=2048,
                             window=window, sinks=sinks)
                    out = (C.c_int32 * 8)()
                    assert lib.fq_paged_attention_launch(C.byref(a), C.byref(c), out) == 0
                    G = heads[0] // heads[1]
                    assert out[1] * out[2] >= max_q * G
                    assert out[5] == out[2] * out[3] * n_seqs * heads[1]
                    # keys seen by out[1] neighbouring rows anywhere, in whole 32-key tiles
                    tokens = min(max_q, (out[1] - 1) // G + 2)
                    for p in {0, 1, 31, 32, 1000, max_kv - tokens, max_kv - 1}:
                        p_lo, p_hi = max(0, min(p, max_kv - 1)), max(0, min(p + tokens - 1, max_kv - 1))
                        j = np.arange(0, max_kv)
                        see = (j <= p_hi) & ((j > p_lo - window) | (j < sinks) if window else True)
                        assert len(set((j[see] // 32).tolist())) <= out[3] * (out[4] // 32), (max_q, max_kv, window)


@pytest.mark.parametrize("group", [1, 3, 4, 8, 24])
def test_attention_blocks_of_many_rows_are_numbered_once(group):
    """The numbers that the kernel for many rows gives its blocks (the rows before them / 128
    + the sequence + the block) differ and stay below total rows / 128 + sequences, whatever
    the lengths."""
    rng = np.random.default_rng(group)
    for case in range(300):
        q = rng.integers(0, [2, 40, 400][case % 3], int(rng.integers(1, 12)))
        max_q = int(q.max()) if case % 2 else int(rng.integers(1, 400))
        cu = np.concatenate([[0], np.cumsum(q)])
        seen = [cu[b] * group // 128 + b + rb for b in range(len(q))
                for rb in range(-(-min(int(q[b]), max_q) * group // 128))]
        assert len(set(seen)) == len(seen)
        assert all(0 <= n < cu[-1] * group // 128 + len(q) for n in seen)


def test_norm_refuses(lib):
    def call(x=FAKE, res=FAKE, post=FAKE, gate=FAKE, pre=FAKE, out=FAKE, h=FAKE, **kw):
        d = dict(rows=4, cols=128, x_dtype=0, residual_dtype=0, eps=1e-5, residual_scale=1.0, x_stride=128,
                 residual_stride=128, gate_stride=0, residual_out_stride=128, h_stride=128)
        d.update(kw)
        return name(lib.fq_gated_residual_norm(C.byref(fq.fq_norm(**d)), x, res, post, gate, pre, out, h, None))

    assert name(lib.fq_gated_residual_norm(None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None)) == "FQ_ERR_NULL"
    assert call(x=None) == "FQ_ERR_NULL" and call(pre=None) == "FQ_ERR_NULL"
    assert call(out=None, h=None) == "FQ_ERR_NULL"
    for kw in (dict(rows=-1), dict(cols=0), dict(x_stride=-1), dict(gate_stride=-1), dict(eps=-1.0),
               dict(eps=math.nan), dict(residual_scale=math.inf)):
        assert call(**kw) == "FQ_ERR_SHAPE", kw
    for kw in (dict(cols=32769), dict(x_dtype=2), dict(residual_dtype=-1), dict(rows=1 << 31)):
        assert call(**kw) == "FQ_ERR_UNSUPPORTED", kw
    assert call(x=FAKE + 1) == "FQ_ERR_ALIGN" and call(x=FAKE + 2, x_dtype=1) == "FQ_ERR_ALIGN"
    assert call(out=FAKE + 2, residual_dtype=1) == "FQ_ERR_ALIGN" and call(h=FAKE + 1) == "FQ_ERR_ALIGN"
    assert call(rows=0, x=None) == "FQ_OK"


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    t = torch.zeros((2, 1, 16, 128), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        fq.KVCache(t, t)                                   # not on a GPU
    with pytest.raises(ValueError):
        fq.KVCache(t, t, kind="fp8")
    with pytest.raises(ValueError):
        fq.KVCache(t[0], t[0])
    with pytest.raises(ValueError):
        fq.PagedBatch(t, t, t, 1, 1)
    with pytest.raises(ValueError):
        fq.fq_paged_attention(t, None, None)
    with pytest.raises(ValueError):
        fq.fq_gated_residual_norm(t)


def test_norm_refuses_host_tensors(lib):
    torch = pytest.importorskip("torch")
    x, w = torch.zeros((2, 64), dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="CUDA"):
        fq.fq_gated_residual_norm(x, x, w)


@pytest.mark.parametrize("name", ["max_q", "max_kv", "window", "sinks"])
def test_numbers_beyond_32_bits_are_refused(name):
    from types import SimpleNamespace
    v = dict(max_q=1, max_kv=500, window=0, sinks=0)
    cache = SimpleNamespace(head_dim=128)

    def call(v):
        batch = SimpleNamespace(n_seqs=1, max_q=v["max_q"], max_kv=v["max_kv"], table_stride=10, _table_cols=10)
        return fq._attention(8, (1024, 128), (1024, 128), 1, cache, batch, None, v["window"], v["sinks"])

    assert getattr(call({**v, name: 2**31 - 1}), name) == 2**31 - 1
    with pytest.raises(ValueError):
        call({**v, name: 2**32 + 5})


# ----------------------------------------------------------- oracle pins --

def test_oracle_bf16_ceil():
    def up(x):   # by the bits
        b = np.float32(x).view(np.uint32)
        return float(((b + np.uint32(0xFFFF)) & np.uint32(0xFFFF0000)).view(np.float32))

    for x in (1.0, 1.0000001, 1.0078125, 3.14159, 255.1, 2.0 ** -126, 1.5 * 2.0 ** -130, 2.0 ** -133, 3e38):
        x = float(np.float32(x))
        assert L.bf16_ceil(x) == up(x), x


def test_oracle_quantiser():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 128))
    for kind, top in L.LEVELS.items():
        c, s, z = L.quantise_rows(x, kind)
        assert c.min() >= 0 and c.max() <= top and (c == np.rint(c)).all()
        # within half a step (the widened range covers every value)
        assert (np.abs(s * (c - z) - x) <= 0.5 * s * (1 + 1e-12) + 0.5 * s * (np.abs(c - top) < 1)).all()
        # exactly representable rows come back exactly
        y = np.arange(top + 1.0)[None] * 0.25
        assert (L.held_rows(y, kind) == y).all()
    assert (L.held_rows(np.zeros((1, 64)), "int4") == 0).all()
    assert np.isnan(L.held_rows(np.array([[1.0, np.inf]]), "int8")).all()


def test_oracle_attention_closed_forms():
    rng = np.random.default_rng(1)
    k, v, q = rng.standard_normal((9, 4)), rng.standard_normal((9, 4)), rng.standard_normal(4)
    see = np.ones(9, bool)
    # equal scores: the mean
    o, lse, _, _ = L.attention_row(np.zeros(4), k, v, see, 1.0)
    np.testing.assert_allclose(o, v.mean(0))
    np.testing.assert_allclose(lse, np.log(9))
    # one key: its value
    one = np.zeros(9, bool)
    one[4] = True
    o, lse, _, _ = L.attention_row(q, k, v, one, 0.5)
    np.testing.assert_allclose(o, v[4])
    np.testing.assert_allclose(lse, 0.5 * k[4] @ q)
    # two keys: the logistic function of the scores' difference
    two = np.zeros(9, bool)
    two[[2, 7]] = True
    p = 1 / (1 + np.exp(-(k[2] - k[7]) @ q))
    np.testing.assert_allclose(L.attention_row(q, k, v, two, 1.0)[0], p * v[2] + (1 - p) * v[7])
    # what is not seen takes no part
    k[0], v[1] = np.nan, np.inf
    np.testing.assert_allclose(L.attention_row(q, k, v, two, 1.0)[0], p * v[2] + (1 - p) * v[7])
    assert L.attention_row(q, k, v, np.zeros(9, bool), 1.0)[1] == -np.inf
    assert L.visible(5, 8, 0, 0).tolist() == [1, 1, 1, 1, 1, 1, 0, 0]
    assert L.visible(5, 8, 2, 1).tolist() == [1, 0, 0, 0, 1, 1, 0, 0]
    assert not L.visible(-1, 8, 0, 0).any()


def test_oracle_norm_closed_forms():
    x = np.array([[3.0, -3.0], [1.0, 1.0]])
    r, h, _ = L.gated_residual_norm(x, np.ones((2, 2)), np.array([2.0, 1.0]), np.ones(2), np.array([1.0, 0.5]), 2.0, 0.0)
    np.testing.assert_allclose(r, [[3.0, 1.5], [3.0, 2.5]])
    np.testing.assert_allclose(h[0], np.array([6.0, 1.5]) / np.sqrt((9 + 2.25) / 2))
    r, h, _ = L.gated_residual_norm(x, None, None, None, None, 1.0, 1e-5)
    assert (r == x).all() and h is None


@pytest.mark.parametrize("scale,want", [(2.358e38, "FQ_OK"), (-2.358e38, "FQ_OK"), (2.36e38, "FQ_ERR_SHAPE"),
                                        (-3.4e38, "FQ_ERR_SHAPE")])
def test_attention_scales_beyond_its_powers_of_two(lib, scale, want):
    """The kernels multiply by scale log2(e), which has to be finite too."""
    c, a, n = cache(), attn(scale=scale), C.c_size_t(7)
    assert name(lib.fq_paged_attention_workspace_bytes(C.byref(a), C.byref(c), C.byref(n))) == want


@pytest.mark.parametrize("name", ["max_q", "max_kv", "window", "sinks"])
@pytest.mark.parametrize("value", [-2**31 - 1, -2**32 + 5])
def test_numbers_below_32_bits_are_refused(name, value):
    """Which 32 bits would make positive; other negative ones reach the library's check."""
    from types import SimpleNamespace

    def call(value):
        v = {**dict(max_q=1, max_kv=500, window=0, sinks=0), name: value}
        batch = SimpleNamespace(n_seqs=1, max_q=v["max_q"], max_kv=v["max_kv"], table_stride=10, _table_cols=10)
        return fq._attention(8, (1024, 128), (1024, 128), 1, SimpleNamespace(head_dim=128), batch, None, v["window"],
                             v["sinks"])

    with pytest.raises(ValueError):
        call(value)
    assert getattr(call(-1), name) == -1


@pytest.mark.parametrize("heads", [(32, 8), (64, 64), (8, 1), (24, 1)])
@pytest.mark.parametrize("total", [1, 5000, 1 << 22])
def test_attention_grids_stay_within_hip_limits(lib, heads, total):
    """Fewer than 2^32 threads in one dimension of a grid, of the kernel and of its join, for any
    bounds; what cannot be launched so is refused."""
    c = cache(n_kv_heads=heads[1], kind=fq.FQ_KV_BF16, n_pages=1 << 20)
    launched = set()
    for bits in range(8, 29, 2):
        for max_kv in (100, 30000, 1 << 20):
            for n_seqs in (1, 3, 100):
                a = attn(n_seqs=n_seqs, n_heads=heads[0], max_q=1 << bits, max_kv=max_kv, total_q=total,
                         table_cols=1 << 14)
                out, n = (C.c_int32 * 8)(), C.c_size_t(0)
                status = name(lib.fq_paged_attention_launch(C.byref(a), C.byref(c), out))
                blocks = -(-(heads[0] // heads[1] << bits) // 128) * heads[1]
                where = (bits, max_kv, n_seqs, list(out))
                if blocks >= 1 << 24 or blocks * n_seqs >= 1 << 31:
                    assert status == "FQ_ERR_UNSUPPORTED", where
                    continue
                assert status == "FQ_OK", where
                launched.add(bits)
                assert out[5] == out[2] * out[3] * heads[1] * n_seqs, where
                assert out[5] // n_seqs * 256 < 1 << 32, where
                if out[3] > 1 and out[0] == fq.FQ_ATTN_TILES:
                    assert out[2] * heads[1] * 8 * 256 < 1 << 32, where
                assert lib.fq_paged_attention_workspace_bytes(C.byref(a), C.byref(c), C.byref(n)) == 0
    assert max(launched) >= 20


@pytest.mark.parametrize("dtype", ["f16", "float16", "int8", None])
def test_cache_read_refuses_other_types(lib, dtype):
    from types import SimpleNamespace
    torch = pytest.importorskip("torch")
    c = SimpleNamespace(_index=-1, n_kv_heads=1, head_dim=64, device="cpu", _ref=None)
    with pytest.raises(ValueError, match="dtype"):
        fq.fq_kv_cache_read(c, torch.zeros(0, dtype=torch.int64), dtype=dtype)


def test_workspaces_of_the_caller_are_checked():
    """One in host memory, on another device or with gaps would be written where it is not."""
    torch = pytest.importorskip("torch")
    t = torch.zeros(64, dtype=torch.int32)
    assert fq._check_workspace(t, -1) == 256   # -1: host memory, as the device asked for
    for bad in (t[::2], None, 5):
        with pytest.raises(ValueError, match="ws"):
            fq._check_workspace(bad, -1)
    with pytest.raises(ValueError, match="ws"):
        fq._check_workspace(t, 0)


@pytest.mark.parametrize("call", ["write", "read", "attention"])
def test_calls_make_the_tensors_device_current(lib, monkeypatch, call):
    """With another device current its default stream, which has the same handle, would run the
    kernel.  (The calls then stop at their first tensor check: there is no GPU here.)"""
    from types import SimpleNamespace
    torch = pytest.importorskip("torch")
    current, seen = [0], []

    class device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, current[0] = current[0], self.index
            seen.append(self.index)

        def __exit__(self, *exc):
            current[0] = self.before

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(fq, "_current_device", lambda: current[0])
    c = SimpleNamespace(_index=1, n_kv_heads=1, head_dim=64, device="cuda:1", _ref=None)
    t = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    with pytest.raises((TypeError, ValueError)):
        if call == "write":
            fq.fq_kv_cache_write(c, t, t, None)
        elif call == "read":
            fq.fq_kv_cache_read(c, None)
        else:
            fq.fq_paged_attention(t, c, SimpleNamespace(_index=1))
    assert seen == [1] and current == [0]


def test_streams_of_other_devices_are_refused():
    from types import SimpleNamespace
    with pytest.raises(ValueError, match="stream"):
        fq._stream_of(SimpleNamespace(device_index=1, cuda_stream=5), 0)
    assert fq._stream_of(SimpleNamespace(device_index=1, cuda_stream=5), 1) == 5


def test_overlapping_outputs_are_refused(lib):
    """Rows over one another would be written by several workgroups; inputs may repeat rows."""
    def write(**kw):
        return name(lib.fq_kv_cache_write(C.byref(cache(**kw)), FAKE, FAKE, 0, 0, 0, 0, FAKE, 0, None))

    assert write() == "FQ_OK"
    for kw in (dict(head_stride=0), dict(token_stride=0), dict(page_stride=64), dict(meta_head_stride=32),
               dict(meta_page_stride=0), dict(kind=fq.FQ_KV_BF16, token_stride=128)):
        assert write(**kw) == "FQ_ERR_SHAPE", kw
    assert write(n_pages=1, page_stride=0, meta_page_stride=0) == "FQ_OK"
    assert write(kind=fq.FQ_KV_BF16, meta_page_stride=0, meta_head_stride=0) == "FQ_OK"

    c = cache()

    def attend(**kw):
        a = attn(**kw)
        return name(lib.fq_paged_attention(C.byref(a), FAKE, C.byref(c), FAKE, FAKE, FAKE, None, None, FAKE, 1 << 40, None))

    assert attend() == "FQ_ERR_NULL"   # O: checked after the strides
    assert attend(q_token_stride=0, q_head_stride=0) == "FQ_ERR_NULL"
    for kw in (dict(o_token_stride=0), dict(o_head_stride=64), dict(o_head_stride=0)):
        assert attend(**kw) == "FQ_ERR_SHAPE", kw
    assert attend(total_q=1, o_token_stride=0) == "FQ_ERR_NULL"

    def norm(out=FAKE, h=FAKE, **kw):
        d = dict(rows=4, cols=128, x_dtype=0, residual_dtype=0, eps=1e-5, residual_scale=1.0, x_stride=0,
                 residual_stride=0, gate_stride=0, residual_out_stride=128, h_stride=128)
        d.update(kw)
        return name(lib.fq_gated_residual_norm(C.byref(fq.fq_norm(**d)), None, FAKE, None, None, FAKE, out, h, None))

    assert norm() == "FQ_ERR_NULL"     # x: checked after the strides
    assert norm(residual_out_stride=0) == norm(h_stride=127) == "FQ_ERR_SHAPE"
    assert norm(out=None, residual_out_stride=0) == norm(rows=1, h_stride=0) == "FQ_ERR_NULL"
