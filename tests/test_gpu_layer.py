"""The operators around the matmuls on the GPU against the float64 oracle: paged KV
cache (written, read back), attention over it, gated residual norms.

Tolerances, all elementwise, from the formats and the order of the operations:
* A result rounded once to bf16 is off by up to half a unit in the last place of its
  8 bits, 2^-8 of it.
* Attention rounds each softmax weight (times V's scale) to bf16, 2^-8 relative, so a
  row is off by up to 2^-8 sum w |v| more.  Scores are fp32 sums of D products of
  magnitude sum |q||k| scale (with codes: of s (c + z + 128) instead of |k|), off by
  d <= (D + 8) 2^-24 of that; a weight then by a factor e^(2 d).  The sums of p v are
  fp32 sums of the codes' magnitude as well; 64 2^-24 of it covers their tree.
* The norm's fp32 steps stay within 2^-20 of the sum of magnitudes.
Codes, scales, zero-points and values read back in fp32 are exact.
"""

import numpy as np
import pytest
import torch

from oracle import layer as L

pytestmark = pytest.mark.gpu

KINDS = ("bf16", "int8", "int4")
B8 = 2.0 ** -8


def log(msg):
    print(msg, flush=True)


def rand_bf16(shape, seed, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + shift).to(torch.bfloat16)


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def make_cache(fq, kind, n_pages, page, heads, D, order="hnd", fill="nan"):
    """A cache whose unwritten places hold garbage: NaN rows (bf16), NaN scales (codes)."""
    row, dt = (D // 2, torch.uint8) if kind == "int4" else (D, torch.uint8 if kind == "int8" else torch.bfloat16)
    bad = float("nan") if kind == "bf16" else 0xA5

    def pool(last, dtype, value, o):
        if o == "hnd":
            return torch.full((n_pages, heads, page, last), value, dtype=dtype, device="cuda")
        if o == "nhd":
            return torch.full((n_pages, page, heads, last), value, dtype=dtype, device="cuda").transpose(1, 2)
        # K beside V in one pool, pages further apart than they need
        return torch.full((n_pages, 2, heads, page, last), value, dtype=dtype, device="cuda")

    if order == "paired":
        kv = pool(row, dt, bad, order)
        k, v = kv[:, 0], kv[:, 1]
    else:
        k, v = pool(row, dt, bad, order), pool(row, dt, bad, order)
    if kind == "bf16":
        return fq.KVCache(k, v, kind=kind)
    km, vm = pool(2, torch.bfloat16, float("nan"), "hnd"), pool(2, torch.bfloat16, float("nan"), "hnd")
    return fq.KVCache(k, v, km, vm, kind=kind)


def codes_of(cache, slots):
    """Codes, scales and zero-points that the cache holds at `slots`, K and V."""
    page, off = slots // cache.page_size, slots % cache.page_size
    out = []
    for rows, meta in ((cache.k, cache.k_meta), (cache.v, cache.v_meta)):
        c = rows.cpu()[page, :, off]
        if cache.kind == "int4":
            c = torch.stack((c & 15, c >> 4), -1).flatten(-2)
        m = meta.cpu()[page, :, off].to(torch.float64).numpy()
        out.append((c.numpy().astype(np.float64), m[..., :1], m[..., 1:]))
    return out


# ------------------------------------------------------------------- cache --

@pytest.mark.parametrize("order", ["hnd", "nhd", "paired"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", KINDS)
def test_cache_write_and_read(gpu_lib, kind, D, order):
    fq = gpu_lib
    heads, page, n_pages, n = 3, 48, 9, 101
    log(f"cache {kind} D={D} {order}")
    cache = make_cache(fq, kind, n_pages, page, heads, D, order)
    # columns of a wider matrix, as the qkv product gives them
    wide = rand_bf16((n, 5 * heads * D), 7, 2.0).cuda()
    k = wide[:, heads * D:2 * heads * D].unflatten(1, (heads, D))
    v = wide[:, 3 * heads * D:4 * heads * D].unflatten(1, (heads, D))
    k[5, 1] = 0                                       # a row of zeros
    k[6, 0] = 1.5                                     # one value all over
    v[7, 2] = -0.25
    k[8] *= 2.0 ** -120                               # near the smallest scales
    v[9] *= 2.0 ** 100
    k[10, 1, 3] = float("inf")                        # rows that no code can hold
    v[11, 0, D - 1] = float("nan")
    k[12, 2, 0], k[12, 2, 1] = 3e38, -3e38
    k[13, 0] = torch.arange(D).to(torch.bfloat16).cuda()   # span / top on a boundary, ties
    v[13, 0] = (torch.arange(D) % 31 * 0.5).to(torch.bfloat16).cuda()
    g = torch.Generator().manual_seed(3)
    slots = torch.randperm(n_pages * page, generator=g)[:n]
    slots[20], slots[21] = -1, n_pages * page         # not stored
    keep = np.ones(n, bool)
    keep[[20, 21]] = False
    before = cache.k.clone()
    fq.fq_kv_cache_write(cache, k, v, slots.cuda())
    torch.cuda.synchronize()
    src = [f64(k), f64(v)]
    if kind != "bf16":
        for (c, s, z), x in zip(codes_of(cache, slots[torch.from_numpy(keep)]), src):
            ec, es, ez = L.quantise_rows(x[keep], kind)
            np.testing.assert_array_equal(s, es)
            ok = ~np.isnan(es[..., 0])
            np.testing.assert_array_equal(z[ok], ez[ok])
            np.testing.assert_array_equal(c[ok], ec[ok])
    untouched = np.ones(n_pages * page, bool)
    untouched[slots[torch.from_numpy(keep)].numpy()] = False
    a, b = (t.transpose(1, 2).reshape(n_pages * page, -1).view(torch.uint8).cpu().numpy()[untouched]
            for t in (before.contiguous(), cache.k.contiguous()))
    np.testing.assert_array_equal(a, b)
    for dtype in ("f32", "bf16"):
        got = fq.fq_kv_cache_read(cache, slots.cuda(), dtype=dtype)
        for y, x in zip(got, src):
            assert y.shape == (n, heads, D)
            y = y.cpu()
            assert (y[[20, 21]] == 0).all()
            want = torch.from_numpy(L.held_rows(x, kind)).to(torch.float32)
            if dtype == "bf16":
                want = want.to(torch.bfloat16)
            want[[20, 21]] = 0
            np.testing.assert_array_equal(y.float().numpy(), want.float().numpy())


@pytest.mark.parametrize("page,n_pages", [(16, 400), (592, 11), (4112, 3), (65536, 2)])
@pytest.mark.parametrize("kind", ["int8", "int4"])
def test_cache_codes_over_sizes(gpu_lib, kind, page, n_pages):
    """Scales, zero-points and codes of rows of all sizes, those at the ends of the quick
    division's range (spans of 2^-90 and 2^90) among them, are exact; pages of any size."""
    fq = gpu_lib
    heads, D, n = 2, 64, 1500
    log(f"cache sizes {kind} page={page}")
    cache = make_cache(fq, kind, n_pages, page, heads, D, "hnd")
    g = torch.Generator().manual_seed(page)
    k, v = (rand_bf16((n, heads, D), page + i, 1.0) for i in (1, 2))
    e = torch.randint(-124, 118, (n,), generator=g)
    e[:40] = torch.arange(40) % 8 - 94
    e[40:80] = torch.arange(40) % 8 + 84
    k = (k.double() * torch.exp2(e.double())[:, None, None]).to(torch.bfloat16)
    k[100:200, :, 1:] = 0                                  # one value, on either side of 0
    v[200:300] = v[200:300].abs()                          # nothing below 0
    v[300:400] = -v[300:400].abs()
    v[400:500] = (torch.randint(-255, 256, (100, heads, D), generator=g) / 2).to(torch.bfloat16)   # ties
    slots = torch.randperm(n_pages * page, generator=g)[:n]
    slots[0] = n_pages * page - 1
    slots = slots.unique()
    k, v = k[:len(slots)], v[:len(slots)]
    fq.fq_kv_cache_write(cache, k.cuda(), v.cuda(), slots.cuda())
    torch.cuda.synchronize()
    for (c, s, z), x in zip(codes_of(cache, slots), (f64(k), f64(v))):
        ec, es, ez = L.quantise_rows(x, kind)
        np.testing.assert_array_equal(s, es)
        np.testing.assert_array_equal(z, ez)
        np.testing.assert_array_equal(c, ec)


def test_cache_of_no_and_one_token_and_repeats(gpu_lib):
    fq = gpu_lib
    cache = make_cache(fq, "int8", 2, 16, 1, 128)
    empty = torch.empty((0, 1, 128), dtype=torch.bfloat16, device="cuda")
    none = torch.empty((0,), dtype=torch.int64, device="cuda")
    fq.fq_kv_cache_write(cache, empty, empty, none)
    k, v = fq.fq_kv_cache_read(cache, none)
    assert k.shape == v.shape == (0, 1, 128)
    x = rand_bf16((1, 1, 128), 5).cuda()
    fq.fq_kv_cache_write(cache, x, -x, torch.tensor([31], device="cuda"))
    k, v = fq.fq_kv_cache_read(cache, torch.tensor([31, 31, -5, 31], device="cuda"), dtype="f32")
    want = L.held_rows(f64(x), "int8")[0]
    for i in (0, 1, 3):
        np.testing.assert_array_equal(k[i].cpu().numpy(), want.astype(np.float32))
    assert (k[2] == 0).all() and (v[2] == 0).all()
    np.testing.assert_array_equal(v[0].cpu().numpy(), L.held_rows(-f64(x), "int8")[0].astype(np.float32))


# --------------------------------------------------------------- attention --

class Step:
    """Sequences with random K and V in a cache with garbage elsewhere."""

    def __init__(self, fq, kind, D, hq, hkv, page, q_lens, kv_lens, seed, order="hnd", spare=2, max_q=None,
                 max_kv=None, k_scale=1.0, edit=None):
        self.fq, self.kind, self.D, self.hq, self.hkv = fq, kind, D, hq, hkv
        self.q_lens, self.kv_lens = q_lens, kv_lens
        need = [-(-n // page) for n in kv_lens]
        n_pages = sum(need) + spare
        self.cache = make_cache(fq, kind, n_pages, page, hkv, D, order)
        g = torch.Generator().manual_seed(seed)
        perm = torch.randperm(n_pages, generator=g)
        cols = max(need + [1]) + 1
        # the last column and unused entries are no pages at all
        self.table = torch.full((len(q_lens), cols), -1, dtype=torch.int32)
        at, ks, vs, slots = 0, [], [], []
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            t = torch.arange(kv_lens[b])
            slots.append(perm[at:at + n][t // page] * page + t % page)
            at += n
            ks.append(rand_bf16((kv_lens[b], hkv, D), seed + 10 * b + 1, k_scale, 0.1))
            vs.append(rand_bf16((kv_lens[b], hkv, D), seed + 10 * b + 2, 1.0, 0.3))
            if edit is not None:
                edit(b, ks[-1], vs[-1])
        self.k, self.v = ks, vs
        if sum(kv_lens):
            fq.fq_kv_cache_write(self.cache, torch.cat(ks).cuda(), torch.cat(vs).cuda(), torch.cat(slots).cuda())
        T = sum(q_lens)
        wide = rand_bf16((T, (hq + 2) * D), seed + 5).cuda()
        self.q = wide[:, D:(hq + 1) * D].unflatten(1, (hq, D))
        cu = np.concatenate([[0], np.cumsum(q_lens)])
        self.cu = cu
        self.batch = fq.PagedBatch(torch.tensor(cu, dtype=torch.int32).cuda(),
                                   torch.tensor(kv_lens, dtype=torch.int32).cuda(), self.table.cuda(),
                                   max_q or max(q_lens), max_kv or max(max(kv_lens), 1))

    def check(self, out, lse, window, sinks, scale=None, rows=None):
        scale = 1.0 / np.sqrt(self.D) if scale is None else scale
        scale = float(np.float32(scale))
        out, q, G = f64(out), f64(self.q), self.hq // self.hkv
        lse = None if lse is None else f64(lse)
        rng = np.random.default_rng(1)
        for b, (n, S) in enumerate(zip(self.q_lens, self.kv_lens)):
            if n == 0:
                continue
            held, size = [], []
            for x in (self.k[b], self.v[b]):
                x = f64(x)
                if self.kind == "bf16":
                    held.append(x)
                    size.append(np.abs(x))
                else:
                    c, s, z = L.quantise_rows(x, self.kind)
                    held.append(s * (c - z))
                    size.append(s * (c + z + 128))
            tokens = range(n) if rows is None or n <= rows else \
                sorted(set([0, 1, n - 2, n - 1]) | set(rng.choice(n, rows, replace=False).tolist()))
            for i in tokens:
                see = L.visible(S - n + i, S, window, sinks)
                t = self.cu[b] + i
                for h in range(self.hq):
                    o, e, A, _ = L.attention_row(q[t, h], held[0][:, h // G], held[1][:, h // G], see, scale)
                    where = f"sequence {b} token {i} head {h}"
                    if see.any() and np.isfinite(e):
                        big = (size[0][see, h // G] @ np.abs(q[t, h])).max() * abs(scale)
                        d = (self.D + 8) * 2.0 ** -24 * big
                        S_v = size[1][see, h // G].max(0) if self.kind != "bf16" else A
                        tol = B8 * 1.05 * np.abs(o) + (B8 * 1.05 + 2.5 * d) * A + 64 * 2.0 ** -24 * S_v + 1e-30
                    else:
                        d, tol = 0.0, np.zeros_like(o)
                    err = np.abs(out[t, h] - o)
                    assert (err <= tol).all(), (where, float((err - tol).max()), np.flatnonzero(err > tol)[:4])
                    if lse is not None:
                        if np.isfinite(e):
                            assert abs(lse[t, h] - e) <= d + 2.0 ** -20 * (1 + abs(e)), (where, lse[t, h], e)
                        else:
                            assert lse[t, h] == e, where


# (query heads, KV heads, page, new tokens, whole lengths, window, sinks)
STEPS = {
    "one_token_one_key": (4, 4, 16, [1], [1], 0, 0),
    "decode_ragged": (8, 2, 16, [1, 1, 1, 1, 1], [1, 31, 32, 33, 200], 0, 0),
    "no_keys": (4, 2, 16, [1, 1, 2], [0, 5, 0], 0, 0),
    "more_tokens_than_keys": (4, 2, 16, [5, 3], [2, 3], 0, 0),
    "no_tokens_of_a_sequence": (4, 2, 32, [0, 2, 0], [40, 40, 0], 0, 0),
    "mha_chunk": (2, 2, 16, [37], [70], 0, 0),
    "gqa_chunk_from_zero": (8, 2, 48, [50], [50], 0, 0),
    "group_of_three": (6, 2, 16, [11, 7], [43, 90], 0, 0),
    "group_of_24": (24, 1, 16, [3], [77], 0, 0),
    "window": (4, 2, 16, [1, 9, 40], [100, 64, 41], 17, 0),
    "window_and_sinks": (4, 2, 16, [1, 9, 40], [300, 164, 141], 17, 4),
    "window_of_one": (4, 2, 16, [3], [70], 1, 0),
    "window_of_one_far_sinks": (4, 2, 16, [3], [150], 1, 40),
    "sinks_reach_the_window": (4, 2, 16, [20], [90], 30, 64),
    "window_wider_than_all": (4, 1, 32, [4, 1], [60, 9], 1000, 3),
    "long_window": (8, 2, 64, [2], [1500], 500, 33),
    "mixed": (8, 2, 32, [1, 70, 5], [333, 170, 5], 0, 0),
}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(STEPS))
def test_attention(gpu_lib, name, kind, D):
    fq = gpu_lib
    hq, hkv, page, q_lens, kv_lens, window, sinks = STEPS[name]
    log(f"attention {name} {kind} D={D}")
    st = Step(fq, kind, D, hq, hkv, page, q_lens, kv_lens, seed=len(name) + D)
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, window=window, sinks=sinks, return_lse=True)
    torch.cuda.synchronize()
    st.check(out, lse, window, sinks)


def tiles_bounds(st, window=0, sinks=0, by_keys=False):
    """Raises the step's bounds of the new tokens, or of the keys, until the kernel for many
    rows is the one to run; returns the launch."""
    q, kv, b = st.batch.max_q, st.batch.max_kv, st.batch
    while True:
        if by_keys:
            kv *= 2
        else:
            q *= 2
        cols = -(-kv // st.cache.page_size)
        table = torch.full((len(st.q_lens), max(cols, st.table.shape[1])), -1, dtype=torch.int32)
        table[:, :st.table.shape[1]] = st.table
        st.batch = st.fq.PagedBatch(b.cu_q, b.kv_lens, table.cuda(), q, kv)
        c = st.fq.fq_paged_attention_launch(st.hq, sum(st.q_lens), st.cache, st.batch, window=window, sinks=sinks)
        if c["kernel"] == "tiles":
            return c


# (query heads, KV heads, page, new tokens, whole lengths, window, sinks)
MANY = {
    "chunk_on_a_prefix": (8, 2, 16, [90], [400], 0, 0),
    "prompts_from_zero": (4, 1, 48, [64, 130, 1], [64, 130, 1], 0, 0),
    "mixed_with_decoding": (8, 2, 64, [1, 120, 33], [500, 260, 33], 0, 0),
    "window": (4, 2, 16, [130, 60], [300, 60], 50, 0),
    "window_and_sinks": (8, 2, 32, [100, 1, 40], [420, 700, 41], 70, 5),
    "window_of_one": (4, 2, 16, [70], [190], 1, 0),
    "far_sinks": (4, 2, 16, [70], [500], 30, 129),
    "more_tokens_than_keys": (8, 4, 16, [100, 70], [40, 0], 0, 0),
    "mha": (2, 2, 16, [140], [300], 0, 0),
    "group_of_three": (6, 2, 16, [45, 80], [100, 200], 0, 0),
    "split_prefix": (4, 1, 16, [40], [3000], 0, 0),
    "split_ragged": (8, 2, 16, [40, 1, 64], [2500, 900, 64], 0, 0),
    "split_window": (4, 1, 64, [64], [2600], 1500, 70),
}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(MANY))
def test_attention_many_rows(gpu_lib, name, kind, D):
    """The kernel for many rows, and the join of its ranges."""
    fq = gpu_lib
    hq, hkv, page, q_lens, kv_lens, window, sinks = MANY[name]
    st = Step(fq, kind, D, hq, hkv, page, q_lens, kv_lens, seed=3 * len(name) + D)
    c = tiles_bounds(st, window, sinks, by_keys=name.startswith("split") and not window)
    log(f"attention {name} {kind} D={D} {c}")
    assert c["kernel"] == "tiles"
    assert c["split"] > 1 or not name.startswith("split")
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, window=window, sinks=sinks, return_lse=True)
    torch.cuda.synchronize()
    st.check(out, lse, window, sinks, rows=24)
    again = fq.fq_paged_attention(st.q, st.cache, st.batch, window=window, sinks=sinks)
    assert torch.equal(again, out)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("q_lens,kv_lens", [([2, 1], [300, 40]), ([60], [140])], ids=["rows", "tiles"])
@pytest.mark.parametrize("scale", [-0.07, 0.0, 1e-30])
def test_attention_scales(gpu_lib, scale, q_lens, kv_lens, kind):
    """A scale that is negative, zero (the mean of the values) or next to it."""
    fq = gpu_lib
    st = Step(fq, kind, 128, 4, 2, 16, q_lens, kv_lens, seed=17)
    if len(q_lens) == 1:
        tiles_bounds(st)
    log(f"attention scale {scale} {kind}")
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, scale=scale, return_lse=True)
    torch.cuda.synchronize()
    st.check(out, lse, 0, 0, scale=scale, rows=12)


def test_attention_kernel_by_rows_and_bytes(gpu_lib):
    """Up to 32 rows the kernel for few; above by what the blocks of 16 rows read."""
    fq = gpu_lib
    small = make_cache(fq, "int4", 4, 16, 8, 128)
    i32 = dict(dtype=torch.int32, device="cuda")

    def kernel(max_q, max_kv, n_seqs):
        b = fq.PagedBatch(torch.zeros(n_seqs + 1, **i32), torch.zeros(n_seqs, **i32), torch.zeros((n_seqs, 4096), **i32),
                          max_q, max_kv)
        return fq.fq_paged_attention_launch(32, 100, small, b)["kernel"]

    assert kernel(8, 65536, 64) == "rows" and kernel(9, 65536, 64) == "tiles"
    assert kernel(20, 8000, 1) == "rows" and kernel(20, 8000, 8) == "tiles"


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [5000, 1234]), ([4], [9001]), ([100], [3000])],
                         ids=["decode", "draft", "chunk"])
def test_attention_split_over_the_keys(gpu_lib, kind, q_lens, kv_lens):
    """Long keys and few rows: ranges joined by the last workgroup, the same bits each
    time, the counters back at zero (a second call on the same workspace)."""
    fq = gpu_lib
    st = Step(fq, kind, 128, 8, 2, 64, q_lens, kv_lens, seed=9)
    c = fq.fq_paged_attention_launch(8, sum(q_lens), st.cache, st.batch)
    log(f"attention split {kind} {q_lens} {kv_lens} {c}")
    assert c["split"] > 1
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, return_lse=True)
    torch.cuda.synchronize()
    st.check(out, lse, 0, 0, rows=6)
    for _ in range(3):
        again = fq.fq_paged_attention(st.q, st.cache, st.batch)
        assert torch.equal(again, out)


@pytest.mark.parametrize("order", ["nhd", "paired"])
@pytest.mark.parametrize("kind", KINDS)
def test_attention_orders_and_output_strides(gpu_lib, kind, order):
    fq = gpu_lib
    st = Step(fq, kind, 128, 4, 2, 16, [1, 30], [77, 64], seed=4, order=order)
    log(f"attention {order} {kind}")
    buf = torch.full((31, 6, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[:, 1:5, 8:]
    got = fq.fq_paged_attention(st.q, st.cache, st.batch, out=out, scale=0.25)
    torch.cuda.synchronize()
    assert got.data_ptr() == out.data_ptr()
    st.check(out, None, 0, 0, scale=0.25)
    assert (buf[:, 0] == 7).all() and (buf[:, 5] == 7).all() and (buf[:, :, :8] == 7).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tiles", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("q", [4, 60], ids=["few", "many"])
def test_attention_unseen_infinities_and_nan(gpu_lib, kind, q, tiles):
    """Keys that some tokens see and others do not hold infinities and NaN in K and V:
    only the rows of the former may show them."""
    fq = gpu_lib
    S, D = 130, 128
    bad = S - 2                                   # seen by the last two tokens only

    def edit(b, k, v):
        k[bad, 0, 5] = float("nan")
        v[bad, 1, 7] = float("inf")
        v[bad, 1, 8] = float("-inf")
        v[bad, 1, 9] = float("nan")

    st = Step(fq, kind, D, 4, 2, 16, [q], [S], seed=3, edit=edit)
    if tiles:
        tiles_bounds(st, by_keys=q > 50)
    log(f"attention unseen NaN {kind} q={q} tiles={tiles}")
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, return_lse=True)
    torch.cuda.synchronize()
    o, e = f64(out), f64(lse)
    assert np.isfinite(o[:q - 2]).all() and np.isfinite(e[:q - 2]).all()
    for t in (q - 2, q - 1):
        assert np.isnan(o[t, :2]).all() and np.isnan(e[t, :2]).all()        # K's NaN: KV head 0
        if kind == "bf16":
            assert np.isfinite(e[t, 2:]).all()
            for h in (2, 3):
                assert o[t, h, 7] == np.inf and o[t, h, 8] == -np.inf and np.isnan(o[t, h, 9])
                assert np.isfinite(np.delete(o[t, h], [7, 8, 9])).all()
        else:
            assert np.isnan(o[t, 2:]).all()       # a row that no code can hold reads as NaN
    # the other rows are those of a cache without them
    clean = Step(fq, kind, D, 4, 2, 16, [q], [S], seed=3)
    if tiles:
        tiles_bounds(clean, by_keys=q > 50)
    want = fq.fq_paged_attention(clean.q, clean.cache, clean.batch)
    assert torch.equal(out[:q - 2], want[:q - 2])


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_attention_nan_left_behind_by_the_window(gpu_lib, kind):
    fq = gpu_lib

    def edit(b, k, v):
        k[60], v[60] = float("nan"), float("inf")

    st = Step(fq, kind, 128, 4, 2, 16, [8], [96], seed=6, edit=edit)   # positions 88 .. 95
    log(f"attention NaN behind the window {kind}")
    out = fq.fq_paged_attention(st.q, st.cache, st.batch, window=32, sinks=3)
    torch.cuda.synchronize()
    o = f64(out)
    for t in range(8):
        sees = 60 > 88 + t - 32
        assert np.isnan(o[t]).all() if sees else np.isfinite(o[t]).all(), t


def test_attention_extreme_scores(gpu_lib):
    """Scores of +-1e4 (one key takes all) and rows whose every score is -infinity."""
    fq = gpu_lib
    st = Step(fq, "bf16", 128, 4, 2, 16, [3, 2], [70, 33], seed=8, k_scale=100.0)
    log("attention extreme scores")
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, scale=10.0, return_lse=True)
    torch.cuda.synchronize()
    st.check(out, lse, 0, 0, scale=10.0)

    def edit(b, k, v):
        k[:] = float("-inf")

    st = Step(fq, "bf16", 128, 2, 2, 16, [1], [40], seed=8, edit=edit)
    st.q.fill_(1.0)
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, return_lse=True)
    assert (out == 0).all() and (lse == float("-inf")).all()


def test_attention_bounds_above_the_lengths(gpu_lib):
    """max_q and max_kv are bounds: larger ones change nothing but the kernel, the split and
    with them the rounding; tokens beyond max_q are left alone."""
    fq = gpu_lib
    st = Step(fq, "int8", 128, 8, 2, 16, [1, 3], [100, 50], seed=2)
    wide = torch.full((2, 4096), -1, dtype=torch.int32)
    wide[:, :st.table.shape[1]] = st.table
    big = fq.PagedBatch(st.batch.cu_q, st.batch.kv_lens, wide.cuda(), 64, 65536)
    log(f"attention bounds {fq.fq_paged_attention_launch(8, 4, st.cache, big)}")
    out, lse = fq.fq_paged_attention(st.q, st.cache, big, return_lse=True)
    torch.cuda.synchronize()
    st.check(out, lse, 0, 0)
    small = fq.PagedBatch(st.batch.cu_q, st.batch.kv_lens, st.batch.block_table, 2, 100)
    keep = torch.full_like(out, 9.0)
    fq.fq_paged_attention(st.q, st.cache, small, out=keep)
    torch.cuda.synchronize()
    assert (keep[3] == 9).all()
    st.check(torch.cat([keep[:3], out[3:]]), None, 0, 0)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("window", [1 << 30, 2**31 - 1])
def test_attention_widest_windows(gpu_lib, window, kind):
    """Windows at the end of their type see what no window sees, with tokens before the first
    key in the same wave as others."""
    fq = gpu_lib
    st = Step(fq, kind, 128, 2, 2, 16, [140, 20], [130, 5], seed=21)
    c = tiles_bounds(st, window)
    log(f"attention window {window} {kind} {c}")
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, window=window, return_lse=True)
    torch.cuda.synchronize()
    st.check(out, lse, 0, 0)


def test_attention_offsets_beyond_32_bits(gpu_lib):
    """Pages that start beyond 4 GiB of the pool, and slots there."""
    fq = gpu_lib
    n_pages, page, D = 80000, 64, 128          # 80000 x 64 KiB per K and V: 5.2 GB each
    k = torch.empty((n_pages, 4, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    cache = fq.KVCache(k, v)
    table = torch.tensor([[n_pages - 1, 3, n_pages - 2]], dtype=torch.int32)
    S = 150
    t = torch.arange(S)
    slots = (table[0].long()[t // page] * page + t % page).cuda()
    x, y = rand_bf16((S, 4, D), 1).cuda(), rand_bf16((S, 4, D), 2).cuda()
    log("attention beyond 32 bits")
    fq.fq_kv_cache_write(cache, x, y, slots)
    a, b = fq.fq_kv_cache_read(cache, slots)
    assert torch.equal(a, x) and torch.equal(b, y)
    st = Step(fq, "bf16", D, 4, 4, page, [2], [S], seed=1)
    st.cache, st.k, st.v = cache, [x.cpu()], [y.cpu()]
    batch = fq.PagedBatch(st.batch.cu_q, st.batch.kv_lens, table.cuda(), 2, S)
    out, lse = fq.fq_paged_attention(st.q, cache, batch, return_lse=True)
    torch.cuda.synchronize()
    st.check(out, lse, 0, 0)


# ------------------------------------------------------------------- norms --

def _norm_inputs(M, H, xt, rt, post, gate, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, H), generator=g).to(xt)
    res = None if rt is None else (3 * torch.randn((M, H), generator=g)).to(rt)
    w = lambda: (1 + 0.3 * torch.randn((H,), generator=g)).to(torch.bfloat16)   # noqa: E731
    gt = {"none": None, "channel": torch.rand((H,), generator=g), "row": torch.rand((M, H), generator=g)}[gate]
    return x, res, w(), w() if post else None, None if gt is None else gt.to(torch.bfloat16)


def _check_norm(got, x, res, pre, post, gate, alpha, eps, rt):
    n64 = lambda t: None if t is None else f64(t)   # noqa: E731
    r, h, mag = L.gated_residual_norm(n64(x), n64(res), n64(pre), n64(post), n64(gate), alpha, eps)
    E = 2.0 ** -20
    tol_r = E * mag + (B8 * np.abs(r) if rt == torch.bfloat16 else 0) + 1e-38
    assert (np.abs(f64(got[0]) - r) <= tol_r).all()
    if pre is not None:
        # the row's rms is off by no more than its largest relative share
        rms = np.sqrt((r * r).mean(-1, keepdims=True) + eps)
        share = E * (np.sqrt((mag * mag).mean(-1, keepdims=True)) / rms + 1)
        tol_h = (B8 + share) * np.abs(h) + E * mag / rms * np.abs(f64(pre)) + 1e-38
        assert (np.abs(f64(got[1]) - h) <= tol_h).all()


@pytest.mark.parametrize("H", [1, 7, 8, 64, 130, 512, 1000, 1024, 1032, 2048, 4096, 4099, 8192, 10240, 16384, 32768])
@pytest.mark.parametrize("M", [1, 5])
def test_norm_sizes(gpu_lib, M, H):
    fq = gpu_lib
    log(f"norm {M} x {H}")
    x, res, pre, post, gate = _norm_inputs(M, H, torch.bfloat16, torch.bfloat16, True, "row", H + M)
    dev = [None if t is None else t.cuda() for t in (x, res, pre, post, gate)]
    got = fq.fq_gated_residual_norm(dev[0], dev[1], dev[2], post_weight=dev[3], gate=dev[4], residual_scale=0.5)
    torch.cuda.synchronize()
    _check_norm(got, x, res, pre, post, gate, 0.5, 1e-5, torch.bfloat16)


@pytest.mark.parametrize("gate", ["none", "channel", "row"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("xt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rt", [None, torch.bfloat16, torch.float32])
def test_norm_types(gpu_lib, rt, xt, post, gate):
    fq = gpu_lib
    M, H = 9, 1000
    log(f"norm types {rt} {xt} {post} {gate}")
    x, res, pre, post_w, gt = _norm_inputs(M, H, xt, rt, post, gate, 5)
    dev = [None if t is None else t.cuda() for t in (x, res, pre, post_w, gt)]
    got = fq.fq_gated_residual_norm(dev[0], dev[1], dev[2], post_weight=dev[3], gate=dev[4], residual_scale=0.75,
                                    eps=1e-3)
    torch.cuda.synchronize()
    out_t = xt if rt is None else rt
    assert got[0].dtype == out_t and got[1].dtype == torch.bfloat16
    _check_norm(got, x, res, pre, post_w, gt, 0.75, 1e-3, out_t)
    only = fq.fq_gated_residual_norm(dev[0], dev[1], post_weight=dev[3], gate=dev[4], residual_scale=0.75, eps=1e-3)
    assert only[1] is None and torch.equal(only[0], got[0])


def test_norm_in_place_strided_and_misaligned(gpu_lib):
    """residual_out = residual; rows of wider matrices that start at odd elements."""
    fq = gpu_lib
    M, H = 6, 520
    log("norm strided")
    x, res, pre, post, gate = _norm_inputs(M, H, torch.bfloat16, torch.bfloat16, True, "row", 3)

    def inside(t, off, width):
        big = torch.full((M, width), 5.0, dtype=t.dtype, device="cuda")
        big[:, off:off + H] = t.cuda()
        return big, big[:, off:off + H]

    _, xs = inside(x, 1, H + 3)
    big, rs = inside(res, 3, H + 7)
    _, gs = inside(gate, 5, H + 11)
    hb = torch.full((M, H + 9), 5.0, dtype=torch.bfloat16, device="cuda")
    hs = hb[:, 7:7 + H]
    got = fq.fq_gated_residual_norm(xs, rs, pre.cuda(), post_weight=post.cuda(), gate=gs, residual_out=rs, h=hs)
    torch.cuda.synchronize()
    assert got[0].data_ptr() == rs.data_ptr() and got[1].data_ptr() == hs.data_ptr()
    _check_norm((rs, hs), x, res, pre, post, gate, 1.0, 1e-5, torch.bfloat16)
    assert (big[:, :3] == 5).all() and (big[:, 3 + H:] == 5).all()
    assert (hb[:, :7] == 5).all() and (hb[:, 7 + H:] == 5).all()


def test_norm_special_rows(gpu_lib):
    """Zeros, infinities and NaN stay in their rows; large values do not overflow where the
    formula in fp32 does not."""
    fq = gpu_lib
    M, H = 8, 256
    x = rand_bf16((M, H), 1).cuda()
    res = rand_bf16((M, H), 2).cuda()
    w = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    x[1], res[1] = 0, 0
    x[2, 3] = float("nan")
    x[3, 200] = float("inf")
    x[4] *= 1e15
    r, h = fq.fq_gated_residual_norm(x, res, w)
    torch.cuda.synchronize()
    assert (r[1] == 0).all() and (h[1] == 0).all()
    assert torch.isnan(h[2]).all() and torch.isnan(r[2, 3]) and torch.isfinite(r[2, :3]).all()
    assert r[3, 200] == float("inf")
    for i in (0, 4, 5, 6, 7):
        assert torch.isfinite(h[i]).all()
    empty = torch.empty((0, H), dtype=torch.bfloat16, device="cuda")
    r, h = fq.fq_gated_residual_norm(empty, empty, w)
    assert r.shape == h.shape == (0, H)


# ------------------------------------------------------- streams and graphs --

def test_layer_operators_on_another_stream(gpu_lib):
    """Calls given a stream run there: behind work of that stream that they depend on."""
    fq = gpu_lib
    st = Step(fq, "int4", 128, 8, 2, 64, [1, 1], [4000, 77], seed=12)
    want = fq.fq_paged_attention(st.q, st.cache, st.batch)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    log("layer operators on a side stream")
    x = torch.randn((64, 4096), device="cuda").to(torch.bfloat16)
    w = torch.ones(4096, dtype=torch.bfloat16, device="cuda")
    q2 = torch.zeros_like(st.q)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.mm(x, x.t().contiguous())        # keeps the stream busy
        q2.copy_(st.q)
    out = fq.fq_paged_attention(q2, st.cache, st.batch, stream=side)
    r, h = fq.fq_gated_residual_norm(x, x, w, stream=side)
    k, v = fq.fq_kv_cache_read(st.cache, torch.arange(64, device="cuda"), stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    assert torch.equal(r, fq.fq_gated_residual_norm(x, x, w)[0])


@pytest.mark.parametrize("kind", KINDS)
def test_layer_operators_in_a_graph(gpu_lib, kind):
    """Write, attend and norm captured once and replayed with other contents, eager work in
    between: every replay equals the eager calls."""
    fq = gpu_lib
    st = Step(fq, kind, 128, 8, 2, 64, [1, 1, 1], [3000, 64, 700], seed=21)
    T, H = 3, 1024
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    lens = st.batch.kv_lens
    k_new, v_new = rand_bf16((T, 2, 128), 31).cuda(), rand_bf16((T, 2, 128), 32).cuda()
    page = st.cache.page_size
    slots = torch.zeros(T, dtype=torch.int64, device="cuda")
    res = rand_bf16((T, H), 33).cuda()
    w = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    out, out_e = (torch.empty((T, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    r, h = torch.empty_like(res), torch.empty_like(res)
    log(f"layer graph {kind}")

    def step(o):
        fq.fq_kv_cache_write(st.cache, k_new, v_new, slots)
        fq.fq_paged_attention(st.q, st.cache, st.batch, out=o, ws=ws)
        fq.fq_gated_residual_norm(o.view(T, H), res, w, residual_out=r, h=h)

    def place(shorter):
        n = torch.tensor([3000, 64, 700], dtype=torch.int32) - shorter
        lens.copy_(n)
        last = (n - 1).long()
        slots.copy_(st.table[torch.arange(T), last // page].long() * page + last % page)

    place(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out)
    for i in range(4):
        place(13 * i)
        k_new.copy_(rand_bf16((T, 2, 128), 40 + i))
        step(out_e)
        eager = [t.clone() for t in (out_e, r, h)]
        torch.cuda.synchronize()
        for t in (out, r, h):
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip((out, r, h), eager):
            assert torch.equal(a, b), f"replay {i}"
