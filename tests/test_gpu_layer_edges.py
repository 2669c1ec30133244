"""The cache and attention on the GPU where contents or arguments are unusual, against the
float64 oracle.

Tolerances, elementwise, from the formats and the order of the operations:
* One rounding to bf16: 2^-8 of the value (7 bits follow the leading one); the softmax weights
  (times V's scale) are rounded so too, which moves a row by 2^-8 sum w |v| at most.
* Scores: fp32 sums of D products and, with codes, of D numbers times the zero-point, of
  magnitude |q| s (c + |z|) (4 bits: 16 + c in one kernel), each addition off by 2^-23 at most
  (the matrix instructions need not round to nearest); d of the row's largest such sum moves
  a weight by a factor of up to e^(2 d), and with it a row by 2.5 d sum w |v|.
* The sums of n weights times codes: n additions of magnitude max s (c + |z|) at most, 2^-23 each.
* The log-sum: d, and 2^-20 of it and of 1 for the exponentials and the logarithm.
"""

import numpy as np
import pytest
import torch

from oracle import layer as L
from test_gpu_layer import MANY, STEPS, Step, codes_of, f64, log, tiles_bounds

pytestmark = pytest.mark.gpu


def check_rows(out, lse, q, cu, held, size, q_lens, kv_lens, D, scale, window=0, sinks=0, every=1, unit=2 * 2.0 ** -23):
    """out, lse of each sequence's every `every`-th token against attention over `held`
    (K, V by sequence, [keys][heads][D]), whose summands have the magnitudes `size`; unit: what
    one addition of a score is off by."""
    out, lse, q = f64(out), f64(lse), f64(q)
    hq, hkv = q.shape[1], held[0][0].shape[1]
    G = hq // hkv
    for b, (n, S) in enumerate(zip(q_lens, kv_lens)):
        for i in sorted(set(range(0, n, every)) | set(range(n)[-1:])):
            see = L.visible(S - n + i, S, window, sinks)
            t = cu[b] + i
            for h in range(hq):
                K, V = (held[x][b][:, h // G] for x in (0, 1))
                o, e, A, _ = L.attention_row(q[t, h], K, V, see, scale)
                where = f"sequence {b} token {i} head {h}"
                if not see.any():
                    assert (out[t, h] == 0).all() and lse[t, h] == -np.inf, where
                    continue
                d = (D + 8) * unit * abs(scale) * (size[0][b][see, h // G] @ np.abs(q[t, h])).max()
                tol = 2.0 ** -8 * 1.01 * np.abs(o) + (2.0 ** -8 * 1.01 + 2.5 * d) * A + \
                    see.sum() * 2.0 ** -23 * size[1][b][see, h // G].max(0) + 1e-30
                err = np.abs(out[t, h] - o)
                assert (err <= tol).all(), (where, float((err - tol).max()), np.flatnonzero(~(err <= tol))[:4])
                assert abs(lse[t, h] - e) <= d + 2.0 ** -20 * (1 + abs(e)), (where, lse[t, h], e)


def held_codes(st):
    """(K, V) that the step's cache holds by sequence, and the magnitudes of their summands."""
    held, size = ([], []), ([], [])
    page = st.cache.page_size
    for b, n in enumerate(st.kv_lens):
        t = torch.arange(n)
        slots = st.table[b].long()[t // page] * page + t % page
        for x, (c, s, z) in enumerate(codes_of(st.cache, slots)):
            held[x].append(s * (c - z))
            size[x].append(np.abs(s) * (c + np.abs(z) + (16 if st.kind == "int4" else 0)))
    return held, size


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["int8", "int4"])
@pytest.mark.parametrize("q_lens,kv_lens,window", [([3, 1], [120, 77], 0), ([70, 9], [330, 20], 0), ([70], [330], 40),
                                                   ([30], [2100], 0)],
                         ids=["rows", "tiles", "tiles_window", "tiles_split"])
def test_attention_over_any_zero_points(gpu_lib, q_lens, kv_lens, window, kind, D):
    """A row stands for s (c - z) with any bf16 z: below 0, above the codes, not whole."""
    fq = gpu_lib
    hq, hkv, page = 4, 2, 16
    st = Step(fq, kind, D, hq, hkv, page, q_lens, kv_lens, seed=31 + D)
    g = torch.Generator().manual_seed(5)
    values = torch.tensor([-3.0, 12.5, 300.0, -0.25, 0.0, 7.75, 255.0, -120.0]).to(torch.bfloat16).cuda()
    for b, n in enumerate(kv_lens):
        t = torch.arange(n)
        at, off = st.table[b].long()[t // page].cuda(), (t % page).cuda()
        for meta in (st.cache.k_meta, st.cache.v_meta):
            meta[at, :, off, 1] = values[torch.randint(0, 8, (n, hkv), generator=g).cuda()]
    if q_lens[0] > 3:
        c = tiles_bounds(st, window, by_keys=kv_lens[0] > 2000)
        assert c["kernel"] == "tiles" and (c["split"] > 1 or kv_lens[0] < 2000)
    log(f"attention zero-points {kind} D={D} {q_lens} {kv_lens} window {window}")
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, window=window, return_lse=True)
    torch.cuda.synchronize()
    held, size = held_codes(st)
    check_rows(out, lse, st.q, st.cu, held, size, q_lens, kv_lens, D, float(np.float32(D ** -0.5)), window, every=5)


@pytest.mark.parametrize("kind", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("q_lens,kv_lens", [([2, 1], [300, 40]), ([60], [140]), ([60], [2500])],
                         ids=["rows", "tiles", "tiles_split"])
@pytest.mark.parametrize("scale", [1.5e-38, 1e-38, -1e-40, 1e-45])
def test_attention_smallest_scales(gpu_lib, scale, q_lens, kv_lens, kind):
    """Scales whose inverse is beyond fp32: the mean of the values, ln of the keys."""
    fq = gpu_lib
    st = Step(fq, kind, 128, 4, 2, 16, q_lens, kv_lens, seed=19)
    if len(q_lens) == 1:
        c = tiles_bounds(st, by_keys=kv_lens[0] > 2000)
        assert c["split"] > 1 or kv_lens[0] < 2000
    log(f"attention scale {scale} {kind} {kv_lens}")
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, scale=scale, return_lse=True)
    torch.cuda.synchronize()
    held, size = rows_held([[f64(t) for t in ts] for ts in (st.k, st.v)]) if kind == "bf16" else held_codes(st)
    check_rows(out, lse, st.q, st.cu, held, size, q_lens, kv_lens, 128, float(np.float32(scale)), every=13)


@pytest.mark.parametrize("kind", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("scale", [1e38, -1e38])
@pytest.mark.parametrize("q_lens,kv_lens", [([2, 1], [300, 40]), ([60], [140]), ([60], [2500])],
                         ids=["rows", "tiles", "tiles_split"])
def test_attention_scores_beyond_fp32(gpu_lib, q_lens, kv_lens, scale, kind):
    """128 scale is no fp32 number: the rows are NaN, not zeros."""
    fq = gpu_lib

    def edit(b, k, v):
        k[:] = 1.0

    st = Step(fq, kind, 128, 4, 2, 16, q_lens, kv_lens, seed=23, edit=edit)
    st.q.fill_(1.0)
    if len(q_lens) == 1:
        c = tiles_bounds(st, by_keys=kv_lens[0] > 2000)
        assert c["split"] > 1 or kv_lens[0] < 2000
    log(f"attention scores beyond fp32 {kind} {kv_lens} {scale}")
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, scale=scale, return_lse=True)
    torch.cuda.synchronize()
    assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("tiles", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("at", [3, 70, 137], ids=["whole", "whole_later", "partial"])
def test_attention_infinities_of_no_weight(gpu_lib, at, tiles, kind):
    """V holds an infinity under a seen key whose weight is far below fp32: that channel (with
    codes, the row) is not finite, wherever the key lies, and the others are as without it."""
    fq = gpu_lib
    S, n = 140, 4   # tokens at 136 .. 139

    def edit(bad):
        def f(b, k, v):
            k[:] = 1.0
            k[at] = -1.0
            if bad:
                v[at, :, 7] = float("inf")
                v[at, :, 9] = float("-inf")
        return f

    outs = []
    for bad in (True, False):
        st = Step(fq, kind, 128, 4, 2, 16, [n], [S], seed=27, edit=edit(bad))
        st.q.fill_(3.0)
        if tiles:
            tiles_bounds(st)
        log(f"attention infinity of no weight {kind} at {at} tiles={tiles} bad={bad}")
        out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, scale=1.0, return_lse=True)   # scores of +-384
        torch.cuda.synchronize()
        outs.append((out, lse))
    (out, lse), (clean, clean_lse) = outs
    first = max(0, at - (S - n))   # the first token that sees it
    assert torch.equal(out[:first], clean[:first]) and torch.equal(lse, clean_lse)
    if kind == "bf16":
        assert not torch.isfinite(out[first:, :, [7, 9]]).any()
        keep = [c for c in range(128) if c not in (7, 9)]
        assert torch.equal(out[:, :, keep], clean[:, :, keep])
    else:
        assert torch.isnan(out[first:]).all()


def rows_held(held):
    """K and V of a bf16 step as check_rows takes them."""
    return held, [[np.abs(t) for t in ts] for ts in held]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("name", list(STEPS) + ["many_" + n for n in MANY])
def test_attention_within_the_magnitudes_of_its_summands(gpu_lib, name, kind, D):
    """The steps of the other file with the tolerance that each kernel's own summands give: an
    addition rounded to nearest (2^-24) of |q| s (c + z), with 4 bits of |q| s (16 + c + z),
    and one rounding to bf16 (2^-8) of a weight and of the result."""
    fq = gpu_lib
    many = name.startswith("many_")
    hq, hkv, page, q_lens, kv_lens, window, sinks = MANY[name[5:]] if many else STEPS[name]
    st = Step(fq, kind, D, hq, hkv, page, q_lens, kv_lens, seed=5 * len(name) + D)
    if many:
        tiles_bounds(st, window, sinks, by_keys="split" in name and not window)
    log(f"attention magnitudes {name} {kind} D={D}")
    out, lse = fq.fq_paged_attention(st.q, st.cache, st.batch, window=window, sinks=sinks, return_lse=True)
    torch.cuda.synchronize()
    held, size = rows_held([[f64(t) for t in ts] for ts in (st.k, st.v)]) if kind == "bf16" else held_codes(st)
    check_rows(out, lse, st.q, st.cu, held, size, q_lens, kv_lens, D, float(np.float32(D ** -0.5)), window, sinks,
               every=11 if many else 3, unit=2.0 ** -24)


@pytest.mark.parametrize("kind", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("given", [True, False], ids=["stream_given", "stream_current"])
def test_every_operator_runs_on_its_stream(gpu_lib, kind, given):
    """All inputs of write, read, attention and norm are made on a side stream behind work that
    keeps it busy, over contents that give other results: on any other stream the calls would
    take those."""
    fq = gpu_lib
    st = Step(fq, kind, 128, 8, 2, 64, [1, 1], [4000, 77], seed=12)
    slots = torch.cat([st.table[b].long()[t // 64] * 64 + t % 64 for b, t in ((0, torch.arange(4000)), (1, torch.arange(77)))])
    names = ["q", "k", "v", "slots", "x", "res", "w"]
    g = torch.Generator().manual_seed(9)
    made = [st.q.clone(), torch.cat(st.k).cuda(), torch.cat(st.v).cuda(), slots.cuda(),
            *(torch.randn(s, generator=g).to(torch.bfloat16).cuda() for s in ((64, 4096), (64, 4096), (4096,)))]
    cache = fq.KVCache.empty(st.cache.n_pages, 64, 2, 128, kind)

    def calls(t, stream):
        fq.fq_kv_cache_write(cache, t["k"], t["v"], t["slots"], stream=stream)
        k, v = fq.fq_kv_cache_read(cache, t["slots"], dtype="f32", stream=stream)
        out, lse = fq.fq_paged_attention(t["q"], cache, st.batch, return_lse=True, stream=stream)
        r, h = fq.fq_gated_residual_norm(t["x"], t["res"], t["w"], stream=stream)
        return k, v, out, lse, r, h

    want = [t.clone() for t in calls(dict(zip(names, made)), None)]
    c = fq.fq_paged_attention_launch(8, 2, cache, st.batch)
    assert c["split"] > 1
    empty = {n: torch.full_like(t, -1) if n == "slots" else torch.zeros_like(t) for n, t in zip(names, made)}
    busy = torch.randn((4096, 4096), device="cuda").to(torch.bfloat16)
    for t in (cache.k, cache.v):
        t.view(torch.uint8).zero_()
    side, end = torch.cuda.Stream(), torch.cuda.Event()
    log(f"operators on a side stream {kind} given={given}")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(400):
            torch.mm(busy, busy)
        for n, t in zip(names, made):
            empty[n].copy_(t)
        if not given:
            got = calls(empty, None)
    if given:
        got = calls(empty, side)
    end.record(side)
    assert not end.query()   # the work before them was still under way when all had been enqueued
    side.synchronize()
    for n, a, b in zip(("k", "v", "out", "lse", "r", "h"), got, want):
        assert torch.equal(a, b), n


def test_norm_of_more_rows_than_one_launch_takes(gpu_lib):
    """2^26 rows of 64 threads are the 2^32 that no grid holds: rows at the ends of the launches
    they are done in are those of calls of a few rows."""
    fq = gpu_lib
    M, H = (1 << 26) + 5, 4
    log(f"norm {M} x {H}")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((M, H), generator=g, device="cuda", dtype=torch.bfloat16)
    res = torch.randn((M, H), generator=g, device="cuda", dtype=torch.bfloat16)
    gate = torch.rand((M, 8), generator=g, device="cuda").to(torch.bfloat16)[:, 2:6]
    w = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    r, h = fq.fq_gated_residual_norm(x, res, w, post_weight=w, gate=gate)
    for first in [0, *((p << 21) - 3 for p in (1, 2, 17, 31, 32))]:
        at = slice(first, min(first + 8, M))
        a, b = fq.fq_gated_residual_norm(x[at], res[at], w, post_weight=w, gate=gate[at])
        torch.cuda.synchronize()
        assert torch.equal(r[at], a) and torch.equal(h[at], b), first
    assert torch.isfinite(h.view(-1)[::4097]).all() and (h != 0).any(1).all()


def test_norm_of_wide_rows_over_launches(gpu_lib):
    """fp32 and strided rows over the end of a launch."""
    fq = gpu_lib
    M, H = (1 << 21) + 7, 8
    log(f"norm {M} x {H}")
    wide = torch.randn((M, 24), device="cuda")
    x, res = wide[:, 1:9], wide[:, 11:19]
    w = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    r, h = fq.fq_gated_residual_norm(x, res, w, residual_scale=0.5)
    at = slice(M - 12, M)
    a, b = fq.fq_gated_residual_norm(x[at], res[at], w, residual_scale=0.5)
    torch.cuda.synchronize()
    assert torch.equal(r[at], a) and torch.equal(h[at], b)


def test_cache_of_more_tokens_than_one_launch_takes(gpu_lib):
    """2^29 tokens of 8 threads are the 2^32 that no grid holds; here nearly all of them are not
    stored.  And a read over the end of a launch."""
    fq = gpu_lib
    n = (1 << 29) + 3
    log(f"cache of {n} tokens")
    cache = fq.KVCache.empty(2, 16, 1, 64, "int8")
    row = torch.randn((1, 1, 64), device="cuda").to(torch.bfloat16)
    slots = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    at = [0, (1 << 24) - 1, 1 << 24, (1 << 28) + 1, n - 1]
    slots[at] = torch.arange(5, device="cuda") * 3
    fq.fq_kv_cache_write(cache, row.expand(n, 1, 64), (-row).expand(n, 1, 64), slots)
    del slots
    k, v = fq.fq_kv_cache_read(cache, torch.arange(5, device="cuda") * 3, dtype="f32")
    torch.cuda.synchronize()
    for t, x in ((k, f64(row)), (v, -f64(row))):
        want = L.held_rows(x, "int8").astype(np.float32)
        assert (t.cpu().numpy() == want).all()
    n = (1 << 24) + 9
    slots = torch.arange(n, device="cuda") % 32
    k, v = fq.fq_kv_cache_read(cache, slots)
    part = fq.fq_kv_cache_read(cache, slots[(1 << 24) - 16:])
    torch.cuda.synchronize()
    stored = torch.isin(slots[(1 << 24) - 16:], torch.arange(5, device="cuda") * 3)
    assert stored.any()
    for t, p in ((k, part[0]), (v, part[1])):
        assert torch.equal(t[(1 << 24) - 16:][stored], p[stored])


def test_workspaces_that_no_kernel_may_write_are_refused(gpu_lib):
    """Before anything is launched; a workspace of any type counts by its bytes."""
    fq = gpu_lib
    st = Step(fq, "bf16", 128, 8, 2, 64, [1], [5000], seed=9)
    need = fq.fq_paged_attention_workspace_bytes(8, 1, st.cache, st.batch)
    log(f"workspaces of the caller, {need} bytes")
    for bad in (torch.zeros(need, dtype=torch.uint8), torch.zeros(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="ws"):
            fq.fq_paged_attention(st.q, st.cache, st.batch, ws=bad)
    with pytest.raises(fq.FqError):
        fq.fq_paged_attention(st.q, st.cache, st.batch, ws=torch.zeros(need - 4, dtype=torch.uint8, device="cuda"))
    ws = torch.zeros(-(-need // 4), dtype=torch.int32, device="cuda")
    assert torch.equal(fq.fq_paged_attention(st.q, st.cache, st.batch, ws=ws), fq.fq_paged_attention(st.q, st.cache, st.batch))
