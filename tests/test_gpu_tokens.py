"""GPU: the operators on packed tokens against their definitions in 64 bits (oracle/tokens.py), at the sizes and masks where they can go wrong.
Tolerances are the bounds derived there from the roundings that the kernels make."""
import numpy as np
import pytest
import torch

from oracle import tokens as ot

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.fixture(scope="module")
def bbm():
    import paper_2409_15097_amd as m
    return m


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def normal(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(torch.bfloat16).cuda()


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def in_layout(x, layout):
    """The packed tensor with the same values: contiguous, as a part of a wider projection, or with the heads outermost."""
    T, H, d = x.shape
    if layout == "fused":
        wide = torch.full((T, (H + 3) * d + 8), NAN, dtype=x.dtype, device=x.device)
        part = wide[:, d:(H + 1) * d].unflatten(1, (H, d))
        part.copy_(x)
        return part
    return x.transpose(0, 1).contiguous().transpose(0, 1) if layout == "heads" else x


def close(name, got, want, tol):
    got = f64(got)
    bad = ~(np.abs(got - want) <= tol) & ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} values off, the worst {np.abs(got - want)[bad].max()} against {tol[bad].min()}; at {np.argwhere(bad)[:4].tolist()}"


# ---- slots


@pytest.mark.parametrize("R, new, ctx, page, short_list, narrow", [
    (1, 1, 0, 16, 0, 0), (1, 200, 70, 64, 0, 0), (3, 5, 40, 16, 2, 0), (64, 1, 500, 64, 0, 0), (65, 3, 17, 32, 0, 1), (1000, 9, 300, 16, 40, 0),
    (1500, 130, 100, 128, 0, 2), (8200, 2, 64, 16, 0, 0), (16384, 2, 33, 32, 100, 1)])
def test_slots(bbm, R, new, ctx, page, short_list, narrow):
    g = np.random.default_rng(R)
    c, a = g.integers(0, ctx + 1, R), g.integers(0, new + 1, R)
    c[g.random(R) < 0.1] = 0
    a[-1], c[-1] = new, ctx
    if R > 2:
        c[0], a[1] = -3, -1                                              # stand for none
    width = max(1, -(-(ctx + new) // page) - narrow)
    held, want = (np.minimum(-(-np.maximum(x, 0) // page), width) for x in (c, np.maximum(c, 0) + np.maximum(a, 0)))
    ids = g.permutation(int(want.sum()) + 40).astype(np.int32)
    wide = np.full((R, width + 3), -7, np.int32)
    wide[:, :width] = np.where(np.arange(width) < held[:, None], np.arange(R)[:, None] % 5 * 1000 + np.arange(width), -2)
    first, n_free = 3, max(0, 3 + int((want - held).sum()) - short_list)
    T = max(0, int(np.maximum(a, 0).sum()) + (7 if R % 2 else -2))
    free = ids[:n_free]
    wt, wcu, wlens, wpos, wslots, wnext = ot.build_slots(c, a, wide[:, :width], free, first, T, page)
    buf = i32(wide)
    for _ in range(2):                                                   # a repeated call finds what it left
        r = bbm.bbm_build_slots(i32(c), i32(a), buf[:, :width], i32(free), i32([first]), T, page)
        got = buf.cpu().numpy()
        assert np.array_equal(got[:, :width], wt) and (got[:, width:] == -7).all()
        for x, y in ((r.cu_new, wcu), (r.lens, wlens), (r.positions, wpos), (r.slots, wslots), (r.free_next, [wnext])):
            assert np.array_equal(x.cpu().numpy(), y)


# ---- rotary positions


@pytest.mark.parametrize("T, H, Hk, d, rot, interleaved, layout", [
    (1, 1, 1, 16, 2, False, "plain"), (1, 4, 0, 64, 64, True, "plain"), (33, 32, 8, 128, 128, False, "fused"), (7, 3, 1, 64, 62, False, "fused"),
    (7, 3, 1, 64, 62, True, "heads"), (130, 8, 2, 128, 64, True, "fused"), (130, 8, 2, 128, 40, False, "heads"), (65, 5, 5, 80, 20, False, "plain"),
    (65, 5, 5, 80, 6, True, "plain"), (3000, 4, 2, 128, 96, False, "plain"), (5000, 2, 1, 512, 512, True, "plain"), (40, 2, 1, 112, 112, False, "heads"),
    (300, 40, 8, 80, 74, False, "heads"), (4100, 2, 1, 512, 510, False, "fused"), (9, 24, 3, 144, 24, False, "plain"), (2, 70, 3, 16, 2, False, "plain")])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope(bbm, T, H, Hk, d, rot, interleaved, layout, inverse):
    g = np.random.default_rng(T + rot)
    pos = g.integers(-5, 1 << 20, T)
    pos[0] = (1 << 31) - 1
    freqs, mscale = bbm.rope_freqs(rot, factor=8.0, method="yarn", trained_len=4096)
    q, k = normal(1, T, H, d), normal(2, T, Hk, d) if Hk else None
    ql, kl = in_layout(q, layout), None if k is None else in_layout(k, layout)
    got = bbm.bbm_rope(ql, kl, i32(pos), freqs, interleaved=interleaved, mscale=mscale, inverse=inverse)
    for name, x, y in (("q", q, got[0]), ("k", k, got[1])):
        if x is None:
            assert y is None
            continue
        want = ot.rope(f64(x), pos, f64(freqs), interleaved, mscale, inverse)
        x = f64(x)
        one = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
        two = one + (1 if interleaved else rot // 2)
        size = np.zeros_like(want)
        size[..., one] = size[..., two] = mscale * (np.abs(x[..., one]) + np.abs(x[..., two]))
        close(name, y, want, ot.B * np.abs(want) + 16 * ot.F * size)     # a sine off by a few steps of 1, three products and a sum
        assert (f64(y)[..., rot:] == x[..., rot:]).all()
    # in place, and back again
    a, b = bbm.bbm_rope(ql, kl, i32(pos), freqs, interleaved=interleaved, mscale=mscale, inverse=inverse, out_q=ql, out_k=kl)
    assert a is ql and torch.equal(ql, got[0]) and (k is None or torch.equal(kl, got[1]))


# ---- prompts


LENS = {
    "one": [1], "two": [2, 1], "empty": [0, 5, 0, 0, 70, 0], "tiles": [64, 65, 63, 128, 127, 129], "crowd": [int(x) for x in np.random.default_rng(4).integers(0, 4, 700)], "throng": [1] * 4200,
    "ragged": [1, 200, 3, 33, 257, 2, 1, 90],
    "many": [int(x) for x in np.random.default_rng(3).integers(0, 12, 150)], "long": [700, 1], "longer": [1300],
}


def prompt_case(name, H, Hk, d, layout, seed=0, before=2, behind=3, scale=1.0):
    lens = LENS[name]
    cu = np.concatenate([[0], np.cumsum(lens)]) + before                   # rows in front of the first sequence and behind the last
    T = int(cu[-1]) + behind
    x = {n: normal(seed + i, T, h, d, scale=scale) for i, (n, h) in enumerate((("q", H), ("k", Hk), ("v", Hk), ("d_o", H)))}
    for t in x.values():                                                   # rows of nobody hold anything
        t[:before] = NAN
        t[cu[-1]:] = float("inf")
    return cu, T, {n: in_layout(t, layout) for n, t in x.items()}


def check_prompt(bbm, cu, T, x, H, Hk, d, scale=None, bwd=True):
    sm = d ** -0.5 if scale is None else scale
    out = torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((H, T), 7.0, device="cuda")
    o, lse = bbm.bbm_prompt_attn_fwd(x["q"], x["k"], x["v"], i32(cu), softmax_scale=scale, out=out, lse=lse)
    grads = [torch.full((T, h, d), 7.0, dtype=torch.bfloat16, device="cuda") for h in (H, Hk, Hk)]
    if bwd:
        bbm.bbm_prompt_attn_bwd(x["q"], x["k"], x["v"], o, x["d_o"], lse, i32(cu), softmax_scale=scale, dq=grads[0], dk=grads[1], dv=grads[2])
    real = np.zeros(T, bool)
    real[cu[0]:cu[-1]] = True
    for t in [o, lse.t()] + grads:
        assert (f64(t)[~real] == 7.0).all(), "rows of nobody are left as they were"
    n = {a: f64(t) for a, t in x.items()}
    oo, ll, gg = f64(o), f64(lse), [f64(t) for t in grads]
    worst = 0.0
    for a, b in zip(cu[:-1], cu[1:]):
        if a == b:
            continue
        seen = np.tril(np.ones((b - a, b - a), bool))
        for hk in range(Hk):
            k, v = n["k"][a:b, hk], n["v"][a:b, hk]
            dk, dv, e_dk, e_dv = (np.zeros((b - a, d)) for _ in range(4))
            for h in range(hk * (H // Hk), (hk + 1) * (H // Hk)):
                q, d_o = n["q"][a:b, h], n["d_o"][a:b, h]
                wo, wl, p = ot.attention(q, k, v, seen, sm)
                at = f"rows {a}..{b}, head {h}: "
                if not bwd:
                    e_o, e_l = ot.bounds(q, k, v, seen, sm, p, wo, wl)
                    close(at + "O", o[a:b, h], wo, e_o), close(at + "lse", lse[h, a:b], wl, e_l)
                    continue
                delta = (d_o * oo[a:b, h]).sum(1)
                g = ot.attention_bwd(q, k, v, d_o, p, sm, delta)
                e_o, e_l, e_dq, e1, e2 = ot.bounds(q, k, v, seen, sm, p, wo, wl, d_o, delta, g)
                close(at + "O", o[a:b, h], wo, e_o), close(at + "lse", lse[h, a:b], wl, e_l), close(at + "dQ", grads[0][a:b, h], g[0], e_dq)
                dk, dv, e_dk, e_dv = dk + g[1], dv + g[2], e_dk + e1, e_dv + e2
            if bwd:
                close(f"rows {a}..{b}, key head {hk}: dK", grads[1][a:b, hk], dk, e_dk), close(f"rows {a}..{b}, key head {hk}: dV", grads[2][a:b, hk], dv, e_dv)
    return o, lse, grads


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name, H, Hk, layout", [("one", 1, 1, "plain"), ("two", 6, 2, "fused"), ("empty", 4, 4, "heads"), ("tiles", 3, 1, "plain"),
                                                 ("ragged", 8, 2, "fused"), ("many", 4, 1, "heads"), ("long", 2, 2, "plain"), ("longer", 5, 1, "fused")])
def test_prompt(bbm, name, H, Hk, d, layout):
    cu, T, x = prompt_case(name, H, Hk, d, layout)
    o, lse, grads = check_prompt(bbm, cu, T, x, H, Hk, d)
    # the same bits again, and without a log-sum-exp in the C call's place of one
    o2, lse2 = bbm.bbm_prompt_attn_fwd(x["q"], x["k"], x["v"], i32(cu))
    g2 = bbm.bbm_prompt_attn_bwd(x["q"], x["k"], x["v"], o2, x["d_o"], lse2, i32(cu))
    a, b = int(cu[0]), int(cu[-1])
    assert torch.equal(o[a:b], o2[a:b]) and torch.equal(lse[:, a:b], lse2[:, a:b]) and all(torch.equal(u[a:b], w[a:b]) for u, w in zip(grads, g2))


@pytest.mark.parametrize("name, H, Hk, d", [("longer", 40, 8, 128), ("longer", 64, 8, 64), ("ragged", 64, 16, 64), ("ragged", 64, 64, 128)])
def test_prompt_with_many_heads(bbm, name, H, Hk, d):
    """Launches that fill the chip: a group of waves a piece, and (64 heads over 8 of 64) the heads of a group in three uneven parts."""
    cu, T, x = prompt_case(name, H, Hk, d, "plain", seed=3)
    check_prompt(bbm, cu, T, x, H, Hk, d)


@pytest.mark.parametrize("name, d", [("crowd", 64), ("throng", 128)])
def test_prompt_with_many_sequences(bbm, name, d):
    """More requests than are counted through: their pieces are searched for."""
    cu, T, x = prompt_case(name, 2, 1, d, "plain", seed=6)
    check_prompt(bbm, cu, T, x, 2, 1, d)


def test_prompt_with_heads_that_share_values(bbm):
    """Keys and values expanded over the heads (stride 0) give the gradients of each head."""
    cu, T, x = prompt_case("ragged", 4, 1, 64, "plain", seed=7)
    x["k"], x["v"] = (x[n].expand(T, 4, 64) for n in ("k", "v"))
    check_prompt(bbm, cu, T, x, 4, 4, 64)


@pytest.mark.parametrize("scale, size", [(1.0, 1.0), (0.01, 1.0), (0.125, 6.0)])
def test_prompt_with_other_scales(bbm, scale, size):
    cu, T, x = prompt_case("ragged", 2, 1, 64, "plain", seed=9, scale=size)
    check_prompt(bbm, cu, T, x, 2, 1, 64, scale=scale)


def test_prompt_rows_that_see_large_values(bbm):
    """Keys and values of 1e30 behind a query leave its row alone; a row of equal large scores is an average."""
    cu, T, x = prompt_case("long", 1, 1, 64, "plain", seed=4)
    a, b = int(cu[0]), int(cu[1])
    x["k"][b - 40:b] = 1e30
    x["v"][b - 40:b] = -1e30
    o, lse = bbm.bbm_prompt_attn_fwd(x["q"], x["k"], x["v"], i32(cu))
    n = {m: f64(t)[a:b - 40, 0] for m, t in x.items()}
    seen = np.tril(np.ones((b - 40 - a,) * 2, bool))
    wo, wl, p = ot.attention(n["q"], n["k"], n["v"], seen, 0.125)
    e_o, e_l = ot.bounds(n["q"], n["k"], n["v"], seen, 0.125, p, wo, wl)
    close("O", o[a:b - 40, 0], wo, e_o), close("lse", lse[0, a:b - 40], wl, e_l)


# ---- the cache in 4 bits


def host_cache(c):
    k, v = (ot.unpack_nibbles(t.cpu().numpy()) for t in (c.k, c.v))
    return ot.kv4_decode(k, c.k_scale.cpu().numpy()), ot.kv4_decode(v, c.v_scale.transpose(-1, -2).cpu().numpy())     # [pages, Hk, page, d]


@pytest.mark.parametrize("T, Hk, d, page, layout", [(1, 1, 64, 16, "plain"), (3, 2, 128, 32, "fused"), (130, 3, 64, 64, "heads"), (700, 2, 128, 128, "fused"), (2100, 1, 64, 16, "plain")])
def test_append_and_read(bbm, T, Hk, d, page, layout):
    g = np.random.default_rng(T)
    pages = -(-T // page) + 2
    c = bbm.kv4_cache(pages, Hk, d, page)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        t.fill_(0x55)
    spread = torch.exp2(torch.from_numpy(g.integers(-20, 20, (T, Hk, 1))).cuda().float())
    k = (normal(1, T, Hk, d).float() * spread).to(torch.bfloat16)
    v = normal(2, T, Hk, d)
    grid = torch.tensor([0, .25, .5, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, -.25, -2.5, -5, -7, 0.0])
    v[0, 0, :16] = grid.to(torch.bfloat16).cuda()                          # halfway values
    v[0, 0, 16:32] = 0
    if T > 1:
        k[1] = 0
        k[2, 0, :32], k[2, 0, 32:64] = 3.3e38, -1e-38                      # the largest and smallest scales
        k[2, 0, 7] = 2.0 ** -133
    slots = g.permutation(pages * page - 1)[:T].astype(np.int64)
    if T > 2:
        slots[1::7] = -1
        slots[2] = pages * page - 1
        slots[5::100] = pages * page + 3
    inside = (slots >= 0) & (slots < pages * page)
    bbm.bbm_kv4_append(in_layout(k, layout), in_layout(v, layout), i32(slots), c)
    pg, at = slots[inside] // page, slots[inside] % page
    for x, codes, scales, v_order in ((k, c.k, c.k_scale, False), (v, c.v, c.v_scale, True)):
        want_codes, want_scales = ot.kv4_encode(f64(x)[inside])
        got_codes, got_scales = ot.unpack_nibbles(codes.cpu().numpy()), scales.cpu().numpy()
        got_scales = got_scales.swapaxes(-1, -2) if v_order else got_scales
        assert np.array_equal(got_scales[pg, :, at], want_scales)
        assert np.array_equal(ot.kv4_decode(got_codes[pg, :, at], got_scales[pg, :, at]), ot.kv4_decode(want_codes, want_scales))
        got_codes[pg, :, at], got_scales[pg, :, at] = 5, 0x55
        assert (got_codes == 5).all() and (got_scales == 0x55).all(), "other slots are left as they were"
    rk, rv = (in_layout(torch.full((T, Hk, d), NAN, dtype=torch.bfloat16, device="cuda"), layout) for _ in range(2))
    bbm.bbm_kv4_read(i32(slots), c, out_k=rk, out_v=rv)
    hk, hv = host_cache(c)
    for got, want in ((rk, hk), (rv, hv)):
        assert np.array_equal(f64(got)[inside], want[pg, :, at]) and (f64(got)[~inside] == 0).all()


def test_groups_that_are_not_finite(bbm):
    c = bbm.kv4_cache(1, 1, 64, 16)
    k, v = normal(1, 2, 1, 64), normal(2, 2, 1, 64)
    k[0, 0, 3], v[1, 0, 40] = float("inf"), NAN
    bbm.bbm_kv4_append(k, v, i32([4, 5]), c)
    rk, rv = bbm.bbm_kv4_read(i32([4, 5]), c)
    assert torch.isnan(rk[0, 0, :32]).all() and torch.isfinite(rk[0, 0, 32:]).all() and torch.isfinite(rk[1]).all()
    assert torch.isnan(rv[1, 0, 32:]).all() and torch.isfinite(rv[1, 0, :32]).all() and torch.isfinite(rv[0]).all()


def cached_case(bbm, lens, news, H, Hk, d, page, layout="plain", seed=0, tree=None, before=0, behind=0, extra_pages=2, width=None):
    """Random pages; slots behind a request's length and pages of nobody hold NaN scales."""
    g = np.random.default_rng(seed)
    R = len(lens)
    need = [-(-n // page) for n in lens]
    width = max(1, max(need) + 1) if width is None else width
    pages = sum(need) + extra_pages
    ids = g.permutation(pages)
    table = np.full((R, width), -1, np.int64)
    c = bbm.kv4_cache(pages, Hk, d, page)
    c.k.copy_(torch.from_numpy(g.integers(0, 256, c.k.shape, dtype=np.uint8)))
    c.v.copy_(torch.from_numpy(g.integers(0, 256, c.v.shape, dtype=np.uint8)))
    ks, vs = np.full(c.k_scale.shape, 255, np.uint8), np.full(c.v_scale.shape, 255, np.uint8)
    at = 0
    for r, n in enumerate(lens):
        for p in range(need[r]):
            if p < width:
                table[r, p] = ids[at]
            m = min(page, n - p * page)
            ks[ids[at], :, :m] = g.integers(125, 128, (Hk, m, d // 32))
            vs[ids[at], :, :, :m] = g.integers(125, 128, (Hk, d // 32, m))
            at += 1
    c.k_scale.copy_(torch.from_numpy(ks)), c.v_scale.copy_(torch.from_numpy(vs))
    cu = np.concatenate([[0], np.cumsum(news)]) + before
    T = int(cu[-1]) + behind
    q = normal(seed + 5, T, H, d)
    words = None
    if tree is not None:
        words = g.integers(0, 1 << 62, (T, tree), dtype=np.int64) * 2 + g.integers(0, 2, (T, tree))
        words[g.random(T) < 0.2] = 0                                       # nodes that see none of the new tokens
    return c, table, cu, T, in_layout(q, layout), words


def check_cached(bbm, c, table, lens, cu, T, q, words, H, Hk, d, page, **kw):
    out, lse = torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((H, T), 7.0, device="cuda")
    bbm.bbm_kv4_attn(q, c, i32(table), i32(lens), i32(cu), mask=None if words is None else torch.from_numpy(words).cuda(), out=out, lse=lse, **kw)
    real = np.zeros(T, bool)
    real[max(0, cu[0]):cu[-1]] = True
    assert (f64(out)[~real] == 7.0).all() and (f64(lse)[:, ~real] == 7.0).all()
    hk, hv = host_cache(c)
    nq, G = f64(q), H // Hk
    for r, n in enumerate(lens):
        a, b, new = max(0, int(cu[r])), min(T, int(cu[r + 1])), int(cu[r + 1] - cu[r])
        if b <= a:
            continue
        m = min(max(n, 0), table.shape[1] * page)
        pg = table[r, np.arange(m) // page]
        ok = (pg >= 0) & (pg < c.k.shape[0])
        j, i = np.arange(m), np.arange(a, b)[:, None] - int(cu[r])
        if words is None:
            seen = (j <= n - new + i) & ok
        else:
            nj = j - (n - new)
            bit = np.zeros((b - a, m), bool)
            inside = (nj >= 0) & (nj < 64 * words.shape[1])
            bit[:, inside] = (words[a:b][:, nj[inside] // 64] >> (nj[inside] % 64)) & 1 != 0
            seen = ((nj < 0) | bit) & ok
        for h in range(H):
            k, v = (np.where(ok[:, None], x[np.where(ok, pg, 0), h // G, j % page], 0.0) if m else np.zeros((0, d)) for x in (hk, hv))
            wo, wl, p = ot.attention(nq[a:b, h], k, v, seen, d ** -0.5)
            e_o, e_l = ot.bounds(nq[a:b, h], k, v, seen, d ** -0.5, p, wo, wl)
            close(f"request {r}, head {h}: O", out[a:b, h], wo, e_o), close(f"request {r}, head {h}: lse", lse[h, a:b], wl, e_l)
    return out, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens, news, H, Hk, page, layout, tree", [
    ([1], [1], 1, 1, 16, "plain", None), ([0, 3, 17], [1, 1, 1], 4, 2, 16, "fused", None), ([63, 64, 65, 200, 1, 0], [1] * 6, 8, 1, 32, "plain", None),
    ([130, 300, 31], [1, 0, 1], 6, 2, 64, "heads", None), ([40, 500, 7], [5, 33, 7], 6, 2, 16, "fused", None), ([40, 90], [40, 60], 32, 2, 128, "plain", None),
    ([20, 70, 5], [20, 6, 5], 4, 4, 16, "plain", 1), ([300, 129], [70, 129], 3, 1, 64, "heads", 2), ([300, 150], [100, 100], 5, 1, 32, "plain", 1),
    ([3, 2], [5, 4], 4, 2, 16, "plain", None), ([2900, 9, 1700], [1, 1, 2], 12, 4, 64, "plain", None), ([2500, 2100], [40, 30], 8, 2, 32, "fused", None), ([2500, 2100], [70, 20], 4, 2, 64, "plain", 1),
    ([20] * 600, [1] * 600, 2, 1, 16, "plain", None), ([33] * 70, [1] * 70, 2, 1, 16, "plain", None)])
def test_cached(bbm, lens, news, H, Hk, d, page, layout, tree):
    c, table, cu, T, q, words = cached_case(bbm, lens, news, H, Hk, d, page, layout, seed=len(lens), tree=tree, before=2, behind=3)
    first = check_cached(bbm, c, table, lens, cu, T, q, words, H, Hk, d, page)
    again = check_cached(bbm, c, table, lens, cu, T, q, words, H, Hk, d, page, max_len=max(1, max(lens)))
    some = check_cached(bbm, c, table, lens, cu, T, q, words, H, Hk, d, page)
    assert all(torch.equal(x, y) for x, y in zip(first, some)) and again is not None


def test_cached_pages_outside_and_a_narrow_table(bbm):
    lens, news, H, Hk, d, page = [500, 300, 90], [1, 3, 2], 4, 2, 128, 32
    c, table, cu, T, q, _ = cached_case(bbm, lens, news, H, Hk, d, page, seed=3)
    table[0, 3], table[0, 15], table[1, 0], table[2, :] = -1, 1 << 30, c.k.shape[0], -5
    check_cached(bbm, c, table, lens, cu, T, q, None, H, Hk, d, page)
    check_cached(bbm, c, table[:, :5], lens, cu, T, q, None, H, Hk, d, page)
    check_cached(bbm, c, table[:, :5], [700, -4, 1 << 30], cu, T, q, None, H, Hk, d, page)


@pytest.mark.parametrize("H, lens, news, tree", [(4, [300, 90, 70], [40, 30, 60], None), (4, [300, 90, 70], [40, 30, 60], 1), (40, [700, 900, 700], [240, 230, 260], None)])
@pytest.mark.parametrize("front, rows", [(0, 3), (17, 5)])
def test_cached_rows_that_are_not_there(bbm, H, lens, news, tree, front, rows):
    """Offsets that begin in front of the first row or end behind the last: the tokens without a row are in the cache all the same."""
    c, table, cu, T, q, words = cached_case(bbm, lens, news, H, 2, 64, 32, seed=11, tree=tree)
    a, b = front, news[0] + news[1] + rows
    check_cached(bbm, c, table, lens, cu - a, b - a, q[a:b].contiguous(), None if words is None else words[a:b].copy(), H, 2, 64, 32)


@pytest.mark.parametrize("max_len", [1, 300, 5000, 1 << 40])
def test_cached_with_a_wrong_hint(bbm, max_len):
    c, table, cu, T, q, _ = cached_case(bbm, [2300, 40], [1, 2], 4, 2, 64, 64, seed=5)
    check_cached(bbm, c, table, [2300, 40], cu, T, q, None, 4, 2, 64, 64, max_len=max_len)


def test_cached_many_heads_a_key_head(bbm):
    c, table, cu, T, q, _ = cached_case(bbm, [200, 77], [1, 3], 71, 1, 64, 16, seed=6)
    check_cached(bbm, c, table, [200, 77], cu, T, q, None, 71, 1, 64, 16)


@pytest.mark.parametrize("d, tree, layout", [(64, None, "fused"), (128, None, "plain"), (128, 3, "heads")])
def test_cached_wide_in_parts(bbm, d, tree, layout):
    lens, news = [2500, 2100], [130, 130]
    c, table, cu, T, q, words = cached_case(bbm, lens, news, 64, 8, d, 32, layout, seed=9, tree=tree, before=1, behind=2)
    check_cached(bbm, c, table, lens, cu, T, q, words, 64, 8, d, 32, max_len=2500)


def test_cached_wide_with_pages_outside(bbm):
    """The kernel of many columns (more than 16384 rows of all heads), its last tile of a few keys, a page outside and a mask."""
    lens, news = [300, 150], [140, 130]
    for tree in (None, 3):
        c, table, cu, T, q, words = cached_case(bbm, lens, news, 64, 64, 64, 16, seed=7, tree=tree)
        table[0, 4], table[1, 0] = -1, c.k.shape[0] + 1
        check_cached(bbm, c, table, lens, cu, T, q, words, 64, 64, 64, 16)


def test_cached_pages_shared_by_requests(bbm):
    """A common prefix is kept once."""
    lens, H, Hk, d, page = [200, 200, 200], 4, 1, 64, 64
    c, table, cu, T, q, _ = cached_case(bbm, lens, [1, 2, 1], H, Hk, d, page, seed=8)
    table[1, :3] = table[2, :3] = table[0, :3]
    check_cached(bbm, c, table, lens, cu, T, q, None, H, Hk, d, page)


def test_offsets_past_32_bits(bbm):
    """A cache whose codes take more than 2^32 bytes: its last pages are written, read and attended."""
    Hk, d, page = 8, 128, 128
    pages = (1 << 32) // (Hk * page * d // 2) + 64
    c = bbm.kv4_cache(pages, Hk, d, page)
    T = 150
    k, v, q = normal(1, T, Hk, d), normal(2, T, Hk, d), normal(3, 1, Hk, d)
    slots = np.arange(T) + (pages - 2) * page
    bbm.bbm_kv4_append(k, v, i32(slots), c)
    rk, rv = bbm.bbm_kv4_read(i32(slots), c)
    small = bbm.kv4_cache(2, Hk, d, page)
    bbm.bbm_kv4_append(k, v, i32(np.arange(T)), small)
    sk, sv = bbm.bbm_kv4_read(i32(np.arange(T)), small)
    assert torch.equal(rk, sk) and torch.equal(rv, sv) and not (rk == 0).all()
    a = bbm.bbm_kv4_attn(q, c, i32([[pages - 2, pages - 1]]), i32([T]), i32([0, 1]))
    b = bbm.bbm_kv4_attn(q, small, i32([[0, 1]]), i32([T]), i32([0, 1]))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ---- together


def layer(bbm, s, w):
    """A step of one attention layer over the cache: slots, rotary positions, attention of prompts or of new tokens, and the cache behind it."""
    r = bbm.bbm_build_slots(s["ctx"], s["new"], s["table"], s["free"], s["at"], w.shape[0], s["cache"].k.shape[2])
    H, Hk, d = s["H"], s["Hk"], s["cache"].k.shape[3] * 2
    q, k, v = w[:, :H * d].unflatten(1, (H, d)), w[:, H * d:(H + Hk) * d].unflatten(1, (Hk, d)), w[:, (H + Hk) * d:].unflatten(1, (Hk, d))
    q, k = bbm.bbm_rope(q, k, r.positions, s["freqs"])
    bbm.bbm_kv4_append(k, v, r.slots, s["cache"])
    if s["prompt"]:
        return (r, q, k, v) + bbm.bbm_prompt_attn_fwd(q, k, v, r.cu_new)
    return (r, q, k, v) + bbm.bbm_kv4_attn(q, s["cache"], s["table"], r.lens, r.cu_new)


def test_prompt_then_steps(bbm):
    H, Hk, d, page, lens = 4, 2, 64, 16, [30, 1, 47, 16]
    R = len(lens)
    s = dict(H=H, Hk=Hk, cache=bbm.kv4_cache(40, Hk, d, page), table=i32(np.full((R, 6), -1)), free=i32(np.random.default_rng(1).permutation(40)), at=i32([0]),
             freqs=bbm.rope_freqs(d)[0], ctx=i32([0] * R), new=i32(lens), prompt=True)
    w = normal(1, sum(lens) + 3, (H + 2 * Hk) * d)
    r, q, k, v, o, lse = layer(bbm, s, w)
    n = {a: f64(t) for a, t in (("q", q), ("k", k), ("v", v))}
    cu = np.concatenate([[0], np.cumsum(lens)])
    for h in range(H):
        for a, b in zip(cu, cu[1:]):
            seen = np.tril(np.ones((b - a, b - a), bool))
            x = n["q"][a:b, h], n["k"][a:b, h // 2], n["v"][a:b, h // 2]
            wo, wl, p = ot.attention(*x, seen, d ** -0.5)
            e_o, e_l = ot.bounds(*x, seen, d ** -0.5, p, wo, wl)
            close("O", o[a:b, h], wo, e_o), close("lse", lse[h, a:b], wl, e_l)
    past = [[n[x][a:b] for a, b in zip(cu, cu[1:])] for x in "kv"]
    for step, new in enumerate(([1, 1, 1, 1], [1, 0, 3, 1], [2, 1, 1, 0])):
        s |= dict(ctx=r.lens, at=r.free_next, new=i32(new), prompt=False)
        w = normal(10 + step, sum(new) + 2, (H + 2 * Hk) * d)
        r, q, k, v, o, lse = layer(bbm, s, w)
        cu = np.concatenate([[0], np.cumsum(new)])
        pos = r.positions.cpu().numpy()
        assert r.free_next.item() == sum(-(-len(x) // page) for x in past[0]) + sum(-(-(len(x) + m) // page) - -(-len(x) // page) for x, m in zip(past[0], new))
        for i, (x, t) in enumerate((("k", k), ("v", v))):
            past[i] = [np.concatenate([y, f64(t)[a:b]]) for y, a, b in zip(past[i], cu, cu[1:])]
        for i in range(R):
            a, b, m = cu[i], cu[i + 1], len(past[0][i])
            assert list(pos[a:b]) == list(range(m - new[i], m))
            kk, vv = (ot.kv4_decode(*ot.kv4_encode(y[i])) for y in past)
            seen = np.arange(m) <= m - new[i] + np.arange(new[i])[:, None]
            for h in range(H):
                x = f64(q)[a:b, h], kk[:, h // 2], vv[:, h // 2]
                wo, wl, p = ot.attention(*x, seen, d ** -0.5)
                if new[i]:
                    e_o, e_l = ot.bounds(*x, seen, d ** -0.5, p, wo, wl)
                    close(f"step {step}: O", o[a:b, h], wo, e_o), close("lse", lse[h, a:b], wl, e_l)


def test_training_step_through_the_rotation(bbm):
    """Gradients of w in <attention(rope(q), rope(k), v), d_o>, against differences of the definition in 64 bits."""
    H, Hk, d, lens = 2, 1, 64, [5, 9]
    T, cu = sum(lens), np.concatenate([[0], np.cumsum(lens)])
    pos = np.concatenate([np.arange(n) for n in lens])
    freqs = bbm.rope_freqs(d)[0]
    q, k, v, d_o = normal(1, T, H, d), normal(2, T, Hk, d), normal(3, T, Hk, d), normal(4, T, H, d)
    rq, rk = bbm.bbm_rope(q, k, i32(pos), freqs)
    o, lse = bbm.bbm_prompt_attn_fwd(rq, rk, v, i32(cu))
    dq, dk, dv = bbm.bbm_prompt_attn_bwd(rq, rk, v, o, d_o, lse, i32(cu))
    dq, dk = bbm.bbm_rope(dq, dk, i32(pos), freqs, inverse=True)

    def loss(q, k, v):
        q, k, total = ot.rope(q, pos, f64(freqs), False), ot.rope(k, pos, f64(freqs), False), 0.0
        for a, b in zip(cu, cu[1:]):
            for h in range(H):
                total += (ot.attention(q[a:b, h], k[a:b, 0], v[a:b, 0], np.tril(np.ones((b - a, b - a), bool)), d ** -0.5)[0] * f64(d_o)[a:b, h]).sum()
        return total
    x, grads = [f64(q), f64(k), f64(v)], [f64(dq), f64(dk), f64(dv)]
    g = np.random.default_rng(0)
    for at in range(3):
        step = g.standard_normal(x[at].shape)
        up, down = (loss(*[y + s * 1e-5 * step if i == at else y for i, y in enumerate(x)]) for s in (1, -1))
        want, got = (up - down) / 2e-5, (grads[at] * step).sum()
        # seven roundings to bf16 on the way (rotated q or k, P, dS twice, the gradient, its rotation, O): each moves a term of the sum by at most half
        # a step; with signs at random over the terms, eight times the root of the sum of squares is far out
        size = np.sqrt(((np.abs(grads[at]) + np.abs(grads[at]).mean()) ** 2 * step ** 2).sum())
        assert abs(got - want) <= 8 * 7 * ot.B * size, (at, got, want)


@pytest.mark.parametrize("prompt", [True, False])
def test_graphs_replay(bbm, prompt):
    """A step recorded into a graph: replays give the eager results bit for bit, with eager work between them and other inputs; two graphs of
    one stream do not share memory."""
    H, Hk, d, page, R = 8, 2, 128, 32, 5
    g = np.random.default_rng(2)
    ctx, new = ([0] * R, [40, 3, 100, 1, 64]) if prompt else ([700, 33, 4000, 0, 64], [1, 1, 2, 1, 1])
    T = sum(new) + 4

    def state(seed):
        s = dict(H=H, Hk=Hk, cache=bbm.kv4_cache(200, Hk, d, page), free=i32(np.arange(160, 200)), at=i32([0]), freqs=bbm.rope_freqs(d)[0], ctx=i32(ctx),
                 new=i32(new), prompt=prompt, table=i32(np.arange(R * 140).reshape(R, 140) % 160))
        for t, lo, hi in ((s["cache"].k, 0, 256), (s["cache"].v, 0, 256), (s["cache"].k_scale, 120, 128), (s["cache"].v_scale, 120, 128)):
            t.copy_(torch.from_numpy(np.random.default_rng(seed).integers(lo, hi, t.shape, dtype=np.uint8)))
        return s, normal(seed, T, (H + 2 * Hk) * d)

    def step(s, w):
        r, q, k, v, o, lse = layer(bbm, s, w)
        n = sum(new)
        out = [r.slots, r.positions, q, k, o[:n], lse[:, :n]]
        if prompt:
            out += [t[:n] for t in bbm.bbm_prompt_attn_bwd(q, k, v, o, q, lse, r.cu_new)]
        return out
    states = [state(1), state(2)]
    want = [[t.clone() for t in step(*s)] for s in states]
    torch.cuda.synchronize()
    side, graphs, outs = torch.cuda.Stream(), [], []
    for s in states:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            outs.append(step(*s))
    other = torch.cuda.Stream()
    for replay in range(3):
        for out in outs:
            for t in out:
                t.fill_(5)
        step(*state(7 + replay))                                           # eager work on the default stream
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(other):
            graphs[1].replay()
        torch.cuda.synchronize()
        for i in range(2):
            for n, (a, b) in enumerate(zip(outs[i], want[i])):
                assert torch.equal(a, b), (replay, i, n)


def test_another_stream(bbm):
    """Inputs that a stream still writes when the call is made on it."""
    cu, T, x = prompt_case("ragged", 4, 2, 128, "plain", before=0, behind=0)
    want = bbm.bbm_prompt_attn_fwd(x["q"], x["k"], x["v"], i32(cu))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    cuu = i32(cu)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            a = a @ a * 1e-3
        late = x["q"] + (a[0, 0] * 0).to(torch.bfloat16).nan_to_num()
    late.record_stream(side)
    got = bbm.bbm_prompt_attn_fwd(late, x["k"], x["v"], cuu, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_binding_refuses(bbm):
    q, k = normal(1, 4, 4, 64), normal(2, 4, 2, 64)
    cu, pos, f = i32([0, 4]), i32([0, 1, 2, 3]), bbm.rope_freqs(64)[0]
    c = bbm.kv4_cache(2, 2, 64, 16)
    for bad in (lambda: bbm.bbm_prompt_attn_fwd(q.float(), k, k, cu), lambda: bbm.bbm_prompt_attn_fwd(q, k, k[:3], cu), lambda: bbm.bbm_prompt_attn_fwd(q, k, k, cu.long()),
                lambda: bbm.bbm_prompt_attn_fwd(q.cpu(), k, k, cu), lambda: bbm.bbm_prompt_attn_fwd(q.transpose(0, 2).contiguous().transpose(0, 2), k, k, cu),
                lambda: bbm.bbm_rope(q, k, pos[:3], f), lambda: bbm.bbm_rope(q, k, pos, f.double()), lambda: bbm.bbm_kv4_append(q, q, pos, c),
                lambda: bbm.bbm_kv4_append(k, k, pos.long(), c), lambda: bbm.bbm_kv4_attn(q, c, pos[None], i32([4]), i32([0, 4, 4])),
                lambda: bbm.bbm_kv4_attn(q, c, pos[None], i32([4]), cu, mask=torch.zeros(4, 1, device="cuda")),
                lambda: bbm.bbm_build_slots(pos, pos[:2], pos[:, None], pos, pos[:1], 4, 16)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(bbm.BbmError):
        bbm.bbm_prompt_attn_fwd(normal(1, 4, 3, 64), k, k, cu)
    with pytest.raises(bbm.BbmError):
        bbm.bbm_rope(normal(1, 4, 4, 72), None, pos, f)


def test_slots_of_a_step_without_tokens_or_free_pages(bbm):
    """Outputs of no elements, and an empty list of pages, may lie where the next one begins."""
    ctx, new = i32([40, 16]), i32([3, 0])
    table = i32([[7, 8, 9, -2], [5, -2, -2, -2]])
    for T, free in ((0, i32([3, 4])), (5, table.flatten()[:0]), (0, i32([]))):
        mine = table.clone()
        free = mine.flatten()[:0] if T else free
        r = bbm.bbm_build_slots(ctx, new, mine, free, i32([0]), T, 16)
        assert r.cu_new.tolist() == [0, 3, 3] and r.lens.tolist() == [43, 16] and r.free_next.tolist() == [0] and torch.equal(mine, table)
        assert r.positions.tolist() == [40, 41, 42, 0, 0][:T] and r.slots.tolist() == [9 * 16 + 8, 9 * 16 + 9, 9 * 16 + 10, -1, -1][:T]


# ---- scores of any size


# Scores of 2^base + j 2^gap (j of 0 .. 6, exact in fp32) times 2^scale: small ones, where one step of the running maximum's exponent begins to count, and so on up
# to fp32's range; the later ones are ties of the largest j.
SIZES = [(10, -1, 0), (16, -4, 3), (20, -2, -1), (30, 8, -8), (30, 8, -5), (30, 8, 4), (60, 38, -20), (100, 78, -20), (20, -2, 95), (20, -2, 99), (-80, -100, 99), (100, 78, -100)]


def sized_rows(seed, T, heads, d, sign, base, gap):
    """Keys whose product with sized_query is sign * 2^base + j * 2^gap: two groups of 32 elements that the 4-bit cache holds exactly."""
    g = torch.Generator().manual_seed(seed)
    k = torch.zeros(T, heads, d)
    k[..., 1] = sign * 2.0 ** (base - base // 2)
    k[..., 33] = torch.tensor([0.0, 1, 2, 3, 4, 6])[torch.randint(0, 6, (T, heads), generator=g)] * 2.0 ** gap
    return k.to(torch.bfloat16).cuda()


def sized_query(T, heads, d, base):
    q = torch.zeros(T, heads, d)
    q[..., 1], q[..., 33] = 2.0 ** (base // 2), 1.0
    q[1::3] *= 2.0 ** -20                                                  # rows of other sizes side by side
    return q.to(torch.bfloat16).cuda()


def sized_bounds(seen, p, v, o, lse):
    """Differences of these scores are exact, so an exponent is off by its product's rounding (2^-16 at 2^8, where probabilities end), or by the running maximum's (2^-13 where
    that is kept as a rounded product); the rest as in ot.bounds: P rounded to bf16, sums of n terms, five roundings of the log-sum-exp's own size."""
    n = max(1, int(seen.sum(1).max(initial=0)))
    e_p = 2.0 ** -12 + (n + 32) * ot.F
    return ot.U + ot.B * np.abs(o) + (ot.B * (1 + ot.B) + e_p) * (p @ np.abs(v)), e_p + 8 * ot.F * np.abs(np.where(np.isfinite(lse), lse, 0.0))


@pytest.mark.parametrize("base, gap, scale", SIZES)
@pytest.mark.parametrize("name, H, Hk, d, sign", [("long", 2, 1, 64, 1), ("tiles", 2, 2, 128, -1), ("ragged", 64, 64, 64, 1), ("ragged", 24, 24, 128, -1)])
def test_prompt_scores_of_any_size(bbm, name, H, Hk, d, sign, base, gap, scale):
    lens = LENS[name]
    cu, T = np.concatenate([[0], np.cumsum(lens)]), sum(lens)
    q, k, v = sized_query(T, H, d, base), sized_rows(1, T, Hk, d, sign, base, gap), normal(2, T, Hk, d)
    o, lse = bbm.bbm_prompt_attn_fwd(q, k, v, i32(cu), softmax_scale=2.0 ** scale)
    q, k, v = f64(q), f64(k), f64(v)
    for a, b in zip(cu, cu[1:]):
        seen = np.tril(np.ones((b - a, b - a), bool))
        for h in range(0, H, max(1, H // 6)):
            kk, vv = k[a:b, h * Hk // H], v[a:b, h * Hk // H]
            wo, wl, p = ot.attention(q[a:b, h], kk, vv, seen, 2.0 ** scale)
            e_o, e_l = sized_bounds(seen, p, vv, wo, wl)
            close(f"rows {a}..{b}, head {h}: O", o[a:b, h], wo, e_o), close(f"rows {a}..{b}, head {h}: lse", lse[h, a:b], wl, e_l)


@pytest.mark.parametrize("base, gap, scale", SIZES)
@pytest.mark.parametrize("lens, news, H, Hk, d, sign", [([70, 200], [3, 1], 4, 2, 64, 1), ([2300, 40, 900], [1, 1, 2], 8, 2, 128, -1), ([300, 150], [140, 130], 64, 64, 64, 1),
                                                        ([2500, 2100], [130, 130], 64, 8, 128, -1)])
def test_cached_scores_of_any_size(bbm, lens, news, H, Hk, d, sign, base, gap, scale):
    """The narrow and the wide kernel, whole and in parts."""
    page, n = 32, sum(lens)
    c = bbm.kv4_cache(-(-n // page) + len(lens), Hk, d, page)
    width = max(-(-m // page) for m in lens)
    table, slots, at = np.full((len(lens), width), -1), [], 0
    for r, m in enumerate(lens):
        pages = -(-m // page)
        table[r, :pages] = np.arange(at, at + pages)
        slots += list(at * page + np.arange(m))
        at += pages
    v = normal(2, n, Hk, d)
    bbm.bbm_kv4_append(sized_rows(1, n, Hk, d, sign, base, gap), v, i32(slots), c)
    hk, hv = host_cache(c)
    cu, T = np.concatenate([[0], np.cumsum(news)]), sum(news)
    q = sized_query(T, H, d, base)
    o, lse = bbm.bbm_kv4_attn(q, c, i32(table), i32(lens), i32(cu), softmax_scale=2.0 ** scale, max_len=max(lens))
    q = f64(q)
    for r, m in enumerate(lens):
        a, b = cu[r], cu[r + 1]
        seen = np.arange(m) <= m - news[r] + np.arange(b - a)[:, None]
        pg, j = table[r, np.arange(m) // page], np.arange(m) % page
        for h in range(0, H, max(1, H // 6)):
            kk, vv = hk[pg, h * Hk // H, j], hv[pg, h * Hk // H, j]
            assert np.abs(kk).max() >= 2.0 ** (base // 2)
            wo, wl, p = ot.attention(q[a:b, h], kk, vv, seen, 2.0 ** scale)
            e_o, e_l = sized_bounds(seen, p, vv, wo, wl)
            close(f"request {r}, head {h}: O", o[a:b, h], wo, e_o), close(f"request {r}, head {h}: lse", lse[h, a:b], wl, e_l)


def test_prompt_rows_that_see_keys_of_1e30(bbm):
    """Keys of 1e30 share a row among themselves where their scores are positive, and leave it to the others where they are not."""
    cu, T, x = prompt_case("long", 1, 1, 64, "plain", seed=4)
    a, b, m = int(cu[0]), int(cu[1]), 40
    x["k"][b - m:b], x["v"][b - m:b] = 1e30, -1e30
    o, lse = bbm.bbm_prompt_attn_fwd(x["q"], x["k"], x["v"], i32(cu))
    n = {t: f64(y)[a:b, 0] for t, y in x.items()}
    rows = np.arange(b - m, b) - a
    large = n["q"][rows].sum(1) > 0
    assert 5 < large.sum() < m - 5
    seen = (np.arange(b - a) <= rows[:, None]) & ((np.arange(b - a) >= b - m - a) == large[:, None])     # (the weight of the other keys is an exact zero)
    q = n["q"][rows]
    wo, wl, p = ot.attention(q, n["k"], n["v"], seen, 0.125)
    e_o, e_l = ot.bounds(q, n["k"], n["v"], seen, 0.125, p, wo, wl)
    got_o, got_l = o[a + rows, 0], lse[0, a + rows]
    close("O, others", got_o[torch.from_numpy(~large).cuda()], wo[~large], e_o[~large]), close("lse, others", got_l[torch.from_numpy(~large).cuda()], wl[~large], e_l[~large])
    # equal scores, an average of equal values: P is 1 or a power of two's neighbour, rounded once, and so is the result
    close("O", got_o[torch.from_numpy(large).cuda()], wo[large], (2 * ot.B + 2.0 ** -12) * np.abs(wo[large]))
    close("lse", got_l[torch.from_numpy(large).cuda()], wl[large], e_l[large])


def test_gradients_of_scores_up_to_2000(bbm):
    cu, T, x = prompt_case("ragged", 4, 2, 64, "plain", seed=12, scale=8.0)
    check_prompt(bbm, cu, T, x, 4, 2, 64, scale=1.0)


# ---- outputs in other layouts, and without a log-sum-exp


def output_in(layout, T, H, d):
    """(packed output, the memory that it is a part of), all sevens."""
    if layout == "fused":
        whole = torch.full((T, (H + 3) * d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
        return whole[:, d:(H + 1) * d].unflatten(1, (H, d)), whole
    whole = torch.full((H + 2, T + 3, d), 7.0, dtype=torch.bfloat16, device="cuda")
    return whole[1:H + 1, 2:T + 2].transpose(0, 1), whole


def same_and_nothing_else(part, whole, want, rows):
    """`want` in these rows of the part, and sevens in the rest of what it is a part of."""
    assert torch.equal(part[rows], want[rows])
    part[rows] = 7.0
    assert (whole == 7.0).all(), "written outside the output's rows"


OUT_LAYOUTS = pytest.mark.parametrize("layout", ["fused", "heads"])


@OUT_LAYOUTS
@pytest.mark.parametrize("name, H, Hk, d", [("ragged", 4, 2, 64), ("longer", 5, 1, 64), ("longer", 5, 1, 128), ("tiles", 3, 1, 128), ("longer", 40, 8, 128), ("longer", 64, 16, 64), ("many", 2, 2, 64)])
def test_prompt_outputs_in_other_layouts(bbm, name, H, Hk, d, layout):
    """Whole and halved tiles, dK and dV whole and in parts."""
    cu, T, x = prompt_case(name, H, Hk, d, "plain", seed=14)
    rows = slice(int(cu[0]), int(cu[-1]))
    args = x["q"], x["k"], x["v"]
    wo, wl = bbm.bbm_prompt_attn_fwd(*args, i32(cu))
    wg = bbm.bbm_prompt_attn_bwd(*args, wo, x["d_o"], wl, i32(cu))
    o, o_all = output_in(layout, T, H, d)
    grads = [output_in(layout, T, h, d) for h in (H, Hk, Hk)]
    got, _ = bbm.bbm_prompt_attn_fwd(*args, i32(cu), out=o)
    assert got is o
    bbm.bbm_prompt_attn_bwd(*args, o, x["d_o"], wl, i32(cu), **{n: g[0] for n, g in zip(("dq", "dk", "dv"), grads)})
    same_and_nothing_else(o, o_all, wo, rows)
    for (part, whole), want in zip(grads, wg):
        same_and_nothing_else(part, whole, want, rows)


CACHED = [([63, 200, 1, 0], [1, 3, 1, 1], 8, 2, 64), ([63, 200, 1, 0], [1, 3, 1, 1], 3, 1, 128), ([2900, 9, 1700], [1, 1, 2], 12, 4, 64), ([9000, 40], [1, 2], 4, 2, 128),
          ([300, 150], [140, 130], 64, 64, 64), ([300, 150], [140, 130], 64, 64, 128), ([2500, 2100], [130, 130], 64, 8, 64), ([2500, 2100], [130, 130], 64, 8, 128)]


@OUT_LAYOUTS
@pytest.mark.parametrize("lens, news, H, Hk, d", CACHED)
def test_cached_outputs_in_other_layouts(bbm, lens, news, H, Hk, d, layout):
    """Few columns and many, whole, in a few parts and in more than four."""
    c, table, cu, T, q, _ = cached_case(bbm, lens, news, H, Hk, d, 32, seed=15, before=2, behind=3)
    args = q, c, i32(table), i32(lens), i32(cu)
    want, _ = bbm.bbm_kv4_attn(*args, max_len=max(lens))
    o, o_all = output_in(layout, T, H, d)
    bbm.bbm_kv4_attn(*args, max_len=max(lens), out=o)
    same_and_nothing_else(o, o_all, want, slice(int(cu[0]), int(cu[-1])))


@OUT_LAYOUTS
@pytest.mark.parametrize("rot, interleaved", [(64, False), (62, False), (40, True)])
def test_rope_and_read_into_other_layouts(bbm, rot, interleaved, layout):
    T, H, Hk, d, page = 70, 6, 2, 64, 16
    q, k, pos, f = normal(1, T, H, d), normal(2, T, Hk, d), i32(np.arange(T) * 3), bbm.rope_freqs(rot)[0]
    want = bbm.bbm_rope(q, k, pos, f, interleaved=interleaved)
    (oq, q_all), (ok, k_all) = output_in(layout, T, H, d), output_in(layout, T, Hk, d)
    bbm.bbm_rope(q, k, pos, f, interleaved=interleaved, out_q=oq, out_k=ok)
    c = bbm.kv4_cache(6, Hk, d, page)
    slots = i32(np.arange(T))
    bbm.bbm_kv4_append(k, q[:, :Hk], slots, c)
    read = bbm.bbm_kv4_read(slots, c)
    (rk, rk_all), (rv, rv_all) = output_in(layout, T, Hk, d), output_in(layout, T, Hk, d)
    bbm.bbm_kv4_read(slots, c, out_k=rk, out_v=rv)
    for part, whole, x in ((oq, q_all, want[0]), (ok, k_all, want[1]), (rk, rk_all, read[0]), (rv, rv_all, read[1])):
        same_and_nothing_else(part, whole, x, slice(0, T))


def c_packed(x):
    """The C structure of a packed tensor."""
    import ctypes
    from paper_2409_15097_amd.tokens import _CPacked
    return ctypes.byref(_CPacked(x.data_ptr(), x.stride(0), x.stride(1)))


@pytest.mark.parametrize("name, H, Hk, d", [("ragged", 4, 2, 64), ("longer", 40, 8, 128)])
def test_prompt_without_a_log_sum_exp(bbm, name, H, Hk, d):
    cu, T, x = prompt_case(name, H, Hk, d, "plain", seed=16)
    want, _ = bbm.bbm_prompt_attn_fwd(x["q"], x["k"], x["v"], i32(cu))
    o, offsets = torch.full_like(want, 7.0), i32(cu)
    stream = torch.cuda.current_stream().cuda_stream
    assert bbm.lib.bbm_prompt_attn_fwd(*(c_packed(x[n]) for n in "qkv"), c_packed(o), None, T, len(cu) - 1, offsets.data_ptr(), H, Hk, d, d ** -0.5, stream) == bbm.BBM_OK
    rows = slice(int(cu[0]), int(cu[-1]))
    assert torch.equal(o[rows], want[rows])


@pytest.mark.parametrize("lens, news, H, Hk, d", CACHED)
def test_cached_without_a_log_sum_exp(bbm, lens, news, H, Hk, d):
    import ctypes
    c, table, cu, T, q, _ = cached_case(bbm, lens, news, H, Hk, d, 32, seed=17)
    tab, ln, offsets, R = i32(table), i32(lens), i32(cu), len(lens)
    want, _ = bbm.bbm_kv4_attn(q, c, tab, ln, offsets, max_len=max(lens))
    need = bbm.bbm_kv4_attn_workspace_bytes(T, R, H, Hk, d, max(lens))
    ws, o = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), torch.full_like(want, 7.0)
    assert bbm.lib.bbm_kv4_attn(c_packed(q), c_packed(o), None, T, R, offsets.data_ptr(), ln.data_ptr(), tab.data_ptr(), tab.stride(0), tab.shape[1], None, 0,
                                ctypes.byref(c.c_struct), H, d ** -0.5, max(lens), ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == bbm.BBM_OK
    assert torch.equal(o, want)


@pytest.mark.parametrize("d", [64, 128])
def test_gradients_round_the_score_gradient_once(bbm, d):
    """Pairs of tokens: a row of dK (and dQ) is one or two terms, so a second rounding on the way to it shows.  The bound is that of ot.bounds with one rounding of dS to bf16, from
    an fp32 probability, and one of the result."""
    pairs, H = 300, 4
    cu, T = np.arange(pairs + 1) * 2, 2 * pairs
    q, k, v, d_o = (normal(30 + i, T, H, d) for i in range(4))
    o, lse = bbm.bbm_prompt_attn_fwd(q, k, v, i32(cu))
    dq, dk, _ = bbm.bbm_prompt_attn_bwd(q, k, v, o, d_o, lse, i32(cu))
    q, k, v, d_o, o = (f64(t) for t in (q, k, v, d_o, o))
    want, tol = ([np.zeros((T, H, d)) for _ in range(2)] for _ in range(2))
    sm, seen = d ** -0.5, np.tril(np.ones((2, 2), bool))
    for a in cu[:-1]:
        for h in range(H):
            at = slice(a, a + 2), h
            wo, wl, p = ot.attention(q[at], k[at], v[at], seen, sm)
            delta = (d_o[at] * o[at]).sum(1)
            g = ot.attention_bwd(q[at], k[at], v[at], d_o[at], p, sm, delta)
            e_l = ot.bounds(q[at], k[at], v[at], seen, sm, p, wo, wl)[1]
            e_s = ((d + 8) * ot.F + 32 * ot.F) * sm * (np.abs(q[at]) @ np.abs(k[at]).T) + 32 * ot.F
            dp_mag = np.abs(d_o[at]) @ np.abs(v[at]).T + (np.abs(d_o[at]) * np.abs(o[at])).sum(1)[:, None]
            ds = p * np.abs(d_o[at] @ v[at].T - delta[:, None])
            e_ds = (ot.B + e_s + e_l[:, None] + 32 * ot.F) * ds + p * (d + 8) * ot.F * dp_mag
            for i, (x, e) in enumerate(((k[at], e_ds), (q[at], e_ds.T))):
                want[i][at] = g[i]
                tol[i][at] = ot.U + ot.B * np.abs(g[i]) + (1 + ot.B) * sm * (e @ np.abs(x)) + 4 * ot.F * sm * ((ds if i == 0 else ds.T) @ np.abs(x))
    close("dQ", dq, want[0], tol[0]), close("dK", dk, want[1], tol[1])
