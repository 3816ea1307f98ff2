"""GPU: the operators on the cache of many and long answers against their definitions in 64 bits (oracle/tokens.py), at the sizes, groups and masks where they can go wrong.
Tolerances are the bounds derived there from the roundings that the kernels make."""
import numpy as np
import pytest
import torch

from oracle import tokens as ot
from test_gpu_tokens import (OUT_LAYOUTS, SIZES, c_packed, cached_case, check_cached, close, f64, host_cache, i32, normal, output_in, same_and_nothing_else, sized_bounds, sized_query,
                             sized_rows)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bbm():
    import paper_2409_15097_amd as m
    return m


# ---- attention behind shared prefixes


class Behind:
    """bbm_kv4_attn by way of the groups."""

    def __init__(self, bbm, group_cu, shared):
        self.bbm, self.groups = bbm, (None if group_cu is None else i32(group_cu), None if shared is None else i32(shared))
        self.kv4_cache = bbm.kv4_cache

    def bbm_kv4_attn(self, q, cache, table, lens, cu, **kw):
        return self.bbm.bbm_kv4_shared_attn(q, cache, table, lens, cu, *self.groups, **kw)


def grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, page, **kw):
    """cached_case whose groups have the pages of their shared keys in common (a page that they share in part is each request's own)."""
    case = cached_case(bbm, lens, news, H, Hk, d, page, **kw)
    table = case[1]
    for g, n in enumerate(shared):
        first = group_cu[g]
        for r in range(first + 1, group_cu[g + 1]):
            table[r, :max(0, n) // page] = table[first, :max(0, n) // page]
    return case


def check_grouped(bbm, group_cu, shared, lens, news, H, Hk, d, page, hints=({},), **kw):
    c, table, cu, T, q, words = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, page, **kw)
    by = Behind(bbm, group_cu, shared)
    for hint in hints:
        a = check_cached(by, c, table, lens, cu, T, q, words, H, Hk, d, page, **hint)
        out, lse = torch.full_like(a[0], 7.0), torch.full_like(a[1], 7.0)
        by.bbm_kv4_attn(q, c, i32(table), i32(lens), i32(cu), mask=None if words is None else torch.from_numpy(words).cuda(), out=out, lse=lse, **hint)
        assert torch.equal(a[0], out) and torch.equal(a[1], lse)
    return c, table, cu, T, q, words


# What the work split goes by, besides the table (None).
NEAR = [{}, dict(max_shared=300, max_own=40), dict(max_shared=5000, max_own=40), dict(max_shared=1200, max_own=5000)]   # (short ones: each request for itself)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group_cu, shared, lens, news, H, Hk, page, layout, tree", [
    ([0, 1], [16], [17], [1], 1, 1, 16, "plain", None),
    ([0, 4], [48], [49, 60, 52, 100], [1] * 4, 8, 2, 16, "fused", None),
    ([1, 3, 3, 6], [37, 500, 130], [20, 40, 38, 131, 150, 300, 9], [1, 2, 1, 1, 0, 5, 3], 6, 2, 32, "heads", None),     # alone in front and behind, a group of nobody, keys that end inside a page
    ([0, 2, 5], [0, -3], [30, 1, 70, 0, 2], [1, 1, 9, 0, 2], 4, 4, 16, "plain", None),                                     # nothing is shared
    ([0, 3], [15], [20, 19, 16], [1, 4, 1], 4, 1, 16, "plain", None),                                                        # less than a block
    ([0, 3], [200], [206, 230, 204], [6, 30, 4], 3, 1, 64, "plain", 1),
    ([0, 2, 4], [128, 64], [200, 270, 150, 64], [70, 129, 66, 0], 5, 1, 128, "heads", 2),
    ([0, 30], [96], [100 + i for i in range(30)], [1 + i % 3 for i in range(30)], 16, 2, 32, "plain", None),
    ([0, 2], [2304], [2400, 2310], [3, 1], 12, 4, 64, "fused", None)])
def test_shared(bbm, group_cu, shared, lens, news, H, Hk, d, page, layout, tree):
    check_grouped(bbm, group_cu, shared, lens, news, H, Hk, d, page, hints=NEAR, layout=layout, tree=tree, seed=len(lens), before=2, behind=3)


@pytest.mark.parametrize("d, H, Hk, tree", [(64, 64, 8, None), (128, 64, 8, None), (128, 64, 16, 1), (64, 40, 40, None)])
def test_shared_by_many_columns(bbm, d, H, Hk, tree):
    """The kernel of many columns for the groups, in parts; alone and beside requests of few and of many."""
    for lens, news in (([2100, 2088], [60, 70]), ([1100 + i for i in range(40)], [1 + i % 15 for i in range(40)])):
        check_grouped(bbm, [0, len(lens)], [1072 if len(lens) > 2 else 2016], lens, news, H, Hk, d, 16, hints=[{}, dict(max_shared=2048, max_own=100), dict(max_shared=20000, max_own=5000)], tree=tree, seed=9, before=1, behind=2)


def test_shared_by_one_and_by_many_requests(bbm):
    """More requests, and more groups, than are counted or read at once."""
    R = 600
    lens, hints = [33 + i % 9 for i in range(R)], [{}, dict(max_shared=4096, max_own=16)]
    check_grouped(bbm, [0, R], [32], lens, [1] * R, 2, 1, 64, 16, hints=hints)
    check_grouped(bbm, list(range(0, R + 1, 8)), [16 * (i % 3) for i in range(75)], lens, [1] * R, 2, 1, 64, 16, hints=hints)
    check_grouped(bbm, list(range(R + 1)), [16 * (i % 3) for i in range(R)], lens, [1] * R, 2, 1, 64, 16, hints=hints)


def test_shared_pages_outside_and_a_narrow_table(bbm):
    group_cu, shared, lens, news, H, Hk, d, page = [0, 2, 4], [256, 64], [500, 300, 90, 70], [1, 3, 2, 1], 4, 2, 128, 32
    c, table, cu, T, q, _ = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, page, seed=3)
    table[:2, 3], table[0, 15], table[2:, 0], table[3, 2] = -1, 1 << 30, c.k.shape[0], -5
    by = Behind(bbm, group_cu, shared)
    check_cached(by, c, table, lens, cu, T, q, None, H, Hk, d, page, max_shared=4096)
    check_cached(by, c, table[:, :9], lens, cu, T, q, None, H, Hk, d, page)
    check_cached(by, c, table[:, :9], lens, cu, T, q, None, H, Hk, d, page, max_shared=4096)
    # a prefix that ends behind the table, and one of which no page is there: the queries behind it see what is left, or nothing
    check_cached(by, c, table[:, :5], [700, 600, 90, 70], cu, T, q, None, H, Hk, d, page, max_shared=4096)
    gone = table.copy()
    gone[2:] = -1
    check_cached(by, c, gone, lens, cu, T, q, None, H, Hk, d, page, max_shared=4096)


@pytest.mark.parametrize("tree", [None, 1])
@pytest.mark.parametrize("front, rows", [(0, 3), (17, 5)])
def test_shared_rows_that_are_not_there(bbm, tree, front, rows):
    """Offsets that begin in front of the first row or end behind the last: the tokens without a row are in the cache all the same."""
    lens, news, H = [300, 290, 170], [40, 30, 60], 4
    c, table, cu, T, q, words = grouped_case(bbm, [0, 3], [96], lens, news, H, 2, 64, 32, seed=11, tree=tree)
    a, b = front, news[0] + news[1] + rows
    for hint in ({}, dict(max_shared=4096)):
        check_cached(Behind(bbm, [0, 3], [96]), c, table, lens, cu - a, b - a, q[a:b].contiguous(), None if words is None else words[a:b].copy(), H, 2, 64, 32, **hint)


@pytest.mark.parametrize("max_shared, max_own", [(1, 1), (300, 5000), (5000, 1), (1 << 40, 1 << 40)])
def test_shared_with_a_wrong_hint(bbm, max_shared, max_own):
    check_grouped(bbm, [0, 2], [2048], [2300, 2100], [1, 2], 4, 2, 64, 64, hints=[dict(max_shared=max_shared, max_own=max_own)], seed=5)


@pytest.mark.parametrize("lens, news", [([2300, 40, 900], [1, 2, 1]), ([300, 150], [140, 130])])
def test_shared_by_nobody_is_the_attention_of_each(bbm, lens, news):
    """Without groups the results are those of bbm_kv4_attn, bit for bit."""
    c, table, cu, T, q, _ = cached_case(bbm, lens, news, 64, 8, 64, 32, seed=4)
    args = q, c, i32(table), i32(lens), i32(cu)
    want = bbm.bbm_kv4_attn(*args, max_len=2300)
    for groups in ((None, None), (i32([0]), i32([]))):
        got = bbm.bbm_kv4_shared_attn(*args, *groups, max_own=2300)
        assert all(torch.equal(x, y) for x, y in zip(got, want))


GROUPED = [([2300, 2290, 2400], [1, 1, 2], 8, 2, 64), ([2300, 2290, 2400], [1, 1, 2], 8, 2, 128), ([2300, 2320, 2350], [130, 130, 130], 8, 1, 64), ([2300, 2320, 2350], [130, 130, 130], 8, 1, 128)]


@pytest.mark.parametrize("base, gap, scale", SIZES)
@pytest.mark.parametrize("lens, news, H, Hk, d, sign", [([170, 200, 165], [3, 1, 1], 4, 2, 64, 1), ([1300, 1290], [130, 130], 8, 2, 128, -1)])
def test_shared_scores_of_any_size(bbm, lens, news, H, Hk, d, sign, base, gap, scale):
    """Sums of a prefix and of what lies behind it meet under one maximum: few columns and many."""
    page, shared = 32, 96 if len(lens) == 3 else 1024
    n, R = sum(lens), len(lens)
    c = bbm.kv4_cache(-(-n // page) + R, Hk, d, page)
    width = max(-(-m // page) for m in lens)
    table, slots, at = np.full((R, width), -1), [], 0
    for r, m in enumerate(lens):
        pages = -(-m // page)
        table[r, :pages] = np.arange(at, at + pages)
        slots += list(at * page + np.arange(m))
        at += pages
    bbm.bbm_kv4_append(sized_rows(1, n, Hk, d, sign, base, gap), normal(2, n, Hk, d), i32(slots), c)
    table[1:, :shared // page] = table[0, :shared // page]
    hk, hv = host_cache(c)
    cu, T = np.concatenate([[0], np.cumsum(news)]), sum(news)
    q = sized_query(T, H, d, base)
    o, lse = bbm.bbm_kv4_shared_attn(q, c, i32(table), i32(lens), i32(cu), i32([0, R]), i32([shared]), softmax_scale=2.0 ** scale, max_shared=4096, max_own=300)
    q = f64(q)
    for r, m in enumerate(lens):
        a, b = cu[r], cu[r + 1]
        seen = np.arange(m) <= m - news[r] + np.arange(b - a)[:, None]
        pg, j = table[r, np.arange(m) // page], np.arange(m) % page
        for h in range(0, H, max(1, H // 4)):
            kk, vv = hk[pg, h * Hk // H, j], hv[pg, h * Hk // H, j]
            wo, wl, p = ot.attention(q[a:b, h], kk, vv, seen, 2.0 ** scale)
            e_o, e_l = sized_bounds(seen, p, vv, wo, wl)
            close(f"request {r}, head {h}: O", o[a:b, h], wo, e_o), close(f"request {r}, head {h}: lse", lse[h, a:b], wl, e_l)


@OUT_LAYOUTS
@pytest.mark.parametrize("lens, news, H, Hk, d", GROUPED)
def test_shared_outputs_in_other_layouts(bbm, lens, news, H, Hk, d, layout):
    c, table, cu, T, q, _ = grouped_case(bbm, [0, 3], [2048], lens, news, H, Hk, d, 32, seed=15, before=2, behind=3)
    args = q, c, i32(table), i32(lens), i32(cu), i32([0, 3]), i32([2048])
    want, _ = bbm.bbm_kv4_shared_attn(*args)
    o, o_all = output_in(layout, T, H, d)
    bbm.bbm_kv4_shared_attn(*args, out=o)
    same_and_nothing_else(o, o_all, want, slice(int(cu[0]), int(cu[-1])))


@pytest.mark.parametrize("rows", [[0], [5], [1, 2, 40]])
@pytest.mark.parametrize("group_cu, shared, lens, news, H, Hk, d, tree", [
    ([0, 3], [48], [55, 60, 52], [3, 4, 2], 6, 2, 64, None), ([0, 2], [2304], [2400, 2310], [3, 3], 12, 4, 128, 1), ([0, 40], [640], [660 + i for i in range(40)], [3] * 40, 6, 2, 128, None),
    ([0, 70], [2048], [2060 + i for i in range(70)], [1] * 70, 8, 2, 64, None), ([0, 2], [256], [400, 420], [130, 90], 8, 2, 128, None)])
def test_shared_queries_that_are_no_numbers(bbm, group_cu, shared, lens, news, H, Hk, d, tree, rows):
    """Rows beside one whose query holds no number are what they should be (to the bit they need not be: a maximum moves when one of its wave's does)."""
    c, table, cu, T, q, words = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, 16, seed=9, tree=tree)
    rows = [r for r in rows if r < T]

    class Beside(Behind):
        def bbm_kv4_attn(self, q, *args, out, lse, **kw):
            super().bbm_kv4_attn(q, *args, out=out, lse=lse, **kw)
            bad, o, l = q.clone(), out.clone(), lse.clone()
            bad[rows] = value
            super().bbm_kv4_attn(bad, *args, out=o, lse=l, **kw)
            others = [r for r in range(T) if r not in rows]
            out[others], lse[:, others] = o[others], l[:, others]
            return out, lse

    for value in (float("nan"), float("inf")):
        for hint in NEAR:
            check_cached(Beside(bbm, group_cu, shared), c, table, lens, cu, T, q, words, H, Hk, d, 16, **hint)


@pytest.mark.parametrize("lens, news, H, Hk, d", GROUPED)
def test_shared_without_a_log_sum_exp(bbm, lens, news, H, Hk, d):
    import ctypes
    c, table, cu, T, q, _ = grouped_case(bbm, [0, 3], [2048], lens, news, H, Hk, d, 32, seed=17)
    tab, ln, offsets, gc, sh = i32(table), i32(lens), i32(cu), i32([0, 3]), i32([2048])
    want, _ = bbm.bbm_kv4_shared_attn(q, c, tab, ln, offsets, gc, sh, max_shared=2048, max_own=400)
    need = bbm.bbm_kv4_shared_attn_workspace_bytes(T, 3, 1, H, Hk, d, 2048, 400)
    ws, o = torch.full((need,), 255, dtype=torch.uint8, device="cuda"), torch.full_like(want, 7.0)
    assert bbm.lib.bbm_kv4_shared_attn(c_packed(q), c_packed(o), None, T, 3, offsets.data_ptr(), ln.data_ptr(), tab.data_ptr(), tab.stride(0), tab.shape[1], 1, gc.data_ptr(), sh.data_ptr(),
                                       None, 0, ctypes.byref(c.c_struct), H, d ** -0.5, 2048, 400, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == bbm.BBM_OK
    assert torch.equal(o, want)


def test_groups_whose_numbers_are_wrong_stay_inside(bbm):
    """Offsets outside the requests or out of order, and prefixes longer than requests: nobody else's rows change, and other groups keep their results."""
    group_cu, shared, lens, news, H, Hk, d, page = [0, 2, 4], [64, 32], [90, 80, 70, 60], [1, 1, 1, 1], 4, 2, 64, 16
    c, table, cu, T, q, _ = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, page, seed=8, before=2, behind=2)
    args = q, c, i32(table), i32(lens), i32(cu)
    want = bbm.bbm_kv4_shared_attn(*args, i32(group_cu), i32(shared), max_shared=4096)
    for wrong, n in (([0, 2, 9], [64, 32]), ([-7, 2, 4], [64, 32]), ([0, 2, 4], [64, 1 << 30]), ([0, 2, 1], [64, 32]), ([0, 2, 4], [64, 80])):
        out, lse = torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((H, T), 7.0, device="cuda")
        bbm.bbm_kv4_shared_attn(*args, i32(wrong), i32(n), out=out, lse=lse, max_shared=4096)
        assert (f64(out)[:2] == 7).all() and (f64(out)[-2:] == 7).all() and torch.equal(out[2:4], want[0][2:4]) and torch.equal(lse[:, 2:4], want[1][:, 2:4])


# ---- weights of the keys


def check_weights(bbm, group_cu, shared, c, table, lens, cu, T, q, words, H, Hk, d, page, lse=None, decay=0.75, seed=0, hints=({},)):
    """Against the definition; returns what was gathered."""
    mask = None if words is None else torch.from_numpy(words).cuda()
    groups = (None, None) if group_cu is None else (i32(group_cu), i32(shared))
    args = c, i32(table), i32(lens), i32(cu)
    if lse is None:
        _, lse = bbm.bbm_kv4_attn(q, *args, mask=mask)
    g = torch.Generator().manual_seed(seed)
    old = torch.rand(c.k.shape[:3], generator=g).mul_(3)
    R, G, page_n = len(lens), H // Hk, c.k.shape[0]
    hk, _ = host_cache(c)
    nq, nl = f64(q), f64(lse)
    want, tol, written = f64(old), np.zeros(old.shape), np.zeros(old.shape, bool)
    of = {r: g for g in range(len(shared or [])) for r in range(group_cu[g], group_cu[g + 1])}
    decayed = set()
    fresh_slots = []
    for r, n in enumerate(lens):
        a, b, new = max(0, int(cu[r])), min(T, int(cu[r + 1])), int(cu[r + 1] - cu[r])
        if b <= a:
            continue
        m = min(max(n, 0), table.shape[1] * page)
        common = min(max(0, shared[of[r]]) // 16 * 16, m) if r in of else 0
        j, i = np.arange(m), np.arange(a, b)[:, None] - int(cu[r])
        row = np.where(j < common, group_cu[of[r]] if r in of else r, r)
        pg = table[row, j // page]
        ok = (pg >= 0) & (pg < page_n)
        if words is None:
            seen = (j <= n - new + i) & ok
        else:
            nj = j - (n - new)
            bit = np.zeros((b - a, m), bool)
            inside = (nj >= 0) & (nj < 64 * words.shape[1])
            bit[:, inside] = (words[a:b][:, nj[inside] // 64] >> (nj[inside] % 64)) & 1 != 0
            seen = ((nj < 0) | bit) & ok
        for h in range(Hk):
            k = np.where(ok[:, None], hk[np.where(ok, pg, 0), h, j % page], 0.0)
            gained = [ot.key_weights(nq[a:b, h * G + x], k, seen, d ** -0.5, nl[h * G + x, a:b]) for x in range(G)]
            for jj in np.nonzero(ok)[0]:
                at = (int(pg[jj]), h, int(jj) % page)
                if at not in decayed:
                    decayed.add(at)
                    want[at] = 0.0 if jj >= n - new else want[at] * np.float64(np.float32(decay))
                    tol[at] += 4 * ot.F * want[at]
                want[at] += sum(x[0][jj] for x in gained)
                tol[at] += sum(x[1][jj] for x in gained)
                written[at] = True
        if words is not None or n - new < m:
            fresh_slots += [(int(table[r, jj // page]), jj % page) for jj in range(max(0, n - new, common), m) if 0 <= table[r, jj // page] < page_n]
    # the sums of all queries of a group meet in one number: as many half steps of it as there are terms
    tol += 2 * ot.F * (T * G + 16) * np.abs(want)
    got = None
    for hint in hints:
        for inplace in (False, True):
            w = old.clone().cuda()
            for p, at in fresh_slots:                                     # whatever lay where new tokens went
                w[p, :, at] = float("nan")
            src, out = w.clone(), (w if inplace else torch.full_like(w, 7.0))
            r = bbm.bbm_kv4_weights(q, lse, *args, src if not inplace else w, *groups, mask=mask, decay=decay, out=None if inplace else out, **hint)
            assert r is out
            now = f64(out)
            close("weights", torch.from_numpy(now[written]), want[written], tol[written])
            rest = now[~written]
            assert np.array_equal(rest, f64(src)[~written], equal_nan=True) if inplace else (rest == 7.0).all()
            assert got is None or hint or torch.equal(got[torch.from_numpy(written).cuda()], out[torch.from_numpy(written).cuda()])
            got = out.clone() if not hint else got
    return got


WEIGHTS = [
    ([0], [], [1], [1], 1, 1, 16, "plain", None),
    ([0], [], [0, 3, 17, 40], [1, 1, 1, 0], 4, 2, 16, "fused", None),
    ([0], [], [63, 64, 65, 200, 1, 0], [1] * 6, 8, 1, 32, "plain", None),
    ([0], [], [130, 300, 31], [30, 17, 31], 6, 2, 64, "heads", None),                  # a prompt's part; a whole prompt
    ([0], [], [2900, 9, 1700], [1, 1, 2], 12, 4, 64, "plain", None),
    ([0], [], [300, 129], [70, 129], 3, 1, 128, "heads", 2),
    ([0], [], [20, 70, 5], [20, 6, 5], 4, 4, 16, "plain", 1),
    ([0], [], [40, 90], [40, 60], 71, 1, 32, "plain", None),
    ([0, 4], [48], [49, 60, 52, 100], [1] * 4, 8, 2, 16, "fused", None),
    ([1, 3, 3, 6], [37, 500, 130], [20, 40, 38, 131, 150, 300, 9], [1, 2, 1, 1, 0, 5, 3], 6, 2, 32, "heads", None),
    ([0, 3], [200], [206, 230, 204], [6, 30, 4], 3, 1, 64, "plain", 1),
    ([0, 30], [96], [100 + i for i in range(30)], [1 + i % 3 for i in range(30)], 16, 2, 32, "plain", None),
    ([0, 2], [2304], [2400, 2310], [3, 1], 12, 4, 64, "fused", None)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group_cu, shared, lens, news, H, Hk, page, layout, tree", WEIGHTS)
def test_weights(bbm, group_cu, shared, lens, news, H, Hk, d, page, layout, tree):
    c, table, cu, T, q, words = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, page, layout=layout, tree=tree, seed=len(lens), before=2, behind=3)
    check_weights(bbm, group_cu if shared else None, shared, c, table, lens, cu, T, q, words, H, Hk, d, page, seed=1, hints=[{}, dict(max_shared=300, max_own=40), dict(max_shared=1, max_own=1)])


def test_weights_pages_outside_and_a_narrow_table(bbm):
    group_cu, shared, lens, news, H, Hk, d, page = [0, 2, 4], [256, 64], [500, 300, 90, 70], [1, 3, 2, 1], 4, 2, 128, 32
    c, table, cu, T, q, _ = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, page, seed=3)
    table[:2, 3], table[0, 15], table[2:, 0], table[3, 2] = -1, 1 << 30, c.k.shape[0], -5
    for t, n in ((table, lens), (table[:, :9], lens), (table[:, :5], [700, 600, 90, 70])):
        check_weights(bbm, group_cu, shared, c, t, n, cu, T, q, None, H, Hk, d, page)


@pytest.mark.parametrize("front, rows", [(0, 3), (17, 5)])
@pytest.mark.parametrize("tree", [None, 1])
def test_weights_rows_that_are_not_there(bbm, tree, front, rows):
    lens, news, H = [300, 290, 170], [40, 30, 60], 4
    c, table, cu, T, q, words = grouped_case(bbm, [0], [], lens, news, H, 2, 64, 32, seed=11, tree=tree)
    a, b = front, news[0] + news[1] + rows
    check_weights(bbm, None, None, c, table, lens, cu - a, b - a, q[a:b].contiguous(), None if words is None else words[a:b].copy(), H, 2, 64, 32)


def test_weights_of_many_requests(bbm):
    R = 600
    c, table, cu, T, q, _ = grouped_case(bbm, list(range(0, R + 1, 8)), [16 * (i % 3) for i in range(75)], [33 + i % 9 for i in range(R)], [1] * R, 2, 1, 64, 16)
    check_weights(bbm, list(range(0, R + 1, 8)), [16 * (i % 3) for i in range(75)], c, table, [33 + i % 9 for i in range(R)], cu, T, q, None, 2, 1, 64, 16)


def test_weights_of_rows_that_saw_nothing(bbm):
    """A log-sum-exp of -infinity gives nothing; what a step's keys get adds up to its queries."""
    lens, news, H, Hk, d, page = [300, 40], [3, 1], 8, 2, 64, 16
    c, table, cu, T, q, _ = cached_case(bbm, lens, news, H, Hk, d, page, seed=2)
    _, lse = bbm.bbm_kv4_attn(q, c, i32(table), i32(lens), i32(cu))
    got = bbm.bbm_kv4_weights(q, lse, c, i32(table), i32(lens), i32(cu), bbm.kv4_weights(c))
    assert np.abs(f64(got).sum((0, 2)) - T * (H // Hk)).max() <= 400 * ot.F * T * H * 40
    lse[:, 1] = -float("inf")
    check_weights(bbm, None, None, c, table, lens, cu, T, q, None, H, Hk, d, page, lse=lse)


@pytest.mark.parametrize("rows", [[0], [5], [0, 1, 40, 41]])
@pytest.mark.parametrize("group_cu, shared, lens, news, H, Hk, d, tree", [
    ([0], [], [3, 300, 50], [3, 4, 2], 3, 1, 64, None),                         # few columns, the first request's new tokens all there is of it
    ([0], [], [8, 300, 50], [8, 4, 2], 3, 1, 128, 1),
    ([0], [], [70, 300, 50], [70, 30, 20], 6, 2, 128, None),                    # many; 63 of a tile's 64 are used
    ([0], [], [70, 300, 50], [60, 64, 20], 12, 2, 64, 1),
    ([0], [], [200, 300], [130, 90], 8, 2, 128, None),
    ([0, 3], [48], [55, 60, 52], [3, 4, 2], 6, 2, 64, None),
    ([0, 40], [96], [100 + i for i in range(40)], [3] * 40, 6, 2, 128, None)])
def test_weights_of_queries_that_are_no_numbers(bbm, group_cu, shared, lens, news, H, Hk, d, tree, rows):
    """What such a row holds reaches the keys that it sees, and none at all if its log-sum-exp is -infinity."""
    c, table, cu, T, q, words = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, 16, seed=9, tree=tree)
    rows = [r for r in rows if r < T]
    if tree:
        words[rows] = 0
    mask = None if words is None else torch.from_numpy(words).cuda()
    groups = (i32(group_cu), i32(shared)) if shared else (None, None)
    old = bbm.kv4_weights(c).fill_(1.5)

    def gather(q, lse, decay=0.5):
        return bbm.bbm_kv4_weights(q, lse, c, i32(table), i32(lens), i32(cu), old, *groups, mask=mask, decay=decay, out=torch.zeros_like(old))

    _, lse = bbm.bbm_kv4_attn(q, c, i32(table), i32(lens), i32(cu), mask=mask)
    none, only = lse.clone(), torch.full_like(lse, -float("inf"))
    none[:, rows] = -float("inf")
    only[:, rows] = lse[:, rows]
    only[:, rows] = torch.where(torch.isinf(only[:, rows]), only[:, rows], torch.zeros_like(only[:, rows]))
    want = gather(q, none)
    seen = gather(q, only, 0.0) > 0
    assert want.isfinite().all()
    for value in (float("nan"), float("inf")):
        bad, bad_lse = q.clone(), none.clone()
        bad[rows] = value
        assert torch.equal(gather(bad, none), want)
        bad_lse[:, rows] = float("nan")
        got = gather(bad, bad_lse)
        assert torch.equal(got[~seen], want[~seen]) and got[seen].isnan().all()


@pytest.mark.parametrize("max_own", [1, 1 << 40])
def test_weights_of_many_columns_and_requests(bbm, max_own):
    """Pieces that a work-group takes one after the other, and hints beyond any table."""
    R = 20
    lens, news = [300 + 11 * i for i in range(R)], [40 + i for i in range(R)]
    c, table, cu, T, q, _ = cached_case(bbm, lens, news, 2, 2, 64, 16, seed=6)
    check_weights(bbm, None, None, c, table, lens, cu, T, q, None, 2, 2, 64, 16, hints=[dict(max_own=max_own)])


def test_weights_of_heads_far_apart(bbm):
    """Heads so far apart that a tile's columns are one head's tokens; and the layout with all tokens of a head side by side."""
    lens, news, H, Hk, d, page = [300, 170], [70, 45], 4, 2, 64, 16
    c, table, cu, T, q, _ = cached_case(bbm, lens, news, H, Hk, d, page, seed=8)
    _, lse = bbm.bbm_kv4_attn(q, c, i32(table), i32(lens), i32(cu))
    store = torch.empty((1 << 29) + 8 + T * 2 * d, dtype=torch.bfloat16, device="cuda")
    far = store.as_strided((T, 2, d), (2 * d, (1 << 29) + 8, 1))
    args = c, i32(table), i32(lens), i32(cu)
    one = bbm.kv4_cache(c.k.shape[0], 1, d, page)
    for x in ("k", "v", "k_scale", "v_scale"):
        getattr(one, x).copy_(getattr(c, x)[:, :1])
    far.copy_(q[:, :2])
    want = bbm.bbm_kv4_weights(q[:, :2].contiguous(), lse[:2].contiguous(), one, *args[1:], bbm.kv4_weights(one))
    got = bbm.bbm_kv4_weights(far, lse[:2].contiguous(), one, *args[1:], bbm.kv4_weights(one))
    # (the same terms in another order: two heads' tokens in one tile, or one behind the other)
    tol = 2 * ot.F * (T * 2 + 16) * f64(want)
    close("weights", got, f64(want), tol)
    heads = q[:, :2].transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(bbm.bbm_kv4_weights(heads, lse[:2].contiguous(), one, *args[1:], bbm.kv4_weights(one)), want)


class SharedInPart:
    """bbm_kv4_weights with the shared lengths as they are, where the definition has those of whole pages."""

    def __init__(self, bbm, shared):
        self.bbm, self.shared, self.bbm_kv4_attn = bbm, i32(shared), bbm.bbm_kv4_attn

    def bbm_kv4_weights(self, q, lse, c, table, lens, cu, w, group_cu, shared_lens, **kw):
        return self.bbm.bbm_kv4_weights(q, lse, c, table, lens, cu, w, group_cu, self.shared, **kw)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group_cu, shared, lens, news, H, Hk, page", [
    ([0, 3], [100], [140, 130, 101], [1, 1, 1], 4, 2, 64),
    ([0, 2], [40], [60, 50], [1, 2], 4, 1, 128),                              # no page is whole
    ([1, 3, 5], [47, 80], [30, 60, 50, 90, 100], [1, 1, 3, 2, 1], 6, 2, 32),
    ([0, 2], [300], [340, 333], [30, 33], 8, 2, 32),                          # many columns
    ([0, 2], [300], [340, 333], [30, 33], 8, 2, 128),
    ([0, 40], [112], [120 + i for i in range(40)], [2] * 40, 8, 2, 64),       # for the group alone
    ([0, 2], [2300], [2400, 2310], [3, 1], 12, 4, 128)])
def test_weights_behind_a_page_shared_in_part(bbm, group_cu, shared, lens, news, H, Hk, d, page):
    """A prefix that ends inside a page, of which each request has a copy of its own, since it goes on there: the copies' keys gather for themselves, and attention is the same either way."""
    c, table, cu, T, q, _ = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, page, seed=6, before=1, behind=2)
    for g, n in enumerate(shared):
        for r in range(group_cu[g] + 1, group_cu[g + 1]):
            a, b = table[group_cu[g], n // page], table[r, n // page]
            for x in (c.k, c.v, c.k_scale):
                x[b, :, :n % page] = x[a, :, :n % page]
            c.v_scale[b, ..., :n % page] = c.v_scale[a, ..., :n % page]
    hints = [{}, dict(max_shared=4096, max_own=40), dict(max_shared=1, max_own=1)]
    check_weights(SharedInPart(bbm, shared), group_cu, [n // page * page for n in shared], c, table, lens, cu, T, q, None, H, Hk, d, page, hints=hints)
    for hint in hints:
        check_cached(Behind(bbm, group_cu, shared), c, table, lens, cu, T, q, None, H, Hk, d, page, **hint)


def gathered(c, table, lens, cu, T, q, lse, old, H, Hk, page, scale, decay, gain=ot.key_weights):
    """(what causal requests' keys hold behind a step, how far it may be off), [pages, Hk, page] in 64 bits; pages that requests share are decayed once."""
    (hk, _), nq, nl, G = host_cache(c), f64(q), f64(lse), H // Hk
    there, fresh = np.zeros((c.k.shape[0], page), bool), np.zeros((c.k.shape[0], page), bool)
    at = [(table[r, np.arange(n) // page], np.arange(n) % page) for r, n in enumerate(lens)]
    for r, (pg, j) in enumerate(at):
        new = int(cu[r + 1] - cu[r])
        there[pg, j] = True
        fresh[pg[len(pg) - new:], j[len(pg) - new:]] = True
    want = np.where(there[:, None], np.where(fresh[:, None], 0.0, np.float64(np.float32(decay)) * old), old)
    tol = np.where(there[:, None], 4 * ot.F * want, 0.0)
    for r, (pg, j) in enumerate(at):
        a, b, n = int(cu[r]), int(cu[r + 1]), len(pg)
        seen = np.arange(n) <= n - (b - a) + np.arange(b - a)[:, None]
        for h in range(H):
            w, e = gain(nq[a:b, h], hk[pg, h // G, j], seen, scale, nl[h, a:b])
            want[pg, h // G, j] += w
            tol[pg, h // G, j] += e
    # the sums of all queries of a group meet in one number: as many half steps of it as there are terms
    return want, tol + np.where(there[:, None], 2 * ot.F * (T * G + 16) * want, 0.0)


SCALED = [([0], [], [70, 200], [3, 1], 4, 2, 64, 1), ([0, 3], [96], [170, 200, 165], [3, 1, 1], 4, 2, 128, -1), ([0], [], [300, 150], [140, 130], 8, 2, 64, -1),
          ([0], [], [300, 150], [140, 130], 8, 2, 128, 1), ([0, 40], [96], [120 + i for i in range(40)], [2] * 40, 8, 2, 128, 1)]


def check_scaled(bbm, group_cu, shared, c, table, lens, cu, T, q, H, Hk, page, scale, gain=ot.key_weights):
    args, groups = (c, i32(table), i32(lens), i32(cu)), (i32(group_cu), i32(shared)) if shared else (None, None)
    _, lse = bbm.bbm_kv4_shared_attn(q, *args, *groups, softmax_scale=scale, max_shared=4096)
    old = torch.rand(c.k.shape[:3], generator=torch.Generator().manual_seed(3)).mul_(3)
    want, tol = gathered(c, table, lens, cu, T, q, lse, f64(old), H, Hk, page, scale, 0.75, gain)
    close("weights", bbm.bbm_kv4_weights(q, lse, *args, old.cuda(), *groups, decay=0.75, softmax_scale=scale), want, tol)


@pytest.mark.parametrize("scale", [2.0 ** -7, 0.3, 2.0])
@pytest.mark.parametrize("group_cu, shared, lens, news, H, Hk, d, sign", SCALED)
def test_weights_with_other_scales(bbm, group_cu, shared, lens, news, H, Hk, d, sign, scale):
    c, table, cu, T, q, _ = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, 32, seed=21)
    check_scaled(bbm, group_cu, shared, c, table, lens, cu, T, q, H, Hk, 32, scale)


def sized_gain(q, k, seen, scale, lse):
    """ot.key_weights of scores that fp32 holds exactly: an exponent is off by the roundings of lse and of the scale in units of log2, relative to lse and to the score, and by
    those of their difference x (the constant, the multiply-add) and of the exponential."""
    s = scale * (q @ k.T)
    x = np.where(seen, s - lse[:, None], -np.inf)
    p = np.exp(x)
    e = ot.F * (np.abs(lse)[:, None] + np.abs(s) + 3 * np.abs(np.where(seen, x, 0.0)) + 8)
    return p.sum(0), (1.001 * e * p).sum(0) + len(q) * ot.U


@pytest.mark.parametrize("base, gap, scale", [(2, -2, 3), (10, -1, 0), (12, -1, 0), (16, -4, -4), (20, -2, -8), (30, 8, -18)])
@pytest.mark.parametrize("group_cu, shared, lens, news, H, Hk, d, sign", SCALED)
def test_weights_of_scores_up_to_2_to_the_12(bbm, group_cu, shared, lens, news, H, Hk, d, sign, base, gap, scale):
    page = 32
    c, table, cu, T, _, _ = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, page, seed=22)
    slots = np.concatenate([table[r, np.arange(n) // page] * page + np.arange(n) % page for r, n in enumerate(lens)])
    slots = np.unique(slots)
    bbm.bbm_kv4_append(sized_rows(1, len(slots), Hk, d, sign, base, gap), normal(2, len(slots), Hk, d), i32(slots), c)
    check_scaled(bbm, group_cu, shared, c, table, lens, cu, T, sized_query(T, H, d, base), H, Hk, page, 2.0 ** scale, sized_gain)


@pytest.mark.parametrize("cut", [1, 3, 5])
def test_weights_of_a_step_in_two_calls(bbm, cut):
    """Requests of few and of many new tokens in calls of their own, on the step's tensors: parts of offsets, lengths and table, whose other rows are nobody's."""
    lens, news, H, Hk, d, page = [300, 170, 250, 90, 400, 333], [130, 1, 1, 2, 1, 1], 8, 2, 64, 16
    c, table, cu, T, q, _ = cached_case(bbm, lens, news, H, Hk, d, page, seed=12, before=1, behind=2)
    tab, ln, offsets = i32(table), i32(lens), i32(cu)
    _, lse = bbm.bbm_kv4_attn(q, c, tab, ln, offsets)
    old = torch.rand(c.k.shape[:3], generator=torch.Generator().manual_seed(3)).mul_(3)
    want, tol = gathered(c, table, lens, cu, T, q, lse, f64(old), H, Hk, page, d ** -0.5, 0.75)
    w = old.cuda()
    for a, b in ((0, cut), (cut, 6)):
        bbm.bbm_kv4_weights(q, lse, c, tab[a:b], ln[a:b], offsets[a:b + 1], w, decay=0.75)
    close("weights", w, want, tol)


@pytest.mark.parametrize("H, Hk", [(4, 2), (64, 1)])
def test_weights_of_groups_whose_numbers_are_wrong_stay_inside(bbm, H, Hk):
    """Few columns and many: keys of other groups get what they get, pages of nobody keep what they hold."""
    group_cu, shared, lens, news, d, page = [0, 2, 4], [64, 32], [90, 80, 70, 60], [1, 1, 1, 1], 64, 16
    c, table, cu, T, q, _ = grouped_case(bbm, group_cu, shared, lens, news, H, Hk, d, page, seed=8, before=2, behind=2)
    args = c, i32(table), i32(lens), i32(cu)
    _, lse = bbm.bbm_kv4_attn(q, *args)
    old = torch.rand(c.k.shape[:3], generator=torch.Generator().manual_seed(1)).cuda()
    want = bbm.bbm_kv4_weights(q, lse, *args, old, i32(group_cu), i32(shared), out=old.clone())
    sure, nobody = np.unique(table[:2][table[:2] >= 0]), np.setdiff1d(np.arange(c.k.shape[0]), table)
    for wrong, n in (([0, 2, 9], [64, 32]), ([-7, 2, 4], [64, 32]), ([0, 2, 4], [64, 1 << 30]), ([0, 2, 1], [64, 32]), ([0, 2, 4], [64, 80]), ([0, 2, 4], [64, -5])):
        got = bbm.bbm_kv4_weights(q, lse, *args, old, i32(wrong), i32(n), out=old.clone())
        assert len(nobody) > 0 and torch.equal(got[sure], want[sure]) and torch.equal(got[nobody], old[nobody])


# ---- eviction


def check_evict(bbm, lens, H, d, page, budget, recent, first=None, weigh=None, spoil=None, free=None, width=None, seed=0, hints=({},), short_by=0):
    """Against the definition, key by key; whole tensors are compared, so that nothing else may change."""
    Hk = H
    c, table, _, _, _, _ = cached_case(bbm, [max(0, n) for n in lens], [0] * len(lens), Hk, Hk, d, page, seed=seed, behind=1)
    if width is not None:
        table = table[:, :width]
    if spoil is not None:
        spoil(table, c)
    g = np.random.default_rng(seed + 1)
    w = g.random(tuple(c.k.shape[:3])).astype(np.float32) ** 4
    if weigh is not None:
        w = weigh(g, w)
    R, pages = len(lens), c.k.shape[0]
    names = ("k", "v", "k_scale", "v_scale")
    was = {x: getattr(c, x).cpu().numpy() for x in names}
    want, want_w = {x: y.copy() for x, y in was.items()}, w.copy()
    free = g.permutation(pages + 40).astype(np.int32) if free is None else free
    at = len(free) if short_by else min(len(free), pages + 3)             # (of a list that was too short more was asked for than it had)
    given, left = [], []
    for r, n in enumerate(lens):
        n = min(max(0, n), table.shape[1] * page)
        page_of = lambda j: table[r, j // page] if 0 <= table[r, j // page] < pages else -1  # noqa: E731
        f = 0 if first is None else first[r]
        for h in range(Hk):
            ws = [w[page_of(j), h, j % page] if page_of(j) >= 0 else None for j in range(n)]
            moves, b = ot.evict(n, budget, recent, f, ws)
            for a, z in moves:
                if page_of(a) < 0 or page_of(z) < 0:
                    continue
                src, dst = (page_of(a), h, a % page), (page_of(z), h, z % page)
                for x in ("k", "v", "k_scale"):
                    want[x][dst] = was[x][src]
                want["v_scale"][dst[0], h, :, dst[2]] = was["v_scale"][src[0], h, :, src[2]]
                want_w[dst] = w[src]
        left.append(b)
        given += [int(table[r, p]) for p in range(-(-b // page), -(-n // page)) if 0 <= table[r, p] < pages]
    list_want = free.copy()
    for i, p in enumerate(given):
        if at - len(given) + i >= 0:
            list_want[at - len(given) + i] = p
    for hint in hints:
        for x in names:
            getattr(c, x).copy_(torch.from_numpy(was[x]))
        wt, ft, tt = torch.from_numpy(w.copy()).cuda(), i32(free), i32(table)
        fi = None if first is None else i32(first)
        lens_t = i32(lens)
        e = bbm.bbm_kv4_evict(c, wt, tt, lens_t, budget, recent=recent, first=fi, free_pages=ft, free_at=i32([at + short_by]), new_lens=lens_t if hint else None, **hint)
        assert e.lens.cpu().tolist() == left and int(e.free_next) == at - len(given)
        assert np.array_equal(ft.cpu().numpy(), list_want) and np.array_equal(tt.cpu().numpy(), table)
        for x in names:
            assert np.array_equal(getattr(c, x).cpu().numpy(), want[x]), x
        assert np.array_equal(wt.cpu().numpy().view(np.int32), want_w.view(np.int32))
    return left


def few_values(g, w):
    """Many equal weights, of both signs, zeros of both signs, infinities and NaNs."""
    return g.choice(np.array([0.0, -0.0, 1.0, 0.5, -1.0, np.inf, -np.inf, np.nan, 1e-40], np.float32), w.shape)


@pytest.mark.parametrize("lens, H, d, page, budget, recent, first", [
    ([1], 1, 64, 16, 1, 0, None), ([2], 1, 64, 16, 1, 0, None), ([2, 3, 0], 2, 128, 16, 1, 1, None), ([40, 41, 60, -3], 2, 64, 16, 40, 10, [4, 0, 4, 4]),
    ([100, 33, 300], 3, 128, 32, 32, 0, [0, 5, 90]), ([200, 70], 1, 64, 64, 64, 64, None), ([130, 129, 128, 127], 2, 128, 128, 100, 99, [1, 1, 0, 500]),
    ([2112, 2048, 2049, 900], 2, 64, 64, 2048, 256, [4, 4, 4, 4]), ([5000, 700], 2, 128, 16, 600, 530, [3, 70]), ([3000, 3100], 1, 64, 32, 2900, 1100, None),
    ([9000], 2, 64, 128, 1000, 7, [64])])
@pytest.mark.parametrize("weigh", [None, few_values])
def test_evict(bbm, lens, H, d, page, budget, recent, first, weigh):
    check_evict(bbm, lens, H, d, page, budget, recent, first, weigh, hints=[{}, dict(max_len=max(1, max(lens))), dict(max_len=1)])


def test_evict_equal_weights_goes_by_position(bbm):
    check_evict(bbm, [3000, 200], 2, 64, 16, 150, 20, weigh=lambda g, w: w * 0 + 1)


def test_evict_pages_outside_and_a_narrow_table(bbm):
    def spoil(table, c):
        table[0, 3], table[0, 30], table[1, 1], table[1, -1], table[2, :] = -1, 1 << 30, c.k.shape[0], -5, -1
    check_evict(bbm, [1000, 500, 300], 2, 128, 16, 200, 30, [5, 5, 5], spoil=spoil, weigh=few_values)
    check_evict(bbm, [1000, 500, 300], 2, 64, 16, 300, 30, None, width=25)


@pytest.mark.parametrize("n_free", [0, 3, 30])
def test_evict_into_a_short_list(bbm, n_free):
    """Pages without a place in the list are not written anywhere."""
    check_evict(bbm, [300, 200, 400], 1, 64, 16, 64, 8, free=np.arange(n_free, dtype=np.int32) + 100)


def test_evict_into_a_list_that_was_too_short(bbm):
    """What the last step asked for and did not get is not where pages go back to."""
    check_evict(bbm, [300, 200, 400], 1, 64, 16, 64, 8, free=np.arange(60, dtype=np.int32) + 100, short_by=7)


def test_evict_of_many_requests(bbm):
    R = 500
    check_evict(bbm, [30 + i * 7 % 90 for i in range(R)], 1, 64, 16, 48, 5, [i % 9 for i in range(R)])


@pytest.mark.parametrize("lens, budget, recent, table_pages", [([25000, 9000], 3000, 700, 1600), ([45000], 600, 16, 2900)])
def test_evict_of_long_requests_in_a_graph(bbm, lens, budget, recent, table_pages):
    """Weights that take most of a CU's LDS, and more than fit; recorded before it has run once, replayed on what other requests left."""
    Hk, d, page, R = 2, 64, 16, len(lens)
    g = np.random.default_rng(5)
    pages = sum(-(-n // page) for n in lens) + 5
    ids, table, at = g.permutation(pages), np.full((R, table_pages), -1), 0
    for r, n in enumerate(lens):
        table[r, :-(-n // page)] = ids[at:at + -(-n // page)]
        at += -(-n // page)
    c = bbm.kv4_cache(pages, Hk, d, page)
    names = ("k", "v", "k_scale", "v_scale")
    was = {x: g.integers(0, 255, getattr(c, x).shape, dtype=np.uint8) for x in names}
    w = g.random(tuple(c.k.shape[:3])).astype(np.float32)
    want, want_w = {x: y.copy() for x, y in was.items()}, w.copy()
    for r, n in enumerate(lens):
        slot = lambda j: (table[r, j // page], j % page)  # noqa: E731
        for h in range(Hk):
            ws = w[table[r, np.arange(n) // page], h, np.arange(n) % page]
            between = np.lexsort((np.arange(n - recent), -ws[:n - recent]))
            kept, edge = np.zeros(n, bool), budget - recent
            kept[between[:edge]] = True
            src = np.concatenate([np.nonzero(kept[edge:n - recent])[0] + edge, np.arange(n - recent, n)])
            dst = np.concatenate([np.nonzero(~kept[:edge])[0], np.arange(edge, budget)])
            (a, i), (b, j) = slot(src), slot(dst)
            for x in ("k", "v", "k_scale"):
                want[x][b, h, j] = was[x][a, h, i]
            want["v_scale"][b, h, :, j] = was["v_scale"][a, h, :, i]
            want_w[b, h, j] = w[a, h, i]
    wt, tt, ln = torch.empty(w.shape, device="cuda"), i32(table), i32(lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e = bbm.bbm_kv4_evict(c, wt, tt, ln, budget, recent=recent, max_len=max(lens))
    for _ in range(3):
        for x in names:
            getattr(c, x).copy_(torch.from_numpy(was[x]))
        wt.copy_(torch.from_numpy(w))
        graph.replay()
        torch.cuda.synchronize()
        assert e.lens.tolist() == [budget] * R and np.array_equal(wt.cpu().numpy(), want_w)
        for x in names:
            assert np.array_equal(getattr(c, x).cpu().numpy(), want[x]), x


@pytest.mark.parametrize("lens, budget, recent, hint", [([45000, 3000, 38000], 22000, 300, 45000), ([60000], 40000, 0, 60000), ([9000, 8000, 700], 4000, 100, 1), ([9000, 5000], 4992, 64, 1)])
@pytest.mark.parametrize("shares", [(0.5, 0.3, 0.2), (0.9, 0.02, 0.08), (0.05, 0.9, 0.05), (0.3, 0.0, 0.7)])
def test_evict_of_equal_weights_read_from_memory(bbm, lens, budget, recent, hint, shares):
    """Requests whose weights do not fit into LDS, and the same by a hint that is too small: keys move while others still look for theirs among weights of few values."""
    Hk, d, page = 2, 64, 16
    g = np.random.default_rng(len(lens) + budget)
    pages, width = sum(-(-n // page) for n in lens) + 5, -(-max(lens) // page)
    ids, table, at = g.permutation(pages), np.full((len(lens), width), -1), 0
    for r, n in enumerate(lens):
        table[r, :-(-n // page)] = ids[at:at + -(-n // page)]
        at += -(-n // page)
    c = bbm.kv4_cache(pages, Hk, d, page)
    names = ("k", "v", "k_scale", "v_scale")
    was = {x: g.integers(0, 255, getattr(c, x).shape, dtype=np.uint8) for x in names}
    w = g.choice(np.array([0.0, 0.5, 2.0], np.float32), c.k.shape[:3], p=shares)
    want, want_w = {x: y.copy() for x, y in was.items()}, w.copy()
    for r, n in enumerate(lens):
        if n <= budget:
            continue
        pg, j = table[r, np.arange(n) // page], np.arange(n) % page
        for h in range(Hk):
            between = np.lexsort((np.arange(n - recent), -w[pg, h, j][:n - recent]))
            kept, edge = np.zeros(n, bool), budget - recent
            kept[between[:edge]] = True
            src = np.concatenate([np.nonzero(kept[edge:n - recent])[0] + edge, np.arange(n - recent, n)])
            dst = np.concatenate([np.nonzero(~kept[:edge])[0], np.arange(edge, budget)])
            for x in ("k", "v", "k_scale"):
                want[x][pg[dst], h, j[dst]] = was[x][pg[src], h, j[src]]
            want["v_scale"][pg[dst], h, :, j[dst]] = was["v_scale"][pg[src], h, :, j[src]]
            want_w[pg[dst], h, j[dst]] = w[pg[src], h, j[src]]
    tt, ln = i32(table), i32(lens)
    for _ in range(2):
        for x in names:
            getattr(c, x).copy_(torch.from_numpy(was[x]))
        wt = torch.from_numpy(w).cuda()
        e = bbm.bbm_kv4_evict(c, wt, tt, ln, budget, recent=recent, max_len=hint)
        assert e.lens.tolist() == [min(n, budget) for n in lens] and np.array_equal(wt.cpu().numpy(), want_w)
        for x in names:
            assert np.array_equal(getattr(c, x).cpu().numpy(), want[x]), x


def test_evict_without_a_list(bbm):
    c = bbm.kv4_cache(4, 1, 64, 16)
    e = bbm.bbm_kv4_evict(c, bbm.kv4_weights(c), i32([[0, 1, 2, 3]]), i32([60]), 20)
    assert e.free_next is None and e.lens.tolist() == [20]


def test_evict_keeps_what_requests_share(bbm):
    """Requests of a common prefix, all heads at once: the prefix is within `first`, and its pages stay as they are."""
    c, table, _, _, _, _ = cached_case(bbm, [200, 230, 210], [0, 0, 0], 2, 2, 64, 16, seed=3, behind=1)
    table[1:, :6] = table[0, :6]
    before = [x.clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]
    e = bbm.bbm_kv4_evict(c, torch.rand(c.k.shape[:3], device="cuda"), i32(table), i32([200, 230, 210]), 120, recent=10, first=i32([96] * 3))
    assert e.lens.tolist() == [120] * 3
    p = table[0, :6]
    assert all(torch.equal(x[p], y[p]) for x, y in zip(before, (c.k, c.v, c.k_scale, c.v_scale)))


# ---- together


def answers(bbm, s, w, weights, page, shared, budget):
    """A decoding step of answers behind a common prompt: slots, rotary positions, the cache, attention, what the keys gathered, and eviction behind the step."""
    cache, H, Hk, d = s["cache"], s["H"], s["Hk"], s["d"]
    r = bbm.bbm_build_slots(s["ctx"], s["new"], s["table"], s["free"], s["at"], w.shape[0], page)
    q, k, v = w[:, :H * d].unflatten(1, (H, d)), w[:, H * d:(H + Hk) * d].unflatten(1, (Hk, d)), w[:, (H + Hk) * d:].unflatten(1, (Hk, d))
    q, k = bbm.bbm_rope(q, k, r.positions + s["gone"].repeat_interleave(s["new"], output_size=w.shape[0]), s["freqs"])
    bbm.bbm_kv4_append(k, v, r.slots, cache)
    o, lse = bbm.bbm_kv4_shared_attn(q, cache, s["table"], r.lens, r.cu_new, s["group_cu"], s["shared"], max_shared=s.get("max_shared"))
    bbm.bbm_kv4_weights(q, lse, cache, s["table"], r.lens, r.cu_new, weights, s["group_cu"], s["shared"])
    e = bbm.bbm_kv4_evict(cache, weights, s["table"], r.lens, budget, recent=4, first=s["first"], free_pages=s["free"], free_at=r.free_next)
    return r, e, q, o, lse


def answers_state(bbm, H, Hk, d, page, R, shared, seed):
    g = np.random.default_rng(seed)
    pages, width = 80, 20
    ids = g.permutation(pages)
    table = np.full((R, width), -1)
    table[:, :shared // page] = ids[:shared // page]
    cache = bbm.kv4_cache(pages, Hk, d, page)
    for t, lo, hi in ((cache.k, 0, 256), (cache.v, 0, 256), (cache.k_scale, 120, 128), (cache.v_scale, 120, 128)):
        t.copy_(torch.from_numpy(g.integers(lo, hi, t.shape, dtype=np.uint8)))
    return dict(H=H, Hk=Hk, d=d, cache=cache, table=i32(table), free=i32(np.concatenate([ids[:shared // page], ids[shared // page:]])), at=i32([shared // page]), freqs=bbm.rope_freqs(d)[0],
                ctx=i32([shared] * R), new=i32([1] * R), group_cu=i32([0, R]), shared=i32([shared]), first=i32([shared] * R), gone=i32([0] * R))


def test_answers_of_one_prompt(bbm):
    """Steps of answers behind a common prompt against the same steps by bbm_kv4_attn on tables of their own; pages that eviction frees are taken again."""
    H, Hk, d, page, R, shared, budget = 8, 2, 64, 16, 3, 48, 80
    s = answers_state(bbm, H, Hk, d, page, R, shared, 1) | dict(max_shared=4096)
    weights = bbm.kv4_weights(s["cache"])
    used = set()
    for step in range(70):
        w = normal(100 + step, R, (H + 2 * Hk) * d)
        want_ctx = s["ctx"].tolist()
        r, e, q, o, lse = answers(bbm, s, w, weights, page, shared, budget)
        assert r.lens.tolist() == [c + 1 for c in want_ctx] and (r.slots >= 0).all()
        if step % 9 == 0 or step > 66:
            # (eviction has moved keys since: attention of the step itself was checked by its own test; here the sums of weights)
            assert e.lens.tolist() == [min(c + 1, budget) for c in want_ctx]
        used.update((r.slots // page).tolist())
        s["gone"] = s["gone"] + (r.lens - e.lens)
        s["ctx"], s["at"] = e.lens, e.free_next
        tables = s["table"].cpu().numpy()
        live = [[int(p) for p in tables[i, shared // page:-(-int(n) // page)]] for i, n in enumerate(e.lens.tolist())]
        flat = sum(live, [])
        assert len(set(flat)) == len(flat) and not set(flat) & set(tables[0, :shared // page].tolist())   # nobody's page is another's
        free = s["free"][int(s["at"]):].tolist()
        assert len(set(free)) == len(free) and not set(free) & set(flat) and len(free) + len(flat) == 80 - shared // page
    assert len(used) < R * 70 // page                                       # (pages came back)
    # the last step's attention once more, on what the cache holds now, with and without the groups
    q = normal(7, R, H, d)
    lens, cu = s["ctx"], i32(range(R + 1))
    a, b = bbm.bbm_kv4_shared_attn(q, s["cache"], s["table"], lens, cu, s["group_cu"], s["shared"]), bbm.bbm_kv4_attn(q, s["cache"], s["table"], lens, cu)
    check_cached(Behind(bbm, [0, R], [shared]), s["cache"], s["table"].cpu().numpy(), lens.tolist(), np.arange(R + 1), R, q, None, H, Hk, d, page)
    assert (a[1] - b[1]).abs().max() <= 64 * ot.F * 64
    assert torch.isfinite(weights).all() and float(weights[s["table"][0, 0]].sum()) > 0


class Given:
    """An attention whose results are there already."""

    def __init__(self, o, lse):
        self.o, self.lse = o, lse

    def bbm_kv4_attn(self, *args, out, lse, **kw):
        out.copy_(self.o), lse.copy_(self.lse)


@pytest.mark.parametrize("H, Hk, d, page, R, shared, budget, recent, steps", [(8, 2, 64, 16, 3, 48, 80, 4, 60), (8, 2, 128, 32, 2, 64, 100, 30, 50), (4, 4, 64, 16, 5, 0, 40, 7, 50)])
def test_answers_step_by_step(bbm, H, Hk, d, page, R, shared, budget, recent, steps):
    """What every step of answers behind a common prompt gives: attention, gathered weights and evicted caches against their definitions, from what the step before left."""
    s = answers_state(bbm, H, Hk, d, page, R, shared, 2)
    cache, tab = s["cache"], s["table"]
    names = ("k", "v", "k_scale", "v_scale")
    weights, evictions = bbm.kv4_weights(cache), 0
    for step in range(steps):
        w = normal(200 + step, R, (H + 2 * Hk) * d)
        q, k, v = w[:, :H * d].unflatten(1, (H, d)), w[:, H * d:(H + Hk) * d].unflatten(1, (Hk, d)), w[:, (H + Hk) * d:].unflatten(1, (Hk, d))
        r = bbm.bbm_build_slots(s["ctx"], s["new"], tab, s["free"], s["at"], R, page)
        positions = r.positions + s["gone"]
        assert positions.tolist() == [shared + step] * R                    # (as if nothing had ever gone)
        q, k = bbm.bbm_rope(q, k, positions, s["freqs"])
        bbm.bbm_kv4_append(k, v, r.slots, cache)
        table, lens, cu = tab.cpu().numpy(), r.lens.tolist(), np.arange(R + 1)
        o, lse = bbm.bbm_kv4_shared_attn(q, cache, tab, r.lens, r.cu_new, s["group_cu"], s["shared"], max_shared=4096)
        check_cached(Given(o, lse), cache, table, lens, cu, R, q, None, H, Hk, d, page)
        want, tol = gathered(cache, table, lens, cu, R, q, lse, f64(weights), H, Hk, page, d ** -0.5, 0.9)
        bbm.bbm_kv4_weights(q, lse, cache, tab, r.lens, r.cu_new, weights, s["group_cu"], s["shared"], decay=0.9)
        close(f"step {step}: weights", weights, want, tol)
        was, was_w = {x: getattr(cache, x).cpu().numpy() for x in names}, weights.cpu().numpy()
        e = bbm.bbm_kv4_evict(cache, weights, tab, r.lens, budget, recent=recent, first=s["first"], free_pages=s["free"], free_at=r.free_next)
        want, want_w, left = {x: y.copy() for x, y in was.items()}, was_w.copy(), []
        for i, n in enumerate(lens):
            pg, j = table[i, np.arange(n) // page], np.arange(n) % page
            for h in range(Hk):
                moves, b = ot.evict(n, budget, recent, shared, list(was_w[pg, h, j]))
                evictions += len(moves) > 0
                for a, z in moves:
                    for x in ("k", "v", "k_scale"):
                        want[x][pg[z], h, j[z]] = was[x][pg[a], h, j[a]]
                    want["v_scale"][pg[z], h, :, j[z]] = was["v_scale"][pg[a], h, :, j[a]]
                    want_w[pg[z], h, j[z]] = was_w[pg[a], h, j[a]]
            left.append(b)
        assert e.lens.tolist() == left and np.array_equal(weights.cpu().numpy(), want_w)
        for x in names:
            assert np.array_equal(getattr(cache, x).cpu().numpy(), want[x]), (step, x)
        s["gone"] = s["gone"] + (r.lens - e.lens)
        s["ctx"], s["at"] = e.lens, e.free_next
    assert evictions > steps // 4


def test_answers_in_graphs(bbm):
    """A step recorded into a graph: replays give the eager results bit for bit, with eager work between them; two graphs of one stream do not share memory."""
    H, Hk, d, page, R, shared, budget = 8, 2, 128, 16, 5, 64, 65
    names = ("k", "v", "k_scale", "v_scale")

    def state(seed):
        s = answers_state(bbm, H, Hk, d, page, R, shared, seed)
        s |= dict(max_shared=4096, w=normal(seed, R, (H + 2 * Hk) * d), weights=torch.rand(s["cache"].k.shape[:3], generator=torch.Generator().manual_seed(seed)).cuda())
        s["ctx"].copy_(i32([70, 64, 90, 65, 64])), s["table"][:, 4:7].copy_(s["free"][10:10 + 3 * R].view(R, 3))
        s["was"] = [getattr(s["cache"], x).clone() for x in names] + [s["weights"].clone(), s["free"].clone(), s["table"].clone()]
        return s

    def step(s):
        for t, was in zip([getattr(s["cache"], x) for x in names] + [s["weights"], s["free"], s["table"]], s["was"]):
            t.copy_(was)
        r, e, q, o, lse = answers(bbm, s, s["w"], s["weights"], page, shared, budget)
        return [o, lse, r.slots, e.lens, e.free_next, s["weights"], s["free"]] + [getattr(s["cache"], x) for x in names]
    states = [state(1), state(2)]
    want = [[t.clone() for t in step(s)] for s in states]
    torch.cuda.synchronize()
    side, graphs, outs = torch.cuda.Stream(), [], []
    for s in states:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            outs.append(step(s))
    other = torch.cuda.Stream()
    eager = state(9)
    for replay in range(4):
        for out in outs:
            for t in out[:5]:
                t.fill_(5)
        step(eager)                                                        # eager work on the default stream
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(other):
            graphs[1].replay()
        torch.cuda.synchronize()
        for i in range(2):
            for n, (a, b) in enumerate(zip(outs[i], want[i])):
                assert torch.equal(a, b), (replay, i, n)


def test_cache_operators_on_another_stream(bbm):
    """Inputs that a stream still writes when the calls are made on it."""
    lens, news, H, Hk, d, page = [300, 290], [1, 1], 8, 2, 64, 16
    c, table, cu, T, q, _ = grouped_case(bbm, [0, 2], [160], lens, news, H, Hk, d, page, seed=2)
    args = c, i32(table), i32(lens), i32(cu)
    groups = i32([0, 2]), i32([160])
    want = bbm.bbm_kv4_shared_attn(q, *args, *groups, max_shared=4096)
    want_w = bbm.bbm_kv4_weights(q, want[1], *args, bbm.kv4_weights(c), *groups)
    keep = [x.clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]         # (eviction moves all four)
    want_e = bbm.bbm_kv4_evict(c, want_w.clone(), args[1], args[2], 200, first=i32([160, 160]))
    after = c.k.clone()
    for x, y in zip((c.k, c.v, c.k_scale, c.v_scale), keep):
        x.copy_(y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    fresh = bbm.kv4_weights(c)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            a = a @ a * 1e-3
        late = q + (a[0, 0] * 0).to(torch.bfloat16).nan_to_num()
    got = bbm.bbm_kv4_shared_attn(late, *args, *groups, max_shared=4096, stream=side)
    got_w = bbm.bbm_kv4_weights(late, got[1], *args, fresh, *groups, stream=side)
    got_e = bbm.bbm_kv4_evict(c, got_w, args[1], args[2], 200, first=i32([160, 160]), stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got_e.lens, want_e.lens) and torch.equal(c.k, after)


def test_weights_on_another_stream(bbm):
    """Queries that a stream still writes when the call is made on it, few columns and many."""
    for lens, news in (([300, 290], [1, 1]), ([300, 290], [40, 30])):
        H, Hk, d, page = 8, 2, 64, 16
        c, table, cu, T, q, _ = grouped_case(bbm, [0, 2], [160], lens, news, H, Hk, d, page, seed=2)
        args, groups = (c, i32(table), i32(lens), i32(cu)), (i32([0, 2]), i32([160]))
        _, lse = bbm.bbm_kv4_shared_attn(q, *args, *groups)
        want = bbm.bbm_kv4_weights(q, lse, *args, bbm.kv4_weights(c), *groups)
        fresh, side = bbm.kv4_weights(c), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        late = torch.zeros_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            a = torch.randn(4096, 4096, device="cuda")
            for _ in range(20):
                a = a @ a * 1e-3
            late.copy_(q)
        got = bbm.bbm_kv4_weights(late, lse, *args, fresh, *groups, stream=side)
        torch.cuda.synchronize()
        assert got is fresh and torch.equal(got, want) and float(want.sum()) > 0


def test_cache_binding_refuses(bbm):
    q, c = normal(1, 4, 4, 64), bbm.kv4_cache(2, 2, 64, 16)
    lens, cu, table, lse, w = i32([4]), i32([0, 4]), i32([[0, 1]]), torch.zeros(4, 4, device="cuda"), bbm.kv4_weights(c)
    for bad in (lambda: bbm.bbm_kv4_shared_attn(q, c, table, lens, cu, i32([0, 1]), None), lambda: bbm.bbm_kv4_shared_attn(q, c, table, lens, cu, i32([0, 1]), i32([0, 0])),
                lambda: bbm.bbm_kv4_shared_attn(q, c, table, lens, cu, i32([0, 1]).long(), i32([0])), lambda: bbm.bbm_kv4_shared_attn(q.float(), c, table, lens, cu, None, None),
                lambda: bbm.bbm_kv4_shared_attn(q, c, table, lens, cu, None, None, mask=torch.zeros(3, 1, dtype=torch.int64, device="cuda")),
                lambda: bbm.bbm_kv4_weights(q, lse.t()[:3], c, table, lens, cu, w), lambda: bbm.bbm_kv4_weights(q, lse.double(), c, table, lens, cu, w),
                lambda: bbm.bbm_kv4_weights(q, lse, c, table, lens, cu, w[:1]), lambda: bbm.bbm_kv4_weights(q, lse, c, table, lens, cu, w.transpose(1, 2).contiguous().transpose(1, 2)),
                lambda: bbm.bbm_kv4_weights(q, lse, c, table, lens, cu, w, out=w.cpu()), lambda: bbm.bbm_kv4_evict(c, w.half(), table, lens, 2),
                lambda: bbm.bbm_kv4_evict(c, w, table, lens, 2, first=i32([0, 0])), lambda: bbm.bbm_kv4_evict(c, w, table, lens, 2, free_pages=i32([0])),
                lambda: bbm.bbm_kv4_evict(c, w, table, lens, 2, free_pages=i32([0]), free_at=i32([0, 1])), lambda: bbm.bbm_kv4_evict(c, w, table[0], lens, 2)):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: bbm.bbm_kv4_evict(c, w, table, lens, 0), lambda: bbm.bbm_kv4_weights(q, lse, c, table, lens, cu, w, decay=2.0),
                lambda: bbm.bbm_kv4_shared_attn(q, c, table, lens, cu, i32([0, 1, 1]), i32([0, 0]))):
        with pytest.raises(bbm.BbmError):
            bad()


def test_cache_operators_past_32_bits(bbm):
    """A cache whose codes take more than 2^32 bytes: its last pages are attended, weighed and thinned like those of a small one."""
    Hk, d, page, T = 8, 128, 128, 500
    pages = (1 << 32) // (Hk * page * d // 2) + 64
    big, small = bbm.kv4_cache(pages, Hk, d, page), bbm.kv4_cache(4, Hk, d, page)
    k, v, q = normal(1, T, Hk, d), normal(2, T, Hk, d), normal(3, 2, 16, d)
    out = []
    for c, p0 in ((big, pages - 4), (small, 0)):
        bbm.bbm_kv4_append(k, v, i32(np.arange(T) + p0 * page), c)
        table, lens, cu, groups = i32([[p0, p0 + 1, p0 + 2], [p0, p0 + 1, p0 + 3]]), i32([384, 372]), i32([0, 1, 2]), (i32([0, 2]), i32([256]))
        o, lse = bbm.bbm_kv4_shared_attn(q, c, table, lens, cu, *groups, max_shared=4096)
        w = bbm.bbm_kv4_weights(q, lse, c, table, lens, cu, bbm.kv4_weights(c), *groups)
        kept = w[p0:].clone()
        e = bbm.bbm_kv4_evict(c, w, table, lens, 300, recent=10, first=i32([256, 256]))
        out.append([o, lse, kept, e.lens, w[p0:].clone()] + [x[p0:].clone() for x in (c.k, c.v, c.k_scale, c.v_scale)])
    assert all(torch.equal(x, y) for x, y in zip(*out))
