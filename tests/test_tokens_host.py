"""CPU checks of the operators on packed tokens: exported symbols, refusals on the host (also under the host sanitizers), frequencies, and
the oracle's formulas against differences."""
import ctypes as C
import math
import os
import re
import subprocess
import sys

import numpy as np
import pytest

from oracle import tokens as ot

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000          # a pointer that is never dereferenced: validation fails first


@pytest.fixture(scope="module")
def bbm():
    import paper_2409_15097_amd as m
    return m


def test_every_declared_symbol_is_exported_and_bound(bbm):
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "bbm_tokens.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(bbm_[a-z0-9_]+)\s*\(", hdr))
    assert names == {"bbm_build_slots", "bbm_rope", "bbm_prompt_attn_fwd", "bbm_prompt_attn_bwd_workspace_bytes", "bbm_prompt_attn_bwd",
                     "bbm_kv4_append", "bbm_kv4_read", "bbm_kv4_attn_workspace_bytes", "bbm_kv4_attn"}
    raw = C.CDLL(bbm.library_path())
    for n in names:
        assert getattr(raw, n) is not None and callable(getattr(bbm, n))


def pk(ptr=P, row=1024, head=128):
    from paper_2409_15097_amd.tokens import _CPacked
    return None if ptr is None else C.byref(_CPacked(ptr, row, head))


def slots(bbm, ctx=P, new=P, R=4, table=P, stride=8, width=8, page=64, free=P, n_free=9, at=P, T=5, cu=2 * P, lens=3 * P, pos=4 * P, sl=5 * P, nxt=6 * P):
    return bbm.lib.bbm_build_slots(ctx, new, R, table, stride, width, page, free, n_free, at, T, cu, lens, pos, sl, nxt, None)


def test_slots_refuses(bbm):
    for kw in (dict(ctx=None), dict(new=None), dict(table=None), dict(free=None), dict(at=None), dict(cu=None), dict(lens=None), dict(pos=None), dict(sl=None),
               dict(nxt=None), dict(R=0), dict(T=-1), dict(width=0), dict(n_free=-1), dict(stride=7), dict(cu=P + 2), dict(nxt=P), dict(lens=P)):
        assert slots(bbm, **kw) == bbm.BBM_EINVAL, kw
    for kw in (dict(page=0), dict(page=48), dict(R=16385), dict(T=(1 << 30) + 1), dict(R=16384, width=1 << 17, stride=1 << 17)):
        assert slots(bbm, **kw) == bbm.BBM_EUNSUPPORTED, kw


def rope(bbm, q=pk, qo=pk, H=4, k=pk, ko=pk, Hk=2, T=3, d=64, rot=64, pos=P, freqs=P, mscale=1.0):
    f = lambda x: x() if callable(x) else x  # noqa: E731
    return bbm.lib.bbm_rope(f(q), f(qo), H, f(k), f(ko), Hk, T, d, rot, 0, 0, pos, freqs, mscale, None)


BAD_PACKED = [None, pk(0), pk(P + 8), pk(row=1020), pk(head=100), pk(row=-8), pk(head=-8)]
OVERLAP = [dict(row=0), dict(head=0), dict(row=64, head=64), dict(row=120, head=64), dict(head=56)]


def test_rope_refuses(bbm):
    for bad in BAD_PACKED:
        for name in ("q", "qo", "k", "ko"):
            assert rope(bbm, **{name: bad}) == bbm.BBM_EINVAL
    for bad in OVERLAP:
        assert rope(bbm, qo=pk(**bad)) == bbm.BBM_EINVAL and rope(bbm, ko=pk(2 * P, **({**bad, "head": 0}))) == bbm.BBM_EINVAL
    for kw in (dict(T=-1), dict(H=0), dict(Hk=-1), dict(rot=0), dict(rot=63), dict(rot=66), dict(pos=None), dict(freqs=None), dict(pos=P + 1),
               dict(mscale=math.inf), dict(mscale=math.nan), dict(qo=pk(row=2048))):
        assert rope(bbm, **kw) == bbm.BBM_EINVAL, kw
    for kw in (dict(d=72, rot=2), dict(d=528), dict(d=0), dict(T=1 << 31), dict(q=pk(row=(1 << 22) + 8)), dict(T=1 << 30)):
        assert rope(bbm, **kw) == bbm.BBM_EUNSUPPORTED, kw
    assert rope(bbm, T=0) == bbm.BBM_OK
    for kw in (dict(k=pk(2 * P)), dict(ko=pk(2 * P)), dict(q=pk(2 * P), qo=pk(2 * P), k=pk(3 * P), ko=pk(2 * P))):
        assert rope(bbm, **kw) == bbm.BBM_EINVAL, kw


def fwd(bbm, q=pk, k=pk, v=pk, o=pk, lse=P, T=3, R=2, cu=P, H=4, Hk=2, d=64, scale=0.125):
    f = lambda x: x() if callable(x) else x  # noqa: E731
    return bbm.lib.bbm_prompt_attn_fwd(f(q), f(k), f(v), f(o), lse, T, R, cu, H, Hk, d, scale, None)


def bwd(bbm, ws=P, ws_bytes=1 << 20, lse=P, T=3, R=2, cu=P, H=4, Hk=2, d=64, scale=0.125, **kw):
    t = {n: pk() for n in ("q", "k", "v", "o", "d_o", "dq", "dk", "dv")} | kw
    return bbm.lib.bbm_prompt_attn_bwd(t["q"], t["k"], t["v"], t["o"], t["d_o"], lse, t["dq"], t["dk"], t["dv"], T, R, cu, H, Hk, d, scale, ws, ws_bytes, None)


def test_prompt_attention_refuses(bbm):
    for call in (fwd, bwd):
        for bad in BAD_PACKED:
            for name in ("q", "k", "v", "o") if call is fwd else ("q", "k", "v", "o", "d_o", "dq", "dk", "dv"):
                assert call(bbm, **{name: bad}) == bbm.BBM_EINVAL
        for kw in (dict(T=-1), dict(R=0), dict(H=0), dict(Hk=0), dict(H=3), dict(cu=None), dict(cu=P + 2), dict(lse=P + 2), dict(scale=0.0), dict(scale=-1.0),
                   dict(scale=math.inf), dict(scale=math.nan)):
            assert call(bbm, **kw) == bbm.BBM_EINVAL, kw
        for kw in (dict(d=96), dict(T=1 << 31), dict(R=1 << 31), dict(H=1 << 17), dict(scale=2.0 ** -101), dict(scale=2.0 ** 101)):
            assert call(bbm, **kw) == bbm.BBM_EUNSUPPORTED, kw
        assert call(bbm, T=0) == bbm.BBM_OK
    for bad in OVERLAP:
        assert fwd(bbm, o=pk(**bad)) == bbm.BBM_EINVAL and bwd(bbm, dk=pk(**bad)) == bbm.BBM_EINVAL
    apart = {n: pk((i + 1) * P) for i, n in enumerate(("q", "k", "v", "o", "d_o", "dq", "dk", "dv"))}
    for out, other in (("dq", "q"), ("dk", "k"), ("dv", "d_o"), ("dv", "dk")):
        assert bwd(bbm, **apart | {out: apart[other]}) == bbm.BBM_EINVAL
    assert fwd(bbm, k=pk(2 * P), v=pk(3 * P)) == bbm.BBM_EINVAL and fwd(bbm, q=pk(2 * P), v=pk(3 * P)) == bbm.BBM_EINVAL
    assert bwd(bbm, lse=None) == bbm.BBM_EINVAL and bwd(bbm, ws=P + 8) == bbm.BBM_EINVAL
    assert bbm.bbm_prompt_attn_bwd_workspace_bytes(0, 1, 4, 2, 64) == 0 and bbm.bbm_prompt_attn_bwd_workspace_bytes(3, 1, 4, 3, 64) == 0
    need = bbm.bbm_prompt_attn_bwd_workspace_bytes(3, 2, 4, 2, 64)
    assert need > 0 and bwd(bbm, ws_bytes=need - 1) == bbm.BBM_EWORKSPACE and bwd(bbm, ws=None) == bbm.BBM_EWORKSPACE


def cache(k=P, ks=P, v=P, vs=P, pages=8, Hk=2, page=64, d=64):
    from paper_2409_15097_amd.tokens import _CCache
    return C.byref(_CCache(k, ks, v, vs, pages, Hk, page, d))


BAD_CACHE = [dict(k=None), dict(ks=None), dict(v=None), dict(vs=None), dict(k=P + 8), dict(vs=P + 4), dict(pages=0), dict(Hk=0)]
ODD_CACHE = [dict(d=96), dict(d=32), dict(page=8), dict(page=48), dict(pages=1 << 25), dict(Hk=1 << 17)]


def attn(bbm, q=None, o=None, lse=P, T=3, R=2, cu=P, lens=P, table=P, stride=4, width=4, mask=None, words=0, c=None, H=4, scale=0.125, max_len=256, ws=P,
         ws_bytes=1 << 30):
    return bbm.lib.bbm_kv4_attn(q or pk(), o or pk(), lse, T, R, cu, lens, table, stride, width, mask, words, c or cache(), H, scale, max_len, ws, ws_bytes, None)


def test_cache_refuses(bbm):
    move = lambda k=pk, v=pk, T=3, slots=P, c=None: (  # noqa: E731
        bbm.lib.bbm_kv4_append(k and k(), v and v(), T, slots, c or cache(), None), bbm.lib.bbm_kv4_read(slots, T, c or cache(), k and k(), v and v(), None))
    EINVAL, EUN = (bbm.BBM_EINVAL,) * 2, (bbm.BBM_EUNSUPPORTED,) * 2
    for bad in BAD_CACHE:
        assert move(c=cache(**bad)) == EINVAL and attn(bbm, c=cache(**bad)) == bbm.BBM_EINVAL
    for bad in ODD_CACHE:
        assert move(c=cache(**bad)) == EUN and attn(bbm, c=cache(**bad)) == bbm.BBM_EUNSUPPORTED
    assert bbm.lib.bbm_kv4_append(pk(), pk(), 3, P, None, None) == bbm.BBM_EINVAL
    for bad in BAD_PACKED:
        assert move(k=lambda: bad) == EINVAL and move(v=lambda: bad) == EINVAL
    for bad in OVERLAP:
        assert bbm.lib.bbm_kv4_read(P, 3, cache(), pk(**bad), pk(), None) == bbm.BBM_EINVAL
    assert move(T=-1) == EINVAL and move(slots=None) == EINVAL and move(slots=P + 2) == EINVAL and move(T=1 << 31) == EUN and move(T=0) == (0, 0)
    for kw in (dict(q=pk(P + 8)), dict(o=pk(row=0)), dict(T=-1), dict(R=0), dict(H=3), dict(cu=None), dict(lens=None), dict(table=None), dict(lens=P + 2),
               dict(lse=P + 2), dict(stride=3), dict(width=0), dict(max_len=0), dict(mask=P + 4, words=1), dict(mask=P, words=0), dict(words=1), dict(scale=0.0),
               dict(scale=math.nan), dict(ws=P + 8)):
        assert attn(bbm, **kw) == bbm.BBM_EINVAL, kw
    for kw in (dict(T=1 << 31), dict(T=1 << 30), dict(scale=2.0 ** -101), dict(width=(1 << 24) + 1, stride=1 << 26), dict(mask=P, words=(1 << 20) + 1)):
        assert attn(bbm, **kw) == bbm.BBM_EUNSUPPORTED, kw
    assert attn(bbm, T=0) == bbm.BBM_OK and attn(bbm) == bbm.BBM_EINVAL and bbm.lib.bbm_kv4_read(P, 3, cache(), pk(), pk(), None) == bbm.BBM_EINVAL
    need = bbm.bbm_kv4_attn_workspace_bytes(1, 1, 8, 1, 128, 1 << 16)
    long = dict(T=1, R=1, H=8, c=cache(Hk=1, d=128), max_len=1 << 16)
    assert need > 0 and attn(bbm, **long, ws_bytes=need - 1) == bbm.BBM_EWORKSPACE and attn(bbm, **long, ws=None) == bbm.BBM_EWORKSPACE
    assert bbm.bbm_kv4_attn_workspace_bytes(0, 1, 8, 1, 128, 64) == 0 and bbm.bbm_kv4_attn_workspace_bytes(1, 1, 8, 3, 128, 64) == 0


def test_refusals_pass_under_host_sanitizers(tmp_path):
    if os.environ.get("BBM_LIBRARY"):
        pytest.skip("this is the sanitized run")
    from test_abi_sanitized import _build_module
    build = _build_module()
    lib = build.build_host_sanitized(str(tmp_path / "hostsan"))
    env = dict(os.environ, BBM_LIBRARY=lib, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    env["LD_PRELOAD"] = ":".join(x for x in (build.sanitizer_runtime(), env.get("LD_PRELOAD", "")) if x)
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-p", "no:cacheprovider", "-k", "refuses or symbol"], cwd=ROOT, env=env,
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert r.returncode == 0 and "AddressSanitizer" not in r.stdout and "runtime error:" not in r.stdout and " passed" in r.stdout, r.stdout[-4000:]


def test_frequencies(bbm):
    f, m = bbm.rope_freqs(64, device="cpu")
    assert m == 1.0 and np.array_equal(f.numpy(), (10000.0 ** (-np.arange(0, 64, 2) / 64)).astype(np.float32))
    lin, _ = bbm.rope_freqs(64, factor=4, method="linear", device="cpu")
    assert np.allclose(lin.numpy(), f.numpy() / 4, rtol=2 ** -23)
    ntk, _ = bbm.rope_freqs(64, factor=4, method="ntk", device="cpu")
    assert ntk[0] == f[0] and abs(float(ntk[-1] / f[-1]) - 0.25) < 1e-6 and np.all(np.diff((ntk / f).numpy()) <= 0)
    yarn, m = bbm.rope_freqs(64, factor=4, method="yarn", trained_len=4096, device="cpu")
    turns, ratio = 4096 * f.numpy() / (2 * np.pi), (yarn / f).numpy()
    assert abs(m - (0.1 * math.log(4) + 1)) < 1e-12 and np.allclose(ratio[turns > 32], 1) and np.allclose(ratio[turns < 1], 0.25) and np.all(np.diff(ratio) <= 1e-7)
    for bad in (dict(rot=0), dict(rot=7), dict(rot=8, base=0.0), dict(rot=8, factor=0.5), dict(rot=8, method="other"), dict(rot=8, method="yarn", factor=2.0), dict(rot=2, method="ntk")):
        with pytest.raises(ValueError):
            bbm.rope_freqs(device="cpu", **bad)


def test_oracle_gradients_are_differences():
    g = np.random.default_rng(5)
    n, d, scale = 7, 8, 0.4
    q, k, v, d_o = (g.standard_normal((n, d)) for _ in range(4))
    seen = np.tril(np.ones((n, n), bool))
    loss = lambda q, k, v: float((ot.attention(q, k, v, seen, scale)[0] * d_o).sum())  # noqa: E731
    o, _, p = ot.attention(q, k, v, seen, scale)
    grads = ot.attention_bwd(q, k, v, d_o, p, scale, (d_o * o).sum(1))
    for at, want in enumerate(grads):
        step = g.standard_normal((n, d))
        x = [q, k, v]
        up, down = ([y + s * 1e-6 * step if i == at else y for i, y in enumerate(x)] for s in (1, -1))
        assert abs((loss(*up) - loss(*down)) / 2e-6 - (want * step).sum()) < 1e-7
    pos, f = np.array([0, 3, 70000]), np.array([1.0, 0.01])
    x, y = g.standard_normal((3, 2, 6)), g.standard_normal((3, 2, 6))
    for inter in (False, True):                                          # <R x, y> = <x, R' y>, and the map is linear
        assert abs((ot.rope(x, pos, f, inter, 1.1) * y).sum() - (x * ot.rope(y, pos, f, inter, 1.1, inverse=True)).sum()) < 1e-12


def test_oracle_of_the_cache_format():
    x = np.zeros((1, 32))
    x[0, :12] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, -0.3, -5.1, 6, 0.26]
    c, s = ot.kv4_encode(x)
    assert s[0, 0] == 127 and list(ot.kv4_decode(c, s)[0, :12]) == [0, 1, 1, 2, 2, 4, 4, 6, -0.5, -6, 6, 0.5]
    x[0, 7] = 7.01
    assert ot.kv4_encode(x)[1][0, 0] == 128


APART = {n: pk((i + 20) * P) for i, n in enumerate(("q", "qo", "k", "ko", "v", "o"))}


def test_refuses_sizes_whose_product_wraps(bbm):
    """Products of two arguments that pass 2^64 and come out small are refused like those just above a limit."""
    for kw in (dict(R=16384, width=1 << 50, stride=1 << 50), dict(R=4, width=1 << 62, stride=1 << 62), dict(R=16384, width=1 << 17, stride=1 << 17)):
        assert slots(bbm, ctx=11 * P, new=12 * P, table=13 * P, free=14 * P, at=15 * P, **kw) == bbm.BBM_EUNSUPPORTED, kw
    for kw in (dict(width=1 << 58, stride=1 << 58), dict(c=cache(pages=1 << 58)), dict(c=cache(pages=1 << 57, page=128)), dict(c=cache(pages=(1 << 60) + 1, page=16)),
               dict(c=cache(Hk=1 << 62), H=1 << 62)):
        assert attn(bbm, q=APART["q"], o=APART["o"], **kw) == bbm.BBM_EUNSUPPORTED, kw
    a = APART
    for pages, T in ((1 << 58, 3), (8, 1 << 62), (8, (1 << 63) - 1)):
        assert bbm.lib.bbm_kv4_append(a["k"], a["v"], T, P, cache(pages=pages), None) == bbm.BBM_EUNSUPPORTED
        assert bbm.lib.bbm_kv4_read(P, T, cache(pages=pages), a["k"], a["v"], None) == bbm.BBM_EUNSUPPORTED
    for H, Hk in ((1 << 62, 1 << 62), ((1 << 63) - 1, 2), (65535, 1), (1, 65535)):
        assert rope(bbm, **{n: a[n] for n in ("q", "qo", "k", "ko")}, H=H, Hk=Hk) == bbm.BBM_EUNSUPPORTED, (H, Hk)


def test_refuses_outputs_at_the_address_of_anything_else(bbm):
    """Every output and workspace against every input and every other output, each of which has an address of its own otherwise."""
    def check(call, outputs, inputs, allowed=()):
        at = {n: (i + 50) * P for i, n in enumerate(outputs + inputs)}
        for out in outputs:
            for other in outputs + inputs:
                if other != out and (out, other) not in allowed and (other, out) not in allowed:
                    assert call(at | {out: at[other]}) == bbm.BBM_EINVAL, (out, other)
                    assert "must not be" in bbm.bbm_last_error(), (out, other, bbm.bbm_last_error())
    check(lambda a: slots(bbm, **a), ["cu", "lens", "pos", "sl", "nxt", "table"], ["ctx", "new", "free", "at"])
    tensors = lambda a, *names: {n: pk(a[n]) for n in names}  # noqa: E731
    check(lambda a: rope(bbm, **tensors(a, "q", "qo", "k", "ko"), pos=a["pos"], freqs=a["freqs"]), ["qo", "ko"], ["q", "k", "pos", "freqs"], [("qo", "q"), ("ko", "k")])
    check(lambda a: fwd(bbm, **tensors(a, "q", "k", "v", "o"), lse=a["lse"], cu=a["cu"]), ["o", "lse"], ["q", "k", "v", "cu"])
    names = ("q", "k", "v", "o", "d_o", "dq", "dk", "dv")
    check(lambda a: bwd(bbm, **tensors(a, *names), lse=a["lse"], cu=a["cu"], ws=a["ws"]), ["dq", "dk", "dv", "ws"], ["q", "k", "v", "o", "d_o", "lse", "cu"])
    parts = ["k", "ks", "v", "vs"]
    c = lambda a: cache(**{n: a["c" + n] for n in parts})  # noqa: E731
    in_cache = ["c" + n for n in parts]
    check(lambda a: bbm.lib.bbm_kv4_append(pk(a["k"]), pk(a["v"]), 3, a["slots"], c(a), None), in_cache, ["k", "v", "slots"])
    check(lambda a: bbm.lib.bbm_kv4_read(a["slots"], 3, c(a), pk(a["k"]), pk(a["v"]), None), ["k", "v"], ["slots"] + in_cache)
    long = dict(T=1, R=1, H=2, max_len=1 << 16, mask=None)
    check(lambda a: attn(bbm, **long | dict(q=pk(a["q"]), o=pk(a["o"]), lse=a["lse"], cu=a["cu"], lens=a["lens"], table=a["table"], ws=a["ws"], c=c(a), mask=a["mask"], words=1)),
          ["o", "lse", "ws"], ["q", "cu", "lens", "table", "mask"] + in_cache)


def test_frequencies_of_a_longer_context_need_a_method(bbm):
    with pytest.raises(ValueError, match="method"):
        bbm.rope_freqs(64, factor=8.0, device="cpu")
    assert bbm.rope_freqs(64, factor=1, device="cpu")[0].equal(bbm.rope_freqs(64, device="cpu")[0])


def test_signatures_are_declared_with_the_library(bbm):
    """`lib` alone, before any name of the operators on packed tokens is used: 64-bit arguments arrive as such."""
    code = """
import re
import paper_2409_15097_amd as bbm
L = bbm.lib
for h in ("bbm.h", "bbm_mask_index.h", "bbm_tokens.h"):
    hdr = re.sub(r"/\\*.*?\\*/", "", open("include/" + h).read(), flags=re.S)
    for name in set(re.findall(r"\\b(bbm_[a-z0-9_]+)\\s*\\(", hdr)):
        assert getattr(L, name).argtypes is not None, name
assert L.bbm_build_slots(1, 1, 4, 1, 8, 8, 64, 1, 9, 1, -(1 << 40), 1, 1, 1, 1, 1, None) == bbm.BBM_EINVAL
assert "T=-1099511627776" in bbm.bbm_last_error(), bbm.bbm_last_error()
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:]
