"""CPU checks of the operators on the cache of many and long answers: exported symbols and refusals on the host (also under the host sanitizers)."""
import ctypes as C
import math
import os
import re
import subprocess
import sys

import pytest

from test_tokens_host import BAD_CACHE, BAD_PACKED, ODD_CACHE, OVERLAP, P, ROOT, cache, pk

NAMES = {"bbm_kv4_shared_attn_workspace_bytes", "bbm_kv4_shared_attn", "bbm_kv4_weights", "bbm_kv4_evict_workspace_bytes", "bbm_kv4_evict"}


@pytest.fixture(scope="module")
def bbm():
    import paper_2409_15097_amd as m
    return m


def test_every_declared_symbol_is_exported_and_bound(bbm):
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "bbm_cache.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(bbm_[a-z0-9_]+)\s*\(", hdr))
    assert names == NAMES
    raw = C.CDLL(bbm.library_path())
    for n in names:
        assert getattr(raw, n) is not None and callable(getattr(bbm, n)) and n in dir(bbm)


def shared(bbm, q=None, o=None, lse=2 * P, T=3, R=2, cu=3 * P, lens=4 * P, table=5 * P, stride=4, width=4, S=1, group=6 * P, shared=7 * P, mask=None, words=0, c=None, H=4, scale=0.125,
           max_shared=4096, max_own=64, ws=8 * P, ws_bytes=1 << 40):
    return bbm.lib.bbm_kv4_shared_attn(q or pk(), o or pk(9 * P), lse, T, R, cu, lens, table, stride, width, S, group, shared, mask, words, c or cache(k=10 * P), H, scale, max_shared,
                                       max_own, ws, ws_bytes, None)


def test_shared_attention_refuses(bbm):
    for bad in BAD_CACHE:
        assert shared(bbm, c=cache(**bad)) == bbm.BBM_EINVAL
    for bad in ODD_CACHE:
        assert shared(bbm, c=cache(**bad)) == bbm.BBM_EUNSUPPORTED
    for bad in BAD_PACKED:
        if bad is not None:
            assert shared(bbm, q=bad) == bbm.BBM_EINVAL and shared(bbm, o=bad) == bbm.BBM_EINVAL
    for bad in OVERLAP:
        assert shared(bbm, o=pk(**bad)) == bbm.BBM_EINVAL
    for kw in (dict(T=-1), dict(R=0), dict(H=3), dict(cu=None), dict(lens=None), dict(table=None), dict(lens=P + 2), dict(lse=P + 2), dict(stride=3), dict(width=0), dict(max_shared=0),
               dict(max_own=0), dict(mask=P + 4, words=1), dict(mask=P, words=0), dict(words=1), dict(scale=0.0), dict(scale=math.nan), dict(ws=P + 8), dict(S=-1), dict(S=3),
               dict(group=None), dict(shared=None), dict(group=P + 2), dict(shared=P + 1)):
        assert shared(bbm, **kw) == bbm.BBM_EINVAL, kw
    for kw in (dict(T=1 << 31), dict(T=1 << 30), dict(scale=2.0 ** -101), dict(width=(1 << 24) + 1, stride=1 << 26), dict(mask=P, words=(1 << 20) + 1)):
        assert shared(bbm, **kw) == bbm.BBM_EUNSUPPORTED, kw
    # an output or the workspace in the place of an input or of another output
    for kw in (dict(o=pk()), dict(lse=9 * P), dict(lse=P), dict(o=pk(3 * P)), dict(o=pk(6 * P)), dict(lse=7 * P), dict(o=pk(10 * P)), dict(ws=4 * P), dict(ws=9 * P), dict(ws=6 * P)):
        assert shared(bbm, **kw) == bbm.BBM_EINVAL, kw
    assert shared(bbm, T=0) == bbm.BBM_OK and shared(bbm, T=0, S=0, group=None, shared=None) == bbm.BBM_OK
    sizes = bbm.bbm_kv4_shared_attn_workspace_bytes
    need = sizes(3, 2, 1, 4, 2, 64, 4096, 64)
    assert need > 0 and shared(bbm, ws_bytes=need - 1) == bbm.BBM_EWORKSPACE and shared(bbm, ws=None) == bbm.BBM_EWORKSPACE
    assert sizes(3, 2, 0, 4, 2, 64, 4096, 64) == 0 and sizes(3, 2, 1, 4, 2, 64, 256, 64) == 0   # one part of each request: nothing to join
    assert shared(bbm, max_shared=256, ws=None, ws_bytes=0, T=0) == bbm.BBM_OK
    assert sizes(0, 2, 1, 4, 2, 64, 4096, 64) == 0 and sizes(3, 2, 3, 4, 2, 64, 4096, 64) == 0 and sizes(3, 2, 1, 4, 3, 64, 4096, 64) == 0 and sizes(3, 2, 1, 4, 2, 96, 4096, 64) == 0
    assert sizes(1 << 20, 1 << 20, 1 << 20, 256, 1, 128, 1 << 62, 1 << 62) > 1 << 35   # (no product wraps)


def weights(bbm, q=None, lse=2 * P, T=3, R=2, cu=3 * P, lens=4 * P, table=5 * P, stride=4, width=4, S=1, group=6 * P, shared=7 * P, mask=None, words=0, c=None, H=4, scale=0.125, decay=0.5,
            w=8 * P, out=9 * P, max_shared=256, max_own=64):
    return bbm.lib.bbm_kv4_weights(q or pk(), lse, T, R, cu, lens, table, stride, width, S, group, shared, mask, words, c or cache(k=10 * P), H, scale, decay, w, out, max_shared, max_own, None)


def test_weights_refuses(bbm):
    for bad in BAD_CACHE:
        assert weights(bbm, c=cache(**bad)) == bbm.BBM_EINVAL
    for bad in ODD_CACHE:
        assert weights(bbm, c=cache(**bad)) == bbm.BBM_EUNSUPPORTED
    for bad in BAD_PACKED:
        if bad is not None:
            assert weights(bbm, q=bad) == bbm.BBM_EINVAL
    for kw in (dict(T=-1), dict(R=0), dict(H=3), dict(cu=None), dict(lens=None), dict(table=None), dict(lens=P + 2), dict(lse=P + 2), dict(lse=None), dict(stride=3), dict(width=0),
               dict(max_shared=0), dict(max_own=0), dict(mask=P + 4, words=1), dict(mask=P, words=0), dict(words=1), dict(scale=0.0), dict(scale=math.nan), dict(S=-1), dict(S=3),
               dict(group=None), dict(shared=None), dict(group=P + 2), dict(shared=P + 1), dict(decay=-0.5), dict(decay=1.5), dict(decay=math.nan), dict(w=None), dict(out=None),
               dict(w=P + 4), dict(out=P + 8), dict(out=P), dict(out=2 * P), dict(out=5 * P), dict(out=6 * P), dict(out=10 * P)):
        assert weights(bbm, **kw) == bbm.BBM_EINVAL, kw
    for kw in (dict(T=1 << 31), dict(T=1 << 30), dict(scale=2.0 ** -101), dict(width=(1 << 24) + 1, stride=1 << 26), dict(mask=P, words=(1 << 20) + 1),
               dict(R=1 << 18), dict(R=1 << 24)):
        assert weights(bbm, **kw) == bbm.BBM_EUNSUPPORTED, kw
    assert weights(bbm, T=0) == bbm.BBM_OK and weights(bbm, T=0, S=0, group=None, shared=None, lse=None) == bbm.BBM_OK


def evict(bbm, c=None, w=P, R=2, lens=2 * P, table=3 * P, stride=4, width=4, budget=100, recent=10, first=4 * P, new=5 * P, free=6 * P, n_free=9, at=7 * P, nxt=8 * P, max_len=256, ws=9 * P,
          ws_bytes=8):
    return bbm.lib.bbm_kv4_evict(c or cache(k=10 * P, ks=11 * P, v=12 * P, vs=13 * P), w, R, lens, table, stride, width, budget, recent, first, new, free, n_free, at, nxt, max_len, ws, ws_bytes,
                                 None)


def test_evict_refuses(bbm):
    for bad in BAD_CACHE:
        assert evict(bbm, c=cache(**bad)) == bbm.BBM_EINVAL
    for bad in ODD_CACHE:
        assert evict(bbm, c=cache(**bad)) == bbm.BBM_EUNSUPPORTED
    for kw in (dict(w=None), dict(w=P + 4), dict(R=0), dict(lens=None), dict(lens=P + 2), dict(table=None), dict(stride=3), dict(width=0), dict(budget=0), dict(recent=-1), dict(first=P + 2),
               dict(new=None), dict(new=P + 1), dict(free=None), dict(at=None), dict(nxt=None), dict(n_free=-1), dict(free=P + 2), dict(at=P + 2), dict(nxt=P + 2), dict(max_len=0),
               dict(ws=P + 8), dict(w=3 * P), dict(new=3 * P), dict(nxt=7 * P), dict(free=2 * P), dict(ws=2 * P), dict(new=4 * P), dict(new=P), dict(ws=8 * P), dict(w=10 * P)):
        assert evict(bbm, **kw) == bbm.BBM_EINVAL, kw
    for kw in (dict(R=16385, ws_bytes=1 << 20), dict(width=(1 << 24) + 1, stride=1 << 26), dict(budget=(1 << 19) + 1, width=1 << 20, stride=1 << 20),
               dict(R=16384, ws_bytes=1 << 20, c=cache(k=10 * P, ks=11 * P, v=12 * P, vs=13 * P, Hk=257))):
        assert evict(bbm, **kw) == bbm.BBM_EUNSUPPORTED, kw
    assert evict(bbm, ws=None) == bbm.BBM_EWORKSPACE and evict(bbm, ws_bytes=7) == bbm.BBM_EWORKSPACE
    assert bbm.bbm_kv4_evict_workspace_bytes(2, 2, 256) == 8 and bbm.bbm_kv4_evict_workspace_bytes(0, 2, 256) == 0


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
