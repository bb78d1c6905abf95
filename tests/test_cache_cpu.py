"""Host side of the cache's entry points without a GPU: sizes, and what is refused before anything touches CUDA."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2505_21036_b200 import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, SMALL = 1, 2, 3


def cache(**kw):
    a = dict(n_seqs=2, heads=3, D=64, n_pages=10, max_pages=4, k=4096, v=4096, k_scale=4096, v_scale=4096, k_sum=4096, page_table=4096, seq_len=4096)
    a.update(kw)
    return api.rf_cache(*(a[n] for n, _ in api.rf_cache._fields_))


def query(H=6, M=5, causal=0, scale=0.0):
    return api.rf_cache_query(H, M, causal, scale)


def calls(c, ws=4096, ws_bytes=1 << 40, u=None, q=4096, o=4096, sched=None):
    """The codes of every entry point given this cache (all pointers are made up: a call that got past the checks would launch)."""
    lib, c, u = api.load(), C.byref(c), C.byref(u or query())
    s = C.byref(sched or api.rf_schedule(4096, 4096, None, None, 1, 4))
    return [lib.rf_cache_append(c, q, q, 5, None, ws, ws_bytes, None, None), lib.rf_cache_fork(c, 4096, None, None),
            lib.rf_cache_drop(c, None, None, 4096, None, None), lib.rf_cache_compact(c, 4096, ws, ws_bytes, None, None),
            lib.rf_cache_select(c, u, q, None, 0, 0, 4, s, None, None), lib.rf_cache_attn_fwd(c, u, q, None, None, o, None, ws, ws_bytes, None, None)]


@pytest.mark.parametrize("kw,code", [(dict(n_seqs=0), INVALID), (dict(heads=0), INVALID), (dict(D=0), INVALID), (dict(D=80), UNSUPPORTED), (dict(D=256), UNSUPPORTED),
                                     (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=-1), INVALID), (dict(n_seqs=1025), UNSUPPORTED),
                                     (dict(n_seqs=1000, heads=66), UNSUPPORTED), (dict(n_pages=(1 << 19) + 1), UNSUPPORTED), (dict(max_pages=(1 << 23) + 1), UNSUPPORTED),
                                     (dict(n_pages=1 << 19, heads=5000, n_seqs=1), UNSUPPORTED), (dict(k=None), INVALID), (dict(v=4104), INVALID), (dict(k_scale=None), INVALID),
                                     (dict(v_scale=4097), INVALID), (dict(k_sum=4100), INVALID), (dict(page_table=None), INVALID), (dict(seq_len=4098), INVALID)])
def test_bad_caches(kw, code):
    c = cache(**kw)
    assert calls(c) == [code] * 6
    assert api.load().rf_cache_workspace_bytes(C.byref(c)) == 0
    assert api.load().rf_cache_attn_workspace_bytes(C.byref(c), C.byref(query())) == 0


def test_null_structs():
    lib = api.load()
    assert lib.rf_cache_workspace_bytes(None) == 0 and lib.rf_cache_fork(None, 4096, None, None) == INVALID
    assert lib.rf_cache_attn_workspace_bytes(C.byref(cache()), None) == 0
    assert lib.rf_cache_attn_fwd(C.byref(cache()), None, 4096, None, None, 4096, None, 4096, 1 << 40, None, None) == INVALID
    assert lib.rf_cache_select(C.byref(cache()), C.byref(query()), 4096, None, 0, 0, 1, None, None, None) == INVALID


@pytest.mark.parametrize("u,code", [(query(H=0), INVALID), (query(H=7), INVALID), (query(M=0), INVALID), (query(causal=-1), INVALID), (query(scale=float("nan")), INVALID),
                                    (query(scale=float("inf")), INVALID), (query(scale=-0.1), INVALID), (query(H=3, M=(1 << 30) + 1), UNSUPPORTED), (query(H=6, M=1 << 30), UNSUPPORTED)])
def test_bad_queries(u, code):
    assert calls(cache(), u=u)[4:] == [code] * 2
    assert api.load().rf_cache_attn_workspace_bytes(C.byref(cache()), C.byref(u)) == 0


def test_bad_pointers_workspaces_and_lists():
    lib, c, u = api.load(), cache(), query()
    ref, uref = C.byref(c), C.byref(u)
    need, attn = lib.rf_cache_workspace_bytes(ref), lib.rf_cache_attn_workspace_bytes(ref, uref)
    assert need >= 8 * 10 and attn > 0
    got = calls(c, ws=None)
    assert [got[i] for i in (0, 3, 5)] == [INVALID] * 3
    got = calls(c, ws=4096 + 128)
    assert [got[i] for i in (0, 3, 5)] == [INVALID] * 3
    assert lib.rf_cache_append(ref, 4096, 4096, 5, None, 4096, need - 1, None, None) == SMALL
    assert lib.rf_cache_compact(ref, 4096, 4096, need - 1, None, None) == SMALL
    assert lib.rf_cache_attn_fwd(ref, uref, 4096, None, None, 4096, None, 4096, attn - 1, None, None) == SMALL
    for q in (None, 4104):
        got = calls(c, q=q)
        assert [got[i] for i in (0, 4, 5)] == [INVALID] * 3
    assert calls(c, o=None)[5] == INVALID and calls(c, o=4104)[5] == INVALID
    assert lib.rf_cache_append(ref, 4096, 4096, 0, None, 4096, need, None, None) == INVALID
    assert lib.rf_cache_append(ref, 4096, 4096, (1 << 30) + 1, None, 4096, need, None, None) == UNSUPPORTED
    assert lib.rf_cache_fork(ref, None, None, None) == INVALID
    assert lib.rf_cache_drop(ref, None, None, None, None, None) == INVALID
    assert lib.rf_cache_drop(ref, 4096, None, None, None, None) == INVALID and lib.rf_cache_drop(ref, None, 4096, 4096, None, None) == INVALID
    assert lib.rf_cache_compact(ref, None, 4096, need, None, None) == INVALID
    for s in (api.rf_schedule(None, 4096, None, None, 1, 4), api.rf_schedule(4096, None, None, None, 1, 4), api.rf_schedule(4096, 4096, None, None, 2, 4),
              api.rf_schedule(4096, 4096, None, None, 1, 0)):
        assert calls(c, sched=s)[4] == INVALID
        assert lib.rf_cache_attn_fwd(ref, uref, 4096, None, C.byref(s), 4096, None, 4096, attn, None, None) == INVALID
    s = api.rf_schedule(4096, 4096, None, None, 1, 3)
    for first, last, top in ((-1, 0, 1), (0, -1, 1), (0, 0, -1), (0, 0, 4), (2, 1, 1), (1 << 30, 1 << 30, 1 << 30)):
        assert lib.rf_cache_select(ref, uref, 4096, None, first, last, top, C.byref(s), None, None) == INVALID
    long = cache(max_pages=16385)
    s = api.rf_schedule(4096, 4096, None, None, 1, 4)
    assert lib.rf_cache_select(C.byref(long), uref, 4096, None, 0, 0, 4, C.byref(s), None, None) == UNSUPPORTED


def test_status_strings_of_the_cache():
    lib = api.load()
    assert b"room" in lib.rf_status_string(8) and b"NaN" in lib.rf_status_string(9)


def test_structures_as_plain_c_sees_them(tmp_path):
    src = tmp_path / "probe.c"
    src.write_text('#include <stdio.h>\n#include "rainfusion.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu %zu %d %d %d\\n", sizeof(rf_cache), offsetof(rf_cache, k), '
                   'offsetof(rf_cache, k_sum), offsetof(rf_cache, seq_len), sizeof(rf_cache_query), offsetof(rf_cache_query, causal_block), '
                   'offsetof(rf_cache_query, scale), RF_CACHE_PAGE, RF_ERR_CACHE_FULL, RF_ERR_NOT_FINITE); return 0; }\n')
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    A, Q = api.rf_cache, api.rf_cache_query
    assert got == [C.sizeof(A), A.k.offset, A.k_sum.offset, A.seq_len.offset, C.sizeof(Q), Q.causal_block.offset, Q.scale.offset, api.CACHE_PAGE, 8, 9]
