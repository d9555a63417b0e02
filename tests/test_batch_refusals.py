"""What the batched attention and the calls that move tokens refuse, before anything is launched (no GPU needed: the
descriptors point nowhere)."""
import ctypes as C

import pytest

from paper_2401_18079_amd import binding as B

INVALID, UNSUPPORTED, CAPACITY, NOT_LOADED = 1, 2, 3, 5
PLACE = [1 << 20]


def cache(**ov):
    c = B._CCache()
    c.bits, c.head_dim, c.n_kv_heads, c.n_q_heads, c.k_side_v, c.loaded = 3, 128, 2, 4, 2, 1
    c.cap_tokens, c.n_tokens_k, c.n_tokens_v, c.cap_nnz_k, c.cap_nnz_v = 256, 100, 100, 4096, 4096
    c.rope_base = 10000.0
    for name in ("params", "k_codes", "v_codes", "v_sz", "k_ptr", "v_ptr", "k_idx", "k_val", "v_idx", "v_val", "d_status",
                 "workspace", "sink_k", "sink_v"):
        PLACE[0] += 1 << 20
        setattr(c, name, PLACE[0])
    c.workspace_bytes = 1 << 20
    for k, v in ov.items():
        setattr(c, k, v)
    return c


def table(cs):
    return (C.c_void_p * len(cs))(*[None if c is None else C.addressof(c) for c in cs])


def attend(prefix, own, n=None, q=1 << 16, out=1 << 16, ws=1 << 16, ws_bytes=1 << 40):
    lib = B.load_library()
    return lib.kvq_attention_decode_batch(None if prefix is None else C.byref(prefix), None if own is None else table(own),
                                          len(own) if n is None else n, q, 1.0, out, ws, ws_bytes, None)


def test_attention_refusals():
    a, b = cache(), cache()
    assert attend(None, None, 2) == INVALID and attend(None, [None, None]) == INVALID
    assert attend(a, [b], 0) == INVALID and attend(a, [b], -1) == INVALID
    for bad, status in ((dict(bits=4), INVALID), (dict(n_q_heads=2), INVALID), (dict(n_kv_heads=1), INVALID),
                        (dict(rope_base=5e5), INVALID), (dict(n_tokens_v=99), INVALID), (dict(loaded=0), NOT_LOADED),
                        (dict(k_codes=8), INVALID), (dict(v_ptr=0), INVALID), (dict(head_dim=64), UNSUPPORTED),
                        (dict(cap_tokens=250), INVALID), (dict(n_sink=5), INVALID), (dict(bits=5), UNSUPPORTED)):
        assert attend(a, [b, cache(**bad)]) == status, bad
    assert attend(a, [b], q=None) == INVALID and attend(a, [b], out=None) == INVALID and attend(a, [b], q=(1 << 16) + 2) == INVALID
    assert attend(a, [b], ws=None) == INVALID and attend(a, [b], ws=(1 << 16) + 8) == INVALID
    need = B.load_library().kvq_attention_decode_batch_workspace_bytes(C.byref(a), table([b]), 1)
    assert need > 0 and attend(a, [b], ws_bytes=need - 1) == CAPACITY
    assert B.load_library().kvq_attention_decode_batch_workspace_bytes(None, None, 1) == 0


def test_workspace_grows_with_the_tokens_only():
    f = B.load_library().kvq_attention_decode_batch_workspace_bytes
    a = cache(cap_tokens=1 << 20, n_tokens_k=1000, n_tokens_v=1000, cap_nnz_k=1 << 30, cap_nnz_v=1 << 30)
    small = f(C.byref(a), None, 1)
    a.n_tokens_k = a.n_tokens_v = 2000
    assert small < f(C.byref(a), None, 1) < 3 * small


def copy(dst, src, first, count):
    n = len(dst)
    return B.load_library().kvq_cache_copy(table(dst), table(src), (C.c_int64 * n)(*first), (C.c_int64 * n)(*count), n, None)


def test_copy_refusals():
    src = cache()
    for ov, first, count, status in (
            (dict(bits=2), 0, 10, INVALID), (dict(n_kv_heads=4), 0, 10, INVALID), (dict(rope_base=5e5), 0, 10, INVALID),
            (dict(n_tokens_v=3), 0, 10, INVALID), (dict(), 0, 157, CAPACITY), (dict(), 0, 101, INVALID), (dict(), 90, 11, INVALID),
            (dict(), -1, 5, INVALID), (dict(), 0, -1, INVALID), (dict(loaded=0), 0, 10, NOT_LOADED), (dict(k_ptr=0), 0, 1, INVALID),
            (dict(n_tokens_k=0, n_tokens_v=0, n_sink=2), 0, 10, INVALID),      # the source keeps no sink rows
            (dict(k_codes=src.k_codes), 0, 1, INVALID), (dict(v_codes=src.v_codes), 0, 1, INVALID)):
        d = cache(**ov)
        assert copy([d], [src], [first], [count]) == status, ov
        assert d.n_tokens_k == ov.get("n_tokens_k", 100)
    assert copy([src], [src], [0], [1]) == INVALID
    a, b = cache(), cache()
    assert copy([a, a], [src, src], [0, 0], [1, 1]) == INVALID               # a destination twice
    assert copy([a, b], [src, a], [0, 0], [1, 1]) == INVALID                 # a destination that is a source
    assert copy([a, cache(n_kv_heads=4, n_q_heads=4)], [src, cache(n_kv_heads=4, n_q_heads=4)], [0, 0], [1, 1]) == INVALID
    assert copy([a, None], [src, src], [0, 0], [1, 1]) == INVALID and copy([a], [None], [0], [1]) == INVALID
    assert copy([a], [cache(loaded=0)], [0], [1]) == NOT_LOADED
    lib = B.load_library()
    assert lib.kvq_cache_copy(None, None, None, None, 1, None) == INVALID and lib.kvq_cache_copy(None, None, None, None, -1, None) == INVALID
    assert lib.kvq_cache_copy(None, None, None, None, 0, None) == 0
    assert copy([a], [src], [0], [0]) == 0 and a.n_tokens_k == 100           # nothing to copy


def test_gather_and_truncate_refusals():
    lib = B.load_library()
    src, dst = cache(), cache()
    g = lambda d, s, t=1 << 16, n=5: lib.kvq_cache_gather(C.byref(d), C.byref(s), t, n, None)
    assert g(dst, src, None) == INVALID and g(dst, src, (1 << 16) + 2) == INVALID and g(dst, src, n=-1) == INVALID
    assert g(dst, src, n=157) == CAPACITY and g(src, src) == INVALID and g(cache(bits=2), src) == INVALID
    assert g(dst, cache(n_tokens_v=50)) == INVALID and g(dst, cache(n_tokens_k=0, n_tokens_v=0)) == INVALID
    assert g(cache(workspace=0), src) == CAPACITY and g(cache(workspace_bytes=7), src) == CAPACITY
    assert g(dst, src, n=0) == 0 and g(dst, cache(loaded=0)) == NOT_LOADED
    t = lambda c, n: lib.kvq_cache_truncate(C.byref(c), n)
    assert t(dst, 101) == INVALID and t(dst, -1) == INVALID and t(cache(n_tokens_v=50), 60) == INVALID and lib.kvq_cache_truncate(None, 0) == INVALID
    c = cache(n_tokens_v=50)
    assert t(c, 50) == 0 and (c.n_tokens_k, c.n_tokens_v) == (50, 50)
    assert t(c, 0) == 0 and (c.n_tokens_k, c.n_tokens_v) == (0, 0)
