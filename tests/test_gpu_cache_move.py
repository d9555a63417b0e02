"""kvq_cache_copy, kvq_cache_gather and kvq_cache_truncate: the destination's stored arrays are, bit for bit, those of the CPU
oracle's cache to which the same tokens were appended (quantization depends on a token alone, so no tolerance is needed)."""
import numpy as np
import pytest

import kvq_synth as S
from kvq_testlib import Setup, compare_caches
from test_gpu_batch_attention import SCALE, Seqs, both, call, close, queries, reference

pytestmark = pytest.mark.gpu

INVALID_ARG, NNZ_OVERFLOW = 1, 4


def moved(oc, src_rows, tokens):
    """Appends the listed rows of (k, v) to an oracle cache."""
    k, v = src_rows
    for t in range(0, len(tokens), 512):
        oc.append_k(k[tokens[t:t + 512]]); oc.append_v(v[tokens[t:t + 512]])


def setup(bits=3, heads=2, n=300, **ov):
    st = Setup(S.workload("c2", bits=bits, n_kv_heads=heads, n_q_heads=heads, **ov))
    return st, (st.k(0, n), st.v(0, n))


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("first,count,at", [(0, 300, 0), (0, 1, 0), (299, 1, 1), (31, 200, 33), (32, 64, 5), (1, 127, 64), (5, 258, 0),
                                            (64, 129, 127), (7, 2, 63), (100, 0, 10)])
def test_copy_of_a_run(bits, first, count, at):
    import torch
    import paper_2401_18079_amd as K
    st, rows = setup(bits, 3)
    sq = Seqs(st)
    _, src = sq.make(300)
    oc, dst = sq.make(at, seq=5, cap=512)
    K.kvq_cache_copy(dst, src, first, count)
    moved(oc, rows, np.arange(first, first + count))
    torch.cuda.synchronize()
    assert dst.status() == 0 and dst.n_tokens_k == dst.n_tokens_v == at + count
    assert not compare_caches(oc, dst)


@pytest.mark.parametrize("bits,heads,blocked_src,blocked_dst", [(3, 40, False, False), (2, 8, True, False), (4, 8, False, True), (3, 16, True, True)])
def test_copy_between_storages_and_longer_runs(bits, heads, blocked_src, blocked_dst):
    import paper_2401_18079_amd as K
    st, rows = setup(bits, heads, 1200)
    sq = Seqs(st)
    _, src = sq.make(1200, blocked=blocked_src)
    oc, dst = sq.make(77, seq=5, cap=1408, blocked=blocked_dst)
    K.kvq_cache_copy(dst, src, 101)
    moved(oc, rows, np.arange(101, 1200))
    assert not compare_caches(oc, dst)


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("kind", ["ascending", "any order", "repeats", "pairs", "one", "long"])
def test_gather(bits, kind):
    import torch
    import paper_2401_18079_amd as K
    n = 1500 if kind == "long" else 300
    st, rows = setup(bits, 3, n)
    sq = Seqs(st)
    _, src = sq.make(n, blocked=kind == "repeats")
    r = np.random.RandomState(bits)
    at = {"ascending": 0, "any order": 33, "repeats": 1, "pairs": 64, "one": 127, "long": 5}[kind]
    tokens = {"ascending": np.sort(r.permutation(n)[:130]), "any order": r.permutation(n), "repeats": r.randint(0, n, 400),
              "pairs": (2 * np.sort(r.permutation(n // 2)[:70])[:, None] + np.arange(2)).reshape(-1), "one": np.array([299]),
              "long": np.sort(r.permutation(n)[:1100])}[kind].astype(np.int32)
    oc, dst = sq.make(at, seq=5, cap=1280, blocked=kind == "any order")
    K.kvq_cache_gather(dst, src, torch.from_numpy(tokens).cuda())
    moved(oc, rows, tokens)
    assert dst.status() == 0 and not compare_caches(oc, dst)


def test_more_copies_than_one_launch_describes_and_shared_parents():
    import paper_2401_18079_amd as K
    st, _ = setup(3, 2)
    sq = Seqs(st)
    parents = [sq.make(40 + 9 * i, seq=i) for i in range(6)]
    r = np.random.RandomState(0)
    which = r.randint(0, 6, 29)
    first = [int(r.randint(0, 40)) for _ in which]
    count = [int(r.randint(0, parents[p][1].n_tokens_k - f + 1)) for p, f in zip(which, first)]
    dst = [sq.make(int(i % 5), seq=9, cap=256) for i in range(29)]
    K.kvq_cache_copy([d[1] for d in dst], [parents[p][1] for p in which], first, count)
    for d, p, f, c in zip(dst, which, first, count):
        n = parents[p][1].n_tokens_k
        moved(d[0], (st.k(0, n, p), st.v(0, n, p)), np.arange(f, f + c))
        assert d[1].status() == 0 and not compare_caches(*d)


def test_sink_rows_and_constants_of_an_empty_destination():
    import torch
    import paper_2401_18079_amd as K
    st, rows = setup(3, 2)
    sq = Seqs(st)
    so, src = sq.make(200, n_sink=3)
    for n_sink in (0, 1, 3):
        oc, _ = sq.make(0, n_sink=n_sink, cap=256)
        # not loaded: takes the source's constants
        dst = K.KvqCache(3, 2, 2, 256, st.k_side, st.wl.rope_base, 4096, n_sink=n_sink)
        K.kvq_cache_copy(dst, src, 0, 150)
        moved(oc, rows, np.arange(150))
        assert dst.c.loaded == src.c.loaded and torch.equal(dst.params, src.params)
        assert not compare_caches(oc, dst)
        q = queries(st.wl, 1)
        close(call(dst, None, q), *reference(oc, [None], q, SCALE, st.wl.rope_base))
    # a list: kept sinks in their places
    oc, dst = sq.make(0, n_sink=2, cap=256)
    tokens = np.array([0, 2, 5, 9, 100, 199], np.int32)
    K.kvq_cache_gather(dst, src, torch.from_numpy(tokens).cuda())
    moved(oc, rows, tokens)
    assert dst.status() == 0 and not compare_caches(oc, dst)
    assert np.array_equal(dst.sink_k.cpu().numpy().view(np.uint16), oc.sink_k.reshape(-1))
    # a token without an fp16 row in a sink's place
    _, bad = sq.make(0, n_sink=2, cap=256)
    K.kvq_cache_gather(bad, src, torch.from_numpy(tokens[2:]).cuda())
    assert bad.status() == INVALID_ARG


def test_thresholds_without_outliers_do_not_hide_copied_ones():
    """A destination whose own thresholds admit no Key outlier holds the source's after a copy: the mat-vecs must see them."""
    import torch
    import paper_2401_18079_amd as K
    st, rows = setup(3, 2)
    sq = Seqs(st)
    so, src = sq.make(200)
    wide = np.full(256, 65504.0, np.float16)
    dst = K.KvqCache(3, 2, 2, 256, st.k_side, st.wl.rope_base, 4096)
    K.kvq_lut_load(dst, st.lut_k, st.lut_v, st.s, st.z, -wide, wide)
    K.kvq_cache_copy(dst, src)
    q = torch.from_numpy(queries(st.wl, 1)[0]).cuda()
    a, b = torch.zeros(2, 256, device="cuda"), torch.zeros(2, 256, device="cuda")
    K.kvq_qk_matvec(src, q, SCALE, a)
    K.kvq_qk_matvec(dst, q, SCALE, b)
    assert int(src.k_ptr[200]) > 100 and torch.equal(a, b)


def test_indices_outside_the_source():
    import torch
    import paper_2401_18079_amd as K
    st, rows = setup(4, 2)
    sq = Seqs(st)
    _, src = sq.make(100)
    oc, dst = sq.make(0, cap=128)
    K.kvq_cache_gather(dst, src, torch.tensor([3, -1, 100, 7, 2 ** 31 - 1, -2 ** 31, 99], dtype=torch.int32, device="cuda"))
    assert dst.status() == INVALID_ARG
    k, v = rows
    z = np.zeros_like(k[:1])
    for t in (3, None, None, 7, None, None, 99):           # the good tokens are where they belong
        oc.append_k(z if t is None else k[t:t + 1]); oc.append_v(v[t:t + 1] if t is not None else np.zeros_like(v[:1]))
    for t in (0, 3, 6):
        assert np.array_equal(unpacked(dst, "k")[t], oc.unpack_k(t, 1)[0]) and np.array_equal(unpacked(dst, "v")[t], oc.unpack_v(t, 1)[0])
    p = dst.k_ptr.cpu().numpy()
    assert p[2] == p[1] and p[3] == p[2] and p[4] - p[3] == src.k_ptr[8].item() - src.k_ptr[7].item()


def unpacked(gc, side):
    """Codes [n, D] of a GPU cache by the oracle's reader."""
    from oracle import kvq_oracle as O
    n, c = gc.n_tokens_k, gc.c
    out = np.zeros((n, gc.D), np.uint8)
    f = O._unpack_k if side == "k" else O._unpack_v
    f((gc.k_codes if side == "k" else gc.v_codes).cpu().numpy(), c.bits, c.n_kv_heads, c.cap_tokens, 0, n, out)
    return out


@pytest.mark.parametrize("how", ["copy", "gather"])
def test_outliers_that_do_not_fit(how):
    """As an append into the same room leaves them: entries up to the capacity, pointers that stop there, the status set."""
    import torch
    import paper_2401_18079_amd as K
    st, rows = setup(3, 4, 300)
    sq = Seqs(st)
    _, src = sq.make(300)
    room = 704                                             # about half of the entries
    make = lambda: K.KvqCache(3, 4, 4, 384, st.k_side, st.wl.rope_base, room, room)  # noqa: E731
    want, got = make(), make()
    for c in (want, got):
        K.kvq_lut_load(c, st.lut_k, st.lut_v, st.s, st.z, st.lo, st.hi)
    K.kvq_quantize_append_k(want, torch.from_numpy(rows[0]).cuda())
    K.kvq_quantize_append_v(want, torch.from_numpy(rows[1]).cuda())
    if how == "copy":
        K.kvq_cache_copy(got, src)
    else:
        K.kvq_cache_gather(got, src, torch.arange(300, dtype=torch.int32, device="cuda"))
    assert want.status() == got.status() == NNZ_OVERFLOW
    for name in ("k_codes", "v_codes", "v_sz", "k_ptr", "v_ptr", "k_idx", "k_val", "v_idx", "v_val"):
        assert torch.equal(getattr(want, name), getattr(got, name)), name


def test_truncate_then_append():
    import torch
    import paper_2401_18079_amd as K
    st, rows = setup(3, 2)
    sq = Seqs(st)
    oc, dst = sq.make(0, cap=384, blocked=True)
    _, src = sq.make(300)
    K.kvq_cache_copy(dst, src)
    blocks = len(dst.blocks["k_idx"])
    K.kvq_cache_truncate(dst, 101)
    freed = dst.free_nnz_blocks()
    assert freed >= 0 and len(dst.blocks["k_idx"]) <= blocks and dst.c.cap_nnz_k == len(dst.blocks["k_idx"]) * 1024
    dst.ensure_nnz_room(199 * dst.D, 199 * 2 * st.k_side)
    K.kvq_quantize_append_kv(dst, torch.from_numpy(rows[0][150:250].copy()).cuda(), torch.from_numpy(rows[1][150:250].copy()).cuda())
    K.kvq_cache_copy(dst, src, 7, 99)
    moved(oc, rows, np.concatenate([np.arange(101), np.arange(150, 250), np.arange(7, 106)]))
    oc_codes = oc.k_codes.copy()
    assert dst.status() == 0 and not compare_caches(oc, dst)
    assert np.array_equal(oc_codes, dst.k_codes.cpu().numpy())


def test_graph_of_copies_replayed():
    """A captured copy and gather, replayed over changed sources with eager work between."""
    import torch
    import paper_2401_18079_amd as K
    st, rows = setup(4, 2)
    sq = Seqs(st)
    _, src = sq.make(300)
    _, a = sq.make(0, cap=384)
    _, b = sq.make(0, cap=384)
    tokens = torch.arange(0, 300, 3, dtype=torch.int32, device="cuda")
    K.kvq_cache_copy(a, src); K.kvq_cache_gather(b, src, tokens)          # modules loaded before the capture
    torch.cuda.synchronize()
    K.kvq_cache_truncate(a, 0); K.kvq_cache_truncate(b, 0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        K.kvq_cache_copy(a, src, 1, 250)
        K.kvq_cache_gather(b, src, tokens)
    for r in range(3):
        K.kvq_cache_truncate(src, 0)
        k, v = st.k(0, 300, seq=20 + r), st.v(0, 300, seq=20 + r)
        K.kvq_quantize_append_kv(src, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda())
        g.replay()
        for gc, which in ((a, np.arange(1, 251)), (b, np.arange(0, 300, 3))):
            oc, _ = sq.make(0, cap=384)
            moved(oc, (k, v), which)
            assert gc.status() == 0
            bad = [x for x in compare_caches(oc, gc) if "codes" not in x]  # behind the tokens the codes of earlier rounds remain
            assert not bad, bad
            assert np.array_equal(unpacked(gc, "k"), oc.unpack_k(0, len(which))) and np.array_equal(unpacked(gc, "v"), oc.unpack_v(0, len(which)))


def test_serving_run():
    """As a server uses them together: a prompt, four continuations forked behind it, steps of a beam search (append, attend
    over prompt and own tokens, take over parents), a draft rejected, the prompt compacted and attended to again."""
    import torch
    import paper_2401_18079_amd as K
    wl = S.workload("c4", bits=3, n_kv_heads=2, n_q_heads=8)
    st = Setup(wl)
    sq = Seqs(st)
    po, pg = sq.make(333, n_sink=1)
    B = 4
    cur = [sq.make(0, cap=128) for _ in range(B)]
    spare = [sq.make(0, cap=128) for _ in range(B)]
    r = np.random.RandomState(5)
    hist = [[] for _ in range(B)]                          # (seq, token) of every own token
    for step in range(6):
        for b in range(B):
            k, v = st.k(step, 1, seq=30 + b), st.v(step, 1, seq=30 + b)
            cur[b][0].append_k(k); cur[b][0].append_v(v)
            K.kvq_quantize_append_kv(cur[b][1], torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda())
            hist[b].append((30 + b, step))
        q = queries(wl, B, seed=step)
        got = call(pg, both(cur, 1), q)
        close(got, *reference(po, both(cur, 0), q, SCALE, wl.rope_base))
        parents = [int(x) for x in r.randint(0, B, B)]
        for s in spare:
            K.kvq_cache_truncate(s[1], 0)
        K.kvq_cache_copy([s[1] for s in spare], [cur[p][1] for p in parents])
        hist = [list(hist[p]) for p in parents]
        fresh = [sq.make(0, cap=128) for _ in range(B)]
        for b in range(B):
            for s, t in hist[b]:
                fresh[b][0].append_k(st.k(t, 1, seq=s)); fresh[b][0].append_v(st.v(t, 1, seq=s))
            assert np.array_equal(unpacked(spare[b][1], "v"), fresh[b][0].unpack_v(0, len(hist[b])))
        cur, spare = [(fresh[b][0], spare[b][1]) for b in range(B)], cur
    # drafts of two tokens rejected
    for b in range(B):
        K.kvq_cache_truncate(cur[b][1], 4)
        oc, _ = sq.make(0, cap=128)
        for s, t in hist[b][:4]:
            oc.append_k(st.k(t, 1, seq=s)); oc.append_v(st.v(t, 1, seq=s))
        cur[b] = (oc, cur[b][1])
    # the prompt keeps its first and its latest tokens and some between
    keep = np.concatenate([[0], np.sort(1 + r.permutation(250)[:60]), np.arange(260, 333)]).astype(np.int32)
    co, cg = sq.make(0, n_sink=1, cap=256)
    K.kvq_cache_gather(cg, pg, torch.from_numpy(keep).cuda())
    moved(co, (st.k(0, 333), st.v(0, 333)), keep)
    assert cg.status() == 0 and not compare_caches(co, cg)
    q = queries(wl, B, seed=9)
    close(call(cg, both(cur, 1), q), *reference(co, both(cur, 0), q, SCALE, wl.rope_base))
