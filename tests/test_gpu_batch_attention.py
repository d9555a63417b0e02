"""kvq_attention_decode_batch against the softmax of paper Sec. 3 in 64 bits, over Keys and Values reconstructed by the CPU
oracle from its own codes and outliers (the GPU caches hold the same bits).

Tolerance, from the arithmetic.  A rotated pair is off by the angle's and the hardware's errors: a product of position and
frequency in two floats (1e-7 revolutions, 6.3e-7 rad), plus one rounding of an angle of at most 6 revolutions (2^-22
revolutions, 1.5e-6 rad), plus 1e-6 of the sine and cosine: 3.2e-6 of |k_i| + |k_i+64| for either channel.  Two-part factors
leave 2^-21 (Keys, truncated twice) and 2^-22 (query) of a product, the fp32 sum over 3 * 128 products 384 * 2^-24 of the
sum of their sizes at worst.  With A = scale * sum over pairs (|q_i| + |q_i+64|) (|k_i| + |k_i+64|) a score is off by at most
dx = A * (3.2e-6 + 0.8e-6 + 23e-6); the rounding of the sum is a random walk, sqrt(384) * 2^-24 = 1.2e-6, and 4 times that is
taken: dx = A * 9e-6.  A weight is off by dx, twice that relative to the others; its two parts leave 2^-21, and the sums over
n tokens another random walk, 4 * sqrt(4 n) * 2^-24.  So |out - ref| <= (2 max dx + 2^-21 + sqrt(n) * 4.8e-7) * sum p |v| with |v| the
sum of the sizes of the parts (dense, zero-point, residual): at most |vhat| + 2 |residual + z|, taken as 3 max |v| of the channel.
Where the two parts end at fp16's smallest step, 2^-24, |k| below 1/64 loses that much more: such cases say so.
"""
import numpy as np
import pytest

import kvq_synth as S
from oracle import kvq_oracle as O
from kvq_testlib import Setup, compare_caches

pytestmark = pytest.mark.gpu

SCALE = float(np.float32(1.0 / np.sqrt(128.0)))


class Seqs:
    """Caches of one layer, each on the GPU and in the oracle with the same tokens."""

    def __init__(self, st):
        self.st = st

    def make(self, tokens, seq=0, n_sink=0, blocked=False, cap=None, k_rows=None, v_rows=None, nnz=None):
        import torch
        import paper_2401_18079_amd as K
        st, wl = self.st, self.st.wl
        cap = cap or max(128, (tokens + 127) // 128 * 128)
        nnz = nnz or max(1024, min(cap * wl.D, 4 * st.cap_nnz_k(cap)))
        oc = O.OracleCache(wl.bits, wl.n_kv_heads, wl.n_q_heads, cap, st.k_side, wl.rope_base, st.lut_k, st.lut_v, st.s, st.z,
                           st.lo, st.hi, cap_nnz_k=nnz, n_sink=n_sink)
        gc = K.KvqCache(wl.bits, wl.n_kv_heads, wl.n_q_heads, cap, st.k_side, wl.rope_base, nnz, n_sink=n_sink,
                        nnz_block_entries=1024 if blocked else None)
        K.kvq_lut_load(gc, st.lut_k, st.lut_v, st.s, st.z, st.lo, st.hi)
        for t in range(0, tokens, 512):
            T = min(512, tokens - t)
            k = st.k(t, T, seq) if k_rows is None else k_rows[t:t + T]
            v = st.v(t, T, seq) if v_rows is None else v_rows[t:t + T]
            oc.append_k(k); oc.append_v(v)
            K.kvq_quantize_append_k(gc, torch.from_numpy(k).cuda())
            K.kvq_quantize_append_v(gc, torch.from_numpy(v).cuda())
        return oc, gc


def rows(oc):
    """(Keys, Values) [n, D] in 64 bits as the mat-vecs see them: sink tokens from their fp16 rows."""
    n, D = oc.n_k, oc.D
    if n == 0:
        return np.zeros((0, D)), np.zeros((0, D))
    k, v = oc.reconstruct_k(0, n), oc.reconstruct_v(0, n)
    s = min(oc.n_sink, n)
    k[:s], v[:s] = oc.sink_k[:s].view(np.float16), oc.sink_v[:s].view(np.float16)
    return k, v


def reference(prefix, own, q, scale, base):
    """(out, tolerance) [B, Hq, 128] for sequences prefix + own[b] (oracle caches or None)."""
    B, Hq, _ = q.shape
    out, tol = np.zeros((B, Hq, 128)), np.zeros((B, Hq, 128))
    some = next(c for c in [prefix] + list(own) if c is not None)
    R = Hq // some.H
    theta = base ** (-np.arange(64) / 64.0)
    for b in range(B):
        parts = [rows(c) for c in (prefix, own[b]) if c is not None]
        k, v = (np.concatenate([p[i] for p in parts]) if parts else np.zeros((0, some.D)) for i in (0, 1))
        n = len(k)
        if n == 0:
            continue
        ang = np.outer(np.arange(n), theta)
        c, s = np.cos(ang), np.sin(ang)
        for h in range(some.H):
            kh, vh = k[:, h * 128:h * 128 + 128], v[:, h * 128:h * 128 + 128]
            rot = np.concatenate([kh[:, :64] * c - kh[:, 64:] * s, kh[:, 64:] * c + kh[:, :64] * s], 1)
            size_k = np.abs(kh[:, :64]) + np.abs(kh[:, 64:])
            for r in range(R):
                x = q[b, h * R + r].astype(np.float64)
                sc = rot @ x * scale
                p = np.exp(sc - sc.max())
                p /= p.sum()
                out[b, h * R + r] = p @ vh
                dx = 9e-6 * abs(scale) * (size_k @ (np.abs(x[:64]) + np.abs(x[64:]))).max()
                tol[b, h * R + r] = (2 * dx + 2.0 ** -21 + np.sqrt(n) * 4.8e-7) * 3 * (p @ np.abs(vh) + np.abs(vh).max() * 2.0 ** -10)
    return out, tol


def close(got, ref, tol):
    got = got.cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all()
    err = np.abs(got - ref)
    worst = float(np.max(err / np.maximum(tol, 1e-300), initial=0.0, where=tol > 0))
    assert np.all(err <= tol), f"worst error / tolerance {worst:.3f}"
    return worst


def queries(wl, B, seed=0, gain=1.0):
    r = np.random.RandomState(seed + 11)
    return (r.standard_normal((B, wl.n_q_heads, 128)) * gain).astype(np.float32)


def call(prefix, own, q, **kw):
    import torch
    import paper_2401_18079_amd as K
    out = torch.full(q.shape, 77.0, device="cuda")
    K.kvq_attention_decode_batch(prefix, own, torch.from_numpy(q).cuda() if isinstance(q, np.ndarray) else q, SCALE, out, **kw)
    return out


def both(pairs, i):
    return None if pairs is None else [None if p is None else p[i] for p in pairs]


@pytest.mark.parametrize("name,ov,prefix,own,sink,blocked", [
    ("c2", dict(n_kv_heads=2, n_q_heads=2), 300, [1, 0, 33], 0, False),
    ("c2", dict(n_kv_heads=1, n_q_heads=1), 1, [0, 1], 0, False),                          # the smallest lengths
    ("c2", dict(n_kv_heads=3, n_q_heads=3, bits=2), 129, [31, 32, 65, 64], 0, False),
    ("c2", dict(n_kv_heads=2, n_q_heads=16, bits=4), 257, [5] * 3, 0, True),               # 24 queries: two blocks of 16
    ("c4", dict(n_kv_heads=2, n_q_heads=8), 1000, [0, 7, 200, 1, 2], 1, False),            # grouped, one sink, 2-bit
    ("c2", dict(n_kv_heads=1, n_q_heads=5), 96, [40, 3], 0, False),                        # five query heads per KV head
    ("c3", dict(n_kv_heads=1, n_q_heads=40), 70, [90, 0], 2, False),                       # 40 of them: own tokens in blocks of 64
    ("c2", dict(n_kv_heads=2, n_q_heads=4, outlier_fraction=0.3), 161, [50, 60], 0, True), # more outliers of a head and 32 tokens than lanes
    ("c2", dict(n_kv_heads=2, n_q_heads=2, outlier_fraction=0.0), 200, [10, 20], 0, False),
    ("c2", dict(n_kv_heads=8, n_q_heads=8), 2100, [3] * 40, 4, False),                     # 40 queries, prefix in several workgroups
    ("c2", dict(n_kv_heads=1, n_q_heads=2), 3, [2, 0], 4, False),                          # fewer tokens than sinks
    # more than 32 queries of a KV head: tiles of 64 tokens shared by 64 or 128 of them
    ("c2", dict(n_kv_heads=2, n_q_heads=16, bits=2), 385, [0, 9, 40, 1, 2], 2, False),     # 40, sinks, last tile of one token
    ("c2", dict(n_kv_heads=1, n_q_heads=8, outlier_fraction=0.3), 290, [3] * 8, 0, False), # 64, more outliers than lanes
    ("c2", dict(n_kv_heads=1, n_q_heads=9, outlier_fraction=0.2, bits=4), 225, [3] * 8, 1, True),   # 72, likewise, blocked storage
    ("c4", dict(n_kv_heads=1, n_q_heads=8), 2500, [1] * 20, 0, False),                     # 160: two blocks of 128, many tiles
    ("c2", dict(n_kv_heads=1, n_q_heads=70), 33, [65, 1], 0, False),                       # 70 of one sequence
    ("c2", dict(n_kv_heads=2, n_q_heads=66, outlier_fraction=0.0), 64, [31, 0], 0, False), # 33 of one sequence, no outliers
])
def test_batch_matches_the_definition(name, ov, prefix, own, sink, blocked):
    wl = S.workload(name, **ov)
    sq = Seqs(Setup(wl))
    pre = sq.make(prefix, n_sink=sink, blocked=blocked)
    per = [sq.make(n, seq=1 + i) if n or i % 2 else None for i, n in enumerate(own)]
    assert not compare_caches(*pre)
    q = queries(wl, len(own))
    got = call(pre[1], both(per, 1), q)
    ref, tol = reference(pre[0], both(per, 0), q, SCALE, wl.rope_base)
    close(got, ref, tol)
    # the same without the sequences' own tokens, and without the prefix
    got = call(pre[1], None, q)
    close(got, *reference(pre[0], [None] * len(own), q, SCALE, wl.rope_base))
    if any(p is not None for p in per):
        got = call(None, both(per, 1), q)
        close(got, *reference(None, both(per, 0), q, SCALE, wl.rope_base))


@pytest.mark.parametrize("heads,ratio,fraction,bits", [(16, 1, 0.01, 3), (17, 1, 0.01, 3), (17, 2, 0.3, 4), (64, 1, 0.05, 2), (80, 1, 0.01, 3)])
def test_wide_layers(heads, ratio, fraction, bits):
    """Outliers of a token over 16, 17, 64 and 80 heads: both sizes of the sort, more than one head a lane, lists read twice."""
    wl = S.workload("c2", n_kv_heads=heads, n_q_heads=heads * ratio, outlier_fraction=fraction, bits=bits)
    sq = Seqs(Setup(wl))
    pre = sq.make(101)
    per = [sq.make(n, seq=1 + n) for n in (3, 70)]
    assert not compare_caches(*pre)
    q = queries(wl, 2)
    close(call(pre[1], both(per, 1), q), *reference(pre[0], both(per, 0), q, SCALE, wl.rope_base))


def test_two_calls_at_once():
    """Two streams, each with its workspace, over the same caches."""
    import torch
    import paper_2401_18079_amd as K
    wl = S.workload("c2", n_kv_heads=4, n_q_heads=8)
    sq = Seqs(Setup(wl))
    pre, per = sq.make(700), [sq.make(20 + i, seq=1 + i) for i in range(3)]
    q = [torch.from_numpy(queries(wl, 3, seed=s)).cuda() for s in range(2)]
    ref = [call(pre[1], both(per, 1), x) for x in q]
    outs = [[torch.zeros_like(ref[0]) for _ in range(8)] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(8):
        for j in range(2):
            K.kvq_attention_decode_batch(pre[1], both(per, 1), q[j], SCALE, outs[j][i], stream=streams[j])
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref[j]) for j in range(2) for o in outs[j])


def test_more_sequences_than_one_launch_describes():
    wl = S.workload("c2", n_kv_heads=2, n_q_heads=4)
    sq = Seqs(Setup(wl))
    lens = [(7 * i) % 50 for i in range(53)]
    pre = sq.make(150)
    per = [sq.make(n, seq=i) for i, n in enumerate(lens)]
    q = queries(wl, len(lens))
    close(call(pre[1], both(per, 1), q), *reference(pre[0], both(per, 0), q, SCALE, wl.rope_base))


def test_one_cache_several_times_and_an_empty_batch():
    import torch
    wl = S.workload("c2", n_kv_heads=2, n_q_heads=2)
    sq = Seqs(Setup(wl))
    a, b, empty = sq.make(70), sq.make(40, seq=2), sq.make(0)
    q = queries(wl, 4)
    per = [b, a, b, empty]
    before = [t.clone() for t in (a[1].k_codes, a[1].v_codes, a[1].v_sz, a[1].k_ptr, a[1].v_ptr, a[1].k_idx, a[1].v_val, a[1].workspace)]
    close(call(a[1], both(per, 1), q), *reference(a[0], both(per, 0), q, SCALE, wl.rope_base))
    after = (a[1].k_codes, a[1].v_codes, a[1].v_sz, a[1].k_ptr, a[1].v_ptr, a[1].k_idx, a[1].v_val, a[1].workspace)
    assert all(torch.equal(x, y) for x, y in zip(before, after))
    assert torch.all(call(empty[1], None, q) == 0.0)
    assert torch.all(call(empty[1], [None, empty[1], empty[1], None], q) == 0.0)
    got = call(empty[1], both(per, 1), q)
    assert torch.all(got[3] == 0.0)
    close(got[:3], *reference(None, both(per[:3], 0), q[:3], SCALE, wl.rope_base))


@pytest.mark.parametrize("what", ["large scores", "large keys", "uneven value scales", "tiny values", "large values"])
def test_extreme_inputs(what):
    """Inputs at the ends of fp16's range, through both parts of the call."""
    wl = S.workload("c2", n_kv_heads=2, n_q_heads=4)
    st = Setup(wl)
    sq = Seqs(st)
    n, gain = 200, 1.0
    k, v = st.k(0, n).astype(np.float32), st.v(0, n).astype(np.float32)
    if what == "large scores":
        gain = 40.0
    elif what == "large keys":
        k[5::17, 3] = 65504.0                 # outliers of 65504, both channels of a pair in some tokens
        k[5::34, 67] = -65504.0
        gain = 1e-3
    elif what == "uneven value scales":
        v *= np.exp2(np.linspace(-9, 9, n))[:, None]
    elif what == "tiny values":
        v *= 2.0 ** -12
    else:
        v = np.clip(v * 12000.0, -65504, 65504)
    k, v = k.astype(np.float16), v.astype(np.float16)
    pre = sq.make(n, k_rows=k, v_rows=v)
    per = [sq.make(90, k_rows=k[::-1].copy(), v_rows=v[::-1].copy()), None, sq.make(33, k_rows=k[40:], v_rows=v[40:])]
    q = queries(wl, 3, gain=gain)
    close(call(pre[1], both(per, 1), q), *reference(pre[0], both(per, 0), q, SCALE, wl.rope_base))


@pytest.mark.parametrize("ratio", [2, 8])
def test_what_a_sink_token_holds_in_codes_is_not_read(ratio):
    """Sink tokens come from their fp16 rows: infinite residuals and scales in their compressed form reach no sum."""
    import torch
    wl = S.workload("c2", n_kv_heads=2, n_q_heads=2 * ratio)
    sq = Seqs(Setup(wl))
    pre = sq.make(300, n_sink=3)
    per = [sq.make(40, seq=1 + i, n_sink=2, blocked=i == 1) for i in range(6)]
    for oc, gc in [pre] + per:
        n = int(gc.v_ptr[oc.n_sink].item())
        assert n > 0
        if gc.block_entries:
            assert n <= gc.block_entries
            gc.blocks["v_val"][0][:n] = 0x7C00
            gc.blocks["k_val"][0][:int(gc.k_ptr[oc.n_sink].item())] = 0x7C00
        else:
            gc.v_val[:n] = 0x7C00
            gc.k_val[:int(gc.k_ptr[oc.n_sink].item())] = 0x7C00
        gc.v_sz[:2 * oc.n_sink] = 0x7C00
    q = queries(wl, 6)
    close(call(pre[1], both(per, 1), q), *reference(pre[0], both(per, 0), q, SCALE, wl.rope_base))


@pytest.mark.parametrize("ratio", [1, 8])
def test_smallest_queries_and_one_of_nan(ratio):
    """Queries of zeros, of denormal numbers and of the largest ones with empty places beside them; a NaN stays in its own row."""
    wl = S.workload("c2", n_kv_heads=2, n_q_heads=2 * ratio)
    sq = Seqs(Setup(wl))
    pre, per = sq.make(70), [sq.make(3 + i, seq=1 + i) for i in range(6)]
    q = queries(wl, 6)
    q[0], q[1], q[2] = 0.0, 1e-41, q[2] * 1e-35
    q[4, 1, 77] = np.nan
    clean = np.where(np.isnan(q), np.float32(0.0), q)
    got = call(pre[1], both(per, 1), q).cpu()
    ref, tol = reference(pre[0], both(per, 0), clean, SCALE, wl.rope_base)
    assert got[4, 1].isnan().all()
    got[4, 1], ref[4, 1] = 0.0, 0.0
    close(got, ref, tol)


def test_far_positions_of_own_tokens():
    """Own tokens behind a prefix of 70001: their Keys are rotated by that much more than their index says."""
    import torch
    import paper_2401_18079_amd as K
    wl = S.workload("c4", n_kv_heads=1, n_q_heads=8)
    sq = Seqs(Setup(wl))
    pre = sq.make(70001)
    per = [sq.make(37, seq=3), sq.make(2, seq=4), None]
    q = queries(wl, 3)
    close(call(pre[1], both(per, 1), q), *reference(pre[0], both(per, 0), q, SCALE, wl.rope_base))


def test_streams_workspaces_and_graphs():
    """Garbage in the workspace, a guard behind it, another stream, and two graphs captured and replayed among eager calls."""
    import torch
    import paper_2401_18079_amd as K
    wl = S.workload("c2", n_kv_heads=2, n_q_heads=4)
    sq = Seqs(Setup(wl))
    pre, per = sq.make(500), [sq.make(n, seq=n) for n in (1, 60, 130)]
    own = both(per, 1)
    q = [torch.from_numpy(queries(wl, 3, seed=s)).cuda() for s in range(3)]
    ref = [call(pre[1], own, x).clone() for x in q]
    for i in range(3):
        close(ref[i], *reference(pre[0], both(per, 0), q[i].cpu().numpy(), SCALE, wl.rope_base))
    need = K.kvq_attention_decode_batch_workspace_bytes(pre[1], own, 3)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(call(pre[1], own, q[0], workspace=ws[:need]), ref[0])
    assert torch.all(ws[need:] == 0xFF)
    with pytest.raises(K.KvqError):
        call(pre[1], own, q[0], workspace=ws[:need - 256])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call(pre[1], own, q[1])
    side.synchronize()
    assert torch.equal(got, ref[1])
    got = torch.zeros_like(ref[2])
    torch.cuda.synchronize()
    K.kvq_attention_decode_batch(pre[1], own, q[2], SCALE, got, stream=side)
    side.synchronize()
    assert torch.equal(got, ref[2])
    graphs = []
    for j in range(2):
        x, o = torch.zeros_like(q[0]), torch.zeros_like(ref[0])
        w = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            K.kvq_attention_decode_batch(pre[1], own, x, SCALE, o, workspace=w)
        graphs.append((g, x, o, w))
    for i in (0, 1, 2, 0, 2):
        for j, (g, x, o, w) in enumerate(graphs):
            x.copy_(q[(i + j) % 3])
            g.replay()
        eager = call(pre[1], own, q[i])
        torch.cuda.synchronize()
        assert torch.equal(eager, ref[i])
        for j, (g, x, o, w) in enumerate(graphs):
            assert torch.equal(o, ref[(i + j) % 3])


def test_agrees_with_the_single_sequence_call():
    """A batch of one over one cache: kvq_attention_decode's result to the two tolerances' sum."""
    import torch
    import paper_2401_18079_amd as K
    wl = S.workload("c2", n_kv_heads=8, n_q_heads=8)
    sq = Seqs(Setup(wl))
    oc, gc = sq.make(1500, n_sink=1)
    q = queries(wl, 1)
    scores, out = torch.zeros((8, 1500), device="cuda"), torch.zeros((8, 128), device="cuda")
    K.kvq_attention_decode(gc, torch.from_numpy(q[0]).cuda(), SCALE, scores, out)
    ref, tol = reference(oc, [None], q, SCALE, wl.rope_base)
    got = call(gc, None, q)
    close(got, ref, tol)
    close(got, out[None].cpu().numpy().astype(np.float64), 2 * tol)
