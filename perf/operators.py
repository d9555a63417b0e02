"""Operators for serving several sequences from quantized KV caches, as cases that can be timed and compared.

Two things a server does with the caches that the library's decoder fills: it answers a batch of sequences that share a
long prompt (one decode step's attention for all of them, the prompt's cache read once: "attend"), and it makes the caches of
new sequences out of those of old ones (copying runs of tokens, as forks and beam search do: "copy"; keeping listed
tokens, as compaction after an eviction does: "gather").

A cache here is the library's storage format: packed 2-, 3- or 4-bit codes of Keys (not yet rotated, two channels that rotate
together in one field) and Values (two tokens of a channel in one field), per-channel Key constants, a scale and a
zero-point per Value token, and the outliers' residuals per token in ascending channel order.  `prepare` draws such caches
directly, several of them side by side in one tensor per array; with `own` it also makes the library's handles on them.

Plain form: everything unpacked to 32-bit floats, angles in 64 bits.  `exact`: the same definition in 64 bits, sequence by
sequence and head by head, unpacked bit by bit.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
SCALE = 1.0 / math.sqrt(128.0)
ARRAYS = ("k_codes", "v_codes", "v_sz", "k_ptr", "v_ptr", "k_idx", "k_val", "v_idx", "v_val")


def _attend(name, bits, kv_heads, q_heads, seqs, prefix, own_lo, own_hi, outliers=0.01, rope_base=10000.0, sink=0):
    return {"name": name, "op": "attend", "bits": bits, "kv_heads": kv_heads, "q_heads": q_heads, "seqs": seqs, "prefix": prefix,
            "own_lo": own_lo, "own_hi": own_hi, "outliers": outliers, "rope_base": rope_base, "sink": sink}


def _copy(name, bits, kv_heads, copies, tokens, first, count, at, outliers=0.01):
    return {"name": name, "op": "copy", "bits": bits, "kv_heads": kv_heads, "copies": copies, "tokens": tokens, "first": first,
            "count": count, "at": at, "outliers": outliers}


def _gather(name, bits, kv_heads, tokens, keep, at, outliers=0.01):
    return {"name": name, "op": "gather", "bits": bits, "kv_heads": kv_heads, "tokens": tokens, "keep": keep, "at": at,
            "outliers": outliers}


def listed():
    return [
        # the smallest step: two replies to a short prompt, one head; launches and latency are all there is to it
        _attend("attend_2x1head_300", 3, 1, 1, 2, 300, 0, 3),
        # sixteen conversations behind one system prompt of 33K tokens, grouped queries, the attention-sink token in fp16
        _attend("attend_16x_grouped_33k", 4, 8, 32, 16, 33001, 1, 600, rope_base=500000.0, sink=1),
        # eight samples drawn from one prompt of 128K tokens, the layer of the repository's benchmark
        _attend("attend_8x_128k", 3, 32, 32, 8, 131072, 1, 64),
        # a search that keeps 64 continuations of a document of 16K tokens
        _attend("attend_64x_16k", 3, 32, 32, 64, 16384, 33, 400),
        # 32 readers of one very long context, 2-bit codes, grouped queries: the largest prefix
        _attend("attend_32x_grouped_512k", 2, 8, 32, 32, 524287, 100, 2000, rope_base=500000.0),
        # 48 unrelated sequences of uneven length, some of them empty: a batch without a prefix
        _attend("attend_48x_uneven", 3, 8, 32, 48, 0, 0, 9000, rope_base=500000.0),
        # the smallest copy: the last 65 tokens of a short cache behind 33 others
        _copy("copy_65", 3, 8, 1, 300, 235, 65, 33),
        # a step of beam search: 32 hypotheses of 777 tokens take over their parents' caches
        _copy("copy_32x777", 4, 8, 32, 777, 0, 777, 0),
        # a run of 50001 tokens from the middle of one 40-head cache to an odd place in another
        _copy("copy_50001_40heads", 2, 40, 1, 51000, 129, 50001, 1002),
        # a whole cache of 128K tokens forked: the largest copy
        _copy("copy_128k", 3, 32, 1, 131072, 0, 131072, 0),
        # a cache of 300 tokens compacted to 100
        _gather("gather_100_of_300", 4, 1, 300, 100, 0),
        # a quarter of 128K tokens kept
        _gather("gather_32k_of_128k", 3, 32, 131072, 32768, 0),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    bits = rng.choice([2, 3, 4])
    kv = rng.choice([1, 2, 3, 4, 8, 8, 16, 32, 32, 40])
    p = rng.choice([0.01, 0.01, 0.01, 0.001, 0.0])
    most = min(400000, int(1.8e8 / (kv * 16 * bits)))                # tokens of a cache
    op = rng.choice(["attend"] * 3 + ["copy", "copy", "gather"])
    if op == "attend":
        ratio = rng.choice([r for r in (1, 1, 2, 4, 8) if kv * r <= 64])
        prefix = rng.choice([0, 1, 1, 1]) * spread(100, most)
        seqs = spread(1, max(2, min(64, int(5e8 / (kv * ratio * max(1, prefix))))))
        hi = spread(1, max(2, min(6000, int(2.0e5 / (kv * seqs)))))
        return _attend("", bits, kv, kv * ratio, seqs, prefix, rng.choice([0, 1, hi // 2]), hi, p,
                       rng.choice([10000.0, 500000.0]), rng.choice([0, 0, 0, 1, 4]) if prefix >= 4 else 0) | {"name": ""}
    if op == "copy":
        copies = rng.choice([1, 1, 2, spread(2, 48)])
        tokens = spread(2, max(3, most // copies))
        count = max(1, int(tokens * rng.random()))
        return _copy("", bits, kv, copies, tokens, rng.randrange(tokens - count + 1), count, rng.choice([0, 0, 1, spread(1, 5000)]), p)
    tokens = spread(2, most)
    return _gather("", bits, kv, tokens, max(1, int(tokens * rng.random())), rng.choice([0, 0, 1, spread(1, 5000)]), p)


# ---- caches as a decoder leaves them ------------------------------------------------------------------------

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(((int(seed) * 1000003 + salt) * 2654435761) & 0x7FFFFFFFFFFF)
    return g


def _up(n):
    return max(128, (n + 127) // 128 * 128)


def _layer(case, seed):
    """What the sequences of one layer have in common: signposts and per-channel Key constants, fp16, on the host."""
    r = np.random.RandomState((int(seed) * 7 + 13) & 0x7FFFFFFF)
    n, D = 1 << case["bits"], case["kv_heads"] * 128

    def signposts():
        u = np.linspace(-1.0, 1.0, n) + r.uniform(-0.25, 0.25, n) * (2.0 / (n - 1))
        u = np.sign(u) * np.abs(u) ** 1.25
        u[0], u[-1] = -1.0, 1.0
        return np.sort(u).astype(np.float16).astype(np.float32)

    a = np.clip(np.abs(r.standard_t(4, D)), 0.05, 20.0)                 # a few channels are much larger
    s, z = (2.5 * a).astype(np.float16), (0.5 * a * r.standard_normal(D)).astype(np.float16)
    wide = 65504.0 if case["outliers"] == 0 else 3.0
    lo, hi = (np.clip(z.astype(np.float32) + d * wide * s.astype(np.float32), -65504, 65504).astype(np.float16) for d in (-1, 1))
    return {"lut_k": signposts(), "lut_v": signposts(), "s": s, "z": z, "lo": lo, "hi": hi}


def _pointers(B, cap):
    """Zeros [B, cap + 1], each row 16-byte aligned as the library's caches are."""
    return torch.zeros(B, cap + 4, dtype=torch.int32, device=DEV)[:, :cap + 1]


def _strata(case):
    return max(1, int(math.ceil(case["outliers"] * case["kv_heads"] * 128))) if case["outliers"] > 0 else 0


def _codes(g, case, B, planes, chunks):
    """Packed codes [B, planes * chunks * 16 * bits]: fields of two codes, values near the middle more often than the ends."""
    b = case["bits"]
    n = 1 << b
    out = torch.empty(B, planes, chunks // 64, b, 64, 16, dtype=torch.uint8, device=DEV)
    edges = [int(256 / (1 + math.exp(-1.702 * 2.2 * (2.0 * j / n - 1.0)))) for j in range(1, n)]
    for i in range(B):
        for h0 in range(0, planes, 8):
            h1 = min(planes, h0 + 8)
            u = torch.randint(0, 256, (h1 - h0, chunks, 128), generator=g, device=DEV, dtype=torch.uint8)
            c = torch.zeros_like(u)
            for t in edges:
                c += u >= t
            c = c.view(h1 - h0, chunks, 16, 8).to(torch.int32)              # eight codes are `bits` bytes
            w = sum(c[..., j] << (j * b) for j in range(8))
            by = torch.stack([(w >> (8 * j)) & 255 for j in range(b)], -1).to(torch.uint8)
            out[i, h0:h1] = by.view(h1 - h0, chunks // 64, 64, b, 16).permute(0, 1, 3, 2, 4)
    return out.view(B, -1)


def _outliers(g, case, lens, cap, scales, thin):
    """ptr [B, cap + 1], idx and val [B, entries]: one channel of each of n equal strata of a token, some left out."""
    B, D, n = len(lens), case["kv_heads"] * 128, _strata(case)
    room = max(8, n * cap)
    ptr = _pointers(B, cap)
    idx = torch.zeros(B, room, dtype=torch.int16, device=DEV)
    val = torch.zeros(B, room, dtype=torch.int16, device=DEV)
    for i in range(B if n else 0):
        T = lens[i]
        u = torch.rand(T, n, generator=g, device=DEV)
        ch = ((torch.arange(n, device=DEV) + u) * (D / n)).to(torch.int32).clamp_(max=D - 1)
        ch = torch.cummax(ch, 1)[0]
        keep = torch.rand(T, n, generator=g, device=DEV) < (0.9 if thin else 2.0)
        keep[:, 1:] &= ch[:, 1:] > ch[:, :-1]
        r = (torch.randn(T, n, generator=g, device=DEV) * 2.0).clamp_(-8, 8)
        r = (r * (scales[ch.long()] if scales is not None else 1.0)).half().view(torch.int16)
        ptr[i, 1:T + 1] = keep.sum(1).cumsum(0)
        ptr[i, T + 1:] = ptr[i, T]
        m = int(ptr[i, T])
        idx[i, :m], val[i, :m] = ch[keep].to(torch.int16), r[keep]
    return ptr, idx, val


def _caches(case, seed, salt, lens, cap, layer):
    """Caches of lens[i] tokens each, side by side: one tensor per array, the sequence first."""
    g, B, H = _gen(seed, salt), len(lens), case["kv_heads"]
    s = {"k_codes": _codes(g, case, B, H, cap), "v_codes": _codes(g, case, B, 2 * H, cap // 2)}
    sz = torch.stack([0.8 * torch.exp(0.5 * torch.randn(B, cap, generator=g, device=DEV)),
                      0.1 * torch.randn(B, cap, generator=g, device=DEV)], -1)
    s["v_sz"] = sz.half().view(torch.int16).reshape(B, 2 * cap)
    ks = torch.from_numpy(layer["s"].astype(np.float32)).to(DEV)
    s["k_ptr"], s["k_idx"], s["k_val"] = _outliers(g, case, lens, cap, ks, True)
    s["v_ptr"], s["v_idx"], s["v_val"] = _outliers(g, case, lens, cap, None, False)
    return s


def _empty(case, B, cap):
    b, H, n = case["bits"], case["kv_heads"], _strata(case)
    z = lambda m, t: torch.zeros(B, m, dtype=t, device=DEV)  # noqa: E731
    room = max(8, n * cap)
    return {"k_codes": z(cap * H * 16 * b, torch.uint8), "v_codes": z(cap * H * 16 * b, torch.uint8), "v_sz": z(2 * cap, torch.int16),
            "k_ptr": _pointers(B, cap), "v_ptr": _pointers(B, cap), "k_idx": z(room, torch.int16),
            "k_val": z(room, torch.int16), "v_idx": z(room, torch.int16), "v_val": z(room, torch.int16)}


def _begun(case, seed, salt, B, at, cap, layer):
    """Caches that hold `at` tokens and have room for `cap`."""
    s = _empty(case, B, cap)
    if at:
        t = _caches(case, seed, salt, [at] * B, _up(at), layer)
        for i in range(B):
            _copy_plain(case, {n: s[n][i:i + 1] for n in ARRAYS}, {n: t[n][i:i + 1] for n in ARRAYS}, 0,
                        torch.arange(at, device=DEV)[None])
    return s


def _handles(case, arrays, cap, lens, layer, sink_rows=None):
    """The library's caches on these arrays, as a program keeps them."""
    import paper_2401_18079_amd as K
    got = []
    for i, n in enumerate(lens):
        c = K.KvqCache(case["bits"], case["kv_heads"], case.get("q_heads", case["kv_heads"]), cap, max(1, _strata(case) // 2),
                       case.get("rope_base", 10000.0), 8, 8, max_append=1, device="cuda:0",
                       n_sink=0 if sink_rows is None else sink_rows[0].shape[0])
        K.kvq_lut_load(c, layer["lut_k"], layer["lut_v"], layer["s"], layer["z"], layer["lo"], layer["hi"])
        for name in ARRAYS:
            t = arrays[name][i]
            setattr(c, name, t)
            setattr(c.c, name, t.data_ptr())
        c.c.cap_nnz_k, c.c.cap_nnz_v = arrays["k_idx"].shape[1], arrays["v_idx"].shape[1]
        if sink_rows is not None:
            c.sink_k.copy_(sink_rows[0].view(torch.int16).reshape(-1))
            c.sink_v.copy_(sink_rows[1].view(torch.int16).reshape(-1))
        c.c.n_tokens_k = c.c.n_tokens_v = n
        got.append(c)
    return got


def _lengths(case, seed):
    r = np.random.RandomState((int(seed) * 31 + 5) & 0x7FFFFFFF)
    return [int(x) for x in r.randint(case["own_lo"], case["own_hi"] + 1, case["seqs"])]


def _sink_rows(case, seed):
    g, D = _gen(seed, 9), case["kv_heads"] * 128
    return tuple(torch.randn(case["sink"], D, generator=g, device=DEV).half() for _ in range(2)) if case["sink"] else None


def prepare(case, seed):
    layer = _layer(case, seed)
    dev = {k: torch.from_numpy(v.astype(np.float32)).to(DEV) for k, v in layer.items()}
    s = {"case": case, "layer": dev}
    if case["op"] == "attend":
        lens = _lengths(case, seed)
        cap = _up(max(lens))
        s["lens"], s["lens_dev"] = lens, torch.tensor(lens, device=DEV)
        s["own"] = _caches(case, seed, 1, lens, cap, layer)
        s["prefix"] = _caches(case, seed, 2, [case["prefix"]], _up(case["prefix"]), layer) if case["prefix"] else None
        s["sink"] = _sink_rows(case, seed)
        s["q"] = torch.randn(case["seqs"], case["q_heads"], 128, generator=_gen(seed, 3), device=DEV)
        s["out"] = torch.zeros(case["seqs"], case["q_heads"], 128, device=DEV)
        if own:
            s["caches"] = _handles(case, s["own"], cap, lens, layer)
            s["prefix_cache"] = (_handles(case, s["prefix"], _up(case["prefix"]), [case["prefix"]], layer, s["sink"])[0]
                                 if case["prefix"] else None)
        return s
    B = case.get("copies", 1)
    new = case.get("count", case.get("keep"))
    s["src"] = _caches(case, seed, 1, [case["tokens"]] * B, _up(case["tokens"]), layer)
    cap = _up(case["at"] + new)
    s["dst"] = _begun(case, seed, 2, B, case["at"], cap, layer)
    r = np.random.RandomState((int(seed) * 17 + 3) & 0x7FFFFFFF)
    s["parents"] = [int(x) for x in r.randint(0, B, B)]
    s["parents_dev"] = torch.tensor(s["parents"], device=DEV)
    if case["op"] == "gather":
        kept = np.sort(r.permutation(case["tokens"])[:new]).astype(np.int32)
        s["kept"] = torch.from_numpy(kept).to(DEV)
    if own:
        s["src_caches"] = _handles(case, s["src"], _up(case["tokens"]), [case["tokens"]] * B, layer)
        s["dst_caches"] = _handles(case, s["dst"], cap, [case["at"]] * B, layer)
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------

def _fields(case, codes, planes, chunks):
    """[B, planes, chunks, 64] fields of two codes each."""
    b = case["bits"]
    by = codes.view(-1, planes, chunks // 64, b, 64, 16).permute(0, 1, 2, 4, 3, 5).reshape(-1, planes, chunks, 16 * b)
    bit = torch.arange(64, device=DEV) * 2 * b
    lo, hi = bit // 8, (bit // 8 + 1).clamp(max=16 * b - 1)
    w = by[..., lo].to(torch.int16) | (by[..., hi].to(torch.int16) << 8)
    return (w >> (bit % 8).to(torch.int16)) & ((1 << 2 * b) - 1)


def _packed(case, f, planes, chunks):
    """The inverse: fields [B, planes, chunks, 64] as stored bytes."""
    b = case["bits"]
    c = f.view(-1, planes, chunks, 16, 4).to(torch.int32)                  # four fields are `bits` bytes
    w = c[..., 0] | (c[..., 1] << 2 * b) | (c[..., 2] << 4 * b) | (c[..., 3] << 6 * b)
    by = torch.stack([(w >> (8 * j)) & 255 for j in range(b)], -1).to(torch.uint8)
    return by.view(-1, planes, chunks // 64, 64, b, 16).permute(0, 1, 2, 4, 3, 5).reshape(f.shape[0], -1)


def _residuals(case, x, ptr, idx, val):
    """Adds the outliers' residuals to x [B, cap, D]."""
    B, cap, D = x.shape
    e = torch.arange(idx.shape[1], device=DEV, dtype=torch.int32)[None].expand(B, -1).contiguous()
    t = torch.searchsorted(ptr.contiguous(), e, right=True) - 1
    there = e < ptr[:, -1:]
    at = torch.where(there, (t.clamp(0, cap - 1) * D + (idx.to(torch.int64) & 0xFFFF)), e.to(torch.int64) % (cap * D))
    at = at + torch.arange(B, device=DEV)[:, None] * (cap * D)
    return x.view(-1).index_add_(0, at.view(-1), torch.where(there, val.view(torch.float16).float(), 0.0).view(-1)).view(x.shape)


def _keys(case, s, layer, cap, start, sink):
    """Rotated Keys [B, H, cap, 128], token t at position start + t."""
    b, H = case["bits"], case["kv_heads"]
    f = _fields(case, s["k_codes"], H, cap)
    k = torch.cat([layer["lut_k"][(f & ((1 << b) - 1)).to(torch.int32)], layer["lut_k"][(f >> b).to(torch.int32)]], -1)
    k = k.permute(0, 2, 1, 3).reshape(-1, cap, H * 128) * layer["s"] + layer["z"]
    k = _residuals(case, k, s["k_ptr"], s["k_idx"], s["k_val"])
    if sink is not None:
        k[:, :sink[0].shape[0]] = sink[0].float()
    k = k.view(-1, cap, H, 128).transpose(1, 2).contiguous()
    theta = case["rope_base"] ** (-torch.arange(64, device=DEV, dtype=torch.float64) / 64.0)
    ang = (start + torch.arange(cap, device=DEV, dtype=torch.float64))[:, None] * theta
    c, sn = torch.cos(ang).float(), torch.sin(ang).float()
    return torch.cat([k[..., :64] * c - k[..., 64:] * sn, k[..., 64:] * c + k[..., :64] * sn], -1)


def _values(case, s, layer, cap, sink):
    """Values [B, H, cap, 128]."""
    b, H = case["bits"], case["kv_heads"]
    f = _fields(case, s["v_codes"], 2 * H, cap // 2)
    v = torch.stack([layer["lut_v"][(f & ((1 << b) - 1)).to(torch.int32)], layer["lut_v"][(f >> b).to(torch.int32)]], 3)
    v = v.view(-1, H, 2, cap, 64).permute(0, 3, 1, 2, 4).reshape(-1, cap, H * 128)
    sz = s["v_sz"].view(torch.float16).float().view(-1, cap, 1, 2)
    v = v * sz[..., 0] + sz[..., 1]
    v = _residuals(case, v, s["v_ptr"], s["v_idx"], s["v_val"])
    if sink is not None:
        v[:, :sink[1].shape[0]] = sink[1].float()
    return v.view(-1, cap, H, 128).transpose(1, 2).contiguous()


def _long_product(y, v, n=8192):
    """y @ v, [H, M, T] by [H, T, 128], summed n tokens at a time: one 32-bit sum over half a million is 2e-5 off."""
    H, M, T = y.shape
    if T <= n:
        return y @ v
    k = (T + n - 1) // n
    y = torch.nn.functional.pad(y, (0, k * n - T)).view(H, M, k, n).transpose(1, 2).contiguous()
    return (y @ torch.nn.functional.pad(v, (0, 0, 0, k * n - T)).view(H, k, n, 128)).sum(1)


def _attend_plain(s):
    case, layer = s["case"], s["layer"]
    B, H, R, P = case["seqs"], case["kv_heads"], case["q_heads"] // case["kv_heads"], case["prefix"]
    cap = s["own"]["k_ptr"].shape[1] - 1
    q = s["q"].view(B, H, R, 128) * SCALE
    x = q @ _keys(case, s["own"], layer, cap, P, None).transpose(2, 3).contiguous()              # [B, H, R, cap]
    there = torch.arange(cap, device=DEV)[None, :] < s["lens_dev"][:, None]
    x = torch.where(there[:, None, None, :], x, -math.inf)
    m = x.max(-1, keepdim=True)[0]
    if P:
        k = _keys(case, s["prefix"], layer, _up(P), 0, s["sink"])[0, :, :P]
        y = (q.permute(1, 0, 2, 3).reshape(H, B * R, 128) @ k.transpose(1, 2).contiguous())        # [H, B * R, P]
        my = y.max(-1, keepdim=True)[0]
        m = torch.maximum(m, my.view(H, B, R, 1).permute(1, 0, 2, 3))
        y = torch.exp(y - m.permute(1, 0, 2, 3).reshape(H, B * R, 1))
        o2 = _long_product(y, _values(case, s["prefix"], layer, _up(P), s["sink"])[0, :, :P]).view(H, B, R, 128).permute(1, 0, 2, 3)
        l2 = y.sum(-1).view(H, B, R, 1).permute(1, 0, 2, 3)
    m = torch.where(m == -math.inf, 0.0, m)
    x = torch.exp(x - m)
    o, l = x @ _values(case, s["own"], layer, cap, None), x.sum(-1, keepdim=True)
    if P:
        o, l = o + o2, l + l2
    return torch.where(l > 0, o / torch.where(l > 0, l, 1.0), 0.0).reshape(B, H * R, 128)


def _copy_plain(case, dst, src, at, tokens):
    """Token tokens[i, j] of src's cache i becomes token at + j of dst's cache i."""
    b, H = case["bits"], case["kv_heads"]
    B, n = tokens.shape
    scap, dcap = src["k_ptr"].shape[1] - 1, dst["k_ptr"].shape[1] - 1
    i = torch.arange(B, device=DEV)[:, None]
    to = at + torch.arange(n, device=DEV)[None].expand(B, n)
    k = src["k_codes"].view(B, H, scap // 64, b, 64, 16)
    dst["k_codes"].view(B, H, dcap // 64, b, 64, 16)[i, :, to // 64, :, to % 64] = k[i, :, tokens // 64, :, tokens % 64]
    f = _fields(case, src["v_codes"], 2 * H, scap // 2)[i, :, tokens // 2]                                 # [B, n, 2 H, 64]
    f = (f >> ((tokens % 2) * b)[..., None, None].to(torch.int16)) & ((1 << b) - 1)
    old = _fields(case, dst["v_codes"], 2 * H, dcap // 2)
    both = torch.stack([old & ((1 << b) - 1), old >> b], 3).view(B, 2 * H, dcap, 64)
    both[i, :, to] = f
    both = both.view(B, 2 * H, dcap // 2, 2, 64)
    dst["v_codes"].copy_(_packed(case, both[:, :, :, 0] | (both[:, :, :, 1] << b), 2 * H, dcap // 2))
    dst["v_sz"].view(B, dcap, 2)[i, to] = src["v_sz"].view(B, scap, 2)[i, tokens]
    for x in ("k", "v"):
        sp, dp = src[x + "_ptr"], dst[x + "_ptr"]
        cnt = torch.gather(sp, 1, tokens + 1) - torch.gather(sp, 1, tokens)
        new = (dp[:, at:at + 1] + cnt.cumsum(1)).to(torch.int32)
        dp[:, at + 1:at + n + 1] = new
        room = dst[x + "_idx"].shape[1]
        e = torch.arange(room, device=DEV, dtype=torch.int32)[None].expand(B, room).contiguous()
        j = (torch.searchsorted(new, e, right=True)).clamp(max=n - 1)
        there = (e >= dp[:, at:at + 1]) & (e < new[:, -1:])
        begin = torch.gather(new - cnt, 1, j)
        fr = (torch.gather(sp, 1, torch.gather(tokens, 1, j)) + e - begin).clamp(0, src[x + "_idx"].shape[1] - 1).long()
        for a in (x + "_idx", x + "_val"):
            dst[a].copy_(torch.where(there, torch.gather(src[a], 1, fr), dst[a]))


def run(s):
    case = s["case"]
    if own:
        import paper_2401_18079_amd as K
        if case["op"] == "attend":
            K.kvq_attention_decode_batch(s["prefix_cache"], s["caches"], s["q"], SCALE, s["out"])
            return s["out"]
        for c in s["dst_caches"]:
            K.kvq_cache_truncate(c, case["at"])
        if case["op"] == "copy":
            K.kvq_cache_copy(s["dst_caches"], [s["src_caches"][p] for p in s["parents"]], case["first"], case["count"])
        else:
            K.kvq_cache_gather(s["dst_caches"][0], s["src_caches"][0], s["kept"])
        return s["dst"]
    if case["op"] == "attend":
        return _attend_plain(s)
    if case["op"] == "copy":
        src = {a: s["src"][a][s["parents_dev"]] for a in ARRAYS}
        tokens = (case["first"] + torch.arange(case["count"], device=DEV))[None].expand(case["copies"], -1).contiguous()
    else:
        src, tokens = s["src"], s["kept"].long()[None]
    _copy_plain(case, s["dst"], src, case["at"], tokens)
    return s["dst"]


# ---- what a pass cannot do without, and how exact it is ------------------------------------------------------

def work(case):
    b, D, n = case["bits"], case["kv_heads"] * 128, _strata(case)
    token = D * b / 8 * 2 + 4 + 2 * 4 + 4 * (0.9 * n + n)                 # codes, Value scale, pointers, outliers
    if case["op"] == "attend":
        own_tokens = case["seqs"] * (case["own_lo"] + case["own_hi"]) / 2
        q = case["seqs"] * case["q_heads"]
        pairs = q * case["prefix"] + case["q_heads"] * own_tokens            # (query head, token)
        return {"bytes": token * (case["prefix"] + own_tokens) + 2 * q * 512 + 28 * D, "flops": pairs * 4 * 128}
    if case["op"] == "copy":
        # a parent that several hypotheses share has to be read once only
        sources = case["copies"] * (1 - (1 - 1 / case["copies"]) ** case["copies"])
        return {"bytes": token * case["count"] * (case["copies"] + sources), "flops": 0}
    return {"bytes": (2 * token + 4) * case["keep"], "flops": 0}


def exact(case, seed):
    if case["op"] != "attend":
        return None                                      # stored bits: whole numbers, the same or wrong
    st = prepare_plain(case, seed)
    b, H, R = case["bits"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    layer = {k: v.double() for k, v in st["layer"].items()}
    power = (2 ** torch.arange(b, device=DEV)).to(torch.uint8)
    theta = torch.tensor([case["rope_base"] ** (-2.0 * i / 128.0) for i in range(64)], dtype=torch.float64, device=DEV)

    def unpacked(codes, plane, chunks):
        """Codes [chunks, 64, 2] of one plane, bit by bit."""
        size = chunks * 16 * b
        x = codes[plane * size:(plane + 1) * size].view(chunks // 64, b, 64, 16).transpose(1, 2).reshape(chunks, 16 * b)
        bits = (x[..., None] >> torch.arange(8, device=DEV, dtype=torch.uint8)) & 1
        return (bits.view(chunks, 64, 2, b) * power).sum(-1)

    def residual(s, i, side, n, cap):
        """Dense [n, D] residuals of cache i."""
        ptr, D = s[side + "_ptr"][i].long(), H * 128
        m = int(ptr[n])
        t = torch.repeat_interleave(torch.arange(n, device=DEV), ptr[1:n + 1] - ptr[:n])
        r = torch.zeros(n, D, dtype=torch.float64, device=DEV)
        r[t, s[side + "_idx"][i, :m].long() & 0xFFFF] = s[side + "_val"][i, :m].view(torch.float16).double()
        return r

    def part(s, i, n, start, sink, q):
        """(scores, Values) per head of the n tokens of cache i against q [H, queries, 128]."""
        cap = s["k_ptr"].shape[1] - 1
        rk, rv = residual(s, i, "k", n, cap), residual(s, i, "v", n, cap)
        ang = torch.outer(torch.arange(start, start + n, dtype=torch.float64, device=DEV), theta)
        turn = torch.polar(torch.ones_like(ang), ang)
        sz = s["v_sz"][i].view(torch.float16).double().view(cap, 2)[:n]
        for h in range(H):
            ch = slice(h * 128, h * 128 + 128)
            k = layer["lut_k"][unpacked(s["k_codes"][i], h, cap)[:n].transpose(1, 2).reshape(n, 128)]
            k = k * layer["s"][ch] + layer["z"][ch] + rk[:, ch]
            v = torch.cat([layer["lut_v"][unpacked(s["v_codes"][i], 2 * h + g, cap // 2).transpose(1, 2).reshape(cap, 64)[:n]]
                           for g in (0, 1)], 1)
            v = v * sz[:, :1] + sz[:, 1:] + rv[:, ch]
            if sink is not None:
                k[:sink[0].shape[0]], v[:sink[0].shape[0]] = sink[0][:, ch].double(), sink[1][:, ch].double()
            k = torch.complex(k[:, :64], k[:, 64:]) * turn
            yield q[h] @ torch.cat([k.real, k.imag], 1).T, v

    B = case["seqs"]
    q = (st["q"].double() * SCALE).view(B, H, R, 128)
    out = torch.zeros(B, H, R, 128, dtype=torch.float64, device=DEV)
    top = torch.full((B, H, R, 1), -math.inf, dtype=torch.float64, device=DEV)
    den = torch.zeros_like(top)

    def join(i, h, x, v):
        m = torch.maximum(top[i, h], x.amax(-1, keepdim=True))
        old = torch.exp(top[i, h] - m)
        e = torch.exp(x - m)
        out[i, h], den[i, h], top[i, h] = out[i, h] * old + e @ v, den[i, h] * old + e.sum(-1, keepdim=True), m

    for i in range(B):
        if st["lens"][i]:
            for h, (x, v) in enumerate(part(st["own"], i, st["lens"][i], case["prefix"], None, q[i])):
                join(i, h, x, v)
    if case["prefix"]:
        every = q.transpose(0, 1).reshape(H, B * R, 128)
        for h, (x, v) in enumerate(part(st["prefix"], 0, case["prefix"], 0, st["sink"], every)):
            for i in range(B):
                join(i, h, x[i * R:(i + 1) * R], v)
    return torch.where(den > 0, out / torch.where(den > 0, den, 1.0), 0.0).view(B, H * R, 128)


def prepare_plain(case, seed):
    """The inputs alone, without handles."""
    global own
    kept, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = kept
