// Tokens from cache to cache: runs of them (forks, beam search), listed ones (compaction after an eviction).  Keys are
// stored before the rotation (paper Sec. 3.2) and positions are indices, so a token may land at any place with its bits as
// they are; only the packing of the Values, two tokens to a field, and the outlier lists depend on the place.
//
// Everything here is moved once, in 16-byte pieces where the format has them; the bound is HBM, read and written.
//   Keys    a lane takes a token's chunk of a head: `bits` pieces, each 1 KiB contiguous over a wavefront at both ends.
//   Values  a lane takes the pair of tokens that share a destination chunk: one chunk if they shared the source's, else two,
//           their halves of every field put together with a shift of the whole chunk by one code.
//   outliers, scales and pointers: 256 tokens a workgroup, a run's entries as one contiguous piece.
// A run's pointers are the source's plus a constant, so a copy is one launch; a list's need the sum of the counts before
// them, which the first of two launches, a short one, leaves per 256 tokens.  (32768 of 131072 tokens of 32 heads: 145 us with the
// codes in the first launch and the lists alone in the second, 133 so.)
#include <string.h>
#include "kvq_append_keys.hpp"
#include "kvq_common.hpp"

namespace {

constexpr int MV_NT = 256;              // threads of a workgroup
constexpr int MV_GROUP = 256;           // tokens of a workgroup of the outlier role
constexpr int MV_JOBS = 16;             // copies whose descriptors travel in one launch's arguments: as many as 4 KiB hold

struct MvSide {
    const uint32_t *s_ptr;
    uint32_t *d_ptr;
    const void *s_idx, *s_val;          // flat arrays, or tables of blocks (shift != 0)
    void *d_idx, *d_val;
};

struct MvJob {
    const uint8_t *s_kc, *s_vc;
    uint8_t *d_kc, *d_vc;
    const uint32_t *s_sz;
    uint32_t *d_sz;
    MvSide k, v;
    uint32_t k_room, v_room;            // the destination's capacity in entries
    int32_t *status;
    const uint16_t *s_sink_k, *s_sink_v;
    uint16_t *d_sink_k, *d_sink_v;
    const uint32_t *s_params;           // null: the destination has its constants
    uint32_t *d_params;
    int32_t s_n, s_cap, d_cap;
    int32_t first, at, n;               // source token of the first one, its place, how many
    int16_t s_shift, d_shift, s_sink, d_sink;       // of outlier blocks; attention-sink tokens kept in fp16
};

struct MvArgs {
    int32_t heads, n_jobs, param_words;
    int32_t wg0[MV_JOBS + 1];           // first workgroup of each
    MvJob job[MV_JOBS];
};
static_assert(sizeof(MvArgs) + 16 <= 4096 && KVQ_MAX_SINK < 32768, "kernel arguments");

__host__ __device__ inline int mv_groups(int n) { return (n + MV_GROUP - 1) / MV_GROUP; }
__host__ __device__ inline int mv_key_items(int at, int n) { return ((at + n + 63) >> 6) - (at >> 6); }
__host__ __device__ inline int mv_value_items(int at, int n) { return ((at + n + 127) >> 7) - (at >> 7); }

// Source token of the i-th one; -1 where a list has none of the source's.
template <bool LIST>
__device__ __forceinline__ int mv_source(const MvJob &j, const int32_t *tokens, int i)
{
    if (!LIST) return j.first + i;
    const int t = tokens[i];
    return t >= 0 && t < j.s_n ? t : -1;
}

// Bits of dword w of a chunk that belong to the first of a field's two codes.
template <int BITS>
__device__ constexpr uint32_t mv_low_mask(int w)
{
    uint32_t m = 0;
    for (int i = 0; i < 32; ++i)
        if ((32 * w + i) % (2 * BITS) < BITS) m |= 1u << i;
    return m;
}

template <int BITS>
__device__ __forceinline__ void mv_load(uint32_t (&c)[4 * BITS], const uint8_t *p)
{
#pragma unroll
    for (int i = 0; i < BITS; ++i) {
        const uint4 v = kvq_load_stream16(p + i * 1024);
        c[4 * i + 0] = v.x; c[4 * i + 1] = v.y; c[4 * i + 2] = v.z; c[4 * i + 3] = v.w;
    }
}

template <int BITS, bool LIST>
__device__ void mv_keys(const MvJob &j, const int32_t *tokens, int item, int lane)
{
    const int per = mv_key_items(j.at, j.n), h = item / per, d = ((j.at >> 6) + item % per) * 64 + lane, i = d - j.at;
    if (i < 0 || i >= j.n) return;
    const int t = mv_source<LIST>(j, tokens, i);
    const uint8_t *s = j.s_kc + kvq_k_piece0(BITS, j.s_cap, t < 0 ? 0 : t, h);
    uint8_t *o = j.d_kc + kvq_k_piece0(BITS, j.d_cap, d, h);
#pragma unroll
    for (int p = 0; p < BITS; ++p) {
        uint4 v = kvq_load_stream16(s + p * 1024);
        if (LIST && t < 0) v = uint4{0u, 0u, 0u, 0u};
        *(uint4 *)(o + p * 1024) = v;
    }
}

template <int BITS, bool LIST>
__device__ void mv_values(const MvJob &j, const int32_t *tokens, int item, int lane)
{
    constexpr int CW = 4 * BITS;
    const int per = mv_value_items(j.at, j.n), plane = item / per, m = ((j.at >> 7) + item % per) * 64 + lane;
    const int h = plane >> 1, g = plane & 1, i0 = 2 * m - j.at, i1 = i0 + 1;
    const bool in0 = i0 >= 0 && i0 < j.n, in1 = i1 >= 0 && i1 < j.n;
    if (!in0 && !in1) return;
    const int t0 = in0 ? mv_source<LIST>(j, tokens, i0) : -1, t1 = in1 ? mv_source<LIST>(j, tokens, i1) : -1;
    uint8_t *o = j.d_vc + kvq_v_piece0(BITS, j.d_cap, m, h, g);
    uint32_t c[CW];
    if (t0 >= 0 && t1 == t0 + 1 && !(t0 & 1)) {
        mv_load<BITS>(c, j.s_vc + kvq_v_piece0(BITS, j.s_cap, t0 >> 1, h, g));
    } else {
        uint32_t a[CW], b[CW];
        if (!in0 || !in1) mv_load<BITS>(c, o);           // the other token of the pair stays
#pragma unroll
        for (int w = 0; w < CW; ++w) a[w] = b[w] = 0u;
        if (t0 >= 0) mv_load<BITS>(a, j.s_vc + kvq_v_piece0(BITS, j.s_cap, t0 >> 1, h, g));
        if (t1 >= 0) mv_load<BITS>(b, j.s_vc + kvq_v_piece0(BITS, j.s_cap, t1 >> 1, h, g));
#pragma unroll
        for (int w = 0; w < CW; ++w) {
            // the first token's codes down from the upper half of their fields, the second's up from the lower
            const uint32_t low = mv_low_mask<BITS>(w);
            const uint32_t down = __builtin_amdgcn_alignbit(w + 1 < CW ? a[w + 1 < CW ? w + 1 : w] : 0u, a[w], BITS);
            const uint32_t up = __builtin_amdgcn_alignbit(b[w], w > 0 ? b[w > 0 ? w - 1 : 0] : 0u, 32 - BITS);
            const uint32_t x = in0 ? ((t0 & 1) ? down : a[w]) : c[w], y = in1 ? ((t1 & 1) ? b[w] : up) : c[w];
            c[w] = (x & low) | (y & ~low);
        }
    }
#pragma unroll
    for (int p = 0; p < BITS; ++p) *(uint4 *)(o + p * 1024) = uint4{c[4 * p], c[4 * p + 1], c[4 * p + 2], c[4 * p + 3]};
}

// (A block's address comes out of memory: the cast says that it points to global memory.)
__device__ __forceinline__ uint16_t *mv_block(const void *arr, uint32_t b)
{
    return (uint16_t *)(__attribute__((address_space(1))) uint16_t *)(uintptr_t)((uint16_t *const *)arr)[b];
}
__device__ __forceinline__ uint16_t mv_get(const void *arr, int shift, uint32_t e)
{
    return shift == 0 ? ((const uint16_t *)arr)[e] : mv_block(arr, e >> shift)[e & ((1u << shift) - 1u)];
}
__device__ __forceinline__ void mv_put(void *arr, int shift, uint32_t e, uint16_t x)
{
    if (shift == 0) ((uint16_t *)arr)[e] = x;
    else mv_block(arr, e >> shift)[e & ((1u << shift) - 1u)] = x;
}

// n consecutive 16-bit entries from place s to place d, by the whole workgroup: where both ends are flat arrays in pieces of 16
// bytes at the destination's alignment (a source may lie at any even address), four of a thread's under way at a time.
struct __attribute__((packed, aligned(2))) MvPiece {
    uint32_t w[4];
};
__device__ void mv_entries(const void *src, void *dst, int s_shift, int d_shift, uint32_t s, uint32_t d, uint32_t n)
{
    const uint32_t tid = threadIdx.x;
    if (s_shift | d_shift) {
        for (uint32_t i = tid; i < n; i += MV_NT) mv_put(dst, d_shift, d + i, mv_get(src, s_shift, s + i));
        return;
    }
    const uint16_t *from = (const uint16_t *)src + s;
    uint16_t *to = (uint16_t *)dst + d;
    const uint32_t off = (uint32_t)((8 - (((uintptr_t)to >> 1) & 7)) & 7), head = off < n ? off : n, pieces = (n - head) / 8;
    if (tid < head) to[tid] = from[tid];
    from += head;
    to += head;
    for (uint32_t i = tid; i < pieces; i += 4 * MV_NT) {
        MvPiece v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k * MV_NT < pieces) v[k] = *(const MvPiece *)(from + 8 * (size_t)(i + k * MV_NT));
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k * MV_NT < pieces) *(uint4 *)(to + 8 * (size_t)(i + k * MV_NT)) = uint4{v[k].w[0], v[k].w[1], v[k].w[2], v[k].w[3]};
    }
    const uint32_t done = pieces * 8;
    if (tid < n - head - done) to[done + tid] = from[done + tid];
}

// A run's outliers of up to MV_GROUP tokens: pointers are the source's moved by a constant, entries a contiguous piece.
__device__ void mv_run_side(const MvSide &a, uint32_t room, int s_shift, int d_shift, int s0, int d0, int at, int first, int n, int32_t *status)
{
    const uint32_t base = a.d_ptr[at], from = a.s_ptr[first];
    const int tid = threadIdx.x;
    bool over = false;
    auto place = [&](uint32_t s) {                          // where the destination's entries end for a source pointer
        const uint64_t e = (uint64_t)base + (s - from);
        return e < room ? (uint32_t)e : room;
    };
    const uint32_t p0 = a.s_ptr[s0], e0 = place(p0), e1 = place(a.s_ptr[s0 + n]);
    if (tid < n) {
        const uint32_t s = a.s_ptr[s0 + tid + 1];
        over = (uint64_t)base + (s - from) > room;
        a.d_ptr[d0 + tid + 1] = place(s);
    }
    mv_entries(a.s_idx, a.d_idx, s_shift, d_shift, p0, e0, e1 - e0);
    mv_entries(a.s_val, a.d_val, s_shift, d_shift, p0, e0, e1 - e0);
    if (over) atomicExch(status, (int32_t)KVQ_ERR_NNZ_OVERFLOW);
}

// What a workgroup of either launch does for tokens `i0` on besides outliers: scales, and (the first one) sink rows.
template <bool LIST>
__device__ void mv_scales(const MvJob &j, const int32_t *tokens, int heads, int i0, int n)
{
    const int tid = threadIdx.x;
    if (tid < n) {
        const int t = mv_source<LIST>(j, tokens, i0 + tid);
        j.d_sz[j.at + i0 + tid] = t < 0 ? 0u : j.s_sz[t];
        if (LIST && t < 0) atomicExch(j.status, (int32_t)KVQ_ERR_INVALID_ARG);
    }
    if (i0 != 0) return;
    for (int i = 0; i < j.n && j.at + i < j.d_sink; ++i) {
        const int t = mv_source<LIST>(j, tokens, i), D = heads * KVQ_HEAD_DIM;
        const bool have = t >= 0 && t < j.s_sink;             // a list may name a token whose fp16 row is not kept
        if (LIST && !have && tid == 0) atomicExch(j.status, (int32_t)KVQ_ERR_INVALID_ARG);
        for (int c = tid; c < D; c += MV_NT) {
            j.d_sink_k[(int64_t)(j.at + i) * D + c] = have ? j.s_sink_k[(int64_t)t * D + c] : 0;
            j.d_sink_v[(int64_t)(j.at + i) * D + c] = have ? j.s_sink_v[(int64_t)t * D + c] : 0;
        }
    }
}

// First kernel of a gather: the counts of every MV_GROUP listed tokens.
__global__ __launch_bounds__(MV_NT) void kvq_move_counts(MvJob j, const int32_t *__restrict__ tokens, uint32_t *__restrict__ sums)
{
    __shared__ uint32_t part[MV_NT / 64][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = blockIdx.x * MV_GROUP + tid;
    const int t = i < j.n ? mv_source<true>(j, tokens, i) : -1;
    uint32_t k = t < 0 ? 0u : j.k.s_ptr[t + 1] - j.k.s_ptr[t], v = t < 0 ? 0u : j.v.s_ptr[t + 1] - j.v.s_ptr[t];
    for (int d = 32; d; d >>= 1) {
        k += (uint32_t)__shfl_xor((int)k, d);
        v += (uint32_t)__shfl_xor((int)v, d);
    }
    if (lane == 0) {
        part[wave][0] = k;
        part[wave][1] = v;
    }
    __syncthreads();
    if (tid < 2) sums[2 * blockIdx.x + tid] = part[0][tid] + part[1][tid] + part[2][tid] + part[3][tid];
}

// Pointers and entries of MV_PART listed tokens on one side, behind the sums of the groups before theirs.  A workgroup counts its whole
// group; a wavefront copies a token's entries at once, MV_HELD tokens of them under way.
constexpr int MV_PART = 64, MV_HELD = 4, MV_LIST_WGS = 2 * MV_GROUP / MV_PART;          // workgroups of a group
struct MvListShared {
    uint32_t wave_sum[2][MV_NT / 64], begin[MV_GROUP + 1], from[MV_GROUP];
};
__device__ void mv_list_part(const MvJob &j, const int32_t *__restrict__ tokens, const uint32_t *__restrict__ sums, int wg, int side, int quarter,
                             MvListShared &sh)
{
    auto &wave_sum = sh.wave_sum;
    auto &begin = sh.begin;
    auto &from = sh.from;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const MvSide &s = side == 0 ? j.k : j.v;
    const uint32_t room = side == 0 ? j.k_room : j.v_room;
    const int i0 = wg * MV_GROUP, n = j.n - i0 < MV_GROUP ? j.n - i0 : MV_GROUP;
    if (quarter * MV_PART >= n) return;
    const int t = tid < n ? mv_source<true>(j, tokens, i0 + tid) : -1;
    const uint32_t p = t < 0 ? 0u : s.s_ptr[t], c = t < 0 ? 0u : s.s_ptr[t + 1] - p;
    uint32_t before = 0;
    for (int i = tid; i < wg; i += MV_NT) before += sums[2 * i + side];
    for (int d = 32; d; d >>= 1) before += (uint32_t)__shfl_xor((int)before, d);
    uint32_t sum = c;
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == 63) {
        wave_sum[0][wave] = before;
        wave_sum[1][wave] = sum;
    }
    __syncthreads();
    const uint64_t base = (uint64_t)s.d_ptr[j.at] + wave_sum[0][0] + wave_sum[0][1] + wave_sum[0][2] + wave_sum[0][3];
    for (int w = 0; w < wave; ++w) sum += wave_sum[1][w];
    const uint64_t end = base + sum;
    const uint32_t clipped = end < room ? (uint32_t)end : room;
    begin[tid] = end - c < room ? (uint32_t)(end - c) : room;
    from[tid] = p;
    if (tid == MV_GROUP - 1) begin[MV_GROUP] = clipped;
    if (tid < n && wave == quarter) {
        s.d_ptr[j.at + i0 + tid + 1] = clipped;
        if (end > room) atomicExch(j.status, (int32_t)KVQ_ERR_NNZ_OVERFLOW);
    }
    __syncthreads();
    const int last = (quarter + 1) * MV_PART < n ? (quarter + 1) * MV_PART : n;
    for (int r = quarter * MV_PART + wave * MV_HELD; r < last; r += MV_NT / 64 * MV_HELD) {
        uint16_t x[MV_HELD], y[MV_HELD];
#pragma unroll
        for (int k = 0; k < MV_HELD; ++k)
            if (r + k < last && begin[r + k] + lane < begin[r + k + 1]) {
                x[k] = mv_get(s.s_idx, j.s_shift, from[r + k] + lane);
                y[k] = mv_get(s.s_val, j.s_shift, from[r + k] + lane);
            }
#pragma unroll
        for (int k = 0; k < MV_HELD; ++k)
            if (r + k < last && begin[r + k] + lane < begin[r + k + 1]) {
                mv_put(s.d_idx, j.d_shift, begin[r + k] + lane, x[k]);
                mv_put(s.d_val, j.d_shift, begin[r + k] + lane, y[k]);
            }
        for (int k = 0; k < MV_HELD && r + k < last; ++k)          // tokens of more outliers than lanes
            for (uint32_t e = lane + 64; begin[r + k] + e < begin[r + k + 1]; e += 64) {
                mv_put(s.d_idx, j.d_shift, begin[r + k] + e, mv_get(s.s_idx, j.s_shift, from[r + k] + e));
                mv_put(s.d_val, j.d_shift, begin[r + k] + e, mv_get(s.s_val, j.s_shift, from[r + k] + e));
            }
    }
}

// The kernel of a copy, and the second of a gather (LIST).
template <int BITS, bool LIST>
__global__ __launch_bounds__(MV_NT) void kvq_move(MvArgs a, const int32_t *__restrict__ tokens, const uint32_t *__restrict__ sums)
{
    int wg = blockIdx.x, i = 0;
    if (!LIST) {                                            // (a gather is one job: a fixed place in the arguments)
        while (i + 1 < a.n_jobs && wg >= a.wg0[i + 1]) ++i;
        wg -= a.wg0[i];
    }
    const MvJob &j = a.job[LIST ? 0 : i];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = LIST ? MV_LIST_WGS : 2, groups = mv_groups(j.n) * per;
    if (wg < groups) {
        const int i0 = wg / per * MV_GROUP, n = j.n - i0 < MV_GROUP ? j.n - i0 : MV_GROUP;
        if (wg % per == 1) mv_scales<LIST>(j, tokens, a.heads, i0, n);
        if constexpr (LIST) {
            __shared__ MvListShared sh;
            mv_list_part(j, tokens, sums, wg / per, wg & 1, (wg % per) >> 1, sh);
        } else {
            mv_run_side((wg & 1) ? j.v : j.k, (wg & 1) ? j.v_room : j.k_room, j.s_shift, j.d_shift, j.first + i0, j.at + i0, j.at, j.first, n, j.status);
        }
        return;
    }
    wg -= groups;
    if (j.s_params) {
        const int wgs = (a.param_words + 16 * MV_NT - 1) / (16 * MV_NT);
        if (wg < wgs) {
            for (int w = wg * 16 * MV_NT + tid; w < a.param_words && w < (wg + 1) * 16 * MV_NT; w += MV_NT) j.d_params[w] = j.s_params[w];
            return;
        }
        wg -= wgs;
    }
    const int key_items = mv_key_items(j.at, j.n) * a.heads, value_items = 2 * mv_value_items(j.at, j.n) * a.heads;
    const int key_wgs = (key_items + 3) / 4;
    if (wg < key_wgs) {
        const int item = wg * 4 + wave;
        if (item < key_items) mv_keys<BITS, LIST>(j, tokens, item, lane);
    } else {
        const int item = (wg - key_wgs) * 4 + wave;
        if (item < value_items) mv_values<BITS, LIST>(j, tokens, item, lane);
    }
}

// Whether tokens may go from `src` to `dst`.
kvq_status mv_check(const kvq_cache *dst, const kvq_cache *src, int64_t n)
{
    kvq_status st = kvq_check_cache(dst);
    if (st == KVQ_OK) st = kvq_check_cache(src);
    if (st != KVQ_OK) return st;
    if (n < 0 || dst->bits != src->bits || dst->n_kv_heads != src->n_kv_heads || dst->rope_base != src->rope_base) return KVQ_ERR_INVALID_ARG;
    if (dst->n_tokens_k != dst->n_tokens_v) return KVQ_ERR_INVALID_ARG;
    if (dst == src || dst->k_codes == src->k_codes || dst->v_codes == src->v_codes) return KVQ_ERR_INVALID_ARG;
    if (!src->loaded) return KVQ_ERR_NOT_LOADED;
    if (!dst->loaded && dst->n_tokens_k > 0) return KVQ_ERR_NOT_LOADED;
    if (n > dst->cap_tokens - dst->n_tokens_k) return KVQ_ERR_CAPACITY;
    return KVQ_OK;
}

void mv_job(MvJob &j, const kvq_cache *dst, const kvq_cache *src, int64_t first, int64_t n)
{
    memset(&j, 0, sizeof j);
    j.s_kc = src->k_codes; j.s_vc = src->v_codes; j.d_kc = dst->k_codes; j.d_vc = dst->v_codes;
    j.s_sz = (const uint32_t *)src->v_sz; j.d_sz = (uint32_t *)dst->v_sz;
    j.s_shift = (int16_t)src->nnz_block_shift; j.d_shift = (int16_t)dst->nnz_block_shift;
    j.k.s_ptr = src->k_ptr; j.k.d_ptr = dst->k_ptr; j.v.s_ptr = src->v_ptr; j.v.d_ptr = dst->v_ptr;
    j.k.s_idx = j.s_shift ? (const void *)src->k_idx_blocks : src->k_idx;
    j.k.s_val = j.s_shift ? (const void *)src->k_val_blocks : src->k_val;
    j.v.s_idx = j.s_shift ? (const void *)src->v_idx_blocks : src->v_idx;
    j.v.s_val = j.s_shift ? (const void *)src->v_val_blocks : src->v_val;
    j.k.d_idx = j.d_shift ? (void *)dst->k_idx_blocks : dst->k_idx;
    j.k.d_val = j.d_shift ? (void *)dst->k_val_blocks : dst->k_val;
    j.v.d_idx = j.d_shift ? (void *)dst->v_idx_blocks : dst->v_idx;
    j.v.d_val = j.d_shift ? (void *)dst->v_val_blocks : dst->v_val;
    j.k_room = (uint32_t)(dst->cap_nnz_k < 0xFFFFFFFFll ? dst->cap_nnz_k : 0xFFFFFFFFll);
    j.v_room = (uint32_t)(dst->cap_nnz_v < 0xFFFFFFFFll ? dst->cap_nnz_v : 0xFFFFFFFFll);
    j.status = dst->d_status;
    j.s_sink_k = src->sink_k; j.s_sink_v = src->sink_v; j.d_sink_k = dst->sink_k; j.d_sink_v = dst->sink_v;
    if (!dst->loaded) {
        j.s_params = (const uint32_t *)src->params;
        j.d_params = (uint32_t *)dst->params;
    }
    j.s_n = (int32_t)(src->n_tokens_k < src->n_tokens_v ? src->n_tokens_k : src->n_tokens_v);
    j.s_cap = (int32_t)src->cap_tokens; j.d_cap = (int32_t)dst->cap_tokens;
    j.first = (int32_t)first; j.at = (int32_t)dst->n_tokens_k; j.n = (int32_t)n;
    j.s_sink = (int16_t)src->n_sink; j.d_sink = (int16_t)dst->n_sink;
}

int64_t mv_wgs(const MvJob &j, int heads, int param_words, bool list)
{
    const int64_t keys = (int64_t)mv_key_items(j.at, j.n) * heads, values = 2 * (int64_t)mv_value_items(j.at, j.n) * heads;
    return mv_groups(j.n) * (list ? MV_LIST_WGS : 2) + (j.s_params ? (param_words + 16 * MV_NT - 1) / (16 * MV_NT) : 0) + (keys + 3) / 4 + (values + 3) / 4;
}

template <bool LIST>
kvq_status mv_launch(const MvArgs &a, int bits, int64_t wgs, const int32_t *tokens, const uint32_t *sums, hipStream_t s)
{
    const dim3 grid((unsigned)wgs), block(MV_NT);
    if (bits == 2) kvq_move<2, LIST><<<grid, block, 0, s>>>(a, tokens, sums);
    else if (bits == 3) kvq_move<3, LIST><<<grid, block, 0, s>>>(a, tokens, sums);
    else kvq_move<4, LIST><<<grid, block, 0, s>>>(a, tokens, sums);
    KVQ_HIP_CHECK(hipGetLastError());
    return KVQ_OK;
}

void mv_done(kvq_cache *dst, const kvq_cache *src, int64_t n)
{
    if (!dst->loaded) dst->loaded = src->loaded;
    else if (!(src->loaded & 2)) dst->loaded &= ~2;       // the destination may hold Key outliers now, whatever its thresholds admit
    dst->n_tokens_k += n;
    dst->n_tokens_v += n;
}

}  // namespace

extern "C" kvq_status kvq_cache_copy(kvq_cache *const *dst, const kvq_cache *const *src, const int64_t *first, const int64_t *count,
                                     int32_t n_copies, void *stream)
{
    if (n_copies < 0 || (n_copies > 0 && (!dst || !src || !first || !count))) return KVQ_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n_copies; ++i) {
        const kvq_status st = mv_check(dst[i], src[i], count[i]);
        if (st != KVQ_OK) return st;
        if (first[i] < 0 || first[i] > src[i]->n_tokens_k - count[i] || first[i] > src[i]->n_tokens_v - count[i]) return KVQ_ERR_INVALID_ARG;
        // sink tokens have their fp16 rows only where they are sink tokens of the source
        const int64_t at = dst[i]->n_tokens_k, sinks = dst[i]->n_sink - at < count[i] ? dst[i]->n_sink - at : count[i];
        if (sinks > 0 && first[i] + sinks > src[i]->n_sink) return KVQ_ERR_INVALID_ARG;
        if (dst[i]->bits != dst[0]->bits || dst[i]->n_kv_heads != dst[0]->n_kv_heads) return KVQ_ERR_INVALID_ARG;
    }
    // no destination is another's source or destination as well
    for (int32_t i = 0; i < n_copies; ++i)
        for (int32_t k = 0; k < n_copies; ++k)
            if (dst[i]->k_codes == src[k]->k_codes || (k < i && dst[i]->k_codes == dst[k]->k_codes)) return KVQ_ERR_INVALID_ARG;
    MvArgs a;
    memset(&a, 0, sizeof a);
    int64_t wgs = 0;
    int32_t started = 0;                                    // copies launched before the ones in `a`
    for (int32_t i = 0; i < n_copies; ++i) {
        a.heads = dst[i]->n_kv_heads;
        a.param_words = (int32_t)(kvq_params_bytes(a.heads) / 4);
        MvJob &j = a.job[a.n_jobs];
        mv_job(j, dst[i], src[i], first[i], count[i]);
        a.wg0[a.n_jobs++] = (int32_t)wgs;
        wgs += (count[i] > 0 || j.s_params) ? mv_wgs(j, a.heads, a.param_words, false) : 0;
        a.wg0[a.n_jobs] = (int32_t)wgs;
        if (a.n_jobs == MV_JOBS || i + 1 == n_copies || wgs > (1 << 28)) {
            if (wgs > 0) {
                const kvq_status st = mv_launch<false>(a, dst[i]->bits, wgs, nullptr, nullptr, (hipStream_t)stream);
                if (st != KVQ_OK) return st;
            }
            for (int32_t k = started; k <= i; ++k) mv_done(dst[k], src[k], count[k]);
            started = i + 1;
            a.n_jobs = 0;
            wgs = 0;
        }
    }
    return KVQ_OK;
}

extern "C" kvq_status kvq_cache_gather(kvq_cache *dst, const kvq_cache *src, const int32_t *d_tokens, int64_t n, void *stream)
{
    const kvq_status st = mv_check(dst, src, n);
    if (st != KVQ_OK) return st;
    if (src->n_tokens_k != src->n_tokens_v) return KVQ_ERR_INVALID_ARG;
    if (n == 0) return KVQ_OK;
    if (!d_tokens || ((uintptr_t)d_tokens & 3) || src->n_tokens_k == 0) return KVQ_ERR_INVALID_ARG;
    const int64_t groups = (n + MV_GROUP - 1) / MV_GROUP;
    if (!dst->workspace || dst->workspace_bytes < groups * 8) return KVQ_ERR_CAPACITY;
    MvArgs a;
    memset(&a, 0, sizeof a);
    a.heads = dst->n_kv_heads;
    a.n_jobs = 1;
    a.param_words = (int32_t)(kvq_params_bytes(a.heads) / 4);
    mv_job(a.job[0], dst, src, 0, n);
    const int64_t wgs = mv_wgs(a.job[0], a.heads, a.param_words, true);
    a.wg0[1] = (int32_t)wgs;
    if (wgs >= ((int64_t)1 << 31)) return KVQ_ERR_UNSUPPORTED;
    uint32_t *sums = (uint32_t *)dst->workspace;
    kvq_move_counts<<<dim3((unsigned)groups), dim3(MV_NT), 0, (hipStream_t)stream>>>(a.job[0], d_tokens, sums);
    KVQ_HIP_CHECK(hipGetLastError());
    const kvq_status go = mv_launch<true>(a, dst->bits, wgs, d_tokens, sums, (hipStream_t)stream);
    if (go != KVQ_OK) return go;
    mv_done(dst, src, n);
    return KVQ_OK;
}

extern "C" kvq_status kvq_cache_truncate(kvq_cache *cache, int64_t n_tokens)
{
    const kvq_status st = kvq_check_cache(cache);
    if (st != KVQ_OK) return st;
    if (n_tokens < 0 || n_tokens > cache->n_tokens_k || n_tokens > cache->n_tokens_v) return KVQ_ERR_INVALID_ARG;
    cache->n_tokens_k = cache->n_tokens_v = n_tokens;
    return KVQ_OK;
}
