// One decode step's attention for a batch of sequences that share a prefix (paper Sec. 3: generation-time attention over
// the quantized cache; Sec. 3.2: Keys rotated after de-quantisation).
//
//   out[b][q] = sum_n softmax_n(x[b][q][.])[n] vhat[n],   x[b][q][n] = scale <q_rot[b][q], R_n khat[n]>,
//
// n over the prefix's tokens and the sequence's own, whose positions follow the prefix's.  A token's Key is de-quantised
// and rotated once for all queries that see it, so the work per element no longer depends on the batch until the products
// do: they run on the matrix cores, the only units with the rate for (tokens x queries x 128) twice.
//
// Numbers.  The products are fp16 with fp32 sums, yet as exact as fp32 ones: a factor that is not an fp16 number goes in as
// two (x = hi + lo, 22 bits or 2^-24 absolute, whichever is coarser), lo * lo left out.
//   scores  K' = R_n khat in two parts, the query in two parts (scaled by a power of two per query): three products.
//   output  vhat = s_n lut[code] + z_n + residual.  lut[code] and the residuals are fp16 numbers as they are stored, so
//           sum_n (p_n s_n) lut[code] + sum_n p_n (residual + z_n) needs only the weights in two parts: two products each.
// Weights are scaled by 2^kappa, which keeps p_n and p_n s_n below 2^15 and the absolute error of the small ones at 2^-24 / 2^kappa.
//
// Layout.  A wavefront takes 32 tokens at a time.  Operands of v_mfma_f32_16x16x32_f16 hold eight k-indices per lane, and
// a k-index may stand for any channel (any token) as long as both operands agree.  So a lane (token r, group g) de-quantises
// the 16 channel pairs 16 g .. 16 g + 15 of its token, which are consecutive fields of its chunk, straight into operand
// registers; the scores come out with a query per lane column and tokens 4 g .. 4 g + 3 in its registers, which is the
// weights' operand of the second product as it stands; and the Values' operand, two tokens to a field, comes from one look-up
// per field.  Nothing crosses lanes but the maximum of a query's 32 scores.
//
// Outliers reach their element through LDS: a first kernel sorts the entries of every 32 tokens by head, and the wavefront
// scatters its head's residuals into a zeroed patch that it reads beside the codes.
#include <math.h>
#include <string.h>
#include <type_traits>
#include "kvq_common.hpp"
#include "kvq_qk_sparse.hpp"

namespace {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr int BT_BLOCK = 32;            // tokens a wavefront takes at a time
constexpr int BT_WAVES = 4;             // wavefronts of a workgroup
constexpr int BT_NT = 64 * BT_WAVES;
constexpr int BT_ROW = 256;             // halves of a query's row: 128 high parts, 128 low parts
constexpr int BT_SEGS = 24;             // descriptors that travel in one launch's arguments
constexpr int BT_MAX_HEADS = 512;
constexpr int BT_PATCH = 8192;          // bytes of a wavefront's patch
constexpr float BT_MAX_SLACK = 6.0f;    // the running maximum follows a larger score from 2^6 times the weight on
constexpr int64_t BT_OWN_ROUNDS = 3;    // workgroups of a batch without a prefix, in times what the chip holds
constexpr int BT_KAPPA = 9;             // 2^(6 + 9) is the largest weight then

// One cache as the kernels see it.
struct BtSeg {
    const uint8_t *k_codes, *v_codes;
    const uint32_t *v_sz;               // fp16 scale, zero-point of a token
    const uint32_t *k_ptr, *v_ptr;
    const void *k_idx, *k_val, *v_idx, *v_val;     // flat arrays, or tables of blocks (shift != 0)
    const void *params;
    const uint16_t *sink_k, *sink_v;
    int64_t k_list, v_list;             // places of its sorted entries
    uint32_t k_room, v_room;
    int32_t n, cap, shift, n_sink;
    int32_t blk0;                       // number of its first 32-token block
    int32_t chunk0;                     // number of its first workgroup's tokens among those of its launch
    int32_t wg0, pad;                   // its first workgroup of the first kernel
};

struct BtWork {                         // the workspace
    BtSeg *segs;                        // [0] the prefix, [1 + b] sequence b's own
    uint32_t *k_start, *v_start;        // [block][heads + 1]: first entry of a head
    float *smax;                        // [block]: largest Value scale
    _Float16 *rows[2];                  // query rows: for the prefix [head][b][r], for the own tokens [b][head][r]
    float *row_scale[2];
    uint32_t *k_list, *v_list;          // entries: residual << 16 | token << 7 | channel
    float *part_o[2], *part_ml[2];      // [chunk][head][query] sums of a workgroup: output; maximum, weights
    int32_t *owner;                     // [chunk of own tokens]: whose
};

struct BtArgs {
    BtWork w;
    const float *q;
    float *out;
    float scale;
    int32_t n_seqs, heads, ratio, prefix, own;     // own: some sequence has tokens of its own
    int32_t chunk[2], n_chunks[2], mp[2];          // blocks per workgroup, workgroups per head, queries per slot (padded)
};

struct BtSegs {
    BtSeg seg[BT_SEGS];
    int32_t first, n;                              // number of the first, how many
};

static_assert(sizeof(BtArgs) + sizeof(BtSegs) + 16 <= 4096, "kernel arguments");

// A pointer that came out of memory, as one to global memory: the compiler takes it for one that may point to LDS as well, and loads
// through such a pointer are waited for together with the LDS, the requests of the next step among them.  (128 queries on each of
// 8 heads, 524287 tokens: 1132 us with such loads, 1074 with these.)
template <class T>
__device__ __forceinline__ T *bt_global(T *p)
{
    return (T *)(__attribute__((address_space(1))) T *)(uintptr_t)p;
}
__device__ __forceinline__ BtSeg bt_seg(const BtSeg &g)
{
    BtSeg s = g;
    s.k_codes = bt_global(g.k_codes); s.v_codes = bt_global(g.v_codes); s.v_sz = bt_global(g.v_sz);
    s.k_ptr = bt_global(g.k_ptr); s.v_ptr = bt_global(g.v_ptr);
    s.k_idx = bt_global(g.k_idx); s.k_val = bt_global(g.k_val); s.v_idx = bt_global(g.v_idx); s.v_val = bt_global(g.v_val);
    s.params = bt_global(g.params); s.sink_k = bt_global(g.sink_k); s.sink_v = bt_global(g.sink_v);
    return s;
}

template <bool BLOCKED>
__device__ __forceinline__ uint32_t bt_entry(const void *arr, int shift, uint32_t e)
{
    if (!BLOCKED) return ((const uint16_t *)arr)[e];
    return bt_global(((const uint16_t *const *)arr)[e >> shift])[e & ((1u << shift) - 1u)];
}

// The entries of SORT blocks of 32 tokens sorted by block and head: eight lanes a token, an entry's rank among its head's from the count
// that it adds to, its place from the sums of the counts.  (The order within a head is any: every entry has an element of its own.)
// A lane keeps up to HELD entries of each block in registers from the count to the placing; where a token has more they are read
// twice.  Attention-sink tokens (before `first`) have none: nothing reads them in this form, and what they hold (an infinite
// residual, say) is to reach no sum.
// Each stage is a round trip to memory or to LDS, and how many blocks a compute unit has under way decides: 131072 tokens of 32
// heads take 40 us with one block per workgroup, 31 with two, 35 with four; to LDS first and from there in order to memory 32; 64
// tokens' entries dealt out evenly, with a search for each lane's token, 69.  Layers of few heads have few entries a token:
// 524287 tokens of 8 heads take 76 us with two blocks, 62 with four of half the registers, 57 with eight, which take 8 us for 300
// tokens where the others take 6.
constexpr int BT_HELD = 6, BT_SORT = 2, BT_HELD_FEW = 3, BT_SORT_FEW = 4, BT_FEW_HEADS = 16;

template <bool BLOCKED, int SORT, int HELD>
__device__ void bt_sort_side(const uint32_t *ptr, const void *idx, const void *val, int shift, uint32_t room, int n0, int first,
                             int n, int heads, uint32_t *start, uint32_t *list, uint32_t *count)
{
    const int tid = threadIdx.x, t = tid >> 3, l = tid & 7, lane = tid & 63, wave = tid >> 6;
    for (int h = tid; h < SORT * heads; h += BT_NT) count[h] = 0u;
    uint32_t p0[SORT], p1[SORT], x[SORT][HELD], v[SORT][HELD], rank[SORT][HELD];
    uint32_t base[(SORT + BT_WAVES - 1) / BT_WAVES];             // first entries of the blocks whose sums this wavefront takes
#pragma unroll
    for (int k = 0; k < (SORT + BT_WAVES - 1) / BT_WAVES; ++k) {
        const int m = n0 + (wave + k * BT_WAVES) * BT_BLOCK;
        base[k] = ptr[m < n ? m : n];
    }
#pragma unroll
    for (int b = 0; b < SORT; ++b) {
        const int m = n0 + b * BT_BLOCK + t;
        p0[b] = ptr[m < n ? m : n];
        p1[b] = ptr[m < n ? m + 1 : n];
    }
    bool more = false;
#pragma unroll
    for (int b = 0; b < SORT; ++b) {
        p1[b] = n0 + b * BT_BLOCK + t < first ? 0u : p1[b] < room ? p1[b] : room;
        more |= p1[b] > p0[b] + 8 * HELD;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const uint32_t e = p0[b] + l + 8 * i;
            if (e < p1[b]) {
                x[b][i] = bt_entry<BLOCKED>(idx, shift, e);
                v[b][i] = bt_entry<BLOCKED>(val, shift, e);      // (put together below, behind the asm: in here each pair would be waited for by itself)
            }
        }
    }
#pragma unroll
    for (int b = 0; b < SORT; ++b)
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            asm volatile("" : "+v"(v[b][i]));
            x[b][i] |= v[b][i] << 16;
        }
    const bool many = __syncthreads_or(more) != 0;
#pragma unroll
    for (int b = 0; b < SORT; ++b) {
        uint32_t *const mine = count + b * heads;
        if (!many) {
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (p0[b] + l + 8 * i < p1[b] && ((x[b][i] & 0xFFFFu) >> 7) < (uint32_t)heads) rank[b][i] = atomicAdd(&mine[(x[b][i] & 0xFFFFu) >> 7], 1u);
        } else {
            for (uint32_t e = p0[b] + l; e < p1[b]; e += 8) {
                const uint32_t h = bt_entry<BLOCKED>(idx, shift, e) >> 7;
                if (h < (uint32_t)heads) atomicAdd(&mine[h], 1u);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < (SORT + BT_WAVES - 1) / BT_WAVES; ++k) {            // exclusive sums, a wavefront a block, up to eight heads a lane
        const int b = wave + k * BT_WAVES;
        if (b >= SORT) break;
        uint32_t c[BT_MAX_HEADS / 64], s = 0, *const mine = count + b * heads;
        const int per = (heads + 63) / 64;
#pragma unroll
        for (int i = 0; i < BT_MAX_HEADS / 64; ++i) {
            const int h = lane * per + i;
            c[i] = (i < per && h < heads) ? mine[h] : 0u;
            s += c[i];
        }
        uint32_t before = s;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = (uint32_t)__shfl_up((int)before, d);
            if (lane >= d) before += o;
        }
        before += base[k] - s;
#pragma unroll
        for (int i = 0; i < BT_MAX_HEADS / 64; ++i) {
            const int h = lane * per + i;
            if (i < per && h < heads) {
                mine[h] = before;
                if (n0 + b * BT_BLOCK < n) {
                    start[b * (heads + 1) + h] = before;
                    if (h == heads - 1) start[b * (heads + 1) + heads] = before + c[i];
                }
                before += c[i];
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < SORT; ++b) {
        uint32_t *const mine = count + b * heads;
        if (!many) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const uint32_t c = x[b][i] & 0xFFFFu;
                if (p0[b] + l + 8 * i < p1[b] && (c >> 7) < (uint32_t)heads) {
                    const uint32_t at = mine[c >> 7] + rank[b][i];
                    if (at < room) list[at] = (x[b][i] & 0xFFFF0000u) | ((uint32_t)t << 7) | (c & 127u);
                }
            }
        } else {
            for (uint32_t e = p0[b] + l; e < p1[b]; e += 8) {
                const uint32_t c = bt_entry<BLOCKED>(idx, shift, e);
                if ((c >> 7) < (uint32_t)heads) {
                    const uint32_t at = atomicAdd(&mine[c >> 7], 1u);
                    if (at < room) list[at] = (bt_entry<BLOCKED>(val, shift, e) << 16) | ((uint32_t)t << 7) | (c & 127u);
                }
            }
        }
    }
}

// Rows of the scaled query: rotated back by the prefix's length for the own tokens (whose positions then start at 0), a power
// of two to bring the largest to [2^13, 2^14), two parts.  The element order is that of the operand: eight halves for
// (step t, group g) are the pairs 16 g + 4 t .. + 3.
__device__ void bt_query_row(const BtArgs &a, const KvqParamsHeader *hdr, int which, int row, int lane)
{
    // row: [b][query head]
    const int b = row / (a.heads * a.ratio), qh = row % (a.heads * a.ratio), h = qh / a.ratio, r = qh % a.ratio;
    const float f = a.scale * KVQ_LOG2E;
    float x = a.q[(int64_t)row * 128 + lane] * f, y = a.q[(int64_t)row * 128 + 64 + lane] * f;
    if (which == 1 && a.prefix > 0) {
        float c, s;
        sincospif(2.0f * rope_rev((float)a.prefix, hdr->rope_vh[lane], hdr->rope_vl[lane]), &s, &c);
        const float x0 = x, y0 = y;
        x = __builtin_fmaf(x0, c, y0 * s);
        y = __builtin_fmaf(y0, c, -(x0 * s));
    }
    const float m = kvq_wave_max(__builtin_fmaxf(__builtin_fabsf(x), __builtin_fabsf(y)));
    int e = 0;
    if (m > 0.0f && m < __builtin_inff()) (void)frexpf(m, &e);
    e = e > -100 ? e : -100;                        // smaller ones have scores of nothing; a scale of zero would make NaN of a masked one
    x = ldexpf(x, 14 - e);
    y = ldexpf(y, 14 - e);
    const int64_t at = which == 0 ? ((int64_t)h * a.n_seqs + b) * a.ratio + r : (int64_t)row;
    const half2_t hi = {(_Float16)x, (_Float16)y};
    const half2_t lo = {(_Float16)(x - (float)hi.x), (_Float16)(y - (float)hi.y)};
    const int g = lane >> 4, t = (lane >> 2) & 3, u = lane & 3;
    half2_t *o = (half2_t *)(a.w.rows[which] + at * BT_ROW) + (t * 4 + g) * 4 + u;
    o[0] = hi;
    o[64] = lo;
    if (lane == 0) a.w.row_scale[which][at] = ldexpf(1.0f, e - 14);
}

// Descriptors from the arguments to memory.
__device__ __forceinline__ void bt_upload(const BtArgs &a, const BtSegs &s)
{
    const uint32_t *from = (const uint32_t *)s.seg;
    uint32_t *to = (uint32_t *)(a.w.segs + s.first);
    for (int i = threadIdx.x; i < s.n * (int)(sizeof(BtSeg) / 4); i += BT_NT) to[i] = from[i];
}
__global__ __launch_bounds__(BT_NT) void kvq_batch_upload(BtArgs a, BtSegs s) { bt_upload(a, s); }

// First kernel: query rows; outliers by head, SORT blocks of 32 tokens and a side per workgroup.  A call whose descriptors fit in the
// arguments brings them along; otherwise (`total` > s.n) they are in memory already.
template <int SORT, int HELD>
__global__ __launch_bounds__(BT_NT) void kvq_batch_prepare(BtArgs a, BtSegs s, int row_wgs, int total)
{
    __shared__ uint32_t count[SORT * (SORT == BT_SORT ? BT_MAX_HEADS : BT_FEW_HEADS)];
    const int tid = threadIdx.x, lane = tid & 63;
    int wg = blockIdx.x;
    if (wg == 0 && total == s.n) bt_upload(a, s);
    if (wg < row_wgs) {
        const int rows = a.n_seqs * a.heads * a.ratio, row = wg * BT_WAVES + (tid >> 6);
        if (row >= rows) return;
        const KvqParamsHeader *hdr = (const KvqParamsHeader *)bt_global(s.seg[0].params);       // the rotary constants are one layer's
        if (a.prefix > 0) bt_query_row(a, hdr, 0, row, lane);
        if (a.own) bt_query_row(a, hdr, 1, row, lane);
        return;
    }
    wg -= row_wgs;
    const bool values = wg & 1;                     // a workgroup per side: the chain of each is latency
    wg >>= 1;
    int i = 0;
    if (total == s.n) {
        while (i + 1 < s.n && wg >= s.seg[i + 1].wg0) ++i;
    } else {                                        // the last whose first workgroup is not after this one
        int found = 0;
        for (int b = 0; b < total; b += 64) {
            const int k = b + lane;
            found += __popcll(__ballot(k < total && a.w.segs[k].wg0 <= wg));
        }
        i = __builtin_amdgcn_readfirstlane(found) - 1;
    }
    const BtSeg g = total == s.n ? bt_seg(s.seg[i]) : bt_seg(a.w.segs[i]);
    const int blk = SORT * (wg - g.wg0), n0 = blk * BT_BLOCK;
    if (n0 >= g.n) return;
    const int64_t at = (int64_t)(g.blk0 + blk) * (a.heads + 1);
    const uint32_t *ptr = values ? g.v_ptr : g.k_ptr;
    const void *idx = values ? g.v_idx : g.k_idx, *val = values ? g.v_val : g.k_val;
    const uint32_t room = values ? g.v_room : g.k_room;
    if (blk == 0 && values && i > 0)                // the workgroups of a sequence's own tokens find it by their number
        for (int c = tid; c < (g.n + a.chunk[1] * BT_BLOCK - 1) / (a.chunk[1] * BT_BLOCK); c += BT_NT) a.w.owner[g.chunk0 + c] = i;
    uint32_t *start = (values ? a.w.v_start : a.w.k_start) + at, *list = values ? a.w.v_list + g.v_list : a.w.k_list + g.k_list;
    if (g.shift == 0) bt_sort_side<false, SORT, HELD>(ptr, idx, val, 0, room, n0, g.n_sink, g.n, a.heads, start, list, count);
    else bt_sort_side<true, SORT, HELD>(ptr, idx, val, g.shift, room, n0, g.n_sink, g.n, a.heads, start, list, count);
    if (values && tid < SORT * BT_BLOCK) {
        float m = 0.0f;
        if (n0 + tid >= g.n_sink && n0 + tid < g.n) m = __builtin_fabsf(kvq_h2f((uint16_t)(g.v_sz[n0 + tid] & 0xFFFFu)));
        for (int d = 16; d; d >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, d));
        if ((tid & 31) == 0 && n0 + tid < g.n) a.w.smax[g.blk0 + blk + (tid >> 5)] = m;
    }
}

__device__ __forceinline__ void bt_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Maximum over the four lanes of a column.
__device__ __forceinline__ float bt_column_max(float v)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    const u32x2 r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    v = __builtin_fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
    const uint32_t d = __builtin_bit_cast(uint32_t, v);
    const u32x2 q = __builtin_amdgcn_permlane16_swap(d, d, false, false);
    return __builtin_fmaxf(__builtin_bit_cast(float, (uint32_t)q[0]), __builtin_bit_cast(float, (uint32_t)q[1]));
}

// (hi, lo) parts of two numbers, packed; `minus_one` is opaque to the compiler, so that hi - x stays one instruction.
__device__ __forceinline__ void bt_split(float x, float y, float minus_one, uint32_t &hi, uint32_t &lo)
{
    const auto h = __builtin_amdgcn_cvt_pkrtz(x, y);
    const half2_t hh = __builtin_bit_cast(half2_t, h);
    const float a = __builtin_fmaf((float)hh.x, minus_one, x), b = __builtin_fmaf((float)hh.y, minus_one, y);
    hi = __builtin_bit_cast(uint32_t, h);
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}

__device__ __forceinline__ half8_t bt_half8(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_bit_cast(half8_t, uint4{a, b, c, d});
}

__device__ __forceinline__ float4_t bt_mfma(half8_t a, half8_t b, float4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Byte of a wavefront's patch for an entry.  Keys: [token block][step t][lane (g, token)][pair u][channel half]; Values:
// [channel block][lane (g, channel)][token block][token].
__device__ __forceinline__ uint32_t bt_key_place(uint32_t x)
{
    const uint32_t t = (x >> 7) & 31u, c = x & 127u, p = c & 63u;
    return ((((t >> 4) * 4 + ((p >> 2) & 3)) * 64 + (p >> 4) * 16 + (t & 15)) * 4 + (p & 3)) * 4 + (c >> 6) * 2;
}
__device__ __forceinline__ uint32_t bt_value_place(uint32_t x)
{
    const uint32_t t = (x >> 7) & 31u, c = x & 127u, j = c & 63u;
    return ((((c >> 6) * 4 + (j & 3)) * 64 + ((t >> 2) & 3) * 16 + (j >> 2)) * 8 + (t >> 4) * 4 + (t & 3)) * 2;
}

// ---- what the two forms of the second kernel share ---------------------------------------------------------------

// A workgroup's tokens and queries.
struct BtPart {
    int si, h, ch, qb, n, first, b0, b1, n_q;
    int64_t row0;                       // its queries' first row
};

template <int WHICH>
__device__ __forceinline__ BtPart bt_part(const BtArgs &a, int wg, int queries)
{
    BtPart p;
    // workgroups: query blocks innermost (they read the same codes), then heads, then chunks
    const int qblocks = a.mp[WHICH] / queries;
    p.qb = wg % qblocks;
    p.h = (wg / qblocks) % a.heads;
    p.ch = wg / (qblocks * a.heads);
    p.si = WHICH == 1 ? a.w.owner[p.ch] : 0;
    const BtSeg &sg = a.w.segs[p.si];
    p.n = sg.n;
    const int n_blocks = (p.n + BT_BLOCK - 1) / BT_BLOCK;
    p.b0 = (p.ch - (WHICH == 1 ? sg.chunk0 : 0)) * a.chunk[WHICH];
    p.b1 = p.b0 + a.chunk[WHICH] < n_blocks ? p.b0 + a.chunk[WHICH] : n_blocks;
    p.first = sg.n_sink < p.n ? sg.n_sink : p.n;           // sink tokens are not attended to here
    p.n_q = WHICH == 0 ? a.n_seqs * a.ratio : a.ratio;
    p.row0 = WHICH == 0 ? (int64_t)p.h * p.n_q : ((int64_t)(p.si - 1) * a.heads + p.h) * p.n_q;
    return p;
}

// The layer's and the head's constants in LDS.
template <int BITS>
struct BtConst {
    static constexpr int NE = 1 << BITS, FB = 2 * BITS;
    static constexpr uint32_t FMASK = (1u << FB) - 1u;
    uint32_t lut_k[NE * NE], lut_v[NE * NE];               // pairs of signposts by field
    __attribute__((aligned(16))) uint32_t s[64], z[64];    // Key scales and zero-points: (channel i, channel i + 64) fp16
    __attribute__((aligned(16))) float vh[64];             // theta_i / 2 pi
    float red[BT_WAVES];
    // What a thread brings along: requested together, put into LDS when the other requests of the start are under way as well.
    struct Brought {
        float k0, k1, v0, v1, vh, m;
        uint16_t s0, s1, z0, z1;
    };
    static __device__ __forceinline__ Brought load(const BtArgs &a, const BtSeg &sg, const BtPart &p)
    {
        static_assert(NE * NE <= BT_NT, "a field per thread");
        const int tid = threadIdx.x, f = tid & (NE * NE - 1), c = p.h * 128 + (tid & 63), b = p.b0 + tid;
        const KvqParamsView pv = kvq_params_view(sg.params, a.heads * KVQ_HEAD_DIM);
        Brought t;
        t.k0 = pv.hdr->lut_k[f & (NE - 1)];
        t.k1 = pv.hdr->lut_k[f >> BITS];
        t.v0 = pv.hdr->lut_v[f & (NE - 1)];
        t.v1 = pv.hdr->lut_v[f >> BITS];
        t.s0 = pv.s16[c];
        t.s1 = pv.s16[c + 64];
        t.z0 = pv.z16[c];
        t.z1 = pv.z16[c + 64];
        t.vh = pv.hdr->rope_vh[tid & 63];
        t.m = a.w.smax[sg.blk0 + (b < p.b1 ? b : p.b1 - 1)];
        return t;
    }
    __device__ __forceinline__ void stage(const BtArgs &a, const BtSeg &sg, const BtPart &p, const Brought &t)
    {
        const int tid = threadIdx.x;
        if (tid < NE * NE) {
            const half2_t k = {(_Float16)t.k0, (_Float16)t.k1}, v = {(_Float16)t.v0, (_Float16)t.v1};
            lut_k[tid] = __builtin_bit_cast(uint32_t, k);
            lut_v[tid] = __builtin_bit_cast(uint32_t, v);
        }
        if (tid < 64) {
            s[tid] = t.s0 | ((uint32_t)t.s1 << 16);
            z[tid] = t.z0 | ((uint32_t)t.z1 << 16);
            vh[tid] = t.vh;
        }
        float m = t.m;
        for (int b = p.b0 + tid + BT_NT; b < p.b1; b += BT_NT) m = __builtin_fmaxf(m, a.w.smax[sg.blk0 + b]);
        m = kvq_wave_max(m);
        if ((tid & 63) == 0) red[tid >> 6] = m;
    }
    // Exponent of the weights' scale: p <= 2^(BT_MAX_SLACK + kappa) and p s as well stay below 2^15 (every scale < 2^e).
    __device__ __forceinline__ float kappa() const
    {
        const float m = __builtin_fmaxf(__builtin_fmaxf(red[0], red[1]), __builtin_fmaxf(red[2], red[3]));
        int e = 0;
        if (m > 0.0f) (void)frexpf(m, &e);
        return (float)(e > 0 ? BT_KAPPA - e : BT_KAPPA);
    }
};

// This lane's dwords of a chunk.  Keys: BITS of them from dword BITS * g on; Values: those with bits 8 BITS r16 on.
template <int BITS>
struct BtLane {
    uint32_t k_off[BITS], v_off0, v_off1, v_shift;
    __device__ __forceinline__ BtLane(int r16, int g)
    {
#pragma unroll
        for (int i = 0; i < BITS; ++i) k_off[i] = (uint32_t)(((BITS * g + i) >> 2) * 1024 + ((BITS * g + i) & 3) * 4 + r16 * 16);
        const int bit = 8 * BITS * r16, d0 = bit >> 5, d1 = (BITS == 3 && d0 < 11) ? d0 + 1 : d0;
        v_shift = (uint32_t)(bit & 31);
        v_off0 = (uint32_t)((d0 >> 2) * 1024 + (d0 & 3) * 4 + g * 32);
        v_off1 = (uint32_t)((d1 >> 2) * 1024 + (d1 & 3) * 4 + g * 32);
    }
};

// The dwords with this lane's four fields of a half of 32 tokens' Values: [token block][pair].
template <int BITS>
struct BtCodes {
    uint32_t c0[2][2], c1[BITS == 3 ? 2 : 1][2];
    __device__ __forceinline__ void load(const uint8_t *half, int n0, const BtLane<BITS> &l)
    {
        const uint8_t *vc = half + (int64_t)(n0 >> 7) * (64 * 16 * BITS) + ((n0 >> 1) & 63) * 16;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int pr = 0; pr < 2; ++pr) {
                const uint8_t *p = vc + tb * 128 + pr * 16;
                c0[tb][pr] = *(const uint32_t *)(p + l.v_off0);
                if (BITS == 3) c1[tb][pr] = *(const uint32_t *)(p + l.v_off1);
            }
    }
    // The fields at the bottom of a word each.
    __device__ __forceinline__ void align(uint32_t (&w)[4], uint32_t shift) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = c0[i >> 1][i & 1];
            if (BITS == 3) w[i] = __builtin_amdgcn_alignbit(c1[BITS == 3 ? i >> 1 : 0][i & 1], w[i], shift);
            if (BITS == 2) w[i] >>= shift;
        }
    }
};
// Operand of one of the half's channel blocks: channels 4 r16 + sub of the half.
template <int BITS>
__device__ __forceinline__ half8_t bt_value_operand(const uint32_t (&w)[4], int sub, const uint32_t *lut)
{
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int sh = 2 * BITS * sub - 2;
        x[i] = *(const uint32_t *)((const uint8_t *)lut + ((sh < 0 ? w[i] << -sh : w[i] >> sh) & (((1u << 2 * BITS) - 1u) << 2)));
    }
    return bt_half8(x[0], x[1], x[2], x[3]);
}
// (scale, zero-point) of this lane's tokens: 4 g .. 4 g + 3 of both blocks.
__device__ __forceinline__ void bt_scales(uint32_t (&sz)[2][4], const uint32_t *v_sz, int n0, int g)
{
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
        const uint4 v = *(const uint4 *)(v_sz + n0 + tb * 16 + g * 4);
        sz[tb][0] = v.x; sz[tb][1] = v.y; sz[tb][2] = v.z; sz[tb][3] = v.w;
    }
}

// One pair (i, i + 64) of a token: de-quantised, its residuals added, rotated, in two parts.
template <bool PATCHED>
__device__ __forceinline__ void bt_key_pair(uint32_t field_lut, uint32_t sc2, uint32_t zc2, uint32_t re2, float rev, float minus_one, float one,
                                            uint32_t &hi, uint32_t &lo)
{
    const half2_t l = __builtin_bit_cast(half2_t, field_lut), sc = __builtin_bit_cast(half2_t, sc2), zc = __builtin_bit_cast(half2_t, zc2),
                  re = __builtin_bit_cast(half2_t, re2);
    float ka = __builtin_fmaf((float)l.x, (float)sc.x, (float)zc.x), kb = __builtin_fmaf((float)l.y, (float)sc.y, (float)zc.y);
    if (PATCHED) {
        ka = __builtin_fmaf((float)re.x, one, ka);
        kb = __builtin_fmaf((float)re.y, one, kb);
    }
    const float c = __builtin_amdgcn_cosf(rev), sn = __builtin_amdgcn_sinf(rev);
    bt_split(__builtin_fmaf(ka, c, -(kb * sn)), __builtin_fmaf(kb, c, ka * sn), minus_one, hi, lo);
}

template <int BITS>
__device__ __forceinline__ uint32_t bt_key_field(const uint32_t (&w)[BITS], int j)
{
    constexpr int FB = 2 * BITS;
    const int bit = j * FB, wi = bit >> 5, sh = bit & 31;
    const uint32_t f = sh + FB <= 32 ? w[wi] >> sh : __builtin_amdgcn_alignbit(w[wi + (sh + FB > 32)], w[wi], sh);
    return f & ((1u << FB) - 1u);
}

// Running sums of MB blocks of 16 queries: a query per column of the lanes, in log2 units with its own maximum.
template <int MB>
struct BtSums {
    float4_t o[8][MB];                  // output by channel block
    float2_t lz[MB];                    // (sum of p z, sum of p) in the first 16 lanes
    float m[MB], inv[MB];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            m[mb] = KVQ_STAT_FLOOR;
            lz[mb] = float2_t{0.f, 0.f};
#pragma unroll
            for (int cb = 0; cb < 8; ++cb) o[cb][mb] = float4_t{0.f, 0.f, 0.f, 0.f};
        }
    }
};
struct BtWeights {                      // p and p s in two parts
    half8_t ph, pl, wh, wl;
};

// Tokens outside [first, n) of the 32 from n0 on get no weight.
template <int MB>
__device__ __forceinline__ void bt_mask(float4_t (&s)[2][MB], uint32_t (&sz)[2][4], int n0, int first, int n, int g)
{
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = n0 + tb * 16 + g * 4 + i;
            const bool in = t >= first && t < n;
            if (!in) sz[tb][i] = 0u;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
                if (!in) s[tb][mb][i] = -__builtin_inff();
        }
}

// The running maximum of block mb's queries over GROUPS x 32 more scores; where it grows by much (2^BT_MAX_SLACK in the weights) the sums
// move to the new one.
template <int MB, int GROUPS>
__device__ __forceinline__ void bt_maximum(const float4_t (&s)[GROUPS][2][MB], BtSums<MB> &sum, int mb)
{
    float m = s[0][0][mb][0];
#pragma unroll
    for (int gr = 0; gr < GROUPS; ++gr)
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int i = 0; i < 4; ++i) m = __builtin_fmaxf(m, s[gr][tb][mb][i]);
    m = bt_column_max(m) * sum.inv[mb];
    if (!(m >= KVQ_STAT_FLOOR)) m = KVQ_STAT_FLOOR;          // no token at all (-inf, or -inf * 0 in a column without a query)
    if (__ballot(m > sum.m[mb] + BT_MAX_SLACK) != 0ull) {
        const float up = m > sum.m[mb] ? m : sum.m[mb], f = __builtin_amdgcn_exp2f(sum.m[mb] - up);
        sum.m[mb] = up;
        sum.lz[mb].x *= f;
        sum.lz[mb].y *= f;
#pragma unroll
        for (int cb = 0; cb < 8; ++cb) sum.o[cb][mb] *= f;
    }
}

// Scores of 32 tokens to weights, and the sums of p z and of p (a channel block of their own with rows (z, 1, 0 ...)).  These two grow
// with every token: they are taken from zero for 32 tokens and added in fp32, which rounds to nearest.  (Left in the products'
// own sums, whose error has a direction, 524287 tokens came out 3.4e-6 to 5.2e-6 off, now 2.0e-6 to 2.4e-6, in
// the same time; 64 queries over 16384 tokens take 163 us instead of 159.)
template <int MB>
__device__ __forceinline__ void bt_weights(const float4_t (&s)[2][MB], const uint32_t (&sz)[2][4], BtSums<MB> &sum, BtWeights (&w)[MB], int r16,
                                           float kap, float minus_one)
{
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const float shift = kap - sum.m[mb];
        uint32_t a_h[4], a_l[4], w_h[4], w_l[4];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tb][mb][i], sum.inv[mb], shift));
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tb][mb][i + 1], sum.inv[mb], shift));
                const float s0 = (float)__builtin_bit_cast(half2_t, sz[tb][i]).x, s1 = (float)__builtin_bit_cast(half2_t, sz[tb][i + 1]).x;
                bt_split(p0, p1, minus_one, a_h[tb * 2 + i / 2], a_l[tb * 2 + i / 2]);
                bt_split(p0 * s0, p1 * s1, minus_one, w_h[tb * 2 + i / 2], w_l[tb * 2 + i / 2]);
            }
        w[mb].ph = bt_half8(a_h[0], a_h[1], a_h[2], a_h[3]);
        w[mb].pl = bt_half8(a_l[0], a_l[1], a_l[2], a_l[3]);
        w[mb].wh = bt_half8(w_h[0], w_h[1], w_h[2], w_h[3]);
        w[mb].wl = bt_half8(w_l[0], w_l[1], w_l[2], w_l[3]);
    }
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t z2 = __builtin_amdgcn_perm(sz[i >> 1][(i & 1) * 2 + 1], sz[i >> 1][(i & 1) * 2], 0x07060302u);
        x[i] = r16 == 0 ? z2 : r16 == 1 ? 0x3C003C00u : 0u;
    }
    const half8_t zf = bt_half8(x[0], x[1], x[2], x[3]);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const float4_t t = bt_mfma(zf, w[mb].ph, bt_mfma(zf, w[mb].pl, float4_t{0.f, 0.f, 0.f, 0.f}));
        sum.lz[mb].x += t[0];
        sum.lz[mb].y += t[1];
    }
}

// The output's products with one block of channels: `vf` its signposts, `rf` its residuals.
template <int MB>
__device__ __forceinline__ void bt_products(half8_t vf, half8_t rf, const BtWeights (&w)[MB], BtSums<MB> &sum, int cb)
{
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) sum.o[cb][mb] = bt_mfma(rf, w[mb].pl, sum.o[cb][mb]);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) sum.o[cb][mb] = bt_mfma(vf, w[mb].wl, sum.o[cb][mb]);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) sum.o[cb][mb] = bt_mfma(rf, w[mb].ph, sum.o[cb][mb]);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) sum.o[cb][mb] = bt_mfma(vf, w[mb].wh, sum.o[cb][mb]);
}

// Four consecutive channels (64 hf + 16 g + 4 i ..) of block mb's query of this lane, with the zero-points' part.
template <int MB>
__device__ __forceinline__ float4_t bt_channels(const BtSums<MB> &sum, int mb, int hf, int i, float z)
{
    return float4_t{sum.o[hf * 4 + 0][mb][i] + z, sum.o[hf * 4 + 1][mb][i] + z, sum.o[hf * 4 + 2][mb][i] + z, sum.o[hf * 4 + 3][mb][i] + z};
}

// A list's places, 64 steps at a time: lane i holds those of step i.
struct BtTable {
    uint32_t k0, k1, v0, v1;
    __device__ __forceinline__ void load(const BtArgs &a, int64_t at)
    {
        k0 = a.w.k_start[at];
        k1 = a.w.k_start[at + 1];
        v0 = a.w.v_start[at];
        v1 = a.w.v_start[at + 1];
    }
};
struct BtPlaces {
    uint32_t k0, k1, v0, v1;
    __device__ __forceinline__ BtPlaces(const BtTable &t, int i)
        : k0((uint32_t)__builtin_amdgcn_readlane((int)t.k0, i)), k1((uint32_t)__builtin_amdgcn_readlane((int)t.k1, i)),
          v0((uint32_t)__builtin_amdgcn_readlane((int)t.v0, i)), v1((uint32_t)__builtin_amdgcn_readlane((int)t.v1, i)) {}
};

// Second kernel, up to 32 queries: a workgroup takes `chunk` blocks of one cache for one KV head and 16 MB queries, each of its
// wavefronts every fourth block from the codes to the output.  WHICH = 0: the prefix, every sequence's queries; 1: a sequence's
// own tokens, its own queries.
template <int BITS, int MB, int WHICH>
struct BtAlone {
    static constexpr int PER_CU = MB == 1 ? 3 : 2;
    static constexpr int QBYTES = 8192 * MB, PATCHES = BT_WAVES * BT_PATCH;
    static_assert(QBYTES == 2 * MB * BT_NT * 16, "two pieces of a block's rows per thread");
    static_assert(16 * 128 * 4 == BT_PATCH, "the sums of 16 queries take a patch's place");
    struct Shared {
        __attribute__((aligned(16))) uint8_t area[PATCHES], qfrag[QBYTES];
        __attribute__((aligned(16))) float base[BT_WAVES][64];                      // angles at a block's first token
        BtConst<BITS> con;
        float wave_m[BT_WAVES][16 * MB], wave_l[BT_WAVES][16 * MB];
    };
    static __device__ void run(const BtArgs &a, int wg, Shared &sh);
};

template <int BITS, int MB, int WHICH>
__device__ __forceinline__ void BtAlone<BITS, MB, WHICH>::run(const BtArgs &a, int wg, Shared &sh)
{
    auto &area = sh.area;
    auto &qfrag = sh.qfrag;
    auto &con = sh.con;
    auto &base = sh.base;
    auto &wave_m = sh.wave_m;
    auto &wave_l = sh.wave_l;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const BtPart p = bt_part<WHICH>(a, wg, 16 * MB);
    const BtSeg sg = bt_seg(a.w.segs[p.si]);

    uint8_t *const patch = area + wave * BT_PATCH;
    const uint8_t *const k_plane = sg.k_codes + (int64_t)sg.cap * 16 * BITS * p.h, *const v_plane = sg.v_codes + (int64_t)sg.cap * 16 * BITS * p.h;
    const int64_t v_half = (int64_t)(sg.cap >> 1) * 16 * BITS;
    const BtLane<BITS> my(r16, g);

    // What a step reads is requested by the step before, as soon as the registers it lands in are free: codes of the Keys after
    // the scores, scales after the weights, codes of the Values after the output's products, a list's entries (one a lane; lists
    // of more go on from memory) after the patch has been zeroed.  (Eight queries, 131072 tokens, 32 heads: 381 -> 302 us.)
    const int steps = p.b1 - p.b0 > wave ? (p.b1 - p.b0 - wave + BT_WAVES - 1) / BT_WAVES : 0;
    const uint32_t *k_list = a.w.k_list + sg.k_list, *v_list = a.w.v_list + sg.v_list;
    uint32_t kw[2][BITS], ke = 0, ve = 0, sz[2][4];
    BtCodes<BITS> vc[2];
    BtTable tab = {0, 0, 0, 0};
    auto block_of = [&](int step) { return p.b0 + wave + BT_WAVES * (step < steps ? step : steps - 1); };
    auto place_of = [&](int step) { return (int64_t)(sg.blk0 + block_of(step)) * (a.heads + 1) + p.h; };
    auto load_keys = [&](int n0) {
        const uint8_t *kc = k_plane + (int64_t)(n0 >> 6) * (64 * 16 * BITS) + (n0 & 63) * 16;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int i = 0; i < BITS; ++i) kw[tb][i] = *(const uint32_t *)(kc + my.k_off[i] + tb * 256);
    };
    if (steps > 0) {
        const int n0 = block_of(0) * BT_BLOCK;
        tab.load(a, place_of(lane));
        load_keys(n0);
        bt_scales(sz, sg.v_sz, n0, g);
        vc[0].load(v_plane, n0, my);
        vc[1].load(v_plane + v_half, n0, my);
    }
    // Everything else the start reads, before anything of it is waited for; the lists' entries behind their places.
    const typename BtConst<BITS>::Brought brought = BtConst<BITS>::load(a, sg, p);
    uint4 rows[2 * MB];
#pragma unroll
    for (int k = 0; k < 2 * MB; ++k) {
        const int i = tid + k * BT_NT, l = i & 63, t = (i >> 6) & 3, part = (i >> 8) & 1, mb = i >> 9;
        const int row = (p.qb * MB + mb) * 16 + (l & 15);
        rows[k] = uint4{0u, 0u, 0u, 0u};
        if (row < p.n_q) rows[k] = *(const uint4 *)(a.w.rows[WHICH] + (p.row0 + row) * BT_ROW + part * 128 + (t * 4 + (l >> 4)) * 8);
    }
    const KvqParamsHeader *hdr = (const KvqParamsHeader *)sg.params;
    const float my_vh = hdr->rope_vh[lane], my_vl = hdr->rope_vl[lane];
    BtSums<MB> sum;
    sum.clear();
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = (p.qb * MB + mb) * 16 + r16;
        sum.inv[mb] = row < p.n_q ? a.w.row_scale[WHICH][p.row0 + row] : 0.0f;
    }
    BtPlaces at(tab, 0);
    if (at.k0 + lane < at.k1) ke = k_list[at.k0 + lane];
    if (at.v0 + lane < at.v1) ve = v_list[at.v0 + lane];
    for (int i = tid; i < PATCHES / 16; i += BT_NT) *(uint4 *)(area + i * 16) = uint4{0u, 0u, 0u, 0u};
    con.stage(a, sg, p, brought);
#pragma unroll
    for (int k = 0; k < 2 * MB; ++k) *(uint4 *)(qfrag + (tid + k * BT_NT) * 16) = rows[k];
    __syncthreads();
    const float kap = con.kappa();
    float minus_one = -1.0f, one = 1.0f;
    asm("" : "+v"(minus_one), "+v"(one));

    for (int step = 0; step < steps; ++step) {
        const int n0 = block_of(step) * BT_BLOCK, next = step + 1, n0_next = block_of(next) * BT_BLOCK;
        const bool edge = n0 < p.first || n0 + BT_BLOCK > p.n;
        if ((next & 63) == 0) tab.load(a, place_of(next + lane));
        const BtPlaces at_next(tab, next & 63);

        // ---- Keys: angles of this lane's pairs at the block's first token; residuals into the patch
        base[wave][lane] = rope_rev((float)n0, my_vh, my_vl);
        const uint32_t kp = bt_key_place(ke);
        if (at.k0 + lane < at.k1) *(uint16_t *)(patch + kp) = (uint16_t)(ke >> 16);
        for (uint32_t e = at.k0 + 64 + lane; e < at.k1; e += 64) {
            const uint32_t x = k_list[e];
            *(uint16_t *)(patch + bt_key_place(x)) = (uint16_t)(x >> 16);
        }
        bt_lds_order();
        float4_t sc[1][2][MB], (&s)[2][MB] = sc[0];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) s[tb][mb] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint4 sv = *(const uint4 *)&con.s[g * 16 + t * 4], zv = *(const uint4 *)&con.z[g * 16 + t * 4];
            const float4_t vh = *(const float4_t *)&con.vh[g * 16 + t * 4], ba = *(const float4_t *)&base[wave][g * 16 + t * 4];
            const uint32_t s4[4] = {sv.x, sv.y, sv.z, sv.w}, z4[4] = {zv.x, zv.y, zv.z, zv.w};
            half8_t hi[2], lo[2];
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                const uint4 rv = *(const uint4 *)(patch + ((tb * 4 + t) * 64 + lane) * 16);
                const uint32_t r4[4] = {rv.x, rv.y, rv.z, rv.w};
                uint32_t kh[4], kl[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    bt_key_pair<true>(con.lut_k[bt_key_field<BITS>(kw[tb], 4 * t + u)], s4[u], z4[u], r4[u],
                                      __builtin_fmaf((float)(tb * 16 + r16), vh[u], ba[u]), minus_one, one, kh[u], kl[u]);
                hi[tb] = bt_half8(kh[0], kh[1], kh[2], kh[3]);
                lo[tb] = bt_half8(kl[0], kl[1], kl[2], kl[3]);
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                const half8_t qh = *(const half8_t *)(qfrag + ((mb * 2 * 4 + t) * 64 + lane) * 16);
                const half8_t ql = *(const half8_t *)(qfrag + (((mb * 2 + 1) * 4 + t) * 64 + lane) * 16);
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) {
                    s[tb][mb] = bt_mfma(lo[tb], qh, s[tb][mb]);
                    s[tb][mb] = bt_mfma(hi[tb], ql, s[tb][mb]);
                    s[tb][mb] = bt_mfma(hi[tb], qh, s[tb][mb]);
                }
            }
        }
        load_keys(n0_next);
        // ---- the patch again zero, then the Values' residuals
        bt_lds_order();
        if (at.k0 + lane < at.k1) *(uint16_t *)(patch + kp) = 0;
        for (uint32_t e = at.k0 + 64 + lane; e < at.k1; e += 64) *(uint16_t *)(patch + bt_key_place(k_list[e])) = 0;
        if (at_next.k0 + lane < at_next.k1) ke = k_list[at_next.k0 + lane];
        bt_lds_order();
        const uint32_t vp = bt_value_place(ve);
        if (at.v0 + lane < at.v1) *(uint16_t *)(patch + vp) = (uint16_t)(ve >> 16);
        for (uint32_t e = at.v0 + 64 + lane; e < at.v1; e += 64) {
            const uint32_t x = v_list[e];
            *(uint16_t *)(patch + bt_value_place(x)) = (uint16_t)(x >> 16);
        }
        BtWeights w[MB];
        if (edge) bt_mask<MB>(s, sz, n0, p.first, p.n, g);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) bt_maximum<MB, 1>(sc, sum, mb);
        bt_weights<MB>(s, sz, sum, w, r16, kap, minus_one);
        bt_scales(sz, sg.v_sz, n0_next, g);
        bt_lds_order();
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            uint32_t f[4];
            vc[hf].align(f, my.v_shift);
#pragma unroll
            for (int sub = 0; sub < 4; ++sub)
                bt_products<MB>(bt_value_operand<BITS>(f, sub, con.lut_v), *(const half8_t *)(patch + ((hf * 4 + sub) * 64 + lane) * 16), w, sum, hf * 4 + sub);
        }
        vc[0].load(v_plane, n0_next, my);
        vc[1].load(v_plane + v_half, n0_next, my);
        bt_lds_order();
        if (at.v0 + lane < at.v1) *(uint16_t *)(patch + vp) = 0;
        for (uint32_t e = at.v0 + 64 + lane; e < at.v1; e += 64) *(uint16_t *)(patch + bt_value_place(v_list[e])) = 0;
        if (at_next.v0 + lane < at_next.v1) ve = v_list[at_next.v0 + lane];
        bt_lds_order();
        at = at_next;
    }

    // ---- the wavefronts' sums to one: each leaves a block of 16 queries where its patch was (pieces of four channels, in an order that
    // spreads the queries over the banks), then every thread adds the four
    if (g == 0)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            wave_m[wave][mb * 16 + r16] = sum.m[mb];
            wave_l[wave][mb * 16 + r16] = sum.lz[mb].y;
        }
    __syncthreads();
    const int64_t slot0 = ((int64_t)p.ch * a.heads + p.h) * a.mp[WHICH] + (int64_t)p.qb * 16 * MB;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int c = mb * 16 + r16;
        const float m = __builtin_fmaxf(__builtin_fmaxf(wave_m[0][c], wave_m[1][c]), __builtin_fmaxf(wave_m[2][c], wave_m[3][c]));
        const float fac = __builtin_amdgcn_exp2f(sum.m[mb] - m - kap), z = __shfl(sum.lz[mb].x, r16);
        if (mb > 0) __syncthreads();
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(float4_t *)(patch + (r16 * 32 + ((hf * 16 + g * 4 + i) ^ r16)) * 16) = bt_channels<MB>(sum, mb, hf, i, z) * fac;
        __syncthreads();
        for (int i = tid; i < 16 * 32; i += BT_NT) {
            const int row = i >> 5, c4 = i & 31;
            float4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < BT_WAVES; ++w) v += *(const float4_t *)(area + w * BT_PATCH + (row * 32 + (c4 ^ row)) * 16);
            if (p.qb * 16 * MB + mb * 16 + row < p.n_q) *(float4_t *)(a.w.part_o[WHICH] + (slot0 + mb * 16 + row) * 128 + c4 * 4) = v;
        }
    }
    if (tid < 16 * MB && p.qb * 16 * MB + tid < p.n_q) {
        float m = KVQ_STAT_FLOOR, l = 0.0f;
        for (int w = 0; w < BT_WAVES; ++w) m = __builtin_fmaxf(m, wave_m[w][tid]);
        for (int w = 0; w < BT_WAVES; ++w) l += wave_l[w][tid] * __builtin_amdgcn_exp2f(wave_m[w][tid] - m - kap);
        *(float2_t *)(a.w.part_ml[WHICH] + (slot0 + tid) * 2) = float2_t{m, l};
    }
}

// Second kernel, more than 32 queries: a workgroup takes them 32 QW at a time and `chunk` blocks, in tiles of 64 tokens.  Each
// wavefront rotates 16 tokens' Keys into LDS, in the operands' layout and in two parts; then it multiplies all 64 tokens (QW = 4), or 32 of
// them (QW = 2), with 32 queries that it keeps in registers.  De-quantising is shared by 64 or 128 queries, and while one workgroup of a
// compute unit does that (vector instructions) the other one's products keep the matrix cores busy.
// The Keys' residuals are added where the rotated pairs lie, by a lane per entry: entries of channels below 64 first, so that two of
// one pair never meet.
template <int BITS, int QW, int WHICH>
struct BtTogether {
    static constexpr int PER_CU = 2;
    static constexpr int MB = 2, TW = BT_WAVES / QW, GROUPS = 2 / TW;       // blocks of 32 tokens that a wavefront multiplies per tile
    static constexpr int OROW = 132, KEYS = 4 * 4 * 2 * 1024;
    static_assert(TW == 1 || QW * 32 * OROW * 4 <= KEYS + 4 * BT_PATCH, "the sums take the tiles' place");
    struct Shared {
        // [block of 16][step t][part][lane] Keys; [block of 32][channel block][lane] residuals; the same of signposts of the Values
        __attribute__((aligned(16))) uint8_t keys[KEYS + 4 * BT_PATCH];
        __attribute__((aligned(16))) float base[BT_WAVES][64];
        BtConst<BITS> con;
        float wave_m[BT_WAVES][16 * MB], wave_l[BT_WAVES][16 * MB];
    };
    static __device__ void run(const BtArgs &a, int wg, Shared &sh);
};

template <int BITS, int QW, int WHICH>
__device__ __forceinline__ void BtTogether<BITS, QW, WHICH>::run(const BtArgs &a, int wg, Shared &sh)
{
    auto &keys = sh.keys;
    auto &con = sh.con;
    auto &base = sh.base;
    auto &wave_m = sh.wave_m;
    auto &wave_l = sh.wave_l;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g = lane >> 4, qg = wave % QW, tg = wave / QW;
    const BtPart p = bt_part<WHICH>(a, wg, 32 * QW);
    const BtSeg sg = bt_seg(a.w.segs[p.si]);
    uint8_t *const patches = keys + KEYS, *const values = patches + 2 * BT_PATCH;

    const typename BtConst<BITS>::Brought brought = BtConst<BITS>::load(a, sg, p);
    const int q0 = (p.qb * QW + qg) * 32;
    half8_t qf[MB][4][2];
    BtSums<MB> sum;
    sum.clear();
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = q0 + mb * 16 + r16;
        const bool in = row < p.n_q;
        sum.inv[mb] = in ? a.w.row_scale[WHICH][p.row0 + row] : 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                uint4 v = {0u, 0u, 0u, 0u};
                if (in) v = *(const uint4 *)(a.w.rows[WHICH] + (p.row0 + row) * BT_ROW + part * 128 + (t * 4 + g) * 8);
                qf[mb][t][part] = __builtin_bit_cast(half8_t, v);
            }
    }
    const KvqParamsHeader *hdr = (const KvqParamsHeader *)sg.params;
    const float my_vh = hdr->rope_vh[lane], my_vl = hdr->rope_vl[lane];
    const uint8_t *const k_plane = sg.k_codes + (int64_t)sg.cap * 16 * BITS * p.h, *const v_plane = sg.v_codes + (int64_t)sg.cap * 16 * BITS * p.h;
    const int64_t v_half = (int64_t)(sg.cap >> 1) * 16 * BITS;
    const BtLane<BITS> my(r16, g);
    const uint32_t *k_list = a.w.k_list + sg.k_list, *v_list = a.w.v_list + sg.v_list;

    // Tiles of two blocks; the second one of the last may lie behind the tokens: it is read where the first is and has no weights.
    const int tiles = (p.b1 - p.b0 + 1) / 2;
    auto block_of = [&](int tile, int which) {
        const int b = p.b0 + 2 * (tile < tiles ? tile : tiles - 1) + which;
        return b < p.b1 ? b : p.b1 - 1;
    };
    const int mine = wave >> 1, half = wave & 1;                 // the block this wavefront rotates, and which half of it
    auto place_of = [&](int tile) { return (int64_t)(sg.blk0 + block_of(tile, mine)) * (a.heads + 1) + p.h; };
    uint32_t kw[BITS], ke = 0, ve = 0;
    auto load_keys = [&](int tile) {
        const int n0 = block_of(tile, mine) * BT_BLOCK + half * 16;
        const uint8_t *kc = k_plane + (int64_t)(n0 >> 6) * (64 * 16 * BITS) + (n0 & 63) * 16;
#pragma unroll
        for (int i = 0; i < BITS; ++i) kw[i] = *(const uint32_t *)(kc + my.k_off[i]);
    };
    BtTable tab;
    tab.load(a, place_of(lane));
    BtPlaces at(tab, 0);
    BtCodes<BITS> vc[2];                                         // of both blocks, the half of the channels that has this wavefront's two blocks
    load_keys(0);
    const uint8_t *const my_half = v_plane + (wave >> 1) * v_half;
#pragma unroll
    for (int gr = 0; gr < 2; ++gr) vc[gr].load(my_half, block_of(0, gr) * BT_BLOCK, my);
    if (at.k0 + lane < at.k1) ke = k_list[at.k0 + lane];
    if (at.v0 + lane < at.v1) ve = v_list[at.v0 + lane];
    for (int i = tid; i < 2 * BT_PATCH / 16; i += BT_NT) *(uint4 *)(patches + i * 16) = uint4{0u, 0u, 0u, 0u};
    con.stage(a, sg, p, brought);
    __syncthreads();
    const float kap = con.kappa();
    float minus_one = -1.0f;
    asm("" : "+v"(minus_one));
    uint8_t *const my_keys = keys + wave * 8192;
    uint8_t *const my_patch = patches + mine * BT_PATCH;

    for (int tile = 0; tile < tiles; ++tile) {
        const int next = tile + 1;
        if ((next & 63) == 0) tab.load(a, place_of(next + lane));
        const BtPlaces at_next(tab, next & 63);
        // ---- this wavefront's 16 tokens
        {
            const int n0 = block_of(tile, mine) * BT_BLOCK + half * 16;
            base[wave][lane] = rope_rev((float)n0, my_vh, my_vl);
            bt_lds_order();
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint4 sv = *(const uint4 *)&con.s[g * 16 + t * 4], zv = *(const uint4 *)&con.z[g * 16 + t * 4];
                const float4_t vh = *(const float4_t *)&con.vh[g * 16 + t * 4], ba = *(const float4_t *)&base[wave][g * 16 + t * 4];
                const uint32_t s4[4] = {sv.x, sv.y, sv.z, sv.w}, z4[4] = {zv.x, zv.y, zv.z, zv.w};
                uint32_t kh[4], kl[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    bt_key_pair<false>(con.lut_k[bt_key_field<BITS>(kw, 4 * t + u)], s4[u], z4[u], 0u, __builtin_fmaf((float)r16, vh[u], ba[u]),
                                       minus_one, 0.f, kh[u], kl[u]);
                *(uint4 *)(my_keys + (t * 2 * 64 + lane) * 16) = uint4{kh[0], kh[1], kh[2], kh[3]};
                *(uint4 *)(my_keys + ((t * 2 + 1) * 64 + lane) * 16) = uint4{kl[0], kl[1], kl[2], kl[3]};
            }
            bt_lds_order();
            auto add_residual = [&](uint32_t x, bool upper) {
                const uint32_t t = (x >> 7) & 31u, c = x & 127u, pr = c & 63u;
                if ((int)(t >> 4) != half || (c >= 64u) != upper) return;
                uint8_t *at_hi = my_keys + ((((pr >> 2) & 3) * 2 * 64 + (pr >> 4) * 16 + (t & 15)) * 4 + (pr & 3)) * 4;
                const half2_t h2 = *(const half2_t *)at_hi, l2 = *(const half2_t *)(at_hi + 1024);
                const float r = kvq_h2f((uint16_t)(x >> 16)), rev = __builtin_fmaf((float)(t & 15), con.vh[pr], base[wave][pr]);
                const float c1 = __builtin_amdgcn_cosf(rev), s1 = __builtin_amdgcn_sinf(rev);
                const float k0 = (float)h2.x + (float)l2.x, k1 = (float)h2.y + (float)l2.y;
                uint32_t hi, lo;
                bt_split(__builtin_fmaf(r, upper ? -s1 : c1, k0), __builtin_fmaf(r, upper ? c1 : s1, k1), minus_one, hi, lo);
                *(uint32_t *)at_hi = hi;
                *(uint32_t *)(at_hi + 1024) = lo;
            };
#pragma unroll
            for (int upper = 0; upper < 2; ++upper) {
                if (at.k0 + lane < at.k1) add_residual(ke, upper != 0);
                for (uint32_t e = at.k0 + 64 + lane; e < at.k1; e += 64) add_residual(k_list[e], upper != 0);
                bt_lds_order();
            }
        }
        load_keys(next);
        if (at_next.k0 + lane < at_next.k1) ke = k_list[at_next.k0 + lane];
        // ---- Values: signposts of two blocks of channels for all 64 tokens; residuals of this wavefront's 16
        uint32_t sz[GROUPS][2][4];
#pragma unroll
        for (int gr = 0; gr < GROUPS; ++gr) bt_scales(sz[gr], sg.v_sz, block_of(tile, TW == 1 ? gr : tg) * BT_BLOCK, g);
#pragma unroll
        for (int gr = 0; gr < 2; ++gr) {
            uint32_t f[4];
            vc[gr].align(f, my.v_shift);
            if (wave & 1)
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] >>= 4 * BITS;       // its two blocks are the half's third and fourth
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
                *(half8_t *)(values + ((gr * 8 + 2 * wave + sub) * 64 + lane) * 16) = bt_value_operand<BITS>(f, sub, con.lut_v);
        }
        // (requested ahead of the products where there are registers for it: with 128 queries there are not)
        if (TW == 2)
#pragma unroll
            for (int gr = 0; gr < 2; ++gr) vc[gr].load(my_half, block_of(next, gr) * BT_BLOCK, my);
        const uint32_t vp = bt_value_place(ve);
        const bool v_mine = at.v0 + lane < at.v1 && (int)((ve >> 11) & 1u) == half;
        if (v_mine) *(uint16_t *)(my_patch + vp) = (uint16_t)(ve >> 16);
        for (uint32_t e = at.v0 + 64 + lane; e < at.v1; e += 64) {
            const uint32_t x = v_list[e];
            if ((int)((x >> 11) & 1u) == half) *(uint16_t *)(my_patch + bt_value_place(x)) = (uint16_t)(x >> 16);
        }
        __syncthreads();
        // ---- products with this wavefront's queries: all scores, their maximum, then weights and output without a branch
        float4_t s[GROUPS][2][MB];
#pragma unroll
        for (int gr = 0; gr < GROUPS; ++gr) {
            const int grp = TW == 1 ? gr : tg;
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) s[gr][tb][mb] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                half8_t hi[2], lo[2];
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) {
                    const uint8_t *k = keys + (((grp * 2 + tb) * 4 + t) * 2 * 64 + lane) * 16;
                    hi[tb] = *(const half8_t *)k;
                    lo[tb] = *(const half8_t *)(k + 1024);
                }
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) s[gr][tb][mb] = bt_mfma(lo[tb], qf[mb][t][0], s[gr][tb][mb]);
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) s[gr][tb][mb] = bt_mfma(hi[tb], qf[mb][t][1], s[gr][tb][mb]);
#pragma unroll
                for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) s[gr][tb][mb] = bt_mfma(hi[tb], qf[mb][t][0], s[gr][tb][mb]);
            }
        }
#pragma unroll
        for (int gr = 0; gr < GROUPS; ++gr) {
            const int blk = p.b0 + 2 * tile + (TW == 1 ? gr : tg), n0 = blk * BT_BLOCK;
            if (n0 < p.first || n0 + BT_BLOCK > p.n || blk >= p.b1) bt_mask<MB>(s[gr], sz[gr], n0, p.first, blk >= p.b1 ? 0 : p.n, g);
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) bt_maximum<MB, GROUPS>(s, sum, mb);
#pragma unroll
        for (int gr = 0; gr < GROUPS; ++gr) {
            const int grp = TW == 1 ? gr : tg;
            BtWeights w[MB];
            bt_weights<MB>(s[gr], sz[gr], sum, w, r16, kap, minus_one);
#pragma unroll
            for (int cb = 0; cb < 8; ++cb)
                bt_products<MB>(*(const half8_t *)(values + ((grp * 8 + cb) * 64 + lane) * 16), *(const half8_t *)(patches + ((grp * 8 + cb) * 64 + lane) * 16),
                                w, sum, cb);
        }
        if (TW == 1)
#pragma unroll
            for (int gr = 0; gr < 2; ++gr) vc[gr].load(my_half, block_of(next, gr) * BT_BLOCK, my);
        __syncthreads();
        if (v_mine) *(uint16_t *)(my_patch + vp) = 0;
        for (uint32_t e = at.v0 + 64 + lane; e < at.v1; e += 64) {
            const uint32_t x = v_list[e];
            if ((int)((x >> 11) & 1u) == half) *(uint16_t *)(my_patch + bt_value_place(x)) = 0;
        }
        if (at_next.v0 + lane < at_next.v1) ve = v_list[at_next.v0 + lane];
        at = at_next;
    }

    // ---- sums to memory; with two wavefronts per query the second's go through LDS
    const int64_t slot0 = ((int64_t)p.ch * a.heads + p.h) * a.mp[WHICH];
    if (TW == 2) {
        __syncthreads();
        if (g == 0)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                wave_m[wave][mb * 16 + r16] = sum.m[mb];
                wave_l[wave][mb * 16 + r16] = sum.lz[mb].y;
            }
        __syncthreads();
    }
    float *sums = (float *)keys + qg * 32 * OROW;
#pragma unroll
    for (int turn = 0; turn < TW; ++turn) {
        // the second wavefront first, then the first adds its own and writes
        if (TW == 1 || tg == 1 - turn) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                const int c = mb * 16 + r16;
                float m = sum.m[mb], l = sum.lz[mb].y;
                if (TW == 2) {
                    m = __builtin_fmaxf(wave_m[qg][c], wave_m[(QW + qg) % BT_WAVES][c]);
                    l = wave_l[qg][c] * __builtin_amdgcn_exp2f(wave_m[qg][c] - m) +
                        wave_l[(QW + qg) % BT_WAVES][c] * __builtin_amdgcn_exp2f(wave_m[(QW + qg) % BT_WAVES][c] - m);
                }
                const float fac = __builtin_amdgcn_exp2f(sum.m[mb] - m - kap), z = __shfl(sum.lz[mb].x, r16);
                const bool in = q0 + c < p.n_q;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int ch = hf * 64 + g * 16 + i * 4;
                        float4_t v = bt_channels<MB>(sum, mb, hf, i, z) * fac;
                        float4_t *q = (float4_t *)(sums + c * OROW + ch);
                        if (TW == 2 && turn == 0) *q = v;
                        else {
                            if (TW == 2) v += *q;
                            if (in) *(float4_t *)(a.w.part_o[WHICH] + (slot0 + q0 + c) * 128 + ch) = v;
                        }
                    }
                if ((TW == 1 || turn == 1) && g == 0 && in)
                    *(float2_t *)(a.w.part_ml[WHICH] + (slot0 + q0 + c) * 2) = float2_t{m, l * __builtin_amdgcn_exp2f(-kap)};
            }
        }
        if (TW == 2) __syncthreads();
    }
}

// The launch: the prefix's workgroups (queries in blocks of 16 MBP), then those of the sequences' own tokens (MBO); 0: none of the kind.
struct BtNone {
    static constexpr int PER_CU = 3;
    struct Shared {
        int none;
    };
    static __device__ __forceinline__ void run(const BtArgs &, int, Shared &) {}
};
template <int BITS, int MB, int WHICH>
struct BtFormOf {
    typedef std::conditional_t<(MB <= 2), BtAlone<BITS, (MB == 2 ? 2 : 1), WHICH>, BtTogether<BITS, (MB >= 4 ? MB / 2 : 2), WHICH>> some;
    typedef std::conditional_t<MB == 0, BtNone, some> type;
};
constexpr int bt_per_cu(int mbp, int mbo) { return mbp <= 1 && mbo <= 1 ? 3 : 2; }

template <int BITS, int MBP, int MBO>
__global__ __launch_bounds__(BT_NT, bt_per_cu(MBP, MBO)) void kvq_batch_attend(BtArgs a, int prefix_wgs)
{
    typedef typename BtFormOf<BITS, MBP, 0>::type P;
    typedef typename BtFormOf<BITS, MBO, 1>::type O;
    __shared__ __attribute__((aligned(16))) uint8_t mem[sizeof(typename P::Shared) > sizeof(typename O::Shared) ? sizeof(typename P::Shared) : sizeof(typename O::Shared)];
    if (MBO == 0 || (MBP > 0 && (int)blockIdx.x < prefix_wgs)) P::run(a, blockIdx.x, *(typename P::Shared *)mem);
    else O::run(a, (int)blockIdx.x - prefix_wgs, *(typename O::Shared *)mem);
}

// Third kernel: a workgroup per (sequence, query head) joins the workgroups' sums and the attention-sink tokens.  Eight slices of
// 32 threads take every eighth sum, four channels a thread.
__global__ __launch_bounds__(256) void kvq_batch_join(BtArgs a)
{
    __shared__ float sink_x[2 * KVQ_MAX_SINK], red[4];
    __shared__ __attribute__((aligned(16))) float sum[8][128], weight[8];
    const int tid = threadIdx.x, hq = a.heads * a.ratio, b = blockIdx.x / hq, qh = blockIdx.x % hq;
    const int h = qh / a.ratio, r = qh % a.ratio, c4 = (tid & 31) * 4, slice = tid >> 5;
    const int64_t q0 = (int64_t)blockIdx.x * 128;
    const int n_pre = a.n_chunks[0];
    const int c_own = a.own ? a.w.segs[1 + b].chunk0 : 0;
    const int n_own = a.own ? (a.w.segs[1 + b].n + a.chunk[1] * BT_BLOCK - 1) / (a.chunk[1] * BT_BLOCK) : 0;
    const int64_t at_pre = (int64_t)h * a.mp[0] + b * a.ratio + r, step_pre = (int64_t)a.heads * a.mp[0];
    const int64_t at_own = ((int64_t)c_own * a.heads + h) * a.mp[1] + r, step_own = (int64_t)a.heads * a.mp[1];
    const int n = n_pre + n_own;
    auto which = [&](int i) { return i < n_pre ? 0 : 1; };
    auto slot = [&](int i) { return i < n_pre ? at_pre + i * step_pre : at_own + (int64_t)(i - n_pre) * step_own; };
    float m = KVQ_STAT_FLOOR;
    for (int i = tid; i < n; i += 256) m = __builtin_fmaxf(m, a.w.part_ml[which(i)][slot(i) * 2]);
    // sink tokens: scores from their fp16 rows
    int n_sink[2];
    for (int k = 0; k < 2; ++k) {
        const BtSeg sg = bt_seg(a.w.segs[k == 0 ? 0 : 1 + b]);
        n_sink[k] = sg.n_sink < sg.n ? sg.n_sink : sg.n;
        for (int j = 0; j < n_sink[k]; ++j)
            if (tid < 64) {
                const KvqParamsHeader *hdr = (const KvqParamsHeader *)sg.params;
                double rev = (double)(j + (k == 0 ? 0 : a.prefix)) * ((double)hdr->rope_vh[tid] + (double)hdr->rope_vl[tid]);
                rev -= floor(rev);
                float c, s;
                sincospif(2.0f * (float)rev, &s, &c);
                const uint16_t *row = sg.sink_k + (int64_t)j * a.heads * 128 + h * 128;
                const float ka = kvq_h2f(row[tid]), kb = kvq_h2f(row[tid + 64]);
                float x = a.q[q0 + tid] * (ka * c - kb * s) + a.q[q0 + 64 + tid] * (kb * c + ka * s);
                for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
                x *= a.scale * KVQ_LOG2E;
                if (tid == 0) sink_x[k * KVQ_MAX_SINK + j] = x;
                m = __builtin_fmaxf(m, x);
            }
    }
    m = kvq_wave_max(m);
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
    m = __builtin_fmaxf(__builtin_fmaxf(red[0], red[1]), __builtin_fmaxf(red[2], red[3]));
    float l = 0.0f;
    float4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = slice; i < n; i += 8) {
        const int64_t at = slot(i);
        const float2_t ml = *(const float2_t *)(a.w.part_ml[which(i)] + at * 2);
        const float f = __builtin_amdgcn_exp2f(ml.x - m);
        l = __builtin_fmaf(ml.y, f, l);
        acc += *(const float4_t *)(a.w.part_o[which(i)] + at * 128 + c4) * f;
    }
    if (slice == 0)
        for (int k = 0; k < 2; ++k) {
            const BtSeg sg = bt_seg(a.w.segs[k == 0 ? 0 : 1 + b]);
            for (int j = 0; j < n_sink[k]; ++j) {
                const float f = __builtin_amdgcn_exp2f(sink_x[k * KVQ_MAX_SINK + j] - m);
                const uint16_t *row = sg.sink_v + (int64_t)j * a.heads * 128 + h * 128 + c4;
                l += f;
                for (int i = 0; i < 4; ++i) acc[i] = __builtin_fmaf(kvq_h2f(row[i]), f, acc[i]);
            }
        }
    *(float4_t *)&sum[slice][c4] = acc;
    if (c4 == 0) weight[slice] = l;
    __syncthreads();
    if (tid < 128) {
        float o = 0.0f, w = 0.0f;
        for (int i = 0; i < 8; ++i) {
            o += sum[i][tid];
            w += weight[i];
        }
        a.out[q0 + tid] = w == 0.0f ? 0.0f : o / w;          // (a NaN stays one)
    }
}

// ---- host ---------------------------------------------------------------------------------------------------

struct BtPlan {
    BtArgs a;
    int64_t bytes;
    int mb[2];
    int64_t blocks;
};

int64_t bt_up(int64_t n) { return (n + 255) & ~(int64_t)255; }

// Blocks of 16 queries that a workgroup takes: one or two, each of its wavefronts alone; four or eight, together.  (A sequence's own
// queries rarely fill more than one: two and eight have no form of their own there.)
int bt_mb_prefix(int64_t queries) { return queries <= 16 ? 1 : queries <= 32 ? 2 : queries <= 64 ? 4 : 8; }
int bt_mb_own(int64_t queries) { return queries <= 16 ? 1 : 4; }

// The tokens of a call and the places of everything in the workspace (from `base`, which may be null).
kvq_status bt_plan(const kvq_cache *prefix, const kvq_cache *const *caches, int32_t n_seqs, char *base, BtPlan &p)
{
    memset(&p, 0, sizeof p);
    const kvq_cache *one = prefix;
    if (n_seqs < 1 || n_seqs > (1 << 20)) return KVQ_ERR_INVALID_ARG;
    int64_t own_blocks = 0, own_seqs = 0, k_entries = 0, v_entries = 0;
    auto add = [&](const kvq_cache *c, int64_t &blocks) -> kvq_status {
        const kvq_status st = kvq_check_cache(c);
        if (st != KVQ_OK) return st;
        if (!one) one = c;
        if (!c->loaded) return KVQ_ERR_NOT_LOADED;
        if (c->n_tokens_k != c->n_tokens_v) return KVQ_ERR_INVALID_ARG;
        if (c->bits != one->bits || c->n_kv_heads != one->n_kv_heads || c->n_q_heads != one->n_q_heads || c->rope_base != one->rope_base)
            return KVQ_ERR_INVALID_ARG;
        const int64_t n = c->n_tokens_k, most = n * c->n_kv_heads * KVQ_HEAD_DIM;
        blocks += (n + BT_BLOCK - 1) / BT_BLOCK;
        k_entries += c->cap_nnz_k < most ? c->cap_nnz_k : most;
        v_entries += c->cap_nnz_v < most ? c->cap_nnz_v : most;
        return KVQ_OK;
    };
    int64_t pre_blocks = 0;
    if (prefix) {
        const kvq_status st = add(prefix, pre_blocks);
        if (st != KVQ_OK) return st;
    }
    for (int32_t b = 0; caches && b < n_seqs; ++b)
        if (caches[b]) {
            const kvq_status st = add(caches[b], own_blocks);
            if (st != KVQ_OK) return st;
            own_seqs += caches[b]->n_tokens_k > 0;
        }
    if (!one) return KVQ_ERR_INVALID_ARG;
    BtArgs &a = p.a;
    a.n_seqs = n_seqs;
    a.heads = one->n_kv_heads;
    a.ratio = one->n_q_heads / one->n_kv_heads;
    a.prefix = prefix ? (int32_t)prefix->n_tokens_k : 0;
    a.own = own_blocks > 0;
    p.blocks = pre_blocks + own_blocks;
    if (p.blocks * (a.heads + 1) >= ((int64_t)1 << 40) || (int64_t)n_seqs * one->n_q_heads >= ((int64_t)1 << 28)) return KVQ_ERR_UNSUPPORTED;
    const int64_t m[2] = {(int64_t)n_seqs * a.ratio, a.ratio};
    const int64_t blocks[2] = {pre_blocks, own_blocks}, used[2] = {1, own_seqs};
    for (int k = 0; k < 2; ++k) {
        p.mb[k] = blocks[k] == 0 ? 0 : k == 0 ? bt_mb_prefix(m[k]) : bt_mb_own(m[k]);
        const int q = 16 * (p.mb[k] ? p.mb[k] : 1);
        a.mp[k] = (int32_t)((m[k] + q - 1) / q * q);
    }
    // Workgroups: none with less than a block per wavefront.  A prefix is cut into as many as the chip holds at once.  Sequences are
    // not cut together and their last pieces are short, so without a prefix there are three times as many, dealt out as places
    // fall free (8 heads, 48 sequences of up to 9000 tokens: 219 us in one round, 182 in two, 177 in three, 181 in four; 48 of 4500
    // tokens each: 160, 156, 160, 177).  Behind a prefix the sequences' own workgroups are many and short: they are cut fine and get
    // the places that their work, start included, would keep busy meanwhile.
    auto pieces = [&](int k, int64_t c) {
        if (k == 0) return (pre_blocks + c - 1) / c;
        int64_t sum = 0;
        for (int32_t b = 0; caches && b < n_seqs; ++b)
            if (caches[b]) sum += ((caches[b]->n_tokens_k + BT_BLOCK - 1) / BT_BLOCK + c - 1) / c;
        return sum;
    };
    auto fit = [&](int k, int64_t slots) {                   // blocks per workgroup for so many workgroups per head and query block
        int64_t chunk = slots > 0 ? (blocks[k] + slots - 1) / slots : blocks[k];
        chunk = chunk < BT_WAVES ? BT_WAVES : (chunk + BT_WAVES - 1) / BT_WAVES * BT_WAVES;
        if (k == 0 || used[k] >= slots) return chunk;
        for (int64_t c = chunk; c < 2 * chunk; c += (c / 16 / BT_WAVES + 1) * BT_WAVES)
            if (pieces(k, c) <= slots) return c;
        return chunk;
    };
    const int64_t places = (int64_t)kvq_cu_count() * bt_per_cu(p.mb[0], p.mb[1]);
    const int64_t wide[2] = {(int64_t)a.heads * (a.mp[0] / (16 * (p.mb[0] ? p.mb[0] : 1))), (int64_t)a.heads * (a.mp[1] / (16 * (p.mb[1] ? p.mb[1] : 1)))};
    int64_t own_places = p.mb[0] ? 0 : places;
    a.chunk[0] = a.chunk[1] = BT_WAVES;
    if (p.mb[0] == 8 && p.mb[1]) {                           // two launches (bt_launch_bits)
        a.chunk[0] = (int32_t)fit(0, (int64_t)kvq_cu_count() * bt_per_cu(8, 0) / wide[0]);
        a.chunk[1] = (int32_t)fit(1, BT_OWN_ROUNDS * kvq_cu_count() * bt_per_cu(0, p.mb[1]) / wide[1]);
    } else if (p.mb[0] && p.mb[1]) {
        // in steps of a block and wavefront: a workgroup's start and end are worth three, a block for 64 or 128 queries three
        const int64_t cost = p.mb[0] == 4 ? 3 : 1;
        for (int i = 0; i < 4; ++i) {
            int64_t left = (places - own_places) / wide[0];
            if (left < 1) left = 1;
            a.chunk[0] = (int32_t)fit(0, left);
            a.chunk[1] = (int32_t)fit(1, own_places > 0 ? 2 * own_places / wide[1] + 1 : 1);
            const int64_t last = a.chunk[0] / BT_WAVES * cost + 3, each = a.chunk[1] / BT_WAVES + 3;
            if (each > last / 2 + 3) a.chunk[1] = (int32_t)((last / 2 > 1 ? last / 2 : 1) * BT_WAVES);
            own_places = (pieces(1, a.chunk[1]) * wide[1] * (a.chunk[1] / BT_WAVES + 3) + last - 1) / last;
            if (own_places > places / 2) own_places = places / 2;
        }
        a.chunk[0] = (int32_t)fit(0, (places - own_places) / wide[0] > 0 ? (places - own_places) / wide[0] : 1);
    } else if (p.mb[0]) {
        a.chunk[0] = (int32_t)fit(0, places / wide[0]);
    } else if (p.mb[1]) {
        a.chunk[1] = (int32_t)fit(1, BT_OWN_ROUNDS * places / wide[1]);
    }
    const int64_t n_chunks[2] = {pieces(0, a.chunk[0]), pieces(1, a.chunk[1])};
    a.n_chunks[0] = (int32_t)n_chunks[0];
    const int64_t own_chunks = n_chunks[1];
    if (own_chunks >= (1 << 24) || n_chunks[0] * wide[0] + own_chunks * wide[1] >= ((int64_t)1 << 31)) return KVQ_ERR_UNSUPPORTED;
    a.n_chunks[1] = (int32_t)own_chunks;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        char *q = base + at;
        at += bt_up(bytes);
        return q;
    };
    BtWork &w = a.w;
    w.segs = (BtSeg *)take((int64_t)sizeof(BtSeg) * (1 + n_seqs));
    w.k_start = (uint32_t *)take(4 * p.blocks * (a.heads + 1));
    w.v_start = (uint32_t *)take(4 * p.blocks * (a.heads + 1));
    w.smax = (float *)take(4 * p.blocks);
    w.owner = (int32_t *)take(4 * own_chunks);
    const int64_t rows = (int64_t)n_seqs * one->n_q_heads;
    for (int k = 0; k < 2; ++k) {
        const int64_t here = blocks[k] > 0 ? rows : 0;
        w.rows[k] = (_Float16 *)take(here * BT_ROW * 2);
        w.row_scale[k] = (float *)take(here * 4);
        const int64_t slots = (int64_t)a.n_chunks[k] * a.heads * a.mp[k];
        w.part_o[k] = (float *)take(slots * 512);
        w.part_ml[k] = (float *)take(slots * 8);
    }
    w.k_list = (uint32_t *)take(4 * k_entries);
    w.v_list = (uint32_t *)take(4 * v_entries);
    p.bytes = at > 256 ? at : 256;
    return KVQ_OK;
}

template <int BITS, int MBP>
kvq_status bt_launch_own(const BtArgs &a, int mbo, int64_t prefix_wgs, int64_t wgs, hipStream_t s)
{
    const dim3 grid((unsigned)wgs), block(BT_NT);
    if constexpr (MBP == 8) kvq_batch_attend<BITS, 8, 0><<<grid, block, 0, s>>>(a, (int)prefix_wgs);
    else if (mbo == 1) kvq_batch_attend<BITS, MBP, 1><<<grid, block, 0, s>>>(a, (int)prefix_wgs);
    else if (mbo == 4) kvq_batch_attend<BITS, MBP, 4><<<grid, block, 0, s>>>(a, (int)prefix_wgs);
    else if constexpr (MBP > 0) kvq_batch_attend<BITS, MBP, 0><<<grid, block, 0, s>>>(a, (int)prefix_wgs);
    KVQ_HIP_CHECK(hipGetLastError());
    return KVQ_OK;
}

template <int BITS>
kvq_status bt_launch_bits(const BtPlan &p, hipStream_t s)
{
    const BtArgs &a = p.a;
    int64_t wgs[2];
    for (int k = 0; k < 2; ++k) wgs[k] = p.mb[k] ? (int64_t)a.n_chunks[k] * a.heads * (a.mp[k] / (16 * p.mb[k])) : 0;
    const int64_t all = wgs[0] + wgs[1];
    if (all == 0) return KVQ_OK;
    if (p.mb[0] == 8) {
        // The form for 128 queries has no register to spare: beside another form in one kernel it spills more, and its launches are long
        // enough to stand alone (32 sequences of 32 heads on 8 behind 524287 tokens: 1212 us in one launch, 1087 in two).
        const kvq_status st = bt_launch_own<BITS, 8>(a, 0, wgs[0], wgs[0], s);
        return st != KVQ_OK || wgs[1] == 0 ? st : bt_launch_own<BITS, 0>(a, p.mb[1], 0, wgs[1], s);
    }
    switch (p.mb[0]) {
    case 0: return bt_launch_own<BITS, 0>(a, p.mb[1], 0, all, s);
    case 1: return bt_launch_own<BITS, 1>(a, p.mb[1], wgs[0], all, s);
    case 2: return bt_launch_own<BITS, 2>(a, p.mb[1], wgs[0], all, s);
    default: return bt_launch_own<BITS, 4>(a, p.mb[1], wgs[0], all, s);
    }
}

kvq_status bt_launch(const BtPlan &p, int bits, hipStream_t s)
{
    return bits == 2 ? bt_launch_bits<2>(p, s) : bits == 3 ? bt_launch_bits<3>(p, s) : bt_launch_bits<4>(p, s);
}

}  // namespace

extern "C" int64_t kvq_attention_decode_batch_workspace_bytes(const kvq_cache *prefix, const kvq_cache *const *caches, int32_t n_seqs)
{
    BtPlan p;
    return bt_plan(prefix, caches, n_seqs, nullptr, p) == KVQ_OK ? p.bytes : 0;
}

extern "C" kvq_status kvq_attention_decode_batch(const kvq_cache *prefix, const kvq_cache *const *caches, int32_t n_seqs,
                                                 const float *d_q_rot, float scale, float *d_out, void *d_workspace,
                                                 int64_t workspace_bytes, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    BtPlan p;
    kvq_status st = bt_plan(prefix, caches, n_seqs, (char *)d_workspace, p);
    if (st != KVQ_OK) return st;
    if (!d_q_rot || !d_out || ((uintptr_t)d_q_rot & 3) || ((uintptr_t)d_out & 3)) return KVQ_ERR_INVALID_ARG;
    if (!d_workspace || ((uintptr_t)d_workspace & 15)) return KVQ_ERR_INVALID_ARG;
    if (workspace_bytes < p.bytes) return KVQ_ERR_CAPACITY;
    BtArgs &a = p.a;
    a.q = d_q_rot;
    a.out = d_out;
    a.scale = scale;
    const kvq_cache *one = prefix;
    for (int32_t b = 0; caches && !one && b < n_seqs; ++b) one = caches[b];

    // ---- descriptors, BT_SEGS at a time in the arguments of the first kernel
    BtSegs part;
    int64_t k_list = 0, v_list = 0, blk = 0, chunk = 0, wgs = 0;
    const int sort = one->n_kv_heads <= BT_FEW_HEADS ? BT_SORT_FEW : BT_SORT;
    memset(&part, 0, sizeof part);
    for (int32_t i = 0; i <= n_seqs; ++i) {
        const kvq_cache *c = i == 0 ? prefix : caches ? caches[i - 1] : nullptr;
        BtSeg &g = part.seg[part.n];
        memset(&g, 0, sizeof g);
        g.params = one->params;
        g.blk0 = (int32_t)blk;
        g.chunk0 = (int32_t)chunk;
        g.wg0 = (int32_t)wgs;
        g.k_list = k_list;
        g.v_list = v_list;
        if (c && c->n_tokens_k > 0) {
            g.k_codes = c->k_codes;
            g.v_codes = c->v_codes;
            g.v_sz = (const uint32_t *)c->v_sz;
            g.k_ptr = c->k_ptr;
            g.v_ptr = c->v_ptr;
            g.shift = c->nnz_block_shift;
            g.k_idx = g.shift ? (const void *)c->k_idx_blocks : c->k_idx;
            g.k_val = g.shift ? (const void *)c->k_val_blocks : c->k_val;
            g.v_idx = g.shift ? (const void *)c->v_idx_blocks : c->v_idx;
            g.v_val = g.shift ? (const void *)c->v_val_blocks : c->v_val;
            g.params = c->params;
            g.sink_k = c->sink_k;
            g.sink_v = c->sink_v;
            g.n = (int32_t)c->n_tokens_k;
            g.cap = (int32_t)c->cap_tokens;
            g.n_sink = c->n_sink;
            const int64_t most = c->n_tokens_k * c->n_kv_heads * KVQ_HEAD_DIM;
            const int64_t kr = c->cap_nnz_k < most ? c->cap_nnz_k : most, vr = c->cap_nnz_v < most ? c->cap_nnz_v : most;
            g.k_room = (uint32_t)(kr > 0xFFFFFFFFll ? 0xFFFFFFFFll : kr);
            g.v_room = (uint32_t)(vr > 0xFFFFFFFFll ? 0xFFFFFFFFll : vr);
            k_list += kr;
            v_list += vr;
            const int64_t nb = (c->n_tokens_k + BT_BLOCK - 1) / BT_BLOCK;
            blk += nb;
            wgs += (nb + sort - 1) / sort;
            if (i > 0) chunk += (nb + a.chunk[1] - 1) / a.chunk[1];
        }
        if (++part.n < BT_SEGS && i < n_seqs) continue;
        if (n_seqs + 1 > BT_SEGS) {
            kvq_batch_upload<<<dim3(1), dim3(BT_NT), 0, s>>>(a, part);
            KVQ_HIP_CHECK(hipGetLastError());
        }
        if (i < n_seqs) {
            part.first += part.n;
            part.n = 0;
        }
    }
    const int64_t row_wgs = ((int64_t)n_seqs * one->n_q_heads + BT_WAVES - 1) / BT_WAVES;
    if (row_wgs + 2 * wgs >= ((int64_t)1 << 31)) return KVQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)(row_wgs + 2 * wgs)), block(BT_NT);
    if (sort == BT_SORT) kvq_batch_prepare<BT_SORT, BT_HELD><<<grid, block, 0, s>>>(a, part, (int)row_wgs, n_seqs + 1);
    else kvq_batch_prepare<BT_SORT_FEW, BT_HELD_FEW><<<grid, block, 0, s>>>(a, part, (int)row_wgs, n_seqs + 1);
    KVQ_HIP_CHECK(hipGetLastError());
    st = bt_launch(p, one->bits, s);
    if (st != KVQ_OK) return st;
    kvq_batch_join<<<dim3((unsigned)(n_seqs * one->n_q_heads)), dim3(256), 0, s>>>(a);
    KVQ_HIP_CHECK(hipGetLastError());
    return KVQ_OK;
}
