// Attention over the 4-bit cache.
//
// Query i of the T_b queries of request b stands at position n_b - T_b + i and sees
// the keys up to it. With s = c * q.k in log2 units, p = 2^(s - lse), lse = log2 sum
// 2^s: out = sum p v; weight[j] += (1/Hq) sum over heads and queries of p.
//
// attend_split_kernel, for up to 32 rows a key head (a row is a query with one of the
// head's query heads; cache_tile.cu has the kernel for more): a CTA takes a key head of
// a request, a tile of 8 or 16 rows and all keys, or a chunk of them. Its four warps
// work on their own: a warp copies groups of 16 keys into its ring in shared memory,
// two groups at a time, makes f16 values of codes and scales in registers (exact), and
// multiplies with the keys as the M rows and the query rows as the N columns
// (m16n8k16): a tile of 8 rows, the usual one of a single token, then costs no
// padding, where a contraction of the fifth generation takes 64 or 128 rows. Channels of a
// contraction may come in any order, so a lane takes the 32 (QK) or 16 (PV) neighbouring
// channels that one load brings. The rows' references
// move only when a score passes them by 15 (see kRefBelow); sums and
// statistics are fp32. P is rounded to f16 (11 bits) for the second product, the
// output once to bf16 (8 bits).
// attend_finish_kernel: the chunks of a row joined under the largest reference, and
// the weights of calls of up to 32 rows a key head, whose scores the first kernel has
// kept: 4 bytes a row and key written and read, mostly in L2.
// The probabilities of a key are added in a fixed order; no atomics.
//
// What bounds it: a byte of codes costs instructions (its conversion to f16 pairs, loads,
// contractions) beside its 1/6780 ns of memory, and registers limit an SM to 16 (one row, 8
// rows) or 12 (16 rows) warps. By cases, all with weights:
//   a token of 128 requests of about 1130, 32 heads (669 MB): 126 us, 10 of them for the weights;
//     5.7 TB/s, issue and the integer pipe 57%
//   a token of four requests of 40 Ki to 127 Ki, 28 / 4 heads (217 MB): 68 us, 16 for the weights; 4.5 TB/s, issue 47%
//   1 to 8 e4m3 queries of 32 requests, 32 / 8 heads (139 MB): 110 us, 22 for the weights; 2.7 TB/s with the kept
//     scores, issue 39%: 12 warps do not cover one another's latencies, and requests of different rows
//     leave a sixth of the SMs' time idle
// Dropped: values from codes by masks and shifts (20 pairs a clock and SM; the conversion 50),
// the weights from K read again (190 us of the first case where the kept scores take 10),
// tiles of 32 rows (155 us of the third: 255 registers), rings of three spans (no change), two or four chains
// of contractions a score (no change), 16 warps of 128 registers for tiles of 16 rows (123 us of the third).

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cache_attend.cuh"

namespace lvs {

namespace {

constexpr int kAttWarps = 4;
constexpr int kAttThreads = 32 * kAttWarps;
constexpr int kAttStages = 2;        // spans of 32 keys of a warp's ring
// Of a single row p times the scale is rounded to f16, times a power of two that follows the block's largest
// scale so far: with e at or above the exponent field of that scale (below 1.875 * 2^(e - 7)) and p at most 2^2 the
// product with 2^(20 - e) stays below 2^16, and what falls below f16's normal range is off by at most 2^-34 of the
// largest value, whatever the scales' size. (With 2^5 throughout, which suits the largest scale, the smallest lost
// p below 2^-20.) A larger scale moves e two beyond its field, so that this happens once or twice a warp: 128 requests
// of about 1130 keys, 32 heads, 126 us so, 128 with e at the field, 125 with 2^5.
constexpr float kRefSlack1 = 2.f, kBoost1 = 0x1p20f;  // (the factor for e = 0)

// D += A B: 16 keys (or channels) x 8 rows, f16 operands, fp32 sums
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}


// A group of 16 keys of one head in shared memory.
template <int D>
struct Group {
    static constexpr int kCodes = 16 * D / 2, kScales = 16 * D / 16;
    static constexpr int kK = 0, kKs = kCodes, kV = kCodes + kScales, kVs = 2 * kCodes + kScales;
    static constexpr int kBytes = 2 * (kCodes + kScales);
};

// Starts a warp's copies of the two groups of 16 keys from j0 on, of K and V of head h:
// lanes 0 to 15 copy the first group, the others the second. A group lies in one page;
// `page` is the lane's (-1: zeros).
template <int D>
__device__ __forceinline__ void load_span(const CachePages& c, int32_t page, int h, int j0, uint32_t dst)
{
    using G = Group<D>;
    const int lane = threadIdx.x & 31, l = lane & 15, half = lane >> 4;
    const bool ok = page >= 0;
    const int64_t row =
        cache_row(ok ? page : 0, c.hkv, h, c.page_shift, (j0 + 16 * half) & ((1 << c.page_shift) - 1));
    dst += half * G::kBytes + l * 16;
    const uint8_t* k = c.codes[0] + row * (D / 2) + l * 16;
#pragma unroll
    for (int i = 0; i < G::kCodes / 256; ++i) copy_async16(dst + G::kK + i * 256, k + i * 256, ok);
    const uint8_t* v = c.codes[1] + row * (D / 2) + l * 16;
#pragma unroll
    for (int i = 0; i < G::kCodes / 256; ++i) copy_async16(dst + G::kV + i * 256, v + i * 256, ok);
    // scales: the first lanes those of K, the next those of V
    constexpr int SL = G::kScales / 16;
    const int t = l / SL;
    if (t < 2)
        copy_async16(dst + (t ? G::kVs - SL * 16 : G::kKs), c.scales[t] + row * (D / 16) + (l - t * SL) * 16, ok);
}

// B operands of 8 query rows (columns of the contraction): lane (g, c) holds row
// g's channels [c * D/4, (c + 1) * D/4) as f16, scaled by a power of two that puts
// the row's largest magnitude at about 2^10 (no bf16 value that matters to the
// sums leaves f16's range). `back` receives what undoes the scaling. A row with an
// infinite or NaN channel has no finite score: it is NaN throughout.
template <int D, bool FP8>
__device__ __forceinline__ void load_q(const void* q, int64_t at, bool real, uint32_t (&f)[D / 8], float& back)
{
    constexpr int N = D / 4;
    back = 1.f;
    if constexpr (FP8) {
        const uint4* s = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(q) + at);
#pragma unroll
        for (int i = 0; i < N / 16; ++i) {
            const uint4 v = real ? __ldg(s + i) : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                __half2 x[2];
                e4m3x4_value(w[k], x);
                f[i * 8 + 2 * k] = h2_bits(x[0]), f[i * 8 + 2 * k + 1] = h2_bits(x[1]);
            }
        }
    } else {
        uint32_t w[N / 2];
        const uint4* s = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(q) + at);
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const uint4 v = real ? __ldg(s + i) : make_uint4(0u, 0u, 0u, 0u);
            w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
        }
        // the largest magnitude's bits (as integers they order the magnitudes, NaN above infinity above the rest)
        uint32_t top = 0u;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) top = __vmaxu2(top, w[i] & 0x7FFF7FFFu);
        top = max(top & 0xFFFFu, top >> 16);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // exponent field of the factor: 127 + 10 - (that of top - 127), at most 2^126
        const int e = min(264 - (int)(top >> 7), 253);
        const float up = __int_as_float(top >= 0x7F80u ? 0x7FC00000 : e << 23);
        back = __int_as_float((254 - e) << 23);
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
            f[i] = pack_h2(__uint_as_float(w[i] << 16) * up, __uint_as_float(w[i] & 0xFFFF0000u) * up);
    }
}

// Scores of a group's 16 keys against the tile's rows: S^T[key][row], unscaled.
template <int D, int NT, typename QF>
__device__ __forceinline__ void score_group(const uint8_t* grp, int lane, QF qf, float (&s)[NT][4])
{
    using G = Group<D>;
    const int g = lane >> 2, c = lane & 3;
    constexpr int WORDS = D / 32;  // words of 8 codes of a lane's D/4 channels
    uint32_t w0[WORDS], w1[WORDS];
    __half2 s0[(WORDS + 1) / 2], s1[(WORDS + 1) / 2];
    if constexpr (D == 128) {
        const uint4 a = *reinterpret_cast<const uint4*>(grp + G::kK + g * 64 + c * 16);
        const uint4 b = *reinterpret_cast<const uint4*>(grp + G::kK + (g + 8) * 64 + c * 16);
        w0[0] = a.x, w0[1] = a.y, w0[2] = a.z, w0[3] = a.w;
        w1[0] = b.x, w1[1] = b.y, w1[2] = b.z, w1[3] = b.w;
        const __half2 x = e4m3x2_value(*reinterpret_cast<const uint16_t*>(grp + G::kKs + g * 8 + c * 2));
        const __half2 y = e4m3x2_value(*reinterpret_cast<const uint16_t*>(grp + G::kKs + (g + 8) * 8 + c * 2));
        s0[0] = __low2half2(x), s0[1] = __high2half2(x);
        s1[0] = __low2half2(y), s1[1] = __high2half2(y);
    } else {
        const uint2 a = *reinterpret_cast<const uint2*>(grp + G::kK + g * 32 + c * 8);
        const uint2 b = *reinterpret_cast<const uint2*>(grp + G::kK + (g + 8) * 32 + c * 8);
        w0[0] = a.x, w0[1] = a.y;
        w1[0] = b.x, w1[1] = b.y;
        s0[0] = __low2half2(e4m3x2_value(grp[G::kKs + g * 4 + c]));
        s1[0] = __low2half2(e4m3x2_value(grp[G::kKs + (g + 8) * 4 + c]));
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[t][i] = 0.f;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {  // 8 channels of every lane, two contractions of 16
        __half2 x[4], y[4];
        e2m1x8_value(w0[w], x);
        e2m1x8_value(w1[w], y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = __hmul2(x[i], s0[w / 2]);
            y[i] = __hmul2(y[i], s1[w / 2]);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint2 q = qf(t, 2 * w + e);
                mma16816(s[t], h2_bits(x[2 * e]), h2_bits(y[2 * e]), h2_bits(x[2 * e + 1]), h2_bits(y[2 * e + 1]), q.x,
                         q.y);
            }
    }
}

template <int D>
constexpr int kRingBytes = kAttWarps * kAttStages * 2 * Group<D>::kBytes;

// NT: tiles of 8 rows of a CTA; 0: a single row (a decoded token of a head with keys of its
// own). The eight columns of the contractions, of which a single row would use one, then
// take the scales, which costs no multiplication of the values: column n of QK holds the
// row's channels of scale block n alone, and the score is the sum of the columns times the
// key's scales; column n of PV holds p times the scales of block n, and the channels of
// block n are read from column n.
// WHOLE: the keys are not split (the request is then known to be the same for a whole CTA,
// which keeps addresses out of the lanes' registers: the sweep's 128 requests take 127 us
// and not 135).
// (CTAs of an SM as the plan of the split counts them.)
enum class Picked { kNone, kQuery, kTile, kQueryCluster, kTileCluster };  // (the chunks of a list are a cluster's CTAs)
constexpr int kPickCluster = 8;  // chunks of a list that a cluster joins, at most
// PICKED: the keys are those of picked pages, and a CTA's rows are those of one query, over the pages of its own list, or
// of a tile of queries, over the list of the pages that any of them has (a key of a page that a row's query has not is as
// masked); a CTA takes all of the list or a chunk of it.
template <int D, int NT_, bool FP8, bool WHOLE, Picked PICK = Picked::kNone>
__global__ void __launch_bounds__(kAttThreads, NT_ == 2 ? 3 : 4) attend_split_kernel(const __grid_constant__ AttendArgs a)
{
    constexpr bool PICKED = PICK != Picked::kNone, LISTS = PICK == Picked::kTile || PICK == Picked::kTileCluster;
    constexpr bool CLUSTER = PICK == Picked::kQueryCluster || PICK == Picked::kTileCluster;
    constexpr bool SINGLE = NT_ == 0;
    constexpr int NT = SINGLE ? 1 : NT_;
    using G = Group<D>;
    constexpr int ROWS = 8 * NT;
    constexpr int MT = D / 16;
    // the rings; behind the loop the same memory takes a row tile of every warp's sums
    constexpr int kRing = kRingBytes<D>, kJoin = kAttWarps * 8 * (D + 4) * 4;
    static_assert(kRing >= kJoin, "the sums fit the rings");
    // CLUSTER: the CTA's own sums behind them
    constexpr int kOut = ROWS * D * 4;
    static_assert(!CLUSTER || kRing >= kJoin + kOut, "the CTA's sums fit the rings, too");
    __shared__ float2 ml_s[CLUSTER ? ROWS : 1];
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float s_m[kAttWarps][ROWS], s_l[kAttWarps][ROWS];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, c = lane & 3;
    const int h = blockIdx.y % a.cache.hkv, tile = blockIdx.y / a.cache.hkv;
    griddep_wait();
    griddep_launch_dependents();
    // the request, and its part of the keys: all, or the chunk of this CTA's slot
    int b = blockIdx.z, chunk = kMostKeys, k0 = 0;
    __shared__ int split_s[3];
    QueryTile qt{0, 0, 1};
    const int64_t pick_tile = PICKED ? blockIdx.x / a.pick_chunks : 0;
    const int64_t pick_list = pick_tile * a.cache.hkv + h;
    int listed = 0;  // keys of the list
    if constexpr (PICKED) {
        if constexpr (LISTS) {
            const int4 head = __ldg(a.list_heads + pick_list);
            qt = QueryTile{uniform(head.x), uniform(head.y), uniform(head.z)};
            listed = uniform(head.w) << a.cache.page_shift;
        } else {
            // (as many queries as requests: one each, as no request has two)
            qt.b = a.pick_all ? (int)pick_tile : uniform(find_request(a.q_off, a.batch, pick_tile));
            qt.i0 = 0, qt.queries = 1;
            listed = a.budget << a.cache.page_shift;
        }
        if (qt.queries <= 0) return;
        b = qt.b;
        chunk = LISTS ? list_chunk(listed, a.pick_chunks, 32) : a.pick_chunk;
        k0 = min((int)(blockIdx.x % a.pick_chunks) * chunk, listed);
    } else if (!WHOLE && a.slots > 0) {
        if (threadIdx.x < 32) {
            chunk = chunk_keys(a);
            find_slot(a, blockIdx.x, chunk, b, k0);
            if (threadIdx.x == 0) split_s[0] = chunk, split_s[1] = b, split_s[2] = k0;
        }
        __syncthreads();
        chunk = uniform(split_s[0]), b = uniform(split_s[1]), k0 = uniform(split_s[2]);
        if (b == a.batch) return;
        // (for the launch that joins the chunks: their length, and the request's first slot)
        if (k0 == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.split[b] = make_int2(chunk, (int)blockIdx.x);
    }
    RowTile rt = row_tile(a, b, tile, ROWS);
    const int q0 = a.q_off[b];
    if constexpr (PICKED) {
        rt.row0 = qt.i0 * a.group + tile * ROWS;
        rt.rows = min(ROWS, qt.queries * a.group - tile * ROWS);
    }
    if (rt.rows <= 0) return;
    const int i_last = rt.query(rt.row0 + rt.rows - 1);
    // keys that the tile's last row sees, and this CTA's part of them (PICKED: keys of the list)
    const int seen = PICKED ? listed : min(rt.len, rt.last0 + i_last + 1);
    const int k1 = chunk_end(seen, k0, chunk);
    if (!PICKED && k0 >= k1 && !WHOLE && a.slots > 0) return;  // (without chunks the tile's zeros are written here, else by the join)
    const int all_see = rt.last0 + rt.query(rt.row0);  // the last key that every row sees

    constexpr int SPAN = 2 * G::kBytes;
    uint8_t* my = ring + warp * kAttStages * SPAN;
    const uint32_t my_s = smem_u32(my);
    const int spans = k1 > k0 ? (k1 - k0 + 31) / 32 : 0;
    const int n_mine = spans > warp ? (spans - warp + kAttWarps - 1) / kAttWarps : 0;
    const int last_see = rt.last0 + i_last;  // the last key that any row sees
    const uint32_t all_have = (1u << qt.queries) - 1u;  // PICKED: a bit for every query of the rows
    // page of the lane's group of the warp's n-th span (-1: none; no keys from k1 on are copied), and of a listed page
    // the position of the group's first key and the queries that have it
    int next_pos = 0;
    uint32_t next_have = 0u;
    auto page_of = [&](int n) -> int32_t {
        const int j = k0 + (warp + n * kAttWarps) * 32 + (lane & 16);
        if constexpr (PICKED) {
            next_have = 0u;
            if (j >= k1) return -1;
            int32_t p, o;
            if constexpr (LISTS) {
                const int4 v = __ldg(a.lists + pick_list * a.list_cap + (j >> a.cache.page_shift));
                p = v.x, o = v.y;
                next_have = p >= 0 ? (uint32_t)v.z : 0u;
            } else {
                o = __ldg(a.picked + pick_list * a.budget + (j >> a.cache.page_shift));
                if (o < 0 || o > all_see >> a.cache.page_shift) return -1;
                p = cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, b,
                               (int64_t)o << a.cache.page_shift);
                if (p >= 0) next_have = 1u;
                else if ((lane & 15) == 0) atomicOr(a.err, kErrBounds);
            }
            next_pos = (o << a.cache.page_shift) + (j & ((1 << a.cache.page_shift) - 1));
            if (next_pos > last_see) next_have = 0u;
            return next_have ? p : -1;
        }
        if (j >= k1) return -1;
        const int32_t p = cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, b, j);
        if (p < 0 && (lane & 15) == 0) atomicOr(a.err, kErrBounds);
        return p;
    };
    // whether the lane's group has a page, a bit for every span on its way, the last one's lowest
    uint32_t named = 0;
#pragma unroll
    for (int i = 0; i < kAttStages - 1; ++i) {
        const int32_t page = page_of(i);
        if (i < n_mine) load_span<D>(a.cache, page, h, k0 + (warp + i * kAttWarps) * 32, my_s + i * SPAN);
        copy_async_commit();
        named = named << 1 | (page >= 0);
    }
    static_assert(kAttStages == 2, "one span is on its way beside the one in hand");
    int pos = next_pos;           // PICKED: of the span in hand
    uint32_t have = next_have;
    int32_t next_page = page_of(kAttStages - 1);  // (read a span ahead: nothing waits for the table)

    // ---- the tile's rows
    uint32_t qr[NT][D / 8];
    float fac[NT][2];  // log2-unit scale of rows 2c and 2c + 1
    int vis[NT][2];    // last key they see
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = t * 8 + g;
        const bool real = r < rt.rows;
        const int row = rt.row0 + (real ? r : 0);
        const int i = rt.query(row);
        const int64_t at =
            (int64_t)(q0 + i) * a.q_stride + (int64_t)(h * a.group + row - i * a.group) * D + c * (D / 4);
        float back;
        load_q<D, FP8>(a.q, at, SINGLE || real, qr[t], back);
        if constexpr (SINGLE) {  // (every lane has read row 0; lane (g, c) keeps what lies in block g)
#pragma unroll
            for (int k = 0; k < D / 8; ++k)
                if (D == 128 ? g != 2 * c + k / 8 : g != c) qr[0][k] = 0u;
        }
        fac[t][0] = row_factor(a.c_log2, __shfl_sync(0xffffffffu, back, 8 * c));
        fac[t][1] = row_factor(a.c_log2, __shfl_sync(0xffffffffu, back, 8 * c + 4));
#pragma unroll
        for (int e = 0; e < 2; ++e) vis[t][e] = rt.last0 + rt.query(rt.row0 + t * 8 + 2 * c + e);
    }
    auto qf = [&](int t, int k) -> uint2 {
        return make_uint2(qr[t][2 * k], qr[t][2 * k + 1]);
    };

    float o[NT][MT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[t][i][e] = 0.f;
        m[t][0] = m[t][1] = kNoRef;
        l[t][0] = l[t][1] = 0.f;
    }

    // SINGLE: the factor of block g of V, and what brings any larger exponent field of a scale, in the four bytes of a
    // word, to the byte's highest bit: 0x78 - 8 e
    float boost = kBoost1;
    uint32_t room = 0x78787878u;

    float* logits = a.logits + (h * a.head_rows + (int64_t)q0 * a.group + rt.row0 + 2 * c) * a.logit_stride;
    bool nan_value = false;

    // a group of 16 keys from j0 on, for a single row
    int pos_of[2] = {0, 0};  // PICKED: of a span's two groups
    uint32_t have_of[2] = {0u, 0u};
    uint32_t my_bit[NT][2];  // PICKED: of the queries of rows 2c and 2c + 1
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) my_bit[t][e] = PICKED ? 1u << ((vis[t][e] - all_see) & 31) : 0u;
    auto group1 = [&](const uint8_t* grp, int j0, bool there, int n_sees, auto check) {
        constexpr bool CHECK = decltype(check)::value;
        constexpr int WORDS = D / 32;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        float ks[2][2];  // scales of the keys g and g + 8 in the blocks 2c and 2c + 1
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int at = G::kKs + (g + 8 * e) * (D / 16) + 2 * c;
            const float2 f = __half22float2(e4m3x2_value(*reinterpret_cast<const uint16_t*>(grp + (D == 128 || c < 2 ? at : 0))));
            ks[e][0] = D == 128 || c < 2 ? f.x : 0.f;
            ks[e][1] = D == 128 || c < 2 ? f.y : 0.f;
        }
        uint32_t w0[WORDS], w1[WORDS];
        if constexpr (D == 128) {
            const uint4 x = *reinterpret_cast<const uint4*>(grp + G::kK + g * 64 + c * 16);
            const uint4 y = *reinterpret_cast<const uint4*>(grp + G::kK + (g + 8) * 64 + c * 16);
            w0[0] = x.x, w0[1] = x.y, w0[2] = x.z, w0[3] = x.w;
            w1[0] = y.x, w1[1] = y.y, w1[2] = y.z, w1[3] = y.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(grp + G::kK + g * 32 + c * 8);
            const uint2 y = *reinterpret_cast<const uint2*>(grp + G::kK + (g + 8) * 32 + c * 8);
            w0[0] = x.x, w0[1] = x.y;
            w1[0] = y.x, w1[1] = y.y;
        }
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            __half2 x[4], y[4];
            e2m1x8_value(w0[w], x);
            e2m1x8_value(w1[w], y);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                mma16816(s, h2_bits(x[2 * e]), h2_bits(y[2 * e]), h2_bits(x[2 * e + 1]), h2_bits(y[2 * e + 1]),
                         qr[0][4 * w + 2 * e], qr[0][4 * w + 2 * e + 1]);
        }
        float z[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            z[e] = fmaf(s[2 * e], ks[e][0], s[2 * e + 1] * ks[e][1]);
            z[e] += __shfl_xor_sync(0xffffffffu, z[e], 1);
            z[e] += __shfl_xor_sync(0xffffffffu, z[e], 2);
            z[e] *= fac[0][0];
            if (CHECK && (PICKED ? g + 8 * e >= n_sees : !there || j0 + g + 8 * e >= k1)) z[e] = -INFINITY;
        }
        if (a.logits && c == 0) {
            __stcg(logits + j0 + g, z[0]);
            __stcg(logits + j0 + g + 8, z[1]);
        }
        // scales of the lane's keys of the second product, a byte each
        uint32_t scales = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int key = 2 * c + (e & 1) + 8 * (e >> 1);
            uint32_t sc = grp[G::kVs + (D == 128 ? key * 8 + g : key * 4 + g / 2)];
            if (CHECK && (PICKED ? key >= n_sees : j0 + key >= k1)) sc = 0u;  // (bytes behind the last key may be anything)
            scales |= sc << (8 * e);
        }
        const bool larger = (((scales + room) | scales) & 0x80808080u) != 0u;
        if (__any_sync(0xffffffffu, larger || fmaxf(z[0], z[1]) > m[0][0] + kRefSlack1)) {
            float x = fmaxf(z[0], z[1]);
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            const float mn = fmaxf(m[0][0], x);
            const float f = ex2(m[0][0] - mn);
            m[0][0] = mn;
            l[0][0] *= f;
            float f0 = f, f1 = f;  // of the columns 2c and 2c + 1
            if (__any_sync(0xffffffffu, larger)) {
                const uint32_t fields = scales & 0x78787878u;
                uint32_t e8 = max(max(fields & 0xFFu, (fields >> 8) & 0xFFu), max((fields >> 16) & 0xFFu, fields >> 24));
                e8 = max(e8, __shfl_xor_sync(0xffffffffu, e8, 1));
                e8 = max(e8, __shfl_xor_sync(0xffffffffu, e8, 2));
                const uint32_t before = 0x78u - (room & 0xFFu);
                e8 = e8 > before ? min(e8 + 16u, 0x78u) : before;
                room = 0x01010101u * (0x78u - e8);
                boost = __uint_as_float((147u - e8 / 8u) << 23);
                const float less = __uint_as_float((127u - (e8 - before) / 8u) << 23);
                f0 *= __shfl_sync(0xffffffffu, less, 8 * c);
                f1 *= __shfl_sync(0xffffffffu, less, 8 * c + 4);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                o[0][i][0] *= f0, o[0][i][1] *= f1;
                o[0][i][2] *= f0, o[0][i][3] *= f1;
            }
        }
        const float p0 = ex2(z[0] - m[0][0]), p1 = ex2(z[1] - m[0][0]);
        l[0][0] += p0 + p1;
        // probabilities of the lane's keys of the second product (2c, 2c+1, 2c+8, 2c+9)
        float pk[4];
        pk[0] = __shfl_sync(0xffffffffu, p0, 8 * c);
        pk[1] = __shfl_sync(0xffffffffu, p0, 8 * c + 4);
        pk[2] = __shfl_sync(0xffffffffu, p1, 8 * c);
        pk[3] = __shfl_sync(0xffffffffu, p1, 8 * c + 4);
        constexpr int VW = D / 64;
        uint32_t x[4][VW];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int key = 2 * c + (e & 1) + 8 * (e >> 1);
            if constexpr (D == 128) {
                const uint2 v = *reinterpret_cast<const uint2*>(grp + G::kV + key * 64 + g * 8);
                x[e][0] = v.x, x[e][1] = v.y;
            } else {
                x[e][0] = *reinterpret_cast<const uint32_t*>(grp + G::kV + key * 32 + g * 4);
            }
        }
        const float2 sa = __half22float2(e4m3x2_value(scales & 0xFFFFu)), sb = __half22float2(e4m3x2_value(scales >> 16));
        const uint32_t b0 = pack_h2(pk[0] * (sa.x * boost), pk[1] * (sa.y * boost));
        const uint32_t b1 = pack_h2(pk[2] * (sb.x * boost), pk[3] * (sb.y * boost));
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            const uint32_t lo = 0x0F0F0F0Fu;
            const uint32_t ae = (x[0][w] & lo) | ((x[1][w] << 4) & ~lo), ao = ((x[0][w] >> 4) & lo) | (x[1][w] & ~lo);
            const uint32_t be = (x[2][w] & lo) | ((x[3][w] << 4) & ~lo), bo = ((x[2][w] >> 4) & lo) | (x[3][w] & ~lo);
            __half2 a0[4], a1[4], a2[4], a3[4];
            e2m1x8_value(ae, a0);
            e2m1x8_value(ao, a1);
            e2m1x8_value(be, a2);
            e2m1x8_value(bo, a3);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                mma16816(o[0][w * 4 + i], h2_bits(a0[i]), h2_bits(a1[i]), h2_bits(a2[i]), h2_bits(a3[i]), b0, b1);
        }
    };

    // a span of 32 keys from j0 on, two groups at a time (one after the other: 114 us where this takes 110, 1 to 8
    // queries of 32 requests, 32 / 8 heads); `there`: their keys that have a page; CHECK: some of
    // the rows do not see all of them
    auto span_of = [&](const uint8_t* grp0, int j0, uint32_t there, auto check, bool late = true) {
        constexpr bool CHECK = decltype(check)::value;
        float s[2][NT][4];
#pragma unroll
        for (int x = 0; x < 2; ++x) score_group<D, NT>(grp0 + x * G::kBytes, lane, qf, s[x]);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[x][t][e] *= fac[t][e & 1];
                    if (CHECK && (PICKED ? !(have_of[x] & my_bit[t][e & 1]) ||
                                               (late && pos_of[x] + g + 8 * (e >> 1) > vis[t][e & 1])
                                         : !(there >> (16 * x) & 1u) ||
                                               j0 + 16 * x + g + 8 * (e >> 1) > min(vis[t][e & 1], k1 - 1)))
                        s[x][t][e] = -INFINITY;
                }
        if (a.logits) {
            float* to = logits + j0 + g;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (t * 8 + 2 * c + e < rt.rows) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            __stcg(to + (t * 8 + e) * a.logit_stride + 16 * x, s[x][t][e]);
                            __stcg(to + (t * 8 + e) * a.logit_stride + 16 * x + 8, s[x][t][e + 2]);
                        }
                    }
        }
        bool move = false;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                move |= fmaxf(fmaxf(s[0][t][e], s[0][t][e + 2]), fmaxf(s[1][t][e], s[1][t][e + 2])) > m[t][e] + kRefSlack;
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = fmaxf(fmaxf(s[0][t][e], s[0][t][e + 2]), fmaxf(s[1][t][e], s[1][t][e + 2]));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                    const float mn = fmaxf(m[t][e], x - kRefBelow);
                    const float f = ex2(m[t][e] - mn);
                    m[t][e] = mn;
                    l[t][e] *= f;
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[t][i][e] *= f;
                        o[t][i][e + 2] *= f;
                    }
                }
        }
        uint32_t pb[2][NT][2];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = ex2(s[x][t][e] - m[t][e & 1]);
                l[t][0] += p[0] + p[2];
                l[t][1] += p[1] + p[3];
                pb[x][t][0] = transpose8x8(pack_h2(p[0], p[1]));
                pb[x][t][1] = transpose8x8(pack_h2(p[2], p[3]));
            }
        // ---- values: lane (g, c) takes keys 2c, 2c+1, 2c+8, 2c+9 and channels [g * D/8, (g + 1) * D/8)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint8_t* grp = grp0 + x * G::kBytes;
            constexpr int VW = D / 64;  // words of a lane's channels
            uint32_t w4[4][VW];
            uint32_t sc[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = 2 * c + (e & 1) + 8 * (e >> 1);
                if constexpr (D == 128) {
                    const uint2 v = *reinterpret_cast<const uint2*>(grp + G::kV + key * 64 + g * 8);
                    w4[e][0] = v.x, w4[e][1] = v.y;
                    sc[e] = grp[G::kVs + key * 8 + g];
                } else {
                    w4[e][0] = *reinterpret_cast<const uint32_t*>(grp + G::kV + key * 32 + g * 4);
                    sc[e] = grp[G::kVs + key * 4 + g / 2];
                }
                if constexpr (CHECK && !PICKED) {
                    const int at = j0 + 16 * x + key;
                    // what lies behind the last key may be anything, a NaN scale among it
                    if (at >= k1) sc[e] = 0u;
                    // a NaN value must not reach the rows that do not see it (0 * NaN): put in at the end
                    if (at > all_see && (sc[e] & 0x7Fu) == 0x7Fu) {
                        sc[e] = 0u;
                        nan_value = true;
                    }
                }
                if (CHECK && PICKED && late && pos_of[x] + key > last_see) sc[e] = 0u;  // (behind the last key, as above)
            }
            if constexpr (CHECK && LISTS) {
                // NaN among the scales, for rows that may not see it, as above
                const uint32_t four = sc[0] | sc[1] << 8 | sc[2] << 16 | sc[3] << 24;
                if (((four & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if ((sc[e] & 0x7Fu) == 0x7Fu) sc[e] = 0u;
                    nan_value = true;
                }
            }
            const __half2 sa = e4m3x2_value(sc[0] | (sc[1] << 8)), sb = e4m3x2_value(sc[2] | (sc[3] << 8));
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                // bytes of (code of the first key, code of the second) for the even and the odd channels
                const uint32_t lo = 0x0F0F0F0Fu;
                const uint32_t ae = (w4[0][w] & lo) | ((w4[1][w] << 4) & ~lo), ao = ((w4[0][w] >> 4) & lo) | (w4[1][w] & ~lo);
                const uint32_t be = (w4[2][w] & lo) | ((w4[3][w] << 4) & ~lo), bo = ((w4[2][w] >> 4) & lo) | (w4[3][w] & ~lo);
                __half2 a0[4], a1[4], a2[4], a3[4];
                e2m1x8_value(ae, a0);
                e2m1x8_value(ao, a1);
                e2m1x8_value(be, a2);
                e2m1x8_value(bo, a3);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t f0 = h2_bits(__hmul2(a0[i], sa)), f1 = h2_bits(__hmul2(a1[i], sa));
                    const uint32_t f2 = h2_bits(__hmul2(a2[i], sb)), f3 = h2_bits(__hmul2(a3[i], sb));
#pragma unroll
                    for (int t = 0; t < NT; ++t) mma16816(o[t][w * 4 + i], f0, f1, f2, f3, pb[x][t][0], pb[x][t][1]);
                }
            }
        }
    };

    int stage = 0;
#pragma unroll 1
    for (int n = 0; n < n_mine; ++n) {
        copy_async_wait<kAttStages - 2>();
        __syncwarp();  // every lane's copies are there, and the span before is no longer read
        const int j0 = k0 + (warp + n * kAttWarps) * 32;
        const bool mine = named >> (kAttStages - 2) & 1u;  // the lane's group of this span has a page
        const int now_pos = pos;
        const uint32_t now_have = have;
        if constexpr (PICKED) pos = next_pos, have = next_have;  // (those of next_page)
        {
            const int nx = n + kAttStages - 1;
            const int to = stage == 0 ? kAttStages - 1 : stage - 1;
            if (nx < n_mine)
                load_span<D>(a.cache, next_page, h, j0 + (kAttStages - 1) * kAttWarps * 32, my_s + to * SPAN);
            copy_async_commit();
            named = named << 1 | (next_page >= 0);
            next_page = page_of(nx + 1);
        }
        const uint8_t* span = my + stage * SPAN;
        stage = stage + 1 == kAttStages ? 0 : stage + 1;
        const uint32_t there = __ballot_sync(0xffffffffu, mine);
        if (PICKED && there == 0u) continue;
        const bool all = PICKED ? __all_sync(0xffffffffu, now_have == all_have && now_pos + 15 <= all_see)
                                : there == 0xFFFFFFFFu && j0 + 31 <= all_see;
        if constexpr (PICKED) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                pos_of[x] = __shfl_sync(0xffffffffu, now_pos, 16 * x);
                have_of[x] = __shfl_sync(0xffffffffu, now_have, 16 * x);
            }
        }
        if constexpr (SINGLE) {
            if (all) {
#pragma unroll
                for (int x = 0; x < 2; ++x) group1(span + x * G::kBytes, j0 + 16 * x, true, 16, std::false_type{});
            } else {
#pragma unroll 1
                for (int x = 0; x < 2; ++x) {
                    const int n_sees = (x ? have_of[1] : have_of[0]) ? last_see - (x ? pos_of[1] : pos_of[0]) + 1 : 0;
                    if (PICKED ? n_sees > 0 : j0 + 16 * x < k1)
                        group1(span + x * G::kBytes, j0 + 16 * x, there >> (16 * x) & 1u, n_sees, std::true_type{});
                }
            }
        } else {
            if (all) span_of(span, j0, there, std::false_type{});
            else span_of(span, j0, there, std::true_type{},
                         !LISTS || __any_sync(0xffffffffu, now_have != 0u && now_pos + 15 > all_see));
        }
    }
    copy_async_wait<0>();

    // ---- the four warps joined, 8 rows at a time
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[t][e] += __shfl_xor_sync(0xffffffffu, l[t][e], d);
            if (g == 0) {
                s_m[warp][t * 8 + 2 * c + e] = m[t][e];
                s_l[warp][t * 8 + 2 * c + e] = l[t][e];
            }
        }
    nan_value = __syncthreads_or(nan_value);
    float* jo = reinterpret_cast<float*>(ring);  // [warp][row][D + 4]
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int rows = min(8, rt.rows - t * 8);
        if (rows <= 0) break;
        if (t > 0) __syncthreads();
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (!SINGLE && 2 * c + e < rows) {
                float* to = jo + (warp * 8 + 2 * c + e) * (D + 4) + g * (D / 8);
#pragma unroll
                for (int i = 0; i < MT; ++i) *reinterpret_cast<float2*>(to + 2 * i) = make_float2(o[t][i][e], o[t][i][e + 2]);
            }
        if (SINGLE && c == g >> 1) {  // column g holds the channels of lane g
            float* to = jo + warp * 8 * (D + 4) + g * (D / 8);
            const float back = 1.f / boost;
#pragma unroll
            for (int i = 0; i < MT; ++i)
                *reinterpret_cast<float2*>(to + 2 * i) = g & 1 ? make_float2(o[0][i][1] * back, o[0][i][3] * back)
                                                               : make_float2(o[0][i][0] * back, o[0][i][2] * back);
        }
        __syncthreads();
        for (int x = tid; x < rows * D; x += kAttThreads) {
            const int r = x / D, ch = x % D;
            const int row = t * 8 + r;
            float M = kNoRef;
#pragma unroll
            for (int w = 0; w < kAttWarps; ++w) M = fmaxf(M, s_m[w][row]);
            float L = 0.f, O = 0.f;
#pragma unroll
            for (int w = 0; w < kAttWarps; ++w) {
                const float f = ex2(s_m[w][row] - M);
                L += s_l[w][row] * f;
                O += jo[(w * 8 + r) * (D + 4) + ch] * f;
            }
            const int rr = rt.row0 + row, i = rt.query(rr);
            const int64_t at = (int64_t)(q0 + i) * a.hq + h * a.group + rr - i * a.group;
            if (LISTS && nan_value) {
                for (int j = k0; j < k1; ++j) {
                    const int4 v = __ldg(a.lists + pick_list * a.list_cap + (j >> a.cache.page_shift));
                    const int slot = j & ((1 << a.cache.page_shift) - 1);
                    if (v.x < 0 || !((uint32_t)v.z >> (i - qt.i0) & 1u) || (v.y << a.cache.page_shift) + slot > rt.last0 + i)
                        continue;
                    const int64_t at_row = cache_row(v.x, a.cache.hkv, h, a.cache.page_shift, slot);
                    if ((a.cache.scales[1][at_row * (D / 16) + ch / 16] & 0x7Fu) == 0x7Fu) O = __int_as_float(0x7FC00000);
                }
            }
            if (!PICKED && nan_value) {
                for (int j = max(k0, all_see + 1); j < min(k1, rt.last0 + i + 1); ++j) {
                    const int32_t page =
                        cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, b, j);
                    if (page < 0) continue;
                    const int64_t at_row =
                        cache_row(page, a.cache.hkv, h, a.cache.page_shift, j & ((1 << a.cache.page_shift) - 1));
                    if ((a.cache.scales[1][at_row * (D / 16) + ch / 16] & 0x7Fu) == 0x7Fu) O = __int_as_float(0x7FC00000);
                }
            }
            if (CLUSTER) {
                jo[kJoin / 4 + row * D + ch] = O;
                if (ch == 0) ml_s[row] = make_float2(M, L);
            } else if (PICKED ? a.pick_chunks == 1 : WHOLE || a.slots == 0) {
                // (a row that sees no key is 0; the comparison keeps a NaN sum)
                a.out[at * D + ch] = __float2bfloat16_rn(L == 0.f ? 0.f : O / L * a.cache.scale[1]);
                if (a.lse && ch == 0) a.lse[at] = L == 0.f ? INFINITY : M + log2f(L);
            } else {
                const int64_t part = ((int64_t)blockIdx.x * a.cache.hkv + h) * a.max_rows + (PICKED ? rr - qt.i0 * a.group : rr);
                a.part_o[part * D + ch] = O;
                if (ch == 0) a.part_ml[part] = make_float2(M, L);
            }
        }
    }
    if constexpr (CLUSTER) {
        // the chunks of a list are a cluster's CTAs: each joins a part of the rows from all CTAs' shared memory
        cluster_sync_all();
        const uint32_t n = cluster_nctarank();
        for (int x = (int)cluster_ctarank() * kAttThreads + tid; x < rt.rows * D / 2; x += (int)n * kAttThreads) {
            const int row = 2 * x / D;
            const uint32_t at_ml = smem_u32(&ml_s[row]), at_o = smem_u32(jo + kJoin / 4 + 2 * x);
            float2 ml[kPickCluster], o[kPickCluster];
            float M = kNoRef;
#pragma unroll
            for (uint32_t r = 0; r < kPickCluster; ++r)
                if (r < n) {
                    ml[r] = ld_shared_cluster_f2(mapa_shared(at_ml, r));
                    o[r] = ld_shared_cluster_f2(mapa_shared(at_o, r));
                    M = fmaxf(M, ml[r].x);
                }
            float L = 0.f, O0 = 0.f, O1 = 0.f;
#pragma unroll
            for (uint32_t r = 0; r < kPickCluster; ++r)
                if (r < n) {
                    const float f = ex2(ml[r].x - M);
                    L += ml[r].y * f;
                    O0 += o[r].x * f, O1 += o[r].y * f;
                }
            const int rr = rt.row0 + row, i = rt.query(rr);
            const int64_t to = ((int64_t)(q0 + i) * a.hq + h * a.group + rr - i * a.group) * D + 2 * x % D;
            const float f = a.cache.scale[1] / L;
            *reinterpret_cast<__nv_bfloat162*>(a.out + to) =
                __floats2bfloat162_rn(L == 0.f ? 0.f : O0 * f, L == 0.f ? 0.f : O1 * f);
        }
        cluster_sync_all();  // (no CTA ends while another reads its memory)
    }
}

// Reference and sum of a row from those of its n chunks (`step` apart), by a warp.
__device__ __forceinline__ float2 join_stats(const float2* ml, int64_t step, int n)
{
    const int lane = threadIdx.x & 31;
    float M = kNoRef, L = 0.f;
    constexpr int U = 4;
    for (int x0 = 0; x0 < n; x0 += 32 * U) {
        float2 v[U];
        float mx = M;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * 32 + lane;
            v[u] = x < n ? __ldcg(ml + x * step) : make_float2(kNoRef, 0.f);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) mx = fmaxf(mx, v[u].x);
        L *= ex2(M - mx);
        M = mx;
#pragma unroll
        for (int u = 0; u < U; ++u) L += v[u].y * ex2(v[u].x - M);
    }
    float top = M;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    L *= ex2(M - top);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) L += __shfl_xor_sync(0xffffffffu, L, d);
    return make_float2(top, L);
}

constexpr int kFinishThreads = 512;
constexpr int kFinishWarps = kFinishThreads / 32;
// Warps of a CTA that share a key's rows in adding weights: the fewer, the more keys a CTA takes at a time
// (128 for each of the others) and the fewer CTAs read the chunks' statistics; the more rows (query and
// head), the longer a CTA would have. 28 rows (four requests of up to 127 Ki keys): 67 us for the call with 2,
// 70 with 4, 75 with 8; 32 to 256 rows (32 requests of up to 8152, before other steps brought 115.5 to 110): 125, 119
// and 115.5. Where CTAs of 256
// keys are so few that all run at once, more share too (16 rows, 524 keys: 8.4 us with 2, 7.7 with 8).
int weight_parts(int rows, int64_t ctas, int num_sms) { return rows <= 64 && ctas > 3 * num_sms ? 2 : 8; }
constexpr int kLogitRows = 2048;  // rows of a request whose scores are kept for the weights

// Sums over the rows [x0, x1) of the probabilities of four neighbouring keys. CHECK: some
// of the rows do not see all of them.
template <bool CHECK>
__device__ __forceinline__ float4 add_weights(const float* s, int64_t stride, const int2* rows, const float* lse, int x0,
                                              int x1, int j)
{
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int U = 8;
    for (int x = x0; x < x1; x += U) {
        float4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            v[u] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (x + u < x1 && (!CHECK || j <= rows[x + u].y))
                v[u] = __ldcg(reinterpret_cast<const float4*>(s + (int64_t)rows[x + u].x * stride));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x + u >= x1) break;
            const float e = lse[x + u];
            const int last = CHECK ? rows[x + u].y : 0;
            sum.x += CHECK && j > last ? 0.f : ex2(v[u].x - e);
            sum.y += CHECK && j + 1 > last ? 0.f : ex2(v[u].y - e);
            sum.z += CHECK && j + 2 > last ? 0.f : ex2(v[u].z - e);
            sum.w += CHECK && j + 3 > last ? 0.f : ex2(v[u].w - e);
        }
    }
    return sum;
}

// The first `join_blocks` CTAs of a request join its rows' chunks, `row_warps` warps a row;
// the others add weights from the kept scores, 256 to 1024 keys at a time, over the rows in order.
// Where some requests have no queries (`active` > 0: those that have), the grid's first axis holds the join CTAs of
// these, then the weight CTAs of all; else its second axis is the request.
// A weight CTA finds the rows' lse from the chunks' statistics by itself, which saves a
// launch between the two. 10 us of the 128-request step; 16 of the four long requests' (40 Ki to
// 127 Ki keys x 28 rows of kept scores, 47 MB; each of 568 CTAs finds all 28 rows' lse from about 150 chunks before its
// first scores), 22 of the drafts' (80 MB).
template <int D, int PARTS>
__global__ void __launch_bounds__(kFinishThreads) attend_finish_kernel(const __grid_constant__ AttendArgs a,
                                                                       int join_blocks, int weight_blocks, int row_warps,
                                                                       int active)
{
    extern __shared__ uint8_t rows_s[];
    // the warps' parts: four weights a lane, or a row of outputs a warp (D <= 128)
    __shared__ __align__(16) float join_s[kFinishWarps][128];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int b = blockIdx.y, block = blockIdx.x;
    griddep_wait();
    griddep_launch_dependents();
    if (active > 0) {
        const int joins = active * join_blocks;
        if (block < joins) {
            b = find_active(a, block / join_blocks);
            block %= join_blocks;
            if (b == a.batch) return;
        } else {
            b = (block - joins) / weight_blocks;
            block = join_blocks + (block - joins) % weight_blocks;
        }
    }
    bool bad;
    const int len = cache_len(a.lens[b], a.limit, bad);
    const int q0 = a.q_off[b], t = a.q_off[b + 1] - q0;
    int chunk = kMostKeys, slot0 = 0;
    if (a.slots > 0 && t > 0 && len > 0) {
        const int2 v = __ldcg(a.split + b);
        chunk = v.x, slot0 = v.y;
    }
    const int64_t step = (int64_t)a.cache.hkv * a.max_rows;  // from a chunk's statistics to the next's
    // chunks with keys that query i sees
    auto chunks_seen = [&](int i) -> int {
        const int seen = len - t + i + 1;
        return seen > 0 ? chunks_of(seen, chunk) : 0;
    };
    if (block >= join_blocks) {
        const int rows = t * a.group, n = rows * a.cache.hkv;
        constexpr int across = kFinishWarps / PARTS, keys = 128 * across;
        const int tiles = (len + keys - 1) / keys;
        int tile = block - join_blocks;
        if (tile >= tiles) return;
        float* lse_s = reinterpret_cast<float*>(rows_s);
        int2* row_s = reinterpret_cast<int2*>(rows_s + (size_t)((n + 1) & ~1) * 4);  // scores' row, last key seen
        const int most = t > 0 ? chunks_seen(t - 1) : 0;
        const bool by_warp = most > 16;
        for (int x = by_warp ? warp : tid; x < n; x += by_warp ? kFinishWarps : kFinishThreads) {
            const int h = x / rows, r = x % rows, i = r / a.group;
            float lse;
            if (a.slots == 0) {
                lse = __ldcg(a.lse + (int64_t)(q0 + i) * a.hq + h * a.group + r % a.group);
            } else {
                const float2* from = a.part_ml + ((int64_t)slot0 * a.cache.hkv + h) * a.max_rows + r;
                float2 ml = make_float2(kNoRef, 0.f);
                if (by_warp) {
                    ml = join_stats(from, step, chunks_seen(i));
                } else {
                    float2 v[16];
                    const int m = chunks_seen(i);
#pragma unroll
                    for (int y = 0; y < 16; ++y) v[y] = y < m ? __ldcg(from + y * step) : make_float2(kNoRef, 0.f);
#pragma unroll
                    for (int y = 0; y < 16; ++y) ml.x = fmaxf(ml.x, v[y].x);
#pragma unroll
                    for (int y = 0; y < 16; ++y) ml.y += v[y].y * ex2(v[y].x - ml.x);
                }
                lse = ml.y == 0.f ? INFINITY : ml.x + log2f(ml.y);
            }
            if (!by_warp || lane == 0) {
                lse_s[x] = lse;
                row_s[x] = make_int2(h * (int)a.head_rows + r, len - t + i);
            }
        }
        __syncthreads();
        const int part = warp / across, per = (n + PARTS - 1) / PARTS;
        const int x0 = min(n, part * per), x1 = min(n, x0 + per);
        for (; tile < tiles; tile += weight_blocks) {
            // four neighbouring keys a lane (the scores' rows are padded to a whole number of them)
            const int j0 = tile * keys, j = j0 + warp % across * 128 + 4 * lane;
            int64_t at = -1;
            float before[4];
            if (part == 0 && j < len) {
                const int32_t page =
                    cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, b, j);
                if (page >= 0) at = ((int64_t)page << a.cache.page_shift) + (j & ((1 << a.cache.page_shift) - 1));
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) before[e] = at >= 0 && j + e < len ? a.weights_in[at + e] : 0.f;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            if (j < len) {
                const float* s = a.logits + (int64_t)q0 * a.group * a.logit_stride + j;
                sum = j0 + keys - 1 <= len - t ? add_weights<false>(s, a.logit_stride, row_s, lse_s, x0, x1, j)
                                                      : add_weights<true>(s, a.logit_stride, row_s, lse_s, x0, x1, j);
            }
            float4* sums = reinterpret_cast<float4*>(&join_s[0][0]);  // [part][128 lanes of the tile]
            sums[warp * 32 + lane] = sum;
            __syncthreads();
            if (at >= 0) {
#pragma unroll
                for (int p = 1; p < PARTS; ++p) {
                    const float4 v = sums[(warp + across * p) * 32 + lane];
                    sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
                }
                const float add[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j + e < len) a.weights_out[at + e] = before[e] + add[e] / (float)a.hq;
            }
            __syncthreads();
        }
        return;
    }
    const int part = warp % row_warps, join_rows = kFinishWarps / row_warps, rows = t * a.hq;
    __shared__ float2 ml_s[kFinishWarps];
    // where a row (query and head) has its chunks' sums, and how many chunks there are
    auto place = [&](int r, int64_t& from) -> int {
        if (r >= rows) return 0;
        const int i = r / a.hq, hq = r - i * a.hq, h = hq / a.group;
        from = ((int64_t)slot0 * a.cache.hkv + h) * a.max_rows + i * a.group + hq - h * a.group;
        return chunks_seen(i);
    };
    // four of the warp's chunks, from x0 on
    constexpr int U = 4;
    auto load = [&](int64_t from, int n, int x0, float2 (&ml)[U], float (&v)[U][D / 32]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * row_warps;
            const float* p = a.part_o + (from + x * step) * D + lane * (D / 32);
            ml[u] = make_float2(kNoRef, 0.f);
#pragma unroll
            for (int e = 0; e < D / 32; ++e) v[u][e] = 0.f;
            if (x < n) {
                ml[u] = __ldcg(a.part_ml + from + x * step);
                if constexpr (D == 128) {
                    const float4 w = __ldcg(reinterpret_cast<const float4*>(p));
                    v[u][0] = w.x, v[u][1] = w.y, v[u][2] = w.z, v[u][3] = w.w;
                } else {
                    const float2 w = __ldcg(reinterpret_cast<const float2*>(p));
                    v[u][0] = w.x, v[u][1] = w.y;
                }
            }
        }
    };
    int64_t from = 0;
    int r = block * join_rows + warp / row_warps, n = place(r, from);
    float2 ml[U];
    float v[U][D / 32];
    load(from, n, part, ml, v);
    const int next_r = join_blocks * join_rows;
    for (int r0 = block * join_rows; r0 < rows; r0 += next_r, r += next_r) {
        // chunks under a running reference
        float M = kNoRef, L = 0.f, O[D / 32];
#pragma unroll
        for (int e = 0; e < D / 32; ++e) O[e] = 0.f;
        auto add = [&](float m2, float l2, const float* o2) {
            const float top = fmaxf(M, m2), f = ex2(M - top), f2 = ex2(m2 - top);
            M = top;
            L = L * f + l2 * f2;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) O[e] = O[e] * f + o2[e] * f2;
        };
        for (int x0 = part; x0 < n; x0 += U * row_warps) {
            if (x0 > part) load(from, n, x0, ml, v);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (x0 + u * row_warps < n) add(ml[u].x, ml[u].y, v[u]);
        }
        const bool real = r < rows;
        n = place(r + next_r, from);  // the next row's sums are on their way while this one is written
        load(from, n, part, ml, v);
        if (row_warps > 1) {
#pragma unroll
            for (int e = 0; e < D / 32; ++e) join_s[warp][lane * (D / 32) + e] = O[e];
            if (lane == 0) ml_s[warp] = make_float2(M, L);
            __syncthreads();
            if (part == 0) {
                for (int w = 1; w < row_warps; ++w) {
                    float o2[D / 32];
#pragma unroll
                    for (int e = 0; e < D / 32; ++e) o2[e] = join_s[warp + w][lane * (D / 32) + e];
                    add(ml_s[warp + w].x, ml_s[warp + w].y, o2);
                }
            }
            __syncthreads();
        }
        if (part == 0 && real) {
            const int64_t at = (int64_t)q0 * a.hq + r;
            const float f = a.cache.scale[1] / L;
#pragma unroll
            for (int e = 0; e < D / 32; e += 2)
                *reinterpret_cast<__nv_bfloat162*>(a.out + at * D + lane * (D / 32) + e) =
                    __floats2bfloat162_rn(L == 0.f ? 0.f : O[e] * f, L == 0.f ? 0.f : O[e + 1] * f);
            if (a.lse && lane == 0) a.lse[at] = L == 0.f ? INFINITY : M + log2f(L);
        }
    }
}

template <int D, bool FP8>
cudaError_t launch_all(const AttendArgs& a, const AttendPlan& plan, int max_rows, int64_t total_rows, int max_len,
                       cudaStream_t stream, int32_t* launches)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.stream = stream;
    cudaError_t e = cudaSuccess;
    if (total_rows > 0) {
        const int tiles = (max_rows + plan.row_tile - 1) / plan.row_tile;
        if (plan.row_tile >= 128) {
            e = launch_attend_tiles(a, D, FP8, plan.row_tile, tiles, stream);
            if (e != cudaSuccess) return e;
            ++*launches;
        } else {
            cfg.gridDim = plan.slots > 0 ? dim3((unsigned)plan.slots, (unsigned)(tiles * a.cache.hkv), 1)
                                         : dim3(1, (unsigned)(tiles * a.cache.hkv), (unsigned)a.batch);
            cfg.blockDim = dim3(kAttThreads, 1, 1);
            const bool whole = plan.slots == 0;
            auto kern = max_rows == 1 ? (whole ? attend_split_kernel<D, 0, FP8, true> : attend_split_kernel<D, 0, FP8, false>)
                        : plan.row_tile == 8
                            ? (whole ? attend_split_kernel<D, 1, FP8, true> : attend_split_kernel<D, 1, FP8, false>)
                            : attend_split_kernel<D, 2, FP8, false>;
            cfg.dynamicSmemBytes = kRingBytes<D>;
            static_assert(kRingBytes<D> + 10 * 1024 <= 48 * 1024, "no more shared memory than a launch has without asking");
            e = cudaLaunchKernelEx(&cfg, kern, a);
            if (e != cudaSuccess) return e;
            ++*launches;
            cfg.dynamicSmemBytes = 0;
        }
    }
    const int most = max_rows / a.group * a.hq;  // rows of the longest request
    // warps of a row by the chunks that a request with queries has where all are alike
    const int chunks = (plan.slots + plan.active - 1) / std::max(plan.active, 1);
    const int row_warps = chunks <= 4 ? 1 : (chunks <= 16 ? 4 : kFinishWarps);
    const int join_rows = kFinishWarps / row_warps;  // of a CTA
    // (a warp joins row after row, the next one's sums on their way: a chunk of a prompt 234 to 224 us)
    const int join_blocks =
        total_rows > 0 && plan.slots > 0
            ? std::min((most + join_rows - 1) / join_rows, std::max(1, 4 * a.num_sms / plan.active)) : 0;
    // weight CTAs: one for the keys that it takes at a time, as many as run in a round or two
    const int parts = weight_parts(most, (int64_t)(max_len + 255) / 256 * a.batch, a.num_sms);
    const int keys = 128 * kFinishWarps / parts;
    const int weight_blocks =
        a.logits ? std::min((max_len + keys - 1) / keys, std::max(1, (parts == 8 ? 6 : 3) * a.num_sms / a.batch)) : 0;
    if (weight_blocks + join_blocks > 0) {
        const bool all = plan.active == a.batch;
        cfg.gridDim = all ? dim3((unsigned)(join_blocks + weight_blocks), (unsigned)a.batch, 1)
                          : dim3((unsigned)(plan.active * join_blocks + a.batch * weight_blocks), 1, 1);
        cfg.blockDim = dim3(kFinishThreads, 1, 1);
        cfg.dynamicSmemBytes = a.logits ? (size_t)(most + 2) * 12 : 0;
        e = cudaLaunchKernelEx(&cfg, parts == 2 ? attend_finish_kernel<D, 2> : attend_finish_kernel<D, 8>, a, join_blocks,
                               weight_blocks, row_warps, all ? 0 : plan.active);
        if (e != cudaSuccess) return e;
        ++*launches;
        cfg.dynamicSmemBytes = 0;
    }
    if (a.weights_out && !a.logits && max_len > 0) {
        e = launch_attend_weights(a, D, FP8, max_len, stream);
        if (e != cudaSuccess) return e;
        *launches += a.row_tiles > 0 ? 2 : 1;
    }
    return e;
}

// The list of a tile's queries for a key head: the pages that any of them has and sees, ascending, with the queries that
// have each. A bit for every page of the request in shared memory (65536 of them at a time), the number of bits before
// each word, and a second pass over the queries' own lists, which finds every page's place by them. What bounds it: a chain
// of loads, offsets - length - lists - table - lists; 9 us of a cold cache for 32 requests of up to 8 queries and 48 pages,
// which the next kernel saves many times: of the 37 queries of a tile of 256 rows with 32 pages each, most have
// the same 120.
constexpr int kListThreads = 256;
constexpr int kListWords = 2048;
__global__ void __launch_bounds__(kListThreads) picked_list_kernel(const __grid_constant__ AttendArgs a)
{
    __shared__ uint32_t bits_s[kListWords];
    __shared__ int before_s[kListWords];
    __shared__ int warp_s[kListThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    griddep_wait();
    griddep_launch_dependents();
    const int64_t list = blockIdx.x, tile = list / a.cache.hkv;
    const int h = (int)(list - tile * a.cache.hkv);
    // the tile's request: the requests' tiles one after the other, 256 requests at a time
    __shared__ int found_s[2];
    if (tid == 0) found_s[0] = -1;
    int64_t tiles_before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kListThreads) {
        const int b = b0 + tid;
        const int n = b < a.batch ? tiles_of(__ldg(a.q_off + b + 1) - __ldg(a.q_off + b), a.pick_queries) : 0;
        int sum = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += y;
        }
        if (lane == 31) warp_s[warp] = sum;
        __syncthreads();
        int64_t at = tiles_before + sum - n;
#pragma unroll
        for (int w = 0; w < kListThreads / 32; ++w) {
            if (w < warp) at += warp_s[w];
            tiles_before += warp_s[w];
        }
        if (tile >= at && tile < at + n) found_s[0] = b, found_s[1] = (int)(tile - at) * a.pick_queries;
        __syncthreads();
        if (found_s[0] >= 0) break;
    }
    QueryTile qt;
    qt.b = found_s[0];
    if (qt.b < 0) {
        if (tid == 0) a.list_heads[list] = make_int4(0, 0, 0, 0);
        return;
    }
    qt.i0 = found_s[1];
    qt.queries = min(a.pick_queries, __ldg(a.q_off + qt.b + 1) - __ldg(a.q_off + qt.b) - qt.i0);
    bool bad;
    const int len = cache_len(__ldg(a.lens + qt.b), a.limit, bad);
    if (bad && tid == 0) atomicOr(a.err, kErrBounds);
    const int q0 = __ldg(a.q_off + qt.b), t = __ldg(a.q_off + qt.b + 1) - q0;
    const int first = len - t + qt.i0;                    // position of the first query
    const int last = first + qt.queries - 1, shift = a.cache.page_shift;
    const int pages = last < 0 ? 0 : (last >> shift) + 1;  // that the last query sees
    const int32_t* picked = a.picked + ((int64_t)(q0 + qt.i0) * a.cache.hkv + h) * a.budget;
    int4* out = a.lists + list * a.list_cap;
    uint32_t* rows = a.list_bits ? a.list_bits + list * a.pick_queries * a.list_words : nullptr;
    // calls f(query, page from w0 on) for the lists' pages in [w0, w0 + n) that their queries see; a warp has 64 entries
    // of four queries on their way at once
    auto each = [&](int w0, int n, auto f) {
        constexpr int W = kListThreads / 32, U = 4;
        for (int q0 = warp; q0 < qt.queries; q0 += W * U)
            for (int x0 = lane; x0 < a.budget; x0 += 64) {
                int o[U][2];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        o[u][y] = q0 + u * W < qt.queries && x0 + 32 * y < a.budget
                                      ? __ldg(picked + (int64_t)(q0 + u * W) * a.cache.hkv * a.budget + x0 + 32 * y)
                                      : -1;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int q = q0 + u * W, sees = first + q < 0 ? -1 : (first + q) >> shift;
                        if (o[u][y] >= 0 && o[u][y] <= sees && o[u][y] >= w0 && o[u][y] - w0 < n) f(q, o[u][y] - w0);
                    }
            }
    };
    int base = 0;
    for (int w0 = 0; w0 < pages; w0 += 32 * kListWords) {
        const int n = min(pages - w0, 32 * kListWords), words = (n + 31) / 32;
        for (int x = tid; x < words; x += kListThreads) bits_s[x] = 0u;
        __syncthreads();
        each(w0, n, [&](int, int o) { atomicOr(bits_s + (o >> 5), 1u << (o & 31)); });
        __syncthreads();
        // bits before each word: a thread has `per` neighbouring words
        const int per = (words + kListThreads - 1) / kListThreads, x0 = min(words, tid * per), x1 = min(words, x0 + per);
        int mine = 0;
        for (int x = x0; x < x1; ++x) mine += __popc(bits_s[x]);
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += y;
        }
        if (lane == 31) warp_s[warp] = sum;
        __syncthreads();
        int at = base + sum - mine, all = base;
#pragma unroll
        for (int w = 0; w < kListThreads / 32; ++w) {
            if (w < warp) at += warp_s[w];
            all += warp_s[w];
        }
        for (int x = x0; x < x1; ++x) {
            before_s[x] = at;
            at += __popc(bits_s[x]);
        }
        if (rows) {  // words that only bits of this pass reach
            const int z0 = (base + 31) / 32, z1 = (all + 31) / 32;
            for (int q = warp; q < qt.queries; q += kListThreads / 32)
                for (int z = z0 + lane; z < z1; z += 32) rows[(int64_t)q * a.list_words + z] = 0u;
        }
        __syncthreads();
        for (int x = tid; x < n; x += kListThreads)
            if (bits_s[x >> 5] >> (x & 31) & 1u) {
                const int to = before_s[x >> 5] + __popc(bits_s[x >> 5] & ((1u << (x & 31)) - 1u));
                const int32_t p = cache_page(a.cache.table, a.cache.width, a.cache.num_pages, shift, qt.b,
                                             (int64_t)(w0 + x) << shift);
                if (p < 0) atomicOr(a.err, kErrBounds);
                out[to] = make_int4(p, w0 + x, 0, 0);
            }
        __syncthreads();
        each(w0, n, [&](int q, int o) {
            const int to = before_s[o >> 5] + __popc(bits_s[o >> 5] & ((1u << (o & 31)) - 1u));
            if (rows) atomicOr(rows + (int64_t)q * a.list_words + (to >> 5), 1u << (to & 31));
            else atomicOr(reinterpret_cast<uint32_t*>(&out[to].z), 1u << q);
        });
        base = all;
        __syncthreads();
    }
    if (tid == 0) a.list_heads[list] = make_int4(qt.b, qt.i0, qt.queries, base);
    if (h == 0 && tid < qt.queries) a.tile_of[q0 + qt.i0 + tid] = make_int2((int)tile, tid);
}

// The chunks of a tile's list joined, a row (query and head) a warp: chunk x of a tile has its sums at
// ((tile * chunks + x) * hkv + key head) * rows of a tile + row.
template <int D>
__global__ void __launch_bounds__(kAttThreads) picked_join_kernel(const __grid_constant__ AttendArgs a, int64_t rows)
{
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kAttWarps + (threadIdx.x >> 5);
    griddep_wait();
    griddep_launch_dependents();
    if (row >= rows) return;
    const int64_t r = row / a.hq;
    const int hq = (int)(row % a.hq), h = hq / a.group;
    int64_t tile = r;
    int in = hq % a.group;
    if (a.lists) {
        const int2 v = __ldg(a.tile_of + r);
        tile = v.x;
        in += v.y * a.group;
    }
    const int64_t from = (tile * a.pick_chunks * a.cache.hkv + h) * a.max_rows + in, step = (int64_t)a.cache.hkv * a.max_rows;
    float M = kNoRef, L = 0.f, O[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; ++e) O[e] = 0.f;
    constexpr int U = 4;
    for (int x0 = 0; x0 < a.pick_chunks; x0 += U) {
        float2 ml[U];
        float v[U][D / 32];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = from + min(x0 + u, a.pick_chunks - 1) * step;
            ml[u] = __ldcg(a.part_ml + at);
            if constexpr (D == 128) {
                const float4 w = __ldcg(reinterpret_cast<const float4*>(a.part_o + at * D) + lane);
                v[u][0] = w.x, v[u][1] = w.y, v[u][2] = w.z, v[u][3] = w.w;
            } else {
                const float2 w = __ldcg(reinterpret_cast<const float2*>(a.part_o + at * D) + lane);
                v[u][0] = w.x, v[u][1] = w.y;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x0 + u >= a.pick_chunks) break;
            const float top = fmaxf(M, ml[u].x), f = ex2(M - top), f2 = ex2(ml[u].x - top);
            M = top;
            L = L * f + ml[u].y * f2;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) O[e] = O[e] * f + v[u][e] * f2;
        }
    }
    const float f = a.cache.scale[1] / L;
#pragma unroll
    for (int e = 0; e < D / 32; e += 2)
        *reinterpret_cast<__nv_bfloat162*>(a.out + row * D + lane * (D / 32) + e) =
            __floats2bfloat162_rn(L == 0.f ? 0.f : O[e] * f, L == 0.f ? 0.f : O[e + 1] * f);
}

template <int D, bool FP8>
cudaError_t launch_picked(const AttendArgs& a, const PickedPlan& plan, int64_t queries, cudaStream_t stream, int32_t* launches)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.stream = stream;
    cudaError_t e = cudaSuccess;
    if (plan.lists) {
        cfg.gridDim = dim3((unsigned)(plan.tiles * a.cache.hkv), 1, 1);
        cfg.blockDim = dim3(kListThreads, 1, 1);
        e = cudaLaunchKernelEx(&cfg, picked_list_kernel, a);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    if (plan.row_tile >= 128) {
        e = launch_picked_tiles(a, plan, D, FP8, stream);
    } else {
        const int subs = (plan.queries * a.group + plan.row_tile - 1) / plan.row_tile;
        cfg.gridDim = dim3((unsigned)(plan.tiles * plan.chunks), (unsigned)(subs * a.cache.hkv), 1);
        cfg.blockDim = dim3(kAttThreads, 1, 1);
        cfg.dynamicSmemBytes = kRingBytes<D>;
        auto pick = [&](auto q, auto t) {
            constexpr Picked Q = decltype(q)::value, T = decltype(t)::value;
            return plan.lists ? (plan.row_tile == 8 ? attend_split_kernel<D, 1, FP8, false, T>
                                                    : attend_split_kernel<D, 2, FP8, false, T>)
                   : a.group == 1 ? attend_split_kernel<D, 0, FP8, false, Q>
                                  : (plan.row_tile == 8 ? attend_split_kernel<D, 1, FP8, false, Q>
                                                        : attend_split_kernel<D, 2, FP8, false, Q>);
        };
        using Own = std::integral_constant<Picked, Picked::kQuery>;
        using Tile = std::integral_constant<Picked, Picked::kTile>;
        using OwnC = std::integral_constant<Picked, Picked::kQueryCluster>;
        using TileC = std::integral_constant<Picked, Picked::kTileCluster>;
        auto kern = plan.cluster ? pick(OwnC{}, TileC{}) : pick(Own{}, Tile{});
        if (plan.cluster) {
            attr[1].id = cudaLaunchAttributeClusterDimension;
            attr[1].val.clusterDim = {(unsigned)plan.chunks, 1, 1};
            cfg.numAttrs = 2;
        }
        e = cudaLaunchKernelEx(&cfg, kern, a);
        cfg.numAttrs = 1;
    }
    if (e != cudaSuccess) return e;
    ++*launches;
    if (plan.chunks > 1 && !plan.cluster) {
        const int64_t rows = queries * a.hq;
        cfg.gridDim = dim3((unsigned)((rows + kAttWarps - 1) / kAttWarps), 1, 1);
        cfg.blockDim = dim3(kAttThreads, 1, 1);
        cfg.dynamicSmemBytes = 0;
        e = cudaLaunchKernelEx(&cfg, picked_join_kernel<D>, a, rows);
        if (e == cudaSuccess) ++*launches;
    }
    return e;
}

}  // namespace

// A call of single tokens has a tile for each query, with the pages of its own list. Else neighbouring queries of a
// request, which mostly have the same pages, share a tile of up to 16, 128 or 256 rows and read its pages once.
// Tiles of 128 rows from 17 rows of the longest request on: 24 and 32 rows of 32 requests, 32 / 8 heads, 48 pages of 32,
// 84 and 89 us where tiles of 16 take 158 and 174; 12 and 16 rows 76 and 82 with either. Up to 32 rows tiles of 16 all
// the same where a tile of 128 for each request and head left seven eighths of its places empty: four queries of one
// request, 28 / 4 heads, 32 pages of 64, 25 us (128 rows: 33), of eight 27 (29); 30 of four, 16 heads, 47 (41).
// The lists are split where the tiles alone leave the GPU's places empty: as for whole requests, n chunks take
// rounds / n of the list and the writing and joining of a chunk's sums. A shared list is taken to grow by half of a
// query's own for each doubling of the queries: of 32 pages each, picked as neighbours mostly agree on, 18 queries
// have 117 and 36 124. A chunk of a prompt (777 to 1024 queries of two requests, 28 / 4 heads, 32 pages of 64): whole
// 237 us, two chunks 216, three 252.
PickedPlan plan_attend_picked(int batch, int hkv, int group, const int32_t* q_off, int page_shift, int width, int budget,
                              int num_sms)
{
    PickedPlan p{};
    int max_t = 0;
    for (int b = 0; b < batch; ++b) max_t = std::max(max_t, q_off[b + 1] - q_off[b]);
    const int64_t max_rows = (int64_t)max_t * group;
    p.lists = max_t > 1;
    int active = 0;
    for (int b = 0; b < batch; ++b) active += q_off[b + 1] > q_off[b];
    const int64_t few = max_rows <= 32 && (int64_t)active * hkv * 4 <= num_sms ? 32 : 16;
    p.row_tile = p.lists ? (max_rows <= 8 ? 8 : (max_rows <= few ? 16 : (max_rows <= 128 ? 128 : 256))) : (group <= 8 ? 8 : 16);
    p.queries = p.lists ? std::max(1, p.row_tile / group) : 1;
    int64_t keys = (int64_t)budget << page_shift;
    const int64_t subs = ((int64_t)p.queries * group + p.row_tile - 1) / p.row_tile;
    for (int b = 0; b < batch; ++b) p.tiles += tiles_of(q_off[b + 1] - q_off[b], p.queries);
    const int64_t items = p.tiles * hkv * subs;
    if (p.lists) {
        p.list_cap = (int32_t)std::min<int64_t>(width, (int64_t)p.queries * budget);
        p.list_words = (p.list_cap + 31) / 32;
        keys = std::min((int64_t)((double)keys * (1.0 + std::log2((double)p.queries) / 2.0)), (int64_t)p.list_cap << page_shift);
    }
    const bool many = p.row_tile >= 128;
    const int64_t places = (int64_t)num_sms * (p.row_tile == 256 ? 1 : (p.row_tile == 128 ? 2 : (p.row_tile == 16 ? 3 : 4)));
    const int64_t units = std::max<int64_t>(1, (keys + 127) / 128);
    int64_t best = 1;
    if (items > 0 && items < places) {
        best = std::min(units, places / items);
    } else if (items < 3 * places) {
        double cost = 1e30;
        for (int64_t n = 1; n <= std::min<int64_t>(units, 8); ++n) {
            const double whole = (double)((items * n + places - 1) / places);
            const double r = many ? (whole + (double)(items * n) / (double)places) / 2.0 : whole;
            const double more = (many ? 250.0 : 0.0) + (n > 1 ? (many ? 0.75 : 1.25) * p.row_tile : 0.0);
            const double c = r / (double)n + r * more / (double)std::max<int64_t>(keys, 1);
            if (c < cost) cost = c, best = n;
        }
    }
    // chunks of few rows are joined within a cluster where it holds them: a launch less, and no sums in memory
    p.cluster = !many && best > 1 && best <= kPickCluster;
    p.chunk = (int32_t)(((keys + best - 1) / best + 31) & ~31ll);
    p.chunks = (int32_t)(p.lists ? best : std::max<int64_t>(1, (keys + p.chunk - 1) / p.chunk));
    if (p.chunks == 1) p.cluster = false;
    return p;
}

cudaError_t launch_attend_picked(const AttendArgs& a, const PickedPlan& plan, int head_dim, bool fp8, int64_t queries,
                                 cudaStream_t stream, int32_t* launches)
{
    *launches = 0;
    if (queries == 0) return cudaSuccess;
    if (fp8) return launch_picked<128, true>(a, plan, queries, stream, launches);
    return head_dim == 128 ? launch_picked<128, false>(a, plan, queries, stream, launches)
                           : launch_picked<64, false>(a, plan, queries, stream, launches);
}

// Rows of a request's key head up to which the kernel for few rows is taken. A key costs it less
// and it splits finer, but it makes a key's values again for every 16 rows; the other makes them once for
// 128 or 256 rows, takes as long for fewer, and makes the scores twice where weights are wanted. 16 requests of
// 4096 keys, 32 / 8 heads: 12 rows 53 us (other 50), with weights 63 (95); 20 rows 71 (51), with weights 84
// (96); 32 rows 79 (51), 97.5 (96). One of 8000 keys: 20 rows 19.6 (19.7). 32 ragged requests of 4 to 32 rows and up to
// 8200 keys: 88 (128), with weights 111 (243). A call's rows are those of its longest request, so the border
// lies where ragged calls and those with weights gain more than the others lose. For the same reason prompts and
// single tokens are better two calls: 1024 queries beside 63 single ones, 4096 keys each, 28 / 4 heads, take 212 us,
// each alone 69 and 43.
constexpr int kFewRows = 32;

// 128 rows a CTA, or two row tiles that share the K and V that it makes: 192 rows 97 (one) and 72 us
// (two), 256 rows 92 and 79.
int attend_row_tile(int64_t max_rows) { return max_rows <= 8 ? 8 : (max_rows <= kFewRows ? 16 : (max_rows <= 128 ? 128 : 256)); }
bool attend_keeps_scores(int64_t max_rows, int hkv)
{
    return max_rows > 0 && max_rows <= kFewRows && max_rows * hkv <= kLogitRows;
}

AttendPlan plan_cache_attend(int batch, int hkv, int group, const int32_t* q_off, int64_t max_len, int num_sms)
{
    AttendPlan p;
    int max_t = 0;
    p.active = 0;
    for (int b = 0; b < batch; ++b) {
        max_t = std::max(max_t, q_off[b + 1] - q_off[b]);
        p.active += q_off[b + 1] > q_off[b];
    }
    const int64_t max_rows = (int64_t)max_t * group;
    p.row_tile = attend_row_tile(max_rows);
    int64_t items = 0;  // CTAs where each takes all keys of its rows
    for (int b = 0; b < batch; ++b)
        items += ((int64_t)(q_off[b + 1] - q_off[b]) * group + p.row_tile - 1) / p.row_tile * hkv;
    // The keys are split into n chunks a request where that fills the GPU better: items * n CTAs of
    // 1/n of the work run in rounds of as many as fit at once (by the kernels' registers and tensor
    // memory), and the writing and joining of a chunk's sums takes a CTA as long as about five
    // keys for every four rows. A CTA of the kernel for many rows, alone on its SM or in a pair, takes as long
    // as 700 keys to start and to end, and its chunks are joined in as long as 2.3 keys a row; its rounds are between
    // the whole number and the fraction, as its CTAs' keys differ. (2 x 700 queries over 2048 keys, 32 / 8
    // heads: whole 73 us, three chunks, as for few rows, 103; 1023 and 873 over 5928 and 6517, 28 / 4 heads: 195 and
    // 213; 512 over 8192, half the SMs: whole 129, two chunks 80.)
    const int64_t places = (int64_t)num_sms * (p.row_tile == 256 ? 1 : (p.row_tile == 128 ? 2 : (p.row_tile == 16 ? 3 : 4)));
    // (three rounds of smaller chunks for 9 to 32 rows, whose requests have different numbers of rows too)
    const int rounds = p.row_tile == 16 && batch > 1 ? 3 : 1;
    const int64_t units = std::max<int64_t>(1, (max_len + 63) / 64);
    int64_t best = 1;
    if (items > 0 && items < places) {
        best = std::min(units, rounds * places / items);
    } else if (items < 3 * places) {
        // (From three rounds on the last one's idle places matter little where the requests are alike. Where one is far
        // longer than the rest, the CTAs of its heads are left alone with all of its keys: 127 requests of 1000 tokens
        // and one of 131072, 32 heads, take 1110 us, where 128 of 1000 take 125.)
        double cost = 1e30;
        for (int64_t n = 1; n <= std::min<int64_t>(units, 8); ++n) {
            const bool many = p.row_tile >= 128;
            const double whole = (double)((items * n + places - 1) / places);
            const double r = many ? (whole + (double)(items * n) / (double)places) / 2.0 : whole;
            const double more = (many ? 700.0 : 0.0) + (n > 1 ? (many ? 2.3 : 1.25) * p.row_tile : 0.0);
            const double c = r / (double)n + r * more / (double)std::max<int64_t>(max_len, 1);
            if (c < cost) cost = c, best = n;
        }
    }
    // (a request without queries has no keys to read: one of 4096 keys beside 255 such takes 18 us, with slots
    // for each of those too 1780)
    p.slots = best > 1 ? (int32_t)std::min<int64_t>(best * p.active, 1 << 20) : 0;
    p.logits = attend_keeps_scores(max_rows, hkv);
    return p;
}

cudaError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& plan, int head_dim, bool fp8, int max_rows,
                                int64_t total_rows, int max_len, cudaStream_t stream, int32_t* launches)
{
    *launches = 0;
    if (fp8) return launch_all<128, true>(a, plan, max_rows, total_rows, max_len, stream, launches);
    return head_dim == 128 ? launch_all<128, false>(a, plan, max_rows, total_rows, max_len, stream, launches)
                           : launch_all<64, false>(a, plan, max_rows, total_rows, max_len, stream, launches);
}

}  // namespace lvs
