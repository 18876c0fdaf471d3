// The pages that a query attends to, picked by the ranges of their keys.
//
// A query's score of a page is the largest product that a key of the page's ranges can have with it: with the query
// as whole numbers r of a power of two, S(page) = 2^e max over the key head's query heads of sum over channels of
// r * (r > 0 ? hi : lo). The sums are whole numbers below 2^22, exact in fp32 and in s32 in any order, so
// the same inputs pick the same pages whatever kernel adds them up.
//
// The scores are a product [pages, 2 d] x [2 d, columns] with max(r, 0) against hi and min(r, 0) against lo, a
// column for each query head of a key head (a query's columns padded to a power of two or whole tiles of eight):
//   pick_token_kernel, one tile of columns: 32 caches of 30 Ki to 127 Ki tokens in pages of 32, 32 / 8 heads (180 MB): 41 us,
//     4.3 TB/s, a fifth of it the CTAs' start; one of 40 Ki, 28 / 4 heads, 7 us with the launch
//   pick_score_kernel, up to 64 columns a request: a warp keeps 16 pages as f16 in registers and goes over the columns'
//     tiles in shared memory. The caches above with 2 to 8 queries each take 96 us, the picking with them; the prompts
//     below took 74 with it
//   cache_pick_tile.cu, more: 777 to 1024 queries of two requests of 20 Ki to 32 Ki in pages of 64, 28 / 4 heads: 27 us
// pick_select_kernel: the budget-th largest score of a query by counting its scores in buckets, then the
// pages above it and the lowest of those at it, in order. 256 lists of up to 4096 pages 10.5 us, 7204 of about 400 14
// (bit by bit 13 and 18).

#include <algorithm>

#include "cache_pick.cuh"

namespace lvs {

namespace {

constexpr int kScoreThreads = 128;
constexpr int kScorePages = 16 * kScoreThreads / 32;  // of a CTA at a time
constexpr int kScoreCols = 64;                        // columns of a request up to which a CTA has them all

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint2 b)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y));
}

// A lane's codes of two pages as they are in memory, and their units.
template <int D>
struct PageCodes {
    uint4 w[2][2 * D / 64];
    float unit[2];  // 0: none

    // pages p[0] and p[1] of the pool (-1: none): channels [c * 16, c * 16 + 16) of each 64
    __device__ __forceinline__ void load(const PickArgs& a, const int32_t (&p)[2], int h, int c)
    {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int64_t row = (int64_t)max(p[e], 0) * a.hkv + h;
            const int x = min(max((int)__ldg(a.exps + row), -100), 100);
            unit[e] = p[e] >= 0 ? __uint_as_float((uint32_t)(127 + x) << 23) : 0.f;
            const uint4* from = reinterpret_cast<const uint4*>(a.codes + row * 2 * D) + c;
#pragma unroll
            for (int k = 0; k < 2 * D / 64; ++k) w[e][k] = __ldg(from + k * 4);
        }
    }
    // the A operand of contraction k
    __device__ __forceinline__ void operand(int k, uint32_t (&f)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint4 v = w[e][k / 4];
            s8x4_value(k % 4 == 0 ? v.x : (k % 4 == 1 ? v.y : (k % 4 == 2 ? v.z : v.w)), f[e], f[2 + e]);
        }
    }
};

// Key heads of a CTA of the kernel for few queries, a warp each (or two, or four).
__host__ __device__ __forceinline__ int score_heads(int hkv) { return hkv % 4 == 0 ? 4 : (hkv % 2 == 0 ? 2 : 1); }

// The lane's pages g and g + 8 from `from` on in the pool (-1: none).
__device__ __forceinline__ void find_pages(const PickArgs& a, int b, int from, int pages, int32_t (&p)[2])
{
    const int g = (threadIdx.x & 31) >> 2;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int o = from + g + 8 * e;
        p[e] = -1;
        if (o < pages) {
            p[e] = cache_page(a.table, a.width, a.num_pages, a.page_shift, b, (int64_t)o << a.page_shift);
            if (p[e] < 0 && (threadIdx.x & 3) == 0) atomicOr(a.err, kErrBounds);
        }
    }
}

// Scores of a contraction's 16 pages (from `base` on) and a tile x of eight columns: d of page g and columns 2c and 2c + 1,
// then of page g + 8; their units (0: the pool has no such page). `best` carries the largest over the tiles of a query of more than eight heads.
__device__ __forceinline__ void store_scores(const PickArgs& a, const ScoreTile& st, int h, int padded, int base, int x,
                                             const float (&unit)[2], const float (&d)[4], float (&best)[2])
{
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int64_t keys_step = (int64_t)a.hkv * a.key_stride, keys_at = (int64_t)(st.q0 + st.i0) * keys_step + h * a.key_stride;
    auto put = [&](int i, int e, float s) {  // score of the CTA's query i and page g + 8 e
        const int o = base + g + 8 * e;
        if (i < st.queries && o < st.pages)
            a.keys[keys_at + i * keys_step + o] =
                (e ? unit[1] : unit[0]) > 0.f ? score_key(s * (e ? unit[1] : unit[0])) : 1u;
    };
    if (padded == 1) {
        const int i = x * 8 + 2 * c;
        put(i, 0, d[0]), put(i + 1, 0, d[1]);
        put(i, 1, d[2]), put(i + 1, 1, d[3]);
        return;
    }
    float s0 = fmaxf(d[0], d[1]), s1 = fmaxf(d[2], d[3]);
    if (padded >= 4) {
        s0 = fmaxf(s0, __shfl_xor_sync(0xffffffffu, s0, 1));
        s1 = fmaxf(s1, __shfl_xor_sync(0xffffffffu, s1, 1));
    }
    if (padded >= 8) {
        s0 = fmaxf(s0, __shfl_xor_sync(0xffffffffu, s0, 2));
        s1 = fmaxf(s1, __shfl_xor_sync(0xffffffffu, s1, 2));
        best[0] = fmaxf(best[0], s0), best[1] = fmaxf(best[1], s1);
        const int tiles_of = padded / 8;
        if (x % tiles_of != tiles_of - 1) return;
        if (c < 2) put(x / tiles_of, c, c ? best[1] : best[0]);
        best[0] = best[1] = -INFINITY;
    } else if (padded == 4) {
        put(x * 2 + (c >> 1), c & 1, c & 1 ? s1 : s0);
    } else {
        put(x * 4 + c, 0, s0);
        put(x * 4 + c, 1, s1);
    }
}

// D += A B in whole numbers: 16 pages x 8 columns, 32 channels
__device__ __forceinline__ void mma16832(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint2 b)
{
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y));
}

// Pages of request b whose scores are wanted.
__device__ __forceinline__ int scored_pages(const PickArgs& a, int b)
{
    bool bad;
    const int len = cache_len(__ldg(a.lens + b), a.limit, bad);
    const int pages = len > 0 ? ((len - 1) >> a.page_shift) + 1 : 0;
    return pages > a.budget && (a.single || __ldg(a.off + b + 1) > __ldg(a.off + b)) ? pages : 0;
}
// The requests' pages in equal chunks, a multiple of `unit`, so that there are no more than `slots` of them however the
// lengths differ (at least one a request), and the chunk of this CTA: its request (a.batch: none) and its first page. Both
// by a warp.
__device__ __forceinline__ int score_chunk(const PickArgs& a, int slots, int unit)
{
    if (a.batch == 1) {
        const int n = (scored_pages(a, 0) + slots - 1) / slots;
        return max(unit, (n + unit - 1) / unit * unit);
    }
    const int lane = threadIdx.x & 31;
    long long total = 0;
    int some = 0;  // requests with pages
    for (int b = lane; b < a.batch; b += 32) {
        const int n = scored_pages(a, b);
        total += n, some += n > 0;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    some = __reduce_add_sync(0xffffffffu, some);
    // sum of ceil(n / chunk) <= total / chunk + some
    const long long per = (total + max(1, slots - some) - 1) / max(1, slots - some);
    return (int)min((long long)kMostKeys, (per + unit - 1) / unit * unit);
}
__device__ __forceinline__ void find_chunk(const PickArgs& a, int chunk, int& b, int& first)
{
    if (a.batch == 1) {
        b = 0;
        first = (int)blockIdx.x * chunk;
        return;
    }
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
        const int pages = b0 + lane < a.batch ? scored_pages(a, b0 + lane) : 0;
        const int n = pages > 0 ? (pages - 1) / chunk + 1 : 0;
        int sum = n;  // inclusive
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += y;
        }
        const uint32_t hit = __ballot_sync(0xffffffffu, (int)blockIdx.x < before + sum);
        if (hit) {
            const int x = __ffs(hit) - 1;
            b = b0 + x;
            first = ((int)blockIdx.x - before - __shfl_sync(0xffffffffu, sum - n, x)) * chunk;
            return;
        }
        before += __shfl_sync(0xffffffffu, sum, 31);
    }
    b = a.batch;
    first = 0;
}

// Single tokens, and a few queries of few heads: one tile of columns. The codes go into the contraction as they are in
// memory (s8: this GPU's slow kind, a third of the time here, but f16 made of them took as many instructions again as
// all else), the queries' whole numbers stay in registers. A warp has a key head of its own where there are enough, so
// that a CTA reads neighbouring heads' codes of a page, which lie side by side, at the same time. Codes come by asynchronous
// copies of whole rows: read into registers, a lane's 16 bytes of each of eight rows at a time, they came at 3 TB/s.
template <int D>
struct TokenRing {
    static constexpr int ROW = 2 * D, STAGE = 16 * ROW, STAGES = 2;
    // byte of 16-byte part x of row r: odd rows have their halves swapped, so that two rows' parts cover all banks
    __device__ static __forceinline__ int at(int r, int x) { return r * ROW + (x ^ ((r & 1) << 2)) * 16; }
};
template <int D, bool FP8>
__global__ void __launch_bounds__(kScoreThreads, 5) pick_token_kernel(const __grid_constant__ PickArgs a, int slots)
{
    using R = TokenRing<D>;
    constexpr int STEPS = 2 * D / 32;                       // contractions of 32 channels
    __shared__ uint2 frag_s[kScoreThreads / 32][STEPS][32];
    __shared__ __align__(16) uint8_t ring_s[kScoreThreads / 32][R::STAGES * R::STAGE];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int heads = score_heads(a.hkv);  // of a CTA
    const int h = blockIdx.y * heads + warp % heads, step = kScorePages / heads;
    griddep_wait();
    griddep_launch_dependents();
    const int padded = padded_group(a.group);
    int b, first;
    const int chunk = score_chunk(a, slots, step);
    find_chunk(a, chunk, b, first);
    if (b == a.batch) return;
    const ScoreTile st = score_tile(a, b, 0, 8 / padded);
    const int pages = min(st.pages, first + chunk);
    int base = first + warp / heads * 16;
    if (base >= pages) return;

    // page of row lane % 16 of the 16 pages from `from` on (-1: none), and its unit
    auto find = [&](int from) -> int32_t {
        const int o = from + (lane & 15);
        if (o >= pages) return -1;
        const int32_t p = cache_page(a.table, a.width, a.num_pages, a.page_shift, b, (int64_t)o << a.page_shift);
        if (p < 0 && lane < 16) atomicOr(a.err, kErrBounds);
        return p;
    };
    auto load = [&](int32_t page, int stage) -> float {
        constexpr int LANES = R::ROW / 16, PER = 32 / LANES;
        const int64_t row = (int64_t)max(page, 0) * a.hkv + h;
        const uint32_t to = smem_u32(&ring_s[warp][stage * R::STAGE]);
#pragma unroll
        for (int i = 0; i < 16 / PER; ++i) {
            const int r = i * PER + lane / LANES, x = lane % LANES;
            const int64_t at = __shfl_sync(0xffffffffu, row, r);
            copy_async16(to + R::at(r, x), a.codes + at * R::ROW + x * 16, true);
        }
        const int e = min(max((int)__ldg(a.exps + row), -100), 100);
        return page >= 0 ? __uint_as_float((uint32_t)(127 + e) << 23) : 0.f;  // (0: none)
    };
    // two steps' codes are on their way, the page of the one behind them found
    float unit[R::STAGES];
    int32_t page = find(base);
#pragma unroll
    for (int u = 0; u < R::STAGES; ++u) {
        unit[u] = load(page, u);
        copy_async_commit();
        page = find(base + (u + 1) * step);
    }
    for (int x = 0; x < 8 / padded; ++x)
        stage_query<D, FP8>(a, st.q0 + st.i0 + min(x, st.queries - 1), h, x < st.queries, padded, x * padded,
                            [&](int col, int ch, __half2 r0, __half2 r1) {
                                // channels [ch, ch + 4): word (ch % 16) / 4 of lane (ch / 16) % 4 and load ch / 64, two
                                // words a contraction
                                const int k = ch / 64 * 2 + ch % 16 / 8;
                                uint32_t v;  // the four as bytes, then by their signs
                                asm("{\n\t.reg .b32 t;\n\t"
                                    "cvt.pack.sat.s8.s32.b32 t, %2, %1, 0;\n\t"
                                    "cvt.pack.sat.s8.s32.b32 %0, %4, %3, t;\n\t}"
                                    : "=r"(v)
                                    : "r"(__half2int_rn(__low2half(r1))), "r"(__half2int_rn(__high2half(r1))),
                                      "r"(__half2int_rn(__low2half(r0))), "r"(__half2int_rn(__high2half(r0))));
                                const uint32_t less = (v >> 7 & 0x01010101u) * 255u;
                                const uint32_t up = v & ~less, down = v & less;
                                uint2* to = &frag_s[warp][k][col * 4 + ch / 16 % 4];
                                if (ch % 8) to[0].y = up, to[STEPS / 2 * 32].y = down;
                                else to[0].x = up, to[STEPS / 2 * 32].x = down;
                            });
    __syncwarp();
    uint2 q[STEPS];
#pragma unroll
    for (int k = 0; k < STEPS; ++k) q[k] = frag_s[warp][k][lane];
    for (; base < pages; base += 2 * step) {
#pragma unroll
        for (int u = 0; u < R::STAGES; ++u) {
            const int from = base + u * step;
            if (from >= pages) break;
            copy_async_wait<R::STAGES - 1>();
            __syncwarp();
            const uint8_t* ring = &ring_s[warp][u * R::STAGE];
            int d[2][4] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
            for (int k = 0; k < STEPS; k += 2) {
                const uint4 v = *reinterpret_cast<const uint4*>(ring + R::at(g, k / 2 * 4 + c));
                const uint4 w = *reinterpret_cast<const uint4*>(ring + R::at(g + 8, k / 2 * 4 + c));
                mma16832(d[0], v.x, w.x, v.y, w.y, q[k]);
                mma16832(d[1], v.z, w.z, v.w, w.w, q[k + 1]);
            }
            const float now = unit[u];
            __syncwarp();  // (every lane has read the stage)
            if (from + 2 * step < pages) {
                unit[u] = load(page, u);
                page = find(from + 3 * step);
            }
            copy_async_commit();
            const float units[2] = {__shfl_sync(0xffffffffu, now, g), __shfl_sync(0xffffffffu, now, g + 8)};
            float f[4], best[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = (float)(d[0][i] + d[1][i]);
            store_scores(a, st, h, padded, from, 0, units, f, best);
        }
    }
    copy_async_wait<0>();
}

// Some queries: up to eight tiles of columns, four at a time, chains of contractions that do not wait for one another.
template <int D, bool FP8>
__global__ void __launch_bounds__(kScoreThreads, 3) pick_score_kernel(const __grid_constant__ PickArgs a, int blocks)
{
    constexpr int STEPS = 2 * D / 16, GROUP = 4;            // contractions of 16 channels
    extern __shared__ __align__(16) uint2 frag_s[];         // [tile][step][lane]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane & 3;
    const int h = blockIdx.y, b = blockIdx.z;
    griddep_wait();
    griddep_launch_dependents();
    const int padded = padded_group(a.group);
    const ScoreTile st = score_tile(a, b, 0, kScoreCols / padded);
    const int step = blocks * kScorePages;
    int base = blockIdx.x * kScorePages + warp * 16;
    if (blockIdx.x * kScorePages >= st.pages) return;
    const int tiles = (st.queries * padded + 7) / 8;
    int32_t page[2];
    PageCodes<D> next;
    find_pages(a, b, base, st.pages, page);
    next.load(a, page, h, c);
    find_pages(a, b, base + step, st.pages, page);
    for (int x = warp; x < tiles * 8 / padded; x += kScoreThreads / 32)  // (zeros behind the last query)
        stage_query<D, FP8>(a, st.q0 + st.i0 + min(x, st.queries - 1), h, x < st.queries, padded, x * padded,
                            [&](int col, int ch, __half2 r0, __half2 r1) {
                                // channels [ch, ch + 4): word (ch % 16) / 4 of lane (ch / 16) % 4 and load ch / 64
                                const int k = ch / 64 * 4 + ch % 16 / 4;
                                uint2* to = frag_s + ((col >> 3) * STEPS + k) * 32 + (col & 7) * 4 + ch / 16 % 4;
                                const __half2 zero = bits_h2(0u);
                                to[0] = make_uint2(h2_bits(__hmax2(r0, zero)), h2_bits(__hmax2(r1, zero)));
                                to[STEPS / 2 * 32] = make_uint2(h2_bits(__hmin2(r0, zero)), h2_bits(__hmin2(r1, zero)));
                            });
    __syncthreads();
    for (; base < st.pages; base += step) {
        const PageCodes<D> now = next;
        uint32_t f[STEPS][4];
#pragma unroll
        for (int k = 0; k < STEPS; ++k) now.operand(k, f[k]);
        if (base + step < st.pages) {
            next.load(a, page, h, c);
            find_pages(a, b, base + 2 * step, st.pages, page);
        }
        float best[2] = {-INFINITY, -INFINITY};
        for (int x0 = 0; x0 < tiles; x0 += GROUP) {
            float d[GROUP][4];
#pragma unroll
            for (int u = 0; u < GROUP; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) d[u][i] = 0.f;
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
#pragma unroll
                for (int u = 0; u < GROUP; ++u)  // (a tile behind the last: that one again)
                    mma16816(d[u], f[k], frag_s[(min(x0 + u, tiles - 1) * STEPS + k) * 32 + lane]);
#pragma unroll
            for (int u = 0; u < GROUP; ++u)
                if (x0 + u < tiles) store_scores(a, st, h, padded, base, x0 + u, now.unit, d[u], best);
        }
    }
}

constexpr int kKeep = 16;  // keys of a thread that stay in registers

// The pages of a query and key head, by WARPS warps (one: four such pairs a CTA).
template <int WARPS>
__global__ void __launch_bounds__(WARPS == 1 ? 128 : 32 * WARPS) pick_select_kernel(const __grid_constant__ PickArgs a)
{
    constexpr int T = 32 * WARPS;
    constexpr int BITS = WARPS == 1 ? 6 : 8, BUCKETS = 1 << BITS;
    __shared__ int count_s[WARPS == 1 ? 4 * BUCKETS : BUCKETS];
    __shared__ uint32_t range_s[2][WARPS];
    __shared__ int before_s[2][WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = WARPS == 1 ? lane : threadIdx.x;
    griddep_wait();
    griddep_launch_dependents();
    const int64_t pair = WARPS == 1 ? (int64_t)blockIdx.x * 4 + warp : (int64_t)blockIdx.x;
    if (pair >= a.rows * a.hkv) return;
    const int64_t r = pair / a.hkv;
    int b = (int)r, t1 = (int)r + 1;
    if (!a.single) {
        b = find_request(a.off, a.batch, r);
        t1 = __ldg(a.off + b + 1);
    }
    bool bad;
    const int len = cache_len(__ldg(a.lens + b), a.limit, bad);
    if (bad && tid == 0) atomicOr(a.err, kErrBounds);
    const int64_t pos = min((int64_t)len - t1 + r, (int64_t)len - 1);  // of the query
    const int pages = pos < 0 ? 0 : (int)(pos >> a.page_shift) + 1;
    int32_t* out = a.picked + pair * a.budget;
    if (pages <= a.budget) {
        for (int x = tid; x < a.budget; x += T) out[x] = x < pages ? x : -1;
        return;
    }
    const uint32_t* keys = a.keys + pair * a.key_stride;
    auto key_at = [&](int j) -> uint32_t {
        return j >= pages ? 0u : (j < a.sink || j >= pages - a.recent ? 0xFFFFFFFFu : __ldcg(keys + j));
    };
    // pages j = part * chunk + i * 32 + lane of warp `part`
    const int chunk = WARPS == 1 ? (pages + 31) & ~31 : ((pages + T - 1) / T) * 32;
    const int first = (WARPS == 1 ? 0 : warp * chunk), steps = chunk / 32;
    uint32_t k[kKeep];
    uint32_t top = 0u, low = 0xFFFFFFFFu;
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
        k[i] = i < steps ? key_at(first + i * 32 + lane) : 0u;
        if (k[i] != 0u && k[i] != 0xFFFFFFFFu) top = max(top, k[i]), low = min(low, k[i]);
    }
    for (int i = kKeep; i < steps; ++i) {
        const uint32_t v = key_at(first + i * 32 + lane);
        if (v != 0u && v != 0xFFFFFFFFu) top = max(top, v), low = min(low, v);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    low = __reduce_min_sync(0xffffffffu, low);
    if constexpr (WARPS > 1) {
        if (lane == 0) range_s[0][warp] = top, range_s[1][warp] = low;
        __syncthreads();
#pragma unroll 1
        for (int w = 0; w < WARPS; ++w) top = max(top, range_s[0][w]), low = min(low, range_s[1][w]);
    }
    auto visit = [&](auto f) {
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            if (i >= steps) break;
            f(first + i * 32 + lane, k[i]);
        }
        for (int i = kKeep; i < steps; ++i) f(first + i * 32 + lane, key_at(first + i * 32 + lane));
    };
    // ---- x, which the budget's keys reach: the keys between the smallest and the largest counted in buckets of a power
    // of two, the bucket that the budget ends in counted in finer ones, and so on: with 64 buckets up to six times (keys
    // that differ in all 32 bits, as scores of both signs nearly do: by 26, 20, 14, 8, 2 and 0 bits), with 256 four times
    int want = a.budget - a.sink - a.recent;  // of the keys that are not picked anyway
    uint32_t x = 0xFFFFFFFFu;
    bool exact = true;  // all that reach x are taken
    if (want > 0) {
        uint32_t lo = low, hi = top;
        int* bucket = count_s + (WARPS == 1 ? warp * BUCKETS : 0);
        auto sync = [&]() {
            if constexpr (WARPS == 1) __syncwarp();
            else __syncthreads();
        };
        for (;;) {
            const int shift = max(0, 32 - __clz(hi - lo) - BITS);
            for (int i = tid; i < BUCKETS; i += T) bucket[i] = 0;
            sync();
            visit([&](int, uint32_t v) {
                if (v >= lo && v <= hi) atomicAdd(bucket + ((v - lo) >> shift), 1);
            });
            sync();
            // by every warp: lane i has the buckets [i * PER, (i + 1) * PER), counted from the last one down
            constexpr int PER = BUCKETS / 32;
            int mine[PER], sum = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) mine[i] = bucket[lane * PER + i], sum += mine[i];
            int from = sum;  // of this lane's buckets and those behind them
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_down_sync(0xffffffffu, from, d);
                if (lane + d < 32) from += y;
            }
            int above = from - sum, at = -1, in = 0;
#pragma unroll
            for (int i = PER - 1; i >= 0; --i) {
                if (at < 0 && above < want && above + mine[i] >= want) at = lane * PER + i, in = mine[i];
                if (at < 0) above += mine[i];
            }
            const int who = __ffs(__ballot_sync(0xffffffffu, at >= 0)) - 1;
            at = __shfl_sync(0xffffffffu, at, who);
            in = __shfl_sync(0xffffffffu, in, who);
            want -= __shfl_sync(0xffffffffu, above, who);
            lo += (uint32_t)at << shift;
            x = lo;
            exact = in == want;
            if (exact || shift == 0) break;
            hi = lo + ((1u << shift) - 1u);  // (no more than the largest key and a bucket, 2^26: below 2^32)
            sync();  // (the counts have been read)
        }
    }
    // ---- keys above x, and the first of those at it (where x was reached by `budget` keys: all that reach it)
    const uint32_t above = exact ? x - 1u : x;
    int mine = 0, ties = 0;  // of this warp
    visit([&](int, uint32_t v) {
        mine += __popc(__ballot_sync(0xffffffffu, v > above));
        ties += exact ? 0 : __popc(__ballot_sync(0xffffffffu, v == x));
    });
    int all = mine, my_at = 0, ties_before = 0;
    if constexpr (WARPS > 1) {
        if (lane == 0) before_s[0][warp] = mine, before_s[1][warp] = ties;
        __syncthreads();
        all = 0;
#pragma unroll 1
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) my_at += before_s[0][w], ties_before += before_s[1][w];
            all += before_s[0][w];
        }
    }
    // of ties; keys that the scores' kernel gave up on can be anything: then none behind the list, and none before it
    const int room = max(0, a.budget - all);
    my_at += min(ties_before, room);
    visit([&](int j, uint32_t v) {
        const uint32_t tie = exact ? 0u : __ballot_sync(0xffffffffu, v == x);
        const uint32_t below = (1u << lane) - 1u;
        const bool take = v > above || ((tie >> lane & 1u) && ties_before + __popc(tie & below) < room);
        const uint32_t m = __ballot_sync(0xffffffffu, take);
        if (take && my_at + __popc(m & below) < a.budget) out[my_at + __popc(m & below)] = j;
        my_at += __popc(m);
        ties_before += __popc(tie);
    });
}

template <int D, bool FP8>
cudaError_t launch_scores(const PickArgs& a, int max_t, int max_pages, int num_sms, cudaLaunchConfig_t cfg)
{
    const int padded = padded_group(a.group);
    cfg.blockDim = dim3(kScoreThreads, 1, 1);
    if (max_t * padded <= 8) {  // one tile of columns
        const int groups = a.hkv / score_heads(a.hkv), step = kScorePages / score_heads(a.hkv);
        // as many CTAs as run at once: each takes as long to start as for ten steps
        const int64_t slots = std::max<int64_t>(2 * (int64_t)a.batch, (int64_t)num_sms * 5 / groups);
        cfg.gridDim = dim3((unsigned)std::min<int64_t>(slots, (int64_t)a.batch * ((max_pages + step - 1) / step)),
                           (unsigned)groups, 1);
        return cudaLaunchKernelEx(&cfg, pick_token_kernel<D, FP8>, a, (int)cfg.gridDim.x);
    }
    constexpr int kTileBytes = 2 * D / 16 * 32 * (int)sizeof(uint2);
    static_assert(kScoreCols / 8 * kTileBytes <= 48 * 1024, "the columns fit shared memory as it is");
    cfg.dynamicSmemBytes = (size_t)((max_t * padded + 7) / 8) * kTileBytes;
    // CTAs of a request's pages: 64 pages at a time, two rounds of what runs at once
    const int64_t others = (int64_t)a.hkv * a.batch, steps = (max_pages + kScorePages - 1) / kScorePages;
    const int64_t times = std::max<int64_t>(1, std::min<int64_t>(steps, others * steps / (2 * 3 * (int64_t)num_sms)));
    const int64_t blocks = (steps + times - 1) / times;
    cfg.gridDim = dim3((unsigned)blocks, (unsigned)a.hkv, (unsigned)a.batch);
    return cudaLaunchKernelEx(&cfg, pick_score_kernel<D, FP8>, a, (int)blocks);
}

}  // namespace

int64_t pick_key_stride(int64_t max_len, int page_shift, int budget)
{
    const int64_t pages = (max_len + (1 << page_shift) - 1) >> page_shift;
    return pages <= budget ? 0 : (pages + 31) & ~31ll;
}

int pick_col_tiles(int64_t max_t, int group)
{
    if (max_t * padded_group(group) <= kScoreCols) return max_t > 0;
    const int per = pick_tile_queries(group);
    return (int)((max_t + per - 1) / per);
}

cudaError_t launch_cache_pick(const PickArgs& a, int head_dim, bool fp8, int max_t, int max_len, int num_sms,
                              cudaStream_t stream, int32_t* launches)
{
    *launches = 0;
    if (a.rows == 0) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.stream = stream;
    const int max_pages = (int)(((int64_t)max_len + (1 << a.page_shift) - 1) >> a.page_shift);
    cudaError_t e = cudaSuccess;
    if (a.key_stride > 0) {
        const int64_t columns = (int64_t)max_t * padded_group(a.group);
        if (columns > kScoreCols) e = launch_pick_tiles(a, head_dim, fp8, max_t, max_pages, num_sms, stream);
        else e = fp8 ? launch_scores<128, true>(a, max_t, max_pages, num_sms, cfg)
                : (head_dim == 128 ? launch_scores<128, false>(a, max_t, max_pages, num_sms, cfg)
                                   : launch_scores<64, false>(a, max_t, max_pages, num_sms, cfg));
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    const int64_t pairs = a.rows * a.hkv;
    cfg.dynamicSmemBytes = 0;
    if (max_pages <= 32 * kKeep) {
        cfg.gridDim = dim3((unsigned)((pairs + 3) / 4), 1, 1);
        cfg.blockDim = dim3(128, 1, 1);
        e = cudaLaunchKernelEx(&cfg, pick_select_kernel<1>, a);
    } else {
        cfg.gridDim = dim3((unsigned)pairs, 1, 1);
        if (max_pages <= 32 * 8 * kKeep) {
            cfg.blockDim = dim3(32 * 8, 1, 1);
            e = cudaLaunchKernelEx(&cfg, pick_select_kernel<8>, a);
        } else {
            cfg.blockDim = dim3(32 * 32, 1, 1);
            e = cudaLaunchKernelEx(&cfg, pick_select_kernel<32>, a);
        }
    }
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace lvs
