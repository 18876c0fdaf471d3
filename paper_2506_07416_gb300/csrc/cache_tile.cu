// Attention over the 4-bit cache for calls of many rows (drafts of grouped heads, chunks of
// a prompt), on the fifth-generation tensor cores.
//
// A CTA takes a key head of a request, NR tiles of 128 rows (a row is a query with one of
// the head's query heads) and all keys that they see, or one chunk of them, 128 keys at a
// time. Its warps:
//   four make f16 values of codes and scales (exact) and lay them out for the
//     contractions: K rows with their channels, V transposed, so that both are K-major
//     128-byte swizzled operands; the next tile's codes are on their way meanwhile;
//   one issues S = Q K^T of each row tile into 128 columns of tensor memory and, once the probabilities
//     are there, O += P V with P read from tensor memory;
//   4 NR hold a row a thread: they read S twice (its largest score, then the
//     exponentials), write P as f16 over S, and keep the row's reference and sum. A
//     reference moves only when a score passes it by 15; O is then rescaled in place.
// What bounds it: the chain of a row tile. The exponentials take at least 1024 clocks of an
// SM for 128 x 128, each contraction 516, and S, softmax and the product with V follow one
// another: about 3600 clocks for a tile of 256 rows by 128 keys. So two row tiles are always in flight:
//   NR = 1, up to 128 rows: two CTAs on an SM, 256 columns and at most 113 KB each, one stage of K and V
//   NR = 2: one CTA with two row tiles, for which K and V are made once, in two stages
// (192 rows of 16 requests of 4096 keys: 72 us with NR = 2 and 97 with 1). Start and end of a CTA take about as
// long as seven of those tiles. A chunk of a prompt, 1023 and 873 queries of 28 / 4 heads over 5928 and 6517 keys
// (156 GFLOP): 186 us, the tensor pipe active half of the time: its 208 nearly equal tiles of 256 rows take two rounds of
// 152 SMs where 1.37 would do, and a CTA's own chain the rest; with the contractions of the warp-wide instructions 617.
// Dropped for that chunk: P and the product by halves of a tile's keys (233 us where the whole took 224), S by
// halves too (263), two threads a row (245 against 218), a quarter of the exponentials by a polynomial (241 against
// 217): a warp's own latencies bound the softmax, and the warps share their SM with those that make the values.

#include <type_traits>

#include "cache_attend.cuh"
#include "pipe.cuh"

namespace lvs {

namespace {

constexpr int kTileKeys = 128;
// Barriers: operands of a stage written, operands of a stage read (two stages), and for each
// of two row tiles scores there, probabilities there, their product there.
enum { B_K_FULL = 0, B_V_FULL = 2, B_K_FREE = 4, B_V_FREE = 6, B_S_FULL = 8, B_P_FULL = 10, B_PV_DONE = 12, B_DRAIN = 14, B_Q_FULL = 15, B_COUNT };

// Warps of a CTA of NR row tiles: 4 NR for the rows, 4 for the values, 1 for the contractions.
template <int NR>
constexpr int kTileThreads = 32 * (4 * NR + 5);

template <int D, int NR>
struct TileLayout {
    static constexpr int ATOM = 128 * 128;                 // 128 rows of 64 f16
    static constexpr int STAGES = NR;                      // of K and V
    static constexpr int ROWS = D / 64 * ATOM;             // a row tile, or a stage of K: [D / 64] atoms
    static constexpr int VALUES = 2 * D * 128;             // a stage of V: [2] halves of the keys, D channels x 64 keys
    static constexpr int Q = 0;
    static constexpr int K = Q + NR * ROWS;
    static constexpr int V = K + STAGES * ROWS;
    static constexpr int BAR = V + STAGES * VALUES;
    static constexpr int MISC = BAR + 8 * B_COUNT;
    // at least 77 KB (115): no more than two CTAs of 256 columns each (one of 512) on an SM
    static constexpr int NEED = MISC + 16 + 1024, LEAST = NR == 1 ? 77 * 1024 : 115 * 1024;
    static constexpr int ALLOC = NEED > LEAST ? NEED : LEAST;
};

// O += P V: A from tensor memory
__device__ __forceinline__ void mma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// 32 rows of the tile (row0 + lane; my_at: where the lane's row starts in q, -1: zeros) as f16 into shared
// memory, by a warp, scaled as in the kernel for few rows (a power of two that puts a row's largest magnitude at about
// 2^10; NaN throughout where a channel is infinite or NaN). Returns what undoes the scaling of the lane's row. A
// row's 16-byte parts go to neighbouring lanes, all rows on their way at once: with a row a lane a
// CTA's start took several us more (a chunk of a prompt 218 and not 208 us).
template <int D, bool FP8>
__device__ __forceinline__ float stage_rows(const void* q, int64_t my_at, uint32_t q_s, int row0)
{
    constexpr int LANES = D * (FP8 ? 1 : 2) / 16, PER = 32 / LANES, STEPS = 32 / PER;
    const int lane = threadIdx.x & 31, sub = lane % LANES;
    float back = 1.f;
    uint4 v[STEPS];
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
        const int64_t at = __shfl_sync(0xffffffffu, my_at, u * PER + lane / LANES);
        v[u] = make_uint4(0u, 0u, 0u, 0u);
        if (at >= 0)
            v[u] = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(q) + at * (FP8 ? 1 : 2)) + sub);
    }
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
        const int row = row0 + u * PER + lane / LANES;
        auto put = [&](int x, uint32_t f0, uint32_t f1, uint32_t f2, uint32_t f3) {  // 8 channels
            st_shared16(q_s + (x >> 3) * TileLayout<D, 1>::ATOM + row * 128 + (((x & 7) ^ (row & 7)) << 4), f0, f1, f2,
                        f3);
        };
        const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
        if constexpr (FP8) {
            uint32_t f[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                __half2 x[2];
                e4m3x4_value(w[k], x);
                f[2 * k] = h2_bits(x[0]), f[2 * k + 1] = h2_bits(x[1]);
            }
            put(2 * sub, f[0], f[1], f[2], f[3]);
            put(2 * sub + 1, f[4], f[5], f[6], f[7]);
        } else {
            // the largest magnitude's bits (as integers they order the magnitudes, NaN above infinity above the rest)
            uint32_t top = __vmaxu2(__vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu),
                                    __vmaxu2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
            top = max(top & 0xFFFFu, top >> 16);
#pragma unroll
            for (int d = 1; d < LANES; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
            const int e = min(264 - (int)(top >> 7), 253);
            const float up = __int_as_float(top >= 0x7F80u ? 0x7FC00000 : e << 23);
            uint32_t f[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                f[k] = pack_h2(__uint_as_float(w[k] << 16) * up, __uint_as_float(w[k] & 0xFFFF0000u) * up);
            put(sub, f[0], f[1], f[2], f[3]);
            const float mine =
                __shfl_sync(0xffffffffu, __int_as_float((254 - e) << 23), lane % PER * LANES);
            if (lane / PER == u) back = mine;
        }
    }
    return back;
}

// A thread's part of a tile's K: 32 channels (D = 64: 16) of each of four keys, 8 apart: of warp
// w of four the channels [c * D/4, ..), c = lane / 8, of the keys w * 32 + lane % 8 + 8 i. A warp's
// loads then cover whole rows, and the stores of eight neighbouring lanes all banks.
template <int D>
struct KPart {
    uint4 code[4];   // D = 64: the first two words
    uint32_t scale[4];

    // from the pages p0 and p1 of the warp's two groups of 16 keys (-1: zeros)
    __device__ __forceinline__ void load(const CachePages& C, int32_t p0, int32_t p1, int h, int j0, int w)
    {
        const int lane = threadIdx.x & 31, c = lane >> 3, smask = (1 << C.page_shift) - 1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t page = i < 2 ? p0 : p1;
            code[i] = make_uint4(0u, 0u, 0u, 0u);
            scale[i] = 0u;
            if (page >= 0) {
                const int64_t at =
                    cache_row(page, C.hkv, h, C.page_shift, (j0 + w * 32 + (lane & 7) + 8 * i) & smask);
                if constexpr (D == 128) {
                    code[i] = __ldg(reinterpret_cast<const uint4*>(C.codes[0] + at * 64 + c * 16));
                    scale[i] = __ldg(reinterpret_cast<const uint16_t*>(C.scales[0] + at * 8 + c * 2));
                } else {
                    const uint2 v = __ldg(reinterpret_cast<const uint2*>(C.codes[0] + at * 32 + c * 8));
                    code[i].x = v.x, code[i].y = v.y;
                    scale[i] = __ldg(C.scales[0] + at * 4 + c);
                }
            }
        }
    }

    // as f16 values into a K-major operand of 128 keys
    __device__ __forceinline__ void store(uint32_t k_s, int w) const
    {
        const int lane = threadIdx.x & 31, c = lane >> 3;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = w * 32 + (lane & 7) + 8 * i;
            const uint32_t words[4] = {code[i].x, code[i].y, code[i].z, code[i].w};
            const __half2 sc = e4m3x2_value(scale[i]);
            const __half2 sb[2] = {__low2half2(sc), D == 128 ? __high2half2(sc) : __low2half2(sc)};
#pragma unroll
            for (int q = 0; q < D / 32; ++q) {  // 8 channels
                __half2 x[4];
                e2m1x8_value(words[q], x);
                const __half2 s = sb[q / 2];
                const int u = c * (D / 32) + q;
                st_shared16(k_s + (u >> 3) * (128 * 128) + key * 128 + (((u & 7) ^ (key & 7)) << 4),
                            h2_bits(__hmul2(x[0], s)), h2_bits(__hmul2(x[1], s)), h2_bits(__hmul2(x[2], s)),
                            h2_bits(__hmul2(x[3], s)));
            }
        }
    }
};
// ... and of its V: 8 neighbouring keys, the 16 channels of one scale block.
struct VPart {
    uint2 code[8];
    uint32_t scale[8];
};

// PICKED: the rows are whole queries of a tile, and the keys those of the pages that any of them has, in the list's order; a
// key of a page that a row's query has not is as masked. Of 64 or 32 keys that no row of a warp has, the warp
// makes no exponentials. Few rows stand in the tile more than once, so that all four warps make exponentials: drafts of
// 32 ragged requests, 4 to 32 rows a head, 48 pages of 32: 82 us without, 77 with. What bounds those: a tile takes 3000
// clocks of a CTA (1000 are the tensor pipe's, which two CTAs share), half of them the warps that make the values.
// Dropped there: lines fetched into the L2 three tiles ahead and loads in another order (78 us).
template <int D, bool FP8, int NR, bool PICKED = false>
__global__ void __launch_bounds__(kTileThreads<NR>, NR == 1 ? 2 : 1) attend_tile_kernel(const __grid_constant__ AttendArgs a)
{
    using L = TileLayout<D, NR>;
    constexpr int SOFT = 4 * NR, MMA_WARP = SOFT + 4, ST = L::STAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - raw);
    auto BAR = [&](int i) { return base + L::BAR + 8 * i; };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::MISC);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::MISC + 4);
    volatile int* nan_flag = reinterpret_cast<volatile int*>(smem + L::MISC + 8);

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = uniform(tid >> 5);
    // the last rows, which see the most keys, first: 2048 queries over themselves 63 to 49 us, a chunk of a prompt 195 to 186
    const int h = blockIdx.y % a.cache.hkv, tile = (gridDim.y - 1 - blockIdx.y) / a.cache.hkv;
    griddep_wait();
    griddep_launch_dependents();
    int b = blockIdx.z, chunk = kMostKeys, k0 = 0;
    __shared__ int split_s[3];
    QueryTile qt{0, 0, 0};
    const int64_t pick_tile = PICKED ? blockIdx.x / a.pick_chunks : 0;
    const int64_t pick_list = pick_tile * a.cache.hkv + h;
    int listed = 0;  // keys of the list
    if constexpr (PICKED) {
        const int4 head = __ldg(a.list_heads + pick_list);
        qt = QueryTile{uniform(head.x), uniform(head.y), uniform(head.z)};
        if (qt.queries <= 0) return;
        b = qt.b;
        listed = uniform(head.w) << a.cache.page_shift;
        chunk = list_chunk(listed, a.pick_chunks, kTileKeys);
        k0 = min((int)(blockIdx.x % a.pick_chunks) * chunk, listed);
    } else if (a.slots > 0) {
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
    RowTile rt = row_tile(a, b, tile, 128 * NR);
    if constexpr (PICKED) {
        rt.row0 = qt.i0 * a.group + tile * 128 * NR;
        rt.rows = min(128 * NR, qt.queries * a.group - tile * 128 * NR);
    }
    if (rt.rows <= 0) return;
    const int q0 = a.q_off[b];
    const int seen = PICKED ? listed : min(rt.len, rt.last0 + rt.query(rt.row0 + rt.rows - 1) + 1);
    const int k1 = chunk_end(seen, k0, chunk);
    if (!PICKED && k0 >= k1 && a.slots > 0) return;  // (without chunks the tile's zeros are written here, else by the join)
    const int all_see = rt.last0 + rt.query(rt.row0);  // the last key that every row sees
    const int4* list = PICKED ? a.lists + pick_list * a.list_cap : nullptr;  // page in the pool, page of the request
    const int n_tiles = uniform(k1 > k0 ? (k1 - k0 + kTileKeys - 1) / kTileKeys : 0);
    // PICKED: up to 64 rows stand in the tile twice, up to 32 four times; each copy of a row makes the probabilities of its
    // own half or quarter of a tile's keys, the others' being 0, and the copies' sums are joined at the end
    const int copies = PICKED && NR == 1 ? uniform(rt.rows <= 32 ? 4 : (rt.rows <= 64 ? 2 : 1)) : 1;
    const int copy_rows = 128 * NR / copies;
    const int live = copies > 1 ? 4 : (rt.rows + 31) / 32;  // softmax warps with rows
    const int row_tiles = NR > 1 ? uniform((rt.rows + 127) / 128) : 1;

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(BAR(B_K_FULL + i), 4);
            mbar_init(BAR(B_V_FULL + i), 4);
            mbar_init(BAR(B_K_FREE + i), 1);
            mbar_init(BAR(B_V_FREE + i), 1);
            mbar_init(BAR(B_S_FULL + i), 1);
            mbar_init(BAR(B_P_FULL + i), (uint32_t)max(1, min(4, live - 4 * i)));
            mbar_init(BAR(B_PV_DONE + i), 1);
        }
        mbar_init(BAR(B_DRAIN), 1);
        mbar_init(BAR(B_Q_FULL), 4 * (uint32_t)row_tiles);
        *abort_flag = 0;
        *nan_flag = 0;
        fence_mbar_init_cluster();
    }
    if (warp == MMA_WARP) {
        tmem_alloc(smem_u32(tmem_slot), 256 * NR);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(*tmem_slot);
    const Ctl ctl{abort_flag, a.err, a.wait_budget};
    float m = kNoRef, l = 0.f;
    const int in_copy = copies > 1 ? tid & (copy_rows - 1) : tid;
    const bool real = tid < 32 * SOFT && in_copy < rt.rows;  // (the softmax warps' threads)
    const int row = rt.row0 + (real ? in_copy : 0), query = rt.query(row);

    const int rtile = warp >> 2;  // the softmax warps' row tile
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    if (warp < SOFT) {
        // ---------------------------------------------------------------- softmax: a row a thread
        float fac = 0.f;
        if (rtile < row_tiles) {  // (rows that are not there are zeros)
            const int64_t at =
                (int64_t)(q0 + query) * a.q_stride + (int64_t)(h * a.group + row - query * a.group) * D;
            fac = row_factor(a.c_log2, stage_rows<D, FP8>(a.q, real ? at : -1, base + L::Q + rtile * L::ROWS,
                                                          (warp & 3) * 32));
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(B_Q_FULL));
        }
        if (warp < live) {
            const uint32_t ts = tmem + lanes + 256 * rtile, to = ts + 128;
            // the last key that the row sees here (PICKED: the last position)
            const int vis = PICKED ? rt.last0 + query : min(rt.last0 + query, k1 - 1);
            // the pages that the row's query has, a bit for each of the list, 32 at a time
            const uint32_t* bits = PICKED ? a.list_bits + (pick_list * a.pick_queries + query - qt.i0) * a.list_words : nullptr;
            uint32_t bit_word = 0u;
            // the groups of 16 keys of a tile that are the copy's
            const uint32_t own = copies == 4 ? 3u << 2 * warp : (copies == 2 ? 15u << 4 * (warp >> 1) : 255u);
            int next_pos = 0;  // PICKED: position of the group's first key
            // page of a tile's group of 16 keys (lanes 0 to 7); groups without one are as masked
            auto page_of = [&](int t) -> int32_t {
                const int j = k0 + t * kTileKeys + lane * 16;
                if constexpr (PICKED) {
                    if (lane >= 8) return 0;
                    if (j >= k1) return -1;
                    const int4 v = __ldg(list + (j >> a.cache.page_shift));
                    next_pos = (v.y << a.cache.page_shift) + (j & ((1 << a.cache.page_shift) - 1));
                    return v.x;
                }
                return lane < 8 && j < k1
                           ? cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, b, j)
                           : 0;
            };
            auto rows = [&](auto rounded) {  // rounded: the scores, as they are read
                const float unit = rounded.value ? 1.f : fac;
                const float2 fac2 = make_float2(unit, unit);
                int32_t next_page = page_of(0);
                for (int t = 0; t < n_tiles; ++t) {
                    const int j0 = k0 + t * kTileKeys;
                    const uint32_t gone = __ballot_sync(0xffffffffu, next_page < 0);
                    const int pos = next_pos;
                    // PICKED: whether some key is behind a row's position; the groups that the row has, and that any of the warp has
                    const bool late = PICKED && __any_sync(0xffffffffu, lane < 8 && next_page >= 0 && pos + 15 > all_see);
                    [[maybe_unused]] uint32_t has = 0u, any_has = 0u;
                    if constexpr (PICKED) {
                        const int shift = a.cache.page_shift, x0 = j0 >> shift;
                        if (t == 0 || (x0 & 31) == 0) bit_word = real ? __ldg(bits + (x0 >> 5)) : 0u;
                        const uint32_t b8 = bit_word >> (x0 & 31);
#pragma unroll
                        for (int g = 0; g < 8; ++g) has |= (b8 >> ((16 * g) >> shift) & 1u) << g;
                        has &= own & ~gone;
                        any_has = __reduce_or_sync(0xffffffffu, has);
                    }
                    next_page = page_of(t + 1);
                    const bool check = PICKED ? late : j0 + kTileKeys > min(k1, all_see + 1) || gone != 0;
                    if (!poll_phase_warp(BAR(B_S_FULL + rtile), (uint32_t)t & 1u, ctl)) break;
                    tc_fence_after();
                    // columns of a chunk of 32 that the row sees, as a mask
                    auto mask_of = [&](int c0) -> uint32_t {
                        if constexpr (PICKED) {
                            uint32_t k = 0u;
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const int n = vis - __shfl_sync(0xffffffffu, pos, c0 / 16 + x) + 1;
                                k |= (n >= 16 ? 0xFFFFu : (n <= 0 ? 0u : (1u << n) - 1u)) << (16 * x);
                            }
                            return k;
                        } else {
                            const int n = vis - (j0 + c0) + 1;
                            uint32_t k = n >= 32 ? 0xFFFFFFFFu : (n <= 0 ? 0u : (1u << n) - 1u);
                            if (gone >> (c0 / 16) & 1u) k &= 0xFFFF0000u;
                            if (gone >> (c0 / 16 + 1) & 1u) k &= 0x0000FFFFu;
                            return k;
                        }
                    };
                    // the columns, STEP at a time from the last on, read for their maximum; the first STEP
                    // are still there when the exponentials are made
                    constexpr int STEP = NR > 1 ? 64 : 32;
                    float mx = -INFINITY;
                    float v[STEP];
                    int held = PICKED ? -1 : 0;  // the first column of those there
                    auto mask = [&](int c0, float* x) {
                        const uint32_t k = mask_of(c0);
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = k >> i & 1u ? x[i] : -INFINITY;
                    };
                    auto read = [&](int c0) {
#pragma unroll
                        for (int x = 0; x < STEP; x += 32) tmem_ld32(ts + c0 + x, v + x);
                        tmem_wait_ld();
                        if constexpr (rounded.value) {
#pragma unroll
                            for (int i = 0; i < STEP; ++i) v[i] *= fac;
                        }
                        if (check) {
#pragma unroll
                            for (int x = 0; x < STEP; x += 32) mask(c0 + x, v + x);
                        }
                    };
#pragma unroll 1
                    for (int c0 = kTileKeys - STEP; c0 >= 0; c0 -= STEP) {
                        if (PICKED && !(any_has >> (c0 / 16) & ((1u << STEP / 16) - 1u))) continue;
                        read(c0);
                        if constexpr (PICKED) {
                            held = c0;
#pragma unroll
                            for (int x = 0; x < STEP / 16; ++x) {
                                const float top = row_max<16>(v + 16 * x);
                                if (has >> (c0 / 16 + x) & 1u) mx = fmaxf(mx, top);
                            }
                        } else {
                            mx = fmaxf(mx, row_max<STEP>(v));
                        }
                    }
                    mx *= unit;  // (> 0, see row_factor)
                    if (__any_sync(0xffffffffu, mx > m + kRefSlack)) {
                        const float mn = fmaxf(m, mx - kRefBelow);
                        const float f = ex2(m - mn);
                        m = mn;
                        l *= f;
                        if (t > 0) {  // (the product with the last tile's values is done: S came behind it)
#pragma unroll 1
                            for (int c0 = 0; c0 < D; c0 += 16) {
                                float x[16];
                                tmem_ld16(to + c0, x);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 16; ++i) x[i] *= f;
                                tmem_st16(to + c0, x);
                            }
                            tmem_wait_st();
                        }
                    }
                    const float2 nm2 = make_float2(-m, -m);
                    float2 s0 = make_float2(0.f, 0.f), s1 = make_float2(0.f, 0.f);
                    auto chunk_of = [&](int c0, const float* x_) {
                        float p[16];
                        if constexpr (PICKED) {
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const bool mine = has >> (c0 / 16 + x) & 1u;
                                const uint32_t keep = mine ? 0xFFFFFFFFu : 0u;
                                float2 t0 = make_float2(0.f, 0.f), t1 = t0;
#pragma unroll
                                for (int i = 16 * x; i < 16 * x + 16; i += 4) {
                                    const float2 x0 = ffma2(make_float2(x_[i], x_[i + 1]), fac2, nm2);
                                    const float2 x1 = ffma2(make_float2(x_[i + 2], x_[i + 3]), fac2, nm2);
                                    const float2 p0 = make_float2(ex2(x0.x), ex2(x0.y)), p1 = make_float2(ex2(x1.x), ex2(x1.y));
                                    t0 = fadd2(t0, p0);
                                    t1 = fadd2(t1, p1);
                                    p[i / 2] = __uint_as_float(pack_h2(p0.x, p0.y) & keep);
                                    p[i / 2 + 1] = __uint_as_float(pack_h2(p1.x, p1.y) & keep);
                                }
                                if (mine) s0 = fadd2(s0, t0), s1 = fadd2(s1, t1);
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; i += 4) {
                                const float2 x0 = ffma2(make_float2(x_[i], x_[i + 1]), fac2, nm2);
                                const float2 x1 = ffma2(make_float2(x_[i + 2], x_[i + 3]), fac2, nm2);
                                const float2 p0 = make_float2(ex2(x0.x), ex2(x0.y)), p1 = make_float2(ex2(x1.x), ex2(x1.y));
                                s0 = fadd2(s0, p0);
                                s1 = fadd2(s1, p1);
                                p[i / 2] = __uint_as_float(pack_h2(p0.x, p0.y));
                                p[i / 2 + 1] = __uint_as_float(pack_h2(p1.x, p1.y));
                            }
                        }
                        tmem_st16(ts + c0 / 2, p);
                    };
                    // (P of columns c is written to the columns from c / 2 on, which have been read)
#pragma unroll 1
                    for (int c0 = 0; c0 < kTileKeys; c0 += STEP) {
                        if (PICKED && !(any_has >> (c0 / 16) & ((1u << STEP / 16) - 1u))) {
                            const float none[16] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f,
                                                    0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int x = 0; x < STEP; x += 32) tmem_st16(ts + (c0 + x) / 2, none);
                            continue;
                        }
                        if (c0 != held) read(c0);
#pragma unroll
                        for (int x = 0; x < STEP; x += 32) chunk_of(c0 + x, v + x);
                    }
                    l += (s0.x + s0.y) + (s1.x + s1.y);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(BAR(B_P_FULL + rtile));
                }
            };
            if (__any_sync(0xffffffffu, fac > kFusedFactor)) rows(std::true_type{});
            else rows(std::false_type{});
        }
    } else if (warp < MMA_WARP) {
        // ---------------------------------------------------------------- codes to values
        const int w = warp - SOFT;
        const CachePages& C = a.cache;
        const int smask = (1 << C.page_shift) - 1;
        // V: keys kg * 8 .., block vb: a warp's loads cover whole rows, and the stores of eight
        // neighbouring lanes, four groups of keys of two blocks, all banks: odd blocks take their
        // channels 4 to 7 first (their words are turned by half)
        const int kg = 4 * w + (lane & 3), vb = lane >> 2, turn = (vb & 1) * 4;
        const uint32_t v_at = (kg >> 3) * (D * 128) + vb * 16 * 128;
        const uint32_t v_x = (uint32_t)(turn << 7 | ((kg & 7) ^ turn) << 4);
        const bool v_part = vb < D / 16;
        int pv_pos = 0;  // PICKED: position of the thread's first key of V
        auto page_at = [&](int j) -> int32_t {
            if constexpr (PICKED) return j < k1 ? __ldg(&list[j >> C.page_shift].x) : -1;
            else return j < k1 ? cache_page(C.table, C.width, C.num_pages, C.page_shift, b, j) : -1;
        };
        auto report = [&](int32_t page, int j) {
            if (!PICKED && page < 0 && j < k1) atomicOr(a.err, kErrBounds);
        };
        auto load_v = [&](VPart& x, int32_t page, int j0) {
            const int64_t at = cache_row(page >= 0 ? page : 0, C.hkv, h, C.page_shift, (j0 + kg * 8) & smask);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x.code[i] = make_uint2(0u, 0u);
                x.scale[i] = 0u;
                if (page >= 0 && v_part) {
                    x.code[i] = __ldg(reinterpret_cast<const uint2*>(C.codes[1] + (at + i) * (D / 2) + vb * 8));
                    x.scale[i] = __ldg(C.scales[1] + (at + i) * (D / 16) + vb);
                }
            }
        };
        // pages of the thread's keys (a group of 16 lies in one), a tile ahead of the loads of the codes
        int32_t pk0, pk1, pv;
        int next_pv_page = 0;  // PICKED: page of the request of the thread's next keys of V
        auto pos_of = [&](int j0) { return PICKED ? (next_pv_page << C.page_shift) + ((j0 + kg * 8) & smask) : 0; };
        auto pages = [&](int j0) {
            pk0 = page_at(j0 + w * 32);
            pk1 = page_at(j0 + w * 32 + 16);
            if constexpr (PICKED) {
                // (both words at once, and nothing that waits for them here)
                const int j = j0 + kg * 8;
                const int2 e = j < k1 ? __ldg(reinterpret_cast<const int2*>(list + (j >> C.page_shift))) : make_int2(-1, 0);
                pv = e.x;
                next_pv_page = e.y;
            } else {
                pv = page_at(j0 + kg * 8);
            }
        };
        auto report_pages = [&](int j0) {
            if ((lane & 15) == 0) report(lane ? pk1 : pk0, j0 + w * 32 + lane);
        };
        KPart<D> kp;
        VPart vp;
        pages(k0);
        report_pages(k0);
        kp.load(C, pk0, pk1, h, k0, w);
        load_v(vp, pv, k0);
        pv_pos = pos_of(k0);
        pages(k0 + kTileKeys);
        for (int t = 0; t < n_tiles; ++t) {
            const int j0 = k0 + t * kTileKeys, jn = j0 + kTileKeys;
            const bool more = t + 1 < n_tiles;
            if (a.stall && t == min(1, n_tiles - 1)) break;
            // the stage, and the parity of its last use's end
            const int st = t % ST;
            const uint32_t past = (uint32_t)(t / ST - 1) & 1u, k_s = base + L::K + st * L::ROWS;
            const uint32_t v_s = base + L::V + st * L::VALUES;
            if (t >= ST && !poll_phase_warp(BAR(B_K_FREE + st), past, ctl)) break;
            kp.store(k_s, w);
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(B_K_FULL + st));
            if (more) {
                report_pages(jn);
                kp.load(C, pk0, pk1, h, jn, w);
            }
            if (t >= ST && !poll_phase_warp(BAR(B_V_FREE + st), past, ctl)) break;
            if (v_part) {
                if constexpr (PICKED) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (pv_pos + i >= rt.len) vp.scale[i] = 0u;  // behind the last token
                        if ((vp.scale[i] & 0x7Fu) == 0x7Fu) {        // (some of the rows may not have the page)
                            vp.scale[i] = 0u;
                            *nan_flag = 1;
                        }
                    }
                } else if (j0 + kTileKeys - 1 > all_see) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int j = j0 + kg * 8 + i;
                        // what lies behind the last key may be anything, a NaN scale among it
                        if (j >= k1) vp.scale[i] = 0u;
                        // a NaN value must not reach the rows that do not see it (0 * NaN): put in at the end
                        if (j > all_see && (vp.scale[i] & 0x7Fu) == 0x7Fu) {
                            vp.scale[i] = 0u;
                            *nan_flag = 1;
                        }
                    }
                }
                __half2 s[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) s[p] = e4m3x2_value(vp.scale[2 * p] | (vp.scale[2 * p + 1] << 8));
#pragma unroll
                for (int q = 0; q < 2; ++q) {  // 8 channels: even ones from the low codes, odd ones from the high
                    __half2 ev[4][4], od[4][4];
                    const uint32_t lo = 0x0F0F0F0Fu;
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        uint32_t x = q ? vp.code[2 * p].y : vp.code[2 * p].x;
                        uint32_t y = q ? vp.code[2 * p + 1].y : vp.code[2 * p + 1].x;
                        x = __funnelshift_l(x, x, 4 * turn);
                        y = __funnelshift_l(y, y, 4 * turn);
                        e2m1x8_value((x & lo) | ((y << 4) & ~lo), ev[p]);
                        e2m1x8_value(((x >> 4) & lo) | (y & ~lo), od[p]);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {  // channel i ^ turn of the eight
                        uint32_t f[4];
#pragma unroll
                        for (int p = 0; p < 4; ++p) f[p] = h2_bits(__hmul2(i & 1 ? od[p][i / 2] : ev[p][i / 2], s[p]));
                        st_shared16(v_s + v_at + q * 1024 + ((uint32_t)(i << 7 | i << 4) ^ v_x), f[0], f[1], f[2], f[3]);
                    }
                }
            }
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(B_V_FULL + st));
            if (more) load_v(vp, pv, jn);
            pv_pos = pos_of(jn);
            pages(jn + kTileKeys);
        }
    } else {
        // ---------------------------------------------------------------- contractions
        // S of row tile r and key tile t, into the place of its last P: behind the product that read it
        const uint32_t idesc_s = idesc_make(128, kTileKeys, 0u), idesc_o = idesc_make(128, D, 0u);
        auto scores = [&](int r, int t) -> bool {
            const int st = t % ST;
            if (r == 0 && !poll_phase_warp(BAR(B_K_FULL + st), (uint32_t)(t / ST) & 1u, ctl)) return false;
            if (t > 0 && !poll_phase_warp(BAR(B_PV_DONE + r), (uint32_t)(t - 1) & 1u, ctl)) return false;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    const uint32_t off = (x >> 2) * L::ATOM + (x & 3) * 32;
                    mma_f16(tmem + 256 * r, sdesc_k_sw128(base + L::Q + r * L::ROWS + off),
                            sdesc_k_sw128(base + L::K + st * L::ROWS + off), idesc_s, x > 0);
                }
                mma_commit(BAR(B_S_FULL + r));
                if (r == row_tiles - 1) mma_commit(BAR(B_K_FREE + st));
            }
            __syncwarp();
            return true;
        };
        // O of row tile r += P of key tile t times its values
        auto values = [&](int r, int t) -> bool {
            const int st = t % ST;
            if (r == 0 && !poll_phase_warp(BAR(B_V_FULL + st), (uint32_t)(t / ST) & 1u, ctl)) return false;
            if (!poll_phase_warp(BAR(B_P_FULL + r), (uint32_t)t & 1u, ctl)) return false;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int x = 0; x < kTileKeys / 16; ++x)
                    mma_f16_ta(tmem + 256 * r + 128, tmem + 256 * r + x * 8,
                               sdesc_k_sw128(base + L::V + st * L::VALUES + (x >> 2) * (D * 128) + (x & 3) * 32), idesc_o,
                               t > 0 || x > 0);
                mma_commit(BAR(B_PV_DONE + r));
                if (r == row_tiles - 1) mma_commit(BAR(B_V_FREE + st));
            }
            __syncwarp();
            return true;
        };
        // while one row tile's scores become probabilities, the other's contractions run
        bool ok = poll_phase_warp(BAR(B_Q_FULL), 0u, ctl);
        for (int r = 0; r < row_tiles && n_tiles > 0 && ok; ++r) ok = scores(r, 0);
        for (int t = 0; t < n_tiles && ok; ++t)
            for (int r = 0; r < row_tiles && ok; ++r) {
                ok = values(r, t);
                if (ok && t + 1 < n_tiles) ok = scores(r, t + 1);
            }
        // every contraction issued has ended before tensor memory is read or released, also where
        // a wait gave up
        if (elect_one()) mma_commit(BAR(B_DRAIN));
        __syncwarp();
        volatile int no_abort = 0;
        const Ctl drain{&no_abort, a.err, kWaitBudgetCycles};
        wait_phase(BAR(B_DRAIN), 0u, drain);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();

    // ---- the rows' results
    // values that are NaN, for the rows that see them: whether block x of 16 channels has one
    auto nan_block = [&](int x, int i) -> bool {
        if constexpr (PICKED) {
            const uint32_t* has = a.list_bits + (pick_list * a.pick_queries + i - qt.i0) * a.list_words;
            const int shift = a.cache.page_shift, smask = (1 << shift) - 1;
            for (int j = k0; j < k1; ++j) {
                const int4 v = __ldg(list + (j >> shift));
                if (v.x < 0 || !(__ldg(has + (j >> shift >> 5)) >> (j >> shift & 31) & 1u) ||
                    (v.y << shift) + (j & smask) > rt.last0 + i)
                    continue;
                const int64_t r = cache_row(v.x, a.cache.hkv, h, shift, j & smask);
                if ((a.cache.scales[1][r * (D / 16) + x] & 0x7Fu) == 0x7Fu) return true;
            }
        } else {
            for (int j = max(k0, all_see + 1); j < min(k1, rt.last0 + i + 1); ++j) {
                const int32_t page = cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, b, j);
                if (page < 0) continue;
                const int64_t r = cache_row(page, a.cache.hkv, h, a.cache.page_shift, j & ((1 << a.cache.page_shift) - 1));
                if ((a.cache.scales[1][r * (D / 16) + x] & 0x7Fu) == 0x7Fu) return true;
            }
        }
        return false;
    };
    const uint32_t to = tmem + lanes + 256 * (NR > 1 ? rtile : 0) + 128;
    if (warp < live && !*abort_flag) {  // (live <= 4 NR)
        // through shared memory (the operands have been read), so that a store covers whole rows: 32 rows of
        // a warp, padded to keep the lanes' rows in different banks
        constexpr int PITCH = D + 4;
        static_assert(NR * 4 * 32 * PITCH * 4 <= L::BAR, "the rows fit the operands' memory");
        float* mine = reinterpret_cast<float*>(smem) + warp * 32 * PITCH;
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 16) {
            float v[16];
            if (n_tiles > 0) {
                tmem_ld16(to + c0, v);
                tmem_wait_ld();
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = 0.f;
            }
            if (real && *nan_flag && nan_block(c0 / 16, query)) {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __int_as_float(0x7FC00000);
            }
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<float4*>(mine + lane * PITCH + c0 + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        }
        __syncwarp();
        if (PICKED && NR == 1 && copies > 1) {
            // a row's copies joined: of the four warps each takes every fourth row
            float2* ml = reinterpret_cast<float2*>(reinterpret_cast<float*>(smem) + 128 * PITCH);
            static_assert(!(PICKED && NR == 1) || 128 * (PITCH * 4 + 8) <= L::BAR, "the rows fit the operands' memory");
            ml[tid] = make_float2(m, l);
            asm volatile("bar.sync 1, 128;" ::: "memory");
            constexpr int N = D / 32;
            for (int r = warp; r < rt.rows; r += 4) {
                float M = kNoRef, L_ = 0.f, O[N];
#pragma unroll
                for (int i = 0; i < N; ++i) O[i] = 0.f;
                for (int c = 0; c < copies; ++c) M = fmaxf(M, ml[c * copy_rows + r].x);
                for (int c = 0; c < copies; ++c) {
                    const int from = c * copy_rows + r;
                    const float f = ex2(ml[from].x - M);
                    L_ += ml[from].y * f;
#pragma unroll
                    for (int i = 0; i < N; i += 2) {
                        const float2 x =
                            *reinterpret_cast<const float2*>(reinterpret_cast<float*>(smem) + from * PITCH + lane * N + i);
                        O[i] += x.x * f, O[i + 1] += x.y * f;
                    }
                }
                const int i_row = rt.row0 + r, i_query = rt.query(rt.row0 + r);
                if (a.pick_chunks > 1) {
                    const int64_t part =
                        ((int64_t)blockIdx.x * a.cache.hkv + h) * a.max_rows + i_row - qt.i0 * a.group;
                    float* out = a.part_o + part * D + lane * N;
#pragma unroll
                    for (int i = 0; i < N; i += 2) __stcg(reinterpret_cast<float2*>(out + i), make_float2(O[i], O[i + 1]));
                    if (lane == 0) a.part_ml[part] = make_float2(M, L_);
                } else {
                    const int64_t at = (int64_t)(q0 + i_query) * a.hq + h * a.group + i_row - i_query * a.group;
                    const float f = a.cache.scale[1] / L_;
                    __nv_bfloat16* out = a.out + at * D + lane * N;
#pragma unroll
                    for (int i = 0; i < N; i += 2)
                        *reinterpret_cast<__nv_bfloat162*>(out + i) =
                            __floats2bfloat162_rn(L_ == 0.f ? 0.f : O[i] * f, L_ == 0.f ? 0.f : O[i + 1] * f);
                }
            }
        } else {
            const int64_t at = (int64_t)(q0 + query) * a.hq + h * a.group + row - query * a.group;
            const int64_t part = ((int64_t)blockIdx.x * a.cache.hkv + h) * a.max_rows + row - (PICKED ? qt.i0 * a.group : 0);
            const bool split = PICKED ? a.pick_chunks > 1 : a.slots > 0;
            const float f = l == 0.f ? 0.f : a.cache.scale[1] / l;
            const int rows = min(32, rt.rows - warp * 32);
            constexpr int N = D / 32;  // channels of a lane
#pragma unroll 4
            for (int r = 0; r < rows; ++r) {
                float v[N];
#pragma unroll
                for (int i = 0; i < N; i += 2)
                    *reinterpret_cast<float2*>(v + i) = *reinterpret_cast<const float2*>(mine + r * PITCH + lane * N + i);
                if (split) {
                    float* out = a.part_o + __shfl_sync(0xffffffffu, part, r) * D + lane * N;
                    if constexpr (N == 4) __stcg(reinterpret_cast<float4*>(out), make_float4(v[0], v[1], v[2], v[3]));
                    else __stcg(reinterpret_cast<float2*>(out), make_float2(v[0], v[1]));
                } else {
                    // (a row that sees no key is 0, whatever the columns hold)
                    const float fr = __shfl_sync(0xffffffffu, f, r);
                    const bool none = __shfl_sync(0xffffffffu, l, r) == 0.f;
                    __nv_bfloat16* out = a.out + __shfl_sync(0xffffffffu, at, r) * D + lane * N;
#pragma unroll
                    for (int i = 0; i < N; i += 2)
                        *reinterpret_cast<__nv_bfloat162*>(out + i) =
                            __floats2bfloat162_rn(none ? 0.f : v[i] * fr, none ? 0.f : v[i + 1] * fr);
                }
            }
            if (real && split) a.part_ml[part] = make_float2(m, l);
            if (!PICKED && real && a.slots == 0 && a.lse) a.lse[at] = l == 0.f ? INFINITY : m + log2f(l);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == MMA_WARP) {
        tc_fence_after();
        tmem_dealloc(tmem, 256 * NR);
    }
}

// ---------------------------------------------------------------------------------------
// The weights of calls of many rows. With every row's lse known, a CTA takes 128 rows of a
// key head and all keys that they see (or a chunk of them), makes their scores again, this
// time with the keys as the rows of the contraction, and each thread adds up the
// probabilities of one key over the columns, in order. The sums of a tile of rows are kept
// for every key; attend_fold_kernel adds those of all tiles and heads, in order. Bound by the
// exponentials and the contraction, as the first pass, with no second product: the chunk of a
// prompt above takes 360 us with weights and 186 without (with rows as the contraction's rows and
// sums over lanes about 3 ms).
enum { W_K_FULL = 0, W_K_FREE = 2, W_S_FULL = 4, W_S_FREE = 6, W_DRAIN = 8, W_COUNT };

template <int D>
struct WeightLayout {
    static constexpr int ROWS = TileLayout<D, 1>::ROWS;
    static constexpr int Q = 0, K = ROWS;                   // two stages of K
    static constexpr int CONST = 3 * ROWS;                  // factor and lse of every row
    static constexpr int BAR = CONST + 128 * 8;
    static constexpr int MISC = BAR + 8 * W_COUNT;
    static constexpr int NEED = MISC + 16 + 1024;           // (at least 77 KB, as above)
    static constexpr int ALLOC = NEED > 77 * 1024 ? NEED : 77 * 1024;
};

template <int D, bool FP8>
__global__ void __launch_bounds__(kTileThreads<1>, 2) attend_weight_kernel(const __grid_constant__ AttendArgs a)
{
    using L = WeightLayout<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - raw);
    auto BAR = [&](int i) { return base + L::BAR + 8 * i; };
    float2* row_s = reinterpret_cast<float2*>(smem + L::CONST);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::MISC);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::MISC + 4);

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = uniform(tid >> 5);
    const int h = blockIdx.y % a.cache.hkv, tile = (gridDim.y - 1 - blockIdx.y) / a.cache.hkv;
    griddep_wait();
    griddep_launch_dependents();
    int b = blockIdx.z, chunk = kMostKeys, k0 = 0;
    __shared__ int split_s[3];
    if (a.slots > 0) {
        if (threadIdx.x < 32) {
            chunk = chunk_keys(a);
            find_slot(a, blockIdx.x, chunk, b, k0);
            if (threadIdx.x == 0) split_s[0] = chunk, split_s[1] = b, split_s[2] = k0;
        }
        __syncthreads();
        chunk = uniform(split_s[0]), b = uniform(split_s[1]), k0 = uniform(split_s[2]);
        if (b == a.batch) return;
    }
    const RowTile rt = row_tile(a, b, tile, 128);
    if (rt.rows <= 0) return;
    const int q0 = a.q_off[b];
    const int seen = min(rt.len, rt.last0 + rt.query(rt.row0 + rt.rows - 1) + 1);
    const int k1 = chunk_end(seen, k0, chunk);
    if (k0 >= k1) return;
    int all_see = rt.last0 + rt.query(rt.row0);
    const int n_tiles = uniform((k1 - k0 + kTileKeys - 1) / kTileKeys);

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(BAR(W_K_FULL + i), 4);
            mbar_init(BAR(W_K_FREE + i), 1);
            mbar_init(BAR(W_S_FULL + i), 1);
            mbar_init(BAR(W_S_FREE + i), 4);
        }
        mbar_init(BAR(W_DRAIN), 1);
        *abort_flag = 0;
        fence_mbar_init_cluster();
    }
    if (warp == 8) {
        tmem_alloc(smem_u32(tmem_slot), 256);
        tmem_relinquish();
    }
    bool apart = false;  // a factor beyond kFusedFactor
    if (tid < 128) {
        const bool real = tid < rt.rows;
        const int row = rt.row0 + (real ? tid : 0), query = rt.query(row), head = h * a.group + row - query * a.group;
        const int64_t at = (int64_t)(q0 + query) * a.q_stride + (int64_t)head * D;
        const float fac = row_factor(a.c_log2, stage_rows<D, FP8>(a.q, real ? at : -1, base + L::Q, warp * 32));
        row_s[tid] = real ? make_float2(fac, -__ldcg(a.lse + (int64_t)(q0 + query) * a.hq + head))
                          : make_float2(0.f, -INFINITY);  // (no probability)
        apart = fac > kFusedFactor;
        fence_proxy_async_shared();
    }
    tc_fence_before();
    // (no tile then counts as one that every row sees: the sums of the others round each score, then subtract the
    // lse. With a branch of its own in the loop the chunk of a prompt took 377 to 380 us, so 373, without 369)
    if (__syncthreads_or(apart)) all_see = -1;
    tc_fence_after();
    const uint32_t tmem = uniform(*tmem_slot);
    const Ctl ctl{abort_flag, a.err, a.wait_budget};

    if (warp < 4) {
        // ---------------------------------------------------------------- sums: a key a thread
        float* out = a.part_w + (h * a.head_tiles + tile_at((int64_t)q0 * a.group, b) + tile) * a.logit_stride;
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        for (int t = 0; t < n_tiles; ++t) {
            const int st = t & 1, j = k0 + t * kTileKeys + tid;
            if (!poll_phase_warp(BAR(W_S_FULL + st), (uint32_t)(t >> 1) & 1u, ctl)) break;
            tc_fence_after();
            // the first row that sees the key (rows ascend with their queries)
            const int from = j <= all_see ? 0 : (int)min((int64_t)128, (int64_t)(j - rt.last0) * a.group - rt.row0);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll 1
            for (int c0 = 0; c0 < 128; c0 += 32) {
                float v[32];
                tmem_ld32(tmem + lanes + 128 * st + c0, v);
                tmem_wait_ld();
                if (c0 == 96) {  // all have been read
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(BAR(W_S_FREE + st));
                }
                const float4* k = reinterpret_cast<const float4*>(row_s + c0);
                if (k0 + t * kTileKeys + kTileKeys - 1 <= all_see) {
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float4 x = k[i / 2];
                        const float2 e = ffma2(make_float2(v[i], v[i + 1]), make_float2(x.x, x.z), make_float2(x.y, x.w));
                        sum = fadd2(sum, make_float2(ex2(e.x), ex2(e.y)));
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float4 x = k[i / 2];
                        const float p0 = ex2(__fadd_rn(__fmul_rn(v[i], x.x), x.y));
                        const float p1 = ex2(__fadd_rn(__fmul_rn(v[i + 1], x.z), x.w));
                        sum.x += c0 + i >= from ? p0 : 0.f;
                        sum.y += c0 + i + 1 >= from ? p1 : 0.f;
                    }
                }
            }
            if (j < k1) __stcg(out + j, sum.x + sum.y);
        }
    } else if (warp < 8) {
        // ---------------------------------------------------------------- codes to values
        const int w = warp - 4;
        const CachePages& C = a.cache;
        auto page_at = [&](int j) -> int32_t {
            return j < k1 ? cache_page(C.table, C.width, C.num_pages, C.page_shift, b, j) : -1;
        };
        KPart<D> kp;
        int32_t p0 = page_at(k0 + w * 32), p1 = page_at(k0 + w * 32 + 16);
        kp.load(C, p0, p1, h, k0, w);
        p0 = page_at(k0 + kTileKeys + w * 32), p1 = page_at(k0 + kTileKeys + w * 32 + 16);
        for (int t = 0; t < n_tiles; ++t) {
            const int st = t & 1, jn = k0 + (t + 1) * kTileKeys;
            if (t >= 2 && !poll_phase_warp(BAR(W_K_FREE + st), (uint32_t)((t >> 1) - 1) & 1u, ctl)) break;
            kp.store(base + L::K + st * L::ROWS, w);
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(BAR(W_K_FULL + st));
            if (t + 1 < n_tiles) kp.load(C, p0, p1, h, jn, w);
            p0 = page_at(jn + kTileKeys + w * 32), p1 = page_at(jn + kTileKeys + w * 32 + 16);
        }
    } else {
        // ---------------------------------------------------------------- contractions
        const uint32_t idesc = idesc_make(128, 128, 0u);
        for (int t = 0; t < n_tiles; ++t) {
            const int st = t & 1;
            if (!poll_phase_warp(BAR(W_K_FULL + st), (uint32_t)(t >> 1) & 1u, ctl)) break;
            if (t >= 2 && !poll_phase_warp(BAR(W_S_FREE + st), (uint32_t)((t >> 1) - 1) & 1u, ctl)) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    const uint32_t off = (x >> 2) * (128 * 128) + (x & 3) * 32;
                    mma_f16(tmem + 128 * st, sdesc_k_sw128(base + L::K + st * L::ROWS + off),
                            sdesc_k_sw128(base + L::Q + off), idesc, x > 0);
                }
                mma_commit(BAR(W_S_FULL + st));
                mma_commit(BAR(W_K_FREE + st));
            }
            __syncwarp();
        }
        if (elect_one()) mma_commit(BAR(W_DRAIN));
        __syncwarp();
        volatile int no_abort = 0;
        const Ctl drain{&no_abort, a.err, kWaitBudgetCycles};
        wait_phase(BAR(W_DRAIN), 0u, drain);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, 256);
    }
}

// 128 keys of a request a CTA: the sums of all heads' row tiles that see a key, four warps
// sharing them, then the weights.
constexpr int kFoldThreads = 512;
__global__ void __launch_bounds__(kFoldThreads) attend_fold_kernel(const __grid_constant__ AttendArgs a)
{
    __shared__ float part_s[4][128];
    const int b = blockIdx.y, j = blockIdx.x * 128 + (threadIdx.x & 127), part = threadIdx.x >> 7;
    griddep_wait();
    griddep_launch_dependents();
    bool bad;
    const int len = cache_len(a.lens[b], a.limit, bad);
    const int t = a.q_off[b + 1] - a.q_off[b], rows = t * a.group;
    if (blockIdx.x * 128 >= len) return;
    float sum = 0.f;
    if (j < len) {
        // the row tiles from the one on whose last row is the first that sees the key
        const int tiles = (rows + 127) / 128, query = max(0, j - (len - t));
        const int first = (int)((int64_t)query * a.group / 128);
        const float* p = a.part_w + tile_at((int64_t)a.q_off[b] * a.group, b) * a.logit_stride + j;
        const int n = max(0, tiles - first), all = n * a.cache.hkv, per = (all + 3) / 4;
        const int x0 = min(all, part * per), x1 = min(all, x0 + per);
        int h = n > 0 ? x0 / n : 0, r = first + (n > 0 ? x0 - h * n : 0);
#pragma unroll 8
        for (int x = x0; x < x1; ++x) {
            sum += __ldcg(p + (h * a.head_tiles + r) * a.logit_stride);
            if (++r == tiles) r = first, ++h;
        }
    }
    part_s[part][threadIdx.x & 127] = sum;
    __syncthreads();
    if (part != 0 || j >= len) return;
    const int32_t page = cache_page(a.cache.table, a.cache.width, a.cache.num_pages, a.cache.page_shift, b, j);
    if (page < 0) return;
    const int64_t at = ((int64_t)page << a.cache.page_shift) + (j & ((1 << a.cache.page_shift) - 1));
    const float all = ((sum + part_s[1][threadIdx.x]) + part_s[2][threadIdx.x]) + part_s[3][threadIdx.x];
    a.weights_out[at] = a.weights_in[at] + all / (float)a.hq;
}

template <int D, bool FP8, int NR>
cudaError_t launch_variant(const AttendArgs& a, int tiles, cudaStream_t stream)
{
    using L = TileLayout<D, NR>;
    auto kern = attend_tile_kernel<D, FP8, NR>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::ALLOC);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = a.slots > 0 ? dim3((unsigned)a.slots, (unsigned)(tiles * a.cache.hkv), 1)
                              : dim3(1, (unsigned)(tiles * a.cache.hkv), (unsigned)a.batch);
    cfg.blockDim = dim3(kTileThreads<NR>, 1, 1);
    cfg.dynamicSmemBytes = L::ALLOC;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

template <int D, bool FP8, int NR>
cudaError_t launch_picked_variant(const AttendArgs& a, const PickedPlan& plan, cudaStream_t stream)
{
    using L = TileLayout<D, NR>;
    auto kern = attend_tile_kernel<D, FP8, NR, true>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::ALLOC);
    if (e != cudaSuccess) return e;
    const int subs = (plan.queries * a.group + 128 * NR - 1) / (128 * NR);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(plan.tiles * plan.chunks), (unsigned)(subs * a.cache.hkv), 1);
    cfg.blockDim = dim3(kTileThreads<NR>, 1, 1);
    cfg.dynamicSmemBytes = L::ALLOC;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

}  // namespace

cudaError_t launch_picked_tiles(const AttendArgs& a, const PickedPlan& plan, int head_dim, bool fp8, cudaStream_t stream)
{
    if (plan.row_tile == 256) {
        if (fp8) return launch_picked_variant<128, true, 2>(a, plan, stream);
        return head_dim == 128 ? launch_picked_variant<128, false, 2>(a, plan, stream)
                               : launch_picked_variant<64, false, 2>(a, plan, stream);
    }
    if (fp8) return launch_picked_variant<128, true, 1>(a, plan, stream);
    return head_dim == 128 ? launch_picked_variant<128, false, 1>(a, plan, stream)
                           : launch_picked_variant<64, false, 1>(a, plan, stream);
}

cudaError_t launch_attend_tiles(const AttendArgs& a, int head_dim, bool fp8, int row_tile, int tiles, cudaStream_t stream)
{
    if (row_tile == 256) {
        if (fp8) return launch_variant<128, true, 2>(a, tiles, stream);
        return head_dim == 128 ? launch_variant<128, false, 2>(a, tiles, stream)
                               : launch_variant<64, false, 2>(a, tiles, stream);
    }
    if (fp8) return launch_variant<128, true, 1>(a, tiles, stream);
    return head_dim == 128 ? launch_variant<128, false, 1>(a, tiles, stream)
                           : launch_variant<64, false, 1>(a, tiles, stream);
}

namespace {

template <int D, bool FP8>
cudaError_t launch_weights(const AttendArgs& a, int max_len, cudaStream_t stream)
{
    using L = WeightLayout<D>;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1] = {pdl_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.stream = stream;
    cudaError_t e = cudaSuccess;
    if (a.row_tiles > 0) {
        auto kern = attend_weight_kernel<D, FP8>;
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::ALLOC);
        if (e != cudaSuccess) return e;
        cfg.gridDim = a.slots > 0 ? dim3((unsigned)a.slots, (unsigned)(a.row_tiles * a.cache.hkv), 1)
                                  : dim3(1, (unsigned)(a.row_tiles * a.cache.hkv), (unsigned)a.batch);
        cfg.blockDim = dim3(kTileThreads<1>, 1, 1);
        cfg.dynamicSmemBytes = L::ALLOC;
        e = cudaLaunchKernelEx(&cfg, kern, a);
        if (e != cudaSuccess) return e;
        cfg.dynamicSmemBytes = 0;
    }
    cfg.gridDim = dim3((unsigned)((max_len + 127) / 128), (unsigned)a.batch, 1);
    cfg.blockDim = dim3(kFoldThreads, 1, 1);
    return cudaLaunchKernelEx(&cfg, attend_fold_kernel, a);
}

}  // namespace

cudaError_t launch_attend_weights(const AttendArgs& a, int head_dim, bool fp8, int max_len, cudaStream_t stream)
{
    if (fp8) return launch_weights<128, true>(a, max_len, stream);
    return head_dim == 128 ? launch_weights<128, false>(a, max_len, stream) : launch_weights<64, false>(a, max_len, stream);
}

}  // namespace lvs
