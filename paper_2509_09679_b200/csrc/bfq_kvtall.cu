// Attention of many query rows over the same keys of the paged low-bit cache (a shared prefix for a batch, chunks of a prompt) on the
// fifth-generation tensor cores: the same formula, references and scales as the kernel for few rows (bfq_kvattn.cu).
//
// A CTA has up to 256 rows, two M = 128 tiles, and takes its keys in units of 128:
//   warps 0 .. 3, 4 .. 7  softmax of tile 0, 1: a thread owns a row (a lane of tensor memory).  Two walks over the row's 128 scores, the first
//                         for the largest (a new reference and a pass over the products only where a score passes the old one by more than
//                         8, as there), the second for exp2, sum, value scales and the rounding to fp16, which goes back to tensor memory over the
//                         scores;
//   warps 8 .. 11         codes to fp16: a unit's keys and values into one of two stages, loaded one unit ahead into registers;
//   warp 12, one thread   the MMAs: S = Q K^T (both operands in shared memory), O += P V (P from tensor memory).
// The order of the MMAs, S0 S1 | O0 S0' O1 S1' | ..., lets the softmax of one tile run beside the products of the other; scores and
// probabilities share their columns, so tensor memory holds 2 x 128 columns of scores and 2 x D of products.
// Shared-memory operands have the 128-byte swizzle: a row of 128 bytes is 64 elements d of one key (or query row), the two halves of
// D = 128 lie one after the other; K is K-major, V the same bytes read MN-major.  The d within a 16-byte chunk stand in the order in which a
// code word's pairs come out (0 4 1 5 2 6 3 7, or 0 2 1 3 of each four): Q's rows are stored in that order too, and O's columns are
// put back where they are written.
#include "bfq_kvattn.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kTallThreads = 13 * 32;
constexpr int kConvert = 128;  // threads that turn codes into operands

template <int D>
struct TallSmem {
    static constexpr uint32_t kHalves = D / 64, kTile = kHalves * 128 * 128;  // 128 rows
    static constexpr uint32_t kQ = 0, kStages = 2 * kTile, kStage = 2 * kTile;  // a stage: keys, values
    static constexpr uint32_t kScales = kStages + 2 * kStage;  // per stage: 128 key scales, 128 value scales (fp32), factor, unit
    static constexpr uint32_t kScalesBytes = 2 * 128 * 4 + 16;
    static constexpr uint32_t kBars = kScales + 2 * kScalesBytes;
    static constexpr uint32_t kBytes = kBars + 16 * 8 + 1024;  // and what rounding the base up to 1024 takes
};
enum Bar { kKvFull = 0, kKvEmpty = 2, kSFull = 4, kPFull = 6, kQFull = 8, kOFull = 10, kBarCount = 12 };

__device__ __forceinline__ void fence_operands() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void store16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ float4 load_shared4(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
// 128-byte swizzle, 8-row groups 1024 bytes apart; MN-major operands: blocks of 64 elements `leading` bytes apart
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t leading) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(leading >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
           (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}
// fp16 x fp16 -> fp32, M = 128
__host__ __device__ constexpr uint32_t instruction(int n, int v_mn_major) {
    return (1u << 4) | (uint32_t(v_mn_major) << 16) | (uint32_t(n >> 3) << 17) | (uint32_t(128 >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                 "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc),
                 "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Place i of a 16-byte chunk holds element order(i) of its eight.
template <int BITS>
__host__ __device__ constexpr int order(int i) {
    return BITS == 4 ? (i >> 1) + 4 * (i & 1) : (i & 4) + ((i >> 1) & 1) + 2 * (i & 1);
}

template <int D, int BITS>
__global__ void __launch_bounds__(kTallThreads, 1) k_attend_tall(const AttendParams p) {
    using M = TallSmem<D>;
    constexpr int kRow = D * BITS / 8;
    extern __shared__ uint8_t smem_raw[];
    __shared__ long long scan[kTallThreads / 32 + 2];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int dead;
    __shared__ float warp_top[kConvert / 32];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto bar = [&](int b) { return base + M::kBars + 8u * b; };
    auto stage_at = [&](int s) { return base + M::kStages + s * M::kStage; };
    auto scales_at = [&](int s) { return base + M::kScales + s * M::kScalesBytes; };
    grid_dep_wait();
    const Part& part = p.tall;
    Walk walk;
    const Run run = find_run<kTallThreads>(p, part, scan, &walk);
    if (run.count == 0) return;
    if (tid == 0) {
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(kKvFull + s), kConvert), mbar_init(bar(kKvEmpty + s), 1);
            mbar_init(bar(kSFull + s), 1), mbar_init(bar(kPFull + s), 128), mbar_init(bar(kQFull + s), 128), mbar_init(bar(kOFull + s), 1);
        }
        mbar_init_fence();
        dead = 0;
    }
    if (warp == 12) tmem_alloc512(smem_u32(&tmem_at));
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = tmem_at;
    auto scores = [&](int tile) { return tmem + 128u * tile; };
    auto products = [&](int tile) { return tmem + 256u + D * tile; };
    const int count = run.count;

    if (warp < 8) {
        // ---- softmax ---------------------------------------------------------------------------------------------------------
        const int tile = warp >> 2, row_of_tile = tid & 127;
        const uint32_t lanes = uint32_t(warp & 3) << 21;  // 32 lanes of tensor memory
        const uint32_t s_at = scores(tile) + lanes, o_at = products(tile) + lanes, q_at = base + M::kQ + tile * M::kTile + row_of_tile * 128;
        float m = -INFINITY, l = 0.f, row_scale = 0.f, unit = 0.f;
        int limit = 0, least = 0;  // keys of the row; of the warp's rows, at least
        uint32_t s_phase = 0, o_phase = 0;
        bool active = false;
        long long pair_from = run.from - walk.unit;
        auto open = [&]() {
            const Tile& t = walk.tile;
            active = t.rows > 128 * tile;
            if (!active) return;
            const int r = 128 * tile + row_of_tile, row = t.row0 + r;
            const bool there = r < t.rows;
            const int token = t.token0 + row / p.group, head = walk.head * p.group + row % p.group;
            const uint4* at = reinterpret_cast<const uint4*>(p.q.data + (there ? (token * p.q.token + head * p.q.head) * 2 : 0));
            float top = 0.f;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const uint4 v = there ? load_plain(at + c) : make_uint4(0, 0, 0, 0);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xFFFF0000u))));
            }
            const RowPower power(top);
            const float up = p.scale_log2 < 0.f ? -power.up : power.up;
            row_scale = fabsf(p.scale_log2) * power.down;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const uint4 v = there ? load_plain(at + c) : make_uint4(0, 0, 0, 0);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                auto element = [&](int i) { return up * __uint_as_float(order<BITS>(i) & 1 ? w[order<BITS>(i) / 2] & 0xFFFF0000u : w[order<BITS>(i) / 2] << 16); };
                store16(q_at + (c >> 3) * 16384 + (((c & 7) ^ (row_of_tile & 7)) << 4), half_pair(element(0), element(1)), half_pair(element(2), element(3)),
                        half_pair(element(4), element(5)), half_pair(element(6), element(7)));
            }
            fence_operands();
            arrive(bar(kQFull + tile));
            m = -INFINITY, l = 0.f;
            const int own = t.last0 + row / p.group + 1;
            limit = there ? (own < t.keys ? (own > 0 ? own : 0) : t.keys) : 0;
            least = __reduce_min_sync(0xFFFFFFFFu, there ? limit : 1 << 30);
        };
        auto close = [&](long long done) {
            const int pair = walk.pair(p);
            if (active) {
                wait_for(bar(kOFull + tile), o_phase, &dead, p.status);
                o_phase ^= 1;
                tmem_fence_after();
                const int r = 128 * tile + row_of_tile;
                const bool there = r < walk.tile.rows;
                const long long entry = static_cast<long long>(blockIdx.x) + pair;
                float* const to = part.parts + (entry * kTallRows + r) * D;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t v[32];
                    tmem_ld32(o_at + 32 * c, v);
                    tmem_wait_ld32(v);
                    if (there) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float x[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[order<BITS>(i)] = __uint_as_float(v[8 * q + i]) * unit;
                            reinterpret_cast<float4*>(to + 32 * c + 8 * q)[0] = make_float4(x[0], x[1], x[2], x[3]);
                            reinterpret_cast<float4*>(to + 32 * c + 8 * q)[1] = make_float4(x[4], x[5], x[6], x[7]);
                        }
                    }
                }
                tmem_fence_before();
                if (there) part.sums[entry * kTallRows + r] = make_float2(m, l);
            }
            if (tid == 0 && pair_from >= run.from) part.pairs[pair] = make_int2(blockIdx.x, static_cast<int>((pair_from + walk.units - 1) / run.per - blockIdx.x + 1));
            pair_from = done;
        };
        bool first = true;
        open();
        for (int i = 0; i < count; ++i) {
            if (active) {
                const uint32_t k_scales = scales_at(i & 1), v_scales = k_scales + 512;
                const int key0 = walk.unit * kUnit;
                const bool edge = key0 + kUnit > least;  // some row of the warp ends in this unit, or has ended
                wait_for(bar(kKvFull + (i & 1)), (i >> 1) & 1, &dead, p.status);  // for the scales
                wait_for(bar(kSFull + tile), s_phase, &dead, p.status);
                s_phase ^= 1;
                tmem_fence_after();
                const float4 head = load_shared4(k_scales + 1024);
                const float less = head.x;
                unit = head.y;
                float most = -INFINITY;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[32];
                    tmem_ld32(s_at + 32 * c, v);
                    tmem_wait_ld32(v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float4 ks = load_shared4(k_scales + 16 * (8 * c + j));
                        float x[4];
                        unpack2(mul2(pack2u(v[4 * j], v[4 * j + 1]), pack2(ks.x, ks.y)), x[0], x[1]);
                        unpack2(mul2(pack2u(v[4 * j + 2], v[4 * j + 3]), pack2(ks.z, ks.w)), x[2], x[3]);
                        if (edge) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) x[e] = key0 + 32 * c + 4 * j + e < limit ? x[e] : -INFINITY;
                        }
                        most = fmaxf(fmaxf(most, fmaxf(x[0], x[1])), fmaxf(x[2], x[3]));
                    }
                }
                most = most == -INFINITY ? most : most * row_scale;
                const bool over = most > m + 8.f;
                if (first) {
                    m = most;
                } else if (__any_sync(0xFFFFFFFFu, over) || less != 1.f) {
                    float f = less;
                    if (over) f *= exp2_fast(m - most), l *= exp2_fast(m - most), m = most;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t v[16];
                        tmem_ld16(o_at + 16 * c, v);
                        tmem_wait_ld16(v);
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
                        tmem_st16(o_at + 16 * c, v);
                    }
                }
                first = false;
                const float ref = m == -INFINITY ? 0.f : m;
                const u64 scale2 = pack2(row_scale, row_scale), ref2 = pack2(-ref, -ref);
                u64 sum2 = pack2(0.f, 0.f);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[32], out[16];
                    tmem_ld32(s_at + 32 * c, v);
                    tmem_wait_ld32(v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float4 ks = load_shared4(k_scales + 16 * (8 * c + j)), us = load_shared4(v_scales + 16 * (8 * c + j));
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float a, b;
                            const u64 kk = h ? pack2(ks.z, ks.w) : pack2(ks.x, ks.y);
                            unpack2(fma2(mul2(pack2u(v[4 * j + 2 * h], v[4 * j + 2 * h + 1]), kk), scale2, ref2), a, b);
                            if (edge) {
                                const int key = key0 + 32 * c + 4 * j + 2 * h;
                                a = key < limit ? a : -INFINITY, b = key + 1 < limit ? b : -INFINITY;
                            }
                            const u64 e2 = pack2(exp2_fast(a), exp2_fast(b));
                            sum2 = add2(sum2, e2);
                            unpack2(mul2(e2, h ? pack2(us.z, us.w) : pack2(us.x, us.y)), a, b);
                            out[2 * j + h] = half_pair(a, b);
                        }
                    }
                    tmem_st16(s_at + 16 * c, out);
                }
                float a, b;
                unpack2(sum2, a, b);
                l += a + b;
                tmem_wait_st();
                tmem_fence_before();
                arrive(bar(kPFull + tile));
            }
            if (walk.unit + 1 == walk.units || i + 1 == count) {
                close(run.from + i + 1);
                walk.next_pair(p, part);
                first = true;
                if (i + 1 < count) open();
            } else {
                ++walk.unit;
            }
        }
    } else if (warp < 12) {
        // ---- codes to operands -------------------------------------------------------------------------------------------------
        const int r = tid - 256, w = r >> 5;
        const Unpack<BITS> unpack;
        // 16-byte pieces: the eight lanes of a phase of the stores below write chunks of one half to eight different places of 16 bytes
        constexpr int kPer = BITS == 4 ? 2 : 4;          // pieces of 64 elements
        constexpr int kKeys = 32 / (kPer * (D / 64));    // keys of a warp's 32 pieces
        constexpr int kTurns = kUnit / kKeys / 4;
        const int part_of = lane % kPer, key_low = lane / kPer % (8 / kPer);
        const int half = D == 128 ? lane >> 3 & 1 : 0, key_of = key_low + (8 / kPer) * (D == 128 ? lane >> 4 : lane >> 3);
        uint4 k_raw[kTurns], v_raw[kTurns];
        uint32_t scale_raw = 0;
        auto load = [&]() {
            const int mask = (1 << p.cache.page_shift) - 1;
#pragma unroll
            for (int c = 0; c < kTurns; ++c) {
                const int key = walk.unit * kUnit + (c * 4 + w) * kKeys + key_of;
                const int64_t page = key < walk.tile.keys ? page_of(p, walk.tile, key) : -1;
                k_raw[c] = v_raw[c] = make_uint4(0, 0, 0, 0);
                if (page >= 0) {
                    const int at = 16 * (half * kPer + part_of);
                    k_raw[c] = load_plain(reinterpret_cast<const uint4*>(codes_of<kRow>(p.cache.k, p.cache.page_shift, page, walk.head, key & mask) + at));
                    v_raw[c] = load_plain(reinterpret_cast<const uint4*>(codes_of<kRow>(p.cache.v, p.cache.page_shift, page, walk.head, key & mask) + at));
                }
            }
            const int key = walk.unit * kUnit + r;
            const int64_t page = key < walk.tile.keys ? page_of(p, walk.tile, key) : -1;
            scale_raw = 0;
            if (page >= 0) {
                const uint32_t a = *static_cast<volatile const uint16_t*>(scale_of(p.cache.k, p.cache.page_shift, page, walk.head, key & mask));
                const uint32_t b = *static_cast<volatile const uint16_t*>(scale_of(p.cache.v, p.cache.page_shift, page, walk.head, key & mask));
                scale_raw = a | b << 16;
            }
        };
        auto store = [&](uint32_t to, const uint4 (&raw)[kTurns]) {
#pragma unroll
            for (int c = 0; c < kTurns; ++c) {
                const int key = (c * 4 + w) * kKeys + key_of;
                const uint32_t row = to + half * 16384 + key * 128;
                const uint32_t x[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
                if constexpr (BITS == 4) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        store16(row + (((4 * part_of + j) ^ (key & 7)) << 4), unpack(x[j], 0), unpack(x[j], 1), unpack(x[j], 2), unpack(x[j], 3));
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        store16(row + (((2 * part_of + j) ^ (key & 7)) << 4), unpack(x[2 * j], 0), unpack(x[2 * j], 1), unpack(x[2 * j + 1], 0), unpack(x[2 * j + 1], 1));
                }
            }
        };
        float u_top = 0.f;
        bool first = true;
        load();
        for (int i = 0; i < count; ++i) {
            const int s = i & 1;
            if (i >= 2) wait_for(bar(kKvEmpty + s), ((i >> 1) - 1) & 1, &dead, p.status);
            store(stage_at(s), k_raw);
            store(stage_at(s) + M::kTile, v_raw);
            const float ks = half_value(static_cast<uint16_t>(scale_raw & 0xFFFFu)), us = half_value(static_cast<uint16_t>(scale_raw >> 16));
            const bool last_of_pair = walk.unit + 1 == walk.units;
            walk.next(p, part);
            if (i + 1 < count) load();
            // the power of two above all value scales of the pair so far
            const float top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(us)));  // not negative: ordered as integers
            if (lane == 0) warp_top[w] = top;
            bar_sync(1, kConvert);
            const float most = fmaxf(fmaxf(warp_top[0], warp_top[1]), fmaxf(warp_top[2], warp_top[3]));
            bar_sync(1, kConvert);
            float less = 1.f;
            if (first) u_top = 0x1p-24f, first = false;
            if (most > u_top) {
                const float next = __uint_as_float((__float_as_uint(most) & 0x7F800000u) + 0x00800000u);
                less = u_top / next, u_top = next;
            }
            if (last_of_pair) first = true;
            const uint32_t to = scales_at(s);
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + 4 * r), "f"(ks) : "memory");
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + 512 + 4 * r), "f"(us * (128.f / u_top)) : "memory");
            if (r == 0) asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(to + 1024), "f"(less), "f"(u_top * (1.f / 128.f)) : "memory");
            fence_operands();
            arrive(bar(kKvFull + s));
        }
    } else {
        // ---- MMAs ----------------------------------------------------------------------------------------------------------------
        if (lane == 0) {
            uint32_t p_phase[2] = {0, 0}, q_phase[2] = {0, 0};
            constexpr uint32_t kScoresDesc = instruction(128, 0), kProductsDesc = instruction(D, 1);
            auto issue_scores = [&](int tile, int s) {
                const uint32_t a = base + M::kQ + tile * M::kTile, b = stage_at(s);
    #pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t off = (k >> 2) * 16384 + (k & 3) * 32;
                    mma_ss(scores(tile), operand(a + off, 0), operand(b + off, 0), kScoresDesc, k > 0);
                }
                commit_to(bar(kSFull + tile));
            };
            auto issue_products = [&](int tile, int s, bool accumulate) {
                const uint32_t b = stage_at(s) + M::kTile;
    #pragma unroll
                for (int k = 0; k < kUnit / 16; ++k) mma_ts(products(tile), scores(tile) + 8 * k, operand(b + 2048 * k, 16384), kProductsDesc, accumulate || k > 0);
            };
            bool first = true;
            for (int i = 0; i < count; ++i) {
                const int s = i & 1, tiles = walk.tile.rows > 128 ? 2 : 1;
                const bool last = walk.unit + 1 == walk.units || i + 1 == count;
                if (first) {
                    wait_for(bar(kKvFull + s), (i >> 1) & 1, &dead, p.status);
                    for (int t = 0; t < tiles; ++t) {
                        wait_for(bar(kQFull + t), q_phase[t], &dead, p.status);
                        q_phase[t] ^= 1;
                        tmem_fence_after();
                        issue_scores(t, s);
                    }
                }
                for (int t = 0; t < tiles; ++t) {
                    wait_for(bar(kPFull + t), p_phase[t], &dead, p.status);
                    p_phase[t] ^= 1;
                    tmem_fence_after();
                    issue_products(t, s, !first);
                    if (last) {
                        commit_to(bar(kOFull + t));
                    } else {
                        if (t == 0) wait_for(bar(kKvFull + (s ^ 1)), ((i + 1) >> 1) & 1, &dead, p.status);
                        issue_scores(t, s ^ 1);
                    }
                }
                commit_to(bar(kKvEmpty + s));
                first = last;
                walk.next(p, part);
            }
            wait_for(bar(kKvEmpty + ((count - 1) & 1)), ((count - 1) >> 1) & 1, &dead, p.status);  // the last arrival has come
        }
        __syncwarp();
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 12) tmem_dealloc512(tmem);
}

template <int D, int BITS>
static cudaError_t prepare(const bfq_plan* plan) {
    static bool done[kMaxDevices] = {false};
    if (done[plan->device]) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(k_attend_tall<D, BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(TallSmem<D>::kBytes));
    done[plan->device] = e == cudaSuccess;
    return e;
}
cudaError_t tall_ctas(const bfq_plan* plan, int bits, int* ctas) {
    *ctas = plan->sm_count;
    return plan->n == 64 ? (bits == 4 ? prepare<64, 4>(plan) : prepare<64, 8>(plan)) : (bits == 4 ? prepare<128, 4>(plan) : prepare<128, 8>(plan));
}
cudaError_t tall_launch(const bfq_plan* plan, const AttendParams& p, int ctas, cudaStream_t st) {
    const dim3 grid{unsigned(ctas)}, block{unsigned(kTallThreads)};
    if (plan->n == 64)
        return p.cache.bits == 4 ? launch_overlapped(k_attend_tall<64, 4>, grid, block, TallSmem<64>::kBytes, st, p)
                                 : launch_overlapped(k_attend_tall<64, 8>, grid, block, TallSmem<64>::kBytes, st, p);
    return p.cache.bits == 4 ? launch_overlapped(k_attend_tall<128, 4>, grid, block, TallSmem<128>::kBytes, st, p)
                             : launch_overlapped(k_attend_tall<128, 8>, grid, block, TallSmem<128>::kBytes, st, p);
}

}  // namespace kv
}  // namespace bfq
