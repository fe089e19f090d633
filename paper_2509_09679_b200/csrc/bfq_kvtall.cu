// Attention of many query rows over the same keys of the paged low-bit cache (a shared prefix for a batch, chunks of a prompt) on the
// fifth-generation tensor cores: the same formula and references as the kernel for few rows (bfq_kvattn.cu).
//
// A CTA has up to 256 rows, two M = 128 tiles, and takes its keys in units of 128:
//   warps 0 .. 3, 4 .. 7  softmax of tile 0, 1: a thread owns a row (a lane of tensor memory).  Two walks over the row's 128 scores, the first
//                         for the largest (a new reference and a pass over the products only where a score passes the old one by more than
//                         8, as there), the second for exp2, sum and the rounding to fp16, which goes back to tensor memory over the scores;
//   warps 8 .. 11         codes to fp16: a unit's keys and values into one of two stages, loaded one unit ahead into registers;
//   warp 12, one thread   the MMAs: S = Q K^T (both operands in shared memory), O += P V (P from tensor memory).
// The order of the MMAs, S0 S1 | O0 S0' O1 S1' | ..., lets the softmax of one tile run beside the products of the other; scores and
// probabilities share their columns, so tensor memory holds 2 x 128 columns of scores and 2 x D of products.
// Keys and values are multiplied by their scales on the way into shared memory, over a power of two for all of a pair so far: one rounding to
// fp16 of each element, 2^-12 on average and independent of its neighbours, a fraction of the output's own rounding.  Applied exactly, to
// scores and probabilities, the scales would be read from shared memory 256 times by every softmax warp for a unit, which took three times as
// long as everything else.
// Shared-memory operands have the 128-byte swizzle: a row of 128 bytes is 64 elements d of one key (or query row), the two halves of
// D = 128 lie one after the other; K is K-major, V the same bytes read MN-major.  The d within a 16-byte chunk stand in the order in which a
// code word's pairs come out (0 4 1 5 2 6 3 7, or 0 2 1 3 of each four): Q's rows are stored in that order too, and O's columns are
// put back where they are written.
#include "bfq_kvattn.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kTallThreads = 16 * 32;  // warps 13 .. 15 only lend their registers
constexpr int kConvert = 128;  // threads that turn codes into operands

template <int D>
struct TallSmem {
    static constexpr uint32_t kHalves = D / 64, kTile = kHalves * 128 * 128;  // 128 rows
    static constexpr uint32_t kQ = 0, kStages = 2 * kTile, kStage = 2 * kTile;  // a stage: keys, values
    static constexpr uint32_t kFactors = kStages + 2 * kStage;  // per stage: less, unit of the products, unit of the scores
    static constexpr uint32_t kBars = kFactors + 2 * 16;
    static constexpr uint32_t kBytes = kBars + 16 * 8 + 1024;  // and what rounding the base up to 1024 takes
};
enum Bar { kKvFull = 0, kKvEmpty = 2, kSFull = 4, kPFull = 6, kQFull = 8, kOFull = 10, kBarCount = 12 };

__device__ __forceinline__ void fence_operands() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// the wait of a converged warp
__device__ __forceinline__ void wait_all(uint32_t bar, uint32_t parity, volatile int* dead, int* status) {
    wait_for(bar, parity, dead, status);
    __syncwarp();
}
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
// Issued by the one thread of a converged warp whose `lead` is set: a predicate on the instruction and no branch around it, so that the
// operands can stay in uniform registers.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void mma_ss(uint32_t lead, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
        "l"(b), "r"(idesc), "r"(accumulate), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t lead, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a),
        "l"(b), "r"(idesc), "r"(accumulate), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t lead, uint32_t bar) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(lead)
                 : "memory");
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
    __shared__ float2 warp_top[2][kConvert / 32];  // of the keys' scales, the values'
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto bar = [&](int b) { return base + M::kBars + 8u * b; };
    auto stage_at = [&](int s) { return base + M::kStages + s * M::kStage; };
    auto factors_at = [&](int s) { return base + M::kFactors + 16u * s; };
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

    // registers: 256 x 168 + 128 x 112 + 128 x 64 = 512 x 128, what the block was launched with
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
        // ---- softmax ---------------------------------------------------------------------------------------------------------
        const int tile = warp >> 2, row_of_tile = tid & 127;
        const uint32_t lanes = uint32_t(warp & 3) << 21;  // 32 lanes of tensor memory
        const uint32_t s_at = scores(tile) + lanes, o_at = products(tile) + lanes;
        float m = -INFINITY, l = 0.f, row_scale = 0.f, unit = 0.f;
        int limit = 0, least = 0;  // keys of the row; of the warp's rows, at least
        uint32_t s_phase = 0, o_phase = 0;
        bool active = false;
        long long pair_from = run.from - walk.unit;
        auto open = [&]() {
            const Tile& t = walk.tile;
            active = t.rows > 128 * tile;
            if (!active) return;
            constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes;  // of a row
            const int first_row = 128 * tile + 32 * (warp & 3), part_of = lane % kLanes;
            const float sign = p.scale_log2 < 0.f ? -1.f : 1.f;
            // eight loads on their way at a time
            constexpr int kLoads = 8;
#pragma unroll 1
            for (int n0 = 0; n0 < 32; n0 += kLoads * kRowsAtOnce) {
                uint4 v[kLoads];
#pragma unroll
                for (int x = 0; x < kLoads; ++x) {
                    const int r = first_row + n0 + x * kRowsAtOnce + lane / kLanes, row = t.row0 + r, token = row / p.group;
                    v[x] = make_uint4(0, 0, 0, 0);
                    if (r < t.rows)
                        v[x] = load_plain(reinterpret_cast<const uint4*>(p.q.data + ((t.token0 + token) * p.q.token + (walk.head * p.group + row - token * p.group) * p.q.head + 8 * part_of) * 2));
                }
#pragma unroll
                for (int x = 0; x < kLoads; ++x) {
                    const int n = n0 + x * kRowsAtOnce;
                    const uint32_t w[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
                    float top = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xFFFF0000u))));
#pragma unroll
                    for (int y = 1; y < kLanes; y <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, y));
                    const RowPower power(top);
                    const float up = sign * power.up;
                    auto element = [&](int i) { return up * __uint_as_float(order<BITS>(i) & 1 ? w[order<BITS>(i) / 2] & 0xFFFF0000u : w[order<BITS>(i) / 2] << 16); };
                    const int at = 32 * (warp & 3) + n + lane / kLanes;  // of the tile
                    store16(base + M::kQ + tile * M::kTile + at * 128 + (part_of >> 3) * 16384 + (((part_of & 7) ^ (at & 7)) << 4), half_pair(element(0), element(1)),
                            half_pair(element(2), element(3)), half_pair(element(4), element(5)), half_pair(element(6), element(7)));
                    const float down = __shfl_sync(0xFFFFFFFFu, power.down, (lane % kRowsAtOnce) * kLanes);
                    if (lane / kRowsAtOnce == n / kRowsAtOnce) row_scale = fabsf(p.scale_log2) * down;  // the lane's own row
                }
            }
            const int r = 128 * tile + row_of_tile, row = t.row0 + r;
            const bool there = r < t.rows;
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
                // half of 32 rows at a time through the warp's part of the query tile, which no product reads any more, so that rows are written
                // whole: 16 bytes at place (chunk ^ row) of a row's half
                constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes;
                const uint32_t own = base + M::kQ + tile * M::kTile + (warp & 3) * (M::kTile / 4);
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) {
                        uint32_t v[32];
                        tmem_ld32(o_at + (D / 2) * h + 32 * c, v);
                        tmem_wait_ld32(v);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float x[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[order<BITS>(i)] = __uint_as_float(v[8 * q + i]) * unit;
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                store16(own + lane * 2 * D + (((8 * c + 2 * q + i) ^ (lane & (kLanes - 1))) << 4), __float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]),
                                        __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
                        }
                    }
                    __syncwarp();
                    const int chunk = lane % kLanes;
#pragma unroll 4
                    for (int n = 0; n < 32; n += kRowsAtOnce) {
                        const int row = n + lane / kLanes, to = 128 * tile + 32 * (warp & 3) + row;
                        const float4 x = load_shared4(own + row * 2 * D + ((chunk ^ (row & (kLanes - 1))) << 4));
                        if (to < walk.tile.rows) *reinterpret_cast<float4*>(part.parts + (entry * kTallRows + to) * D + (D / 2) * h + 4 * chunk) = x;
                    }
                    __syncwarp();
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
                const int key0 = walk.unit * kUnit;
                const bool edge = key0 + kUnit > least;  // some row of the warp ends in this unit, or has ended
                wait_for(bar(kKvFull + (i & 1)), (i >> 1) & 1, &dead, p.status);  // for the factors
                wait_for(bar(kSFull + tile), s_phase, &dead, p.status);
                s_phase ^= 1;
                tmem_fence_after();
                const float4 factors = load_shared4(factors_at(i & 1));
                const float less = factors.x, scale = fmaxf(row_scale * factors.z, 1e-30f);  // -infinity times it is that
                unit = factors.y;
                float most = -INFINITY;
                // compact loops: unrolled over the whole row, with the masks that few units need, the instruction cache missed all the time
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[32];
                    tmem_ld32(s_at + 32 * c, v);
                    tmem_wait_ld32(v);
                    if (edge) {
                        const int n = limit - key0 - 32 * c;
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = j < n ? v[j] : 0xFF800000u;
                    }
                    float x[4] = {most, most, most, most};
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j & 3] = fmaxf(x[j & 3], __uint_as_float(v[j]));
                    most = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
                }
                most = most == -INFINITY ? most : most * scale;
                const bool over = most > m + 8.f;
                if (first) {
                    m = most;
                } else if (__any_sync(0xFFFFFFFFu, over) || less != 1.f) {
                    float f = less;
                    if (over) f *= exp2_fast(m - most), l *= exp2_fast(m - most), m = most;
#pragma unroll 1
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t w[16];
                        tmem_ld16(o_at + 16 * c, w);
                        tmem_wait_ld16(w);
#pragma unroll
                        for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * f);
                        tmem_st16(o_at + 16 * c, w);
                    }
                }
                first = false;
                const float ref = m == -INFINITY ? 0.f : m;
                const u64 scale2 = pack2(scale, scale), ref2 = pack2(-ref, -ref);
                u64 sum2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[32], out[16];
                    tmem_ld32(s_at + 32 * c, v);
                    tmem_wait_ld32(v);
                    if (edge) {
                        const int n = limit - key0 - 32 * c;
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = j < n ? v[j] : 0xFF800000u;
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float a, b;
                        unpack2(fma2(pack2u(v[2 * j], v[2 * j + 1]), scale2, ref2), a, b);
                        a = exp2_fast(a), b = exp2_fast(b);
                        sum2[j & 1] = add2(sum2[j & 1], pack2(a, b));
                        out[j] = half_pair(a, b);
                    }
                    tmem_st16(s_at + 16 * c, out);
                }
                float a, b;
                unpack2(add2(sum2[0], sum2[1]), a, b);
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
        asm volatile("setmaxnreg.dec.sync.aligned.u32 112;");
        // ---- codes to operands -------------------------------------------------------------------------------------------------
        const int w = warp - 8;
        const Unpack<BITS> unpack;
        // 16-byte pieces: the eight lanes of a phase of the stores below write chunks of one half to eight different places of 16 bytes
        constexpr int kPer = BITS == 4 ? 2 : 4;        // pieces of 64 elements
        constexpr int kKeys = 32 / (kPer * (D / 64));  // keys of a warp's 32 pieces: of one page
        constexpr int kTurns = kUnit / kKeys / 4;
        const int part_of = lane % kPer, key_low = lane / kPer % (8 / kPer);
        const int half = D == 128 ? lane >> 3 & 1 : 0, key_of = key_low + (8 / kPer) * (D == 128 ? lane >> 4 : lane >> 3);
        uint4 k_raw[kTurns], v_raw[kTurns];
        uint16_t k_scale[kTurns], v_scale[kTurns];
        constexpr int64_t kNone = -(int64_t(1) << 32);
        int64_t page = kNone;  // lane c: of turn c; kNone: it has no keys
        auto look = [&]() {
            const int key = walk.unit * kUnit + (lane * 4 + w) * kKeys;
            page = lane < kTurns && key < walk.tile.keys ? load_plain(walk.tile.pages + (key >> p.cache.page_shift)) : kNone;
        };
        auto load = [&]() {
            const int mask = (1 << p.cache.page_shift) - 1;
            if (page != kNone && (page < 0 || page >= p.cache.pages)) atomicExch(p.status, kBadIndex), page = kNone;
#pragma unroll
            for (int c = 0; c < kTurns; ++c) {
                const int key = walk.unit * kUnit + (c * 4 + w) * kKeys + key_of;
                const int64_t at = __shfl_sync(0xFFFFFFFFu, page, c);
                k_raw[c] = v_raw[c] = make_uint4(0, 0, 0, 0), k_scale[c] = v_scale[c] = 0;
                if (at >= 0 && key < walk.tile.keys) {
                    const int64_t row = (static_cast<int64_t>(walk.head) << p.cache.page_shift) + (key & mask);
                    const int off = 16 * (half * kPer + part_of);
                    k_raw[c] = load_plain(reinterpret_cast<const uint4*>(p.cache.k.codes + at * p.cache.k.codes_page + row * kRow + off));
                    v_raw[c] = load_plain(reinterpret_cast<const uint4*>(p.cache.v.codes + at * p.cache.v.codes_page + row * kRow + off));
                    k_scale[c] = *static_cast<volatile const uint16_t*>(p.cache.k.scales + at * p.cache.k.scales_page + row);
                    v_scale[c] = *static_cast<volatile const uint16_t*>(p.cache.v.scales + at * p.cache.v.scales_page + row);
                }
            }
        };
        auto times = [](uint32_t a, uint32_t b) {
            uint32_t d;
            asm("mul.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
            return d;
        };
        auto store = [&](uint32_t to, const uint4& raw, int key, float scale) {
            const uint32_t row = to + half * 16384 + key * 128, s2 = half_pair(scale, scale);
            const uint32_t x[4] = {raw.x, raw.y, raw.z, raw.w};
            if constexpr (BITS == 4) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    store16(row + (((4 * part_of + j) ^ (key & 7)) << 4), times(unpack(x[j], 0), s2), times(unpack(x[j], 1), s2), times(unpack(x[j], 2), s2),
                            times(unpack(x[j], 3), s2));
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    store16(row + (((2 * part_of + j) ^ (key & 7)) << 4), times(unpack(x[2 * j], 0), s2), times(unpack(x[2 * j], 1), s2),
                            times(unpack(x[2 * j + 1], 0), s2), times(unpack(x[2 * j + 1], 1), s2));
            }
        };
        // the power of two above all scales of the pair so far, at most that of 65504
        auto above = [](float top, float most) { return most > top ? __uint_as_float((__float_as_uint(most) & 0x7F800000u) + 0x00800000u) : top; };
        float k_top = 0.f, v_top = 0.f;
        bool first = true;
        look();
        load();
        for (int i = 0; i < count; ++i) {
            const int s = i & 1;
            float2 most = make_float2(0.f, 0.f);
#pragma unroll
            for (int c = 0; c < kTurns; ++c)
                most.x = fmaxf(most.x, half_value(k_scale[c])), most.y = fmaxf(most.y, half_value(v_scale[c]));
            most.x = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most.x)));  // not negative: ordered as integers
            most.y = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most.y)));
            if (lane == 0) warp_top[s][w] = most;
            bar_sync(1, kConvert);
#pragma unroll
            for (int n = 0; n < kConvert / 32; ++n) most.x = fmaxf(most.x, warp_top[s][n].x), most.y = fmaxf(most.y, warp_top[s][n].y);
            if (first) k_top = v_top = 0x1p-24f;
            const float v_before = v_top;
            k_top = above(k_top, most.x), v_top = above(v_top, most.y);
            const float k_factor = 128.f / k_top, v_factor = 128.f / v_top;  // codes times scales: at most 2^14
            first = walk.unit + 1 == walk.units;
            walk.next(p, part);
            if (i + 1 < count) look();
            if (i >= 2) wait_for(bar(kKvEmpty + s), ((i >> 1) - 1) & 1, &dead, p.status);
#pragma unroll
            for (int c = 0; c < kTurns; ++c) {
                const int key = (c * 4 + w) * kKeys + key_of;
                store(stage_at(s), k_raw[c], key, k_factor * half_value(k_scale[c]));
                store(stage_at(s) + M::kTile, v_raw[c], key, v_factor * half_value(v_scale[c]));
            }
            if (warp == 8 && lane == 0)
                asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(factors_at(s)), "f"(v_before / v_top), "f"(v_top * (1.f / 128.f)), "f"(k_top * (1.f / 128.f)), "f"(0.f)
                             : "memory");
            fence_operands();
            arrive(bar(kKvFull + s));
            if (i + 1 < count) load();
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        // ---- MMAs ----------------------------------------------------------------------------------------------------------------
        if (warp == 12) {
            const uint32_t lead = elect_one();
            uint32_t p_phase[2] = {0, 0}, q_phase[2] = {0, 0};
            constexpr uint32_t kScoresDesc = instruction(128, 0), kProductsDesc = instruction(D, 1);
            auto issue_scores = [&](int tile, int s) {
                const uint32_t a = base + M::kQ + tile * M::kTile, b = stage_at(s);
    #pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t off = (k >> 2) * 16384 + (k & 3) * 32;
                    mma_ss(lead, scores(tile), operand(a + off, 0), operand(b + off, 0), kScoresDesc, k > 0);
                }
                commit_to(lead, bar(kSFull + tile));
            };
            auto issue_products = [&](int tile, int s, bool accumulate) {
                const uint32_t b = stage_at(s) + M::kTile;
    #pragma unroll
                for (int k = 0; k < kUnit / 16; ++k) mma_ts(lead, products(tile), scores(tile) + 8 * k, operand(b + 2048 * k, 16384), kProductsDesc, accumulate || k > 0);
            };
            bool first = true;
            for (int i = 0; i < count; ++i) {
                const int s = i & 1, tiles = walk.tile.rows > 128 ? 2 : 1;
                const bool last = walk.unit + 1 == walk.units || i + 1 == count;
                if (first) {
                    wait_all(bar(kKvFull + s), (i >> 1) & 1, &dead, p.status);
                    for (int t = 0; t < tiles; ++t) {
                        wait_all(bar(kQFull + t), q_phase[t], &dead, p.status);
                        q_phase[t] ^= 1;
                        tmem_fence_after();
                        issue_scores(t, s);
                    }
                }
                for (int t = 0; t < tiles; ++t) {
                    wait_all(bar(kPFull + t), p_phase[t], &dead, p.status);
                    p_phase[t] ^= 1;
                    tmem_fence_after();
                    issue_products(t, s, !first);
                    if (last) {
                        commit_to(lead, bar(kOFull + t));
                    } else {
                        if (t == 0) wait_all(bar(kKvFull + (s ^ 1)), ((i + 1) >> 1) & 1, &dead, p.status);
                        issue_scores(t, s ^ 1);
                    }
                }
                commit_to(lead, bar(kKvEmpty + s));
                first = last;
                walk.next(p, part);
            }
            wait_all(bar(kKvEmpty + ((count - 1) & 1)), ((count - 1) >> 1) & 1, &dead, p.status);  // the last arrival has come
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
