// Attention of a few queries for each sequence over the paged low-bit cache (decoding), and the joining of partial results.
//
//     out = Q^T sum_j softmax_j(scale q . (s_j k_j)) (u_j v_j),  k, v the codes of the rotated rows, s, u their fp16 scales, q rotated by Q.
//
// The codes are exact in fp16, so both products run on the tensor cores without the scales: a row of q is taken times a power of two
// that puts its largest element in [2^10, 2^11) (elements down to 2^-24 of that stay exact), q . k_j is summed in fp32 and multiplied by
// s_j; probabilities times u_j are rounded once to fp16 (2^-11 of each, independent of its neighbours; bf16 would cost more than the output's own
// rounding), on a power of two that follows the largest u so far.  Softmax is taken in one pass over the keys: m is a reference that is
// at most 8 (a factor of 256) below the largest score so far, so that it, the sum and the products change only when a score passes it by more
// than that.
//
// A CTA of four warps takes units of 128 keys, 32 keys to a warp, each warp from a ring of its own that it fills ahead by TMA (a box for each page and half,
// swizzled so that the reads below hit every bank once).  mma.m16n8k16 with the keys, then the values' elements, as its 16 rows and 8 queries
// as its columns: with the queries as rows a group of four would leave three quarters of the tensor cores' work idle and twice
// the registers taken.  Keys come as words of a row, 8 (4) codes at a time; which k index of the product an element gets is
// free as long as the queries' fragments have the same order, so no code moves between lanes.  Values come by ldmatrix.trans on 16-bit
// units of 4 (2) codes: the halves of a register are two keys' codes of the same element, which is what the second product needs of its
// left operand; the probabilities, keys by queries, are turned by movmatrix into its right one.
//
// What bounds it: long contexts of 8-bit codes, memory (0.85 of the copy's rate).  4-bit codes, instructions and their latencies together: of 720 for 32
// keys 272 turn codes into fp16 (9 for 8 codes of 4 bits, 10 for 8 of 8); the schedulers issue in 0.59 of their cycles, ALU 49 %.
#include <algorithm>

#include "bfq_kvattn.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kWarps = 4, kAttendThreads = 32 * kWarps;

constexpr int kKeys = kFewUnit / kWarps;  // of a warp

// Shared memory: for each warp kCount stages of its 32 keys' and values' codes, the same of their scales, a tile's merged products, sums, barriers.
template <int D, int BITS, int NB>
struct Stage {
    static constexpr int kRow = D * BITS / 8;  // bytes of a row's codes
    static constexpr int kCount = kRow == 128 ? 2 : 3;
    static constexpr uint32_t kBytes = 2 * kKeys * kRow, kScaleBytes = 4 * kKeys;
    static constexpr int kPitch = D + (BITS == 4 ? 1 : 8);  // of a merged row, floats: lanes are kPer g + 2 t rows apart, two to a bank
    static constexpr uint32_t kScales = kWarps * kCount * kBytes, kMerge = kScales + kWarps * kCount * kScaleBytes, kSums = kMerge + 8 * NB * kPitch * 4,
                              kBars = kSums + kWarps * 8 * NB * 8;
    static constexpr uint32_t kSmem = kBars + kWarps * kCount * 8 + 1024;  // and what rounding the base up to 1024 takes
};

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float lds_half(uint32_t at) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
    return half_value(v);
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
struct Maps {
    CUtensorMap k_codes, v_codes;
};

// NB: blocks of 8 queries
template <int D, int BITS, int NB>
__global__ void __launch_bounds__(kAttendThreads, NB == 2 ? 2 : (D * BITS == 1024 ? 3 : 4)) k_attend(const AttendParams p, const __grid_constant__ Maps maps) {
    using S = Stage<D, BITS, NB>;
    constexpr int kSteps = D / 16, kRows = 8 * NB;
    extern __shared__ uint8_t smem_raw[];
    __shared__ int scan[kWarps + 2];
    __shared__ volatile int dead;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    float* const merge = reinterpret_cast<float*>(smem_raw + (base - smem_u32(smem_raw)) + S::kMerge);  // [rows][pitch]
    float2* const warp_sums = reinterpret_cast<float2*>(smem_raw + (base - smem_u32(smem_raw)) + S::kSums);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const Unpack<BITS> unpack;
    auto full = [&](int s) { return base + S::kBars + 8u * (warp * S::kCount + s); };
    auto stage_at = [&](int s) { return base + (warp * S::kCount + s) * S::kBytes; };
    auto scales_at = [&](int s) { return base + S::kScales + (warp * S::kCount + s) * S::kScaleBytes; };
    // Beside the tall kernel, which has waited for all that came before and shares nothing with this one: it is waited for at the end, so that
    // this kernel's end is the end of both.
    if (!p.beside_tall) grid_dep_wait();
    grid_dep_launch();
    const Part& part = p.few;
    Walk ahead;
    const Run run = find_run<kAttendThreads>(p, part, scan, &ahead);
    if (run.count == 0) {
        if (p.beside_tall) grid_dep_wait();
        return;
    }
    Walk now = ahead;
    const int count = run.count;
    if (tid == 0) {
        for (int s = 0; s < kWarps * S::kCount; ++s) mbar_init(base + S::kBars + 8u * s, 1);
        mbar_init_fence();
        dead = 0;
    }
    __syncthreads();

    // ---- the warp's keys of the unit ahead, a page to a lane; the pages' numbers are looked up one unit earlier still -----------
    const int page_keys = 1 << p.cache.page_shift, box = page_keys < kKeys ? page_keys : kKeys, own = kKeys * warp + lane * box;
    const bool a_box = lane * box < kKeys;
    constexpr int64_t kNone = -(int64_t(1) << 32);
    int64_t page = kNone;  // of the lane's box; kNone: it has no keys
    int sent = 0;          // units; above count: a wait has given up
    auto look = [&]() {
        const int key = ahead.unit * kFewUnit + own;
        page = sent < count && a_box && key < ahead.tile.keys ? load_plain(ahead.tile.pages + (key >> p.cache.page_shift)) : kNone;
    };
    auto fetch = [&](int slot) {
        if (sent >= count) return;
        ++sent;
        const int row = (ahead.head << p.cache.page_shift) + ((ahead.unit * kFewUnit + own) & (page_keys - 1));
        const uint32_t boxes = __popc(__ballot_sync(0xFFFFFFFFu, page != kNone));
        if (lane == 0) mbar_expect_tx(full(slot), boxes * box * (2 * S::kRow + 4));
        __syncwarp();
        if (page != kNone) {
            if (page < 0 || page >= p.cache.pages) atomicExch(p.status, kBadIndex), page = 0;
            const int at = static_cast<int>(page);
            const uint32_t codes = stage_at(slot) + lane * box * S::kRow, scales = scales_at(slot) + lane * box * 2;
            tma_load_3d(codes, &maps.k_codes, 0, row, at, full(slot));
            tma_load_3d(codes + kKeys * S::kRow, &maps.v_codes, 0, row, at, full(slot));
            bulk_load(scales, p.cache.k.scales + page * p.cache.k.scales_page + row, box * 2, full(slot));
            bulk_load(scales + kKeys * 2, p.cache.v.scales + page * p.cache.v.scales_page + row, box * 2, full(slot));
        }
        __syncwarp();
        ahead.next(p, part);
        look();
    };
    look();
#pragma unroll
    for (int i = 0; i < S::kCount; ++i) fetch(i);
    // place of 16-byte chunk c of row r of a swizzled half of a stage: r kRow + 16 (c ^ its swizzle), which rows 8 apart share
    auto swizzle = [](int r) { return S::kRow == 128 ? r & 7 : (S::kRow == 64 ? r >> 1 & 3 : r >> 2 & 1); };
    const uint32_t k_lane = g * S::kRow + 16 * ((t * S::kRow / 64) ^ swizzle(g)) + (S::kRow == 32 ? 8 * (t & 1) : 0);  // its first chunk of row g
    const uint32_t v_lane = kKeys * S::kRow + lane * S::kRow + 16 * swizzle(lane & 7);

    // ---- a pair's state: fragments of the queries, reference, sums and products -------------------------------------------
    uint32_t qb[NB][kSteps][2];
    float m[NB][2], l[NB][2], o[NB][kSteps][4];  // of queries 8 b + 2 t and + 1; o: element rows of 16
    // m and scores are in units of the row's power of two; times `unit`, softmax scale * log2 e over it, they are exponents of 2
    float unit[NB][2], over_at[NB][2];  // a score above over_at moves m
    int limit[NB][2], least;            // keys of the row; of the tile's rows, at least
    float u_top, u_unit;  // power of two that no u so far passes; 128 / u_top: probabilities (at most 2^8) times u stay below 2^15
    auto open = [&]() {
        const Tile& tl = now.tile;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int r = 8 * b + g, row = tl.row0 + r;  // the row that the lane holds a part of
            const bool there = r < tl.rows;
            const int token = tl.token0 + row / p.group, head = now.head * p.group + row % p.group;
            const uint4* at = reinterpret_cast<const uint4*>(p.q.data + (there ? (token * p.q.token + head * p.q.head + t * (D / 4)) * 2 : 0));
            uint32_t w[D / 8];  // the lane's D / 4 elements of the row, two in a word
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                const uint4 v = there ? load_plain(at + c) : make_uint4(0, 0, 0, 0);
                w[4 * c] = v.x, w[4 * c + 1] = v.y, w[4 * c + 2] = v.z, w[4 * c + 3] = v.w;
            }
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xFFFF0000u))));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const RowPower power(top);
            const float up = p.scale_log2 < 0.f ? -power.up : power.up;
            auto element = [&](int i) { return up * __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16); };
            auto pair = [&](int i, int j) { return half_pair(element(i), element(j)); };
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if constexpr (BITS == 4) {
                    const int d = 8 * (s / 2) + 2 * (s & 1);
                    qb[b][s][0] = pair(d, d + 4), qb[b][s][1] = pair(d + 1, d + 5);
                } else {
                    qb[b][s][0] = pair(4 * s, 4 * s + 2), qb[b][s][1] = pair(4 * s + 1, 4 * s + 3);
                }
            }
            const int own = tl.last0 + row / p.group + 1, keys = there ? (own < tl.keys ? own : tl.keys) : 0;
#pragma unroll
            for (int c = 0; c < 2; ++c) {  // from the lanes of the rows that this lane's columns are
                unit[b][c] = fmaxf(fabsf(p.scale_log2) * __shfl_sync(0xFFFFFFFFu, power.down, 4 * (2 * t + c)), 1e-30f);  // times -infinity is that
                limit[b][c] = __shfl_sync(0xFFFFFFFFu, keys, 4 * (2 * t + c));
                m[b][c] = over_at[b][c] = -INFINITY, l[b][c] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[b][i][j] = 0.f;
        }
        u_top = 0.f, u_unit = 0.f;
        least = tl.keys;
#pragma unroll
        for (int b = 0; b < NB; ++b) least = min(least, 8 * b + g < tl.rows ? tl.last0 + (tl.row0 + 8 * b + g) / p.group + 1 : least);
        least = __reduce_min_sync(0xFFFFFFFFu, least);
    };
    int pair_from = run.from - now.unit;  // number of the pair's unit 0
    auto close = [&](int done) {          // after unit `done` (exclusive) of the numbering
        const int pair = now.pair(p);
        const long long entry = blockIdx.x + pair;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[b][c] += __shfl_xor_sync(0xFFFFFFFFu, l[b][c], x);
                if (g == 0) warp_sums[warp * kRows + 8 * b + 2 * t + c] = make_float2(m[b][c] * unit[b][c], l[b][c]);
            }
        __syncthreads();
        float f[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int r = 8 * b + 2 * t + c;
                float top = -INFINITY, sum = 0.f;
                float2 ml[kWarps];
#pragma unroll
                for (int w = 0; w < kWarps; ++w) ml[w] = warp_sums[w * kRows + r], top = fmaxf(top, ml[w].x);
                const float safe = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) sum += ml[w].y * exp2_fast(ml[w].x - safe);
                f[b][c] = exp2_fast(m[b][c] * unit[b][c] - safe) * (u_top * (1.f / 128.f));
                if (warp == 0 && g == 0 && r < now.tile.rows) part.sums[entry * kRows + r] = make_float2(top, sum);
            }
        // element of accumulator i, row g + 8 j: see the values' order below
        auto element_of = [&](int i, int j) {
            constexpr int kPer = 16 / BITS;  // codes of a 16-bit unit
            const int n = 2 * i + j;         // chunk n / kPer, unit g, code n % kPer of the unit
            return (n / kPer) * 8 * kPer + kPer * g + n % kPer;
        };
        // a quarter of the elements from each warp at a time, all four in turn: an element's sum starts with another warp, but always the same
#pragma unroll
        for (int turn = 0; turn < kWarps; ++turn) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                if (i / (kSteps / kWarps) == ((warp + turn) & (kWarps - 1))) {
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float* at = merge + (8 * b + 2 * t + (j & 1)) * S::kPitch + element_of(i, j >> 1);
                            const float v = o[b][i][j] * f[b][j & 1];
                            *at = turn > 0 ? *at + v : v;
                        }
                }
            __syncthreads();
        }
        for (int i = tid; i < now.tile.rows * D; i += kAttendThreads) part.parts[(entry * kRows) * D + i] = merge[(i / D) * S::kPitch + i % D];
        if (tid == 0 && pair_from >= run.from) part.pairs[pair] = make_int2(blockIdx.x, (pair_from + now.units - 1) / run.per - static_cast<int>(blockIdx.x) + 1);
        pair_from = done;
    };

    open();
    int slot = 0;
    uint32_t phase = 0;
    for (int i = 0; i < count; ++i) {
        const int key0 = now.unit * kFewUnit + kKeys * warp;
        const uint32_t stage = stage_at(slot), scales = scales_at(slot);
        const bool stuck = sent <= count && !wait_for(full(slot), phase, &dead, p.status);
        if (key0 < now.tile.keys) {
            // ---- scores of 32 keys: rows g and g + 8 of product j are keys 16 j + g and 16 j + 8 + g of the warp's
            float s[NB][2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                constexpr int kWords = D * BITS / 128;  // of a lane and key
                uint32_t w[2][kWords];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t at = stage + k_lane + (16 * j + 8 * h) * S::kRow;
                    if constexpr (kWords == 2) {
                        const uint2 v = lds64(at);
                        w[h][0] = v.x, w[h][1] = v.y;
                    } else {
#pragma unroll
                        for (int c = 0; c < kWords / 4; ++c) {
                            const uint4 v = lds128(at ^ (16 * c));
                            w[h][4 * c] = v.x, w[h][4 * c + 1] = v.y, w[h][4 * c + 2] = v.z, w[h][4 * c + 3] = v.w;
                        }
                    }
                }
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int c = 0; c < 4; ++c) s[b][j][c] = 0.f;
#pragma unroll
                for (int st = 0; st < kSteps; ++st) {
                    uint32_t a[4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if constexpr (BITS == 4) a[h] = unpack(w[h][st / 2], 2 * (st & 1)), a[2 + h] = unpack(w[h][st / 2], 2 * (st & 1) + 1);
                        else a[h] = unpack(w[h][st], 0), a[2 + h] = unpack(w[h][st], 1);
                    }
#pragma unroll
                    for (int b = 0; b < NB; ++b) mma16816(s[b][j], a[0], a[1], a[2], a[3], qb[b][st][0], qb[b][st][1]);
                }
            }
            // ---- scales, masks, probabilities
            float u[4];  // keys 8 x + g
            bool over = false;
            const bool edge = key0 + kKeys > least;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t at = scales + 2 * (8 * x + g);
                const float f = lds_half(at);
                u[x] = lds_half(at + 2 * kKeys);
#pragma unroll
                for (int b = 0; b < NB; ++b) s[b][x >> 1][2 * (x & 1)] *= f, s[b][x >> 1][2 * (x & 1) + 1] *= f;
                if (edge) {
                    const int key = key0 + 8 * x + g;
                    // of a key that some rows do not see: a value's scale that is not finite (append_kv writes none) becomes a score of NaN for those
                    // that do; where all rows see it, it makes NaN of their products below
                    const bool fine = u[x] <= 65504.f;
                    u[x] = fine && key < now.tile.keys ? u[x] : 0.f;
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float& e = s[b][x >> 1][2 * (x & 1) + c];
                            e = key < limit[b][c] ? (fine ? e : NAN) : -INFINITY;
                        }
                }
                over |= u[x] > u_top;
#pragma unroll
                for (int b = 0; b < NB; ++b) over |= s[b][x >> 1][2 * (x & 1)] > over_at[b][0] || s[b][x >> 1][2 * (x & 1) + 1] > over_at[b][1];
            }
            if (__any_sync(0xFFFFFFFFu, over)) {
                float most = fmaxf(fmaxf(u[0], u[1]), fmaxf(u[2], u[3]));
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, x));
                float less = 1.f;  // on the products
                if (most > u_top) {
                    const float top = __uint_as_float((__float_as_uint(most) & 0x7F800000u) + 0x00800000u);  // above it
                    less = u_top / top, u_top = top, u_unit = 128.f / top;
                }
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float top = fmaxf(fmaxf(s[b][0][c], s[b][0][2 + c]), fmaxf(s[b][1][c], s[b][1][2 + c]));
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
                        top = fmaxf(top, m[b][c]);
                        const float f = top == -INFINITY ? 1.f : exp2_fast((m[b][c] - top) * unit[b][c]);
                        m[b][c] = top, l[b][c] *= f, over_at[b][c] = top == -INFINITY ? top : top + 8.f / unit[b][c];
#pragma unroll
                        for (int k = 0; k < kSteps; ++k) o[b][k][c] *= f * less, o[b][k][2 + c] *= f * less;
                    }
            }
            uint32_t pb[NB][4];  // keys 8 x + 2 t and + 1 of query 8 b + g
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const float r0 = m[b][0] == -INFINITY ? 0.f : -m[b][0] * unit[b][0], r1 = m[b][1] == -INFINITY ? 0.f : -m[b][1] * unit[b][1];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float e0 = exp2_fast(fmaf(s[b][x >> 1][2 * (x & 1)], unit[b][0], r0)), e1 = exp2_fast(fmaf(s[b][x >> 1][2 * (x & 1) + 1], unit[b][1], r1)),
                                v = u[x] * u_unit;
                    l[b][0] += e0, l[b][1] += e1;
                    pb[b][x] = transpose8(half_pair(e0 * v, e1 * v));
                }
            }
            // ---- values: matrix (8 keys) x (a 16-byte chunk), its 16-bit units across the lanes
            constexpr int kPer = 16 / BITS, kMats = S::kRow / 16;
#pragma unroll
            for (int c = 0; c < kMats; ++c) {
                uint32_t r[4];  // keys 8 x of chunk c
                ldmatrix4_trans((stage + v_lane) ^ (16 * c), r);
#pragma unroll
                for (int n = 0; n < kPer; n += 2)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t a[4];
#pragma unroll
                        for (int h = 0; h < 2; ++h) a[h] = unpack(r[2 * j], n + h), a[2 + h] = unpack(r[2 * j + 1], n + h);
#pragma unroll
                        for (int b = 0; b < NB; ++b) mma16816(o[b][(c * kPer + n) / 2], a[0], a[1], a[2], a[3], pb[b][2 * j], pb[b][2 * j + 1]);
                    }
            }
        }
        if (__any_sync(0xFFFFFFFFu, stuck)) {
            // no copies go to a slot whose last ones have not come; those in flight, of up to kCount units, are waited for
            uint32_t parity = phase;
            for (int k = 0, x = slot; k < S::kCount && i + k < sent; ++k) {
                drain(full(x), parity);
                if (++x == S::kCount) x = 0, parity ^= 1;
            }
            sent = count + 1;
        }
        fetch(slot);
        if (++slot == S::kCount) slot = 0, phase ^= 1;
        if (now.unit + 1 == now.units || i + 1 == count) {
            close(run.from + i + 1);
            now.next_pair(p, part);
            if (i + 1 < count) open();
        } else {
            ++now.unit;
        }
    }
    if (p.beside_tall) grid_dep_wait();
}

// Joins a row's partial results (the shared prefix's, then its sequence's), turns it back by Q^T and rounds it once.  A row is a (token, query
// head); a warp takes `each` consecutive ones.
template <int D>
__global__ void __launch_bounds__(128) k_join(const AttendParams p, int each) {
    constexpr int kE = D / 32;
    const int lane = threadIdx.x & 31;
    // The kernel before has let this one start after it had waited for all that came before itself: constants, lengths and starts can be read
    // while it still works.
    const int rows_all = static_cast<int>(p.tokens) * p.q.heads, row0 = (blockIdx.x * 4 + (threadIdx.x >> 5)) * each;
    Turn<D, kE, true> turn;
    turn.load(p.tw, lane);
    bool waited = false;
    const int q_heads = p.q.heads, begin = first_token(p, 0), end = first_token(p, p.batch);
    int of = -1, b = 0, place = 0, news = 0;  // token that b, its place in it, the sequence's tokens and tall are of
    bool tall = false;
    for (int row = row0; row < row0 + each && row < rows_all; ++row) {
        const int token = row / q_heads, head = row - token * q_heads, h = head / p.group;
        if (token < begin || token >= end) continue;  // rows of no sequence stay as they are
        if (token != of) {
            of = b = token, place = 0;
            if (p.q_starts != nullptr) {  // the last sequence that starts at or before this token
                int lo = 0, hi = p.batch;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    if (first_token(p, mid) <= token) lo = mid;
                    else hi = mid;
                }
                b = lo, place = token - first_token(p, b);
            }
            news = first_token(p, b + 1) - first_token(p, b);
            tall = p.seq_tall && news * p.group > kFewMost;
        }
        if (tall && p.join_tall) {  // k_join_tall has these
            row += q_heads - 1 - head;
            continue;
        }
        float m = -INFINITY, l = 0.f, o[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) o[e] = 0.f;
        auto join = [&](bool tall, int b, int row) {  // b < 0: the prefix
            const Part& part = tall ? p.tall : p.few;
            const int rows = part.rows, r = row % rows, entry = (b < 0 ? 0 : part.tiles_prefix + b * part.tiles_seq) + row / rows;
            const Tile tile = tile_of(p, part, entry);
            const int pair = tile.place * p.cache.heads + h;
            if (tile.keys == 0) return;
            if (!waited) grid_dep_wait(), waited = true;
            const int2 found = ctas_of(part, pair);
            const int64_t first = static_cast<int64_t>(found.x) + pair;
            constexpr int kAtOnce = 4;  // results on their way
            float v[kAtOnce][kE];
            auto load = [&](int i, float (&to)[kE]) {
                const float* at = part.parts + ((first + i) * rows + r) * D + kE * lane;
                if constexpr (kE == 4) {
                    const float4 u = load_plain(reinterpret_cast<const float4*>(at));
                    to[0] = u.x, to[1] = u.y, to[2] = u.z, to[3] = u.w;
                } else {
                    const float2 u = load_plain(reinterpret_cast<const float2*>(at));
                    to[0] = u.x, to[1] = u.y;
                }
            };
            for (int i0 = 0; i0 < found.y; i0 += 32) {  // a lane has one of 32 results' m and l
                const int n = found.y - i0 < 32 ? found.y - i0 : 32;
                const float2 ml = lane < n ? load_plain(part.sums + (first + i0 + lane) * rows + r) : make_float2(-INFINITY, 0.f);
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) load(i0 + (k < n ? k : 0), v[k]);
                float top = ml.x;
#pragma unroll
                for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
                top = fmaxf(top, m);
                const float safe = top == -INFINITY ? 0.f : top, old = exp2_fast(m - safe), mine = exp2_fast(ml.x - safe);
                float sum = mine * ml.y;
#pragma unroll
                for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
                m = top, l = l * old + sum;
#pragma unroll
                for (int e = 0; e < kE; ++e) o[e] *= old;
                for (int i = 0; i < n; i += kAtOnce) {
#pragma unroll
                    for (int k = 0; k < kAtOnce; ++k) {
                        const float f = __shfl_sync(0xFFFFFFFFu, mine, (i + k) & 31);
#pragma unroll
                        for (int e = 0; e < kE; ++e) o[e] = i + k < n ? fmaf(f, v[k][e], o[e]) : o[e];
                        if (i + kAtOnce + k < n) load(i0 + i + kAtOnce + k, v[k]);
                    }
                }
            }
        };
        if (p.prefix_length > 0) join(p.prefix_tall != 0, -1, token * p.group + head % p.group);
        // rows that have no tile: of tokens beyond max_new, or of starts that fall
        if (place < p.max_new && place < news) join(tall, b, place * p.group + head % p.group);
        const float f = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
        for (int e = 0; e < kE; ++e) o[e] *= f;
        turn.apply(o);
        if (!waited) grid_dep_wait(), waited = true;  // what came before may still read where this is written
        uint8_t* out = const_cast<uint8_t*>(p.out.data) + (token * p.out.token + head * p.out.head + kE * lane) * 2;
        if constexpr (kE == 4) *reinterpret_cast<uint2*>(out) = make_uint2(bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3]));
        else *reinterpret_cast<uint32_t*>(out) = bf16_pair(o[0], o[1]);
        if (p.lse != nullptr && lane == 0) p.lse[row] = l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
    // from the last CTA on, which has no rows
    for (int b = (gridDim.x - 1 - blockIdx.x) * blockDim.x + threadIdx.x; b < p.batch; b += gridDim.x * blockDim.x)
        if (out_of_range(p, b)) atomicExch(p.status, kBadIndex);
    if (!waited) grid_dep_wait();
}

// A half of the cache's codes as boxes of a page's rows of a head, at most kKeys of them: {bytes of a row, rows of a page, pages}
static bool encode_half(CUtensorMap* map, const Half& half, const Cache& cache, int row_bytes) {
    const EncodeTiledFn encode = encode_tiled();
    if (encode == nullptr) return false;
    const int page = 1 << cache.page_shift;
    const cuuint64_t dims[3] = {cuuint64_t(row_bytes), cuuint64_t(cache.heads) << cache.page_shift, cuuint64_t(cache.pages > 0 ? cache.pages : 1)};
    const cuuint64_t strides[2] = {cuuint64_t(row_bytes), cuuint64_t(half.codes_page)};
    const cuuint32_t box[3] = {cuuint32_t(row_bytes), cuuint32_t(page < kKeys ? page : kKeys), 1}, estr[3] = {1, 1, 1};
    const CUtensorMapSwizzle swizzle = row_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : (row_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B);
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, half.codes, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// One of the kernel's forms: all CTAs that the chip runs at once (ctas), or a launch of `grid` on st.
template <int D, int BITS, int NB>
static cudaError_t attend_form(const bfq_plan* plan, const AttendParams& p, int* ctas, int grid, cudaStream_t st) {
    using S = Stage<D, BITS, NB>;
    static int per_sm[kMaxDevices] = {0};
    int& occ = per_sm[plan->device];
    if (occ == 0) {
        cudaError_t e = cudaFuncSetAttribute(k_attend<D, BITS, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(S::kSmem));
        int n = 0;
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k_attend<D, BITS, NB>, kAttendThreads, S::kSmem);
        if (e != cudaSuccess) return e;
        occ = n > 0 ? n : 1;
    }
    if (ctas != nullptr) {
        *ctas = plan->sm_count * occ;
        return cudaSuccess;
    }
    Maps maps;
    if (!encode_half(&maps.k_codes, p.cache.k, p.cache, S::kRow) || !encode_half(&maps.v_codes, p.cache.v, p.cache, S::kRow)) return cudaErrorInvalidValue;
    return launch_overlapped(k_attend<D, BITS, NB>, dim3(unsigned(grid)), dim3(kAttendThreads), S::kSmem, st, p, maps);
}
template <int D, int BITS>
static cudaError_t attend_rows(const bfq_plan* plan, const AttendParams& p, int* ctas, int grid, cudaStream_t st) {
    return p.few.rows == 8 ? attend_form<D, BITS, 1>(plan, p, ctas, grid, st) : attend_form<D, BITS, 2>(plan, p, ctas, grid, st);
}
static cudaError_t attend(const bfq_plan* plan, const AttendParams& p, int* ctas, int grid = 0, cudaStream_t st = nullptr) {
    return plan->n == 64 ? (p.cache.bits == 4 ? attend_rows<64, 4>(plan, p, ctas, grid, st) : attend_rows<64, 8>(plan, p, ctas, grid, st))
                         : (p.cache.bits == 4 ? attend_rows<128, 4>(plan, p, ctas, grid, st) : attend_rows<128, 8>(plan, p, ctas, grid, st));
}

// Tiles of 256 rows where there are rows enough to pay for them.  The kernel for few rows against the one for many, us (4-bit cache, n = 128, 8 key
// heads): 16 sequences of 4096 keys, 32 rows each 63 / 88, 48 rows 91 / 91, 64 rows 114 / 95, 256 rows 422 / 137; 64 of 2048 keys, 48 rows
// 193 / 221, 64 rows 251 / 226.  One sequence of 2048 keys alone fills no more than the start of either: 64 rows 14 / 18, 256 rows 27 / 23.
// Other forms, 16 sequences of 4096 keys that come from memory (as above: 48 rows 102 / 121, 64 rows 127 / 123): n = 128 at 8 bits, 48 rows 107 / 145, 64 rows
// 135 / 147, 96 rows 188 / 152; n = 64 at 4 bits, 48 rows 86 / 94, 64 rows 107 / 96, at 8 bits 92 / 96 and 115 / 98.
static bool use_tall(int64_t rows) { return rows > kFewMost; }
// A prefix too, but where the sequences do not need that kernel's launch beside theirs only from five units of 16 rows and 128 keys to an SM on:
// 8192 keys, 32 rows 28 / 30, 64 rows 48 / 31; 1024 keys, 64 rows 17 / 23, 128 rows (3.5 units) 23 / 25, 256 rows (7) 38 / 27.
static bool prefix_use_tall(int64_t rows, bool seq_tall, int64_t keys, int heads, int sm_count) {
    return use_tall(rows) && (seq_tall || ((rows + 15) / 16) * ((keys + kFewUnit - 1) / kFewUnit) * heads > 5 * sm_count);
}
// A row to a thread in the join where the rows fill the chip so; else a row to a warp, whose lanes have the results' weights at once.  Whole calls
// with k_join_tall against k_join, us: one sequence, 512 rows 46 / 18; 16 sequences of 2048 keys from memory, 8192, 16384 and 32768 rows of results:
// n = 128 at 4 bits 84 / 82, 90 / 90, 98 / 117, at 8 bits 98 / 94, 102 / 104, 113 / 129; n = 64 at 4 bits 66 / 64, 66 / 72, 78 / 96, at 8 bits 68 / 66, 70 / 74,
// 78 / 98.
constexpr int64_t kJoinTallRows = 16384;

// The workspace: for each of the two kernels pairs, sums and parts.  Lays them out from `at` on (null: only counts); returns the bytes.
static size_t lay_out(AttendParams* p, int n, int ctas_few, int ctas_tall, uint8_t* at) {
    size_t bytes = 0;
    auto take = [&](size_t b) {
        uint8_t* here = at != nullptr ? at + bytes : nullptr;
        bytes += (b + 255) / 256 * 256;
        return here;
    };
    for (const bool tall : {false, true}) {
        Part& part = tall ? p->tall : p->few;
        const size_t pairs = size_t(p->places(part)) * p->cache.heads, rows = (pairs + (tall ? ctas_tall : ctas_few)) * part.rows;
        if (pairs == 0) continue;
        part.pairs = reinterpret_cast<int2*>(take(pairs * sizeof(int2)));
        part.sums = reinterpret_cast<float2*>(take(rows * sizeof(float2)));
        part.parts = reinterpret_cast<float*>(take(rows * n * sizeof(float)));
    }
    return bytes;
}

// checks everything that the host can see and lays the work out
static int set_up(const bfq_plan* plan, const bfq_kv_cache* cache, const bfq_kv_queries* in, AttendParams* p) {
    int rc = check_cache(plan, cache, &p->cache);
    if (rc != BFQ_OK) return rc;
    if (in == nullptr) return BFQ_ERR_NULL;
    if (in->tokens < 0 || in->tokens >= int64_t(1) << 24 || in->batch < 0 || in->batch > 1 << 20 || in->table_width < 0 ||
        in->table_ld < in->table_width || in->prefix_length < 0 || in->prefix_pages < 0)
        return BFQ_ERR_STRIDE;
    if ((int64_t(in->table_width) << p->cache.page_shift) >= int64_t(1) << 30 || in->prefix_length >= int64_t(1) << 30 ||
        in->prefix_length > int64_t(in->prefix_pages) << p->cache.page_shift || (in->prefix_length > 0 && cache->pages == 0))
        return BFQ_ERR_STRIDE;
    if (!(in->scale == in->scale) || in->scale - in->scale != 0.f) return BFQ_ERR_STRIDE;  // not finite
    if (in->tokens == 0 || in->batch == 0) return BFQ_OK;
    rc = check_heads(&in->q, plan->n, 2, &p->q);
    if (rc == BFQ_OK) rc = check_heads(&in->out, plan->n, 2, &p->out);
    if (rc != BFQ_OK) return rc;
    if (in->out.heads != in->q.heads || in->q.heads % cache->heads != 0 || in->q.heads / cache->heads > 128 || in->tokens * in->q.heads >= int64_t(1) << 31)
        return BFQ_ERR_STRIDE;
    if (in->lengths == nullptr || (in->table_width > 0 && in->block_table == nullptr) || (in->prefix_length > 0 && in->prefix == nullptr)) return BFQ_ERR_NULL;
    for (const void* at : {static_cast<const void*>(in->lengths), static_cast<const void*>(in->block_table), static_cast<const void*>(in->q_starts),
                           static_cast<const void*>(in->prefix), static_cast<const void*>(in->lse)})
        if ((reinterpret_cast<uintptr_t>(at) & 3u) != 0) return BFQ_ERR_ALIGN;
    if (in->q_starts == nullptr ? in->tokens < in->batch : in->max_new < 1) return BFQ_ERR_STRIDE;
    p->lse = in->lse, p->block_table = in->block_table, p->table_ld = in->table_ld, p->table_width = in->table_width, p->lengths = in->lengths;
    p->q_starts = in->q_starts, p->prefix = in->prefix, p->prefix_pages = in->prefix_pages, p->prefix_length = cache->pages > 0 ? int(in->prefix_length) : 0;
    p->tokens = in->tokens, p->batch = in->batch, p->group = in->q.heads / cache->heads, p->max_new = in->q_starts == nullptr ? 1 : int(std::min<int64_t>(in->max_new, in->tokens));
    const int64_t rows = (in->q_starts == nullptr ? in->batch : in->tokens) * int64_t(p->group), rows_seq = int64_t(p->max_new) * p->group;
    p->seq_tall = use_tall(rows_seq), p->prefix_tall = prefix_use_tall(rows, p->seq_tall, in->prefix_length, cache->heads, plan->sm_count);
    p->join_tall = p->seq_tall && p->prefix_length == 0 && in->tokens * in->q.heads > kJoinTallRows;
    p->tall.rows = kTallRows, p->tall.unit_shift = 6, p->few.unit_shift = 7;
    static_assert(kTallUnit == 1 << 6 && kFewUnit == 1 << 7, "shifts");
    // sequences of the kernel for few rows: all of them, or those up to kFewMost rows of a batch with larger ones, mostly single tokens
    const int64_t rows_few = p->seq_tall ? kFewMost : rows_seq;
    // a tile of 8 rows where they fit, against 16 (us, as above): 16 sequences of 4096 keys 30 / 37, 64 of 2048 keys 51 / 69, one 10.9 / 11.9
    p->few.rows = (p->seq_tall ? p->group : rows_few) <= 8 && (in->prefix_length == 0 || p->prefix_tall || rows <= 8) ? 8 : 16;
    p->few.seq_from = 1, p->few.seq_to = p->seq_tall ? kFewMost : INT32_MAX, p->tall.seq_from = kFewMost + 1, p->tall.seq_to = INT32_MAX;
    Part& front = p->prefix_tall ? p->tall : p->few;
    const int64_t tiles_prefix = in->prefix_length > 0 ? (rows + front.rows - 1) / front.rows : 0, tiles_few = (rows_few + p->few.rows - 1) / p->few.rows,
                  tiles_seq = (p->seq_tall ? (rows_seq + kTallRows - 1) / kTallRows : 0) + tiles_few;
    front.tiles_prefix = int(tiles_prefix), p->few.tiles_seq = int(tiles_few), p->tall.tiles_seq = int(tiles_seq - tiles_few);
    int64_t pairs = 0;
    for (Part* part : {&p->few, &p->tall}) {
        part->rows_shift = part->rows == 8 ? 3 : (part->rows == 16 ? 4 : 8);
        if (part->tiles_prefix + int64_t(in->batch) * part->tiles_seq >= int64_t(1) << 30) return BFQ_ERR_TOO_LARGE;
        part->by_tokens = in->q_starts != nullptr && part->tiles_seq > 0 && p->places_by_tokens(*part) < p->entries(*part);
        const int64_t places = p->places(*part);  // as many as tiles, or more
        auto units = [&](int64_t keys) { return (keys + (1 << part->unit_shift) - 1) >> part->unit_shift; };
        const int64_t most = part->tiles_prefix * units(in->prefix_length) + (places - part->tiles_prefix) * units(int64_t(in->table_width) << p->cache.page_shift);
        if (most > ((1 << 30) - 1) / cache->heads) return BFQ_ERR_TOO_LARGE;
        part->most = int(most), pairs += places * cache->heads;
    }
    if (pairs >= int64_t(1) << 27) return BFQ_ERR_TOO_LARGE;
    static_assert(kTallRows == 1 << 8, "shift");
    p->scale_log2 = in->scale * 1.4426950408889634f;
    p->tw = plan->tw, p->status = plan->status_word;
    return BFQ_OK;
}

}  // namespace kv
}  // namespace bfq

using namespace bfq;

namespace {
// CTAs of the two launches, no more than there can be units; a kernel that has no work: 0
cudaError_t ctas_of_both(const bfq_plan* plan, const kv::AttendParams& p, int* few, int* tall) {
    *few = *tall = 0;
    auto least = [&](const kv::Part& part, int ctas) {
        const int most = part.most * p.cache.heads;
        return most < ctas ? (most > 1 ? most : 1) : ctas;
    };
    cudaError_t e = cudaSuccess;
    if (p.entries(p.few) > 0) e = kv::attend(plan, p, few), *few = least(p.few, *few);
    if (e == cudaSuccess && p.entries(p.tall) > 0) e = kv::tall_ctas(plan, p.cache.bits, tall), *tall = least(p.tall, *tall);
    return e;
}
}  // namespace

extern "C" size_t bfq_kv_attend_workspace(const bfq_plan* plan, const bfq_kv_cache* cache, const bfq_kv_queries* in) {
    kv::AttendParams p{};
    if (kv::set_up(plan, cache, in, &p) != BFQ_OK || p.batch == 0) return 0;
    kv::OnDevice guard(plan->device);
    int few = 0, tall = 0;
    if (!guard.ok || ctas_of_both(plan, p, &few, &tall) != cudaSuccess) return 0;
    return kv::lay_out(&p, plan->n, few, tall, nullptr);
}

extern "C" int bfq_kv_attend(bfq_plan* plan, const bfq_kv_cache* cache, const bfq_kv_queries* in, void* workspace, size_t workspace_bytes, void* stream) {
    kv::AttendParams p{};
    const int rc = kv::set_up(plan, cache, in, &p);
    if (rc != BFQ_OK || p.batch == 0) return rc;
    kv::OnDevice guard(plan->device);
    if (!guard.ok) return BFQ_ERR_CUDA;
    int few = 0, tall = 0;
    cudaError_t e = ctas_of_both(plan, p, &few, &tall);
    if (e == cudaSuccess) {
        if (workspace == nullptr || workspace_bytes < kv::lay_out(&p, plan->n, few, tall, nullptr)) return BFQ_ERR_WORKSPACE;
        if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return BFQ_ERR_ALIGN;
        kv::lay_out(&p, plan->n, few, tall, static_cast<uint8_t*>(workspace));
        cudaStream_t st = static_cast<cudaStream_t>(stream);
        p.beside_tall = tall > 0, p.few.ctas = few, p.tall.ctas = tall;
        if (tall > 0) e = kv::tall_launch(plan, p, tall, st);
        if (e == cudaSuccess && few > 0) e = kv::attend(plan, p, nullptr, few, st);
        if (e == cudaSuccess && p.join_tall) e = kv::join_tall_launch(plan, p, st);
        if (e == cudaSuccess) {
            // a warp for each row where that is fewer than the chip runs at once; more would only load the butterfly's constants again
            const int64_t rows = p.tokens * p.q.heads, warps = int64_t(plan->sm_count) * 16, each = (rows + warps - 1) / warps;
            const dim3 grid(unsigned((rows + 4 * each - 1) / (4 * each)) + 1);
            e = plan->n == 64 ? launch_overlapped(kv::k_join<64>, grid, dim3(128), 0, st, p, int(each)) : launch_overlapped(kv::k_join<128>, grid, dim3(128), 0, st, p, int(each));
        }
    }
    if (e == cudaSuccess) return BFQ_OK;
    plan->last_cuda_error = static_cast<int>(e);
    return BFQ_ERR_CUDA;
}
