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
// A CTA of four warps takes units of 64 keys, 16 keys to a warp, through a ring of stages that cp.async fills some units ahead
// (16-byte chunks, chunk i of a unit at place i ^ (i / 8 mod 8): the reads below hit every bank once).  mma.m16n8k16: the 16 rows are
// the queries of a key head's group.  Keys come as words of a row, 8 (4) codes at a time; which k index of the product an element gets is
// free as long as the queries' fragments have the same order, so no code moves between lanes.  Values come by ldmatrix.trans on 16-bit
// units of 4 (2) codes: the halves of a register are two keys' codes of the same elements, which is what the second product needs.
#include "bfq_kvattn.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kWarps = 4, kAttendThreads = 32 * kWarps;

template <int D, int BITS>
struct Stage {
    static constexpr int kRow = D * BITS / 8;             // bytes of a row's codes
    static constexpr int kChunks = kFewUnit * kRow / 16;     // of a unit's keys (and as many of its values)
    static constexpr int kScales = 2 * kFewUnit * kRow;      // keys' scales behind both, then the values'
    static constexpr int kBytes = kScales + 4 * kFewUnit;
    static constexpr int kCount = kBytes > 12000 ? 4 : 6;
};
constexpr int kMergeRows = 2 * kFewRows;
template <int D, int BITS>
constexpr size_t attend_smem() {
    return size_t(Stage<D, BITS>::kCount) * Stage<D, BITS>::kBytes + sizeof(float) * kMergeRows * (D + 4) + 4 * kFewRows * sizeof(float2);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16u : 0u) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
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
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
template <int D, int BITS>
__global__ void __launch_bounds__(kAttendThreads) k_attend(const AttendParams p) {
    using S = Stage<D, BITS>;
    constexpr int kSteps = D / 16, kTilesD = D / 8;
    extern __shared__ __align__(128) uint8_t smem[];
    float* const merge = reinterpret_cast<float*>(smem + S::kCount * S::kBytes);  // [2][16][D + 4]
    float2* const warp_sums = reinterpret_cast<float2*>(merge + kMergeRows * (D + 4));
    __shared__ long long scan[kWarps + 3];
    const uint32_t ring = smem_u32(smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    grid_dep_wait();

    const Part& part = p.few;
    Walk<kFewRows, kFewUnit> ahead;
    const Run run = find_run<kAttendThreads>(p, part, scan, &ahead);
    if (run.count == 0) return;
    Walk<kFewRows, kFewUnit> now = ahead;
    const int count = run.count, heads = p.cache.heads;

    // ---- copies ----------------------------------------------------------------------------------------------------------
    auto fetch = [&](int i) {
        if (i < count) {
            const uint32_t stage = ring + (i % S::kCount) * S::kBytes;
            const int key0 = ahead.unit * kFewUnit;
            const int mask = (1 << p.cache.page_shift) - 1;
#pragma unroll
            for (int c = 0; c < S::kChunks; c += kAttendThreads) {
                const int i16 = c + tid;
                if (S::kChunks % kAttendThreads != 0 && i16 >= S::kChunks) break;
                const int key = key0 + i16 / (S::kRow / 16), part = i16 % (S::kRow / 16);
                const int64_t found = key < ahead.tile.keys ? page_of(p, ahead.tile, key) : -1, page = found < 0 ? 0 : found;
                const bool there = found >= 0;  // else zeros
                const uint32_t dst = stage + 16 * (i16 ^ ((i16 >> 3) & 7));
                copy16(dst, codes_of<S::kRow>(p.cache.k, p.cache.page_shift, page, ahead.head, key & mask) + 16 * part, there);
                copy16(dst + kFewUnit * S::kRow, codes_of<S::kRow>(p.cache.v, p.cache.page_shift, page, ahead.head, key & mask) + 16 * part, there);
            }
            if (tid < 2 * kFewUnit / 8) {
                const int key = key0 + 8 * (tid % (kFewUnit / 8));
                const bool values = tid >= kFewUnit / 8;
                const int64_t found = key < ahead.tile.keys ? page_of(p, ahead.tile, key) : -1, page = found < 0 ? 0 : found;
                const bool there = found >= 0;
                copy16(stage + S::kScales + 16 * tid, scale_of(values ? p.cache.v : p.cache.k, p.cache.page_shift, page, ahead.head, key & mask), there);
            }
            ahead.next(p, part);
        }
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < S::kCount - 1; ++i) fetch(i);

    // ---- a pair's state: fragments of the queries, reference, sums and products -------------------------------------------
    uint32_t qa[kSteps][4];
    float m[2], l[2], o[kTilesD][4];
    float row_scale_log2[2];  // softmax scale * log2 e over the row's power of two
    float u_top, u_unit;      // power of two that no u so far passes; 128 / u_top: probabilities (at most 2^8) times u stay below 2^15
    int limit[2];             // keys of rows g and g + 8
    bool two;                 // there are rows 8 and up
    auto open = [&]() {
        const Tile& tl = now.tile;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = g + 8 * half, row = tl.row0 + r;
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
            row_scale_log2[half] = p.scale_log2 * power.down;
            auto element = [&](int i) { return power.up * __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16); };
            auto pair = [&](int i, int j) { return half_pair(element(i), element(j)); };
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if constexpr (BITS == 4) {
                    const int d = 8 * (s / 2) + 2 * (s & 1);
                    qa[s][half] = pair(d, d + 4), qa[s][2 + half] = pair(d + 1, d + 5);
                } else {
                    qa[s][half] = pair(4 * s, 4 * s + 2), qa[s][2 + half] = pair(4 * s + 1, 4 * s + 3);
                }
            }
            m[half] = -INFINITY, l[half] = 0.f;
            const int own = tl.last0 + row / p.group + 1;
            limit[half] = there ? (own < tl.keys ? own : tl.keys) : 0;
        }
        two = tl.rows > 8, u_top = 0.f, u_unit = 0.f;
#pragma unroll
        for (int i = 0; i < kTilesD; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
    };
    long long pair_from = run.from - now.unit;  // number of the pair's unit 0
    auto close = [&](long long done) {      // after unit `done` (exclusive) of the numbering
        const int pair = now.pair(p);
        const long long entry = blockIdx.x + pair;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            l[half] += __shfl_xor_sync(0xFFFFFFFFu, l[half], 1);
            l[half] += __shfl_xor_sync(0xFFFFFFFFu, l[half], 2);
            if (t == 0) warp_sums[warp * kFewRows + g + 8 * half] = make_float2(m[half], l[half]);
        }
        __syncthreads();
        float f[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float top = -INFINITY, sum = 0.f;
            float2 ml[kWarps];
#pragma unroll
            for (int w = 0; w < kWarps; ++w) ml[w] = warp_sums[w * kFewRows + g + 8 * half], top = fmaxf(top, ml[w].x);
            const float safe = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) sum += ml[w].y * exp2_fast(ml[w].x - safe);
            f[half] = exp2_fast(m[half] - safe) * (u_top * (1.f / 128.f));
            if (warp == 0 && t == 0 && g + 8 * half < now.tile.rows) part.sums[entry * kFewRows + g + 8 * half] = make_float2(top, sum);
        }
        // d of accumulator i, column 2 t + j: see the values' order below
        auto column = [&](int i, int j) {
            constexpr int kPer = 32 / BITS / 2;  // codes of a 16-bit unit
            return (i / kPer) * 8 * kPer + kPer * (2 * t + j) + i % kPer;
        };
        auto put = [&](float* to, bool add) {
#pragma unroll
            for (int i = 0; i < kTilesD; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float* at = to + (g + 8 * (j >> 1)) * (D + 4) + column(i, j & 1);
                    const float v = o[i][j] * f[j >> 1];
                    *at = add ? *at + v : v;
                }
        };
        if (warp >= 2) put(merge + (warp - 2) * kFewRows * (D + 4), false);
        __syncthreads();
        if (warp < 2) put(merge + warp * kFewRows * (D + 4), true);
        __syncthreads();
        for (int i = tid; i < now.tile.rows * (D / 4); i += kAttendThreads) {
            const int r = i / (D / 4), c = 4 * (i % (D / 4));
            const float4 a = *reinterpret_cast<const float4*>(merge + r * (D + 4) + c), b = *reinterpret_cast<const float4*>(merge + (kFewRows + r) * (D + 4) + c);
            *reinterpret_cast<float4*>(part.parts + (entry * kFewRows + r) * D + c) = make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
        }
        if (tid == 0 && pair_from >= run.from) part.pairs[pair] = make_int2(blockIdx.x, static_cast<int>((pair_from + now.units - 1) / run.per - blockIdx.x + 1));
        pair_from = done;
    };

    open();
    for (int i = 0; i < count; ++i) {
        copies_wait<S::kCount - 2>();
        __syncthreads();
        fetch(i + S::kCount - 1);
        const uint32_t stage = ring + (i % S::kCount) * S::kBytes;
        const int key0 = now.unit * kFewUnit + 16 * warp;
        // ---- scores of 16 keys: key 8 j + g of the warp's is column g of tile j
        float s[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = 16 * warp + 8 * j + g;
            constexpr int kWords = D * BITS / 128;  // of a lane
            uint32_t w[kWords];
            if constexpr (kWords == 2) {
                const int i16 = key * (S::kRow / 16) + (t >> 1);
                const uint2 v = lds64(stage + 16 * (i16 ^ ((i16 >> 3) & 7)) + 8 * (t & 1));
                w[0] = v.x, w[1] = v.y;
            } else {
#pragma unroll
                for (int c = 0; c < kWords / 4; ++c) {
                    const int i16 = key * (S::kRow / 16) + t * (kWords / 4) + c;
                    const uint4 v = lds128(stage + 16 * (i16 ^ ((i16 >> 3) & 7)));
                    w[4 * c] = v.x, w[4 * c + 1] = v.y, w[4 * c + 2] = v.z, w[4 * c + 3] = v.w;
                }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) s[j][c] = 0.f;
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                uint32_t b0, b1;
                if constexpr (BITS == 4) b0 = pair4(w[st / 2], 2 * (st & 1)), b1 = pair4(w[st / 2], 2 * (st & 1) + 1);
                else b0 = pair8(w[st], 0), b1 = pair8(w[st], 1);
                mma16816(s[j], qa[st][0], qa[st][1], qa[st][2], qa[st][3], b0, b1);
            }
        }
        // ---- scales, masks, probabilities
        float u[2][2];
        bool over = false;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t at = stage + S::kScales + 2 * (16 * warp + 8 * j + 2 * t);
            const uint32_t ks = lds32(at), vs = lds32(at + 2 * kFewUnit);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int key = key0 + 8 * j + 2 * t + c;
                const float f = half_value(static_cast<uint16_t>(ks >> (16 * c)));
                u[j][c] = key < now.tile.keys ? half_value(static_cast<uint16_t>(vs >> (16 * c))) : 0.f;
                over |= u[j][c] > u_top;
                s[j][c] = key < limit[0] ? s[j][c] * f * row_scale_log2[0] : -INFINITY;
                over |= s[j][c] > m[0] + 8.f;
                if (two) {
                    s[j][2 + c] = key < limit[1] ? s[j][2 + c] * f * row_scale_log2[1] : -INFINITY;
                    over |= s[j][2 + c] > m[1] + 8.f;
                }
            }
        }
        if (__any_sync(0xFFFFFFFFu, over)) {
            float most = fmaxf(fmaxf(u[0][0], u[0][1]), fmaxf(u[1][0], u[1][1]));
            most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
            float less = 1.f;  // on the products
            if (most > u_top) {
                const float top = __uint_as_float((__float_as_uint(most) & 0x7F800000u) + 0x00800000u);  // above it
                less = u_top / top, u_top = top, u_unit = 128.f / top;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float f = 1.f;
                if (half == 0 || two) {
                    float top = fmaxf(fmaxf(s[0][2 * half], s[0][2 * half + 1]), fmaxf(s[1][2 * half], s[1][2 * half + 1]));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                    top = fmaxf(top, m[half]);
                    f = top == -INFINITY ? 1.f : exp2_fast(m[half] - top);
                    m[half] = top, l[half] *= f;
                }
                f *= less;
#pragma unroll
                for (int i = 0; i < kTilesD; ++i) o[i][2 * half] *= f, o[i][2 * half + 1] *= f;
            }
        }
        uint32_t pa[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j) u[j][0] *= u_unit, u[j][1] *= u_unit;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half == 1 && !two) break;
            const float ref = m[half] == -INFINITY ? 0.f : m[half];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float a = exp2_fast(s[j][2 * half] - ref), b = exp2_fast(s[j][2 * half + 1] - ref);
                l[half] += a + b;
                pa[half + 2 * j] = half_pair(a * u[j][0], b * u[j][1]);
            }
        }
        // ---- values: matrix (8 keys) x (a 16-byte chunk), its 16-bit units across the lanes
        constexpr int kPer = 16 / BITS, kMats = S::kRow / 16;
#pragma unroll
        for (int c = 0; c < kMats; c += 2) {
            const int key = 16 * warp + (lane & 15), i16 = key * kMats + c + (lane >> 4);
            uint32_t r[4];  // keys 0 .. 7 and 8 .. 15 of chunk c, then of chunk c + 1
            ldmatrix4_trans(stage + kFewUnit * S::kRow + 16 * (i16 ^ ((i16 >> 3) & 7)), r);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < kPer; ++n) {
                    uint32_t b0, b1;
                    if constexpr (BITS == 4) b0 = pair4(r[2 * h], n), b1 = pair4(r[2 * h + 1], n);
                    else b0 = pair8(r[2 * h], n), b1 = pair8(r[2 * h + 1], n);
                    mma16816(o[(c + h) * kPer + n], pa[0], pa[1], pa[2], pa[3], b0, b1);
                }
        }
        if (now.unit + 1 == now.units || i + 1 == count) {
            close(run.from + i + 1);
            now.next(p, part);
            if (i + 1 < count) open();
        } else {
            ++now.unit;
        }
    }
    copies_wait<0>();
}

// Joins a row's partial results (the shared prefix's, then its sequence's), turns it back by Q^T and rounds it once.  A warp for each
// (token, query head).
template <int D>
__global__ void __launch_bounds__(128) k_join(const AttendParams p) {
    constexpr int kE = D / 32;
    const int lane = threadIdx.x & 31;
    grid_dep_wait();
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
    const int q_heads = p.q.heads;
    if (row >= p.tokens * q_heads) return;
    const int token = static_cast<int>(row / q_heads), head = static_cast<int>(row % q_heads), h = head / p.group;
    int b = token, place = 0;
    if (token < first_token(p, 0) || token >= first_token(p, p.batch)) return;  // rows of no sequence stay as they are
    if (p.q_starts != nullptr) {                   // the last sequence that starts at or before this token
        int lo = 0, hi = p.batch;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (first_token(p, mid) <= token) lo = mid;
            else hi = mid;
        }
        b = lo, place = token - first_token(p, b);
    }
    Turn<D, kE, true> turn;
    turn.load(p.tw, lane);
    float m = -INFINITY, l = 0.f, o[kE];
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = 0.f;
    auto join = [&](bool tall, int b, int row) {  // b < 0: the prefix
        const Part& part = tall ? p.tall : p.few;
        const int rows = tall ? kTallRows : kFewRows, r = row % rows, entry = (b < 0 ? 0 : part.tiles_prefix + b * part.tiles_seq) + row / rows;
        if ((tall ? tile_of<kTallRows>(p, part, entry) : tile_of<kFewRows>(p, part, entry)).keys == 0) return;
        const int pair = entry * p.cache.heads + h;
        const int2 ctas = load_plain(part.pairs + pair);
        const int64_t first = static_cast<int64_t>(ctas.x) + pair;
        for (int i = 0; i < ctas.y; ++i) {
            const int64_t at = (first + i) * rows + r;
            const float2 ml = load_plain(part.sums + at);
            const float top = fmaxf(m, ml.x), safe = top == -INFINITY ? 0.f : top;
            const float fa = exp2_fast(m - safe), fb = exp2_fast(ml.x - safe);
            float v[kE];
            if constexpr (kE == 4) {
                const float4 u = load_plain(reinterpret_cast<const float4*>(part.parts + at * D) + lane);
                v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
            } else {
                const float2 u = load_plain(reinterpret_cast<const float2*>(part.parts + at * D) + lane);
                v[0] = u.x, v[1] = u.y;
            }
            m = top, l = l * fa + ml.y * fb;
#pragma unroll
            for (int e = 0; e < kE; ++e) o[e] = o[e] * fa + v[e] * fb;
        }
    };
    if (p.prefix_length > 0) join(p.prefix_tall != 0, -1, token * p.group + head % p.group);
    if (place < p.max_new) join(p.seq_tall != 0, b, place * p.group + head % p.group);
    else if (lane == 0) atomicExch(p.status, kBadIndex);  // more new tokens than the call was told
    const float f = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] *= f;
    turn.apply(o);
    uint8_t* out = const_cast<uint8_t*>(p.out.data) + (token * p.out.token + head * p.out.head + kE * lane) * 2;
    if constexpr (kE == 4) *reinterpret_cast<uint2*>(out) = make_uint2(bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3]));
    else *reinterpret_cast<uint32_t*>(out) = bf16_pair(o[0], o[1]);
    if (p.lse != nullptr && lane == 0) p.lse[row] = l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    // a length or a start outside its range was taken as the nearest one inside
    if (lane == 0 && head == 0 && place == 0) {
        const int n = load_plain(p.lengths + b);
        if (n < 0 || n > p.table_width << p.cache.page_shift) atomicExch(p.status, kBadIndex);
    }
}

// CTAs of the first kernel: all that the chip runs at once
template <int D, int BITS>
static cudaError_t attend_ctas(const bfq_plan* plan, int* ctas) {
    static int per_sm[kMaxDevices] = {0};
    int& occ = per_sm[plan->device];
    if (occ == 0) {
        cudaError_t e = cudaFuncSetAttribute(k_attend<D, BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(attend_smem<D, BITS>()));
        int n = 0;
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k_attend<D, BITS>, kAttendThreads, attend_smem<D, BITS>());
        if (e != cudaSuccess) return e;
        occ = n > 0 ? n : 1;
    }
    *ctas = plan->sm_count * occ;
    return cudaSuccess;
}
template <int D, int BITS>
static cudaError_t launch_attend(const AttendParams& p, int ctas, cudaStream_t st) {
    return launch_overlapped(k_attend<D, BITS>, dim3(unsigned(ctas)), dim3(kAttendThreads), attend_smem<D, BITS>(), st, p);
}
static cudaError_t ctas_of(const bfq_plan* plan, int bits, int* ctas) {
    return plan->n == 64 ? (bits == 4 ? attend_ctas<64, 4>(plan, ctas) : attend_ctas<64, 8>(plan, ctas))
                         : (bits == 4 ? attend_ctas<128, 4>(plan, ctas) : attend_ctas<128, 8>(plan, ctas));
}

// Tiles of 256 rows where there are rows enough to pay for them.
static bool use_tall(int64_t rows) { return rows > 48; }

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
        const size_t pairs = size_t(p->entries(part)) * p->cache.heads, rows = (pairs + (tall ? ctas_tall : ctas_few)) * (tall ? kTallRows : kFewRows);
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
        in->prefix_length > int64_t(in->prefix_pages) << p->cache.page_shift)
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
    if (in->q_starts == nullptr ? in->tokens < in->batch : in->max_new < 1 || in->max_new > in->tokens) return BFQ_ERR_STRIDE;
    p->lse = in->lse, p->block_table = in->block_table, p->table_ld = in->table_ld, p->table_width = in->table_width, p->lengths = in->lengths;
    p->q_starts = in->q_starts, p->prefix = in->prefix, p->prefix_pages = in->prefix_pages, p->prefix_length = int(in->prefix_length);
    p->tokens = in->tokens, p->batch = in->batch, p->group = in->q.heads / cache->heads, p->max_new = in->q_starts == nullptr ? 1 : in->max_new;
    const int64_t rows = (in->q_starts == nullptr ? in->batch : in->tokens) * int64_t(p->group), rows_seq = int64_t(p->max_new) * p->group;
    p->prefix_tall = use_tall(rows), p->seq_tall = use_tall(rows_seq);
    const int tile_prefix = p->prefix_tall ? kTallRows : kFewRows, tile_seq = p->seq_tall ? kTallRows : kFewRows;
    const int64_t tiles_prefix = in->prefix_length > 0 ? (rows + tile_prefix - 1) / tile_prefix : 0, tiles_seq = (rows_seq + tile_seq - 1) / tile_seq;
    if ((tiles_prefix + tiles_seq * in->batch) * cache->heads >= int64_t(1) << 30) return BFQ_ERR_TOO_LARGE;
    (p->prefix_tall ? p->tall : p->few).tiles_prefix = int(tiles_prefix), (p->seq_tall ? p->tall : p->few).tiles_seq = int(tiles_seq);
    p->scale_log2 = in->scale * 1.4426950408889634f;
    p->tw = plan->tw, p->status = plan->status_word;
    return BFQ_OK;
}

}  // namespace kv
}  // namespace bfq

using namespace bfq;

namespace {
// CTAs of the two launches; a kernel that has no work: 0
cudaError_t ctas_of_both(const bfq_plan* plan, const kv::AttendParams& p, int* few, int* tall) {
    *few = *tall = 0;
    cudaError_t e = cudaSuccess;
    if (p.entries(p.few) > 0) e = kv::ctas_of(plan, p.cache.bits, few);
    if (e == cudaSuccess && p.entries(p.tall) > 0) e = kv::tall_ctas(plan, p.cache.bits, tall);
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
        const bool four = cache->bits == 4;
        if (tall > 0) e = kv::tall_launch(plan, p, tall, st);
        if (e == cudaSuccess && few > 0)
            e = plan->n == 64 ? (four ? kv::launch_attend<64, 4>(p, few, st) : kv::launch_attend<64, 8>(p, few, st))
                              : (four ? kv::launch_attend<128, 4>(p, few, st) : kv::launch_attend<128, 8>(p, few, st));
        if (e == cudaSuccess) {
            const dim3 grid(unsigned((p.tokens * p.q.heads + 3) / 4));
            e = plan->n == 64 ? launch_overlapped(kv::k_join<64>, grid, dim3(128), 0, st, p) : launch_overlapped(kv::k_join<128>, grid, dim3(128), 0, st, p);
        }
    }
    if (e == cudaSuccess) return BFQ_OK;
    plan->last_cuda_error = static_cast<int>(e);
    return BFQ_ERR_CUDA;
}
