// Rows into and out of the paged low-bit key/value cache.
//
// bfq_kv_append, one pass over a step's new tokens:  z = w x / sqrt(mean x^2 + eps) per head (queries and keys, where norms are given),
// the position's rotation on the first R elements of a head (pairs (i, i + R/2) or (2i, 2i + 1), cos and sin from a table), y = Q z, and
//     queries      y as bf16
//     keys, values s = fp16(max |y| / qmax), codes = clip(round(y / s)) in the page and place of the token's slot.
// Values are rotated by Q alone.  bfq_kv_read: x = Q^T (s code), the rows at any slots in the model's basis.
//
// The kernels below are for many rows (bfq_kvrows_few.cu has those for few): the butterfly as one dense product on the tensor cores, 128
// rows to a tcgen05.mma.  A thread owns a row of D = 64 or 128 elements, all of it in registers, so that norms and maxima need no exchange; a
// warp's 32 consecutive rows (a token's heads share its angles) come through shared memory 16 bytes a lane, the next ones while these are worked
// on.  A row z, times the power of two that puts its largest element in [2^10, 2^11), is split into two fp16 terms, h + l, 22 bits; so is Q, times
// 2^10, built from the stages' cosines and sines in fp32 by each CTA.  y = h Qh + h Ql + l Qh in fp32: off by at most 2^-20 of |z| (both
// splits 2^-22 of their elements, l Ql 2^-22, the rest for the sums).  Rows read back are exact in one term: the codes, times their scale
// afterwards.  The terms go straight into tensor memory as the product's left operand; two groups of four warps take tiles in turn, one
// working while the other's product runs.
// For 16384 tokens of 32 + 2 x 8 heads this takes 162 us (119 without norms and rotation) of 2500 instructions for 32 rows.  Other forms: a row on 16
// lanes, stages by shuffles, 420 us; a row to a thread, stages in registers with their constants broadcast from shared memory, 235 us;
// this one with two threads to a row and twice the warps, which repeats a row's addresses, angles and partners, 191 us.
#include "bfq_generic.cuh"
#include "bfq_kvmma.cuh"
#include "bfq_kvrows.cuh"
#include "bfq_kvturn.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kGroups = 2, kRowsThreads = 128 * kGroups;  // groups of four warps

// Which tiles of 128 rows a group has: a CTA's consecutive, its groups' in turn.
struct Tiles {
    int at, end;
    __device__ __forceinline__ explicit Tiles(int rows) {
        const int tiles = (rows + 127) / 128, per = (tiles + gridDim.x - 1) / gridDim.x, from = per * blockIdx.x;
        end = from + per < tiles ? from + per : tiles;
        at = from + (threadIdx.x >> 7);
    }
    __device__ __forceinline__ bool there() const { return at < end; }
    // the thread's row of a tile; -1: of none
    __device__ __forceinline__ int row(int tile, int rows) const {
        const int r = tile * 128 + (threadIdx.x & 127);
        return tile < end && r < rows ? r : -1;
    }
};

// 16 bytes of a row as numbers, in pairs
template <bool F32>
__device__ __forceinline__ void unpack_chunk(uint4 v, u64* x) {  // bf16: 4 pairs, fp32: 2
    if constexpr (F32) {
        x[0] = pack2u(v.x, v.y), x[1] = pack2u(v.z, v.w);
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = pack2u(w[i] << 16, w[i] & 0xFFFF0000u);
    }
}
template <int D>
__device__ __forceinline__ float largest(const u64 (&x)[D / 2]) {  // NaN elements do not count, as in the other quantizers
    float top[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < D / 2; ++r) {
        float a, b;
        unpack2(x[r], a, b);
        top[r & 3] = fmaxf(top[r & 3], fmaxf(fabsf(a), fabsf(b)));
    }
    return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}
// An infinity as the largest number, so that its two terms are not NaN: with its row's factor infinite afterwards, a row with one becomes
// infinities of Q's signs, as the stages one by one make of it.
__device__ __forceinline__ uint32_t finite_pair(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// pairs (i, i + R / 2), R known to the compiler so that the row stays in registers
template <int D, int R>
__device__ __forceinline__ void turn_halves(u64 (&x)[D / 2], const float* table) {
#pragma unroll
    for (int i = 0; i < R / 8; ++i) {
        const uint4 c = load_plain(reinterpret_cast<const uint4*>(table) + i), s = load_plain(reinterpret_cast<const uint4*>(table + R / 2) + i);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u64 cc = h ? pack2u(c.z, c.w) : pack2u(c.x, c.y), ss = h ? pack2u(s.z, s.w) : pack2u(s.x, s.y), a = x[2 * i + h], b = x[R / 4 + 2 * i + h];
            x[2 * i + h] = sub2(mul2(cc, a), mul2(ss, b)), x[R / 4 + 2 * i + h] = fma2(ss, a, mul2(cc, b));
        }
    }
}
template <int D, int R = D>
__device__ __forceinline__ void turn_halves_of(int dims, u64 (&x)[D / 2], const float* table) {
    if (dims == R) turn_halves<D, R>(x, table);
    else if constexpr (R > 16) turn_halves_of<D, R - 16>(dims, x, table);
}
template <int D>
__device__ __forceinline__ void turn_neighbours(int dims, u64 (&x)[D / 2], const float* table) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
        if (8 * i < dims) {
            const float4 c = load_plain(reinterpret_cast<const float4*>(table) + i), s = load_plain(reinterpret_cast<const float4*>(table + dims / 2) + i);
            const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float a, b;
                unpack2(x[4 * i + r], a, b);
                x[4 * i + r] = pack2(fmaf(a, cs[r], -b * sn[r]), fmaf(b, cs[r], a * sn[r]));
            }
        }
}

// Place in its eight of element i, for left operands whose elements stand in the order that codes come out in.
template <int BITS>
__host__ __device__ constexpr int place_of(int i) {
    return BITS == 4 ? (i < 4 ? 2 * i : 2 * i - 7) : (i & 4) + ((i >> 1) & 1) + 2 * (i & 1);
}

// Q (or, for rows read back, Q^T) as right operand, K-major, times 2^10 in two fp16 terms: [2 terms][D / 64 halves of k][D rows n][128 bytes].
// Entry (i, j) of Q is a product over the stages: when stage s comes, the element that leads from j to i has i's bits below s and j's from s
// on; its pair gives c if bit s of i and j are the same, else s (i's is 1) or -s.  Products over the stages from s on depend on j's bits from s on
// alone, so that a thread with half a row of Q makes D / 2 entries with D / 2 multiplications and a few.
template <int D, bool READ, int BITS>
__device__ __forceinline__ void build_matrix(uint32_t to, const float2* tw) {
    constexpr int kStages = D == 64 ? 6 : 7;
    constexpr uint32_t kTerm = D * D * 2;
    const int i = threadIdx.x % D, w = threadIdx.x / D;  // row, upper bit of j
    if (w < 2) {
        float v[D / 2];
        v[0] = 1.f;
        int n = 1;
#pragma unroll
        for (int s = kStages - 1; s >= 0; --s) {
            const bool one = i >> s & 1;
            if (s == kStages - 1) {
                const float2 t = load_plain(tw + s * (D / 2) + (i & ((1 << s) - 1)));
                v[0] = (one == (w == 1)) ? t.x : (one ? t.y : -t.y);
            } else {
#pragma unroll
                for (int k = D / 4 - 1; k >= 0; --k)
                    if (k < n) {
                        const float2 t = load_plain(tw + s * (D / 2) + (((w * n + k) << s) | (i & ((1 << s) - 1))));
                        const float x = v[k];
                        v[2 * k] = x * (one ? t.y : t.x), v[2 * k + 1] = x * (one ? t.x : -t.y);
                    }
                n *= 2;
            }
        }
        auto split = [](float x, uint16_t& hi, uint16_t& lo) {
            const __half h = __float2half_rn(x);
            hi = __half_as_ushort(h), lo = __half_as_ushort(__float2half_rn(x - __half2float(h)));
        };
        if constexpr (!READ) {  // n = i, k = j
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint16_t h[2], l[2];
                    split(v[8 * c + 2 * e] * 1024.f, h[0], l[0]), split(v[8 * c + 2 * e + 1] * 1024.f, h[1], l[1]);
                    hi[e] = h[0] | uint32_t(h[1]) << 16, lo[e] = l[0] | uint32_t(l[1]) << 16;
                }
                const int j = w * (D / 2) + 8 * c;
                const uint32_t at = to + (j >> 6) * (D * 128) + i * 128 + (((j >> 3 & 7) ^ (i & 7)) << 4);
                store16(at, hi[0], hi[1], hi[2], hi[3]), store16(at + kTerm, lo[0], lo[1], lo[2], lo[3]);
            }
        } else {  // n = j, k = the place of i
            const int k = (i & ~7) + place_of<BITS>(i & 7);
#pragma unroll
            for (int c = 0; c < D / 2; ++c) {
                const int j = w * (D / 2) + c;
                const uint32_t at = to + (k >> 6) * (D * 128) + j * 128 + (((k >> 3 & 7) ^ (j & 7)) << 4) + 2 * (k & 7);
                uint16_t hi, lo;
                split(v[c] * 1024.f, hi, lo);
                asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(hi) : "memory");
                asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + kTerm), "h"(lo) : "memory");
            }
        }
    }
    fence_operands();
}

// Shared memory: the matrix, weights of queries' and keys' norms and ones, each warp's rows in and out.
template <int D, int IN, int OUT, bool ONE>  // bytes of a row; ONE: rows go out through the place of those that came in
struct RowsSmem {
    static constexpr int kInPitch = IN + 16, kOutPitch = OUT + 16;
    static constexpr uint32_t kNorms = 4 * D * D, kBars = kNorms + 3 * D * 4, kWarps = kBars + 64, kOut = ONE ? 0 : 32 * kInPitch,
                              kWarp = ONE ? 32 * (kInPitch > kOutPitch ? kInPitch : kOutPitch) : 32 * (kInPitch + kOutPitch);
    static constexpr uint32_t kBytes = kWarps + (kRowsThreads / 32) * kWarp + 1024;  // and what rounding the base up to 1024 takes
    static constexpr int kCtas = kBytes < 110000 ? 2 : 1;                            // on an SM; they share tensor memory
};
template <int COLUMNS>
__device__ __forceinline__ void tensor_memory(uint32_t at) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(at), "n"(COLUMNS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int COLUMNS>
__device__ __forceinline__ void tensor_memory_free(uint32_t at) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "n"(COLUMNS) : "memory");
}

// The product of a group's 128 rows, whose TERMS terms of fp16 are in tensor memory (D / 2 columns each, then the result's D): all threads of the
// group call it, and have the result in tensor memory when it returns.
template <int D, int TERMS>
__device__ __forceinline__ void multiply(uint32_t columns, uint32_t matrix, uint32_t bar, uint32_t& phase, volatile int* dead, int* status) {
    tmem_wait_st();
    tmem_fence_before();
    bar_sync(1 + (threadIdx.x >> 7), 128);
    if ((threadIdx.x >> 5 & 3) == 0) {
        tmem_fence_after();
        const uint32_t lead = elect_one();
#pragma unroll
        for (int term = 0; term < TERMS + 1; ++term)  // h Qh, h Ql, l Qh
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                mma_ts(lead, columns + D, columns + (term == 2 ? D / 2 : 0) + 8 * k, operand(matrix + (term == 1 ? D * D * 2 : 0) + (k >> 2) * (D * 128) + (k & 3) * 32, 0),
                       instruction(D, 0), term > 0 || k > 0);
        commit_to(lead, bar);
    }
    wait_for(bar, phase, dead, status);
    phase ^= 1;
    tmem_fence_after();
}
// Before the CTA ends: products in flight after a wait has given up.  done: a barrier of the group's own.
__device__ __forceinline__ void products_done(uint32_t done, volatile int* dead) {
    if ((threadIdx.x >> 5 & 3) == 0 && __any_sync(0xFFFFFFFFu, *dead)) {
        commit_to(elect_one(), done);
        drain(done, 0);
    }
}
// the result's row, times f
template <int D>
__device__ __forceinline__ void result_row(uint32_t at, float f, u64 (&x)[D / 2]) {
    const u64 f2 = pack2(f, f);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        uint32_t v[32];
        tmem_ld32(at + 32 * c, v);
        tmem_wait_ld32(v);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[16 * c + i] = mul2(pack2u(v[2 * i], v[2 * i + 1]), f2);
    }
}

template <int D, bool F32>
using AppendSmem = RowsSmem<D, D*(F32 ? 4 : 2), 2 * D, F32>;

template <int D, bool F32, int BITS>
__global__ void __launch_bounds__(kRowsThreads, AppendSmem<D, F32>::kCtas) k_append(const AppendParams p) {
    using S = AppendSmem<D, F32>;
    constexpr int kIn = D * (F32 ? 4 : 2), kCodes = D * BITS / 8;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int dead;
    grid_dep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, norms = base + S::kNorms, in = base + S::kWarps + warp * S::kWarp, out = in + S::kOut,
                   bar = base + S::kBars + 8 * (warp >> 2);
    const int heads = p.q.heads + 2 * p.cache.heads, rows = static_cast<int>(p.tokens) * heads;  // rows of a token: queries, keys, values
    Tiles tiles(rows);
    // The thread's row of a tile.  Found anew wherever it is needed, so that it takes no registers while the row is worked on.
    struct Row {
        int token, kind, head;  // 0 query, 1 key, 2 value, -1 none
    };
    auto find = [&](int tile) {
        const int row = tiles.row(tile, rows);
        Row r{row / heads, -1, 0};
        if (row < 0) return Row{0, -1, 0};
        const int i = row - r.token * heads;
        r.kind = i < p.q.heads ? 0 : (i < p.q.heads + p.cache.heads ? 1 : 2);
        r.head = r.kind == 0 ? i : (r.kind == 1 ? i - p.q.heads : i - p.q.heads - p.cache.heads);
        return r;
    };
    auto fetch = [&](const Row& r) {
        const Heads& from = r.kind == 0 ? p.q : (r.kind == 1 ? p.k : p.v);
        each_chunk<kIn, S::kInPitch>(from.data + (r.token * from.token + r.head * from.head) * (F32 ? 4 : 2), r.kind >= 0 ? kIn : 0,
                                     [&](uint32_t at, uint8_t* data) { copy_in(in + at, data); });
    };
    auto position_of = [&](const Row& r) { return p.positions != nullptr && (r.kind == 0 || r.kind == 1) ? load_plain(p.positions + r.token) : 0; };
    auto angles_of = [&](int position) { return p.rope + (position >= 0 && position < p.rope_rows ? position : 0) * int64_t(p.rope_dims); };
    fetch(find(tiles.at));
    if (threadIdx.x == 0) {
        for (int g = 0; g < 2 * kGroups; ++g) mbar_init(base + S::kBars + 8 * g, 1);  // of a product, of all after a wait has given up
        mbar_init_fence();
        dead = 0;
    }
    if (warp == 0) tensor_memory<4 * D>(smem_u32(&tmem_at));
    for (int i = threadIdx.x; i < D; i += kRowsThreads) {
        float* w = reinterpret_cast<float*>(smem_raw + (norms - smem_u32(smem_raw)));
        w[i] = p.q_norm != nullptr ? load_plain(p.q_norm + i) : 1.f, w[D + i] = p.k_norm != nullptr ? load_plain(p.k_norm + i) : 1.f, w[2 * D + i] = 1.f;
    }
    build_matrix<D, false, BITS>(base, p.tw);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t columns = tmem_at + 2 * D * (warp >> 2), mine = columns + (uint32_t(warp & 3) << 21);  // the group's; the warp's 32 lanes of them
    const bool normed = p.q_norm != nullptr || p.k_norm != nullptr;
    uint32_t phase = 0;
    for (; tiles.there(); tiles.at += kGroups) {
        const Row now = find(tiles.at), next = find(tiles.at + kGroups);
        const bool turned = p.positions != nullptr && (now.kind == 0 || now.kind == 1);
        const int position = position_of(now);
        float down;
        {
            u64 x[D / 2];
            copies_done();
            __syncwarp();
#pragma unroll
            for (int c = 0; c < kIn / 16; ++c) unpack_chunk<F32>(shared_load(in + lane * S::kInPitch + 16 * c), x + (F32 ? 2 : 4) * c);
            __syncwarp();
            if (!F32) fetch(next);  // fp32: the place is for the rows out first
            if (normed) {
                u64 sum = pack2(0.f, 0.f);
#pragma unroll
                for (int r = 0; r < D / 2; ++r) sum = fma2(x[r], x[r], sum);
                float a, b;
                unpack2(sum, a, b);
                const bool own = (now.kind == 0 && p.q_norm != nullptr) || (now.kind == 1 && p.k_norm != nullptr);
                const float f = own ? rsqrtf((a + b) * (1.f / D) + p.eps) : 1.f;
                const u64 f2 = pack2(f, f);
                const uint32_t w = norms + (own ? now.kind : 2) * D * 4;
#pragma unroll
                for (int k = 0; k < D / 4; ++k) {
                    const uint4 c = shared_load(w + 16 * k);
                    x[2 * k] = mul2(x[2 * k], mul2(f2, pack2u(c.x, c.y))), x[2 * k + 1] = mul2(x[2 * k + 1], mul2(f2, pack2u(c.z, c.w)));
                }
            }
            if (turned) {
                if (position < 0 || position >= p.rope_rows) atomicExch(p.status, kBadIndex);
                const float* const angles = angles_of(position);
                if (p.interleaved) turn_neighbours<D>(p.rope_dims, x, angles);
                else turn_halves_of<D>(p.rope_dims, x, angles);
            }
            const float top = largest<D>(x);
            const RowPower power(top);
            down = top == INFINITY ? INFINITY : power.down * (1.f / 1024.f);
            const u64 up2 = pack2(power.up, power.up);
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t h[16], l[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const u64 y = mul2(x[16 * c + i], up2);
                    float a, b;
                    unpack2(y, a, b);
                    h[i] = finite_pair(a, b);
                    const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
                    unpack2(sub2(y, pack2(back.x, back.y)), a, b);
                    l[i] = finite_pair(a, b);
                }
                tmem_st16(mine + 16 * c, h);
                tmem_st16(mine + D / 2 + 16 * c, l);
            }
        }
        multiply<D, 2>(columns, base, bar, phase, &dead, p.status);
        u64 x[D / 2];
        result_row<D>(mine + D, down, x);
        uint8_t* to = nullptr;
        int bytes = 0;
        if (now.kind == 0) {
            store_bf16<D>(out + lane * S::kOutPitch, x);
            to = const_cast<uint8_t*>(p.q_out.data) + (now.token * p.q_out.token + now.head * p.q_out.head) * 2, bytes = 2 * D;
        } else if (now.kind > 0) {
            constexpr float kTop = (1 << (BITS - 1)) - 1;
            const float top = largest<D>(x), scale = fminf(top * (1.f / kTop), 65504.f);
            const uint16_t stored = __half_as_ushort(__float2half_rn(scale));
            const float s = half_value(stored), inv = s > 0.f ? __fdividef(1.f, s) : 0.f;
            const u64 inv2 = pack2(inv, inv), magic = pack2(12582912.f, 12582912.f);  // the sum's low bits are the nearest integer
            const bool clip = !(top * inv < kTop + 0.499f);                           // a scale that was rounded down far, or cut
#pragma unroll
            for (int c = 0; c < kCodes / 16; ++c) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    constexpr int kCodesOfWord = 32 / BITS;
                    uint32_t v[kCodesOfWord];
#pragma unroll
                    for (int e = 0; e < kCodesOfWord; e += 2) {
                        u64 y = mul2(x[((4 * c + i) * kCodesOfWord + e) / 2], inv2);
                        if (clip) {
                            float a, b;
                            unpack2(y, a, b);
                            y = pack2(fminf(fmaxf(a, -kTop - 1.f), kTop), fminf(fmaxf(b, -kTop - 1.f), kTop));
                        }
                        unpack2u(add2(y, magic), v[e], v[e + 1]);
                    }
                    if constexpr (BITS == 4) {
                        uint32_t b[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) b[e] = (v[2 * e] & 15u) | (v[2 * e + 1] << 4);
                        w[i] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
                    } else {
                        w[i] = __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
                    }
                }
                shared_store(out + lane * S::kOutPitch + 16 * c, make_uint4(w[0], w[1], w[2], w[3]));
            }
            const int64_t slot = load_plain(p.slots + now.token), page = slot >> p.cache.page_shift;
            if (slot >= 0 && page >= p.cache.pages) atomicExch(p.status, kBadIndex);
            if (slot >= 0 && page < p.cache.pages) {
                const int place = static_cast<int>(slot) & ((1 << p.cache.page_shift) - 1);
                const Half& half = now.kind == 1 ? p.cache.k : p.cache.v;
                to = codes_of<kCodes>(half, p.cache.page_shift, page, now.head, place), bytes = kCodes;
                *scale_of(half, p.cache.page_shift, page, now.head, place) = stored;
            }
        }
        __syncwarp();
        each_chunk<2 * D, S::kOutPitch>(to, bytes, [&](uint32_t at, uint8_t* dst) { *reinterpret_cast<uint4*>(dst) = shared_load(out + at); });
        __syncwarp();
        if (F32) fetch(next);
    }
    copies_done();
    products_done(bar + 8 * kGroups, &dead);
    tmem_fence_before();
    __syncthreads();
    if (warp == 0) tensor_memory_free<4 * D>(tmem_at);
}

template <int D, bool F32, int BITS>
using ReadSmem = RowsSmem<D, D * BITS / 8, D*(F32 ? 4 : 2), F32>;

template <int D, bool F32, int BITS>
__global__ void __launch_bounds__(kRowsThreads, ReadSmem<D, F32, BITS>::kCtas) k_read(const ReadParams p) {
    using S = ReadSmem<D, F32, BITS>;
    constexpr int kIn = D * BITS / 8, kOut = D * (F32 ? 4 : 2);
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int dead;
    grid_dep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, in = base + S::kWarps + warp * S::kWarp, out = in + S::kOut, bar = base + S::kBars + 8 * (warp >> 2);
    const int heads = 2 * p.cache.heads, rows = static_cast<int>(p.tokens) * heads;  // rows of a token: keys, values
    Tiles tiles(rows);
    struct Row {
        const uint8_t* data;  // null: zeros
        uint16_t scale;
    };
    auto find = [&](int tile) {
        Row r{};
        const int row = tiles.row(tile, rows);
        if (row < 0) return r;
        const int token = row / heads, i = row - token * heads, head = i < p.cache.heads ? i : i - p.cache.heads;
        const int64_t slot = load_plain(p.slots + token), page = slot >> p.cache.page_shift;
        if (slot < 0) return r;
        if (page >= p.cache.pages) {
            atomicExch(p.status, kBadIndex);
            return r;
        }
        const int place = static_cast<int>(slot) & ((1 << p.cache.page_shift) - 1);
        const Half& half = i < p.cache.heads ? p.cache.k : p.cache.v;
        r.data = codes_of<kIn>(half, p.cache.page_shift, page, head, place);
        r.scale = *static_cast<volatile const uint16_t*>(scale_of(half, p.cache.page_shift, page, head, place));
        return r;
    };
    auto fetch = [&](const Row& r) { each_chunk<kIn, S::kInPitch>(r.data, r.data != nullptr ? kIn : 0, [&](uint32_t at, uint8_t* from) { copy_in(in + at, from); }); };
    Row now = find(tiles.at);
    fetch(now);
    if (threadIdx.x == 0) {
        for (int g = 0; g < 2 * kGroups; ++g) mbar_init(base + S::kBars + 8 * g, 1);  // of a product, of all after a wait has given up
        mbar_init_fence();
        dead = 0;
    }
    if (warp == 0) tensor_memory<4 * D>(smem_u32(&tmem_at));
    build_matrix<D, true, BITS>(base, p.tw);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t columns = tmem_at + 2 * D * (warp >> 2), mine = columns + (uint32_t(warp & 3) << 21);
    const Unpack<BITS> unpack;
    uint32_t phase = 0;
    for (; tiles.there(); tiles.at += kGroups) {
        copies_done();
        __syncwarp();
        uint4 raw[kIn / 16];
#pragma unroll
        for (int c = 0; c < kIn / 16; ++c) raw[c] = now.data != nullptr ? shared_load(in + lane * S::kInPitch + 16 * c) : make_uint4(0, 0, 0, 0);
        __syncwarp();
        const Row next = find(tiles.at + kGroups);
        if (!F32) fetch(next);  // fp32: the place is for the rows out first
        constexpr int kWords = D * BITS / 32, kPairs = 16 / BITS;  // of a row; of a word
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            uint32_t h[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int pair = 16 * c + i, word = pair / kPairs;
                static_assert(kWords * kPairs == D / 2, "a row");
                const uint32_t w = (word & 3) == 0 ? raw[word / 4].x : ((word & 3) == 1 ? raw[word / 4].y : ((word & 3) == 2 ? raw[word / 4].z : raw[word / 4].w));
                h[i] = unpack(w, pair % kPairs);
            }
            tmem_st16(mine + 16 * c, h);
        }
        multiply<D, 1>(columns, base, bar, phase, &dead, p.status);
        u64 x[D / 2];
        result_row<D>(mine + D, half_value(now.scale) * (1.f / 1024.f), x);
        if constexpr (F32) {
#pragma unroll
            for (int c = 0; c < D / 4; ++c) {
                uint4 v;
                unpack2u(x[2 * c], v.x, v.y), unpack2u(x[2 * c + 1], v.z, v.w);
                shared_store(out + lane * S::kOutPitch + 16 * c, v);
            }
        } else {
            store_bf16<D>(out + lane * S::kOutPitch, x);
        }
        __syncwarp();
        const int row = tiles.row(tiles.at, rows), token = row / heads, i = row - token * heads;
        uint8_t* const to = (i < p.cache.heads ? p.k : p.v) + (int64_t(token) * p.cache.heads + (i < p.cache.heads ? i : i - p.cache.heads)) * kOut;
        each_chunk<kOut, S::kOutPitch>(to, row >= 0 ? kOut : 0, [&](uint32_t at, uint8_t* dst) { *reinterpret_cast<uint4*>(dst) = shared_load(out + at); });
        __syncwarp();
        if (F32) fetch(next);
        now = next;
    }
    copies_done();
    products_done(bar + 8 * kGroups, &dead);
    tmem_fence_before();
    __syncthreads();
    if (warp == 0) tensor_memory_free<4 * D>(tmem_at);
}

// Rows of a call: below what a whole tile more for each group can bring past 31 bits.
constexpr int64_t kMostRows = (int64_t(1) << 31) - 128 * (kGroups + 1);

// as many CTAs as their shared memory lets run at once
template <class S, class Kernel, class Params>
static cudaError_t launch_rows(const bfq_plan* plan, Kernel kern, bool* ready, int64_t rows, const Params& p, cudaStream_t st) {
    if (!ready[plan->device]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(S::kBytes));
        if (e != cudaSuccess) return e;
        ready[plan->device] = true;
    }
    const int64_t want = (rows + 128 * kGroups - 1) / (128 * kGroups), most = int64_t(plan->sm_count) * S::kCtas;
    return launch_overlapped(kern, dim3(unsigned(want < most ? want : most)), dim3(kRowsThreads), S::kBytes, st, p);
}
// One line for appending and reading, either width and type.  Measured either side (us, few : many; 32 + 2 x 8 heads with norms and positions):
//     rows                  6144         9216         12288        16368        24576
//     append, n = 64, bf16  4.7 : 7.9    7.2 : 8.1    6.0 : 8.1    8.8 : 8.0    11.6 : 8.1
//                     fp32  4.9 : 8.6    7.1 : 8.5    6.0 : 8.6    9.1 : 8.5    11.7 : 8.5
//            n = 128, bf16  7.2 : 12.7  11.9 : 12.6  14.4 : 12.9  16.7 : 13.1  21.4 : 13.2
//                     fp32  7.2 : 13.8  12.3 : 14.1  14.7 : 13.8  16.4 : 14.2  22.1 : 14.2
//     read, n = 64          4.0 : 5.0    4.5 : 5.0    5.1 : 5.0    5.5 : 5.4     6.1 : 5.5
//           n = 128         6.7 : 8.1    7.0 : 8.1    7.7 : 8.2    8.6 : 8.1    10.1 : 8.5
// Appending at n = 128 would cross at some 10000 rows: up to 3.6 us are lost there between them and the line.
static bool few_rows(int64_t rows) { return rows < 16384; }

template <int D, bool F32, int BITS>
static cudaError_t launch_append_bits(const bfq_plan* plan, const AppendParams& p, cudaStream_t st) {
    static bool ready[kMaxDevices] = {false};
    return launch_rows<AppendSmem<D, F32>>(plan, k_append<D, F32, BITS>, ready, p.tokens * (p.q.heads + 2 * p.cache.heads), p, st);
}
template <int D, bool F32>
static cudaError_t launch_append(const bfq_plan* plan, const AppendParams& p, cudaStream_t st) {
    if (few_rows(p.tokens * (p.q.heads + 2 * p.cache.heads))) return append_few_launch(plan, p, F32, st);
    return p.cache.bits == 4 ? launch_append_bits<D, F32, 4>(plan, p, st) : launch_append_bits<D, F32, 8>(plan, p, st);
}
template <int D, bool F32, int BITS>
static cudaError_t launch_read_bits(const bfq_plan* plan, const ReadParams& p, cudaStream_t st) {
    static bool ready[kMaxDevices] = {false};
    return launch_rows<ReadSmem<D, F32, BITS>>(plan, k_read<D, F32, BITS>, ready, p.tokens * 2 * p.cache.heads, p, st);
}
template <int D, bool F32>
static cudaError_t launch_read(const bfq_plan* plan, const ReadParams& p, cudaStream_t st) {
    if (few_rows(p.tokens * 2 * p.cache.heads)) return read_few_launch(plan, p, F32, st);
    return p.cache.bits == 4 ? launch_read_bits<D, F32, 4>(plan, p, st) : launch_read_bits<D, F32, 8>(plan, p, st);
}

}  // namespace kv
}  // namespace bfq

using namespace bfq;

extern "C" int bfq_kv_append(bfq_plan* plan, const bfq_kv_cache* cache, const int64_t* slots, int64_t tokens, bfq_dtype xt, const bfq_heads* k,
                             const bfq_heads* v, const bfq_heads* q, const bfq_heads* q_out, const bfq_kv_positions* at, void* stream) {
    kv::AppendParams p{};
    int rc = kv::check_cache(plan, cache, &p.cache);
    if (rc != BFQ_OK) return rc;
    if (xt != BFQ_F32 && xt != BFQ_BF16) return BFQ_ERR_DTYPE;
    if (tokens < 0 || tokens >= int64_t(1) << 31) return BFQ_ERR_STRIDE;
    if (tokens == 0) return BFQ_OK;
    if (slots == nullptr || k == nullptr || v == nullptr || (q == nullptr) != (q_out == nullptr)) return BFQ_ERR_NULL;
    const int n = plan->n, esize = xt == BFQ_F32 ? 4 : 2;
    rc = kv::check_heads(k, n, esize, &p.k);
    if (rc == BFQ_OK) rc = kv::check_heads(v, n, esize, &p.v);
    if (rc == BFQ_OK && q != nullptr) rc = kv::check_heads(q, n, esize, &p.q);
    if (rc == BFQ_OK && q != nullptr) rc = kv::check_heads(q_out, n, 2, &p.q_out);
    if (rc != BFQ_OK) return rc;
    if (tokens * (p.q.heads + 2 * int64_t(cache->heads)) > kv::kMostRows) return BFQ_ERR_STRIDE;
    if (k->heads != cache->heads || v->heads != cache->heads || (q != nullptr && q_out->heads != q->heads)) return BFQ_ERR_STRIDE;
    if ((reinterpret_cast<uintptr_t>(slots) & 7u) != 0) return BFQ_ERR_ALIGN;
    if (at != nullptr) {
        if (at->positions != nullptr) {
            if (at->table == nullptr) return BFQ_ERR_NULL;
            if (at->dims < 16 || at->dims > n || at->dims % 16 != 0 || at->rows < 1) return BFQ_ERR_STRIDE;
            if ((reinterpret_cast<uintptr_t>(at->table) & 15u) != 0 || (reinterpret_cast<uintptr_t>(at->positions) & 3u) != 0) return BFQ_ERR_ALIGN;
            p.positions = at->positions, p.rope = at->table, p.rope_rows = at->rows, p.rope_dims = at->dims, p.interleaved = at->interleaved != 0;
        }
        if ((reinterpret_cast<uintptr_t>(at->q_norm) & 15u) != 0 || (reinterpret_cast<uintptr_t>(at->k_norm) & 15u) != 0) return BFQ_ERR_ALIGN;
        p.q_norm = at->q_norm, p.k_norm = at->k_norm, p.eps = at->eps;
    }
    p.slots = slots, p.tw = plan->tw, p.tokens = tokens, p.status = plan->status_word;
    kv::OnDevice guard(plan->device);
    if (!guard.ok) return BFQ_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = n == 64 ? (xt == BFQ_F32 ? kv::launch_append<64, true>(plan, p, st) : kv::launch_append<64, false>(plan, p, st))
                                  : (xt == BFQ_F32 ? kv::launch_append<128, true>(plan, p, st) : kv::launch_append<128, false>(plan, p, st));
    if (e == cudaSuccess) return BFQ_OK;
    plan->last_cuda_error = static_cast<int>(e);
    return BFQ_ERR_CUDA;
}

extern "C" int bfq_kv_read(bfq_plan* plan, const bfq_kv_cache* cache, const int64_t* slots, int64_t tokens, bfq_dtype t, void* k, void* v, void* stream) {
    kv::ReadParams p{};
    const int rc = kv::check_cache(plan, cache, &p.cache);
    if (rc != BFQ_OK) return rc;
    if (t != BFQ_F32 && t != BFQ_BF16) return BFQ_ERR_DTYPE;
    if (tokens < 0 || tokens >= int64_t(1) << 31 || tokens * 2 * cache->heads > kv::kMostRows) return BFQ_ERR_STRIDE;
    if (tokens == 0) return BFQ_OK;
    if (slots == nullptr || k == nullptr || v == nullptr) return BFQ_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(slots) & 7u) != 0 || ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u) != 0) return BFQ_ERR_ALIGN;
    p.slots = slots, p.tw = plan->tw, p.k = static_cast<uint8_t*>(k), p.v = static_cast<uint8_t*>(v), p.tokens = tokens, p.status = plan->status_word;
    kv::OnDevice guard(plan->device);
    if (!guard.ok) return BFQ_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = plan->n == 64 ? (t == BFQ_F32 ? kv::launch_read<64, true>(plan, p, st) : kv::launch_read<64, false>(plan, p, st))
                                        : (t == BFQ_F32 ? kv::launch_read<128, true>(plan, p, st) : kv::launch_read<128, false>(plan, p, st));
    if (e == cudaSuccess) return BFQ_OK;
    plan->last_cuda_error = static_cast<int>(e);
    return BFQ_ERR_CUDA;
}
