// Rows into and out of the paged low-bit key/value cache.
//
// bfq_kv_append, one pass over a step's new tokens:  z = w x / sqrt(mean x^2 + eps) per head (queries and keys, where norms are given),
// the position's rotation on the first R elements of a head (pairs (i, i + R/2) or (2i, 2i + 1), cos and sin from a table), y = Q z, and
//     queries      y as bf16
//     keys, values s = fp16(max |y| / qmax), codes = clip(round(y / s)) in the page and place of the token's slot.
// Values are rotated by Q alone.  bfq_kv_read: x = Q^T (s code), the rows at any slots in the model's basis.
//
// A thread owns a row of D = 64 or 128 elements, all of it in registers, so that norms, maxima and the stages of the butterfly need no
// exchange between lanes; a warp takes 32 consecutive rows (a token's heads share its angles), copied into shared memory 16 bytes a lane, the next
// 32 while these are worked on, and results go out the same way.  The butterfly's constants are the same for all lanes: they come from
// shared memory by broadcast.  Its stages run in the scaled form, two FMAs a pair: with z = P w, P the product of the cosines
// that an element has been through,
//     lo: w <- w_lo - tan(t) (P_hi / P_lo) w_hi,   hi: w <- w_hi + tan(t) (P_lo / P_hi) w_lo,   P <- P cos(t)
// and P multiplied in at the end.  Where some |P| is below 2^-40 (an angle close to an odd multiple of pi/2), and for 32 rows of which
// one is not finite in that form, the plain stages are taken, four operations a pair.  All sums in fp32.
//
// What bounds it: fp32 operations, about 14 an element at 128 a cycle and SM, which is what the memory's rate leaves room for, too.  With a row
// on 16 lanes (exchanges by shuffles, constants in registers, 12 warps on an SM) 16384 tokens of 32 + 2 x 8 heads took 420 us.
#include "bfq_generic.cuh"
#include "bfq_kvrows.cuh"
#include "bfq_kvturn.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kMostWarps = 4;  // of a CTA

// Which rows a warp has: chunks of 32 rows, a CTA's consecutive, its warps' in turn.
struct Chunks {
    int at, end, step;
    __device__ __forceinline__ explicit Chunks(int rows) {
        const int chunks = (rows + 31) / 32, per = (chunks + gridDim.x - 1) / gridDim.x, from = per * blockIdx.x;
        step = blockDim.x >> 5;
        end = from + per < chunks ? from + per : chunks;
        at = from + (threadIdx.x >> 5);
    }
    __device__ __forceinline__ bool there() const { return at < end; }
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
// whether an infinity or a NaN is among them: a sum of zeros otherwise
template <int D>
__device__ __forceinline__ bool all_finite(const u64 (&x)[D / 2]) {
    u64 sum = pack2(0.f, 0.f);
    const u64 zero = pack2(0.f, 0.f);
#pragma unroll
    for (int r = 0; r < D / 2; ++r) sum = fma2(x[r], zero, sum);
    float a, b;
    unpack2(sum, a, b);
    return a + b == 0.f;
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

template <int D, bool F32, int BITS>
struct AppendSmem {
    static constexpr int kIn = D * (F32 ? 4 : 2), kInPitch = kIn + 16, kOutPitch = 2 * D + 16, kCodes = D * BITS / 8;
    static constexpr uint32_t kTable = RowTurn<D, false>::kBytes, kNorms = kTable, kProducts = kNorms + 3 * D * 4;  // weights of queries, keys, ones
    static constexpr uint32_t kWarps = kProducts + D * 4, kWarp = 32 * (kInPitch + kOutPitch);
    static constexpr uint32_t bytes(int warps) { return kWarps + warps * kWarp; }
};

template <int D, bool F32, int BITS>
__global__ void __launch_bounds__(32 * kMostWarps, D == 128 ? 3 : 5) k_append(const AppendParams p) {
    using S = AppendSmem<D, F32, BITS>;
    extern __shared__ __align__(16) uint8_t smem[];
    grid_dep_wait();
    const int lane = threadIdx.x & 31;
    const uint32_t table = smem_u32(smem), norms = table + S::kNorms, in = table + S::kWarps + (threadIdx.x >> 5) * S::kWarp, out = in + 32 * S::kInPitch;
    const int heads = p.q.heads + 2 * p.cache.heads, rows = static_cast<int>(p.tokens) * heads;  // rows of a token: queries, keys, values
    Chunks chunks(rows);
    // The lane's row of a chunk.  Found anew wherever it is needed, so that it takes no registers while the row is worked on.
    struct Row {
        int token, kind, head;  // 0 query, 1 key, 2 value, -1 none
    };
    auto find = [&](int chunk) {
        const int row = chunk * 32 + lane;
        Row r{row / heads, -1, 0};
        if (row < 0 || row >= rows) return Row{0, -1, 0};
        const int i = row - r.token * heads;
        r.kind = i < p.q.heads ? 0 : (i < p.q.heads + p.cache.heads ? 1 : 2);
        r.head = r.kind == 0 ? i : (r.kind == 1 ? i - p.q.heads : i - p.q.heads - p.cache.heads);
        return r;
    };
    auto data_of = [&](const Row& r) {
        const Heads& from = r.kind == 0 ? p.q : (r.kind == 1 ? p.k : p.v);
        return from.data + (r.token * from.token + r.head * from.head) * (F32 ? 4 : 2);
    };
    auto fetch = [&](const Row& r) { each_chunk<S::kIn, S::kInPitch>(data_of(r), r.kind >= 0 ? S::kIn : 0, [&](uint32_t at, uint8_t* from) { copy_in(in + at, from); }); };
    auto position_of = [&](const Row& r) { return p.positions != nullptr && (r.kind == 0 || r.kind == 1) ? load_plain(p.positions + r.token) : 0; };
    auto angles_of = [&](int position) { return p.rope + (position >= 0 && position < p.rope_rows ? position : 0) * int64_t(p.rope_dims); };
    auto prefetch = [&](const Row& r, int position) {  // a row's angles, into the cache
        if (p.positions == nullptr || r.kind < 0 || r.kind > 1) return;
        const float* at = angles_of(position);
        for (int i = 0; i < p.rope_dims; i += 32) asm volatile("prefetch.global.L1 [%0];" ::"l"(at + i));
    };
    {
        const Row first = find(chunks.there() ? chunks.at : -1);
        fetch(first);
        prefetch(first, position_of(first));
    }
    for (int i = threadIdx.x; i < D; i += blockDim.x) {
        float* w = reinterpret_cast<float*>(smem + S::kNorms);
        w[i] = p.q_norm != nullptr ? load_plain(p.q_norm + i) : 1.f, w[D + i] = p.k_norm != nullptr ? load_plain(p.k_norm + i) : 1.f, w[2 * D + i] = 1.f;
    }
    const bool scaled = RowTurn<D, false>::build(reinterpret_cast<float*>(smem), reinterpret_cast<float*>(smem + S::kProducts), p.tw);
    const bool normed = p.q_norm != nullptr || p.k_norm != nullptr;
    for (; chunks.there(); chunks.at += chunks.step) {
        u64 x[D / 2];
        copies_done();
        __syncwarp();
        const Row now = find(chunks.at), next = find(chunks.at + chunks.step < chunks.end ? chunks.at + chunks.step : -1);
        const bool turned = p.positions != nullptr && (now.kind == 0 || now.kind == 1);
        const int position = position_of(now), position_next = position_of(next);
        if (turned && (position < 0 || position >= p.rope_rows)) atomicExch(p.status, kBadIndex);
        const float* const angles = angles_of(position);
        auto prepare = [&]() {  // norm and position
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
                if (p.interleaved) turn_neighbours<D>(p.rope_dims, x, angles);
                else turn_halves_of<D>(p.rope_dims, x, angles);
            }
        };
        constexpr int kPairs = F32 ? 2 : 4;  // of 16 bytes
        for (bool plain = !scaled, again = false;; plain = again = true) {  // once, or again from memory in the plain form
#pragma unroll
            for (int c = 0; c < S::kIn / 16; ++c) {
                uint4 v;
                if (!again) v = shared_load(in + lane * S::kInPitch + 16 * c);
                else v = now.kind >= 0 ? load_plain(reinterpret_cast<const uint4*>(data_of(now)) + c) : make_uint4(0, 0, 0, 0);
                unpack_chunk<F32>(v, x + kPairs * c);
            }
            if (!again) {
                __syncwarp();
                fetch(next);
            }
            prepare();
            if (!again) prefetch(next, position_next);
            if (plain) RowTurn<D, false>::plain(x, p.tw);
            else RowTurn<D, false>::scaled(x, table);
            if (plain || __all_sync(0xFFFFFFFFu, now.kind < 0 || all_finite<D>(x))) break;
        }
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
            for (int c = 0; c < S::kCodes / 16; ++c) {
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
                to = codes_of<S::kCodes>(half, p.cache.page_shift, page, now.head, place), bytes = S::kCodes;
                *scale_of(half, p.cache.page_shift, page, now.head, place) = stored;
            }
        }
        __syncwarp();
        each_chunk<2 * D, S::kOutPitch>(to, bytes, [&](uint32_t at, uint8_t* dst) { *reinterpret_cast<uint4*>(dst) = shared_load(out + at); });
    }
}

template <int D, bool F32, int BITS>
struct ReadSmem {
    static constexpr int kIn = D * BITS / 8, kInPitch = kIn + 16, kOut = D * (F32 ? 4 : 2), kOutPitch = kOut + 16;
    static constexpr uint32_t kTable = RowTurn<D, true>::kBytes, kProducts = kTable, kWarps = kProducts + D * 4, kWarp = 32 * (kInPitch + kOutPitch);
    static constexpr uint32_t bytes(int warps) { return kWarps + warps * kWarp; }
};

template <int D, bool F32, int BITS>
__global__ void __launch_bounds__(32 * kMostWarps, D == 128 ? 3 : 5) k_read(const ReadParams p) {
    using S = ReadSmem<D, F32, BITS>;
    extern __shared__ __align__(16) uint8_t smem[];
    grid_dep_wait();
    const int lane = threadIdx.x & 31;
    const uint32_t table = smem_u32(smem), in = table + S::kWarps + (threadIdx.x >> 5) * S::kWarp, out = in + 32 * S::kInPitch;
    const int heads = 2 * p.cache.heads, rows = static_cast<int>(p.tokens) * heads;  // rows of a token: keys, values
    Chunks chunks(rows);
    struct Row {
        const uint8_t* data;  // null: zeros
        uint16_t scale;
    };
    auto find = [&](int chunk) {
        Row r{};
        const int row = chunk * 32 + lane;
        if (row < 0 || row >= rows) return r;
        const int token = row / heads, i = row - token * heads, head = i < p.cache.heads ? i : i - p.cache.heads;
        const int64_t slot = load_plain(p.slots + token), page = slot >> p.cache.page_shift;
        if (slot < 0) return r;
        if (page >= p.cache.pages) {
            atomicExch(p.status, kBadIndex);
            return r;
        }
        const int place = static_cast<int>(slot) & ((1 << p.cache.page_shift) - 1);
        const Half& half = i < p.cache.heads ? p.cache.k : p.cache.v;
        r.data = codes_of<S::kIn>(half, p.cache.page_shift, page, head, place);
        r.scale = *static_cast<volatile const uint16_t*>(scale_of(half, p.cache.page_shift, page, head, place));
        return r;
    };
    auto to_of = [&](int chunk) -> uint8_t* {
        const int row = chunk * 32 + lane, token = row / heads, i = row - token * heads;
        if (row >= rows) return nullptr;
        return (i < p.cache.heads ? p.k : p.v) + (int64_t(token) * p.cache.heads + (i < p.cache.heads ? i : i - p.cache.heads)) * S::kOut;
    };
    auto fetch = [&](const Row& r) { each_chunk<S::kIn, S::kInPitch>(r.data, r.data != nullptr ? S::kIn : 0, [&](uint32_t at, uint8_t* from) { copy_in(in + at, from); }); };
    Row now = find(chunks.there() ? chunks.at : -1);
    fetch(now);
    const bool scaled = RowTurn<D, true>::build(reinterpret_cast<float*>(smem), reinterpret_cast<float*>(smem + S::kProducts), p.tw);
    for (; chunks.there(); chunks.at += chunks.step) {
        copies_done();
        __syncwarp();
        uint4 raw[S::kIn / 16];
#pragma unroll
        for (int c = 0; c < S::kIn / 16; ++c) raw[c] = now.data != nullptr ? shared_load(in + lane * S::kInPitch + 16 * c) : make_uint4(0, 0, 0, 0);
        __syncwarp();
        const Row next = find(chunks.at + chunks.step < chunks.end ? chunks.at + chunks.step : -1);
        fetch(next);
        // codes are at most 128 and scales at most 65504: the scaled form, at most 2^40 times that, stays finite
        const float s = half_value(now.scale);
        const u64 s2 = pack2(s, s), base = pack2(-8388608.f - (1 << (BITS - 1)), -8388608.f - (1 << (BITS - 1)));
        u64 x[D / 2];
#pragma unroll
        for (int c = 0; c < S::kIn / 16; ++c) {
            const uint32_t w[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                constexpr int kCodesOfWord = 32 / BITS;
                const uint32_t v = w[i] ^ (BITS == 4 ? 0x88888888u : 0x80808080u);  // code + 2^(bits - 1): low bits on top of 2^23
#pragma unroll
                for (int e = 0; e < kCodesOfWord; e += 2) {
                    const uint32_t lo = (v >> (e * BITS)) & ((1u << BITS) - 1), hi = (v >> (e * BITS + BITS)) & ((1u << BITS) - 1);
                    x[((4 * c + i) * kCodesOfWord + e) / 2] = mul2(s2, add2(pack2u(lo | 0x4B000000u, hi | 0x4B000000u), base));
                }
            }
        }
        if (scaled) RowTurn<D, true>::scaled(x, table);
        else RowTurn<D, true>::plain(x, p.tw);
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
        uint8_t* const to = to_of(chunks.at);
        each_chunk<S::kOut, S::kOutPitch>(to, to != nullptr ? S::kOut : 0, [&](uint32_t at, uint8_t* dst) { *reinterpret_cast<uint4*>(dst) = shared_load(out + at); });
        now = next;
    }
}

template <class S, class Kernel, class Params>
static cudaError_t launch_rows(const bfq_plan* plan, Kernel kern, int* per_sm, int64_t rows, const Params& p, cudaStream_t st) {
    int& occ = per_sm[plan->device];
    if (occ == 0) {
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(S::bytes(kMostWarps)));
        int n = 0;
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, 32 * kMostWarps, S::bytes(kMostWarps));
        if (e != cudaSuccess) return e;
        occ = n > 0 ? n : 1;
    }
    const int64_t want = (rows + 32 * kMostWarps - 1) / (32 * kMostWarps), most = int64_t(plan->sm_count) * occ;
    return launch_overlapped(kern, dim3(unsigned(want < most ? want : most)), dim3(32 * kMostWarps), S::bytes(kMostWarps), st, p);
}
static bool few_rows(int64_t rows) { return rows < 65536; }

template <int D, bool F32, int BITS>
static cudaError_t launch_append_bits(const bfq_plan* plan, const AppendParams& p, cudaStream_t st) {
    static int per_sm[kMaxDevices] = {0};
    return launch_rows<AppendSmem<D, F32, BITS>>(plan, k_append<D, F32, BITS>, per_sm, p.tokens * (p.q.heads + 2 * p.cache.heads), p, st);
}
template <int D, bool F32>
static cudaError_t launch_append(const bfq_plan* plan, const AppendParams& p, cudaStream_t st) {
    if (few_rows(p.tokens * (p.q.heads + 2 * p.cache.heads))) return append_few_launch(plan, p, F32, st);
    return p.cache.bits == 4 ? launch_append_bits<D, F32, 4>(plan, p, st) : launch_append_bits<D, F32, 8>(plan, p, st);
}
template <int D, bool F32, int BITS>
static cudaError_t launch_read_bits(const bfq_plan* plan, const ReadParams& p, cudaStream_t st) {
    static int per_sm[kMaxDevices] = {0};
    return launch_rows<ReadSmem<D, F32, BITS>>(plan, k_read<D, F32, BITS>, per_sm, p.tokens * 2 * p.cache.heads, p, st);
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
    if (tokens * (p.q.heads + 2 * int64_t(cache->heads)) >= (int64_t(1) << 31) - 64) return BFQ_ERR_STRIDE;
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
    if (tokens < 0 || tokens >= int64_t(1) << 31 || tokens * cache->heads >= int64_t(1) << 30) return BFQ_ERR_STRIDE;
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
