// Rows into and out of the paged low-bit key/value cache where rows are few (a decode step): the operations of bfq_kvrows.cu with a row of
// D = 64 or 128 elements on D / 8 lanes, 8 elements (one 16-byte load of bf16) each.  Three stages of the butterfly in a lane, the others by
// exchanges; constants in registers.  More instructions than with a row to a thread, but a loop of a few hundred of them instead of
// thousands in a line, which a call that runs through them once waits for.
#include "bfq_generic.cuh"
#include "bfq_kvrows.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kRowThreads = 128;

// 8 elements of a row as they lie in memory, and as numbers
template <bool F32>
struct Raw {
    uint4 w[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const uint8_t* at) {
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) w[i] = load_plain(reinterpret_cast<const uint4*>(at) + i);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        if constexpr (F32) {
            const uint32_t v[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(v[i]);
        } else {
            const uint32_t v[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(v[i] << 16), x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
        }
    }
};
__device__ __forceinline__ void load_floats8(const float* at, float (&x)[8]) {
    Raw<true> r;
    r.load(reinterpret_cast<const uint8_t*>(at));
    r.get(x);
}

// 8 elements -> codes of 4 bits (one word) or 8 (two): quant1's codes (clip(x inv), then round to nearest even), the rounding by an addition
// that leaves the integer in the low bits
template <int BITS>
__device__ __forceinline__ void codes8(const float (&x)[8], float inv, uint32_t (&w)[BITS / 4]) {
    constexpr float kTop = (1 << (BITS - 1)) - 1;
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = __float_as_uint(__fadd_rn(fminf(fmaxf(__fmul_rn(x[e], inv), -kTop - 1.f), kTop), 12582912.f));
    if constexpr (BITS == 4) {
        w[0] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[0] |= (c[e] & 15u) << (4 * e);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            w[i] = __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x0040), __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x0040), 0x5410);
    }
}

// The rows of a CTA are consecutive (a token's rows share its position's angles and its slot), kRowThreads / (D / 8) at a time.  A lane's row
// by token and row of the token, without a division at each step.
struct RowAt {
    int64_t token, left;  // rows from this one to the CTA's last (<= 0: none)
    int r;                // of the token's `heads`
    __device__ __forceinline__ void start(int64_t rows, int heads, int rows_per_step) {
        const int64_t steps = (rows + rows_per_step - 1) / rows_per_step, per = (steps + gridDim.x - 1) / gridDim.x * rows_per_step;
        const int64_t from = per * blockIdx.x, to = from + per < rows ? from + per : rows, row = from + threadIdx.x / (kRowThreads / rows_per_step);
        left = to - row, token = row / heads, r = static_cast<int>(row - token * heads);
    }
    __device__ __forceinline__ void next(int heads, int rows_per_step) {
        left -= rows_per_step;
        r += rows_per_step;
        while (r >= heads) r -= heads, ++token;
    }
    __device__ __forceinline__ bool there() const { return left > 0; }
};

// Of a row's token: what the row after next needs is on its way while this one is worked on.
template <int D, bool F32, int BITS>
__global__ void __launch_bounds__(kRowThreads) k_append_few(const AppendParams p) {
    constexpr int kLanes = D / 8, kStep = kRowThreads / kLanes;
    grid_dep_wait();
    const int lane = threadIdx.x & 31, l = lane % kLanes;
    const int heads = p.q.heads + 2 * p.cache.heads;  // rows of a token: queries, keys, values
    auto kind_of = [&](const RowAt& a) { return a.r < p.q.heads ? 0 : (a.r < p.q.heads + p.cache.heads ? 1 : 2); };
    auto head_of = [&](const RowAt& a, int kind) { return a.r - (kind == 0 ? 0 : (kind == 1 ? p.q.heads : p.q.heads + p.cache.heads)); };
    auto fetch = [&](const RowAt& a, Raw<F32>& raw) {
        if (!a.there()) return;
        const int kind = kind_of(a), head = head_of(a, kind);
        const uint8_t* data = kind == 0 ? p.q.data : (kind == 1 ? p.k.data : p.v.data);
        const int64_t st = kind == 0 ? p.q.token : (kind == 1 ? p.k.token : p.v.token), sh = kind == 0 ? p.q.head : (kind == 1 ? p.k.head : p.v.head);
        raw.load(data + (a.token * st + head * sh + 8 * l) * (F32 ? 4 : 2));
    };
    RowAt at, ahead;
    at.start(p.tokens * heads, heads, kStep);
    Raw<F32> raw, raw_next;
    fetch(at, raw);
    int position = at.there() && p.positions != nullptr ? load_plain(p.positions + at.token) : 0, position_next = 0;
    int64_t slot = at.there() ? load_plain(p.slots + at.token) : -1, slot_next = -1;
    Turn<D, 8, false> turn;
    turn.load(p.tw, lane);
    for (; __any_sync(0xFFFFFFFFu, at.there()); at = ahead, raw = raw_next, position = position_next, slot = slot_next) {
        const bool there = at.there();
        const int kind = kind_of(at), head = head_of(at, kind);
        const bool turned = there && p.positions != nullptr && kind < 2 && 8 * l < p.rope_dims, upper = !p.interleaved && 16 * l >= p.rope_dims;
        float cs[8], sn[8];
        if (turned) {
            const bool fine = position >= 0 && position < p.rope_rows;
            if (!fine) atomicExch(p.status, kBadIndex);
            const float* table = p.rope + (fine ? position : 0) * int64_t(p.rope_dims);
            if (p.interleaved) {
                const float4 c = load_plain(reinterpret_cast<const float4*>(table + 4 * l)), s = load_plain(reinterpret_cast<const float4*>(table + p.rope_dims / 2 + 4 * l));
                cs[0] = c.x, cs[1] = c.y, cs[2] = c.z, cs[3] = c.w, sn[0] = s.x, sn[1] = s.y, sn[2] = s.z, sn[3] = s.w;
            } else {
                const float* t = table + 8 * l - (upper ? p.rope_dims / 2 : 0);
                load_floats8(t, cs), load_floats8(t + p.rope_dims / 2, sn);
            }
        }
        ahead = at;
        ahead.next(heads, kStep);
        fetch(ahead, raw_next);
        if (ahead.there()) {
            slot_next = load_plain(p.slots + ahead.token);
            if (p.positions != nullptr) position_next = load_plain(p.positions + ahead.token);
        }
        float x[8];
        raw.get(x);
        const float* norm = kind == 0 ? p.q_norm : (kind == 1 ? p.k_norm : nullptr);
        if (__any_sync(0xFFFFFFFFu, norm != nullptr)) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            if (norm != nullptr) {
                const float f = 1.f / sqrtf(sum * (1.f / D) + p.eps);
                float w[8];
                load_floats8(norm + 8 * l, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= f * w[e];
            }
        }
        if (__any_sync(0xFFFFFFFFu, turned)) {
            if (p.interleaved) {
                if (turned) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = x[2 * i], b = x[2 * i + 1];
                        x[2 * i] = fmaf(a, cs[i], -b * sn[i]);
                        x[2 * i + 1] = fmaf(b, cs[i], a * sn[i]);
                    }
                }
            } else {
                const int half = p.rope_dims / 16, other = turned ? (upper ? lane - half : lane + half) : lane;  // `half` lanes have a half
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float o = __shfl_sync(0xFFFFFFFFu, x[e], other);
                    if (turned) x[e] = fmaf(x[e], cs[e], (upper ? o : -o) * sn[e]);
                }
            }
        }
        turn.apply(x);
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (!there) continue;
        if (kind == 0) {
            const uint4 v = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
            *reinterpret_cast<uint4*>(const_cast<uint8_t*>(p.q_out.data) + (at.token * p.q_out.token + head * p.q_out.head + 8 * l) * 2) = v;
            continue;
        }
        const int64_t page = slot >> p.cache.page_shift;
        if (slot < 0) continue;
        if (page >= p.cache.pages) {
            atomicExch(p.status, kBadIndex);
            continue;
        }
        const int place = static_cast<int>(slot) & ((1 << p.cache.page_shift) - 1);
        const Half to = kind == 1 ? p.cache.k : p.cache.v;
        float inv;
        const uint16_t scale = row_scale(top, (1 << (BITS - 1)) - 1, &inv);
        uint32_t w[BITS / 4];
        codes8<BITS>(x, inv, w);
        uint8_t* c = codes_of<D * BITS / 8>(to, p.cache.page_shift, page, head, place) + l * BITS;
        if constexpr (BITS == 4) *reinterpret_cast<uint32_t*>(c) = w[0];
        else *reinterpret_cast<uint2*>(c) = make_uint2(w[0], w[1]);
        if (l == 0) *scale_of(to, p.cache.page_shift, page, head, place) = scale;
    }
}

template <int D, bool F32, int BITS>
__global__ void __launch_bounds__(kRowThreads) k_read_few(const ReadParams p) {
    constexpr int kLanes = D / 8, kStep = kRowThreads / kLanes;
    grid_dep_wait();
    const int lane = threadIdx.x & 31, l = lane % kLanes;
    const int heads = 2 * p.cache.heads;  // rows of a token: keys, values
    struct Codes {
        uint32_t w[2];
        uint16_t scale;
    };
    auto slot_of = [&](const RowAt& a) { return a.there() ? load_plain(p.slots + a.token) : int64_t(-1); };
    auto fetch = [&](const RowAt& a, int64_t slot) {
        Codes c{};
        const int64_t page = slot >> p.cache.page_shift;
        if (slot < 0) return c;
        if (page >= p.cache.pages) {
            atomicExch(p.status, kBadIndex);
            return c;
        }
        const bool is_k = a.r < p.cache.heads;
        const int place = static_cast<int>(slot) & ((1 << p.cache.page_shift) - 1), head = is_k ? a.r : a.r - p.cache.heads;
        const Half from = is_k ? p.cache.k : p.cache.v;
        const uint8_t* at = codes_of<D * BITS / 8>(from, p.cache.page_shift, page, head, place) + l * BITS;
        if constexpr (BITS == 4) {
            c.w[0] = load_plain(reinterpret_cast<const uint32_t*>(at));
        } else {
            const uint2 u = load_plain(reinterpret_cast<const uint2*>(at));
            c.w[0] = u.x, c.w[1] = u.y;
        }
        c.scale = *static_cast<volatile const uint16_t*>(scale_of(from, p.cache.page_shift, page, head, place));
        return c;
    };
    RowAt at, ahead;
    at.start(p.tokens * heads, heads, kStep);
    ahead = at;
    ahead.next(heads, kStep);
    Codes codes = fetch(at, slot_of(at)), codes_next{};
    int64_t slot = slot_of(ahead);  // of the next row
    Turn<D, 8, true> turn;
    turn.load(p.tw, lane);
    for (; __any_sync(0xFFFFFFFFu, at.there()); codes = codes_next) {
        codes_next = fetch(ahead, slot);
        const RowAt now = at;
        at = ahead;
        ahead.next(heads, kStep);
        slot = slot_of(ahead);
        const float s = half_value(codes.scale);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = s * static_cast<float>(static_cast<int32_t>(codes.w[e * BITS / 32] << (32 - BITS - e * BITS % 32)) >> (32 - BITS));
        turn.apply(x);
        if (!now.there()) continue;
        const bool is_k = now.r < p.cache.heads;
        uint8_t* out = (is_k ? p.k : p.v) + ((now.token * p.cache.heads + (is_k ? now.r : now.r - p.cache.heads)) * D + 8 * l) * (F32 ? 4 : 2);
        if constexpr (F32) {
            reinterpret_cast<float4*>(out)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4*>(out)[1] = make_float4(x[4], x[5], x[6], x[7]);
        } else {
            *reinterpret_cast<uint4*>(out) = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
        }
    }
}

// enough CTAs for every row, at most four on an SM
static dim3 row_grid(const bfq_plan* plan, int64_t rows, int rows_per_step) {
    const int64_t want = (rows + rows_per_step - 1) / rows_per_step, most = int64_t(plan->sm_count) * 4;
    return dim3(unsigned(want < most ? want : most));
}
template <int D, bool F32>
static cudaError_t launch_append(const bfq_plan* plan, const AppendParams& p, cudaStream_t st) {
    const dim3 grid = row_grid(plan, p.tokens * (p.q.heads + 2 * p.cache.heads), kRowThreads / (D / 8));
    return p.cache.bits == 4 ? launch_overlapped(k_append_few<D, F32, 4>, grid, dim3(kRowThreads), 0, st, p)
                             : launch_overlapped(k_append_few<D, F32, 8>, grid, dim3(kRowThreads), 0, st, p);
}
template <int D, bool F32>
static cudaError_t launch_read(const bfq_plan* plan, const ReadParams& p, cudaStream_t st) {
    const dim3 grid = row_grid(plan, p.tokens * 2 * p.cache.heads, kRowThreads / (D / 8));
    return p.cache.bits == 4 ? launch_overlapped(k_read_few<D, F32, 4>, grid, dim3(kRowThreads), 0, st, p)
                             : launch_overlapped(k_read_few<D, F32, 8>, grid, dim3(kRowThreads), 0, st, p);
}
cudaError_t append_few_launch(const bfq_plan* plan, const AppendParams& p, bool f32, cudaStream_t st) {
    return plan->n == 64 ? (f32 ? launch_append<64, true>(plan, p, st) : launch_append<64, false>(plan, p, st))
                         : (f32 ? launch_append<128, true>(plan, p, st) : launch_append<128, false>(plan, p, st));
}
cudaError_t read_few_launch(const bfq_plan* plan, const ReadParams& p, bool f32, cudaStream_t st) {
    return plan->n == 64 ? (f32 ? launch_read<64, true>(plan, p, st) : launch_read<64, false>(plan, p, st))
                         : (f32 ? launch_read<128, true>(plan, p, st) : launch_read<128, false>(plan, p, st));
}

}  // namespace kv
}  // namespace bfq
