// Rows into and out of the paged low-bit key/value cache.
//
// bfq_kv_append, one pass over a step's new tokens:  z = w x / sqrt(mean x^2 + eps) per head (queries and keys, where norms are given),
// the position's rotation on the first R elements of a head (pairs (i, i + R/2) or (2i, 2i + 1), cos and sin from a table), y = Q z, and
//     queries      y as bf16
//     keys, values s = fp16(max |y| / qmax), codes = clip(round(y / s)) in the page and place of the token's slot.
// Values are rotated by Q alone.  bfq_kv_read: x = Q^T (s code), the rows at any slots in the model's basis.
//
// A row of D = 64 or 128 elements lies on D / 8 lanes, 8 elements (one 16-byte load of bf16) each: three stages of the butterfly in
// a lane, the others by exchanges; more elements per lane would save exchanges and cost 16 registers of constants each per stage.
// All sums in fp32.  What bounds it: instructions (about 30 per element and lane against 14 that the memory's rate would leave).
#include "bfq_generic.cuh"
#include "bfq_kv.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kRowThreads = 128;

struct AppendParams {
    Cache cache;
    Heads q, k, v, q_out;  // q.heads = 0: no queries
    const int64_t* slots;
    const int32_t* positions;  // null: no rotation by position
    const float* rope;         // [rope_rows][rope_dims]: cos of rope_dims / 2 frequencies, then sin
    const float* q_norm;
    const float* k_norm;
    const float2* tw;
    int64_t rope_rows, tokens;
    float eps;
    int rope_dims, interleaved;
    int* status;
};

template <bool F32>
__device__ __forceinline__ void load8(const uint8_t* at, float (&x)[8]) {
    if constexpr (F32) {
        const float4 a = load_plain(reinterpret_cast<const float4*>(at)), b = load_plain(reinterpret_cast<const float4*>(at) + 1);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        const uint4 a = load_plain(reinterpret_cast<const uint4*>(at));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// 8 elements -> codes of 4 bits (one word) or 8 (two)
template <int BITS>
__device__ __forceinline__ void codes8(const float (&x)[8], float inv, uint32_t (&w)[BITS / 4]) {
    constexpr int kTop = (1 << (BITS - 1)) - 1;
#pragma unroll
    for (int i = 0; i < BITS / 4; ++i) w[i] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t c = static_cast<uint32_t>(quant1(x[e], inv, -kTop - 1, kTop)) & ((1u << BITS) - 1);
        w[e * BITS / 32] |= c << (e * BITS % 32);
    }
}

template <int D, bool F32, int BITS>
__global__ void __launch_bounds__(kRowThreads) k_append(const AppendParams p) {
    constexpr int kLanes = D / 8, kRowsPerWarp = 32 / kLanes;
    grid_dep_wait();
    const int lane = threadIdx.x & 31, l = lane % kLanes;
    Turn<D, 8> turn;
    turn.load(p.tw, lane);
    const int heads = p.q.heads + 2 * p.cache.heads;  // of a token, queries first
    const int64_t rows = p.tokens * heads;
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kRowThreads / 32);
    for (int64_t at = (static_cast<int64_t>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5)) * kRowsPerWarp; at < rows; at += warps * kRowsPerWarp) {
        const int64_t row = at + lane / kLanes;
        const bool there = row < rows;
        const int64_t token = there ? row / heads : 0;
        const int r = there ? static_cast<int>(row - token * heads) : 0;
        const bool is_q = r < p.q.heads, is_k = !is_q && r < p.q.heads + p.cache.heads;
        const int head = is_q ? r : (is_k ? r - p.q.heads : r - p.q.heads - p.cache.heads);
        const Heads& from = is_q ? p.q : (is_k ? p.k : p.v);
        float x[8];
        load8<F32>(from.data + (token * from.token + head * from.head + 8 * l) * (F32 ? 4 : 2), x);
        const float* norm = is_q ? p.q_norm : (is_k ? p.k_norm : nullptr);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (norm != nullptr) {
            const float f = 1.f / sqrtf(sum * (1.f / D) + p.eps);
            const float4 a = load_plain(reinterpret_cast<const float4*>(norm + 8 * l)), b = load_plain(reinterpret_cast<const float4*>(norm + 8 * l + 4));
            const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= f * w[e];
        }
        if (p.positions != nullptr) {
            const bool turned = (is_q || is_k) && 8 * l < p.rope_dims;
            int64_t pos = there ? load_plain(p.positions + token) : 0;
            if (pos < 0 || pos >= p.rope_rows) {
                if (there) atomicExch(p.status, kBadIndex);
                pos = 0;
            }
            const float* table = p.rope + pos * p.rope_dims;
            if (p.interleaved) {
                if (turned) {
                    const float4 c = load_plain(reinterpret_cast<const float4*>(table + 4 * l)), s = load_plain(reinterpret_cast<const float4*>(table + p.rope_dims / 2 + 4 * l));
                    const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = x[2 * i], b = x[2 * i + 1];
                        x[2 * i] = fmaf(a, cs[i], -b * sn[i]);
                        x[2 * i + 1] = fmaf(b, cs[i], a * sn[i]);
                    }
                }
            } else {
                const int half = p.rope_dims / 16;  // lanes of one half
                const bool upper = l >= half;
                const int other = (lane - l) + (turned ? (upper ? l - half : l + half) : l);
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = __shfl_sync(0xFFFFFFFFu, x[e], other);
                if (turned) {
                    const float* t = table + 8 * (upper ? l - half : l);
                    float cs[8], sn[8];
                    load8<true>(reinterpret_cast<const uint8_t*>(t), cs);
                    load8<true>(reinterpret_cast<const uint8_t*>(t + p.rope_dims / 2), sn);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = fmaf(x[e], cs[e], (upper ? o[e] : -o[e]) * sn[e]);
                }
            }
        }
        turn.forward(x);
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (!there) continue;
        if (is_q) {
            uint4 v = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
            *reinterpret_cast<uint4*>(const_cast<uint8_t*>(p.q_out.data) + (token * p.q_out.token + head * p.q_out.head + 8 * l) * 2) = v;
            continue;
        }
        const int64_t slot = load_plain(p.slots + token), page = slot >> p.cache.page_shift;
        if (slot < 0) continue;
        if (page >= p.cache.pages) {
            atomicExch(p.status, kBadIndex);
            continue;
        }
        const int place = static_cast<int>(slot) & ((1 << p.cache.page_shift) - 1);
        const Half& to = is_k ? p.cache.k : p.cache.v;
        float inv;
        const uint16_t scale = row_scale(top, (1 << (BITS - 1)) - 1, &inv);
        uint32_t w[BITS / 4];
        codes8<BITS>(x, inv, w);
        uint8_t* c = codes_of<D * BITS / 8>(to, p.cache.heads, p.cache.page_shift, page, head, place) + l * BITS;
        if constexpr (BITS == 4) *reinterpret_cast<uint32_t*>(c) = w[0];
        else *reinterpret_cast<uint2*>(c) = make_uint2(w[0], w[1]);
        if (l == 0) *scale_of(to, p.cache.heads, p.cache.page_shift, page, head, place) = scale;
    }
}

struct ReadParams {
    Cache cache;
    const int64_t* slots;
    const float2* tw;
    uint8_t *k, *v;  // [tokens][heads][D]
    int64_t tokens;
    int* status;
};

template <int D, bool F32, int BITS>
__global__ void __launch_bounds__(kRowThreads) k_read(const ReadParams p) {
    constexpr int kLanes = D / 8, kRowsPerWarp = 32 / kLanes;
    grid_dep_wait();
    const int lane = threadIdx.x & 31, l = lane % kLanes;
    Turn<D, 8> turn;
    turn.load(p.tw, lane);
    const int heads = 2 * p.cache.heads;
    const int64_t rows = p.tokens * heads;
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kRowThreads / 32);
    for (int64_t at = (static_cast<int64_t>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5)) * kRowsPerWarp; at < rows; at += warps * kRowsPerWarp) {
        const int64_t row = at + lane / kLanes;
        const bool there = row < rows;
        const int64_t token = there ? row / heads : 0;
        const int r = there ? static_cast<int>(row - token * heads) : 0;
        const bool is_k = r < p.cache.heads;
        const int head = is_k ? r : r - p.cache.heads;
        const int64_t slot = there ? load_plain(p.slots + token) : -1, page = slot >> p.cache.page_shift;
        float x[8];
        if (slot < 0 || page >= p.cache.pages) {
            if (slot >= 0) atomicExch(p.status, kBadIndex);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
        } else {
            const int place = static_cast<int>(slot) & ((1 << p.cache.page_shift) - 1);
            const Half& from = is_k ? p.cache.k : p.cache.v;
            const uint8_t* c = codes_of<D * BITS / 8>(from, p.cache.heads, p.cache.page_shift, page, head, place) + l * BITS;
            const float s = half_value(*static_cast<volatile const uint16_t*>(scale_of(from, p.cache.heads, p.cache.page_shift, page, head, place)));
            uint32_t w[2];
            if constexpr (BITS == 4) {
                w[0] = load_plain(reinterpret_cast<const uint32_t*>(c));
            } else {
                const uint2 u = load_plain(reinterpret_cast<const uint2*>(c));
                w[0] = u.x, w[1] = u.y;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = s * static_cast<float>(static_cast<int32_t>(w[e * BITS / 32] << (32 - BITS - e * BITS % 32)) >> (32 - BITS));
        }
        turn.inverse(x);
        if (!there) continue;
        uint8_t* out = (is_k ? p.k : p.v) + ((token * p.cache.heads + head) * D + 8 * l) * (F32 ? 4 : 2);
        if constexpr (F32) {
            reinterpret_cast<float4*>(out)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4*>(out)[1] = make_float4(x[4], x[5], x[6], x[7]);
        } else {
            *reinterpret_cast<uint4*>(out) = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
        }
    }
}

// enough CTAs for every row, at most `per_sm` on an SM
static dim3 row_grid(const bfq_plan* plan, int64_t rows, int rows_per_warp, int per_sm) {
    const int64_t rows_per_cta = rows_per_warp * (kRowThreads / 32), want = (rows + rows_per_cta - 1) / rows_per_cta;
    const int64_t most = int64_t(plan->sm_count) * per_sm;
    return dim3(unsigned(want < most ? want : most));
}

template <int D, bool F32>
static cudaError_t launch_append(const bfq_plan* plan, const AppendParams& p, cudaStream_t st) {
    const dim3 grid = row_grid(plan, p.tokens * (p.q.heads + 2 * p.cache.heads), 256 / D, 4);
    return p.cache.bits == 4 ? launch_overlapped(k_append<D, F32, 4>, grid, dim3(kRowThreads), 0, st, p)
                             : launch_overlapped(k_append<D, F32, 8>, grid, dim3(kRowThreads), 0, st, p);
}
template <int D, bool F32>
static cudaError_t launch_read(const bfq_plan* plan, const ReadParams& p, cudaStream_t st) {
    const dim3 grid = row_grid(plan, p.tokens * 2 * p.cache.heads, 256 / D, 4);
    return p.cache.bits == 4 ? launch_overlapped(k_read<D, F32, 4>, grid, dim3(kRowThreads), 0, st, p)
                             : launch_overlapped(k_read<D, F32, 8>, grid, dim3(kRowThreads), 0, st, p);
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
    if (tokens < 0 || tokens >= int64_t(1) << 40) return BFQ_ERR_STRIDE;
    if (tokens == 0) return BFQ_OK;
    if (slots == nullptr || k == nullptr || v == nullptr || (q == nullptr) != (q_out == nullptr)) return BFQ_ERR_NULL;
    const int n = plan->n, esize = xt == BFQ_F32 ? 4 : 2;
    rc = kv::check_heads(k, n, esize, &p.k);
    if (rc == BFQ_OK) rc = kv::check_heads(v, n, esize, &p.v);
    if (rc == BFQ_OK && q != nullptr) rc = kv::check_heads(q, n, esize, &p.q);
    if (rc == BFQ_OK && q != nullptr) rc = kv::check_heads(q_out, n, 2, &p.q_out);
    if (rc != BFQ_OK) return rc;
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
    if (tokens < 0 || tokens >= int64_t(1) << 40) return BFQ_ERR_STRIDE;
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
