// What the kernels on the paged low-bit key/value cache share: the cache as they see it, the butterfly on a row of one head
// spread over a few lanes, and how codes become bf16 operands of the tensor cores.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/bfq.h"
#include "bfq_plan.h"
#include "bfq_ptx.cuh"

namespace bfq {
namespace kv {
using namespace ptx;

struct Half {  // keys or values
    uint8_t* codes;
    uint16_t* scales;
    int64_t codes_page, scales_page;  // from page to page: bytes, scales
};
struct Cache {
    Half k, v;
    int64_t pages;
    int heads, page_shift, bits;
};
struct Heads {
    const uint8_t* data;
    int64_t token, head;  // strides in elements
    int heads;
};

// Where row (page, head, place) lies.  All products in 64 bits: a cache is larger than 4 GB.
template <int ROW_BYTES>
__device__ __forceinline__ uint8_t* codes_of(const Half& h, int page_shift, int64_t page, int head, int place) {
    return h.codes + page * h.codes_page + ((static_cast<int64_t>(head) << page_shift) + place) * ROW_BYTES;
}
__device__ __forceinline__ uint16_t* scale_of(const Half& h, int page_shift, int64_t page, int head, int place) {
    return h.scales + page * h.scales_page + (static_cast<int64_t>(head) << page_shift) + place;
}

// The butterfly (or, BACK, its transpose) on rows of D elements, a row on D / E consecutive lanes of a warp, lane l with elements
// E l .. E l + E - 1, two in a 64-bit register.  Stages of stride below E stay in a lane, the others are one exchange with the lane at that
// distance: (a, b) -> (c a - s b, s a + c b), so a lane with the lower element of a pair takes c x - s x', one with the upper c x + s x'.
// The constants are the lane's own, read once and used for every row that the lane works on.
template <int D, int E, bool BACK>
struct Turn {
    static constexpr int kLanes = D / E;
    static constexpr int kStages = D == 64 ? 6 : 7;
    static constexpr int kIn = E == 2 ? 1 : (E == 4 ? 2 : 3);  // stages within a lane
    static_assert((D == 64 || D == 128) && (E == 2 || E == 4 || E == 8), "rows of a head");
    float2 first[E / 2];                              // stage 0: (c, s) of the pair in each register
    u64 in_c[kIn][E / 4 + 1], in_s[kIn][E / 4 + 1];   // stages 1 .. kIn - 1: of the pairs of registers (entry 0 and those behind E / 4: unused)
    u64 c[kStages - kIn][E / 2], s[kStages - kIn][E / 2];

    __device__ __forceinline__ void load(const float2* tw, int lane) {
        const int base = (lane % kLanes) * E;
        auto at = [&](int st, int i) {  // the constants of element i's pair
            float2 v = load_plain(tw + st * (D / 2) + (((i >> (st + 1)) << st) | (i & ((1 << st) - 1))));
            if (BACK) v.y = -v.y;
            return v;
        };
#pragma unroll
        for (int r = 0; r < E / 2; ++r) first[r] = at(0, base + 2 * r);
#pragma unroll
        for (int st = 1; st < kStages; ++st) {
            const int h = 1 << st;
            int n = 0;
#pragma unroll
            for (int r = 0; r < E / 2; ++r) {
                const int i = base + 2 * r;
                if (st < kIn && ((2 * r) & h) != 0) continue;
                float2 a = at(st, i), b = at(st, i + 1);
                if (st < kIn) {
                    in_c[st][n] = pack2(a.x, b.x), in_s[st][n++] = pack2(a.y, b.y);
                } else {
                    if ((i & h) == 0) a.y = -a.y, b.y = -b.y;
                    c[st - kIn][r] = pack2(a.x, b.x), s[st - kIn][r] = pack2(a.y, b.y);
                }
            }
        }
    }
    __device__ __forceinline__ void stage(u64 (&x)[E / 2], int st) const {
        const int h = 1 << st;
        if (st == 0) {
#pragma unroll
            for (int r = 0; r < E / 2; ++r) {
                float a, b;
                unpack2(x[r], a, b);
                x[r] = pack2(fmaf(first[r].x, a, -first[r].y * b), fmaf(first[r].y, a, first[r].x * b));
            }
        } else if (st < kIn) {
            int n = 0;
#pragma unroll
            for (int r = 0; r < E / 2; ++r) {
                if (((2 * r) & h) != 0) continue;
                const u64 cc = in_c[st][n], ss = in_s[st][n++], a = x[r], b = x[r + h / 2];
                x[r] = sub2(mul2(cc, a), mul2(ss, b));
                x[r + h / 2] = fma2(ss, a, mul2(cc, b));
            }
        } else {
#pragma unroll
            for (int r = 0; r < E / 2; ++r) {
                uint32_t lo, hi;
                unpack2u(x[r], lo, hi);
                lo = __shfl_xor_sync(0xFFFFFFFFu, lo, h / E), hi = __shfl_xor_sync(0xFFFFFFFFu, hi, h / E);
                x[r] = fma2(c[st - kIn][r], x[r], mul2(s[st - kIn][r], pack2u(lo, hi)));
            }
        }
    }
    __device__ __forceinline__ void apply(float (&v)[E]) const {
        u64 x[E / 2];
#pragma unroll
        for (int r = 0; r < E / 2; ++r) x[r] = pack2(v[2 * r], v[2 * r + 1]);
#pragma unroll
        for (int st = 0; st < kStages; ++st) stage(x, BACK ? kStages - 1 - st : st);
#pragma unroll
        for (int r = 0; r < E / 2; ++r) unpack2(x[r], v[2 * r], v[2 * r + 1]);
    }
};

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float half_value(uint16_t bits) { return __half2float(__ushort_as_half(bits)); }

// ---- host side ----------------------------------------------------------------------------------------------------------
inline int shift_of(int page_size) {  // -1: not a power of two from 16 to 256
    for (int s = 4; s <= 8; ++s)
        if (page_size == 1 << s) return s;
    return -1;
}
// What every call refuses of a cache; fills `c`.
inline int check_cache(const bfq_plan* plan, const bfq_kv_cache* in, Cache* c) {
    if (plan == nullptr || in == nullptr) return BFQ_ERR_NULL;
    if (plan->n != 64 && plan->n != 128) return BFQ_ERR_UNSUPPORTED_N;
    if (in->bits != 4 && in->bits != 8) return BFQ_ERR_BITS;
    const int shift = shift_of(in->page_size);
    if (shift < 0 || in->heads < 1 || in->heads > 1024 || in->pages < 0 || in->pages >= int64_t(1) << 31) return BFQ_ERR_STRIDE;
    if (in->k_codes == nullptr || in->k_scales == nullptr || in->v_codes == nullptr || in->v_scales == nullptr) return BFQ_ERR_NULL;
    if (!plan->angles_set) return BFQ_ERR_WORKSPACE;
    const int64_t rows = int64_t(in->heads) << shift, bytes = rows * plan->n * in->bits / 8;
    const int64_t strides[4] = {in->k_codes_page, in->v_codes_page, in->k_scales_page * 2, in->v_scales_page * 2};
    const int64_t least[4] = {bytes, bytes, rows * 2, rows * 2};
    for (int i = 0; i < 4; ++i)
        if (strides[i] < least[i] || (strides[i] & 15) != 0) return BFQ_ERR_STRIDE;
    const void* at[4] = {in->k_codes, in->v_codes, in->k_scales, in->v_scales};
    for (const void* p : at)
        if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return BFQ_ERR_ALIGN;
    c->k = Half{in->k_codes, in->k_scales, in->k_codes_page, in->k_scales_page};
    c->v = Half{in->v_codes, in->v_scales, in->v_codes_page, in->v_scales_page};
    c->pages = in->pages, c->heads = in->heads, c->page_shift = shift, c->bits = in->bits;
    return BFQ_OK;
}
// rows of heads: 16-byte aligned, every stride a multiple of 16 bytes
inline int check_heads(const bfq_heads* h, int n, int esize, Heads* out) {
    if (h->data == nullptr) return BFQ_ERR_NULL;
    if (h->heads < 1 || h->heads > 1 << 20) return BFQ_ERR_STRIDE;
    if ((reinterpret_cast<uintptr_t>(h->data) & 15u) != 0) return BFQ_ERR_ALIGN;
    if (h->token < 0 || h->head < (h->heads > 1 ? n : 0) || (h->token * esize) % 16 != 0 || (h->head * esize) % 16 != 0) return BFQ_ERR_STRIDE;
    *out = Heads{static_cast<const uint8_t*>(h->data), h->token, h->head, h->heads};
    return BFQ_OK;
}

struct OnDevice {  // makes the plan's device current for a call
    int prev = -1;
    bool ok = false, switched = false;
    explicit OnDevice(int device) {
        if (cudaGetDevice(&prev) != cudaSuccess) return;
        if (prev != device) {
            if (cudaSetDevice(device) != cudaSuccess) return;
            switched = true;
        }
        ok = true;
    }
    ~OnDevice() {
        if (switched) cudaSetDevice(prev);
    }
};

}  // namespace kv
}  // namespace bfq
