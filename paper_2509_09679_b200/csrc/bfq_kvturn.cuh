// A row of a head in the registers of one thread: the inverse butterfly on it, and the way of a warp's 32 rows in and out through shared memory.
#pragma once
#include "bfq_kv.cuh"

namespace bfq {
namespace kv {

__device__ __forceinline__ uint4 shared_load(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void shared_store(uint32_t at, uint4 v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void copy_in(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Q^T on a row in a thread's registers, elements 2 r and 2 r + 1 in register r.  A stage's lo <- c lo + s hi, hi <- c hi - s lo is four
// operations a pair.  With each element kept as x / p, p the product of the cosines that it has met, it is two: lo' <- lo' + a hi',
// hi' <- hi' + b lo' with a = (s / c) (q / p), b = -(s / c) (p / q) for the factors p of lo and q of hi before the stage, and one
// multiplication by P, the products of all stages, at the end.  Every rounding is relative to what the plain stage would have there times 1 / p, so that the
// error is the same; the form is taken while all |P| >= 2^-40, which no row of the cache can bring past fp32's range.
// Table in shared memory, 16 bytes an entry: stage 0: (a, b) of registers 2 k and 2 k + 1; the other stages: (a, a', b, b') of the k-th pair of
// registers; then P, four elements an entry.
template <int D>
struct RowTurn {
    static constexpr int kStages = D == 64 ? 6 : 7, kPerStage = D / 4;
    static constexpr uint32_t kBytes = 16 * (kStages * kPerStage + D / 4);

    // All threads of the CTA; products: D floats of shared memory.  Returns whether the scaled form can be taken.
    __device__ static bool build(float* table, float* products, const float2* tw) {
        float* const out = table + 4 * kStages * kPerStage;
        for (int i = threadIdx.x; i < D; i += blockDim.x) products[i] = 1.f;
        __syncthreads();
        for (int n = 0; n < kStages; ++n) {
            const int st = kStages - 1 - n;
            for (int j = threadIdx.x; j < D / 2; j += blockDim.x) {
                const float2 t = load_plain(tw + st * (D / 2) + j);
                const int lo = ((j >> st) << (st + 1)) | (j & ((1 << st) - 1)), hi = lo + (1 << st);
                const float tangent = -t.y / t.x, p = products[lo], q = products[hi], a = -tangent * (q / p), b = tangent * (p / q);
                if (st == 0) {
                    table[2 * j] = a, table[2 * j + 1] = b;
                } else {  // pair j is half j & 1 of the registers' pair j / 2
                    float* at = table + 4 * (st * kPerStage + (j >> 1)) + (j & 1);
                    at[0] = a, at[2] = b;
                }
                products[lo] = p * t.x, products[hi] = q * t.x;
            }
            __syncthreads();
        }
        int fine = 1;
        for (int i = threadIdx.x; i < D; i += blockDim.x) {
            out[i] = products[i];
            fine &= fabsf(products[i]) >= 0x1p-40f;  // false for NaN too
        }
        return __syncthreads_and(fine) != 0;
    }
    __device__ __forceinline__ static void scaled(u64 (&x)[D / 2], uint32_t table) {
#pragma unroll
        for (int n = 0; n < kStages; ++n) {
            const int st = kStages - 1 - n;
            if (st == 0) {
#pragma unroll
                for (int k = 0; k < D / 4; ++k) {
                    const uint4 c = shared_load(table + 16 * k);
                    float a, b;
                    unpack2(x[2 * k], a, b);
                    x[2 * k] = pack2(fmaf(__uint_as_float(c.x), b, a), fmaf(__uint_as_float(c.y), a, b));
                    unpack2(x[2 * k + 1], a, b);
                    x[2 * k + 1] = pack2(fmaf(__uint_as_float(c.z), b, a), fmaf(__uint_as_float(c.w), a, b));
                }
            } else {
                const int h = 1 << (st - 1);  // in registers
#pragma unroll
                for (int k = 0; k < kPerStage; ++k) {
                    const int lo = ((k / h) * 2 * h) + k % h, hi = lo + h;
                    const uint4 c = shared_load(table + 16 * (st * kPerStage + k));
                    const u64 a = x[lo], b = x[hi];
                    x[lo] = fma2(pack2u(c.x, c.y), b, a), x[hi] = fma2(pack2u(c.z, c.w), a, b);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < D / 4; ++k) {
            const uint4 c = shared_load(table + 16 * (kStages * kPerStage + k));
            x[2 * k] = mul2(x[2 * k], pack2u(c.x, c.y)), x[2 * k + 1] = mul2(x[2 * k + 1], pack2u(c.z, c.w));
        }
    }
    __device__ __forceinline__ static void plain(u64 (&x)[D / 2], const float2* tw) {
#pragma unroll
        for (int n = 0; n < kStages; ++n) {
            const int st = kStages - 1 - n;
#pragma unroll
            for (int j = 0; j < D / 2; ++j) {
                const float2 t = load_plain(tw + st * (D / 2) + j);
                const int lo = ((j >> st) << (st + 1)) | (j & ((1 << st) - 1)), hi = lo + (1 << st);
                float v[2], w[2];
                unpack2(x[lo / 2], v[0], v[1]), unpack2(x[hi / 2], w[0], w[1]);
                const float s = -t.y, a = v[lo & 1], b = st == 0 ? v[1] : w[hi & 1];
                const float na = fmaf(t.x, a, -s * b), nb = fmaf(s, a, t.x * b);
                if (st == 0) {
                    x[lo / 2] = pack2(na, nb);
                } else {
                    v[lo & 1] = na, w[hi & 1] = nb;
                    x[lo / 2] = pack2(v[0], v[1]), x[hi / 2] = pack2(w[0], w[1]);
                }
            }
        }
    }
};

// A warp's 32 rows of BYTES bytes each between memory and shared memory (PITCH apart there), 16 bytes a lane; `row` is the lane's own
// row's address.  f(place in shared memory, address, row) for each 16 bytes of a row of which `bytes`, the row's own, covers them.
template <int BYTES, int PITCH, class F>
__device__ __forceinline__ void each_chunk(const uint8_t* row, int bytes, F&& f) {
    constexpr int kLanes = BYTES / 16 < 32 ? BYTES / 16 : 32, kRows = 32 / kLanes, kTurns = BYTES / 16 / kLanes;
    const int lane = threadIdx.x & 31, part = lane % kLanes;
    const uint64_t address = reinterpret_cast<uint64_t>(row);
#pragma unroll
    for (int r = 0; r < 32; r += kRows) {
        const int from = r + lane / kLanes;
        const uint32_t lo = __shfl_sync(0xFFFFFFFFu, static_cast<uint32_t>(address), from), hi = __shfl_sync(0xFFFFFFFFu, static_cast<uint32_t>(address >> 32), from);
        const int size = __shfl_sync(0xFFFFFFFFu, bytes, from);
        uint8_t* const base = reinterpret_cast<uint8_t*>(static_cast<uint64_t>(hi) << 32 | lo);
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const int off = 16 * (part + t * kLanes);
            if (off < size) f(static_cast<uint32_t>(from * PITCH + off), base + off);
        }
    }
}

template <int D>
__device__ __forceinline__ void store_bf16(uint32_t to, const u64 (&x)[D / 2]) {
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a, b;
            unpack2(x[4 * c + i], a, b);
            w[i] = bf16_pair(a, b);
        }
        shared_store(to + 16 * c, make_uint4(w[0], w[1], w[2], w[3]));
    }
}

}  // namespace kv
}  // namespace bfq
