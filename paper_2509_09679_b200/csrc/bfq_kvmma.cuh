// Codes and rows as fp16 operands of the tensor cores, and what the kernels that use tcgen05 share: waits, descriptors, products.
#pragma once
#include "bfq_kv.cuh"

namespace bfq {
namespace kv {

__device__ __forceinline__ uint32_t sub_pair(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t fma_pair(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// Codes of a word as exact fp16 pairs (one of the lower half, one of the upper): the code's bits, its top one inverted, lie in the mantissa of
// 1024 .. 2047.  4 bits: codes i and i + 4, i < 4; the odd ones lie four places up there, 1152 + 16 code.  8 bits: codes i and i + 2, i < 2.
// Masks and bases are kept in registers that the compiler cannot see through: as constants, two of them in one operation, it makes two
// operations of each (of the kernel for few rows' 850 instructions for 32 keys of 4 bits 130).
template <int BITS>
struct Unpack {
    uint32_t mask, base, mask_up, base_up;
    __device__ __forceinline__ Unpack() {
        asm volatile("mov.u32 %0, %1;" : "=r"(mask) : "n"(BITS == 4 ? 0x000F000F : 0x00FF00FF));
        asm volatile("mov.u32 %0, %1;" : "=r"(base) : "n"(BITS == 4 ? 0x64086408 : 0x64806480));  // 1032, 1152
        if constexpr (BITS == 4) {
            asm volatile("mov.u32 %0, %1;" : "=r"(mask_up) : "n"(0x00F000F0));
            asm volatile("mov.u32 %0, %1;" : "=r"(base_up) : "n"(0x64806480));  // 1152
        }
    }
    __device__ __forceinline__ static uint32_t and_xor(uint32_t a, uint32_t b, uint32_t c) {
        uint32_t d;
        asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
        return d;
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t w, int i) const {
        if constexpr (BITS == 4) {
            if (i >= 2) w >>= 8;
            return i & 1 ? fma_pair(and_xor(w, mask_up, base_up), 0x2C002C00u, 0xD480D480u)  // / 16 - 72
                         : sub_pair(and_xor(w, mask, base), base);
        } else {
            if (i) w >>= 8;
            return sub_pair(and_xor(w, mask, base), base);
        }
    }
};
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The power of two that puts a row's largest element `top` in [2^10, 2^11): elements down to 2^-24 of it stay exact in fp16.
struct RowPower {
    float up, down;  // 2^e and 2^-e
    __device__ __forceinline__ explicit RowPower(float top) {
        const int field = 264 - static_cast<int>(__float_as_uint(top) >> 23), e = field > 253 ? 253 : field;
        up = __uint_as_float(uint32_t(e) << 23), down = __uint_as_float(uint32_t(254 - e) << 23);
    }
};

// Waits for a phase, with a limit; false: gave up.  Once one wait has given up all others of the CTA return at once (what they wait for may never
// come): the kernel ends with meaningless outputs and the status word says so, after it has drained what it has in flight.
constexpr long long kWaitCycles = 1ll << 31;  // about a second
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int* dead, int* status, long long cycles = kWaitCycles) {
    if (mbar_try_wait(bar, parity)) return true;
    const long long since = clock64();
    while (!mbar_try_wait(bar, parity)) {
        if (*dead) return false;
        if (clock64() - since > cycles) {
            *dead = 1;
            atomicExch(status, 3);
            return false;
        }
    }
    return true;
}
// After a wait has given up: copies or products in flight still read and write the CTA's memory, which must not end before them.  A limit of its own.
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) {
    const long long since = clock64();
    while (!mbar_try_wait(bar, parity) && clock64() - since <= kWaitCycles) {}
}
__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

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

}  // namespace kv
}  // namespace bfq
