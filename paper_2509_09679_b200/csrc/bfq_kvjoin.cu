// Joining the results of the kernel for many rows (bfq_kvtall.cu) where sequences have them alone: a row to a thread, as rows go into and out of
// the cache (bfq_kvrows.cu).  A warp takes 32 rows of a tile, which have the same results: those of the CTAs that had a part of the
// pair, mostly one.  Per result rows are copied into shared memory 16 bytes a lane, weighted and summed, then turned back by Q^T and rounded once.
// With a row to a warp (k_join: four elements to a lane, exchanges by shuffles) the 5632 tokens of 32 heads of a prompt's chunks took 184 us.
#include "bfq_kvattn.cuh"
#include "bfq_kvturn.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kJoinWarps = 4;
template <int D>
struct JoinSmem {
    static constexpr int kIn = 4 * D, kInPitch = kIn + 16, kOut = 2 * D, kOutPitch = kOut + 16;
    static constexpr uint32_t kProducts = RowTurn<D>::kBytes, kWarps = kProducts + D * 4, kWarp = 32 * kInPitch;  // rows out: in the place of rows in
    static constexpr uint32_t kBytes = kWarps + kJoinWarps * kWarp;
};

template <int D>
__global__ void __launch_bounds__(32 * kJoinWarps, D == 128 ? 3 : 5) k_join_tall(const AttendParams p, int chunks) {  // 32 rows of a place and a head each
    using S = JoinSmem<D>;
    extern __shared__ __align__(16) uint8_t smem[];
    grid_dep_wait();
    const int lane = threadIdx.x & 31, heads = p.cache.heads;
    const uint32_t table = smem_u32(smem), rows_at = table + S::kWarps + (threadIdx.x >> 5) * S::kWarp;
    const Part& part = p.tall;
    const bool scaled = RowTurn<D>::build(reinterpret_cast<float*>(smem), reinterpret_cast<float*>(smem + S::kProducts), p.tw);
    int of = -1;
    Tile tile{};
    for (int c = blockIdx.x * kJoinWarps + (threadIdx.x >> 5); c < chunks; c += gridDim.x * kJoinWarps) {
        const int numbered = c / (kTallRows / 32), place = numbered / heads, head = numbered - place * heads, r = c % (kTallRows / 32) * 32 + lane;
        if (place != of) {
            const int entry = entry_at(p, part, place);
            tile = tile_of(p, part, max(entry, 0)), of = place;
            if (entry < 0) tile.rows = 0;
        }
        if (r - lane >= tile.rows) continue;
        const bool there = r < tile.rows;
        const int pair = tile.place * heads + head;
        const int2 ctas = tile.keys > 0 ? ctas_of(part, pair) : make_int2(0, 0);
        const int64_t first = (static_cast<int64_t>(ctas.x) + pair) * kTallRows + r;
        u64 x[D / 2];
#pragma unroll
        for (int i = 0; i < D / 2; ++i) x[i] = pack2(0.f, 0.f);
        float m = -INFINITY, l = 0.f;
        for (int i = 0; i < ctas.y; ++i) {
            const int64_t at = first + static_cast<int64_t>(i) * kTallRows;
            each_chunk<S::kIn, S::kInPitch>(reinterpret_cast<const uint8_t*>(part.parts + at * D), there ? S::kIn : 0, [&](uint32_t to, uint8_t* from) { copy_in(rows_at + to, from); });
            const float2 ml = there ? load_plain(part.sums + at) : make_float2(-INFINITY, 0.f);
            const float top = fmaxf(m, ml.x), safe = top == -INFINITY ? 0.f : top, old = exp2_fast(m - safe), own = exp2_fast(ml.x - safe);
            m = top, l = l * old + ml.y * own;
            copies_done();
            __syncwarp();
            const u64 old2 = pack2(old, old), own2 = pack2(own, own);
#pragma unroll
            for (int k = 0; k < D / 4; ++k) {
                const uint4 v = shared_load(rows_at + lane * S::kInPitch + 16 * k);
                x[2 * k] = fma2(own2, pack2u(v.x, v.y), mul2(old2, x[2 * k])), x[2 * k + 1] = fma2(own2, pack2u(v.z, v.w), mul2(old2, x[2 * k + 1]));
            }
            __syncwarp();
        }
        const float f = l > 0.f || l != l ? 1.f / l : 0.f;
        const u64 f2 = pack2(f, f);
#pragma unroll
        for (int i = 0; i < D / 2; ++i) x[i] = mul2(x[i], f2);
        // an average of cached rows: at most 128 x 65504, which the scaled form leaves finite
        if (scaled) RowTurn<D>::scaled(x, table);
        else RowTurn<D>::plain(x, p.tw);
        const int row = tile.row0 + r, token = tile.token0 + row / p.group, q_head = head * p.group + row % p.group;
        store_bf16<D>(rows_at + lane * S::kOutPitch, x);
        __syncwarp();
        uint8_t* const to = const_cast<uint8_t*>(p.out.data) + (token * p.out.token + q_head * p.out.head) * 2;
        each_chunk<S::kOut, S::kOutPitch>(to, there ? S::kOut : 0, [&](uint32_t from, uint8_t* dst) { *reinterpret_cast<uint4*>(dst) = shared_load(rows_at + from); });
        if (p.lse != nullptr && there) p.lse[static_cast<int64_t>(token) * p.q.heads + q_head] = l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
        __syncwarp();
    }
}

template <int D>
static cudaError_t launch(const bfq_plan* plan, const AttendParams& p, cudaStream_t st) {
    static int per_sm[kMaxDevices] = {0};
    int& occ = per_sm[plan->device];
    if (occ == 0) {
        cudaError_t e = cudaFuncSetAttribute(k_join_tall<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(JoinSmem<D>::kBytes));
        int n = 0;
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k_join_tall<D>, 32 * kJoinWarps, JoinSmem<D>::kBytes);
        if (e != cudaSuccess) return e;
        occ = n > 0 ? n : 1;
    }
    const int64_t chunks = p.places(p.tall) * p.cache.heads * (kTallRows / 32), want = (chunks + kJoinWarps - 1) / kJoinWarps, most = int64_t(plan->sm_count) * occ;
    return launch_overlapped(k_join_tall<D>, dim3(unsigned(want < most ? want : most)), dim3(32 * kJoinWarps), JoinSmem<D>::kBytes, st, p, int(chunks));
}
cudaError_t join_tall_launch(const bfq_plan* plan, const AttendParams& p, cudaStream_t st) { return plan->n == 64 ? launch<64>(plan, p, st) : launch<128>(plan, p, st); }

}  // namespace kv
}  // namespace bfq
