// Attention of many query rows over the same keys of the paged low-bit cache (a shared prefix for a batch, chunks of a prompt) on the
// fifth-generation tensor cores: the same formula and references as the kernel for few rows (bfq_kvattn.cu).
//
// A CTA has up to 256 rows, two M = 128 tiles, and takes its keys in units of 64:
//   warps 0 .. 3, 4 .. 7  softmax of tile 0, 1: a thread owns a row (a lane of tensor memory) and has its 64 scores in registers: the largest
//                         (a new reference and a pass over the products only where a score passes the old one by more than 8, as
//                         there), exp2, sum and the rounding to fp16, which goes back to tensor memory over the scores;
//   warps 8 .. 15         codes to fp16: a unit's keys and values into one of four stages, loaded two units ahead into registers;
//   warp 16               the MMAs: S = Q K^T (both operands in shared memory), O += P V (P from tensor memory).
// Two buffers of scores for each tile: S of the next unit is there while the products of this one run, so that a tile's softmax waits
// for nothing but itself.  With one buffer of 128 keys a unit's chain, softmax 2500 cycles and then both products 1600, was the kernel's period.  Tensor
// memory: 2 x 2 x 64 columns of scores (probabilities in the same place), 2 x D of products.
// Keys and values are multiplied by their scales on the way into shared memory, over a power of two for all of a pair so far: one rounding to
// fp16 of each element, 2^-12 on average and independent of its neighbours, a fraction of the output's own rounding.  Applied exactly, to
// scores and probabilities, the scales would be read from shared memory 256 times by every softmax warp for a unit, which took three times as
// long as everything else.
// Probabilities go to fp16 times 2^7: the reference is at most 2^8 below the largest, so that they stay below 2^15, and one of 2^-32 of the row's
// largest is still half a step there.  Without it what is below 2^-25 of the reference counted in the sum of the exponentials alone: beside a
// large score whose value is near zero, as a prompt's first token has it, nothing was left of the result.
// Shared-memory operands have the 128-byte swizzle: a row of 128 bytes is 64 elements d of one key (or query row), the two halves of
// D = 128 lie one after the other; K is K-major, V the same bytes read MN-major.  The d within a 16-byte chunk stand in the order in which a
// code word's pairs come out (0 4 1 5 2 6 3 7, or 0 2 1 3 of each four): Q's rows are stored in that order too, and O's columns are
// put back where they are written.
#include "bfq_kvattn.cuh"
#include "bfq_n4096.cuh"

namespace bfq {
namespace kv {

constexpr int kTallThreads = 20 * 32;  // warps 17 .. 19 only lend their registers
constexpr int kConvert = 256;          // threads that turn codes into operands
constexpr int kStageCount = 4;

template <int D>
struct TallSmem {
    static constexpr uint32_t kHalves = D / 64, kTile = kHalves * 128 * 128;     // 128 query rows
    static constexpr uint32_t kKeysHalf = kTallUnit * 128, kKeys = kHalves * kKeysHalf;  // 64 elements of a unit's keys, all of them
    static constexpr uint32_t kQ = 0, kStages = 2 * kTile, kStage = 2 * kKeys;   // a stage: keys, values
    static constexpr uint32_t kFactors = kStages + kStageCount * kStage;          // per stage: less, unit of the products, unit of the scores
    static constexpr uint32_t kBars = kFactors + kStageCount * 16;
    static constexpr uint32_t kBytes = kBars + 24 * 8 + 1024;  // and what rounding the base up to 1024 takes
};
// per stage: operands there, free; per tile and buffer: scores there, probabilities there; per tile: queries there, products of a unit done, of a pair; all
// products done (after a wait has given up)
enum Bar { kKvFull = 0, kKvEmpty = 4, kSFull = 8, kPFull = 12, kQFull = 16, kDone = 18, kOFull = 20, kAllDone = 22, kBarCount = 23 };

template <int D, int BITS>
__global__ void __launch_bounds__(kTallThreads, 1) k_attend_tall(const AttendParams p) {
    using M = TallSmem<D>;
    constexpr int kRow = D * BITS / 8;
    extern __shared__ uint8_t smem_raw[];
    __shared__ int scan[kTallThreads / 32 + 2];
    __shared__ uint32_t tmem_at;
    __shared__ volatile int dead;
    __shared__ float2 warp_top[2][kConvert / 32];  // of the keys' scales, the values'
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto bar = [&](int b) { return base + M::kBars + 8u * b; };
    auto stage_at = [&](int s) { return base + M::kStages + s * M::kStage; };
    auto factors_at = [&](int s) { return base + M::kFactors + 16u * s; };
    grid_dep_wait();
    grid_dep_launch();
    const Part& part = p.tall;
    Walk walk;
    const Run run = find_run<kTallThreads>(p, part, scan, &walk);
    if (run.count == 0) return;
    if (tid == 0) {
        for (int s = 0; s < 4; ++s) {
            mbar_init(bar(kKvFull + s), kConvert), mbar_init(bar(kKvEmpty + s), 1);
            mbar_init(bar(kSFull + s), 1), mbar_init(bar(kPFull + s), 128);
        }
        for (int t = 0; t < 2; ++t) mbar_init(bar(kQFull + t), 128), mbar_init(bar(kDone + t), 1), mbar_init(bar(kOFull + t), 1);
        mbar_init(bar(kAllDone), 1);
        mbar_init_fence();
        dead = 0;
    }
    if (warp == 16) tmem_alloc512(smem_u32(&tmem_at));
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = tmem_at;
    auto scores = [&](int tile, int buffer) { return tmem + 128u * tile + 64u * buffer; };
    auto products = [&](int tile) { return tmem + 256u + D * tile; };
    const int count = run.count;

    // registers: 256 x 136 + 256 x 80 + 128 x 48 = 640 x 96, what the block was launched with
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
        // ---- softmax ---------------------------------------------------------------------------------------------------------
        const int tile = warp >> 2, row_of_tile = tid & 127;
        const uint32_t lanes = uint32_t(warp & 3) << 21;  // 32 lanes of tensor memory
        const uint32_t o_at = products(tile) + lanes;
        float m = -INFINITY, l = 0.f, row_scale = 0.f, unit = 0.f;
        int limit = 0, least = 0;  // keys of the row; of the warp's rows, at least
        // s_phase: a bit for each buffer; done_phase: of the last products that were asked for.  When a unit's scores are there, the products of the
        // unit before the last are done, so that a wait for the last one's parity means that one; at a pair's end they may not be
        uint32_t s_phase = 0, done_phase = 0, o_phase = 0;
        bool active = false;
        int pair_from = run.from - walk.unit;
        auto open = [&]() {
            const Tile& t = walk.tile;
            active = t.rows > 128 * tile;
            if (!active) return;
            constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes;  // of a row
            const int first_row = 128 * tile + 32 * (warp & 3), part_of = lane % kLanes;
            const float sign = p.scale_log2 < 0.f ? -1.f : 1.f;
            // eight loads on their way at a time
            constexpr int kLoads = 8;
#pragma unroll 1
            for (int n0 = 0; n0 < 32; n0 += kLoads * kRowsAtOnce) {
                uint4 v[kLoads];
#pragma unroll
                for (int x = 0; x < kLoads; ++x) {
                    const int r = first_row + n0 + x * kRowsAtOnce + lane / kLanes, row = t.row0 + r, token = row / p.group;
                    v[x] = make_uint4(0, 0, 0, 0);
                    if (r < t.rows)
                        v[x] = load_plain(reinterpret_cast<const uint4*>(p.q.data + ((t.token0 + token) * p.q.token + (walk.head * p.group + row - token * p.group) * p.q.head + 8 * part_of) * 2));
                }
#pragma unroll
                for (int x = 0; x < kLoads; ++x) {
                    const int n = n0 + x * kRowsAtOnce;
                    const uint32_t w[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
                    float top = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xFFFF0000u))));
#pragma unroll
                    for (int y = 1; y < kLanes; y <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, y));
                    const RowPower power(top);
                    const float up = sign * power.up;
                    auto element = [&](int i) { return up * __uint_as_float(order<BITS>(i) & 1 ? w[order<BITS>(i) / 2] & 0xFFFF0000u : w[order<BITS>(i) / 2] << 16); };
                    const int at = 32 * (warp & 3) + n + lane / kLanes;  // of the tile
                    store16(base + M::kQ + tile * M::kTile + at * 128 + (part_of >> 3) * 16384 + (((part_of & 7) ^ (at & 7)) << 4), half_pair(element(0), element(1)),
                            half_pair(element(2), element(3)), half_pair(element(4), element(5)), half_pair(element(6), element(7)));
                    const float down = __shfl_sync(0xFFFFFFFFu, power.down, (lane % kRowsAtOnce) * kLanes);
                    if (lane / kRowsAtOnce == n / kRowsAtOnce) row_scale = fabsf(p.scale_log2) * down;  // the lane's own row
                }
            }
            const int r = 128 * tile + row_of_tile, row = t.row0 + r;
            const bool there = r < t.rows;
            fence_operands();
            arrive(bar(kQFull + tile));
            m = -INFINITY, l = 0.f;
            const int own = t.last0 + row / p.group + 1;
            limit = there ? (own < t.keys ? (own > 0 ? own : 0) : t.keys) : 0;
            least = __reduce_min_sync(0xFFFFFFFFu, there ? limit : 1 << 30);
        };
        auto close = [&](int done) {
            const int pair = walk.pair(p);
            if (active) {
                wait_for(bar(kOFull + tile), o_phase, &dead, p.status);
                o_phase ^= 1;
                tmem_fence_after();
                const int r = 128 * tile + row_of_tile;
                const bool there = r < walk.tile.rows;
                const long long entry = static_cast<long long>(blockIdx.x) + pair;
                // half of 32 rows at a time through the places of the warp's own query rows, which no product reads any more, so that rows are written
                // whole: 16 bytes at place (chunk ^ row) of a row's half.  Those places are, as open writes them, 4096 bytes at 4096 (warp & 3) of
                // each half of D: one block of 32 rows at 64 elements, two blocks of 16 rows 16384 apart at 128.  Other warps may still
                // be here, or write their rows of the next pair already: nothing orders the four of a tile between close and open.
                constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes, kBlockRows = 4096 / (2 * D);
                const uint32_t own = base + M::kQ + tile * M::kTile + (warp & 3) * 4096;
                auto staged = [&](int row, int chunk) {
                    return own + (row / kBlockRows) * 16384 + (row % kBlockRows) * 2 * D + ((chunk ^ (row & (kLanes - 1))) << 4);
                };
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) {
                        uint32_t v[32];
                        tmem_ld32(o_at + (D / 2) * h + 32 * c, v);
                        tmem_wait_ld32(v);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float x[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[order<BITS>(i)] = __uint_as_float(v[8 * q + i]) * unit;
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                store16(staged(lane, 8 * c + 2 * q + i), __float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]),
                                        __float_as_uint(x[4 * i + 3]));
                        }
                    }
                    __syncwarp();
                    const int chunk = lane % kLanes;
#pragma unroll 4
                    for (int n = 0; n < 32; n += kRowsAtOnce) {
                        const int row = n + lane / kLanes, to = 128 * tile + 32 * (warp & 3) + row;
                        const float4 x = load_shared4(staged(row, chunk));
                        if (to < walk.tile.rows) *reinterpret_cast<float4*>(part.parts + (entry * kTallRows + to) * D + (D / 2) * h + 4 * chunk) = x;
                    }
                    __syncwarp();
                }
                tmem_fence_before();
                if (there) part.sums[entry * kTallRows + r] = make_float2(m, l * 0x1p-7f);
            }
            if (tid == 0 && pair_from >= run.from) part.pairs[pair] = make_int2(blockIdx.x, (pair_from + walk.units - 1) / run.per - static_cast<int>(blockIdx.x) + 1);
            pair_from = done;
        };
        bool first = true;
        open();
        for (int i = 0; i < count; ++i) {
            if (active) {
                const int key0 = walk.unit * kTallUnit, buffer = i & 1;
                const bool edge = key0 + kTallUnit > least;  // some row of the warp ends in this unit, or has ended
                const uint32_t s_at = scores(tile, buffer) + lanes;
                // the factors and the scores, usually both there: one latency.  The warps of tile 1 pass over pairs that have no rows for it, and
                // may be here while all of the run before is still to be done: a wait is given 2^14 cycles for each unit of it (2350 are usual)
                const long long cycles = kWaitCycles + (static_cast<long long>(i) << 14);
                const bool kv_there = mbar_try_wait(bar(kKvFull + (i & 3)), (i >> 2) & 1), s_there = mbar_try_wait(bar(kSFull + 2 * tile + buffer), s_phase >> buffer & 1);
                if (!kv_there) wait_for(bar(kKvFull + (i & 3)), (i >> 2) & 1, &dead, p.status, cycles);
                if (!s_there) wait_for(bar(kSFull + 2 * tile + buffer), s_phase >> buffer & 1, &dead, p.status, cycles);
                s_phase ^= 1u << buffer;
                tmem_fence_after();
                uint32_t v[2][32];
                tmem_ld32(s_at, v[0]);
                tmem_ld32(s_at + 32, v[1]);
                const float4 factors = load_shared4(factors_at(i & 3));
                const float less = factors.x, scale = fmaxf(row_scale * factors.z, 1e-30f);  // -infinity times it is that
                unit = factors.y;
                tmem_wait_ld32(v[0]);
                tmem_wait_ld32(v[1]);
                if (edge) {
                    const int n = limit - key0;
#pragma unroll
                    for (int j = 0; j < 64; ++j) v[j >> 5][j & 31] = j < n ? v[j >> 5][j & 31] : 0xFF800000u;
                }
                float x[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int j = 0; j < 64; j += 2)
                    x[j >> 1 & 3] = fmaxf(fmaxf(x[j >> 1 & 3], __uint_as_float(v[j >> 5][j & 31])), __uint_as_float(v[j >> 5][(j & 31) + 1]));
                float most = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
                most = most == -INFINITY ? most : most * scale;
                const bool over = most > m + 8.f;
                if (first) {
                    m = most;
                } else if (__any_sync(0xFFFFFFFFu, over) || less != 1.f) {
                    wait_for(bar(kDone + tile), done_phase ^ 1, &dead, p.status);  // the products of the unit before
                    tmem_fence_after();
                    float f = less;
                    if (over) f *= exp2_fast(m - most), l *= exp2_fast(m - most), m = most;
#pragma unroll 1
                    for (int c = 0; c < D / 8; ++c) {
                        uint32_t w[8];
                        tmem_ld8(o_at + 8 * c, w);
                        tmem_wait_ld8(w);
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * f);
                        tmem_st8(o_at + 8 * c, w);
                    }
                }
                first = false;
                const float ref = m == -INFINITY ? 0.f : m;
                const u64 scale2 = pack2(scale, scale), ref2 = pack2(7.f - ref, 7.f - ref);
                u64 sum2[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t out[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float a, b;
                        unpack2(fma2(pack2u(v[c][2 * j], v[c][2 * j + 1]), scale2, ref2), a, b);
                        a = exp2_fast(a), b = exp2_fast(b);
                        sum2[j & 1] = add2(sum2[j & 1], pack2(a, b));
                        out[j] = half_pair(a, b);
                    }
                    tmem_st16(s_at + 16 * c, out);
                }
                float a, b;
                unpack2(add2(sum2[0], sum2[1]), a, b);
                l += a + b;
                tmem_wait_st();
                tmem_fence_before();
                done_phase ^= 1;
                arrive(bar(kPFull + 2 * tile + buffer));
            }
            if (walk.unit + 1 == walk.units || i + 1 == count) {
                close(run.from + i + 1);
                walk.next_pair(p, part);
                first = true;
                if (i + 1 < count) open();
            } else {
                ++walk.unit;
            }
        }
    } else if (warp < 16) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        // ---- codes to operands -------------------------------------------------------------------------------------------------
        const int w = warp - 8;
        const Unpack<BITS> unpack;
        // 16-byte pieces: the eight lanes of a phase of the stores below write chunks of one half to eight different places of 16 bytes
        constexpr int kPer = BITS == 4 ? 2 : 4;        // pieces of 64 elements
        constexpr int kKeys = 32 / (kPer * (D / 64));  // keys of a warp's 32 pieces: of one page
        constexpr int kTurns = kTallUnit / kKeys / 8 > 0 ? kTallUnit / kKeys / 8 : 1;  // D = 64 at 4 bits: half of the warps have all
        const int part_of = lane % kPer, key_low = lane / kPer % (8 / kPer);
        const int half = D == 128 ? lane >> 3 & 1 : 0, key_of = key_low + (8 / kPer) * (D == 128 ? lane >> 4 : lane >> 3);
        const bool busy = w * kKeys < kTallUnit;
        struct Raw {
            uint4 k[kTurns], v[kTurns];
            uint16_t k_scale[kTurns], v_scale[kTurns];
            bool first;  // unit of its pair
        };
        constexpr int64_t kNone = -(int64_t(1) << 32);
        int64_t page = kNone;  // lane c: of turn c; kNone: it has no keys
        int sent = 0;          // units loaded
        bool opens = true;     // the unit ahead is its pair's first here
        auto look = [&]() {    // pages of the unit ahead, a load earlier than they are needed
            const int key = walk.unit * kTallUnit + (lane * 8 + w) * kKeys;
            page = sent < count && busy && lane < kTurns && key < walk.tile.keys ? load_plain(walk.tile.pages + (key >> p.cache.page_shift)) : kNone;
        };
        auto load = [&](Raw& raw) {
            if (sent >= count) return;
            const int mask = (1 << p.cache.page_shift) - 1;
            if (page != kNone && (page < 0 || page >= p.cache.pages)) atomicExch(p.status, kBadIndex), page = kNone;
#pragma unroll
            for (int c = 0; c < kTurns; ++c) {
                const int key = walk.unit * kTallUnit + (c * 8 + w) * kKeys + key_of;
                const int64_t at = __shfl_sync(0xFFFFFFFFu, page, c);
                raw.k[c] = raw.v[c] = make_uint4(0, 0, 0, 0), raw.k_scale[c] = raw.v_scale[c] = 0;
                if (at >= 0 && key < walk.tile.keys) {
                    const int row = (walk.head << p.cache.page_shift) + (key & mask), off = row * kRow + 16 * (half * kPer + part_of);
                    raw.k[c] = load_plain(reinterpret_cast<const uint4*>(p.cache.k.codes + at * p.cache.k.codes_page + off));
                    raw.v[c] = load_plain(reinterpret_cast<const uint4*>(p.cache.v.codes + at * p.cache.v.codes_page + off));
                    raw.k_scale[c] = *static_cast<volatile const uint16_t*>(p.cache.k.scales + at * p.cache.k.scales_page + row);
                    raw.v_scale[c] = *static_cast<volatile const uint16_t*>(p.cache.v.scales + at * p.cache.v.scales_page + row);
                }
            }
            raw.first = opens;
            opens = walk.unit + 1 == walk.units;
            ++sent;
            walk.next(p, part);
            look();
        };
        auto times = [](uint32_t a, uint32_t b) {
            uint32_t d;
            asm("mul.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
            return d;
        };
        auto store = [&](uint32_t to, const uint4& raw, int key, float scale) {
            const uint32_t row = to + half * M::kKeysHalf + key * 128, s2 = half_pair(scale, scale);
            const uint32_t x[4] = {raw.x, raw.y, raw.z, raw.w};
            if constexpr (BITS == 4) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    store16(row + (((4 * part_of + j) ^ (key & 7)) << 4), times(unpack(x[j], 0), s2), times(unpack(x[j], 1), s2), times(unpack(x[j], 2), s2),
                            times(unpack(x[j], 3), s2));
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    store16(row + (((2 * part_of + j) ^ (key & 7)) << 4), times(unpack(x[2 * j], 0), s2), times(unpack(x[2 * j], 1), s2),
                            times(unpack(x[2 * j + 1], 0), s2), times(unpack(x[2 * j + 1], 1), s2));
            }
        };
        // the power of two above all scales of the pair so far, at most that of 65504
        auto above = [](float top, float most) { return most > top ? __uint_as_float((__float_as_uint(most) & 0x7F800000u) + 0x00800000u) : top; };
        float k_top = 0.f, v_top = 0.f;
        auto step = [&](int i, Raw& raw) {
            const int s = i & 3;
            float2 most = make_float2(0.f, 0.f);
            // a scale that is not finite (append_kv writes none): a key of NaN, for the rows that see it
#pragma unroll
            for (int c = 0; c < kTurns; ++c)
                if ((raw.k_scale[c] & 0x7C00) == 0x7C00 || (raw.v_scale[c] & 0x7C00) == 0x7C00) raw.k_scale[c] = 0x7FFF, raw.v_scale[c] = 0;
#pragma unroll
            for (int c = 0; c < kTurns; ++c) most.x = fmaxf(most.x, half_value(raw.k_scale[c])), most.y = fmaxf(most.y, half_value(raw.v_scale[c]));
            most.x = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most.x)));  // not negative: ordered as integers
            most.y = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most.y)));
            if (lane == 0) warp_top[i & 1][w] = most;
            bar_sync(1, kConvert);
#pragma unroll
            for (int n = 0; n < kConvert / 32; ++n) most.x = fmaxf(most.x, warp_top[i & 1][n].x), most.y = fmaxf(most.y, warp_top[i & 1][n].y);
            if (raw.first) k_top = v_top = 0x1p-24f;
            const float v_before = v_top;
            k_top = above(k_top, most.x), v_top = above(v_top, most.y);
            const float k_factor = 128.f / k_top, v_factor = 128.f / v_top;  // codes times scales: at most 2^14
            if (i >= kStageCount) wait_for(bar(kKvEmpty + s), ((i >> 2) - 1) & 1, &dead, p.status);
            if (busy) {
#pragma unroll
                for (int c = 0; c < kTurns; ++c) {
                    const int key = (c * 8 + w) * kKeys + key_of;
                    store(stage_at(s), raw.k[c], key, k_factor * half_value(raw.k_scale[c]));
                    store(stage_at(s) + M::kKeys, raw.v[c], key, v_factor * half_value(raw.v_scale[c]));
                }
            }
            if (warp == 8 && lane == 0)
                asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(factors_at(s)), "f"(v_before / v_top), "f"(v_top * 0x1p-14f), "f"(k_top * 0x1p-7f), "f"(0.f)
                             : "memory");
            fence_operands();
            arrive(bar(kKvFull + s));
            load(raw);
        };
        Raw even, odd;
        look();
        load(even);
        load(odd);
        for (int i = 0; i < count; i += 2) {
            step(i, even);
            if (i + 1 < count) step(i + 1, odd);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        // ---- MMAs ----------------------------------------------------------------------------------------------------------------
        if (warp == 16) {
            const uint32_t lead = elect_one();
            uint32_t p_phase = 0, done_phase = 0, q_phase[2] = {0, 0};  // a bit for each tile and buffer, for each tile
            constexpr uint32_t kScoresDesc = instruction(kTallUnit, 0), kProductsDesc = instruction(D, 1);
            auto issue_scores = [&](int tile, int i) {
                const uint32_t a = base + M::kQ + tile * M::kTile, b = stage_at(i & 3);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_ss(lead, scores(tile, i & 1), operand(a + (k >> 2) * 16384 + (k & 3) * 32, 0), operand(b + (k >> 2) * M::kKeysHalf + (k & 3) * 32, 0), kScoresDesc, k > 0);
                commit_to(lead, bar(kSFull + 2 * tile + (i & 1)));
            };
            auto issue_products = [&](int tile, int i, bool accumulate) {
                const uint32_t b = stage_at(i & 3) + M::kKeys;
#pragma unroll
                for (int k = 0; k < kTallUnit / 16; ++k)
                    mma_ts(lead, products(tile), scores(tile, i & 1) + 8 * k, operand(b + 2048 * k, M::kKeysHalf), kProductsDesc, accumulate || k > 0);
                commit_to(lead, bar(kDone + tile));
            };
            auto operands_there = [&](int i) { wait_all(bar(kKvFull + (i & 3)), (i >> 2) & 1, &dead, p.status); };
            for (int i0 = 0; i0 < count;) {  // a pair's units here: i0 .. i1 - 1
                const int left = walk.units - walk.unit, i1 = i0 + left < count ? i0 + left : count, tiles = walk.tile.rows > 128 ? 2 : 1;
                operands_there(i0);
                for (int t = 0; t < tiles; ++t) {
                    wait_all(bar(kQFull + t), q_phase[t], &dead, p.status);
                    q_phase[t] ^= 1;
                    tmem_fence_after();
                    issue_scores(t, i0);
                }
                if (i0 + 1 < i1) {
                    operands_there(i0 + 1);
                    for (int t = 0; t < tiles; ++t) issue_scores(t, i0 + 1);
                }
                for (int i = i0; i < i1; ++i) {
                    for (int t = 0; t < tiles; ++t) {
                        const int which = 2 * t + (i & 1);
                        wait_all(bar(kPFull + which), p_phase >> which & 1, &dead, p.status);
                        p_phase ^= 1u << which;
                        tmem_fence_after();
                        issue_products(t, i, i > i0);
                        if (i + 1 == i1) commit_to(lead, bar(kOFull + t));
                    }
                    commit_to(lead, bar(kKvEmpty + (i & 3)));
                    if (i + 2 < i1) operands_there(i + 2);
                    for (int t = 0; t < tiles; ++t) {
                        // scores of another shape in the place of probabilities: products of different shapes are not ordered by themselves
                        wait_all(bar(kDone + t), done_phase >> t & 1, &dead, p.status);
                        done_phase ^= 1u << t;
                        if (i + 2 < i1) {
                            tmem_fence_after();
                            issue_scores(t, i + 2);
                        }
                    }
                }
                i0 = i1;
                walk.next_pair(p, part);
            }
            for (int i = count > kStageCount ? count - kStageCount : 0; i < count; ++i)  // the last arrivals have come
                wait_all(bar(kKvEmpty + (i & 3)), (i >> 2) & 1, &dead, p.status);
            if (__any_sync(0xFFFFFFFFu, dead)) {
                commit_to(lead, bar(kAllDone));
                drain(bar(kAllDone), 0);
            }
        }
        __syncwarp();
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 16) tmem_dealloc512(tmem);
}

template <int D, int BITS>
static cudaError_t prepare(const bfq_plan* plan) {
    static bool done[kMaxDevices] = {false};
    if (done[plan->device]) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(k_attend_tall<D, BITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(TallSmem<D>::kBytes));
    done[plan->device] = e == cudaSuccess;
    return e;
}
cudaError_t tall_ctas(const bfq_plan* plan, int bits, int* ctas) {
    *ctas = plan->sm_count;
    return plan->n == 64 ? (bits == 4 ? prepare<64, 4>(plan) : prepare<64, 8>(plan)) : (bits == 4 ? prepare<128, 4>(plan) : prepare<128, 8>(plan));
}
cudaError_t tall_launch(const bfq_plan* plan, const AttendParams& p, int ctas, cudaStream_t st) {
    const dim3 grid{unsigned(ctas)}, block{unsigned(kTallThreads)};
    if (plan->n == 64)
        return p.cache.bits == 4 ? launch_overlapped(k_attend_tall<64, 4>, grid, block, TallSmem<64>::kBytes, st, p)
                                 : launch_overlapped(k_attend_tall<64, 8>, grid, block, TallSmem<64>::kBytes, st, p);
    return p.cache.bits == 4 ? launch_overlapped(k_attend_tall<128, 4>, grid, block, TallSmem<128>::kBytes, st, p)
                             : launch_overlapped(k_attend_tall<128, 8>, grid, block, TallSmem<128>::kBytes, st, p);
}

}  // namespace kv
}  // namespace bfq
