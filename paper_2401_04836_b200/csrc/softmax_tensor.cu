// The passes of the softmax loss on the tensor cores.
//
// A block holds 256 own rows (two tiles of 128) in shared memory and streams tiles of other rows past them.  For each tile of
// scores:  S = Own Other^T  (tcgen05, both operands in shared memory) into tensor memory;  128 threads, one a row, turn S into
// shares  P = 2^(a S - base)  in place;  O = P Other  (P from tensor memory, the same bytes of Other as MN-major operand);  O is
// added in registers to the sums of earlier tiles.  Products of fp32 operands are lo hi + hi lo + hi hi of their fp16 terms, shares
// likewise two terms: 22 bits.  The tensor cores add up one tile alone (its chain is short, because what they cut off at each
// addition would not average out over a long one).
//
// Two tiles of rows take turns: while the tensor cores work on one, the threads of the other make shares.  One warp loads (bulk
// copies of whole images' rows, `stages` deep), one issues products.  The running maximum is a whole power of two that moves only
// when a score exceeds it by 2^11 (fp16 has room for that), so rescaling is rare and exact.
#include <cuda_fp16.h>

#include <algorithm>

#include "softmax_loss.cuh"
#include "umma.cuh"

namespace cb {
namespace loss {
namespace {

using namespace umma;

constexpr int kRows = 128;                       // of a tile of own rows: lanes of tensor memory
constexpr int kMaxTiles = 2;                     // tiles of own rows a block has
constexpr int kTile = 128;                       // other rows of a tile, half of them to each of two warpgroups
constexpr int kHalf = kTile / 2;
constexpr int kMaxStages = 4;
constexpr int kShift = 4;                        // shares are 2^kShift times too large: small ones stay in fp16's range
constexpr float kSlack = 11.f;                   // by how much a score may exceed the base (2^(kShift + kSlack) < 65504)

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct Barriers {
    uint64_t own_full, own_free;                 // own rows in shared memory: there, read for the last time
    uint64_t full[kMaxStages], free[kMaxStages]; // a tile of other rows
    uint64_t done[2 * kMaxTiles];                // S of a warpgroup, and every product that it issued before, is complete
};

// A place in the ring of stages and the parity of its turn.
struct Place {
    uint32_t at = 0, turn = 0;
    __device__ __forceinline__ void next(uint32_t stages) {
        if (++at == stages) at = 0, turn ^= 1;
    }
};

__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
__device__ __forceinline__ void expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t to, const void *from, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// A wait that gives up after `polls` polls, or soon after another thread of the block has given up.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, int polls, volatile int *failed) {
    if (mbar_wait(bar, parity, 1)) return true;
    for (int n = 0; n < polls; n += 64) {
        if (mbar_wait(bar, parity, 64)) return true;
        if (*failed) return false;
    }
    *failed = 1;
    return false;
}

__device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }

__host__ __device__ constexpr int tiles_of(int columns) { return columns <= 64 ? 2 : 1; }
__host__ __device__ constexpr int threads_of(int columns) { return 128 * (2 * tiles_of(columns) + 1); }
// whether tensor memory has room for the own rows' terms beside S and O
__host__ __device__ constexpr bool own_in_tensor(int columns) { return columns != 64; }

// two fp32 values in one register pair: one instruction for both
using Two = unsigned long long;
__device__ __forceinline__ Two two(float x, float y) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 both(Two v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// RP: room for sums in registers.  QT, KT: terms of own and other rows; PT: terms of a share (its product takes as many of Other).
template <int RP, int PASS, int QT, int KT, int PT>
__global__ void __launch_bounds__(threads_of(RP), 1) loss_tensor(const __grid_constant__ TensorArgs a) {
    constexpr bool kSums = PASS != kLossAlone;
    constexpr int kTiles = tiles_of(RP);                             // tiles of own rows
    constexpr int kTeams = 2 * kTiles;                               // warpgroups that make shares: two a tile, 64 other rows each
    constexpr bool kOwnInTensor = own_in_tensor(RP);
    // columns of tensor memory: S of every team (P takes its place), own rows of every tile, O of every team
    constexpr int kOwnAt = kHalf * kTeams, kOwnWide = kOwnInTensor ? RP : 0;
    constexpr int kSumsAt = kOwnAt + kOwnWide * kTiles;
    static_assert(kSumsAt + RP * kTeams <= 512);
    constexpr int kStep = RP <= 32 ? 32 : 16;                        // scores a thread has in registers at once
    constexpr int kLoader = 4 * kTeams;                              // warp
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ Barriers bars;
    __shared__ float2 merged[kTiles][kRows];                         // maximum and sum of the second team
    __shared__ uint32_t tmem_at;
    __shared__ int failed_s, team_gave_up[kTeams][2], tile_gave_up[kTiles];
    volatile int *failed = &failed_s;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t row_bytes = 2u * a.columns;
    const uint32_t own_term = kRows * row_bytes, other_term = kTile * row_bytes;
    const uint32_t stage_bytes = KT * other_term + (PASS == kByColumns ? 8u * kTile : 0u);
    const uint32_t own_at = smem_u32(smem), other_at = own_at + (kOwnInTensor ? 0 : kTiles * QT * own_term);

    if (threadIdx.x == 0) {
        failed_s = 0;
        for (int w = 0; w < kTeams; ++w) team_gave_up[w][0] = team_gave_up[w][1] = 0;
        for (int t = 0; t < kTiles; ++t) tile_gave_up[t] = 0;
        auto init = [](uint64_t *b, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_u32(b)), "r"(n) : "memory"); };
        init(&bars.own_full, 1);
        init(&bars.own_free, kTeams);
        for (int s = 0; s < kMaxStages; ++s) init(&bars.full[s], 1), init(&bars.free[s], kTeams);
        for (int w = 0; w < kTeams; ++w) init(&bars.done[w], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kLoader) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_at;
    after_last_kernel();

    const int64_t u0 = (int64_t)blockIdx.x * a.each, u1 = min(u0 + a.each, a.groups * a.tiles);
    if (warp >= kLoader) {
        // of the launch's registers (5 x 96 or 3 x 168, by warpgroups) these warps leave the teams 4 x 112 or 2 x 224
        if constexpr (kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == kLoader && elect_one()) {
            Place place;
            uint32_t run = 0, loads = 0;                             // runs begun; tiles loaded, up to the number of stages
            bool ok = true;
            for (int64_t u = u0; u < u1 && ok;) {
                const int64_t g = u / a.tiles, t0 = u - g * a.tiles, t1 = min(a.tiles, t0 + (u1 - u));
                if (!kOwnInTensor) {
                    const int live = (int)min((a.n_own - g * kTiles * kRows + kRows - 1) / kRows, (int64_t)kTiles);
                    if (!(ok = wait_for(smem_u32(&bars.own_free), (run & 1) ^ 1, a.polls, failed))) break;
                    const uint32_t bar = smem_u32(&bars.own_full);
                    expect(bar, live * QT * own_term);
                    ++run;
                    for (int t = 0; t < live; ++t)
                        for (int q = 0; q < QT; ++q)
                            bulk_load(own_at + (t * QT + q) * own_term, (q ? a.own.lo : a.own.hi) + (g * kTiles + t) * kRows * a.columns, own_term, bar);
                }
                for (int64_t t = t0; t < t1; ++t) {
                    if (!(ok = wait_for(smem_u32(&bars.free[place.at]), place.turn ^ 1, a.polls, failed))) break;
                    const uint32_t full = smem_u32(&bars.full[place.at]), to = other_at + place.at * stage_bytes;
                    expect(full, stage_bytes);
                    for (int q = 0; q < KT; ++q) bulk_load(to + q * other_term, (q ? a.other.lo : a.other.hi) + t * kTile * a.columns, other_term, full);
                    if (PASS == kByColumns) {
                        bulk_load(to + KT * other_term, a.base + t * kTile, 4 * kTile, full);
                        bulk_load(to + KT * other_term + 4 * kTile, a.pull + t * kTile, 4 * kTile, full);
                    }
                    place.next(a.stages);
                    loads = min(loads + 1, (uint32_t)a.stages);
                }
                u += t1 - t0;
            }
            // nothing of this block is under way when it ends, whatever the others did
            if (!ok) {
                if (run) mbar_wait(smem_u32(&bars.own_full), (run & 1) ^ 1, 1 << 14);
                for (uint32_t i = 0; i < loads; ++i) {               // the last ones, backwards
                    if (place.at == 0) place.at = a.stages, place.turn ^= 1;
                    --place.at;
                    mbar_wait(smem_u32(&bars.full[place.at]), place.turn, 1 << 14);
                }
            }
        }
        __syncwarp();
    } else {
        if constexpr (kTiles == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int team = warp / 4, t = team / 2, h = team % 2;       // tile of own rows, half of the other rows
        const bool issues = warp % 4 == team;                        // the warp that issues the team's products: one on each scheduler
        const uint32_t s_at = tmem + kHalf * team, own_tmem = tmem + kOwnAt + kOwnWide * t, sums_at = tmem + kSumsAt + RP * team;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;           // 32 lanes a warp
        const int in_tile = 32 * (warp % 4) + lane;
        // from accumulated scores to units of log 2, and what undoes the scales of the sums
        const int e_own = image_exponent(a.words[a.own_word]), e_other = image_exponent(a.words[a.other_word]);
        const float unit = kLog2e * exp2f((float)-e_own) * exp2f((float)-e_other);
        const Two unit2 = two(unit, unit);
        const uint32_t done = smem_u32(&bars.done[team]);
        uint32_t turn = 0, runs = 0, beat = 0;                       // parity of `done`; runs; tiles
        Place place;
        bool ok = true;
        auto arrived = [&](uint32_t bar, uint32_t parity) {          // for the whole warp or not at all
            ok = __all_sync(0xffffffffu, wait_for(bar, parity, a.polls, failed));
            fence_after();
            return ok;
        };
        // descriptors of the first 16 columns (scores) or rows (sums); further ones, terms and stages lie a constant apart
        const uint32_t group_rows = 8 * row_bytes;                   // bytes of 8 rows: 8 columns of them are 128 bytes
        const uint64_t own_k = smem_desc(own_at + t * QT * own_term, 128, group_rows);
        const uint64_t other_k = smem_desc(other_at + h * kHalf * row_bytes, 128, group_rows), other_mn = smem_desc(other_at + h * kHalf * row_bytes, group_rows, 128);
        const uint32_t q_term = own_term >> 4, k_term = other_term >> 4, k_stage = stage_bytes >> 4, mn_step = (2 * group_rows) >> 4;
        const uint32_t i_scores = idesc_f16(kRows, kHalf, false), i_sums = idesc_f16(kRows, a.columns, true);
        const int deep = a.columns / 16;
        auto scores = [&](uint32_t stage) {
            const uint64_t k = other_k + stage * k_stage;
            if (!a.withhold && elect_one()) {
                bool first = true;
                auto product = [&](int q, uint64_t ka) {             // term q of own rows
#pragma unroll
                    for (int c = 0; c < RP / 16; ++c, first = false) {
                        if (c >= deep) break;
                        if (kOwnInTensor) umma_f16_ts(s_at, own_tmem + q * (RP / 2) + 8 * c, ka + c * 16, i_scores, first ? 0u : 1u);
                        else umma_f16(s_at, own_k + q * q_term + c * 16, ka + c * 16, i_scores, first ? 0u : 1u);
                    }
                };
                if (QT == 2) product(1, k);
                if (KT == 2) product(0, k + k_term);
                product(0, k);
                umma_commit(done);
            }
            __syncwarp();
        };
        auto sums = [&](uint32_t stage, bool last) {
            const uint64_t k = other_mn + stage * k_stage;
            if (!a.withhold && elect_one()) {
                bool first = true;
                auto product = [&](uint32_t pa, uint64_t ka) {
#pragma unroll
                    for (int c = 0; c < kHalf / 16; ++c, first = false) umma_f16_ts(sums_at, pa + c * 16, ka + c * mn_step, i_sums, first ? 0u : 1u);
                };
                if (kSums) {
                    if (PT == 2) {
                        product(s_at + 8, k);
                        product(s_at, k + k_term);
                    }
                    product(s_at, k);
                }
                umma_commit(smem_u32(&bars.free[stage]));
                if (last) umma_commit(done);
            }
            __syncwarp();
        };
        for (int64_t u = u0; u < u1 && ok; ++runs) {
            const int64_t g = u / a.tiles, t0 = u - g * a.tiles, t1 = min(a.tiles, t0 + (u1 - u));
            if ((g * kTiles + t) * kRows >= a.n_own) {               // no such rows: only what the loader waits for
                for (int64_t tile = t0; tile < t1 && ok; ++tile) {
                    if (issues && arrived(smem_u32(&bars.full[place.at]), place.turn) && lane == 0) arrive(smem_u32(&bars.free[place.at]));
                    place.next(a.stages);
                }
                if (!kOwnInTensor && issues && lane == 0) arrive(smem_u32(&bars.own_free));
                u += t1 - t0;
                continue;
            }
            float top = -INFINITY, total = 0.f;
            float sum[kSums ? RP : 1];
#pragma unroll
            for (int r = 0; r < (kSums ? RP : 1); ++r) sum[r] = 0.f;
            auto take = [&](float late) {                            // adds O of a tile, made from shares `late` times too large
                if constexpr (kSums) {
                    constexpr int kPiece = RP >= 32 ? 32 : 16;
                    const Two late2 = two(late, late);
#pragma unroll
                    for (int c = 0; c < RP / kPiece; ++c) {
                        if (kPiece * c >= a.columns) break;
                        uint32_t o[kPiece];
                        tmem_load(sums_at + lanes + kPiece * c, o);
                        tmem_landed(o);
#pragma unroll
                        for (int r = 0; r < kPiece; r += 2) {
                            const Two add = two(__uint_as_float(o[r]), __uint_as_float(o[r + 1])), old = two(sum[kPiece * c + r], sum[kPiece * c + r + 1]);
                            const float2 v = both(PASS == kByRows ? fma2(late2, add, old) : add2(add, old));
                            sum[kPiece * c + r] = v.x;
                            sum[kPiece * c + r + 1] = v.y;
                        }
                    }
                }
            };
            if constexpr (kOwnInTensor) {                            // a row a thread, one term a team
                for (int q = h; q < QT; q += 2) {
                    const uint4 *from = reinterpret_cast<const uint4 *>((q ? a.own.lo : a.own.hi) + ((g * kTiles + t) * kRows + in_tile / 8 * 8) * a.columns) + in_tile % 8;
#pragma unroll
                    for (int c = 0; c < RP / 16; ++c) {
                        if (c >= deep) break;
                        const uint4 x = __ldg(from + 16 * c), y = __ldg(from + 16 * c + 8);
                        const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                        tmem_store(own_tmem + lanes + q * (RP / 2) + 8 * c, w);
                    }
                }
                tmem_stored();
                fence_before();
                asm volatile("bar.sync %0, 256;" :: "r"(1 + t) : "memory");
                fence_after();
            }
            if (issues) {
                if ((kOwnInTensor || arrived(smem_u32(&bars.own_full), runs & 1)) && arrived(smem_u32(&bars.full[place.at]), place.turn)) scores(place.at);
            }
            for (int64_t tile = t0; tile < t1; ++tile, ++beat) {
                if (arrived(done, turn)) {
                    float late = 1.f;
                    const int valid = (int)min(a.n_other - tile * kTile - kHalf * h, (int64_t)kHalf);
                    const float *vec = reinterpret_cast<const float *>(smem + (other_at - own_at) + place.at * stage_bytes + KT * other_term) + kHalf * h;
                    if (PASS == kByColumns) arrived(smem_u32(&bars.full[place.at]), place.turn);    // base and pull came with the tile
                    Two part[2] = {0, 0};
#pragma unroll
                    for (int c = 0; c < kHalf / kStep; ++c) {
                        uint32_t s[kStep];
                        tmem_load(s_at + lanes + kStep * c, s);
                        tmem_landed(s);
                        if (PASS != kByColumns) {
                            if (valid < kHalf)
#pragma unroll
                                for (int j = 0; j < kStep; ++j)
                                    if (kStep * c + j >= valid) s[j] = 0xff800000u;    // -inf
                            float m = __uint_as_float(s[0]);
#pragma unroll
                            for (int j = 1; j < kStep; ++j) m = fmaxf(m, __uint_as_float(s[j]));
                            m *= unit;
                            const bool raise = m > top + (PASS == kLossAlone ? 60.f : kSlack);
                            if (__any_sync(0xffffffffu, raise)) {
                                const float now = raise ? ceilf(m) : top, keep = raise ? exp2f(top - now) : 1.f;
                                top = now;
                                total *= keep;
                                late *= keep;
#pragma unroll
                                for (int q = 0; q < 2; ++q) part[q] = mul2(part[q], two(keep, keep));
                                if (kSums) {
#pragma unroll
                                    for (int r = 0; r < RP; ++r) sum[r] *= keep;
#pragma unroll 1
                                    for (int k = 0; k < c * kStep / 16; ++k) {          // shares of this tile that are written already
                                        uint32_t p[16], w[8];
                                        tmem_stored();
                                        tmem_load(s_at + lanes + 16 * k, p);
                                        tmem_landed(p);
#pragma unroll
                                        for (int j = 0; j < 8; ++j) {
                                            float2 v = unpack(p[j]);
                                            if (PT == 2) {
                                                const float2 lo = unpack(p[8 + j]);
                                                v.x = (v.x + lo.x) * keep;
                                                v.y = (v.y + lo.y) * keep;
                                            } else {
                                                v.x *= keep;
                                                v.y *= keep;
                                            }
                                            w[j] = pack(v.x, v.y);
                                            const float2 hi = unpack(w[j]);
                                            p[j] = pack(v.x - hi.x, v.y - hi.y);
                                        }
                                        tmem_store(s_at + lanes + 16 * k, w);
                                        if (PT == 2) {
#pragma unroll
                                            for (int j = 0; j < 8; ++j) w[j] = p[j];
                                            tmem_store(s_at + lanes + 16 * k + 8, w);
                                        }
                                    }
                                }
                            }
                        }
                        // no score yet (a half without other rows): nothing to subtract, the shares are 2^-inf
                        const float base = top == -INFINITY ? 0.f : (PASS == kLossAlone ? 0.f : (float)kShift) - top;
                        const Two base2 = two(base, base);
#pragma unroll
                        for (int k = 0; k < kStep / 16; ++k) {
                            uint32_t hi[8], lo[8];
#pragma unroll
                            for (int j = 0; j < 8; j += 2) {
                                const int at = 16 * k + 2 * j;
                                Two p[2];
                                ulonglong2 pull;
                                if (PASS == kByColumns) {
                                    const ulonglong2 bs = *reinterpret_cast<const ulonglong2 *>(vec + kStep * c + at);
                                    pull = *reinterpret_cast<const ulonglong2 *>(vec + kTile + kStep * c + at);
                                    p[0] = bs.x;
                                    p[1] = bs.y;
                                }
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    const Two e = fma2(two(__uint_as_float(s[at + 2 * i]), __uint_as_float(s[at + 2 * i + 1])), unit2, PASS == kByColumns ? p[i] : base2);
                                    p[i] = two(exp2_fast(both(e).x), exp2_fast(both(e).y));
                                    if (PASS == kByColumns) p[i] = mul2(p[i], i ? pull.y : pull.x);
                                    else part[i] = add2(part[i], p[i]);
                                    if (!kSums) continue;
                                    const float2 v = both(p[i]);
                                    hi[j + i] = pack(v.x, v.y);
                                    if (PT == 2) {
                                        const float2 f = unpack(hi[j + i]);
                                        const float2 l = both(fma2(two(f.x, f.y), two(-1.f, -1.f), p[i]));
                                        lo[j + i] = pack(l.x, l.y);
                                    }
                                }
                            }
                            if (kSums) {
                                tmem_store(s_at + lanes + kStep * c + 16 * k, hi);
                                if (PT == 2) tmem_store(s_at + lanes + kStep * c + 16 * k + 8, lo);
                            }
                        }
                    }
                    if (PASS != kByColumns) {
                        const float2 x = both(add2(part[0], part[1]));
                        total += x.x + x.y;
                    }
                    if (kSums) {
                        if (tile > t0) take(late);                   // O of the tile before is complete: it was issued in front of these scores
                        tmem_stored();
                    }
                    turn ^= 1;
                }
                fence_before();
                if (!ok) *(volatile int *)&team_gave_up[team][beat & 1] = 1;
                asm volatile("bar.sync %0, 128;" :: "r"(1 + kTiles + team) : "memory");
                ok = *(volatile int *)&team_gave_up[team][beat & 1] == 0;        // the same for the whole team
                const uint32_t stage = place.at;
                place.next(a.stages);
                if (!ok) break;
                if (issues) {
                    fence_after();
                    sums(stage, tile + 1 == t1);
                    if (tile + 1 < t1 && arrived(smem_u32(&bars.full[place.at]), place.turn)) scores(place.at);   // behind the products that read the shares in their place
                }
            }
            if (ok && arrived(done, turn)) {
                turn ^= 1;
                take(1.f);
            }
            // The second team hands its sums to the first where its O was.
            if (h == 1) {
                if constexpr (kSums) {
#pragma unroll
                    for (int c = 0; c < RP / 8; ++c) {
                        if (8 * c >= a.columns) break;
                        uint32_t w[8];
#pragma unroll
                        for (int r = 0; r < 8; ++r) w[r] = __float_as_uint(sum[8 * c + r]);
                        tmem_store(sums_at + lanes + 8 * c, w);
                    }
                    tmem_stored();
                }
                merged[t][in_tile] = make_float2(top, total);
                fence_before();
            }
            if (!ok) *(volatile int *)&tile_gave_up[t] = 1;
            asm volatile("bar.sync %0, 256;" :: "r"(1 + t) : "memory");
            ok = *(volatile int *)&tile_gave_up[t] == 0;             // the same for both teams: both go on or neither
            if (!kOwnInTensor && issues && lane == 0) arrive(smem_u32(&bars.own_free));    // every product of the team is complete
            if (h == 0) {
                fence_after();
                const int64_t part = (g * a.parts + ((int64_t)blockIdx.x - g * a.tiles / a.each)) * (kTiles * kRows) + kRows * t + in_tile;
                const float2 other = merged[t][in_tile];
                const float shift = PASS == kByRows ? 1.f / (1 << kShift) : 1.f;
                float mine = 1.f, theirs = 1.f;
                if (PASS != kByColumns) {
                    const float most = fmaxf(top, other.x);
                    mine = top == -INFINITY ? 0.f : exp2f(top - most);
                    theirs = other.x == -INFINITY ? 0.f : exp2f(other.x - most);
                    a.top[part] = most;
                    a.total[part] = (total * mine + other.y * theirs) * shift;
                }
                if constexpr (kSums) {
                    const float undo = exp2f((float)-e_other) * shift, undo2 = PASS == kByColumns ? exp2f((float)-image_exponent(a.words[kMaxWeight])) : 1.f;
                    float4 *to = reinterpret_cast<float4 *>(a.sum + part * a.width);
#pragma unroll
                    for (int c = 0; c < RP / 16; ++c) {
                        if (16 * c >= a.columns) break;
                        uint32_t o[16];
                        tmem_load(sums_at + RP + lanes + 16 * c, o);
                        tmem_landed(o);
                        float x[16];
#pragma unroll
                        for (int r = 0; r < 16; ++r) x[r] = fmaf(sum[16 * c + r], mine, __uint_as_float(o[r]) * theirs) * undo * undo2;
#pragma unroll
                        for (int q = 0; q < 4; ++q) to[4 * c + q] = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                    }
                }
                fence_before();
            }
            asm volatile("bar.sync %0, 256;" :: "r"(1 + t) : "memory");
            fence_after();
            u += t1 - t0;
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == kLoader) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    if (threadIdx.x == 0 && failed_s) atomicExch(a.gave_up, 1u);
    start_next_kernel();
}

template <int RP, int PASS, int QT, int KT, int PT>
cudaError_t launch(TensorArgs a, int blocks, cudaStream_t stream) {
    constexpr int kMost = 224 * 1024;                                // of 227 KB: barriers and what halves exchange are apart
    const int own = own_in_tensor(RP) ? 0 : tiles_of(RP) * QT * kRows * 2 * a.columns, stage = KT * kTile * 2 * a.columns + (PASS == kByColumns ? 8 * kTile : 0);
    a.stages = std::min<int>(kMaxStages, (kMost - own) / stage);
    const int bytes = own + a.stages * stage;
    static PerDeviceOnce once;
    const cudaError_t e = once_per_device(once, [] {
        return cudaFuncSetAttribute(loss_tensor<RP, PASS, QT, KT, PT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    });
    if (e != cudaSuccess) return e;
    return launch_early(loss_tensor<RP, PASS, QT, KT, PT>, dim3(blocks), threads_of(RP), bytes, stream, a);
}

template <int RP, bool WIDE>
cudaError_t by_pass(int pass, const TensorArgs &a, int blocks, cudaStream_t stream) {
    constexpr int PT = WIDE ? 2 : 1;
    if (pass == kLossAlone) return launch<RP, kLossAlone, 2, WIDE ? 2 : 1, PT>(a, blocks, stream);
    if (pass == kByRows) return launch<RP, kByRows, 2, WIDE ? 2 : 1, PT>(a, blocks, stream);
    return launch<RP, kByColumns, WIDE ? 2 : 1, 2, PT>(a, blocks, stream);
}

template <bool WIDE>
cudaError_t by_rank(int pass, const TensorArgs &a, int blocks, cudaStream_t stream) {
    if (a.columns <= 16) return by_pass<16, WIDE>(pass, a, blocks, stream);
    if (a.columns <= 32) return by_pass<32, WIDE>(pass, a, blocks, stream);
    if (a.columns <= 64) return by_pass<64, WIDE>(pass, a, blocks, stream);
    return by_pass<128, WIDE>(pass, a, blocks, stream);
}

}  // namespace

int tensor_rows(int rank) { return kRows * tiles_of(image_columns(rank)); }

cudaError_t tensor_pass(int pass, bool wide, const TensorArgs &a, int blocks, cudaStream_t stream) {
    return wide ? by_rank<true>(pass, a, blocks, stream) : by_rank<false>(pass, a, blocks, stream);
}

}  // namespace loss
}  // namespace cb
