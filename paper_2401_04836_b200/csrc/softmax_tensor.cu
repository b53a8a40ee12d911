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
    uint64_t own_full, own_free;                 // the own rows of a run of tiles: there, read for the last time
    uint64_t full[kMaxStages], free[kMaxStages]; // a tile of other rows
    uint64_t scores[kMaxTiles][2];               // S of a tile is complete, and every product issued before it (by buffer)
    uint64_t shares[kMaxTiles][2];               // P of a tile is written, or S read for the last time (by buffer)
    uint64_t sums[kMaxTiles];                    // O of a tile is complete, where no S issued later says so
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
    constexpr int kBuffers = kTiles == 1 || !kSums ? 2 : 1;          // of S; tensor memory holds kTiles x (S, and O of both halves)
    constexpr int kSpan = 512 / kTiles;                              // columns of tensor memory a tile has
    constexpr int kSumsAt = 128 * (kTiles == 1 ? 2 : 1);             // O of half 0 and, kSumsWide further, of half 1
    constexpr int kSumsWide = kTiles == 1 ? 128 : 64;
    constexpr int kStep = RP <= 32 ? 32 : 16;                        // scores a thread has in registers at once
    constexpr int kLoader = 8 * kTiles, kIssuer = kLoader + 1;       // warps; those in front of them make the shares
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ Barriers bars;
    __shared__ float2 merged[kTiles][kRows];                         // maximum and sum of half 1
    __shared__ uint32_t tmem_at;
    __shared__ int failed_s, gave_up[kTiles];
    volatile int *failed = &failed_s;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t row_bytes = 2u * a.columns;
    const uint32_t own_term = kRows * row_bytes, other_term = kTile * row_bytes;
    const uint32_t stage_bytes = KT * other_term + (PASS == kByColumns ? 8u * kTile : 0u);
    const uint32_t own_at = smem_u32(smem), other_at = own_at + kTiles * QT * own_term;

    if (threadIdx.x == 0) {
        failed_s = 0;
        for (int t = 0; t < kTiles; ++t) gave_up[t] = 0;
        auto init = [](uint64_t *b, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_u32(b)), "r"(n) : "memory"); };
        init(&bars.own_full, 1);
        init(&bars.own_free, 1);
        for (int s = 0; s < kMaxStages; ++s) init(&bars.full[s], 1), init(&bars.free[s], 1);
        for (int t = 0; t < kMaxTiles; ++t)
            for (int b = 0; b < 2; ++b) {
                init(&bars.scores[t][b], 1);
                init(&bars.shares[t][b], 8);
            }
        for (int t = 0; t < kMaxTiles; ++t) init(&bars.sums[t], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssuer) {
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
        // of the launch's registers (5 x 96 or 3 x 168, by warpgroups) these warps leave the others 4 x 104 or 2 x 208
        if constexpr (kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == kLoader && elect_one()) {
            Place place;
            uint32_t run = 0, loads = 0;                             // runs begun; tiles loaded, up to the number of stages
            bool ok = true;
            for (int64_t u = u0; u < u1 && ok;) {
                const int64_t g = u / a.tiles, t0 = u - g * a.tiles, t1 = min(a.tiles, t0 + (u1 - u));
                const int live = (int)min((a.n_own - g * kTiles * kRows + kRows - 1) / kRows, (int64_t)kTiles);
                if (!(ok = wait_for(smem_u32(&bars.own_free), (run & 1) ^ 1, a.polls, failed))) break;
                const uint32_t bar = smem_u32(&bars.own_full);
                expect(bar, live * QT * own_term);
                ++run;
                for (int t = 0; t < live; ++t)
                    for (int q = 0; q < QT; ++q)
                        bulk_load(own_at + (t * QT + q) * own_term, (q ? a.own.lo : a.own.hi) + (g * kTiles + t) * kRows * a.columns, own_term, bar);
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
        } else if (warp == kIssuer) {                                // the whole warp: its operands stay in uniform registers
            const uint32_t i_scores = idesc_f16(kRows, kTile, false), i_sums = idesc_f16(kRows, a.columns, true);
            const uint32_t group_rows = 8 * row_bytes;               // bytes of 8 rows: 8 columns of them are 128 bytes
            const int deep = a.columns / 16;
            // descriptors of the first 16 columns (scores) or rows (sums); further ones, terms and stages lie a constant apart
            const uint64_t own_k = smem_desc(own_at, 128, group_rows), other_k = smem_desc(other_at, 128, group_rows);
            const uint64_t other_mn = smem_desc(other_at, group_rows, 128);
            const uint32_t q_term = own_term >> 4, k_term = other_term >> 4, k_stage = stage_bytes >> 4, mn_step = (2 * group_rows) >> 4;
            uint32_t run = 0, made = 0;                              // runs; tiles whose scores were issued in all runs before
            uint32_t made_t[kTiles] = {};                            // the same of each tile of own rows
            Place place;
            auto commit = [&](uint64_t *b) { if (!a.withhold && elect_one()) umma_commit(smem_u32(b)); };
            auto scores = [&](int t, uint32_t stage, uint32_t b) {
                const uint32_t to = tmem + kSpan * t + 128 * b;
                const uint64_t q = own_k + t * QT * q_term, k = other_k + stage * k_stage;
                bool first = true;
                auto product = [&](uint64_t qa, uint64_t ka) {
#pragma unroll
                    for (int c = 0; c < RP / 16; ++c, first = false) {
                        if (c >= deep) break;
                        umma_f16(to, qa + c * 16, ka + c * 16, i_scores, first ? 0u : 1u);
                    }
                };
                if (!a.withhold && elect_one()) {
                    if (QT == 2) product(q + q_term, k);
                    if (KT == 2) product(q, k + k_term);
                    product(q, k);
                    umma_commit(smem_u32(&bars.scores[t][b]));
                }
                __syncwarp();
            };
            auto sums = [&](int t, uint32_t stage, uint32_t b) {
                const uint64_t k = other_mn + stage * k_stage;
                const uint32_t to = tmem + kSpan * t + kSumsAt, p = tmem + kSpan * t + 128 * b;
                if (!a.withhold && elect_one()) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        bool first = true;
                        auto product = [&](uint32_t pa, uint64_t ka) {
#pragma unroll
                            for (int c = h * kHalf / 16; c < (h + 1) * kHalf / 16; ++c, first = false)
                                umma_f16_ts(to + kSumsWide * h, pa + c * 16, ka + c * mn_step, i_sums, first ? 0u : 1u);
                        };
                        if (PT == 2) {
                            product(p + 8, k);
                            product(p, k + k_term);
                        }
                        product(p, k);
                    }
                }
                __syncwarp();
            };
            bool ok = true;
            auto arrived = [&](uint64_t *b, uint32_t parity) {
                ok = __all_sync(0xffffffffu, wait_for(smem_u32(b), parity, a.polls, failed));
                fence_after();
                return ok;
            };
            auto loaded = [&](const Place &w) { return arrived(&bars.full[w.at], w.turn); };
            for (int64_t u = u0; u < u1 && ok; ++run) {
                const int64_t g = u / a.tiles, t0 = u - g * a.tiles;
                const uint32_t tiles = (uint32_t)(min(a.tiles, t0 + (u1 - u)) - t0);
                const int live = (int)min((a.n_own - g * kTiles * kRows + kRows - 1) / kRows, (int64_t)kTiles);
                if (!arrived(&bars.own_full, run & 1)) break;
                if constexpr (!kSums) {
                    for (uint32_t i = 0; i < tiles && loaded(place); ++i) {
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            if (t >= live || !ok) break;
                            const uint32_t b = made_t[t] & 1;
                            if (!arrived(&bars.shares[t][b], (made_t[t] / 2 & 1) ^ 1)) break;
                            scores(t, place.at, b);
                            ++made_t[t];
                        }
                        if (!ok) break;
                        commit(&bars.free[place.at]);
                        place.next(a.stages);
                    }
                } else if constexpr (kBuffers == 1) {
                    if (!loaded(place)) break;
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
                        if (t < live) scores(t, place.at, 0);
                    for (uint32_t i = 0; i < tiles && ok; ++i) {
                        Place after = place;
                        after.next(a.stages);
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            if (t >= live || !ok) break;
                            if (!arrived(&bars.shares[t][0], made_t[t]++ & 1)) break;
                            sums(t, place.at, 0);
                            if (t == live - 1) commit(&bars.free[place.at]);
                            if (i + 1 == tiles) commit(&bars.sums[t]);
                            else if (t > 0 || loaded(after)) scores(t, after.at, 0);   // behind the products that read the shares in their place
                        }
                        place = after;
                    }
                } else {
                    if (!loaded(place)) break;
                    scores(0, place.at, made & 1);
                    for (uint32_t i = 0; i < tiles && ok; ++i, ++made) {
                        Place after = place;
                        after.next(a.stages);
                        if (i + 1 < tiles) {
                            if (!loaded(after)) break;
                            scores(0, after.at, (made + 1) & 1);     // behind the products of the tile before, which read that buffer
                        }
                        if (!arrived(&bars.shares[0][made & 1], made / 2 & 1)) break;
                        sums(0, place.at, made & 1);
                        commit(&bars.sums[0]);
                        commit(&bars.free[place.at]);
                        place = after;
                    }
                }
                if (ok) commit(&bars.own_free);
                u += tiles;
            }
        }
        __syncwarp();
    } else {
        if constexpr (kTiles == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int t = warp / 8, h = warp / 4 % 2;                    // tile of own rows, half of the other rows
        const uint32_t lanes = tmem + kSpan * t + ((uint32_t)(warp % 4) << 21);        // 32 lanes a warp
        const uint32_t sums_at = lanes + kSumsAt + kSumsWide * h;
        const int in_tile = 32 * (warp % 4) + lane;
        // from accumulated scores to units of log 2, and what undoes the scales of the sums
        const int e_own = image_exponent(a.words[a.own_word]), e_other = image_exponent(a.words[a.other_word]);
        const float unit = kLog2e * exp2f((float)-e_own) * exp2f((float)-e_other);
        const Two unit2 = two(unit, unit);
        uint32_t seen = 0, runs = 0;                                 // tiles and runs of these rows
        Place place;
        bool ok = true;
        auto arrived = [&](uint64_t *b, uint32_t parity) {           // for the whole warp or not at all
            ok = __all_sync(0xffffffffu, wait_for(smem_u32(b), parity, a.polls, failed));
            fence_after();
            return ok;
        };
        for (int64_t u = u0; u < u1 && ok;) {
            const int64_t g = u / a.tiles, t0 = u - g * a.tiles, t1 = min(a.tiles, t0 + (u1 - u));
            if ((g * kTiles + t) * kRows >= a.n_own) {
                if (PASS == kByColumns)
                    for (int64_t tile = t0; tile < t1; ++tile) place.next(a.stages);
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
                        tmem_load(sums_at + kPiece * c, o);
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
            for (int64_t tile = t0; tile < t1; ++tile, ++seen) {
                const uint32_t b = seen % kBuffers, s_at = lanes + 128 * b + kHalf * h;
                if (!arrived(&bars.scores[t][b], (seen / kBuffers) & 1)) break;
                float late = 1.f;
                const int valid = (int)min(a.n_other - tile * kTile - kHalf * h, (int64_t)kHalf);
                const float *vec = reinterpret_cast<const float *>(smem + (other_at - own_at) + place.at * stage_bytes + KT * other_term) + kHalf * h;
                if (PASS == kByColumns) {                            // base and pull came with the tile
                    if (!arrived(&bars.full[place.at], place.turn)) break;
                    place.next(a.stages);
                }
                Two part[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < kHalf / kStep; ++c) {
                    uint32_t s[kStep];
                    tmem_load(s_at + kStep * c, s);
                    tmem_landed(s);
                    if (PASS != kByColumns) {
                        if (valid < kHalf)
#pragma unroll
                            for (int j = 0; j < kStep; ++j)
                                if (kStep * c + j >= valid) s[j] = 0xff800000u;        // -inf
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
                                for (int k = 0; k < c * kStep / 16; ++k) {              // shares of this tile that are written already
                                    uint32_t p[16], w[8];
                                    tmem_stored();
                                    tmem_load(s_at + 16 * k, p);
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
                                    tmem_store(s_at + 16 * k, w);
                                    if (PT == 2) {
#pragma unroll
                                        for (int j = 0; j < 8; ++j) w[j] = p[j];
                                        tmem_store(s_at + 16 * k + 8, w);
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
                            tmem_store(s_at + kStep * c + 16 * k, hi);
                            if (PT == 2) tmem_store(s_at + kStep * c + 16 * k + 8, lo);
                        }
                    }
                }
                if (PASS != kByColumns) {
                    const float2 x = both(add2(part[0], part[1]));
                    total += x.x + x.y;
                }
                if (kSums) {
                    if (tile > t0) {                                 // O of the tile before, which the next product overwrites
                        if (kBuffers == 2 && !arrived(&bars.sums[t], (seen - 1) & 1)) break;
                        take(late);
                    }
                    tmem_stored();
                }
                fence_before();
                __syncwarp();
                if (lane == 0) arrive(smem_u32(&bars.shares[t][b]));
            }
            if (kSums && ok && arrived(&bars.sums[t], (kBuffers == 2 ? seen - 1 : runs) & 1)) take(1.f);
            ++runs;
            // Half 1 hands its sums to half 0 where O was: nothing writes there before the shares of half 1 in the next run.
            if (h == 1) {
                if constexpr (kSums) {
#pragma unroll
                    for (int c = 0; c < RP / 8; ++c) {
                        if (8 * c >= a.columns) break;
                        uint32_t w[8];
#pragma unroll
                        for (int r = 0; r < 8; ++r) w[r] = __float_as_uint(sum[8 * c + r]);
                        tmem_store(sums_at + 8 * c, w);
                    }
                    tmem_stored();
                }
                merged[t][in_tile] = make_float2(top, total);
                fence_before();
            }
            if (!ok) *(volatile int *)&gave_up[t] = 1;
            asm volatile("bar.sync %0, 256;" :: "r"(1 + t) : "memory");
            ok = *(volatile int *)&gave_up[t] == 0;                  // the same for both halves: both go on or neither
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
                        tmem_load(sums_at + kSumsWide + 16 * c, o);
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
    if (warp == kIssuer) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    if (threadIdx.x == 0 && failed_s) atomicExch(a.gave_up, 1u);
    start_next_kernel();
}

template <int RP, int PASS, int QT, int KT, int PT>
cudaError_t launch(TensorArgs a, int blocks, cudaStream_t stream) {
    constexpr int kMost = 224 * 1024;                                // of 227 KB: barriers and what halves exchange are apart
    const int own = tiles_of(RP) * QT * kRows * 2 * a.columns, stage = KT * kTile * 2 * a.columns + (PASS == kByColumns ? 8 * kTile : 0);
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
