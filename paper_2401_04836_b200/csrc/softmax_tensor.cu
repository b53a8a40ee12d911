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

constexpr int kGroups = 2;                       // tiles of own rows
constexpr int kRows = 128;                       // of a tile: lanes of tensor memory
constexpr int kLoader = 4 * kGroups, kIssuer = kLoader + 1;
constexpr int kThreads = 32 * (kIssuer + 1);
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
    uint64_t scores[kGroups][2];                 // S of a tile is complete (kLossAlone: two buffers)
    uint64_t shares[kGroups][2];                 // P of a tile is written (kLossAlone: S has been read)
    uint64_t sums[kGroups];                      // O of the last tile of a run is complete
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

// RP: room for sums in registers.  QT, KT: terms of own and other rows; PT: terms of a share (its product takes as many of Other).
template <int RP, int PASS, int QT, int KT, int PT, int TN>
__global__ void __launch_bounds__(kThreads, 1) loss_tensor(const __grid_constant__ TensorArgs a) {
    constexpr bool kSums = PASS != kLossAlone;
    constexpr int kBuffers = RP <= 64 ? 2 : 1;                       // of O in tensor memory, which S and O of two tiles share
    constexpr int kStep = RP <= 64 ? 32 : 16;                        // scores a thread has in registers at once
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ Barriers bars;
    __shared__ uint32_t tmem_at;
    __shared__ int failed_s;
    volatile int *failed = &failed_s;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t row_bytes = 2u * a.columns;
    const uint32_t own_term = kRows * row_bytes, other_term = TN * row_bytes;
    const uint32_t stage_bytes = KT * other_term + (PASS == kByColumns ? 8u * TN : 0u);
    const uint32_t own_at = smem_u32(smem), other_at = own_at + kGroups * QT * own_term;

    if (threadIdx.x == 0) {
        failed_s = 0;
        auto init = [](uint64_t *b, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_u32(b)), "r"(n) : "memory"); };
        init(&bars.own_full, 1);
        init(&bars.own_free, 1);
        for (int s = 0; s < kMaxStages; ++s) init(&bars.full[s], 1), init(&bars.free[s], 1);
        for (int t = 0; t < kGroups; ++t) {
            for (int b = 0; b < 2; ++b) init(&bars.scores[t][b], 1), init(&bars.shares[t][b], 4);
            init(&bars.sums[t], 1);
        }
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
    if (warp == kLoader) {
        if (lane == 0) {
            uint32_t n = 0, run = 0, held = 0;                       // tiles, runs and loads of own rows so far
            bool ok = true;
            for (int64_t u = u0; u < u1 && ok; ++run) {
                const int64_t g = u / a.tiles, t0 = u - g * a.tiles, t1 = min(a.tiles, t0 + (u1 - u));
                const int live = (g * kGroups + 1) * kRows < a.n_own ? 2 : 1;
                if (run && !(ok = wait_for(smem_u32(&bars.own_free), (run - 1) & 1, a.polls, failed))) break;
                const uint32_t bar = smem_u32(&bars.own_full);
                expect(bar, live * QT * own_term);
                ++held;
                for (int t = 0; t < live; ++t)
                    for (int q = 0; q < QT; ++q)
                        bulk_load(own_at + (t * QT + q) * own_term, (q ? a.own.lo : a.own.hi) + (g * kGroups + t) * kRows * a.columns, own_term, bar);
                for (int64_t t = t0; t < t1; ++t, ++n) {
                    const uint32_t s = n % a.stages;
                    if (n >= (uint32_t)a.stages && !(ok = wait_for(smem_u32(&bars.free[s]), (n / a.stages - 1) & 1, a.polls, failed))) break;
                    const uint32_t full = smem_u32(&bars.full[s]), to = other_at + s * stage_bytes;
                    expect(full, stage_bytes);
                    for (int q = 0; q < KT; ++q) bulk_load(to + q * other_term, (q ? a.other.lo : a.other.hi) + t * TN * a.columns, other_term, full);
                    if (PASS == kByColumns) {
                        bulk_load(to + KT * other_term, a.base + t * TN, 4 * TN, full);
                        bulk_load(to + KT * other_term + 4 * TN, a.pull + t * TN, 4 * TN, full);
                    }
                }
                u += t1 - t0;
            }
            // nothing of this block is under way when it ends, whatever the others did
            if (!ok) {
                if (held) mbar_wait(smem_u32(&bars.own_full), (held - 1) & 1, 1 << 14);
                for (uint32_t i = n > (uint32_t)a.stages ? n - a.stages : 0; i < n; ++i)
                    mbar_wait(smem_u32(&bars.full[i % a.stages]), (i / a.stages) & 1, 1 << 14);
            }
        }
        __syncwarp();
    } else if (warp == kIssuer) {
        if (elect_one()) {
            const uint32_t i_scores = idesc_f16(kRows, TN, false), i_sums = idesc_f16(kRows, a.columns, true);
            const uint32_t group_rows = 8 * row_bytes;               // bytes of 8 rows: 8 columns of them are 128 bytes
            const int deep = a.columns / 16;
            uint32_t n = 0, run = 0, made[kGroups] = {0, 0};
            // descriptors of the first 16 columns (scores) or rows (sums); further ones, terms and stages lie a constant apart
            const uint64_t own_k = smem_desc(own_at, 128, group_rows), other_k = smem_desc(other_at, 128, group_rows);
            const uint64_t other_mn = smem_desc(other_at, group_rows, 128);
            const uint32_t q_term = own_term >> 4, k_term = other_term >> 4, k_stage = stage_bytes >> 4, mn_step = (2 * group_rows) >> 4;
            auto scores = [&](int t, uint32_t i, uint32_t to) {
                if (a.withhold) return;
                const uint64_t q = own_k + t * QT * q_term, k = other_k + (i % a.stages) * k_stage;
                bool first = true;
                auto product = [&](uint64_t qa, uint64_t ka) {
#pragma unroll
                    for (int c = 0; c < RP / 16; ++c, first = false) {
                        if (c >= deep) break;
                        umma_f16(to, qa + c * 16, ka + c * 16, i_scores, first ? 0u : 1u);
                    }
                };
                if (QT == 2) product(q + q_term, k);
                if (KT == 2) product(q, k + k_term);
                product(q, k);
            };
            auto sums = [&](int t, uint32_t i, uint32_t p, uint32_t to) {
                if (a.withhold) return;
                const uint64_t k = other_mn + (i % a.stages) * k_stage;
                bool first = true;
                auto product = [&](uint32_t pa, uint64_t ka) {
#pragma unroll
                    for (int c = 0; c < TN / 16; ++c, first = false) umma_f16_ts(to, pa + c * 16, ka + c * mn_step, i_sums, first ? 0u : 1u);
                };
                if (PT == 2) {
                    product(p + 8, k);
                    product(p, k + k_term);
                }
                product(p, k);
            };
            auto commit = [&](uint64_t *b) { if (!a.withhold) umma_commit(smem_u32(b)); };
            bool ok = true;
            for (int64_t u = u0; u < u1 && ok; ++run) {
                const int64_t g = u / a.tiles, t0 = u - g * a.tiles;
                const uint32_t tiles = (uint32_t)(min(a.tiles, t0 + (u1 - u)) - t0);
                const int live = (g * kGroups + 1) * kRows < a.n_own ? 2 : 1;
                if (!(ok = wait_for(smem_u32(&bars.own_full), run & 1, a.polls, failed))) break;
                auto arrived = [&](uint32_t i) {
                    ok = wait_for(smem_u32(&bars.full[i % a.stages]), (i / a.stages) & 1, a.polls, failed);
                    fence_after();
                    return ok;
                };
                if (!kSums) {
                    for (uint32_t i = 0; i < tiles && arrived(n); ++i, ++n) {
                        for (int t = 0; t < live && ok; ++t) {
                            const uint32_t b = made[t] & 1, turn = made[t] / 2;
                            if (turn) ok = wait_for(smem_u32(&bars.shares[t][b]), (turn - 1) & 1, a.polls, failed);
                            if (!ok) break;
                            fence_after();
                            scores(t, n, tmem + 256 * t + 128 * b);
                            commit(&bars.scores[t][b]);
                            ++made[t];
                        }
                        if (ok) commit(&bars.free[n % a.stages]);
                    }
                } else {
                    if (!arrived(n)) break;
                    for (int t = 0; t < live; ++t) {
                        scores(t, n, tmem + 256 * t);
                        commit(&bars.scores[t][0]);
                    }
                    for (uint32_t i = 0; i < tiles && ok; ++i, ++n) {
                        for (int t = 0; t < live; ++t) {
                            if (!(ok = wait_for(smem_u32(&bars.shares[t][0]), made[t] & 1, a.polls, failed))) break;
                            fence_after();
                            sums(t, n, tmem + 256 * t, tmem + 256 * t + 128 + (made[t] % kBuffers) * 64);
                            ++made[t];
                            if (t == live - 1) commit(&bars.free[n % a.stages]);
                            if (i + 1 == tiles) {
                                commit(&bars.sums[t]);
                            } else {
                                if (t == 0 && !arrived(n + 1)) break;
                                scores(t, n + 1, tmem + 256 * t);   // behind the product that reads the shares in its place
                                commit(&bars.scores[t][0]);
                            }
                        }
                    }
                }
                if (ok) commit(&bars.own_free);
                u += tiles;
            }
        }
        __syncwarp();
    } else {
        const int t = warp / 4;
        const uint32_t mine = tmem + 256 * t + ((uint32_t)(warp % 4) << 21);           // 32 lanes a warp
        const int row = kRows * t + 32 * (warp % 4) + lane;
        // from accumulated scores to units of log 2, and what undoes the scales of the sums
        const int e_own = image_exponent(a.words[a.own_word]), e_other = image_exponent(a.words[a.other_word]);
        const float unit = kLog2e * exp2f((float)-e_own) * exp2f((float)-e_other);
        uint32_t run = 0, seen = 0, turns = 0;                                         // runs and tiles of this row tile; turns: tiles of all
        bool ok = true;
        for (int64_t u = u0; u < u1 && ok;) {
            const int64_t g = u / a.tiles, t0 = u - g * a.tiles, t1 = min(a.tiles, t0 + (u1 - u));
            const bool live = (g * kGroups + t) * kRows < a.n_own;
            if (!live) {
                turns += (uint32_t)(t1 - t0);
                u += t1 - t0;
                continue;
            }
            float top = -INFINITY, total = 0.f;
            float sum[kSums ? RP : 1];
#pragma unroll
            for (int r = 0; r < (kSums ? RP : 1); ++r) sum[r] = 0.f;
            auto take = [&](uint32_t buffer, float late) {                             // adds O of a tile, made from shares `late` times too large
#pragma unroll
                for (int c = 0; c < RP / 16; ++c) {
                    if (16 * c >= a.columns) break;
                    uint32_t o[16];
                    tmem_load(mine + 128 + 64 * buffer + 16 * c, o);
                    tmem_landed(o);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if constexpr (kSums) sum[16 * c + r] = PASS == kByRows ? fmaf(late, __uint_as_float(o[r]), sum[16 * c + r]) : sum[16 * c + r] + __uint_as_float(o[r]);
                }
            };
            auto arrived = [&](uint64_t *b, uint32_t parity) {                         // for the whole warp or not at all
                ok = __all_sync(0xffffffffu, wait_for(smem_u32(b), parity, a.polls, failed));
                fence_after();
                return ok;
            };
            for (int64_t tile = t0; tile < t1; ++tile, ++seen, ++turns) {
                const uint32_t b = kSums ? 0 : seen & 1, s_at = mine + 128 * b;
                if (!arrived(&bars.scores[t][b], kSums ? seen & 1 : (seen / 2) & 1)) break;
                float late = 1.f;
                // the products of the tile before are complete too: they were issued in front of these scores
                if (kSums && kBuffers == 1 && tile > t0) take(0, 1.f);
                const int valid = (int)min(a.n_other - tile * TN, (int64_t)TN);
                const float *vec = reinterpret_cast<const float *>(smem + (other_at - own_at) + (turns % a.stages) * stage_bytes + KT * other_term);
                if (PASS == kByColumns && !arrived(&bars.full[turns % a.stages], (turns / a.stages) & 1)) break;   // base and pull came with the tile
                float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < TN / kStep; ++c) {
                    uint32_t s[kStep];
                    tmem_load(s_at + kStep * c, s);
                    tmem_landed(s);
                    if (PASS != kByColumns) {
                        if (valid < TN)
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
                            for (int q = 0; q < 4; ++q) part[q] *= keep;
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
                    const float base = (PASS == kLossAlone ? 0.f : (float)kShift) - top;
#pragma unroll
                    for (int k = 0; k < kStep / 16; ++k) {
                        uint32_t hi[8], lo[8];
#pragma unroll
                        for (int j = 0; j < 8; j += 2) {
                            float p[4];
                            const int at = 16 * k + 2 * j;
                            if (PASS == kByColumns) {
                                const float4 bs = *reinterpret_cast<const float4 *>(vec + kStep * c + at);
                                const float4 pl = *reinterpret_cast<const float4 *>(vec + TN + kStep * c + at);
                                p[0] = exp2_fast(fmaf(__uint_as_float(s[at]), unit, -bs.x)) * pl.x;
                                p[1] = exp2_fast(fmaf(__uint_as_float(s[at + 1]), unit, -bs.y)) * pl.y;
                                p[2] = exp2_fast(fmaf(__uint_as_float(s[at + 2]), unit, -bs.z)) * pl.z;
                                p[3] = exp2_fast(fmaf(__uint_as_float(s[at + 3]), unit, -bs.w)) * pl.w;
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    p[i] = exp2_fast(fmaf(__uint_as_float(s[at + i]), unit, base));
                                    part[i] += p[i];
                                }
                            }
                            if (!kSums) continue;
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                hi[j + i] = pack(p[2 * i], p[2 * i + 1]);
                                if (PT == 2) {
                                    const float2 h = unpack(hi[j + i]);
                                    lo[j + i] = pack(p[2 * i] - h.x, p[2 * i + 1] - h.y);
                                }
                            }
                        }
                        if (kSums) {
                            tmem_store(s_at + kStep * c + 16 * k, hi);
                            if (PT == 2) tmem_store(s_at + kStep * c + 16 * k + 8, lo);
                        }
                    }
                }
                if (kSums) tmem_stored();
                fence_before();
                __syncwarp();
                if (lane == 0) arrive(smem_u32(&bars.shares[t][b]));
                total += (part[0] + part[1]) + (part[2] + part[3]);
                if (kSums && kBuffers == 2 && tile > t0) take((seen - 1) & 1, late);
            }
            if (ok && kSums && arrived(&bars.sums[t], run++ & 1)) take(kBuffers == 2 ? (seen - 1) & 1 : 0, 1.f);
            const int64_t part = (g * a.parts + ((int64_t)blockIdx.x - g * a.tiles / a.each)) * (kGroups * kRows) + row;
            if (ok) {
                const float shift = PASS == kByRows ? 1.f / (1 << kShift) : 1.f;
                if (PASS != kByColumns) {
                    a.top[part] = top;
                    a.total[part] = total * shift;
                }
                if (kSums) {
                    const float undo = exp2f((float)-e_other) * shift;
                    float undo2 = 1.f;
                    if (PASS == kByColumns) undo2 = exp2f((float)-image_exponent(a.words[kMaxWeight]));
                    float4 *to = reinterpret_cast<float4 *>(a.sum + part * a.width);
#pragma unroll
                    for (int c = 0; c < RP / 4; ++c)
                        if (4 * c < a.columns)
                            to[c] = make_float4(sum[4 * c] * undo * undo2, sum[4 * c + 1] * undo * undo2, sum[4 * c + 2] * undo * undo2, sum[4 * c + 3] * undo * undo2);
                }
            }
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

template <int RP, int PASS, int QT, int KT, int PT, int TN>
cudaError_t launch(TensorArgs a, int blocks, cudaStream_t stream) {
    constexpr int kMost = 226 * 1024;                                // of 227 KB: the barriers are apart
    const int own = kGroups * QT * kRows * 2 * a.columns, stage = KT * TN * 2 * a.columns + (PASS == kByColumns ? 8 * TN : 0);
    a.stages = std::min<int>(kMaxStages, (kMost - own) / stage);
    const int bytes = own + a.stages * stage;
    static PerDeviceOnce once;
    const cudaError_t e = once_per_device(once, [] {
        return cudaFuncSetAttribute(loss_tensor<RP, PASS, QT, KT, PT, TN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    });
    if (e != cudaSuccess) return e;
    return launch_early(loss_tensor<RP, PASS, QT, KT, PT, TN>, dim3(blocks), kThreads, bytes, stream, a);
}

template <int RP, int TN, bool WIDE>
cudaError_t by_pass(int pass, const TensorArgs &a, int blocks, cudaStream_t stream) {
    constexpr int PT = WIDE ? 2 : 1;
    if (pass == kLossAlone) return launch<RP, kLossAlone, 2, WIDE ? 2 : 1, PT, TN>(a, blocks, stream);
    if (pass == kByRows) return launch<RP, kByRows, 2, WIDE ? 2 : 1, PT, TN>(a, blocks, stream);
    return launch<RP, kByColumns, WIDE ? 2 : 1, 2, PT, TN>(a, blocks, stream);
}

template <bool WIDE>
cudaError_t by_rank(int pass, const TensorArgs &a, int blocks, cudaStream_t stream) {
    if (a.columns <= 16) return by_pass<16, 128, WIDE>(pass, a, blocks, stream);
    if (a.columns <= 32) return by_pass<32, 128, WIDE>(pass, a, blocks, stream);
    if (a.columns <= 64) return by_pass<64, 128, WIDE>(pass, a, blocks, stream);
    return by_pass<128, WIDE ? 64 : 128, WIDE>(pass, a, blocks, stream);
}

}  // namespace

// Tiles of 128 other rows, or of 64 where 256 own rows of two terms leave no room for two of 128.
int tensor_tile(int rank, bool wide) { return wide && image_columns(rank) > 64 ? 64 : 128; }

cudaError_t tensor_pass(int pass, bool wide, const TensorArgs &a, int blocks, cudaStream_t stream) {
    return wide ? by_rank<true>(pass, a, blocks, stream) : by_rank<false>(pass, a, blocks, stream);
}

}  // namespace loss
}  // namespace cb
