// Differential attention, gradients on the tensor cores: bf16, head dim 64 or 128.  With P_c the two maps (recomputed from
// the scores and their saved log-sum-exp), dA = dO V^T and d_c = <dO, P_c V> row by row:
//
//     dV = (P_1 - lambda P_2)^T dO      dS_1 = P_1 o (dA - d_1)      dS_2 = -lambda P_2 o (dA - d_2)
//     dQ_c = scale dS_c K_c             dK_c = scale dS_c^T Q_c      dlambda = -sum P_2 o dA
//
// dA and dV are shared by the maps, so a visible pair costs 10 D multiply-adds.  Two kernels that each recompute the maps:
// one walks the keys of a query tile (dQ, dlambda: 6 D... of scores, dA and dQ), one the queries of a key block (dK, dV).
// A single kernel would save the second recomputation, but every dQ would be summed over key blocks by atomics in fp32
// (order not fixed, 2 x 4 bytes per element and key block) and P, dS would have to go through shared memory twice, whose
// bandwidth the operand reads already fill; here every sum has one place and one order, and the weights are operands
// from tensor memory.
//
// Both run as two chains of 64-wide half tiles that alternate on the tensor pipe, each with a warpgroup of its own: one
// chain's exponentials run under the other chain's products.  One CTA per SM, persistent; warp 0 loads (TMA), warp 1
// issues the MMAs in a fixed order.  Every wait is bounded; on expiry the CTA raises a flag that ends all roles, lets
// its copies land, frees its tensor memory and returns.
#include "ta_diff_tc.cuh"

namespace ta {
namespace {

constexpr int kThreads = 384;
constexpr int kRows = 128, kHalf = 64;

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

struct BwdArgs {
    int B, H, H_kv, g, Nq, Nk, causal;
    int tiles, tile_major;         // query tiles / key blocks per head
    int gi, hsplit;                // dK, dV: query heads per item, items per (key block, KV head)
    long long total_items, prow;
    float scale, scale_log2;
    const int *q_lens, *kv_lens;
    const float *lambda;
    int lambda_count;
    const float4 *stats;
    __nv_bfloat16 *dq, *dk, *dv;
    float *part, *dlam_part;
    long long kv_elems;
};

__device__ __forceinline__ long long item_of_round(const BwdArgs &a, long long k) {
    const long long g = gridDim.x, b = blockIdx.x;
    const long long item = k * g + ((k & 1) ? g - 1 - b : b);
    return item < a.total_items ? item : -1;
}

// Remembers the copies a producer has started, so that they can be waited for when it gives up.
struct Armed {
    uint32_t mask = 0, par = 0;
    __device__ __forceinline__ void arm(int bar, uint32_t parity) {
        mask |= 1u << bar;
        par = parity ? (par | 1u << bar) : (par & ~(1u << bar));
    }
    __device__ __forceinline__ void drain(uint32_t bar0, int bars) const {
        const unsigned long long t0 = globaltimer_ns();
        for (int i = 0; i < bars; ++i) {
            if (!(mask & (1u << i))) continue;
            while (!mbar_try_wait(bar0 + 8u * (uint32_t)i, (par >> i) & 1u) && globaltimer_ns() - t0 < 10000000ull) {
            }
        }
    }
};

// ------------------------------------------------------------------ dQ and dlambda: one query tile, all its keys

template <int D>
struct DqCfg {
    static constexpr int kSlabs = D / 64, kd = D / 2;
    static constexpr uint32_t kSlab = kRows * 128, kTile = kSlabs * kSlab;
    static constexpr int kNKV = D == 128 ? 2 : 4;
    static constexpr uint32_t kOffQ = 0, kOffG = kTile, kOffK = 2 * kTile, kOffV = kOffK + kNKV * kTile;
    static constexpr uint32_t kOffBar = kOffV + kNKV * kTile;
    static constexpr int kNumBars = 2 + 3 * kNKV + 6;
    static constexpr uint32_t kSmem = kOffBar + kNumBars * 8 + 16 + 1024;
    // per chain (64 keys): S_1, S_2 (dS_c over their first 32 columns), dA; then dQ
    static constexpr uint32_t kColChain = 192, kColDQ = 384;
};

struct DqItem {
    int b, h, hk, t0, tile;
    DiffSpan sp;
    int keys_end, nhalf;
};
__device__ __forceinline__ DqItem decode_dq(const BwdArgs &a, long long item) {
    DqItem c;
    long long bh;
    const long long heads = (long long)a.B * a.H;
    if (a.tile_major) {
        c.tile = a.tiles - 1 - (int)(item / heads);
        bh = item % heads;
    } else {
        c.tile = a.tiles - 1 - (int)(item % a.tiles);
        bh = item / a.tiles;
    }
    c.b = (int)(bh / a.H);
    c.h = (int)(bh - (long long)c.b * a.H);
    c.hk = c.h / a.g;
    c.t0 = c.tile * kRows;
    c.sp = diff_span(a.q_lens, a.kv_lens, c.b, a.Nq, a.Nk);
    const int last = min(c.t0 + kRows, c.sp.ql) - 1;
    c.keys_end = last >= c.t0 ? c.sp.keys(last, a.causal) : 0;
    c.nhalf = (c.keys_end + kHalf - 1) / kHalf;
    return c;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
diff_tc_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_g,
                  const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ BwdArgs a) {
    using C = DqCfg<D>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t s0 = smem_u32(smem);
    const uint32_t sQ = s0 + C::kOffQ, sG = s0 + C::kOffG;
    auto sK = [&](int i) { return s0 + C::kOffK + (uint32_t)i * C::kTile; };
    auto sV = [&](int i) { return s0 + C::kOffV + (uint32_t)i * C::kTile; };
    const uint32_t bar0 = s0 + C::kOffBar;
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
    // barriers 0 .. 2 kNKV are those copies complete on
    const uint32_t q_full = bar(0);
    auto k_full = [&](int i) { return bar(1 + i); };
    auto v_full = [&](int i) { return bar(1 + C::kNKV + i); };
    auto kv_free = [&](int i) { return bar(1 + 2 * C::kNKV + i); };
    constexpr int kB = 1 + 3 * C::kNKV;
    const uint32_t q_free = bar(kB);
    auto s_full = [&](int c) { return bar(kB + 1 + c); };      // S_1, S_2, dA of chain c complete
    auto ds_full = [&](int c) { return bar(kB + 3 + c); };     // dS_1, dS_2 of chain c written (4 warps)
    const uint32_t dq_full = bar(kB + 5), dq_free = bar(kB + 6);
    uint32_t *tmem_slot = (uint32_t *)(smem + C::kOffBar + C::kNumBars * 8);
    volatile uint32_t *abort_flag = tmem_slot + 1;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < C::kNumBars; ++i) mbar_init(bar(i), i == kB + 3 || i == kB + 4 ? 4 : i == kB + 6 ? 8 : 1);
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp == 0) {
        // =============================================================== TMA producer
        if (lane == 0) {
            uint32_t ic = 0, g = 0;
            Armed armed;
            bool ok = true;
            for (long long round = 0; ok && round * gridDim.x < a.total_items; ++round) {
                const long long item = item_of_round(a, round);
                if (item < 0) continue;
                const DqItem c = decode_dq(a, item);
                if (c.nhalf == 0) continue;
                ok = mbar_wait_abortable(q_free, (ic & 1) ^ 1, 0x110, abort_flag);
                if (!ok) break;
                mbar_expect_tx(q_full, 2 * C::kTile);
                armed.arm(0, ic & 1);
                ++ic;
#pragma unroll
                for (int s = 0; s < C::kSlabs; ++s) {
                    tma_load_5d(sQ + s * C::kSlab, &map_q, q_full, 64 * s, c.t0, 0, c.h, c.b);
                    tma_load_5d(sG + s * C::kSlab, &map_g, q_full, 64 * s, c.t0, 0, c.h, c.b);
                }
                for (int j = 0; 2 * j < c.nhalf; ++j, ++g) {
                    const int st = g % C::kNKV;
                    const uint32_t par = (g / C::kNKV) & 1;
                    ok = mbar_wait_abortable(kv_free(st), par ^ 1, 0x111, abort_flag);
                    if (!ok) break;
                    mbar_expect_tx(k_full(st), C::kTile);
                    armed.arm(1 + st, par);
#pragma unroll
                    for (int s = 0; s < C::kSlabs; ++s)
                        tma_load_5d(sK(st) + s * C::kSlab, &map_k, k_full(st), 64 * s, kRows * j, 0, c.hk, c.b);
                    mbar_expect_tx(v_full(st), C::kTile);
                    armed.arm(1 + C::kNKV + st, par);
#pragma unroll
                    for (int s = 0; s < C::kSlabs; ++s)
                        tma_load_5d(sV(st) + s * C::kSlab, &map_v, v_full(st), 64 * s, kRows * j, 0, c.hk, c.b);
                }
            }
            if (!ok) armed.drain(bar0, 1 + 2 * C::kNKV);
        }
    } else if (warp == 1) {
        // =============================================================== MMA issuer
        constexpr uint32_t idesc_s = instr_desc(kHalf, 0);
        constexpr uint32_t idesc_q = instr_desc(C::kd, 1);
        uint32_t ic = 0, g0 = 0, sc[2] = {0, 0};     // items, key blocks before this item, half tiles of each chain
        bool ok = true;
        // S_1, S_2, dA of half tile i of the item (keys 64 i ..)
        auto scores = [&](const DqItem &c, int i) {
            const uint32_t g = g0 + (uint32_t)(i >> 1);
            const int st = g % C::kNKV, ch = i & 1;
            bool fine = true;
            if (ch == 0) {
                fine = warp_wait(k_full(st), (g / C::kNKV) & 1, 0x120, abort_flag);
                if (fine) fine = warp_wait(v_full(st), (g / C::kNKV) & 1, 0x121, abort_flag);
                if (!fine) return false;
                // keys the tensor has but the call does not count: they meet dS = 0 in the product for dQ
                if (c.sp.kl < a.Nk && c.sp.kl < kRows * (i >> 1) + kRows) {
                    zero_rows(sK(st), C::kSlab, C::kSlabs, c.sp.kl - kRows * (i >> 1), kRows);
                    fence_proxy_async_smem();
                    __syncwarp();
                }
            }
            tc_fence_after();
            if (lane == 0) {
                const uint32_t rows = (uint32_t)ch * kHalf * 128u;
                const uint32_t col = tmem_base + ch * C::kColChain;
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int kb = 0; kb < C::kd / 16; ++kb) {
                        const uint32_t off = map_k_off<D>(m, kb, C::kSlab);
                        tc_mma_ss(col + 64 * m, smem_desc_sw128(sQ + off, 16, 1024), smem_desc_sw128(sK(st) + rows + off, 16, 1024),
                                  idesc_s, kb > 0);
                    }
#pragma unroll
                for (int kb = 0; kb < D / 16; ++kb) {
                    const uint32_t off = (kb >> 2) * C::kSlab + (kb & 3) * 32;
                    tc_mma_ss(col + 128, smem_desc_sw128(sG + off, 16, 1024), smem_desc_sw128(sV(st) + rows + off, 16, 1024), idesc_s,
                              kb > 0);
                }
                tc_commit(s_full(ch));
            }
            __syncwarp();
            return true;
        };
        for (long long round = 0; ok && round * gridDim.x < a.total_items; ++round) {
            const long long item = item_of_round(a, round);
            if (item < 0) continue;
            const DqItem c = decode_dq(a, item);
            if (c.nhalf == 0) continue;
            ok = warp_wait(q_full, ic & 1, 0x122, abort_flag);
            if (ok) ok = scores(c, 0);
            if (ok && c.nhalf > 1) ok = scores(c, 1);
            for (int i = 0; ok && i < c.nhalf; ++i) {
                const int ch = i & 1;
                const uint32_t g = g0 + (uint32_t)(i >> 1);
                const int st = g % C::kNKV;
                ok = warp_wait(ds_full(ch), sc[ch] & 1, 0x123, abort_flag);
                ++sc[ch];
                if (ok && i == 0) ok = warp_wait(dq_free, (ic & 1) ^ 1, 0x124, abort_flag);
                if (!ok) break;
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t col = tmem_base + ch * C::kColChain;
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int kb = 0; kb < kHalf / 16; ++kb)
                            tc_mma_ts(tmem_base + C::kColDQ + m * C::kd, col + 64 * m + 8 * kb,
                                      smem_desc_sw128(sK(st) + map_n_off<D>(m, C::kSlab) + (uint32_t)(ch * kHalf + 16 * kb) * 128u,
                                                      C::kSlab, 1024),
                                      idesc_q, (kb > 0 || i > 0) ? 1u : 0u);
                    if (ch == 1 || i + 1 == c.nhalf) tc_commit(kv_free(st));
                    if (i + 1 == c.nhalf) {
                        tc_commit(dq_full);
                        tc_commit(q_free);
                    }
                }
                __syncwarp();
                if (i + 2 < c.nhalf) ok = scores(c, i + 2);
            }
            g0 += (uint32_t)((c.nhalf + 1) >> 1);
            ++ic;
        }
    } else if (warp >= 4) {
        // =============================================================== weights, dS, epilogue
        const int ch = (warp - 4) >> 2, wq = warp & 3;
        const uint32_t tmem_lane = tmem_base + ((uint32_t)(wq * 32) << 16);
        const uint32_t col = tmem_lane + ch * C::kColChain;
        const int r = wq * 32 + lane;
        bool ok = true;
        uint32_t ic = 0, sc = 0;
        for (long long round = 0; ok && round * gridDim.x < a.total_items; ++round) {
            const long long item = item_of_round(a, round);
            if (item < 0) continue;
            const DqItem c = decode_dq(a, item);
            const int t = c.t0 + r;
            const int row_keys = c.sp.keys(t, a.causal);
            const long long bh = (long long)c.b * a.H + c.h;
            const float4 st = __ldg(a.stats + bh * a.prow + t);       // (rows are padded to whole tiles)
            const float2 sl2 = make_float2(a.scale_log2, a.scale_log2);
            const float2 n1 = make_float2(-st.x, -st.x), n2 = make_float2(-st.y, -st.y);
            const float2 d1 = make_float2(-st.z, -st.z), d2 = make_float2(-st.w, -st.w);
            float2 dl = make_float2(0.f, 0.f);
            for (int i = ch; i < c.nhalf; i += 2, ++sc) {
                ok = warp_wait(s_full(ch), sc & 1, 0x130, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const int c_hi = row_keys - kHalf * i;
                const bool whole = __all_sync(0xffffffffu, c_hi >= kHalf);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    uint32_t x1[32], x2[32], y[32];
                    tmem_ld32_nowait(col + 32 * q, x1);
                    tmem_ld32_nowait(col + 64 + 32 * q, x2);
                    tmem_ld32_nowait(col + 128 + 32 * q, y);
                    tmem_ld_wait();
                    if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (32 * q + e >= c_hi) {
                                x1[e] = x2[e] = 0xFF800000u;
                                y[e] = 0u;
                            }
                    }
                    uint32_t p1[16], p2[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float2 w1 = fma2(make_float2(__uint_as_float(x1[2 * e]), __uint_as_float(x1[2 * e + 1])), sl2, n1);
                        float2 w2 = fma2(make_float2(__uint_as_float(x2[2 * e]), __uint_as_float(x2[2 * e + 1])), sl2, n2);
                        w1.x = fast_exp2(w1.x);
                        w1.y = fast_exp2(w1.y);
                        w2.x = fast_exp2(w2.x);
                        w2.y = fast_exp2(w2.y);
                        const float2 da = make_float2(__uint_as_float(y[2 * e]), __uint_as_float(y[2 * e + 1]));
                        dl = fma2(w2, da, dl);
                        w1 = mul2(w1, add2(da, d1));
                        w2 = mul2(w2, add2(da, d2));
                        p1[e] = pack_bf16x2(w1.x, w1.y);
                        p2[e] = pack_bf16x2(w2.x, w2.y);
                    }
                    tmem_st16(col + 16 * q, p1);
                    tmem_st16(col + 64 + 16 * q, p2);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(ds_full(ch));
            }
            if (!ok) break;
            // this warp's share of sum P_2 o dA
            float s = dl.x + dl.y;
#pragma unroll
            for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
            if (lane == 0) a.dlam_part[(bh * a.tiles + c.tile) * 8 + (warp - 4)] = s;
            // dQ of one map per warpgroup; -lambda and the scale are applied here, in fp32
            if (c.nhalf > 0) {
                ok = warp_wait(dq_full, ic & 1, 0x131, abort_flag);
                ++ic;
                if (!ok) break;
                tc_fence_after();
            }
            const float f = ch ? -a.scale * __ldg(a.lambda + (a.lambda_count > 1 ? c.h : 0)) : a.scale;
            __nv_bfloat16 *dst = a.dq + (bh * a.Nq + t) * D + ch * C::kd;
#pragma unroll 1
            for (int i = 0; i < C::kd / 32; ++i) {
                uint32_t v[32];
                tmem_ld32(tmem_lane + C::kColDQ + ch * C::kd + 32 * i, v);
                if (t >= a.Nq) continue;
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        w[k] = row_keys > 0 ? pack_bf16x2(__uint_as_float(v[e + 2 * k]) * f, __uint_as_float(v[e + 2 * k + 1]) * f) : 0u;
                    *reinterpret_cast<uint4 *>(dst + 32 * i + e) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (c.nhalf > 0 && lane == 0) mbar_arrive(dq_free);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 3) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

// ------------------------------------------------------------------ dK, dV: one key block, all query rows that see it
//
// Scores transposed (rows: keys, columns: 64 query rows), so that P^T and dS^T are operands from tensor memory.  Per chain
// two slots of 64 columns: X takes S_1, then dA, then dS_2; Y takes S_2, then P_1 - lambda P_2 and dS_1.

template <int D>
struct DkvCfg {
    static constexpr int kSlabs = D / 64, kd = D / 2;
    static constexpr uint32_t kSlab = kRows * 128, kTile = kSlabs * kSlab;        // K, V block
    static constexpr uint32_t kQSlab = kHalf * 128, kQTile = kSlabs * kQSlab;     // Q, dO step
    static constexpr int kStages = 4;
    static constexpr uint32_t kStat = kHalf * 16;
    static constexpr uint32_t kOffK = 0, kOffV = kTile, kOffQ = 2 * kTile, kOffG = kOffQ + kStages * kQTile;
    static constexpr uint32_t kOffStat = kOffG + kStages * kQTile;
    static constexpr uint32_t kOffBar = kOffStat + kStages * kStat;
    static constexpr int kNumBars = 1 + kStages + kStages + 1 + 2 + 2 + 2 + 2 + 2;
    static constexpr uint32_t kSmem = kOffBar + kNumBars * 8 + 16 + 1024;
    static constexpr uint32_t kColDV = 256, kColDK = 384;
};

struct DkvItem {
    int b, hk, h0, hs, u0;
    DiffSpan sp;
    int t_lo, per_head, n;        // first query row (a multiple of 64), steps per head, steps of the item
};
__device__ __forceinline__ DkvItem decode_dkv(const BwdArgs &a, long long item) {
    DkvItem c;
    // earlier (longer, when causal) key blocks first
    const long long per_tile = a.total_items / a.tiles;
    int tile;
    long long rest;
    if (a.tile_major) {
        tile = (int)(item / per_tile);
        rest = item % per_tile;
    } else {
        tile = (int)(item % a.tiles);
        rest = item / a.tiles;
    }
    c.hs = (int)(rest % a.hsplit); rest /= a.hsplit;
    c.hk = (int)(rest % a.H_kv);
    c.b = (int)(rest / a.H_kv);
    c.h0 = c.hk * a.g + c.hs * a.gi;
    c.u0 = tile * kRows;
    c.sp = diff_span(a.q_lens, a.kv_lens, c.b, a.Nq, a.Nk);
    c.t_lo = a.causal ? max(0, c.u0 - c.sp.off) / kHalf * kHalf : 0;
    c.per_head = c.u0 < c.sp.kl && c.t_lo < c.sp.ql ? (c.sp.ql - c.t_lo + kHalf - 1) / kHalf : 0;
    c.n = c.per_head * a.gi;
    return c;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
diff_tc_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_g,
                   const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ BwdArgs a) {
    using C = DkvCfg<D>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t s0 = smem_u32(smem);
    const uint32_t sK = s0 + C::kOffK, sV = s0 + C::kOffV;
    auto sQ = [&](int i) { return s0 + C::kOffQ + (uint32_t)i * C::kQTile; };
    auto sG = [&](int i) { return s0 + C::kOffG + (uint32_t)i * C::kQTile; };
    const uint32_t bar0 = s0 + C::kOffBar;
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
    // barriers 0 .. kStages are those copies complete on
    const uint32_t kv_full = bar(0);
    auto q_full = [&](int i) { return bar(1 + i); };
    auto q_free = [&](int i) { return bar(1 + C::kStages + i); };      // (products read it, then 4 warps its statistics)
    constexpr int kB = 1 + 2 * C::kStages;
    const uint32_t kv_free = bar(kB);
    auto s_full = [&](int c) { return bar(kB + 1 + c); };      // S_1, S_2 of chain c complete
    auto s_read = [&](int c) { return bar(kB + 3 + c); };      // and read into registers (4 warps)
    auto dp_full = [&](int c) { return bar(kB + 5 + c); };     // dA of chain c complete
    auto ds_full = [&](int c) { return bar(kB + 7 + c); };     // weights and dS of chain c written (4 warps)
    const uint32_t acc_full = bar(kB + 9), acc_free = bar(kB + 10);
    uint32_t *tmem_slot = (uint32_t *)(smem + C::kOffBar + C::kNumBars * 8);
    volatile uint32_t *abort_flag = tmem_slot + 1;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < C::kNumBars; ++i) {
            const int k = i - kB;
            mbar_init(bar(i), k == 3 || k == 4 || k == 7 || k == 8 ? 4 : k == 10 ? 8 : 1);
        }
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp < 4) {
        if (warp == 0) {
            // =========================================================== TMA producer
            if (lane == 0) {
                uint32_t ic = 0, g = 0;
                Armed armed;
                bool ok = true;
                for (long long round = 0; ok && round * gridDim.x < a.total_items; ++round) {
                    const long long item = item_of_round(a, round);
                    if (item < 0) continue;
                    const DkvItem c = decode_dkv(a, item);
                    if (c.n == 0) continue;
                    ok = mbar_wait_abortable(kv_free, (ic & 1) ^ 1, 0x210, abort_flag);
                    if (!ok) break;
                    mbar_expect_tx(kv_full, 2 * C::kTile);
                    armed.arm(0, ic & 1);
                    ++ic;
#pragma unroll
                    for (int s = 0; s < C::kSlabs; ++s) {
                        tma_load_5d(sK + s * C::kSlab, &map_k, kv_full, 64 * s, c.u0, 0, c.hk, c.b);
                        tma_load_5d(sV + s * C::kSlab, &map_v, kv_full, 64 * s, c.u0, 0, c.hk, c.b);
                    }
                    for (int i = 0; i < c.n; ++i, ++g) {
                        const int st = g % C::kStages;
                        const uint32_t par = (g / C::kStages) & 1;
                        const int h = c.h0 + i / c.per_head, t0 = c.t_lo + kHalf * (i % c.per_head);
                        ok = mbar_wait_abortable(q_free(st), par ^ 1, 0x211, abort_flag);
                        if (!ok) break;
                        mbar_expect_tx(q_full(st), 2 * C::kQTile + C::kStat);
                        armed.arm(1 + st, par);
#pragma unroll
                        for (int s = 0; s < C::kSlabs; ++s) {
                            tma_load_5d(sQ(st) + s * C::kQSlab, &map_q, q_full(st), 64 * s, t0, 0, h, c.b);
                            tma_load_5d(sG(st) + s * C::kQSlab, &map_g, q_full(st), 64 * s, t0, 0, h, c.b);
                        }
                        // (the statistics are padded to whole tiles of rows)
                        bulk_load(s0 + C::kOffStat + st * C::kStat, a.stats + ((long long)c.b * a.H + h) * a.prow + t0, C::kStat,
                                  q_full(st));
                    }
                }
                if (!ok) armed.drain(bar0, 1 + C::kStages);
            }
        } else if (warp == 1) {
            // =========================================================== MMA issuer
            constexpr uint32_t idesc_s = instr_desc(kHalf, 0);
            constexpr uint32_t idesc_v = instr_desc(D, 1);
            constexpr uint32_t idesc_k = instr_desc(C::kd, 1);
            uint32_t ic = 0, g0 = 0, sr[2] = {0, 0}, sd[2] = {0, 0};
            bool ok = true;
            auto scores = [&](const DkvItem &c, int i) {
                const uint32_t g = g0 + (uint32_t)i;
                const int st = g % C::kStages, ch = i & 1;
                if (!warp_wait(q_full(st), (g / C::kStages) & 1, 0x220, abort_flag)) return false;
                const int t0 = c.t_lo + kHalf * (i % c.per_head);
                // rows the tensors have but the call does not count: they meet weights of 0 in the products for dK, dV
                if (c.sp.ql < a.Nq && c.sp.ql < t0 + kHalf) {
                    zero_rows(sQ(st), C::kQSlab, C::kSlabs, c.sp.ql - t0, kHalf);
                    zero_rows(sG(st), C::kQSlab, C::kSlabs, c.sp.ql - t0, kHalf);
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                tc_fence_after();
                if (lane == 0) {
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int kb = 0; kb < C::kd / 16; ++kb)
                            tc_mma_ss(tmem_base + ch * 128 + 64 * m, smem_desc_sw128(sK + map_k_off<D>(m, kb, C::kSlab), 16, 1024),
                                      smem_desc_sw128(sQ(st) + map_k_off<D>(m, kb, C::kQSlab), 16, 1024), idesc_s, kb > 0);
                    tc_commit(s_full(ch));
                }
                __syncwarp();
                return true;
            };
            for (long long round = 0; ok && round * gridDim.x < a.total_items; ++round) {
                const long long item = item_of_round(a, round);
                if (item < 0) continue;
                const DkvItem c = decode_dkv(a, item);
                if (c.n == 0) continue;
                ok = warp_wait(kv_full, ic & 1, 0x221, abort_flag);
                if (ok) ok = scores(c, 0);
                if (ok && c.n > 1) ok = scores(c, 1);
                for (int i = 0; ok && i <= c.n; ++i) {
                    if (i < c.n) {
                        // dA of step i, once its scores are in registers
                        const int ch = i & 1, st = (g0 + (uint32_t)i) % C::kStages;
                        ok = warp_wait(s_read(ch), sr[ch] & 1, 0x222, abort_flag);
                        ++sr[ch];
                        if (!ok) break;
                        tc_fence_after();
                        if (lane == 0) {
#pragma unroll
                            for (int kb = 0; kb < D / 16; ++kb)
                                tc_mma_ss(tmem_base + ch * 128, smem_desc_sw128(sV + (kb >> 2) * C::kSlab + (kb & 3) * 32, 16, 1024),
                                          smem_desc_sw128(sG(st) + (kb >> 2) * C::kQSlab + (kb & 3) * 32, 16, 1024), idesc_s, kb > 0);
                            tc_commit(dp_full(ch));
                            if (i + 1 == c.n) tc_commit(kv_free);
                        }
                        __syncwarp();
                    }
                    if (i >= 1) {
                        // dV, dK of step i - 1, then the scores of step i + 1 in the same slots
                        const int k = i - 1, ch = k & 1, st = (g0 + (uint32_t)k) % C::kStages;
                        ok = warp_wait(ds_full(ch), sd[ch] & 1, 0x223, abort_flag);
                        ++sd[ch];
                        if (ok && k == 0) ok = warp_wait(acc_free, (ic & 1) ^ 1, 0x224, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                        if (lane == 0) {
                            const uint32_t x = tmem_base + ch * 128, y = x + 64;
#pragma unroll
                            for (int kb = 0; kb < kHalf / 16; ++kb)
                                tc_mma_ts(tmem_base + C::kColDV, y + 8 * kb, smem_desc_sw128(sG(st) + kb * 2048, C::kQSlab, 1024),
                                          idesc_v, (kb > 0 || k > 0) ? 1u : 0u);
#pragma unroll
                            for (int kb = 0; kb < kHalf / 16; ++kb)
                                tc_mma_ts(tmem_base + C::kColDK, y + 32 + 8 * kb,
                                          smem_desc_sw128(sQ(st) + map_n_off<D>(0, C::kQSlab) + kb * 2048, C::kQSlab, 1024), idesc_k,
                                          (kb > 0 || k > 0) ? 1u : 0u);
#pragma unroll
                            for (int kb = 0; kb < kHalf / 16; ++kb)
                                tc_mma_ts(tmem_base + C::kColDK + C::kd, x + 8 * kb,
                                          smem_desc_sw128(sQ(st) + map_n_off<D>(1, C::kQSlab) + kb * 2048, C::kQSlab, 1024), idesc_k,
                                          (kb > 0 || k > 0) ? 1u : 0u);
                            tc_commit(q_free(st));
                            if (i == c.n) tc_commit(acc_full);
                        }
                        __syncwarp();
                        if (i + 1 < c.n) ok = scores(c, i + 1);
                    }
                }
                g0 += (uint32_t)c.n;
                ++ic;
            }
        }
    } else {
        // =============================================================== weights, dS, epilogue
        const int ch = (warp - 4) >> 2, wq = warp & 3;
        const uint32_t tmem_lane = tmem_base + ((uint32_t)(wq * 32) << 16);
        const uint32_t x = tmem_lane + ch * 128, y = x + 64;
        const int r = wq * 32 + lane;
        bool ok = true;
        uint32_t ic = 0, g0 = 0, sc = 0;
        for (long long round = 0; ok && round * gridDim.x < a.total_items; ++round) {
            const long long item = item_of_round(a, round);
            if (item < 0) continue;
            const DkvItem c = decode_dkv(a, item);
            const int u = c.u0 + r;
            const float2 sl2 = make_float2(a.scale_log2, a.scale_log2);
            for (int i = ch; i < c.n; i += 2, ++sc) {
                const uint32_t g = g0 + (uint32_t)i;
                const int st = g % C::kStages;
                const int h = c.h0 + i / c.per_head, t0 = c.t_lo + kHalf * (i % c.per_head);
                const float4 *stat = (const float4 *)(smem + C::kOffStat + st * C::kStat);
                const float lam = __ldg(a.lambda + (a.lambda_count > 1 ? h : 0));
                const float2 lam2 = make_float2(lam, lam), neg = make_float2(-1.f, -1.f);
                // (its copies complete before the scores that read them)
                ok = warp_wait(q_full(st), (g / C::kStages) & 1, 0x230, abort_flag);
                if (ok) ok = warp_wait(s_full(ch), sc & 1, 0x231, abort_flag);
                if (!ok) break;
                tc_fence_after();
                float w1[64], w2[64];
                tmem_ld32_nowait(x, (uint32_t *)w1);
                tmem_ld32_nowait(x + 32, (uint32_t *)w1 + 32);
                tmem_ld32_nowait(y, (uint32_t *)w2);
                tmem_ld32_nowait(y + 32, (uint32_t *)w2 + 32);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(s_read(ch));
                // columns from c_lo on see this key (all of them below the diagonal); rows without a visible key and the
                // padding have a log-sum-exp of +inf, which makes their weights 0
                const int c_lo = a.causal ? u - c.sp.off - t0 : 0;
                const bool whole = __all_sync(0xffffffffu, c_lo <= 0);
                if (!whole) {
#pragma unroll
                    for (int e = 0; e < 64; ++e)
                        if (e < c_lo) w1[e] = w2[e] = -INFINITY;
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        // (keeps the statistics' loads near their use: all of them at once would spill)
                        if (e % 4 == 0) asm volatile("" ::: "memory");
                        const int k = 32 * q + 2 * e;
                        const float4 sa = stat[k], sb = stat[k + 1];
                        float2 p1 = fma2(make_float2(w1[k], w1[k + 1]), sl2, make_float2(-sa.x, -sb.x));
                        float2 p2 = fma2(make_float2(w2[k], w2[k + 1]), sl2, make_float2(-sa.y, -sb.y));
                        p1.x = fast_exp2(p1.x);
                        p1.y = fast_exp2(p1.y);
                        p2.x = fast_exp2(p2.x);
                        p2.y = fast_exp2(p2.y);
                        p2 = mul2(p2, lam2);                           // from here on lambda P_2
                        w1[k] = p1.x; w1[k + 1] = p1.y;
                        w2[k] = p2.x; w2[k + 1] = p2.y;
                        const float2 d = fma2(p2, neg, p1);
                        pk[e] = pack_bf16x2(d.x, d.y);
                    }
                    tmem_st16(y + 16 * q, pk);
                }
                ok = warp_wait(dp_full(ch), sc & 1, 0x232, abort_flag);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t v[16], p1[8], p2[8];
                    tmem_ld16_nowait(x + 16 * q, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (e % 4 == 0) asm volatile("" ::: "memory");
                        const int k = 16 * q + 2 * e;
                        const float2 sa = *(const float2 *)&stat[k].z, sb = *(const float2 *)&stat[k + 1].z;
                        const float2 da = make_float2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
                        const float2 s1 = mul2(make_float2(w1[k], w1[k + 1]), add2(da, make_float2(-sa.x, -sb.x)));
                        const float2 s2 = mul2(make_float2(w2[k], w2[k + 1]), fma2(da, neg, make_float2(sa.y, sb.y)));
                        p1[e] = pack_bf16x2(s1.x, s1.y);
                        p2[e] = pack_bf16x2(s2.x, s2.y);
                    }
                    tmem_st8(y + 32 + 8 * q, p1);
                    tmem_st8(x + 8 * q, p2);                           // (columns of dA already read)
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(ds_full(ch));
            }
            if (!ok) break;
            g0 += (uint32_t)c.n;
            if (c.n > 0) {
                ok = warp_wait(acc_full, ic & 1, 0x233, abort_flag);
                ++ic;
                if (!ok) break;
                tc_fence_after();
            }
            // warpgroup 0 writes dK (scaled), warpgroup 1 dV
            const bool in = u < a.Nk, any = c.n > 0 && u < c.sp.kl;
            const float f = ch ? 1.f : a.scale;
            const long long row = (((long long)c.b * a.H_kv + c.hk) * a.Nk + u) * D;
#pragma unroll 1
            for (int i = 0; i < D / 32; ++i) {
                uint32_t v[32];
                tmem_ld32(tmem_lane + (ch ? C::kColDV : C::kColDK) + 32 * i, v);
                if (!in) continue;
                if (a.hsplit > 1) {
                    float *dst = a.part + (ch * a.hsplit + c.hs) * a.kv_elems + row + 32 * i;
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<float4 *>(dst + e) =
                            any ? make_float4(__uint_as_float(v[e]) * f, __uint_as_float(v[e + 1]) * f, __uint_as_float(v[e + 2]) * f,
                                              __uint_as_float(v[e + 3]) * f)
                                : make_float4(0.f, 0.f, 0.f, 0.f);
                } else {
                    __nv_bfloat16 *dst = (ch ? a.dv : a.dk) + row + 32 * i;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            w[k] = any ? pack_bf16x2(__uint_as_float(v[e + 2 * k]) * f, __uint_as_float(v[e + 2 * k + 1]) * f) : 0u;
                        *reinterpret_cast<uint4 *>(dst + e) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (c.n > 0 && lane == 0) mbar_arrive(acc_free);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 3) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

template <int D>
int launch_d(const DiffProblem &p, const DiffGrads &g) {
    CUtensorMap mq, mg, mk, mv, mqh, mgh;
    int rc;
    if ((rc = make_strided_map(&mq, p.q, &p.sq.b, p.B, p.H, p.Nq, D, kRows)) != TA_OK) return rc;
    if ((rc = make_strided_map(&mg, p.dout, &p.sdo.b, p.B, p.H, p.Nq, D, kRows)) != TA_OK) return rc;
    if ((rc = make_strided_map(&mk, p.k, &p.sk.b, p.B, p.H_kv, p.Nk, D, kRows)) != TA_OK) return rc;
    if ((rc = make_strided_map(&mv, p.v, &p.sv.b, p.B, p.H_kv, p.Nk, D, kRows)) != TA_OK) return rc;
    if ((rc = make_strided_map(&mqh, p.q, &p.sq.b, p.B, p.H, p.Nq, D, kHalf)) != TA_OK) return rc;
    if ((rc = make_strided_map(&mgh, p.dout, &p.sdo.b, p.B, p.H, p.Nq, D, kHalf)) != TA_OK) return rc;
    int dev = 0;
    const int num_sms = current_device_sms(&dev);
    static PerDeviceOnce configured;
    if (!configured.is_done(dev)) {
        const auto dyn = cudaFuncAttributeMaxDynamicSharedMemorySize;
        cudaError_t e = cudaFuncSetAttribute(diff_tc_dq_kernel<D>, dyn, (int)DqCfg<D>::kSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(diff_tc_dkv_kernel<D>, dyn, (int)DkvCfg<D>::kSmem);
        if (e != cudaSuccess) return cuda_fail(e);
        configured.mark(dev);
    }
    BwdArgs a = {};
    a.B = p.B; a.H = p.H; a.H_kv = p.H_kv; a.g = p.H / p.H_kv; a.Nq = p.Nq; a.Nk = p.Nk; a.causal = p.causal;
    a.prow = diff_padded_rows(p.Nq);
    a.scale = p.scale;
    a.scale_log2 = p.scale * 1.4426950408889634f;
    a.q_lens = p.q_lens; a.kv_lens = p.kv_lens;
    a.lambda = p.lambda; a.lambda_count = p.lambda_count;
    a.stats = g.stats;
    a.dq = (__nv_bfloat16 *)g.dq; a.dk = (__nv_bfloat16 *)g.dk; a.dv = (__nv_bfloat16 *)g.dv;
    a.part = g.part; a.dlam_part = g.dlam_part;
    a.kv_elems = (long long)p.B * p.H_kv * p.Nk * D;
    a.hsplit = g.hsplit;
    a.gi = a.g / g.hsplit;

    a.tiles = (p.Nq + kRows - 1) / kRows;
    a.total_items = (long long)p.B * p.H * a.tiles;
    a.tile_major = 2ull * p.B * p.H_kv * p.Nk * D * 2 <= (96ull << 20) ? 1 : 0;
    rc = launch_kernel(diff_tc_dq_kernel<D>, (unsigned)(a.total_items < num_sms ? a.total_items : num_sms), kThreads,
                       DqCfg<D>::kSmem, p.stream, false, mq, mg, mk, mv, a);
    if (rc != TA_OK) return rc;
    a.tiles = (p.Nk + kRows - 1) / kRows;
    a.total_items = (long long)p.B * p.H_kv * g.hsplit * a.tiles;
    a.tile_major = 2ull * p.B * p.H * p.Nq * D * 2 <= (96ull << 20) ? 1 : 0;
    return launch_kernel(diff_tc_dkv_kernel<D>, (unsigned)(a.total_items < num_sms ? a.total_items : num_sms), kThreads,
                         DkvCfg<D>::kSmem, p.stream, false, mqh, mgh, mk, mv, a);
}

}  // namespace

int launch_diff_tc_bwd(const DiffProblem &p, const DiffGrads &g) {
    if (p.D == 128) return launch_d<128>(p, g);
    if (p.D == 64) return launch_d<64>(p, g);
    return TA_ERR_UNSUPPORTED;
}

int read_status_diff_tc_bwd(unsigned int *word) {
    if (cudaMemcpyFromSymbol(word, g_status_word, sizeof(*word)) != cudaSuccess) return TA_ERR_CUDA;
    if (*word != 0) {
        unsigned int z = 0;
        cudaMemcpyToSymbol(g_status_word, &z, sizeof(z));
    }
    return TA_OK;
}

}  // namespace ta
