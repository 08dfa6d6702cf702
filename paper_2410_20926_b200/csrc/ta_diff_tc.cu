// Differential attention, forward pass on the tensor cores: bf16, head dim 64 or 128.
//
//     out = (A_1 - lambda A_2) V,   A_c = softmax(Q_c K_c^T scale o M)
//
// A work item is one tile of 128 query rows of one head.  Its keys go by once in blocks of 128; the two maps are two
// chains that share the K and V blocks and alternate on the tensor pipe.  Per chain c and key block j
//     S_c = Q_c K_c^T                      (half the head dim, fp32 in tensor memory)
//     m <- max(m, rowmax),  P = 2^(S scale log2 e - m) -> bf16, over S in tensor memory,  l <- l alpha + rowsum P
//     O_c <- alpha O_c + P V               (whole head dim)
// and at the end out = O_1 / l_1 - lambda O_2 / l_2: the sums l_c are known only then, so the maps cannot be subtracted
// before the value product, and the pass needs 6 D multiply-adds per visible pair where the definition has 4 D.
// S_1, S_2, O_1, O_2 fill the tensor memory (4 x 128 columns).
//
// One CTA per SM, persistent: warp 0 loads (TMA), warp 1 issues the MMAs in a fixed order -- P V of block j, then S of
// block j + 1, chain after chain, so that one chain's exponentials run under the other chain's products --, warps 4-7 and
// 8-11 are the softmax of chain 1 and 2 (one query row per thread, its 128 scores in registers).  A running maximum
// is moved (and O rescaled) only when it has grown by more than 2^8: weights up to 256 lose nothing in bf16 or fp32.
// Every wait is bounded; when one expires the CTA raises a flag that ends all roles, lets its copies land, frees its
// tensor memory and returns.
#include "ta_diff_tc.cuh"

namespace ta {
namespace {

constexpr int kRows = 128;
constexpr int kThreads = 384;
constexpr uint32_t kSlab = kRows * 128;

template <int D>
struct Cfg {
    static constexpr int kSlabs = D / 64;
    static constexpr int kd = D / 2;
    static constexpr uint32_t kTile = kSlabs * kSlab;
    static constexpr int kNQ = 2;
    static constexpr int kNKV = D == 128 ? 2 : 4;
    static constexpr uint32_t kOffQ = 0;
    static constexpr uint32_t kOffK = kOffQ + kNQ * kTile;
    static constexpr uint32_t kOffV = kOffK + kNKV * kTile;
    static constexpr uint32_t kOffBar = kOffV + kNKV * kTile;
    static constexpr int kNumBars = 2 * kNQ + 3 * kNKV + 2 + 2 + 2 + 2;
    static constexpr uint32_t kOffX = kOffBar + ((kNumBars * 8 + 16 + 15) & ~15);      // 1 / l of both maps, 128 rows
    static constexpr uint32_t kSmem = kOffX + 2 * kRows * 4 + 1024;
    static constexpr uint32_t kColS = 0, kColO = 256;
};

struct TcArgs {
    int B, H, H_kv, g, Nq, Nk, causal;
    int qtiles, tile_major;
    long long total_items;
    float scale_log2;
    const int *q_lens, *kv_lens;
    const float *lambda;
    int lambda_count;
    __nv_bfloat16 *out;
    Strides3 so;
    float2 *lse;
    short *o16;
    float2 *ostep;
};

struct Item {
    int b, h, hk, t0;
    DiffSpan sp;
    int keys_end, nblocks;       // keys any row of the tile sees
};
__device__ __forceinline__ Item decode(const TcArgs &a, long long item) {
    Item c;
    int tile;
    long long bh;
    const long long heads = (long long)a.B * a.H;
    // Later (longer, when causal) tiles first.  While all K and V fit the L2 the tile is the slowest index, so the
    // numbering runs from the longest items to the shortest over the whole launch; beyond that the tiles of a head
    // stay together.
    if (a.tile_major) {
        tile = a.qtiles - 1 - (int)(item / heads);
        bh = item % heads;
    } else {
        tile = a.qtiles - 1 - (int)(item % a.qtiles);
        bh = item / a.qtiles;
    }
    c.b = (int)(bh / a.H);
    c.h = (int)(bh - (long long)c.b * a.H);
    c.hk = c.h / a.g;
    c.t0 = tile * kRows;
    c.sp = diff_span(a.q_lens, a.kv_lens, c.b, a.Nq, a.Nk);
    const int last = min(c.t0 + kRows, c.sp.ql) - 1;      // the last valid row sees the most
    c.keys_end = last >= c.t0 ? c.sp.keys(last, a.causal) : 0;
    c.nblocks = (c.keys_end + kRows - 1) / kRows;
    return c;
}
// the item of a CTA's k-th round: forth and back over the CTAs, so that long and short items pair up
__device__ __forceinline__ long long item_of_round(const TcArgs &a, long long k) {
    const long long g = gridDim.x, b = blockIdx.x;
    const long long item = k * g + ((k & 1) ? g - 1 - b : b);
    return item < a.total_items ? item : -1;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
diff_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
               const __grid_constant__ CUtensorMap map_v, const __grid_constant__ TcArgs a) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t s0 = smem_u32(smem);
    auto sQ = [&](int i) { return s0 + C::kOffQ + (uint32_t)i * C::kTile; };
    auto sK = [&](int i) { return s0 + C::kOffK + (uint32_t)i * C::kTile; };
    auto sV = [&](int i) { return s0 + C::kOffV + (uint32_t)i * C::kTile; };
    const uint32_t bar0 = s0 + C::kOffBar;
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
    auto q_full = [&](int i) { return bar(i); };
    auto q_free = [&](int i) { return bar(C::kNQ + i); };
    auto k_full = [&](int i) { return bar(2 * C::kNQ + i); };
    auto v_full = [&](int i) { return bar(2 * C::kNQ + C::kNKV + i); };
    auto kv_free = [&](int i) { return bar(2 * C::kNQ + 2 * C::kNKV + i); };
    constexpr int kB = 2 * C::kNQ + 3 * C::kNKV;
    auto s_full = [&](int c) { return bar(kB + c); };          // scores of chain c complete
    auto p_full = [&](int c) { return bar(kB + 2 + c); };      // weights of chain c written (4 warps)
    auto o_full = [&](int c) { return bar(kB + 4 + c); };      // value sum of chain c complete
    const uint32_t o_free = bar(kB + 6);                       // both value sums read (8 warps)
    const uint32_t x_full = bar(kB + 7);                       // 1 / l of both maps written (8 warps)
    uint32_t *tmem_slot = (uint32_t *)(smem + C::kOffBar + C::kNumBars * 8);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    float *s_inv = (float *)(smem + C::kOffX);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // rows a tensor does not have arrive as zeros (TMA fill); nothing reads shared memory before it is loaded
    if (tid == 0) {
        for (int i = 0; i < C::kNumBars; ++i)
            mbar_init(bar(i), i == kB + 2 || i == kB + 3 ? 4 : i >= kB + 6 ? 8 : 1);
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
            uint32_t armed = 0, last_par = 0;        // bits: q, k, v slots
            auto arm = [&](int slot, uint32_t parity) {
                const uint32_t bit = 1u << slot;
                armed |= bit;
                last_par = parity ? (last_par | bit) : (last_par & ~bit);
            };
            bool ok = true;
            for (long long round = 0; ok && round * gridDim.x < a.total_items; ++round) {
                const long long item = item_of_round(a, round);
                if (item < 0) continue;
                const Item c = decode(a, item);
                if (c.nblocks == 0) continue;
                const int qs = ic % C::kNQ;
                const uint32_t qp = (ic / C::kNQ) & 1;
                ++ic;
                ok = mbar_wait_abortable(q_free(qs), qp ^ 1, 0xD10, abort_flag);
                if (!ok) break;
                mbar_expect_tx(q_full(qs), C::kTile);
                arm(qs, qp);
#pragma unroll
                for (int s = 0; s < C::kSlabs; ++s)
                    tma_load_5d(sQ(qs) + s * kSlab, &map_q, q_full(qs), 64 * s, c.t0, 0, c.h, c.b);
                for (int j = 0; j < c.nblocks; ++j, ++g) {
                    const int st = g % C::kNKV;
                    const uint32_t par = (g / C::kNKV) & 1;
                    ok = mbar_wait_abortable(kv_free(st), par ^ 1, 0xD11, abort_flag);
                    if (!ok) break;
                    mbar_expect_tx(k_full(st), C::kTile);
                    arm(C::kNQ + st, par);
#pragma unroll
                    for (int s = 0; s < C::kSlabs; ++s)
                        tma_load_5d(sK(st) + s * kSlab, &map_k, k_full(st), 64 * s, kRows * j, 0, c.hk, c.b);
                    mbar_expect_tx(v_full(st), C::kTile);
                    arm(C::kNQ + C::kNKV + st, par);
#pragma unroll
                    for (int s = 0; s < C::kSlabs; ++s)
                        tma_load_5d(sV(st) + s * kSlab, &map_v, v_full(st), 64 * s, kRows * j, 0, c.hk, c.b);
                }
            }
            if (!ok) {
                const unsigned long long t0 = globaltimer_ns();
                for (int slot = 0; slot < C::kNQ + 2 * C::kNKV; ++slot) {
                    if (!(armed & (1u << slot))) continue;
                    const uint32_t b = slot < C::kNQ ? q_full(slot) : bar(2 * C::kNQ + slot - C::kNQ);
                    while (!mbar_try_wait(b, (last_par >> slot) & 1u) && globaltimer_ns() - t0 < 10000000ull) {
                    }
                }
            }
        }
    } else if (warp == 1) {
        // =============================================================== MMA issuer (lane 0 issues, the warp waits)
        constexpr uint32_t idesc_s = instr_desc(128, 0);
        constexpr uint32_t idesc_o = instr_desc(D, 1);
        uint32_t ic = 0, g = 0, pc = 0;              // items, key blocks, blocks of weights so far
        bool ok = true;
        auto scores = [&](int c, int qs, int st) {
            const uint32_t ql = desc_low(sQ(qs), 16), kl = desc_low(sK(st), 16);
            if (elect_one()) {
#pragma unroll
                for (int kb = 0; kb < C::kd / 16; ++kb) {
                    const uint32_t off = map_k_off<D>(c, kb, kSlab) >> 4;
                    mma_ss(tmem_base + C::kColS + c * 128, ql + off, kl + off, idesc_s, kb > 0);
                }
                tc_commit(s_full(c));
            }
            __syncwarp();
        };
        for (long long round = 0; ok && round * gridDim.x < a.total_items; ++round) {
            const long long item = item_of_round(a, round);
            if (item < 0) continue;
            const Item c = decode(a, item);
            if (c.nblocks == 0) continue;
            const int qs = ic % C::kNQ;
            ok = warp_wait(q_full(qs), (ic / C::kNQ) & 1, 0xE10, abort_flag);
            if (ok) ok = warp_wait(k_full(g % C::kNKV), (g / C::kNKV) & 1, 0xE11, abort_flag);
            if (!ok) break;
            tc_fence_after();
            scores(0, qs, g % C::kNKV);
            scores(1, qs, g % C::kNKV);
            for (int j = 0; j < c.nblocks; ++j, ++g, ++pc) {
                const int st = g % C::kNKV, nx = (g + 1) % C::kNKV;
                const bool more = j + 1 < c.nblocks;
                ok = warp_wait(v_full(st), (g / C::kNKV) & 1, 0xE12, abort_flag);
                if (ok && more) ok = warp_wait(k_full(nx), ((g + 1) / C::kNKV) & 1, 0xE13, abort_flag);
                if (!ok) break;
                const int keys = min(kRows, c.keys_end - kRows * j);
                const int ksteps = (keys + 15) >> 4;
                if (c.sp.kl < a.Nk && c.sp.kl - kRows * j < 16 * ksteps) {
                    zero_rows(sV(st), kSlab, C::kSlabs, c.sp.kl - kRows * j, 16 * ksteps);
                    fence_proxy_async_smem();
                    __syncwarp();
                }
#pragma unroll
                for (int ch = 0; ch < 2; ++ch) {
                    ok = warp_wait(p_full(ch), pc & 1, 0xE14, abort_flag);
                    if (ok && j == 0 && ch == 0) ok = warp_wait(o_free, (ic & 1) ^ 1, 0xE15, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t vl = desc_low(sV(st), kSlab), o = tmem_base + C::kColO + ch * 128, w = tmem_base + C::kColS + ch * 128;
                    const uint32_t first = j > 0 ? 1u : 0u;
                    if (elect_one()) {
                        // (weights beyond ksteps are zeros that nothing has to multiply)
#pragma unroll
                        for (int kb = 0; kb < kRows / 16; ++kb)
                            if (kb < ksteps) mma_ts(o, w + kb * 8, vl + 128u * kb, idesc_o, kb > 0 ? 1u : first);
                        if (ch == 1) tc_commit(kv_free(st));
                        if (!more) tc_commit(o_full(ch));
                        if (!more && ch == 1) tc_commit(q_free(qs));
                    }
                    __syncwarp();
                    if (more) scores(ch, qs, nx);
                }
                if (!ok) break;
            }
            ++ic;
        }
    } else if (warp >= 4) {
        // =============================================================== softmax, epilogue
    
        const int ch = (warp - 4) >> 2, wq = warp & 3;
        const uint32_t tmem_lane = tmem_base + ((uint32_t)(wq * 32) << 16);
        const uint32_t s_col = tmem_lane + C::kColS + ch * 128;
        const uint32_t o_col = tmem_lane + C::kColO + ch * 128;
        const int r = wq * 32 + lane;
        bool ok = true;
        uint32_t ic = 0, sc = 0;
        for (long long round = 0; ok && round * gridDim.x < a.total_items; ++round) {
            const long long item = item_of_round(a, round);
            if (item < 0) continue;
            const Item c = decode(a, item);
            const int t = c.t0 + r;
            const int row_keys = c.sp.keys(t, a.causal);
            float m = -INFINITY, l = 0.f;               // running maximum (scaled, log2) and sum
            for (int j = 0; j < c.nblocks; ++j, ++sc) {
                ok = warp_wait(s_full(ch), sc & 1, 0xF10, abort_flag);
                if (!ok) break;
                tc_fence_after();
                // pass over the scores for the row maximum; they are read again for the weights (128 of them held
                // across the rescaling would spill)
                const int c_hi = row_keys - kRows * j;
                const bool whole = __all_sync(0xffffffffu, c_hi >= kRows);
                float bm0 = -INFINITY, bm1 = -INFINITY, bm2 = -INFINITY, bm3 = -INFINITY;
                uint32_t v[2][32];
                tmem_ld32_nowait(s_col, v[0]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    tmem_ld_wait();
                    if (i < 3) tmem_ld32_nowait(s_col + 32 * (i + 1), v[(i + 1) & 1]);
                    uint32_t *x = v[i & 1];
                    if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (32 * i + e >= c_hi) x[e] = 0xFF800000u;      // -inf
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        bm0 = fmaxf(bm0, fmaxf(__uint_as_float(x[e]), __uint_as_float(x[e + 1])));
                        bm1 = fmaxf(bm1, fmaxf(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3])));
                        bm2 = fmaxf(bm2, fmaxf(__uint_as_float(x[e + 4]), __uint_as_float(x[e + 5])));
                        bm3 = fmaxf(bm3, fmaxf(__uint_as_float(x[e + 6]), __uint_as_float(x[e + 7])));
                    }
                }
                const float bm = fmaxf(fmaxf(bm0, bm1), fmaxf(bm2, bm3)) * a.scale_log2;
                if (__any_sync(0xffffffffu, bm > m + 8.f)) {
                    // the first block, or the maximum has outgrown the reference: move it, rescale what was summed so far
                    const float mn = fmaxf(m, bm);
                    const float alpha = m == -INFINITY ? 0.f : fast_exp2(m - mn);
                    l *= alpha;
                    if (j > 0) {
                        // (S of this block was issued behind the previous value product: that one is complete)
#pragma unroll 1
                        for (int i = 0; i < D / 32; ++i) {
                            uint32_t o[32];
                            tmem_ld32(o_col + 32 * i, o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                            tmem_st32(o_col + 32 * i, o);
                        }
                    }
                    m = mn;
                }
                const float ref = m == -INFINITY ? 0.f : m;
                const float2 nref = make_float2(-ref, -ref), sl2 = make_float2(a.scale_log2, a.scale_log2);
                float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
                tmem_ld32_nowait(s_col, v[0]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    tmem_ld_wait();
                    if (i < 3) tmem_ld32_nowait(s_col + 32 * (i + 1), v[(i + 1) & 1]);
                    uint32_t *x = v[i & 1];
                    if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (32 * i + e >= c_hi) x[e] = 0xFF800000u;
                    }
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float2 y = fma2(make_float2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), sl2, nref);
                        y.x = fast_exp2(y.x);
                        y.y = fast_exp2(y.y);
                        pk[e] = pack_bf16x2(y.x, y.y);
                        if (e & 1) sum1 = add2(sum1, y); else sum0 = add2(sum0, y);
                    }
                    // (columns 16 i .. of the scores have been read: the next chunk, at 32 (i + 1), has been waited for or
                    // lies behind)
                    tmem_st16(s_col + 16 * i, pk);
                }
                l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(ch));
            }
            if (!ok) break;

            // ---- epilogue: every thread half the columns of its row of the result
            const float lam = __ldg(a.lambda + (a.lambda_count > 1 ? c.h : 0));
            const float inv = l > 0.f || l != l ? 1.f / l : 0.f;         // (NaN stays NaN)
            const long long row = ((long long)c.b * a.H + c.h) * a.Nq + t;
            float i1 = 0.f, i2 = 0.f;
            if (c.nblocks > 0) {
                // (the other chain has read the last item's numbers: no value product of this item starts before)
                s_inv[ch * kRows + r] = inv;
                __syncwarp();
                if (lane == 0) mbar_arrive(x_full);
                ok = warp_wait(x_full, ic & 1, 0xF13, abort_flag);
                if (ok) ok = warp_wait(o_full(0), ic & 1, 0xF11, abort_flag);
                if (ok) ok = warp_wait(o_full(1), ic & 1, 0xF12, abort_flag);
                ++ic;
                i1 = s_inv[r];
                i2 = s_inv[kRows + r] * lam;
            }
            if (!ok) break;
            tc_fence_after();
            const bool row_in = t < a.Nq, any = row_keys > 0;
            __nv_bfloat16 *dst = a.out + (long long)c.b * a.so.b + (long long)c.h * a.so.h + (long long)t * a.so.n;
#pragma unroll 1
            for (int i = ch * (D / 64); i < (ch + 1) * (D / 64); ++i) {
                uint32_t o1[32], o2[32];
                // (an item without blocks reads what the last one left, and drops it)
                tmem_ld32_nowait(tmem_lane + C::kColO + 32 * i, o1);
                tmem_ld32_nowait(tmem_lane + C::kColO + 128 + 32 * i, o2);
                tmem_ld_wait();
                if (!row_in) continue;
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const int x = e + 2 * f;
                        const float lo = __uint_as_float(o1[x]) * i1 - __uint_as_float(o2[x]) * i2;
                        const float hi = __uint_as_float(o1[x + 1]) * i1 - __uint_as_float(o2[x + 1]) * i2;
                        w[f] = any ? pack_bf16x2(lo, hi) : 0u;
                    }
                    *reinterpret_cast<uint4 *>(dst + 32 * i + e) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            if (a.lse != nullptr) {
                // for the backward: this map's log-sum-exp and value sum
                if (row_in) reinterpret_cast<float *>(a.lse)[2 * row + ch] = any ? m + log2f(l) : INFINITY;
                float most = 0.f;
#pragma unroll 1
                for (int i = 0; i < D / 32; ++i) {
                    uint32_t o[32];
                    tmem_ld32(o_col + 32 * i, o);
#pragma unroll
                    for (int e = 0; e < 32; ++e) most = fmaxf(most, fabsf(__uint_as_float(o[e])));
                }
                if (!any) most = 0.f;
                const float n = diff_inv_step(most);
                if (row_in) reinterpret_cast<float *>(a.ostep)[2 * row + ch] = most * inv * (1.f / 32767.f);
                short *o16 = a.o16 + (2 * row + ch) * D;
#pragma unroll 1
                for (int i = 0; i < D / 32; ++i) {
                    uint32_t o[32];
                    tmem_ld32(o_col + 32 * i, o);
                    if (!row_in) continue;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int f = 0; f < 4; ++f)
                            w[f] = any ? diff_pack16(__uint_as_float(o[e + 2 * f]) * n, __uint_as_float(o[e + 2 * f + 1]) * n) : 0u;
                        *reinterpret_cast<uint4 *>(o16 + 32 * i + e) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (c.nblocks > 0 && lane == 0) mbar_arrive(o_free);
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
int launch_d(const DiffProblem &p) {
    using C = Cfg<D>;
    CUtensorMap mq, mk, mv;
    int rc;
    if ((rc = make_strided_map(&mq, p.q, &p.sq.b, p.B, p.H, p.Nq, D, kRows)) != TA_OK) return rc;
    if ((rc = make_strided_map(&mk, p.k, &p.sk.b, p.B, p.H_kv, p.Nk, D, kRows)) != TA_OK) return rc;
    if ((rc = make_strided_map(&mv, p.v, &p.sv.b, p.B, p.H_kv, p.Nk, D, kRows)) != TA_OK) return rc;
    TcArgs a = {};
    a.B = p.B; a.H = p.H; a.H_kv = p.H_kv; a.g = p.H / p.H_kv; a.Nq = p.Nq; a.Nk = p.Nk; a.causal = p.causal;
    a.qtiles = (p.Nq + kRows - 1) / kRows;
    a.total_items = (long long)p.B * p.H * a.qtiles;
    // K and V of all heads against the 126 MB L2
    a.tile_major = 2ull * p.B * p.H_kv * p.Nk * D * 2 <= (96ull << 20) ? 1 : 0;
    a.scale_log2 = p.scale * 1.4426950408889634f;
    a.q_lens = p.q_lens; a.kv_lens = p.kv_lens;
    a.lambda = p.lambda; a.lambda_count = p.lambda_count;
    a.out = (__nv_bfloat16 *)p.out;
    a.so = p.so;
    a.lse = p.lse; a.o16 = p.o16; a.ostep = p.ostep;
    int dev = 0;
    const int num_sms = current_device_sms(&dev);
    static PerDeviceOnce configured;
    if (!configured.is_done(dev)) {
        const cudaError_t e = cudaFuncSetAttribute(diff_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem);
        if (e != cudaSuccess) return cuda_fail(e);
        configured.mark(dev);
    }
    const unsigned grid = (unsigned)(a.total_items < num_sms ? a.total_items : num_sms);
    return launch_kernel(diff_tc_kernel<D>, grid, kThreads, C::kSmem, p.stream, false, mq, mk, mv, a);
}

}  // namespace

int launch_diff_tc(const DiffProblem &p) {
    if (p.D == 128) return launch_d<128>(p);
    if (p.D == 64) return launch_d<64>(p);
    return TA_ERR_UNSUPPORTED;
}

int read_status_diff_tc(unsigned int *word) {
    if (cudaMemcpyFromSymbol(word, g_status_word, sizeof(*word)) != cudaSuccess) return TA_ERR_CUDA;
    if (*word != 0) {
        unsigned int z = 0;
        cudaMemcpyToSymbol(g_status_word, &z, sizeof(z));
    }
    return TA_OK;
}

}  // namespace ta
