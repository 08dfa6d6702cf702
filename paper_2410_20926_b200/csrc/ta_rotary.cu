// Rotary positions with several axes (ta_rotary): pairs of features (x1, x2) of every q and k row turned by an
// angle that comes from one of the token's coordinates (time / height / width, or the coordinates of the
// n_1 x .. x n_m tensor),
//     y1 = x1 cos - x2 sin,   y2 = x2 cos + x1 sin,   angle = pos[axis(c)] * freq(c),
// with the opposite angle for the gradient.  The paper says a token's position is the vector of its coordinates
// (Section 3.2); here every pair of features belongs to one axis and q and k are rotated once.
//
// Bound by memory: every element is read and written once.  A block works out the sines and cosines of its tokens into
// shared memory; then a thread owns V neighbouring pairs of one token (16 bytes and 16 bytes), keeps their sines and
// cosines in registers and walks a chunk of the heads, q's and k's alike, which all share them.  With few tokens
// (decoding) the chunks shrink until the launch fills the GPU.
//
// Angles: freq(c) / (2 pi) is kept as a 64-bit fixed-point fraction of a turn, so pos * fraction modulo 2^64 is the
// angle modulo a turn, exact to pos * 2^-64 for every 32-bit position of either sign; sincospif then sees a value in
// [-1, 1).  (An fp32 product is off by milliradians at position 10^5.)
#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "ta_internal.h"
#include "ta_ptx.cuh"

namespace ta {
namespace {

constexpr int kMaxPairs = TA_MAX_HEAD_DIM / 2;
constexpr int kThreads = 256;

struct RotaryArgs {
    const void *src[2];                  // q, k
    void *dst[2];
    long long ss[2][3], ds[2][3];        // strides (batch, head, token) in elements
    int heads_q, heads;                  // H, H + H_kv
    int N, parts, part_dim, half;     // half: rotated pairs per part
    int units;                           // units of V pairs per (token, part): rotated ones, then copies
    int heads_per_block, tokens;         // heads and tokens of a block
    long long total_tokens;              // B * N
    int inverse;
    int small;                           // thread and token indices fit 32 bits
    const int *positions;
    long long pos_axis_stride, pos_batch_stride;
    long long token_offset;
    long long dim_stride[TA_MAX_DIMS];
    int dim[TA_MAX_DIMS];
    unsigned long long freq[kMaxPairs];  // turns per position, 0.64 fixed point
    unsigned char axis[kMaxPairs];
};

template <typename T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// V neighbouring features as they stand in memory
template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    static constexpr bool kWords = sizeof(T) * V >= 4;
    using Word = typename std::conditional<kWords, uint32_t, uint16_t>::type;
    static constexpr int kNum = kWords ? (int)sizeof(T) * V / 4 : 1;
    Word w[kNum];

    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else if constexpr (!kWords) return __uint_as_float((uint32_t)w[0] << 16);
        else return __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    // features i, i + 1 (i even), or feature 0 of a vector of one
    __device__ __forceinline__ void put2(int i, float lo, float hi) {
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(lo);
            if (V > 1) w[i + 1 < V ? i + 1 : i] = __float_as_uint(hi);
        } else if constexpr (!kWords) {
            w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(lo));
        } else {
            w[i / 2] = pack_bf16x2(lo, hi);
        }
    }
};

// Turns the unit's pairs in place.  Halves: pair i is (x1[i], x2[i]).  Interleaved: pair i is features 2 i, 2 i + 1 of
// the 2 V that x1 | x2 hold, and only the first nrot pairs turn (the others keep their bits).
template <typename T, int V, bool kInterleaved>
__device__ __forceinline__ void turn(Vec<T, V> &x1, Vec<T, V> &x2, const float *cs, const float *sn, int nrot) {
    if constexpr (kInterleaved && V == 1) {
        if (nrot) {
            const float va = x1.get(0), vb = x2.get(0);
            x1.put2(0, va * cs[0] - vb * sn[0], 0.f);
            x2.put2(0, vb * cs[0] + va * sn[0], 0.f);
        }
    } else if constexpr (kInterleaved) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < nrot) {
                Vec<T, V> &x = 2 * i < V ? x1 : x2;
                const int f = (2 * i) % V;
                const float va = x.get(f), vb = x.get(f + 1);
                x.put2(f, va * cs[i] - vb * sn[i], vb * cs[i] + va * sn[i]);
            }
    } else {
        if (nrot == 0) return;
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const int j = i + 1 < V ? i + 1 : i;
            const float a0 = x1.get(i), b0 = x2.get(i), a1 = x1.get(j), b1 = x2.get(j);
            x1.put2(i, a0 * cs[i] - b0 * sn[i], a1 * cs[j] - b1 * sn[j]);
            x2.put2(i, b0 * cs[i] + a0 * sn[i], b1 * cs[j] + a1 * sn[j]);
        }
    }
}

// Halves layout: a unit is V pairs (c .. c+V-1, half + c ..).  Interleaved: the 2 V neighbouring features of V pairs.
// Features behind the rotated ones are copied bit for bit, in units of 2 V features.
template <typename T, int V, bool kInterleaved>
__global__ void __launch_bounds__(kThreads, 4)
rotary_kernel(const __grid_constant__ RotaryArgs a) {
    extern __shared__ float2 s_turn[];                    // [tokens of the block][half]: cosine, sine
    __shared__ unsigned long long s_freq[kMaxPairs];
    __shared__ unsigned char s_axis[kMaxPairs];
    // (a table in parameter space that lanes index differently is read lane by lane: once per block is enough)
    for (int i = threadIdx.x; i < a.half; i += kThreads) {
        s_freq[i] = a.freq[i];
        s_axis[i] = a.axis[i];
    }
    __syncthreads();
    const long long tok0 = (long long)blockIdx.x * a.tokens;
    const int ntok = (int)min((long long)a.tokens, a.total_tokens - tok0);
    for (int i = threadIdx.x; i < ntok * a.half; i += kThreads) {
        const int t = i / a.half, c = i - t * a.half;
        const int ax = s_axis[c];
        const unsigned b = a.N == 1 ? (unsigned)(tok0 + t) : a.small ? (unsigned)(tok0 + t) / (unsigned)a.N : (unsigned)((tok0 + t) / a.N);
        const int n = (int)(tok0 + t - (long long)b * a.N);
        int pos;
        if (a.positions != nullptr)
            pos = __ldg(a.positions + ax * a.pos_axis_stride + b * a.pos_batch_stride + n);
        else
            pos = a.small ? (int)(((unsigned)a.token_offset + n) / (unsigned)a.dim_stride[ax] % (unsigned)a.dim[ax])
                          : (int)(((a.token_offset + n) / a.dim_stride[ax]) % a.dim[ax]);
        const unsigned long long turns = (unsigned long long)(long long)pos * s_freq[c] + 0x80000000ull;
        float2 cs;
        sincospif((float)(int)(turns >> 32) * 4.656612873077392578125e-10f, &cs.y, &cs.x);   // 2^-31: half turns
        if (a.inverse) cs.y = -cs.y;
        s_turn[i] = cs;
    }
    __syncthreads();

    // this thread: one unit of one token, every (kThreads / slots)-th head of the block's chunk
    const int slots = a.tokens * a.parts * a.units;
    const int lane_head = threadIdx.x / slots, slot = threadIdx.x - lane_head * slots;
    const int step = kThreads / slots;
    const int tp = slot / a.units, unit = slot - tp * a.units;
    const int tok = tp / a.parts, part = tp - tok * a.parts;
    if (lane_head >= step || tok >= ntok) return;
    const unsigned b = a.small ? (unsigned)(tok0 + tok) / (unsigned)a.N : (unsigned)((tok0 + tok) / a.N);
    const int n = (int)(tok0 + tok - (long long)b * a.N);
    const int c0 = unit * V;                              // first pair of the unit
    const int nrot = kInterleaved ? min(max(a.half - c0, 0), V) : (c0 < a.half ? V : 0);
    float cs[V], sn[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < nrot) {
            const float2 t = s_turn[tok * a.half + c0 + i];
            cs[i] = t.x;
            sn[i] = t.y;
        }
    // feature offsets of the unit's two vectors
    int o1, o2;
    if (kInterleaved) {
        o1 = part * a.part_dim + 2 * c0;
        o2 = o1 + V;
    } else {
        // units behind the rotated ones: 2 V features each from 2 * half on, which is 2 * c0
        o1 = part * a.part_dim + (nrot ? c0 : 2 * c0);
        o2 = nrot ? o1 + a.half : o1 + V;
    }
    using VT = Vec<T, V>;
    const int h1 = min(a.heads, (int)(blockIdx.y + 1) * a.heads_per_block);
    // In the last unit the copied tail may be shorter than 2 V features (interleaved and copied units alike).
    const bool whole = 2 * c0 + 2 * V <= a.part_dim;
    const int h0 = blockIdx.y * a.heads_per_block + lane_head;
    auto source = [&](int h) {
        const int w = h >= a.heads_q ? 1 : 0;
        return reinterpret_cast<const T *>(a.src[w]) + b * a.ss[w][0] + (h - (w ? a.heads_q : 0)) * a.ss[w][1] + n * a.ss[w][2];
    };
    auto target = [&](int h) {
        const int w = h >= a.heads_q ? 1 : 0;
        return reinterpret_cast<T *>(a.dst[w]) + b * a.ds[w][0] + (h - (w ? a.heads_q : 0)) * a.ds[w][1] + n * a.ds[w][2];
    };
    if (!whole) {
        const int have = a.part_dim - 2 * c0;             // features left, 1 .. 2 V - 1; o1 is their first
        for (int h = h0; h < h1; h += step) {
            const T *s = source(h) + o1;
            T *d = target(h) + o1;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (kInterleaved && j < nrot) {
                    const float x1 = to_f(s[2 * j]), x2 = to_f(s[2 * j + 1]);
                    d[2 * j] = from_f<T>(x1 * cs[j] - x2 * sn[j]);
                    d[2 * j + 1] = from_f<T>(x2 * cs[j] + x1 * sn[j]);
                }
            for (int i = 2 * nrot; i < have; ++i) d[i] = s[i];
        }
        return;
    }
    // (the next head's loads are in flight while one is turned; two or three ahead cost registers and with them warps:
    // 125 and 141 us instead of 123 for 32k tokens of 40 heads)
    VT x1, x2;
    if (h0 < h1) {
        const T *s = source(h0);
        x1 = *reinterpret_cast<const VT *>(s + o1);
        x2 = *reinterpret_cast<const VT *>(s + o2);
    }
    for (int h = h0; h < h1; h += step) {
        VT y1 = x1, y2 = x2;
        if (h + step < h1) {
            const T *s = source(h + step);
            x1 = *reinterpret_cast<const VT *>(s + o1);
            x2 = *reinterpret_cast<const VT *>(s + o2);
        }
        turn<T, V, kInterleaved>(y1, y2, cs, sn, nrot);
        T *d = target(h);
        *reinterpret_cast<VT *>(d + o1) = y1;
        *reinterpret_cast<VT *>(d + o2) = y2;
    }
}

template <typename T, int V, bool kInterleaved>
int launch_rotary(RotaryArgs &a, cudaStream_t stream) {
    // units per part: the rotated pairs (a multiple of V in the halves layout), then the copied features
    a.units = (a.part_dim + 2 * V - 1) / (2 * V);
    // tokens of a block: as many as its threads cover with one unit each, and 16 KB of sines and cosines
    const int per_token = a.parts * a.units;              // at most 2/3 of D: a part rotates at least one pair
    a.tokens = kThreads / per_token;
    if (a.tokens > 2048 / a.half) a.tokens = 2048 / a.half;
    if ((long long)a.tokens > a.total_tokens) a.tokens = (int)a.total_tokens;
    // Heads of a block: up to 64 share its angles (32k tokens of 40 heads: 123 us with all in a block, 129 with 20, 150 with
    // 10).  While the launch has less than two blocks per SM, first the tokens and then the heads of a block are halved.
    const long long want = 2ll * current_device_sms(nullptr);
    int hpb = a.heads < 64 ? a.heads : 64;
    auto blocks = [&] { return (a.total_tokens + a.tokens - 1) / a.tokens; };
    auto chunks = [&] { return (a.heads + hpb - 1) / hpb; };
    while (a.tokens > 1 && blocks() * chunks() < want) a.tokens = (a.tokens + 1) / 2;
    while (hpb > kThreads / (a.tokens * per_token) && hpb > 1 && blocks() * chunks() < want) hpb = (hpb + 1) / 2;
    while (chunks() > 65535) hpb <<= 1;
    if (blocks() > 0x7FFFFFFFll) return TA_ERR_TOO_LARGE;
    a.heads_per_block = hpb;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks(), (unsigned)chunks());
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(float2) * (size_t)a.tokens * a.half;
    cfg.stream = stream;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, rotary_kernel<T, V, kInterleaved>, a);
    if (e != cudaSuccess) return cuda_fail(e);
    count_launch();
    return TA_OK;
}

template <typename T, int V>
int launch_layout(RotaryArgs &a, int interleaved, cudaStream_t stream) {
    return interleaved ? launch_rotary<T, V, true>(a, stream) : launch_rotary<T, V, false>(a, stream);
}

}  // namespace

// strides of a contiguous [B][heads][N][D] tensor where the caller left them all zero
void take_strides(const long long *given, int heads, int N, int D, long long *s) {
    if (given[0] == 0 && given[1] == 0 && given[2] == 0) {
        s[0] = (long long)heads * N * D;
        s[1] = (long long)N * D;
        s[2] = D;
    } else {
        for (int i = 0; i < 3; ++i) s[i] = given[i];
    }
}

// bytes [lo, hi) a strided tensor spans
void strided_extent(const void *p, const long long *s, int B, int heads, int N, int D, int elem, uintptr_t *lo, uintptr_t *hi) {
    const long long n[3] = {B, heads, N};
    long long a = 0, b = 0;
    for (int i = 0; i < 3; ++i) {
        const long long reach = s[i] * (n[i] - 1);
        if (reach < 0) a += reach; else b += reach;
    }
    *lo = (uintptr_t)p + a * elem;
    *hi = (uintptr_t)p + (b + D) * elem;
}

// Whether two elements of a tensor that is written share an address (or may): its dimensions, by growing stride,
// have to nest.
bool strides_nest(const long long *s, int B, int heads, int N, int D) {
    long long st[3] = {s[0], s[1], s[2]}, n[3] = {B, heads, N};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (llabs(st[j]) < llabs(st[i])) {
                long long x = st[i]; st[i] = st[j]; st[j] = x;
                x = n[i]; n[i] = n[j]; n[j] = x;
            }
    long long span = D;
    for (int i = 0; i < 3; ++i) {
        if (n[i] == 1) continue;
        if (llabs(st[i]) < span) return false;
        span += llabs(st[i]) * (n[i] - 1);
    }
    return true;
}

static int rotary_impl(const ta_rotary_params &p) {
    if (!p.q || !p.q_out || !p.sections || p.B < 1 || p.H < 1 || p.N < 1 || p.D < 1 || p.H_kv < 0 || p.parts < 1)
        return TA_ERR_INVALID_ARG;
    if ((p.H_kv > 0) != (p.k != nullptr) || (p.H_kv > 0) != (p.k_out != nullptr)) return TA_ERR_INVALID_ARG;
    if ((p.positions == nullptr) == (p.dims == nullptr)) return TA_ERR_INVALID_ARG;   // one of the two
    if (p.naxes < 1 || p.naxes > TA_MAX_DIMS || !(p.base > 0.) || !isfinite(p.base)) return TA_ERR_INVALID_ARG;
    if (p.dtype != TA_DTYPE_BF16 && p.dtype != TA_DTYPE_F32) return TA_ERR_UNSUPPORTED;
    if (p.D > TA_MAX_HEAD_DIM) return TA_ERR_UNSUPPORTED;
    if ((long long)p.H + p.H_kv > 0x7FFFFFFFll) return TA_ERR_TOO_LARGE;
    if (p.D % p.parts) return TA_ERR_SHAPE;
    const int elem = p.dtype == TA_DTYPE_F32 ? 4 : 2;
    RotaryArgs a;
    a.part_dim = p.D / p.parts;
    a.parts = p.parts;
    long long pairs = 0;
    for (int i = 0; i < p.naxes; ++i) {
        if (p.sections[i] < 0) return TA_ERR_INVALID_ARG;
        pairs += p.sections[i];
    }
    if (pairs < 1 || 2 * pairs > a.part_dim) return TA_ERR_SHAPE;
    a.half = (int)pairs;
    a.small = 1;
    a.positions = p.positions;
    a.pos_axis_stride = p.pos_axis_stride;
    a.pos_batch_stride = p.pos_batch_stride;
    a.token_offset = 0;
    if (p.dims) {
        long long total = 1;
        for (int i = p.naxes - 1; i >= 0; --i) {
            if (p.dims[i] < 1) return TA_ERR_INVALID_ARG;
            a.dim[i] = p.dims[i];
            a.dim_stride[i] = total;
            if (total > (1ll << 62) / p.dims[i]) return TA_ERR_TOO_LARGE;
            total *= p.dims[i];
        }
        if (p.token_offset < 0) return TA_ERR_INVALID_ARG;
        if (p.token_offset > total - p.N) return TA_ERR_SHAPE;      // tokens outside the tensor
        a.token_offset = p.token_offset;
        a.small = total <= 0x7FFFFFFFll;
    }
    a.src[0] = p.q; a.src[1] = p.k;
    a.dst[0] = p.q_out; a.dst[1] = p.k_out;
    take_strides(p.q_strides, p.H, p.N, p.D, a.ss[0]);
    take_strides(p.q_out_strides, p.H, p.N, p.D, a.ds[0]);
    take_strides(p.k_strides, p.H_kv, p.N, p.D, a.ss[1]);
    take_strides(p.k_out_strides, p.H_kv, p.N, p.D, a.ds[1]);
    const int nt = p.H_kv > 0 ? 2 : 1;
    const int heads[2] = {p.H, p.H_kv};
    // widest vector every row and unit starts on a boundary of
    int v = 16 / elem;
    auto fits = [&](int w) {
        const int bytes = w * elem;
        if (!p.interleaved && a.half % w) return false;
        if (a.parts > 1 && a.part_dim % w) return false;
        for (int t = 0; t < nt; ++t) {
            if ((uintptr_t)a.src[t] % bytes || (uintptr_t)a.dst[t] % bytes) return false;
            const long long n[3] = {p.B, heads[t], p.N};
            for (int i = 0; i < 3; ++i)
                if (n[i] > 1 && (a.ss[t][i] % w || a.ds[t][i] % w)) return false;
        }
        return true;
    };
    for (int t = 0; t < nt; ++t) {
        if ((uintptr_t)a.src[t] % elem || (uintptr_t)a.dst[t] % elem) return TA_ERR_ALIGNMENT;
        if (!strides_nest(a.ds[t], p.B, heads[t], p.N, p.D)) return TA_ERR_INVALID_ARG;
    }
    // An output may be its own input (same address and strides); otherwise it may not share memory with an input or
    // the other output.  Interleaved views of one buffer span one another without sharing an element, so only
    // tensors without gaps are compared.
    auto dense = [&](const long long *s, int h) {
        return s[2] == p.D && s[1] == (long long)p.N * p.D && s[0] == (long long)h * p.N * p.D;
    };
    for (int i = 0; i < nt; ++i) {
        if (!dense(a.ds[i], heads[i])) continue;
        uintptr_t lo, hi, l2, h2;
        strided_extent(a.dst[i], a.ds[i], p.B, heads[i], p.N, p.D, elem, &lo, &hi);
        for (int j = 0; j < nt; ++j) {
            strided_extent(a.src[j], a.ss[j], p.B, heads[j], p.N, p.D, elem, &l2, &h2);
            if (dense(a.ss[j], heads[j]) && lo < h2 && l2 < hi && !(i == j && a.dst[i] == a.src[j])) return TA_ERR_INVALID_ARG;
            strided_extent(a.dst[j], a.ds[j], p.B, heads[j], p.N, p.D, elem, &l2, &h2);
            if (i != j && dense(a.ds[j], heads[j]) && lo < h2 && l2 < hi) return TA_ERR_INVALID_ARG;
        }
    }
    int rc = check_arch();
    if (rc != TA_OK) return rc;
    // Frequencies, in long double (64-bit mantissa): the fraction of a turn per position as 0.64 fixed point.  One power
    // per ladder and one product per pair; the products' roundings leave an angle off by pairs * position * 2^-64.
    const long double unit_turn = 1.0L / 6.283185307179586476925286766559005768L;
    int c = 0;
    long double freq = 1.0L, ratio = p.per_axis_ladder ? 1.0L : powl((long double)p.base, -1.0L / a.half);
    for (int ax = 0; ax < p.naxes; ++ax) {
        if (p.per_axis_ladder && p.sections[ax] > 0) {
            ratio = powl((long double)p.base, -1.0L / p.sections[ax]);
            freq = 1.0L;
        }
        for (int i = 0; i < p.sections[ax]; ++i, ++c, freq *= ratio) {
            long double turns = freq * unit_turn;
            if (turns >= 1.0L) turns -= floorl(turns);            // whole turns per position do not count
            a.axis[c] = (unsigned char)ax;
            a.freq[c] = (unsigned long long)(turns * 18446744073709551616.0L);
        }
    }
    a.heads_q = p.H;
    a.heads = p.H + p.H_kv;
    a.N = p.N;
    a.total_tokens = (long long)p.B * p.N;
    if (a.total_tokens > 0x7FFFFFFFll) a.small = 0;
    a.inverse = p.inverse ? 1 : 0;
    while (v > 1 && !fits(v)) v >>= 1;
    cudaStream_t stream = (cudaStream_t)p.stream;
    if (p.dtype == TA_DTYPE_F32) {
        if (v == 4) return launch_layout<float, 4>(a, p.interleaved, stream);
        if (v == 2) return launch_layout<float, 2>(a, p.interleaved, stream);
        return launch_layout<float, 1>(a, p.interleaved, stream);
    }
    if (v == 8) return launch_layout<__nv_bfloat16, 8>(a, p.interleaved, stream);
    if (v == 4) return launch_layout<__nv_bfloat16, 4>(a, p.interleaved, stream);
    if (v == 2) return launch_layout<__nv_bfloat16, 2>(a, p.interleaved, stream);
    return launch_layout<__nv_bfloat16, 1>(a, p.interleaved, stream);
}

}  // namespace ta

extern "C" int ta_rotary(const ta_rotary_params *p) {
    if (!p || p->struct_bytes != sizeof(ta_rotary_params)) return TA_ERR_INVALID_ARG;
    ta::tl_last_cuda_error = 0;
    return ta::rotary_impl(*p);
}
