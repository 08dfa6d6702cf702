// Rotary positions with several axes (ta_rotary): pairs of features (x1, x2) of every q and k row turned by an
// angle that comes from one of the token's coordinates (time / height / width, or the coordinates of the
// n_1 x .. x n_m tensor),
//     y1 = x1 cos - x2 sin,   y2 = x2 cos + x1 sin,   angle = pos[axis(c)] * freq(c),
// with the opposite angle for the gradient.  The paper says a token's position is the vector of its coordinates
// (Section 3.2); here every pair of features belongs to one axis and q and k are rotated once.
//
// Bound by memory: every element is read and written once.  A thread owns V neighbouring pairs of one token, works
// out their V sines and cosines once and then walks a chunk of the heads (q's and k's alike), which all share them;
// at 8 pairs and 8 heads the angles cost about half a microsecond of issue slots per microsecond of traffic and hide
// under it.  With few tokens (decoding) the chunks shrink until the launch fills the GPU.
//
// Angles: freq(c) / (2 pi) is kept as a 64-bit fixed-point fraction of a turn, so pos * fraction modulo 2^64 is the
// angle modulo a turn, exact to pos * 2^-64 for every 32-bit position of either sign; sincospif then sees a value in
// [-1, 1).  (An fp32 product is off by milliradians at position 10^5.)
#include <cuda_bf16.h>
#include <math.h>

#include "ta_internal.h"

namespace ta {
namespace {

constexpr int kMaxPairs = TA_MAX_HEAD_DIM / 2;
constexpr int kThreads = 256;

struct RotaryArgs {
    const void *src[2];                  // q, k
    void *dst[2];
    long long ss[2][3], ds[2][3];        // strides (batch, head, token) in elements
    int heads_q, heads;                  // H, H + H_kv
    int B, N, parts, part_dim, half;     // half: rotated pairs per part
    int units;                           // units of V pairs per (token, part): rotated ones, then copies
    int heads_per_thread;
    int naxes, inverse;
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

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};

// Halves layout: a unit is V pairs (c .. c+V-1, half + c ..).  Interleaved: the 2 V neighbouring features of V pairs.
// Features behind the rotated ones are copied bit for bit, in units of 2 V features.
template <typename T, int V, bool kInterleaved>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const __grid_constant__ RotaryArgs a) {
    __shared__ unsigned long long s_freq[kMaxPairs];
    __shared__ unsigned char s_axis[kMaxPairs];
    for (int i = threadIdx.x; i < a.half; i += kThreads) {
        s_freq[i] = a.freq[i];
        s_axis[i] = a.axis[i];
    }
    __syncthreads();
    const long long per_token = (long long)a.parts * a.units;
    const long long idx = blockIdx.x * (long long)kThreads + threadIdx.x;
    const long long bt = idx / per_token;
    if (bt >= (long long)a.B * a.N) return;
    const int in_token = (int)(idx - bt * per_token);
    const int part = in_token / a.units, unit = in_token - part * a.units;
    const int b = (int)(bt / a.N), n = (int)(bt - (long long)b * a.N);
    const int c0 = unit * V;                              // first pair of the unit
    const int nrot = kInterleaved ? min(max(a.half - c0, 0), V) : (c0 < a.half ? V : 0);

    float cs[V], sn[V];
    if (nrot > 0) {
        int last_axis = -1, pos = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (i < nrot) {
                const int ax = s_axis[c0 + i];
                if (ax != last_axis) {
                    last_axis = ax;
                    if (a.positions != nullptr) {
                        pos = __ldg(a.positions + ax * a.pos_axis_stride + b * a.pos_batch_stride + n);
                    } else {
                        pos = (int)(((a.token_offset + n) / a.dim_stride[ax]) % a.dim[ax]);
                    }
                }
                const unsigned long long turns = (unsigned long long)(long long)pos * s_freq[c0 + i] + 0x80000000ull;
                sincospif((float)(int)(turns >> 32) * 4.656612873077392578125e-10f, &sn[i], &cs[i]);   // 2^-31: half turns
                if (a.inverse) sn[i] = -sn[i];
            }
        }
    }
    // feature offsets of the unit's two vectors
    long long o1, o2;
    if (kInterleaved) {
        o1 = (long long)part * a.part_dim + 2 * c0;
        o2 = o1 + V;
    } else {
        // units behind the rotated ones: 2 V features each from 2 * half on, which is 2 * c0
        o1 = (long long)part * a.part_dim + (nrot ? c0 : 2 * c0);
        o2 = nrot ? o1 + a.half : o1 + V;
    }
    using VT = Vec<T, V>;
    const int h0 = blockIdx.y * a.heads_per_thread, h1 = min(a.heads, h0 + a.heads_per_thread);
    auto source = [&](int h) {
        const int w = h >= a.heads_q ? 1 : 0;
        return reinterpret_cast<const T *>(a.src[w]) + b * a.ss[w][0] + (h - (w ? a.heads_q : 0)) * a.ss[w][1] + n * a.ss[w][2];
    };
    auto target = [&](int h) {
        const int w = h >= a.heads_q ? 1 : 0;
        return reinterpret_cast<T *>(a.dst[w]) + b * a.ds[w][0] + (h - (w ? a.heads_q : 0)) * a.ds[w][1] + n * a.ds[w][2];
    };
    // In the last unit the copied tail may be shorter than 2 V features (interleaved and copied units alike).
    const bool whole = 2 * c0 + 2 * V <= a.part_dim;
    if (!whole) {
        const int have = a.part_dim - 2 * c0;             // features left, 1 .. 2 V - 1
        for (int h = h0; h < h1; ++h) {
            const T *s = source(h) + (long long)part * a.part_dim + 2 * c0;
            T *d = target(h) + (long long)part * a.part_dim + 2 * c0;
            for (int i = 0; i < have; ++i) {
                if (i / 2 < nrot) {                       // (interleaved only)
                    if (i & 1) continue;
                    const float x1 = to_f(s[i]), x2 = to_f(s[i + 1]);
                    float c_ = 1.f, s_ = 0.f;
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (j == i / 2) { c_ = cs[j]; s_ = sn[j]; }
                    d[i] = from_f<T>(x1 * c_ - x2 * s_);
                    d[i + 1] = from_f<T>(x2 * c_ + x1 * s_);
                } else {
                    d[i] = s[i];
                }
            }
        }
        return;
    }
    constexpr int kAhead = 4;                             // heads whose loads are in flight together
    for (int h = h0; h < h1; h += kAhead) {
        VT x1[kAhead], x2[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (h + j < h1) {
                const T *s = source(h + j);
                x1[j] = *reinterpret_cast<const VT *>(s + o1);
                x2[j] = *reinterpret_cast<const VT *>(s + o2);
            }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (h + j < h1) {
                T *d = target(h + j);
                if (kInterleaved) {
                    // features 2 i, 2 i + 1 of the 2 V that x1 | x2 hold
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        if (i < nrot) {
                            T &ra = 2 * i < V ? x1[j].e[(2 * i) % V] : x2[j].e[(2 * i) % V];
                            T &rb = 2 * i + 1 < V ? x1[j].e[(2 * i + 1) % V] : x2[j].e[(2 * i + 1) % V];
                            const float va = to_f(ra), vb = to_f(rb);
                            ra = from_f<T>(va * cs[i] - vb * sn[i]);
                            rb = from_f<T>(vb * cs[i] + va * sn[i]);
                        }
                    }
                } else if (nrot) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float va = to_f(x1[j].e[i]), vb = to_f(x2[j].e[i]);
                        x1[j].e[i] = from_f<T>(va * cs[i] - vb * sn[i]);
                        x2[j].e[i] = from_f<T>(vb * cs[i] + va * sn[i]);
                    }
                }
                *reinterpret_cast<VT *>(d + o1) = x1[j];
                *reinterpret_cast<VT *>(d + o2) = x2[j];
            }
    }
}

template <typename T, int V, bool kInterleaved>
int launch_rotary(RotaryArgs &a, cudaStream_t stream) {
    // units per part: the rotated pairs (a multiple of V in the halves layout), then the copied features
    a.units = (a.part_dim + 2 * V - 1) / (2 * V);
    const long long threads = (long long)a.B * a.N * a.parts * a.units;
    const long long blocks = (threads + kThreads - 1) / kThreads;
    if (blocks > 0x7FFFFFFFll) return TA_ERR_TOO_LARGE;
    // 8 heads share a thread's angles; fewer while the launch has less than two resident waves of threads
    // (one token for each of 64 requests: 40 chunks of one head 4.1 us, 5 of eight 6.9 us)
    const long long want = 2ll * 2048 * current_device_sms(nullptr);
    int hpt = 8;
    while (hpt > 1 && threads * ((a.heads + hpt - 1) / hpt) < want) hpt >>= 1;
    while ((a.heads + hpt - 1) / hpt > 65535) hpt <<= 1;
    a.heads_per_thread = hpt;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks, (unsigned)((a.heads + hpt - 1) / hpt));
    cfg.blockDim = dim3(kThreads);
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
    a.naxes = p.naxes;
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
    // frequencies, in long double: fraction of a turn per position
    int c = 0;
    for (int ax = 0; ax < p.naxes; ++ax)
        for (int i = 0; i < p.sections[ax]; ++i, ++c) {
            const long double expo = p.per_axis_ladder ? (long double)i / p.sections[ax] : (long double)c / a.half;
            const long double turns = powl((long double)p.base, -expo) / 6.283185307179586476925286766559005768L;
            a.axis[c] = (unsigned char)ax;
            a.freq[c] = (unsigned long long)ldexpl(turns - floorl(turns), 64);
            if (turns - floorl(turns) >= 1.0L) a.freq[c] = 0;
        }
    a.heads_q = p.H;
    a.heads = p.H + p.H_kv;
    a.B = p.B; a.N = p.N;
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
