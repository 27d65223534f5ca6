// Group normalisation of channel-last activations with an activation behind it, forward and backward.
//
// Of image n, group g holds cg = C / G neighbouring channels, M = P * cg values over P pixels:
//   mean = sum x / M,  rstd = 1 / sqrt(sum (x - mean)^2 / M + eps),  h = (x - mean) * rstd,  z = gamma_c * h + beta_c,  y = act(z)
//   dz = dy * act'(z),  A_c = sum_p dz,  B_c = sum_p dz * h   (of each image and channel)
//   dx = rstd * (gamma_c * dz - (sum_g gamma A) / M - h * (sum_g gamma B) / M),  dbeta = sum_n A,  dgamma = sum_n B
//
// Bound by memory; the statistics stand between the first read of a value and its second one.  Here the tensor is read twice: a pass that
// leaves sums of each image, chunk of pixels and channel, a small one that adds them up, and a pass that writes the result.
//
// Sums.  A thread owns a vector of channels and strides over pixels, in 32 bits: forward about a value of its own (the first it reads),
// which keeps the digits of values far from zero.  Sums of different threads meet in 64 bits, where sum x^2 / M - mean^2 loses nothing that
// matters.  The order is fixed by the sizes alone.
//
// Which side of zero a ReLU's input was on is decided exactly, for the given mean and rstd: z > 0 is x > t (x < t where gamma < 0) with
// t = mean - beta / (rstd * gamma), formed in 64 bits once per thread and channel and rounded to the next value in 32 bits that no x lies between.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "asgd_internal.h"
#include "stream.h"

namespace asgd {

namespace {

constexpr int kThreads = 256, kUnroll = 4;

// V values of type T as they lie in memory.
template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T e[V]; };

template <int ACT> __device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == kActRelu) return z < 0.f ? 0.f : z;
    if constexpr (ACT == kActSilu) return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
    return z;
}
// y = z s(z): y' = s (1 + z (1 - s))
__device__ __forceinline__ float silu_slope(float z)
{
    const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
    return s * __builtin_fmaf(z, 1.f - s, 1.f);
}

__device__ __forceinline__ float round_down(double t)
{
    const float f = (float)t;
    if (!((double)f > t)) return f;
    const uint32_t u = __float_as_uint(f);
    return __uint_as_float(f > 0.f ? u - 1 : f < 0.f ? u + 1 : 0x80000001u);
}

// What the backward pass knows of one channel of one image.
template <int ACT> struct Channel {
    float mean, a, beta;    // z = (x - mean) * a + beta
    float sign, edge;       // ReLU: z > 0 is sign * x > edge
    __device__ __forceinline__ void set(float m, float rstd, float gamma, float b)
    {
        mean = m; a = rstd * gamma; beta = b; sign = edge = 0.f;
        if constexpr (ACT == kActRelu) {
            if (gamma == 0.f) {
                edge = b > 0.f ? -1.f : 1.f;
            } else {
                sign = gamma > 0.f ? 1.f : -1.f;
                edge = round_down((double)sign * ((double)m - (double)b / ((double)rstd * (double)gamma)));
            }
        }
    }
    __device__ __forceinline__ float slope(float dy, float x) const   // dz
    {
        if constexpr (ACT == kActRelu) return sign * x > edge ? dy : 0.f;
        if constexpr (ACT == kActSilu) return dy * silu_slope(__builtin_fmaf(x - mean, a, beta));
        return dy;
    }
};

struct GnShape {
    int N, P, C, G, cg;
    long ldx, lddy, ldo;
    int chunks, pc;          // chunks of pc pixels
    int cbs, bx, rows;       // channel blocks of bx vectors, pixels that a workgroup takes at a time
    FastDiv dcbs, dchunks;
};

// Where a thread of the passes over the tensor works.
struct Place { int n, chunk, p0, p1, row, vec, c0; bool live; };
template <int V> __device__ __forceinline__ Place place(const GnShape &s)
{
    Place w;
    const unsigned r = fdiv(blockIdx.x, s.dcbs), cb = blockIdx.x - r * s.cbs;
    w.n = (int)fdiv(r, s.dchunks);
    w.chunk = (int)(r - (unsigned)w.n * s.chunks);
    w.p0 = w.chunk * s.pc;
    w.p1 = min(s.P, w.p0 + s.pc);
    w.row = (int)threadIdx.x / s.bx;
    w.vec = (int)threadIdx.x - w.row * s.bx;
    w.c0 = ((int)cb * s.bx + w.vec) * V;
    w.live = w.row < s.rows && w.c0 < s.C;
    return w;
}

template <typename T, int V> __device__ __forceinline__ Pack<T, V> load_pack(const T *p) { return *reinterpret_cast<const Pack<T, V> *>(p); }

// The two sums of every channel over the rows of a workgroup, in 64 bits: from each thread's V pairs (u, v) and what add() makes of them.
template <int V, class F>
__device__ __forceinline__ void channel_sums(const GnShape &s, const Place &w, const float (&u)[V], const float (&v)[V], double *part, F &&add)
{
    __shared__ float2 lds[kThreads * V];
    __shared__ double2 sums[kThreads];
    const int width = s.bx * V;
    if (w.row < s.rows) {
#pragma unroll
        for (int e = 0; e < V; ++e) lds[w.row * width + w.vec * V + e] = make_float2(u[e], v[e]);
    }
    __syncthreads();
    const int c_first = w.c0 - w.vec * V;     // of the channel block
    double *out = part + (((size_t)w.n * s.chunks + w.chunk) * s.C + c_first) * 2;
    const int used = min(s.rows, w.p1 - w.p0);
    const int split = width < kThreads ? kThreads / width : 1;   // threads that share a channel
    for (int base = 0; base < width; base += kThreads) {         // the same number of turns in all threads
        const int q = (int)threadIdx.x / (split > 1 ? width : kThreads), ch = split > 1 ? (int)threadIdx.x - q * width : base + (int)threadIdx.x;
        double2 t = make_double2(0, 0);
        if (q < split && ch < width)
            for (int r = q; r < used; r += split) add(t, lds[r * width + ch], r);
        if (split > 1) {
            sums[threadIdx.x] = t;
            __syncthreads();
            if (q == 0)
                for (int k = 1; k < split; ++k) { t.x += sums[k * width + ch].x; t.y += sums[k * width + ch].y; }
        }
        if (q == 0 && ch < width && c_first + ch < s.C) { out[2 * ch] = t.x; out[2 * ch + 1] = t.y; }
    }
}

// Sums of x and x^2 of each image, chunk and channel.
template <typename T, int V> __global__ __launch_bounds__(kThreads) void gn_fwd_sums_kernel(GnShape s, const T *x, double *part)
{
    const Place w = place<V>(s);
    float mean[V], m2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) mean[e] = m2[e] = 0.f;
    if (w.live && w.p0 + w.row < w.p1) {
        const T *px = x + ((size_t)w.n * s.P + w.p0 + w.row) * s.ldx + w.c0;
        const size_t step = (size_t)s.rows * s.ldx;
        float pivot[V];
        const Pack<T, V> first = load_pack<T, V>(px);
#pragma unroll
        for (int e = 0; e < V; ++e) pivot[e] = ldf(&first.e[e]);
        int count = 0;
        for (int p = w.p0 + w.row; p < w.p1; p += kUnroll * s.rows, px += kUnroll * step) {
            Pack<T, V> v[kUnroll];
#pragma unroll
            for (int k = 0; k < kUnroll; ++k)
                if (p + k * (long)s.rows < w.p1) v[k] = load_pack<T, V>(px + k * step);
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                if (p + k * (long)s.rows >= w.p1) continue;
                ++count;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float d = ldf(&v[k].e[e]) - pivot[e];
                    mean[e] += d;
                    m2[e] = __builtin_fmaf(d, d, m2[e]);
                }
            }
        }
        const float inv = 1.f / (float)count;
#pragma unroll
        for (int e = 0; e < V; ++e) {   // of this thread's values: their mean, and the squares about it
            const float d = mean[e] * inv;
            m2[e] = __builtin_fmaf(-mean[e], d, m2[e]);
            mean[e] = pivot[e] + d;
        }
    }
    const int span = w.p1 - w.p0;
    channel_sums<V>(s, w, mean, m2, part, [&](double2 &t, float2 v, int r) ASGD_INLINE {
        const double n = (double)((span - r + s.rows - 1) / s.rows), m = (double)v.x;
        t.x = __builtin_fma(n, m, t.x);
        t.y += __builtin_fma(n * m, m, (double)v.y);
    });
}

// Sums of two values over a wave, the same in all lanes.
__device__ __forceinline__ void wave_sum(double &a, double &b)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) { a += __shfl_xor(a, d); b += __shfl_xor(b, d); }
}

// One wave per image and group: its mean and rstd.
__global__ __launch_bounds__(kThreads) void gn_fwd_stats_kernel(GnShape s, const double *part, float eps, float *mean, float *rstd)
{
    const unsigned i = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (i >= (unsigned)s.N * (unsigned)s.G) return;
    const unsigned n = i / s.G, g = i - n * s.G;
    const double *p = part + ((size_t)n * s.chunks * s.C + (size_t)g * s.cg) * 2;
    double a = 0, b = 0;
    const long entries = (long)s.chunks * s.cg;
    for (long j = threadIdx.x & 63; j < entries; j += 64) {
        const long k = j / s.cg, c = j - k * s.cg;
        const double *q = p + ((size_t)k * s.C + c) * 2;
        a += q[0]; b += q[1];
    }
    wave_sum(a, b);
    if ((threadIdx.x & 63) == 0) {
        const double M = (double)s.P * s.cg, m = a / M, var = b / M - m * m;
        mean[i] = (float)m;
        rstd[i] = (float)(1.0 / __builtin_sqrt((var > 0 ? var : var == var ? 0.0 : var) + (double)eps));
    }
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void gn_fwd_apply_kernel(GnShape s, const T *x, const T *gamma, const T *beta, const float *mean, const float *rstd, T *y)
{
    const Place w = place<V>(s);
    if (!w.live) return;
    float m[V], a[V], b[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = w.c0 + e, i = w.n * s.G + c / s.cg;
        m[e] = mean[i];
        a[e] = rstd[i] * (gamma ? ldf(&gamma[c]) : 1.f);
        b[e] = beta ? ldf(&beta[c]) : 0.f;
    }
    const size_t at = (size_t)w.n * s.P + w.p0 + w.row;
    const T *px = x + at * s.ldx + w.c0;
    T *py = y + at * s.ldo + w.c0;
    const size_t step = (size_t)s.rows * s.ldx, ostep = (size_t)s.rows * s.ldo;
    for (int p = w.p0 + w.row; p < w.p1; p += kUnroll * s.rows, px += kUnroll * step, py += kUnroll * ostep) {
        Pack<T, V> v[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k)
            if (p + k * (long)s.rows < w.p1) v[k] = load_pack<T, V>(px + k * step);
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            if (p + k * (long)s.rows >= w.p1) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) stf(&v[k].e[e], activate<ACT>(__builtin_fmaf(ldf(&v[k].e[e]) - m[e], a[e], b[e])));
            *reinterpret_cast<Pack<T, V> *>(py + k * ostep) = v[k];
        }
    }
}

template <typename T, int V, int ACT>
__device__ __forceinline__ void load_channels(const GnShape &s, const Place &w, const T *gamma, const T *beta, const float *mean, const float *rstd,
                                              Channel<ACT> (&ch)[V], float (&r)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = w.c0 + e, i = w.n * s.G + c / s.cg;
        r[e] = rstd[i];
        ch[e].set(mean[i], r[e], gamma ? ldf(&gamma[c]) : 1.f, beta ? ldf(&beta[c]) : 0.f);
    }
}

// A and B of each image, chunk and channel.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void gn_bwd_sums_kernel(GnShape s, const T *dy, const T *x, const T *gamma, const T *beta, const float *mean,
                                                               const float *rstd, double *part)
{
    const Place w = place<V>(s);
    float sa[V], sb[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sa[e] = sb[e] = 0.f;
    if (w.live) {
        Channel<ACT> ch[V];
        float r[V];
        load_channels<T, V, ACT>(s, w, gamma, beta, mean, rstd, ch, r);
        const size_t at = (size_t)w.n * s.P + w.p0 + w.row;
        const T *px = x + at * s.ldx + w.c0, *pd = dy + at * s.lddy + w.c0;
        const size_t xstep = (size_t)s.rows * s.ldx, dstep = (size_t)s.rows * s.lddy;
        for (int p = w.p0 + w.row; p < w.p1; p += kUnroll * s.rows, px += kUnroll * xstep, pd += kUnroll * dstep) {
            Pack<T, V> vx[kUnroll], vd[kUnroll];
#pragma unroll
            for (int k = 0; k < kUnroll; ++k)
                if (p + k * (long)s.rows < w.p1) { vx[k] = load_pack<T, V>(px + k * xstep); vd[k] = load_pack<T, V>(pd + k * dstep); }
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                if (p + k * (long)s.rows >= w.p1) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float xv = ldf(&vx[k].e[e]), dz = ch[e].slope(ldf(&vd[k].e[e]), xv);
                    sa[e] += dz;
                    sb[e] = __builtin_fmaf(dz, xv - ch[e].mean, sb[e]);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) sb[e] *= r[e];
    }
    channel_sums<V>(s, w, sa, sb, part, [](double2 &t, float2 v, int) ASGD_INLINE { t.x += (double)v.x; t.y += (double)v.y; });
}

// The first workgroups: one wave per image and group, (sum gamma A) / M and (sum gamma B) / M into coef.  The others: dgamma and dbeta of four
// channels, 64 threads each over images and chunks.
template <typename T>
__global__ __launch_bounds__(kThreads) void gn_bwd_stats_kernel(GnShape s, const double *part, const T *gamma, float2 *coef, float *dgamma, float *dbeta,
                                                                unsigned group_blocks)
{
    __shared__ double2 lds[kThreads];
    if (blockIdx.x < group_blocks) {
        const unsigned i = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
        if (i >= (unsigned)s.N * (unsigned)s.G) return;
        const unsigned n = i / s.G, g = i - n * s.G;
        const double *p = part + ((size_t)n * s.chunks * s.C + (size_t)g * s.cg) * 2;
        double a = 0, b = 0;
        const long entries = (long)s.chunks * s.cg;
        for (long j = threadIdx.x & 63; j < entries; j += 64) {
            const long k = j / s.cg, c = j - k * s.cg;
            const double *q = p + ((size_t)k * s.C + c) * 2;
            const double w = gamma ? (double)ldf(&gamma[g * s.cg + c]) : 1.0;
            a = __builtin_fma(w, q[0], a); b = __builtin_fma(w, q[1], b);
        }
        wave_sum(a, b);
        const double M = (double)s.P * s.cg;
        if ((threadIdx.x & 63) == 0) coef[i] = make_float2((float)(a / M), (float)(b / M));
        return;
    }
    const int c = (int)(blockIdx.x - group_blocks) * 4 + ((int)threadIdx.x & 3);
    double2 t = make_double2(0, 0);
    if (c < s.C) {
        const long entries = (long)s.N * s.chunks;
        for (long j = threadIdx.x >> 2; j < entries; j += kThreads / 4) {
            const double2 v = *reinterpret_cast<const double2 *>(part + ((size_t)j * s.C + c) * 2);
            t.x += v.x; t.y += v.y;
        }
    }
    lds[threadIdx.x] = t;
    __syncthreads();
    for (int d = kThreads / 2; d >= 4; d >>= 1) {
        if ((int)threadIdx.x < d) { lds[threadIdx.x].x += lds[threadIdx.x + d].x; lds[threadIdx.x].y += lds[threadIdx.x + d].y; }
        __syncthreads();
    }
    if (threadIdx.x < 4 && c < s.C) {
        if (dbeta) dbeta[c] = (float)lds[threadIdx.x].x;
        if (dgamma) dgamma[c] = (float)lds[threadIdx.x].y;
    }
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void gn_bwd_apply_kernel(GnShape s, const T *dy, const T *x, const T *gamma, const T *beta, const float *mean,
                                                                const float *rstd, const float2 *coef, T *dx)
{
    const Place w = place<V>(s);
    if (!w.live) return;
    Channel<ACT> ch[V];
    float c0[V], c2[V];   // dx = a * dz - c0 - c2 * (x - mean)
    load_channels<T, V, ACT>(s, w, gamma, beta, mean, rstd, ch, c2);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float2 k = coef[w.n * s.G + (w.c0 + e) / s.cg];
        c0[e] = c2[e] * k.x;
        c2[e] = c2[e] * c2[e] * k.y;
    }
    const size_t at = (size_t)w.n * s.P + w.p0 + w.row;
    const T *px = x + at * s.ldx + w.c0, *pd = dy + at * s.lddy + w.c0;
    T *po = dx + at * s.ldo + w.c0;
    const size_t xstep = (size_t)s.rows * s.ldx, dstep = (size_t)s.rows * s.lddy, ostep = (size_t)s.rows * s.ldo;
    for (int p = w.p0 + w.row; p < w.p1; p += kUnroll * s.rows, px += kUnroll * xstep, pd += kUnroll * dstep, po += kUnroll * ostep) {
        Pack<T, V> vx[kUnroll], vd[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k)
            if (p + k * (long)s.rows < w.p1) { vx[k] = load_pack<T, V>(px + k * xstep); vd[k] = load_pack<T, V>(pd + k * dstep); }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            if (p + k * (long)s.rows >= w.p1) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xv = ldf(&vx[k].e[e]), dz = ch[e].slope(ldf(&vd[k].e[e]), xv);
                stf(&vd[k].e[e], __builtin_fmaf(-c2[e], xv - ch[e].mean, __builtin_fmaf(ch[e].a, dz, -c0[e])));
            }
            *reinterpret_cast<Pack<T, V> *>(po + k * ostep) = vd[k];
        }
    }
}

// ---- host side

// Chunks of pixels: 2048 workgroups in all (eight a CU), of at least 32 KiB of a tensor each.
void gn_chunks(int batch, int pixels, int channels, int dtype, int &chunks, int &pc)
{
    const long bytes = (long)channels * (long)dtype_size(dtype);
    const long least = std::max<long>(1, (32768 + bytes - 1) / bytes);
    long want = std::min<long>((2048 + batch - 1) / batch, (pixels + least - 1) / least);
    want = std::max<long>(1, want);
    pc = (int)((pixels + want - 1) / want);
    chunks = (pixels + pc - 1) / pc;
}

// Values a vector holds: as many as divide the channels and the strides and as every pointer is aligned to.
int gn_vector(int dtype, long channels, uintptr_t pointers, long strides)
{
    const int es = (int)dtype_size(dtype);
    int v = 16 / es;
    while (v > 1 && ((channels % v) || (strides % v) || (pointers % ((unsigned)v * es)))) v /= 2;
    return v;
}

bool gn_shape(const GroupNorm &q, int V, GnShape &s)
{
    s.N = q.batch; s.P = q.pixels; s.C = q.channels; s.G = q.groups; s.cg = q.channels / q.groups;
    s.ldx = q.ldx; s.lddy = q.lddy; s.ldo = q.ldo;
    gn_chunks(q.batch, q.pixels, q.channels, q.dtype, s.chunks, s.pc);
    const int cv = s.C / V;
    s.cbs = (cv + kThreads - 1) / kThreads;
    s.bx = (cv + s.cbs - 1) / s.cbs;
    s.rows = kThreads / s.bx;
    s.dcbs = make_fastdiv((uint32_t)s.cbs);
    s.dchunks = make_fastdiv((uint32_t)s.chunks);
    return (double)s.N * s.chunks * s.cbs < 2147483648.0 && (double)s.N * s.G < 2147483648.0;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

template <class F> void by_act(int act, F &&f)
{
    if (act == kActRelu) f(std::integral_constant<int, kActRelu>{});
    else if (act == kActSilu) f(std::integral_constant<int, kActSilu>{});
    else f(std::integral_constant<int, kActNone>{});
}
template <class F> void by_vector(int dtype, int v, F &&f)
{
    const auto go = [&](auto t) {
        using T = decltype(t);
        constexpr int W = 16 / (int)sizeof(T);
        if (v == W) f(t, std::integral_constant<int, W>{});
        else if (v == W / 2) f(t, std::integral_constant<int, W / 2>{});
        else if (W == 8 && v == 2) f(t, std::integral_constant<int, 2>{});
        else f(t, std::integral_constant<int, 1>{});
    };
    if (dtype == kBF16) go(bf16_t{});
    else go(float{});
}

}  // namespace

size_t group_norm_ws(int batch, int pixels, int channels, int groups, int dtype)
{
    if (batch == 0 || pixels == 0) return 256;
    int chunks, pc;
    gn_chunks(batch, pixels, channels, dtype, chunks, pc);
    return round256((size_t)batch * chunks * channels * 16) + round256((size_t)batch * groups * 8);
}

int launch_group_norm_fwd(const GroupNorm &q, const void *x, const void *gamma, const void *beta, void *y, float *mean, float *rstd, float eps, void *ws,
                          hipStream_t st)
{
    const int V = gn_vector(q.dtype, q.channels, (uintptr_t)x | (uintptr_t)y, q.ldx | q.ldo);
    GnShape s;
    if (!gn_shape(q, V, s)) return -1;
    double *part = static_cast<double *>(ws);
    float *own = reinterpret_cast<float *>(static_cast<char *>(ws) + round256((size_t)s.N * s.chunks * s.C * 16));   // where the caller wants none
    if (!mean) mean = own;
    if (!rstd) rstd = own + (size_t)s.N * s.G;
    const unsigned blocks = (unsigned)s.N * s.chunks * s.cbs;
    by_vector(q.dtype, V, [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int W = decltype(v)::value;
        const T *xx = static_cast<const T *>(x);
        hipLaunchKernelGGL((gn_fwd_sums_kernel<T, W>), dim3(blocks), dim3(kThreads), 0, st, s, xx, part);
        hipLaunchKernelGGL(gn_fwd_stats_kernel, dim3(blocks_for((size_t)s.N * s.G, kThreads / 64)), dim3(kThreads), 0, st, s, part, eps, mean, rstd);
        by_act(q.act, [&](auto a) {
            hipLaunchKernelGGL((gn_fwd_apply_kernel<T, W, decltype(a)::value>), dim3(blocks), dim3(kThreads), 0, st, s, xx, static_cast<const T *>(gamma),
                               static_cast<const T *>(beta), mean, rstd, static_cast<T *>(y));
        });
    });
    return launch_ok();
}

int launch_group_norm_bwd(const GroupNorm &q, const void *dy, const void *x, const void *gamma, const void *beta, const float *mean, const float *rstd, void *dx,
                          float *dgamma, float *dbeta, void *ws, hipStream_t st)
{
    const int V = gn_vector(q.dtype, q.channels, (uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx, q.ldx | q.lddy | q.ldo);
    GnShape s;
    if (!gn_shape(q, V, s)) return -1;
    double *part = static_cast<double *>(ws);
    float2 *coef = reinterpret_cast<float2 *>(static_cast<char *>(ws) + round256((size_t)s.N * s.chunks * s.C * 16));
    const unsigned blocks = (unsigned)s.N * s.chunks * s.cbs, group_blocks = blocks_for((size_t)s.N * s.G, kThreads / 64);
    by_vector(q.dtype, V, [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int W = decltype(v)::value;
        const T *xx = static_cast<const T *>(x), *dd = static_cast<const T *>(dy), *gg = static_cast<const T *>(gamma), *bb = static_cast<const T *>(beta);
        by_act(q.act, [&](auto a) {
            constexpr int ACT = decltype(a)::value;
            hipLaunchKernelGGL((gn_bwd_sums_kernel<T, W, ACT>), dim3(blocks), dim3(kThreads), 0, st, s, dd, xx, gg, bb, mean, rstd, part);
            hipLaunchKernelGGL(gn_bwd_stats_kernel<T>, dim3(group_blocks + (dgamma || dbeta ? blocks_for(s.C, 4) : 0)), dim3(kThreads), 0, st, s, part, gg, coef,
                               dgamma, dbeta, group_blocks);
            hipLaunchKernelGGL((gn_bwd_apply_kernel<T, W, ACT>), dim3(blocks), dim3(kThreads), 0, st, s, dd, xx, gg, bb, mean, rstd, coef, static_cast<T *>(dx));
        });
    });
    return launch_ok();
}

}  // namespace asgd
