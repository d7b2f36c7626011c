// Group norm with an activation, channels last, forward and backward.
//
//     xhat = (x - mean) rstd,  z = w xhat + b,  y = act(z)       mean, rstd over a group's channels and an image's pixels
//     dz = dy act'(z),  db = sum dz,  dw = sum dz xhat,  dx = rstd (w dz - mean(w dz) - xhat mean(w dz xhat))
//
// What bounds it: memory.  Forward cannot do without reading x and writing y, backward without reading x and dy and writing
// dx; the sums that every element waits for lie between.  So a cluster of blocks takes a slice of an image (all pixels, as
// many whole groups of channels as make long enough rows), each block a share of the pixels.  A block reads its share once,
// keeps the raw values in shared memory while it adds up, exchanges sums of channels with the other blocks of the
// cluster through their shared memory, and finishes from there.  What a block cannot keep it reads again.
//
// A thread has the same few channels throughout (one access of up to 16 bytes to a pixel), so sums and parameters of
// channels live in registers, and a value it kept is its own: no barrier between writing and reading it.
#include <algorithm>
#include <cmath>
#include <new>

#include "common.cuh"
#include "dtypes.cuh"
#include "tensor.cuh"

namespace choco {
namespace {

enum Activation { kNone, kRelu, kSilu, kGelu };

constexpr int kNormThreads = 256;
constexpr int kNormWarps = kNormThreads / 32;
constexpr int kAtOnce = 4;              // pixels whose loads a thread has under way
constexpr int64_t kMostSlice = 4096;    // channels of a slice, and of a group: their sums are in shared memory

struct Pixels {                         // element (i, b, p, c) at i worker + b image + p pixel + c
    void* data;
    int64_t worker, image, pixel;
};
struct NormArgs {
    Pixels x, y;                        // backward: y is dy
    Pixels dx;
    const void* weight;                 // null: 1
    const void* bias;                   // null: 0
    int64_t param_ld;
    float* mean;
    float* rstd;
    float2* sums;                       // backward: of the channels of every image
    int64_t pixels;
    int32_t images, channels, per_group, groups;
    int32_t slice, slices;              // channels of a slice, slices of an image
    int32_t cluster;
    int32_t kept;                       // pixels of a thread whose values it keeps
    int32_t param_dtype, activation;
    double eps;
};

__device__ __forceinline__ float2 load_peer(const float2* p, uint32_t rank) // of another block of the cluster
{
    float2 v;
    asm volatile("{\n\t.reg .b32 r;\n\tmapa.shared::cluster.u32 r, %2, %3;\n\tld.shared::cluster.v2.f32 {%0, %1}, [r];\n\t}"
                 : "=f"(v.x), "=f"(v.y)
                 : "r"(smem_u32(p)), "r"(rank)
                 : "memory");
    return v;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }

// 16-bit results carry 8 or 11 bits: the fast exponential and quotient (2 units in the last place of float32 and 2^-21 |z|) do for them
template <bool FAST>
__device__ __forceinline__ float sigmoid(float z)
{
    return FAST ? __fdividef(1.f, 1.f + __expf(-z)) : 1.f / (1.f + expf(-z));
}
template <int ACT, bool FAST>
__device__ __forceinline__ float act_of(float z)
{
    if constexpr (ACT == kRelu) return z < 0.f ? 0.f : z; // NaN stays one
    else if constexpr (ACT == kSilu) return z * sigmoid<FAST>(z);
    else if constexpr (ACT == kGelu) return z * (0.5f * (1.f + erff(z * 0.70710678f)));
    else return z;
}
template <int ACT, bool FAST>
__device__ __forceinline__ float slope_of(float z) // relu is decided elsewhere
{
    if constexpr (ACT == kSilu) {
        const float s = sigmoid<FAST>(z);
        return s * fmaf(z, 1.f - s, 1.f);
    } else if constexpr (ACT == kGelu) {
        const float e = FAST ? __expf(-0.5f * z * z) : expf(-0.5f * z * z);
        return fmaf(z * 0.39894228f, e, 0.5f * (1.f + erff(z * 0.70710678f)));
    } else {
        return 1.f;
    }
}

// The part of a block: which channels and pixels are a thread's.  A slice of more columns (of VEC channels) than the
// block has threads is gone through in rounds.
template <int VEC>
struct Share {
    int columns;                        // of the slice
    int rounds;
    int lanes;                          // threads that share a column
    int lane, column;                   // (of a round)
    int64_t begin, end;                 // pixels of the block
    int steps;                          // pixels of a thread, at most
    bool folds;                         // columns of a warp repeat: lanes are added up by shuffles first
    int rows;                           // partial sums of a column in shared memory

    __device__ Share(const NormArgs& a, uint32_t rank)
    {
        columns = a.slice / VEC;
        rounds = (columns + kNormThreads - 1) / kNormThreads;
        lanes = rounds > 1 ? 1 : kNormThreads / columns;
        lane = rounds > 1 ? 0 : (int)threadIdx.x / columns;
        column = rounds > 1 ? (int)threadIdx.x : (int)threadIdx.x % columns;
        begin = a.pixels * rank / a.cluster;
        end = a.pixels * (rank + 1) / a.cluster;
        steps = (int)((end - begin + lanes - 1) / lanes);
        folds = columns < 32 && (columns & (columns - 1)) == 0;
        rows = folds ? kNormWarps : lanes;
    }
    __device__ bool active(int round) const { return lane < lanes && round * kNormThreads + column < columns; }
    __device__ int channel(int round) const { return (round * kNormThreads + column) * VEC; }
    __device__ int64_t pixel(int step) const { return begin + lane + (int64_t)step * lanes; }
};

// Adds up a round's sums of channels over the block; `part` receives them.
template <int VEC>
__device__ __forceinline__ void add_up(const Share<VEC>& sh, const NormArgs& a, int round, float* s1, float* s2, float2* red, float2* part)
{
    const int first = round * kNormThreads * VEC, width = (sh.rounds > 1 ? min(kNormThreads, sh.columns - round * kNormThreads) : sh.columns) * VEC;
    int row = sh.lane;
    bool writes = sh.active(round);
    if (sh.folds) {
        for (int o = sh.columns; o < 32; o <<= 1)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                s1[e] += __shfl_xor_sync(0xffffffffu, s1[e], o);
                s2[e] += __shfl_xor_sync(0xffffffffu, s2[e], o);
            }
        row = (int)threadIdx.x >> 5;
        writes = (int)(threadIdx.x & 31) < sh.columns;
    }
    if (writes) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) red[row * width + sh.column * VEC + e] = make_float2(s1[e], s2[e]);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += kNormThreads) {
        float2 v = red[c];
        for (int r = 1; r < sh.rows; ++r) {
            const float2 w = red[r * width + c];
            v.x += w.x;
            v.y += w.y;
        }
        part[first + c] = v;
    }
    __syncthreads();
}

// Sums of channels over the cluster, in the order of its blocks.  Ends with an arrival at the cluster's barrier that the
// caller waits for before it leaves: until then others read `part`.
__device__ __forceinline__ void exchange(const NormArgs& a, const float2* part, float2* total)
{
    if (a.cluster > 1) {
        cluster_arrive();
        cluster_wait();
    }
    for (int c = threadIdx.x; c < a.slice; c += kNormThreads) {
        float2 v = part[c];
        if (a.cluster > 1) {
            v = make_float2(0.f, 0.f);
            for (int k = 0; k < a.cluster; ++k) {
                const float2 w = load_peer(part + c, k);
                v.x += w.x;
                v.y += w.y;
            }
        }
        total[c] = v;
    }
    if (a.cluster > 1) cluster_arrive();
    __syncthreads();
}

__device__ __forceinline__ double warp_add(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float param(const void* p, int64_t at, int32_t dtype, float other)
{
    return p ? bits_to_float(load_bits(p, at, dtype), dtype) : other;
}

// Shared memory of a block: sums of the slice's channels (own and all), two numbers for each of its groups, partial sums of
// threads, a number for each channel, and the values that are kept.
struct Layout {
    float2 *part, *total, *group, *red;
    float* first;
    uint8_t* kept;
};
__host__ __device__ constexpr size_t fixed_bytes(int vec, int slice, int per_group)
{
    return ((size_t)(2 * slice + slice / per_group + kNormThreads * vec) * sizeof(float2) + (size_t)slice * sizeof(float) + 15) & ~(size_t)15;
}
template <int VEC>
__device__ __forceinline__ Layout layout_of(uint8_t* raw, const NormArgs& a)
{
    Layout l;
    l.part = reinterpret_cast<float2*>(raw);
    l.total = l.part + a.slice;
    l.group = l.total + a.slice;
    l.red = l.group + a.slice / a.per_group;
    l.first = reinterpret_cast<float*>(l.red + kNormThreads * VEC);
    l.kept = raw + fixed_bytes(VEC, a.slice, a.per_group);
    return l;
}

template <typename T, int VEC>
__device__ __forceinline__ void keep(uint8_t* kept, int slot, const Raw<T, VEC>& r)
{
    constexpr int b = Raw<T, VEC>::kBytes;
    uint8_t* p = kept + ((size_t)slot * kNormThreads + threadIdx.x) * b;
    if constexpr (b == 16) *reinterpret_cast<uint4*>(p) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    else if constexpr (b == 8) *reinterpret_cast<uint2*>(p) = make_uint2(r.w[0], r.w[1]);
    else if constexpr (b == 4) *reinterpret_cast<uint32_t*>(p) = r.w[0];
    else *reinterpret_cast<unsigned short*>(p) = (unsigned short)r.w[0];
}
template <typename T, int VEC>
__device__ __forceinline__ void kept_raw(Raw<T, VEC>& r, const uint8_t* kept, int slot)
{
    load_raw(r, reinterpret_cast<const T*>(kept + ((size_t)slot * kNormThreads + threadIdx.x) * Raw<T, VEC>::kBytes));
}

// ---------------------------------------------------------------------------------------- forward
template <typename XT, typename YT, int VEC, int ACT>
__device__ __forceinline__ void finish_forward(const NormArgs& a, const Share<VEC>& sh, const Layout& l, const XT* x, YT* y, int worker, int slice0)
{
    for (int round = 0; round < sh.rounds; ++round) {
        if (!sh.active(round)) continue;
        const int c0 = sh.channel(round);
        float m[VEC], scale[VEC], shift[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float2 st = l.group[(c0 + e) / a.per_group];
            const int64_t at = (int64_t)worker * a.param_ld + slice0 + c0 + e;
            m[e] = st.x;
            scale[e] = st.y * param(a.weight, at, a.param_dtype, 1.f);
            shift[e] = param(a.bias, at, a.param_dtype, 0.f);
        }
        for (int i0 = 0; i0 < sh.steps; i0 += kAtOnce) {
            Raw<XT, VEC> r[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int slot = round * sh.steps + i0 + j;
                if (i0 + j < sh.steps && sh.pixel(i0 + j) < sh.end) {
                    if (slot < a.kept) kept_raw(r[j], l.kept, slot);
                    else load_raw(r[j], x + sh.pixel(i0 + j) * a.x.pixel + c0);
                }
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                if (i0 + j >= sh.steps || sh.pixel(i0 + j) >= sh.end) continue;
                float f[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = act_of<ACT, sizeof(YT) == 2>(fmaf(raw_get(r[j], e) - m[e], scale[e], shift[e]));
                store_vec<YT, VEC>(y + sh.pixel(i0 + j) * a.y.pixel + c0, f);
            }
        }
    }
}

template <typename XT, typename YT, int VEC>
__global__ void __launch_bounds__(kNormThreads) forward_kernel(NormArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    const uint32_t rank = blockIdx.x % (uint32_t)a.cluster, item = blockIdx.x / (uint32_t)a.cluster;
    const int row = (int)(item / (uint32_t)a.slices), slice0 = (int)(item % (uint32_t)a.slices) * a.slice;
    const int worker = row / a.images, image = row % a.images;
    const Share<VEC> sh(a, rank);
    const Layout l = layout_of<VEC>(raw, a);
    const XT* x = static_cast<const XT*>(a.x.data) + worker * a.x.worker + image * a.x.image + slice0;
    YT* y = static_cast<YT*>(a.y.data) + worker * a.y.worker + image * a.y.image + slice0;
    allow_next_kernel();
    wait_for_previous_kernel();
    // Sums of x - p and (x - p)^2 with p the channel's value at the image's first pixel: float32 loses nothing where
    // the mean is far from zero
    for (int round = 0; round < sh.rounds; ++round) {
        float s1[VEC], s2[VEC], p[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) s1[e] = s2[e] = 0.f;
        if (sh.active(round)) {
            const int c0 = sh.channel(round);
            Raw<XT, VEC> first;
            load_raw(first, x + c0);
            for (int i0 = 0; i0 < sh.steps; i0 += kAtOnce) {
                Raw<XT, VEC> r[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (i0 + j < sh.steps && sh.pixel(i0 + j) < sh.end) load_raw(r[j], x + sh.pixel(i0 + j) * a.x.pixel + c0);
                if (i0 == 0) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        p[e] = raw_get(first, e);
                        if (sh.lane == 0) l.first[c0 + e] = p[e];
                    }
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    if (i0 + j >= sh.steps || sh.pixel(i0 + j) >= sh.end) continue;
                    const int slot = round * sh.steps + i0 + j;
                    if (slot < a.kept) keep(l.kept, slot, r[j]);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float d = raw_get(r[j], e) - p[e];
                        s1[e] += d;
                        s2[e] = fmaf(d, d, s2[e]);
                    }
                }
            }
        }
        add_up(sh, a, round, s1, s2, l.red, l.part);
    }
    exchange(a, l.part, l.total);
    // groups: a warp each; the sums of x and x^2 in float64, which bears the difference of the two
    const double count = (double)a.pixels, inverse = 1.0 / (count * a.per_group);
    for (int g = threadIdx.x >> 5; g < a.slice / a.per_group; g += kNormWarps) {
        double t1 = 0.0, t2 = 0.0;
        for (int c = threadIdx.x & 31; c < a.per_group; c += 32) {
            const float2 v = l.total[g * a.per_group + c];
            const double p = (double)l.first[g * a.per_group + c];
            t1 += fma(count, p, (double)v.x);
            t2 += (double)v.y + p * fma(count, p, 2.0 * (double)v.x);
        }
        t1 = warp_add(t1) * inverse;
        t2 = warp_add(t2) * inverse;
        const double var = t2 - t1 * t1;
        const float2 st = make_float2((float)t1, (float)(1.0 / sqrt((var > 0.0 || var != var ? var : 0.0) + a.eps)));
        if ((threadIdx.x & 31) == 0) {
            l.group[g] = st;
            const int64_t at = (int64_t)row * a.groups + slice0 / a.per_group + g;
            if (rank == 0 && a.mean) a.mean[at] = st.x;
            if (rank == 0 && a.rstd) a.rstd[at] = st.y;
        }
    }
    __syncthreads();
    switch (a.activation) {
    case kRelu: finish_forward<XT, YT, VEC, kRelu>(a, sh, l, x, y, worker, slice0); break;
    case kSilu: finish_forward<XT, YT, VEC, kSilu>(a, sh, l, x, y, worker, slice0); break;
    case kGelu: finish_forward<XT, YT, VEC, kGelu>(a, sh, l, x, y, worker, slice0); break;
    default: finish_forward<XT, YT, VEC, kNone>(a, sh, l, x, y, worker, slice0); break;
    }
    if (a.cluster > 1) {
        __syncwarp();
        cluster_wait();
    }
}

// ---------------------------------------------------------------------------------------- backward
// Of a channel, in the registers of the threads that have it.  relu's slope is 1 where x is past `border` on the side that the sign of
// the scale says: the border is formed in float64 and rounded so that float32 values compare with it as with the exact
// one, which no z near 0 in float32 does.
struct Channel {
    float mean, scale, shift;           // z = (x - mean) scale + shift
    float border;
    uint32_t flip;                      // sign bit where x has to be below
};
__device__ __forceinline__ Channel channel_of(const NormArgs& a, float2 st, int64_t at)
{
    const float w = param(a.weight, at, a.param_dtype, 1.f), b = param(a.bias, at, a.param_dtype, 0.f);
    Channel ch;
    ch.mean = st.x;
    ch.scale = st.y * w;
    ch.shift = b;
    ch.border = __int_as_float(0x7f800000);
    ch.flip = 0;
    if (a.activation == kRelu) {
        const double slope = (double)st.y * (double)w;
        if (slope == 0.0) {
            if (b > 0.f) ch.border = __int_as_float(0xff800000);
        } else {
            // x > edge, or -x > -edge
            double edge = (double)st.x - (double)b / slope;
            if (slope < 0.0) {
                edge = -edge;
                ch.flip = 0x80000000u;
            }
            ch.border = __double2float_rd(edge);
        }
    }
    return ch;
}
template <int ACT, bool FAST>
__device__ __forceinline__ float dz_of(const Channel& ch, float x, float dy)
{
    if constexpr (ACT == kRelu) return __uint_as_float(__float_as_uint(x) ^ ch.flip) > ch.border ? dy : 0.f;
    else if constexpr (ACT == kNone) return dy;
    else return dy * slope_of<ACT, FAST>(fmaf(x - ch.mean, ch.scale, ch.shift));
}

// Both passes over a block's share: sums of dz and dz (x - mean) by channel, or dx.
template <typename XT, typename YT, int VEC, int ACT, bool FINISH>
__device__ __forceinline__ void backward_pass(const NormArgs& a, const Share<VEC>& sh, const Layout& l, const XT* x, const YT* dy, XT* dx,
                                              int row, int worker, int slice0)
{
    constexpr bool kFast = sizeof(XT) == 2 && sizeof(YT) == 2;
    uint8_t* kept_dy = l.kept + (size_t)a.kept * kNormThreads * Raw<XT, VEC>::kBytes;
    for (int round = 0; round < sh.rounds; ++round) {
        float s1[VEC], s2[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) s1[e] = s2[e] = 0.f;
        if (sh.active(round)) {
            const int c0 = sh.channel(round);
            Channel ch[VEC];
            float k1[VEC], k2[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int g = (c0 + e) / a.per_group;
                const int64_t at = (int64_t)row * a.groups + slice0 / a.per_group + g;
                const float2 st = make_float2(a.mean[at], a.rstd[at]);
                ch[e] = channel_of(a, st, (int64_t)worker * a.param_ld + slice0 + c0 + e);
                if (FINISH) {
                    k1[e] = l.group[g].x;
                    k2[e] = l.group[g].y;
                }
            }
            for (int i0 = 0; i0 < sh.steps; i0 += kAtOnce) {
                Raw<XT, VEC> rx[kAtOnce];
                Raw<YT, VEC> ry[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    const int slot = round * sh.steps + i0 + j;
                    if (i0 + j < sh.steps && sh.pixel(i0 + j) < sh.end) {
                        if (FINISH && slot < a.kept) {
                            kept_raw(rx[j], l.kept, slot);
                            kept_raw(ry[j], kept_dy, slot);
                        } else {
                            load_raw(rx[j], x + sh.pixel(i0 + j) * a.x.pixel + c0);
                            load_raw(ry[j], dy + sh.pixel(i0 + j) * a.y.pixel + c0);
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    if (i0 + j >= sh.steps || sh.pixel(i0 + j) >= sh.end) continue;
                    const int slot = round * sh.steps + i0 + j;
                    if (!FINISH && slot < a.kept) {
                        keep(l.kept, slot, rx[j]);
                        keep(kept_dy, slot, ry[j]);
                    }
                    float f[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float xe = raw_get(rx[j], e), dz = dz_of<ACT, kFast>(ch[e], xe, raw_get(ry[j], e)), d = xe - ch[e].mean;
                        if (FINISH) {
                            f[e] = fmaf(dz, ch[e].scale, -fmaf(d, k2[e], k1[e]));
                        } else {
                            s1[e] += dz;
                            s2[e] = fmaf(dz, d, s2[e]);
                        }
                    }
                    if (FINISH) store_vec<XT, VEC>(dx + sh.pixel(i0 + j) * a.dx.pixel + c0, f);
                }
            }
        }
        if (!FINISH) add_up(sh, a, round, s1, s2, l.red, l.part);
    }
}

template <typename XT, typename YT, int VEC, bool FINISH>
__device__ __forceinline__ void backward_pass_act(const NormArgs& a, const Share<VEC>& sh, const Layout& l, const XT* x, const YT* dy, XT* dx,
                                                  int row, int worker, int slice0)
{
    switch (a.activation) {
    case kRelu: backward_pass<XT, YT, VEC, kRelu, FINISH>(a, sh, l, x, dy, dx, row, worker, slice0); break;
    case kSilu: backward_pass<XT, YT, VEC, kSilu, FINISH>(a, sh, l, x, dy, dx, row, worker, slice0); break;
    case kGelu: backward_pass<XT, YT, VEC, kGelu, FINISH>(a, sh, l, x, dy, dx, row, worker, slice0); break;
    default: backward_pass<XT, YT, VEC, kNone, FINISH>(a, sh, l, x, dy, dx, row, worker, slice0); break;
    }
}

template <typename XT, typename YT, int VEC>
__global__ void __launch_bounds__(kNormThreads) backward_kernel(NormArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    const uint32_t rank = blockIdx.x % (uint32_t)a.cluster, item = blockIdx.x / (uint32_t)a.cluster;
    const int row = (int)(item / (uint32_t)a.slices), slice0 = (int)(item % (uint32_t)a.slices) * a.slice;
    const int worker = row / a.images, image = row % a.images;
    const Share<VEC> sh(a, rank);
    const Layout l = layout_of<VEC>(raw, a);
    const XT* x = static_cast<const XT*>(a.x.data) + worker * a.x.worker + image * a.x.image + slice0;
    const YT* dy = static_cast<const YT*>(a.y.data) + worker * a.y.worker + image * a.y.image + slice0;
    XT* dx = a.dx.data ? static_cast<XT*>(a.dx.data) + worker * a.dx.worker + image * a.dx.image + slice0 : nullptr;
    allow_next_kernel();
    wait_for_previous_kernel();
    backward_pass_act<XT, YT, VEC, false>(a, sh, l, x, dy, dx, row, worker, slice0);
    exchange(a, l.part, l.total);
    if (rank == 0 && a.sums)
        for (int c = threadIdx.x; c < a.slice; c += kNormThreads) {
            const float r = a.rstd[(int64_t)row * a.groups + (slice0 + c) / a.per_group];
            a.sums[(int64_t)row * a.channels + slice0 + c] = make_float2(l.total[c].x, l.total[c].y * r);
        }
    if (dx) {
        // dx = scale dz - (k1 + (x - mean) k2):  k1 = rstd mean(w dz), k2 = rstd^3 mean(w dz (x - mean))
        const double inverse = 1.0 / ((double)a.pixels * a.per_group);
        for (int g = threadIdx.x >> 5; g < a.slice / a.per_group; g += kNormWarps) {
            double t1 = 0.0, t2 = 0.0;
            for (int c = threadIdx.x & 31; c < a.per_group; c += 32) {
                const float2 v = l.total[g * a.per_group + c];
                const double w = (double)param(a.weight, (int64_t)worker * a.param_ld + slice0 + g * a.per_group + c, a.param_dtype, 1.f);
                t1 += w * (double)v.x;
                t2 += w * (double)v.y;
            }
            const double r = (double)a.rstd[(int64_t)row * a.groups + slice0 / a.per_group + g];
            t1 = warp_add(t1) * inverse * r;
            t2 = warp_add(t2) * inverse * r * r * r;
            if ((threadIdx.x & 31) == 0) l.group[g] = make_float2((float)t1, (float)t2);
        }
        __syncthreads();
        backward_pass_act<XT, YT, VEC, true>(a, sh, l, x, dy, dx, row, worker, slice0);
    }
    if (a.cluster > 1) {
        __syncwarp();
        cluster_wait();
    }
}

// dw and db: sums over a worker's images, in float64.  A block has 32 channels of a worker, its warps every eighth image.
struct GradArgs {
    const float2* sums;
    void* dweight;
    void* dbias;
    int64_t grad_ld;
    int32_t images, channels, blocks;   // blocks to a worker
    int32_t grad_dtype, accumulate;
};
__global__ void __launch_bounds__(kNormThreads) grad_kernel(GradArgs a)
{
    __shared__ double2 part[kNormWarps][32];
    const int worker = blockIdx.x / (uint32_t)a.blocks, c = (int)(blockIdx.x % (uint32_t)a.blocks) * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5;
    allow_next_kernel();
    wait_for_previous_kernel();
    double2 v = make_double2(0.0, 0.0);
    if (c < a.channels) {
        const float2* s = a.sums + (int64_t)worker * a.images * a.channels + c;
#pragma unroll 4
        for (int b = warp; b < a.images; b += kNormWarps) {
            const float2 w = s[(int64_t)b * a.channels];
            v.x += (double)w.x;
            v.y += (double)w.y;
        }
    }
    part[warp][threadIdx.x & 31] = v;
    __syncthreads();
    if (warp >= 2 || c >= a.channels) return;
    void* out = warp ? a.dweight : a.dbias; // one warp to each
    if (!out) return;
    double t = 0.0;
    for (int k = 0; k < kNormWarps; ++k) t += warp ? part[k][threadIdx.x & 31].y : part[k][threadIdx.x & 31].x;
    const int64_t at = (int64_t)worker * a.grad_ld + c;
    if (a.accumulate) t += (double)bits_to_float(load_bits(out, at, a.grad_dtype), a.grad_dtype);
    store_from_float(out, at, a.grad_dtype, (float)t);
}

// ---------------------------------------------------------------------------------------- host
using NormKernel = void (*)(NormArgs);
template <typename XT, typename YT, int VEC>
NormKernel pick(bool backward) { return backward ? (NormKernel)backward_kernel<XT, YT, VEC> : (NormKernel)forward_kernel<XT, YT, VEC>; }

// arrays of one type: accesses of 16 bytes, two elements or one; of two types: four elements or one
template <typename XT, typename YT>
NormKernel kernel_of(bool backward, int vec)
{
    if constexpr (std::is_same_v<XT, YT>) {
        constexpr int kFull = 16 / (int)sizeof(XT);
        return vec == kFull ? pick<XT, YT, kFull>(backward) : vec == 2 ? pick<XT, YT, 2>(backward) : pick<XT, YT, 1>(backward);
    } else {
        return vec == 4 ? pick<XT, YT, 4>(backward) : pick<XT, YT, 1>(backward);
    }
}
template <typename XT>
NormKernel kernel_of(bool backward, int32_t y, int vec)
{
    return y == CHOCO_F32 ? kernel_of<XT, float>(backward, vec) : y == CHOCO_BF16 ? kernel_of<XT, __nv_bfloat16>(backward, vec) : kernel_of<XT, __half>(backward, vec);
}
NormKernel kernel_of(bool backward, int32_t x, int32_t y, int vec)
{
    return x == CHOCO_F32 ? kernel_of<float>(backward, y, vec) : x == CHOCO_BF16 ? kernel_of<__nv_bfloat16>(backward, y, vec) : kernel_of<__half>(backward, y, vec);
}

constexpr int kMostShared = 227 * 1024;
constexpr int64_t kMostSize = (int64_t)1 << 40; // elements that strides may span

} // namespace
} // namespace choco

using namespace choco;

struct choco_group_norm {
    choco_group_norm_params params;
    int device;
    float2* sums;          // [n max_images, channels]
    NormKernel allowed[2]; // the last kernels that were allowed their shared memory: forward, backward
};

namespace {

bool on_device(const choco_group_norm* o)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == o->device;
}
int status_of(cudaError_t e)
{
    if (e == cudaSuccess) return CHOCO_OK;
    cudaGetLastError();
    return CHOCO_ERR_CUDA;
}

// An array as a call describes it.  `written`: no element may belong to two places.
int check(const choco_group_norm_params& p, int64_t images, int64_t pixels, const choco_pixels* a, bool written)
{
    if (!a || !a->data || !dtype_ok(a->dtype) || a->worker < 0 || a->image < 0 || a->pixel < 0) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(a->data, dtype_size(a->dtype))) return CHOCO_ERR_MISALIGNED;
    struct { int64_t count, stride; } dims[3] = {{pixels, a->pixel}, {images, a->image}, {p.n, a->worker}};
    for (auto& d : dims)
        if (d.stride > kMostSize / d.count) return CHOCO_ERR_TOO_LARGE;
    if (!written) return CHOCO_OK;
    std::sort(dims, dims + 3, [](const auto& u, const auto& v) { return u.stride < v.stride; });
    int64_t span = p.channels; // from the first to behind the last element of what smaller strides reach
    for (auto& d : dims) {
        if (d.count == 1) continue;
        if (d.stride < span) return CHOCO_ERR_INVALID_ARG;
        span += (d.count - 1) * d.stride;
    }
    return CHOCO_OK;
}
bool same_place(const choco_pixels& a, const choco_pixels& b)
{
    return a.data == b.data && a.dtype == b.dtype && a.worker == b.worker && a.image == b.image && a.pixel == b.pixel;
}
// Whether an array that is written may share elements with one that is read: their addresses meet, they are not the same array,
// and they are not two sets of channels of one wider array.
bool mixes(const choco_group_norm_params& p, int64_t images, int64_t pixels, const choco_pixels& w, const choco_pixels& r)
{
    if (same_place(w, r)) return false;
    auto end = [&](const choco_pixels& a) {
        return (uintptr_t)a.data + (uintptr_t)(((pixels - 1) * a.pixel + (images - 1) * a.image + (p.n - 1) * a.worker + p.channels) * dtype_size(a.dtype));
    };
    if (end(w) <= (uintptr_t)r.data || end(r) <= (uintptr_t)w.data) return false;
    if (w.dtype == r.dtype && w.worker == r.worker && w.image == r.image && w.pixel == r.pixel && pixels > 1) {
        const int64_t apart = ((int64_t)(uintptr_t)w.data - (int64_t)(uintptr_t)r.data) / dtype_size(w.dtype);
        const int64_t to = apart < 0 ? -apart : apart;
        bool grid = to >= p.channels && to + p.channels <= w.pixel;
        grid = grid && (images == 1 || w.image % w.pixel == 0) && (p.n == 1 || w.worker % w.pixel == 0);
        if (grid) return false;
    }
    return true;
}

// Elements that one access may take: all arrays allow it at every pixel
bool allows(const choco_group_norm_params& p, int64_t images, int64_t pixels, const choco_pixels& a, int vec)
{
    const int64_t bytes = std::min<int64_t>(16, vec * dtype_size(a.dtype)), es = dtype_size(a.dtype);
    return aligned_to(a.data, bytes) && (pixels == 1 || a.pixel * es % bytes == 0) && (images == 1 || a.image * es % bytes == 0) &&
           (p.n == 1 || a.worker * es % bytes == 0);
}

int64_t gcd(int64_t a, int64_t b) { return b ? gcd(b, a % b) : a; }

// How a call is cut: channels of a slice, blocks of a cluster, pixels that a thread keeps.
struct Cut {
    int vec, slice, cluster, kept;
    size_t shared;
};
// A slice is a whole number of groups and of accesses.
Cut cut_of(const choco_group_norm_params& p, int64_t images, int64_t pixels, int vec, int64_t bytes /* kept of an element */)
{
    const int64_t per = p.channels / p.groups, unit = per / gcd(per, vec) * vec, rows = p.n * images;
    Cut best = {};
    best.vec = vec;
    // long rows of pixels first, halved while more than eight blocks of 96 KiB would be needed and rows stay at 64 bytes
    int64_t count = p.channels / unit; // units of a slice: a divisor of this
    auto fits = [&](int64_t c) { return c * unit <= kMostSlice && c * unit * bytes * pixels <= (int64_t)8 * 96 * 1024; };
    int64_t units = count;
    while (units > 1 && !fits(units)) {
        int64_t next = units - 1;
        while (count % next) --next;
        if (units * unit <= kMostSlice && next * unit * bytes < 64) break;
        units = next;
    }
    best.slice = (int)(units * unit);
    const int64_t slices = p.channels / best.slice, total = best.slice * bytes * pixels;
    // blocks: enough for 96 KiB each, and for all SMs where there are few rows (but no share below 16 KiB)
    int cluster = 1;
    while (cluster < 8 && (total > (int64_t)cluster * 96 * 1024 || (rows * slices * cluster < 296 && total > (int64_t)cluster * 32 * 1024))) cluster *= 2;
    if (cluster > pixels) cluster = (int)pixels;
    best.cluster = cluster;
    const int columns = best.slice / vec, rounds = (columns + kNormThreads - 1) / kNormThreads, lanes = rounds > 1 ? 1 : kNormThreads / columns;
    const int64_t share = (pixels + cluster - 1) / cluster, steps = rounds * ((share + lanes - 1) / lanes);
    const size_t fixed = fixed_bytes(vec, best.slice, (int)per), each = (size_t)kNormThreads * vec * bytes;
    best.kept = (int)std::min<int64_t>(steps, ((int64_t)kMostShared - (int64_t)fixed) / (int64_t)each);
    best.shared = fixed + each * best.kept;
    return best;
}

cudaError_t launch_clusters(NormKernel kernel, int64_t blocks, int cluster, size_t shared, cudaStream_t st, const NormArgs& a)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kNormThreads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

int32_t widest(const choco_group_norm_params& p, int64_t images, int64_t pixels, const choco_pixels& x, const choco_pixels& y, const choco_pixels* dx)
{
    auto good = [&](int vec) {
        const int64_t per = p.channels / p.groups, unit = per / gcd(per, vec) * vec; // the smallest slice
        return p.channels % vec == 0 && unit <= kMostSlice && allows(p, images, pixels, x, vec) && allows(p, images, pixels, y, vec) && (!dx || allows(p, images, pixels, *dx, vec));
    };
    if (x.dtype == y.dtype) {
        const int full = (int)(16 / dtype_size(x.dtype));
        return good(full) ? full : good(2) ? 2 : 1;
    }
    return good(4) ? 4 : 1;
}

Pixels device_of(const choco_pixels& a) { return {a.data, a.worker, a.image, a.pixel}; }

int fill(const choco_group_norm* gn, int64_t images, int64_t pixels, const void* weight, const void* bias, int64_t param_ld, int32_t param_dtype, NormArgs& a)
{
    const choco_group_norm_params& p = gn->params;
    if ((weight || bias) && (!dtype_ok(param_dtype) || param_ld < 0 || param_ld > kMostSize / p.n)) return CHOCO_ERR_INVALID_ARG;
    if ((weight || bias) && p.n > 1 && param_ld > 0 && param_ld < p.channels) return CHOCO_ERR_INVALID_ARG;
    if ((weight && !aligned_to(weight, dtype_size(param_dtype))) || (bias && !aligned_to(bias, dtype_size(param_dtype)))) return CHOCO_ERR_MISALIGNED;
    a.weight = weight; a.bias = bias;
    a.param_ld = param_ld; a.param_dtype = param_dtype;
    a.pixels = pixels;
    a.images = (int32_t)images; a.channels = (int32_t)p.channels; a.groups = p.groups; a.per_group = (int32_t)(p.channels / p.groups);
    a.activation = p.activation;
    a.eps = p.eps;
    return CHOCO_OK;
}

int launch(choco_group_norm* gn, NormArgs& a, bool backward, const choco_pixels& x, const choco_pixels& y, const choco_pixels* dx, cudaStream_t st)
{
    const choco_group_norm_params& p = gn->params;
    const int vec = widest(p, a.images, a.pixels, x, y, dx);
    const Cut c = cut_of(p, a.images, a.pixels, vec, dtype_size(x.dtype) + (backward ? dtype_size(y.dtype) : 0));
    a.slice = c.slice;
    a.slices = a.channels / c.slice;
    a.cluster = c.cluster;
    a.kept = c.kept;
    const int64_t blocks = (int64_t)p.n * a.images * a.slices * c.cluster;
    if (blocks > 0x7fffffff) return CHOCO_ERR_TOO_LARGE;
    const NormKernel kernel = kernel_of(backward, x.dtype, y.dtype, vec);
    if (gn->allowed[backward] != kernel) {
        if (status_of(cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared)) != CHOCO_OK) return CHOCO_ERR_CUDA;
        gn->allowed[backward] = kernel;
    }
    return status_of(launch_clusters(kernel, blocks, c.cluster, c.shared, st, a));
}

} // namespace

extern "C" {

int choco_group_norm_init(choco_group_norm** out, const choco_group_norm_params* p)
{
    if (!out) return CHOCO_ERR_INVALID_ARG;
    *out = nullptr;
    if (!p || p->n < 1 || p->groups < 1 || p->channels < 1 || p->max_images < 0 || p->channels % p->groups) return CHOCO_ERR_INVALID_ARG;
    if (!(p->eps >= 0.0) || !std::isfinite((float)p->eps) || p->activation < 0 || p->activation > kGelu) return CHOCO_ERR_INVALID_ARG;
    if (p->n > 65535 || p->channels > 1 << 20 || p->channels / p->groups > kMostSlice || p->max_images > ((int64_t)1 << 31) / p->n - 1)
        return CHOCO_ERR_TOO_LARGE;
    choco_group_norm* o = new (std::nothrow) choco_group_norm();
    if (!o) return CHOCO_ERR_ALLOC;
    o->params = *p;
    int rc = cudaGetDevice(&o->device) == cudaSuccess ? CHOCO_OK : CHOCO_ERR_CUDA;
    const size_t bytes = sizeof(float2) * (size_t)p->n * (size_t)p->max_images * (size_t)p->channels;
    if (rc == CHOCO_OK && bytes > 0 && cudaMalloc(&o->sums, bytes) != cudaSuccess) rc = CHOCO_ERR_ALLOC;
    if (rc != CHOCO_OK) {
        cudaGetLastError();
        delete o;
        return rc;
    }
    *out = o;
    return CHOCO_OK;
}

int choco_group_norm_destroy(choco_group_norm* gn)
{
    if (!gn) return CHOCO_ERR_INVALID_ARG;
    cudaFree(gn->sums);
    delete gn;
    return CHOCO_OK;
}

int choco_group_norm_forward(choco_group_norm* gn, int64_t images, int64_t pixels, const choco_pixels* x, const choco_pixels* y, const void* weight,
                             const void* bias, int64_t param_ld, int32_t param_dtype, float* mean, float* rstd, void* stream)
{
    if (!gn || images < 0 || pixels < 0 || !on_device(gn)) return CHOCO_ERR_INVALID_ARG;
    if (images == 0 || pixels == 0) return CHOCO_OK;
    const choco_group_norm_params& p = gn->params;
    if (pixels > 0x7fffffff || images > 0x7fffffff / p.n) return CHOCO_ERR_TOO_LARGE;
    int rc = check(p, images, pixels, x, false);
    if (rc == CHOCO_OK) rc = check(p, images, pixels, y, true);
    if (rc == CHOCO_OK && mixes(p, images, pixels, *y, *x)) rc = CHOCO_ERR_INVALID_ARG;
    if (rc == CHOCO_OK && (!aligned_to(mean, 4) || !aligned_to(rstd, 4))) rc = CHOCO_ERR_MISALIGNED;
    NormArgs a = {};
    if (rc == CHOCO_OK) rc = fill(gn, images, pixels, weight, bias, param_ld, param_dtype, a);
    if (rc != CHOCO_OK) return rc;
    a.x = device_of(*x); a.y = device_of(*y);
    a.mean = mean; a.rstd = rstd;
    return launch(gn, a, false, *x, *y, nullptr, (cudaStream_t)stream);
}

int choco_group_norm_backward(choco_group_norm* gn, int64_t images, int64_t pixels, const choco_pixels* x, const choco_pixels* dy, const choco_pixels* dx,
                              const void* weight, const void* bias, int64_t param_ld, int32_t param_dtype, const float* mean, const float* rstd,
                              void* dweight, void* dbias, int64_t grad_ld, int32_t grad_dtype, int32_t accumulate, void* stream)
{
    if (!gn || images < 0 || pixels < 0 || (accumulate != 0 && accumulate != 1) || !on_device(gn)) return CHOCO_ERR_INVALID_ARG;
    const choco_group_norm_params& p = gn->params;
    const bool grads = dweight || dbias;
    if (grads && (!dtype_ok(grad_dtype) || (p.n > 1 && grad_ld < p.channels) || grad_ld > kMostSize / p.n)) return CHOCO_ERR_INVALID_ARG;
    if (grads && (!aligned_to(dweight, dtype_size(grad_dtype)) || !aligned_to(dbias, dtype_size(grad_dtype)))) return CHOCO_ERR_MISALIGNED;
    if (pixels > 0x7fffffff || images > 0x7fffffff / p.n || (grads && (images > p.max_images || (p.channels + 31) / 32 > 0x7fffffff / p.n)))
        return CHOCO_ERR_TOO_LARGE;
    const bool some = images > 0 && pixels > 0;
    NormArgs a = {};
    if (some) {
        if (!mean || !rstd) return CHOCO_ERR_INVALID_ARG;
        if (!aligned_to(mean, 4) || !aligned_to(rstd, 4)) return CHOCO_ERR_MISALIGNED;
        int rc = check(p, images, pixels, x, false);
        if (rc == CHOCO_OK) rc = check(p, images, pixels, dy, false);
        if (rc == CHOCO_OK && dx) rc = check(p, images, pixels, dx, true);
        if (rc == CHOCO_OK && dx && dx->dtype != x->dtype) rc = CHOCO_ERR_INVALID_ARG;
        if (rc == CHOCO_OK && dx && (mixes(p, images, pixels, *dx, *x) || mixes(p, images, pixels, *dx, *dy))) rc = CHOCO_ERR_INVALID_ARG;
        if (rc == CHOCO_OK) rc = fill(gn, images, pixels, weight, bias, param_ld, param_dtype, a);
        if (rc != CHOCO_OK) return rc;
        a.x = device_of(*x); a.y = device_of(*dy);
        if (dx) a.dx = device_of(*dx);
        a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
        a.sums = grads ? gn->sums : nullptr;
        if (dx || grads) rc = launch(gn, a, true, *x, *dy, dx, (cudaStream_t)stream);
        if (rc != CHOCO_OK) return rc;
    }
    if (!grads || (!some && accumulate)) return CHOCO_OK;
    const GradArgs g = {gn->sums, dweight, dbias, grad_ld, some ? (int32_t)images : 0, (int32_t)p.channels, (int32_t)((p.channels + 31) / 32), grad_dtype, accumulate};
    return status_of(launch_overlapped(grad_kernel, dim3((unsigned)(g.blocks * p.n)), dim3(kNormThreads), 0, (cudaStream_t)stream, HotRange{}, g));
}

} // extern "C"
