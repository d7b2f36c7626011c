// Group norm with an activation, channels last, forward and backward.
//
//     xhat = (x - mean) rstd,  z = w xhat + b,  y = act(z)       mean, rstd over a group's channels and an image's pixels
//     dz = dy act'(z),  db = sum dz,  dw = sum dz xhat,  dx = rstd (w dz - mean(w dz) - xhat mean(w dz xhat))
//
// What bounds it: memory.  Forward cannot do without reading x and writing y, backward without reading x and dy and writing
// dx; the sums that every element waits for lie between.  So a cluster of blocks takes a slice of an image (all pixels, as
// many whole groups of channels as make long enough rows), each block a share of the pixels.  A block reads its share once,
// keeps the raw values in shared memory while it adds up, exchanges sums of channels with the other blocks of the
// cluster through their shared memory, and finishes from there.  What a block cannot keep it reads again.  (2 x 64 images of 112 x 112 x 64
// bf16: forward 117 .. 121 us of 64; of 56 x 56 x 256: backward 187 us of 96; 8 x 128 of 32 x 32 x 16 f32: forward 30 us of 21.)
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

constexpr int kNormThreads = 128;
constexpr int kNormWarps = kNormThreads / 32;
constexpr int kNormBlocks = 4;          // to an SM, by registers
constexpr int kApart = 64;             // pixels that a thread adds up on their own: what is rounded grows with the length of a sum
// Squares about a pivot, over those about the mean, of sums that are good enough: of R, rstd is off by up to 1.5 R roundings (R of the squares'
// sum, twice R of the square of the sum, half of which reaches the root): 4e-7.
constexpr double kMostLost = 4.0;
constexpr int kLookedAt = 4;            // pixels whose mean is the first pivot
constexpr int kWaits = 2;               // groups in which a thread's copies to shared memory are waited for
constexpr int64_t kMostSlice = 2048;    // channels of a slice, and of a group: their sums are in shared memory

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
    int64_t looked_at[kLookedAt];       // of x, in elements from an image's first
    int32_t images, channels, per_group, groups;
    int32_t slice, slices;              // channels of a slice, slices of an image
    int32_t cluster;
    int32_t share;                      // pixels of a block
    int32_t rounds, lanes, steps;       // see Share
    uint32_t per_column;                // 2^16 / columns, rounded up
    int32_t kept;                       // pixels of a thread whose values it keeps
    int32_t param_dtype, activation;
    double eps;
    double inverse;                     // of the values of a group of an image
};

__device__ __forceinline__ void store_peer(float2* p, uint32_t rank, float2 v) // where p is in another block of the cluster
{
    asm volatile("{\n\t.reg .b32 r;\n\tmapa.shared::cluster.u32 r, %0, %1;\n\tst.shared::cluster.v2.f32 [r], {%2, %3};\n\t}" ::"r"(smem_u32(p)), "r"(rank),
                 "f"(v.x), "f"(v.y)
                 : "memory");
}
__device__ __forceinline__ int cluster_at() // of the clusters along the grid's first axis
{
    int c;
    asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(c));
    return c;
}
// (threads of a warp may reach them one by one)
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

__device__ __forceinline__ float or_zero(float v) { return isfinite(v) ? v : 0.f; } // where it is no number to take sums about

// Two neighbouring channels at a time, in the register pairs that sm_100's float32 instructions for two take (as structs of two
// floats the moves between them cost what the instructions save).
using Pair = uint64_t;
__device__ __forceinline__ Pair shuffled(Pair a, int o) { return __shfl_xor_sync(0xffffffffu, a, o); }
__device__ __forceinline__ Pair pair_of(float x, float y)
{
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(x), "f"(y));
    return p;
}
__device__ __forceinline__ float2 floats_of(Pair p)
{
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p));
    return f;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b)
{
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// Values of a pixel: pairs of channels (of VEC = 1 the second one is nothing)
template <typename T, int VEC>
__device__ __forceinline__ Pair raw_pair(const Raw<T, VEC>& r, int p)
{
    if constexpr (std::is_same_v<T, __nv_bfloat16> && VEC > 1)
        return pair_of(__uint_as_float(r.w[p] << 16), __uint_as_float(r.w[p] & 0xffff0000u));
    else
        return pair_of(raw_get(r, 2 * p), VEC > 1 ? raw_get(r, VEC > 1 ? 2 * p + 1 : 0) : 0.f);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_pairs(T* to, const Pair* f)
{
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = e & 1 ? floats_of(f[e / 2]).y : floats_of(f[e / 2]).x;
    store_vec<T, VEC>(to, v);
}

// 16-bit results carry 8 or 11 bits: the fast exponential and quotient (2 units in the last place of float32 and 2^-21 |z|) do for them
template <bool FAST>
__device__ __forceinline__ float sigmoid(float z)
{
    return FAST ? __fdividef(1.f, 1.f + __expf(-z)) : 1.f / (1.f + expf(-z));
}
template <int ACT, bool FAST>
__device__ __forceinline__ float act_of(float z)
{
    if constexpr (ACT == kRelu) {
        float y;
        asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(z));
        return y;
    } else if constexpr (ACT == kSilu) {
        return z * sigmoid<FAST>(z);
    } else if constexpr (ACT == kGelu) {
        return z * (0.5f * (1.f + erff(z * 0.70710678f)));
    } else {
        return z;
    }
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
    int64_t first;                      // pixel of the block's and the lane's first step
    int steps, mine;                    // pixels of a thread at most, and of this one
    bool folds;                         // columns of a warp repeat: lanes are added up by shuffles first
    int rows;                           // partial sums of a column in shared memory

    __device__ Share(const NormArgs& a, uint32_t rank)
    {
        columns = a.slice / VEC;
        rounds = a.rounds;
        lanes = a.lanes;
        lane = rounds > 1 ? 0 : (int)(threadIdx.x * a.per_column >> 16);
        column = rounds > 1 ? (int)threadIdx.x : (int)threadIdx.x - lane * columns;
        const int64_t begin = (int64_t)a.share * rank, left = a.pixels - begin;
        const int count = (int)max((int64_t)0, min((int64_t)a.share, left)) - lane;
        first = begin + lane;
        steps = a.steps;
        mine = count > 0 ? min(steps, (int)(((uint32_t)count + lanes - 1) / (uint32_t)lanes)) : 0;
        folds = columns < 32 && (columns & (columns - 1)) == 0;
        rows = folds ? kNormWarps : lanes;
    }
    __device__ bool active(int round) const { return lane < lanes && round * kNormThreads + column < columns; }
    __device__ int channel(int round) const { return (round * kNormThreads + column) * VEC; }
    __device__ int kept(int most, int round) const { return max(0, min(most - round * steps, mine)); } // of this thread's pixels
};

__device__ __forceinline__ float2 plus(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }

// Adds up a round's sums of channels over the block and hands them to all blocks of the cluster, which keep the sums of each in `parts`.
template <int VEC>
__device__ __forceinline__ void add_up(const Share<VEC>& sh, const NormArgs& a, int round, Pair* s1, Pair* s2, float2* red, float2* parts, uint32_t rank)
{
    constexpr int NP = (VEC + 1) / 2;
    const int first = round * kNormThreads * VEC, width = (sh.rounds > 1 ? min(kNormThreads, sh.columns - round * kNormThreads) : sh.columns) * VEC;
    int row = sh.lane;
    bool writes = sh.active(round);
    if (sh.folds) {
        for (int o = sh.columns; o < 32; o <<= 1) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                s1[p] = add2(s1[p], shuffled(s1[p], o));
                s2[p] = add2(s2[p], shuffled(s2[p], o));
            }
        }
        row = (int)threadIdx.x >> 5;
        writes = (int)(threadIdx.x & 31) < sh.columns;
    }
    if (writes) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            red[row * width + sh.column * VEC + e] = e & 1 ? make_float2(floats_of(s1[e / 2]).y, floats_of(s2[e / 2]).y)
                                                           : make_float2(floats_of(s1[e / 2]).x, floats_of(s2[e / 2]).x);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += kNormThreads) {
        float2 v = red[c];
        for (int r = 1; r < sh.rows; ++r) v = plus(v, red[r * width + c]);
        for (int k = 0; k < a.cluster; ++k) {
            if (a.cluster > 1) store_peer(parts + rank * a.slice + first + c, k, v);
            else parts[first + c] = v;
        }
    }
    __syncthreads();
}

// Sums of channels over the cluster, in the order of its blocks.
__device__ __forceinline__ void exchange(const NormArgs& a, const float2* parts, float2* total)
{
    if (a.cluster > 1) {
        cluster_arrive();
        cluster_wait();
    }
    for (int c = threadIdx.x; c < a.slice; c += kNormThreads) {
        float2 v = parts[c];
        for (int k = 1; k < a.cluster; ++k) v = plus(v, parts[k * a.slice + c]);
        total[c] = v;
    }
    __syncthreads();
}

// Shared memory of a block: four numbers for each channel of the slice, their sums (of each block and of all), partial sums of
// threads, and the values that are kept.
struct Layout {
    float4* channel;
    float2 *parts, *total, *red;
    uint8_t* kept;
};
// partial sums of threads: rows of the slice's channels (Share)
__host__ __device__ constexpr int partial_sums(int vec, int slice)
{
    const int columns = slice / vec;
    if (columns >= kNormThreads) return kNormThreads * vec;
    const bool folds = columns < 32 && (columns & (columns - 1)) == 0;
    return (folds ? kNormWarps : kNormThreads / columns) * slice;
}
__host__ __device__ constexpr size_t fixed_bytes(int vec, int slice, int cluster)
{
    return ((size_t)((3 + cluster) * slice + partial_sums(vec, slice)) * sizeof(float2) + 15) & ~(size_t)15;
}
template <int VEC>
__device__ __forceinline__ Layout layout_of(uint8_t* raw, const NormArgs& a)
{
    Layout l;
    l.channel = reinterpret_cast<float4*>(raw);
    l.total = reinterpret_cast<float2*>(l.channel + a.slice);
    l.parts = l.total + a.slice;
    l.red = l.parts + a.cluster * a.slice;
    l.kept = raw + fixed_bytes(VEC, a.slice, a.cluster);
    return l;
}

// For every channel of the slice what its group says: number(channel, group, first channel to add, step to the next, sum over those
// who add together) and then use(channel, the two numbers).  Small groups are added up by each of their channels, others by a warp.
// A barrier has to follow.
template <typename Number, typename Use>
__device__ __forceinline__ void each_channel(const NormArgs& a, const Layout& l, Number number, Use use)
{
    if (a.per_group <= 8) {
        for (int c = threadIdx.x; c < a.slice; c += kNormThreads) use(c, number(c, c / a.per_group, 0, 1, [](auto v) { return v; }));
    } else {
        for (int g = threadIdx.x >> 5; g < a.slice / a.per_group; g += kNormWarps) {
            const int lane = threadIdx.x & 31;
            const float2 v = number(g * a.per_group + lane, g, lane, 32, [](auto t) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
                return t;
            });
            for (int c = g * a.per_group + lane; c < (g + 1) * a.per_group; c += 32) use(c, v);
        }
    }
}
__device__ __forceinline__ float param(const void* p, int64_t at, int32_t dtype, float other)
{
    return p ? bits_to_float(load_bits(p, at, dtype), dtype) : other;
}

// Pixels whose loads a thread has under way where it keeps no more: short accesses take few registers (us, backward,
// 3 x 24 images of 6762 x 188 bf16 in accesses of 4 bytes: 745 with 4, 545 with 8, 478 with 16)
template <typename T, int VEC>
constexpr int kAtOnce = Raw<T, VEC>::kBytes > 8 ? 4 : Raw<T, VEC>::kBytes > 4 ? 8 : 16;
// One access of a thread from memory to its slot (an address in shared memory): copied past the registers, so that a thread
// has many under way (a copy has 4 bytes at least).  Copies are committed and waited for in groups.
template <typename T, int VEC>
constexpr uint32_t kSlot = kNormThreads * Raw<T, VEC>::kBytes; // from one of a thread's slots to its next
template <typename T, int VEC>
__device__ __forceinline__ uint32_t slot_of(const uint8_t* kept, int slot)
{
    return smem_u32(kept) + slot * kSlot<T, VEC> + threadIdx.x * Raw<T, VEC>::kBytes;
}
template <typename T, int VEC>
__device__ __forceinline__ void keep(uint32_t slot, const T* from)
{
    constexpr int b = Raw<T, VEC>::kBytes;
    if constexpr (b == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot), "l"(from) : "memory");
    else if constexpr (b >= 4) asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(slot), "l"(from), "n"(b) : "memory");
    else asm volatile("st.shared.u16 [%0], %1;" ::"r"(slot), "h"(*reinterpret_cast<const unsigned short*>(from)) : "memory");
}
__device__ __forceinline__ void keep_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void keep_wait(int group) // of kWaits that were committed
{
    if (group == 0) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}
__device__ __forceinline__ int group_begin(int kept, int group) { return group == 0 ? 0 : group == 1 ? kept >> 1 : kept; }
// All copies of a thread for a round, from pixel to pixel of its column
template <typename T, int VEC>
__device__ __forceinline__ void ask(uint32_t slot, const T* from, int64_t step, int begin, int end)
{
    from += begin * step;
    slot += begin * kSlot<T, VEC>;
#pragma unroll 4
    for (int i = begin; i < end; ++i) {
        keep<T, VEC>(slot, from);
        slot += kSlot<T, VEC>;
        from += step;
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void keep_raw(const Raw<T, VEC>& r, uint32_t slot) // VEC elements of 4 bytes or more
{
    constexpr int b = Raw<T, VEC>::kBytes;
    if constexpr (b == 16) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(slot), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]) : "memory");
    else asm volatile("st.shared.b32 [%0], %1;" ::"r"(slot), "r"(r.w[0]) : "memory");
}
template <typename T, int VEC>
__device__ __forceinline__ void kept_raw(Raw<T, VEC>& r, uint32_t slot)
{
    constexpr int b = Raw<T, VEC>::kBytes;
    if constexpr (b == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "r"(slot) : "memory");
    else if constexpr (b == 8) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "r"(slot) : "memory");
    else if constexpr (b == 4) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r.w[0]) : "r"(slot) : "memory");
    else {
        unsigned short h;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(slot) : "memory");
        r.w[0] = h;
    }
}

// ---------------------------------------------------------------------------------------- forward
template <typename XT, typename YT, int VEC, int ACT>
__device__ __forceinline__ void finish_forward(const NormArgs& a, const Share<VEC>& sh, const Layout& l, const XT* x, YT* y)
{
    constexpr int NP = (VEC + 1) / 2;
    for (int round = 0; round < sh.rounds; ++round) {
        if (!sh.active(round)) continue;
        const int c0 = sh.channel(round);
        Pair m[NP], scale[NP], shift[NP]; // -mean, weight rstd, bias
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const float4 u = l.channel[c0 + 2 * p], v = VEC > 1 ? l.channel[c0 + 2 * p + 1] : u;
            m[p] = pair_of(u.x, v.x);
            scale[p] = pair_of(u.y, v.y);
            shift[p] = pair_of(u.z, v.z);
        }
        auto take = [&](const Raw<XT, VEC>& r, YT* to) {
            Pair f[NP];
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                f[p] = fma2(add2(raw_pair(r, p), m[p]), scale[p], shift[p]);
                if constexpr (ACT != kNone) {
                    const float2 z = floats_of(f[p]);
                    f[p] = pair_of(act_of<ACT, sizeof(YT) == 2>(z.x), act_of<ACT, sizeof(YT) == 2>(z.y));
                }
            }
            store_pairs<YT, VEC>(to, f);
        };
        const int kept = sh.kept(a.kept, round);
        const XT* from = x + sh.first * a.x.pixel + c0;
        YT* to = y + sh.first * a.y.pixel + c0;
        const int64_t from_step = sh.lanes * a.x.pixel, to_step = sh.lanes * a.y.pixel;
        uint32_t slot = slot_of<XT, VEC>(l.kept, round * sh.steps);
#pragma unroll 4
        for (int i = 0; i < kept; ++i) {
            Raw<XT, VEC> r;
            kept_raw(r, slot);
            take(r, to);
            to += to_step;
            slot += kSlot<XT, VEC>;
        }
        for (int i0 = kept; i0 < sh.mine; i0 += kAtOnce<XT, VEC>) {
            Raw<XT, VEC> r[kAtOnce<XT, VEC>];
#pragma unroll
            for (int j = 0; j < kAtOnce<XT, VEC>; ++j)
                if (i0 + j < sh.mine) load_raw(r[j], from + (i0 + j) * from_step);
#pragma unroll
            for (int j = 0; j < kAtOnce<XT, VEC>; ++j)
                if (i0 + j < sh.mine) {
                    take(r[j], to);
                    to += to_step;
                }
        }
    }
}

template <typename XT, typename YT, int VEC>
__global__ void __launch_bounds__(kNormThreads, kNormBlocks) forward_kernel(NormArgs a)
{
    constexpr int NP = (VEC + 1) / 2;
    extern __shared__ __align__(16) uint8_t raw[];
    const uint32_t rank = cluster_rank();
    const uint32_t item = cluster_at();                          // slices of an image run side by side: they share memory's rows
    const int row = item / (uint32_t)a.slices, slice0 = item % (uint32_t)a.slices * a.slice, worker = row / (uint32_t)a.images, image = row % (uint32_t)a.images;
    if (a.cluster > 1) cluster_arrive();
    const Share<VEC> sh(a, rank);
    const Layout l = layout_of<VEC>(raw, a);
    const XT* x = static_cast<const XT*>(a.x.data) + worker * a.x.worker + image * a.x.image + slice0;
    YT* y = static_cast<YT*>(a.y.data) + worker * a.y.worker + image * a.y.image + slice0;
    allow_next_kernel();
    wait_for_previous_kernel();
    if (a.cluster > 1) cluster_wait();                           // all blocks are there: they write to each other
    auto ask_round = [&](int round) {
        const int kept = sh.active(round) ? sh.kept(a.kept, round) : 0;
        const XT* from = x + sh.first * a.x.pixel + sh.channel(round);
        for (int g = 0; g < kWaits; ++g) {
            ask<XT, VEC>(slot_of<XT, VEC>(l.kept, round * sh.steps), from, sh.lanes * a.x.pixel, group_begin(kept, g), group_begin(kept, g + 1));
            keep_commit();
        }
    };
    const double count = (double)a.pixels;
    // Sums of x - p and (x - p)^2 with p the mean of the channel's values at a few pixels, so that float32 loses nothing where the mean is far
    // from zero.  Where these pixels turn out to lie far from the others (a border, padding, a spike) the sums are formed once
    // more, with the channels' means as p.  All blocks of a cluster have the same sums, and decide alike.
    for (int pass = 0;; ++pass) {
        for (int round = 0; round < sh.rounds; ++round) {
            if (pass == 0) ask_round(round);
            if (round == 0)
                for (int c = threadIdx.x; c < a.slice; c += kNormThreads) {
                    const int64_t at = (int64_t)worker * a.param_ld + slice0 + c;
                    l.channel[c].y = param(a.weight, at, a.param_dtype, 1.f);
                    l.channel[c].z = param(a.bias, at, a.param_dtype, 0.f);
                }
            Pair s1[NP], s2[NP], pivot[NP];
#pragma unroll
            for (int p = 0; p < NP; ++p) s1[p] = s2[p] = pair_of(0.f, 0.f);
            if (sh.active(round)) {
                const int c0 = sh.channel(round), kept = sh.kept(a.kept, round);
                const XT* from = x + sh.first * a.x.pixel + c0;
                const int64_t from_step = sh.lanes * a.x.pixel;
                if (pass == 0) {
                    Raw<XT, VEC> seen[kLookedAt];
#pragma unroll
                    for (int k = 0; k < kLookedAt; ++k) load_raw(seen[k], x + c0 + a.looked_at[k]);
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        const Pair part = pair_of(1.f / kLookedAt, 1.f / kLookedAt), none = pair_of(0.f, 0.f); // (of each: the sum of all may leave float32)
                        const Pair mean = add2(fma2(raw_pair(seen[0], p), part, fma2(raw_pair(seen[1], p), part, none)),
                                               fma2(raw_pair(seen[2], p), part, fma2(raw_pair(seen[3], p), part, none)));
                        const float2 v = floats_of(mean);
                        const float u = or_zero(v.x), w = or_zero(v.y);
                        pivot[p] = pair_of(-u, -w);
                        if (sh.lane == 0) {
                            l.channel[c0 + 2 * p].w = u;
                            if (VEC > 1) l.channel[c0 + 2 * p + 1].w = w;
                        }
                    }
                } else {
#pragma unroll
                    for (int p = 0; p < NP; ++p) pivot[p] = pair_of(-l.channel[c0 + 2 * p].w, VEC > 1 ? -l.channel[c0 + 2 * p + 1].w : 0.f);
                }
                Pair t1[NP], t2[NP];
                auto take = [&](const Raw<XT, VEC>& r) {
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        const Pair d = add2(raw_pair(r, p), pivot[p]);
                        t1[p] = add2(t1[p], d);
                        t2[p] = fma2(d, d, t2[p]);
                    }
                };
                // Four by themselves first, and up to kApart, before they are added to all: values of 16 bits are few different ones, whose squares
                // a large sum rounds in the same direction each time.
                auto take_four = [&](const Raw<XT, VEC>* r) {
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        Pair u = add2(raw_pair(r[0], p), pivot[p]), v = fma2(u, u, pair_of(0.f, 0.f));
#pragma unroll
                        for (int j = 1; j < 4; ++j) {
                            const Pair d = add2(raw_pair(r[j], p), pivot[p]);
                            u = add2(u, d);
                            v = fma2(d, d, v);
                        }
                        t1[p] = add2(t1[p], u);
                        t2[p] = add2(t2[p], v);
                    }
                };
                auto begin_apart = [&]() {
#pragma unroll
                    for (int p = 0; p < NP; ++p) t1[p] = t2[p] = pair_of(0.f, 0.f);
                };
                auto end_apart = [&]() {
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        s1[p] = add2(s1[p], t1[p]);
                        s2[p] = add2(s2[p], t2[p]);
                    }
                };
                uint32_t slot = slot_of<XT, VEC>(l.kept, round * sh.steps);
#pragma unroll 1
                for (int g = 0; g < kWaits; ++g) {
                    keep_wait(g);
                    const int last = group_begin(kept, g + 1);
#pragma unroll 1
                    for (int i = group_begin(kept, g); i < last;) {
                        const int end = min(i + kApart, last);
                        begin_apart();
#pragma unroll 1
                        for (; i + 4 <= end; i += 4) {
                            Raw<XT, VEC> r[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) kept_raw(r[j], slot + j * kSlot<XT, VEC>);
                            take_four(r);
                            slot += 4 * kSlot<XT, VEC>;
                        }
#pragma unroll 1
                        for (; i < end; ++i) {
                            Raw<XT, VEC> r;
                            kept_raw(r, slot);
                            take(r);
                            slot += kSlot<XT, VEC>;
                        }
                        end_apart();
                    }
                }
                for (int begin = kept; begin < sh.mine; begin += kApart) {
                    const int end = min(begin + kApart, sh.mine);
                    begin_apart();
                    for (int i0 = begin; i0 < end; i0 += kAtOnce<XT, VEC>) {
                        Raw<XT, VEC> r[kAtOnce<XT, VEC>];
#pragma unroll
                        for (int j = 0; j < kAtOnce<XT, VEC>; ++j)
                            if (i0 + j < end) load_raw(r[j], from + (i0 + j) * from_step);
#pragma unroll
                        for (int j = 0; j < kAtOnce<XT, VEC>; j += 4) {
                            if (i0 + j + 4 <= end) {
                                take_four(r + j);
                            } else {
#pragma unroll
                                for (int k = j; k < j + 4; ++k)
                                    if (i0 + k < end) take(r[k]);
                            }
                        }
                    }
                    end_apart();
                }
            }
            add_up(sh, a, round, s1, s2, l.red, l.parts, cluster_rank());
        }
        exchange(a, l.parts, l.total);
        // the sums of x and x^2 of a group in float64, which bears the difference of the two
        bool lost = false;
        each_channel(a, l, [&](int c, int g, int from, int step, auto sum) {
            double t1 = 0.0, t2 = 0.0, squares = 0.0;
            for (int k = g * a.per_group + from; k < (g + 1) * a.per_group; k += step) {
                const float2 v = l.total[k];
                const double p = (double)l.channel[k].w, s = (double)v.x, n = count * p;
                t1 += n + s;
                t2 = fma(p, n + 2.0 * s, t2) + (double)v.y;
                squares += (double)v.y;
            }
            t1 = sum(t1) * a.inverse;
            t2 = sum(t2) * a.inverse;
            const double var = fma(-t1, t1, t2), positive = var > 0.0 || var != var ? var : 0.0;
            if (sum(squares) * a.inverse > kMostLost * (positive + a.eps)) lost = true;
            const float2 st = make_float2((float)t1, 1.f / sqrtf((float)(positive + a.eps)));
            if (rank == 0 && c == g * a.per_group) {
                const int64_t at = (int64_t)row * a.groups + slice0 / a.per_group + g;
                if (a.mean) a.mean[at] = st.x;
                if (a.rstd) a.rstd[at] = st.y;
            }
            return st;
        }, [&](int c, float2 st) {
            l.channel[c].x = -st.x;
            l.channel[c].y *= st.y;
        });
        if (!__syncthreads_or(lost) || pass > 0) break;
        if (a.cluster > 1) {                                         // the others have read what will be written once more
            cluster_arrive();
            cluster_wait();
        }
        for (int c = threadIdx.x; c < a.slice; c += kNormThreads) l.channel[c].w = (float)((double)l.channel[c].w + (double)l.total[c].x / count);
        __syncthreads();
    }
    switch (a.activation) {
    case kRelu: finish_forward<XT, YT, VEC, kRelu>(a, sh, l, x, y); break;
    case kSilu: finish_forward<XT, YT, VEC, kSilu>(a, sh, l, x, y); break;
    case kGelu: finish_forward<XT, YT, VEC, kGelu>(a, sh, l, x, y); break;
    default: finish_forward<XT, YT, VEC, kNone>(a, sh, l, x, y); break;
    }
}

// ---------------------------------------------------------------------------------------- backward
// What the first pass wants of a channel: -mean, weight rstd, bias or (relu) a border, rstd with the sign that goes with it.  relu's slope
// is 1 where x is past the border on the side that the sign of weight rstd says, x ^ sign > border.  The border is formed in float64
// and rounded down, so that values of float32 compare with it as with the number itself, which no z near 0 in float32 does.
__device__ __forceinline__ float4 channel_of(const NormArgs& a, float2 st, int64_t at)
{
    const float w = param(a.weight, at, a.param_dtype, 1.f), b = param(a.bias, at, a.param_dtype, 0.f);
    if (a.activation != kRelu) return make_float4(-st.x, st.y * w, b, st.y);
    const double slope = (double)st.y * (double)w;
    double edge = (double)st.x - (double)b / slope;
    float border = __double2float_rd(slope < 0.0 ? -edge : edge);
    if (slope == 0.0) border = __int_as_float(b > 0.f ? 0xff800000 : 0x7f800000); // all or none
    return make_float4(-st.x, st.y * w, border, slope < 0.0 ? -st.y : st.y);
}

// dz of a thread's channels at a pixel
template <typename XT, typename YT, int VEC, int ACT>
struct Slopes {
    static constexpr int NP = (VEC + 1) / 2;
    static constexpr bool kPacked = ACT == kRelu && sizeof(XT) == 2 && std::is_same_v<XT, YT> && VEC > 1;
    Pair mean[NP], scale[NP], shift[NP];
    uint32_t border[kPacked ? NP : 1], sign[kPacked ? NP : 2 * NP];

    __device__ void load(const float4* channel)
    {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const float4 u = channel[2 * p], v = VEC > 1 ? channel[2 * p + 1] : u;
            mean[p] = pair_of(u.x, v.x);
            scale[p] = pair_of(u.y, v.y);
            shift[p] = pair_of(u.z, v.z);
            if constexpr (kPacked) {
                // past a border of float32 is past the next lower one of the 16-bit type, for its values
                XT lo, hi;
                if constexpr (std::is_same_v<XT, __half>) { lo = __float2half_rd(u.z); hi = __float2half_rd(v.z); }
                else { lo = __float2bfloat16_rd(u.z); hi = __float2bfloat16_rd(v.z); }
                border[p] = (uint32_t) * reinterpret_cast<unsigned short*>(&lo) | (uint32_t) * reinterpret_cast<unsigned short*>(&hi) << 16;
                sign[p] = (__float_as_uint(u.w) >> 16 & 0x8000u) | (__float_as_uint(v.w) & 0x80000000u);
            } else {
                sign[2 * p] = __float_as_uint(u.w) & 0x80000000u;
                sign[2 * p + 1] = __float_as_uint(v.w) & 0x80000000u;
            }
        }
    }
    // relu, 16 bits: dy where the slope is 1, in its own type
    __device__ __forceinline__ void mask(const Raw<XT, VEC>& rx, Raw<YT, VEC>& ry) const
    {
        if constexpr (kPacked) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const uint32_t turned = rx.w[p] ^ sign[p];
                uint32_t past;
                if constexpr (std::is_same_v<XT, __half>)
                    past = __hgt2_mask(*reinterpret_cast<const __half2*>(&turned), *reinterpret_cast<const __half2*>(&border[p]));
                else past = __hgt2_mask(*reinterpret_cast<const __nv_bfloat162*>(&turned), *reinterpret_cast<const __nv_bfloat162*>(&border[p]));
                ry.w[p] &= past;
            }
        }
    }
    __device__ __forceinline__ Pair dz(const Raw<XT, VEC>& rx, const Raw<YT, VEC>& ry, int p, Pair x) const
    {
        if constexpr (kPacked) {
            return raw_pair(ry, p);                              // (masked before)
        } else if constexpr (ACT == kRelu) {
            const float2 dy = floats_of(raw_pair(ry, p)), v = floats_of(x), edge = floats_of(shift[p]);
            return pair_of(__uint_as_float(__float_as_uint(v.x) ^ sign[2 * p]) > edge.x ? dy.x : 0.f,
                           __uint_as_float(__float_as_uint(v.y) ^ sign[2 * p + 1]) > edge.y ? dy.y : 0.f);
        } else if constexpr (ACT == kNone) {
            return raw_pair(ry, p);
        } else {
            constexpr bool kFast = sizeof(XT) == 2 && sizeof(YT) == 2;
            const float2 z = floats_of(fma2(add2(x, mean[p]), scale[p], shift[p])), dy = floats_of(raw_pair(ry, p));
            return pair_of(dy.x * slope_of<ACT, kFast>(z.x), dy.y * slope_of<ACT, kFast>(z.y));
        }
    }
};

template <typename XT, typename YT, int VEC>
__device__ __forceinline__ void ask_both(const NormArgs& a, const Share<VEC>& sh, const Layout& l, const XT* x, const YT* dy, int round)
{
    const int kept = sh.active(round) ? sh.kept(a.kept, round) : 0;
    const uint32_t slot_x = slot_of<XT, VEC>(l.kept, round * sh.steps);
    const uint32_t slot_y = slot_of<YT, VEC>(l.kept + (size_t)a.kept * kSlot<XT, VEC>, round * sh.steps);
    const XT* from_x = x + sh.first * a.x.pixel + sh.channel(round);
    const YT* from_y = dy + sh.first * a.y.pixel + sh.channel(round);
    for (int g = 0; g < kWaits; ++g) {
        ask<XT, VEC>(slot_x, from_x, sh.lanes * a.x.pixel, group_begin(kept, g), group_begin(kept, g + 1));
        ask<YT, VEC>(slot_y, from_y, sh.lanes * a.y.pixel, group_begin(kept, g), group_begin(kept, g + 1));
        keep_commit();
    }
}

// Both passes over a block's share: sums of dz and dz (x - mean) by channel, or dx.
template <typename XT, typename YT, int VEC, int ACT, bool FINISH>
__device__ __forceinline__ void backward_pass(const NormArgs& a, const Share<VEC>& sh, const Layout& l, const XT* x, const YT* dy, XT* dx)
{
    constexpr int NP = (VEC + 1) / 2;
    constexpr bool kFolds = sizeof(XT) == 2;
    const uint8_t* kept_dy = l.kept + (size_t)a.kept * kSlot<XT, VEC>;
    for (int round = 0; round < sh.rounds; ++round) {
        if (!FINISH && round > 0) ask_both<XT, YT, VEC>(a, sh, l, x, dy, round); // (the first round's are under way)
        Pair s1[NP], s2[NP];    // (of the second pass: what is added to weight rstd dz, -k1 - (x - mean) k2)
#pragma unroll
        for (int p = 0; p < NP; ++p) s1[p] = s2[p] = pair_of(0.f, 0.f);
        if (sh.active(round)) {
            const int c0 = sh.channel(round), kept = sh.kept(a.kept, round), slot0 = round * sh.steps;
            const XT* from_x = x + sh.first * a.x.pixel + c0;
            const YT* from_y = dy + sh.first * a.y.pixel + c0;
            const int64_t step_x = sh.lanes * a.x.pixel, step_y = sh.lanes * a.y.pixel, step_to = sh.lanes * a.dx.pixel;
            XT* to = FINISH ? dx + sh.first * a.dx.pixel + c0 : nullptr;
            Slopes<XT, YT, VEC, ACT> sl;
            sl.load(l.channel + c0);
            if (FINISH) {
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const float2 u = l.parts[c0 + 2 * p], v = VEC > 1 ? l.parts[c0 + 2 * p + 1] : u;
                    s1[p] = pair_of(u.x, v.x);
                    s2[p] = pair_of(u.y, v.y);
                    // values of 16 bits lose nothing where x - mean is multiplied out: x k2 + (mean k2 + k1)
                    if constexpr (kFolds) s1[p] = fma2(sl.mean[p], s2[p], s1[p]);
                }
            }
            auto take = [&](const Raw<XT, VEC>& rx, const Raw<YT, VEC>& ry, Pair* t1, Pair* t2) {
                Pair f[NP];
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const Pair xp = raw_pair(rx, p), dz = sl.dz(rx, ry, p, xp);
                    if (FINISH) {
                        f[p] = fma2(dz, sl.scale[p], fma2(kFolds ? xp : add2(xp, sl.mean[p]), s2[p], s1[p]));
                    } else {
                        t1[p] = add2(t1[p], dz);
                        t2[p] = fma2(dz, add2(xp, sl.mean[p]), t2[p]);
                    }
                }
                if (FINISH) {
                    store_pairs<XT, VEC>(to, f);
                    to += step_to;
                }
            };
            uint32_t slot_x = slot_of<XT, VEC>(l.kept, slot0), slot_y = slot_of<YT, VEC>(kept_dy, slot0);
#pragma unroll 1
            for (int g = 0; g < kWaits; ++g) {
                if (!FINISH) keep_wait(g);
                const int end = group_begin(kept, g + 1);
#pragma unroll 2
                for (int i = group_begin(kept, g); i < end; ++i) {
                    Raw<XT, VEC> rx;
                    Raw<YT, VEC> ry;
                    kept_raw(rx, slot_x);
                    kept_raw(ry, slot_y);
                    if constexpr (!FINISH && Slopes<XT, YT, VEC, ACT>::kPacked) {
                        sl.mask(rx, ry);
                        keep_raw(ry, slot_y);                    // for the second pass
                    }
                    take(rx, ry, s1, s2);
                    slot_x += kSlot<XT, VEC>;
                    slot_y += kSlot<YT, VEC>;
                }
            }
            for (int begin = kept; begin < sh.mine; begin += kApart) {
                Pair t1[NP], t2[NP];
#pragma unroll
                for (int p = 0; p < NP; ++p) t1[p] = t2[p] = pair_of(0.f, 0.f);
                for (int i0 = begin; i0 < min(begin + kApart, sh.mine); i0 += kAtOnce<XT, VEC>) {
                    Raw<XT, VEC> rx[kAtOnce<XT, VEC>];
                    Raw<YT, VEC> ry[kAtOnce<XT, VEC>];
#pragma unroll
                    for (int j = 0; j < kAtOnce<XT, VEC>; ++j)
                        if (i0 + j < sh.mine) {
                            load_raw(rx[j], from_x + (i0 + j) * step_x);
                            load_raw(ry[j], from_y + (i0 + j) * step_y);
                        }
#pragma unroll
                    for (int j = 0; j < kAtOnce<XT, VEC>; ++j)
                        if (i0 + j < sh.mine) {
                            sl.mask(rx[j], ry[j]);
                            take(rx[j], ry[j], t1, t2);
                        }
                }
                if (!FINISH) {
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        s1[p] = add2(s1[p], t1[p]);
                        s2[p] = add2(s2[p], t2[p]);
                    }
                }
            }
        }
        if (!FINISH) add_up(sh, a, round, s1, s2, l.red, l.parts, cluster_rank());
    }
}

template <typename XT, typename YT, int VEC, bool FINISH>
__device__ __forceinline__ void backward_pass_act(const NormArgs& a, const Share<VEC>& sh, const Layout& l, const XT* x, const YT* dy, XT* dx)
{
    switch (a.activation) {
    case kRelu: backward_pass<XT, YT, VEC, kRelu, FINISH>(a, sh, l, x, dy, dx); break;
    case kSilu: backward_pass<XT, YT, VEC, kSilu, FINISH>(a, sh, l, x, dy, dx); break;
    case kGelu: backward_pass<XT, YT, VEC, kGelu, FINISH>(a, sh, l, x, dy, dx); break;
    default: backward_pass<XT, YT, VEC, kNone, FINISH>(a, sh, l, x, dy, dx); break;
    }
}

template <typename XT, typename YT, int VEC>
__global__ void __launch_bounds__(kNormThreads, kNormBlocks) backward_kernel(NormArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    const uint32_t rank = cluster_rank();
    const uint32_t item = cluster_at();                          // slices of an image run side by side: they share memory's rows
    const int row = item / (uint32_t)a.slices, slice0 = item % (uint32_t)a.slices * a.slice, worker = row / (uint32_t)a.images, image = row % (uint32_t)a.images;
    if (a.cluster > 1) cluster_arrive();
    const Share<VEC> sh(a, rank);
    const Layout l = layout_of<VEC>(raw, a);
    const XT* x = static_cast<const XT*>(a.x.data) + worker * a.x.worker + image * a.x.image + slice0;
    const YT* dy = static_cast<const YT*>(a.y.data) + worker * a.y.worker + image * a.y.image + slice0;
    XT* dx = a.dx.data ? static_cast<XT*>(a.dx.data) + worker * a.dx.worker + image * a.dx.image + slice0 : nullptr;
    allow_next_kernel();
    wait_for_previous_kernel();
    if (a.cluster > 1) cluster_wait();                           // all blocks are there: they write to each other
    ask_both<XT, YT, VEC>(a, sh, l, x, dy, 0);
    const int64_t stats = (int64_t)row * a.groups + slice0 / a.per_group;
    for (int c = threadIdx.x; c < a.slice; c += kNormThreads) {
        const int g = c / a.per_group;
        l.channel[c] = channel_of(a, make_float2(a.mean[stats + g], a.rstd[stats + g]), (int64_t)worker * a.param_ld + slice0 + c);
    }
    __syncthreads();
    backward_pass_act<XT, YT, VEC, false>(a, sh, l, x, dy, dx);
    exchange(a, l.parts, l.total);
    if (rank == 0 && a.sums)
        for (int c = threadIdx.x; c < a.slice; c += kNormThreads)
            a.sums[(int64_t)row * a.channels + slice0 + c] = make_float2(l.total[c].x, l.total[c].y * fabsf(l.channel[c].w));
    if (dx) {
        // dx = weight rstd dz - k1 - (x - mean) k2:  k1 = mean(weight rstd dz), k2 = rstd^2 mean(weight rstd dz (x - mean))
        const float inverse = (float)a.inverse;
        each_channel(a, l, [&](int c, int g, int from, int step, auto sum) {
            float t1 = 0.f, t2 = 0.f;
            for (int k = g * a.per_group + from; k < (g + 1) * a.per_group; k += step) {
                const float2 v = l.total[k];
                const float scale = l.channel[k].y;
                t1 = fmaf(scale, v.x, t1);
                t2 = fmaf(scale, v.y, t2);
            }
            return make_float2(-sum(t1) * inverse, -sum(t2) * inverse);
        }, [&](int c, float2 k) {
            const float r = l.channel[c].w;
            l.parts[c] = make_float2(k.x, k.y * r * r);  // (the blocks' sums are done with)
        });
        __syncthreads();
        backward_pass_act<XT, YT, VEC, true>(a, sh, l, x, dy, dx);
    }
}

// dw and db: sums over a worker's images, in float64.  A block has 32 channels of a worker, its warps every eighth image.
constexpr int kGradThreads = 256;
struct GradArgs {
    const float2* sums;
    void* dweight;
    void* dbias;
    int64_t grad_ld;
    int32_t images, channels, blocks;   // blocks to a worker
    int32_t grad_dtype, accumulate;
};
__global__ void __launch_bounds__(kGradThreads) grad_kernel(GradArgs a)
{
    __shared__ double2 part[kGradThreads / 32][32];
    const int worker = blockIdx.x / (uint32_t)a.blocks, c = (int)(blockIdx.x % (uint32_t)a.blocks) * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5;
    allow_next_kernel();
    wait_for_previous_kernel();
    double2 v = make_double2(0.0, 0.0);
    if (c < a.channels) {
        const float2* s = a.sums + (int64_t)worker * a.images * a.channels + c;
#pragma unroll 4
        for (int b = warp; b < a.images; b += kGradThreads / 32) {
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
    for (int k = 0; k < kGradThreads / 32; ++k) t += warp ? part[k][threadIdx.x & 31].y : part[k][threadIdx.x & 31].x;
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
// Kept bytes of a block, at most where a cluster can be larger: three and four blocks to an SM, so that some read while others add up or
// write.  (us, forward 2 x 64 images of 112 x 112 x 64 bf16 / 8 x 128 of 32 x 32 x 16 f32: 50 KiB 116 / 37.7, 72 KiB 116 / 30.5, 100 KiB with 256 threads
// 112 / 33.4; backward 2 x 64 of 56 x 56 x 256 bf16 / 4 x 32 of 7 x 7 x 2048 f16: 34 KiB 205 / 66, 50 KiB 190 / 60, 72 KiB 197 / 62.)  And at least
// where few images ask for more blocks.
constexpr int64_t kShareForward = 72 * 1024, kShareBackward = 50 * 1024, kLeast = 32 * 1024;
// A share that is larger, in quarters of that, is kept by that much only and the rest read twice: more blocks to an SM are worth more than
// the bytes.  (us, all that fits / this: forward 6 x 17 images of 91 x 91 x 96 f32, 1.8 times, 211 / 225; 2 x 64 of 112 x 112 x 64 bf16, just
// above it, 122 / 154; backward 10 x 117 of 9717 x 8 f32, 1.5 times, 332 / 246; 4 x 64 of 6000 x 64 bf16, 1.9 times, 209 / 180; 3 x 24 of 6762 x 188, 1290 / 742.)
// Exponentials in full float32 need the warps as well.  (Forward 6 x 17 of 8281 x 96 f32, silu: 560 / 393.)
constexpr int64_t kSlackForward = 8, kSlackSmooth = 4, kSlackBackward = 5;
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
// (strides of axes with one element say nothing)
bool same_place(const choco_group_norm_params& p, int64_t images, int64_t pixels, const choco_pixels& a, const choco_pixels& b)
{
    return a.data == b.data && a.dtype == b.dtype && (p.n == 1 || a.worker == b.worker) && (images == 1 || a.image == b.image) &&
           (pixels == 1 || a.pixel == b.pixel);
}
int64_t gcd(int64_t a, int64_t b) { return b ? gcd(b, a % b) : a; }

// Whether an array that is written may share elements with one that is read: their addresses meet, they are not the same array,
// and they are not two sets of channels of one wider array.
bool mixes(const choco_group_norm_params& p, int64_t images, int64_t pixels, const choco_pixels& w, const choco_pixels& r)
{
    if (same_place(p, images, pixels, w, r)) return false;
    auto end = [&](const choco_pixels& a) {
        return (uintptr_t)a.data + (uintptr_t)(((pixels - 1) * a.pixel + (images - 1) * a.image + (p.n - 1) * a.worker + p.channels) * dtype_size(a.dtype));
    };
    if (end(w) <= (uintptr_t)r.data || end(r) <= (uintptr_t)w.data) return false;
    if (w.dtype != r.dtype) return true;
    // channels of the wider array: what all strides are multiples of (of axes with one element they say nothing)
    int64_t wide = 0;
    const struct { int64_t count, w, r; } dims[3] = {{pixels, w.pixel, r.pixel}, {images, w.image, r.image}, {p.n, w.worker, r.worker}};
    for (const auto& d : dims) {
        if (d.count == 1) continue;
        if (d.w != d.r) return true;
        wide = gcd(d.w, wide);
    }
    const int64_t apart = ((int64_t)(uintptr_t)w.data - (int64_t)(uintptr_t)r.data) / dtype_size(w.dtype);
    const int64_t to = apart < 0 ? -apart : apart;
    return to < p.channels || (wide > 0 && to + p.channels > wide);
}

// Whether rows of two arrays [n, channels] of one pitch share elements
bool rows_meet(const choco_group_norm_params& p, const void* a, const void* b, int64_t ld, int64_t size)
{
    const uintptr_t u = (uintptr_t)a, v = (uintptr_t)b;
    const uintptr_t apart = (u < v ? v - u : u - v) / (uintptr_t)size;
    if (apart < (uintptr_t)p.channels) return true;
    if (p.n == 1) return false;
    const uintptr_t rows = apart / (uintptr_t)ld, rest = apart % (uintptr_t)ld; // from a row of one to that before the other's, and on
    return (rows < (uintptr_t)p.n && rest < (uintptr_t)p.channels) || (rows + 1 < (uintptr_t)p.n && ld - (int64_t)rest < p.channels);
}

// Elements that one access may take: all arrays allow it at every pixel
bool allows(const choco_group_norm_params& p, int64_t images, int64_t pixels, const choco_pixels& a, int vec)
{
    const int64_t bytes = std::min<int64_t>(16, vec * dtype_size(a.dtype)), es = dtype_size(a.dtype);
    return aligned_to(a.data, bytes) && (pixels == 1 || a.pixel * es % bytes == 0) && (images == 1 || a.image * es % bytes == 0) &&
           (p.n == 1 || a.worker * es % bytes == 0);
}

// How a call is cut: channels of a slice, blocks of a cluster, pixels that a thread keeps.
struct Cut {
    int vec, slice, cluster, share, rounds, lanes, steps, kept;
    size_t shared;
};
// A slice is a whole number of groups and of accesses.
Cut cut_of(const choco_group_norm_params& p, int64_t images, int64_t pixels, int vec, int64_t es /* bytes of an element of x */, int64_t bytes /* kept of one */, int64_t most,
           int64_t slack)
{
    const int64_t per = p.channels / p.groups, unit = per / gcd(per, vec) * vec, rows = p.n * images;
    Cut best = {};
    best.vec = vec;
    // The widest slice whose image one block keeps within `most`; if none is, rows of 64 bytes at least and a cluster.
    const int64_t count = p.channels / unit; // slices are whole parts of it
    auto part_below = [&](int64_t u) {       // the next smaller part
        for (--u; u > 1 && count % u;) --u;
        return u;
    };
    int64_t units = part_below(std::min(count, kMostSlice / unit) + 1); // (looked for below kMostSlice, however many channels there are)
    while (units > 1 && units * unit * bytes * pixels > most && part_below(units) * unit * es >= 64) units = part_below(units);
    best.slice = (int)(units * unit);
    const int64_t slices = p.channels / best.slice, total = best.slice * bytes * pixels;
    // blocks: enough for `most` each, and for all SMs where there are few rows (but no share below kLeast)
    int cluster = 1;
    while (cluster < 8 && (total > cluster * most || (rows * slices * cluster < 296 && total > cluster * kLeast))) cluster *= 2;
    if (cluster > pixels) cluster = (int)pixels;
    best.cluster = cluster;
    const int columns = best.slice / vec;
    best.rounds = (columns + kNormThreads - 1) / kNormThreads;
    best.lanes = best.rounds > 1 ? 1 : kNormThreads / columns;
    best.share = (int)((pixels + cluster - 1) / cluster);
    best.steps = (best.share + best.lanes - 1) / best.lanes;
    const int64_t steps = (int64_t)best.rounds * best.steps;
    const size_t fixed = fixed_bytes(vec, best.slice, cluster), each = (size_t)kNormThreads * vec * bytes;
    const bool whole = (int64_t)best.share * best.slice * bytes * 4 <= most * slack;
    const int64_t room = std::min<int64_t>((int64_t)kMostShared - (int64_t)fixed, whole ? kMostShared : most);
    best.kept = (int)std::min<int64_t>(steps, std::max<int64_t>(room / (int64_t)each, 1));
    best.shared = fixed + each * best.kept;
    return best;
}

cudaError_t launch_clusters(NormKernel kernel, dim3 grid, int cluster, size_t shared, cudaStream_t st, const NormArgs& a)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
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
    a.inverse = 1.0 / ((double)pixels * a.per_group);
    // (seventeenths: pixels of different columns in images of the usual widths)
    const int at[kLookedAt] = {1, 6, 10, 15};
    for (int k = 0; k < kLookedAt; ++k) a.looked_at[k] = pixels * at[k] / 17;
    return CHOCO_OK;
}

int launch(choco_group_norm* gn, NormArgs& a, bool backward, const choco_pixels& x, const choco_pixels& y, const choco_pixels* dx, cudaStream_t st)
{
    const choco_group_norm_params& p = gn->params;
    const int vec = widest(p, a.images, a.pixels, x, y, dx);
    const Cut c = cut_of(p, a.images, a.pixels, vec, dtype_size(x.dtype), dtype_size(x.dtype) + (backward ? dtype_size(y.dtype) : 0),
                         backward ? kShareBackward : kShareForward, backward ? kSlackBackward : a.activation >= kSilu && y.dtype == CHOCO_F32 ? kSlackSmooth : kSlackForward);
    if ((int64_t)c.rounds * c.steps > 0x7fffffff) return CHOCO_ERR_TOO_LARGE; // (of arrays that repeat one pixel; steps of all rounds are counted through)
    a.slice = c.slice;
    a.slices = a.channels / c.slice;
    a.cluster = c.cluster;
    a.share = c.share;
    a.kept = c.kept;
    a.rounds = c.rounds; a.lanes = c.lanes; a.steps = c.steps;
    a.per_column = (65536u * vec + c.slice - 1) / c.slice;
    const int64_t along = (int64_t)p.n * a.images * a.slices * c.cluster;
    if (along > 0x7fffffff) return CHOCO_ERR_TOO_LARGE;
    const NormKernel kernel = kernel_of(backward, x.dtype, y.dtype, vec);
    if (gn->allowed[backward] != kernel) {
        if (status_of(cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared)) != CHOCO_OK ||
            status_of(cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributePreferredSharedMemoryCarveout, 100)) != CHOCO_OK)
            return CHOCO_ERR_CUDA;
        gn->allowed[backward] = kernel;
    }
    return status_of(launch_clusters(kernel, dim3((unsigned)along), c.cluster, c.shared, st, a));
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
    for (int64_t& at : a.looked_at) at *= a.x.pixel;
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
    if (dweight && dbias && rows_meet(p, dweight, dbias, grad_ld, dtype_size(grad_dtype))) return CHOCO_ERR_INVALID_ARG;
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
    return status_of(launch_overlapped(grad_kernel, dim3((unsigned)(g.blocks * p.n)), dim3(kGradThreads), 0, (cudaStream_t)stream, HotRange{}, g));
}

} // extern "C"
