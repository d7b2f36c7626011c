// Muon: a momentum step whose update is orthogonalised matrix by matrix.
//
// With U the averaged gradient of a matrix, X_0 = U / |U| (Frobenius) and m its smaller side,
//     S = X X^T,   T = b I + c S,   B = a I + S T,   X <- B X          (`steps` times)
// takes every singular value s to s (a + b s^2 + c s^4): an odd polynomial that drives them towards one.  The
// work is three products per step: X X^T (m x m, symmetric), S T (likewise) and B X (m x k).
//
// Numbers.  The products run on the tensor cores, float16 factors and float32 sums.  X, S and B are scaled
// by powers of two into the middle of float16's range (X by 2^ex with 2^ex ~ sqrt(m k), so that its elements start
// near 1; S, T and B by 2^es ~ m, so that their diagonals do) and kept as a float16 value and, with three products, the
// float16 value of what that leaves: hi hi + hi lo + lo hi carries 22 bits.  Over five steps its roundings come to 4e-7 of the result
// (2-norm) and, the tensor cores' sums cutting bits off, 1e-6 .. 3e-6 together, as with products of plain float32.  One product carries 11
// bits, 0.0012 .. 0.0017 over five steps, as much again as rounding a result to bfloat16 (0.0017): it is taken where the caller asks for it.
//
// Layout.  X, S, T and B lie in the workspace as tiles of 128 rows x 64 halves, in the very bytes that the tensor
// cores read from shared memory (tensor.cuh), high part and low part behind one another.  A tile is one contiguous
// copy in either direction and needs no descriptor.  The side of a matrix with fewer elements is the row side (tall ones
// are turned on the way in and out), padding is zero and stays zero.  S, T and B are symmetric: only tiles on or below the
// diagonal are computed, stored and read; a product that needs one above it reads the stored one turned.
//
// What bounds it.  4096 x 4096 floats, 3.3 ms (2.9 ms in a burst of calls): the tensor cores, 76 .. 80 % of whose cycles three products
// take at the clock that the card's power leaves; 2.5 ms is their floor.  32 of 2600 x 650 bfloat16, 2.4 .. 2.8 ms (1.25 with one
// product): parts have 11 or 41 steps of K, so their beginnings and ends count (with one product 29 .. 53 % of the tensor cores' cycles are
// used, and the reads behind them come to 11 TB/s from L2), and 650 rows are three parts of 256, 1.6 times the useful operations.  The 176
// small matrices of eight ResNet-20, 87 us: the fifteen products of the longest chain, one block's.
#include <math.h>

#include <cstring>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "common.cuh"
#include "dtypes.cuh"
#include "tensor.cuh"

namespace choco {
namespace {

constexpr int kSide = 128;                         // rows of a tile, columns of a product's part
constexpr int kHalves = 64;                        // columns of a tile
constexpr uint32_t kTileBytes = kSide * kHalves * 2;
constexpr uint32_t kPieceBytes = kTileBytes / 2;   // half of its rows
constexpr int kBlock = 256;                        // matrices start on multiples of this in the momentum
constexpr int kUnit = 4096;                        // elements of one block of the momentum kernel
constexpr int kUnitThreads = 256;
constexpr int kMostSplits = 4;                     // of a part of X X^T along K
constexpr int kCutThreads = 256;                  // of the kernels that cut matrices into tiles and put them together

struct Matrix {
    void* x;
    const void* g;
    void* copy;
    int64_t x_ld, g_ld, copy_ld;
    int64_t state;          // first element in m
    int64_t at[2];          // tiles of X and of its successor, in bytes of the workspace
    int64_t s_at, t_at, b_at; // of S, T and B
    int32_t rows, cols;
    int32_t m, k;           // rows and columns of X: the smaller side and the larger
    int32_t mt, nb;         // tiles of X: rows of tiles, tiles in a row (an even number)
    int32_t ex, es;         // powers of two that X, and S and B, are scaled by
    int32_t group;
    float weight_decay, lr_scale;
    int32_t unit0, units;   // blocks of the momentum kernel (small matrices: none)
    int8_t x_dtype, g_dtype, copy_dtype;
    bool tall;              // rows > cols
    bool whole;             // rows of g behind one another
    bool aligned;           // rows of all its arrays start on 16-byte boundaries
};
struct Unit {
    int32_t matrix;
    int32_t part;           // of its units
};
struct Part {               // of a product: kSide CG rows from kSide CG i, and as many columns from kSide CG j
    int32_t matrix;
    int32_t i, j;
    int32_t begin, steps;   // of K, in steps of 64; a part of X X^T may be split along K
    int32_t split, splits;  // which of how many
    int32_t slot;           // where the sums of all its splits lie, and their counter
};
struct Block {              // a tile of X
    int32_t matrix;
    int32_t row, col;
};
struct Scale {              // of a matrix in this step: X_0 = (U first) second; both 0 where it is left alone or zero
    float first, second;
};

__device__ __forceinline__ float averaged(float m, float g, float beta, float omb) { return m * beta + g * omb; }

// N neighbouring elements, of which the first `valid` are there (others: 0): accesses of up to 16 bytes where the address allows
template <int N, typename T>
__device__ __forceinline__ void load_some(const T* p, int valid, float* v)
{
    constexpr int kAlign = N * (int)sizeof(T) < 16 ? N * (int)sizeof(T) : 16;
    if (valid >= N && ((uintptr_t)p & (kAlign - 1)) == 0) {
        Raw<T, N> r;
        load_raw(r, p);
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = raw_get(r, q);
    } else {
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = q < valid ? to_float(p[q]) : 0.f;
    }
}
// ---------------------------------------------------------------------------------------- momentum and norms
struct MomentArgs {
    const Matrix* mats;
    const Unit* units;
    float* m;               // null: no momentum, U = g
    const float* factor;    // null: 1
    double* partial;        // per unit
    uint32_t* done;         // per matrix, 0 between calls
    Scale* scale;           // per matrix
    const uint32_t* errors; // waits of this handle that ran out: nothing is written any more
    float beta, omb;
    int32_t nesterov;
};

// m = beta m + (1 - beta) c g, and the sum of squares of U by unit.  The last unit of a matrix to finish adds its
// units up in their order and forms the scale, in float64: squares of small gradients leave float32's range.
template <int THREADS, typename GT>
__device__ double moment_unit(const MomentArgs& a, const Matrix& t, int64_t begin, int64_t end, float c)
{
    double sum = 0.0;
    float* m = a.m ? a.m + t.state : nullptr;
    const GT* g = static_cast<const GT*>(t.g);
    if (t.whole) {
        const int64_t quads = end / 4 * 4;
#pragma unroll 4
        for (int64_t e = begin + 4 * (int64_t)threadIdx.x; e < quads; e += 4 * THREADS) {
            float ge[4], u[4];
            load_some<4>(g + e, 4, ge);
            if (m) {
                const float4 old = *reinterpret_cast<const float4*>(m + e);
                float v[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float gq = ge[q] * c;
                    v[q] = averaged(v[q], gq, a.beta, a.omb);
                    u[q] = a.nesterov ? averaged(v[q], gq, a.beta, a.omb) : v[q];
                }
                *reinterpret_cast<float4*>(m + e) = make_float4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) u[q] = ge[q] * c;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) sum = fma((double)u[q], (double)u[q], sum);
        }
        begin = quads > begin ? quads : begin;
    }
    // single elements, eight of a thread under way
    for (int64_t e0 = begin + threadIdx.x; e0 < end; e0 += 8 * THREADS) {
        float ge[8], me[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t e = e0 + j * THREADS;
            ge[j] = me[j] = 0.f;
            if (e < end) {
                const int64_t row = (uint32_t)e / (uint32_t)t.cols, col = (uint32_t)e % (uint32_t)t.cols;
                ge[j] = to_float(g[t.g_ld == t.cols ? e : row * t.g_ld + col]);
                if (m) me[j] = m[e];
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t e = e0 + j * THREADS;
            if (e >= end) break;
            float u = ge[j] * c;
            if (m) {
                const float v = averaged(me[j], u, a.beta, a.omb);
                m[e] = v;
                u = a.nesterov ? averaged(v, u, a.beta, a.omb) : v;
            }
            sum = fma((double)u, (double)u, sum);
        }
    }
    return sum;
}

template <int THREADS>
__device__ __forceinline__ double moment_unit(const MomentArgs& a, const Matrix& t, int64_t begin, int64_t end, float c)
{
    if (t.g_dtype == CHOCO_F32) return moment_unit<THREADS, float>(a, t, begin, end, c);
    if (t.g_dtype == CHOCO_BF16) return moment_unit<THREADS, __nv_bfloat16>(a, t, begin, end, c);
    return moment_unit<THREADS, __half>(a, t, begin, end, c);
}
// X_0's scale from the sum of squares
__device__ __forceinline__ Scale scale_of(double sum, int ex)
{
    Scale s = {0.f, 0.f};
    if (sum != 0.0) {
        const double f = ldexp(1.0, ex) / sqrt(sum);     // from 1e-44 to 1e49: in two factors where float32 ends
        const double pre = f > 1e30 ? 0x1p100 : f < 1e-30 ? 0x1p-100 : 1.0;
        s.first = (float)pre;
        s.second = isfinite(sum) ? (float)(f / pre) : __int_as_float(0x7fc00000); // (not 0, which stands for matrices left alone)
    }
    return s;
}

template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* ws) // the sum is thread 0's
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) ws[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < THREADS / 32; ++w) s += ws[w];
    __syncthreads();
    return s;
}

__global__ void __launch_bounds__(kUnitThreads) moment_kernel(MomentArgs a)
{
    __shared__ double ws[kUnitThreads / 32];
    __shared__ bool last;
    const Unit un = a.units[blockIdx.x];
    const Matrix& t = a.mats[un.matrix];
    allow_next_kernel();
    wait_for_previous_kernel();
    const float c = a.factor ? a.factor[t.group] : 1.f;
    const bool skip = !isfinite(c) || __ldcg(a.errors) != 0;
    double sum = 0.0;
    if (!skip) {
        const int64_t begin = (int64_t)un.part * kUnit, all = (int64_t)t.rows * t.cols;
        const int64_t end = begin + kUnit < all ? begin + kUnit : all;
        sum = moment_unit<kUnitThreads>(a, t, begin, end, c);
    }
    sum = block_sum<kUnitThreads>(sum, ws);
    if (threadIdx.x == 0) {
        a.partial[t.unit0 + un.part] = sum;
        __threadfence();
        last = atomicAdd(a.done + un.matrix, 1u) == (uint32_t)t.units - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (int i = threadIdx.x; i < t.units; i += kUnitThreads) sum += __ldcg(a.partial + t.unit0 + i);
    sum = block_sum<kUnitThreads>(sum, ws);
    if (threadIdx.x == 0) {
        a.done[un.matrix] = 0;
        a.scale[un.matrix] = scale_of(skip ? 0.0 : sum, t.ex);
    }
}

// ---------------------------------------------------------------------------------------- matrices <-> tiles
struct TileArgs {
    const Matrix* mats;
    const Block* blocks;
    uint8_t* work;
    const Scale* scale;
    const uint32_t* errors;
    float* m;
    const float* factor;
    float beta, omb, lr;
    int32_t nesterov;
    int32_t planes;         // parts of the tiles that are read (X_0 has two)
    int32_t which;          // of the two X
    int32_t update;         // x -= lr .. O (a step), or x = O
};

__device__ __forceinline__ uint32_t piece_at(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }

__device__ __forceinline__ uint32_t two_halves(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// eight values as float16, and what that leaves as float16
__device__ __forceinline__ void split8(const float* v, uint4& hi, uint4& lo, bool want_lo)
{
    uint32_t h[4], l[4] = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        h[q] = two_halves(v[2 * q], v[2 * q + 1]);
        if (want_lo) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[q]));
            l[q] = two_halves(v[2 * q] - f.x, v[2 * q + 1] - f.y);
        }
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ void join8(uint4 hi, uint4 lo, float* v, bool has_lo)
{
    const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[q]));
        if (has_lo) {
            const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&l[q]));
            f.x += r.x;
            f.y += r.y;
        }
        v[2 * q] = f.x;
        v[2 * q + 1] = f.y;
    }
}

template <int N>
__device__ __forceinline__ void load_some(const void* p, int64_t at, int32_t dtype, int valid, float* v)
{
    if (dtype == CHOCO_F32) load_some<N>(static_cast<const float*>(p) + at, valid, v);
    else if (dtype == CHOCO_BF16) load_some<N>(static_cast<const __nv_bfloat16*>(p) + at, valid, v);
    else load_some<N>(static_cast<const __half*>(p) + at, valid, v);
}
template <int N, typename T>
__device__ __forceinline__ void store_some(T* p, int valid, const float* v)
{
    constexpr int kAlign = N * (int)sizeof(T) < 16 ? N * (int)sizeof(T) : 16;
    if (valid >= N && ((uintptr_t)p & (kAlign - 1)) == 0) {
        store_vec<T, N>(p, v);
    } else {
#pragma unroll
        for (int q = 0; q < N; ++q)
            if (q < valid) p[q] = from_float<T>(v[q]);
    }
}
template <int N>
__device__ __forceinline__ void store_some(void* p, int64_t at, int32_t dtype, int valid, const float* v)
{
    if (dtype == CHOCO_F32) store_some<N>(static_cast<float*>(p) + at, valid, v);
    else if (dtype == CHOCO_BF16) store_some<N>(static_cast<__nv_bfloat16*>(p) + at, valid, v);
    else store_some<N>(static_cast<__half*>(p) + at, valid, v);
}
// U from (row, col) on
template <int N>
__device__ __forceinline__ void update_some(const TileArgs& a, const Matrix& t, int row, int col, int valid, float c, float* u)
{
    load_some<N>(t.g, (int64_t)row * t.g_ld + col, t.g_dtype, valid, u);
#pragma unroll
    for (int q = 0; q < N; ++q) u[q] *= c;
    if (!a.m) return;
    float m[N];
    load_some<N>(a.m + t.state + (int64_t)row * t.cols + col, valid, m);
#pragma unroll
    for (int q = 0; q < N; ++q) u[q] = a.nesterov ? averaged(m[q], u[q], a.beta, a.omb) : m[q];
}
// x (and its copy) from (row, col) on
template <int N>
__device__ __forceinline__ void apply_some(const TileArgs& a, const Matrix& t, int row, int col, int valid, float* o)
{
    const int64_t at = (int64_t)row * t.x_ld + col;
    if (a.update) {
        float x[N];
        load_some<N>(t.x, at, t.x_dtype, valid, x);
        const float lr = a.lr * t.lr_scale, decay = a.lr * t.weight_decay;
#pragma unroll
        for (int q = 0; q < N; ++q) o[q] = x[q] - (o[q] * lr + x[q] * decay);
        if (t.copy) store_some<N>(t.copy, (int64_t)row * t.copy_ld + col, t.copy_dtype, valid, o);
    }
    store_some<N>(t.x, at, t.x_dtype, valid, o);
}

// A turned tile in shared memory, columns as rows: a gap after every eight elements keeps threads that take eight each on banks of their own
constexpr int kTurnRow = kSide + kSide / 8 + 1;
__device__ __forceinline__ int turned_at(int row) { return row + (row >> 3); }

// Where a tile's matrix has its elements, N neighbours to a thread: along rows of the tile, or along its columns where the matrix is tall
template <int N, typename Work>
__device__ __forceinline__ void each_place(const Matrix& t, int row0, int col0, Work work) // work(row of the tile, column, how many are there)
{
    constexpr int kAlong = kSide / N, kAcross = kHalves / N, kUnroll = 16 / N;
#pragma unroll kUnroll
    for (int e = threadIdx.x; e < kSide * kHalves / N; e += kCutThreads) {
        const int r = t.tall ? e % kAlong * N : e / kAcross, q = t.tall ? e / kAlong : e % kAcross * N;
        work(r, q, row0 + r < t.m && col0 + q < t.k ? (t.tall ? t.m - row0 - r : t.k - col0 - q) : 0);
    }
}
template <int N>
__device__ __forceinline__ void apply_turned(const TileArgs& a, const Matrix& t, int row0, int col0, float (*turn)[kTurnRow])
{
    each_place<N>(t, row0, col0, [&](int r, int q, int valid) {
        if (valid <= 0) return;
        float o[N];
#pragma unroll
        for (int k = 0; k < N; ++k) o[k] = turn[t.tall ? q : q + k][turned_at(t.tall ? r + k : r)];
        apply_some<N>(a, t, t.tall ? col0 + q : row0 + r, t.tall ? row0 + r : col0 + q, valid, o);
    });
}

// A tile of X_0: 128 rows x 64 columns of U; those of tall matrices go by way of shared memory.
__global__ void __launch_bounds__(kCutThreads) cut_kernel(TileArgs a)
{
    __shared__ float turn[kHalves][kTurnRow];
    const Block bl = a.blocks[blockIdx.x];
    const Matrix& t = a.mats[bl.matrix];
    const int row0 = bl.row * kSide, col0 = bl.col * kHalves;
    allow_next_kernel();
    wait_for_previous_kernel();
    const Scale sc = a.scale[bl.matrix];
    const bool live = sc.second != 0.f; // (true for NaN)
    const float c = a.factor ? a.factor[t.group] : 1.f;
    if (live && t.tall) {
        each_place<8>(t, row0, col0, [&](int r, int q, int valid) {
            float u[8] = {};
            if (valid > 0) update_some<8>(a, t, col0 + q, row0 + r, valid, c, u);
#pragma unroll
            for (int k = 0; k < 8; ++k) turn[q][turned_at(r + k)] = u[k];
        });
        __syncthreads();
    }
    uint8_t* to = a.work + t.at[0] + ((int64_t)bl.row * t.nb + bl.col) * 2 * kTileBytes;
    const int piece = threadIdx.x & 7, col = col0 + piece * 8;
#pragma unroll 2
    for (int r = threadIdx.x >> 3; r < kSide; r += kCutThreads / 8) {
        float v[8] = {};
        if (live && t.tall) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = turn[piece * 8 + q][turned_at(r)];
        } else if (live && row0 + r < t.m && col < t.k) {
            update_some<8>(a, t, row0 + r, col, t.k - col, c, v);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = v[q] * sc.first * sc.second;
        uint4 hi, lo;
        split8(v, hi, lo, true);
        *reinterpret_cast<uint4*>(to + piece_at(r, piece)) = hi;
        *reinterpret_cast<uint4*>(to + kTileBytes + piece_at(r, piece)) = lo;
    }
}

// The last X of a matrix, tile by tile, to where it goes: by way of shared memory where the matrix is tall, and in pairs of elements, so that a
// warp's accesses lie side by side, where rows are off 16-byte boundaries (32 of 2600 x 650 bf16: 123 -> 100 us).
__global__ void __launch_bounds__(kCutThreads) apply_kernel(TileArgs a)
{
    __shared__ float turn[kHalves][kTurnRow];
    const Block bl = a.blocks[blockIdx.x];
    const Matrix& t = a.mats[bl.matrix];
    const int row0 = bl.row * kSide, col0 = bl.col * kHalves;
    allow_next_kernel();
    wait_for_previous_kernel();
    if ((a.factor && !isfinite(a.factor[t.group])) || __ldcg(a.errors) != 0) return;
    const uint8_t* from = a.work + t.at[a.which] + ((int64_t)bl.row * t.nb + bl.col) * a.planes * kTileBytes;
    const float unscale = exp2f((float)-t.ex);
    const bool straight = t.aligned && !t.tall;
    const int piece = threadIdx.x & 7, col = col0 + piece * 8;
#pragma unroll 2
    for (int r = threadIdx.x >> 3; r < kSide; r += kCutThreads / 8) {
        const uint4 hi = *reinterpret_cast<const uint4*>(from + piece_at(r, piece));
        const uint4 lo = a.planes == 2 ? *reinterpret_cast<const uint4*>(from + kTileBytes + piece_at(r, piece)) : make_uint4(0, 0, 0, 0);
        float v[8];
        join8(hi, lo, v, a.planes == 2);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            v[q] *= unscale;
            if (!straight) turn[piece * 8 + q][turned_at(r)] = v[q];
        }
        if (straight && row0 + r < t.m && col < t.k) apply_some<8>(a, t, row0 + r, col, t.k - col, v);
    }
    if (straight) return;
    __syncthreads();
    if (t.aligned) apply_turned<8>(a, t, row0, col0, turn);
    else apply_turned<2>(a, t, row0, col0, turn);
}

// ---------------------------------------------------------------------------------------- products
enum Kind { kGram, kSquare, kNext };    // S = X X^T and T = b I + c S;  B = a I + S T;  X' = B X

struct ProductArgs {
    const Matrix* mats;
    const Part* parts;
    uint8_t* work;
    uint32_t* errors;
    int32_t count;          // of the parts
    float a, b, c;
    int32_t which;          // of the two X: the one that is read
    uint32_t polls;         // of a wait before it counts as run out
    float* partial;         // sums of split parts, 128 x 128 each
    uint32_t* arrived;      // how many splits are there, 0 between launches
    int32_t planes;         // parts of its tiles in the workspace (S, T and B and the next X have as many as take part in products)
};

// PA, PB: parts of the first and of the second factor.  1, 1: one product; 2, 2: three (low by low is left out); 1, 2: two, for
// the first B X with one: the roundings of X_0 are the ones that all steps magnify.
template <int PA, int PB, int CG>
struct Plan {
    static constexpr uint32_t kFirst = PA * kTileBytes, kSecond = PB * kTileBytes;
    static constexpr uint32_t kStage = kFirst + kSecond;         // of both factors, 64 of K
    static constexpr int kStages = PA == 2 ? 3 : CG == 1 ? 3 : PB == 2 ? 4 : 6; // (one CTA, not three products: two blocks of threads to an SM)
    static constexpr bool kLeave = PA == 2;
    static constexpr uint32_t kColumns = kSide * CG;             // of tensor memory: the part's columns, twice
    static constexpr int kWarps = 4 * CG;                        // that take the sums; two more feed the tensor cores
    static constexpr int kThreads = CG == 2 ? 384 : 192;         // (three whole warpgroups where registers move between them)
    static constexpr int kBlocks = PB == 1 && CG == 1 ? 2 : 1;   // to an SM
    static constexpr uint32_t kSend = kSide / 4 * 128;           // bytes of a warp's rows of a tile
    static constexpr uint32_t kShared = kStages * kStage + kWarps * kSend;
};
// The tensor cores cut sums to float32 towards zero, a bias of half a unit in the last place for every 16 of K.  With three
// products the sums therefore leave tensor memory now and then and are added up in registers, to the nearest (error after five
// steps on 650 x 2600, against 2.8e-6 of plain float32 products: 5e-5 where they stay, 5.6e-6, 3.2e-6 and 1.8e-6 where they leave after 256, 128
// and 64 of K).  Leaving takes tensor memory from the products, 260 cycles each time.  Longer sums leave less often, as the error of plain products grows
// with their length too.
__host__ __device__ constexpr int steps_to_leave(int nk) { return nk >= 64 ? 4 : nk >= 16 ? 2 : 1; }

// Copies of one factor for 64 of K into shared memory.  Rows [128 i, 128 i + 128) of X (along its rows) ...
template <int PL>
__device__ __forceinline__ void fetch_along(uint8_t* to, const uint8_t* x, int64_t tile, int planes, uint64_t* bar)
{
    bulk_load(to, x + tile * planes * kTileBytes, PL * kTileBytes, bar);
}
// ... or 128 columns, of tiles `tile` and `tile + 1`, their upper or lower 64 rows
template <int PL>
__device__ __forceinline__ void fetch_turned(uint8_t* to, const uint8_t* x, int64_t tile, int planes, int lower, uint64_t* bar)
{
#pragma unroll
    for (int cb = 0; cb < 2; ++cb)
#pragma unroll
        for (int p = 0; p < PL; ++p)
            bulk_load(to + p * kTileBytes + cb * kPieceBytes, x + ((tile + cb) * planes + p) * kTileBytes + lower * kPieceBytes, kPieceBytes, bar);
}

template <int THREADS>
__device__ __forceinline__ void warps_sync(int barrier) // of four warps of a block
{
    asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(THREADS) : "memory");
}
template <int THREADS>
__device__ __forceinline__ bool warps_agree(int barrier, bool yes)
{
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(all)
                 : "r"((uint32_t)yes), "r"(barrier), "n"(THREADS)
                 : "memory");
    return all != 0;
}
template <int N>
__device__ __forceinline__ void add_at(float (&w)[N], int column, float x)
{
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e == column) w[e] += x;
}
// A warp's 32 rows of a tile (64 columns a lane, one row each): through 4 KiB of shared memory, high part and low part
// one after the other.  Straight from registers the rows, 128 bytes apart, cost 8000 cycles for 128 x 128 results.
template <int PL>
__device__ __forceinline__ void send_tile(const float (&w)[kHalves], uint8_t* mine, uint8_t* to, int lane)
{
#pragma unroll
    for (int p = 0; p < PL; ++p) {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
#pragma unroll
        for (int piece = 0; piece < 8; ++piece) {
            uint4 hi, lo;
            split8(w + piece * 8, hi, lo, p == 1);
            *reinterpret_cast<uint4*>(mine + piece_at(lane, piece)) = p ? lo : hi;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            bulk_store(to + p * kTileBytes, mine, kSide / 4 * 128);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
    }
}

// What the roles of a block know about a part.
template <int KIND, int CG, bool LEAVE>
struct Job {
    Part part;
    const Matrix* t;
    int it, jt;              // this CTA's rows of tiles of the two factors
    int mt, nb, nk, leave;   // nk: steps of 64 of K, `leave`: after how many sums leave tensor memory
    int columns;             // of tiles of 128 columns of the result
    bool has_a, has_b, same; // same: both factors are the same rows

    __device__ Job(const ProductArgs& a, int index, uint32_t rank)
    {
        part = a.parts[index];
        t = a.mats + part.matrix;
        it = part.i * CG + rank;
        jt = part.j * CG + rank;
        mt = t->mt;
        nb = t->nb;
        columns = KIND == kNext ? nb / 2 : mt;
        has_a = it < mt;
        has_b = jt < columns;
        same = KIND == kGram && part.i == part.j;
        nk = part.steps;
        leave = LEAVE ? steps_to_leave(nk) : nk;
    }
    // a tile above the diagonal's parts is stored turned
    __device__ bool turns_a(int kb) const { return KIND != kGram && (kb >> 1) / CG > part.i; }
    __device__ bool turns_b(int kb) const { return KIND == kNext || (KIND == kSquare && (kb >> 1) / CG > part.j); }
};

// One block (a pair of them) to an SM works on one part after another.  A warp copies factors in, a warp issues products, the
// others take the sums out while the products of the next part are under way: tensor memory holds two sets of sums.
template <int KIND, int PA, int PB, int CG>
__global__ void __launch_bounds__(Plan<PA, PB, CG>::kThreads, Plan<PA, PB, CG>::kBlocks) __cluster_dims__(CG, 1, 1) product_kernel(ProductArgs a)
{
    using L = Plan<PA, PB, CG>;
    constexpr int PL = PA, ST = L::kStages;                      // PL: parts of the results
    extern __shared__ __align__(1024) uint8_t stage[];           // (all other shared memory lies behind it)
    __shared__ uint64_t full[ST], empty[ST], sums[2], taken[2], drained;
    __shared__ uint32_t tmem_at;
    __shared__ volatile uint32_t failed;                         // a wait ran out
    __shared__ volatile bool last[2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const int begin = blockIdx.x / CG, step = gridDim.x / CG;
    if (tid == 0) {
        for (int s = 0; s < ST; ++s) {
            mbar_init(&full[s], CG == 2 && rank == 0 ? 2 : 1);   // the first CTA of a pair hears of the other one's copies too
            mbar_init(&empty[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&sums[s], 1);
            mbar_init(&taken[s], L::kWarps * CG);
        }
        mbar_init(&drained, 1);
        failed = 0;
    }
    __syncwarp();
    if (warp == 0) tmem_alloc<CG>(&tmem_at, 2 * L::kColumns);
    tmem_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    tmem_fence_after();
    const uint32_t acc = tmem_at;
    const Patience patience = {a.polls, &failed};
    const Job<KIND, CG, L::kLeave> first_job(a, begin, rank);    // (the tables do not change: read while the kernel before ends)
    allow_next_kernel();
    wait_for_previous_kernel();

    // (128 sums a thread want more registers than 384 threads can have: 168 each at launch become 224 and 40)
    if (warp < L::kWarps) {                                      // the sums: a thread has 128 columns of a row
        if constexpr (L::kLeave && CG == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const uint32_t from = acc + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * kSide;
        const int r = tid & 127, h = warp >> 2;
        uint8_t* mine = stage + ST * L::kStage + warp * L::kSend;
        const uint32_t rows = (warp & 3) * L::kSend;             // of a tile, in bytes
        bool ok = true;
        auto wait_sums = [&](uint32_t ch) {
            ok = ok && mbar_wait_warp(&sums[ch & 1], (ch >> 1) & 1, patience);
            tmem_fence_after();
            return ok;
        };
        auto leave_sums = [&](uint32_t ch) {
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(&taken[ch & 1], 0);
        };
        uint32_t ch = 0;                                         // sets of sums so far
        // (a warp whose wait gave up goes through all parts nevertheless, without waiting: it is wanted at the votes of split ones)
        for (int index = begin; index < a.count; index += step) {
            const Job<KIND, CG, L::kLeave> job = index == begin ? first_job : Job<KIND, CG, L::kLeave>(a, index, rank);
            const Matrix& t = *job.t;
            float v[L::kLeave ? kSide : 1];
#pragma unroll
            for (int e = 0; e < (L::kLeave ? kSide : 1); ++e) v[e] = 0.f;
            if constexpr (L::kLeave) {
                for (int kb = 0; kb < job.nk; kb += job.leave, ++ch) {
                    if (!wait_sums(ch)) break;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t bits[64];
                        tmem_load64(from + (ch & 1) * L::kColumns + q * 64, bits);
                        if (q == 1) leave_sums(ch);
#pragma unroll
                        for (int e = 0; e < 64; ++e) v[q * 64 + e] += __uint_as_float(bits[e]);
                    }
                }
            } else {
                wait_sums(ch);
            }
            const int tile = job.part.j * CG + h;                // of 128 columns
            const bool there = job.has_a && tile < job.columns;
            const int own = job.it == tile ? r : -1;             // this thread's column on the diagonal
            const int splits = KIND == kGram ? job.part.splits : 1;
            if (!ok && splits == 1) continue;
            float* partial = nullptr;                            // of this CTA's tile: split after split, column after column
            if (KIND == kGram && splits > 1) {
                const int64_t place = ((int64_t)job.part.slot * CG + rank) * CG + h;
                partial = a.partial + place * kMostSplits * (kSide * kSide) + r;
                float* here = partial + job.part.split * (kSide * kSide);
#pragma unroll
                for (int q32 = 0; q32 < kSide / 32; ++q32) {
                    if (!ok) break;
                    uint32_t bits[32];
                    if constexpr (!L::kLeave) tmem_load32(from + (ch & 1) * L::kColumns + q32 * 32, bits);
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        __stcg(here + (q32 * 32 + e) * kSide, L::kLeave ? v[L::kLeave ? q32 * 32 + e : 0] : __uint_as_float(bits[e]));
                }
                if (!L::kLeave && ok) leave_sums(ch);
                // the last split to arrive adds them all up in their order
                __threadfence();
                ok = warps_agree<128>(1 + h, ok);
                if (!ok) continue;
                if (r == 0) last[h] = atomicAdd(a.arrived + place, 1u) == (uint32_t)splits - 1;
                warps_sync<128>(1 + h);
                const bool mine_to_do = last[h];
                warps_sync<128>(1 + h);                          // (read before the next part writes it)
                if (!mine_to_do) {
                    if (!L::kLeave) ++ch;
                    continue;
                }
                __threadfence();
                if (r == 0) a.arrived[place] = 0;
            }
            const int64_t at = (KIND == kNext ? (int64_t)job.it * job.nb + 2 * tile : ((int64_t)job.it * job.mt + tile) * 2) * PL * kTileBytes;
            const float up = exp2f((float)t.es), scale = KIND == kGram ? exp2f((float)(t.es - 2 * t.ex)) : exp2f((float)-t.es);
#pragma unroll
            for (int cb = 0; cb < 2; ++cb) {
                float w[kHalves];
                if (KIND == kGram && splits > 1) {
#pragma unroll
                    for (int e = 0; e < kHalves; ++e) w[e] = 0.f;
                    for (int k = 0; k < splits; ++k) {           // (all loads of a split under way together)
                        const float* sum = partial + k * (kSide * kSide) + cb * kHalves * kSide;
                        float u[kHalves];
#pragma unroll
                        for (int e = 0; e < kHalves; ++e) u[e] = __ldcg(sum + e * kSide);
#pragma unroll
                        for (int e = 0; e < kHalves; ++e) w[e] += u[e];
                    }
#pragma unroll
                    for (int e = 0; e < kHalves; ++e) w[e] *= scale;
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    if (KIND == kGram && splits > 1) break;
                    uint32_t bits[32];
                    if constexpr (!L::kLeave) tmem_load32(from + (ch & 1) * L::kColumns + cb * kHalves + q * 32, bits);
#pragma unroll
                    for (int e = 0; e < 32; ++e) w[q * 32 + e] = (L::kLeave ? v[L::kLeave ? cb * kHalves + q * 32 + e : 0] : __uint_as_float(bits[e])) * scale;
                }
                if (!L::kLeave && cb == 1 && splits == 1) leave_sums(ch);
                if (!there) continue;
                const int column = own - cb * kHalves;           // in this tile
                if (KIND == kSquare) add_at(w, column, a.a * up);
                send_tile<PL>(w, mine, a.work + (KIND == kGram ? t.s_at : KIND == kSquare ? t.b_at : t.at[a.which ^ 1]) + at + cb * PL * kTileBytes + rows, lane);
                if (KIND == kGram) {
#pragma unroll
                    for (int e = 0; e < kHalves; ++e) w[e] *= a.c;
                    add_at(w, column, a.b * up);
                    send_tile<PL>(w, mine, a.work + t.t_at + at + cb * PL * kTileBytes + rows, lane);
                }
            }
            if (!L::kLeave) ++ch;
        }
        if (!ok) failed = 1;
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else {
        if constexpr (L::kLeave && CG == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == L::kWarps) {                                 // the copies
            fence_async();
            uint32_t n = 0;                                      // steps of 64 of K so far
            bool ok = true;
            for (int index = begin; index < a.count && ok; index += step) {
                const Job<KIND, CG, L::kLeave> job = index == begin ? first_job : Job<KIND, CG, L::kLeave>(a, index, rank);
                const uint8_t* x = a.work + job.t->at[a.which];
                const uint8_t* first = KIND == kGram ? x : a.work + (KIND == kSquare ? job.t->s_at : job.t->b_at);
                const bool load_b = job.has_b && !job.same;
                const uint32_t bytes = (job.has_a ? L::kFirst : 0) + (load_b ? L::kSecond : 0);
                for (int kb = 0; kb < job.nk; ++kb, ++n) {
                    const uint32_t s = n % ST;
                    if (n >= ST) ok = mbar_wait_warp(&empty[s], (n / ST - 1) & 1, patience);
                    if (!ok) break;
                    uint8_t* to_a = stage + s * L::kStage;
                    uint8_t* to_b = to_a + L::kFirst;
                    const int ct = kb >> 1;
                    if (elect_one()) {
                        mbar_expect_tx(&full[s], bytes);
                        if (job.has_a) {
                            if (KIND == kGram) fetch_along<PA>(to_a, x, (int64_t)job.it * job.nb + job.part.begin + kb, a.planes, &full[s]);
                            else if (!job.turns_a(kb)) fetch_along<PA>(to_a, first, ((int64_t)job.it * job.mt + ct) * 2 + (kb & 1), PL, &full[s]);
                            else fetch_turned<PA>(to_a, first, ((int64_t)ct * job.mt + job.it) * 2, PL, kb & 1, &full[s]);
                        }
                        if (load_b) {
                            if (KIND == kGram) fetch_along<PB>(to_b, x, (int64_t)job.jt * job.nb + job.part.begin + kb, a.planes, &full[s]);
                            else if (KIND == kNext) fetch_turned<PB>(to_b, x, (int64_t)ct * job.nb + 2 * job.jt, a.planes, kb & 1, &full[s]);
                            else if (!job.turns_b(kb)) fetch_along<PB>(to_b, a.work + job.t->t_at, ((int64_t)job.jt * job.mt + ct) * 2 + (kb & 1), PL, &full[s]);
                            else fetch_turned<PB>(to_b, a.work + job.t->t_at, ((int64_t)ct * job.mt + job.jt) * 2, PL, kb & 1, &full[s]);
                        }
                    }
                    __syncwarp();
                }
            }
            if (!ok) {                                           // copies under way are sat out
                failed = 1;
                for (uint32_t q = n > ST ? n - ST : 0; q < n; ++q) mbar_wait_warp(&full[q % ST], (q / ST) & 1, patience);
            }
        } else if (warp == L::kWarps + 1) {                      // the products
            uint32_t n = 0, ch = 0;
            bool ok = true;
            for (int index = begin; index < a.count && ok; index += step) {
                const Job<KIND, CG, L::kLeave> job = index == begin ? first_job : Job<KIND, CG, L::kLeave>(a, index, rank);
                for (int kb = 0; kb < job.nk; ++kb, ++n) {
                    const uint32_t s = n % ST;
                    if (CG == 2 && rank == 1) {                  // the other CTA of a pair tells the first what has come
                        ok = mbar_wait_warp(&full[s], (n / ST) & 1, patience);
                        if (!ok) break;
                        if (elect_one()) mbar_arrive_at(&full[s], 0);
                        __syncwarp();
                        continue;
                    }
                    const bool begins = kb % job.leave == 0, ends = kb + 1 == job.nk || (kb + 1) % job.leave == 0;
                    if (begins && ch >= 2) ok = mbar_wait_warp(&taken[ch & 1], (ch / 2 - 1) & 1, patience);
                    ok = ok && mbar_wait_warp(&full[s], (n / ST) & 1, patience);
                    if (!ok) break;
                    tmem_fence_after();
                    const bool turn_a = job.turns_a(kb), turn_b = job.turns_b(kb);
                    const uint32_t at_a = smem_u32(stage) + s * L::kStage, at_b = job.same ? at_a : at_a + L::kFirst;
                    const uint32_t shape = product_shape(kSide * CG, kSide * CG) | (turn_a ? kTurnA : 0) | (turn_b ? kTurnB : 0);
                    const uint64_t da = turn_a ? operand_turned(at_a, kPieceBytes) : operand_along(at_a);
                    const uint64_t db = turn_b ? operand_turned(at_b, kPieceBytes) : operand_along(at_b);
                    const uint64_t na = turn_a ? kNextTurned : kNextAlong, nb = turn_b ? kNextTurned : kNextAlong;
                    const uint32_t to = acc + (ch & 1) * L::kColumns;
                    constexpr uint64_t low = kTileBytes >> 4;
                    auto high = [&](int q) { product<CG>(to, da + q * na, db + q * nb, shape, PB == 2 || !begins || q > 0); };
                    if (elect_one()) {
                        if constexpr (PB == 2) {                 // the small products come first, while the sums are small
#pragma unroll
                            for (int q = 0; q < kHalves / 16; ++q) {
                                product<CG>(to, da + q * na, db + q * nb + low, shape, !begins || q > 0);
                                if constexpr (PA == 2) product<CG>(to, da + q * na + low, db + q * nb, shape, true);
                            }
                        }
                        high(0);
                        high(1);
                        high(2);
                        high(3);
                        products_done<CG>(&empty[s]);
                        if (ends) products_done<CG>(&sums[ch & 1]);
                    }
                    __syncwarp();
                    if (ends) ++ch;
                }
            }
            if (!ok) failed = 1;
            // products that nobody waits for any more are sat out too
            if (rank == 0 && elect_one()) products_done<CG>(&drained);
            __syncwarp();
            mbar_wait_warp(&drained, 0, patience);
        }
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if (tid == 0 && failed) atomicAdd(a.errors, 1u);
    __syncwarp();
    if (CG == 2) cluster_sync();
    if (warp == 0) tmem_free<CG>(acc, 2 * L::kColumns);
}

// ---------------------------------------------------------------------------------------- small matrices
// A matrix that fits a block's shared memory takes one launch for the whole step: momentum, norm, all products and the new
// parameters, with X, S, T and B where the tensor cores read them.  (64 x 576 by 17 launches: 187 us; this way: 65.)  Rows of tiles are cut
// to the smaller side, a multiple of 16; the first factor of a product always has 128 rows and reads on into what lies behind, which
// makes rows of sums that nobody looks at.
constexpr int kSmallThreads = 512;
constexpr int kSmallShared = 227 * 1024 - 1024;
constexpr uint32_t kTmemColumns = 512;

struct SmallLayout {
    int rows, blocks, square;   // of tiles: rows; tiles of X; tiles of S in a row
    uint32_t tile;              // bytes of one part of a tile
    uint32_t s_at, t_at, bytes;
    __host__ __device__ SmallLayout(int m, int k)
    {
        rows = (m + 15) / 16 * 16;
        blocks = (k + kHalves - 1) / kHalves;
        square = (rows + kHalves - 1) / kHalves;
        tile = rows * 128;
        s_at = blocks * 2 * tile;
        t_at = s_at + square * 2 * tile;
        bytes = t_at + square * 2 * tile + kTileBytes;
    }
};
__host__ __device__ inline bool is_small(int m, int k) // (only tiles that can fit are multiplied out)
{
    return m > 0 && m <= kSide && k <= 1 << 14 && SmallLayout(m, k).bytes <= (uint32_t)kSmallShared;
}

struct SmallArgs {
    MomentArgs moment;
    TileArgs tile;
    const int32_t* list;
    uint32_t* errors;
    float a, b, c;
    int32_t steps;
    uint32_t polls;
};

__global__ void __launch_bounds__(kSmallThreads, 1) small_kernel(SmallArgs a)
{
    extern __shared__ __align__(1024) uint8_t stage[];
    __shared__ double ws[kSmallThreads / 32];
    __shared__ uint64_t done;
    __shared__ uint32_t tmem_at;
    __shared__ volatile uint32_t failed;                         // a wait ran out
    __shared__ Scale scale;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Matrix& t = a.moment.mats[a.list[blockIdx.x]];
    const SmallLayout l(t.m, t.k);
    if (tid == 0) {
        mbar_init(&done, 1);
        failed = 0;
    }
    __syncwarp();
    if (warp == 0) tmem_alloc<1>(&tmem_at, kTmemColumns);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t acc = tmem_at;
    allow_next_kernel();
    wait_for_previous_kernel();
    const float c = a.moment.factor ? a.moment.factor[t.group] : 1.f;
    const bool skip = __syncthreads_or(!isfinite(c) || __ldcg(a.moment.errors) != 0); // (other blocks may add to the errors)
    bool ok = true;
    if (!skip) {
        const double sum = block_sum<kSmallThreads>(moment_unit<kSmallThreads>(a.moment, t, 0, (int64_t)t.rows * t.cols, c), ws);
        if (tid == 0) scale = scale_of(sum, t.ex);
        __syncthreads();                                         // (and the momentum is written)
        const Scale sc = scale;
        const bool live = sc.second != 0.f;
        auto x_tile = [&](int block, int part) { return stage + (block * 2 + part) * l.tile; };
        auto put = [&](uint8_t* tile, int row, int piece, const float* v) {
            uint4 hi, lo;
            split8(v, hi, lo, true);
            *reinterpret_cast<uint4*>(tile + piece_at(row, piece)) = hi;
            *reinterpret_cast<uint4*>(tile + l.tile + piece_at(row, piece)) = lo;
        };
        if (!t.tall) {
#pragma unroll 3
            for (int e = tid; e < l.rows * l.blocks * 8; e += kSmallThreads) {
                const int row = e / (l.blocks * 8), piece = e % (l.blocks * 8);
                float v[8] = {};
                if (live && row < t.m && piece * 8 < t.k) update_some<8>(a.tile, t, row, piece * 8, t.k - piece * 8, c, v);
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = v[q] * sc.first * sc.second;
                put(x_tile(piece >> 3, 0), row, piece & 7, v);
            }
        } else {
#pragma unroll 3
            for (int e = tid; e < l.blocks * kHalves * (l.rows / 8); e += kSmallThreads) {
                const int col = e % (l.blocks * kHalves), row = e / (l.blocks * kHalves) * 8;
                float v[8] = {};
                if (live && row < t.m && col < t.k) update_some<8>(a.tile, t, col, row, t.m - row, c, v);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float u = v[q] * sc.first * sc.second;
                    const __half hi = __float2half_rn(u);
                    uint8_t* at = x_tile(col >> 6, 0) + piece_at(row + q, (col & 63) >> 3) + (col & 7) * 2;
                    *reinterpret_cast<__half*>(at) = hi;
                    *reinterpret_cast<__half*>(at + l.tile) = __float2half_rn(u - __half2float(hi));
                }
            }
        }
        uint32_t phase = 0;
        auto begin_products = [&]() { // what was written is there for the tensor cores
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tmem_fence_before();
            __syncthreads();
            tmem_fence_after();
        };
        auto wait_products = [&]() {
            ok = __syncthreads_and(mbar_wait(&done, phase, {a.polls, &failed}));
            phase ^= 1;
            tmem_fence_after();
            return ok;
        };
        // Three products of 16 of K from `begin` to `end`, the small ones of all of them first, while the sums are small
        auto products = [&](uint32_t to, uint32_t shape, int begin, int end, auto first, auto second) {
            const uint64_t low = l.tile >> 4;
            for (int q = begin; q < end; ++q) {
                const uint64_t f = first(q), g = second(q);
                product<1>(to, f, g + low, shape, q > begin);
                product<1>(to, f + low, g, shape, true);
            }
            for (int q = begin; q < end; ++q) product<1>(to, first(q), second(q), shape, true);
        };
        const uint32_t base = smem_u32(stage), shape = product_shape(kSide, l.rows);
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const int row = (warp & 3) * 32 + lane, share = warp >> 2;  // a warp has 32 rows and every fourth unit of their columns
        const bool rows_here = (warp & 3) * 32 < l.rows;
        const float up = exp2f((float)t.es), down = exp2f((float)-t.es), gram = exp2f((float)(t.es - 2 * t.ex));
        // sums of X X^T in several parts, added up in registers (see steps_to_leave)
        const int parts = min(min((int)kTmemColumns / l.rows, 16), l.blocks), each = (l.blocks + parts - 1) / parts, used = (l.blocks + each - 1) / each;
        for (int step = 0; step < a.steps && ok; ++step) {
            begin_products();
            if (warp == 0 && elect_one()) {
                auto x = [&](int q) { return operand_along(base + (q >> 2) * 2 * l.tile + (q & 3) * 32); };
                for (int p = 0; p < used; ++p)
                    products(acc + p * l.rows, shape, p * each * (kHalves / 16), min((p + 1) * each, l.blocks) * (kHalves / 16), x, x);
                products_done<1>(&done);
            }
            if (!wait_products()) break;
            if (rows_here)
                for (int piece = share; piece < l.rows / 8; piece += 4) {
                    float f[8] = {};
                    for (int p = 0; p < used; ++p) {
                        uint32_t r[8];
                        tmem_load8(acc + lanes + p * l.rows + piece * 8, r);
#pragma unroll
                        for (int q = 0; q < 8; ++q) f[q] += __uint_as_float(r[q]);
                    }
                    if (row < l.rows) {
#pragma unroll
                        for (int q = 0; q < 8; ++q) f[q] *= gram;
                        put(stage + l.s_at + (piece >> 3) * 2 * l.tile, row, piece & 7, f);
#pragma unroll
                        for (int q = 0; q < 8; ++q) f[q] = f[q] * a.c + (row == piece * 8 + q ? a.b * up : 0.f);
                        put(stage + l.t_at + (piece >> 3) * 2 * l.tile, row, piece & 7, f);
                    }
                }
            begin_products();
            if (warp == 0 && elect_one()) {
                auto at = [&](uint32_t from) { return [=](int q) { return operand_along(from + (q >> 2) * 2 * l.tile + (q & 3) * 32); }; };
                products(acc, shape, 0, l.rows / 16, at(base + l.s_at), at(base + l.t_at));
                products_done<1>(&done);
            }
            if (!wait_products()) break;
            if (rows_here)                                       // B takes the place of S
                for (int piece = share; piece < l.rows / 8; piece += 4) {
                    uint32_t r[8];
                    tmem_load8(acc + lanes + piece * 8, r);
                    if (row < l.rows) {
                        float f[8];
#pragma unroll
                        for (int q = 0; q < 8; ++q) f[q] = __uint_as_float(r[q]) * down + (row == piece * 8 + q ? a.a * up : 0.f);
                        put(stage + l.s_at + (piece >> 3) * 2 * l.tile, row, piece & 7, f);
                    }
                }
            begin_products();
            // B X, 256 columns at a time, two of these under way; the new columns take the place of the old ones
            auto next = [&](int first) {
                const int count = min(4, l.blocks - first);
                const uint32_t wide = product_shape(kSide, count * kHalves) | kTurnB;
                products(acc + (first & 4) * kHalves, wide, 0, l.rows / 16,
                         [&](int q) { return operand_along(base + l.s_at + (q >> 2) * 2 * l.tile + (q & 3) * 32); },
                         [&](int q) { return operand_turned(base + first * 2 * l.tile + q * 2048, 2 * l.tile); });
                products_done<1>(&done);
            };
            if (warp == 0 && elect_one()) next(0);
            for (int first = 0; first < l.blocks && ok; first += 4) {
                if (!wait_products()) break;
                if (warp == 0 && first + 4 < l.blocks && elect_one()) next(first + 4);
                __syncwarp();
                const int units = min(4, l.blocks - first) * 2;
                if (rows_here)
                    for (int u = share; u < units; u += 4) {
                        uint32_t r[32];
                        tmem_load32(acc + (first & 4) * kHalves + lanes + u * 32, r);
                        if (row < l.rows) {
#pragma unroll
                            for (int p = 0; p < 4; ++p) {
                                float f[8];
#pragma unroll
                                for (int q = 0; q < 8; ++q) f[q] = __uint_as_float(r[p * 8 + q]) * down;
                                put(x_tile(first + (u >> 1), 0), row, (u & 1) * 4 + p, f);
                            }
                        }
                    }
                tmem_fence_before();                             // (read before the products after the next ones write there)
            }
        }
        __syncthreads();
        const float unscale = exp2f((float)-t.ex);
        if (failed) {
            if (tid == 0) atomicAdd(a.errors, 1u);
        } else if (!t.tall) {
#pragma unroll 3
            for (int e = tid; e < t.m * l.blocks * 8; e += kSmallThreads) {
                const int r = e / (l.blocks * 8), piece = e % (l.blocks * 8);
                if (piece * 8 >= t.k) continue;
                const uint8_t* at = x_tile(piece >> 3, 0) + piece_at(r, piece & 7);
                float v[8];
                join8(*reinterpret_cast<const uint4*>(at), *reinterpret_cast<const uint4*>(at + l.tile), v, true);
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] *= unscale;
                apply_some<8>(a.tile, t, r, piece * 8, t.k - piece * 8, v);
            }
        } else {
#pragma unroll 3
            for (int e = tid; e < l.blocks * kHalves * (l.rows / 8); e += kSmallThreads) {
                const int col = e % (l.blocks * kHalves), r = e / (l.blocks * kHalves) * 8;
                if (col >= t.k || r >= t.m) continue;
                float v[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const uint8_t* at = x_tile(col >> 6, 0) + piece_at(r + q, (col & 63) >> 3) + (col & 7) * 2;
                    v[q] = (__half2float(*reinterpret_cast<const __half*>(at)) + __half2float(*reinterpret_cast<const __half*>(at + l.tile))) * unscale;
                }
                apply_some<8>(a.tile, t, col, r, t.m - r, v);
            }
        }
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if (warp == 0) tmem_free<1>(acc, kTmemColumns);
}

using ProductKernel = void (*)(ProductArgs);
struct Launch {
    ProductKernel kernel;
    int threads, shared, blocks;    // blocks: to an SM
};
template <int KIND, int PA, int PB, int CG>
Launch launch_of()
{
    using L = Plan<PA, PB, CG>;
    return {product_kernel<KIND, PA, PB, CG>, L::kThreads, (int)L::kShared, L::kBlocks};
}
// `first`: the product reads X_0, which has two parts in any case
template <int CG>
Launch launch_of(int kind, bool three, bool first)
{
    if (three) return kind == kGram ? launch_of<kGram, 2, 2, CG>() : kind == kSquare ? launch_of<kSquare, 2, 2, CG>() : launch_of<kNext, 2, 2, CG>();
    if (kind == kNext) return first ? launch_of<kNext, 1, 2, CG>() : launch_of<kNext, 1, 1, CG>();
    return kind == kGram ? launch_of<kGram, 1, 1, CG>() : launch_of<kSquare, 1, 1, CG>();
}
template <int CG>
cudaError_t allow_shared()
{
    cudaError_t e = cudaSuccess;
    for (int kind = 0; kind < 3; ++kind)
        for (int mode = 0; mode < 3 && e == cudaSuccess; ++mode) {
            const Launch l = launch_of<CG>(kind, mode == 0, mode == 1);
            e = cudaFuncSetAttribute((const void*)l.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, l.shared);
        }
    return e;
}

// matrices of a wave that take the same kernels: one product or three, one CTA to a part or two
struct Class {
    int64_t symmetric, gram_end, symmetric_end; // parts of S, of B
    int64_t next, next_end;             // parts of X'
};
struct Wave {
    int64_t blocks[2], blocks_end[2];   // tiles of X, of matrices with one product and with three
    Class classes[2][2];                // [three products][pairs]
};

// Workspace that matrices are taken together up to.  (Waves that stay in L2 cost more by their launches and their ends than they save: 4 ResNet-50s
// 3.9 ms, in waves of 512 MiB 4.6, of 256 MiB 5.7.)
constexpr int64_t kWaveBytes = (int64_t)2 << 30;
constexpr int64_t kMostElements = (int64_t)1 << 30;
constexpr int32_t kMostSide = 1 << 14;           // of the smaller side: S is m x m

struct Range { // of addresses
    uintptr_t begin, end;
};

} // namespace
} // namespace choco

using namespace choco;

struct choco_muon {
    choco_muon_params params;
    int device, sms;
    bool broken;                   // the table on the device may be half written
    uint32_t polls;                // of a wait in a kernel before it counts as run out
    bool timed_out;                // one was seen to have run out
    std::vector<Matrix> mats;      // as on the device
    std::vector<Range> written;    // in order, disjoint
    std::vector<Range> read;       // gradients likewise, those that meet joined
    std::vector<int64_t> offsets;
    std::vector<Wave> waves;
    std::vector<int32_t> small;    // matrices that one block of threads takes through the whole step
    int64_t small_shared;
    int64_t elements;
    int64_t nunits;
    int32_t* d_small;
    int64_t split_tiles;           // 128 x 128 results that splits are added up for, of one launch
    float* d_split;
    uint32_t* d_arrived;
    void* memory;
    Matrix* d_mats;
    Unit* d_units;
    Part* d_parts;
    Block* d_blocks;
    double* d_partial;
    uint32_t* d_done;
    uint32_t* d_errors;
    Scale* d_scale;
    uint8_t* d_work;
};

namespace {

bool on_device(const choco_muon* o)
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
void free_all(choco_muon* o)
{
    cudaFree(o->memory);
    delete o;
}

Range range_of(const void* p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype)
{
    return {(uintptr_t)p, (uintptr_t)p + (uintptr_t)(((rows - 1) * ld + cols) * dtype_size(dtype))};
}

// Largest singular value that the polynomial makes of one in [0, most], and the largest |a + b s^2 + c s^4| and |b + c s^2| on the way.
void reach(const choco_muon_params& p, double most, double* value, double* slope)
{
    *value = *slope = 0.0;
    for (int i = 0; i <= 4096; ++i) {
        const double s = most * i / 4096, inner = p.b + s * s * p.c, q = std::fabs(p.a + s * s * inner);
        *slope = std::max({*slope, q, std::fabs(inner)});
        *value = std::max(*value, s * q);
    }
}
bool polynomial_ok(const choco_muon_params& p)
{
    if (!std::isfinite(p.a) || !std::isfinite(p.b) || !std::isfinite(p.c)) return false;
    double most = 1.0;
    for (int k = 0; k < p.steps; ++k) {
        double value, slope;
        reach(p, most, &value, &slope);
        if (!(value <= 1.9) || !(slope <= 15.0)) return false; // S, T and B stay inside float16 at their scales
        most = std::max(1.0, value);
    }
    return true;
}

template <typename T>
int64_t carve(int64_t& at, int64_t count)
{
    at = (at + 255) / 256 * 256;
    const int64_t here = at;
    at += (int64_t)sizeof(T) * count;
    return here;
}

// What depends on the gradient's address
void look_at_gradient(Matrix& t)
{
    t.whole = t.g_ld == t.cols || t.rows == 1;
    auto rows = [&](const void* p, int64_t ld, int32_t dtype) { return aligned_to(p, 16) && (t.rows == 1 || ld * dtype_size(dtype) % 16 == 0); };
    t.aligned = rows(t.x, t.x_ld, t.x_dtype) && rows(t.g, t.g_ld, t.g_dtype) && rows(nullptr, t.cols, CHOCO_F32) && (!t.copy || rows(t.copy, t.copy_ld, t.copy_dtype));
}

// Fills the host tables.  Throws std::bad_alloc.
int plan(choco_muon* o, int32_t n, const choco_muon_matrix* ms, std::vector<Unit>& units, std::vector<Part>& parts, std::vector<Block>& blocks,
         int64_t* work)
{
    int64_t at = 0;
    std::vector<int32_t> kinds; // of every matrix: 1 = three products, -1: in no wave
    for (int32_t i = 0; i < n; ++i) {
        const choco_muon_matrix& q = ms[i];
        if (q.rows < 0 || q.cols < 0 || q.x_ld < 0 || q.g_ld < 0 || q.copy_ld < 0) return CHOCO_ERR_INVALID_ARG;
        if (q.group < 0 || q.group >= o->params.groups || !dtype_ok(q.x_dtype) || !dtype_ok(q.g_dtype) || !dtype_ok(q.copy_dtype))
            return CHOCO_ERR_INVALID_ARG;
        if (!(q.weight_decay >= 0.0) || !(q.lr_scale >= 0.0) || !std::isfinite((float)q.weight_decay) || !std::isfinite((float)q.lr_scale))
            return CHOCO_ERR_INVALID_ARG;
        const bool some = q.rows > 0 && q.cols > 0;
        if (some && (!q.x || !q.g)) return CHOCO_ERR_INVALID_ARG;
        if ((q.x_ld && q.x_ld < q.cols) || (q.g_ld && q.g_ld < q.cols) || (q.copy_ld && q.copy_ld < q.cols)) return CHOCO_ERR_INVALID_ARG;
        if (!aligned_to(q.x, dtype_size(q.x_dtype)) || !aligned_to(q.g, dtype_size(q.g_dtype)) || !aligned_to(q.copy, dtype_size(q.copy_dtype)))
            return CHOCO_ERR_MISALIGNED;
        if (some && (std::min(q.rows, q.cols) > kMostSide || std::max(q.rows, q.cols) > kMostElements / std::min(q.rows, q.cols) ||
                     std::max({q.x_ld, q.g_ld, q.copy_ld}) > std::min((int64_t)1 << 38, ((int64_t)1 << 40) / q.rows)))
            return CHOCO_ERR_TOO_LARGE;
        Matrix t = {};
        t.x = q.x; t.g = q.g; t.copy = q.copy;
        t.rows = some ? (int32_t)q.rows : 0; t.cols = some ? (int32_t)q.cols : 0;
        t.x_ld = q.x_ld ? q.x_ld : q.cols; t.g_ld = q.g_ld ? q.g_ld : q.cols; t.copy_ld = q.copy_ld ? q.copy_ld : q.cols;
        t.state = at;
        t.tall = t.rows > t.cols;
        t.m = std::min(t.rows, t.cols); t.k = std::max(t.rows, t.cols);
        t.mt = (t.m + kSide - 1) / kSide;
        t.nb = (t.k + kSide - 1) / kSide * 2;
        if (some) {
            t.ex = std::min(14, (int)std::floor(std::log2(std::sqrt((double)t.m * t.k))));
            t.es = std::min(12, (int)std::ceil(std::log2((double)t.m)));
        }
        t.group = q.group;
        t.weight_decay = (float)q.weight_decay; t.lr_scale = (float)q.lr_scale;
        t.x_dtype = (int8_t)q.x_dtype; t.g_dtype = (int8_t)q.g_dtype; t.copy_dtype = (int8_t)q.copy_dtype;
        look_at_gradient(t);
        t.unit0 = (int32_t)units.size();
        const int64_t count = (int64_t)t.rows * t.cols;
        const bool small = is_small(t.m, t.k);
        if (small) {
            o->small.push_back(i);
            o->small_shared = std::max(o->small_shared, (int64_t)SmallLayout(t.m, t.k).bytes);
        }
        t.units = small ? 0 : (int32_t)((count + kUnit - 1) / kUnit);
        for (int32_t u = 0; u < t.units; ++u) units.push_back({i, u});
        if (units.size() > 0x7fffffff) return CHOCO_ERR_TOO_LARGE;
        o->mats.push_back(t);
        o->offsets.push_back(at);
        kinds.push_back(small || !some ? -1 : o->params.products != 1);
        at += (count + kBlock - 1) / kBlock * kBlock;
        if (at > (int64_t)1 << 38) return CHOCO_ERR_TOO_LARGE;
        if (some) {
            o->written.push_back(range_of(q.x, t.rows, t.cols, t.x_ld, q.x_dtype));
            if (q.copy) o->written.push_back(range_of(q.copy, t.rows, t.cols, t.copy_ld, q.copy_dtype));
        }
    }
    o->elements = at;
    o->nunits = (int64_t)units.size();
    // the longest first, so that the launch ends with short ones
    std::sort(o->small.begin(), o->small.end(), [&](int32_t x, int32_t y) {
        const uint32_t p = SmallLayout(o->mats[x].m, o->mats[x].k).bytes, q = SmallLayout(o->mats[y].m, o->mats[y].k).bytes;
        return p != q ? p > q : x < y;
    });
    // waves: matrices in order, as many as the workspace holds together
    *work = 0;
    for (int32_t i = 0; i < n;) {
        int64_t bytes = 0;
        int32_t end = i;
        for (; end < n; ++end) {
            Matrix& t = o->mats[end];
            if (kinds[end] < 0) continue;
            const int64_t planes = kinds[end] ? 2 : 1, x0 = (int64_t)t.mt * t.nb * 2 * kTileBytes, xb = x0 / 2 * planes, sb = (int64_t)t.mt * t.mt * 2 * planes * kTileBytes;
            if (bytes > 0 && bytes + x0 + xb + 3 * sb > kWaveBytes) break;
            t.at[0] = bytes; t.at[1] = bytes + x0;
            t.s_at = bytes + x0 + xb; t.t_at = t.s_at + sb; t.b_at = t.t_at + sb;
            bytes += x0 + xb + 3 * sb;
        }
        *work = std::max(*work, bytes);
        if (bytes == 0) break;   // (nothing but small ones was left)
        Wave w = {};
        for (int three = 0; three < 2; ++three) {
            w.blocks[three] = (int64_t)blocks.size();
            for (int32_t q = i; q < end; ++q)
                if (kinds[q] == three)
                    for (int32_t r = 0; r < o->mats[q].mt; ++r)
                        for (int32_t c = 0; c < o->mats[q].nb; ++c) blocks.push_back({q, r, c});
            w.blocks_end[three] = (int64_t)blocks.size();
            for (int pairs = 0; pairs < 2; ++pairs) {
                Class& cl = w.classes[three][pairs];
                const int cg = pairs + 1;
                std::vector<int32_t> these;
                for (int32_t q = i; q < end; ++q)
                    if (kinds[q] == three && o->mats[q].mt > 0 && (o->mats[q].mt > 1) == (pairs == 1)) these.push_back(q);
                // the longest first: a launch ends with short ones
                std::sort(these.begin(), these.end(), [&](int32_t x, int32_t y) {
                    return o->mats[x].k != o->mats[y].k ? o->mats[x].k > o->mats[y].k : x < y;
                });
                cl.symmetric = (int64_t)parts.size();
                auto symmetric = [&](auto add) {
                    for (int32_t q : these)
                        for (int32_t r = 0; r < (o->mats[q].mt + cg - 1) / cg; ++r)
                            for (int32_t c = 0; c <= r; ++c) add(o->mats[q], Part{q, r, c, 0, 0, 0, 1, 0});
                };
                auto steps_of = [](int32_t k) { return (k + kHalves - 1) / kHalves; };
                // X X^T: where the parts are too few for all SMs, long ones are split along K, into pieces of eight steps at least
                int64_t few = 0;
                symmetric([&](const Matrix&, const Part&) { ++few; });
                const int64_t room = std::max<int64_t>(1, o->sms / cg / std::max<int64_t>(few, 1));
                int32_t slots = 0;
                symmetric([&](const Matrix& t, Part p) {
                    const int32_t steps = steps_of(t.k);
                    p.splits = (int32_t)std::max<int64_t>(1, std::min({room, (int64_t)kMostSplits, (int64_t)steps / 8}));
                    if (p.splits > 1) p.slot = slots++;
                    for (p.split = 0; p.split < p.splits; ++p.split) {
                        p.begin = (int32_t)((int64_t)steps * p.split / p.splits);
                        p.steps = (int32_t)((int64_t)steps * (p.split + 1) / p.splits) - p.begin;
                        parts.push_back(p);
                    }
                });
                o->split_tiles = std::max(o->split_tiles, (int64_t)slots * cg * cg);
                cl.gram_end = (int64_t)parts.size();
                symmetric([&](const Matrix& t, Part p) {
                    p.steps = steps_of(t.m);
                    parts.push_back(p);
                });
                cl.symmetric_end = cl.next = (int64_t)parts.size();
                std::sort(these.begin(), these.end(), [&](int32_t x, int32_t y) {
                    return o->mats[x].m != o->mats[y].m ? o->mats[x].m > o->mats[y].m : x < y;
                });
                for (int32_t q : these)
                    for (int32_t c = 0; c < (o->mats[q].nb / 2 + cg - 1) / cg; ++c)
                        for (int32_t r = 0; r < (o->mats[q].mt + cg - 1) / cg; ++r)
                            parts.push_back(Part{q, r, c, 0, steps_of(o->mats[q].m), 0, 1, 0});
                cl.next_end = (int64_t)parts.size();
            }
        }
        o->waves.push_back(w);
        i = end;
    }
    return blocks.size() > 0x7fffffff || parts.size() > 0x3fffffff ? CHOCO_ERR_TOO_LARGE : CHOCO_OK;
}

// Whether arrays that a step writes share memory, with each other or with gradients.
bool overlap(choco_muon* o)
{
    std::vector<Range>& w = o->written;
    std::sort(w.begin(), w.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    for (size_t i = 1; i < w.size(); ++i)
        if (w[i].begin < w[i - 1].end) return true;
    return false;
}
bool meets(const std::vector<Range>& ranges, const Range& r)
{
    auto next = std::lower_bound(ranges.begin(), ranges.end(), r.end, [](const Range& a, uintptr_t e) { return a.begin < e; });
    return next != ranges.begin() && (next - 1)->end > r.begin;
}
bool is_written(const choco_muon* o, const Matrix& t, const void* g)
{
    return t.rows > 0 && meets(o->written, range_of(g, t.rows, t.cols, t.g_ld, t.g_dtype));
}
std::vector<Range> gradient_ranges(const std::vector<Matrix>& mats) // throws std::bad_alloc
{
    std::vector<Range> all, joined;
    for (const Matrix& t : mats)
        if (t.rows > 0) all.push_back(range_of(t.g, t.rows, t.cols, t.g_ld, t.g_dtype));
    std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    for (const Range& r : all) {
        if (!joined.empty() && r.begin <= joined.back().end) joined.back().end = std::max(joined.back().end, r.end);
        else joined.push_back(r);
    }
    return joined;
}

int allocate(choco_muon* o, const std::vector<Unit>& units, const std::vector<Part>& parts, const std::vector<Block>& blocks, int64_t work)
{
    int64_t at = 0;
    const int64_t n = (int64_t)o->mats.size();
    const int64_t mats = carve<Matrix>(at, n), un = carve<Unit>(at, (int64_t)units.size()), pa = carve<Part>(at, (int64_t)parts.size()),
                  bl = carve<Block>(at, (int64_t)blocks.size()), pt = carve<double>(at, o->nunits), done = carve<uint32_t>(at, n),
                  err = carve<uint32_t>(at, 1), arr = carve<uint32_t>(at, o->split_tiles), sc = carve<Scale>(at, n), sm = carve<int32_t>(at, (int64_t)o->small.size()),
                  sp = carve<float>(at, o->split_tiles * kMostSplits * kSide * kSide);
    at = (at + 1023) / 1024 * 1024;
    const int64_t wk = at;
    at += work;
    if (cudaMalloc(&o->memory, (size_t)at) != cudaSuccess) return CHOCO_ERR_ALLOC;
    uint8_t* base = static_cast<uint8_t*>(o->memory);
    o->d_mats = reinterpret_cast<Matrix*>(base + mats);
    o->d_units = reinterpret_cast<Unit*>(base + un);
    o->d_parts = reinterpret_cast<Part*>(base + pa);
    o->d_blocks = reinterpret_cast<Block*>(base + bl);
    o->d_partial = reinterpret_cast<double*>(base + pt);
    o->d_done = reinterpret_cast<uint32_t*>(base + done);
    o->d_errors = reinterpret_cast<uint32_t*>(base + err);
    o->d_scale = reinterpret_cast<Scale*>(base + sc);
    o->d_small = reinterpret_cast<int32_t*>(base + sm);
    o->d_arrived = reinterpret_cast<uint32_t*>(base + arr);
    o->d_split = reinterpret_cast<float*>(base + sp);
    o->d_work = base + wk;
    cudaStream_t st;
    if (cudaStreamCreateWithFlags(&st, cudaStreamNonBlocking) != cudaSuccess) return CHOCO_ERR_CUDA;
    auto send = [&](void* to, const auto& from) {
        return from.empty() || cudaMemcpyAsync(to, from.data(), sizeof(from[0]) * from.size(), cudaMemcpyHostToDevice, st) == cudaSuccess;
    };
    bool ok = cudaMemsetAsync(o->d_done, 0, (size_t)(sc - done), st) == cudaSuccess; // counts and errors
    ok = ok && send(o->d_mats, o->mats) && send(o->d_units, units) && send(o->d_small, o->small) && send(o->d_parts, parts) && send(o->d_blocks, blocks);
    ok = cudaStreamSynchronize(st) == cudaSuccess && ok;
    cudaStreamDestroy(st);
    if (!ok) return CHOCO_ERR_CUDA;
    return allow_shared<1>() == cudaSuccess && allow_shared<2>() == cudaSuccess &&
                   cudaFuncSetAttribute((const void*)small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallShared) == cudaSuccess
               ? CHOCO_OK
               : CHOCO_ERR_CUDA;
}

cudaError_t launch_products(const choco_muon* o, const Wave& w, int kind, int step, cudaStream_t st)
{
    const choco_muon_params& p = o->params;
    cudaError_t e = cudaSuccess;
    for (int three = 0; three < 2; ++three)
        for (int pairs = 0; pairs < 2; ++pairs) {
            const Class& cl = w.classes[three][pairs];
            const int64_t begin = kind == kNext ? cl.next : kind == kSquare ? cl.gram_end : cl.symmetric;
            const int64_t end = kind == kNext ? cl.next_end : kind == kSquare ? cl.symmetric_end : cl.gram_end;
            if (begin == end || e != cudaSuccess) continue;
            const ProductArgs a = {o->d_mats, o->d_parts + begin, o->d_work, o->d_errors, (int32_t)(end - begin), (float)p.a, (float)p.b, (float)p.c,
                                   step & 1, o->polls, o->d_split, o->d_arrived, three || step == 0 ? 2 : 1};
            const Launch l = pairs ? launch_of<2>(kind, three, step == 0) : launch_of<1>(kind, three, step == 0);
            const int64_t most = (int64_t)o->sms * l.blocks / (pairs + 1);
            e = launch_overlapped(l.kernel, dim3((unsigned)(std::min(end - begin, most) * (pairs + 1))), dim3(l.threads), l.shared, st, HotRange{}, a);
        }
    return e;
}

int run(choco_muon* o, float* m, double lr, const float* factor, bool update, cudaStream_t st)
{
    const choco_muon_params& p = o->params;
    const MomentArgs ma = {o->d_mats, o->d_units, m, factor, o->d_partial, o->d_done, o->d_scale, o->d_errors, (float)p.beta, (float)(1.0 - p.beta), p.nesterov};
    TileArgs ta = {o->d_mats, nullptr, o->d_work, o->d_scale, o->d_errors, m, factor, (float)p.beta, (float)(1.0 - p.beta), (float)lr, p.nesterov, 0, 0, update};
    cudaError_t e = cudaSuccess;
    if (o->nunits > 0) e = launch_overlapped(moment_kernel, dim3((unsigned)o->nunits), dim3(kUnitThreads), 0, st, HotRange{}, ma);
    for (const Wave& w : o->waves) {
        auto tiles = [&](void (*kernel)(TileArgs)) {
            for (int three = 0; three < 2; ++three) {
                if (w.blocks[three] == w.blocks_end[three] || e != cudaSuccess) continue;
                ta.blocks = o->d_blocks + w.blocks[three];
                ta.planes = three || p.steps == 0 ? 2 : 1;
                e = launch_overlapped(kernel, dim3((unsigned)(w.blocks_end[three] - w.blocks[three])), dim3(kCutThreads), 0, st, HotRange{}, ta);
            }
        };
        tiles(cut_kernel);
        for (int k = 0; k < p.steps; ++k)
            for (int kind : {kGram, kSquare, kNext})
                if (e == cudaSuccess) e = launch_products(o, w, kind, k, st);
        ta.which = p.steps & 1;
        tiles(apply_kernel);
    }
    if (!o->small.empty() && e == cudaSuccess) {
        const SmallArgs sa = {ma, ta, o->d_small, o->d_errors, (float)p.a, (float)p.b, (float)p.c, p.steps, o->polls};
        e = launch_overlapped(small_kernel, dim3((unsigned)o->small.size()), dim3(kSmallThreads), (size_t)o->small_shared, st, HotRange{}, sa);
    }
    return status_of(e);
}

} // namespace

extern "C" {

int choco_muon_init(choco_muon** out, int32_t n_matrices, const choco_muon_matrix* matrices, const choco_muon_params* p)
{
    if (!out) return CHOCO_ERR_INVALID_ARG;
    *out = nullptr;
    if (n_matrices < 1 || !matrices || !p || p->groups < 1) return CHOCO_ERR_INVALID_ARG;
    if (!(p->beta >= 0.0 && p->beta < 1.0) || (p->nesterov != 0 && p->nesterov != 1) || p->steps < 0 || p->steps > 64) return CHOCO_ERR_INVALID_ARG;
    if (p->products != 0 && p->products != 1 && p->products != 3) return CHOCO_ERR_UNSUPPORTED;
    if (!polynomial_ok(*p)) return CHOCO_ERR_INVALID_ARG;
    choco_muon* o = new (std::nothrow) choco_muon();
    if (!o) return CHOCO_ERR_ALLOC;
    o->params = *p;
    o->polls = kSpinLimit;
    int rc = CHOCO_OK;
    try {
        std::vector<Unit> units;
        std::vector<Part> parts;
        std::vector<Block> blocks;
        int64_t work = 0;
        if (cudaGetDevice(&o->device) != cudaSuccess || cudaDeviceGetAttribute(&o->sms, cudaDevAttrMultiProcessorCount, o->device) != cudaSuccess)
            o->sms = 0; // (arguments are refused before the missing device is)
        rc = plan(o, n_matrices, matrices, units, parts, blocks, &work);
        if (rc == CHOCO_OK && overlap(o)) rc = CHOCO_ERR_INVALID_ARG;
        for (const Matrix& t : o->mats)
            if (rc == CHOCO_OK && is_written(o, t, t.g)) rc = CHOCO_ERR_INVALID_ARG;
        if (rc == CHOCO_OK) o->read = gradient_ranges(o->mats);
        if (rc == CHOCO_OK && o->sms == 0) rc = CHOCO_ERR_CUDA;
        if (rc == CHOCO_OK) rc = allocate(o, units, parts, blocks, work);
    } catch (const std::exception&) {
        rc = CHOCO_ERR_ALLOC;
    }
    if (rc != CHOCO_OK) {
        cudaGetLastError();
        free_all(o);
        return rc;
    }
    *out = o;
    return CHOCO_OK;
}

int choco_muon_destroy(choco_muon* opt)
{
    if (!opt) return CHOCO_ERR_INVALID_ARG;
    free_all(opt); // cudaFree waits for what still uses the memory
    return CHOCO_OK;
}

int choco_muon_state_size(const choco_muon* opt, int64_t* elements, int64_t* offsets)
{
    if (!opt || !elements) return CHOCO_ERR_INVALID_ARG;
    *elements = opt->elements;
    if (offsets) std::memcpy(offsets, opt->offsets.data(), sizeof(int64_t) * opt->offsets.size());
    return CHOCO_OK;
}

int choco_muon_set_grads(choco_muon* opt, const void* const* g, void* stream)
{
    if (!opt || !g || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    if (opt->timed_out) return CHOCO_ERR_TIMEOUT;
    for (size_t i = 0; i < opt->mats.size(); ++i) {
        const Matrix& t = opt->mats[i];
        if (t.rows > 0 && !g[i]) return CHOCO_ERR_INVALID_ARG;
        if (!aligned_to(g[i], dtype_size(t.g_dtype))) return CHOCO_ERR_MISALIGNED;
        if (is_written(opt, t, g[i])) return CHOCO_ERR_INVALID_ARG;
    }
    cudaStream_t st = (cudaStream_t)stream;
    try {
        std::vector<Matrix> mats = opt->mats;
        for (size_t i = 0; i < mats.size(); ++i) {
            mats[i].g = g[i];
            look_at_gradient(mats[i]);
        }
        std::vector<Range> read = gradient_ranges(mats);
        if (cudaStreamSynchronize(st) != cudaSuccess) return CHOCO_ERR_CUDA;
        opt->broken = true; // until the table on the device is whole
        if (cudaMemcpyAsync(opt->d_mats, mats.data(), sizeof(Matrix) * mats.size(), cudaMemcpyHostToDevice, st) != cudaSuccess ||
            cudaStreamSynchronize(st) != cudaSuccess)
            return CHOCO_ERR_CUDA;
        opt->mats.swap(mats);
        opt->read.swap(read);
        opt->broken = false;
    } catch (const std::exception&) {
        return CHOCO_ERR_ALLOC;
    }
    return CHOCO_OK;
}

int choco_muon_step(choco_muon* opt, float* m, double lr, const float* factor, void* stream)
{
    if (!opt || !(lr >= 0.0) || !std::isfinite((float)lr) || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    if (opt->elements > 0 && !m) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(m, 16) || !aligned_to(factor, 4)) return CHOCO_ERR_MISALIGNED;
    if (opt->elements > 0) {
        const Range r = range_of(m, 1, opt->elements, 0, CHOCO_F32);
        if (meets(opt->written, r) || meets(opt->read, r)) return CHOCO_ERR_INVALID_ARG;
    }
    if (opt->timed_out) return CHOCO_ERR_TIMEOUT;
    if (opt->broken) return CHOCO_ERR_CUDA;
    return run(opt, m, lr, factor, true, (cudaStream_t)stream);
}

int choco_muon_orthogonalize(choco_muon* opt, void* stream)
{
    if (!opt || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    if (opt->timed_out) return CHOCO_ERR_TIMEOUT;
    if (opt->broken) return CHOCO_ERR_CUDA;
    return run(opt, nullptr, 0.0, nullptr, false, (cudaStream_t)stream);
}

int choco_muon_status(choco_muon* opt, void* stream)
{
    if (!opt || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    uint32_t errors = 0;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemcpyAsync(&errors, opt->d_errors, sizeof(errors), cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return CHOCO_ERR_CUDA;
    if (errors) opt->timed_out = true;
    return opt->timed_out ? CHOCO_ERR_TIMEOUT : CHOCO_OK;
}

int choco_debug_muon_set_wait_polls(choco_muon* opt, uint32_t polls)
{
    if (!opt) return CHOCO_ERR_INVALID_ARG;
    opt->polls = polls > kSpinLimit ? kSpinLimit : polls;
    return CHOCO_OK;
}

} // extern "C"
