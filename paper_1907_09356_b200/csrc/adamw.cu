// AdamW over many tensors at once, with moments in 32 or in 8 bits, and the per-group gradient
// norms that feed it (choco_adamw_* in choco.h).
//
// A list of tensors is cut into chunks of kChunkElems elements of one tensor or fewer (twice as many
// where a long list has 8-bit moments and the chunk is of whole aligned blocks); a table in device
// memory says which tensor a chunk belongs to, so that one launch serves all tensors of all
// workers whatever their sizes.  Inside a chunk every warp owns blocks of kBlock = 256 elements, the
// unit that shares a scale in 8 bits.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "common.cuh"
#include "dtypes.cuh"

using namespace choco;

namespace {

constexpr int kBlock = 256;                 // elements that share a scale; tensors start on multiples of it in m and v
constexpr int kStepThreads = 128;            // short blocks: 256 threads took 5 % more, 64 no less
constexpr int kStepWarps = kStepThreads / 32;
constexpr int kChunkElems = kStepWarps * kBlock;
// Blocks of elements that a warp of the fast path has in flight.  With codes one is too few bytes to cover the
// chain of reads before it (8 x 25.6 M elements: 552 us with one, 505 us with two, though they spill up to 60 bytes
// of a thread's 48 registers, and 670 us with three, which spill 220); with 32-bit moments two, with 92 bytes
// spilled, are slower than one (16 x 28.95 M: 2.32 ms against 2.06 ms).
template <int BITS>
constexpr int kBlocksAtOnce = BITS == 8 ? 2 : 1;
// blocks on an SM: 64 registers a thread with 32-bit moments, 48 with codes, where more warps pay; 72 for single accesses (8 x 65
// small tensors: 12.1 us, 12.8 with six blocks)
constexpr int kStepBlocks32 = 8, kStepBlocks8 = 10, kStepBlocksRest = 7;
constexpr int kNormThreads = 128, kNormThreadsLong = 256; // 8 x 65 small tensors 6.1 us and 7.2 us, 16 x 28.95 M elements 262 us and 256 us
constexpr int64_t kUnitLong = 16384, kUnitShort = 2048; // elements of a unit of the norms
constexpr float kCodesM = 127.0f;           // codes k stand for s k^2, k up to 127 (m) and 255 (sqrt v)
constexpr float kCodesV = 255.0f;
constexpr float kTiny = 1e-30f;             // smallest largest-value of a block: keeps its reciprocal finite
constexpr double kNormEps = 1e-6;

struct Tensor {
    void* x;
    const void* g;
    void* copy;
    int64_t numel;
    int64_t state;          // first element in m and v
    float weight_decay, lr_scale;
    int32_t group;
    int8_t x_dtype, g_dtype, copy_dtype;
    int8_t aligned;         // every array on a 16-byte boundary
};

// A run of elements of one tensor.  `first`: the first one of its group (exactly one per group).
struct Chunk {
    int32_t tensor;
    int32_t first;
    int64_t begin;
};

// A run of elements of one tensor whose squares a block adds up; a group without elements has one of none.
struct Unit {
    int32_t tensor;
    int32_t group;
    int64_t begin;
};

// Steps of a handle, on the device: counts[0], those that the host has counted (calls that were no capture; written
// by each), and for every group counts[1 + group], what it has taken fewer than those.  A captured step knows
// neither when it is captured, so its replays take one off the group's count themselves.
// Correction: what a captured step multiplies with, one per group.
struct Correction {
    float step_size, rsqrt_bc2;
    int64_t n;              // its steps, this one included
};

struct StepScalars {
    float beta1, beta2, omb1, omb2, eps;
    float root_beta2, root_omb2; // sqrt(beta2), sqrt(1 - beta2)
    float lr;
    float step_size;        // lr / (1 - beta1^t)
    float rsqrt_bc2;        // 1 / sqrt(1 - beta2^t)
    float log_beta1, log_beta2; // natural logarithms
    int64_t t;
    int64_t whole_elems;    // of a chunk of whole aligned blocks
    const Correction* corrections; // of a captured step, [groups]; else NULL
    uint64_t seed;          // of the random rounding
};

__host__ __device__ inline double pow_int(double b, int64_t e)
{
    double r = 1.0;
    for (; e > 0; e >>= 1, b *= b)
        if (e & 1) r *= b;
    return r;
}

// largest of a warp's non-negative values (their order is that of their bits)
__device__ __forceinline__ float warp_max(float v)
{
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
}

__device__ __forceinline__ float root_approx(float v) // within 2^-22 of sqrt(v); subnormal numbers are taken for 0
{
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float root_approx_any(float v) // the same without that exception
{
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float reciprocal_approx(float v) // within 2^-22 of 1 / v, v not subnormal
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

constexpr float kRound = 12582912.0f; // 1.5 * 2^23: adding it rounds to an integer, held in the low bits
__device__ __forceinline__ uint32_t pack4(const float* k) // low bytes of four of those
{
    const uint32_t lo = __byte_perm(__float_as_uint(k[0]), __float_as_uint(k[1]), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(k[2]), __float_as_uint(k[3]), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
}
// 2^23 plus byte e of a word
__device__ __forceinline__ float byte_bits(uint32_t w, int e) { return __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540 | e)); }

// (h + 1/2) / 2^16 of 16 bits
__device__ __forceinline__ float unit_of(uint32_t h) { return __fadd_rn(__uint_as_float(0x3F800000u | h << 7), -0x1.ffffp-1f); }

// Codes as byte_bits leaves them (m's with 128 added) to k |k| and k^2: times the block's scale, m and sqrt(v).
__device__ __forceinline__ float square_m(float bits)
{
    const float k = __fadd_rn(bits, -8388736.0f);
    return k * fabsf(k);
}
__device__ __forceinline__ float square_v(float bits)
{
    const float k = __fadd_rn(bits, -8388608.0f);
    return k * k;
}

// 8 elements whose type is known at run time: 16 or 32 bytes, unpacked after all loads are under way
struct Raw8 {
    uint4 a, b;
};
__device__ __forceinline__ Raw8 load8(const void* p, int64_t i, int32_t dtype)
{
    Raw8 r;
    if (dtype == CHOCO_F32) {
        const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
        r.a = q[0];
        r.b = q[1];
    } else {
        r.a = *reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(p) + i);
        r.b = make_uint4(0, 0, 0, 0);
    }
    return r;
}
__device__ __forceinline__ void unpack8(const Raw8& r, int32_t dtype, float (&f)[8])
{
    if (dtype == CHOCO_F32) {
        f[0] = __uint_as_float(r.a.x); f[1] = __uint_as_float(r.a.y); f[2] = __uint_as_float(r.a.z); f[3] = __uint_as_float(r.a.w);
        f[4] = __uint_as_float(r.b.x); f[5] = __uint_as_float(r.b.y); f[6] = __uint_as_float(r.b.z); f[7] = __uint_as_float(r.b.w);
        return;
    }
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (dtype == CHOCO_BF16) {
            f[2 * k] = __uint_as_float(w[k] << 16);
            f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        } else {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
            f[2 * k] = v.x;
            f[2 * k + 1] = v.y;
        }
    }
}
__device__ __forceinline__ void store8(void* p, int64_t i, int32_t dtype, const float* f)
{
    if (dtype == CHOCO_F32) store_vec<float, 8>(static_cast<float*>(p) + i, f);
    else if (dtype == CHOCO_BF16) store_vec<__nv_bfloat16, 8>(static_cast<__nv_bfloat16*>(p) + i, f);
    else store_vec<__half, 8>(static_cast<__half*>(p) + i, f);
}

// What a step multiplies with, for one tensor of one group.
struct Factors {
    float c, step_size, rsqrt_bc2, decay;
    int64_t n;              // steps of the group, this one included
};

struct State {
    void *m, *v;
    float *m_scale, *v_scale;
};

// 8 elements with moments in 32 bits: IEEE operations one by one, so that the result is the
// formula's in float32, bit for bit.
__device__ __forceinline__ void update8(const StepScalars& sc, const Factors& f, float (&g)[8], float (&x)[8], float (&m)[8], float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        g[e] *= f.c;
        m[e] = m[e] * sc.beta1 + g[e] * sc.omb1;
        v[e] = v[e] * sc.beta2 + (g[e] * sc.omb2) * g[e];
        const float den = __fsqrt_rn(v[e]) * f.rsqrt_bc2 + sc.eps;
        x[e] = x[e] - (__fdiv_rn(m[e], den) * f.step_size + x[e] * f.decay);
    }
}

// A lane's 8 elements of a block with moments in 8 bits.  In: the codes as byte_bits leaves them and
// the block's scales; out: x, the new codes as floats that hold them in their low bytes, and the new
// scales.  Here instructions and registers, not bytes, would be the bound (with IEEE roots, quotients
// and separate products 99 instructions an element: 828 us for 8 x 25.6 M elements whose bytes, at
// the rate of a copy, take 507): products are fused, and roots and quotients are the approximate ones, whose 2^-22 is
// nothing beside the per cent that a code rounds by.  Elements past the end of a tensor come as
// zeros and stay zeros.
// RANDOM: a value between two codes' goes to either one, to the upper with the probability that makes
// the expected value (of m and of v, not of their roots) the value itself.  Nearest codes do not
// move while a value moves by less than half the distance to the next (1/k of m, 2/k of v), and v falls
// by no more than 1 - beta2 of itself a step.  `bits`: 16 random bits an element, whose bytes trade places for m.
// The generator and the second rounding cost a third of the time (8 x 25.6 M elements: 505 -> 677 us).
template <bool RANDOM>
__device__ __forceinline__ void update8_codes(const StepScalars& sc, const Factors& f, float (&g)[8], float (&x)[8], float (&m)[8],
                                              float (&v)[8], float& sm, float& sv, const uint32_t (&bits)[4])
{
    float amax = 0.f, rmax = 0.f;
    const float sm1 = sm * sc.beta1, sv2 = sv * sc.root_beta2, gm = f.c * sc.omb1, gv = f.c * sc.root_omb2;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        m[e] = __fmaf_rn(square_m(m[e]), sm1, g[e] * gm);
        const float r0 = square_v(v[e]) * sv2, q = g[e] * gv;
        v[e] = root_approx_any(__fmaf_rn(r0, r0, q * q)); // gradients of 1e-19 have subnormal squares, and a root of 1e-20
        const float ratio = m[e] * reciprocal_approx(__fmaf_rn(v[e], f.rsqrt_bc2, sc.eps));
        x[e] = __fmaf_rn(-f.step_size, ratio, __fmaf_rn(-f.decay, x[e], x[e]));
        amax = fmaxf(amax, fabsf(m[e]));
        rmax = fmaxf(rmax, v[e]);
    }
    amax = fmaxf(warp_max(amax), kTiny);
    rmax = fmaxf(warp_max(rmax), kTiny);
    sm = amax * (1.0f / (kCodesM * kCodesM));
    sv = rmax * (1.0f / (kCodesV * kCodesV));
    const float to_m = kCodesM * rsqrtf(amax), to_v = kCodesV * rsqrtf(rmax);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (RANDOM) {
            const uint32_t h = __byte_perm(bits[e / 2], 0, e & 1 ? 0x4432 : 0x4410), swapped = __byte_perm(h, 0, 0x4401);
            const float y = (fabsf(m[e]) * to_m) * to_m, w = (v[e] * to_v) * to_v;
            const float k = truncf(root_approx(y)), up = (2.f * k + 1.f) * unit_of(swapped) < __fmaf_rn(-k, k, y) ? 1.f : 0.f;
            m[e] = copysignf(fminf(k + up, kCodesM), m[e]) + kRound;
            const float q = truncf(root_approx(w)), q2 = q * q, odd = 2.f * q + 1.f;
            const float over = odd * unit_of(h) * __fmaf_rn(2.f, q2, odd) < __fmaf_rn(-q, q, w) * (w + q2) ? 1.f : 0.f;
            const float code = fminf(q + over, kCodesV) + kRound;
            v[e] = v[e] > 0.f ? fmaxf(code, kRound + 1.0f) : code;
        } else {
            m[e] = __fmaf_rn(copysignf(root_approx(fabsf(m[e])), m[e]), to_m, kRound);
            const float k = __fmaf_rn(root_approx(v[e]), to_v, kRound);
            v[e] = v[e] > 0.f ? fmaxf(k, kRound + 1.0f) : k; // at least 1 where v > 0
        }
    }
}

// The random bits of a lane's 8 consecutive elements of a block of moments, in the halves of four words: they go by the place
// in m and v, the group's step and the seed alone.
__device__ __forceinline__ void random_bits(uint32_t (&bits)[4], const StepScalars& sc, const Factors& f, int64_t block_start)
{
    const uint64_t at = (uint64_t)block_start / 8 + (threadIdx.x & 31);
    const uint4 r = philox4x32_10(make_uint4((uint32_t)at, (uint32_t)(at >> 32), (uint32_t)f.n, ((uint32_t)(f.n >> 32) << 8) | kStreamMoments),
                                  make_uint2((uint32_t)sc.seed, (uint32_t)(sc.seed >> 32)));
    bits[0] = r.x; bits[1] = r.y; bits[2] = r.z; bits[3] = r.w;
}
// The same bits where a lane has every 32nd element: element 32 j + lane is number lane % 8 of lane 4 j + lane / 8.
__device__ __forceinline__ void spread_bits(uint32_t (&bits)[4])
{
    const uint32_t lane = threadIdx.x & 31, which = (lane & 7) >> 1;
    uint32_t mine[4];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t w = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t other = __shfl_sync(0xffffffffu, bits[k], 4 * j + (lane >> 3));
            if (which == k) w = other;
        }
        const uint32_t h = lane & 1 ? w >> 16 : w & 0xffffu;
        mine[j / 2] = j & 1 ? mine[j / 2] | h << 16 : h;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) bits[k] = mine[k];
}

// What a lane needs of a whole block of an aligned tensor: 8 consecutive elements, moved in 128-bit
// accesses.
template <int BITS, typename XT, typename GT>
struct Loaded {
    Raw<GT, 8> g;
    Raw<XT, 8> x;
    Raw<float, BITS == 32 ? 8 : 2> m, v; // in 8 bits the two words are the codes
    float sm, sv;
};

template <int BITS, typename XT, typename GT>
__device__ __forceinline__ void load_block(Loaded<BITS, XT, GT>& l, const Tensor& t, const State& st, int64_t base)
{
    const int64_t i = base + (threadIdx.x & 31) * 8, s = t.state + i;
    load_raw(l.g, static_cast<const GT*>(t.g) + i);
    load_raw(l.x, static_cast<const XT*>(t.x) + i);
    if constexpr (BITS == 32) {
        load_raw(l.m, static_cast<const float*>(st.m) + s);
        load_raw(l.v, static_cast<const float*>(st.v) + s);
    } else {
        load_raw(l.m, reinterpret_cast<const float*>(static_cast<const uint8_t*>(st.m) + s));
        load_raw(l.v, reinterpret_cast<const float*>(static_cast<const uint8_t*>(st.v) + s));
        l.sm = st.m_scale[s / kBlock];
        l.sv = st.v_scale[s / kBlock];
    }
}

template <int BITS, bool RANDOM, typename XT, typename GT>
__device__ __forceinline__ void finish_block(Loaded<BITS, XT, GT>& l, const Tensor& t, const State& st, const StepScalars& sc,
                                             const Factors& f, int64_t base)
{
    const int64_t i = base + (threadIdx.x & 31) * 8, s = t.state + i;
    float g[8], x[8], m[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        g[e] = raw_get(l.g, e);
        x[e] = raw_get(l.x, e);
        if constexpr (BITS == 32) {
            m[e] = raw_get(l.m, e);
            v[e] = raw_get(l.v, e);
        } else {
            m[e] = byte_bits(l.m.w[e / 4] ^ 0x80808080u, e & 3);
            v[e] = byte_bits(l.v.w[e / 4], e & 3);
        }
    }
    if constexpr (BITS == 32) {
        update8(sc, f, g, x, m, v);
        store_vec<float, 8>(static_cast<float*>(st.m) + s, m);
        store_vec<float, 8>(static_cast<float*>(st.v) + s, v);
    } else {
        uint32_t bits[4];
        if constexpr (RANDOM) random_bits(bits, sc, f, t.state + base);
        update8_codes<RANDOM>(sc, f, g, x, m, v, l.sm, l.sv, bits);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(st.m) + s) = make_uint2(pack4(m), pack4(m + 4));
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(st.v) + s) = make_uint2(pack4(v), pack4(v + 4));
        if ((threadIdx.x & 31) == 0) {
            st.m_scale[s / kBlock] = l.sm;
            st.v_scale[s / kBlock] = l.sv;
        }
    }
    store_vec<XT, 8>(static_cast<XT*>(t.x) + i, x);
    if (t.copy) store8(t.copy, i, t.copy_dtype, x);
}

// Any block: a lane owns every 32nd element, so that single elements still make whole lines; the
// last block of a tensor and tensors that do not start on 16 bytes.
template <int BITS, typename XT, typename GT>
struct LoadedAny {
    Raw<GT, 1> g[8];
    Raw<XT, 1> x[8];
    float m[8], v[8], sm, sv;
};
template <int BITS, typename XT, typename GT>
__device__ __forceinline__ void load_block_any(LoadedAny<BITS, XT, GT>& l, const Tensor& t, const State& st, int64_t base, int count)
{
    const int lane = threadIdx.x & 31;
    const int64_t s0 = t.state + base;
    const GT* g = static_cast<const GT*>(t.g) + base + lane;
    const XT* x = static_cast<const XT*>(t.x) + base + lane;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        l.g[j].w[0] = l.x[j].w[0] = 0;
        l.m[j] = BITS == 32 ? 0.f : 8388736.0f; // code 0
        l.v[j] = BITS == 32 ? 0.f : 8388608.0f;
        if (j * 32 + lane >= count) continue;
        load_raw(l.g[j], g + j * 32);
        load_raw(l.x[j], x + j * 32);
        if constexpr (BITS == 32) {
            l.m[j] = static_cast<const float*>(st.m)[s0 + j * 32 + lane];
            l.v[j] = static_cast<const float*>(st.v)[s0 + j * 32 + lane];
        } else {
            l.m[j] = byte_bits(static_cast<const uint8_t*>(st.m)[s0 + j * 32 + lane] ^ 0x80u, 0);
            l.v[j] = byte_bits(static_cast<const uint8_t*>(st.v)[s0 + j * 32 + lane], 0);
        }
    }
    if constexpr (BITS == 8) {
        l.sm = st.m_scale[s0 / kBlock];
        l.sv = st.v_scale[s0 / kBlock];
    }
}
template <int BITS, bool RANDOM, typename XT, typename GT>
__device__ __forceinline__ void finish_block_any(LoadedAny<BITS, XT, GT>& l, const Tensor& t, const State& st, const StepScalars& sc,
                                                 const Factors& f, int64_t base, int count)
{
    const int lane = threadIdx.x & 31;
    const int64_t s0 = t.state + base;
    float g[8], x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        g[j] = raw_get(l.g[j], 0);
        x[j] = raw_get(l.x[j], 0);
    }
    if constexpr (BITS == 32) {
        update8(sc, f, g, x, l.m, l.v);
    } else {
        uint32_t bits[4];
        if constexpr (RANDOM) {
            random_bits(bits, sc, f, s0);
            spread_bits(bits);
        }
        update8_codes<RANDOM>(sc, f, g, x, l.m, l.v, l.sm, l.sv, bits);
        if (lane == 0) {
            st.m_scale[s0 / kBlock] = l.sm;
            st.v_scale[s0 / kBlock] = l.sv;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = j * 32 + lane;
        if (e >= count) continue;
        static_cast<XT*>(t.x)[base + e] = from_float<XT>(x[j]);
        if (t.copy) store_from_float(t.copy, base + e, t.copy_dtype, x[j]);
        if constexpr (BITS == 32) {
            static_cast<float*>(st.m)[s0 + e] = l.m[j];
            static_cast<float*>(st.v)[s0 + e] = l.v[j];
        } else {
            static_cast<uint8_t*>(st.m)[s0 + e] = (uint8_t)__float_as_uint(l.m[j]);
            static_cast<uint8_t*>(st.v)[s0 + e] = (uint8_t)__float_as_uint(l.v[j]);
        }
    }
}

// What this step multiplies with in one tensor; false: its group sits the step out.
// (The group's factor and count come as values, so that both are asked for before either is looked at.)
__device__ __forceinline__ bool factors_of(Factors& f, const Tensor& t, float c, int64_t skipped, const StepScalars& sc)
{
    f.c = c;
    f.step_size = sc.step_size;
    f.rsqrt_bc2 = sc.rsqrt_bc2;
    f.n = sc.t - skipped;
    if (sc.corrections) {
        f.step_size = sc.corrections[t.group].step_size;
        f.rsqrt_bc2 = sc.corrections[t.group].rsqrt_bc2;
        f.n = sc.corrections[t.group].n;
    } else if (skipped != 0) { // the group has taken another number of steps than the host has counted
        const float n = (float)f.n;
        f.step_size = __fdividef(sc.lr, -expm1f(n * sc.log_beta1));
        f.rsqrt_bc2 = rsqrtf(-expm1f(n * sc.log_beta2));
    }
    f.step_size *= t.lr_scale;
    f.decay = t.weight_decay * (sc.lr * t.lr_scale);
    return isfinite(c);
}

// Where the counts go, unless advance_kernel has seen to them.
__device__ __forceinline__ void count_call(int64_t* counts, const StepScalars& sc, int32_t beside)
{
    if (!beside && !sc.corrections && blockIdx.x == 0 && threadIdx.x == 0) counts[0] = sc.t;
}
__device__ __forceinline__ void count_skip(int64_t* counts, const StepScalars& sc, const Chunk& ch, int32_t group)
{
    if (!sc.corrections && ch.first && threadIdx.x == 0) counts[1 + group] += 1;
}

// The launch before a captured step's others: every group's corrections, from the steps it has taken when this
// runs, in float64 as the host forms them, and its new count.  Direct calls save this launch.
__global__ void __launch_bounds__(128) advance_kernel(int64_t* counts, const float* factor, Correction* out, int32_t groups, double beta1,
                                                      double beta2, double lr)
{
    wait_for_previous_kernel();
    allow_next_kernel();
    const int32_t k = blockIdx.x * 128 + threadIdx.x;
    if (k >= groups) return;
    if (factor && !isfinite(factor[k])) return; // sits the step out
    const int64_t n = counts[0] - counts[1 + k] + 1;
    out[k] = {(float)(lr / (1.0 - pow_int(beta1, n))), (float)(1.0 / sqrt(1.0 - pow_int(beta2, n))), n};
    counts[1 + k] -= 1;
}

// A step is, for each pair of types in the list, a launch of `step_rest_kernel` for the blocks that
// need single accesses and one of `step_kernel` for whole blocks of aligned tensors; most lists need one
// or two.  (In one kernel the first would set the registers of the others; a stack frame of 160
// bytes alone cost 40 % of their speed.)  They touch different elements and run side by side: each
// lets the next start as soon as all that came before the step has ended, and waits for the
// one before it only at its end.
// Nobody but the thread that finds `first` uses the count of a group that sits a step out, and no direct call
// reads counts[0].

// one block of threads per chunk, one warp per block of elements
template <int BITS, bool RANDOM, typename XT, typename GT>
__global__ void __launch_bounds__(kStepThreads, kStepBlocksRest)
step_rest_kernel(const Tensor* __restrict__ tensors, const Chunk* __restrict__ chunks, const float* factor,
                 int64_t* counts, State st, StepScalars sc, int32_t beside)
{
    const Chunk ch = chunks[blockIdx.x];
    const Tensor t = tensors[ch.tensor];
    if (!beside) wait_for_previous_kernel();
    allow_next_kernel();
    const int64_t base = ch.begin + (int64_t)(threadIdx.x >> 5) * kBlock;
    if (base < t.numel) {
        const int count = (int)min((int64_t)kBlock, t.numel - base);
        LoadedAny<BITS, XT, GT> l;
        load_block_any(l, t, st, base, count);
        Factors f;
        if (factors_of(f, t, factor ? factor[t.group] : 1.0f, counts[1 + t.group], sc)) finish_block_any<BITS, RANDOM>(l, t, st, sc, f, base, count);
        else count_skip(counts, sc, ch, t.group);
    }
    count_call(counts, sc, beside);
    if (beside) wait_for_previous_kernel();
}

// One block of threads per chunk, one warp per block of elements.  The chunks are taken from the
// last one: choco_adamw_grad_norm has read the gradients from the first one on, and what it read
// last is what the L2 cache still holds.  The list does not change between calls, so it is read
// before the previous kernel has ended; a warp's operands are asked for before the group's factor
// is known, since every latency in this chain is time in which nothing is in flight.
// A resident grid that walks over the chunks, with the list read ahead, was a fifth slower (16 x 28.95 M
// float32: 2.55 ms, now 2.06 ms): short blocks started in order keep what is in flight together
// in memory.
// A chunk may be shorter than what the warps could take: in a short list it holds one block of
// elements for each, and what follows belongs to the next chunk.
template <int BITS, bool RANDOM, typename XT, typename GT>
__global__ void __launch_bounds__(kStepThreads, BITS == 8 && !RANDOM ? kStepBlocks8 : kStepBlocks32)
step_kernel(const Tensor* __restrict__ tensors, const Chunk* __restrict__ chunks, const float* factor,
            int64_t* counts, State st, StepScalars sc, int32_t beside)
{
    constexpr int N = kBlocksAtOnce<BITS>;
    const Chunk ch = chunks[gridDim.x - 1 - blockIdx.x];
    const Tensor t = tensors[ch.tensor];
    if (!beside) wait_for_previous_kernel();
    allow_next_kernel();
    const int64_t base = ch.begin + (int64_t)(threadIdx.x >> 5) * kBlock;
    const int64_t end = min(t.numel / kBlock * kBlock, ch.begin + sc.whole_elems);
    Loaded<BITS, XT, GT> l[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (base + k * kChunkElems < end) load_block(l[k], t, st, base + k * kChunkElems);
    Factors f;
    if (factors_of(f, t, factor ? factor[t.group] : 1.0f, counts[1 + t.group], sc)) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (base + k * kChunkElems < end) finish_block<BITS, RANDOM>(l[k], t, st, sc, f, base + k * kChunkElems);
    } else {
        count_skip(counts, sc, ch, t.group);
    }
    count_call(counts, sc, beside);
    if (beside) wait_for_previous_kernel();
}

// Both kinds of chunks in one launch, for lists so short that a second launch takes longer than
// this kernel's registers cost.
template <int BITS, bool RANDOM, typename XT, typename GT>
__global__ void __launch_bounds__(kStepThreads, kStepBlocksRest)
step_both_kernel(const Tensor* __restrict__ tensors, const Chunk* __restrict__ chunks, const float* factor,
                 int64_t* counts, State st, StepScalars sc, int32_t beside)
{
    const Chunk ch = chunks[blockIdx.x];
    const Tensor t = tensors[ch.tensor];
    if (!beside) wait_for_previous_kernel();
    allow_next_kernel();
    const int64_t base = ch.begin + (int64_t)(threadIdx.x >> 5) * kBlock;
    const int64_t whole = t.aligned ? t.numel / kBlock * kBlock : 0; // where the tensor's other chunks begin
    Factors f;
    bool go = true;
    if (ch.begin < whole) {
        if (base < whole) {
            Loaded<BITS, XT, GT> l;
            load_block(l, t, st, base);
            go = factors_of(f, t, factor ? factor[t.group] : 1.0f, counts[1 + t.group], sc);
            if (go) finish_block<BITS, RANDOM>(l, t, st, sc, f, base);
        }
    } else if (base < t.numel) {
        const int count = (int)min((int64_t)kBlock, t.numel - base);
        LoadedAny<BITS, XT, GT> l;
        load_block_any(l, t, st, base, count);
        go = factors_of(f, t, factor ? factor[t.group] : 1.0f, counts[1 + t.group], sc);
        if (go) finish_block_any<BITS, RANDOM>(l, t, st, sc, f, base, count);
    }
    if (!go) count_skip(counts, sc, ch, t.group);
    count_call(counts, sc, beside);
    if (beside) wait_for_previous_kernel();
}

using StepKernel = void (*)(const Tensor*, const Chunk*, const float*, int64_t*, State, StepScalars, int32_t);
enum StepForm { kRest, kWhole, kBoth };
template <int BITS, bool RANDOM, typename XT, typename GT>
StepKernel step_kernel_of(StepForm form)
{
    return form == kRest    ? step_rest_kernel<BITS, RANDOM, XT, GT>
           : form == kWhole ? step_kernel<BITS, RANDOM, XT, GT>
                            : step_both_kernel<BITS, RANDOM, XT, GT>;
}
template <int BITS, bool RANDOM, typename XT>
StepKernel step_kernel_of(int32_t g, StepForm form)
{
    return g == CHOCO_F32    ? step_kernel_of<BITS, RANDOM, XT, float>(form)
           : g == CHOCO_BF16 ? step_kernel_of<BITS, RANDOM, XT, __nv_bfloat16>(form)
                             : step_kernel_of<BITS, RANDOM, XT, __half>(form);
}
template <int BITS, bool RANDOM>
StepKernel step_kernel_of(int32_t x, int32_t g, StepForm form)
{
    return x == CHOCO_F32    ? step_kernel_of<BITS, RANDOM, float>(g, form)
           : x == CHOCO_BF16 ? step_kernel_of<BITS, RANDOM, __nv_bfloat16>(g, form)
                             : step_kernel_of<BITS, RANDOM, __half>(g, form);
}

// 8 elements per thread; the moments are whole blocks.
template <int BITS>
__global__ void __launch_bounds__(256) read_state_kernel(State st, void* m_out, void* v_out, int32_t dtype, int64_t elements)
{
    wait_for_previous_kernel();
    allow_next_kernel();
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= elements) return;
    float m[8], v[8];
    if constexpr (BITS == 32) {
        if (m_out) unpack8(load8(st.m, i, CHOCO_F32), CHOCO_F32, m);
        if (v_out) unpack8(load8(st.v, i, CHOCO_F32), CHOCO_F32, v);
    } else {
        uint2 km = make_uint2(0, 0), kv = make_uint2(0, 0);
        float sm = 0.f, sv = 0.f;
        if (m_out) { km = *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(st.m) + i); sm = st.m_scale[i / kBlock]; }
        if (v_out) { kv = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(st.v) + i); sv = st.v_scale[i / kBlock]; }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = byte_bits((e < 4 ? km.x : km.y) ^ 0x80808080u, e & 3);
            v[e] = byte_bits(e < 4 ? kv.x : kv.y, e & 3);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = square_m(m[e]) * sm;
            const float r = square_v(v[e]) * sv;
            v[e] = r * r;
        }
    }
    if (m_out) store8(m_out, i, dtype, m);
    if (v_out) store8(v_out, i, dtype, v);
}

// Sums of squares in float64: squares of float32 values neither overflow nor vanish there.  A block
// takes one unit (a run of one tensor's gradient); the last block of a group to finish adds up the
// group's units in their order and forms its norm and factor.  What bounds it is the memory
// (16 x 28.95 M float32: 259 us, 7.2 TB/s; rows off 16-byte boundaries take single loads, 311 us for half
// as many).
template <int THREADS>
__device__ __forceinline__ double sum_of_block(double acc, double* red) // thread 0 has the sum
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = acc;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < THREADS / 32; ++w) acc += red[w];
    return acc;
}

struct NormOut {
    double* partial;             // [units]
    const int64_t* unit_begin;   // [groups + 1]: the units of a group are contiguous
    uint32_t* done;              // [groups] blocks that have finished; all zeros between calls
    float max_norm, unscale;
    float *norm, *factor;
};

template <int THREADS>
__global__ void __launch_bounds__(THREADS)
norm_kernel(const Tensor* __restrict__ tensors, const Unit* __restrict__ units, int64_t unit_elems, NormOut o)
{
    __shared__ double red[THREADS / 32];
    __shared__ bool last;
    const Unit u = units[blockIdx.x];
    const Tensor t = tensors[u.tensor];
    const int64_t u0 = o.unit_begin[u.group], u1 = o.unit_begin[u.group + 1];
    wait_for_previous_kernel();
    allow_next_kernel();
    const int64_t end = min(u.begin + unit_elems, t.numel);
    double acc = 0.0;
    int64_t done = u.begin;
    if (t.aligned) {
        constexpr int kAhead = 4;           // vectors of a thread in flight
        constexpr int kSpanElems = THREADS * 8;
        auto span = [&](auto vectors) {
            constexpr int N = decltype(vectors)::value;
            Raw8 r[N];
#pragma unroll
            for (int k = 0; k < N; ++k) r[k] = load8(t.g, done + k * kSpanElems + threadIdx.x * 8, t.g_dtype);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float g[8];
                unpack8(r[k], t.g_dtype, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc = __fma_rn((double)g[e], (double)g[e], acc);
            }
            done += N * kSpanElems;
        };
        while (done + kAhead * kSpanElems <= end) span(std::integral_constant<int, kAhead>());
        if (done + 2 * kSpanElems <= end) span(std::integral_constant<int, 2>());
        if (done + kSpanElems <= end) span(std::integral_constant<int, 1>());
    }
    constexpr int kSingles = 8;             // single elements of a thread in flight
    for (; done < end; done += kSingles * THREADS) {
        uint32_t g[kSingles];
#pragma unroll
        for (int k = 0; k < kSingles; ++k) {
            const int64_t e = done + k * THREADS + threadIdx.x;
            g[k] = e < end ? load_bits(t.g, e, t.g_dtype) : 0u;
        }
#pragma unroll
        for (int k = 0; k < kSingles; ++k) {
            const double d = (double)bits_to_float(g[k], t.g_dtype);
            acc = __fma_rn(d, d, acc);
        }
    }
    acc = sum_of_block<THREADS>(acc, red);
    if (threadIdx.x == 0) {
        o.partial[blockIdx.x] = acc;
        __threadfence(); // before the count, so that the last block finds it
        last = atomicAdd(&o.done[u.group], 1u) == (uint32_t)(u1 - u0) - 1u;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    acc = 0.0;
    for (int64_t k = u0 + threadIdx.x; k < u1; k += THREADS) acc += __ldcg(o.partial + k);
    acc = sum_of_block<THREADS>(acc, red);
    if (threadIdx.x == 0) {
        o.done[u.group] = 0;
        const double nrm = (double)o.unscale * sqrt(acc);
        const float rounded = (float)nrm; // infinite above float32's largest number too
        o.norm[u.group] = rounded;
        double f = (double)o.unscale;
        if (o.max_norm > 0.f) {
            const double clip = (double)o.max_norm / (nrm + kNormEps);
            f *= clip < 1.0 ? clip : 1.0;
        }
        o.factor[u.group] = isfinite(rounded) ? (float)f : __int_as_float(0x7fc00000);
    }
}

} // namespace

// Lists of up to this many chunks take one launch for both kinds of blocks: 8 x 65 tensors of a ResNet-20, 11.9 us
// against 12.9; 16 M elements, 68.1 against 68.8.  With codes the registers cost more: 4.4 M elements, 14.8 us
// against 16.3; 16 M, 51 against 46.
constexpr int64_t kTogether32 = 32768, kTogether8 = 8192;
constexpr int kPairs = 9;               // of types: 3 x_dtype + g_dtype

namespace {
struct Range { // of addresses
    uintptr_t begin, end;
};
} // namespace

struct choco_adamw {
    choco_adamw_params params;
    int device;
    bool norm_only;                // no parameters: the list serves choco_adamw_grad_norm alone
    bool broken;                   // the tables on the device may be half written (a copy of new ones failed)
    std::vector<Tensor> tensors;   // as on the device
    std::vector<Range> written;    // by a step, in order of their addresses
    std::vector<int64_t> offsets;
    int64_t elements;              // of m and v
    std::vector<int32_t> by_group;  // tensors with elements, group after group
    int64_t most_chunks, nunits, unit_elems;
    bool together;                 // a short list: one launch for all blocks of a pair of types
    int64_t whole_elems;           // of a chunk of whole aligned blocks
    int64_t begin[2 * kPairs + 1]; // in d_chunks, for every pair of types: other blocks, whole blocks of aligned tensors
    int64_t t;                     // step calls so far that were no capture; a group has taken t - d_counts[1 + group] steps
    bool random_codes;             // how 8-bit codes are rounded
    uint64_t seed;
    bool captured;                 // a graph may hold launches over ranges of d_chunks
    void* memory;                  // all that follows
    Tensor* d_tensors;
    Chunk* d_chunks;               // room for most_chunks
    Unit* d_units;
    int64_t* d_unit_begin;         // [groups + 1]
    int64_t* d_counts;             // [1 + groups]
    Correction* d_corrections;     // [groups]
    double* d_partial;             // [nunits]
    uint32_t* d_done;              // [groups]
};

namespace {

bool on_device(const choco_adamw* o)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == o->device;
}

// Device memory for everything, in one allocation, and what of it has a first value in one copy.
// Throws std::bad_alloc.
int allocate(choco_adamw* o, const std::vector<Chunk>& chunks, const std::vector<Unit>& units, const std::vector<int64_t>& unit_begin)
{
    const size_t groups = (size_t)o->params.groups;
    std::vector<char> first;
    size_t at[8];
    auto place = [&](int k, const void* from, size_t bytes, size_t room) {
        at[k] = (first.size() + 255) / 256 * 256;
        first.resize(at[k] + (room > bytes ? room : bytes), 0);
        if (bytes) std::memcpy(first.data() + at[k], from, bytes);
    };
    place(0, o->tensors.data(), sizeof(Tensor) * o->tensors.size(), 0);
    place(1, chunks.data(), sizeof(Chunk) * chunks.size(), sizeof(Chunk) * (size_t)o->most_chunks);
    place(2, units.data(), sizeof(Unit) * units.size(), 0);
    place(3, unit_begin.data(), sizeof(int64_t) * unit_begin.size(), 0);
    place(4, nullptr, 0, sizeof(int64_t) * (1 + groups));
    place(5, nullptr, 0, sizeof(uint32_t) * groups);
    place(6, nullptr, 0, sizeof(Correction) * groups);
    at[7] = (first.size() + 255) / 256 * 256;
    if (cudaMalloc(&o->memory, at[7] + sizeof(double) * units.size()) != cudaSuccess) {
        o->memory = nullptr;
        return CHOCO_ERR_ALLOC;
    }
    // a copy from pageable memory may return before it has arrived, and a call on another stream would not wait for it
    if (cudaMemcpy(o->memory, first.data(), first.size(), cudaMemcpyHostToDevice) != cudaSuccess ||
        cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess)
        return CHOCO_ERR_CUDA;
    char* const m = static_cast<char*>(o->memory);
    o->d_tensors = reinterpret_cast<Tensor*>(m + at[0]);
    o->d_chunks = reinterpret_cast<Chunk*>(m + at[1]);
    o->d_units = reinterpret_cast<Unit*>(m + at[2]);
    o->d_unit_begin = reinterpret_cast<int64_t*>(m + at[3]);
    o->d_counts = reinterpret_cast<int64_t*>(m + at[4]);
    o->d_done = reinterpret_cast<uint32_t*>(m + at[5]);
    o->d_corrections = reinterpret_cast<Correction*>(m + at[6]);
    o->d_partial = reinterpret_cast<double*>(m + at[7]);
    return CHOCO_OK;
}

int status_of(cudaError_t e)
{
    if (e == cudaSuccess) return CHOCO_OK;
    cudaGetLastError();
    return CHOCO_ERR_CUDA;
}

void free_all(choco_adamw* o)
{
    cudaFree(o->memory);
    delete o;
}

bool all_aligned(const Tensor& t) { return aligned_to(t.x, 16) && aligned_to(t.g, 16) && aligned_to(t.copy, 16); }

Range range_of(const void* p, int64_t numel, int32_t dtype)
{
    return {(uintptr_t)p, (uintptr_t)p + (uintptr_t)(numel * dtype_size(dtype))};
}
// What a step writes, in order; false if two of these arrays share memory.  Throws std::bad_alloc.
bool collect_written(choco_adamw* o)
{
    std::vector<Range>& w = o->written;
    for (const Tensor& t : o->tensors) {
        if (t.numel > 0 && t.x) w.push_back(range_of(t.x, t.numel, t.x_dtype));
        if (t.numel > 0 && t.copy) w.push_back(range_of(t.copy, t.numel, t.copy_dtype));
    }
    std::sort(w.begin(), w.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    for (size_t i = 1; i < w.size(); ++i)
        if (w[i].begin < w[i - 1].end) return false;
    return true;
}
bool is_written(const choco_adamw* o, const Tensor& t, const void* g)
{
    if (t.numel == 0) return false;
    const Range r = range_of(g, t.numel, t.g_dtype);
    // of the arrays that begin before r ends the last one reaches furthest
    auto next = std::lower_bound(o->written.begin(), o->written.end(), r.end, [](const Range& a, uintptr_t e) { return a.begin < e; });
    return next != o->written.begin() && (next - 1)->end > r.begin;
}

// Fills the host tables of `o`.  Throws std::bad_alloc.
int plan(choco_adamw* o, int32_t n, const choco_adamw_tensor* ts, std::vector<Unit>& units, std::vector<int64_t>& unit_begin)
{
    const int32_t groups = o->params.groups;
    std::vector<std::vector<int32_t>> members(groups);
    int64_t at = 0, total = 0;
    o->norm_only = false;
    for (int32_t i = 0; i < n; ++i) {
        const choco_adamw_tensor& t = ts[i];
        if (t.numel < 0 || t.numel > (int64_t)1 << 38 || t.group < 0 || t.group >= groups) return CHOCO_ERR_INVALID_ARG;
        if (!dtype_ok(t.x_dtype) || !dtype_ok(t.g_dtype) || !dtype_ok(t.copy_dtype)) return CHOCO_ERR_INVALID_ARG;
        if (!(t.weight_decay >= 0.0) || !(t.lr_scale >= 0.0) || !std::isfinite((float)t.weight_decay) || !std::isfinite((float)t.lr_scale))
            return CHOCO_ERR_INVALID_ARG;
        if (t.numel > 0 && !t.g) return CHOCO_ERR_INVALID_ARG;
        if (t.numel > 0 && !t.x) o->norm_only = true;
        if (!aligned_to(t.x, dtype_size(t.x_dtype)) || !aligned_to(t.g, dtype_size(t.g_dtype)) ||
            !aligned_to(t.copy, dtype_size(t.copy_dtype)))
            return CHOCO_ERR_MISALIGNED;
        Tensor d = {};
        d.x = t.x; d.g = t.g; d.copy = t.copy;
        d.numel = t.numel;
        d.state = at;
        d.weight_decay = (float)t.weight_decay;
        d.lr_scale = (float)t.lr_scale;
        d.group = t.group;
        d.x_dtype = (int8_t)t.x_dtype; d.g_dtype = (int8_t)t.g_dtype; d.copy_dtype = (int8_t)t.copy_dtype;
        d.aligned = all_aligned(d);
        o->tensors.push_back(d);
        o->offsets.push_back(at);
        at += (t.numel + kBlock - 1) / kBlock * kBlock;
        total += t.numel;
        if (at > (int64_t)1 << 38) return CHOCO_ERR_TOO_LARGE;
        if (t.numel > 0) members[t.group].push_back(i);
    }
    o->elements = at;
    if (!o->norm_only) {
        if (!collect_written(o)) return CHOCO_ERR_INVALID_ARG;
        for (const Tensor& t : o->tensors)
            if (is_written(o, t, t.g)) return CHOCO_ERR_INVALID_ARG;
    }
    // short units where the whole list has fewer than four long ones for each SM
    o->unit_elems = total >= kUnitLong * 4 * 148 ? kUnitLong : kUnitShort;
    for (int32_t k = 0; k < groups; ++k) {
        unit_begin.push_back((int64_t)units.size());
        for (int32_t i : members[k]) {
            o->by_group.push_back(i);
            o->most_chunks += o->tensors[i].numel / kChunkElems + 2;
            for (int64_t b = 0; b < o->tensors[i].numel; b += o->unit_elems) units.push_back({i, k, b});
        }
        if (members[k].empty()) units.push_back({0, k, o->tensors[0].numel});
    }
    unit_begin.push_back((int64_t)units.size());
    o->nunits = (int64_t)units.size();
    const bool eight = o->params.state_bits == 8;
    o->together = o->most_chunks <= (eight ? kTogether8 : kTogether32);
    o->whole_elems = kChunkElems * (o->together || !eight ? 1 : kBlocksAtOnce<8>);
    if (o->norm_only) o->most_chunks = 0; // no step
    return o->most_chunks > 0x7fffffff || o->nunits > 0x7fffffff ? CHOCO_ERR_TOO_LARGE : CHOCO_OK;
}

// Cuts the tensors into chunks, never more than most_chunks; begin: where each range starts.  Throws
// std::bad_alloc.
std::vector<Chunk> cut(const choco_adamw* o, const std::vector<Tensor>& tensors, int64_t* begin)
{
    std::vector<Chunk> chunks;
    std::vector<char> seen((size_t)o->params.groups, 0);
    chunks.reserve((size_t)o->most_chunks);
    for (int32_t k = 0; k < 2 * kPairs; ++k) {
        begin[k] = (int64_t)chunks.size();
        for (int32_t i : o->by_group) {
            const Tensor& t = tensors[i];
            if (t.x_dtype * 3 + t.g_dtype != k / 2) continue;
            const int64_t whole = t.aligned ? t.numel / kBlock * kBlock : 0;
            for (int64_t b = k % 2 ? 0 : whole; b < (k % 2 ? whole : t.numel); b += k % 2 ? o->whole_elems : kChunkElems) {
                chunks.push_back({i, !seen[t.group], b});
                seen[t.group] = 1;
            }
        }
    }
    begin[2 * kPairs] = (int64_t)chunks.size();
    return chunks;
}

} // namespace

extern "C" {

int choco_adamw_init(choco_adamw** out, int32_t n_tensors, const choco_adamw_tensor* tensors, const choco_adamw_params* p)
{
    if (!out) return CHOCO_ERR_INVALID_ARG;
    *out = nullptr;
    if (n_tensors < 1 || !tensors || !p || p->groups < 1) return CHOCO_ERR_INVALID_ARG;
    if (!(p->beta1 >= 0.0 && p->beta1 < 1.0) || !(p->beta2 >= 0.0 && p->beta2 < 1.0) || !((float)p->eps > 0.f) || !std::isfinite((float)p->eps))
        return CHOCO_ERR_INVALID_ARG;
    if (p->state_bits != 32 && p->state_bits != 8) return CHOCO_ERR_UNSUPPORTED;
    if (p->state_bits == 8 && (float)p->eps < FLT_MIN) return CHOCO_ERR_INVALID_ARG; // the approximate quotient takes it for 0
    choco_adamw* o = new (std::nothrow) choco_adamw();
    if (!o) return CHOCO_ERR_ALLOC;
    o->params = *p;
    int rc = CHOCO_OK;
    try {
        std::vector<Chunk> chunks;
        std::vector<Unit> units;
        std::vector<int64_t> unit_begin;
        rc = plan(o, n_tensors, tensors, units, unit_begin);
        if (rc == CHOCO_OK && !o->norm_only) chunks = cut(o, o->tensors, o->begin);
        if (rc == CHOCO_OK && cudaGetDevice(&o->device) != cudaSuccess) rc = CHOCO_ERR_CUDA;
        if (rc == CHOCO_OK) rc = allocate(o, chunks, units, unit_begin);
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

int choco_adamw_destroy(choco_adamw* opt)
{
    if (!opt) return CHOCO_ERR_INVALID_ARG;
    free_all(opt); // cudaFree waits for what still uses the memory
    return CHOCO_OK;
}

int choco_adamw_state_size(const choco_adamw* opt, int64_t* elements, int64_t* offsets)
{
    if (!opt || !elements) return CHOCO_ERR_INVALID_ARG;
    *elements = opt->elements;
    if (offsets) std::memcpy(offsets, opt->offsets.data(), sizeof(int64_t) * opt->offsets.size());
    return CHOCO_OK;
}

int choco_adamw_set_grads(choco_adamw* opt, const void* const* g, void* stream)
{
    if (!opt || !g || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    for (size_t i = 0; i < opt->tensors.size(); ++i) {
        if (opt->tensors[i].numel > 0 && !g[i]) return CHOCO_ERR_INVALID_ARG;
        if (!aligned_to(g[i], dtype_size(opt->tensors[i].g_dtype))) return CHOCO_ERR_MISALIGNED;
        if (is_written(opt, opt->tensors[i], g[i])) return CHOCO_ERR_INVALID_ARG;
    }
    cudaStream_t st = (cudaStream_t)stream;
    auto send = [&](auto* to, const auto& from) {
        return from.empty() || cudaMemcpyAsync(to, from.data(), sizeof(from[0]) * from.size(), cudaMemcpyHostToDevice, st) == cudaSuccess;
    };
    try {
        std::vector<Tensor> tensors = opt->tensors;
        std::vector<Chunk> chunks;
        int64_t begin[2 * kPairs + 1];
        bool moved = false; // a tensor's accesses change width with its gradient's alignment
        for (size_t i = 0; i < tensors.size(); ++i) {
            tensors[i].g = g[i];
            tensors[i].aligned = all_aligned(tensors[i]);
            moved |= tensors[i].aligned != opt->tensors[i].aligned;
        }
        moved = moved && !opt->norm_only;
        if (moved && opt->captured) return CHOCO_ERR_UNSUPPORTED; // a replay would find other chunks in the ranges it was captured with
        if (moved) chunks = cut(opt, tensors, begin);
        if (cudaStreamSynchronize(st) != cudaSuccess) return CHOCO_ERR_CUDA;
        // the tables on the device have to agree with each other and with the host's: if one copy fails, no call may use them
        opt->broken = true;
        if (!send(opt->d_tensors, tensors) || !send(opt->d_chunks, chunks) || cudaStreamSynchronize(st) != cudaSuccess)
            return CHOCO_ERR_CUDA;
        opt->tensors.swap(tensors);
        if (moved) std::memcpy(opt->begin, begin, sizeof(begin));
        opt->broken = false;
    } catch (const std::exception&) {
        return CHOCO_ERR_ALLOC;
    }
    return CHOCO_OK;
}

int choco_adamw_set_rounding(choco_adamw* opt, int32_t random, uint64_t seed)
{
    if (!opt || (random != 0 && random != 1)) return CHOCO_ERR_INVALID_ARG;
    if (opt->params.state_bits != 8) return CHOCO_ERR_UNSUPPORTED;
    opt->random_codes = random != 0;
    opt->seed = seed;
    return CHOCO_OK;
}

int choco_adamw_grad_norm(choco_adamw* opt, float max_norm, float unscale, float* norm, float* factor, void* stream)
{
    if (!opt || !norm || !factor || !(max_norm >= 0.f) || !std::isfinite(max_norm) || !(unscale > 0.f) ||
        !std::isfinite(unscale) || !on_device(opt))
        return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(norm, 4) || !aligned_to(factor, 4)) return CHOCO_ERR_MISALIGNED;
    if (opt->broken) return CHOCO_ERR_CUDA;
    const NormOut o = {opt->d_partial, opt->d_unit_begin, opt->d_done, max_norm, unscale, norm, factor};
    const bool many = opt->unit_elems == kUnitLong;
    return status_of(launch_overlapped(many ? norm_kernel<kNormThreadsLong> : norm_kernel<kNormThreads>, dim3((unsigned)opt->nunits),
                                       dim3(many ? kNormThreadsLong : kNormThreads), 0, (cudaStream_t)stream, HotRange{}, opt->d_tensors,
                                       opt->d_units, opt->unit_elems, o));
}

int choco_adamw_step(choco_adamw* opt, void* m, void* v, float* m_scale, float* v_scale, double lr, const float* factor,
                     void* stream)
{
    if (!opt || opt->norm_only || !(lr >= 0.0) || !std::isfinite((float)lr) || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    const bool eight = opt->params.state_bits == 8;
    if (opt->elements > 0 && (!m || !v || (eight && (!m_scale || !v_scale)))) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(m, 16) || !aligned_to(v, 16) || !aligned_to(m_scale, 4) || !aligned_to(v_scale, 4) || !aligned_to(factor, 4))
        return CHOCO_ERR_MISALIGNED;
    if (opt->broken) return CHOCO_ERR_CUDA;
    const choco_adamw_params& p = opt->params;
    StepScalars sc;
    sc.t = opt->t + 1;
    sc.beta1 = (float)p.beta1; sc.beta2 = (float)p.beta2;
    sc.omb1 = (float)(1.0 - p.beta1); sc.omb2 = (float)(1.0 - p.beta2);
    sc.eps = (float)p.eps;
    sc.root_beta2 = (float)std::sqrt(p.beta2);
    sc.root_omb2 = (float)std::sqrt(1.0 - p.beta2);
    sc.lr = (float)lr;
    sc.log_beta1 = (float)std::log(p.beta1); sc.log_beta2 = (float)std::log(p.beta2);
    sc.step_size = (float)(lr / (1.0 - pow_int(p.beta1, sc.t)));
    sc.rsqrt_bc2 = (float)(1.0 / std::sqrt(1.0 - pow_int(p.beta2, sc.t)));
    sc.whole_elems = opt->whole_elems;
    sc.seed = opt->seed;
    cudaStream_t st = (cudaStream_t)stream;
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    cudaError_t err = cudaStreamIsCapturing(st, &capture);
    if (status_of(err) != CHOCO_OK) return CHOCO_ERR_CUDA;
    const bool capturing = capture != cudaStreamCaptureStatusNone;
    sc.corrections = capturing ? opt->d_corrections : nullptr;
    const State state = {m, v, m_scale, v_scale};
    if (capturing) {
        opt->captured = true;
        err = launch_overlapped(advance_kernel, dim3((unsigned)((p.groups + 127) / 128)), dim3(128), 0, st, HotRange{}, opt->d_counts, factor,
                                opt->d_corrections, p.groups, p.beta1, p.beta2, lr);
    }
    int32_t beside = 0;
    auto launch = [&](int32_t pair, StepForm form, int64_t begin, int64_t end) {
        if (begin == end || err != cudaSuccess) return;
        const int32_t x = pair / 3, g = pair % 3;
        const StepKernel kernel = !eight              ? step_kernel_of<32, false>(x, g, form)
                                  : opt->random_codes ? step_kernel_of<8, true>(x, g, form)
                                                      : step_kernel_of<8, false>(x, g, form);
        err = launch_overlapped(kernel, dim3((unsigned)(end - begin)),
                                dim3(kStepThreads), 0, st, HotRange{}, opt->d_tensors, opt->d_chunks + begin, factor, opt->d_counts,
                                state, sc, beside);
        beside = 1;
    };
    for (int32_t pair = 0; pair < kPairs; ++pair) {
        const int64_t* b = opt->begin + 2 * pair;
        if (opt->together && b[0] < b[1] && b[1] < b[2]) {
            launch(pair, kBoth, b[0], b[2]);
        } else {
            launch(pair, kRest, b[0], b[1]);
            launch(pair, kWhole, b[1], b[2]);
        }
    }
    if (status_of(err) != CHOCO_OK) return CHOCO_ERR_CUDA;
    if (!capturing) opt->t += 1;
    return CHOCO_OK;
}

int choco_adamw_read_state(choco_adamw* opt, const void* m, const void* v, const float* m_scale, const float* v_scale,
                           void* m_out, void* v_out, int32_t out_dtype, void* stream)
{
    if (!opt || !dtype_ok(out_dtype) || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    const bool eight = opt->params.state_bits == 8;
    if ((m_out && !m) || (v_out && !v) || (eight && ((m_out && !m_scale) || (v_out && !v_scale)))) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(m, 16) || !aligned_to(v, 16) || !aligned_to(m_scale, 4) || !aligned_to(v_scale, 4) ||
        !aligned_to(m_out, 16) || !aligned_to(v_out, 16))
        return CHOCO_ERR_MISALIGNED;
    if (opt->elements == 0 || (!m_out && !v_out)) return CHOCO_OK;
    const State state = {const_cast<void*>(m), const_cast<void*>(v), const_cast<float*>(m_scale), const_cast<float*>(v_scale)};
    const dim3 grid((unsigned)((opt->elements / 8 + 255) / 256)), threads(256);
    return status_of(launch_overlapped(eight ? read_state_kernel<8> : read_state_kernel<32>, grid, threads, 0, (cudaStream_t)stream,
                                       HotRange{}, state, m_out, v_out, out_dtype, opt->elements));
}

int choco_adamw_get_steps(choco_adamw* opt, int64_t* steps, void* stream)
{
    if (!opt || !steps || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    const size_t bytes = sizeof(int64_t) * (size_t)opt->params.groups;
    if (cudaMemcpyAsync(steps, opt->d_counts + 1, bytes, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess)
        return CHOCO_ERR_CUDA;
    for (int32_t k = 0; k < opt->params.groups; ++k) steps[k] = opt->t - steps[k];
    return CHOCO_OK;
}

int choco_adamw_set_steps(choco_adamw* opt, const int64_t* steps, void* stream)
{
    if (!opt || !steps || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    int64_t most = 0;
    for (int32_t k = 0; k < opt->params.groups; ++k) {
        if (steps[k] < 0) return CHOCO_ERR_INVALID_ARG;
        most = steps[k] > most ? steps[k] : most;
    }
    cudaStream_t st = (cudaStream_t)stream;
    try {
        std::vector<int64_t> counts(1 + (size_t)opt->params.groups);
        counts[0] = most;
        for (int32_t k = 0; k < opt->params.groups; ++k) counts[1 + k] = most - steps[k];
        if (cudaMemcpyAsync(opt->d_counts, counts.data(), sizeof(int64_t) * counts.size(), cudaMemcpyHostToDevice, st) != cudaSuccess ||
            cudaStreamSynchronize(st) != cudaSuccess)
            return CHOCO_ERR_CUDA;
    } catch (const std::exception&) {
        return CHOCO_ERR_ALLOC;
    }
    opt->t = most;
    return CHOCO_OK;
}

} // extern "C"
