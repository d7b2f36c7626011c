// AdamW over many tensors at once, with moments in 32 or in 8 bits, and the per-group gradient
// norms that feed it (choco_adamw_* in choco.h).
//
// A list of tensors is cut into chunks of at most kChunkElems elements of one tensor; a table in
// device memory says which tensor a chunk belongs to, so that one launch serves all tensors of all
// workers whatever their sizes.  Inside a chunk every warp owns blocks of kBlock = 256 elements, the
// unit that shares a scale in 8 bits.
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "common.cuh"
#include "dtypes.cuh"

using namespace choco;

namespace {

constexpr int kBlock = 256;                 // elements that share a scale; tensors start on multiples of it in m and v
constexpr int kStepThreads = 256;
constexpr int kStepWarps = kStepThreads / 32;
constexpr int kChunkElems = kStepWarps * kBlock;
constexpr int kNormThreads = 256;
constexpr float kLevelsM = 127.0f * 127.0f; // codes k stand for s k^2, k up to 127 (m) and 255 (sqrt v)
constexpr float kLevelsV = 255.0f * 255.0f;
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

struct StepScalars {
    float beta1, beta2, omb1, omb2, eps;
    float lr;
    float step_size;        // lr / (1 - beta1^t)
    float rsqrt_bc2;        // 1 / sqrt(1 - beta2^t)
    double beta1d, beta2d, lrd;
    int64_t t;
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

// The nearest k to sqrt(y), y in [0, levels^2]: the number of edges (j - 1/2)^2, j = 1 .., that y
// reaches (the edges are exact in float32, so that the code does not hang on a square root's
// rounding).  The approximate root is off by less than 255 * 2^-21 = 1.22e-4; taken 1.3e-4 too low
// it rounds to k or k - 1, and one comparison decides.  Returned as a float.
__device__ __forceinline__ float nearest_root(float y)
{
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
    constexpr float kRound = 12582912.0f; // 1.5 * 2^23: adding it rounds to an integer
    const float k = __fadd_rn(__fadd_rn(__fadd_rn(r, -1.3e-4f), kRound), -kRound);
    const float edge = k + 0.5f;
    return y >= edge * edge ? k + 1.0f : k;
}
// the low byte of an integer held as a float in [-128, 255]
__device__ __forceinline__ uint32_t byte_of(float k) { return __float_as_uint(__fadd_rn(k, 12582912.0f)); }
__device__ __forceinline__ uint32_t pack4(const float* k)
{
    const uint32_t lo = __byte_perm(byte_of(k[0]), byte_of(k[1]), 0x0040), hi = __byte_perm(byte_of(k[2]), byte_of(k[3]), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
}
// byte e of a word as a float: the byte becomes the last one of 2^23's mantissa
__device__ __forceinline__ float ubyte(uint32_t w, int e)
{
    return __fadd_rn(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540 | e)), -8388608.0f);
}
__device__ __forceinline__ float sbyte(uint32_t w, int e) // of w ^ 0x80808080
{
    return __fadd_rn(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540 | e)), -8388736.0f);
}
__device__ __forceinline__ float moment_m(float k, float scale) { return (k * fabsf(k)) * scale; }
__device__ __forceinline__ float root_v(float k, float scale) { return (k * k) * scale; }

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
};

// One element: m, v and x in, new ones out; returns sqrt(v).
__device__ __forceinline__ float adamw_element(const StepScalars& sc, const Factors& f, float g, float& x, float& m, float& v)
{
    g *= f.c;
    m = m * sc.beta1 + g * sc.omb1;
    v = v * sc.beta2 + (g * sc.omb2) * g;
    const float r = __fsqrt_rn(v);
    const float den = r * f.rsqrt_bc2 + sc.eps;
    x = x - (__fdiv_rn(m, den) * f.step_size + x * f.decay);
    return r;
}

struct State {
    void *m, *v;
    float *m_scale, *v_scale;
};

// A whole block of an aligned tensor: a lane owns 8 consecutive elements, moved in 128-bit accesses.
template <int BITS>
__device__ __forceinline__ void step_block(const Tensor& t, const State& st, const StepScalars& sc, const Factors& f, int64_t base)
{
    const int lane = threadIdx.x & 31;
    const int64_t i = base + lane * 8, s = t.state + i, sb = (t.state + base) / kBlock;
    const Raw8 rg = load8(t.g, i, t.g_dtype), rx = load8(t.x, i, t.x_dtype);
    float g[8], x[8], m[8], v[8];
    if constexpr (BITS == 32) {
        const Raw8 rm = load8(st.m, s, CHOCO_F32), rv = load8(st.v, s, CHOCO_F32);
        unpack8(rm, CHOCO_F32, m);
        unpack8(rv, CHOCO_F32, v);
    } else {
        const uint2 km = *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(st.m) + s);
        const uint2 kv = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(st.v) + s);
        const float sm = st.m_scale[sb], sv = st.v_scale[sb];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = moment_m(sbyte((e < 4 ? km.x : km.y) ^ 0x80808080u, e & 3), sm);
            const float r = root_v(ubyte(e < 4 ? kv.x : kv.y, e & 3), sv);
            v[e] = r * r;
        }
    }
    unpack8(rg, t.g_dtype, g);
    unpack8(rx, t.x_dtype, x);
    float amax = 0.f, rmax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float r = adamw_element(sc, f, g[e], x[e], m[e], v[e]);
        if constexpr (BITS == 8) {
            v[e] = r;
            amax = fmaxf(amax, fabsf(m[e]));
            rmax = fmaxf(rmax, r);
        }
    }
    store8(t.x, i, t.x_dtype, x);
    if (t.copy) store8(t.copy, i, t.copy_dtype, x);
    if constexpr (BITS == 32) {
        store8(st.m, s, CHOCO_F32, m);
        store8(st.v, s, CHOCO_F32, v);
    } else {
        amax = fmaxf(warp_max(amax), kTiny);
        rmax = fmaxf(warp_max(rmax), kTiny);
        const float im = __fdiv_rn(kLevelsM, amax), iv = __fdiv_rn(kLevelsV, rmax);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = copysignf(nearest_root(fabsf(m[e]) * im), m[e]);
            const float k = nearest_root(v[e] * iv);
            v[e] = v[e] > 0.f ? fmaxf(k, 1.0f) : k;
        }
        *reinterpret_cast<uint2*>(static_cast<int8_t*>(st.m) + s) = make_uint2(pack4(m), pack4(m + 4));
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(st.v) + s) = make_uint2(pack4(v), pack4(v + 4));
        if (lane == 0) {
            st.m_scale[sb] = amax * (1.0f / kLevelsM);
            st.v_scale[sb] = rmax * (1.0f / kLevelsV);
        }
    }
}

// Any block: a lane owns every 32nd element, so that single elements still make whole lines; the
// last block of a tensor and tensors that do not start on 16 bytes.
template <int BITS>
__device__ __forceinline__ void step_block_any(const Tensor& t, const State& st, const StepScalars& sc, const Factors& f, int64_t base,
                                               int count)
{
    const int lane = threadIdx.x & 31;
    const int64_t s0 = t.state + base, sb = s0 / kBlock;
    float g[8], x[8], m[8], v[8];
    float sm = 0.f, sv = 0.f;
    if (BITS == 8) { sm = st.m_scale[sb]; sv = st.v_scale[sb]; }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = j * 32 + lane;
        g[j] = x[j] = m[j] = v[j] = 0.f;
        if (e >= count) continue;
        g[j] = load_as_float(t.g, base + e, t.g_dtype);
        x[j] = load_as_float(t.x, base + e, t.x_dtype);
        if constexpr (BITS == 32) {
            m[j] = static_cast<const float*>(st.m)[s0 + e];
            v[j] = static_cast<const float*>(st.v)[s0 + e];
        } else {
            m[j] = (float)static_cast<const int8_t*>(st.m)[s0 + e];
            v[j] = (float)static_cast<const uint8_t*>(st.v)[s0 + e];
        }
    }
    float amax = 0.f, rmax = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = j * 32 + lane;
        if (e >= count) continue;
        if constexpr (BITS == 8) {
            m[j] = moment_m(m[j], sm);
            const float r = root_v(v[j], sv);
            v[j] = r * r;
        }
        const float r = adamw_element(sc, f, g[j], x[j], m[j], v[j]);
        store_from_float(t.x, base + e, t.x_dtype, x[j]);
        if (t.copy) store_from_float(t.copy, base + e, t.copy_dtype, x[j]);
        if constexpr (BITS == 32) {
            static_cast<float*>(st.m)[s0 + e] = m[j];
            static_cast<float*>(st.v)[s0 + e] = v[j];
        } else {
            v[j] = r;
            amax = fmaxf(amax, fabsf(m[j]));
            rmax = fmaxf(rmax, r);
        }
    }
    if constexpr (BITS == 8) {
        amax = fmaxf(warp_max(amax), kTiny);
        rmax = fmaxf(warp_max(rmax), kTiny);
        const float im = __fdiv_rn(kLevelsM, amax), iv = __fdiv_rn(kLevelsV, rmax);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = j * 32 + lane;
            if (e >= count) continue;
            const float km = copysignf(nearest_root(fabsf(m[j]) * im), m[j]);
            float kv = nearest_root(v[j] * iv);
            if (v[j] > 0.f) kv = fmaxf(kv, 1.0f);
            static_cast<uint8_t*>(st.m)[s0 + e] = (uint8_t)byte_of(km);
            static_cast<uint8_t*>(st.v)[s0 + e] = (uint8_t)byte_of(kv);
        }
        if (lane == 0) {
            st.m_scale[sb] = amax * (1.0f / kLevelsM);
            st.v_scale[sb] = rmax * (1.0f / kLevelsV);
        }
    }
}

// One block of threads per chunk, one warp per block of elements.  The chunks are taken from the
// last one: choco_adamw_grad_norm has read the gradients from the first one on, and what it read
// last is what the L2 cache still holds.
template <int BITS>
__global__ void __launch_bounds__(kStepThreads)
step_kernel(const Tensor* __restrict__ tensors, const Chunk* __restrict__ chunks, const float* __restrict__ factor,
            int64_t* __restrict__ skipped, State st, StepScalars sc)
{
    wait_for_previous_kernel();
    allow_next_kernel();
    const Chunk ch = chunks[gridDim.x - 1 - blockIdx.x];
    const Tensor t = tensors[ch.tensor];
    Factors f;
    f.c = 1.0f;
    if (factor) {
        f.c = factor[t.group];
        if (!isfinite(f.c)) { // overflowed gradients: the group sits this step out
            if (ch.first && threadIdx.x == 0) skipped[t.group] += 1;
            return;
        }
    }
    const int64_t base = ch.begin + (int64_t)(threadIdx.x >> 5) * kBlock;
    if (base >= t.numel) return;
    f.step_size = sc.step_size;
    f.rsqrt_bc2 = sc.rsqrt_bc2;
    const int64_t sk = skipped[t.group];
    if (sk != 0) { // this group has taken fewer steps than the others
        const int64_t n = sc.t - sk;
        f.step_size = (float)(sc.lrd / (1.0 - pow_int(sc.beta1d, n)));
        f.rsqrt_bc2 = (float)(1.0 / sqrt(1.0 - pow_int(sc.beta2d, n)));
    }
    f.step_size *= t.lr_scale;
    f.decay = t.weight_decay * (sc.lr * t.lr_scale);
    if (t.aligned && base + kBlock <= t.numel) step_block<BITS>(t, st, sc, f, base);
    else step_block_any<BITS>(t, st, sc, f, base, (int)min((int64_t)kBlock, t.numel - base));
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
            m[e] = moment_m(sbyte((e < 4 ? km.x : km.y) ^ 0x80808080u, e & 3), sm);
            const float r = root_v(ubyte(e < 4 ? kv.x : kv.y, e & 3), sv);
            v[e] = r * r;
        }
    }
    if (m_out) store8(m_out, i, dtype, m);
    if (v_out) store8(v_out, i, dtype, v);
}

// Sum of squares of one unit (a run of one tensor's gradient), in float64: squares of float32
// values neither overflow nor vanish there.
__global__ void __launch_bounds__(kNormThreads) norm_partial_kernel(const Tensor* __restrict__ tensors,
                                                                    const Chunk* __restrict__ units, int64_t unit_elems,
                                                                    double* __restrict__ partial)
{
    __shared__ double red[kNormThreads / 32];
    wait_for_previous_kernel();
    allow_next_kernel();
    const Chunk u = units[blockIdx.x];
    const Tensor t = tensors[u.tensor];
    const int64_t end = min(u.begin + unit_elems, t.numel);
    double acc = 0.0;
    int64_t done = u.begin;
    if (t.aligned) {
        constexpr int kAhead = 4;           // vectors of a thread in flight
        constexpr int kSpanElems = kNormThreads * 8;
        for (; done + kAhead * kSpanElems <= end; done += kAhead * kSpanElems) {
            Raw8 r[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) r[k] = load8(t.g, done + k * kSpanElems + threadIdx.x * 8, t.g_dtype);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                float g[8];
                unpack8(r[k], t.g_dtype, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc = __fma_rn((double)g[e], (double)g[e], acc);
            }
        }
    }
    for (int64_t e = done + threadIdx.x; e < end; e += kNormThreads) {
        const double g = (double)load_as_float(t.g, e, t.g_dtype);
        acc = __fma_rn(g, g, acc);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormThreads / 32; ++w) acc += red[w];
        partial[blockIdx.x] = acc;
    }
}

// One block per group: the units of a group are contiguous.
__global__ void __launch_bounds__(kNormThreads) norm_finish_kernel(const double* __restrict__ partial,
                                                                   const int64_t* __restrict__ unit_begin, float max_norm,
                                                                   float unscale, float* norm, float* factor)
{
    __shared__ double red[kNormThreads / 32];
    wait_for_previous_kernel();
    allow_next_kernel();
    double acc = 0.0;
    for (int64_t u = unit_begin[blockIdx.x] + threadIdx.x; u < unit_begin[blockIdx.x + 1]; u += kNormThreads) acc += partial[u];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormThreads / 32; ++w) acc += red[w];
        const double nrm = (double)unscale * sqrt(acc);
        norm[blockIdx.x] = (float)nrm;
        double f = (double)unscale;
        if (max_norm > 0.f) {
            const double clip = (double)max_norm / (nrm + kNormEps);
            f *= clip < 1.0 ? clip : 1.0;
        }
        factor[blockIdx.x] = isfinite(nrm) ? (float)f : __int_as_float(0x7fc00000);
    }
}

} // namespace

struct choco_adamw {
    choco_adamw_params params;
    int device;
    bool norm_only;                // no parameters: the list serves choco_adamw_grad_norm alone
    std::vector<Tensor> tensors;   // as on the device
    std::vector<int64_t> offsets;
    int64_t elements;              // of m and v
    int64_t nchunks, nunits, unit_elems;
    int64_t t;                     // step calls so far; a group has taken t - skipped[group] steps
    Tensor* d_tensors;
    Chunk* d_chunks;
    Chunk* d_units;
    int64_t* d_unit_begin;         // [groups + 1]
    int64_t* d_skipped;            // [groups]
    double* d_partial;             // [nunits]
};

namespace {

bool on_device(const choco_adamw* o)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == o->device;
}

template <typename T>
bool upload(T** out, const T* src, size_t count)
{
    *out = nullptr;
    const size_t bytes = sizeof(T) * (count ? count : 1);
    if (cudaMalloc((void**)out, bytes) != cudaSuccess) { *out = nullptr; return false; }
    if (!src) return cudaMemset(*out, 0, bytes) == cudaSuccess;
    return count == 0 || cudaMemcpy(*out, src, sizeof(T) * count, cudaMemcpyHostToDevice) == cudaSuccess;
}

int status_of(cudaError_t e)
{
    if (e == cudaSuccess) return CHOCO_OK;
    cudaGetLastError();
    return CHOCO_ERR_CUDA;
}

void free_all(choco_adamw* o)
{
    cudaFree(o->d_tensors);
    cudaFree(o->d_chunks);
    cudaFree(o->d_units);
    cudaFree(o->d_unit_begin);
    cudaFree(o->d_skipped);
    cudaFree(o->d_partial);
    delete o;
}

bool all_aligned(const Tensor& t) { return aligned_to(t.x, 16) && aligned_to(t.g, 16) && aligned_to(t.copy, 16); }

// Fills the host tables of `o`.  Throws std::bad_alloc.
int plan(choco_adamw* o, int32_t n, const choco_adamw_tensor* ts, std::vector<Chunk>& chunks, std::vector<Chunk>& units,
         std::vector<int64_t>& unit_begin)
{
    const int32_t groups = o->params.groups;
    std::vector<std::vector<int32_t>> members(groups);
    int64_t at = 0, total = 0;
    o->norm_only = false;
    for (int32_t i = 0; i < n; ++i) {
        const choco_adamw_tensor& t = ts[i];
        if (t.numel < 0 || t.numel > (int64_t)1 << 38 || t.group < 0 || t.group >= groups) return CHOCO_ERR_INVALID_ARG;
        if (!dtype_ok(t.x_dtype) || !dtype_ok(t.g_dtype) || !dtype_ok(t.copy_dtype)) return CHOCO_ERR_INVALID_ARG;
        if (!(t.weight_decay >= 0.0) || !(t.lr_scale >= 0.0) || !std::isfinite(t.weight_decay) || !std::isfinite(t.lr_scale))
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
    o->unit_elems = 16384;
    for (int32_t k = 0; k < groups; ++k) {
        unit_begin.push_back((int64_t)units.size());
        bool first = true;
        for (int32_t i : members[k]) {
            const int64_t len = o->tensors[i].numel;
            for (int64_t b = 0; b < len; b += kChunkElems) { chunks.push_back({i, first ? 1 : 0, b}); first = false; }
            for (int64_t b = 0; b < len; b += o->unit_elems) units.push_back({i, 0, b});
        }
    }
    unit_begin.push_back((int64_t)units.size());
    o->nchunks = (int64_t)chunks.size();
    o->nunits = (int64_t)units.size();
    if (o->nchunks > 0x7fffffff) return CHOCO_ERR_TOO_LARGE;
    return CHOCO_OK;
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
    choco_adamw* o = new (std::nothrow) choco_adamw();
    if (!o) return CHOCO_ERR_ALLOC;
    o->params = *p;
    int rc = CHOCO_OK;
    try {
        std::vector<Chunk> chunks, units;
        std::vector<int64_t> unit_begin;
        rc = plan(o, n_tensors, tensors, chunks, units, unit_begin);
        if (rc == CHOCO_OK && cudaGetDevice(&o->device) != cudaSuccess) rc = CHOCO_ERR_CUDA;
        if (rc == CHOCO_OK &&
            !(upload(&o->d_tensors, o->tensors.data(), o->tensors.size()) && upload(&o->d_chunks, chunks.data(), chunks.size()) &&
              upload(&o->d_units, units.data(), units.size()) && upload(&o->d_unit_begin, unit_begin.data(), unit_begin.size()) &&
              upload(&o->d_skipped, (const int64_t*)nullptr, (size_t)p->groups) &&
              upload(&o->d_partial, (const double*)nullptr, units.size())))
            rc = CHOCO_ERR_ALLOC;
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
    }
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaStreamSynchronize(st) != cudaSuccess) return CHOCO_ERR_CUDA;
    for (size_t i = 0; i < opt->tensors.size(); ++i) {
        opt->tensors[i].g = g[i];
        opt->tensors[i].aligned = all_aligned(opt->tensors[i]);
    }
    if (cudaMemcpyAsync(opt->d_tensors, opt->tensors.data(), sizeof(Tensor) * opt->tensors.size(), cudaMemcpyHostToDevice, st) !=
            cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess)
        return CHOCO_ERR_CUDA;
    return CHOCO_OK;
}

int choco_adamw_grad_norm(choco_adamw* opt, float max_norm, float unscale, float* norm, float* factor, void* stream)
{
    if (!opt || !norm || !factor || !(max_norm >= 0.f) || !std::isfinite(max_norm) || !(unscale > 0.f) ||
        !std::isfinite(unscale) || !on_device(opt))
        return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(norm, 4) || !aligned_to(factor, 4)) return CHOCO_ERR_MISALIGNED;
    cudaStream_t st = (cudaStream_t)stream;
    const dim3 threads(kNormThreads);
    cudaError_t err = cudaSuccess;
    if (opt->nunits > 0)
        err = launch_overlapped(norm_partial_kernel, dim3((unsigned)opt->nunits), threads, 0, st, HotRange{}, opt->d_tensors, opt->d_units,
                                opt->unit_elems, opt->d_partial);
    if (err == cudaSuccess)
        err = launch_overlapped(norm_finish_kernel, dim3((unsigned)opt->params.groups), threads, 0, st, HotRange{}, opt->d_partial,
                                opt->d_unit_begin, max_norm, unscale, norm, factor);
    return status_of(err);
}

int choco_adamw_step(choco_adamw* opt, void* m, void* v, float* m_scale, float* v_scale, double lr, const float* factor,
                     void* stream)
{
    if (!opt || opt->norm_only || !(lr >= 0.0) || !std::isfinite(lr) || !on_device(opt)) return CHOCO_ERR_INVALID_ARG;
    const bool eight = opt->params.state_bits == 8;
    if (opt->elements > 0 && (!m || !v || (eight && (!m_scale || !v_scale)))) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(m, 16) || !aligned_to(v, 16) || !aligned_to(m_scale, 4) || !aligned_to(v_scale, 4) || !aligned_to(factor, 4))
        return CHOCO_ERR_MISALIGNED;
    const choco_adamw_params& p = opt->params;
    StepScalars sc;
    sc.t = opt->t + 1;
    sc.beta1 = (float)p.beta1; sc.beta2 = (float)p.beta2;
    sc.omb1 = (float)(1.0 - p.beta1); sc.omb2 = (float)(1.0 - p.beta2);
    sc.eps = (float)p.eps;
    sc.lr = (float)lr;
    sc.beta1d = p.beta1; sc.beta2d = p.beta2; sc.lrd = lr;
    sc.step_size = (float)(lr / (1.0 - pow_int(p.beta1, sc.t)));
    sc.rsqrt_bc2 = (float)(1.0 / std::sqrt(1.0 - pow_int(p.beta2, sc.t)));
    cudaStream_t st = (cudaStream_t)stream;
    if (opt->nchunks > 0) {
        const State state = {m, v, m_scale, v_scale};
        const int rc = status_of(launch_overlapped(eight ? step_kernel<8> : step_kernel<32>, dim3((unsigned)opt->nchunks),
                                                   dim3(kStepThreads), 0, st, HotRange{}, opt->d_tensors, opt->d_chunks, factor,
                                                   opt->d_skipped, state, sc));
        if (rc != CHOCO_OK) return rc;
    }
    opt->t += 1;
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
    if (cudaMemcpyAsync(steps, opt->d_skipped, bytes, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
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
        std::vector<int64_t> skipped(opt->params.groups);
        for (int32_t k = 0; k < opt->params.groups; ++k) skipped[k] = most - steps[k];
        if (cudaMemcpyAsync(opt->d_skipped, skipped.data(), sizeof(int64_t) * skipped.size(), cudaMemcpyHostToDevice, st) !=
                cudaSuccess ||
            cudaStreamSynchronize(st) != cudaSuccess)
            return CHOCO_ERR_CUDA;
    } catch (const std::exception&) {
        return CHOCO_ERR_ALLOC;
    }
    opt->t = most;
    return CHOCO_OK;
}

} // extern "C"
