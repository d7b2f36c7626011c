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
    int8_t x_dtype, g_dtype, copy_dtype, pad;
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

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, m));
    return v;
}

// The nearest k to sqrt(y): the code is the number of edges (j - 1/2)^2, j = 1 .., that y reaches
// (the edges are exact in float32).  The square root is only a first guess.
__device__ __forceinline__ int nearest_root(float y, int levels)
{
    int k = (int)__fsqrt_rn(y);
    k = min(k, levels);
    const float up = (float)k + 0.5f;
    if (k < levels && y >= up * up) k += 1;
    const float dn = (float)k - 0.5f;
    if (k > 0 && y < dn * dn) k -= 1;
    return k;
}

template <int BITS>
__global__ void __launch_bounds__(kStepThreads)
step_kernel(const Tensor* __restrict__ tensors, const Chunk* __restrict__ chunks, const float* __restrict__ factor,
            int64_t* __restrict__ skipped, void* m_arr, void* v_arr, float* m_scale, float* v_scale, StepScalars sc)
{
    const Chunk ch = chunks[blockIdx.x];
    const Tensor t = tensors[ch.tensor];
    const int lane = threadIdx.x & 31;
    float c = 1.0f;
    if (factor) {
        c = factor[t.group];
        if (!isfinite(c)) { // overflowed gradients: the group sits this step out
            if (ch.first && threadIdx.x == 0) skipped[t.group] += 1;
            return;
        }
    }
    const int64_t base = ch.begin + (int64_t)(threadIdx.x >> 5) * kBlock;
    if (base >= t.numel) return;
    const int count = (int)min((int64_t)kBlock, t.numel - base);
    float step_size = sc.step_size, rs = sc.rsqrt_bc2;
    const int64_t sk = skipped[t.group];
    if (sk != 0) { // this group has taken fewer steps than the others
        const int64_t n = sc.t - sk;
        step_size = (float)(sc.lrd / (1.0 - pow_int(sc.beta1d, n)));
        rs = (float)(1.0 / sqrt(1.0 - pow_int(sc.beta2d, n)));
    }
    step_size *= t.lr_scale;
    const float lrwd = t.weight_decay * (sc.lr * t.lr_scale);
    const int64_t s0 = t.state + base;
    const int64_t sb = s0 / kBlock;

    float m[8], v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = j * 32 + lane;
        m[j] = 0.f;
        v[j] = 0.f;
        if (e >= count) continue;
        if (BITS == 32) {
            m[j] = static_cast<const float*>(m_arr)[s0 + e];
            v[j] = static_cast<const float*>(v_arr)[s0 + e];
        } else {
            const float km = (float)static_cast<const int8_t*>(m_arr)[s0 + e];
            const float kv = (float)static_cast<const uint8_t*>(v_arr)[s0 + e];
            m[j] = (km * fabsf(km)) * m_scale[sb];
            const float r = (kv * kv) * v_scale[sb];
            v[j] = r * r;
        }
    }
    float amax = 0.f, rmax = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = j * 32 + lane;
        if (e >= count) continue;
        const float g = load_as_float(t.g, base + e, t.g_dtype) * c;
        const float x = load_as_float(t.x, base + e, t.x_dtype);
        m[j] = m[j] * sc.beta1 + g * sc.omb1;
        v[j] = v[j] * sc.beta2 + (g * sc.omb2) * g;
        const float r = __fsqrt_rn(v[j]);
        const float den = r * rs + sc.eps;
        const float nx = x - (__fdiv_rn(m[j], den) * step_size + x * lrwd);
        store_from_float(t.x, base + e, t.x_dtype, nx);
        if (t.copy) store_from_float(t.copy, base + e, t.copy_dtype, nx);
        if (BITS == 32) {
            static_cast<float*>(m_arr)[s0 + e] = m[j];
            static_cast<float*>(v_arr)[s0 + e] = v[j];
        } else {
            v[j] = r;
            amax = fmaxf(amax, fabsf(m[j]));
            rmax = fmaxf(rmax, r);
        }
    }
    if (BITS == 8) {
        amax = fmaxf(warp_max(amax), kTiny);
        rmax = fmaxf(warp_max(rmax), kTiny);
        const float im = __fdiv_rn(kLevelsM, amax), iv = __fdiv_rn(kLevelsV, rmax);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = j * 32 + lane;
            if (e >= count) continue;
            const int km = nearest_root(fabsf(m[j]) * im, 127);
            int kv = nearest_root(v[j] * iv, 255);
            if (kv == 0 && v[j] > 0.f) kv = 1;
            static_cast<int8_t*>(m_arr)[s0 + e] = (int8_t)(m[j] < 0.f ? -km : km);
            static_cast<uint8_t*>(v_arr)[s0 + e] = (uint8_t)kv;
        }
        if (lane == 0) {
            m_scale[sb] = amax * (1.0f / kLevelsM);
            v_scale[sb] = rmax * (1.0f / kLevelsV);
        }
    }
}

__global__ void __launch_bounds__(256) read_state_kernel(const void* m, const void* v, const float* m_scale,
                                                         const float* v_scale, void* m_out, void* v_out, int32_t dtype,
                                                         int32_t bits, int64_t elements)
{
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= elements) return;
    if (m_out) {
        float a;
        if (bits == 32) {
            a = static_cast<const float*>(m)[e];
        } else {
            const float k = (float)static_cast<const int8_t*>(m)[e];
            a = (k * fabsf(k)) * m_scale[e / kBlock];
        }
        store_from_float(m_out, e, dtype, a);
    }
    if (v_out) {
        float a;
        if (bits == 32) {
            a = static_cast<const float*>(v)[e];
        } else {
            const float k = (float)static_cast<const uint8_t*>(v)[e];
            const float r = (k * k) * v_scale[e / kBlock];
            a = r * r;
        }
        store_from_float(v_out, e, dtype, a);
    }
}

// Sum of squares of one unit (a run of one tensor's gradient), in float64: squares of float32
// values neither overflow nor vanish there.
__global__ void __launch_bounds__(kNormThreads) norm_partial_kernel(const Tensor* __restrict__ tensors,
                                                                    const Chunk* __restrict__ units, int64_t unit_elems,
                                                                    double* __restrict__ partial)
{
    __shared__ double red[kNormThreads];
    const Chunk u = units[blockIdx.x];
    const Tensor t = tensors[u.tensor];
    const int64_t end = min(u.begin + unit_elems, t.numel);
    double acc = 0.0;
    for (int64_t e = u.begin + threadIdx.x; e < end; e += kNormThreads) {
        const double g = (double)load_as_float(t.g, e, t.g_dtype);
        acc = __fma_rn(g, g, acc);
    }
    red[threadIdx.x] = acc;
    __syncthreads();
    for (int o = kNormThreads / 2; o > 0; o >>= 1) {
        if (threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) partial[blockIdx.x] = red[0];
}

// One block per group: the units of a group are contiguous.
__global__ void __launch_bounds__(kNormThreads) norm_finish_kernel(const double* __restrict__ partial,
                                                                   const int64_t* __restrict__ unit_begin, float max_norm,
                                                                   float unscale, float* norm, float* factor)
{
    __shared__ double red[kNormThreads];
    double acc = 0.0;
    for (int64_t u = unit_begin[blockIdx.x] + threadIdx.x; u < unit_begin[blockIdx.x + 1]; u += kNormThreads) acc += partial[u];
    red[threadIdx.x] = acc;
    __syncthreads();
    for (int o = kNormThreads / 2; o > 0; o >>= 1) {
        if (threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const double nrm = (double)unscale * sqrt(red[0]);
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

int status_of_launch() { return cudaGetLastError() == cudaSuccess ? CHOCO_OK : CHOCO_ERR_CUDA; }

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
    for (size_t i = 0; i < opt->tensors.size(); ++i) opt->tensors[i].g = g[i];
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
    if (opt->nunits > 0)
        norm_partial_kernel<<<(unsigned)opt->nunits, kNormThreads, 0, st>>>(opt->d_tensors, opt->d_units, opt->unit_elems,
                                                                            opt->d_partial);
    norm_finish_kernel<<<(unsigned)opt->params.groups, kNormThreads, 0, st>>>(opt->d_partial, opt->d_unit_begin, max_norm,
                                                                             unscale, norm, factor);
    return status_of_launch();
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
        if (eight)
            step_kernel<8><<<(unsigned)opt->nchunks, kStepThreads, 0, st>>>(opt->d_tensors, opt->d_chunks, factor, opt->d_skipped, m,
                                                                            v, m_scale, v_scale, sc);
        else
            step_kernel<32><<<(unsigned)opt->nchunks, kStepThreads, 0, st>>>(opt->d_tensors, opt->d_chunks, factor, opt->d_skipped,
                                                                             m, v, m_scale, v_scale, sc);
        const int rc = status_of_launch();
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
    read_state_kernel<<<(unsigned)((opt->elements + 255) / 256), 256, 0, (cudaStream_t)stream>>>(
        m, v, m_scale, v_scale, m_out, v_out, out_dtype, opt->params.state_bits, opt->elements);
    return status_of_launch();
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
