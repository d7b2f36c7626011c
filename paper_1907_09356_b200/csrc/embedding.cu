// Token lookup and its gradient for the tables of all workers (choco_embedding_* in choco.h).
//
// The gradient sorts every worker's tokens with their positions (a stable radix sort), so that the
// rows of dout that belong to one row of the table follow one another in order of position, and
// adds them up in float32: no atomics on values, so the result does not depend on scheduling.
#include <cmath>
#include <new>

#include "common.cuh"
#include "dtypes.cuh"

using namespace choco;

namespace {

constexpr int kEmbThreads = 256;
constexpr int kDigitBits = 8;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortTile = 2048;             // keys a block of the sort takes
constexpr int kSortRounds = kSortTile / kEmbThreads;

struct EmbShape {
    int64_t vocab, dim, table_row, table_ld, padding;
    float scale;
    int32_t n;
    int64_t count;       // tokens per worker
};

// The token at a position, or -1 for one outside the vocabulary.
__device__ __forceinline__ int64_t token_at(const void* tokens, int32_t bits, int64_t at, int64_t vocab)
{
    const int64_t t = bits == 64 ? static_cast<const int64_t*>(tokens)[at] : (int64_t)static_cast<const int32_t*>(tokens)[at];
    return t >= 0 && t < vocab ? t : -1;
}

// One warp per row.
template <typename TT, typename TO>
__global__ void __launch_bounds__(kEmbThreads)
lookup_kernel(EmbShape s, const TT* __restrict__ table, const void* __restrict__ tokens, int32_t index_bits, int64_t tokens_ld,
              TO* __restrict__ out, int64_t out_row, int64_t out_ld)
{
    const int64_t row = (int64_t)blockIdx.x * (kEmbThreads / 32) + (threadIdx.x >> 5);
    if (row >= (int64_t)s.n * s.count) return;
    const int64_t i = row / s.count, t = row - i * s.count;
    const int64_t tok = token_at(tokens, index_bits, i * tokens_ld + t, s.vocab);
    TO* o = out + i * out_ld + t * out_row;
    const TT* w = table + i * s.table_ld + (tok < 0 ? 0 : tok) * s.table_row;
    for (int64_t c = threadIdx.x & 31; c < s.dim; c += 32) o[c] = from_float<TO>(tok < 0 ? 0.f : to_float(w[c]) * s.scale);
}

// The sort's key of a token: tokens that get no gradient go behind all others.
__device__ __forceinline__ uint32_t sort_key(const EmbShape& s, const void* tokens, int32_t bits, int64_t at)
{
    const int64_t t = token_at(tokens, bits, at, s.vocab);
    return t < 0 || t == s.padding ? (uint32_t)s.vocab : (uint32_t)t;
}

struct SortPass {
    const void* tokens;          // first pass: the tokens themselves
    int64_t tokens_ld;
    int32_t index_bits, shift, first;
    int32_t tiles;               // per worker
    const uint32_t *key_in, *pos_in;
    uint32_t *key_out, *pos_out;
    uint32_t* hist;              // [n, kDigits, tiles]
};

__device__ __forceinline__ uint32_t pass_key(const EmbShape& s, const SortPass& p, int32_t worker, int64_t j)
{
    return p.first ? sort_key(s, p.tokens, p.index_bits, worker * p.tokens_ld + j) : p.key_in[worker * s.count + j];
}

__global__ void __launch_bounds__(kEmbThreads) sort_count_kernel(EmbShape s, SortPass p)
{
    __shared__ uint32_t h[kDigits];
    h[threadIdx.x] = 0;
    __syncthreads();
    const int32_t worker = blockIdx.y;
    for (int r = 0; r < kSortRounds; ++r) {
        const int64_t j = (int64_t)blockIdx.x * kSortTile + r * kEmbThreads + threadIdx.x;
        if (j < s.count) atomicAdd(&h[(pass_key(s, p, worker, j) >> p.shift) & (kDigits - 1)], 1u);
    }
    __syncthreads();
    p.hist[((int64_t)worker * kDigits + threadIdx.x) * p.tiles + blockIdx.x] = h[threadIdx.x];
}

// Exclusive sums of a worker's counts, digit by digit and tile by tile: where each tile's keys go.
__global__ void __launch_bounds__(1024) sort_scan_kernel(uint32_t* hist, int64_t per_worker)
{
    __shared__ uint32_t ws[32];
    __shared__ uint32_t carry;
    uint32_t* h = hist + blockIdx.x * per_worker;
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    for (int64_t b = 0; b < per_worker; b += 1024) {
        const int64_t j = b + threadIdx.x;
        const uint32_t mine = j < per_worker ? h[j] : 0u;
        uint32_t v = mine;
        const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        if (lane == 31) ws[w] = v;
        __syncthreads();
        if (w == 0) {
            uint32_t x = ws[lane];
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += u;
            }
            ws[lane] = x;
        }
        __syncthreads();
        const uint32_t before = carry + (w ? ws[w - 1] : 0u) + v - mine;
        if (j < per_worker) h[j] = before;
        __syncthreads();
        if (threadIdx.x == 0) carry += ws[31];
        __syncthreads();
    }
}

// Every warp ranks its slice of the tile in order; equal digits keep their order.
__global__ void __launch_bounds__(kEmbThreads) sort_scatter_kernel(EmbShape s, SortPass p)
{
    __shared__ uint32_t cnt[kEmbThreads / 32][kDigits];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int32_t worker = blockIdx.y;
    for (int d = lane; d < kDigits; d += 32) cnt[w][d] = 0;
    __syncwarp();
    uint32_t key[kSortRounds], pos[kSortRounds], rank[kSortRounds];
    const int64_t j0 = (int64_t)blockIdx.x * kSortTile + w * (kSortRounds * 32) + lane;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const int64_t j = j0 + r * 32;
        const bool in = j < s.count;
        const uint32_t act = __ballot_sync(0xffffffffu, in);
        if (in) {
            key[r] = pass_key(s, p, worker, j);
            pos[r] = p.first ? (uint32_t)j : p.pos_in[worker * s.count + j];
            const uint32_t d = (key[r] >> p.shift) & (kDigits - 1);
            const uint32_t same = __match_any_sync(act, d);
            const uint32_t before = cnt[w][d];
            __syncwarp(act);
            rank[r] = before + __popc(same & ((1u << lane) - 1u));
            if (lane == __ffs(same) - 1) cnt[w][d] = before + __popc(same);
            __syncwarp(act);
        }
    }
    __syncthreads();
    {
        uint32_t at = p.hist[((int64_t)worker * kDigits + threadIdx.x) * p.tiles + blockIdx.x];
        for (int k = 0; k < kEmbThreads / 32; ++k) {
            const uint32_t c = cnt[k][threadIdx.x];
            cnt[k][threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        if (j0 + r * 32 < s.count) {
            const int64_t to = worker * s.count + cnt[w][(key[r] >> p.shift) & (kDigits - 1)] + rank[r];
            p.key_out[to] = key[r];
            p.pos_out[to] = pos[r];
        }
    }
}

template <typename TG>
__global__ void __launch_bounds__(kEmbThreads) zero_rows_kernel(EmbShape s, TG* grad)
{
    TG* g = grad + blockIdx.y * s.table_ld;
    for (int64_t r = blockIdx.x; r < s.vocab; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < s.dim; c += kEmbThreads) g[r * s.table_row + c] = from_float<TG>(0.f);
}

// One warp per sorted entry; the first entry of a token adds up all of them.
template <typename TD, typename TG>
__global__ void __launch_bounds__(kEmbThreads)
sum_rows_kernel(EmbShape s, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ pos, const TD* __restrict__ dout,
                int64_t dout_row, int64_t dout_ld, TG* grad, int32_t accumulate)
{
    const int64_t e = (int64_t)blockIdx.x * (kEmbThreads / 32) + (threadIdx.x >> 5);
    if (e >= (int64_t)s.n * s.count) return;
    const int64_t i = e / s.count, end = (i + 1) * s.count;
    const uint32_t key = keys[e];
    if (key >= (uint32_t)s.vocab || (e > i * s.count && keys[e - 1] == key)) return;
    const TD* d = dout + i * dout_ld;
    TG* g = grad + i * s.table_ld + (int64_t)key * s.table_row;
    for (int64_t c = threadIdx.x & 31; c < s.dim; c += 32) {
        float acc = 0.f;
        for (int64_t k = e; k < end && keys[k] == key; ++k) acc += to_float(d[pos[k] * dout_row + c]);
        acc *= s.scale;
        if (accumulate) acc += to_float(g[c]);
        g[c] = from_float<TG>(acc);
    }
}

template <typename F>
int with_type(int32_t dtype, F f)
{
    if (dtype == CHOCO_F32) return f((float*)nullptr);
    if (dtype == CHOCO_BF16) return f((__nv_bfloat16*)nullptr);
    return f((__half*)nullptr);
}

int status_of_launch() { return cudaGetLastError() == cudaSuccess ? CHOCO_OK : CHOCO_ERR_CUDA; }

} // namespace

struct choco_embedding {
    choco_embedding_params p;
    int device;
    uint32_t* key[2];
    uint32_t* pos[2];
    uint32_t* hist;
};

namespace {

bool on_device(const choco_embedding* e)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == e->device;
}

void free_all(choco_embedding* e)
{
    for (int k = 0; k < 2; ++k) { cudaFree(e->key[k]); cudaFree(e->pos[k]); }
    cudaFree(e->hist);
    delete e;
}

EmbShape shape_of(const choco_embedding* e, int64_t count)
{
    const choco_embedding_params& p = e->p;
    return {p.vocab, p.dim, p.table_row, p.table_ld, p.padding, p.scale, p.n, count};
}

int check_tokens(const choco_embedding* e, const void* tokens, int32_t bits, int64_t count, int64_t ld)
{
    if (!on_device(e) || (bits != 32 && bits != 64) || count < 0 || (e->p.n > 1 && ld < count)) return CHOCO_ERR_INVALID_ARG;
    if (count > 0 && !tokens) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(tokens, bits / 8)) return CHOCO_ERR_MISALIGNED;
    if (count >= ((int64_t)1 << 31) || count * e->p.n >= ((int64_t)1 << 31)) return CHOCO_ERR_TOO_LARGE;
    return CHOCO_OK;
}

} // namespace

extern "C" {

int choco_embedding_init(choco_embedding** out, const choco_embedding_params* p)
{
    if (!out) return CHOCO_ERR_INVALID_ARG;
    *out = nullptr;
    if (!p || p->n < 1 || p->vocab < 1 || p->dim < 1 || p->max_tokens < 0 || !std::isfinite(p->scale)) return CHOCO_ERR_INVALID_ARG;
    if (p->n > 65535 || p->vocab > 0x7ffffffe || p->dim > ((int64_t)1 << 24)) return CHOCO_ERR_TOO_LARGE;
    if (p->max_tokens >= ((int64_t)1 << 31) || p->max_tokens * p->n >= ((int64_t)1 << 31)) return CHOCO_ERR_TOO_LARGE;
    choco_embedding_params q = *p;
    if (q.table_row == 0) q.table_row = q.dim;
    if (q.table_row < q.dim || q.table_row > ((int64_t)1 << 31)) return CHOCO_ERR_INVALID_ARG;
    if (q.table_ld == 0) q.table_ld = q.vocab * q.table_row;
    if (q.n > 1 && q.table_ld < (q.vocab - 1) * q.table_row + q.dim) return CHOCO_ERR_INVALID_ARG;
    choco_embedding* e = new (std::nothrow) choco_embedding();
    if (!e) return CHOCO_ERR_ALLOC;
    e->p = q;
    cudaError_t err = cudaGetDevice(&e->device);
    const size_t total = (size_t)q.n * (size_t)q.max_tokens;
    if (total > 0) {
        const size_t tiles = (size_t)((q.max_tokens + kSortTile - 1) / kSortTile);
        for (int k = 0; k < 2 && err == cudaSuccess; ++k) {
            err = cudaMalloc((void**)&e->key[k], total * 4);
            if (err == cudaSuccess) err = cudaMalloc((void**)&e->pos[k], total * 4);
        }
        if (err == cudaSuccess) err = cudaMalloc((void**)&e->hist, (size_t)q.n * kDigits * tiles * 4);
    }
    if (err != cudaSuccess) {
        cudaGetLastError();
        free_all(e);
        return err == cudaErrorMemoryAllocation ? CHOCO_ERR_ALLOC : CHOCO_ERR_CUDA;
    }
    *out = e;
    return CHOCO_OK;
}

int choco_embedding_destroy(choco_embedding* emb)
{
    if (!emb) return CHOCO_ERR_INVALID_ARG;
    free_all(emb);
    return CHOCO_OK;
}

int choco_embedding_forward(choco_embedding* emb, const void* table, int32_t table_dtype, const void* tokens, int32_t index_bits,
                            int64_t count, int64_t tokens_ld, void* out, int32_t out_dtype, int64_t out_row, int64_t out_ld,
                            void* stream)
{
    if (!emb || !table || !dtype_ok(table_dtype) || !dtype_ok(out_dtype)) return CHOCO_ERR_INVALID_ARG;
    const int rc = check_tokens(emb, tokens, index_bits, count, tokens_ld);
    if (rc != CHOCO_OK) return rc;
    if (count > 0 && (!out || out_row < emb->p.dim || (emb->p.n > 1 && out_ld < 0))) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(table, dtype_size(table_dtype)) || !aligned_to(out, dtype_size(out_dtype))) return CHOCO_ERR_MISALIGNED;
    if (count == 0) return CHOCO_OK;
    const EmbShape s = shape_of(emb, count);
    const int64_t rows = count * s.n;
    cudaStream_t st = (cudaStream_t)stream;
    return with_type(table_dtype, [&](auto* tt) {
        return with_type(out_dtype, [&](auto* to) {
            using TT = std::remove_pointer_t<decltype(tt)>;
            using TO = std::remove_pointer_t<decltype(to)>;
            lookup_kernel<TT, TO><<<(unsigned)((rows + 7) / 8), kEmbThreads, 0, st>>>(
                s, static_cast<const TT*>(table), tokens, index_bits, tokens_ld, static_cast<TO*>(out), out_row, out_ld);
            return status_of_launch();
        });
    });
}

int choco_embedding_backward(choco_embedding* emb, const void* tokens, int32_t index_bits, int64_t count, int64_t tokens_ld,
                             const void* dout, int32_t dout_dtype, int64_t dout_row, int64_t dout_ld, void* grad,
                             int32_t grad_dtype, int32_t accumulate, void* stream)
{
    if (!emb || !grad || !dtype_ok(dout_dtype) || !dtype_ok(grad_dtype)) return CHOCO_ERR_INVALID_ARG;
    const int rc = check_tokens(emb, tokens, index_bits, count, tokens_ld);
    if (rc != CHOCO_OK) return rc;
    if (count > emb->p.max_tokens) return CHOCO_ERR_TOO_LARGE;
    if (count > 0 && (!dout || dout_row < emb->p.dim || (emb->p.n > 1 && dout_ld < 0))) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(grad, dtype_size(grad_dtype)) || !aligned_to(dout, dtype_size(dout_dtype))) return CHOCO_ERR_MISALIGNED;
    const EmbShape s = shape_of(emb, count);
    cudaStream_t st = (cudaStream_t)stream;
    if (!accumulate) {
        const int r = with_type(grad_dtype, [&](auto* tg) {
            using TG = std::remove_pointer_t<decltype(tg)>;
            const dim3 grid((unsigned)(s.vocab < 4096 ? s.vocab : 4096), (unsigned)s.n);
            zero_rows_kernel<TG><<<grid, kEmbThreads, 0, st>>>(s, static_cast<TG*>(grad));
            return status_of_launch();
        });
        if (r != CHOCO_OK) return r;
    }
    if (count == 0) return CHOCO_OK;
    SortPass p = {};
    p.tokens = tokens; p.tokens_ld = tokens_ld; p.index_bits = index_bits;
    p.tiles = (int32_t)((count + kSortTile - 1) / kSortTile);
    p.hist = emb->hist;
    int cur = 0;
    p.first = 1;
    for (p.shift = 0; p.shift == 0 || (s.vocab >> p.shift) != 0; p.shift += kDigitBits) {
        p.key_in = emb->key[cur]; p.pos_in = emb->pos[cur];
        p.key_out = emb->key[cur ^ 1]; p.pos_out = emb->pos[cur ^ 1];
        const dim3 grid((unsigned)p.tiles, (unsigned)s.n);
        sort_count_kernel<<<grid, kEmbThreads, 0, st>>>(s, p);
        sort_scan_kernel<<<(unsigned)s.n, 1024, 0, st>>>(p.hist, (int64_t)kDigits * p.tiles);
        sort_scatter_kernel<<<grid, kEmbThreads, 0, st>>>(s, p);
        p.first = 0;
        cur ^= 1;
    }
    const int64_t rows = count * s.n;
    return with_type(dout_dtype, [&](auto* td) {
        return with_type(grad_dtype, [&](auto* tg) {
            using TD = std::remove_pointer_t<decltype(td)>;
            using TG = std::remove_pointer_t<decltype(tg)>;
            sum_rows_kernel<TD, TG><<<(unsigned)((rows + 7) / 8), kEmbThreads, 0, st>>>(
                s, emb->key[cur], emb->pos[cur], static_cast<const TD*>(dout), dout_row, dout_ld, static_cast<TG*>(grad), accumulate);
            return status_of_launch();
        });
    });
}

} // extern "C"
