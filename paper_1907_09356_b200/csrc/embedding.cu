// Token lookup and its gradient for the tables of all workers (choco_embedding_* in choco.h).
//
// The gradient orders every worker's tokens with their positions, so that the rows of dout that
// belong to one row of the table follow one another in order of position, cuts that list into tiles
// of equal length and adds up each tile's rows in registers, in float32.  A run of one token that
// crosses tiles leaves partial sums, which a last kernel adds in tile order.  No atomics on
// values: the result depends on the tokens and the sizes alone.
#include <algorithm>
#include <cmath>
#include <new>

#include "common.cuh"
#include "dtypes.cuh"

using namespace choco;

namespace {

constexpr int kEmbThreads = 256;
constexpr int kEmbWarps = kEmbThreads / 32;
constexpr int kDigitBits = 8;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortTile = 2048;             // keys a block of the sort takes
constexpr int kSortRounds = kSortTile / kEmbThreads;
constexpr int kTileLong = 32;               // sorted entries per tile of the sums, many rows ...
constexpr int kTileShort = 8;               // ... and few: more warps, shorter chains of loads
constexpr int64_t kShortRows = 16384;
constexpr int kRankKeys = 64;               // keys a block of the rank kernel places
constexpr int64_t kRankPairs = (int64_t)1 << 27; // n count^2 up to which tokens are ordered by ranks
constexpr uint32_t kNoKey = 0xffffffffu;
constexpr int kChainOfWarp = 32;            // chains of partial sums up to this length are added by one warp

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

// ---------------------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------------------

constexpr int kLookupVecs = 4;              // vectors a lane moves: a warp serves 128 V columns of one row

template <typename TT, typename TO, int V>
__global__ void __launch_bounds__(kEmbThreads)
lookup_kernel(EmbShape s, const TT* __restrict__ table, const void* __restrict__ tokens, int32_t index_bits, int64_t tokens_ld,
              TO* __restrict__ out, int64_t out_row, int64_t out_ld, uint32_t slabs)
{
    const uint64_t item = (uint64_t)blockIdx.x * kEmbWarps + (threadIdx.x >> 5);
    const uint32_t row = (uint32_t)(item / slabs), slab = (uint32_t)(item - (uint64_t)row * slabs);
    if (row >= (uint32_t)((int64_t)s.n * s.count)) return;
    const uint32_t i = row / (uint32_t)s.count, t = row - i * (uint32_t)s.count;
    const int64_t tok = token_at(tokens, index_bits, i * tokens_ld + t, s.vocab);
    const int64_t c0 = (int64_t)slab * (32 * V * kLookupVecs) + (threadIdx.x & 31) * V;
    TO* o = out + i * out_ld + t * out_row;
    const TT* w = table + i * s.table_ld + (tok < 0 ? 0 : tok) * s.table_row;
    Raw<TT, V> raw[kLookupVecs];
#pragma unroll
    for (int k = 0; k < kLookupVecs; ++k) {
        const int64_t c = c0 + k * 32 * V;
        if (tok >= 0 && c < s.dim) load_raw(raw[k], w + c);
    }
#pragma unroll
    for (int k = 0; k < kLookupVecs; ++k) {
        const int64_t c = c0 + k * 32 * V;
        if (c >= s.dim) continue;
        float f[V];
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = tok >= 0 ? raw_get(raw[k], e) * s.scale : 0.f;
        store_vec<TO, V>(o + c, f);
    }
}

// ---------------------------------------------------------------------------------------
// order of the tokens
// ---------------------------------------------------------------------------------------

// The key of a token: tokens that get no gradient go behind all others.
__device__ __forceinline__ uint32_t sort_key(const EmbShape& s, const void* tokens, int32_t bits, int64_t at)
{
    const int64_t t = token_at(tokens, bits, at, s.vocab);
    return t < 0 || t == s.padding ? (uint32_t)s.vocab : (uint32_t)t;
}

// Which rows of the tables some token names: a bit per row, a multiple of four bytes per worker.  All
// zeros between calls: whoever zeroes a byte's rows of the gradient clears it.
struct Presence {
    uint8_t* bits;               // nullptr: not wanted (the sums are added to the gradient)
    int64_t bytes;               // per worker
};
__device__ __forceinline__ void mark_present(const Presence& p, int32_t worker, uint32_t key)
{
    uint32_t* w = reinterpret_cast<uint32_t*>(p.bits + worker * p.bytes) + (key >> 5);
    const uint32_t bit = 1u << (key & 31);
    if (!(*reinterpret_cast<volatile uint32_t*>(w) & bit)) atomicOr(w, bit);
}

// A share of the rows that no token names becomes zeros: bytes of the map [begin, end), a warp each.
struct ZeroWork {
    Presence pres;
    void* grad;
    int32_t dtype;
    int32_t wide;                // bytes a store may have: the alignment of every row
    int64_t begin, end;          // of n * pres.bytes
    int32_t blocks;              // blocks of the launch that do this, behind the others
};

__device__ __forceinline__ void zero_run(char* p, int64_t bytes, int wide, int lane)
{
    if (wide == 16) for (int64_t b = lane * 16; b < bytes; b += 512) *reinterpret_cast<uint4*>(p + b) = make_uint4(0, 0, 0, 0);
    else if (wide == 8) for (int64_t b = lane * 8; b < bytes; b += 256) *reinterpret_cast<uint2*>(p + b) = make_uint2(0, 0);
    else if (wide == 4) for (int64_t b = lane * 4; b < bytes; b += 128) *reinterpret_cast<uint32_t*>(p + b) = 0;
    else for (int64_t b = lane * 2; b < bytes; b += 64) *reinterpret_cast<unsigned short*>(p + b) = 0;
}

__device__ __forceinline__ void zero_share(const EmbShape& s, const ZeroWork& z, int32_t block)
{
    const int lane = threadIdx.x & 31;
    const int64_t size = z.dtype == CHOCO_F32 ? 4 : 2;
    const int64_t step = (int64_t)z.blocks * (blockDim.x >> 5);
    for (int64_t u = z.begin + (int64_t)block * (blockDim.x >> 5) + (threadIdx.x >> 5); u < z.end; u += step) {
        const int64_t worker = u / z.pres.bytes, r0 = (u - worker * z.pres.bytes) * 8;
        const uint32_t have = z.pres.bits[u];
        __syncwarp();
        if (have && lane == 0) z.pres.bits[u] = 0;
        if (r0 >= s.vocab) continue;
        const int rows = (int)min((int64_t)8, s.vocab - r0);
        char* p = static_cast<char*>(z.grad) + (worker * s.table_ld + r0 * s.table_row) * size;
        if (!have && s.table_row == s.dim) {
            const int64_t bytes = rows * s.dim * size;
            // eight rows start on 16 bytes if the table does, whatever their length in float32
            const int wide = ((uintptr_t)p | (uint64_t)bytes) % 16 == 0 ? 16 : z.wide;
            zero_run(p, bytes, wide, lane);
        } else {
            for (int r = 0; r < rows; ++r)
                if (!(have >> r & 1)) zero_run(p + r * s.table_row * size, s.dim * size, z.wide, lane);
        }
    }
}

// Few tokens: every key counts the keys before it in order of (token, position).  The pair is
// one 32-bit number, so that is one comparison; all SMs share the count^2 of them.
__global__ void __launch_bounds__(kEmbThreads)
rank_kernel(EmbShape s, const void* __restrict__ tokens, int64_t tokens_ld, int32_t index_bits, int32_t pos_bits, Presence pres,
            uint32_t* __restrict__ keys, uint32_t* __restrict__ pos)
{
    constexpr int kParts = kEmbThreads / kRankKeys;
    extern __shared__ uint32_t all[];       // count pairs, then a multiple of 16 filled up with the largest
    __shared__ uint32_t sums[kParts][kRankKeys];
    wait_for_previous_kernel();
    const int32_t worker = blockIdx.y;
    const int count = (int)s.count, padded = (count + 15) / 16 * 16;
    for (int j = threadIdx.x; j < padded; j += kEmbThreads)
        all[j] = j < count ? sort_key(s, tokens, index_bits, worker * tokens_ld + j) << pos_bits | (uint32_t)j : kNoKey;
    __syncthreads();
    allow_next_kernel();
    const int mine = threadIdx.x % kRankKeys, part = threadIdx.x / kRankKeys;
    const int i = blockIdx.x * kRankKeys + mine;
    const uint32_t key = i < count ? all[i] : 0u;
    const uint4* quads = reinterpret_cast<const uint4*>(all);
    const int per = padded / 4 / kParts;
    uint32_t before = 0;
#pragma unroll 4
    for (int q = part * per; q < (part + 1) * per; ++q) {
        const uint4 v = quads[q];
        before += (v.x < key) + (v.y < key) + (v.z < key) + (v.w < key);
    }
    sums[part][mine] = before;
    __syncthreads();
    if (part == 0 && i < count) {
#pragma unroll
        for (int k = 1; k < kParts; ++k) before += sums[k][mine];
        const uint32_t tok = key >> pos_bits;
        keys[worker * s.count + before] = tok;
        pos[worker * s.count + before] = key & ((1u << pos_bits) - 1u);
        if (pres.bits && tok < (uint32_t)s.vocab) mark_present(pres, worker, tok);
    }
}

// Many tokens: a stable radix sort, three launches per digit.
struct SortPass {
    const void* tokens;          // first pass: the tokens themselves
    int64_t tokens_ld;
    int32_t index_bits, shift, first;
    int32_t tiles;               // per worker
    const uint32_t *key_in, *pos_in;
    uint32_t *key_out, *pos_out;
    uint32_t* hist;              // [n, kDigits, tiles]
    uint32_t* total;             // [n, kDigits]
    Presence pres;
};

__device__ __forceinline__ uint32_t pass_key(const EmbShape& s, const SortPass& p, int32_t worker, int64_t j)
{
    return p.first ? sort_key(s, p.tokens, p.index_bits, worker * p.tokens_ld + j) : p.key_in[worker * s.count + j];
}

__global__ void __launch_bounds__(kEmbThreads) sort_count_kernel(EmbShape s, SortPass p, ZeroWork z)
{
    __shared__ uint32_t h[kDigits];
    wait_for_previous_kernel();
    allow_next_kernel();
    const int32_t blocks = p.tiles * s.n;
    if ((int32_t)blockIdx.x >= blocks) return zero_share(s, z, blockIdx.x - blocks);
    const int32_t worker = blockIdx.x / p.tiles, tile = blockIdx.x - worker * p.tiles;
    h[threadIdx.x] = 0;
    __syncthreads();
    uint32_t key[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const int64_t j = (int64_t)tile * kSortTile + r * kEmbThreads + threadIdx.x;
        key[r] = j < s.count ? pass_key(s, p, worker, j) : kNoKey;
    }
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        if (key[r] == kNoKey) continue;
        atomicAdd(&h[(key[r] >> p.shift) & (kDigits - 1)], 1u);
        if (p.first && p.pres.bits && key[r] < (uint32_t)s.vocab) mark_present(p.pres, worker, key[r]);
    }
    __syncthreads();
    p.hist[((int64_t)worker * kDigits + threadIdx.x) * p.tiles + tile] = h[threadIdx.x];
}

// One warp per digit: exclusive sums of its counts over the tiles, and their total.
__global__ void __launch_bounds__(kEmbThreads) sort_scan_kernel(EmbShape s, SortPass p, ZeroWork z)
{
    wait_for_previous_kernel();
    allow_next_kernel();
    const int32_t blocks = s.n * (kDigits / kEmbWarps);
    if ((int32_t)blockIdx.x >= blocks) return zero_share(s, z, blockIdx.x - blocks);
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kEmbWarps + (threadIdx.x >> 5);
    uint32_t* h = p.hist + row * p.tiles;
    uint32_t carry = 0;
    for (int32_t b = 0; b < p.tiles; b += 32) {
        const int32_t j = b + lane;
        const uint32_t mine = j < p.tiles ? h[j] : 0u;
        uint32_t v = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        if (j < p.tiles) h[j] = carry + v - mine;
        carry += __shfl_sync(0xffffffffu, v, 31);
    }
    if (lane == 0) p.total[row] = carry;
}

// Every warp ranks its slice of the tile in order; equal digits keep their order.
__global__ void __launch_bounds__(kEmbThreads) sort_scatter_kernel(EmbShape s, SortPass p, ZeroWork z)
{
    __shared__ uint32_t cnt[kEmbWarps][kDigits];
    __shared__ uint32_t ws[kEmbWarps];
    wait_for_previous_kernel();
    allow_next_kernel();
    const int32_t blocks = p.tiles * s.n;
    if ((int32_t)blockIdx.x >= blocks) return zero_share(s, z, blockIdx.x - blocks);
    const int32_t worker = blockIdx.x / p.tiles, tile = blockIdx.x - worker * p.tiles;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    // thread d: where digit d of this tile starts = keys with smaller digits + this digit in earlier tiles
    const uint32_t total = p.total[worker * kDigits + threadIdx.x];
    const uint32_t earlier = p.hist[((int64_t)worker * kDigits + threadIdx.x) * p.tiles + tile];
    uint32_t incl = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 31) ws[w] = incl;
    for (int d = lane; d < kDigits; d += 32) cnt[w][d] = 0;
    __syncwarp();
    uint32_t key[kSortRounds], pos[kSortRounds], rank[kSortRounds];
    const int64_t j0 = (int64_t)tile * kSortTile + w * (kSortRounds * 32) + lane;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const int64_t j = j0 + r * 32;
        key[r] = j < s.count ? pass_key(s, p, worker, j) : kNoKey;
        pos[r] = p.first ? (uint32_t)j : j < s.count ? p.pos_in[worker * s.count + j] : 0u;
    }
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const bool in = key[r] != kNoKey;
        const uint32_t d = (key[r] >> p.shift) & (kDigits - 1);
        const uint32_t same = __match_any_sync(0xffffffffu, in ? d : kNoKey);
        const uint32_t before = in ? cnt[w][d] : 0u;
        __syncwarp();
        rank[r] = before + __popc(same & ((1u << lane) - 1u));
        if (in && lane == __ffs(same) - 1) cnt[w][d] = before + __popc(same);
        __syncwarp();
    }
    __syncthreads();
    {
        uint32_t at = earlier + incl - total;
#pragma unroll
        for (int k = 0; k < kEmbWarps; ++k)
            if (k < w) at += ws[k];
#pragma unroll
        for (int k = 0; k < kEmbWarps; ++k) {
            const uint32_t c = cnt[k][threadIdx.x];
            cnt[k][threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        if (key[r] != kNoKey) {
            const int64_t to = worker * s.count + cnt[w][(key[r] >> p.shift) & (kDigits - 1)] + rank[r];
            p.key_out[to] = key[r];
            p.pos_out[to] = pos[r];
        }
    }
}

// ---------------------------------------------------------------------------------------
// sums
// ---------------------------------------------------------------------------------------

struct Sums {
    const uint32_t *keys, *pos;  // [n, count] in order
    const void* dout;
    int64_t dout_row, dout_ld;
    void* grad;
    int32_t grad_dtype, accumulate;
    float* part;                 // [n * tiles, 2, pitch]: a run that comes from the tile before; one that starts here and goes on
    int64_t pitch;
    int32_t tile;                // entries per tile
    int32_t tiles;               // per worker
    uint32_t slabs;              // groups of columns
};

// scale * acc (+ what is there) to V columns of a row of the gradient, whose type is known at run time
template <int V>
__device__ __forceinline__ void store_grad(const EmbShape& s, const Sums& a, int32_t worker, uint32_t key, int64_t c, const float* acc)
{
    const int64_t at = worker * s.table_ld + (int64_t)key * s.table_row + c;
    float f[V];
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = acc[e] * s.scale;
    auto put = [&](auto* g) {
        using TG = std::remove_pointer_t<decltype(g)>;
        if (a.accumulate) {
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] += to_float(g[at + e]);
        }
        store_vec<TG, V>(g + at, f);
    };
    if (a.grad_dtype == CHOCO_F32) put(static_cast<float*>(a.grad));
    else if (a.grad_dtype == CHOCO_BF16) put(static_cast<__nv_bfloat16*>(a.grad));
    else put(static_cast<__half*>(a.grad));
}

// One warp per tile and group of 32 V C columns; B entries' loads are in flight together.
template <typename TD, int V, int C, int B>
__global__ void __launch_bounds__(kEmbThreads) sum_tiles_kernel(EmbShape s, Sums a, ZeroWork z, uint32_t sum_blocks)
{
    wait_for_previous_kernel();
    allow_next_kernel();
    if (blockIdx.x >= sum_blocks) return zero_share(s, z, blockIdx.x - sum_blocks);
    const int lane = threadIdx.x & 31;
    const uint64_t item = (uint64_t)blockIdx.x * kEmbWarps + (threadIdx.x >> 5);
    const uint32_t gt = (uint32_t)(item / a.slabs), slab = (uint32_t)(item - (uint64_t)gt * a.slabs);
    if (gt >= (uint32_t)a.tiles * (uint32_t)s.n) return;
    const int32_t worker = gt / (uint32_t)a.tiles, tile = gt - worker * a.tiles;
    const int64_t first = (int64_t)tile * a.tile, e0 = worker * s.count + first;
    const int cnt = (int)min((int64_t)a.tile, s.count - first);
    const uint32_t key = lane < cnt ? a.keys[e0 + lane] : kNoKey;
    const uint32_t pos = lane < cnt ? a.pos[e0 + lane] : 0u;
    const uint32_t prev = tile > 0 ? a.keys[e0 - 1] : kNoKey;
    const uint32_t next = first + cnt < s.count ? a.keys[e0 + cnt] : kNoKey;
    const int live = __popc(__ballot_sync(0xffffffffu, key < (uint32_t)s.vocab));
    if (live == 0) return;
    uint32_t cur = __shfl_sync(0xffffffffu, key, 0);
    bool head = cur == prev;
    const TD* d = static_cast<const TD*>(a.dout) + worker * a.dout_ld;
    const int64_t c0 = (int64_t)slab * (32 * V * C) + lane * V;
    float acc[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[c][e] = 0.f;
    auto flush = [&](bool goes_on) {
        if (head || goes_on) {
            float* p = a.part + ((int64_t)gt * 2 + (head ? 0 : 1)) * a.pitch;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c0 + c * 32 * V < s.dim) store_vec<float, V>(p + c0 + c * 32 * V, acc[c]);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c0 + c * 32 * V < s.dim) store_grad<V>(s, a, worker, cur, c0 + c * 32 * V, acc[c]);
        }
    };
    for (int b = 0; b < live; b += B) {
        Raw<TD, V> raw[B][C];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const uint32_t p = __shfl_sync(0xffffffffu, pos, (b + j) & 31);
            if (b + j < live) {
                const TD* r = d + p * a.dout_row;
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (c0 + c * 32 * V < s.dim) load_raw(raw[j][c], r + c0 + c * 32 * V);
            }
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const uint32_t k = __shfl_sync(0xffffffffu, key, (b + j) & 31);
            if (b + j >= live) break;
            if (k != cur) {
                flush(false);
                head = false;
                cur = k;
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[c][e] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[c][e] += raw_get(raw[j][c], e);
        }
    }
    flush(live == cnt && next == cur);
}

// Runs that cross tiles: the tile in which one starts adds up the partial sums of all its tiles, in
// order.  A chain of up to kChainOfWarp tiles is one warp's work; longer ones (frequent
// tokens) are shared by the block's warps, a contiguous part each.
constexpr int kJoinCols = 128;              // columns of a warp, four per lane

__global__ void __launch_bounds__(kEmbThreads) join_kernel(EmbShape s, Sums a)
{
    __shared__ float4 sub[kEmbWarps][32];
    __shared__ uint32_t long_tile[kEmbWarps], long_len[kEmbWarps], long_key[kEmbWarps];
    wait_for_previous_kernel();
    allow_next_kernel();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const uint32_t gt = blockIdx.x * kEmbWarps + w;
    const int64_t c0 = (int64_t)blockIdx.y * kJoinCols + lane * 4;
    uint32_t key = kNoKey, len = 0;
    if (gt < (uint32_t)a.tiles * (uint32_t)s.n) {
        const int32_t worker = gt / (uint32_t)a.tiles, tile = gt - worker * a.tiles;
        const uint32_t* k = a.keys + worker * s.count;
        const int64_t first = (int64_t)tile * a.tile, after = first + a.tile;
        if (after < s.count) {
            const uint32_t last = k[after - 1], next = k[after], head = k[first], prev = tile > 0 ? k[first - 1] : kNoKey;
            if (last == next && last < (uint32_t)s.vocab && !(head == last && prev == last)) {
                key = last;
                // further tiles that begin with it
                for (uint32_t all = 0xffffffffu; all == 0xffffffffu; len += __popc(all)) {
                    const int64_t j = after + (int64_t)(len + lane) * a.tile;
                    all = __ballot_sync(0xffffffffu, j < s.count && k[j < s.count ? j : 0] == key);
                }
            }
        }
    }
    if (lane == 0) {
        long_len[w] = len > kChainOfWarp ? len : 0;
        long_tile[w] = gt;
        long_key[w] = key;
    }
    auto part_of = [&](uint32_t t, int slot) {
        return *reinterpret_cast<const float4*>(a.part + ((int64_t)t * 2 + slot) * a.pitch + c0);
    };
    auto add = [](float4& x, const float4 y) { x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w; };
    auto sum_of = [&](uint32_t t0, uint32_t from, uint32_t to, float4 sum) {  // slots 0 of tiles t0 + [from, to)
        for (uint32_t j = from; j < to; j += 8) {
            float4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = j + u < to ? part_of(t0 + j + u, 0) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int u = 0; u < 8; ++u) add(sum, v[u]);
        }
        return sum;
    };
    auto put = [&](uint32_t t, uint32_t k, const float4 sum) {
        const float f[4] = {sum.x, sum.y, sum.z, sum.w};
        const int32_t worker = t / (uint32_t)a.tiles;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c0 + e < s.dim) store_grad<1>(s, a, worker, k, c0 + e, f + e);
    };
    if (len > 0 && len <= kChainOfWarp && c0 < s.dim) put(gt, key, sum_of(gt + 1, 0, len, part_of(gt, 1)));
    __syncthreads();
    for (int q = 0; q < kEmbWarps; ++q) {
        const uint32_t n = long_len[q]; // the same for all threads
        if (n == 0) continue;
        const uint32_t t = long_tile[q], each = (n + kEmbWarps - 1) / kEmbWarps;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c0 < s.dim) sum = sum_of(t + 1, min(n, w * each), min(n, (w + 1) * each), sum);
        sub[w][lane] = sum;
        __syncthreads();
        if (w == 0 && c0 < s.dim) {
            sum = part_of(t, 1);
#pragma unroll
            for (int k = 0; k < kEmbWarps; ++k) add(sum, sub[k][lane]);
            put(t, long_key[q], sum);
        }
        __syncthreads();
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

// The largest number of elements (a power of two, at most `most`) by which every row of an array
// can be cut into aligned vectors.
int vector_of(const void* p, int32_t dtype, int64_t row, int64_t ld, int64_t dim, int n, int most)
{
    const int64_t size = dtype_size(dtype);
    int v = most;
    while (v > 1 && ((uintptr_t)p % (uintptr_t)std::min<int64_t>(v * size, 16) != 0 || row % v != 0 || (n > 1 && ld % v != 0) || dim % v != 0))
        v /= 2;
    return v;
}

} // namespace

struct choco_embedding {
    choco_embedding_params p;
    int device;
    uint32_t* key[2];
    uint32_t* pos[2];
    uint32_t* hist;
    uint32_t* total;
    uint8_t* present;
    int64_t present_bytes;       // per worker
    bool dirty;                  // a call failed half-way: the map may not be clear
    float* part;
    int64_t pitch;
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
    cudaFree(e->total);
    cudaFree(e->present);
    cudaFree(e->part);
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

int tile_of(int64_t rows) { return rows <= kShortRows ? kTileShort : kTileLong; }

// number of bits for positions, if (token, position) pairs fit 32 bits and ordering by ranks pays; else 0
int rank_bits(const EmbShape& s)
{
    int b = 1;
    while (((int64_t)1 << b) < s.count) ++b;
    if ((int64_t)s.n * s.count * s.count > kRankPairs || ((s.vocab + 1) << b) > (int64_t)1 << 32 || s.count > 8192) return 0;
    return b;
}

template <typename TD, int V, int C, int B>
cudaError_t launch_sums(const EmbShape& s, Sums a, const ZeroWork& z, cudaStream_t st)
{
    a.slabs = (uint32_t)((s.dim + 32 * V * C - 1) / (32 * V * C));
    const uint64_t warps = (uint64_t)a.slabs * a.tiles * s.n;
    const uint64_t blocks = (warps + kEmbWarps - 1) / kEmbWarps;
    if (blocks + z.blocks > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_overlapped(sum_tiles_kernel<TD, V, C, B>, dim3((unsigned)(blocks + z.blocks)), dim3(kEmbThreads), 0, st, HotRange{}, s, a,
                             z, (uint32_t)blocks);
}

template <typename TD>
cudaError_t launch_sums_for(const EmbShape& s, const Sums& a, const ZeroWork& z, int v, cudaStream_t st)
{
    // 256 columns of a row to a warp, 128 where one element at a time is all that alignment leaves;
    // narrow rows take fewer vectors per lane
    if constexpr (sizeof(TD) == 2)
        if (v == 8) return launch_sums<TD, 8, 1, 8>(s, a, z, st);
    if (v >= 4) return s.dim <= 128 ? launch_sums<TD, 4, 1, 8>(s, a, z, st) : launch_sums<TD, 4, 2, 4>(s, a, z, st);
    if (v == 2) return s.dim <= 64 ? launch_sums<TD, 2, 1, 8>(s, a, z, st) : launch_sums<TD, 2, 4, 4>(s, a, z, st);
    return launch_sums<TD, 1, 4, 4>(s, a, z, st);
}

} // namespace

extern "C" {

int choco_embedding_init(choco_embedding** out, const choco_embedding_params* p)
{
    if (!out) return CHOCO_ERR_INVALID_ARG;
    *out = nullptr;
    if (!p || p->n < 1 || p->vocab < 1 || p->dim < 1 || p->max_tokens < 0 || !std::isfinite(p->scale)) return CHOCO_ERR_INVALID_ARG;
    if (p->n > 65535 || p->vocab > 0x7ffffffe || p->dim > ((int64_t)1 << 22)) return CHOCO_ERR_TOO_LARGE;
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
    const int64_t total = q.n * q.max_tokens;
    e->pitch = (q.dim + 7) / 8 * 8;
    e->present_bytes = (q.vocab + 31) / 32 * 4;
    if (total > 0) {
        const int64_t sort_tiles = (q.max_tokens + kSortTile - 1) / kSortTile;
        // batches of every size up to the largest have to fit, in tiles of either length
        const int64_t few = std::min(total, kShortRows);
        const int64_t tiles = std::max<int64_t>((q.max_tokens + kTileLong - 1) / kTileLong * q.n, (few + kTileShort - 1) / kTileShort + q.n);
        auto get = [&](auto** ptr, int64_t count) {
            if (err == cudaSuccess) err = cudaMalloc((void**)ptr, (size_t)count * sizeof(**ptr));
        };
        for (int k = 0; k < 2; ++k) { get(&e->key[k], total); get(&e->pos[k], total); }
        get(&e->hist, q.n * kDigits * sort_tiles);
        get(&e->total, (int64_t)q.n * kDigits);
        get(&e->part, tiles * 2 * e->pitch);
    }
    if (q.max_tokens > 0 && err == cudaSuccess) {
        err = cudaMalloc((void**)&e->present, (size_t)(q.n * e->present_bytes));
        if (err == cudaSuccess) err = cudaMemset(e->present, 0, (size_t)(q.n * e->present_bytes));
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
    free_all(emb); // cudaFree waits for what still uses the memory
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
    cudaStream_t st = (cudaStream_t)stream;
    const int most = table_dtype == CHOCO_F32 && out_dtype == CHOCO_F32 ? 4 : 8;
    const int v = std::min(vector_of(table, table_dtype, s.table_row, s.table_ld, s.dim, s.n, most),
                           vector_of(out, out_dtype, out_row, out_ld, s.dim, s.n, most));
    return with_type(table_dtype, [&](auto* tt) {
        return with_type(out_dtype, [&](auto* to) {
            using TT = std::remove_pointer_t<decltype(tt)>;
            using TO = std::remove_pointer_t<decltype(to)>;
            auto go = [&](auto vec) {
                constexpr int V = decltype(vec)::value;
                const int64_t slabs = (s.dim + 32 * V * kLookupVecs - 1) / (32 * V * kLookupVecs);
                const int64_t blocks = (count * s.n * slabs + kEmbWarps - 1) / kEmbWarps;
                if (blocks > 0x7fffffff) return (int)CHOCO_ERR_TOO_LARGE;
                lookup_kernel<TT, TO, V><<<(unsigned)blocks, kEmbThreads, 0, st>>>(
                    s, static_cast<const TT*>(table), tokens, index_bits, tokens_ld, static_cast<TO*>(out), out_row, out_ld,
                    (uint32_t)slabs);
                return status_of_launch();
            };
            if constexpr (sizeof(TT) == 2 || sizeof(TO) == 2)
                if (v == 8) return go(std::integral_constant<int, 8>());
            if (v >= 4) return go(std::integral_constant<int, 4>());
            if (v == 2) return go(std::integral_constant<int, 2>());
            return go(std::integral_constant<int, 1>());
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
    if (emb->p.max_tokens == 0 || count > emb->p.max_tokens) return CHOCO_ERR_TOO_LARGE;
    if (count > 0 && (!dout || dout_row < emb->p.dim || (emb->p.n > 1 && dout_ld < 0))) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(grad, dtype_size(grad_dtype)) || !aligned_to(dout, dtype_size(dout_dtype))) return CHOCO_ERR_MISALIGNED;
    if (count == 0 && accumulate) return CHOCO_OK;
    const EmbShape s = shape_of(emb, count);
    cudaStream_t st = (cudaStream_t)stream;
    const int64_t sort_tiles = (count + kSortTile - 1) / kSortTile;

    Presence pres = {accumulate ? nullptr : emb->present, emb->present_bytes};
    ZeroWork z = {};
    z.pres = pres;
    z.grad = grad;
    z.dtype = grad_dtype;
    z.wide = vector_of(grad, grad_dtype, s.table_row, s.table_ld, s.dim, s.n, 8) * (int)dtype_size(grad_dtype);
    z.wide = std::min(z.wide, 16);
    const int64_t map = accumulate ? 0 : emb->present_bytes * s.n;
    // `part` of `parts` of the rows nobody names, done by blocks behind those of a launch
    auto share = [&](int part, int parts) {
        z.begin = map * part / parts;
        z.end = map * (part + 1) / parts;
        z.blocks = (int32_t)std::min<int64_t>((z.end - z.begin + kEmbWarps - 1) / kEmbWarps, 148 * 8);
    };
    cudaError_t err = cudaSuccess;
    if (!accumulate) {
        if (emb->dirty) err = cudaMemsetAsync(emb->present, 0, (size_t)map, st);
        emb->dirty = true;
    }
    int cur = 0;
    const dim3 threads(kEmbThreads);
    const int bits = rank_bits(s);
    if (count > 0 && bits > 0) {
        const size_t smem = (size_t)(count + 15) / 16 * 16 * 4;
        const dim3 grid((unsigned)((count + kRankKeys - 1) / kRankKeys), (unsigned)s.n);
        if (err == cudaSuccess)
            err = launch_overlapped(rank_kernel, grid, threads, smem, st, HotRange{}, s, tokens, tokens_ld, index_bits, bits, pres,
                                    emb->key[0], emb->pos[0]);
        share(0, 1);
    } else if (count > 0) {
        SortPass p = {};
        p.tokens = tokens; p.tokens_ld = tokens_ld; p.index_bits = index_bits;
        p.tiles = (int32_t)sort_tiles;
        p.hist = emb->hist;
        p.total = emb->total;
        p.pres = pres;
        p.first = 1;
        int passes = 1;
        while ((s.vocab >> (passes * kDigitBits)) != 0) ++passes;
        const int shares = 3 * passes - 1; // every launch but the first, which finds out what is present, zeroes a share
        int done = 0;
        for (int k = 0; k < passes; ++k) {
            p.shift = k * kDigitBits;
            p.key_in = emb->key[cur]; p.pos_in = emb->pos[cur];
            p.key_out = emb->key[cur ^ 1]; p.pos_out = emb->pos[cur ^ 1];
            const unsigned tiles = (unsigned)(sort_tiles * s.n), digits = (unsigned)(s.n * (kDigits / kEmbWarps));
            if (k == 0) z.begin = z.end = z.blocks = 0;
            else share(done++, shares);
            if (err == cudaSuccess) err = launch_overlapped(sort_count_kernel, dim3(tiles + z.blocks), threads, 0, st, HotRange{}, s, p, z);
            share(done++, shares);
            if (err == cudaSuccess) err = launch_overlapped(sort_scan_kernel, dim3(digits + z.blocks), threads, 0, st, HotRange{}, s, p, z);
            share(done++, shares);
            if (err == cudaSuccess) err = launch_overlapped(sort_scatter_kernel, dim3(tiles + z.blocks), threads, 0, st, HotRange{}, s, p, z);
            p.first = 0;
            cur ^= 1;
        }
        z.begin = z.end = z.blocks = 0;
    } else {
        share(0, 1);
    }
    Sums a = {};
    a.keys = emb->key[cur]; a.pos = emb->pos[cur];
    a.dout = dout; a.dout_row = dout_row; a.dout_ld = dout_ld;
    a.grad = grad; a.grad_dtype = grad_dtype; a.accumulate = accumulate;
    a.part = emb->part; a.pitch = emb->pitch;
    a.tile = tile_of(count * s.n);
    a.tiles = (int32_t)((count + a.tile - 1) / a.tile);
    const int v = std::min(vector_of(dout, dout_dtype, dout_row, dout_ld, s.dim, s.n, 8),
                           vector_of(grad, grad_dtype, s.table_row, s.table_ld, s.dim, s.n, 8));
    if (err == cudaSuccess)
        with_type(dout_dtype, [&](auto* td) {
            err = launch_sums_for<std::remove_pointer_t<decltype(td)>>(s, a, z, v, st);
            return 0;
        });
    if (err == cudaSuccess && a.tiles > 1) {
        const dim3 grid((unsigned)(((int64_t)a.tiles * s.n + kEmbWarps - 1) / kEmbWarps), (unsigned)((s.dim + kJoinCols - 1) / kJoinCols));
        err = launch_overlapped(join_kernel, grid, threads, 0, st, HotRange{}, s, a);
    }
    if (err != cudaSuccess || status_of_launch() != CHOCO_OK) {
        cudaGetLastError();
        return CHOCO_ERR_CUDA;
    }
    emb->dirty = false;
    return CHOCO_OK;
}

} // extern "C"
