// Token lookup and its gradient for the tables of all workers (choco_embedding_* in choco.h).
//
// The gradient orders every worker's tokens with their positions, so that the rows of dout that
// belong to one row of the table follow one another in order of position, cuts that list into tiles
// of equal length and adds up each tile's rows in registers, in float32.  A run of one token that
// goes on for more than half a tile leaves partial sums, which a last kernel adds in tile order.
// Every element of the gradient is written, or added to, once: the result depends on the tokens
// and the sizes alone.
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
constexpr int kTileMid = 16;                // ... and fewer: more warps, shorter chains of loads
constexpr int kTileShort = 8;
constexpr int64_t kMidRows = 65536, kShortRows = 16384;
constexpr uint32_t kNoKey = 0xffffffffu;
constexpr int kShortChain = 8;              // tiles behind the first that a run's partial sums are in, for one warp to add
constexpr int64_t kJoinBlocks = 148 * 5;

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

// N vectors of V elements a lane, all its loads in flight together: a warp serves 32 N V columns of
// a row, or where rows are narrow 32 / lanes of them.  The row of the table is known only when the
// token has arrived, so the bytes in flight have to come from many warps, and rows too narrow to
// fill one are served together.
// Where a lane's vectors of one row are small, it takes those of up to three rows together (rows of 650
// bf16: 11.2 us alone, 9.4 us three; of 650 floats: 14.9 and 14.1 us; of 1024 bf16, 16 words of
// a lane, nothing is gained, and with 32 words much is lost).
template <typename TT, int V, int N>
__host__ __device__ constexpr int lookup_rows()
{
    constexpr int words = N * ((V * (int)sizeof(TT) + 3) / 4);
    return words <= 8 ? 3 : words <= 12 ? 2 : 1;
}

template <typename TT, typename TO, int V, int N, bool NARROW>
__global__ void __launch_bounds__(kEmbThreads)
lookup_kernel(EmbShape s, const TT* table, const void* tokens, int32_t index_bits, int64_t tokens_ld,
              TO* out, int64_t out_row, int64_t out_ld, uint32_t slabs, uint32_t narrow_log)
{
    constexpr int R = NARROW ? 1 : lookup_rows<TT, V, N>();
    const uint32_t lanes_log = NARROW ? narrow_log : 5; // lanes of a row
    const uint32_t lane = threadIdx.x & 31, lanes = 1u << lanes_log, mine = lane & (lanes - 1);
    const uint32_t item = ((blockIdx.x * kEmbWarps + (threadIdx.x >> 5)) << (5 - lanes_log)) + (lane >> lanes_log);
    const uint32_t tr = slabs == 1 ? item : item / slabs, slab = slabs == 1 ? 0 : item - tr * slabs;
    const uint32_t t = tr * R;
    wait_for_previous_kernel();
    allow_next_kernel();
    if (t >= (uint32_t)s.count) return;
    const int64_t i = blockIdx.y;
    int64_t tok[R];
#pragma unroll
    for (int r = 0; r < R; ++r) tok[r] = t + r < (uint32_t)s.count ? token_at(tokens, index_bits, i * tokens_ld + t + r, s.vocab) : -1;
    const int32_t step = (int32_t)lanes * V, c0 = (int32_t)slab * step * N + (int32_t)mine * V, dim = (int32_t)s.dim;
    Raw<TT, V> raw[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const TT* w = table + i * s.table_ld + (tok[r] < 0 ? 0 : tok[r]) * s.table_row;
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (tok[r] >= 0 && c0 + k * step < dim) load_raw(raw[r][k], w + c0 + k * step);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (t + r >= (uint32_t)s.count) break;
        TO* o = out + i * out_ld + (int64_t)(t + r) * out_row;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int32_t c = c0 + k * step;
            if (c >= dim) continue;
            float f[V];
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = tok[r] >= 0 ? raw_get(raw[r][k], e) * s.scale : 0.f;
            store_vec<TO, V>(o + c, f);
        }
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

// ---------------------------------------------------------------------------------------
// zeros
// ---------------------------------------------------------------------------------------

// `bytes` bytes from p on (both even), by `of` threads, this one the i-th
__device__ __forceinline__ void zero_run(char* p, int64_t bytes, int i, int of)
{
    char* const end = p + bytes;
    char* const body = p + ((16 - ((uintptr_t)p & 15)) & 15);
    if (body >= end) {
        for (char* q = p + 2 * i; q < end; q += 2 * of) *reinterpret_cast<unsigned short*>(q) = 0;
        return;
    }
    char* const tail = end - ((uintptr_t)end & 15);
    for (char* q = body + 16 * i; q < tail; q += 16 * of) *reinterpret_cast<uint4*>(q) = make_uint4(0, 0, 0, 0);
    if (p + 2 * i < body) *reinterpret_cast<unsigned short*>(p + 2 * i) = 0; // (at most seven each)
    if (tail + 2 * i < end) *reinterpret_cast<unsigned short*>(tail + 2 * i) = 0;
}

constexpr int kZeroSpan = 8192;             // bytes of a block

// All rows of the gradient, before the sums are written to those that tokens name.  Runs beside the
// kernel that puts the tokens in order, which leaves the memory and most SMs idle: that kernel
// lets this one start as soon as all that came before has ended, and the last block here waits for
// it, so that what follows finds both done.  Knowing the named rows first would save their bytes,
// and cost the time the ordering takes.  Short blocks in order reach the memory's rate; a resident
// grid that walks over the table got 5.5 TB/s of 7.3.
__global__ void __launch_bounds__(kEmbThreads) zero_kernel(EmbShape s, char* grad, int32_t size, uint32_t blocks_per_row, int32_t beside)
{
    if (!beside) wait_for_previous_kernel();
    allow_next_kernel();
    char* const table = grad + blockIdx.y * s.table_ld * size;
    if (s.table_row == s.dim) { // one run of bytes
        const int64_t all = s.vocab * s.dim * size, from = (int64_t)blockIdx.x * kZeroSpan;
        zero_run(table + from, min((int64_t)kZeroSpan, all - from), threadIdx.x, kEmbThreads);
    } else {
        const int64_t row = blockIdx.x / blocks_per_row, from = (int64_t)(blockIdx.x - row * blocks_per_row) * kZeroSpan;
        zero_run(table + row * s.table_row * size + from, min((int64_t)kZeroSpan, s.dim * size - from), threadIdx.x, kEmbThreads);
    }
    if (beside && blockIdx.x + 1 == gridDim.x && blockIdx.y + 1 == gridDim.y) wait_for_previous_kernel();
}

// For each of N keys of a lane the lanes whose key has the same digit, a ballot per bit; the keys' votes do
// not wait for one another.  Keys that are none are alike with nobody that is one.  (The match
// instruction takes longer where most digits differ.)
template <int N>
__device__ __forceinline__ void lanes_alike(uint32_t (&alike)[N], const uint32_t (&key)[N], int shift, int bits, int rounds)
{
#pragma unroll
    for (int r = 0; r < N; ++r) alike[r] = __ballot_sync(0xffffffffu, key[r] != kNoKey);
    for (int b = 0; b < bits; ++b) {
#pragma unroll
        for (int r = 0; r < N; ++r) {
            if (r >= rounds) break;
            const bool one = key[r] >> (shift + b) & 1;
            const uint32_t ones = __ballot_sync(0xffffffffu, one);
            alike[r] &= one ? ones : ~ones;
        }
    }
}

// Up to 16 x 8192 tokens per worker: a cluster of blocks keeps a worker's keys and positions in its
// shared memory and sorts them there, digit by digit (stable, from the lowest).  Every block counts
// and ranks its part of the list and puts it in order for itself, the blocks add up each other's
// counts, and each pair goes to its place in the shared memory of the block that holds it next, in
// the last round to global memory.  One launch where a sort in global memory takes three per digit
// (131072 tokens of 16 bits: 27 us against 45 us; 8 x 2240: 12 us), and most SMs stay free for the
// zeros.  What it takes is latency: per digit about 2 us of barriers and exchanged counts, and
// 4 us for 8192 keys to be ranked and sent.
// Up to 4096 tokens of up to 16 bits a block of 512 threads does it alone: fewer warps have counts
// to add up and meet at barriers (8 x 2240 rows of 650 floats added, all three launches: 34.5 -> 32.8 us;
// 4 x 1000 of 200: 15.2 -> 14.1 us).
constexpr int kOrderRounds = 8;             // keys of a thread, at most
constexpr int kOrderThreads = 1024, kOrderThreadsFew = 512;
constexpr int kOrderDigitBits = 9, kOrderDigitBitsFew = 8; // (a digit's counts are one thread's work)
constexpr int kOrderMost = kOrderThreads * kOrderRounds, kOrderMostFew = kOrderThreadsFew * kOrderRounds; // keys of a block
constexpr int kOrderFew = 2048;             // keys that are not worth a second block
constexpr int kOrderCluster = 16;           // blocks of a cluster, at most

struct Order {
    const void* tokens;
    int64_t tokens_ld;
    int32_t index_bits;
    int32_t cluster_log, part_log;          // blocks of a cluster, keys of a block
    int32_t digit_bits, passes;
    int32_t few;                            // one block of kOrderThreadsFew threads
    uint32_t *keys, *pos;                   // out: [n, count]
    uint32_t* chain_count;                  // set to 0 (see Sums)
};

template <int THREADS>
struct OrderSmem {
    static constexpr int kWarps = THREADS / 32, kDigits = 1 << (THREADS == kOrderThreads ? kOrderDigitBits : kOrderDigitBitsFew);
    uint16_t cnt[kWarps][kDigits];
    uint32_t hist[kDigits];                 // read by the other blocks
    uint32_t base[kDigits];
    uint32_t ws[kWarps];
};

__device__ __forceinline__ uint32_t cluster_address(const void* p, uint32_t block) // of block's copy of a shared variable
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(block));
    return a;
}
__device__ __forceinline__ uint32_t load_cluster(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void store_cluster(uint32_t a, uint32_t x, uint32_t y)
{
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(a), "r"(x), "r"(y) : "memory");
}
// (not the forms that a whole warp has to reach together: with fewer digits than lanes, warps come out of a branch)
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

template <int THREADS>
__global__ void __launch_bounds__(THREADS) order_kernel(EmbShape s, Order o)
{
    constexpr int kWarps = THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    OrderSmem<THREADS>& m = *reinterpret_cast<OrderSmem<THREADS>*>(smem);
    uint2* buf = reinterpret_cast<uint2*>(smem + sizeof(OrderSmem<THREADS>)); // two buffers of (key, position)
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int32_t worker = blockIdx.x >> o.cluster_log;
    wait_for_previous_kernel();
    allow_next_kernel();
    if (blockIdx.x == 0 && threadIdx.x < 2) o.chain_count[threadIdx.x] = 0;
    const uint32_t rank = blockIdx.x & ((1u << o.cluster_log) - 1u), blocks = 1u << o.cluster_log;
    const uint32_t part = 1u << o.part_log;
    const uint32_t first = rank << o.part_log;
    const int have = (int)min((int64_t)part, max((int64_t)0, s.count - (int64_t)first));
    const int rounds = part / THREADS, slice = part / kWarps;
    constexpr int kRounds = kOrderRounds;
    uint32_t key[kRounds], pos[kRounds];
    uint16_t place[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int j = w * slice + r * 32 + lane;
        key[r] = kNoKey;
        if (r < rounds && j < have) {
            key[r] = sort_key(s, o.tokens, o.index_bits, worker * o.tokens_ld + first + j);
            pos[r] = first + j;
        }
    }
    const uint32_t digits = 1u << o.digit_bits;
    for (int pass = 0; pass < o.passes; ++pass) {
        const int shift = pass * o.digit_bits;
        uint2* in = buf + (pass & 1) * part;
        uint2* out = buf + ((pass & 1) ^ 1) * part;
        for (uint32_t d = lane; d < digits; d += 32) m.cnt[w][d] = 0;
        if (pass > 0) {
#pragma unroll
            for (int r = 0; r < kRounds; ++r) {
                const int j = w * slice + r * 32 + lane;
                if (r < rounds && j < have) { key[r] = in[j].x; pos[r] = in[j].y; }
            }
        }
        __syncwarp();
        uint32_t alike[kRounds];
        lanes_alike<kRounds>(alike, key, shift, o.digit_bits, rounds);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (r >= rounds) break;
            const bool live = key[r] != kNoKey;
            const uint32_t d = (key[r] >> shift) & (digits - 1);
            const uint32_t before = live ? m.cnt[w][d] : 0u;
            __syncwarp();
            place[r] = (uint16_t)(before + __popc(alike[r] & ((1u << lane) - 1u)));
            if (live && lane == __ffs(alike[r]) - 1) m.cnt[w][d] = (uint16_t)(before + __popc(alike[r]));
            __syncwarp();
        }
        __syncthreads();
        // exclusive sums over the digits, one digit per thread
        auto scan = [&](uint32_t mine) {
            uint32_t incl = mine;
#pragma unroll
            for (int q = 1; q < 32; q <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, incl, q);
                if (lane >= q) incl += u;
            }
            if (lane == 31) m.ws[w] = incl;
            __syncthreads();
            uint32_t v = lane < kWarps ? m.ws[lane] : 0u;
#pragma unroll
            for (int q = 1; q < 32; q <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, v, q);
                if (lane >= q) v += u;
            }
            const uint32_t before = __shfl_sync(0xffffffffu, v, (w + 31) & 31); // up to the warp before
            __syncthreads();
            return incl - mine + (w ? before : 0u);
        };
        uint32_t own = 0;
        if (threadIdx.x < digits) {
#pragma unroll
            for (int k = 0; k < kWarps; ++k) own += m.cnt[k][threadIdx.x];
            m.hist[threadIdx.x] = own;
        }
        if (blocks > 1) cluster_arrive();
        const uint32_t start = scan(own); // where this block's keys with the digit start in its own order
        if (threadIdx.x < digits) {
            uint32_t at = start;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                const uint32_t c = m.cnt[k][threadIdx.x];
                m.cnt[k][threadIdx.x] = (uint16_t)at;
                at += c;
            }
        }
        __syncthreads();
        // the block's pairs in its own order, so that what goes to one place goes there in runs
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (r >= rounds || key[r] == kNoKey) continue;
            in[m.cnt[w][(key[r] >> shift) & (digits - 1)] + place[r]] = make_uint2(key[r], pos[r]);
        }
        uint32_t earlier = 0, total = 0;
        if (blocks > 1) cluster_wait();
        if (blocks > 1 && threadIdx.x < digits) {
            for (uint32_t b = 0; b < blocks; b += 8) {
                uint32_t c[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) c[k] = b + k < blocks ? load_cluster(cluster_address(&m.hist[threadIdx.x], b + k)) : 0u;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (b + k < rank) earlier += c[k];
                    total += c[k];
                }
            }
        }
        if (blocks > 1) {
            const uint32_t base = scan(total);
            if (threadIdx.x < digits) m.base[threadIdx.x] = base + earlier - start;
        } else if (threadIdx.x < digits) {
            m.base[threadIdx.x] = 0; // the block's own order is all
        }
        __syncthreads();
        const bool last = pass + 1 == o.passes;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int j = r * THREADS + threadIdx.x;
            if (r >= rounds || j >= have) break;
            const uint2 kp = in[j];
            const uint32_t to = m.base[(kp.x >> shift) & (digits - 1)] + j;
            if (last) {
                o.keys[worker * s.count + to] = kp.x;
                o.pos[worker * s.count + to] = kp.y;
            } else if (blocks > 1) {
                store_cluster(cluster_address(out + (to & (part - 1)), to >> o.part_log), kp.x, kp.y);
            } else {
                out[to] = kp;
            }
        }
        // what was sent has arrived, and nobody reads these counts any more (nor, at the end, this block's memory)
        if (blocks > 1) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
    }
}

// More tokens: a stable radix sort in global memory, three launches per digit.
struct SortPass {
    const void* tokens;          // first pass: the tokens themselves
    int64_t tokens_ld;
    int32_t index_bits, shift, first;
    int32_t tiles;               // per worker
    const uint32_t *key_in, *pos_in;
    uint32_t *key_out, *pos_out;
    uint32_t* hist;              // [n, kDigits, tiles]
    uint32_t* total;             // [n, kDigits]
    uint32_t* chain_count;       // set to 0 (see Sums)
};

__device__ __forceinline__ uint32_t pass_key(const EmbShape& s, const SortPass& p, int32_t worker, int64_t j)
{
    return p.first ? sort_key(s, p.tokens, p.index_bits, worker * p.tokens_ld + j) : p.key_in[worker * s.count + j];
}

__global__ void __launch_bounds__(kEmbThreads) sort_count_kernel(EmbShape s, SortPass p)
{
    __shared__ uint32_t h[kDigits];
    wait_for_previous_kernel();
    allow_next_kernel();
    const int32_t worker = blockIdx.x / p.tiles, tile = blockIdx.x - worker * p.tiles;
    if (blockIdx.x == 0 && threadIdx.x < 2) p.chain_count[threadIdx.x] = 0;
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
    }
    __syncthreads();
    p.hist[((int64_t)worker * kDigits + threadIdx.x) * p.tiles + tile] = h[threadIdx.x];
}

// One warp per digit: exclusive sums of its counts over the tiles, and their total.
__global__ void __launch_bounds__(kEmbThreads) sort_scan_kernel(EmbShape s, SortPass p)
{
    wait_for_previous_kernel();
    allow_next_kernel();
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kEmbWarps + (threadIdx.x >> 5);
    uint32_t* h = p.hist + row * p.tiles;
    uint32_t carry = 0;
    for (int32_t b = 0; b < p.tiles; b += 32 * 8) { // a lane has eight tiles in a row
        uint32_t c[8], sum = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int32_t j = b + lane * 8 + k;
            c[k] = j < p.tiles ? h[j] : 0u;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += c[k];
        uint32_t v = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        uint32_t at = carry + v - sum;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int32_t j = b + lane * 8 + k;
            if (j < p.tiles) h[j] = at;
            at += c[k];
        }
        carry += __shfl_sync(0xffffffffu, v, 31);
    }
    if (lane == 0) p.total[row] = carry;
}

// Every warp ranks its slice of the tile in order; equal digits keep their order.
__global__ void __launch_bounds__(kEmbThreads) sort_scatter_kernel(EmbShape s, SortPass p)
{
    __shared__ uint32_t cnt[kEmbWarps][kDigits];
    __shared__ uint32_t ws[kEmbWarps];
    wait_for_previous_kernel();
    allow_next_kernel();
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
    uint32_t alike[kSortRounds];
    lanes_alike<kSortRounds>(alike, key, p.shift, kDigitBits, kSortRounds);
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const bool in = key[r] != kNoKey;
        const uint32_t d = (key[r] >> p.shift) & (kDigits - 1);
        const uint32_t same = alike[r];
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
    uint32_t* chains;            // [n * tiles] tiles with a run of the second kind, in no order: those of few tiles from the
    uint32_t chain_room;         // front, long ones from the back
    uint32_t* chain_count;       // [2] their numbers
    int64_t pitch;
    int32_t tile;                // entries per tile
    int32_t tiles;               // per worker
    uint32_t slabs;              // groups of columns
};

// Adds to float32 in memory without reading it first.  Every element gets at most one such addition
// in a call, so their order does not matter (subnormal results become zeros).
template <int V>
__device__ __forceinline__ void add_in_memory(float* p, const float* f)
{
    if constexpr (V >= 4) {
#pragma unroll
        for (int k = 0; k < V; k += 4)
            asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p + k), "f"(f[k]), "f"(f[k + 1]), "f"(f[k + 2]), "f"(f[k + 3])
                         : "memory");
    } else if constexpr (V == 2) {
        asm volatile("red.global.add.v2.f32 [%0], {%1, %2};" ::"l"(p), "f"(f[0]), "f"(f[1]) : "memory");
    } else {
        asm volatile("red.global.add.f32 [%0], %1;" ::"l"(p), "f"(f[0]) : "memory");
    }
}

// scale * acc (+ what is there) to V columns of a row of the gradient, whose type is known at run time
template <int V>
__device__ __forceinline__ void store_grad(const EmbShape& s, void* grad, int32_t dtype, bool accumulate, int32_t worker, uint32_t key,
                                           int64_t c, const float* acc)
{
    const int64_t at = worker * s.table_ld + (int64_t)key * s.table_row + c;
    float f[V];
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = acc[e] * s.scale;
    auto put = [&](auto* g) {
        using TG = std::remove_pointer_t<decltype(g)>;
        if (accumulate) {
            if constexpr (std::is_same_v<TG, float>) {
                add_in_memory<V>(g + at, f);
                return;
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] += to_float(g[at + e]);
            }
        }
        store_vec<TG, V>(g + at, f);
    };
    if (dtype == CHOCO_F32) put(static_cast<float*>(grad));
    else if (dtype == CHOCO_BF16) put(static_cast<__nv_bfloat16*>(grad));
    else put(static_cast<__half*>(grad));
}

// One warp per tile and group of 32 V C columns; B entries' loads are in flight together.  A run that
// starts in the tile and reaches at most half a tile into the next one is added up here (and left out
// there); what reaches further leaves a partial sum for every tile it is in.  What bounds it is the
// memory (131072 rows of 1024 bf16 into 27000 rows of floats: 350 MB in 55 us); the registers are kept
// below 85 so that 24 warps share an SM.
constexpr int kSumThreads = 128, kSumBlocks = 6;

template <typename TD, int V, int C, int B>
__global__ void __launch_bounds__(kSumThreads, kSumBlocks) sum_tiles_kernel(EmbShape s, Sums a)
{
    wait_for_previous_kernel();
    allow_next_kernel();
    // the tile's entries, what is taken from the next one, and room for a batch to look past the end
    __shared__ uint32_t entry_key[kSumThreads / 32][kTileLong * 3 / 2 + B], entry_pos[kSumThreads / 32][kTileLong * 3 / 2 + B];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const uint64_t item = (uint64_t)blockIdx.x * (kSumThreads / 32) + (threadIdx.x >> 5);
    const uint32_t gt = (uint32_t)(item / a.slabs), slab = (uint32_t)(item - (uint64_t)gt * a.slabs);
    if (gt >= (uint32_t)a.tiles * (uint32_t)s.n) return;
    const int32_t worker = gt / (uint32_t)a.tiles, tile = gt - worker * a.tiles;
    const int64_t first = (int64_t)tile * a.tile, e0 = worker * s.count + first;
    const int cnt = (int)min((int64_t)a.tile, s.count - first);
    const uint32_t key = lane < cnt ? a.keys[e0 + lane] : kNoKey;
    const uint32_t pos = lane < cnt ? a.pos[e0 + lane] : 0u;
    const uint32_t prev = tile > 0 ? a.keys[e0 - 1] : kNoKey;
    // what follows the tile, for its last run
    const bool there = first + cnt + lane < s.count;
    const uint32_t more_key = there ? a.keys[e0 + cnt + lane] : kNoKey, more_pos = there ? a.pos[e0 + cnt + lane] : 0u;
    const int64_t far_on = first + (kShortChain + 1) * a.tile;
    const uint32_t far_key = far_on < s.count ? a.keys[worker * s.count + far_on] : kNoKey;
    const int live = __popc(__ballot_sync(0xffffffffu, key < (uint32_t)s.vocab));
    if (live == 0) return;
    // Does the run that ends the tile before start there, and reach at most half a tile into this
    // one?  Then that tile's warp has added it up.
    const int reach = a.tile / 2;
    int from = 0;
    bool head = __shfl_sync(0xffffffffu, key, 0) == prev;
    if (head) {
        const uint32_t before = a.keys[e0 - a.tile], far = tile > 1 ? a.keys[e0 - a.tile - 1] : kNoKey;
        const int lead = __ffs(~__ballot_sync(0xffffffffu, lane < cnt && key == prev)) - 1; // (cnt < 32 or a later key differs, or -1)
        if (lead >= 0 && lead <= reach && !(before == prev && far == prev)) {
            if (lead >= live) return;
            from = lead;
            head = false;
        }
    }
    uint32_t cur = __shfl_sync(0xffffffffu, key, from);
    // And does the last run go on, and if it started here, not further than that?  Then what
    // follows the tile of it is this warp's too.
    const uint32_t last = __shfl_sync(0xffffffffu, key, live - 1);
    bool goes_on = live == cnt && __shfl_sync(0xffffffffu, more_key, 0) == last;
    int end = live;
    if (goes_on && !(head && cur == last)) {
        const int more = __ffs(~__ballot_sync(0xffffffffu, more_key == last)) - 1;
        if (more >= 0 && more <= reach) {
            end += more;
            goes_on = false;
        } else if (slab == 0 && lane == 0) {
            if (far_key == last) a.chains[a.chain_room - 1 - atomicAdd(a.chain_count + 1, 1u)] = gt;
            else a.chains[atomicAdd(a.chain_count, 1u)] = gt;
        }
    }
    if (lane < cnt) {
        entry_key[w][lane] = key;
        entry_pos[w][lane] = pos;
    }
    if (lane < end - cnt) {
        entry_key[w][cnt + lane] = more_key;
        entry_pos[w][cnt + lane] = more_pos;
    }
    __syncwarp();
    const TD* d = static_cast<const TD*>(a.dout) + worker * a.dout_ld;
    const int64_t c0 = (int64_t)slab * (32 * V * C) + lane * V;
    float acc[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[c][e] = 0.f;
    auto flush = [&](bool unfinished) {
        if (head || unfinished) {
            float* p = a.part + ((int64_t)gt * 2 + (head ? 0 : 1)) * a.pitch;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c0 + c * 32 * V < s.dim) store_vec<float, V>(p + c0 + c * 32 * V, acc[c]);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c0 + c * 32 * V < s.dim)
                    store_grad<V>(s, a.grad, a.grad_dtype, a.accumulate, worker, cur, c0 + c * 32 * V, acc[c]);
        }
    };
    for (int b = from; b < end; b += B) {
        Raw<TD, V> raw[B][C];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const uint32_t p = entry_pos[w][b + j];
            if (b + j < end) {
                const TD* r = d + p * a.dout_row;
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (c0 + c * 32 * V < s.dim) load_raw(raw[j][c], r + c0 + c * 32 * V);
            }
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            if (b + j >= end) break;
            const uint32_t k = entry_key[w][b + j];
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
    flush(goes_on);
}

// Runs that reach further than half a tile into the next one: the partial sums of all their tiles,
// in order, 128 columns at a time.  Chains of up to kShortChain tiles are a warp's work, all parts in
// flight together; of longer ones (frequent tokens) a block takes one, a warp a contiguous part.
constexpr int kJoinCols = 128;              // four a lane

template <int V>
__global__ void __launch_bounds__(kEmbThreads) join_kernel(EmbShape s, Sums a, uint32_t slabs)
{
    __shared__ float4 sub[kEmbWarps][32];
    wait_for_previous_kernel();
    allow_next_kernel();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const uint32_t few = a.chain_count[0], many = a.chain_count[1];
    auto add = [](float4& x, const float4 y) { x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w; };
    auto part_of = [&](uint32_t t, int slot, int64_t c) {
        return *reinterpret_cast<const float4*>(a.part + ((int64_t)t * 2 + slot) * a.pitch + c);
    };
    // sum += slots 0 of the tiles t + [from, to)
    auto add_parts = [&](float4& sum, uint32_t t, uint32_t from, uint32_t to, int64_t c) {
        for (uint32_t j = from; j < to; j += kShortChain) {
            float4 v[kShortChain];
#pragma unroll
            for (int u = 0; u < kShortChain; ++u) v[u] = j + u < to ? part_of(t + j + u, 0, c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int u = 0; u < kShortChain; ++u) add(sum, v[u]);
        }
    };
    auto put = [&](int32_t worker, uint32_t key, int64_t c, const float4 sum) {
        const float f[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
        for (int e = 0; e < 4; e += V)
            if (c + e < s.dim) store_grad<V>(s, a.grad, a.grad_dtype, a.accumulate, worker, key, c + e, f + e);
    };
    for (uint64_t task = blockIdx.x; task < (uint64_t)many * slabs; task += gridDim.x) {
        const uint32_t at = (uint32_t)(task / slabs), gt = a.chains[a.chain_room - 1 - at];
        const int64_t c = (int64_t)(task - (uint64_t)at * slabs) * kJoinCols + lane * 4;
        const int32_t worker = gt / (uint32_t)a.tiles, tile = gt - worker * a.tiles;
        const uint32_t* k = a.keys + worker * s.count;
        const uint32_t key = k[(int64_t)(tile + 1) * a.tile - 1];
        // The tiles that begin with this key follow one another: tile + 1 is one, the last is in
        // [lo, hi); 32 places are looked at together.
        int32_t lo = tile + 1, hi = a.tiles;
        while (hi - lo > 1) {
            const int32_t step = (hi - lo + 31) / 32;
            const int64_t j = lo + (int64_t)(lane + 1) * step;
            const int32_t n = __popc(__ballot_sync(0xffffffffu, j < hi && k[(j < hi ? j : lo) * a.tile] == key));
            hi = min(hi, lo + (n + 1) * step);
            lo += n * step;
        }
        const uint32_t len = lo - tile, each = (len + kEmbWarps - 1) / kEmbWarps;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (w == 0 && c < s.dim) sum = part_of(gt, 1, c);
        if (c < s.dim) add_parts(sum, gt + 1, min(len, w * each), min(len, (w + 1) * each), c);
        sub[w][lane] = sum;
        __syncthreads();
        if (w == 0 && c < s.dim) {
#pragma unroll
            for (int p = 1; p < kEmbWarps; ++p) add(sum, sub[p][lane]);
            put(worker, key, c, sum);
        }
        __syncthreads();
    }
    // (the blocks that had nothing above begin here)
    const uint32_t warps = gridDim.x * kEmbWarps;
    for (uint64_t task = (gridDim.x - 1 - blockIdx.x) * kEmbWarps + w; task < (uint64_t)few * slabs; task += warps) {
        const uint32_t at = (uint32_t)(task / slabs), gt = a.chains[at];
        const int64_t c = (int64_t)(task - (uint64_t)at * slabs) * kJoinCols + lane * 4;
        const int32_t worker = gt / (uint32_t)a.tiles, tile = gt - worker * a.tiles;
        const uint32_t* k = a.keys + worker * s.count;
        const uint32_t key = k[(int64_t)(tile + 1) * a.tile - 1];
        const int64_t j = (int64_t)(tile + 1 + lane) * a.tile; // the tiles behind that begin with it
        const uint32_t len = __popc(__ballot_sync(0xffffffffu, lane < kShortChain && j < s.count && k[j < s.count ? j : 0] == key));
        if (c >= s.dim) continue;
        float4 sum = part_of(gt, 1, c);
        add_parts(sum, gt + 1, 0, len, c);
        put(worker, key, c, sum);
    }
}

// ---------------------------------------------------------------------------------------
// a few tokens: everything in one launch
// ---------------------------------------------------------------------------------------

constexpr int kDirectTokens = 256;          // per worker
// Tables up to this are zeroed by the same launch (13 MB: 5.6 us, 6.6 us apart); beyond, a kernel of its own reaches the
// memory's rate (692 MB: 98 us, 120 us together).
constexpr int64_t kDirectZeroBytes = (int64_t)16 << 20;

struct Direct {
    const void* tokens;
    int64_t tokens_ld;
    int32_t index_bits;
    const void* dout;
    int64_t dout_row, dout_ld;
    void* grad;
    int32_t grad_dtype, accumulate;
    uint32_t groups, slabs;      // groups of kEmbWarps positions, of columns
    int64_t eights;              // groups of eight rows of a table, if rows nobody names become zeros, else 0
    uint32_t zero_blocks;        // per worker
};

// Every warp takes one position.  If its token occurs earlier there is nothing to do; otherwise it
// adds up the rows of all later positions with that token, 32 V C columns.  Blocks behind those zero
// rows: a warp compares eight rows with all tokens.
template <typename TD, int V, int C>
__global__ void __launch_bounds__(kEmbThreads) direct_kernel(EmbShape s, Direct d)
{
    __shared__ uint32_t keys[kDirectTokens];
    __shared__ uint8_t list[kEmbWarps][kDirectTokens];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int32_t worker = blockIdx.y;
    const int count = (int)s.count;
    wait_for_previous_kernel();
    allow_next_kernel();
    if (threadIdx.x < count) keys[threadIdx.x] = sort_key(s, d.tokens, d.index_bits, worker * d.tokens_ld + threadIdx.x);
    __syncthreads();
    const uint32_t sum_blocks = d.groups * d.slabs;
    if (blockIdx.x >= sum_blocks) {
        const int64_t step = (int64_t)d.zero_blocks * kEmbWarps;
        for (int64_t u = (int64_t)(blockIdx.x - sum_blocks) * kEmbWarps + w; u < d.eights; u += step) {
            uint32_t named = 0;
            for (int j = lane; j < count; j += 32) {
                const uint32_t r = keys[j] - (uint32_t)(u * 8);
                if (keys[j] < (uint32_t)s.vocab && r < 8) named |= 1u << r;
            }
            named = __reduce_or_sync(0xffffffffu, named);
            const int64_t size = d.grad_dtype == CHOCO_F32 ? 4 : 2;
            char* p = static_cast<char*>(d.grad) + (worker * s.table_ld + u * 8 * s.table_row) * size;
            const int left = (int)min((int64_t)8, s.vocab - u * 8);
            if (named == 0 && s.table_row == s.dim) zero_run(p, left * s.dim * size, lane, 32);
            else
                for (int r = 0; r < left; ++r)
                    if (!(named >> r & 1)) zero_run(p + r * s.table_row * size, s.dim * size, lane, 32);
        }
        return;
    }
    const uint32_t group = blockIdx.x / d.slabs, slab = blockIdx.x - group * d.slabs;
    const int mine = (int)group * kEmbWarps + w;
    if (mine >= count) return;
    const uint32_t key = keys[mine];
    if (key >= (uint32_t)s.vocab) return;
    for (int j = 0; j < mine; j += 32)
        if (__any_sync(0xffffffffu, j + lane < mine && keys[j + lane] == key)) return;
    int n = 0;
    for (int j = mine & ~31; j < count; j += 32) {
        const bool is = j + lane >= mine && j + lane < count && keys[j + lane] == key;
        const uint32_t all = __ballot_sync(0xffffffffu, is);
        if (is) list[w][n + __popc(all & ((1u << lane) - 1u))] = (uint8_t)(j + lane);
        n += __popc(all);
    }
    __syncwarp();
    const TD* rows = static_cast<const TD*>(d.dout) + worker * d.dout_ld;
    const int64_t c0 = (int64_t)slab * (32 * V * C) + lane * V;
    float acc[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[c][e] = 0.f;
    constexpr int B = 8;
    for (int b = 0; b < n; b += B) {
        Raw<TD, V> raw[B][C];
#pragma unroll
        for (int j = 0; j < B; ++j)
            if (b + j < n) {
                const TD* r = rows + list[w][b + j] * d.dout_row;
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (c0 + c * 32 * V < s.dim) load_raw(raw[j][c], r + c0 + c * 32 * V);
            }
#pragma unroll
        for (int j = 0; j < B; ++j)
            if (b + j < n)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[c][e] += raw_get(raw[j][c], e);
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (c0 + c * 32 * V < s.dim)
            store_grad<V>(s, d.grad, d.grad_dtype, d.accumulate, worker, key, c0 + c * 32 * V, acc[c]);
}

template <typename F>
int with_type(int32_t dtype, F f)
{
    if (dtype == CHOCO_F32) return f((float*)nullptr);
    if (dtype == CHOCO_BF16) return f((__nv_bfloat16*)nullptr);
    return f((__half*)nullptr);
}

int status_of(cudaError_t e)
{
    if (e == cudaSuccess) return CHOCO_OK;
    cudaGetLastError();
    return CHOCO_ERR_CUDA;
}

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
    void* memory;                // all that follows
    uint32_t* key[2];            // the second ones, hist and total only where a batch may have to be sorted in global memory
    uint32_t* pos[2];
    uint32_t* hist;
    uint32_t* total;
    float* part;
    int64_t pitch;
    uint32_t* chains;            // two counts, then the tiles
    uint32_t chain_room;
};

namespace {

bool on_device(const choco_embedding* e)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == e->device;
}

void free_all(choco_embedding* e)
{
    cudaFree(e->memory);
    delete e;
}

EmbShape shape_of(const choco_embedding* e, int64_t count)
{
    const choco_embedding_params& p = e->p;
    return {p.vocab, p.dim, p.table_row, p.table_ld, p.padding, p.scale, p.n, count};
}

int check_tokens(const choco_embedding* e, const void* tokens, int32_t bits, int64_t count, int64_t ld)
{
    if (!on_device(e) || (bits != 32 && bits != 64) || count < 0 || (e->p.n > 1 && ld < count && ld != 0)) return CHOCO_ERR_INVALID_ARG;
    if (count > 0 && !tokens) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(tokens, bits / 8)) return CHOCO_ERR_MISALIGNED;
    if (count >= ((int64_t)1 << 31) || count * e->p.n >= ((int64_t)1 << 31)) return CHOCO_ERR_TOO_LARGE;
    return CHOCO_OK;
}

// Whether two of the rows [i, t], i < n, t < count, at i ld + t row, of `dim` elements each share one (ld, row >= 0).
bool rows_overlap(int64_t n, int64_t count, int64_t dim, int64_t ld, int64_t row)
{
    using wide = __int128;
    if (count > 1 && row < dim) return true;
    if (n == 1 || ld >= (wide)(count - 1) * row + dim) return false;          // worker after worker
    if (ld >= dim && row >= (wide)(n - 1) * ld + dim) return false;           // token after token
    for (int64_t i = 1; i < n; ++i) { // row t of worker 0 and the rows of worker i on either side of it
        const wide at = (wide)i * ld, t = at / row, over = at % row;
        if ((t < count && over < dim) || (t + 1 < count && row - over < dim)) return true;
    }
    return false;
}

// (8 x 2240 rows of 650 added: 33.6 us in tiles of 16, 35.5 us of 32; 4 x 1000 rows of 200: 17.4 us of 8, 18.9 us of 16)
int tile_of(int64_t rows) { return rows <= kShortRows ? kTileShort : rows <= kMidRows ? kTileMid : kTileLong; }

// How a cluster of blocks orders the tokens, or false if there are too many for that.
bool plan_order(const EmbShape& s, Order& o)
{
    if (s.count > (int64_t)kOrderCluster * kOrderMost) return false;
    int bits = 1;
    while ((s.vocab >> bits) != 0) ++bits; // keys go up to vocab
    o.few = s.count <= kOrderMostFew && bits <= 2 * kOrderDigitBitsFew;
    const int most = o.few ? kOrderDigitBitsFew : kOrderDigitBits;
    o.passes = (bits + most - 1) / most;
    o.digit_bits = (bits + o.passes - 1) / o.passes;
    // a block for every kOrderFew keys, while all workers' clusters run at once, or as many as their memory needs
    o.cluster_log = 0;
    while (!o.few && (1 << o.cluster_log) < kOrderCluster && ((int64_t)kOrderFew << o.cluster_log) < s.count &&
           (((int64_t)kOrderMost << o.cluster_log) < s.count || ((int64_t)s.n << (o.cluster_log + 1)) <= 148))
        ++o.cluster_log;
    o.part_log = o.few ? 9 : 10; // a key for each thread
    while (((int64_t)1 << (o.part_log + o.cluster_log)) < s.count) ++o.part_log;
    return true;
}

template <int THREADS>
cudaError_t launch_order_of(const EmbShape& s, const Order& o, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(s.n << o.cluster_log));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = sizeof(OrderSmem<THREADS>) + ((size_t)2 * sizeof(uint2) << o.part_log);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1u << o.cluster_log;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, order_kernel<THREADS>, s, o);
}
cudaError_t launch_order(const EmbShape& s, const Order& o, cudaStream_t st)
{
    return o.few ? launch_order_of<kOrderThreadsFew>(s, o, st) : launch_order_of<kOrderThreads>(s, o, st);
}

// dynamic shared memory beyond the default, clusters of more than eight blocks
cudaError_t allow_order()
{
    cudaError_t e = cudaFuncSetAttribute(order_kernel<kOrderThreads>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)(sizeof(OrderSmem<kOrderThreads>) + 2 * sizeof(uint2) * kOrderMost));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(order_kernel<kOrderThreads>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(order_kernel<kOrderThreadsFew>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)(sizeof(OrderSmem<kOrderThreadsFew>) + 2 * sizeof(uint2) * kOrderMostFew));
    return e;
}

template <typename TD, int V, int C, int B>
cudaError_t launch_sums(const EmbShape& s, Sums a, cudaStream_t st)
{
    a.slabs = (uint32_t)((s.dim + 32 * V * C - 1) / (32 * V * C));
    const uint64_t warps = (uint64_t)a.slabs * a.tiles * s.n;
    const uint64_t blocks = (warps + kSumThreads / 32 - 1) / (kSumThreads / 32);
    return launch_overlapped(sum_tiles_kernel<TD, V, C, B>, dim3((unsigned)blocks), dim3(kSumThreads), 0, st, HotRange{}, s, a);
}

template <typename TD>
cudaError_t launch_sums_for(const EmbShape& s, const Sums& a, int v, cudaStream_t st)
{
    // 256 columns of a row to a warp, 128 where one element at a time is all that alignment leaves;
    // narrow rows take fewer vectors per lane
    if constexpr (sizeof(TD) == 2)
        if (v == 8) return launch_sums<TD, 8, 1, 8>(s, a, st);
    if (v >= 4) return s.dim <= 128 ? launch_sums<TD, 4, 1, 8>(s, a, st) : launch_sums<TD, 4, 2, 4>(s, a, st);
    if (v == 2) return s.dim <= 64 ? launch_sums<TD, 2, 1, 8>(s, a, st) : launch_sums<TD, 2, 4, 4>(s, a, st);
    return launch_sums<TD, 1, 4, 4>(s, a, st);
}

template <typename TD, int V, int C>
cudaError_t launch_direct(const EmbShape& s, Direct d, cudaStream_t st)
{
    d.groups = (uint32_t)((s.count + kEmbWarps - 1) / kEmbWarps);
    d.slabs = (uint32_t)((s.dim + 32 * V * C - 1) / (32 * V * C));
    d.zero_blocks = (uint32_t)std::min<int64_t>((d.eights + kEmbWarps - 1) / kEmbWarps, std::max<int64_t>(1, 148 * 8 / s.n));
    return launch_overlapped(direct_kernel<TD, V, C>, dim3(d.groups * d.slabs + d.zero_blocks, (unsigned)s.n), dim3(kEmbThreads), 0, st,
                             HotRange{}, s, d);
}

template <typename TD>
cudaError_t launch_direct_for(const EmbShape& s, const Direct& d, int v, cudaStream_t st)
{
    if constexpr (sizeof(TD) == 2)
        if (v == 8) return launch_direct<TD, 8, 1>(s, d, st);
    if (v >= 4) return launch_direct<TD, 4, 1>(s, d, st);
    if (v == 2) return launch_direct<TD, 2, 2>(s, d, st);
    return launch_direct<TD, 1, 2>(s, d, st);
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
    e->pitch = (q.dim + 7) / 8 * 8;
    if (q.max_tokens > kDirectTokens) {
        const int64_t total = q.n * q.max_tokens;
        const bool sorts = q.max_tokens > (int64_t)kOrderCluster * kOrderMost;
        // batches of every size up to the largest have to fit, in tiles of any length
        const int64_t few = std::min(total, kShortRows), mid = std::min(total, kMidRows);
        const int64_t tiles = std::max({(q.max_tokens + kTileLong - 1) / kTileLong * q.n, mid / kTileMid + q.n, few / kTileShort + q.n});
        e->chain_room = (uint32_t)tiles;
        int64_t bytes = 0;
        auto place = [&](auto** ptr, int64_t count) { // the second time around, when the memory is there
            if (e->memory) *ptr = reinterpret_cast<std::remove_reference_t<decltype(*ptr)>>(static_cast<char*>(e->memory) + bytes);
            bytes += (count * (int64_t)sizeof(**ptr) + 255) / 256 * 256;
        };
        for (int round = 0; round < 2 && err == cudaSuccess; ++round) {
            bytes = 0;
            place(&e->key[0], total);
            place(&e->pos[0], total);
            place(&e->part, tiles * 2 * e->pitch);
            place(&e->chains, tiles + 2);
            if (sorts) {
                place(&e->key[1], total);
                place(&e->pos[1], total);
                place(&e->hist, q.n * kDigits * ((q.max_tokens + kSortTile - 1) / kSortTile));
                place(&e->total, (int64_t)q.n * kDigits);
            }
            if (round == 0 && err == cudaSuccess) err = cudaMalloc(&e->memory, (size_t)bytes);
        }
        if (err == cudaSuccess) err = allow_order();
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
    if (count > 0 && rows_overlap(emb->p.n, count, emb->p.dim, out_ld, out_row)) return CHOCO_ERR_INVALID_ARG;
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
            auto launch = [&](auto vec, auto vectors) {
                constexpr int V = decltype(vec)::value, N = decltype(vectors)::value;
                uint32_t lanes_log = 5;
                while (lanes_log > 2 && ((int64_t)V * N << (lanes_log - 1)) >= s.dim) --lanes_log;
                auto* kernel = lanes_log < 5 ? lookup_kernel<TT, TO, V, N, true> : lookup_kernel<TT, TO, V, N, false>;
                const int64_t slabs = (s.dim + 32 * V * N - 1) / (32 * V * N), per_block = (int64_t)kEmbWarps << (5 - lanes_log);
                const int64_t rows_a_warp = lanes_log < 5 ? 1 : lookup_rows<TT, V, N>();
                const int64_t blocks = ((count + rows_a_warp - 1) / rows_a_warp * slabs + per_block - 1) / per_block;
                if (blocks > 0x1fffffff) return (int)CHOCO_ERR_TOO_LARGE; // (more than the output can have in memory)
                return status_of(launch_overlapped(kernel, dim3((unsigned)blocks, (unsigned)s.n), dim3(kEmbThreads), 0,
                                                   st, HotRange{}, s, static_cast<const TT*>(table), tokens, index_bits, tokens_ld,
                                                   static_cast<TO*>(out), out_row, out_ld, (uint32_t)slabs, lanes_log));
            };
            // 4 or 6 vectors a lane, whichever leaves fewer of them idle
            auto go = [&](auto vec) {
                constexpr int V = decltype(vec)::value;
                auto idle = [&](int64_t cols) { return (s.dim + cols - 1) / cols * cols - s.dim; };
                if (s.dim > 32 * V * 4 && idle(32 * V * 6) < idle(32 * V * 4)) return launch(vec, std::integral_constant<int, 6>());
                return launch(vec, std::integral_constant<int, 4>());
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
    if (count > 0 && (!dout || (dout_row < emb->p.dim && dout_row != 0) || (emb->p.n > 1 && dout_ld < 0))) return CHOCO_ERR_INVALID_ARG;
    if (!aligned_to(grad, dtype_size(grad_dtype)) || !aligned_to(dout, dtype_size(dout_dtype))) return CHOCO_ERR_MISALIGNED;
    if (count == 0 && accumulate) return CHOCO_OK;
    const EmbShape s = shape_of(emb, count);
    cudaStream_t st = (cudaStream_t)stream;
    const int v = std::min(vector_of(dout, dout_dtype, dout_row, dout_ld, s.dim, s.n, 8),
                           vector_of(grad, grad_dtype, s.table_row, s.table_ld, s.dim, s.n, 8));
    cudaError_t err = cudaSuccess;

    // every launch's size is known, and refused if it is too large, before the first goes out
    const int32_t size = (int32_t)dtype_size(grad_dtype);
    const int64_t per_row = (s.dim * size + kZeroSpan - 1) / kZeroSpan;
    const int64_t zero_blocks = s.table_row == s.dim ? (s.vocab * s.dim * size + kZeroSpan - 1) / kZeroSpan : s.vocab * per_row;
    // (no form of the sums has a warp take fewer than 64 columns)
    const int64_t tiles = (count + tile_of(count * s.n) - 1) / tile_of(count * s.n);
    if ((!accumulate && zero_blocks > 0x7fffffff) || (s.dim + 63) / 64 * tiles * s.n > 0x7fffffffLL * (kSumThreads / 32)) return CHOCO_ERR_TOO_LARGE;
    auto zero = [&](int32_t beside) {
        if (accumulate || err != cudaSuccess) return;
        err = launch_overlapped(zero_kernel, dim3((unsigned)zero_blocks, (unsigned)s.n), dim3(kEmbThreads), 0, st, HotRange{}, s,
                                static_cast<char*>(grad), size, (uint32_t)per_row, beside);
    };
    if (count <= kDirectTokens) {
        const bool apart = !accumulate && s.n * s.vocab * s.dim * dtype_size(grad_dtype) > kDirectZeroBytes;
        if (apart) zero(0);
        const Direct d = {tokens, tokens_ld, index_bits, dout, dout_row, dout_ld, grad, grad_dtype, accumulate, 0, 0,
                          accumulate || apart ? 0 : (s.vocab + 7) / 8, 0};
        if (err == cudaSuccess && (count > 0 || d.eights > 0))
            with_type(dout_dtype, [&](auto* td) {
                err = launch_direct_for<std::remove_pointer_t<decltype(td)>>(s, d, v, st);
                return 0;
            });
        return status_of(err);
    }

    const dim3 threads(kEmbThreads);
    int cur = 0;
    Order o = {};
    if (plan_order(s, o)) {
        o.tokens = tokens; o.tokens_ld = tokens_ld; o.index_bits = index_bits;
        o.keys = emb->key[0]; o.pos = emb->pos[0];
        o.chain_count = emb->chains;
        err = launch_order(s, o, st);
        zero(1);
    } else {
        SortPass p = {};
        p.tokens = tokens; p.tokens_ld = tokens_ld; p.index_bits = index_bits;
        p.tiles = (int32_t)((count + kSortTile - 1) / kSortTile);
        p.hist = emb->hist;
        p.total = emb->total;
        p.chain_count = emb->chains;
        p.first = 1;
        zero(0);
        for (p.shift = 0; p.shift == 0 || (s.vocab >> p.shift) != 0; p.shift += kDigitBits) {
            p.key_in = emb->key[cur]; p.pos_in = emb->pos[cur];
            p.key_out = emb->key[cur ^ 1]; p.pos_out = emb->pos[cur ^ 1];
            const unsigned tiles = (unsigned)(p.tiles * s.n), digits = (unsigned)(s.n * (kDigits / kEmbWarps));
            if (err == cudaSuccess) err = launch_overlapped(sort_count_kernel, dim3(tiles), threads, 0, st, HotRange{}, s, p);
            if (err == cudaSuccess) err = launch_overlapped(sort_scan_kernel, dim3(digits), threads, 0, st, HotRange{}, s, p);
            if (err == cudaSuccess) err = launch_overlapped(sort_scatter_kernel, dim3(tiles), threads, 0, st, HotRange{}, s, p);
            p.first = 0;
            cur ^= 1;
        }
    }
    Sums a = {};
    a.keys = emb->key[cur]; a.pos = emb->pos[cur];
    a.dout = dout; a.dout_row = dout_row; a.dout_ld = dout_ld;
    a.grad = grad; a.grad_dtype = grad_dtype; a.accumulate = accumulate;
    a.part = emb->part; a.pitch = emb->pitch;
    a.chains = emb->chains + 2; a.chain_room = emb->chain_room; a.chain_count = emb->chains;
    a.tile = tile_of(count * s.n);
    a.tiles = (int32_t)((count + a.tile - 1) / a.tile);
    if (err == cudaSuccess)
        with_type(dout_dtype, [&](auto* td) {
            err = launch_sums_for<std::remove_pointer_t<decltype(td)>>(s, a, v, st);
            return 0;
        });
    if (err == cudaSuccess) {
        const uint32_t slabs = (uint32_t)((s.dim + kJoinCols - 1) / kJoinCols);
        // a resident grid: how many chains there are is known on the device only
        const int64_t blocks = std::min<int64_t>((int64_t)a.tiles * s.n * slabs, kJoinBlocks);
        err = launch_overlapped(v >= 4 ? join_kernel<4> : v == 2 ? join_kernel<2> : join_kernel<1>, dim3((unsigned)blocks), threads, 0, st,
                                HotRange{}, s, a, slabs);
    }
    return status_of(err);
}

} // extern "C"
