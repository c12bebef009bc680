// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   forward    out[t, :] = rn(fl(scale * W[id_t, :]))        0 where id_t is not in [0, rows)
//   backward   dW[v, :] = rn(fl([dW[v, :] +] scale * sum over t with id_t = v of dY[t, :]))
//
// fl rounds to fp32, rn to the stored type.
//
// The backward pass sorts the tokens by id (stable, so a row's tokens keep their order), then
// adds each row's tokens in an order fixed by the ids alone, in fp32.  No element is the target of
// two additions whose order could differ: results are bit-reproducible.
//
// Both are bound by their bytes where there are many tokens (128k x 4096 bf16: lookup 223 us of
// 202 at the measured copy rate; gradient into 32000 rows 229 us of 196, 13 of them the sort that nothing
// overlaps), and by launches and dependent round trips where there are few.
#include "came_ops.cuh"

#include <cooperative_groups.h>

#include <algorithm>

namespace cg = cooperative_groups;

namespace {

using namespace came_ops;

constexpr int kSlice = 256;              // columns one warp works on: 8 per lane

// EV consecutive elements as they are stored: one access of EV * sizeof(T) bytes.  (Volatile, so
// that the loads of a batch stay together in front of what uses them.)
template <int EV, typename T>
struct Raw {
    static constexpr int B = EV * static_cast<int>(sizeof(T));
    static constexpr int W = B < 4 ? 1 : B / 4;
    uint32_t w[W];

    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (B == 32) {
            asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]),
                           "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
        } else if constexpr (B == 16) {
            asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
        } else if constexpr (B == 8) {
            asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
        } else if constexpr (B == 4) {
            asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
        } else {
            uint16_t h;
            asm volatile("ld.global.b16 %0, [%1];" : "=h"(h) : "l"(p));
            w[0] = h;
        }
    }

    // acc[k] += element k: for bf16 the addition that widens one operand, without unpacking
    __device__ __forceinline__ void add_to(float* acc) const
    {
#pragma unroll
        for (int k = 0; k < EV; ++k) {
            if constexpr (sizeof(T) == 4) {
                acc[k] += __uint_as_float(w[k]);
            } else {
                const uint16_t h = static_cast<uint16_t>(k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xffffu);
                asm("add.rn.f32.bf16 %0, %1, %0;" : "+f"(acc[k]) : "h"(h));
            }
        }
    }

    __device__ __forceinline__ float value(int k) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
        else return __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
    }
};

// kStream: marked as first to leave the L2.
template <int EV, bool kStream = false, typename T>
__device__ __forceinline__ void store_ev(T* p, const float* x)
{
    constexpr int B = EV * static_cast<int>(sizeof(T));
    if constexpr (B >= 4) {
        constexpr int W = B / 4;
        uint32_t w[W];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(x[j]);
            else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(x[2 * j + 1]), "f"(x[2 * j]));
        }
        if constexpr (W == 8 && kStream)
            asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                         :: "l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                            "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
        else if constexpr (W == 8)
            asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                         :: "l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                            "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
        else if constexpr (W == 4 && kStream) __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
        else if constexpr (W == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (W == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    } else {
        *p = from_float<T>(x[0]);
    }
}

// p[k] += x[k], EV consecutive fp32
template <int EV>
__device__ __forceinline__ void reduce_ev(float* p, const float* x)
{
    if constexpr (EV >= 4) {
#pragma unroll
        for (int k = 0; k < EV; k += 4)
            asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};"
                         :: "l"(p + k), "f"(x[k]), "f"(x[k + 1]), "f"(x[k + 2]), "f"(x[k + 3]) : "memory");
    } else if constexpr (EV == 2) {
        asm volatile("red.global.add.v2.f32 [%0], {%1, %2};" :: "l"(p), "f"(x[0]), "f"(x[1]) : "memory");
    } else {
        asm volatile("red.global.add.f32 [%0], %1;" :: "l"(p), "f"(x[0]) : "memory");
    }
}

// A lane's eight columns of a slice: 8 / EV groups of EV, 32 * EV columns apart.
template <int EV>
__device__ __forceinline__ long long column(long long slice, int group, int lane)
{
    return slice * kSlice + group * (32 * EV) + lane * EV;
}

// ---- forward --------------------------------------------------------------------------------

// A warp copies S slices of one token's row: S rows' pieces in flight per lane.  Bound by the bytes:
// 128k tokens of 4096 bf16 take 229 / 241 / 338 us with 4 / 2 / 1 slices per warp; rows of one slice, and rows that
// go in accesses below 16 bytes, are faster with one (60000 rows of 1001 bf16: 48 against 145 us).
// stream: the output is larger than the L2 can hold for its reader anyway, so it leaves the
// table's rows there (223 instead of 229 us).
template <typename I, typename T, typename O, int EV, int S>
__global__ void __launch_bounds__(256)
k_embed_forward(const T* __restrict__ table, long long rows, int cols, long long table_ld, const I* __restrict__ ids,
                unsigned tokens, float scale, O* __restrict__ out, long long out_ld, unsigned warps_per_token, int stream)
{
    const unsigned item = blockIdx.x * 8u + (threadIdx.x >> 5);
    const unsigned t = S == 1 && warps_per_token == 1 ? item : item / warps_per_token;
    if (t >= tokens) return;
    const int lane = threadIdx.x & 31;
    const int first = static_cast<int>(item - t * warps_per_token) * (S * kSlice) + lane * EV;
    const long long id = static_cast<long long>(ids[t]);
    const bool hit = id >= 0 && id < rows;
    const T* const src = table + (hit ? id : 0) * table_ld;
    O* const dst = out + t * out_ld;
    Raw<EV, T> x[S][8 / EV];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int g = 0; g < 8 / EV; ++g) {
            const int c = first + s * kSlice + g * (32 * EV);
            if (hit && c < cols) x[s][g].load(src + c);
        }
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int g = 0; g < 8 / EV; ++g) {
            const int c = first + s * kSlice + g * (32 * EV);
            if (c >= cols) continue;
            float y[EV];
#pragma unroll
            for (int k = 0; k < EV; ++k) y[k] = hit ? x[s][g].value(k) * scale : 0.f;
            if (stream) store_ev<EV, true>(dst + c, y);
            else        store_ev<EV>(dst + c, y);
        }
}

// ---- backward: stable sort of the tokens by row ----------------------------------------------
// Least significant digit first.  A warp owns a contiguous run of the input; per digit it knows how
// many equal digits come before its run (in its block: a count per warp and digit; in the grid:
// the blocks' counts; over all digits: a scan), so every element's place is known and nothing
// depends on the order in which atomics arrive.  Ids that are not rows (and the padding row) get the
// key `rows` and end up behind all others.
//
// Four ways by the number of tokens, each launched alone: up to kTinyTokens (below) inside the
// sums' grid; up to kFewTokens 2.0 us; up to kOneTokens one block, 7 us at 2048 and 10 at 4096 tokens; beyond
// that three to five short grids, 14 us at 8192 and 16384 and 23 at 131072 tokens.  Bound by the
// latency of their dependent steps.  (One cluster of eight blocks took 61 us at 131072 tokens: scattered
// stores go one lane per cycle and SM.  Blocks that count all tokens themselves instead of the
// counting grid: 44 instead of 36 us for the whole gradient at 16384 tokens.  kOneTokens 2048: 20.4
// instead of 17.2 us for the whole gradient at 3000.)
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxDigitBits = 9;
constexpr int kMaxBins = 1 << kMaxDigitBits;
constexpr int kMaxPasses = 4;            // keys below 2^31 in digits of 8 bits
constexpr int kFewTokens = 512;          // every token counts the tokens before it
constexpr unsigned kFewRows = 1u << 22;  // (key and position then fit one word)
constexpr int kOneTokens = 4096;         // one block sorts in its shared memory
constexpr int kMoveThreads = 512;        // a grid of blocks that leave room for the zeroing ones on their SM
constexpr int kMoveWarps = kMoveThreads / 32;
constexpr int kMoveTile = 512;           // tokens per block, or a multiple of it ...
constexpr int kMoveBlocks = 148;         // ... so that there are no more blocks than SMs
constexpr size_t kHistBytes = sizeof(unsigned) * kSortWarps * kMaxBins;
constexpr size_t kOneBytes = kHistBytes + sizeof(uint2) * kOneTokens;

struct SortArgs {
    uint2*    pair[2];       // (key, token) ping-pong buffers [tokens]; the result is in the first
    unsigned* count[kMaxPasses];     // [blocks][bins] digits of each pass in each block's part of its input
    unsigned* arrived;       // [n_arrived] counters of the sums' grid, cleared here
    long long tokens, n_arrived;
    unsigned  rows, padding; // padding: its own row, or rows when there is none
    unsigned  tile;          // tokens per block of the counting and moving grids
    int       digit_bits, passes, blocks;
};

// Exclusive sum over the block's WARPS warps; `totals` has room for a warp.
template <int WARPS>
__device__ __forceinline__ unsigned block_exclusive_scan(unsigned v, unsigned* totals)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto warp_scan = [&](unsigned x) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned u = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += u;
        }
        return x;
    };
    const unsigned s = warp_scan(v);
    if (lane == 31) totals[warp] = s;
    __syncthreads();
    const unsigned t = lane < WARPS ? totals[lane] : 0u, upto = warp_scan(t);
    return __shfl_sync(0xffffffffu, upto - t, warp) + s - v;
}

template <typename I>
__device__ __forceinline__ unsigned key_of(I id, const SortArgs& a)
{
    const long long v = static_cast<long long>(id);
    return (v >= 0 && v < a.rows && v != a.padding) ? static_cast<unsigned>(v) : a.rows;
}

// The lanes of `in` whose digit equals this lane's: one vote per bit of the digit.  (The match
// instruction takes its time for every distinct value; votes take the same for all data.)
__device__ __forceinline__ unsigned lanes_with(unsigned digit, unsigned in, int bits)
{
    unsigned m = in;
#pragma unroll
    for (int b = 0; b < kMaxDigitBits; ++b) {
        if (b >= bits) break;
        const bool one = digit >> b & 1u;
        const unsigned v = __ballot_sync(0xffffffffu, one);
        m &= one ? v : ~v;
    }
    return m;
}

// Number of equal digits before this lane's element in the warp's run, which `counts` holds for
// the elements before these 32; adds these 32 to it.  The whole warp calls.
__device__ __forceinline__ unsigned rank_and_count(unsigned digit, bool in, int bits, unsigned* counts)
{
    const unsigned peers = lanes_with(digit, __ballot_sync(0xffffffffu, in), bits);
    const unsigned before = __popc(peers & ((1u << (threadIdx.x & 31)) - 1u));
    const unsigned sum = in ? counts[digit] : 0u;
    __syncwarp();
    if (in && before == 0) counts[digit] = sum + __popc(peers);
    __syncwarp();
    return sum + before;
}

// hist[warp][digit] becomes the count in the warps before; returns the block's count of digit tid.
template <int WARPS>
__device__ __forceinline__ unsigned sum_over_warps(unsigned* hist, int bins)
{
    unsigned s = 0;
    if (static_cast<int>(threadIdx.x) < bins) {
        unsigned v[WARPS];
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v[w] = hist[w * bins + threadIdx.x];
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            hist[w * bins + threadIdx.x] = s;
            s += v[w];
        }
    }
    return s;
}

// Up to kFewTokens tokens: the place of a token is the number of tokens that sort before it.
template <typename I>
__global__ void __launch_bounds__(kFewTokens)
k_embed_sort_few(const I* __restrict__ ids, SortArgs a)
{
    __shared__ __align__(16) unsigned word[kFewTokens];
    release_dependents();
    const unsigned t = threadIdx.x, n = static_cast<unsigned>(a.tokens);
    for (long long k = t; k < a.n_arrived; k += kFewTokens) a.arrived[k] = 0u;
    const unsigned mine = t < n ? key_of(ids[t], a) << 9 | t : 0xffffffffu;
    word[t] = mine;
    __syncthreads();
    if (t >= n) return;
    unsigned before = 0;
    for (unsigned j = 0; j < n; j += 4) {                // words behind the last token are all ones
        const uint4 w = *reinterpret_cast<const uint4*>(word + j);
        before += (w.x < mine) + (w.y < mine) + (w.z < mine) + (w.w < mine);
    }
    a.pair[0][before] = make_uint2(mine >> 9, t);
}

// Up to kOneTokens tokens: one block, the elements stay in registers and shared memory.
template <typename I>
__global__ void __launch_bounds__(kSortThreads)
k_embed_sort_one(const I* __restrict__ ids, SortArgs a)
{
    constexpr int kRounds = kOneTokens / kSortThreads;
    extern __shared__ __align__(16) unsigned hist[];     // [warp][digit], then the elements
    uint2* const s_pair = reinterpret_cast<uint2*>(hist + kSortWarps * kMaxBins);
    __shared__ unsigned base[kMaxBins], scan_totals[32];
    release_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n = static_cast<int>(a.tokens), bins = 1 << a.digit_bits;
    for (long long k = tid; k < a.n_arrived; k += kSortThreads) a.arrived[k] = 0u;
    const int per = (n + kSortThreads - 1) / kSortThreads * 32;
    const int begin = min(n, warp * per), end = min(n, begin + per);
    unsigned* const mine = hist + warp * bins;
    uint2 pair[kRounds];
    unsigned rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int k = begin + r * 32 + lane;
        pair[r] = make_uint2(k < end ? key_of(ids[k], a) : 0u, static_cast<unsigned>(k));
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.digit_bits;
        if (pass > 0) {
#pragma unroll
            for (int r = 0; r < kRounds; ++r) {
                const int k = begin + r * 32 + lane;
                if (k < end) pair[r] = s_pair[k];
            }
        }
        for (int k = lane; k < bins; k += 32) mine[k] = 0u;
        __syncwarp();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (begin + r * 32 >= end) break;
            rank[r] = rank_and_count(pair[r].x >> shift & (bins - 1), begin + r * 32 + lane < end, a.digit_bits, mine);
        }
        __syncthreads();
        const unsigned first = block_exclusive_scan<kSortWarps>(sum_over_warps<kSortWarps>(hist, bins), scan_totals);
        if (tid < bins) base[tid] = first;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (begin + r * 32 + lane >= end) break;
            const unsigned digit = pair[r].x >> shift & (bins - 1);
            s_pair[base[digit] + mine[digit] + rank[r]] = pair[r];
        }
        __syncthreads();
    }
    for (int k = tid; k < n; k += kSortThreads) a.pair[0][k] = s_pair[k];
}

// More tokens: a counting grid, then one moving grid per digit.  Block b has the tokens (in the
// order of the pass's input) from b * tile on.
template <typename I>
__global__ void __launch_bounds__(kMoveThreads)
k_embed_count(const I* __restrict__ ids, SortArgs a)
{
    __shared__ unsigned count[kMaxBins];
    release_dependents();
    const int tid = threadIdx.x, bins = 1 << a.digit_bits;
    const long long at = static_cast<long long>(blockIdx.x) * kMoveThreads + tid;
    const long long all = static_cast<long long>(a.blocks) * kMoveThreads;
    for (long long k = at; k < a.n_arrived; k += all) a.arrived[k] = 0u;
    // the moving grids count the digits of the pass after theirs
    for (int pass = 1; pass < a.passes; ++pass)
        for (int k = tid; k < bins; k += kMoveThreads) a.count[pass][static_cast<long long>(blockIdx.x) * bins + k] = 0u;
    if (tid < bins) count[tid] = 0u;
    __syncthreads();
    const long long begin = static_cast<long long>(blockIdx.x) * a.tile, end = min(a.tokens, begin + a.tile);
#pragma unroll 4
    for (long long k = begin + tid; k < end; k += kMoveThreads) atomicAdd(&count[key_of(ids[k], a) & (bins - 1)], 1u);
    __syncthreads();
    if (tid < bins) a.count[0][static_cast<long long>(blockIdx.x) * bins + tid] = count[tid];
}

template <typename I>
__global__ void __launch_bounds__(kMoveThreads)
k_embed_move(const I* __restrict__ ids, SortArgs a, int pass)
{
    constexpr int kRounds = 4;                           // elements per lane that are loaded at once
    extern __shared__ __align__(16) unsigned hist[];     // [warp][digit]
    __shared__ uint4 sum_before[kMoveThreads], sum_all[kMoveThreads];      // [part of the blocks][digits]
    __shared__ unsigned base[kMaxBins], scan_totals[32];
    release_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int bins = 1 << a.digit_bits, shift = pass * a.digit_bits, me = static_cast<int>(blockIdx.x);
    const int to_buffer = (a.passes - 1 - pass) & 1;
    const uint2* const src = a.pair[to_buffer ^ 1];
    uint2* const dst = a.pair[to_buffer];
    const long long per = a.tile / kMoveWarps;
    const long long begin = min(a.tokens, static_cast<long long>(me) * a.tile + warp * per);
    const long long end = min(a.tokens, begin + per);
    unsigned* const mine = hist + warp * bins;
    for (int k = lane; k < bins; k += 32) mine[k] = 0u;
    wait_for_previous_grid();
    uint2 pair[kRounds];
    unsigned rank[kRounds];
    auto load = [&](long long at) {
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const long long k = at + r * 32 + lane;
            if (k < end) pair[r] = pass > 0 ? __ldcg(src + k) : make_uint2(key_of(ids[k], a), static_cast<unsigned>(k));
            else pair[r] = make_uint2(0u, 0u);
        }
    };
    auto count_ranks = [&](long long at) {
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (at + r * 32 >= end) break;
            rank[r] = rank_and_count(pair[r].x >> shift & (bins - 1), at + r * 32 + lane < end, a.digit_bits, mine);
        }
    };
    const bool kept = per <= 32 * kRounds;               // a warp's run fits its registers
    load(begin);
    // four neighbouring digits per thread: all of them, and what the blocks before this one have
    {
        const int quads = bins >> 2, quad = tid & (quads - 1), step = kMoveThreads / quads;
        const uint4* const count = reinterpret_cast<const uint4*>(a.count[pass]) + quad;
        uint4 before = make_uint4(0u, 0u, 0u, 0u), all = before;
#pragma unroll 8
        for (int b = tid / quads; b < a.blocks; b += step) {
            const uint4 v = __ldcg(count + static_cast<long long>(b) * quads);
            all.x += v.x; all.y += v.y; all.z += v.z; all.w += v.w;
            if (b < me) { before.x += v.x; before.y += v.y; before.z += v.z; before.w += v.w; }
        }
        sum_before[tid] = before;
        sum_all[tid] = all;
    }
    __syncwarp();
    for (long long at = begin; at < end; at += 32 * kRounds) {
        if (at > begin) load(at);
        count_ranks(at);
    }
    __syncthreads();
    sum_over_warps<kMoveWarps>(hist, bins);
    unsigned before = 0, all = 0;
    if (tid < bins)
#pragma unroll 8
        for (int k = tid; k < 4 * kMoveThreads; k += bins) {
            before += reinterpret_cast<const unsigned*>(sum_before)[k];
            all += reinterpret_cast<const unsigned*>(sum_all)[k];
        }
    const unsigned first = block_exclusive_scan<kMoveWarps>(all, scan_totals);
    if (tid < bins) base[tid] = first + before;
    __syncthreads();
    for (long long at = begin; at < end; at += 32 * kRounds) {
        if (!kept) {                                     // counts go on from what the warps before have
            load(at);
            count_ranks(at);
        }
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (at + r * 32 + lane >= end) break;
            const unsigned digit = pair[r].x >> shift & (bins - 1);
            const unsigned to = base[digit] + rank[r] + (kept ? mine[digit] : 0u);
            dst[to] = pair[r];
            if (pass + 1 < a.passes)
                atomicAdd(&a.count[pass + 1][static_cast<long long>(to / a.tile) * bins + (pair[r].x >> (shift + a.digit_bits) & (bins - 1))], 1u);
        }
    }
}

// ---- backward: the sums ----------------------------------------------------------------------------
// A block takes 8 * per_warp consecutive sorted tokens and one slice of the columns, a warp
// per_warp of them: however many tokens a row has, the work is even.  A run of equal keys that
// begins and ends within a warp is stored at once.  A part of a run that crosses warps goes
// through shared memory to the warp in which the run ends; one that crosses blocks goes to
// the workspace, and the block that arrives last for that run adds the parts in order.
//
// The first zero_blocks blocks write the rows without tokens instead.  They need the ids only, so
// they do not wait for the sort: the zeros are written while it runs.
//
// What bounds it: the bytes at 128k tokens (5.7 TB/s of them in the whole grid); a row of one token costs
// a warp about 40 instructions per 512 bytes, so it needs the 32 warps per SM that 64 registers allow
// (24 or 16 warps: 238 and 255 instead of 229 us).  Copies into a ring in shared memory instead of the two
// batches in registers: 247 us, more instructions and fewer warps.
constexpr int kSumWarps = 8;
constexpr int kTinyTokens = 64;          // one block's: no run crosses blocks, and it sorts for itself
// 64 clusters: with 32 the zeroing blocks were packed onto half of the SMs (128256 rows of 4096 fp32, 8192
// tokens: 467 instead of 355 us), with 128 the marking shows (32000 rows, 131072 tokens: 286 instead of 229).
constexpr int kClusterBlocks = 8, kZeroClusters = 64, kZeroBlocks = kClusterBlocks * kZeroClusters;
constexpr int kZeroWords = 2048;         // of the bit map: 65536 of a cluster's rows per round
enum : int { kLinkHead = 1, kLinkTail = 2, kLinkThrough = 4 };

struct SumArgs {
    const uint2* pair;         // sorted (key, token) [tokens]
    float*    part;            // [blocks of tokens][2][slices][kSlice]: 0 = run from before, 1 = run that goes on
    unsigned* arrived;         // [blocks of tokens][slices]
    const void* ids;
    long long tokens, cols, grad_ld;
    unsigned  dy_bytes;        // from row to row of dY
    unsigned  rows, padding;
    int       slices, per_warp, accumulate, id64;
    int       tiny;            // up to kTinyTokens: every block sorts the ids for itself
    int       zero_blocks;     // 0 or kZeroBlocks
    int       zero_group;      // log2 of the neighbouring rows a cluster takes at once
    unsigned  sum_blocks;      // the grid is rounded up to whole clusters
    float     scale;
};

template <typename O, int EV>
__device__ __forceinline__ void store_row(const SumArgs& a, O* grad, unsigned row, int slice, int lane, const float (&sum)[8])
{
    O* const dst = grad + static_cast<long long>(row) * a.grad_ld;
#pragma unroll
    for (int g = 0; g < 8 / EV; ++g) {
        const long long c = column<EV>(slice, g, lane);
        if (c >= a.cols) continue;
        float y[EV];
#pragma unroll
        for (int k = 0; k < EV; ++k) y[k] = a.scale * sum[g * EV + k];
        if (a.accumulate) {
            if constexpr (sizeof(O) == 4) {
                // The only addition to these elements in the whole call, so its order cannot matter;
                // done in the L2, it keeps the warp from waiting for the old value.  (That addition takes
                // subnormal inputs and results as zero.)
                reduce_ev<EV>(dst + c, y);
                continue;
            } else {
                Raw<EV, O> old;
                old.load(dst + c);
#pragma unroll
                for (int k = 0; k < EV; ++k) y[k] += old.value(k);
            }
        }
        store_ev<EV>(dst + c, y);
    }
}

// One block's part of a run that crosses blocks.  The last of the run's blocks to arrive adds
// all parts in the order of the tokens and stores the row.  begins / ends: the run does so here.
template <typename O, int EV>
__device__ __forceinline__ void join_blocks(const SumArgs& a, O* grad, unsigned row, int block, bool begins, bool ends,
                                            int slice, int lane, const float (&sum)[8])
{
    const int size = kSumWarps * a.per_warp;
    auto at = [&](int b, int s) {
        return a.part + ((static_cast<long long>(b) * 2 + s) * a.slices + slice) * kSlice + lane; };
    float* const mine = at(block, begins ? 1 : 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) __stcg(mine + j * 32, sum[j]);
    // the run's first and last block: 32 blocks' borders are looked at at once
    int first = block, last = block;
    while (!begins) {
        const int b = first - 1 - lane;                  // the run reaches back into block first - 1
        const bool here = b <= 0 || __ldcg(&a.pair[static_cast<long long>(b) * size - 1].x) != row;
        const unsigned found = __ballot_sync(0xffffffffu, here);
        first -= found ? __ffs(found) : 32;
        begins = found != 0;
    }
    while (!ends) {
        const int b = last + 1 + lane;
        const long long next = (static_cast<long long>(b) + 1) * size;
        const bool here = next >= a.tokens || __ldcg(&a.pair[next].x) != row;
        const unsigned found = __ballot_sync(0xffffffffu, here);
        last += found ? __ffs(found) : 32;
        ends = found != 0;
    }
    // The warp's parts are ordered before lane 0's fence, and with it before its arrival; what the others
    // have published, behind it, before the warp's reads.  (A shuffle orders no memory.)
    __syncwarp();
    unsigned final = 0;
    if (lane == 0) {
        publish();
        final = atomicAdd(&a.arrived[static_cast<long long>(first) * a.slices + slice], 1u) == static_cast<unsigned>(last - first);
        publish();
    }
    final = __shfl_sync(0xffffffffu, final, 0);
    __syncwarp();
    if (!final) return;
    float total[8];
    {
        const float* const p = at(first, 1);
#pragma unroll
        for (int j = 0; j < 8; ++j) total[j] = __ldcg(p + j * 32);
    }
    for (int b = first + 1; b <= last; b += 4) {
        float x[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float* const p = at(b + u, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[u][j] = b + u <= last ? __ldcg(p + j * 32) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) total[j] += x[u][j];
    }
    store_row<O, EV>(a, grad, row, slice, lane, total);
}

// Cluster c of kZeroClusters takes every kZeroClusters-th group of 2^group rows (frequent ids are
// neighbours in most vocabularies: this spreads them).  Its blocks share the reading of the ids: each
// marks what its part of them touches in a bit map of the cluster's rows, then takes the
// rows that no block has marked, every kClusterBlocks-th group of them, and zeroes them.
//   cluster = (r >> group) mod kZeroClusters,   bit = (r >> group) / kZeroClusters << group | r mod 2^group
// (Every block reading all ids for itself cost 70 us at 131072 tokens.)
template <typename I, typename O, int EV>
__device__ __forceinline__ void zero_rows(const I* __restrict__ ids, O* __restrict__ grad, const SumArgs& a, unsigned* seen)
{
    constexpr int kPer = 16 / static_cast<int>(sizeof(I)), kBatch = 4;       // 16-byte loads, four at a time
    constexpr int kThreads = kSumWarps * 32;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, me = static_cast<int>(cluster.block_rank()), group = a.zero_group;
    const unsigned own = blockIdx.x / kClusterBlocks;
    const unsigned inner = (1u << group) - 1u, mine = own << group, filter = (kZeroClusters - 1u) << group;
    // bits up to the last group of this cluster; rows behind the table's end are left out below
    const unsigned groups = ((a.rows - 1u) >> group) + 1u;
    const unsigned bits = own < groups ? ((groups - 1u - own) / kZeroClusters + 1u) << group : 0u;
    // the ids from the first 16-byte boundary on go in whole loads, the others one by one
    const long long lead = min(a.tokens, static_cast<long long>((16 - reinterpret_cast<uintptr_t>(ids) % 16) % 16 / sizeof(I)));
    const long long whole = (a.tokens - lead) / kPer;
    const uint4* const packs = reinterpret_cast<const uint4*>(ids + lead);
    const int per_row = EV * 32 <= a.cols ? 32 : 1 << (32 - __clz(static_cast<int>((a.cols + EV - 1) / EV - 1)));  // lanes
    const float zeros[EV] = {};
    for (unsigned first = 0; first < bits; first += kZeroWords * 32u) {
        const unsigned count = min(bits - first, kZeroWords * 32u);
        for (unsigned k = tid; k < (count + 31u) / 32u; k += kThreads) seen[k] = 0u;
        __syncthreads();
        auto mark = [&](I raw) {
            if ((static_cast<unsigned>(raw) & filter) != mine) return;
            const long long id = static_cast<long long>(raw);
            if (id < 0 || id >= a.rows || id == a.padding) return;
            const unsigned r = static_cast<unsigned>(id), bit = ((r >> group) / kZeroClusters << group | (r & inner)) - first;
            if (bit < count && !(seen[bit >> 5] >> (bit & 31u) & 1u)) atomicOr(&seen[bit >> 5], 1u << (bit & 31u));
        };
        for (long long k = me * kThreads + tid; k < whole; k += kBatch * kClusterBlocks * kThreads) {
            uint4 w[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const long long q = k + u * (kClusterBlocks * kThreads);
                w[u] = q < whole ? packs[q] : make_uint4(~0u, ~0u, ~0u, ~0u);            // -1: no row
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if constexpr (sizeof(I) == 4) {
                    mark(static_cast<I>(w[u].x)); mark(static_cast<I>(w[u].y));
                    mark(static_cast<I>(w[u].z)); mark(static_cast<I>(w[u].w));
                } else {
                    mark(static_cast<I>(static_cast<unsigned long long>(w[u].y) << 32 | w[u].x));
                    mark(static_cast<I>(static_cast<unsigned long long>(w[u].w) << 32 | w[u].z));
                }
            }
        }
        if (me == 0 && tid < lead) mark(ids[tid]);
        const long long rest = lead + whole * kPer + tid;
        if (me == 0 && rest < a.tokens) mark(ids[rest]);
        cluster.sync();
        // every block's marks together
        constexpr int kWords = kZeroWords / kThreads;
        unsigned m[kWords] = {};
#pragma unroll
        for (int q = 0; q < kWords; ++q)
            if (tid + q * kThreads < static_cast<int>((count + 31u) / 32u))
#pragma unroll
                for (int b = 0; b < kClusterBlocks; ++b) m[q] |= cluster.map_shared_rank(seen, b)[tid + q * kThreads];
        cluster.sync();                                  // nobody overwrites, clears or leaves before all have read
#pragma unroll
        for (int q = 0; q < kWords; ++q) seen[tid + q * kThreads] = m[q];
        __syncthreads();
        const int rows_at_once = 32 / per_row;           // a warp's, where rows are shorter than its store
        for (unsigned k = static_cast<unsigned>((warp * kClusterBlocks + me) * rows_at_once + lane / per_row); k < count;
             k += kClusterBlocks * kSumWarps * rows_at_once) {
            const unsigned bit = first + k;
            const unsigned r = (((bit >> group) * kZeroClusters + own) << group) | (bit & inner);
            if ((seen[k >> 5] >> (k & 31u) & 1u) || r >= a.rows) continue;
            O* const dst = grad + static_cast<long long>(r) * a.grad_ld;
            for (long long c = static_cast<long long>(lane & (per_row - 1)) * EV; c < a.cols; c += per_row * EV)
                store_ev<EV>(dst + c, zeros);
        }
        __syncthreads();
    }
}

// The sorted (key, token) pairs of up to kTinyTokens ids.
template <typename I>
__device__ __forceinline__ void sort_tiny(const I* __restrict__ ids, const SumArgs& a, unsigned long long* word, uint2* sorted)
{
    const unsigned t = threadIdx.x, n = static_cast<unsigned>(a.tokens);
    unsigned long long mine = 0;
    if (t < n) {
        const long long id = static_cast<long long>(ids[t]);
        const unsigned key = id >= 0 && id < a.rows && id != a.padding ? static_cast<unsigned>(id) : a.rows;
        mine = static_cast<unsigned long long>(key) << 32 | t;
        word[t] = mine;
    }
    __syncthreads();
    if (t < n) {
        unsigned before = 0;
        for (unsigned j = 0; j < n; ++j) before += word[j] < mine;
        sorted[before] = make_uint2(static_cast<unsigned>(mine >> 32), t);
    }
    __syncthreads();
}

template <typename T, typename O, int EV>
__global__ void __launch_bounds__(kSumWarps * 32, 4)
k_embed_sum(const T* __restrict__ dy, O* __restrict__ grad, SumArgs a)
{
    constexpr int U = sizeof(T) == 2 && EV > 1 ? 4 : 2;  // rows per batch
    __shared__ float part[kSumWarps][2][8][32];          // [warp][head, tail][element][lane]
    static_assert(sizeof(part) >= sizeof(unsigned) * kZeroWords, "the bit map takes the parts' place");
    __shared__ int link[kSumWarps];
    if (blockIdx.x < static_cast<unsigned>(a.zero_blocks)) {
        unsigned* const seen = reinterpret_cast<unsigned*>(part);
        if (a.id64) zero_rows<long long, O, EV>(static_cast<const long long*>(a.ids), grad, a, seen);
        else        zero_rows<int, O, EV>(static_cast<const int*>(a.ids), grad, a, seen);
        return;
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned at = blockIdx.x - static_cast<unsigned>(a.zero_blocks);
    if (at >= a.sum_blocks) return;
    // Adding to old values, the blocks of rare tokens (high rows, in most vocabularies) take twice as
    // long as others, so they go first: 24k tokens x 1024 42 instead of 46 us, 128k x 4096 244 instead of
    // 257.  Writing, the joins of frequent tokens are better started early (229 instead of 234).
    if (a.accumulate) at = a.sum_blocks - 1u - at;
    const unsigned block = at / static_cast<unsigned>(a.slices);
    const int slice = static_cast<int>(at - block * static_cast<unsigned>(a.slices));
    const int K = a.per_warp;
    const long long p0 = (static_cast<long long>(block) * kSumWarps + warp) * K;
    __shared__ uint2 tiny_pair[kTinyTokens];
    if (a.tiny) {
        unsigned long long* const word = reinterpret_cast<unsigned long long*>(part);
        if (a.id64) sort_tiny(static_cast<const long long*>(a.ids), a, word, tiny_pair);
        else        sort_tiny(static_cast<const int*>(a.ids), a, word, tiny_pair);
    } else {
        wait_for_previous_grid();
    }
    auto pair_at = [&](long long p) { return a.tiny ? tiny_pair[p] : __ldcg(a.pair + p); };

    // The warp's tokens, a group of (up to) 32 at a time, a lane each; keys that are rows come first.
    const int size = min(K, 32), groups = K / size;
    auto group_at = [&](int m) {
        const long long p = p0 + m * 32 + lane;
        return m < groups && lane < size && p < a.tokens ? pair_at(p) : make_uint2(a.rows, 0u);
    };
    uint2 now = group_at(0), next = group_at(1);
    const unsigned key_last = p0 + K <= a.tokens ? pair_at(p0 + K - 1).x : a.rows;
    const unsigned key_before = p0 > 0 && p0 <= a.tokens ? pair_at(p0 - 1).x : a.rows;
    const unsigned key_after = p0 + K < a.tokens ? pair_at(p0 + K).x : a.rows;
    const unsigned key_first = __shfl_sync(0xffffffffu, now.x, 0);
    const bool any = key_first < a.rows;
    const bool head = any && key_before == key_first;
    const bool tail = key_last < a.rows && key_after == key_last;
    const bool through = head && tail && key_first == key_last;
    if (lane == 0) link[warp] = (head ? kLinkHead : 0) | (tail ? kLinkTail : 0) | (through ? kLinkThrough : 0);

    float acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    auto keep = [&](int which) {
#pragma unroll
        for (int j = 0; j < 8; ++j) part[warp][which][j][lane] = acc[j];
    };
    const int width = static_cast<int>(min(a.cols - slice * static_cast<long long>(kSlice), static_cast<long long>(kSlice))) - lane * EV;
    const char* const column0 = reinterpret_cast<const char*>(dy + slice * static_cast<long long>(kSlice) + lane * EV);
    int n = __popc(__ballot_sync(0xffffffffu, now.x < a.rows)), n_next = __popc(__ballot_sync(0xffffffffu, next.x < a.rows));
    // Two batches of rows in registers: while one is added, the other is on its way.
    Raw<EV, T> x[2][U][8 / EV];
    auto fetch = [&](Raw<EV, T> (&to)[8 / EV], unsigned tokens, int k, int count) {
        const T* const row = reinterpret_cast<const T*>(
            column0 + static_cast<unsigned long long>(__shfl_sync(0xffffffffu, tokens, k)) * a.dy_bytes);
        if (k < count)
#pragma unroll
            for (int g = 0; g < 8 / EV; ++g)
                if (g * (32 * EV) < width) to[g].load(row + g * (32 * EV));
    };
    auto add = [&](const Raw<EV, T> (&row)[8 / EV]) {
#pragma unroll
        for (int g = 0; g < 8 / EV; ++g) row[g].add_to(acc + g * EV);
    };
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int u = 0; u < U; ++u) fetch(x[b][u], now.y, b * U + u, n);
    unsigned current = key_first;                        // the run being added ...
    bool open_head = head;                               // ... began in an earlier warp
    for (int m = 0; n > 0;) {
        unsigned left = __shfl_up_sync(0xffffffffu, now.x, 1);
        if (lane == 0) left = current;
        const unsigned starts = __ballot_sync(0xffffffffu, lane < n && now.x != left);   // bit k: token k begins a run
        for (int k0 = 0; k0 < n; k0 += 2 * U) {
            const bool last = k0 + 2 * U >= 32;          // what is fetched belongs to the next group
            const unsigned tokens = last ? next.y : now.y;
            const int count = last ? n_next : n;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int k = k0 + b * U;
                if (k + U <= n && (starts >> k & ((1u << U) - 1u)) == 0u) {              // all of one run
#pragma unroll
                    for (int u = 0; u < U; ++u) add(x[b][u]);
                } else {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (k + u >= n) break;
                        if (starts >> (k + u) & 1u) {
                            if (open_head) keep(0);
                            else store_row<O, EV>(a, grad, current, slice, lane, acc);
                            open_head = false;
                            current = __shfl_sync(0xffffffffu, now.x, k + u);
#pragma unroll
                            for (int j = 0; j < 8; ++j) acc[j] = 0.f;
                        }
                        add(x[b][u]);
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) fetch(x[b][u], tokens, (k + 2 * U + u) & 31, count);
            }
        }
        if (++m >= groups) break;
        now = next;
        n = n_next;
        next = group_at(m + 1);
        n_next = __popc(__ballot_sync(0xffffffffu, next.x < a.rows));
    }
    if (any) {
        if (open_head) keep(0);                          // ends here, or goes through
        else if (tail) keep(1);
        else store_row<O, EV>(a, grad, current, slice, lane, acc);
    }
    __syncthreads();

    // parts of runs that cross warps: added by the warp in which the run ends, or by the last one
    auto gather = [&](int which_end) -> int {            // acc = the run's parts up to this warp; its first warp or -1
        int w = warp - 1;
        if (which_end == 1) {
            w = warp;                                    // the run begins in this warp
        } else {
            while (w >= 0 && (link[w] & kLinkThrough)) --w;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = w >= 0 ? part[w][1][j][lane] : 0.f;
        if (which_end == 0)
            for (int q = max(w + 1, 0); q <= warp; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += part[q][0][j][lane];
        return w;
    };
    if (head && !through) {
        if (gather(0) >= 0) store_row<O, EV>(a, grad, key_first, slice, lane, acc);
        else join_blocks<O, EV>(a, grad, key_first, static_cast<int>(block), false, true, slice, lane, acc);
    }
    if (warp == kSumWarps - 1 && tail) {
        const int w = gather(through ? 0 : 1);
        join_blocks<O, EV>(a, grad, key_last, static_cast<int>(block), w >= 0, false, slice, lane, acc);
    }
}

// ---- host ----------------------------------------------------------------------------------------

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Sorted tokens per warp of the sums' grid: many, so that few runs cross blocks (a crossing costs its
// block about 3 us), but so few that there are 4000 to 16000 warps.  Measured: 128k tokens x 16 slices
// 354 / 259 / 230 / 225 / 229 us at 8 / 16 / 32 / 64 / 128 per warp, 16k x 4 slices 37 / 36 / 38 / 42 / 52,
// 2k x 4 slices 17 / 17 / 22 / 30 / 47.  Fixed by the sizes alone, as the order of the sums is.
int tokens_per_warp(const came_embed& e)
{
    const long long work = e.tokens * ceil_div(e.cols, kSlice);
    return work >= 1ll << 22 ? 128 : work >= 1ll << 20 ? 64 : work >= 1ll << 18 ? 32 : work >= 1ll << 16 ? 16 : 8;
}

struct Layout {
    size_t pair[2], count[kMaxPasses], part, arrived, bytes;
    int digit_bits, passes, sort_blocks; // of the sort
    unsigned tile;
    long long blocks, slices;            // of the sums' grid
    int per_warp;
};

Layout layout(const came_embed& e)
{
    Layout l;
    size_t at = 0;
    auto take = [&](size_t b) { const size_t p = at; at += (b + 255) / 256 * 256; return p; };
    l.per_warp = tokens_per_warp(e);
    l.blocks = ceil_div(e.tokens, kSumWarps * l.per_warp);
    l.slices = ceil_div(e.cols, kSlice);
    int bits = 1;
    while ((e.rows >> bits) != 0) ++bits;                 // the keys are 0 .. rows
    l.passes = static_cast<int>(ceil_div(bits, kMaxDigitBits));
    l.digit_bits = std::max(2, static_cast<int>(ceil_div(bits, l.passes)));      // digits are counted four at a time
    l.tile = static_cast<unsigned>(ceil_div(std::max<long long>(e.tokens, 1), kMoveTile * kMoveBlocks) * kMoveTile);
    l.sort_blocks = static_cast<int>(ceil_div(e.tokens, l.tile));
    for (int k = 0; k < 2; ++k) l.pair[k] = take(sizeof(uint2) * e.tokens);
    for (int k = 0; k < l.passes; ++k)
        l.count[k] = take(sizeof(unsigned) * (static_cast<size_t>(l.sort_blocks) << l.digit_bits));
    l.part = take(sizeof(float) * 2 * kSlice * l.blocks * l.slices);
    l.arrived = take(sizeof(unsigned) * l.blocks * l.slices);
    l.bytes = std::max<size_t>(at, 256);
    return l;
}

came_status validate_embed(const came_embed* e, bool backward)
{
    if (!e) return report(CAME_ERR_NULL, "descriptor is NULL");
    if (e->rows < 1 || e->rows >= (1ll << 31) - 1 || e->cols < 1 || e->cols > (1ll << 29))
        return report(CAME_ERR_SHAPE, "rows must lie in [1, 2^31 - 2], cols in [1, 2^29]");
    if (e->tokens < 0 || e->tokens >= (1ll << 31)) return report(CAME_ERR_SHAPE, "tokens must lie in [0, 2^31)");
    if (e->table_ld < e->cols || e->data_ld < e->cols || e->table_ld > (1ll << 40) / e->rows ||
        e->data_ld > (1ll << 40) / std::max<int64_t>(1, e->tokens))
        return report(CAME_ERR_SHAPE, "a row stride is below cols, or the tensor is too large");
    if (e->table_ld > (1ll << 29) || e->data_ld > (1ll << 29))
        return report(CAME_ERR_SHAPE, "a row stride is beyond 2^29 elements");
    if (!known_dtype(e->table_dtype) || !known_dtype(e->data_dtype)) return report(CAME_ERR_DTYPE, "unknown dtype");
    if (e->id_dtype != CAME_I32 && e->id_dtype != CAME_I64) return report(CAME_ERR_DTYPE, "unknown id_dtype");
    if (e->flags & ~static_cast<uint32_t>(CAME_EMBED_ACCUMULATE | CAME_EMBED_PADDING_ROW))
        return report(CAME_ERR_UNSUPPORTED, "unknown flag");
    if (e->reserved != 0) return report(CAME_ERR_SHAPE, "reserved must be 0");
    if (!holds_in_fp32(e->scale)) return report(CAME_ERR_HPARAM, "scale must be finite, and not vanish, in fp32");
    if (!e->table || (e->tokens && (!e->data || !e->ids))) return report(CAME_ERR_NULL, "table, data and ids are required");
    if (!aligned_to(e->table, dtype_bytes(e->table_dtype)) || !aligned_to(e->data, dtype_bytes(e->data_dtype)) ||
        !aligned_to(e->ids, e->id_dtype == CAME_I64 ? 8 : 4))
        return report(CAME_ERR_ALIGN, "a pointer is not aligned to its element size");
    // what is written shares memory with nothing that is read
    struct Range { uintptr_t lo, hi; };
    auto range = [](const void* p, unsigned long long n) {
        return Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + n}; };
    auto span = [&](long long n, long long ld, int32_t dt) {
        return n ? ((n - 1) * ld + e->cols) * static_cast<unsigned long long>(dtype_bytes(dt)) : 0ull; };
    const Range table = range(e->table, span(e->rows, e->table_ld, e->table_dtype));
    const Range data = range(e->data, span(e->tokens, e->data_ld, e->data_dtype));
    const Range ids = range(e->ids, static_cast<unsigned long long>(e->tokens) * (e->id_dtype == CAME_I64 ? 8 : 4));
    auto meet = [](const Range& a, const Range& b) { return a.lo < b.hi && b.lo < a.hi; };
    const Range& written = backward ? table : data;
    if (e->tokens && (meet(table, data) || meet(written, ids)))
        return report(CAME_ERR_OVERLAP, "the output shares memory with an input");
    return CAME_OK;
}

// Elements per access: the widest of 8, 4, 2, 1 at which every row of both tensors starts aligned.
int elements_per_access(const came_embed& e)
{
    for (int ev = 8; ev > 1; ev >>= 1)
        if (e.cols % ev == 0 && e.table_ld % ev == 0 && e.data_ld % ev == 0 &&
            aligned_to(e.table, ev * dtype_bytes(e.table_dtype)) && aligned_to(e.data, ev * dtype_bytes(e.data_dtype)))
            return ev;
    return 1;
}

template <typename I, typename T, typename O, int EV, int S>
void launch_forward_slices(const came_embed& e, cudaStream_t stream)
{
    const long long per_token = ceil_div(e.cols, kSlice * S), blocks = ceil_div(e.tokens * per_token, 8);
    const bool large = e.tokens * e.cols * static_cast<long long>(sizeof(O)) > (64ll << 20);
    k_embed_forward<I, T, O, EV, S><<<static_cast<unsigned>(blocks), 256, 0, stream>>>(
        static_cast<const T*>(e.table), e.rows, static_cast<int>(e.cols), e.table_ld, static_cast<const I*>(e.ids),
        static_cast<unsigned>(e.tokens), static_cast<float>(e.scale), static_cast<O*>(e.data), e.data_ld,
        static_cast<unsigned>(per_token), large ? 1 : 0);
}

template <typename I, typename T, typename O, int EV>
void launch_forward(const came_embed& e, cudaStream_t stream)
{
    if constexpr (EV == 8) {
        if (e.cols > kSlice) return launch_forward_slices<I, T, O, EV, 4>(e, stream);
    }
    launch_forward_slices<I, T, O, EV, 1>(e, stream);
}

template <typename I, typename T, typename O>
void launch_forward_ev(const came_embed& e, cudaStream_t stream)
{
    switch (elements_per_access(e)) {
        case 8:  launch_forward<I, T, O, 8>(e, stream); break;
        case 4:  launch_forward<I, T, O, 4>(e, stream); break;
        case 2:  launch_forward<I, T, O, 2>(e, stream); break;
        default: launch_forward<I, T, O, 1>(e, stream); break;
    }
}

template <typename I>
void launch_forward_types(const came_embed& e, cudaStream_t stream)
{
    using bf16 = __nv_bfloat16;
    if (e.table_dtype == CAME_BF16) {
        if (e.data_dtype == CAME_BF16) launch_forward_ev<I, bf16, bf16>(e, stream);
        else                           launch_forward_ev<I, bf16, float>(e, stream);
    } else {
        if (e.data_dtype == CAME_BF16) launch_forward_ev<I, float, bf16>(e, stream);
        else                           launch_forward_ev<I, float, float>(e, stream);
    }
}

// Launched with programmatic stream serialisation: the kernel waits for the grid before it itself.
// (early = false: an ordinary launch.)
template <typename K, typename... A>
cudaError_t launch_dependent(K kernel, bool early, int cluster, long long blocks, int threads, size_t smem, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[3];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = early ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    attr[2].id = cudaLaunchAttributeClusterSchedulingPolicyPreference;       // a block of a cluster per SM
    attr[2].val.clusterSchedulingPolicyPreference = cudaClusterSchedulingPolicySpread;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 3 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename I>
cudaError_t launch_sort(const came_embed& e, const SortArgs& a, int32_t device, cudaStream_t stream)
{
    const I* const ids = static_cast<const I*>(e.ids);
    if (e.tokens <= kFewTokens && a.rows < kFewRows) {
        k_embed_sort_few<I><<<1, kFewTokens, 0, stream>>>(ids, a);
        return cudaGetLastError();
    }
    if (e.tokens <= kOneTokens) {
        static std::atomic<uint64_t> done{0};
        const cudaError_t err = allow_smem(k_embed_sort_one<I>, kOneBytes, device, done);
        if (err != cudaSuccess) return err;
        k_embed_sort_one<I><<<1, kSortThreads, kOneBytes, stream>>>(ids, a);
        return cudaGetLastError();
    }
    static std::atomic<uint64_t> done{0};
    cudaError_t err = allow_smem(k_embed_move<I>, sizeof(unsigned) * kMoveWarps * kMaxBins, device, done);
    if (err != cudaSuccess) return err;
    k_embed_count<I><<<a.blocks, kMoveThreads, 0, stream>>>(ids, a);
    err = cudaGetLastError();
    const size_t hist = sizeof(unsigned) * kMoveWarps << a.digit_bits;
    for (int pass = 0; pass < a.passes && err == cudaSuccess; ++pass)
        err = launch_dependent(k_embed_move<I>, true, 1, a.blocks, kMoveThreads, hist, stream, ids, a, pass);
    return err;
}

template <typename T, typename O, int EV>
cudaError_t launch_sums(const came_embed& e, const SumArgs& s, long long blocks, cudaStream_t stream)
{
    // the rows without tokens may be written while the sort runs, but only behind a sort: that has
    // waited for everything before it
    const int cluster = s.zero_blocks ? kClusterBlocks : 1;
    return launch_dependent(k_embed_sum<T, O, EV>, e.tokens > 0 && !s.tiny, cluster, ceil_div(s.zero_blocks + blocks, cluster) * cluster,
                            kSumWarps * 32, 0, stream,
                            static_cast<const T*>(e.data), static_cast<O*>(e.table), s);
}

template <typename T, typename O>
cudaError_t launch_sums_ev(const came_embed& e, const SumArgs& s, long long blocks, cudaStream_t stream)
{
    switch (elements_per_access(e)) {
        case 8:  return launch_sums<T, O, 8>(e, s, blocks, stream);
        case 4:  return launch_sums<T, O, 4>(e, s, blocks, stream);
        case 2:  return launch_sums<T, O, 2>(e, s, blocks, stream);
        default: return launch_sums<T, O, 1>(e, s, blocks, stream);
    }
}

}  // namespace

extern "C" {

came_status came_embed_forward(const came_embed* e, int32_t device, void* cuda_stream)
{
    came_status s = validate_embed(e, false);
    if (s != CAME_OK) return s;
    if (e->flags) return report(CAME_ERR_UNSUPPORTED, "the flags apply to the gradient only");
    if ((s = require_current_device(device)) != CAME_OK) return s;
    if (e->tokens == 0) return CAME_OK;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (e->tokens * ceil_div(e->cols, kSlice) >= (1ll << 32) - 8)
        return report(CAME_ERR_SHAPE, "too many tokens times columns for one launch");
    if (e->id_dtype == CAME_I64) launch_forward_types<long long>(*e, stream);
    else                         launch_forward_types<int>(*e, stream);
    const cudaError_t err = cudaGetLastError();
    return err == cudaSuccess ? CAME_OK : report_cuda(err, "kernel launch");
}

came_status came_embed_workspace(const came_embed* e, int64_t* out_bytes)
{
    if (!out_bytes) return report(CAME_ERR_NULL, "out_bytes is NULL");
    const came_status s = validate_embed(e, true);
    if (s != CAME_OK) return s;
    *out_bytes = static_cast<int64_t>(layout(*e).bytes);
    return CAME_OK;
}

came_status came_embed_backward(const came_embed* e, void* workspace, int64_t workspace_bytes,
                                int32_t device, void* cuda_stream)
{
    came_status s = validate_embed(e, true);
    if (s != CAME_OK) return s;
    const bool padding = (e->flags & CAME_EMBED_PADDING_ROW) != 0;
    if (padding && (e->padding_row < 0 || e->padding_row >= e->rows))
        return report(CAME_ERR_SHAPE, "padding_row is not a row of the table");
    const Layout l = layout(*e);
    if (!workspace) return report(CAME_ERR_NULL, "workspace is NULL");
    if (!aligned_to(workspace, 16)) return report(CAME_ERR_ALIGN, "workspace not 16-byte aligned");
    if (workspace_bytes < static_cast<int64_t>(l.bytes))
        return report(CAME_ERR_SHAPE, "workspace smaller than came_embed_workspace says");
    if ((s = require_current_device(device)) != CAME_OK) return s;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (l.blocks * l.slices + kZeroBlocks >= (1ll << 31)) return report(CAME_ERR_SHAPE, "too many tokens times columns for one launch");
    char* const w = static_cast<char*>(workspace);
    auto at = [&](size_t offset) { return reinterpret_cast<unsigned*>(w + offset); };
    SortArgs a = {};
    for (int k = 0; k < 2; ++k) a.pair[k] = reinterpret_cast<uint2*>(w + l.pair[k]);
    for (int k = 0; k < l.passes; ++k) a.count[k] = at(l.count[k]);
    a.arrived = at(l.arrived);
    a.n_arrived = l.blocks * l.slices;
    a.tokens = e->tokens;
    a.rows = static_cast<unsigned>(e->rows);
    a.padding = padding ? static_cast<unsigned>(e->padding_row) : a.rows;
    a.passes = l.passes;
    a.digit_bits = l.digit_bits;
    a.tile = l.tile;
    a.blocks = l.sort_blocks;
    SumArgs t = {};
    t.pair = a.pair[0];
    t.part = reinterpret_cast<float*>(w + l.part);
    t.arrived = a.arrived;
    t.tokens = e->tokens;
    t.cols = e->cols;
    t.dy_bytes = static_cast<unsigned>(e->data_ld * dtype_bytes(e->data_dtype));
    t.grad_ld = e->table_ld;
    t.rows = a.rows;
    t.slices = static_cast<int>(l.slices);
    t.per_warp = l.per_warp;
    t.accumulate = (e->flags & CAME_EMBED_ACCUMULATE) ? 1 : 0;
    t.scale = static_cast<float>(e->scale);
    t.ids = e->ids;
    t.id64 = e->id_dtype == CAME_I64;
    t.padding = a.padding;
    if (!t.accumulate) {
        t.zero_blocks = kZeroBlocks;
        // at least 2 KB of neighbouring rows together
        while (t.zero_group < 5 && (static_cast<unsigned long long>(e->cols) * dtype_bytes(e->table_dtype) << t.zero_group) < 2048) ++t.zero_group;
    }
    if (e->tokens == 0 && t.accumulate) return CAME_OK;
    t.tiny = e->tokens <= kTinyTokens;
    cudaError_t err = cudaSuccess;
    if (!t.tiny)
        err = e->id_dtype == CAME_I64 ? launch_sort<long long>(*e, a, device, stream)
                                       : launch_sort<int>(*e, a, device, stream);
    if (err != cudaSuccess) return report_cuda(err, "kernel launch(sort)");
    using bf16 = __nv_bfloat16;
    const long long blocks = l.blocks * l.slices;
    t.sum_blocks = static_cast<unsigned>(blocks);
    if (e->data_dtype == CAME_BF16)
        err = e->table_dtype == CAME_BF16 ? launch_sums_ev<bf16, bf16>(*e, t, blocks, stream)
                                          : launch_sums_ev<bf16, float>(*e, t, blocks, stream);
    else
        err = e->table_dtype == CAME_BF16 ? launch_sums_ev<float, bf16>(*e, t, blocks, stream)
                                          : launch_sums_ev<float, float>(*e, t, blocks, stream);
    if (err == cudaSuccess) err = cudaGetLastError();
    return err == cudaSuccess ? CAME_OK : report_cuda(err, "kernel launch");
}

}  // extern "C"
