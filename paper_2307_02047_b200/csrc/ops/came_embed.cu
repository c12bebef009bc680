// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   forward    out[t, :] = rn(scale * W[id_t, :])            0 where id_t is not in [0, rows)
//   backward   dW[v, :] (+)= rn(scale * sum over t with id_t = v of dY[t, :])
//
// The backward pass sorts the tokens by id (stable, so a row's tokens keep their order), then
// adds each row's tokens in that order in fp32: no atomics on floating-point data, results are
// bit-reproducible.
#include "came_ops.cuh"

#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

namespace cg = cooperative_groups;

namespace {

using namespace came_ops;

constexpr int kSlice = 256;              // columns one warp works on: 8 per lane

// EV consecutive elements as they are stored: one access of EV * sizeof(T) bytes.
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
            const uint4 v = *reinterpret_cast<const uint4*>(p);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else if constexpr (B == 8) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x; w[1] = v.y;
        } else if constexpr (B == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else {
            w[0] = *reinterpret_cast<const uint16_t*>(p);
        }
    }

    __device__ __forceinline__ float value(int k) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
        else return __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
    }
};

template <int EV, typename T>
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
        if constexpr (W == 8)
            asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                         :: "l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                            "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
        else if constexpr (W == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (W == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    } else {
        *p = from_float<T>(x[0]);
    }
}

// A lane's eight columns of a slice: 8 / EV groups of EV, 32 * EV columns apart.
template <int EV>
__device__ __forceinline__ long long column(long long slice, int group, int lane)
{
    return slice * kSlice + group * (32 * EV) + lane * EV;
}

// ---- forward --------------------------------------------------------------------------------

constexpr int kFwdSlices = 4;            // slices of one token per warp: loads in flight

template <typename I, typename T, typename O, int EV>
__global__ void __launch_bounds__(256)
k_embed_forward(const T* __restrict__ table, long long rows, long long cols, long long table_ld,
                const I* __restrict__ ids, long long tokens, float scale, O* __restrict__ out,
                long long out_ld, int warps_per_token)
{
    const long long item = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const long long t = item / warps_per_token;
    if (t >= tokens) return;
    const long long s0 = (item - t * warps_per_token) * kFwdSlices;
    const int lane = threadIdx.x & 31;
    const long long id = static_cast<long long>(ids[t]);
    const bool hit = id >= 0 && id < rows;
    const T* const src = table + (hit ? id : 0) * table_ld;
    O* const dst = out + t * out_ld;
    Raw<EV, T> x[kFwdSlices][8 / EV];
#pragma unroll
    for (int s = 0; s < kFwdSlices; ++s)
#pragma unroll
        for (int g = 0; g < 8 / EV; ++g) {
            const long long c = column<EV>(s0 + s, g, lane);
            if (hit && c < cols) x[s][g].load(src + c);
        }
#pragma unroll
    for (int s = 0; s < kFwdSlices; ++s)
#pragma unroll
        for (int g = 0; g < 8 / EV; ++g) {
            const long long c = column<EV>(s0 + s, g, lane);
            if (c < cols) {
                float y[EV];
#pragma unroll
                for (int k = 0; k < EV; ++k) y[k] = hit ? x[s][g].value(k) * scale : 0.f;
                store_ev<EV, O>(dst + c, y);
            }
        }
}

// ---- backward: stable sort of the tokens by row ----------------------------------------------
// One cluster of blocks, least significant digit first.  A warp owns a contiguous run of the
// input; per digit it knows how many equal digits come before its run (in its block: a count per
// warp and digit; in the cluster: the blocks' totals, read through distributed shared memory;
// over all digits: a scan), so every element's place is known and nothing is added by atomics
// whose order matters.  Ids that are not rows (and the padding row) get the key `rows` and end
// up behind all others.
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxDigitBits = 9;
constexpr int kMaxBins = 1 << kMaxDigitBits;
constexpr size_t kSortSmem = sizeof(unsigned) * kSortWarps * kMaxBins;

struct SortArgs {
    unsigned* key[2];        // ping-pong buffers [tokens]
    unsigned* token[2];
    unsigned* row_start;     // [rows] first and last + 1 sorted position of a row's tokens; set
                             // for rows that have some
    unsigned* row_end;
    unsigned* arrived;       // [n_arrived] counters of the sums' grid, cleared here
    long long tokens, n_arrived;
    unsigned  rows, padding; // padding: its own row, or rows when there is none
    int       digit_bits, passes;
};

__device__ __forceinline__ unsigned block_exclusive_scan(unsigned v, unsigned* warp_totals)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
    }
    if (lane == 31) warp_totals[warp] = s;
    __syncthreads();
    unsigned before = 0;
    for (int w = 0; w < warp; ++w) before += warp_totals[w];
    __syncthreads();
    return before + s - v;
}

template <typename I>
__global__ void __launch_bounds__(kSortThreads)
k_embed_sort(const I* __restrict__ ids, SortArgs a)
{
    extern __shared__ unsigned hist[];                   // [warp][digit]
    __shared__ unsigned total[kMaxBins], base[kMaxBins], warp_totals[kSortWarps];
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = static_cast<int>(cluster.num_blocks()), me = static_cast<int>(cluster.block_rank());
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int bins = 1 << a.digit_bits;
    release_dependents();
    for (long long k = static_cast<long long>(me) * kSortThreads + tid; k < a.n_arrived;
         k += static_cast<long long>(blocks) * kSortThreads)
        a.arrived[k] = 0u;
    const long long runs = static_cast<long long>(blocks) * kSortWarps;
    const long long per = ((a.tokens + runs - 1) / runs + 31) / 32 * 32;
    const long long begin = min(a.tokens, (static_cast<long long>(me) * kSortWarps + warp) * per);
    const long long end = min(a.tokens, begin + per);
    unsigned* const mine = hist + warp * kMaxBins;

    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.digit_bits;
        const unsigned* const src_key = a.key[(pass + 1) & 1];
        const unsigned* const src_token = a.token[(pass + 1) & 1];
        unsigned* const dst_key = a.key[pass & 1];
        unsigned* const dst_token = a.token[pass & 1];
        auto key_at = [&](long long k) -> unsigned {
            if (pass > 0) return __ldcg(src_key + k);
            const long long id = static_cast<long long>(ids[k]);
            return (id >= 0 && id < a.rows && id != a.padding) ? static_cast<unsigned>(id) : a.rows;
        };
        for (int k = lane; k < bins; k += 32) mine[k] = 0u;
        __syncwarp();
        for (long long k = begin + lane; k < end; k += 32)
            atomicAdd(&mine[(key_at(k) >> shift) & (bins - 1)], 1u);
        __syncthreads();
        if (tid < bins) {
            unsigned s = 0;
            for (int w = 0; w < kSortWarps; ++w) {
                const unsigned v = hist[w * kMaxBins + tid];
                hist[w * kMaxBins + tid] = s;
                s += v;
            }
            total[tid] = s;
        }
        cluster.sync();
        unsigned before = 0, all = 0;
        if (tid < bins)
            for (int b = 0; b < blocks; ++b) {
                const unsigned v = *cluster.map_shared_rank(&total[tid], b);
                if (b < me) before += v;
                all += v;
            }
        const unsigned first = block_exclusive_scan(all, warp_totals);
        if (tid < bins) base[tid] = first + before;
        __syncthreads();
        for (long long k0 = begin; k0 < end; k0 += 32) {
            const long long k = k0 + lane;
            const bool in = k < end;
            const unsigned active = __ballot_sync(0xffffffffu, in);
            if (in) {
                const unsigned key = key_at(k);
                const unsigned token = pass > 0 ? __ldcg(src_token + k) : static_cast<unsigned>(k);
                const unsigned digit = (key >> shift) & (bins - 1);
                const unsigned peers = __match_any_sync(active, digit);
                const unsigned rank = __popc(peers & ((1u << lane) - 1u));
                const unsigned at = base[digit] + mine[digit] + rank;
                __syncwarp(active);
                if (rank == 0) mine[digit] += __popc(peers);
                __syncwarp(active);
                dst_key[at] = key;
                dst_token[at] = token;
            }
        }
        __threadfence();
        cluster.sync();
    }
    const unsigned* const key = a.key[(a.passes + 1) & 1];
    for (long long k = begin + lane; k < end; k += 32) {
        const unsigned v = __ldcg(key + k);
        if (v >= a.rows) continue;
        if (k == 0 || __ldcg(key + k - 1) != v) a.row_start[v] = static_cast<unsigned>(k);
        if (k + 1 == a.tokens || __ldcg(key + k + 1) != v) a.row_end[v] = static_cast<unsigned>(k + 1);
    }
}

// ---- backward: rows without tokens ---------------------------------------------------------------
// Runs beside the sort (it needs the ids only): block c owns the rows r = c mod gridDim.x (a
// power of two, so that frequent ids, which are neighbours in most vocabularies, spread over the
// blocks), marks those that have tokens in a bit map of its own and writes zeros to the others.
constexpr int kZeroThreads = 512;
constexpr int kZeroWords = 4096;         // bits of rows per round: 131072

template <typename I, typename O, int EV>
__global__ void __launch_bounds__(kZeroThreads)
k_embed_zero(const I* __restrict__ ids, long long tokens, unsigned rows, unsigned padding, long long cols,
             O* __restrict__ grad, long long grad_ld, int log2_blocks)
{
    __shared__ unsigned seen[kZeroWords];
    release_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned own = blockIdx.x, mask = (1u << log2_blocks) - 1u;
    const unsigned owned = own < rows ? ((rows - 1u - own) >> log2_blocks) + 1u : 0u;      // rows of this block
    const float zeros[EV] = {};
    for (unsigned first = 0; first < owned; first += kZeroWords * 32u) {
        const unsigned count = min(owned - first, kZeroWords * 32u);
        for (unsigned k = tid; k < (count + 31u) / 32u; k += kZeroThreads) seen[k] = 0u;
        __syncthreads();
#pragma unroll 4
        for (long long t = tid; t < tokens; t += kZeroThreads) {
            const long long id = static_cast<long long>(ids[t]);
            if (id < 0 || id >= rows || (static_cast<unsigned>(id) & mask) != own || id == padding) continue;
            const unsigned bit = (static_cast<unsigned>(id) >> log2_blocks) - first;
            if (bit < count && !(seen[bit >> 5] >> (bit & 31u) & 1u)) atomicOr(&seen[bit >> 5], 1u << (bit & 31u));
        }
        __syncthreads();
        for (unsigned k = warp; k < count; k += kZeroThreads / 32) {
            if (seen[k >> 5] >> (k & 31u) & 1u) continue;
            O* const dst = grad + (static_cast<long long>(first + k) * (mask + 1u) + own) * grad_ld;
            for (long long c = static_cast<long long>(lane) * EV; c < cols; c += 32 * EV) store_ev<EV, O>(dst + c, zeros);
        }
        __syncthreads();
    }
    // the sums' grid waits for this one; by waiting for the sort here it waits for both
    wait_for_previous_grid();
}

// ---- backward: the sums ----------------------------------------------------------------------------
// A block takes 8 * per_warp consecutive sorted tokens and one slice of the columns, a warp
// per_warp of them: however many tokens a row has, the work is even.  A run of equal keys that
// begins and ends within a warp is stored at once.  A part of a run that crosses warps goes
// through shared memory to the warp in which the run ends; one that crosses blocks goes to
// the workspace, and the block that arrives last for that run adds the parts in order.
constexpr int kSumWarps = 8;
enum : int { kLinkHead = 1, kLinkTail = 2, kLinkThrough = 4 };

struct SumArgs {
    const unsigned* key;       // sorted [tokens]
    const unsigned* token;
    const unsigned* row_start;
    const unsigned* row_end;
    float*    part;            // [blocks of tokens][2][slices][kSlice]: 0 = run from before, 1 = run that goes on
    unsigned* arrived;         // [blocks of tokens][slices]
    long long tokens, cols, dy_ld, grad_ld;
    unsigned  rows;
    int       slices, per_warp, accumulate;
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
        if (a.accumulate) {
            Raw<EV, O> old;
            old.load(dst + c);
#pragma unroll
            for (int k = 0; k < EV; ++k) y[k] = fmaf(a.scale, sum[g * EV + k], old.value(k));
        } else {
#pragma unroll
            for (int k = 0; k < EV; ++k) y[k] = a.scale * sum[g * EV + k];
        }
        store_ev<EV, O>(dst + c, y);
    }
}

// One block's part of a run that crosses blocks.  The last of the run's blocks to arrive adds
// all parts in the order of the tokens and stores the row.
template <typename O, int EV>
__device__ __forceinline__ void join_blocks(const SumArgs& a, O* grad, unsigned row, unsigned block, int slot, int slice,
                                            int lane, const float (&sum)[8])
{
    const unsigned size = static_cast<unsigned>(kSumWarps * a.per_warp);
    const unsigned first = __ldcg(a.row_start + row) / size, last = (__ldcg(a.row_end + row) - 1u) / size;
    auto at = [&](unsigned b, int s) {
        return a.part + ((static_cast<long long>(b) * 2 + s) * a.slices + slice) * kSlice + lane; };
    float* const mine = at(block, slot);
#pragma unroll
    for (int j = 0; j < 8; ++j) __stcg(mine + j * 32, sum[j]);
    __threadfence();
    __syncwarp();
    unsigned final = 0;
    if (lane == 0)
        final = atomicAdd(&a.arrived[static_cast<long long>(first) * a.slices + slice], 1u) == last - first;
    if (!__shfl_sync(0xffffffffu, final, 0)) return;
    __threadfence();
    float total[8];
    {
        const float* const p = at(first, 1);
#pragma unroll
        for (int j = 0; j < 8; ++j) total[j] = __ldcg(p + j * 32);
    }
    for (unsigned b = first + 1; b <= last; b += 4) {
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

template <typename T, typename O, int EV>
__global__ void __launch_bounds__(kSumWarps * 32)
k_embed_sum(const T* __restrict__ dy, O* __restrict__ grad, SumArgs a)
{
    constexpr int U = sizeof(T) == 2 ? 8 : 4;            // rows in flight: 8 * 16 or 4 * 32 bytes per lane
    __shared__ float part[kSumWarps][2][8][32];          // [warp][head, tail][element][lane]
    __shared__ int link[kSumWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned block = blockIdx.x / static_cast<unsigned>(a.slices);
    const int slice = static_cast<int>(blockIdx.x - block * static_cast<unsigned>(a.slices));
    const int K = a.per_warp;
    const long long p0 = (static_cast<long long>(block) * kSumWarps + warp) * K;
    wait_for_previous_grid();

    const long long p = p0 + lane;
    const bool in = lane < K && p < a.tokens;
    const unsigned key = in ? __ldcg(a.key + p) : a.rows;
    const unsigned token = in ? __ldcg(a.token + p) : 0u;
    const int n = __popc(__ballot_sync(0xffffffffu, key < a.rows));          // keys that are rows come first
    const unsigned key_first = __shfl_sync(0xffffffffu, key, 0);
    const unsigned key_last = __shfl_sync(0xffffffffu, key, K - 1);
    const bool head = n > 0 && p0 > 0 && __ldcg(a.key + p0 - 1) == key_first;
    const bool tail = n == K && p0 + K < a.tokens && __ldcg(a.key + p0 + K) == key_last;
    const bool through = head && tail && key_first == key_last;
    if (lane == 0) link[warp] = (head ? kLinkHead : 0) | (tail ? kLinkTail : 0) | (through ? kLinkThrough : 0);

    float acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    auto keep = [&](int which) {
#pragma unroll
        for (int j = 0; j < 8; ++j) part[warp][which][j][lane] = acc[j];
    };
    unsigned current = key_first;
    bool open_head = head;                               // the run being added began in an earlier warp
    for (int k = 0; k < n; k += U) {
        Raw<EV, T> x[U][8 / EV];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned t = __shfl_sync(0xffffffffu, token, (k + u) & 31);
#pragma unroll
            for (int g = 0; g < 8 / EV; ++g) {
                const long long c = column<EV>(slice, g, lane);
                if (k + u < n && c < a.cols) x[u][g].load(dy + static_cast<long long>(t) * a.dy_ld + c);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned v = __shfl_sync(0xffffffffu, key, (k + u) & 31);
            if (k + u < n) {
                if (v != current) {
                    if (open_head) keep(0);
                    else store_row<O, EV>(a, grad, current, slice, lane, acc);
                    open_head = false;
                    current = v;
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] += x[u][j / EV].value(j % EV);
            }
        }
    }
    if (n > 0) {
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
        else join_blocks<O, EV>(a, grad, key_first, block, 0, slice, lane, acc);
    }
    if (warp == kSumWarps - 1 && tail) {
        const int w = gather(through ? 0 : 1);
        join_blocks<O, EV>(a, grad, key_last, block, w >= 0 ? 1 : 0, slice, lane, acc);
    }
}

// ---- host ----------------------------------------------------------------------------------------

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Sorted tokens per warp of the sums' grid: enough to cover the latency of a row's load, few
// enough that there are several thousand warps.  Fixed by the sizes alone, as the order of the sums is.
int tokens_per_warp(const came_embed& e)
{
    const long long work = e.tokens * ceil_div(e.cols, kSlice);
    return work >= 32 * 8192 ? 32 : work >= 16 * 8192 ? 16 : 8;
}

struct Layout {
    size_t key[2], token[2], row_start, row_end, part, arrived, bytes;
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
    for (int k = 0; k < 2; ++k) l.key[k] = take(sizeof(unsigned) * e.tokens);
    for (int k = 0; k < 2; ++k) l.token[k] = take(sizeof(unsigned) * e.tokens);
    l.row_start = take(sizeof(unsigned) * e.rows);
    l.row_end = take(sizeof(unsigned) * e.rows);
    l.part = take(sizeof(float) * 2 * kSlice * l.blocks * l.slices);
    l.arrived = take(sizeof(unsigned) * l.blocks * l.slices);
    l.bytes = at;
    return l;
}

came_status validate_embed(const came_embed* e, bool backward)
{
    if (!e) return report(CAME_ERR_NULL, "descriptor is NULL");
    if (e->rows < 1 || e->rows >= (1ll << 31) - 1 || e->cols < 1 || e->cols >= (1ll << 31))
        return report(CAME_ERR_SHAPE, "rows and cols must be >= 1 and below 2^31 - 1");
    if (e->tokens < 0 || e->tokens >= (1ll << 31)) return report(CAME_ERR_SHAPE, "tokens must lie in [0, 2^31)");
    if (e->table_ld < e->cols || e->data_ld < e->cols || e->table_ld > (1ll << 40) / e->rows ||
        e->data_ld > (1ll << 40) / std::max<int64_t>(1, e->tokens))
        return report(CAME_ERR_SHAPE, "a row stride is below cols, or the tensor is too large");
    if (!known_dtype(e->table_dtype) || !known_dtype(e->data_dtype)) return report(CAME_ERR_DTYPE, "unknown dtype");
    if (e->id_dtype != CAME_I32 && e->id_dtype != CAME_I64) return report(CAME_ERR_DTYPE, "unknown id_dtype");
    if (e->flags & ~static_cast<uint32_t>(CAME_EMBED_ACCUMULATE | CAME_EMBED_PADDING_ROW))
        return report(CAME_ERR_UNSUPPORTED, "unknown flag");
    if (e->reserved != 0) return report(CAME_ERR_SHAPE, "reserved must be 0");
    if (!std::isfinite(e->scale)) return report(CAME_ERR_HPARAM, "scale must be finite");
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

template <typename I, typename T, typename O, int EV>
void launch_forward(const came_embed& e, cudaStream_t stream)
{
    const int per_token = static_cast<int>(ceil_div(e.cols, kSlice * kFwdSlices));
    const long long items = e.tokens * per_token;
    k_embed_forward<I, T, O, EV><<<static_cast<unsigned>(ceil_div(items, 8)), 256, 0, stream>>>(
        static_cast<const T*>(e.table), e.rows, e.cols, e.table_ld, static_cast<const I*>(e.ids), e.tokens,
        static_cast<float>(e.scale), static_cast<O*>(e.data), e.data_ld, per_token);
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
cudaError_t launch_dependent(K kernel, bool early, long long blocks, int threads, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = early ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename I>
cudaError_t launch_sort(const came_embed& e, const SortArgs& a, cudaStream_t stream)
{
    cudaError_t err = cudaFuncSetAttribute(k_embed_sort<I>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                           static_cast<int>(kSortSmem));
    if (err != cudaSuccess) return err;
    cudaLaunchConfig_t cfg = {};
    const unsigned blocks = e.tokens <= 4096 ? 1 : 8;
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = kSortSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = blocks;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_embed_sort<I>, static_cast<const I*>(e.ids), a);
}

template <typename I, typename O, int EV>
cudaError_t launch_zero(const came_embed& e, unsigned padding, cudaStream_t stream)
{
    int lg = 0;
    while (lg < 8 && (2ll << lg) <= e.rows) ++lg;        // at most 256 blocks, two per SM
    // it may start while the sort runs, but only behind a sort: the sort has waited for everything
    // before it, and only then may rows be written
    return launch_dependent(k_embed_zero<I, O, EV>, e.tokens > 0, 1ll << lg, kZeroThreads, stream, static_cast<const I*>(e.ids),
                            static_cast<long long>(e.tokens), static_cast<unsigned>(e.rows), padding,
                            static_cast<long long>(e.cols), static_cast<O*>(e.table),
                            static_cast<long long>(e.table_ld), lg);
}

template <typename T, typename O, int EV>
cudaError_t launch_sums(const came_embed& e, const SumArgs& s, unsigned padding, long long blocks, cudaStream_t stream)
{
    cudaError_t err = cudaSuccess;
    if (!s.accumulate)
        err = e.id_dtype == CAME_I64 ? launch_zero<long long, O, EV>(e, padding, stream) : launch_zero<int, O, EV>(e, padding, stream);
    if (err == cudaSuccess && blocks > 0)
        err = launch_dependent(k_embed_sum<T, O, EV>, true, blocks, kSumWarps * 32, stream, static_cast<const T*>(e.data),
                               static_cast<O*>(e.table), s);
    return err;
}

template <typename T, typename O>
cudaError_t launch_sums_ev(const came_embed& e, const SumArgs& s, unsigned padding, long long blocks, cudaStream_t stream)
{
    switch (elements_per_access(e)) {
        case 8:  return launch_sums<T, O, 8>(e, s, padding, blocks, stream);
        case 4:  return launch_sums<T, O, 4>(e, s, padding, blocks, stream);
        case 2:  return launch_sums<T, O, 2>(e, s, padding, blocks, stream);
        default: return launch_sums<T, O, 1>(e, s, padding, blocks, stream);
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
    if (e->tokens * ceil_div(e->cols, kSlice * kFwdSlices) > (1ll << 33))
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
    if (l.blocks * l.slices >= (1ll << 31)) return report(CAME_ERR_SHAPE, "too many tokens times columns for one launch");
    char* const w = static_cast<char*>(workspace);
    auto at = [&](size_t offset) { return reinterpret_cast<unsigned*>(w + offset); };
    SortArgs a = {};
    for (int k = 0; k < 2; ++k) {
        a.key[k] = at(l.key[k]);
        a.token[k] = at(l.token[k]);
    }
    a.row_start = at(l.row_start);
    a.row_end = at(l.row_end);
    a.arrived = at(l.arrived);
    a.n_arrived = l.blocks * l.slices;
    a.tokens = e->tokens;
    a.rows = static_cast<unsigned>(e->rows);
    a.padding = padding ? static_cast<unsigned>(e->padding_row) : a.rows;
    int bits = 1;
    while ((e->rows >> bits) != 0) ++bits;                // the keys are 0 .. rows
    a.passes = static_cast<int>(ceil_div(bits, kMaxDigitBits));
    a.digit_bits = static_cast<int>(ceil_div(bits, a.passes));
    SumArgs t = {};
    t.key = a.key[(a.passes + 1) & 1];
    t.token = a.token[(a.passes + 1) & 1];
    t.row_start = a.row_start;
    t.row_end = a.row_end;
    t.part = reinterpret_cast<float*>(w + l.part);
    t.arrived = a.arrived;
    t.tokens = e->tokens;
    t.cols = e->cols;
    t.dy_ld = e->data_ld;
    t.grad_ld = e->table_ld;
    t.rows = a.rows;
    t.slices = static_cast<int>(l.slices);
    t.per_warp = l.per_warp;
    t.accumulate = (e->flags & CAME_EMBED_ACCUMULATE) ? 1 : 0;
    t.scale = static_cast<float>(e->scale);
    cudaError_t err = cudaSuccess;
    if (e->tokens > 0)
        err = e->id_dtype == CAME_I64 ? launch_sort<long long>(*e, a, stream) : launch_sort<int>(*e, a, stream);
    if (err != cudaSuccess) return report_cuda(err, "kernel launch(sort)");
    using bf16 = __nv_bfloat16;
    const long long blocks = l.blocks * l.slices;
    if (e->data_dtype == CAME_BF16)
        err = e->table_dtype == CAME_BF16 ? launch_sums_ev<bf16, bf16>(*e, t, a.padding, blocks, stream)
                                          : launch_sums_ev<bf16, float>(*e, t, a.padding, blocks, stream);
    else
        err = e->table_dtype == CAME_BF16 ? launch_sums_ev<float, bf16>(*e, t, a.padding, blocks, stream)
                                          : launch_sums_ev<float, float>(*e, t, a.padding, blocks, stream);
    if (err == cudaSuccess) err = cudaGetLastError();
    return err == cudaSuccess ? CAME_OK : report_cuda(err, "kernel launch");
}

}  // extern "C"
