// Learned relative position bias by buckets of distances, and its gradient.
//
//   out[h, i, j] = table[bucket(j - i - offset), h]
//   dtable[b, h] = sum over (n, i, j) with that bucket of dout[n, h, i, j]
//
// Everything depends on j - i alone.  Forward: a block writes a tile of one head from a line of the tile's
// diagonals in shared memory.  Backward: a warp follows diagonals, whose sums stay in registers, and adds up the buckets,
// which are intervals of diagonals, at the end.
#include "came_vec.cuh"

#include <algorithm>
#include <cmath>

namespace {

using namespace came_ops;

constexpr int kMostBuckets = 1024;
constexpr int kSMs = 148;
constexpr int kWarps = 8;
constexpr int kMostAdditions = 512;
constexpr long long kFar = 1ll << 40;

// Distances of one direction: bucket m begins at start[m].
template <int M>
struct Buckets {
    int n;                               // buckets of a direction, M at most
    int both;
    int start[M];
};
constexpr int kFewBuckets = 64;          // (the tables travel with the launch)

struct BiasArgs {
    void*          table;
    void*          data;
    const int64_t* device_offset;
    long long      offset;
    long long      q, k, batch, table_ld, batch_stride, head_stride, q_stride;
    int            heads, buckets, table_bf16;
    int            tile_rows, tile_vectors;          // forward
    long long      tiles;                // backward: tiles of diagonals, parts of a tile's rows, batches for a warp
    int            chunks, batches, batch_groups, period;
    float*         part;                 // backward: [heads][units][buckets]
};

__device__ __forceinline__ long long offset_of(const BiasArgs& a)
{
    if (!a.device_offset) return a.offset;
    return max(-kFar, min(kFar, static_cast<long long>(*a.device_offset)));
}

// Bucket, within its direction, of a distance: the last m with start[m] <= d.
__device__ __forceinline__ int bucket_of(const int* start, int n, long long d)
{
    int lo = 0, hi = n;                  // start[lo] <= d < start[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= d) lo = mid;
        else hi = mid;
    }
    return lo;
}

__host__ __device__ __forceinline__ long long distance_of(long long relative, int both)
{
    return relative > 0 ? (both ? relative : 0) : -relative;
}

// ---- forward ------------------------------------------------------------------------------------

// A tile: tile_rows rows and tile_vectors accesses of 16 bytes in each, aligned in memory: row i's accesses begin at its
// first aligned column, wherever that is.  The line of the tile's diagonals is kept once for every alignment
// of a group of N values, so that each access is one load from shared memory and one store.
template <typename T, int M>
__global__ void __launch_bounds__(256)
k_posbias_forward(const __grid_constant__ BiasArgs a, const __grid_constant__ Buckets<M> buckets)
{
    constexpr int N = 16 / static_cast<int>(sizeof(T));
    extern __shared__ __align__(16) char dynamic[];
    __shared__ int start[M];
    T* const line = reinterpret_cast<T*>(dynamic);
    const int tr = a.tile_rows, tv = a.tile_vectors, length = (tr + N * tv + N + N - 1) / N * N;
    const int h = blockIdx.z;
    const long long i0 = static_cast<long long>(blockIdx.y) * tr, v0 = static_cast<long long>(blockIdx.x) * tv;
    for (int m = threadIdx.x; m < buckets.n; m += 256) start[m] = buckets.start[m];
    __syncthreads();
    // line[x]: the diagonal of column N v0 + x - (tr - 1) in row i0
    const long long origin = N * v0 - (tr - 1) - i0 - offset_of(a);
    for (int x = threadIdx.x; x < length; x += 256) {
        const long long relative = origin + x;
        const int b = bucket_of(start, buckets.n, distance_of(relative, buckets.both)) + (buckets.both && relative > 0 ? buckets.n : 0);
        const long long at = b * a.table_ld + h;
        const float value = a.table_bf16 ? to_float(static_cast<const __nv_bfloat16*>(a.table)[at]) : static_cast<const float*>(a.table)[at];
        const T t = from_float<T>(value);
#pragma unroll
        for (int s = 0; s < N; ++s)
            if (x >= s) line[s * length + x - s] = t;
    }
    __syncthreads();
    T* const out = static_cast<T*>(a.data) + h * a.q * a.k;
    const unsigned skew = static_cast<unsigned>(reinterpret_cast<uintptr_t>(out) / sizeof(T)), keys = static_cast<unsigned>(a.k);
    const int rows_at_once = 256 / tv, v = threadIdx.x % tv;
    const unsigned vector = static_cast<unsigned>(v0) + v;
    const int rows = static_cast<int>(min(static_cast<long long>(tr), a.q - i0));
    T* row = out + (i0 + threadIdx.x / tv) * a.k;
    for (int r = threadIdx.x / tv; r < rows; r += rows_at_once, row += rows_at_once * a.k) {
        const unsigned ahead = (N - (skew + static_cast<unsigned>(i0 + r) * keys) % N) % N;      // elements before the row's first aligned one
        const unsigned have = keys >= ahead ? (keys - ahead) / N : 0u;                           // whole accesses of the row
        const unsigned x = ahead + N * v + (tr - 1) - r;
        T* const to = row + ahead + static_cast<size_t>(N) * vector;
        if (vector < have) {
            *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(line + (x % N) * length + x / N * N);
        } else if (vector == have) {
            for (unsigned e = 0; e < N && ahead + N * vector + e < keys; ++e) to[e] = line[x + e];
        }
        if (vector == 0)
            for (unsigned e = 0; e < ahead && e < keys; ++e) row[e] = line[e + (tr - 1) - r];
    }
}

// ---- backward -----------------------------------------------------------------------------------

__device__ __forceinline__ void add_value(float& sum, const Vec<float, 8>& v, int k) { sum += v.value(k); }
__device__ __forceinline__ void add_value(float& sum, const Vec<__nv_bfloat16, 8>& v, int k)
{
    const uint16_t h = static_cast<uint16_t>(k & 1 ? v.w[k >> 1] >> 16 : v.w[k >> 1] & 0xffffu);
    asm("add.rn.f32.bf16 %0, %1, %0;" : "+f"(sum) : "h"(h));
}

// Rows of a head that are eight apart begin at the same place relative to an aligned address, whatever their stride is.  A warp takes
// such rows, first + 8 m, and goes down them while its lanes go right, an aligned access of eight elements for a row: the
// differences column - row of a lane's elements stay what they are, so that eight sums in registers are all it needs.  An
// access v of a row covers the columns 8 v - skew to 8 v - skew + 7; lane l has the accesses with v - m = block + l.
// The accesses that reach over an end of the row, one or two for a lane, are made afterwards, element by element.
// (bf16: registers for three blocks per SM, 92 us for 16 heads of 4096 x 4096, 97 with four; fp32: for two)
template <typename T, int M>
__global__ void __launch_bounds__(kWarps * 32, sizeof(T) == 2 ? 3 : 2)
k_posbias_backward(const __grid_constant__ BiasArgs a, const __grid_constant__ Buckets<M> buckets)
{
    constexpr int length = 256;
    __shared__ float lines[kWarps][length];
    __shared__ int start[M];
    release_dependents();
    for (int m = threadIdx.x; m < buckets.n; m += kWarps * 32) start[m] = buckets.start[m];
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long units = 8ll * a.tiles * a.chunks * a.batch_groups;
    const long long unit = static_cast<long long>(blockIdx.x) * kWarps + warp;
    const int h = blockIdx.y;
    if (unit >= units) return;
    // (the warps of a block: the eight places, neighbouring rows)
    const int first = static_cast<int>(unit % 8);
    const long long group = unit / 8, chunk = group / a.batch_groups % a.chunks, tile = group / a.batch_groups / a.chunks;
    const int part_of_batch = static_cast<int>(group % a.batch_groups), place = part_of_batch % a.period;
    const long long n0 = place + static_cast<long long>(part_of_batch - place) * a.batches, n1 = min(a.batch, n0 + static_cast<long long>(a.period) * a.batches);
    const T* const head = static_cast<const T*>(a.data) + h * a.head_stride + first * a.q_stride;
    // (the unit's batches, n0, n0 + period, ..., begin at the same place)
    const int skew = static_cast<int>(reinterpret_cast<uintptr_t>(head + n0 * a.batch_stride) / sizeof(T) & 7);
    const long long rows = (a.q - first + 7) >> 3, vectors = (a.k + skew + 7) >> 3;
    const long long block = 32 * tile - (((a.q + 7) >> 3) - 1);
    const long long low = max(0ll, -(block + 31)), high = min(rows, vectors - block);      // rows that meet the tile
    const long long m0 = low + chunk * a.tile_rows, m1 = min(high, m0 + a.tile_rows);
    float* const part = a.part + (h * units + unit) * a.buckets;
    if (m0 >= m1) {                      // (beside the tile's rows)
        for (int b = lane; b < a.buckets; b += 32) part[b] = 0.f;
        return;
    }
    const long long mine = block + lane;
    float sums[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sums[k] = 0.f;
    // rows for which this lane's access lies within the row
    const long long whole0 = max(m0, (skew ? 1ll : 0ll) - mine), whole1 = min(m1, ((a.k + skew) >> 3) - mine);
    for (long long n = n0; n < n1; n += a.period) {
        const T* const here = head + n * a.batch_stride + 8 * mine - skew;       // row m's access: here + m step
        const long long step = 8 * a.q_stride + 8;
        const T* p = here + m0 * step;
        for (long long m = m0; m < m1; m += 8, p += 8 * step) {
            Vec<T, 8> v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
#pragma unroll
                for (int j = 0; j < Vec<T, 8>::W; ++j) v[u].w[j] = 0u;
                if (m + u >= whole0 && m + u < whole1) v[u].load(p + u * step);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int k = 0; k < 8; ++k) add_value(sums[k], v[u], k);
        }
        // the row's first access, where it begins in front of the row, and its last, where it ends behind it
#pragma unroll 1
        for (int side = 0; side < 2; ++side) {
            const long long vector = side ? vectors - 1 : 0, m = vector - mine;
            const bool part = side ? (a.k + skew) % 8 != 0 && (vector > 0 || !skew) : skew != 0;
            if (!part || m < m0 || m >= m1) continue;
            const long long column = 8 * vector - skew;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (column + k >= 0 && column + k < a.k) sums[k] += to_float(here[m * step + k]);
        }
    }
    float* const line = lines[warp];     // line[x]: the x-th of the tile's diagonals
#pragma unroll
    for (int k = 0; k < 8; ++k) line[8 * lane + k] = sums[k];
    __syncwarp();
    // Buckets are intervals of diagonals: a lane adds a short one up, the warp a long one.
    const long long origin = 8 * block - skew - first - offset_of(a);    // line[x] has key - query - offset = origin + x
    constexpr long long kNone = 4 * kFar;
    for (int b0 = 0; b0 < a.buckets; b0 += 32) {
        const int b = b0 + lane;
        int x0 = 0, x1 = 0;
        if (b < a.buckets) {
            const bool behind = b >= buckets.n;          // (only with buckets.both)
            const int m = behind ? b - buckets.n : b;
            const long long from = start[m], to = m == buckets.n - 1 ? kNone : start[m + 1];     // its distances [from, to)
            long long lo, hi;
            if (behind) {
                lo = max(1ll, from);
                hi = to;
            } else {
                lo = 1 - to;
                hi = m == 0 && !buckets.both ? kNone : 1 - from;
            }
            x0 = static_cast<int>(max(0ll, min(static_cast<long long>(length), lo - origin)));
            x1 = static_cast<int>(max(0ll, min(static_cast<long long>(length), hi - origin)));
        }
        const bool large = x1 - x0 > 32;
        float mine = 0.f;
        if (!large)
            for (int x = x0; x < x1; ++x) mine += line[x];
        for (unsigned todo = __ballot_sync(0xffffffffu, large); todo; todo &= todo - 1) {
            const int owner = __ffs(todo) - 1;
            const int y0 = __shfl_sync(0xffffffffu, x0, owner), y1 = __shfl_sync(0xffffffffu, x1, owner);
            float s = 0.f;
            for (int x = y0 + lane; x < y1; x += 32) s += line[x];
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
            if (lane == owner) mine = s;
        }
        if (b < a.buckets) part[b] = mine;
    }
}

// Adds a head's units: 32 buckets for each block, 32 warps that take every 32nd unit.  There may be many: 16 of a warp's, whose
// loads are on their way together, are added in fp32, from there on in fp64 (each by itself 7 % more for 16 heads of 4096 x 4096 bf16).
__global__ void __launch_bounds__(1024)
k_posbias_finish(const __grid_constant__ BiasArgs a, long long units, int accumulate)
{
    constexpr int kRun = 16;
    __shared__ double s[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.x * 32 + lane, h = blockIdx.y;
    wait_for_previous_grid();
    double v = 0.0;
    if (b < a.buckets)
        for (long long u = warp; u < units; u += 32 * kRun) {
            const float* const from = a.part + (h * units + u) * a.buckets + b;
            float x[kRun], run = 0.f;
#pragma unroll
            for (int j = 0; j < kRun; ++j) x[j] = u + 32 * j < units ? from[32ll * j * a.buckets] : 0.f;
#pragma unroll
            for (int j = 0; j < kRun; ++j) run += x[j];
            v += run;
        }
    s[warp][lane] = v;
    __syncthreads();
    if (warp != 0 || b >= a.buckets) return;
    double t = 0.0;
    for (int g = 0; g < 32; ++g) t += s[g][lane];
    const long long at = b * a.table_ld + h;
    if (a.table_bf16) {
        __nv_bfloat16* const o = static_cast<__nv_bfloat16*>(a.table) + at;
        *o = __double2bfloat16(accumulate ? to_float(*o) + t : t);
    } else {
        float* const o = static_cast<float*>(a.table) + at;
        *o = static_cast<float>(accumulate ? *o + t : t);
    }
}

// ---- host ---------------------------------------------------------------------------------------

came_status validate_buckets(const came_posbias& p)
{
    const bool both = p.flags & CAME_POSBIAS_BIDIRECTIONAL;
    if (p.buckets < (both ? 4 : 2) || p.buckets > kMostBuckets || (both && p.buckets % 2))
        return report(CAME_ERR_SHAPE, "buckets must lie in [2, 1024], bidirectional: be even and at least 4");
    const int n = both ? p.buckets / 2 : p.buckets;
    if (p.max_distance <= n / 2 || p.max_distance > (1 << 29))
        return report(CAME_ERR_HPARAM, "max_distance must lie above the distances that have a bucket each, up to 2^29");
    return CAME_OK;
}

template <int M>
void fill_buckets(const came_posbias& p, Buckets<M>& b)
{
    b.both = (p.flags & CAME_POSBIAS_BIDIRECTIONAL) ? 1 : 0;
    b.n = b.both ? p.buckets / 2 : p.buckets;
    const int e = b.n / 2, steps = b.n - e;
    for (int m = 0; m < b.n; ++m) {
        if (m <= e) { b.start[m] = m; continue; }
        // the smallest d with E (max_distance / E)^((m - E) / steps) <= d; what is this near to a whole number is one
        const double border = e * std::pow(static_cast<double>(p.max_distance) / e, static_cast<double>(m - e) / steps);
        const double whole = std::nearbyint(border);
        b.start[m] = static_cast<int>(std::fabs(border - whole) <= 1e-13 * border ? whole : std::ceil(border));
    }
}

came_status validate_posbias(const came_posbias* p, bool backward)
{
    if (!p) return report(CAME_ERR_NULL, "descriptor is NULL");
    if (p->q_len < 0 || p->q_len > (1ll << 30) || p->k_len < 0 || p->k_len > (1ll << 30) || p->heads < 1 || p->heads > 65535)
        return report(CAME_ERR_SHAPE, "q_len and k_len must lie in [0, 2^30], heads in [1, 65535]");
    if (p->flags & ~static_cast<uint32_t>(CAME_POSBIAS_BIDIRECTIONAL | CAME_POSBIAS_ACCUMULATE)) return report(CAME_ERR_UNSUPPORTED, "unknown flag");
    if ((p->flags & CAME_POSBIAS_ACCUMULATE) && !backward) return report(CAME_ERR_UNSUPPORTED, "accumulation applies to the backward pass only");
    const came_status s = validate_buckets(*p);
    if (s != CAME_OK) return s;
    if (p->offset < -kFar || p->offset > kFar) return report(CAME_ERR_SHAPE, "offset must lie in [-2^40, 2^40]");
    if (p->table_ld < p->heads || p->table_ld > (1ll << 29)) return report(CAME_ERR_SHAPE, "table_ld must lie in [heads, 2^29]");
    if (!known_dtype(p->table_dtype) || !known_dtype(p->data_dtype)) return report(CAME_ERR_DTYPE, "unknown dtype");
    const double most = static_cast<double>(1ll << 40);
    if (static_cast<double>(p->heads) * p->q_len * p->k_len > most) return report(CAME_ERR_SHAPE, "more than 2^40 elements");
    if (backward) {
        if (p->batch < 0 || p->batch > (1 << 20)) return report(CAME_ERR_SHAPE, "batch must lie in [0, 2^20]");
        if (p->batch_stride < 0 || p->head_stride < 0 || p->q_stride < 0 ||
            static_cast<double>(p->batch) * p->batch_stride > most || static_cast<double>(p->heads) * p->head_stride > most ||
            static_cast<double>(p->q_len) * p->q_stride > most)
            return report(CAME_ERR_SHAPE, "a stride is negative, or too large");
    }
    const bool empty = !p->q_len || !p->k_len || (backward && !p->batch);
    if (!p->table || (!empty && !p->data)) return report(CAME_ERR_NULL, "table and data are required");
    if (!aligned_to(p->table, dtype_bytes(p->table_dtype)) || !aligned_to(p->data, dtype_bytes(p->data_dtype)) || !aligned_to(p->device_offset, 8))
        return report(CAME_ERR_ALIGN, "a pointer is not aligned to its element size");
    struct Range { uintptr_t lo, hi; };
    auto range = [](const void* q, unsigned long long n) { return Range{reinterpret_cast<uintptr_t>(q), reinterpret_cast<uintptr_t>(q) + n}; };
    auto meet = [](const Range& x, const Range& y) { return x.lo < y.hi && y.lo < x.hi; };
    const unsigned long long last = backward ? (p->batch - 1) * p->batch_stride + (p->heads - 1) * p->head_stride + (p->q_len - 1) * p->q_stride + p->k_len
                                             : static_cast<unsigned long long>(p->heads) * p->q_len * p->k_len;
    const Range table = range(p->table, ((p->buckets - 1) * p->table_ld + p->heads) * dtype_bytes(p->table_dtype));
    const Range data = range(p->data, empty ? 0 : last * dtype_bytes(p->data_dtype));
    const Range offset = range(p->device_offset, p->device_offset ? 8 : 0);
    if ((!empty && meet(table, data)) || meet(offset, backward ? table : data)) return report(CAME_ERR_OVERLAP, "the output shares memory with an input");
    return CAME_OK;
}

struct BackwardPlan { int tile_rows, chunks, batches, batch_groups, period; long long tiles, units, bytes; };

// Rows that a warp goes down, and batches for a warp: as many as make 32 warps for each SM, of which the kernels' registers let 24
// (fp32: 16) run at a time (9 x 8 x 1023 x 1025 fp32: 72 us, 77 with 24 or 48 warps; 64 x 12 x 512 x 512 bf16: 108, 101 and 105).
BackwardPlan plan_backward(const came_posbias& p)
{
    BackwardPlan b = {};
    const long long rows = std::max<long long>(1, (p.q_len + 7) / 8), vectors = std::max<long long>(1, (p.k_len + 14) / 8);
    const long long batch = std::max<int64_t>(1, p.batch), want = kSMs * 32;
    b.tiles = (rows - 1 + vectors + 31) / 32;
    const long long tall = std::min(rows, vectors + 31);         // rows that meet a tile, at most
    const long long all = 8 * b.tiles * p.heads;
    b.tile_rows = 128;
    auto chunks = [&] { return (tall + b.tile_rows - 1) / b.tile_rows; };
    while (b.tile_rows > 16 && all * chunks() * batch < want) b.tile_rows /= 2;
    b.chunks = static_cast<int>(chunks());
    // A warp's batches begin at one place: every period-th one.
    b.period = 1;
    while (b.period < batch && b.period * p.batch_stride % 8) b.period *= 2;
    b.period = static_cast<int>(std::min<long long>(b.period, batch));
    const long long count = (batch + b.period - 1) / b.period, turns = std::min(count, std::max(1ll, want / (all * b.chunks) / b.period));
    // (and as few that a lane adds kMostAdditions terms of a diagonal at most one after another)
    const long long most = std::max(1ll, kMostAdditions / std::min<long long>(b.tile_rows, tall));
    b.batches = static_cast<int>(std::min(most, (count + turns - 1) / turns));
    b.batch_groups = static_cast<int>((count + b.batches - 1) / b.batches * b.period);
    b.units = 8 * b.tiles * b.chunks * b.batch_groups;
    b.bytes = b.units * p.heads * p.buckets * 4;
    return b;
}

BiasArgs args_of(const came_posbias& p)
{
    BiasArgs a = {};
    a.table = p.table;
    a.data = p.data;
    a.device_offset = p.device_offset;
    a.offset = p.offset;
    a.q = p.q_len;
    a.k = p.k_len;
    a.batch = p.batch;
    a.table_ld = p.table_ld;
    a.batch_stride = p.batch_stride;
    a.head_stride = p.head_stride;
    a.q_stride = p.q_stride;
    a.heads = p.heads;
    a.buckets = p.buckets;
    a.table_bf16 = p.table_dtype == CAME_BF16;
    return a;
}

template <typename T, int M>
came_status launch_forward(const came_posbias& p, cudaStream_t stream)
{
    constexpr int N = 16 / sizeof(T);
    BiasArgs a = args_of(p);
    Buckets<M> b;
    fill_buckets(p, b);
    const long long vectors = p.k_len / N + 1;           // (the last one, or the only one, may be part of one)
    // Tiles of 64 rows; of few rows and a quarter of the columns where that leaves SMs without a block.
    a.tile_vectors = 128;
    a.tile_rows = static_cast<int>(std::min<int64_t>(64, p.q_len));
    auto blocks = [&] { return (vectors + a.tile_vectors - 1) / a.tile_vectors * ((p.q_len + a.tile_rows - 1) / a.tile_rows) * p.heads; };
    if (blocks() < 2 * kSMs) a.tile_vectors = 32;
    while (a.tile_rows > 8 && blocks() < 2 * kSMs) a.tile_rows /= 2;
    const long long x = (vectors + a.tile_vectors - 1) / a.tile_vectors, y = (p.q_len + a.tile_rows - 1) / a.tile_rows;
    if (x > 0x7fffffffll || y > 65535) {
        // (2^30 rows of 64 do not fit a grid's second dimension)
        return report(CAME_ERR_SHAPE, "q_len is beyond 65535 tiles of 64 rows: call for parts of it");
    }
    const size_t length = (a.tile_rows + N * a.tile_vectors + N + N - 1) / N * N;
    k_posbias_forward<T, M><<<dim3(static_cast<unsigned>(x), static_cast<unsigned>(y), p.heads), 256, length * 16, stream>>>(a, b);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? CAME_OK : report_cuda(e, "kernel launch");
}

template <typename T, int M>
cudaError_t launch_backward(const BiasArgs& a, const came_posbias& d, const BackwardPlan& p, cudaStream_t stream)
{
    Buckets<M> b;
    fill_buckets(d, b);
    const dim3 grid(static_cast<unsigned>((p.units + kWarps - 1) / kWarps), a.heads);
    k_posbias_backward<T, M><<<grid, kWarps * 32, 0, stream>>>(a, b);
    return cudaGetLastError();
}

bool few_buckets(const came_posbias& p) { return p.buckets <= kFewBuckets; }

}  // namespace

extern "C" {

came_status came_posbias_bucket(const came_posbias* p, int64_t relative, int32_t* out)
{
    if (!p || !out) return report(CAME_ERR_NULL, "descriptor and out are required");
    const came_status s = validate_buckets(*p);
    if (s != CAME_OK) return s;
    Buckets<kMostBuckets> b;
    fill_buckets(*p, b);
    const long long d = distance_of(std::max<int64_t>(-kFar, std::min<int64_t>(kFar, relative)), b.both);
    const int m = static_cast<int>(std::upper_bound(b.start, b.start + b.n, d) - b.start) - 1;
    *out = m + (b.both && relative > 0 ? b.n : 0);
    return CAME_OK;
}

came_status came_posbias_forward(const came_posbias* p, int32_t device, void* cuda_stream)
{
    came_status s = validate_posbias(p, false);
    if (s != CAME_OK) return s;
    if ((s = require_current_device(device)) != CAME_OK) return s;
    if (!p->q_len || !p->k_len) return CAME_OK;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (few_buckets(*p))
        return p->data_dtype == CAME_BF16 ? launch_forward<__nv_bfloat16, kFewBuckets>(*p, stream) : launch_forward<float, kFewBuckets>(*p, stream);
    return p->data_dtype == CAME_BF16 ? launch_forward<__nv_bfloat16, kMostBuckets>(*p, stream) : launch_forward<float, kMostBuckets>(*p, stream);
}

came_status came_posbias_workspace(const came_posbias* p, int64_t* out_bytes)
{
    if (!out_bytes) return report(CAME_ERR_NULL, "out_bytes is NULL");
    const came_status s = validate_posbias(p, true);
    if (s != CAME_OK) return s;
    *out_bytes = std::max<int64_t>(256, plan_backward(*p).bytes);
    return CAME_OK;
}

came_status came_posbias_backward(const came_posbias* p, void* workspace, int64_t workspace_bytes, int32_t device, void* cuda_stream)
{
    came_status s = validate_posbias(p, true);
    if (s != CAME_OK) return s;
    const BackwardPlan plan = plan_backward(*p);
    if (!workspace) return report(CAME_ERR_NULL, "workspace is NULL");
    if (!aligned_to(workspace, 16)) return report(CAME_ERR_ALIGN, "workspace not 16-byte aligned");
    if (workspace_bytes < plan.bytes) return report(CAME_ERR_SHAPE, "workspace smaller than came_posbias_workspace says");
    if (plan.units > (1ll << 31)) return report(CAME_ERR_SHAPE, "too many tiles for one launch");
    if ((s = require_current_device(device)) != CAME_OK) return s;
    const bool accumulate = p->flags & CAME_POSBIAS_ACCUMULATE, empty = !p->q_len || !p->k_len || !p->batch;
    if (empty && accumulate) return CAME_OK;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    BiasArgs a = args_of(*p);
    a.part = static_cast<float*>(workspace);
    a.tile_rows = plan.tile_rows;
    a.tiles = plan.tiles;
    a.chunks = plan.chunks;
    a.batches = plan.batches;
    a.batch_groups = plan.batch_groups;
    a.period = plan.period;
    cudaError_t e = cudaSuccess;
    const bool small = p->data_dtype == CAME_BF16;
    if (!empty && few_buckets(*p))
        e = small ? launch_backward<__nv_bfloat16, kFewBuckets>(a, *p, plan, stream) : launch_backward<float, kFewBuckets>(a, *p, plan, stream);
    else if (!empty)
        e = small ? launch_backward<__nv_bfloat16, kMostBuckets>(a, *p, plan, stream) : launch_backward<float, kMostBuckets>(a, *p, plan, stream);
    if (e == cudaSuccess) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>((p->buckets + 31) / 32), p->heads);
        cfg.blockDim = dim3(1024);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, k_posbias_finish, a, empty ? 0ll : plan.units, accumulate ? 1 : 0);
        if (e == cudaSuccess) e = cudaGetLastError();
    }
    return e == cudaSuccess ? CAME_OK : report_cuda(e, "kernel launch");
}

}  // extern "C"
