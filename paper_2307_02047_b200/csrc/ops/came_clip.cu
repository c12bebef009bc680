// Global gradient norm over a list of tensors, and clipping.
//
//   n_i  = |s| sqrt(sum_j g_ij^2),   N = sqrt(sum_i n_i^2)
//   coef = 1 if N + eps <= max_norm, else max_norm / (N + eps)
//   out_ij = rn(fl(g_ij * fl(fl(s) * coef)))      fl: rounded to fp32, rn: to the output's type
//
// One grid reads every gradient once: a block per tile of one tensor, the tile's sum of squares
// in fp32 for up to 32 terms and in double from there on.  The sums are finished
// without waiting: the last tile of a tensor to arrive adds that tensor's partials, the last
// tensor adds the tensors', both in a fixed order, so results do not depend on timing.
//
// Bound by the bytes: 13.5 GB of bf16 in 1812 us (7.4 TB/s, 1.14 of the measured copy rate, which also
// writes), 436 MB of fp32 in 71 us (6.1 TB/s); a set of 0.5 MB takes 4.5 us on the device, a
// chain of dependent round trips.  Writing clipped copies reads a set larger than the L2 twice: 709 MB
// bf16 to bf16 in 337 us, 6.0 TB/s of the 2.03 GB that move.
#include "came_ops.cuh"

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
#include <vector>

namespace {

using namespace came_ops;

constexpr int kThreads = 256;
constexpr int kApplyTile = 64 << 10;     // bytes of gradient per block when the outputs are written
constexpr int kApplyUnroll = 2;          // groups of 8 elements in flight per thread when the outputs are written
constexpr int kFlatTiles = 512, kFlatTensors = 64;
constexpr int kWideTile = 128 << 10;     // from this tile size on the norm has eight 32-byte loads in flight per thread, else four

struct ClipTensor {
    const void* g;
    void*       out;
    long long   n;
    int         g_bf16, out_bf16;
    int         tile0, ntiles;           // this tensor's range of the tile list
    int         tile_elems, vec_out;     // vec_out: out can be written in groups of 8
    int         in_place;                // out is the gradient buffer, also after it moves
};

struct ClipTile { int tensor, index; };

struct ClipConsts { double max_norm, eps, scale; };

// ws: partial sums of squares per tile, then per tensor
struct ClipWork {
    double*   tile_sum;     // [tiles]
    double*   tensor_sum;   // [n]
    unsigned* arrived;      // [n] tiles of a tensor that have arrived, [1] finished tensors
};

template <typename T> struct Pack;       // 32 bytes of gradient
template <> struct Pack<float> {
    static constexpr int N = 8;
    float x[8];
    __device__ __forceinline__ void load(const float* p)
    {
        asm volatile("ld.global.nc.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]),
                       "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(p));
    }
    __device__ __forceinline__ void clear() { for (int j = 0; j < 8; ++j) x[j] = 0.f; }
    __device__ __forceinline__ void add_squares(float (&a)[4]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j & 3] = fmaf(x[j], x[j], a[j & 3]);
    }
};
template <> struct Pack<__nv_bfloat16> {
    static constexpr int N = 16;
    uint32_t w[8];
    __device__ __forceinline__ void load(const __nv_bfloat16* p)
    {
        asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]),
                       "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
    }
    __device__ __forceinline__ void clear() { for (int j = 0; j < 8; ++j) w[j] = 0u; }
    __device__ __forceinline__ void add_squares(float (&a)[4]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)                      // bf16 factors, fp32 sum, without unpacking
            asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; fma.rn.f32.bf16 %0, l, l, %0; fma.rn.f32.bf16 %1, h, h, %1; }"
                : "+f"(a[(2 * j) & 3]), "+f"(a[(2 * j + 1) & 3]) : "r"(w[j]));
    }
};

// The elements of one tile: [a, b) is the body, whose start is aligned to `group` elements;
// tile 0 also owns the `head` elements before the tensor's first aligned address.
struct Span { long long a, b; int head; };

template <typename T>
__device__ __forceinline__ Span span_of(const ClipTensor& d, const T* g, int index, int group)
{
    Span s;
    const int off = static_cast<int>((reinterpret_cast<uintptr_t>(g) / sizeof(T)) % group);
    const long long head = min(d.n, static_cast<long long>(off ? group - off : 0));
    s.a = min(d.n, head + static_cast<long long>(index) * d.tile_elems);
    // the list has ceil(n / tile_elems) tiles, so the last one always reaches the end
    s.b = min(d.n, s.a + d.tile_elems);
    s.head = index == 0 ? static_cast<int>(head) : 0;
    return s;
}

// Sum of squares of this thread's share of the tile.  At most 32 squares (and one of the tile's ragged
// ends) go into one fp32 accumulator: what follows is added in double.  Tiles of up to 64 KB have no more than
// that; of larger ones (kUnroll 8) every batch starts anew.  Longer chains lose more than their length
// suggests: the square of a bf16 has so few bits that roundings of one sign prevail (normal values:
// the sum is low by 2.5e-7 at 256 squares, 2e-8 at 32), and squares below half a spacing vanish.
template <int kUnroll, typename T>
__device__ __forceinline__ double tile_squares(const ClipTensor& d, int index)
{
    constexpr int N = Pack<T>::N;
    constexpr bool kAnew = kUnroll == 8;
    const T* const g = static_cast<const T*>(d.g);
    const Span s = span_of<T>(d, g, index, N);
    const int tid = threadIdx.x;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    double sum = 0.0;                                    // of the batches before
    auto joined = [&] { return static_cast<double>((acc[0] + acc[1]) + (acc[2] + acc[3])); };
    const int packs = static_cast<int>((s.b - s.a) / N);
    const T* const body = g + s.a;
    int k = tid;
    for (; k + (kUnroll - 1) * kThreads < packs; k += kUnroll * kThreads) {
        Pack<T> p[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) p[u].load(body + static_cast<long long>(k + u * kThreads) * N);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) p[u].add_squares(acc);
        if constexpr (kAnew) {
            sum += joined();
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = 0.f;
        }
    }
    {
        Pack<T> p[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (k + u * kThreads < packs) p[u].load(body + static_cast<long long>(k + u * kThreads) * N);
            else p[u].clear();
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) p[u].add_squares(acc);
    }
    if (tid < s.head) {
        const float x = to_float(g[tid]);
        acc[0] = fmaf(x, x, acc[0]);
    }
    const long long rest = s.a + static_cast<long long>(packs) * N + tid;
    if (rest < s.b) {
        const float x = to_float(g[rest]);
        acc[1] = fmaf(x, x, acc[1]);
    }
    sum += joined();
    if (isfinite(sum)) return sum;
    // An element beyond 1.8e19 overflows an fp32 square although the norm is finite: the
    // thread adds its share once more, in double.  (Inf and NaN come out as they are.)
    double wide = 0.0;
    for (int q = tid; q < packs; q += kThreads)
        for (int j = 0; j < N; ++j) {
            const double x = to_float(body[static_cast<long long>(q) * N + j]);
            wide += x * x;
        }
    if (tid < s.head) { const double x = to_float(g[tid]); wide += x * x; }
    if (rest < s.b) { const double x = to_float(g[rest]); wide += x * x; }
    return wide;
}

__device__ __forceinline__ void store_total(double sum, const ClipConsts& hc, float* results)
{
    const double norm = fabs(hc.scale) * sqrt(sum);
    const double reach = norm + hc.eps;
    results[0] = static_cast<float>(norm);
    results[1] = static_cast<float>(reach <= hc.max_norm ? 1.0 : hc.max_norm / reach);   // NaN stays NaN
}

// A warp's sum of count values that other blocks have written.
__device__ __forceinline__ double warp_sum_of(const double* p, int count, int lane)
{
    constexpr int B = 8;                                 // loads of one round trip
    double s = 0.0;
    for (int k = lane; k < count; k += B * 32) {
        double v[B];
#pragma unroll
        for (int u = 0; u < B; ++u) v[u] = k + u * 32 < count ? __ldcg(p + k + u * 32) : 0.0;
#pragma unroll
        for (int u = 0; u < B; ++u) s += v[u];
    }
    return warp_sum(s);
}

// kFlat: one count of arrivals, and the last block finishes everything, a warp per tensor.  It
// saves a round of store, fence and atomic (1.5 us of a small call), but one block reads
// all partial sums: for lists of up to kFlatTiles tiles.  Else the last tile of each tensor adds the
// tensor's sums, and the last tensor the tensors'.
//
// Resident blocks: sets of a thousand tiles want them in one wave (32 MB: 12.6 us with seven per SM, 14.0 with
// six); larger ones are better off with five that need no spilled registers (436 MB: 70.7 against 74.2).
template <bool kFlat, int kUnroll>
__global__ void __launch_bounds__(kThreads, kUnroll == 4 ? 7 : 5)
k_clip_norm(const ClipTensor* __restrict__ T, const ClipTile* __restrict__ tiles, int n, ClipWork w,
            ClipConsts hc, float* __restrict__ results)
{
    __shared__ double red[kThreads / 32];
    __shared__ unsigned s_last;
    const ClipTile t = tiles[blockIdx.x];
    const ClipTensor d = T[t.tensor];
    double s = d.g_bf16 ? tile_squares<kUnroll, __nv_bfloat16>(d, t.index) : tile_squares<kUnroll, float>(d, t.index);
    release_dependents();                                // (earlier, waiting blocks would hold the SMs)
    s = warp_sum(s);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) red[warp] = s;
    __syncthreads();
    const double scale = fabs(hc.scale);
    if constexpr (kFlat) {
        if (threadIdx.x == 0) {
            s = 0.0;
            for (int k = 0; k < kThreads / 32; ++k) s += red[k];
            w.tile_sum[blockIdx.x] = s;
            publish();
            s_last = atomicAdd(&w.arrived[n], 1u) == gridDim.x - 1u;
            publish();
        }
        __syncthreads();
        if (!s_last) return;
        double total = 0.0;                              // of this warp's tensors, in their order
        for (int k = warp; k < n; k += kThreads / 32) {
            const int tile0 = T[k].tile0, ntiles = T[k].ntiles;
            s = warp_sum_of(w.tile_sum + tile0, ntiles, lane);
            if (lane == 0) results[2 + k] = static_cast<float>(scale * sqrt(s));
            total += s;
        }
        if (lane == 0) red[warp] = total;
        __syncthreads();
        if (threadIdx.x == 0) {
            w.arrived[n] = 0u;
            s = 0.0;
            for (int k = 0; k < kThreads / 32; ++k) s += red[k];
            store_total(s, hc, results);
        }
    } else {
        if (warp > 0) return;
        // one warp: arrive, and finish the tensor / the whole list when last
        unsigned last = 1;
        if (lane == 0) {
            s = 0.0;
            for (int k = 0; k < kThreads / 32; ++k) s += red[k];
            if (d.ntiles > 1) {
                w.tile_sum[blockIdx.x] = s;
                publish();
                last = atomicAdd(&w.arrived[t.tensor], 1u) == static_cast<unsigned>(d.ntiles - 1);
                publish();
            }
        }
        if (d.ntiles > 1) {                              // (a tensor of one tile is finished)
            last = __shfl_sync(0xffffffffu, last, 0);
            __syncwarp();                                // lane 0's fence holds for the warp's reads (a shuffle orders no memory)
            if (!last) return;
            s = warp_sum_of(w.tile_sum + d.tile0, d.ntiles, lane);
        }
        if (lane == 0) {
            w.arrived[t.tensor] = 0u;
            w.tensor_sum[t.tensor] = s;
            results[2 + t.tensor] = static_cast<float>(scale * sqrt(s));
            publish();
            last = atomicAdd(&w.arrived[n], 1u) == static_cast<unsigned>(n - 1);
            publish();
        }
        last = __shfl_sync(0xffffffffu, last, 0);
        __syncwarp();
        if (!last) return;
        s = warp_sum_of(w.tensor_sum, n, lane);
        if (lane == 0) {
            w.arrived[n] = 0u;
            store_total(s, hc, results);
        }
    }
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
        asm volatile("ld.global.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]),
                       "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(p));
    } else {
        uint32_t w[4];
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
        asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     :: "l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]),
                        "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
    } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(x[2 * j + 1]), "f"(x[2 * j]));
        asm volatile("st.global.cs.v4.b32 [%0], {%1,%2,%3,%4};"
                     :: "l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
}

template <typename T, typename O>
__device__ __forceinline__ void apply_tile(const ClipTensor& d, int index, int part, int parts, float f)
{
    const T* const g = static_cast<const T*>(d.g);
    O* const out = static_cast<O*>(d.out);
    const int tid = threadIdx.x;
    // groups of 8 elements: 16 bytes of bf16, 32 of fp32
    Span s = span_of<T>(d, g, index, 8);
    const long long size = d.tile_elems / parts;         // a multiple of 8: tiles are powers of two
    s.a = min(s.b, s.a + part * size);
    s.b = min(s.b, s.a + size);
    if (part > 0) s.head = 0;
    if (d.vec_out) {
        const int packs = static_cast<int>((s.b - s.a) / 8);
        for (int k = tid; k < packs; k += kApplyUnroll * kThreads) {
            float x[kApplyUnroll][8];
#pragma unroll
            for (int u = 0; u < kApplyUnroll; ++u)
                if (k + u * kThreads < packs) load8<T>(g + s.a + static_cast<long long>(k + u * kThreads) * 8, x[u]);
#pragma unroll
            for (int u = 0; u < kApplyUnroll; ++u)
                if (k + u * kThreads < packs) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[u][j] *= f;
                    store8<O>(out + s.a + static_cast<long long>(k + u * kThreads) * 8, x[u]);
                }
        }
        const long long rest = s.a + static_cast<long long>(packs) * 8 + tid;
        if (rest < s.b) out[rest] = from_float<O>(to_float(g[rest]) * f);
    } else {
        // in and out start at different offsets of a 32-byte (16-byte) line
        for (long long k = s.a + tid; k < s.b; k += kThreads) out[k] = from_float<O>(to_float(g[k]) * f);
    }
    if (tid < s.head) out[tid] = from_float<O>(to_float(g[tid]) * f);
}

// A block per kApplyTile bytes.  They are walked backwards: the norm's grid has just read the last ones, so they come from the L2.
__global__ void __launch_bounds__(kThreads)
k_clip_apply(const ClipTensor* __restrict__ T, const ClipTile* __restrict__ tiles, int parts, float scale,
             const float* __restrict__ results)
{
    const unsigned at = gridDim.x - 1u - blockIdx.x;
    const ClipTile t = tiles[at / parts];
    const int part = static_cast<int>(at % parts);
    const ClipTensor d = T[t.tensor];
    wait_for_previous_grid();
    const float f = scale * __ldcg(results + 1);
    if (d.out == d.g && f == 1.f) return;            // in place and nothing to do
    if (d.g_bf16) {
        if (d.out_bf16) apply_tile<__nv_bfloat16, __nv_bfloat16>(d, t.index, part, parts, f);
        else            apply_tile<__nv_bfloat16, float>(d, t.index, part, parts, f);
    } else {
        if (d.out_bf16) apply_tile<float, __nv_bfloat16>(d, t.index, part, parts, f);
        else            apply_tile<float, float>(d, t.index, part, parts, f);
    }
}

}  // namespace

struct came_clip_ctx {
    int device = 0, n = 0, ntiles = 0, tile_bytes = 0;
    bool has_out = true;                    // no tensor with elements lacks an output
    std::vector<ClipTensor> table;
    char*       d_mem = nullptr;            // table | tiles | sums | counters
    ClipTensor* d_table = nullptr;
    ClipTile*   d_tiles = nullptr;
    ClipWork    work = {};
    // staging of the table when gradients move, made at the first move; two slots, taken in turn, so
    // that a call does not wait for the copy of the call before it
    ClipTensor* pinned[2] = {nullptr, nullptr};
    cudaEvent_t pinned_free[2] = {nullptr, nullptr};
    bool        pinned_used[2] = {false, false};
    int         pinned_next = 0;
};

namespace {

void free_clip(came_clip_ctx* c)
{
    if (!c) return;
    cudaFree(c->d_mem);
    if (c->pinned[0]) cudaFreeHost(c->pinned[0]);
    for (cudaEvent_t e : c->pinned_free)
        if (e) cudaEventDestroy(e);
    delete c;
}

// Whether `out` can be written in groups of 8 wherever `grad` is read in groups of 8.
bool groups_agree(const ClipTensor& d)
{
    const size_t gs = d.g_bf16 ? 2 : 4, os = d.out_bf16 ? 2 : 4;
    return (reinterpret_cast<uintptr_t>(d.g) / gs) % 8 == (reinterpret_cast<uintptr_t>(d.out) / os) % 8;
}

came_status tensor_error(came_status s, int i, const char* what)
{
    char buf[160];
    std::snprintf(buf, sizeof buf, "tensor %d: %s", i, what);
    return report(s, buf);
}

// An output may be its own gradient buffer; it may share memory with nothing else.
came_status check_overlap(const came_clip_tensor* t, int n)
{
    struct Range { uintptr_t lo, hi; int tensor; bool out; };
    std::vector<Range> rs;
    rs.reserve(2 * static_cast<size_t>(n));
    for (int i = 0; i < n; ++i) {
        if (!t[i].numel) continue;
        const uintptr_t g = reinterpret_cast<uintptr_t>(t[i].grad), o = reinterpret_cast<uintptr_t>(t[i].out);
        const uintptr_t gb = t[i].numel * dtype_bytes(t[i].grad_dtype), ob = t[i].numel * dtype_bytes(t[i].out_dtype);
        const bool in_place = o == g && t[i].grad_dtype == t[i].out_dtype;
        if (!in_place) rs.push_back(Range{g, g + gb, i, false});
        if (o) rs.push_back(Range{o, o + ob, i, true});
    }
    std::sort(rs.begin(), rs.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
    uintptr_t reach = 0, reach_out = 0;      // furthest end of any range / of any output so far
    for (const Range& r : rs) {
        if (r.lo < reach_out || (r.out && r.lo < reach))
            return tensor_error(CAME_ERR_OVERLAP, r.tensor, "an output shares memory with another buffer");
        reach = std::max(reach, r.hi);
        if (r.out) reach_out = std::max(reach_out, r.hi);
    }
    return CAME_OK;
}

came_status validate_clip(const came_clip_tensor* t, int n)
{
    bool any_out = false, all_out = true;
    for (int i = 0; i < n; ++i) {
        const came_clip_tensor& x = t[i];
        if (x.numel < 0 || x.numel > (1ll << 40)) return tensor_error(CAME_ERR_SHAPE, i, "numel out of range");
        if (!known_dtype(x.grad_dtype)) return tensor_error(CAME_ERR_DTYPE, i, "unknown grad_dtype");
        if (x.numel && !x.grad) return tensor_error(CAME_ERR_NULL, i, "grad is required");
        if (!aligned_to(x.grad, dtype_bytes(x.grad_dtype)))
            return tensor_error(CAME_ERR_ALIGN, i, "grad not aligned to its element size");
        if (x.out) {
            any_out = true;
            if (!known_dtype(x.out_dtype)) return tensor_error(CAME_ERR_DTYPE, i, "unknown out_dtype");
            if (!aligned_to(x.out, dtype_bytes(x.out_dtype)))
                return tensor_error(CAME_ERR_ALIGN, i, "out not aligned to its element size");
        } else if (x.numel) {
            all_out = false;
        }
    }
    if (any_out && !all_out)
        return report(CAME_ERR_NULL, "either every tensor has an output or none has");
    return check_overlap(t, n);
}

came_status validate_clip_params(const came_clip_params& p)
{
    if (!(p.max_norm > 0)) return report(CAME_ERR_HPARAM, "max_norm must be > 0 (infinity: never clip)");
    if (!std::isfinite(p.eps) || p.eps < 0) return report(CAME_ERR_HPARAM, "eps must be finite and >= 0");
    if (!std::isfinite(p.grad_scale) || p.grad_scale < 0)
        return report(CAME_ERR_HPARAM, "grad_scale must be finite and > 0 (or 0 for 1)");
    return CAME_OK;
}

// Bytes of gradient per tile.  Up to 64 KB: about a thousand tiles, one wave of blocks (32 MB of fp32 took
// 12.2 us, against 14.6 with twice and 13.1 with half as many).  Above: about two thousand of up to
// 512 KB, whose threads have eight loads in flight (436 MB: 70 us, against 76 with 64 KB tiles and four loads).
int tile_bytes_for(double total_bytes)
{
    long long bytes = 16 << 10;
    while (bytes < (64 << 10) && 2.0 * bytes * 592 <= total_bytes) bytes *= 2;
    while (bytes >= (64 << 10) && bytes < (512 << 10) && 2.0 * bytes * 1184 <= total_bytes) bytes *= 2;
    return static_cast<int>(bytes);
}

// The rule of check_overlap for the list that replacing the gradients would make.
came_status check_moved(const came_clip_ctx* c, const void* const* grads)
{
    if (!c->has_out) return CAME_OK;
    try {
        std::vector<came_clip_tensor> t(c->n);
        for (int i = 0; i < c->n; ++i) {
            const ClipTensor& d = c->table[i];
            t[i].grad = grads[i];
            t[i].out = d.in_place ? const_cast<void*>(grads[i]) : d.out;
            t[i].numel = d.n;
            t[i].grad_dtype = d.g_bf16 ? CAME_BF16 : CAME_F32;
            t[i].out_dtype = d.out_bf16 ? CAME_BF16 : CAME_F32;
        }
        return check_overlap(t.data(), c->n);
    } catch (const std::bad_alloc&) {
        return report(CAME_ERR_OOM, "host allocation failed");
    }
}

came_status rebind(came_clip_ctx* c, const void* const* grads, cudaStream_t stream)
{
    bool moved = false;
    for (int i = 0; i < c->n; ++i) {
        const ClipTensor& d = c->table[i];
        if (d.n && !grads[i]) return tensor_error(CAME_ERR_NULL, i, "grad is required");
        if (!aligned_to(grads[i], d.g_bf16 ? 2 : 4))
            return tensor_error(CAME_ERR_ALIGN, i, "grad not aligned to its element size");
        moved |= d.g != grads[i];
    }
    if (!moved) return CAME_OK;
    const came_status s = check_moved(c, grads);
    if (s != CAME_OK) return s;
    // A captured copy would run at the graph's replay, out of the staging buffer as it is then, while
    // the table here would count as copied from now on.
    cudaStreamCaptureStatus capture;
    cudaError_t e = cudaStreamIsCapturing(stream, &capture);
    if (e == cudaErrorStreamCaptureImplicit || (e == cudaSuccess && capture != cudaStreamCaptureStatusNone)) {
        cudaGetLastError();
        return report(CAME_ERR_UNSUPPORTED, "gradients cannot be replaced while the stream captures");
    }
    if (e != cudaSuccess) return report_cuda(e, "cudaStreamIsCapturing");
    if (!c->pinned[0]) {
        for (cudaEvent_t& free : c->pinned_free)
            if (!free && (e = cudaEventCreateWithFlags(&free, cudaEventDisableTiming)) != cudaSuccess)
                return report_cuda(e, "cudaEventCreate");
        if ((e = cudaMallocHost(&c->pinned[0], 2 * sizeof(ClipTensor) * c->n)) != cudaSuccess) {
            c->pinned[0] = nullptr;
            return report_cuda(e, "cudaMallocHost(table)");
        }
        c->pinned[1] = c->pinned[0] + c->n;
    }
    const int k = c->pinned_next;
    if (c->pinned_used[k] && (e = cudaEventSynchronize(c->pinned_free[k])) != cudaSuccess)
        return report_cuda(e, "cudaEventSynchronize(table)");
    ClipTensor* const to = c->pinned[k];
    std::copy(c->table.begin(), c->table.end(), to);
    for (int i = 0; i < c->n; ++i) {
        to[i].g = grads[i];
        if (to[i].in_place) to[i].out = const_cast<void*>(grads[i]);
        to[i].vec_out = groups_agree(to[i]);
    }
    e = cudaMemcpyAsync(c->d_table, to, sizeof(ClipTensor) * c->n, cudaMemcpyHostToDevice, stream);
    if (e != cudaSuccess) return report_cuda(e, "cudaMemcpyAsync(table)");
    // from here on the device has, or will have, these: what is kept here never runs ahead of it
    std::copy(to, to + c->n, c->table.begin());
    if ((e = cudaEventRecord(c->pinned_free[k], stream)) != cudaSuccess) {
        cudaStreamSynchronize(stream);      // (nothing would tell when the slot is free)
        return report_cuda(e, "cudaEventRecord(table)");
    }
    c->pinned_used[k] = true;
    c->pinned_next = k ^ 1;
    return CAME_OK;
}

came_status run_clip(came_clip_ctx* c, const came_clip_params* p, const void* const* grads, float* results,
                     cudaStream_t stream, bool apply)
{
    if (!c || !p || !results) return report(CAME_ERR_NULL, "context, parameters and results are required");
    if (!aligned_to(results, 4)) return report(CAME_ERR_ALIGN, "results not 4-byte aligned");
    came_status s = validate_clip_params(*p);
    if (s != CAME_OK) return s;
    if (apply && !holds_in_fp32(p->grad_scale))
        return report(CAME_ERR_HPARAM, "grad_scale must be finite, and not vanish, in fp32 where outputs are written");
    if (apply && !c->has_out) return report(CAME_ERR_UNSUPPORTED, "the context was created without outputs");
    if ((s = require_current_device(c->device)) != CAME_OK) return s;
    if (grads && (s = rebind(c, grads, stream)) != CAME_OK) return s;
    const double scale = p->grad_scale == 0.0 ? 1.0 : p->grad_scale;
    const ClipConsts hc{p->max_norm, p->eps, scale};
    const bool flat = c->ntiles <= kFlatTiles && c->n <= kFlatTensors;
    auto* const norm = flat ? k_clip_norm<true, 4> : c->tile_bytes < kWideTile ? k_clip_norm<false, 4> : k_clip_norm<false, 8>;
    norm<<<c->ntiles, kThreads, 0, stream>>>(c->d_table, c->d_tiles, c->n, c->work, hc, results);
    if (apply) {
        cudaLaunchConfig_t cfg = {};
        const int parts = std::max(1, c->tile_bytes / kApplyTile);
        cfg.gridDim = dim3(static_cast<unsigned>(c->ntiles) * parts);
        cfg.blockDim = dim3(kThreads);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        cudaLaunchKernelEx(&cfg, k_clip_apply, static_cast<const ClipTensor*>(c->d_table),
                           static_cast<const ClipTile*>(c->d_tiles), parts, static_cast<float>(scale),
                           static_cast<const float*>(results));
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? CAME_OK : report_cuda(e, "kernel launch");
}

}  // namespace

extern "C" {

came_status came_clip_create(came_clip_ctx** out, const came_clip_tensor* t, int32_t n, int32_t device)
{
    if (!out) return report(CAME_ERR_NULL, "out is NULL");
    *out = nullptr;
    if (!t) return report(CAME_ERR_NULL, "tensor array is NULL");
    if (n < 1 || n > (1 << 24)) return report(CAME_ERR_SHAPE, "tensor count out of range");
    came_clip_ctx* c = nullptr;
    try {
        came_status s = validate_clip(t, n);
        if (s != CAME_OK) return s;
        int ndev = 0;
        if (cudaGetDeviceCount(&ndev) != cudaSuccess || ndev < 1) {
            cudaGetLastError();
            return report(CAME_ERR_DEVICE, "no usable CUDA device");
        }
        if (device < 0 || device >= ndev) return report(CAME_ERR_DEVICE, "device ordinal out of range");
        if ((s = require_current_device(device)) != CAME_OK) return s;
        c = new came_clip_ctx;
        c->device = device;
        c->n = n;
        c->table.resize(n);
        double total = 0;
        for (int i = 0; i < n; ++i) total += static_cast<double>(t[i].numel) * dtype_bytes(t[i].grad_dtype);
        c->tile_bytes = tile_bytes_for(total);
        std::vector<ClipTile> tiles;
        for (int i = 0; i < n; ++i) {
            ClipTensor& d = c->table[i];
            std::memset(&d, 0, sizeof d);
            d.g = t[i].grad;
            d.out = t[i].out;
            d.n = t[i].numel;
            d.g_bf16 = t[i].grad_dtype == CAME_BF16;
            d.out_bf16 = t[i].out && t[i].out_dtype == CAME_BF16;
            d.vec_out = groups_agree(d);
            d.in_place = t[i].out && t[i].out == t[i].grad;
            d.tile_elems = c->tile_bytes / static_cast<int>(dtype_bytes(t[i].grad_dtype));
            const long long k = std::max(1ll, (d.n + d.tile_elems - 1) / d.tile_elems);
            if (static_cast<long long>(tiles.size()) + k > (1 << 27)) {
                free_clip(c);
                return report(CAME_ERR_SHAPE, "too many tiles");
            }
            d.tile0 = static_cast<int>(tiles.size());
            d.ntiles = static_cast<int>(k);
            for (int q = 0; q < d.ntiles; ++q) tiles.push_back(ClipTile{i, q});
            c->has_out &= t[i].out != nullptr || t[i].numel == 0;
        }
        c->ntiles = static_cast<int>(tiles.size());
        size_t bytes = 0;
        auto take = [&](size_t b) { const size_t at = bytes; bytes += (b + 255) / 256 * 256; return at; };
        const size_t at_table = take(sizeof(ClipTensor) * n), at_tiles = take(sizeof(ClipTile) * tiles.size());
        const size_t at_tile_sum = take(sizeof(double) * tiles.size()), at_tensor_sum = take(sizeof(double) * n);
        const size_t at_arrived = take(sizeof(unsigned) * (static_cast<size_t>(n) + 1));
        cudaError_t e;
#define CLIP_TRY(call, what) do { if ((e = (call)) != cudaSuccess) { free_clip(c); return report_cuda(e, what); } } while (0)
        CLIP_TRY(cudaMalloc(&c->d_mem, bytes), "cudaMalloc(clip workspace)");
        c->d_table = reinterpret_cast<ClipTensor*>(c->d_mem + at_table);
        c->d_tiles = reinterpret_cast<ClipTile*>(c->d_mem + at_tiles);
        c->work.tile_sum = reinterpret_cast<double*>(c->d_mem + at_tile_sum);
        c->work.tensor_sum = reinterpret_cast<double*>(c->d_mem + at_tensor_sum);
        c->work.arrived = reinterpret_cast<unsigned*>(c->d_mem + at_arrived);
        // one copy: the table, the tiles and (zero) everything behind them
        std::vector<char> host(bytes, 0);
        std::memcpy(host.data() + at_table, c->table.data(), sizeof(ClipTensor) * n);
        std::memcpy(host.data() + at_tiles, tiles.data(), sizeof(ClipTile) * tiles.size());
        CLIP_TRY(cudaMemcpy(c->d_mem, host.data(), bytes, cudaMemcpyHostToDevice), "cudaMemcpy(clip workspace)");
        CLIP_TRY(cudaStreamSynchronize(nullptr), "cudaStreamSynchronize");
#undef CLIP_TRY
    } catch (const std::bad_alloc&) {
        free_clip(c);
        return report(CAME_ERR_OOM, "host allocation failed");
    }
    *out = c;
    return CAME_OK;
}

came_status came_clip_norm(came_clip_ctx* ctx, const came_clip_params* p, const void* const* grads,
                           float* results, void* cuda_stream)
{
    return run_clip(ctx, p, grads, results, static_cast<cudaStream_t>(cuda_stream), false);
}

came_status came_clip_grads(came_clip_ctx* ctx, const came_clip_params* p, const void* const* grads,
                            float* results, void* cuda_stream)
{
    return run_clip(ctx, p, grads, results, static_cast<cudaStream_t>(cuda_stream), true);
}

came_status came_clip_destroy(came_clip_ctx* ctx)
{
    if (!ctx) return CAME_ERR_NULL;
    free_clip(ctx);
    return CAME_OK;
}

}  // extern "C"
