// AdamW over a list of tensors, with the states in fp32 or in 8 bits.
//
//   g = grad * s,  m = b1 m + (1-b1) g,  v = b2 v + (1-b2) g^2,
//   p = p - (lr wd p + lr mhat / (sqrt(vhat) + eps))
//
// A warp takes 256 consecutive elements of a tensor, eight per lane: the elements that share a scale
// where states have 8 bits.  Nothing crosses from one such block to the next, so there is one pass, one
// launch for each type of state and gradient in the list, and no order that could change a result.
//
// Bound by the bytes: 355 M elements with fp32 states and gradients move 9.9 GB in 1450 us (6.8 TB/s); 2^28 with 8-bit
// states, bf16 gradients and bf16 copies 4.3 GB in 655 us (6.6 TB/s, the measured copy rate).  The 8-bit form computes about 70
// instructions for an element, three quarters of what the SMs can issue in that time, a third of them for the random bits
// and the rounding; one hash serves both states.
#include "came_vec.cuh"

#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
#include <type_traits>
#include <vector>

namespace {

using namespace came_ops;

constexpr int kBlock = 256;              // elements per warp and scale
constexpr int kWarps = 8;
constexpr int kMovedPointers = 1000;     // gradient pointers that one launch carries

struct AdamwTensor {
    float*         p;
    void*          m;
    void*          v;
    uint8_t*       ms;
    uint8_t*       vs;
    __nv_bfloat16* copy;
    long long      n;
    unsigned       block0;               // number of the tensor's first block in the whole list
    int            decay;
};

struct AdamwTile { int tensor; unsigned block; };       // blocks of a tensor from `block` on, per_warp for each warp

struct AdamwConsts {
    float b1, c1, b2, c2, eps, decay, scale;
    float step, root;                    // lr / (1 - b1^t), 1 / sqrt(1 - b2^t); not used with a step on the device
    unsigned key;
    unsigned per_warp;
    double lr, log_b1, log_b2;           // used with a step on the device
    unsigned key_seed;
    const float* device_scale;
    const int64_t* device_step;
};

constexpr unsigned kGolden = 0x9E3779B9u;

__host__ __device__ __forceinline__ unsigned mix(unsigned x)
{
    x ^= x >> 16;
    x *= 0xBB67AE85u;
    x ^= x >> 15;
    x *= 0xA54FF53Bu;
    return x ^ (x >> 16);
}
__host__ __device__ __forceinline__ unsigned mix_word(unsigned k, uint64_t w)
{
    k = mix((k ^ static_cast<unsigned>(w)) + 0x3C6EF373u);
    return mix((k ^ static_cast<unsigned>(w >> 32)) + 0x3C6EF373u);
}

// kFull: also of subnormal numbers, which count as zero else.
template <bool kFull>
__device__ __forceinline__ float approx_sqrt(float x)
{
    float y;
    if constexpr (kFull) asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    else asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float approx_rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }
__device__ __forceinline__ float power_of_two(int e) { return e > 0 ? __uint_as_float(static_cast<unsigned>(e) << 23) : __uint_as_float(0x00400000u >> -e); }

// The 8-bit types: magnitudes are the upper bits of an fp32 whose exponent has been lowered by kLow, subnormal
// values included, so that adding a random number below the bits that are dropped and cutting these
// off rounds up with the right probability.
struct E4M3 {
    static constexpr bool kSigned = true;
    static constexpr int kTop = 7, kDrop = 20, kLow = 120;
    static __device__ __forceinline__ unsigned random(unsigned r) { return ((r << 4) & 0xffff0u) | 8u; }
    template <int K> static __device__ __forceinline__ uint32_t halves(uint32_t w)       // bytes K and K + 1
    {
        uint32_t h;
        if constexpr (K == 0) asm("{ .reg .b16 l, u; mov.b32 {l, u}, %1; cvt.rn.f16x2.e4m3x2 %0, l; }" : "=r"(h) : "r"(w));
        else asm("{ .reg .b16 l, u; mov.b32 {l, u}, %1; cvt.rn.f16x2.e4m3x2 %0, u; }" : "=r"(h) : "r"(w));
        return h;
    }
};
struct E5M2 {
    static constexpr bool kSigned = false;
    static constexpr int kTop = 14, kDrop = 21, kLow = 112;
    static __device__ __forceinline__ unsigned random(unsigned r) { return ((r >> 11) & 0x1fffe0u) | 16u; }
    template <int K> static __device__ __forceinline__ uint32_t halves(uint32_t w)       // an e5m2 is the upper byte of a half
    {
        return __byte_perm(w, 0, K == 0 ? 0x1404 : 0x3424);
    }
};

template <typename F>
__device__ __forceinline__ void decode8(const uint32_t (&w)[2], unsigned e, float (&x)[8])
{
    const float scale = power_of_two(static_cast<int>(e));
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const uint32_t h = k & 2 ? F::template halves<2>(w[k >> 2]) : F::template halves<0>(w[k >> 2]);
        const __half2 two = *reinterpret_cast<const __half2*>(&h);
        x[k] = __low2float(two) * scale;
        x[k + 1] = __high2float(two) * scale;
    }
}

// Codes of a block's values (x: this lane's eight; r: their random bits), and the byte of its scale.
template <typename F>
__device__ __forceinline__ unsigned encode8(const float (&x)[8], const unsigned (&r)[8], uint32_t (&w)[2])
{
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = max_nan(most, fabsf(x[k]));
    unsigned top = __reduce_max_sync(0xffffffffu, __float_as_uint(most));
    const bool special = top >= 0x7f800000u;             // an infinity or a NaN somewhere in the block
    if (special) {
        most = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(x[k]) < INFINITY ? fabsf(x[k]) : 0.f);
        top = __reduce_max_sync(0xffffffffu, __float_as_uint(most));
    }
    const int e = max(static_cast<int>(top >> 23) - F::kTop, 0);
    // One factor scales and lowers the exponent: 2^(127 - e - kLow), also where it is subnormal.  Of blocks whose values are
    // so large that it would vanish, 2^-96 is taken first, which leaves at least 2^-144 (e4m3, e = 247) for the largest fp32.  What
    // that loses are values below 2^-30 in a block whose codes' last random bit is worth 2^5 or more.
    int power = 254 - e - F::kLow;
    float first = 1.f;
    if (power < -22) {
        first = 0x1p-96f;
        power += 96;
    }
    const float factor = power_of_two(power);
    uint32_t c[8];                                       // codes in the upper byte
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float z = first == 1.f ? fabsf(x[k]) : fabsf(x[k]) * first;
        unsigned s = __float_as_uint(z * factor) + F::random(r[k]);
        if constexpr (F::kSigned) {
            c[k] = ((s << (24 - F::kDrop)) & 0x7f000000u) | (__float_as_uint(x[k]) & 0x80ffffffu);
        } else {
            if (x[k] > 0.f) s = max(s, 1u << F::kDrop);          // not zero (subnormal values neither): not stored as zero
            c[k] = s << (24 - F::kDrop);
        }
    }
    if (special) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (fabsf(x[k]) < INFINITY) continue;
            c[k] = !F::kSigned && x[k] == INFINITY ? 0x7c000000u : 0x7f000000u;
        }
    }
#pragma unroll
    for (int k = 0; k < 8; k += 4)
        w[k >> 2] = __byte_perm(__byte_perm(c[k], c[k + 1], 0x73), __byte_perm(c[k + 2], c[k + 3], 0x73), 0x5410);
    return static_cast<unsigned>(e);
}

// One element's new p, from its old p, its gradient and its states, which become the new ones.
template <bool kFull>
struct Update {
    float b1, c1, b2, c2, eps, step, root, decay, scale;
    __device__ __forceinline__ float operator()(float p, float g, float& m, float& v) const
    {
        g = __fmul_rn(g, scale);
        m = __fadd_rn(__fmul_rn(b1, m), __fmul_rn(c1, g));
        v = __fadd_rn(__fmul_rn(b2, v), __fmul_rn(c2, __fmul_rn(g, g)));
        const float u = m * approx_rcp(fmaf(approx_sqrt<kFull>(v), root, eps));
        return p - fmaf(step, u, decay * p);
    }
};

// A block as it is stored, eight elements per lane side by side: what a warp has in flight.
template <int BITS, typename G>
struct Stored {
    using S = typename std::conditional<BITS == 32, float, uint8_t>::type;
    Vec<G, 8> g;
    Vec<S, 8> m, v;
    Vec<float, 8> p;
    __device__ __forceinline__ void load(const AdamwTensor& d, const G* grad, unsigned block)
    {
        const long long at = static_cast<long long>(block) * kBlock + 8 * (threadIdx.x & 31);
        g.load(grad + at);
        m.load(static_cast<const S*>(d.m) + at);
        v.load(static_cast<const S*>(d.v) + at);
        p.load(d.p + at);
    }
};

// Updates one block.  kWide: all 256 elements are there, aligned, and loaded; else lane l takes the elements
// l, l + 32, ... of the `left` ones one by one.  `scales`: the bytes of m (low) and v, which become the new ones.
template <int BITS, typename G, bool kFull, bool kWide>
__device__ __forceinline__ void adamw_block(const AdamwTensor& d, const G* grad, const Stored<BITS, G>& in, unsigned block, int left,
                                            const Update<kFull>& f, unsigned key, unsigned& scales)
{
    using S = typename Stored<BITS, G>::S;
    const int lane = threadIdx.x & 31, first = kWide ? 8 * lane : lane, next = kWide ? 1 : 32;
    const long long at = static_cast<long long>(block) * kBlock + first;
    float* const pp = d.p + at;
    S* const pm = static_cast<S*>(d.m) + at;
    S* const pv = static_cast<S*>(d.v) + at;
    float p[8], g[8], m[8], v[8];
    uint32_t wm[2] = {0u, 0u}, wv[2] = {0u, 0u};
    if constexpr (kWide) {
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = in.g.value(k), p[k] = in.p.value(k);
        if constexpr (BITS == 32) {
#pragma unroll
            for (int k = 0; k < 8; ++k) m[k] = in.m.value(k), v[k] = in.v.value(k);
        } else {
            wm[0] = in.m.w[0], wm[1] = in.m.w[1], wv[0] = in.v.w[0], wv[1] = in.v.w[1];
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool there = first + 32 * k < left;
            p[k] = there ? pp[32 * k] : 0.f;
            g[k] = there ? to_float(grad[at + 32 * k]) : 0.f;
            if constexpr (BITS == 32) {
                m[k] = there ? pm[32 * k] : 0.f;
                v[k] = there ? pv[32 * k] : 0.f;
            } else if (there) {
                wm[k >> 2] |= static_cast<uint32_t>(pm[32 * k]) << (8 * (k & 3));
                wv[k >> 2] |= static_cast<uint32_t>(pv[32 * k]) << (8 * (k & 3));
            }
        }
    }
    if constexpr (BITS == 8) {
        decode8<E4M3>(wm, scales & 255u, m);
        decode8<E5M2>(wv, scales >> 8, v);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = f(p[k], g[k], m[k], v[k]);
    if constexpr (BITS == 8) {
        unsigned r[8];
        const unsigned base = mix(key + (d.block0 + block) * kGolden) + static_cast<unsigned>(first) * kGolden;
#pragma unroll
        for (int k = 0; k < 8; ++k) r[k] = mix(base + static_cast<unsigned>(k * next) * kGolden);
        if constexpr (!kWide) {          // elements behind the end stay out of the scales
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (first + 32 * k >= left) m[k] = v[k] = 0.f;
        }
        scales = encode8<E4M3>(m, r, wm);
        scales |= encode8<E5M2>(v, r, wv) << 8;
        if constexpr (kWide) {
            *reinterpret_cast<uint2*>(pm) = make_uint2(wm[0], wm[1]);
            *reinterpret_cast<uint2*>(pv) = make_uint2(wv[0], wv[1]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (first + 32 * k < left) {
                    pm[32 * k] = static_cast<uint8_t>(wm[k >> 2] >> (8 * (k & 3)));
                    pv[32 * k] = static_cast<uint8_t>(wv[k >> 2] >> (8 * (k & 3)));
                }
        }
    } else if constexpr (kWide) {
        Vec<float, 8> x;
        x.set(m);
        x.store(pm);
        x.set(v);
        x.store(pv);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (first + 32 * k < left) pm[32 * k] = m[k], pv[32 * k] = v[k];
    }
    if constexpr (kWide) {
        Vec<float, 8> x;
        x.set(p);
        x.store(pp);
        if (d.copy) {
            Vec<__nv_bfloat16, 8> c;
            c.set(p);
            c.store(d.copy + at);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (first + 32 * k < left) {
                pp[32 * k] = p[k];
                if (d.copy) d.copy[at + 32 * k] = __float2bfloat16_rn(p[k]);
            }
    }
}

// 8 bits: registers for three blocks per SM (2^28 elements with bf16 gradients and copies: 655 us, against 742 with two and 682
// with four, whose registers do not hold the block that is on its way; fp32 gradients, no copies: 636, 712 and 797).
template <int BITS, typename G, bool kFull>
__global__ void __launch_bounds__(kWarps * 32, BITS == 8 ? 3 : 1)
k_adamw(const AdamwTensor* __restrict__ table, const void* const* __restrict__ grads, const AdamwTile* __restrict__ tiles,
        const __grid_constant__ AdamwConsts c)
{
    __shared__ float s_step, s_root;
    __shared__ unsigned s_key;
    const AdamwTile tile = tiles[blockIdx.x];
    const AdamwTensor d = table[tile.tensor];
    const G* const grad = static_cast<const G*>(grads[tile.tensor]);
    Update<kFull> f{c.b1, c.c1, c.b2, c.c2, c.eps, c.step, c.root, d.decay ? c.decay : 0.f, c.scale};
    unsigned key = c.key;
    if (c.device_scale) f.scale = __fmul_rn(f.scale, *c.device_scale);
    if (c.device_step) {
        if (threadIdx.x == 0) {
            const long long t = max(1ll, static_cast<long long>(*c.device_step));
            s_step = static_cast<float>(c.lr / -expm1(static_cast<double>(t) * c.log_b1));
            s_root = static_cast<float>(1.0 / sqrt(-expm1(static_cast<double>(t) * c.log_b2)));
            s_key = mix_word(c.key_seed, static_cast<uint64_t>(t));
        }
        __syncthreads();
        f.step = s_step;
        f.root = s_root;
        key = s_key;
    }
    // The block's warps take turns: neighbouring blocks at the same time (64 M elements: 181 us, against 198 with
    // each warp's blocks side by side).
    const int lane = threadIdx.x & 31;
    const unsigned blocks = static_cast<unsigned>((d.n + kBlock - 1) / kBlock);
    const unsigned begin = tile.block + (threadIdx.x >> 5), end = min(blocks, tile.block + kWarps * c.per_warp);
    const bool aligned = ((reinterpret_cast<uintptr_t>(d.p) & 31) | (reinterpret_cast<uintptr_t>(grad) & (8 * sizeof(G) - 1)) |
                          ((reinterpret_cast<uintptr_t>(d.m) | reinterpret_cast<uintptr_t>(d.v)) & (BITS == 32 ? 31 : 7)) |
                          (reinterpret_cast<uintptr_t>(d.copy) & 15)) == 0;
    const unsigned wide = aligned ? min(end, static_cast<unsigned>(d.n / kBlock)) : 0u;          // the last block may be short
    // The scales of the warp's blocks are read at the start and written at the end, lane j those of its block j: a load
    // from a sector to which neighbours have just written takes the time of several others (64 M elements: 374 us block
    // by block, 181 with the loads at the start).
    const unsigned mine = begin + lane * kWarps;
    unsigned scales = 0;
    if (BITS == 8 && mine < end) scales = d.ms[mine] | d.vs[mine] << 8;
    Stored<BITS, G> now, ahead;
    unsigned b = begin;
    auto turn = [&](auto is_wide) {
        const unsigned j = (b - begin) / kWarps;
        unsigned e = BITS == 8 ? __shfl_sync(0xffffffffu, scales, j) : 0u;
        const int left = static_cast<int>(min(d.n - static_cast<long long>(b) * kBlock, static_cast<long long>(kBlock)));
        adamw_block<BITS, G, kFull, decltype(is_wide)::value>(d, grad, now, b, left, f, key, e);
        if (lane == j) scales = e;
    };
    // 8 bits: the next block is on its way while this one is computed (2^28 elements with bf16 gradients and copies: 655 us, 750
    // without); fp32 states compute so little that it only costs registers (64 M: 276 and 273 us).
    constexpr bool kAhead = BITS == 8;
    if (kAhead && b < wide) ahead.load(d, grad, b);
    for (; b < wide; b += kWarps) {
        if constexpr (kAhead) {
            now = ahead;
            if (b + kWarps < wide) ahead.load(d, grad, b + kWarps);
        } else {
            now.load(d, grad, b);
        }
        turn(std::true_type{});
    }
    for (; b < end; b += kWarps) turn(std::false_type{});
    if (BITS == 8 && mine < end) {
        d.ms[mine] = static_cast<uint8_t>(scales);
        d.vs[mine] = static_cast<uint8_t>(scales >> 8);
    }
}

struct MovedPointers { const void* p[kMovedPointers]; };

__global__ void k_adamw_pointers(const __grid_constant__ MovedPointers from, const void** to, int n)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) to[i] = from.p[i];
}

}  // namespace

struct came_adamw_ctx {
    int device = 0, n = 0;
    unsigned per_warp[2] = {1, 1};       // blocks of a tile for each warp: fp32, 8-bit states
    int first[5] = {0, 0, 0, 0, 0};      // where the tiles of each (state, gradient) type begin
    std::vector<int64_t> numel;
    std::vector<int>     grad_bytes;
    char*         d_mem = nullptr;
    AdamwTensor*  d_table = nullptr;
    AdamwTile*    d_tiles = nullptr;
    const void**  d_grads = nullptr;     // as given at create
    const void**  d_moved = nullptr;     // as given to the call that is running
};

namespace {

void free_adamw(came_adamw_ctx* c)
{
    if (!c) return;
    cudaFree(c->d_mem);
    delete c;
}

came_status tensor_error(came_status s, int i, const char* what)
{
    char buf[160];
    std::snprintf(buf, sizeof buf, "tensor %d: %s", i, what);
    return report(s, buf);
}

came_status validate_adamw(const came_adamw_tensor* t, int n)
{
    struct Range { uintptr_t lo, hi; int tensor; bool out; };
    std::vector<Range> rs;
    rs.reserve(7 * static_cast<size_t>(n));
    for (int i = 0; i < n; ++i) {
        const came_adamw_tensor& x = t[i];
        if (x.numel < 0 || x.numel > (1ll << 39)) return tensor_error(CAME_ERR_SHAPE, i, "numel out of range");
        if (!known_dtype(x.grad_dtype)) return tensor_error(CAME_ERR_DTYPE, i, "unknown grad_dtype");
        if (x.state_bits != 32 && x.state_bits != 8) return tensor_error(CAME_ERR_DTYPE, i, "state_bits must be 32 or 8");
        if (x.flags & ~static_cast<uint32_t>(CAME_T_NO_WEIGHT_DECAY)) return tensor_error(CAME_ERR_UNSUPPORTED, i, "unknown flag");
        if (x.reserved) return tensor_error(CAME_ERR_SHAPE, i, "reserved must be 0");
        if (!x.numel) continue;
        const bool small = x.state_bits == 8;
        if (!x.param || !x.grad || !x.m || !x.v || (small && (!x.m_scale || !x.v_scale)))
            return tensor_error(CAME_ERR_NULL, i, "param, grad and states are required");
        const size_t sb = small ? 1 : 4;
        if (!aligned_to(x.param, 4) || !aligned_to(x.grad, dtype_bytes(x.grad_dtype)) || !aligned_to(x.m, sb) ||
            !aligned_to(x.v, sb) || !aligned_to(x.param_bf16, 2))
            return tensor_error(CAME_ERR_ALIGN, i, "a pointer is not aligned to its element size");
        auto add = [&](const void* p, uintptr_t bytes, bool out) {
            const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
            if (p) rs.push_back(Range{lo, lo + bytes, i, out});
        };
        const uintptr_t count = x.numel, scales = (count + kBlock - 1) / kBlock;
        add(x.param, 4 * count, true);
        add(x.grad, dtype_bytes(x.grad_dtype) * count, false);
        add(x.m, sb * count, true);
        add(x.v, sb * count, true);
        if (small) add(x.m_scale, scales, true), add(x.v_scale, scales, true);
        add(x.param_bf16, 2 * count, true);
    }
    std::sort(rs.begin(), rs.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
    uintptr_t reach = 0, reach_out = 0;      // furthest end of any range / of any that is written so far
    for (const Range& r : rs) {
        if (r.lo < reach_out || (r.out && r.lo < reach))
            return tensor_error(CAME_ERR_OVERLAP, r.tensor, "a buffer that is written shares memory with another");
        reach = std::max(reach, r.hi);
        if (r.out) reach_out = std::max(reach_out, r.hi);
    }
    return CAME_OK;
}

came_status validate_hparams(const came_adamw_hparams& h, bool device_step)
{
    auto in = [](double x, double hi) { return x >= 0 && x < hi; };      // (no NaN passes)
    if (!in(h.beta1, 1.0) || !in(h.beta2, 1.0)) return report(CAME_ERR_HPARAM, "beta1 and beta2 must lie in [0, 1)");
    if (!in(h.lr, FLT_MAX) || !in(h.eps, FLT_MAX) || !in(h.weight_decay, FLT_MAX) || !in(h.lr * h.weight_decay, FLT_MAX))
        return report(CAME_ERR_HPARAM, "lr, eps and weight_decay must be finite and >= 0");
    if (!(h.grad_scale >= 0) || !holds_in_fp32(h.grad_scale))
        return report(CAME_ERR_HPARAM, "grad_scale must be finite, and not vanish, in fp32 (0 for 1)");
    if (static_cast<float>(h.beta1) >= 1.f || static_cast<float>(h.beta2) >= 1.f)
        return report(CAME_ERR_HPARAM, "beta1 and beta2 must be below 1 in fp32");
    if (!device_step && h.step < 1) return report(CAME_ERR_STEP_ORDER, "step must be >= 1");
    return CAME_OK;
}

template <int BITS, typename G>
cudaError_t launch(const came_adamw_ctx* c, int kind, const void* const* grads, AdamwConsts k, bool full, cudaStream_t stream)
{
    k.per_warp = c->per_warp[BITS == 8];
    const int tiles = c->first[kind + 1] - c->first[kind];
    if (!tiles) return cudaSuccess;
    if (full) k_adamw<BITS, G, true><<<tiles, kWarps * 32, 0, stream>>>(c->d_table, grads, c->d_tiles + c->first[kind], k);
    else k_adamw<BITS, G, false><<<tiles, kWarps * 32, 0, stream>>>(c->d_table, grads, c->d_tiles + c->first[kind], k);
    return cudaGetLastError();
}

int kind_of(const came_adamw_tensor& t) { return (t.state_bits == 8 ? 2 : 0) + (t.grad_dtype == CAME_BF16 ? 1 : 0); }

}  // namespace

extern "C" {

came_status came_adamw_create(came_adamw_ctx** out, const came_adamw_tensor* t, int32_t n, int32_t device, uint32_t flags)
{
    if (!out) return report(CAME_ERR_NULL, "out is NULL");
    *out = nullptr;
    if (!t) return report(CAME_ERR_NULL, "tensor array is NULL");
    if (n < 1 || n > (1 << 24)) return report(CAME_ERR_SHAPE, "tensor count out of range");
    if (flags & ~static_cast<uint32_t>(CAME_CREATE_KEEP_STATE)) return report(CAME_ERR_UNSUPPORTED, "unknown flag");
    came_adamw_ctx* c = nullptr;
    try {
        came_status s = validate_adamw(t, n);
        if (s != CAME_OK) return s;
        int ndev = 0;
        if (cudaGetDeviceCount(&ndev) != cudaSuccess || ndev < 1) {
            cudaGetLastError();
            return report(CAME_ERR_DEVICE, "no usable CUDA device");
        }
        if (device < 0 || device >= ndev) return report(CAME_ERR_DEVICE, "device ordinal out of range");
        if ((s = require_current_device(device)) != CAME_OK) return s;
        c = new came_adamw_ctx;
        c->device = device;
        c->n = n;
        long long blocks = 0;
        for (int i = 0; i < n; ++i) blocks += (t[i].numel + kBlock - 1) / kBlock;
        if (blocks > (1ll << 31)) { free_adamw(c); return report(CAME_ERR_SHAPE, "more than 2^39 elements in all"); }
        // 8 bits: up to eight, so that a tile writes whole sectors of scales and loads ahead (64 M elements: 161 us,
        // 230 with one), as long as there are tiles for every SM.  fp32: one (261 us, 272 with eight).
        while (c->per_warp[1] < 8 && blocks >= 148ll * kWarps * c->per_warp[1]) c->per_warp[1] *= 2;
        std::vector<AdamwTensor> table(n);
        std::vector<AdamwTile> tiles;
        long long block0 = 0;
        for (int i = 0; i < n; ++i) {
            const came_adamw_tensor& x = t[i];
            table[i] = AdamwTensor{x.param, x.m, x.v, x.m_scale, x.v_scale, static_cast<__nv_bfloat16*>(x.param_bf16), x.numel,
                                   static_cast<unsigned>(block0), (x.flags & CAME_T_NO_WEIGHT_DECAY) ? 0 : 1};
            block0 += (x.numel + kBlock - 1) / kBlock;
            c->numel.push_back(x.numel);
            c->grad_bytes.push_back(static_cast<int>(dtype_bytes(x.grad_dtype)));
        }
        for (int kind = 0; kind < 4; ++kind) {
            c->first[kind] = static_cast<int>(tiles.size());
            const unsigned per_tile = kWarps * c->per_warp[kind >> 1];
            for (int i = 0; i < n; ++i) {
                if (kind_of(t[i]) != kind) continue;
                const long long have = (t[i].numel + kBlock - 1) / kBlock;
                if (static_cast<long long>(tiles.size()) + have / per_tile + 1 > (1 << 28)) {
                    free_adamw(c);
                    return report(CAME_ERR_SHAPE, "too many tiles");
                }
                for (long long b = 0; b < have; b += per_tile) tiles.push_back(AdamwTile{i, static_cast<unsigned>(b)});
            }
        }
        c->first[4] = static_cast<int>(tiles.size());
        size_t bytes = 0;
        auto take = [&](size_t b) { const size_t at = bytes; bytes += (b + 255) / 256 * 256; return at; };
        const size_t at_table = take(sizeof(AdamwTensor) * n), at_tiles = take(sizeof(AdamwTile) * tiles.size());
        const size_t at_grads = take(sizeof(void*) * n), at_moved = take(sizeof(void*) * n);
        cudaError_t e;
#define ADAMW_TRY(call, what) do { if ((e = (call)) != cudaSuccess) { free_adamw(c); return report_cuda(e, what); } } while (0)
        ADAMW_TRY(cudaMalloc(&c->d_mem, bytes), "cudaMalloc(adamw tables)");
        c->d_table = reinterpret_cast<AdamwTensor*>(c->d_mem + at_table);
        c->d_tiles = reinterpret_cast<AdamwTile*>(c->d_mem + at_tiles);
        c->d_grads = reinterpret_cast<const void**>(c->d_mem + at_grads);
        c->d_moved = reinterpret_cast<const void**>(c->d_mem + at_moved);
        std::vector<char> host(bytes, 0);
        std::memcpy(host.data() + at_table, table.data(), sizeof(AdamwTensor) * n);
        if (!tiles.empty()) std::memcpy(host.data() + at_tiles, tiles.data(), sizeof(AdamwTile) * tiles.size());
        for (int i = 0; i < n; ++i) std::memcpy(host.data() + at_grads + sizeof(void*) * i, &t[i].grad, sizeof(void*));
        ADAMW_TRY(cudaMemcpy(c->d_mem, host.data(), bytes, cudaMemcpyHostToDevice), "cudaMemcpy(adamw tables)");
        if (!(flags & CAME_CREATE_KEEP_STATE)) {
            for (int i = 0; i < n; ++i) {
                const size_t count = static_cast<size_t>(t[i].numel), sb = t[i].state_bits == 8 ? 1 : 4;
                if (!count) continue;
                ADAMW_TRY(cudaMemsetAsync(t[i].m, 0, sb * count, nullptr), "cudaMemset(m)");
                ADAMW_TRY(cudaMemsetAsync(t[i].v, 0, sb * count, nullptr), "cudaMemset(v)");
                if (sb == 1) {
                    const size_t scales = (count + kBlock - 1) / kBlock;
                    ADAMW_TRY(cudaMemsetAsync(t[i].m_scale, 0, scales, nullptr), "cudaMemset(m_scale)");
                    ADAMW_TRY(cudaMemsetAsync(t[i].v_scale, 0, scales, nullptr), "cudaMemset(v_scale)");
                }
            }
        }
        ADAMW_TRY(cudaStreamSynchronize(nullptr), "cudaStreamSynchronize");
#undef ADAMW_TRY
    } catch (const std::bad_alloc&) {
        free_adamw(c);
        return report(CAME_ERR_OOM, "host allocation failed");
    }
    *out = c;
    return CAME_OK;
}

came_status came_adamw_step(came_adamw_ctx* ctx, const came_adamw_hparams* hp, const void* const* grads,
                            const float* device_scale, const int64_t* device_step, void* cuda_stream)
{
    if (!ctx || !hp) return report(CAME_ERR_NULL, "context and hyper-parameters are required");
    came_status s = validate_hparams(*hp, device_step != nullptr);
    if (s != CAME_OK) return s;
    if (!aligned_to(device_scale, 4)) return report(CAME_ERR_ALIGN, "device_scale not 4-byte aligned");
    if (!aligned_to(device_step, 8)) return report(CAME_ERR_ALIGN, "device_step not 8-byte aligned");
    if (grads)
        for (int i = 0; i < ctx->n; ++i) {
            if (ctx->numel[i] && !grads[i]) return tensor_error(CAME_ERR_NULL, i, "grad is required");
            if (!aligned_to(grads[i], ctx->grad_bytes[i])) return tensor_error(CAME_ERR_ALIGN, i, "grad not aligned to its element size");
        }
    if ((s = require_current_device(ctx->device)) != CAME_OK) return s;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const double t = static_cast<double>(device_step ? 1 : hp->step);
    AdamwConsts k = {};
    k.b1 = static_cast<float>(hp->beta1);
    k.c1 = static_cast<float>(1.0 - hp->beta1);
    k.b2 = static_cast<float>(hp->beta2);
    k.c2 = static_cast<float>(1.0 - hp->beta2);
    k.eps = static_cast<float>(hp->eps);
    k.decay = static_cast<float>(hp->lr * hp->weight_decay);
    k.scale = hp->grad_scale == 0.0 ? 1.f : static_cast<float>(hp->grad_scale);
    k.lr = hp->lr;
    k.log_b1 = std::log(hp->beta1);      // (log 0 = -inf, and 1 - exp(-inf) = 1)
    k.log_b2 = std::log(hp->beta2);
    k.step = static_cast<float>(hp->lr / -std::expm1(t * k.log_b1));
    k.root = static_cast<float>(1.0 / std::sqrt(-std::expm1(t * k.log_b2)));
    k.key_seed = mix_word(0u, hp->seed);
    k.key = mix_word(k.key_seed, static_cast<uint64_t>(device_step ? 1 : hp->step));
    k.device_scale = device_scale;
    k.device_step = device_step;
    // The roots of subnormal v are below 2^-63, times 1 / sqrt(1 - beta2) at most: beside an eps of 2^39 times that they are less than
    // 2^-24 of the sum, and left out (355 M elements with 8-bit states and bf16 gradients: 971 us, 997 with them).
    const bool full = !(hp->eps * std::sqrt(1.0 - hp->beta2) >= 0x1p-39);
    cudaError_t e = cudaSuccess;
    const void* const* from = ctx->d_grads;
    if (grads) {
        from = ctx->d_moved;
        for (int i = 0; i < ctx->n && e == cudaSuccess; i += kMovedPointers) {
            const int some = std::min(kMovedPointers, ctx->n - i);
            MovedPointers list;
            std::copy(grads + i, grads + i + some, list.p);
            k_adamw_pointers<<<(some + 255) / 256, 256, 0, stream>>>(list, ctx->d_moved + i, some);
            e = cudaGetLastError();
        }
    }
    if (e == cudaSuccess) e = launch<32, float>(ctx, 0, from, k, full, stream);
    if (e == cudaSuccess) e = launch<32, __nv_bfloat16>(ctx, 1, from, k, full, stream);
    if (e == cudaSuccess) e = launch<8, float>(ctx, 2, from, k, full, stream);
    if (e == cudaSuccess) e = launch<8, __nv_bfloat16>(ctx, 3, from, k, full, stream);
    return e == cudaSuccess ? CAME_OK : report_cuda(e, "kernel launch");
}

came_status came_adamw_destroy(came_adamw_ctx* ctx)
{
    if (!ctx) return CAME_ERR_NULL;
    free_adamw(ctx);
    return CAME_OK;
}

}  // extern "C"
