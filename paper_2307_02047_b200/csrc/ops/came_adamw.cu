// AdamW over a list of tensors, with the states in fp32 or in 8 bits.
//
//   g = grad * s,  m = b1 m + (1-b1) g,  v = b2 v + (1-b2) g^2,
//   p = p - (lr wd p + lr mhat / (sqrt(vhat) + eps))
//
// A warp takes 256 consecutive elements of a tensor, eight per lane: the elements that share a scale
// where states have 8 bits.  Nothing crosses from one such block to the next, so there is one pass, one
// launch for each type of state and gradient in the list, and no order that could change a result.
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

struct AdamwTile { int tensor; unsigned block; };       // blocks [block, block + per_tile) of a tensor

struct AdamwConsts {
    float b1, c1, b2, c2, eps, decay, scale;
    float step, root;                    // lr / (1 - b1^t), 1 / sqrt(1 - b2^t); not used with a step on the device
    unsigned key;
    int per_tile;
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

__device__ __forceinline__ float approx_sqrt(float x) { float y; asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float approx_rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }
__device__ __forceinline__ float power_of_two(int e) { return e > 0 ? __uint_as_float(static_cast<unsigned>(e) << 23) : __uint_as_float(0x00400000u >> -e); }

// The 8-bit types: magnitudes are the upper bits of an fp32 whose exponent has been lowered by kLow, subnormal
// values included, so that adding a random number below the bits that are dropped and cutting these
// off rounds up with the right probability.
struct E4M3 {
    static constexpr int kTop = 7, kDrop = 20;
    static constexpr float kLow = 0x1p-120f;
    static __device__ __forceinline__ unsigned random(unsigned r) { return ((r & 0xffffu) << 4) + 8u; }
    static __device__ __forceinline__ void decode(uint32_t two, float& a, float& b)      // bytes 0 and 1
    {
        uint32_t h;
        asm("{ .reg .b16 t; cvt.u16.u32 t, %1; cvt.rn.f16x2.e4m3x2 %0, t; }" : "=r"(h) : "r"(two));
        const __half2 x = *reinterpret_cast<const __half2*>(&h);
        a = __low2float(x);
        b = __high2float(x);
    }
};
struct E5M2 {
    static constexpr int kTop = 14, kDrop = 21;
    static constexpr float kLow = 0x1p-112f;
    static __device__ __forceinline__ unsigned random(unsigned r) { return ((r >> 16) << 5) + 16u; }
    static __device__ __forceinline__ void decode(uint32_t two, float& a, float& b)
    {
        const uint32_t h = __byte_perm(two, 0, 0x1404);              // an e5m2 is the upper byte of a half
        const __half2 x = *reinterpret_cast<const __half2*>(&h);
        a = __low2float(x);
        b = __high2float(x);
    }
};

template <typename F>
__device__ __forceinline__ void decode8(const uint32_t (&w)[2], uint8_t e, float (&x)[8])
{
    const float scale = power_of_two(e);
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        F::decode(w[k >> 2] >> (k & 2 ? 16 : 0), x[k], x[k + 1]);
        x[k] *= scale;
        x[k + 1] *= scale;
    }
}

// Codes of a block's values (x: this lane's eight), and the byte of its scale.  The order of a lane's elements does
// not matter here: r are their random bits.
template <typename F, bool kSigned>
__device__ __forceinline__ uint8_t encode8(const float (&x)[8], const unsigned (&r)[8], uint32_t (&w)[2])
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
    const float inverse = power_of_two(254 - e);
    w[0] = w[1] = 0u;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float y = __fmul_rn(__fmul_rn(fabsf(x[k]), inverse), F::kLow);
        unsigned code = (__float_as_uint(y) + F::random(r[k])) >> F::kDrop;
        if constexpr (kSigned) {
            if (special && !(fabsf(x[k]) < INFINITY)) code = 0x7fu;
            code |= (__float_as_uint(x[k]) >> 24) & 0x80u;
        } else {
            code = max(code, min(__float_as_uint(x[k]), 1u));       // not zero: not stored as zero
            if (special && !(x[k] < INFINITY)) code = x[k] == INFINITY ? 0x7cu : 0x7fu;
        }
        w[k >> 2] |= code << (8 * (k & 3));
    }
    return static_cast<uint8_t>(e);
}

// One element's new p, from its old p, its gradient and its states, which become the new ones.
struct Update {
    float b1, c1, b2, c2, eps, step, root, decay, scale;
    __device__ __forceinline__ float operator()(float p, float g, float& m, float& v) const
    {
        g = __fmul_rn(g, scale);
        m = __fadd_rn(__fmul_rn(b1, m), __fmul_rn(c1, g));
        v = __fadd_rn(__fmul_rn(b2, v), __fmul_rn(c2, __fmul_rn(g, g)));
        const float u = m * approx_rcp(fmaf(approx_sqrt(v), root, eps));
        return p - fmaf(step, u, decay * p);
    }
};

// 256 elements from `i0` on, `left` of them in the tensor.  kWide: all there, and 8 per lane lie side by side and
// aligned; else lane l takes the elements l, l + 32, ... one by one.
template <int BITS, typename G, bool kWide>
__device__ __forceinline__ void adamw_block(const AdamwTensor& d, const G* grad, unsigned block, int left, const Update& f, unsigned key)
{
    using S = typename std::conditional<BITS == 32, float, uint8_t>::type;
    const int lane = threadIdx.x & 31;
    const long long i0 = static_cast<long long>(block) * kBlock;
    float p[8], g[8], m[8], v[8];
    const int first = kWide ? 8 * lane : lane, next = kWide ? 1 : 32;
    const long long at = i0 + first;
    float* const pp = d.p + at;
    S* const pm = static_cast<S*>(d.m) + at;
    S* const pv = static_cast<S*>(d.v) + at;
    Vec<float, 8> vp;
    if constexpr (kWide) {
        Vec<G, 8> vg;
        Vec<S, 8> vm, vv;
        uint8_t em = 0, ev = 0;
        vg.load(grad + at);
        vm.load(pm);
        vv.load(pv);
        vp.load(pp);
        if constexpr (BITS == 8) em = d.ms[block], ev = d.vs[block];
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = vg.value(k), p[k] = vp.value(k);
        if constexpr (BITS == 32) {
#pragma unroll
            for (int k = 0; k < 8; ++k) m[k] = vm.value(k), v[k] = vv.value(k);
        } else {
            decode8<E4M3>(vm.w, em, m);
            decode8<E5M2>(vv.w, ev, v);
        }
    } else {
        uint32_t wm[2] = {0u, 0u}, wv[2] = {0u, 0u};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool in = first + 32 * k < left;
            p[k] = in ? pp[32 * k] : 0.f;
            g[k] = in ? to_float(grad[at + 32 * k]) : 0.f;
            if constexpr (BITS == 32) {
                m[k] = in ? pm[32 * k] : 0.f;
                v[k] = in ? pv[32 * k] : 0.f;
            } else if (in) {
                wm[k >> 2] |= static_cast<uint32_t>(pm[32 * k]) << (8 * (k & 3));
                wv[k >> 2] |= static_cast<uint32_t>(pv[32 * k]) << (8 * (k & 3));
            }
        }
        if constexpr (BITS == 8) {
            decode8<E4M3>(wm, d.ms[block], m);
            decode8<E5M2>(wv, d.vs[block], v);
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = f(p[k], g[k], m[k], v[k]);
    if constexpr (BITS == 8) {
        unsigned r[8];
        const unsigned base = mix(key + (d.block0 + block) * kGolden) + static_cast<unsigned>(first) * kGolden;
#pragma unroll
        for (int k = 0; k < 8; ++k) r[k] = mix(base + static_cast<unsigned>(k * next) * kGolden);
        if constexpr (!kWide) {          // elements behind the end are zero and stay out of the scales
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (first + 32 * k >= left) m[k] = v[k] = 0.f;
        }
        uint32_t wm[2], wv[2];
        const uint8_t em = encode8<E4M3, true>(m, r, wm), ev = encode8<E5M2, false>(v, r, wv);
        __syncwarp();                    // every lane has read the old scales
        if (lane == 0) d.ms[block] = em, d.vs[block] = ev;
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
        vp.set(m);
        vp.store(pm);
        vp.set(v);
        vp.store(pv);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (first + 32 * k < left) pm[32 * k] = m[k], pv[32 * k] = v[k];
    }
    if constexpr (kWide) {
        vp.set(p);
        vp.store(pp);
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

template <int BITS, typename G>
__global__ void __launch_bounds__(kWarps * 32)
k_adamw(const AdamwTensor* __restrict__ table, const void* const* __restrict__ grads, const AdamwTile* __restrict__ tiles,
        const __grid_constant__ AdamwConsts c)
{
    __shared__ float s_step, s_root;
    __shared__ unsigned s_key;
    const AdamwTile tile = tiles[blockIdx.x];
    const AdamwTensor d = table[tile.tensor];
    const G* const grad = static_cast<const G*>(grads[tile.tensor]);
    Update f{c.b1, c.c1, c.b2, c.c2, c.eps, c.step, c.root, d.decay ? c.decay : 0.f, c.scale};
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
    const unsigned blocks = static_cast<unsigned>((d.n + kBlock - 1) / kBlock);
    const unsigned end = min(blocks, tile.block + static_cast<unsigned>(c.per_tile));
    const uintptr_t states = reinterpret_cast<uintptr_t>(d.m) | reinterpret_cast<uintptr_t>(d.v);
    const bool aligned = ((reinterpret_cast<uintptr_t>(d.p) & 31) | (reinterpret_cast<uintptr_t>(grad) & (8 * sizeof(G) - 1)) |
                          (states & (BITS == 32 ? 31 : 7)) | (reinterpret_cast<uintptr_t>(d.copy) & 15)) == 0;
    for (unsigned b = tile.block + (threadIdx.x >> 5); b < end; b += kWarps) {
        const long long left = d.n - static_cast<long long>(b) * kBlock;
        if (aligned && left >= kBlock) adamw_block<BITS, G, true>(d, grad, b, kBlock, f, key);
        else adamw_block<BITS, G, false>(d, grad, b, static_cast<int>(min(left, static_cast<long long>(kBlock))), f, key);
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
    int device = 0, n = 0, per_tile = 0;
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
cudaError_t launch(const came_adamw_ctx* c, int kind, const void* const* grads, const AdamwConsts& k, cudaStream_t stream)
{
    const int tiles = c->first[kind + 1] - c->first[kind];
    if (!tiles) return cudaSuccess;
    k_adamw<BITS, G><<<tiles, kWarps * 32, 0, stream>>>(c->d_table, grads, c->d_tiles + c->first[kind], k);
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
        // a block per warp in small lists, four in large ones
        c->per_tile = kWarps * (blocks > 148 * 8 * kWarps * 4 ? 4 : 1);
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
            for (int i = 0; i < n; ++i) {
                if (kind_of(t[i]) != kind) continue;
                const long long have = (t[i].numel + kBlock - 1) / kBlock;
                if (static_cast<long long>(tiles.size()) + have / c->per_tile + 1 > (1 << 28)) {
                    free_adamw(c);
                    return report(CAME_ERR_SHAPE, "too many tiles");
                }
                for (long long b = 0; b < have; b += c->per_tile) tiles.push_back(AdamwTile{i, static_cast<unsigned>(b)});
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
    k.per_tile = ctx->per_tile;
    k.device_scale = device_scale;
    k.device_step = device_step;
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
    if (e == cudaSuccess) e = launch<32, float>(ctx, 0, from, k, stream);
    if (e == cudaSuccess) e = launch<32, __nv_bfloat16>(ctx, 1, from, k, stream);
    if (e == cudaSuccess) e = launch<8, float>(ctx, 2, from, k, stream);
    if (e == cudaSuccess) e = launch<8, __nv_bfloat16>(ctx, 3, from, k, stream);
    return e == cudaSuccess ? CAME_OK : report_cuda(e, "kernel launch");
}

came_status came_adamw_destroy(came_adamw_ctx* ctx)
{
    if (!ctx) return CAME_ERR_NULL;
    free_adamw(ctx);
    return CAME_OK;
}

}  // extern "C"
