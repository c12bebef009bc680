// Layer norm over the rows of a matrix, and its backward pass.
//
//   y = (x - mean) rstd w + b
//   dx = rstd (d - mean(d) - h mean(d h)),  d = dy w,  h = (x - mean) rstd
//   dw = sum over rows of dy h,  db = sum over rows of dy
//
// A group of 32 to 1024 threads takes a row: it is read once and stays in registers or shared memory while its sums are
// formed.  In the backward pass a group goes from row to row and keeps, for its columns, the sums over its
// rows in registers; blocks write those to the workspace, and a second, short grid adds them.
//
// fp32 is bound by the bytes (128k x 4096: forward 615 us, 7.0 TB/s; backward 935 us, 6.9 TB/s).  bf16 has half the bytes
// for the same arithmetic: forward 402 us (5.3 TB/s, 0.82 of the measured copy rate), backward 547 us (5.9 TB/s), 584 under
// a load that lowers the clock: about 17 and 22 instructions for an element, 60 % of what can be issued, which is
// what arithmetic on pairs and two sums per exchange of a warp have left.
#include "came_vec.cuh"

#include <algorithm>
#include <atomic>

namespace {

using namespace came_ops;

constexpr int kSMs = 148;
constexpr int kBlockThreads = 512;       // threads of a block whose groups go from row to row, at most
constexpr int kRingBytes = 200 << 10;    // its shared memory for rows on their way
constexpr int kMaxStages = 6;
constexpr int kRun = 256;                // rows longer than a block: additions of a thread one after another
constexpr long long kManyElements = 4ll << 20;      // forward: from here on groups go from row to row

struct LnArgs {
    const void* x;
    const void* w;
    const void* b;
    void*       y;                       // backward: dx
    const void* dy;
    float*      mean;
    float*      rstd;
    float*      part;                    // backward: [blocks][2][cols]
    int         rows, cols;
    long long   x_ld, y_ld, dy_ld;
    float       eps, inv_cols;
    int         tpr;                     // threads per row
    int         stages;                  // places in the ring, 2 to kMaxStages
    int         period;                  // rows until one begins at the same place relative to an aligned address
    int         w_bf16, y_bf16;
};

// Two fp32 in one 64-bit register: additions, products and multiply-adds of both at a time, half the instructions, each rounded
// as ever.
struct Two {
    unsigned long long v;
    __device__ __forceinline__ Two() {}
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
    __device__ __forceinline__ float sum() const { float a, b; get(a, b); return a + b; }
};
__device__ __forceinline__ Two operator+(Two a, Two b) { Two c; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(c.v) : "l"(a.v), "l"(b.v)); return c; }
__device__ __forceinline__ Two operator*(Two a, Two b) { Two c; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(c.v) : "l"(a.v), "l"(b.v)); return c; }
__device__ __forceinline__ Two fma(Two a, Two b, Two c) { Two d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return d; }
__device__ __forceinline__ Two both(float a) { return Two(a, a); }

template <int V>
__device__ __forceinline__ void load_param(const void* p, int is_bf16, int at, float (&out)[V])
{
    if (is_bf16) {
        Vec<__nv_bfloat16, V> v;
        v.load(static_cast<const __nv_bfloat16*>(p) + at);
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = v.value(k);
    } else {
        Vec<float, V> v;
        v.load(static_cast<const float*>(p) + at);
#pragma unroll
        for (int k = 0; k < V; ++k) out[k] = v.value(k);
    }
}

template <int V>
__device__ __forceinline__ void store_as(void* p, int is_bf16, long long at, const float (&x)[V])
{
    if (is_bf16) {
        Vec<__nv_bfloat16, V> v;
        v.set(x);
        v.store(static_cast<__nv_bfloat16*>(p) + at);
    } else {
        Vec<float, V> v;
        v.set(x);
        v.store(static_cast<float*>(p) + at);
    }
}

// Eight columns from `column` on, those of them that the row has (kSkew: perhaps not all).
template <bool kSkew>
__device__ __forceinline__ void load_columns(const void* p, int is_bf16, int column, int cols, float (&x)[8])
{
    if (!p || column >= cols) return;
    if constexpr (!kSkew) {
        load_param<8>(p, is_bf16, column, x);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (static_cast<unsigned>(column + k) < static_cast<unsigned>(cols)) {
                float one[1];
                load_param<1>(p, is_bf16, column + k, one);
                x[k] = one[0];
            }
    }
}

// Zero in the place of the columns that the row does not have.
__device__ __forceinline__ void drop_outside(Two (&x)[4], int column, int cols)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float a, b;
        x[k].get(a, b);
        x[k] = Two(static_cast<unsigned>(column + 2 * k) < static_cast<unsigned>(cols) ? a : 0.f,
                   static_cast<unsigned>(column + 2 * k + 1) < static_cast<unsigned>(cols) ? b : 0.f);
    }
}

template <bool kSkew>
__device__ __forceinline__ void store_columns(void* p, int is_bf16, long long row, int column, int cols, const float (&x)[8])
{
    if constexpr (kSkew) {
        if (column < 0 || column + 8 > cols) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (static_cast<unsigned>(column + k) < static_cast<unsigned>(cols)) {
                    const float one[1] = {x[k]};
                    store_as<1>(p, is_bf16, row + column + k, one);
                }
            return;
        }
    }
    store_as<8>(p, is_bf16, row + column, x);
}

// Backward: places for an eighth of a row's sums in shared memory (an odd number, for the banks).
__host__ __device__ __forceinline__ int sums_width(int cols) { return ((cols + 7) >> 3) | 1; }

__device__ __forceinline__ void group_barrier(int group, int tpr)
{
    asm volatile("bar.sync %0, %1;" :: "r"(group + 1), "r"(tpr) : "memory");
}

// The two sums v over a group's threads, the same in all of them.  The halves of a warp take one sum each after the first
// exchange, so that two sums cost hardly more than one.  `room`: shared memory of the group, an entry per warp; a caller
// that comes back before the group's next barrier takes another one.
__device__ __forceinline__ void group_sum(float (&v)[2], int group, int tpr, int warp, float (*room)[2])
{
    const int lane = threadIdx.x & 31, half = lane >> 4, warps = tpr >> 5;
    float mine = half ? v[1] : v[0];
    mine += __shfl_xor_sync(0xffffffffu, half ? v[0] : v[1], 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (warps > 1) {
        if ((lane & 15) == 0) room[warp][half] = mine;
        group_barrier(group, tpr);
        mine = (lane & 15) < warps ? room[lane & 15][half] : 0.f;
        if (warps > 16 && (lane & 15) + 16 < warps) mine += room[(lane & 15) + 16][half];
#pragma unroll
        for (int o = 8; o > 0; o >>= 1)
            if (o < warps) mine += __shfl_xor_sync(0xffffffffu, mine, o);        // (lanes at `warps` and above hold zeros)
    }
    v[0] = __shfl_sync(0xffffffffu, mine, 0);
    v[1] = __shfl_sync(0xffffffffu, mine, 16);
}
__device__ __forceinline__ float group_sum(float x, int group, int tpr, int warp, float (*room)[2])
{
    float v[2] = {x, 0.f};
    group_sum(v, group, tpr, warp, room);
    return v[0];
}

// Eight elements from global to shared memory, asynchronously; of the `left` elements that there are, the others become zero.
template <typename T, bool kEnd>
__device__ __forceinline__ void copy_async(uint32_t to, const T* from, long long left)
{
    constexpr int N = 16 / static_cast<int>(sizeof(T));
#pragma unroll
    for (int k = 0; k < 8; k += N) {
        if constexpr (kEnd) {
            const int bytes = static_cast<int>(max(0ll, min(static_cast<long long>(N), left - k))) * static_cast<int>(sizeof(T));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to + k * static_cast<int>(sizeof(T))), "l"(bytes ? from + k : from), "r"(bytes) : "memory");
        } else {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + k * static_cast<int>(sizeof(T))), "l"(from + k) : "memory");
        }
    }
}

// W words from shared memory
template <int W>
__device__ __forceinline__ void read_shared(uint32_t at, uint32_t (&w)[W])
{
#pragma unroll
    for (int k = 0; k < W; k += 4)
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[k]), "=r"(w[k + 1]), "=r"(w[k + 2]), "=r"(w[k + 3]) : "r"(at + 4 * k));
}

template <int N>
__device__ __forceinline__ void wait_all_but(int n)      // N at most: the youngest n of the copies committed may be on their way
{
    if constexpr (N > 0)
        if (n < N) return wait_all_but<N - 1>(n);
    asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory");
}

// ---- forward ------------------------------------------------------------------------------------

// R rows of a group at once, C accesses of V elements per thread: the row's column (c tpr + thread) V.
template <typename X, int V, int C, int R>
__global__ void __launch_bounds__(1024)
k_ln_forward(const __grid_constant__ LnArgs a)
{
    __shared__ float room[2][32][2];     // 32 warps at most, of all groups together; one set for each sum
    const int tpr = a.tpr, group = threadIdx.x / tpr, t = threadIdx.x - group * tpr;
    const int row = (blockIdx.x * (blockDim.x / tpr) + group) * R;
    if (row >= a.rows) return;           // (the whole group)
    const int warp0 = group * (tpr >> 5);
    Vec<X, V> raw[R][C];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const X* const x = static_cast<const X*>(a.x) + min(row + r, a.rows - 1) * a.x_ld;       // (a row that is not there: the last once more)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * tpr + t) * V;
            if (col < a.cols) raw[r][c].load(x + col);
        }
    }
    // (few elements per thread: the parameters are on their way while the sums are formed)
    constexpr bool kEarly = C * V <= 8;
    float w[kEarly ? C : 1][V], b[kEarly ? C : 1][V];
    if constexpr (kEarly) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * tpr + t) * V;
            if (a.w && col < a.cols) load_param<V>(a.w, a.w_bf16, col, w[c]);
            if (a.b && col < a.cols) load_param<V>(a.b, a.w_bf16, col, b[c]);
        }
    }
    float sums[2] = {0.f, 0.f}, squares[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < R; ++r) {
        Two sum(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if ((c * tpr + t) * V >= a.cols) continue;
            if constexpr (V == 1) sum = sum + Two(raw[r][c].value(0), 0.f);
            else
#pragma unroll
                for (int k = 0; k < V; k += 2) sum = sum + Two(raw[r][c].value(k), raw[r][c].value(k + 1));
        }
        sums[r] = sum.sum();
    }
    group_sum(sums, group, tpr, t >> 5, room[0] + warp0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float mean = sums[r] *= a.inv_cols;
        Two sum(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if ((c * tpr + t) * V >= a.cols) continue;
            if constexpr (V == 1) {
                const Two d(raw[r][c].value(0) - mean, 0.f);
                sum = fma(d, d, sum);
            } else {
#pragma unroll
                for (int k = 0; k < V; k += 2) {
                    const Two d = Two(raw[r][c].value(k), raw[r][c].value(k + 1)) + both(-mean);
                    sum = fma(d, d, sum);
                }
            }
        }
        squares[r] = sum.sum();
    }
    group_sum(squares, group, tpr, t >> 5, room[1] + warp0);
    float rstd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        rstd[r] = __frsqrt_rn(fmaf(squares[r], a.inv_cols, a.eps));
        if (t == 0 && a.mean && row + r < a.rows) {
            a.mean[row + r] = sums[r];
            a.rstd[row + r] = rstd[r];
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * tpr + t) * V;
        if (col >= a.cols) continue;
        const int at = kEarly ? c : 0;
        if constexpr (!kEarly) {
            if (a.w) load_param<V>(a.w, a.w_bf16, col, w[0]);
            if (a.b) load_param<V>(a.b, a.w_bf16, col, b[0]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row + r >= a.rows) continue;
            float y[V];
#pragma unroll
            for (int k = 0; k < V; ++k) y[k] = __fmul_rn(__fadd_rn(raw[r][c].value(k), -sums[r]), rstd[r]);
            if (a.w)
#pragma unroll
                for (int k = 0; k < V; ++k) y[k] = __fmul_rn(y[k], w[at][k]);
            if (a.b)
#pragma unroll
                for (int k = 0; k < V; ++k) y[k] = __fadd_rn(y[k], b[at][k]);
            store_as<V>(a.y, a.y_bf16, (row + r) * a.y_ld + col, y);
        }
    }
}

// The rows that a group of the kernels below takes, and where its threads' columns lie.  Rows whose stride is no multiple of eight
// elements begin at other places relative to an aligned address, again and again after `period` rows: a group takes rows of one
// such place only, so that it can make aligned accesses and keep its columns.  Thread t's access c is at column (c tpr + t) 8 - skew;
// of the ones that reach over an end of the row, the elements outside are left out.
struct Rows {
    long long first, step;               // rows first, first + step, ...
    int skew;
    __device__ __forceinline__ Rows(const LnArgs& a, int groups, int group, int at_once)
    {
        const long long id = static_cast<long long>(blockIdx.x) * groups + group, per = static_cast<long long>(gridDim.x) * groups / a.period;
        const long long place = id % a.period, turn = id / a.period;
        first = turn < per ? place + a.period * at_once * turn : a.rows;
        step = a.period * at_once * per;
        skew = static_cast<int>((place * a.x_ld) & 7);
    }
};

// Many rows: a group goes from two rows to the next two.  They come through a ring in shared memory (every thread copies and
// reads its own columns, so it waits for nothing but its own copies), the parameters stay in registers, and two rows share each
// barrier.
template <typename X, int C, bool kSkew>
__global__ void __launch_bounds__(kBlockThreads, 1)
k_ln_forward_rows(const __grid_constant__ LnArgs a)
{
    constexpr int kX = 8 * static_cast<int>(sizeof(X));
    extern __shared__ __align__(16) char dynamic[];
    __shared__ float room[2][kBlockThreads / 32][2];
    const int tpr = a.tpr, groups = blockDim.x / tpr, group = threadIdx.x / tpr, t = threadIdx.x - group * tpr;
    const int warp0 = group * (tpr >> 5), stages = a.stages;
    const Rows rows(a, groups, group, 2);
    const int skew = kSkew ? rows.skew : 0;
    const long long other = kSkew ? a.period : 1, end = kSkew ? static_cast<long long>(a.rows - 1) * a.x_ld + a.cols : 0;
    auto column = [&](int c) { return (c * tpr + t) * 8 - skew; };
    auto partial = [&](int c) { return kSkew && (column(c) < 0 || column(c) + 8 > a.cols); };
    const uint32_t base = static_cast<uint32_t>(__cvta_generic_to_shared(dynamic));
    auto place = [&](int stage, int r, int c) { return base + (((stage * 2 + r) * C + c) * blockDim.x + threadIdx.x) * kX; };
    auto start = [&](long long row, int stage) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if (row + r * other < a.rows) {
                const long long at = (row + r * other) * a.x_ld;
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (column(c) < a.cols) copy_async<X, kSkew>(place(stage, r, c), static_cast<const X*>(a.x) + at + column(c), end - at - column(c));
            }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int k = 0; k < stages - 1; ++k) start(rows.first + k * rows.step, k);
    Two w[C][4], b[C][4];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float one[8], zero[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) one[k] = 1.f, zero[k] = 0.f;
        load_columns<kSkew>(a.w, a.w_bf16, column(c), a.cols, one);
        load_columns<kSkew>(a.b, a.w_bf16, column(c), a.cols, zero);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[c][k] = Two(one[2 * k], one[2 * k + 1]), b[c][k] = Two(zero[2 * k], zero[2 * k + 1]);
    }
    int stage = 0;
    for (long long row = rows.first; row < a.rows; row += rows.step) {
        wait_all_but<kMaxStages - 2>(stages - 2);
        Two x[2][C][4], sums[2] = {both(0.f), both(0.f)};
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                Vec<X, 8> v;
                if (column(c) >= a.cols) continue;
                read_shared(place(stage, r, c), v.w);            // (a second row that is not there: whatever the ring holds; not written)
#pragma unroll
                for (int k = 0; k < 4; ++k) x[r][c][k] = Two(v.value(2 * k), v.value(2 * k + 1));
                if (partial(c)) drop_outside(x[r][c], column(c), a.cols);
#pragma unroll
                for (int k = 0; k < 4; ++k) sums[r] = sums[r] + x[r][c][k];
            }
        float s[2] = {sums[0].sum(), sums[1].sum()};
        // two rows into the place of the two before these (which have been read)
        start(row + (stages - 1) * rows.step, stage == 0 ? stages - 1 : stage - 1);
        stage = stage + 1 == stages ? 0 : stage + 1;
        group_sum(s, group, tpr, t >> 5, room[0] + warp0);
        Two squares[2] = {both(0.f), both(0.f)};
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            s[r] *= a.inv_cols;
            const Two minus = both(-s[r]);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (column(c) >= a.cols) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k) x[r][c][k] = x[r][c][k] + minus;
                if (partial(c)) drop_outside(x[r][c], column(c), a.cols);
#pragma unroll
                for (int k = 0; k < 4; ++k) squares[r] = fma(x[r][c][k], x[r][c][k], squares[r]);
            }
        }
        float q[2] = {squares[0].sum(), squares[1].sum()};
        group_sum(q, group, tpr, t >> 5, room[1] + warp0);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const long long here = row + r * other;
            if (here >= a.rows) continue;
            const float rstd = __frsqrt_rn(fmaf(q[r], a.inv_cols, a.eps));
            if (t == 0 && a.mean) {
                a.mean[here] = s[r];
                a.rstd[here] = rstd;
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (column(c) >= a.cols) continue;
                float y[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) fma(x[r][c][k] * both(rstd), w[c][k], b[c][k]).get(y[2 * k], y[2 * k + 1]);
                store_columns<kSkew>(a.y, a.y_bf16, here * a.y_ld, column(c), a.cols, y);
            }
        }
    }
}

// Rows that do not fit a block's registers: three passes over a row.  kRuns: a thread has more than kRun columns to add (the
// loops in two levels cost shorter rows 4 to 8 %).
template <typename X, int V, bool kRuns>
__global__ void __launch_bounds__(1024)
k_ln_forward_long(const __grid_constant__ LnArgs a)
{
    __shared__ float room[2][32][2];
    const int row = blockIdx.x, t = threadIdx.x;
    const X* const x = static_cast<const X*>(a.x) + row * a.x_ld;
    float sum = 0.f, sq = 0.f;
    for (int c0 = 0; c0 < (kRuns ? a.cols : 1); c0 += kRun * 1024 * V) {
        const int c1 = kRuns ? min(a.cols, c0 + kRun * 1024 * V) : a.cols;
        float run = 0.f;
        for (int col = c0 + t * V; col < c1; col += 1024 * V) {
            Vec<X, V> v;
            v.load(x + col);
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k) s += v.value(k);
            run += s;
        }
        sum += run;
    }
    const float mean = group_sum(sum, 0, 1024, t >> 5, room[0]) * a.inv_cols;
    for (int c0 = 0; c0 < (kRuns ? a.cols : 1); c0 += kRun * 1024 * V) {
        const int c1 = kRuns ? min(a.cols, c0 + kRun * 1024 * V) : a.cols;
        float run = 0.f;
        for (int col = c0 + t * V; col < c1; col += 1024 * V) {
            Vec<X, V> v;
            v.load(x + col);
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float d = v.value(k) - mean;
                s = fmaf(d, d, s);
            }
            run += s;
        }
        sq += run;
    }
    sq = group_sum(sq, 0, 1024, t >> 5, room[1]);
    const float rstd = __frsqrt_rn(fmaf(sq, a.inv_cols, a.eps));
    if (t == 0 && a.mean) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
    for (int col = t * V; col < a.cols; col += 1024 * V) {
        Vec<X, V> v;
        v.load(x + col);
        float y[V], p[V];
#pragma unroll
        for (int k = 0; k < V; ++k) y[k] = (v.value(k) - mean) * rstd;
        if (a.w) {
            load_param<V>(a.w, a.w_bf16, col, p);
#pragma unroll
            for (int k = 0; k < V; ++k) y[k] = __fmul_rn(y[k], p[k]);
        }
        if (a.b) {
            load_param<V>(a.b, a.w_bf16, col, p);
#pragma unroll
            for (int k = 0; k < V; ++k) y[k] = __fadd_rn(y[k], p[k]);
        }
        store_as<V>(a.y, a.y_bf16, row * a.y_ld + col, y);
    }
}

// ---- backward -----------------------------------------------------------------------------------

// C accesses of 8 elements per thread.  kHold: the weight and what the second half needs stay in registers; else the ring
// is read again, and the weight is kept in shared memory.
template <typename X, typename G, int C, bool kHold, bool kSkew>
__global__ void __launch_bounds__(kBlockThreads, 1)
k_ln_backward(const __grid_constant__ LnArgs a)
{
    constexpr int kX = 8 * static_cast<int>(sizeof(X)), kG = 8 * static_cast<int>(sizeof(G)), kStage = C * (kX + kG);
    extern __shared__ __align__(16) char dynamic[];      // the ring; at the end the groups' sums
    __shared__ float room[2][kBlockThreads / 32][2];
    release_dependents();
    const int tpr = a.tpr, groups = blockDim.x / tpr, group = threadIdx.x / tpr, t = threadIdx.x - group * tpr;
    const int warp0 = group * (tpr >> 5), stages = a.stages;
    const Rows rows(a, groups, group, 1);
    const int skew = kSkew ? rows.skew : 0;
    const long long end_x = kSkew ? static_cast<long long>(a.rows - 1) * a.x_ld + a.cols : 0, end_g = kSkew ? static_cast<long long>(a.rows - 1) * a.dy_ld + a.cols : 0;
    auto column = [&](int c) { return (c * tpr + t) * 8 - skew; };
    auto outside = [&](int c, int k) { return static_cast<unsigned>(column(c) + k) >= static_cast<unsigned>(a.cols); };
    auto partial = [&](int c) { return kSkew && (column(c) < 0 || column(c) + 8 > a.cols); };
    Two w[kHold ? C : 1][4], dw[C][4], db[C][4];
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int k = 0; k < 4; ++k) dw[c][k] = db[c][k] = both(0.f);
        if constexpr (kHold) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = 1.f;
            load_columns<kSkew>(a.w, a.w_bf16, column(c), a.cols, x);
#pragma unroll
            for (int k = 0; k < 4; ++k) w[c][k] = Two(x[2 * k], x[2 * k + 1]);
        }
    }
    uint32_t base = static_cast<uint32_t>(__cvta_generic_to_shared(dynamic));
    const uint32_t weights = base + threadIdx.x * 32;            // !kHold: as fp32 in front of the ring, each thread its own columns
    if constexpr (!kHold) {
        base += C * 32 * blockDim.x;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = 1.f;
            load_columns<kSkew>(a.w, a.w_bf16, column(c), a.cols, x);
#pragma unroll
            for (int k = 0; k < 8; ++k) reinterpret_cast<float*>(dynamic)[(c * blockDim.x + threadIdx.x) * 8 + k] = x[k];
        }
        __syncthreads();
    }
    auto weight_at = [&](int c) {
        Vec<float, 8> v;
        read_shared(weights + c * blockDim.x * 32, v.w);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[0][k] = Two(v.value(2 * k), v.value(2 * k + 1));
    };
    // (accesses of a warp lie side by side: stage, then access, then thread)
    auto x_at = [&](int stage, int c) { return base + stage * kStage * blockDim.x + (c * blockDim.x + threadIdx.x) * kX; };
    auto g_at = [&](int stage, int c) { return base + (stage * kStage + C * kX) * blockDim.x + (c * blockDim.x + threadIdx.x) * kG; };
    auto start = [&](long long row, int stage) {
        if (row < a.rows) {
            const long long px = row * a.x_ld, pg = row * a.dy_ld;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (column(c) >= a.cols) continue;
                copy_async<X, kSkew>(x_at(stage, c), static_cast<const X*>(a.x) + px + column(c), end_x - px - column(c));
                copy_async<G, kSkew>(g_at(stage, c), static_cast<const G*>(a.dy) + pg + column(c), end_g - pg - column(c));
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // stages - 1 rows are on their way while one is computed
    for (int k = 0; k < stages - 1; ++k) start(rows.first + k * rows.step, k);
    float mean = 0.f, rstd = 0.f;
    if (rows.first < a.rows) mean = a.mean[rows.first], rstd = a.rstd[rows.first];
    int stage = 0, turn = 0;
    for (long long row = rows.first; row < a.rows; row += rows.step, turn ^= 1) {
        Two h[kHold ? C : 1][4], d[kHold ? C : 1][4];
        Two ds = both(0.f), dh = both(0.f);      // sums of d and of d h
        const Two minus = both(-mean), now_rstd = both(rstd);
        const int now = stage;
        Vec<X, 8> vx;
        Vec<G, 8> vg;
        // h and dy of access c; nothing outside the row
        auto take = [&](int c, Two (&hh)[4], Two (&g)[4]) {
            read_shared(x_at(now, c), vx.w);
            read_shared(g_at(now, c), vg.w);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                hh[k] = (Two(vx.value(2 * k), vx.value(2 * k + 1)) + minus) * now_rstd;
                g[k] = Two(vg.value(2 * k), vg.value(2 * k + 1));
            }
            if (partial(c)) {
                drop_outside(hh, column(c), a.cols);
                drop_outside(g, column(c), a.cols);
            }
        };
        wait_all_but<kMaxStages - 2>(stages - 2);
        // the row after the ones on their way takes the place of the one before this (which has been read)
        start(row + (stages - 1) * rows.step, stage == 0 ? stages - 1 : stage - 1);
        if (row + rows.step < a.rows) mean = a.mean[row + rows.step], rstd = a.rstd[row + rows.step];
        stage = stage + 1 == stages ? 0 : stage + 1;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = kHold ? c : 0;
            if (column(c) >= a.cols) continue;
            if constexpr (!kHold) weight_at(c);
            Two g[4];
            take(c, h[at], g);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                d[at][k] = g[k] * w[at][k];
                dw[c][k] = fma(g[k], h[at][k], dw[c][k]);
                db[c][k] = db[c][k] + g[k];
                ds = ds + d[at][k];
                dh = fma(d[at][k], h[at][k], dh);
            }
        }
        if (!a.y) continue;
        float s[2] = {ds.sum(), dh.sum()};
        group_sum(s, group, tpr, t >> 5, room[turn] + warp0);
        const Two c1 = both(-s[0] * a.inv_cols), c2 = both(-s[1] * a.inv_cols);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = kHold ? c : 0;
            if (column(c) >= a.cols) continue;
            float o[8];
            if constexpr (!kHold) {
                weight_at(c);
                take(c, h[0], d[0]);
#pragma unroll
                for (int k = 0; k < 4; ++k) d[0][k] = d[0][k] * w[0][k];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) (fma(h[at][k], c2, d[at][k] + c1) * now_rstd).get(o[2 * k], o[2 * k + 1]);
            store_columns<kSkew>(a.y, a.y_bf16, row * a.y_ld, column(c), a.cols, o);
        }
    }
    if (!a.part) return;
    float* const part = a.part + 2ll * blockIdx.x * a.cols;
    if (groups == 1) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                float p[2], q[2];
                dw[c][k / 2].get(p[0], p[1]);
                db[c][k / 2].get(q[0], q[1]);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (!outside(c, k + j)) part[column(c) + k + j] = p[j], part[a.cols + column(c) + k + j] = q[j];
            }
        return;
    }
    // Every group's sums side by side in shared memory, then added in the groups' order.  Column j is at (j mod 8) wide + j / 8: one
    // of a thread's eight columns at a time, the threads' lie side by side.
    wait_all_but<0>(0);
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(dynamic);
    const int wide = sums_width(a.cols), each = 8 * wide;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            float p[2], q[2];
            dw[c][k / 2].get(p[0], p[1]);
            db[c][k / 2].get(q[0], q[1]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (outside(c, k + j)) continue;
                const int col = column(c) + k + j, at = 2 * group * each + (col & 7) * wide + (col >> 3);
                sums[at] = p[j];
                sums[at + each] = q[j];
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.cols; i += blockDim.x) {
        const int which = i >= a.cols, col = i - which * a.cols;
        const float* const from = sums + which * each + (col & 7) * wide + (col >> 3);
        float s = 0.f;
        for (int g = 0; g < groups; ++g) s += from[2 * g * each];
        part[i] = s;
    }
}

// Rows that do not fit a group: first each row's two sums ...
template <typename X, typename G, int V>
__global__ void __launch_bounds__(1024)
k_ln_backward_rows(const __grid_constant__ LnArgs a, float2* out)
{
    __shared__ float room[32][2];
    const int row = blockIdx.x;
    const X* const x = static_cast<const X*>(a.x) + row * a.x_ld;
    const G* const dy = static_cast<const G*>(a.dy) + row * a.dy_ld;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.f, 0.f};
    for (int c0 = 0; c0 < a.cols; c0 += kRun * blockDim.x * V) {
        const int c1 = min(a.cols, c0 + kRun * static_cast<int>(blockDim.x) * V);
        float run[2] = {0.f, 0.f};
        for (int col = c0 + threadIdx.x * V; col < c1; col += blockDim.x * V) {
            Vec<X, V> vx;
            Vec<G, V> vg;
            vx.load(x + col);
            vg.load(dy + col);
            float w[V], p = 0.f, q = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k) w[k] = 1.f;
            if (a.w) load_param<V>(a.w, a.w_bf16, col, w);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float d = vg.value(k) * w[k];
                p += d;
                q = fmaf(d, (vx.value(k) - mean) * rstd, q);
            }
            run[0] += p;
            run[1] += q;
        }
        s[0] += run[0];
        s[1] += run[1];
    }
    group_sum(s, 0, blockDim.x, threadIdx.x >> 5, room);
    if (threadIdx.x == 0) out[row] = make_float2(s[0] * a.inv_cols, s[1] * a.inv_cols);
}

// ... then everything else by columns: a block of 8 warps has 32 V columns and every gridDim.y-th group of 8 rows.
template <typename X, typename G, int V>
__global__ void __launch_bounds__(256)
k_ln_backward_columns(const __grid_constant__ LnArgs a, const float2* means)
{
    __shared__ float sums[8][2][32 * V];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = (blockIdx.x * 32 + lane) * V;
    const bool in = col < a.cols;
    float w[V], dw[V], db[V];
#pragma unroll
    for (int k = 0; k < V; ++k) w[k] = 1.f, dw[k] = db[k] = 0.f;
    if (a.w && in) load_param<V>(a.w, a.w_bf16, col, w);
    for (long long row = blockIdx.y * 8 + warp; in && row < a.rows; row += 8 * gridDim.y) {
        Vec<X, V> vx;
        Vec<G, V> vg;
        vx.load(static_cast<const X*>(a.x) + row * a.x_ld + col);
        vg.load(static_cast<const G*>(a.dy) + row * a.dy_ld + col);
        const float mean = a.mean[row], rstd = a.rstd[row];
        float o[V];
        float2 c = make_float2(0.f, 0.f);
        if (a.y) c = means[row];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float h = (vx.value(k) - mean) * rstd, g = vg.value(k);
            dw[k] = fmaf(g, h, dw[k]);
            db[k] += g;
            o[k] = rstd * (fmaf(g, w[k], -c.x) - h * c.y);
        }
        if (a.y) store_as<V>(a.y, a.y_bf16, row * a.y_ld + col, o);
    }
    if (!a.part) return;
#pragma unroll
    for (int k = 0; k < V; ++k) sums[warp][0][lane * V + k] = dw[k], sums[warp][1][lane * V + k] = db[k];
    __syncthreads();
    float* const part = a.part + 2ll * blockIdx.y * a.cols;
    for (int i = threadIdx.x; i < 64 * V; i += 256) {
        const int which = i / (32 * V), at = i % (32 * V), column = blockIdx.x * 32 * V + at;
        float s = 0.f;
        for (int g = 0; g < 8; ++g) s += sums[g][which][at];
        if (column < a.cols) part[static_cast<long long>(which) * a.cols + column] = s;
    }
}

// Adds the blocks' sums: 32 columns for each block, 32 warps that take every 32nd partial sum.
struct LnFinish {
    const float* part;
    void*        dw;
    void*        db;
    int          parts, cols, bf16, accumulate;
};

__global__ void __launch_bounds__(1024)
k_ln_finish(const __grid_constant__ LnFinish f)
{
    __shared__ float s[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane, which = blockIdx.y;
    void* const out = which ? f.db : f.dw;
    if (!out) return;
    wait_for_previous_grid();
    float v = 0.f;
    if (col < f.cols)
        for (int p = warp; p < f.parts; p += 32) v += f.part[(2ll * p + which) * f.cols + col];
    s[warp][lane] = v;
    __syncthreads();
    if (warp != 0 || col >= f.cols) return;
    float t = 0.f;
    for (int g = 0; g < 32; ++g) t += s[g][lane];
    if (f.bf16) {
        __nv_bfloat16* const o = static_cast<__nv_bfloat16*>(out) + col;
        *o = __float2bfloat16_rn(f.accumulate ? to_float(*o) + t : t);
    } else {
        float* const o = static_cast<float*>(out) + col;
        *o = f.accumulate ? *o + t : t;
    }
}

// ---- host ---------------------------------------------------------------------------------------

came_status validate_ln(const came_layernorm* l, bool backward)
{
    if (!l) return report(CAME_ERR_NULL, "descriptor is NULL");
    if (l->rows < 0 || l->rows > (1ll << 30) || l->cols < 1 || l->cols > (1ll << 27))
        return report(CAME_ERR_SHAPE, "rows must lie in [0, 2^30], cols in [1, 2^27]");
    const bool dx = backward && l->dx;
    auto ld_ok = [&](int64_t ld) { return ld >= l->cols && ld <= (1ll << 29) && ld <= (1ll << 40) / std::max<int64_t>(1, l->rows); };
    if (!ld_ok(l->x_ld) || !ld_ok(l->y_ld) || (dx && !ld_ok(l->dx_ld)))
        return report(CAME_ERR_SHAPE, "a row stride is below cols, or too large");
    if (!known_dtype(l->x_dtype) || !known_dtype(l->y_dtype) || !known_dtype(l->weight_dtype) || (dx && !known_dtype(l->dx_dtype)))
        return report(CAME_ERR_DTYPE, "unknown dtype");
    if (l->flags & ~static_cast<uint32_t>(CAME_LAYERNORM_ACCUMULATE)) return report(CAME_ERR_UNSUPPORTED, "unknown flag");
    if (l->flags && !backward) return report(CAME_ERR_UNSUPPORTED, "the flags apply to the backward pass only");
    if (l->reserved) return report(CAME_ERR_SHAPE, "reserved must be 0");
    if (!backward && !(l->eps >= 0 && l->eps <= FLT_MAX)) return report(CAME_ERR_HPARAM, "eps must be finite and >= 0");
    if (l->rows) {
        if (!l->x || (backward ? !l->dy || !l->mean || !l->rstd : !l->y)) return report(CAME_ERR_NULL, "a required buffer is NULL");
        if (!l->mean != !l->rstd) return report(CAME_ERR_NULL, "mean and rstd belong together");
    }
    const size_t xs = dtype_bytes(l->x_dtype), ys = dtype_bytes(l->y_dtype), ws = dtype_bytes(l->weight_dtype), ds = dtype_bytes(l->dx_dtype);
    const void* const y = backward ? l->dy : l->y;
    if (!aligned_to(l->x, xs) || !aligned_to(y, ys) || !aligned_to(l->weight, ws) || !aligned_to(l->mean, 4) || !aligned_to(l->rstd, 4) ||
        (backward ? (dx && !aligned_to(l->dx, ds)) || !aligned_to(l->dweight, ws) || !aligned_to(l->dbias, ws) : !aligned_to(l->bias, ws)))
        return report(CAME_ERR_ALIGN, "a pointer is not aligned to its element size");
    struct Range { uintptr_t lo, hi; bool out; } r[9];
    int n = 0;
    auto add = [&](const void* p, unsigned long long bytes, bool out) {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
        if (p && bytes) r[n++] = Range{lo, lo + bytes, out};
    };
    auto span = [&](int64_t ld, size_t b) { return l->rows ? ((l->rows - 1) * ld + l->cols) * static_cast<unsigned long long>(b) : 0ull; };
    add(l->x, span(l->x_ld, xs), false);
    add(y, span(l->y_ld, ys), !backward);
    add(l->weight, l->cols * ws, false);
    add(l->mean, l->rows * 4ull, !backward);
    add(l->rstd, l->rows * 4ull, !backward);
    if (backward) {
        if (dx) add(l->dx, span(l->dx_ld, ds), true);
        add(l->dweight, l->cols * ws, true);
        add(l->dbias, l->cols * ws, true);
    } else {
        add(l->bias, l->cols * ws, false);
    }
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if ((r[i].out || r[j].out) && r[i].lo < r[j].hi && r[j].lo < r[i].hi)
                return report(CAME_ERR_OVERLAP, "a buffer that is written shares memory with another");
    return CAME_OK;
}

// How the rows of all tensors can be accessed: eight elements at a time, aligned, where they begin at the same places.
struct Access {
    bool wide;                           // every row begins at a multiple of eight elements, and has such a length
    int  period;                         // else: rows until the places repeat, 1 to 8; 0: not at the same places
};

Access access_of(const came_layernorm& l, bool backward)
{
    Access a = {true, 0};
    bool same = true;                    // all tensors begin aligned, and their strides agree modulo 8
    auto rows = [&](const void* p, int64_t ld, int32_t dt) {
        same = same && aligned_to(p, 8 * dtype_bytes(dt)) && ld % 8 == l.x_ld % 8;
    };
    rows(l.x, l.x_ld, l.x_dtype);
    rows(backward ? l.dy : l.y, l.y_ld, l.y_dtype);
    if (backward && l.dx) rows(l.dx, l.dx_ld, l.dx_dtype);
    a.wide = same && l.cols % 8 == 0 && l.x_ld % 8 == 0 && aligned_to(l.weight, 8 * dtype_bytes(l.weight_dtype)) &&
             (backward || aligned_to(l.bias, 8 * dtype_bytes(l.weight_dtype)));
    if (same)
        for (a.period = 1; a.period * l.x_ld % 8; a.period *= 2) {}
    return a;
}

// Threads per row, in whole warps, where each holds `held` elements.
int threads_per_row(long long cols, int held) { return static_cast<int>((cols + 32 * held - 1) / (32 * held)) * 32; }

// Blocks of `groups` groups that take `at_once` rows each time: no more than have rows, and groups for every place.
int blocks_for(long long rows, int groups, int at_once, int period)
{
    const long long want = std::min<long long>((rows + at_once * groups - 1) / (at_once * groups), kSMs);
    return static_cast<int>(std::max<long long>({1, want, (period + groups - 1) / groups}));
}

struct BackwardPlan { int held, tpr, threads, stages, blocks, column_blocks; Access access; size_t smem, means, part, bytes; };

BackwardPlan plan_backward(const came_layernorm& l)
{
    BackwardPlan p = {};
    p.access = access_of(l, true);
    const size_t pair = dtype_bytes(l.x_dtype) + dtype_bytes(l.y_dtype);
    const bool sums = l.dweight || l.dbias;
    const int64_t span = l.cols + (p.access.wide ? 0 : 7);       // columns, and the place of the first
    // elements of a row per thread (0: the row does not fit a block, or its tensors' rows begin at different places)
    // 32 for bf16 rows that one warp then holds, without a barrier (131072 x 768: 108 us, 127 with 16; 512 columns 83 and 75), and
    // where 16 would leave the block few threads (65536 x 5120: 384 and 480).  Else 16: what 32 reads again costs more than its fewer
    // barriers save (128k x 4096 under load: 584 us, 605 with 32).  fp32 leaves too few places in the ring for 32 (65536 x 5120:
    // 1068 us, 663 with 16).
    auto busy = [&](int held) { const int tpr = threads_per_row(span, held); return kBlockThreads / tpr * tpr >= kBlockThreads * 7 / 8; };
    if (!p.access.period) p.held = 0;
    else if (span <= 8 * 32) p.held = 8;
    else if (pair <= 4 && span <= 32 * kBlockThreads && ((p.access.wide && l.cols > 512 && l.cols <= 1024) || (!busy(16) && busy(32)))) p.held = 32;
    else if (span <= 16 * kBlockThreads) p.held = 16;
    else if (span <= 32 * kBlockThreads) p.held = 32;
    if (p.held) {
        p.tpr = threads_per_row(span, p.held);
        const int groups = std::max(1, kBlockThreads / p.tpr);
        p.threads = groups * p.tpr;
        const size_t stage = p.held * pair * p.threads, weights = p.held == 32 ? sizeof(float) * 32 * p.threads : 0;
        p.blocks = blocks_for(l.rows, groups, 1, p.access.period);
        // (no more places than a group has rows, and one)
        const long long turns = l.rows / std::max(1, p.blocks * groups / p.access.period * p.access.period) + 2;
        p.stages = static_cast<int>(std::max<long long>(2, std::min<long long>({kMaxStages, static_cast<long long>((kRingBytes - weights) / stage), turns})));
        p.smem = std::max(weights + stage * p.stages, groups > 1 && sums ? sizeof(float) * 16 * groups * sums_width(static_cast<int>(l.cols)) : 0);
        if (p.smem > kRingBytes) p.held = 0;
    }
    if (!p.held) {
        const int v = p.access.wide ? 8 : 1;
        p.column_blocks = static_cast<int>((l.cols + 32 * v - 1) / (32 * v));
        const long long want = (l.rows + 7) / 8;
        // (and at most 512 rows one after another for a warp)
        const long long blocks = std::max<long long>({1, kSMs * 8 / p.column_blocks, (l.rows + 4095) / 4096});
        p.blocks = static_cast<int>(std::max(1ll, std::min({want, blocks, 65535ll})));
    }
    size_t at = 0;
    auto take = [&](size_t b) { const size_t here = at; at += (b + 255) / 256 * 256; return here; };
    p.means = take(!p.held && l.dx ? sizeof(float2) * l.rows : 0);
    p.part = take(sums ? 8ull * p.blocks * l.cols : 0);
    p.bytes = std::max<size_t>(at, 256);
    return p;
}

template <typename X, int E, bool kSkew>
cudaError_t launch_forward_rows(LnArgs a, int32_t device, cudaStream_t stream)
{
    static std::atomic<uint64_t> done{0};
    auto* const kernel = k_ln_forward_rows<X, E / 8, kSkew>;
    const cudaError_t e = allow_smem(kernel, kRingBytes, device, done);
    if (e != cudaSuccess) return e;
    a.tpr = threads_per_row(a.cols + (kSkew ? 7 : 0), E);
    const int groups = std::max(1, kBlockThreads / a.tpr), threads = groups * a.tpr;
    const int stage = 2 * E * static_cast<int>(sizeof(X)) * threads;         // (64 KB at most)
    a.stages = std::min(kMaxStages, kRingBytes / stage);
    kernel<<<blocks_for(a.rows, groups, 2, a.period), threads, static_cast<size_t>(stage) * a.stages, stream>>>(a);
    return cudaGetLastError();
}

template <typename X, int V, int C, int R>
cudaError_t launch_forward_once(LnArgs a, int threads, cudaStream_t stream)
{
    a.tpr = threads_per_row(a.cols, V * C);
    const int groups = std::max(1, threads / a.tpr);
    const long long at_once = static_cast<long long>(groups) * R;
    k_ln_forward<X, V, C, R><<<static_cast<unsigned>((a.rows + at_once - 1) / at_once), groups * a.tpr, 0, stream>>>(a);
    return cudaGetLastError();
}

template <typename X, int V>
cudaError_t launch_forward_v(const LnArgs& a, cudaStream_t stream)
{
    // Few rows: as many threads for each as there are accesses.  More rows: more elements for a thread.
    if (a.rows <= 2 * kSMs && a.cols <= 8 * 1024) return launch_forward_once<X, V, 8 / V, 1>(a, 0, stream);
    if (a.cols <= (V == 8 ? 8 * 32 : 8 * 1024)) return launch_forward_once<X, V, 8 / V, 1>(a, 256, stream);
    if constexpr (V == 8) {
        // (two rows share the parameters and the barriers; rows beyond 8192 columns leave too few warps for that: 32768 rows of
        // 16384 bf16 528 us, 605 in twos)
        if (a.cols <= 16 * 512) return launch_forward_once<X, 8, 2, 2>(a, 256, stream);
        if (a.cols <= 32 * 1024) return launch_forward_once<X, 8, 4, 1>(a, 256, stream);
    }
    if (a.cols > kRun * 1024 * V) k_ln_forward_long<X, V, true><<<a.rows, 1024, 0, stream>>>(a);
    else k_ln_forward_long<X, V, false><<<a.rows, 1024, 0, stream>>>(a);
    return cudaGetLastError();
}

template <typename X>
cudaError_t launch_forward(LnArgs a, const Access& access, int32_t device, cudaStream_t stream)
{
    a.period = std::max(1, access.period);
    const long long span = a.cols + (access.wide ? 0 : 7);
    // Many rows, and a block holds them.  Not wide fp32 rows of more than 256 columns (a block per few rows is faster, 612 against
    // 735 us at 128k x 4096: fewer instructions for a byte, so that occupancy hides the latency), nor wide ones that leave a
    // block few threads (65536 x 5120 bf16: 316 against 377).
    const bool many = static_cast<long long>(a.rows) * a.cols >= kManyElements, narrow = span <= 8 * 32;
    const int tpr = threads_per_row(span, 16);
    if (access.period && span <= 16 * kBlockThreads && many &&
        (!access.wide || narrow || (sizeof(X) == 2 && kBlockThreads / tpr * tpr >= kBlockThreads * 7 / 8))) {
        if (access.wide) return narrow ? launch_forward_rows<X, 8, false>(a, device, stream) : launch_forward_rows<X, 16, false>(a, device, stream);
        return narrow ? launch_forward_rows<X, 8, true>(a, device, stream) : launch_forward_rows<X, 16, true>(a, device, stream);
    }
    return access.wide ? launch_forward_v<X, 8>(a, stream) : launch_forward_v<X, 1>(a, stream);
}

template <typename X, typename G, int E, bool kSkew>
cudaError_t launch_held(LnArgs a, const BackwardPlan& p, int32_t device, cudaStream_t stream)
{
    static std::atomic<uint64_t> done{0};
    auto* const kernel = k_ln_backward<X, G, E / 8, E != 32, kSkew>;
    const cudaError_t e = allow_smem(kernel, kRingBytes, device, done);
    if (e != cudaSuccess) return e;
    a.tpr = p.tpr;
    a.stages = p.stages;
    a.period = p.access.period;
    kernel<<<p.blocks, p.threads, p.smem, stream>>>(a);
    return cudaGetLastError();
}

template <typename X, typename G, int V>
cudaError_t launch_by_columns(const LnArgs& a, const BackwardPlan& p, float2* means, cudaStream_t stream)
{
    const int threads = std::min(1024, threads_per_row(a.cols, V));
    if (a.y) k_ln_backward_rows<X, G, V><<<a.rows, threads, 0, stream>>>(a, means);
    k_ln_backward_columns<X, G, V><<<dim3(p.column_blocks, p.blocks), 256, 0, stream>>>(a, means);
    return cudaGetLastError();
}

template <typename X, typename G>
cudaError_t launch_backward(const LnArgs& a, const BackwardPlan& p, float2* means, int32_t device, cudaStream_t stream)
{
    if (p.access.wide) {
        if (p.held == 8) return launch_held<X, G, 8, false>(a, p, device, stream);
        if (p.held == 16) return launch_held<X, G, 16, false>(a, p, device, stream);
        if (p.held == 32) return launch_held<X, G, 32, false>(a, p, device, stream);
        return launch_by_columns<X, G, 8>(a, p, means, stream);
    }
    if (p.held == 8) return launch_held<X, G, 8, true>(a, p, device, stream);
    if (p.held == 16) return launch_held<X, G, 16, true>(a, p, device, stream);
    if (p.held == 32) return launch_held<X, G, 32, true>(a, p, device, stream);
    return launch_by_columns<X, G, 1>(a, p, means, stream);
}

LnArgs args_of(const came_layernorm& l, bool backward)
{
    LnArgs a = {};
    a.x = l.x;
    a.w = l.weight;
    a.b = backward ? nullptr : l.bias;
    a.y = backward ? l.dx : l.y;
    a.dy = backward ? l.dy : nullptr;
    a.mean = l.mean;
    a.rstd = l.rstd;
    a.rows = static_cast<int>(l.rows);
    a.cols = static_cast<int>(l.cols);
    a.x_ld = l.x_ld;
    a.y_ld = backward ? l.dx_ld : l.y_ld;
    a.dy_ld = l.y_ld;
    a.eps = static_cast<float>(l.eps);
    a.inv_cols = static_cast<float>(1.0 / static_cast<double>(l.cols));
    a.w_bf16 = l.weight_dtype == CAME_BF16;
    a.y_bf16 = (backward ? l.dx_dtype : l.y_dtype) == CAME_BF16;
    return a;
}

}  // namespace

extern "C" {

came_status came_layernorm_forward(const came_layernorm* l, int32_t device, void* cuda_stream)
{
    came_status s = validate_ln(l, false);
    if (s != CAME_OK) return s;
    if ((s = require_current_device(device)) != CAME_OK) return s;
    if (l->rows == 0) return CAME_OK;
    const LnArgs a = args_of(*l, false);
    const Access access = access_of(*l, false);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = l->x_dtype == CAME_BF16 ? launch_forward<__nv_bfloat16>(a, access, device, stream)
                                                  : launch_forward<float>(a, access, device, stream);
    return e == cudaSuccess ? CAME_OK : report_cuda(e, "kernel launch");
}

came_status came_layernorm_workspace(const came_layernorm* l, int64_t* out_bytes)
{
    if (!out_bytes) return report(CAME_ERR_NULL, "out_bytes is NULL");
    const came_status s = validate_ln(l, true);
    if (s != CAME_OK) return s;
    *out_bytes = static_cast<int64_t>(plan_backward(*l).bytes);
    return CAME_OK;
}

came_status came_layernorm_backward(const came_layernorm* l, void* workspace, int64_t workspace_bytes, int32_t device, void* cuda_stream)
{
    came_status s = validate_ln(l, true);
    if (s != CAME_OK) return s;
    const BackwardPlan p = plan_backward(*l);
    if (!workspace) return report(CAME_ERR_NULL, "workspace is NULL");
    if (!aligned_to(workspace, 16)) return report(CAME_ERR_ALIGN, "workspace not 16-byte aligned");
    if (workspace_bytes < static_cast<int64_t>(p.bytes)) return report(CAME_ERR_SHAPE, "workspace smaller than came_layernorm_workspace says");
    if ((s = require_current_device(device)) != CAME_OK) return s;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    char* const ws = static_cast<char*>(workspace);
    const bool sums = l->dweight || l->dbias;
    LnArgs a = args_of(*l, true);
    if (sums) a.part = reinterpret_cast<float*>(ws + p.part);
    float2* const means = reinterpret_cast<float2*>(ws + p.means);
    cudaError_t e = cudaSuccess;
    if (l->rows && (a.y || sums)) {
        if (l->x_dtype == CAME_BF16)
            e = l->y_dtype == CAME_BF16 ? launch_backward<__nv_bfloat16, __nv_bfloat16>(a, p, means, device, stream)
                                        : launch_backward<__nv_bfloat16, float>(a, p, means, device, stream);
        else
            e = l->y_dtype == CAME_BF16 ? launch_backward<float, __nv_bfloat16>(a, p, means, device, stream)
                                        : launch_backward<float, float>(a, p, means, device, stream);
    }
    if (e == cudaSuccess && sums && (l->rows || !(l->flags & CAME_LAYERNORM_ACCUMULATE))) {
        LnFinish f{a.part, l->dweight, l->dbias, l->rows ? p.blocks : 0, a.cols, a.w_bf16, (l->flags & CAME_LAYERNORM_ACCUMULATE) ? 1 : 0};
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>((l->cols + 31) / 32), 2);
        cfg.blockDim = dim3(1024);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, k_ln_finish, f);
        if (e == cudaSuccess) e = cudaGetLastError();
    }
    return e == cudaSuccess ? CAME_OK : report_cuda(e, "kernel launch");
}

}  // extern "C"
