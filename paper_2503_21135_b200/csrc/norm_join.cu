// Where a block's output joins the residual stream: the norm behind the block, its gate, the residual scale, and the norm in
// front of the next block, in one pass; and the gradient.
//
//   s_y = rsqrt(mean(y^2) + eps),  z = y s_y w_post (z = y without that norm),  g = gate of the channel or token, or 1
//   r'  = res_scale r + block_scale g z                       (rounded to the stream's type once, when stored)
//   s_r = rsqrt(mean(r'^2) + eps),  n = r' s_r w_pre          (of r' in fp32, before that rounding)
//
// Gradient, with G the whole gradient of r' and u = w_pre dn:
//   G  = dr' + s_r u - (s_r r') s_r (s_r A / d),    A = sum(u r')
//   dr = res_scale G,  dz = block_scale g G,  dg = block_scale sum(z G) over the channel's tokens or the token's channels
//   dy = s_y v - (s_y y) s_y (s_y sum(v y) / d),  v = dz w_post;   dw_post = sum_t dz y s_y,  dw_pre = sum_t dn r' s_r
// Powers of a factor are never worked out: the cube leaves the range of fp32 at factors of 1e13 and 1e-13 (rows near zero with a tiny
// eps, rows of large values), where the gradient does not.
// sum(v y) is linear in A, so that A, sum(v y) with A = 0 and what multiplies A are summed in ONE reduction over the row.
// The backward pass works r' out again from y and r, in fp32: no rounded r' enters it.
//
// A row is held in registers between its reduction(s) and its stores, so that every byte moves once: bound by memory.
#include <algorithm>
#include <type_traits>

#include "../../include/dynamo.h"
#include "common.cuh"
#include "f32x2.cuh"
#include "vec8.cuh"

namespace dyn {

struct JoinArgs {
    const void* r;        // [T, d] stream in
    const void* y;        // [T, d] block output, or NULL: r' = r, nothing stored
    const void* w_post;   // [d] or NULL: ones
    const void* w_pre;    // [d] or NULL: ones
    const void* gate;     // [d] (of the weights' type) or [T] fp32 or NULL
    void* r_out;          // [T, d] or NULL
    void* n_out;          // [T, d] or NULL
    float* stats;         // [T, 2] s_y, s_r; forward: or NULL
    // backward
    const void* d_n;      // [T, d] or NULL (zero)
    const void* d_r_out;  // [T, d] or NULL (zero)
    void* d_r;            // [T, d] or NULL
    void* d_y;            // [T, d] or NULL
    float* d_gate;        // [T] for a token gate
    float* part;          // [CTA][2][d] sums of a CTA's rows: S1 (see norm_join_grad_kernel), d_w_pre
    int T, d;
    int gate_kind, post, pre, n_f32, w_f32;
    float res_scale, block_scale, eps;
};

// Eight weights from column c on (ones where there are none).
__device__ __forceinline__ void weights8(const void* w, int w_f32, int c, float (&v)[8]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.f;
    } else if (w_f32) {
        const float4 a = *reinterpret_cast<const float4*>((const float*)w + c), b = *reinterpret_cast<const float4*>((const float*)w + c + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
        Raw8<__nv_bfloat16> raw;
        raw.a = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)w + c);
        unpack8(raw, v);
    }
}

__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16>& r, F2 (&v)[4]) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, F2 (&v)[4]) {
    v[0] = f2(__uint_as_float(r.a.x), __uint_as_float(r.a.y));
    v[1] = f2(__uint_as_float(r.a.z), __uint_as_float(r.a.w));
    v[2] = f2(__uint_as_float(r.b.x), __uint_as_float(r.b.y));
    v[3] = f2(__uint_as_float(r.b.z), __uint_as_float(r.b.w));
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const F2 (&v)[4]) {
    const float f[8] = {lo(v[0]), hi(v[0]), lo(v[1]), hi(v[1]), lo(v[2]), hi(v[2]), lo(v[3]), hi(v[3])};
    store8(p, f);
}

// Eight columns that are read twice: by loads that the compiler may not merge with the first ones (the values would stay in registers).
__device__ __forceinline__ uint4 reread16(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ Raw8<__nv_bfloat16> reread8(const __nv_bfloat16* p) { return {reread16(p)}; }
__device__ __forceinline__ Raw8<float> reread8(const float* p) { return {reread16(p), reread16(p + 4)}; }

// Sum of a value over the TPR threads of a row; every thread gets it.  `scratch`: [TPR / 32], two of them in turn.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* scratch) {
    constexpr int W = TPR / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (W > 1) {
        if (lane == 0) scratch[warp] = v;
        __syncthreads();
        v = scratch[lane & (W - 1)];
#pragma unroll
        for (int o = W / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    return v;
}
// Sums of three values.  They are reduced together: at the first two steps a lane gives half of what it holds away and keeps
// half, so that eight lanes end up with one of them each (6 shuffles instead of 15, and 3 instead of 12 across the warps).
// `scratch`: [4][TPR / 32].
template <int TPR>
__device__ __forceinline__ void row_sums(float (&v)[3], float* scratch) {
    constexpr int W = TPR / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool up16 = lane & 16, up8 = lane & 8;
    const float k0 = (up16 ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, up16 ? v[0] : v[2], 16);
    const float k1 = (up16 ? 0.f : v[1]) + __shfl_xor_sync(0xffffffffu, up16 ? v[1] : 0.f, 16);
    float k = (up8 ? k1 : k0) + __shfl_xor_sync(0xffffffffu, up8 ? k0 : k1, 8);   // value lane >> 3 (the fourth: nothing)
#pragma unroll
    for (int o = 4; o; o >>= 1) k += __shfl_xor_sync(0xffffffffu, k, o);
    if constexpr (W > 1) {
        constexpr int PER = W < 8 ? 1 : W / 8;
        if ((lane & 7) == 0) scratch[(lane >> 3) * W + warp] = k;
        __syncthreads();
        const float* at = scratch + (lane >> 3) * W + (lane & (W / PER - 1) & 7) * PER;
        k = at[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) k += at[i];
#pragma unroll
        for (int o = W / PER / 2; o; o >>= 1) k += __shfl_xor_sync(0xffffffffu, k, o);
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] = __shfl_sync(0xffffffffu, k, 8 * i);
}

// A CTA has one row at a time; where a row takes one warp, four.
__host__ __device__ constexpr int threads_of(int tpr) { return tpr < 64 ? 128 : tpr; }
// CTAs of `threads` threads that share an SM when each thread may have `regs` registers.
__host__ __device__ constexpr int ctas_of(int threads, int regs) { return 65536 / regs / threads < 1 ? 1 : 65536 / regs / threads; }
// Registers a thread, forward and backward.  Two CTAs of 512 threads share an SM in the forward pass (4096 columns; one and
// a half times as many registers, 96, 25.1 against 24.7 us, fewer, 42, 34), one in the backward one (64 registers 70 us
// against 42.9).  Two runs a thread instead: forward 25.1, backward 65 us at 128 registers, 44 at 168.
__host__ __device__ constexpr int join_regs() { return 64; }
__host__ __device__ constexpr int grad_regs() { return 128; }

// What a column needs of the weights: the post-norm's times the channel's gate, and the pre-norm's.
__device__ __forceinline__ void post_weights(const JoinArgs& a, int c, F2 (&p)[4]) {
    float w[8], k[8];
    weights8(a.post ? a.w_post : nullptr, a.w_f32, c, w);
    weights8(a.gate_kind == DYNAMO_GATE_CHANNEL ? a.gate : nullptr, a.w_f32, c, k);
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = f2(w[2 * j] * k[2 * j], w[2 * j + 1] * k[2 * j + 1]);
}
__device__ __forceinline__ void pre_weights(const JoinArgs& a, int c, F2 (&q)[4]) {
    float w[8];
    weights8(a.w_pre, a.w_f32, c, w);
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = f2(w[2 * j], w[2 * j + 1]);
}

// Asks for a thread's eight columns of a row that is read later; a line is asked for by the thread whose piece begins it.
template <typename T>
__device__ __forceinline__ void ask_for(const T* p) {
    if (((uintptr_t)p & 127) < 8 * sizeof(T)) asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}

// TPR threads a row, V runs of eight columns a thread (run i of thread t: columns 8 (t + i TPR)).  The CTAs that the SMs hold walk
// the rows, each thread with its columns' weights in registers and the next row on its way while it works on the present one.
// What bounds it is instructions as much as memory: two columns an instruction (f32x2).  4096 rows of 4096, bf16, gate per
// channel: 24.7 us, 5.4 TB/s of rows; 36.7 with a CTA a row that read the weights for it (half as many bytes again as the
// row's), 30.9 with one column an instruction.
// KEEP = false (rows too wide for that): weights and rows are read when they are used, the next row asked for ahead (1024 rows of 16384,
// bf16: 33.2 us; 36.4 without).
template <typename TY, typename TR, int TPR, int V, bool KEEP>
__global__ void __launch_bounds__(threads_of(TPR), ctas_of(threads_of(TPR), join_regs()))
    norm_join_kernel(const __grid_constant__ JoinArgs a) {
    constexpr int THREADS = threads_of(TPR), ROWS = THREADS / TPR, W = TPR / 32;
    __shared__ float scratch[2][W];
    pdl_prologue();
    const int tt = threadIdx.x % TPR, d = a.d;
    const float inv_d = 1.f / (float)d;
    F2 p[V][4], q[V][4];
    struct Row {
        Raw8<TY> y[V];
        Raw8<TR> r[V];
        float gt;
    };
    auto fetch = [&](Row& R, long long t) {
        const bool there = t < a.T;
        R.gt = there && a.gate_kind == DYNAMO_GATE_TOKEN ? ((const float*)a.gate)[t] : 1.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            const bool in = there && c < d;
            R.y[i] = a.y && in ? load8((const TY*)a.y + t * d + c) : zero8<TY>();
            R.r[i] = in ? load8((const TR*)a.r + t * d + c) : zero8<TR>();
        }
    };
    const long long step = (long long)gridDim.x * ROWS;
    long long t = (long long)blockIdx.x * ROWS + threadIdx.x / TPR;
    Row R;
    fetch(R, t);
    if constexpr (KEEP)
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (8 * (tt + i * TPR) < d) {
                post_weights(a, 8 * (tt + i * TPR), p[i]);
                pre_weights(a, 8 * (tt + i * TPR), q[i]);
            }
    const F2 res = f2(a.y ? a.res_scale : 1.f);
    for (; t < a.T; t += step) {
        F2 y[V][4], x[V][4];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            unpack8(R.y[i], y[i]);
            unpack8(R.r[i], x[i]);
        }
        const float gate = a.block_scale * R.gt;
        if constexpr (KEEP) fetch(R, t + step);   // on its way from here on, into the registers that were just read
        else if (t + step < a.T)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = 8 * (tt + i * TPR);
                if (c >= d) continue;
                if (a.y) ask_for((const TY*)a.y + (t + step) * d + c);
                ask_for((const TR*)a.r + (t + step) * d + c);
            }
        float s_y = 1.f;
        if (a.post) {
            F2 sum2 = f2(0.f);
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum2 = fma2(y[i][j], y[i][j], sum2);
            s_y = rsqrtf(fmaf(row_sum<TPR>(lo(sum2) + hi(sum2), scratch[0]), inv_d, a.eps));
        }
        const F2 g = f2(gate * s_y);
        F2 sum2 = f2(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            if (a.y && c < d) {
                if constexpr (!KEEP) post_weights(a, c, p[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i][j] = fma2(g, mul2(p[i][j], y[i][j]), mul2(res, x[i][j]));
                store8((TR*)a.r_out + t * d + c, x[i]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) sum2 = fma2(x[i][j], x[i][j], sum2);
        }
        float s_r = 1.f;
        if (a.pre) {
            s_r = rsqrtf(fmaf(row_sum<TPR>(lo(sum2) + hi(sum2), scratch[1]), inv_d, a.eps));
            const F2 s2 = f2(s_r);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = 8 * (tt + i * TPR);
                if (c >= d) continue;
                if constexpr (!KEEP) pre_weights(a, c, q[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i][j] = mul2(q[i][j], mul2(x[i][j], s2));
                if (a.n_f32) store8((float*)a.n_out + t * d + c, x[i]);
                else store8((__nv_bfloat16*)a.n_out + t * d + c, x[i]);
            }
        }
        if (a.stats && tt == 0) *reinterpret_cast<float2*>(a.stats + 2 * t) = make_float2(s_y, s_r);
        if constexpr (!KEEP) fetch(R, t + step);
        // One reduction a row alone would use the same scratch for the next row's: its readers have to be through.
        if constexpr (TPR > 32)
            if (!(a.post && a.pre)) __syncthreads();
    }
}

// The gradient, laid out the same.  What the first pass over a row has worked out in fp32 (r', dr' + s_r u, y, dn) stays in
// registers for the second; the next row's loads go out once it has read the present one's registers.  4096 rows of 4096, bf16,
// gate per channel: 43.4 us with the launch that adds up the CTAs' sums (4.7 TB/s); 47 with every sum reduced by itself and a
// copy of the row that came, 56 with the rows staged in shared memory and read twice.  The column sums of d_w_post and of a channel gate differ by a factor of the column
// (S1 = sum_t block_scale gate_t G y s_y; d_w_post = gate S1, d_gate = w_post S1), so that two sums a column are kept.
template <typename TY, typename TR, typename TN, int TPR, int V, bool KEEP>
__global__ void __launch_bounds__(threads_of(TPR), ctas_of(threads_of(TPR), grad_regs()))
    norm_join_grad_kernel(const __grid_constant__ JoinArgs a) {
    constexpr int THREADS = threads_of(TPR), ROWS = THREADS / TPR, W = TPR / 32;
    __shared__ float scratch[2][4 * W];
    extern __shared__ __align__(16) float s_sum[];   // several rows a CTA: [2][d] for the CTA's column sums
    pdl_prologue();
    const int tt = threadIdx.x % TPR, d = a.d, row0 = threadIdx.x / TPR;
    const float inv_d = 1.f / (float)d;
    F2 acc[2][V][4];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[k][i][j] = f2(0.f);
    F2 p[V][4], q[V][4];
    struct Row {
        Raw8<TY> y[V];
        Raw8<TR> r[V], dr[V];
        Raw8<TN> dn[V];
        float s_y, s_r, gt;
    };
    auto fetch = [&](Row& R, long long t) {
        const bool there = t < a.T;
        const float2 st = there ? *reinterpret_cast<const float2*>(a.stats + 2 * t) : make_float2(1.f, 1.f);
        R.s_y = a.post ? st.x : 1.f;
        R.s_r = st.y;
        R.gt = there && a.gate_kind == DYNAMO_GATE_TOKEN ? ((const float*)a.gate)[t] : 1.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            const bool in = there && c < d;
            R.y[i] = a.y && in ? load8((const TY*)a.y + t * d + c) : zero8<TY>();
            R.r[i] = in ? load8((const TR*)a.r + t * d + c) : zero8<TR>();
            R.dr[i] = a.d_r_out && in ? load8((const TR*)a.d_r_out + t * d + c) : zero8<TR>();
            R.dn[i] = a.d_n && in ? load8((const TN*)a.d_n + t * d + c) : zero8<TN>();
        }
    };
    const long long step = (long long)gridDim.x * ROWS;
    long long t = (long long)blockIdx.x * ROWS + row0;
    Row R;
    fetch(R, t);
    if constexpr (KEEP)
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (8 * (tt + i * TPR) < d) {
                post_weights(a, 8 * (tt + i * TPR), p[i]);
                pre_weights(a, 8 * (tt + i * TPR), q[i]);
            }
    const F2 res = f2(a.y ? a.res_scale : 1.f);
    int turn = 0;
    for (; t < a.T; t += step, turn ^= 1) {
        const float s_y = R.s_y, s_r = R.s_r, gz = a.block_scale * R.gt;
        F2 y[V][4], x[V][4], g[V][4], dn[V][4];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            unpack8(R.y[i], y[i]);
            unpack8(R.r[i], x[i]);
            unpack8(R.dr[i], g[i]);
            unpack8(R.dn[i], dn[i]);
        }
        if constexpr (KEEP) fetch(R, t + step);   // on its way from here on, into the registers that were just read
        // sums over the row: A = u r', B = k z (dr' + s_r u), C = k z r' with k the gate of the channels (the token's and
        // block_scale are put in afterwards); k z = s_y (p y)
        F2 sum2[3] = {f2(0.f), f2(0.f), f2(0.f)};
        {
            const F2 gy2 = f2(gz * s_y), sr2 = f2(s_r);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = 8 * (tt + i * TPR);
                if (c >= d) continue;
                if constexpr (!KEEP) {
                    post_weights(a, c, p[i]);
                    pre_weights(a, c, q[i]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const F2 py = mul2(p[i][j], y[i][j]);
                    x[i][j] = fma2(gy2, py, mul2(res, x[i][j]));
                    const F2 u = mul2(q[i][j], dn[i][j]);
                    g[i][j] = fma2(sr2, u, g[i][j]);
                    sum2[0] = fma2(u, x[i][j], sum2[0]);
                    sum2[1] = fma2(py, g[i][j], sum2[1]);
                    sum2[2] = fma2(py, x[i][j], sum2[2]);
                }
            }
        }
        float sum[3] = {lo(sum2[0]) + hi(sum2[0]), lo(sum2[1]) + hi(sum2[1]), lo(sum2[2]) + hi(sum2[2])};
        row_sums<TPR>(sum, scratch[turn]);
        const float ca = s_r * (s_r * sum[0] * inv_d);             // G = dr' + s_r u - ca (s_r r')
        const float zg = s_y * (sum[1] - ca * (s_r * sum[2]));     // sum(k z G)
        if (a.d_gate && a.gate_kind == DYNAMO_GATE_TOKEN && tt == 0) a.d_gate[t] = a.block_scale * zg;
        const float cv = a.post ? gz * zg * inv_d : 0.f;        // sum(v y) s_y / d
        const F2 ca2 = f2(-ca), gy2 = f2(gz * s_y), cy2 = f2(-cv * s_y), sy2 = f2(s_y), sr2 = f2(s_r);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            if (c >= d) continue;
            if constexpr (!KEEP) post_weights(a, c, p[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const F2 xn = mul2(x[i][j], sr2), G = fma2(ca2, xn, g[i][j]);
                const F2 gG = mul2(gy2, G);
                acc[0][i][j] = fma2(gG, y[i][j], acc[0][i][j]);
                acc[1][i][j] = fma2(dn[i][j], xn, acc[1][i][j]);
                y[i][j] = fma2(p[i][j], gG, mul2(cy2, mul2(sy2, y[i][j])));
                g[i][j] = mul2(res, G);
            }
            if (a.d_r) store8((TR*)a.d_r + t * d + c, g[i]);
            if (a.d_y) store8((TY*)a.d_y + t * d + c, y[i]);
        }
        if constexpr (!KEEP) fetch(R, t + step);
    }
    if (!a.part) return;
    float* part = a.part + (long long)blockIdx.x * 2 * d;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = 8 * (tt + i * TPR);
                if (c < d) store8(part + k * d + c, acc[k][i]);
            }
    } else {
        // the CTA's rows one after another: the order of the sum is fixed
        for (int o = 0; o < ROWS; ++o) {
            if (row0 == o)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int c = 8 * (tt + i * TPR);
                        if (c >= d) continue;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float2* at = reinterpret_cast<float2*>(s_sum + k * d + c + 2 * j);
                            const float2 was = o ? *at : make_float2(0.f, 0.f);
                            *at = make_float2(was.x + lo(acc[k][i][j]), was.y + hi(acc[k][i][j]));
                        }
                    }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * d; c += THREADS) part[c] = s_sum[c];
    }
}

// Eight column sums, in two halves `apart` from one another.
__device__ __forceinline__ void take8(const float4* at, int apart, F2 (&v)[4]) {
    const float4 x = at[0], y = at[apart];
    v[0] = f2(x.x, x.y), v[1] = f2(x.z, x.w), v[2] = f2(y.x, y.y), v[3] = f2(y.z, y.w);
}
__device__ __forceinline__ void give8(float4* at, int apart, const F2 (&v)[4]) {
    at[0] = make_float4(lo(v[0]), hi(v[0]), lo(v[1]), hi(v[1]));
    at[apart] = make_float4(lo(v[2]), hi(v[2]), lo(v[3]), hi(v[3]));
}
// The gradient of rows too wide for a thread's registers to hold: the first pass keeps the sums alone, the second reads the row again
// (from the L1 or L2; the next row is asked for meanwhile) and works the same values out again.  The weights are read when they
// are used; the column sums stand in shared memory, a thread's own columns: [sum][half][run][4].
constexpr int WIDE_THREADS = 512;
template <typename TY, typename TR, typename TN>
__global__ void __launch_bounds__(WIDE_THREADS, 1) norm_join_grad_wide_kernel(const __grid_constant__ JoinArgs a) {
    constexpr int TPR = WIDE_THREADS;
    __shared__ float scratch[2][4 * TPR / 32];
    extern __shared__ __align__(16) float s_sum[];
    pdl_prologue();
    const int tt = threadIdx.x, d = a.d;
    const float inv_d = 1.f / (float)d;
    const F2 res = f2(a.y ? a.res_scale : 1.f);
    const int runs = d / 8;
    float4* const sums = reinterpret_cast<float4*>(s_sum);
    if (a.part)
        for (int i = tt; i < runs; i += TPR)
#pragma unroll
            for (int h = 0; h < 4; ++h) sums[h * runs + i] = make_float4(0.f, 0.f, 0.f, 0.f);
    int turn = 0;
    for (long long t = blockIdx.x; t < a.T; t += gridDim.x, turn ^= 1) {
        const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * t);
        const float s_y = a.post ? st.x : 1.f, s_r = st.y;
        const float gz = a.block_scale * (a.gate_kind == DYNAMO_GATE_TOKEN ? ((const float*)a.gate)[t] : 1.f);
        const F2 gy2 = f2(gz * s_y), sr2 = f2(s_r);
        // y, dn, r' (x), dr' + s_r u (g), u and p y of eight columns
        struct Columns {
            F2 p[4], y[4], dn[4], x[4], g[4], u[4], py[4];
        };
        auto columns = [&](Columns& C, int c) {
            const long long at = t * d + c;
            F2 q[4];
            unpack8(a.y ? reread8((const TY*)a.y + at) : zero8<TY>(), C.y);
            unpack8(reread8((const TR*)a.r + at), C.x);
            unpack8(a.d_r_out ? reread8((const TR*)a.d_r_out + at) : zero8<TR>(), C.g);
            unpack8(a.d_n ? reread8((const TN*)a.d_n + at) : zero8<TN>(), C.dn);
            post_weights(a, c, C.p);
            pre_weights(a, c, q);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                C.py[j] = mul2(C.p[j], C.y[j]);
                C.x[j] = fma2(gy2, C.py[j], mul2(res, C.x[j]));
                C.u[j] = mul2(q[j], C.dn[j]);
                C.g[j] = fma2(sr2, C.u[j], C.g[j]);
            }
        };
        F2 sum2[3] = {f2(0.f), f2(0.f), f2(0.f)};   // as in norm_join_grad_kernel
#pragma unroll 2
        for (int i = tt; i < runs; i += TPR) {
            const int c = 8 * i;
            Columns C;
            columns(C, c);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum2[0] = fma2(C.u[j], C.x[j], sum2[0]);
                sum2[1] = fma2(C.py[j], C.g[j], sum2[1]);
                sum2[2] = fma2(C.py[j], C.x[j], sum2[2]);
            }
            const long long next = (t + gridDim.x) * d + c;
            if (t + gridDim.x < a.T) {
                if (a.y) ask_for((const TY*)a.y + next);
                ask_for((const TR*)a.r + next);
                if (a.d_r_out) ask_for((const TR*)a.d_r_out + next);
                if (a.d_n) ask_for((const TN*)a.d_n + next);
            }
        }
        float sum[3] = {lo(sum2[0]) + hi(sum2[0]), lo(sum2[1]) + hi(sum2[1]), lo(sum2[2]) + hi(sum2[2])};
        row_sums<TPR>(sum, scratch[turn]);
        const float ca = s_r * (s_r * sum[0] * inv_d), zg = s_y * (sum[1] - ca * (s_r * sum[2]));
        if (a.d_gate && a.gate_kind == DYNAMO_GATE_TOKEN && tt == 0) a.d_gate[t] = a.block_scale * zg;
        const float cv = a.post ? gz * zg * inv_d : 0.f;
        const F2 ca2 = f2(-ca), cy2 = f2(-cv * s_y), sy2 = f2(s_y);
#pragma unroll 2
        for (int i = tt; i < runs; i += TPR) {
            const int c = 8 * i;
            Columns C;
            columns(C, c);
            F2 s1[4] = {f2(0.f), f2(0.f), f2(0.f), f2(0.f)}, s2[4] = {s1[0], s1[0], s1[0], s1[0]};
            if (a.part) {
                take8(sums + i, runs, s1);
                take8(sums + 2 * runs + i, runs, s2);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const F2 xn = mul2(C.x[j], sr2), G = fma2(ca2, xn, C.g[j]);
                const F2 gG = mul2(gy2, G);
                s1[j] = fma2(gG, C.y[j], s1[j]);
                s2[j] = fma2(C.dn[j], xn, s2[j]);
                C.y[j] = fma2(C.p[j], gG, mul2(cy2, mul2(sy2, C.y[j])));
                C.g[j] = mul2(res, G);
            }
            if (a.part) {
                give8(sums + i, runs, s1);
                give8(sums + 2 * runs + i, runs, s2);
            }
            if (a.d_r) store8((TR*)a.d_r + t * d + c, C.g);
            if (a.d_y) store8((TY*)a.d_y + t * d + c, C.y);
        }
    }
    if (!a.part) return;
    float* part = a.part + (long long)blockIdx.x * 2 * d;
    for (int i = tt; i < runs; i += TPR)
#pragma unroll
        for (int h = 0; h < 4; ++h) *reinterpret_cast<float4*>(part + (h >> 1) * d + 8 * i + 4 * (h & 1)) = sums[h * runs + i];
}

// Column sums of the CTAs' partial rows, in a fixed order, and the factors of the two gradients that share one.  grid.y: which
// of the two sums.
__global__ void __launch_bounds__(1024) norm_join_sums_kernel(const __grid_constant__ JoinArgs a, int n_part, float* d_w_post,
                                                             float* d_gate, float* d_w_pre) {
    __shared__ float s[32][32];
    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, d = a.d;
    float sum = 0.f;
    if (c < d)
#pragma unroll 8
        for (int p = warp; p < n_part; p += 32) sum += a.part[((long long)p * 2 + blockIdx.y) * d + c];
    s[warp][lane] = sum;
    __syncthreads();
    if (warp || c >= d) return;
#pragma unroll
    for (int w = 1; w < 32; ++w) sum += s[w][lane];
    if (blockIdx.y) {
        if (d_w_pre) d_w_pre[c] = sum;
        return;
    }
    auto weight = [&](const void* w) { return !w ? 1.f : a.w_f32 ? ((const float*)w)[c] : __bfloat162float(((const __nv_bfloat16*)w)[c]); };
    if (d_w_post) d_w_post[c] = sum * weight(a.gate_kind == DYNAMO_GATE_CHANNEL ? a.gate : nullptr);
    if (d_gate) d_gate[c] = sum * weight(a.post ? a.w_post : nullptr);
}

constexpr int JOIN_MAX_D = 16384;

// Threads a row and runs a thread by the width: a run a thread as far as registers allow, one warp a row (no barrier) while
// that is enough.  The gradient of rows above 8192 has a kernel that keeps no row (V = 0): 1024 rows of 12288 / 16384 bf16 59 / 80 us, 85 / 112
// with two runs in 64 registers of 1024 threads; below, two runs in 128 registers of 512 are faster (2048 rows of 5000 / 8192: 49 / 60 us,
// 70 / 71 without keeping the row).
template <int TPR_, int V_, bool KEEP_>
struct Layout {
    static constexpr int TPR = TPR_, V = V_;
    static constexpr bool KEEP = KEEP_;
};
template <bool GRAD, typename F>
static cudaError_t by_width(int d, F f) {
    if (d <= 256) return f(Layout<32, 1, true>{});
    if (d <= 512) return f(Layout<64, 1, true>{});
    if (d <= 1024) return f(Layout<128, 1, true>{});
    if (d <= 2048) return f(Layout<256, 1, true>{});
    if (d <= 4096) return f(Layout<512, 1, true>{});
    if constexpr (GRAD) return d <= 8192 ? f(Layout<512, 2, false>{}) : f(Layout<WIDE_THREADS, 0, false>{});
    else return d <= 8192 ? f(Layout<1024, 1, true>{}) : f(Layout<1024, 2, false>{});
}
template <typename F>
static cudaError_t by_types(int a, int b, F f) {
    if (a == DYNAMO_BF16) return b == DYNAMO_BF16 ? f((__nv_bfloat16*)nullptr, (__nv_bfloat16*)nullptr) : f((__nv_bfloat16*)nullptr, (float*)nullptr);
    return b == DYNAMO_BF16 ? f((float*)nullptr, (__nv_bfloat16*)nullptr) : f((float*)nullptr, (float*)nullptr);
}

// CTAs of a launch: what the SMs hold at once, and no more than there are rows.
static int join_ctas(int T, int tpr, int per_sm, int n_sms) {
    const int rows = threads_of(tpr) / tpr;
    return (int)std::max(1ll, std::min(((long long)T + rows - 1) / rows, (long long)n_sms * per_sm));
}
static int grad_ctas(int T, int d, int n_sms) {
    int n = 0;
    by_width<true>(d, [&](auto l) {
        constexpr int TPR = decltype(l)::TPR;
        n = join_ctas(T, TPR, ctas_of(threads_of(TPR), grad_regs()), n_sms);
        return cudaSuccess;
    });
    return n;
}

}  // namespace dyn

using namespace dyn;

namespace {

bool dtype_ok(int32_t t) { return t == DYNAMO_BF16 || t == DYNAMO_F32; }

dynamo_status check_join(const dynamo_join_desc* D, int32_t T) {
    if (!D) return DYNAMO_ERR_NULL;
    if (D->d < 8 || D->d % 8 || D->d > JOIN_MAX_D) return DYNAMO_ERR_SHAPE;
    if (!dtype_ok(D->y_dtype) || !dtype_ok(D->r_dtype) || !dtype_ok(D->n_dtype) || !dtype_ok(D->w_dtype)) return DYNAMO_ERR_SHAPE;
    if (D->gate_kind < DYNAMO_GATE_NONE || D->gate_kind > DYNAMO_GATE_TOKEN) return DYNAMO_ERR_ARG;
    if (!(D->eps > 0.f) || !(D->eps < 1e30f)) return DYNAMO_ERR_ARG;   // a row of zeros has a finite norm factor
    if (!(D->res_scale - D->res_scale == 0.f) || !(D->block_scale - D->block_scale == 0.f)) return DYNAMO_ERR_ARG;
    if (T < 0) return DYNAMO_ERR_TOKENS;
    return DYNAMO_OK;
}

JoinArgs join_args(const dynamo_join_desc* D, int32_t T, const void* r, const void* y, const void* w_post, const void* gate,
                   const void* w_pre) {
    JoinArgs a = {};
    a.r = r;
    a.y = y;
    a.w_post = w_post;
    a.w_pre = w_pre;
    a.gate = gate;
    a.T = T;
    a.d = D->d;
    a.gate_kind = y ? D->gate_kind : (int)DYNAMO_GATE_NONE;
    a.post = y && D->post_norm;
    a.pre = D->pre_norm != 0;
    a.n_f32 = D->n_dtype == DYNAMO_F32;
    a.w_f32 = D->w_dtype == DYNAMO_F32;
    a.res_scale = D->res_scale;
    a.block_scale = D->block_scale;
    a.eps = D->eps;
    return a;
}

}  // namespace

namespace dyn {
// What dynamo_norm_join_forward refuses; dynamo_moe_block_forward asks before it launches the layer.
dynamo_status check_join_forward(const dynamo_join_desc* desc, const void* r, const void* y, const void* w_post, const void* gate,
                                      const void* w_pre, int32_t T, const void* r_out, const void* n_out, const float* stats) {
    if (const dynamo_status s = check_join(desc, T); s != DYNAMO_OK) return s;
    if (T == 0) return DYNAMO_OK;
    if (!y && !desc->pre_norm) return DYNAMO_ERR_ARG;   // nothing to do
    if (!r || (y && !r_out) || (desc->pre_norm && !n_out) || (y && desc->gate_kind != DYNAMO_GATE_NONE && !gate)) return DYNAMO_ERR_NULL;
    if (!aligned16(r, y, r_out, n_out) || !aligned16(w_post, w_pre) ||
        (y && desc->gate_kind == DYNAMO_GATE_CHANNEL && !aligned16(gate)) || ((uintptr_t)stats & 7))
        return DYNAMO_ERR_ALIGN;
    return DYNAMO_OK;
}
}  // namespace dyn

extern "C" {

dynamo_status dynamo_norm_join_forward(const dynamo_join_desc* desc, const void* r, const void* y, const void* w_post,
                                       const void* gate, const void* w_pre, int32_t T, void* r_out, void* n_out, float* stats,
                                       void* stream) {
    if (const dynamo_status s = dyn::check_join_forward(desc, r, y, w_post, gate, w_pre, T, r_out, n_out, stats); s != DYNAMO_OK) return s;
    if (T == 0) return DYNAMO_OK;
    int n_sms = 0;
    if (count_sms(&n_sms) != cudaSuccess) return DYNAMO_ERR_CUDA;
    JoinArgs a = join_args(desc, T, r, y, w_post, gate, w_pre);
    a.r_out = y ? r_out : nullptr;
    a.n_out = n_out;
    a.stats = stats;
    const cudaError_t e = by_types(desc->y_dtype, desc->r_dtype, [&](auto* ty, auto* tr) {
        using TY = std::remove_pointer_t<decltype(ty)>;
        using TR = std::remove_pointer_t<decltype(tr)>;
        return by_width<false>(desc->d, [&](auto l) {
            using L = decltype(l);
            constexpr int THREADS = threads_of(L::TPR), PER_SM = ctas_of(THREADS, join_regs());
            return launch_pdl(norm_join_kernel<TY, TR, L::TPR, L::V, L::KEEP>, dim3((unsigned)join_ctas(T, L::TPR, PER_SM, n_sms)),
                              dim3(THREADS), 0, (cudaStream_t)stream, a);
        });
    });
    return e == cudaSuccess ? DYNAMO_OK : DYNAMO_ERR_CUDA;
}

dynamo_status dynamo_norm_join_workspace_bytes(const dynamo_join_desc* desc, int32_t T, size_t* bytes) {
    if (const dynamo_status s = check_join(desc, T); s != DYNAMO_OK) return s;
    if (!bytes) return DYNAMO_ERR_NULL;
    *bytes = (size_t)grad_ctas(T, desc->d, 256) * 2 * desc->d * 4;   // up to 256 SMs are reckoned with
    return DYNAMO_OK;
}

dynamo_status dynamo_norm_join_backward(const dynamo_join_desc* desc, const void* d_n, const void* d_r_out, const void* r,
                                        const void* y, const float* stats, const void* w_post, const void* gate,
                                        const void* w_pre, int32_t T, void* d_r, void* d_y, float* d_w_post, float* d_gate,
                                        float* d_w_pre, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    if (const dynamo_status s = dynamo_norm_join_workspace_bytes(desc, T, &need); s != DYNAMO_OK) return s;
    const bool has_y = y || T == 0;   // an empty array may be NULL
    if (!has_y && !desc->pre_norm) return DYNAMO_ERR_ARG;
    const bool token = has_y && desc->gate_kind == DYNAMO_GATE_TOKEN, channel = has_y && desc->gate_kind == DYNAMO_GATE_CHANNEL;
    if ((d_w_post && !(has_y && desc->post_norm)) || (d_gate && !token && !channel) || (d_w_pre && !desc->pre_norm) || (d_y && !has_y))
        return DYNAMO_ERR_ARG;   // a gradient of something that is not there
    const bool columns = d_w_post || d_w_pre || (channel && d_gate);
    if (T > 0 && (!r || !stats || (desc->pre_norm && !d_n) || ((token || channel) && !gate) || (!desc->pre_norm && !d_r_out)))
        return DYNAMO_ERR_NULL;
    if (columns && !workspace) return DYNAMO_ERR_NULL;
    if (!aligned16(d_n, d_r_out, r, y) || !aligned16(w_post, w_pre, d_r, d_y) || (channel && !aligned16(gate)) || ((uintptr_t)stats & 7) ||
        (columns && ((uintptr_t)workspace & 255)))
        return DYNAMO_ERR_ALIGN;
    if (columns && workspace_bytes < need) return DYNAMO_ERR_ARENA_TOO_SMALL;
    cudaStream_t st = (cudaStream_t)stream;
    int n_sms = 0;
    if (count_sms(&n_sms) != cudaSuccess) return DYNAMO_ERR_CUDA;
    if (T == 0 && !columns) return DYNAMO_OK;
    JoinArgs a = join_args(desc, T, r, y, w_post, gate, w_pre);
    a.stats = const_cast<float*>(stats);
    a.d_n = desc->pre_norm ? d_n : nullptr;
    a.d_r_out = d_r_out;
    a.d_r = d_r;
    a.d_y = d_y;
    a.d_gate = token ? d_gate : nullptr;
    a.part = columns ? (float*)workspace : nullptr;
    const int ctas = grad_ctas(T, desc->d, std::min(n_sms, 256));
    const cudaError_t e = by_types(desc->y_dtype, desc->r_dtype, [&](auto* ty, auto* tr) {
        using TY = std::remove_pointer_t<decltype(ty)>;
        using TR = std::remove_pointer_t<decltype(tr)>;
        return by_width<true>(desc->d, [&](auto l) {
            using L = decltype(l);
            const dim3 grid((unsigned)ctas), block(threads_of(L::TPR));
            const size_t smem = threads_of(L::TPR) > L::TPR ? 2 * desc->d * sizeof(float) : 0;
            if constexpr (L::V == 0) {
                auto wide = [&](auto kernel) {
                    const size_t sums = a.part ? 2 * (size_t)desc->d * sizeof(float) : 0;
                    // (the widest row's, whatever this one's: the limit is the function's, and other threads launch it too)
                    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                               2 * JOIN_MAX_D * (int)sizeof(float));
                    return e != cudaSuccess ? e : launch_pdl(kernel, grid, block, sums, st, a);
                };
                return a.n_f32 ? wide(norm_join_grad_wide_kernel<TY, TR, float>) : wide(norm_join_grad_wide_kernel<TY, TR, __nv_bfloat16>);
            } else {
                return a.n_f32 ? launch_pdl(norm_join_grad_kernel<TY, TR, float, L::TPR, L::V, L::KEEP>, grid, block, smem, st, a)
                               : launch_pdl(norm_join_grad_kernel<TY, TR, __nv_bfloat16, L::TPR, L::V, L::KEEP>, grid, block, smem, st, a);
            }
        });
    });
    if (e != cudaSuccess) return DYNAMO_ERR_CUDA;
    if (columns && launch_pdl(norm_join_sums_kernel, dim3((unsigned)((desc->d + 31) / 32), 2), dim3(1024), 0, st, a, ctas,
                              d_w_post, channel ? d_gate : nullptr, d_w_pre) != cudaSuccess)
        return DYNAMO_ERR_CUDA;
    return DYNAMO_OK;
}

}  // extern "C"
