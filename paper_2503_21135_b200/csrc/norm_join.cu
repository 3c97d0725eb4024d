// Where a block's output joins the residual stream: the norm behind the block, its gate, the residual scale, and the norm in
// front of the next block, in one pass; and the gradient.
//
//   s_y = rsqrt(mean(y^2) + eps),  z = y s_y w_post (z = y without that norm),  g = gate of the channel or token, or 1
//   r'  = res_scale r + block_scale g z                       (rounded to the stream's type once, when stored)
//   s_r = rsqrt(mean(r'^2) + eps),  n = r' s_r w_pre          (of r' in fp32, before that rounding)
//
// Gradient, with G the whole gradient of r' and u = w_pre dn:
//   G  = dr' + s_r u - r' s_r^3 / d * A,            A = sum(u r')
//   dr = res_scale G,  dz = block_scale g G,  dg = block_scale sum(z G) over the channel's tokens or the token's channels
//   dy = s_y (v - y s_y^2 / d * sum(v y)),  v = dz w_post;   dw_post = sum_t dz y s_y,  dw_pre = sum_t dn r' s_r
// sum(v y) is linear in A, so that A, sum(v y) with A = 0 and what multiplies A are summed in ONE reduction over the row.
// The backward pass works r' out again from y and r, in fp32: no rounded r' enters it.
//
// A row is held in registers between its reduction(s) and its stores, so that every byte moves once: bound by memory.
#include <algorithm>
#include <type_traits>

#include "../../include/dynamo.h"
#include "common.cuh"
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

// Sums of N values over the TPR threads of a row; every thread gets them.  `scratch`: [N][TPR / 32], two of them in turn.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* scratch) {
    constexpr int W = TPR / 32;
#pragma unroll
    for (int o = 16; o; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if constexpr (W > 1) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) scratch[i * W + warp] = v[i];
        __syncthreads();
        // the warps' sums by 16-byte reads that all lanes share, added in the order of a tree
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float4 s = *reinterpret_cast<const float4*>(scratch + i * W);
#pragma unroll
            for (int w = 4; w < W; w += 4) {
                const float4 q = *reinterpret_cast<const float4*>(scratch + i * W + w);
                s.x += q.x, s.y += q.y, s.z += q.z, s.w += q.w;
            }
            v[i] = (s.x + s.y) + (s.z + s.w);
        }
    }
}

// CTAs of `threads` threads that share an SM when each thread may have `regs` registers.
__host__ __device__ constexpr int ctas_of(int threads, int regs) { return 65536 / regs / threads < 1 ? 1 : 65536 / regs / threads; }
__host__ __device__ constexpr int threads_of(int tpr) { return tpr < 128 ? 128 : tpr; }
// Registers a thread of the forward kernel: a warp that has a row to itself has several runs' values in flight.
__host__ __device__ constexpr int join_regs(int tpr) { return tpr == 32 ? 128 : 64; }
// What a column needs of the weights: the post-norm's times the channel's gate, and the pre-norm's.
template <int V>
struct ColumnWeights {
    float p[V][8], q[V][8];
    __device__ __forceinline__ void load(const JoinArgs& a, int i, int c) {
        float k[8];
        weights8(a.post ? a.w_post : nullptr, a.w_f32, c, p[i]);
        weights8(a.gate_kind == DYNAMO_GATE_CHANNEL ? a.gate : nullptr, a.w_f32, c, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) p[i][j] *= k[j];
        weights8(a.w_pre, a.w_f32, c, q[i]);
    }
};

// TPR threads a row, V runs of eight columns a thread (run i of thread t: columns 8 (t + i TPR)).  The CTAs that the SMs hold walk
// the rows, each thread with its columns' weights in registers and the next row on its way while it works on the present
// one: at 4096 columns the weights are half as many bytes again as a row's, and with a CTA a row, that read them for it,
// 4096 rows took 36.7 us.  KEEP = false (rows too wide for that): both are read when they are used.
template <typename TY, typename TR, int TPR, int V, bool KEEP>
__global__ void __launch_bounds__(threads_of(TPR), ctas_of(threads_of(TPR), join_regs(TPR))) norm_join_kernel(const __grid_constant__ JoinArgs a) {
    constexpr int THREADS = threads_of(TPR), ROWS = THREADS / TPR, W = TPR / 32;
    __shared__ __align__(16) float scratch[2][W < 4 ? 4 : W];
    pdl_prologue();
    const int tt = threadIdx.x % TPR, d = a.d;
    const float inv_d = 1.f / (float)d;
    ColumnWeights<V> w;
    if constexpr (KEEP)
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (8 * (tt + i * TPR) < d) w.load(a, i, 8 * (tt + i * TPR));
    Raw8<TY> yr[V], yn[V];
    Raw8<TR> rr[V], rn[V];
    auto fetch = [&](Raw8<TY> (&y)[V], Raw8<TR> (&r)[V], long long t) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            const bool in = t < a.T && c < d;
            y[i] = a.y && in ? load8((const TY*)a.y + t * d + c) : zero8<TY>();
            r[i] = in ? load8((const TR*)a.r + t * d + c) : zero8<TR>();
        }
    };
    const long long step = (long long)gridDim.x * ROWS;
    long long t = (long long)blockIdx.x * ROWS + threadIdx.x / TPR;
    if constexpr (KEEP) fetch(yn, rn, t);
    for (; t < a.T; t += step) {
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < V; ++i) yr[i] = yn[i], rr[i] = rn[i];
            fetch(yn, rn, t + step);
        } else {
            fetch(yr, rr, t);
        }
        const float gt = a.gate_kind == DYNAMO_GATE_TOKEN ? ((const float*)a.gate)[t] : 1.f;
        float s_y = 1.f;
        if (a.post) {
            float sum[1] = {0.f};
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float y[8];
                unpack8(yr[i], y);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[0] = fmaf(y[j], y[j], sum[0]);
            }
            row_sums<TPR, 1>(sum, scratch[0]);
            s_y = rsqrtf(fmaf(sum[0], inv_d, a.eps));
        }
        const float g = a.block_scale * gt * s_y;
        float x[V][8];
        float sum[1] = {0.f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            unpack8(rr[i], x[i]);
            if (a.y && c < d) {
                float y[8];
                unpack8(yr[i], y);
                if constexpr (!KEEP) w.load(a, i, c);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = fmaf(g, w.p[i][j] * y[j], a.res_scale * x[i][j]);
                store8((TR*)a.r_out + t * d + c, x[i]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[0] = fmaf(x[i][j], x[i][j], sum[0]);
        }
        float s_r = 1.f;
        if (a.pre) {
            row_sums<TPR, 1>(sum, scratch[1]);
            s_r = rsqrtf(fmaf(sum[0], inv_d, a.eps));
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = 8 * (tt + i * TPR);
                if (c >= d) continue;
                float n[8];
                if constexpr (KEEP) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) n[j] = w.q[i][j];
                } else {
                    weights8(a.w_pre, a.w_f32, c, n);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) n[j] *= x[i][j] * s_r;
                if (a.n_f32) store8((float*)a.n_out + t * d + c, n);
                else store8((__nv_bfloat16*)a.n_out + t * d + c, n);
            }
        }
        if (a.stats && tt == 0) *reinterpret_cast<float2*>(a.stats + 2 * t) = make_float2(s_y, s_r);
        // One reduction a row alone would use the same scratch for the next row's: its readers have to be through.
        if constexpr (TPR > 32)
            if (!(a.post && a.pre)) __syncthreads();
    }
}

// The gradient, laid out the same.  The column sums of d_w_post and of a channel gate differ by a factor of the column
// (S1 = sum_t block_scale gate_t G y s_y; d_w_post = gate S1, d_gate = w_post S1), so that two sums a column are kept.
template <typename TY, typename TR, typename TN, int TPR, int V, bool KEEP>
__global__ void __launch_bounds__(threads_of(TPR), ctas_of(threads_of(TPR), 128)) norm_join_grad_kernel(const __grid_constant__ JoinArgs a) {
    constexpr int THREADS = threads_of(TPR), ROWS = THREADS / TPR, W = TPR / 32;
    __shared__ __align__(16) float scratch[2][3 * (W < 4 ? 4 : W)];
    extern __shared__ float s_sum[];   // several rows a CTA: [2][d] for the CTA's column sums
    pdl_prologue();
    const int tt = threadIdx.x % TPR, d = a.d, row0 = threadIdx.x / TPR;
    const float inv_d = 1.f / (float)d;
    float acc[2][V][8];
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[q][i][j] = 0.f;
    ColumnWeights<V> w;
    if constexpr (KEEP)
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (8 * (tt + i * TPR) < d) w.load(a, i, 8 * (tt + i * TPR));
    struct Row {
        Raw8<TY> y[V];
        Raw8<TR> r[V], dr[V];
        Raw8<TN> dn[V];
        float2 st;
        float gt;
    };
    auto fetch = [&](Row& R, long long t) {
        const bool there = t < a.T;
        R.st = there ? *reinterpret_cast<const float2*>(a.stats + 2 * t) : make_float2(1.f, 1.f);
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
    Row R, next;
    if constexpr (KEEP) fetch(next, t);
    const float res = a.y ? a.res_scale : 1.f;
    int turn = 0;
    for (; t < a.T; t += step, turn ^= 1) {
        if constexpr (KEEP) {
            R = next;
            fetch(next, t + step);
        } else {
            fetch(R, t);
        }
        const float s_y = a.post ? R.st.x : 1.f, s_r = R.st.y, gz = a.block_scale * R.gt;
        // sums over the row: A = u r', B = k z (dr' + s_r u), C = k z r' with k the gate of the channels (the token's and
        // block_scale are put in afterwards)
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            if (c >= d) continue;
            if constexpr (!KEEP) w.load(a, i, c);
            float y[8], r[8], g[8], dn[8];
            unpack8(R.y[i], y);
            unpack8(R.r[i], r);
            unpack8(R.dr[i], g);
            unpack8(R.dn[i], dn);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float kz = w.p[i][j] * (y[j] * s_y);
                const float x = fmaf(gz, kz, res * r[j]);
                const float u = w.q[i][j] * dn[j];
                sum[0] = fmaf(u, x, sum[0]);
                sum[1] = fmaf(kz, fmaf(s_r, u, g[j]), sum[1]);
                sum[2] = fmaf(kz, x, sum[2]);
            }
        }
        row_sums<TPR, 3>(sum, scratch[turn]);
        const float ca = s_r * s_r * s_r * inv_d * sum[0];      // G = dr' + s_r u - ca r'
        const float zg = sum[1] - ca * sum[2];                  // sum(k z G)
        if (a.d_gate && a.gate_kind == DYNAMO_GATE_TOKEN && tt == 0) a.d_gate[t] = a.block_scale * zg;
        const float cv = a.post ? gz * zg * inv_d : 0.f;        // sum(v y) s_y / d
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            if (c >= d) continue;
            if constexpr (!KEEP) w.load(a, i, c);
            float y[8], r[8], g[8], dn[8];
            unpack8(R.y[i], y);
            unpack8(R.r[i], r);
            unpack8(R.dr[i], g);
            unpack8(R.dn[i], dn);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float yn = y[j] * s_y;
                const float x = fmaf(gz, w.p[i][j] * yn, res * r[j]);
                const float G = fmaf(-ca, x, fmaf(s_r, w.q[i][j] * dn[j], g[j]));
                const float gG = gz * G;
                r[j] = res * G;
                y[j] = s_y * fmaf(-cv, yn, w.p[i][j] * gG);
                acc[0][i][j] = fmaf(gG, yn, acc[0][i][j]);
                acc[1][i][j] = fmaf(dn[j], x * s_r, acc[1][i][j]);
            }
            if (a.d_r) store8((TR*)a.d_r + t * d + c, r);
            if (a.d_y) store8((TY*)a.d_y + t * d + c, y);
        }
    }
    if (!a.part) return;
    float* part = a.part + (long long)blockIdx.x * 2 * d;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = 8 * (tt + i * TPR);
                if (c < d) store8(part + q * d + c, acc[q][i]);
            }
    } else {
        // the CTA's rows one after another: the order of the sum is fixed
        for (int o = 0; o < ROWS; ++o) {
            if (row0 == o)
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int c = 8 * (tt + i * TPR);
                        if (c >= d) continue;
#pragma unroll
                        for (int j = 0; j < 8; ++j) s_sum[q * d + c + j] = (o ? s_sum[q * d + c + j] : 0.f) + acc[q][i][j];
                    }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * d; c += THREADS) part[c] = s_sum[c];
    }
}

// Column sums of the CTAs' partial rows, in a fixed order, and the factors of the two gradients that share one.  grid.y: which
// of the two sums.
__global__ void __launch_bounds__(256) norm_join_sums_kernel(const __grid_constant__ JoinArgs a, int n_part, float* d_w_post,
                                                             float* d_gate, float* d_w_pre) {
    __shared__ float s[8][32];
    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, d = a.d;
    float sum = 0.f;
    if (c < d)
#pragma unroll 8
        for (int p = warp; p < n_part; p += 8) sum += a.part[((long long)p * 2 + blockIdx.y) * d + c];
    s[warp][lane] = sum;
    __syncthreads();
    if (warp || c >= d) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) sum += s[w][lane];
    if (blockIdx.y) {
        if (d_w_pre) d_w_pre[c] = sum;
        return;
    }
    auto weight = [&](const void* w) { return !w ? 1.f : a.w_f32 ? ((const float*)w)[c] : __bfloat162float(((const __nv_bfloat16*)w)[c]); };
    if (d_w_post) d_w_post[c] = sum * weight(a.gate_kind == DYNAMO_GATE_CHANNEL ? a.gate : nullptr);
    if (d_gate) d_gate[c] = sum * weight(a.post ? a.w_post : nullptr);
}

constexpr int JOIN_MAX_D = 16384;

// Threads a row and runs a thread by the width: a warp where its four runs cover the row (no barrier), else as many threads as
// there are runs, up to the 1024 of a CTA.
template <int TPR_, int V_, bool KEEP_>
struct Layout {
    static constexpr int TPR = TPR_, V = V_;
    static constexpr bool KEEP = KEEP_;
};
template <bool GRAD, typename F>
static cudaError_t by_width(int d, F f) {
    if (d <= 256) return f(Layout<32, 1, true>{});
    if (d <= 512) return f(Layout<32, 2, !GRAD>{});
    if (d <= 1024) return f(Layout<128, 1, true>{});
    if (d <= 2048) return f(Layout<256, 1, true>{});
    if (d <= 4096) return f(Layout<512, 1, true>{});
    if (d <= 8192) return f(Layout<1024, 1, !GRAD>{});
    return f(Layout<1024, 2, false>{});
}
template <typename F>
static cudaError_t by_types(int a, int b, F f) {
    if (a == DYNAMO_BF16) return b == DYNAMO_BF16 ? f((__nv_bfloat16*)nullptr, (__nv_bfloat16*)nullptr) : f((__nv_bfloat16*)nullptr, (float*)nullptr);
    return b == DYNAMO_BF16 ? f((float*)nullptr, (__nv_bfloat16*)nullptr) : f((float*)nullptr, (float*)nullptr);
}

// CTAs of a launch: what the SMs hold at once, and no more than there are rows.
template <typename L>
static int ctas_for(int T, int regs, int n_sms) {
    constexpr int THREADS = threads_of(L::TPR), ROWS = THREADS / L::TPR;
    return (int)std::max(1ll, std::min({((long long)T + ROWS - 1) / ROWS, (long long)n_sms * ctas_of(THREADS, regs)}));
}
static int grad_ctas(int T, int d, int n_sms) {
    int n = 0;
    by_width<true>(d, [&](auto l) {
        n = ctas_for<decltype(l)>(T, 128, n_sms);
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

extern "C" {

dynamo_status dynamo_norm_join_forward(const dynamo_join_desc* desc, const void* r, const void* y, const void* w_post,
                                       const void* gate, const void* w_pre, int32_t T, void* r_out, void* n_out, float* stats,
                                       void* stream) {
    if (const dynamo_status s = check_join(desc, T); s != DYNAMO_OK) return s;
    if (T == 0) return DYNAMO_OK;
    if (!y && !desc->pre_norm) return DYNAMO_ERR_ARG;   // nothing to do
    if (!r || (y && !r_out) || (desc->pre_norm && !n_out) || (y && desc->gate_kind != DYNAMO_GATE_NONE && !gate)) return DYNAMO_ERR_NULL;
    if (!aligned16(r, y, r_out, n_out) || !aligned16(w_post, w_pre) ||
        (y && desc->gate_kind == DYNAMO_GATE_CHANNEL && !aligned16(gate)) || ((uintptr_t)stats & 7))
        return DYNAMO_ERR_ALIGN;
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
            return launch_pdl(norm_join_kernel<TY, TR, L::TPR, L::V, L::KEEP>, dim3((unsigned)ctas_for<L>(T, join_regs(L::TPR), n_sms)),
                              dim3(threads_of(L::TPR)), 0, (cudaStream_t)stream, a);
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
            const size_t smem = L::TPR < 128 ? 2 * desc->d * sizeof(float) : 0;
            return a.n_f32 ? launch_pdl(norm_join_grad_kernel<TY, TR, float, L::TPR, L::V, L::KEEP>, grid, block, smem, st, a)
                           : launch_pdl(norm_join_grad_kernel<TY, TR, __nv_bfloat16, L::TPR, L::V, L::KEEP>, grid, block, smem, st, a);
        });
    });
    if (e != cudaSuccess) return DYNAMO_ERR_CUDA;
    if (columns && launch_pdl(norm_join_sums_kernel, dim3((unsigned)((desc->d + 31) / 32), 2), dim3(256), 0, st, a, ctas,
                              d_w_post, channel ? d_gate : nullptr, d_w_pre) != cudaSuccess)
        return DYNAMO_ERR_CUDA;
    return DYNAMO_OK;
}

}  // extern "C"
