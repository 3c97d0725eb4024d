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
    float* part;          // [CTA][3][d] sums of a CTA's rows: d_w_post, d_w_pre, d_gate of the channels
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

// Sums of N values over the TPR threads of a row; every thread gets them.  `scratch`: [TPR / 32][N], two of them in turn.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* scratch) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 16; o; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if constexpr (TPR > 32) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) scratch[warp * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = lane < TPR / 32 ? scratch[lane * N + i] : 0.f;
#pragma unroll
            for (int o = TPR / 64; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            v[i] = __shfl_sync(0xffffffffu, s, 0);
        }
    }
}

// TPR threads a row, V runs of eight columns a thread (run i of thread t: columns 8 (t + i TPR)).
template <typename TY, typename TR, int TPR, int V>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) norm_join_kernel(JoinArgs a) {
    constexpr int THREADS = TPR < 128 ? 128 : TPR, ROWS = THREADS / TPR, W = TPR / 32;
    __shared__ float scratch[2][W];
    pdl_prologue();
    const int tt = threadIdx.x % TPR, d = a.d;
    const float inv_d = 1.f / (float)d;
    for (long long t = (long long)blockIdx.x * ROWS + threadIdx.x / TPR; t < a.T; t += (long long)gridDim.x * ROWS) {
        Raw8<TY> yr[V];
        Raw8<TR> rr[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            yr[i] = a.y && c < d ? load8((const TY*)a.y + t * d + c) : zero8<TY>();
            rr[i] = c < d ? load8((const TR*)a.r + t * d + c) : zero8<TR>();
        }
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
        float g = a.block_scale * s_y;
        if (a.gate_kind == DYNAMO_GATE_TOKEN) g *= ((const float*)a.gate)[t];
        float x[V][8];
        float sum[1] = {0.f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            float r[8];
            unpack8(rr[i], r);
            if (a.y && c < d) {
                float y[8], w[8];
                unpack8(yr[i], y);
                if (a.post) {
                    weights8(a.w_post, a.w_f32, c, w);
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] *= w[j];
                }
                if (a.gate_kind == DYNAMO_GATE_CHANNEL) {
                    weights8(a.gate, a.w_f32, c, w);
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] *= w[j];
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = fmaf(g, y[j], a.res_scale * r[j]);
                if (a.r_out) store8((TR*)a.r_out + t * d + c, x[i]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = r[j];
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
                float w[8];
                weights8(a.w_pre, a.w_f32, c, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] *= x[i][j] * s_r;
                if (a.n_f32) store8((float*)a.n_out + t * d + c, w);
                else store8((__nv_bfloat16*)a.n_out + t * d + c, w);
            }
        }
        if (a.stats && tt == 0) *reinterpret_cast<float2*>(a.stats + 2 * t) = make_float2(s_y, s_r);
        // One reduction a row alone would use the same scratch for the next row's: its readers have to be through.
        if constexpr (TPR > 32)
            if (!(a.post && a.pre)) __syncthreads();
    }
}

template <typename TY, typename TR, int TPR, int V>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) norm_join_grad_kernel(JoinArgs a) {
    constexpr int THREADS = TPR < 128 ? 128 : TPR, ROWS = THREADS / TPR, W = TPR / 32;
    __shared__ float scratch[2][W * 3];
    extern __shared__ float s_sum[];   // several rows a CTA: [3][d] for the CTA's column sums
    pdl_prologue();
    const int tt = threadIdx.x % TPR, d = a.d, row0 = threadIdx.x / TPR;
    const float inv_d = 1.f / (float)d;
    float acc[3][V][8];
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[q][i][j] = 0.f;
    int turn = 0;
    for (long long t = (long long)blockIdx.x * ROWS + row0; t < a.T; t += (long long)gridDim.x * ROWS, turn ^= 1) {
        Raw8<TY> yr[V];
        Raw8<TR> rr[V], dr[V];
        float dn[V][8];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            yr[i] = a.y && c < d ? load8((const TY*)a.y + t * d + c) : zero8<TY>();
            rr[i] = c < d ? load8((const TR*)a.r + t * d + c) : zero8<TR>();
            dr[i] = a.d_r_out && c < d ? load8((const TR*)a.d_r_out + t * d + c) : zero8<TR>();
            if (a.d_n && c < d) {
                if (a.n_f32) unpack8(load8((const float*)a.d_n + t * d + c), dn[i]);
                else unpack8(load8((const __nv_bfloat16*)a.d_n + t * d + c), dn[i]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) dn[i][j] = 0.f;
            }
        }
        const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * t);
        const float s_y = a.post ? st.x : 1.f, s_r = st.y;
        const float gt = a.gate_kind == DYNAMO_GATE_TOKEN ? ((const float*)a.gate)[t] : 1.f;
        // sums over the row: A = u r', B = k z (dr' + s_r u), C = k z r' with k the gate of the channels (the token's and
        // block_scale are put in afterwards)
        float sum[3] = {0.f, 0.f, 0.f};
        const float gz = a.block_scale * gt;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = 8 * (tt + i * TPR);
            if (c >= d) continue;
            float y[8], r[8], g[8], wp[8], wq[8], k[8];
            unpack8(yr[i], y);
            unpack8(rr[i], r);
            unpack8(dr[i], g);
            weights8(a.post ? a.w_post : nullptr, a.w_f32, c, wp);
            weights8(a.w_pre, a.w_f32, c, wq);
            weights8(a.gate_kind == DYNAMO_GATE_CHANNEL ? a.gate : nullptr, a.w_f32, c, k);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float kz = k[j] * wp[j] * y[j] * s_y;
                const float x = a.y ? fmaf(gz, kz, a.res_scale * r[j]) : r[j];
                const float u = wq[j] * dn[i][j];
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
            float y[8], r[8], g[8], wp[8], wq[8], k[8];
            unpack8(yr[i], y);
            unpack8(rr[i], r);
            unpack8(dr[i], g);
            weights8(a.post ? a.w_post : nullptr, a.w_f32, c, wp);
            weights8(a.w_pre, a.w_f32, c, wq);
            weights8(a.gate_kind == DYNAMO_GATE_CHANNEL ? a.gate : nullptr, a.w_f32, c, k);
            float dy[8], drv[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float yn = y[j] * s_y, z = wp[j] * yn;
                const float x = a.y ? fmaf(gz, k[j] * z, a.res_scale * r[j]) : r[j];
                const float G = fmaf(-ca, x, fmaf(s_r, wq[j] * dn[i][j], g[j]));
                const float dz = gz * k[j] * G;
                drv[j] = a.y ? a.res_scale * G : G;
                dy[j] = s_y * fmaf(-cv, yn, dz * wp[j]);
                acc[0][i][j] = fmaf(dz, yn, acc[0][i][j]);
                acc[1][i][j] = fmaf(dn[i][j], x * s_r, acc[1][i][j]);
                acc[2][i][j] = fmaf(gz * z, G, acc[2][i][j]);
            }
            if (a.d_r) store8((TR*)a.d_r + t * d + c, drv);
            if (a.d_y) store8((TY*)a.d_y + t * d + c, dy);
        }
    }
    if (!a.part) return;
    float* part = a.part + (long long)blockIdx.x * 3 * d;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = 8 * (tt + i * TPR);
                if (c < d) store8(part + q * d + c, acc[q][i]);
            }
    } else {
        // the CTA's rows one after another: the order of the sum is fixed
        for (int w = 0; w < ROWS; ++w) {
            if (row0 == w)
#pragma unroll
                for (int q = 0; q < 3; ++q)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int c = 8 * (tt + i * TPR);
                        if (c >= d) continue;
#pragma unroll
                        for (int j = 0; j < 8; ++j) s_sum[q * d + c + j] = (w ? s_sum[q * d + c + j] : 0.f) + acc[q][i][j];
                    }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 3 * d; c += THREADS) part[c] = s_sum[c];
    }
}

// Column sums of the CTAs' partial rows, in the order of the CTAs.  grid.y: which of the three vectors.
__global__ void __launch_bounds__(256) norm_join_sums_kernel(const float* __restrict__ part, int n_part, int d, float* d_w_post,
                                                             float* d_w_pre, float* d_gate) {
    __shared__ float s[8][32];
    pdl_prologue();
    float* out = blockIdx.y == 0 ? d_w_post : (blockIdx.y == 1 ? d_w_pre : d_gate);
    if (!out) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float sum = 0.f;
    if (c < d)
#pragma unroll 4
        for (int p = warp; p < n_part; p += 8) sum += part[((long long)p * 3 + blockIdx.y) * d + c];
    s[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < d) {
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += s[w][lane];
        out[c] = sum;
    }
}

constexpr int JOIN_MAX_D = 16384;
constexpr int JOIN_MAX_CTAS = 1024;   // of a backward launch

template <typename F>
static cudaError_t by_width(int d, F f) {
    using std::integral_constant;
    if (d <= 256) return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    if (d <= 512) return f(integral_constant<int, 32>{}, integral_constant<int, 2>{});
    if (d <= 1024) return f(integral_constant<int, 128>{}, integral_constant<int, 1>{});
    if (d <= 2048) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    if (d <= 4096) return f(integral_constant<int, 512>{}, integral_constant<int, 1>{});
    if (d <= 8192) return f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
    return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}
template <typename F>
static cudaError_t by_types(int a, int b, F f) {
    if (a == DYNAMO_BF16) return b == DYNAMO_BF16 ? f((__nv_bfloat16*)nullptr, (__nv_bfloat16*)nullptr) : f((__nv_bfloat16*)nullptr, (float*)nullptr);
    return b == DYNAMO_BF16 ? f((float*)nullptr, (__nv_bfloat16*)nullptr) : f((float*)nullptr, (float*)nullptr);
}

// CTAs of a backward launch: what the SMs hold at once, and no more than there are rows.
static int grad_ctas(int T, int d, int n_sms) {
    const int tpr = d <= 512 ? 32 : d <= 1024 ? 128 : d <= 2048 ? 256 : d <= 4096 ? 512 : 1024;
    const int rows = tpr < 128 ? 128 / tpr : 1, threads = tpr * rows;
    const int per_sm = std::max(1, 512 / threads);
    return std::max(1, std::min({(T + rows - 1) / rows, n_sms * per_sm, JOIN_MAX_CTAS}));
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
    JoinArgs a = join_args(desc, T, r, y, w_post, gate, w_pre);
    a.r_out = y ? r_out : nullptr;
    a.n_out = n_out;
    a.stats = stats;
    const cudaError_t e = by_types(desc->y_dtype, desc->r_dtype, [&](auto* ty, auto* tr) {
        using TY = std::remove_pointer_t<decltype(ty)>;
        using TR = std::remove_pointer_t<decltype(tr)>;
        return by_width(desc->d, [&](auto tprc, auto vc) {
            constexpr int TPR = decltype(tprc)::value, V = decltype(vc)::value;
            constexpr int THREADS = TPR < 128 ? 128 : TPR, ROWS = THREADS / TPR;
            const long long ctas = ((long long)T + ROWS - 1) / ROWS;
            return launch_pdl(norm_join_kernel<TY, TR, TPR, V>, dim3((unsigned)ctas), dim3(THREADS), 0, (cudaStream_t)stream, a);
        });
    });
    return e == cudaSuccess ? DYNAMO_OK : DYNAMO_ERR_CUDA;
}

dynamo_status dynamo_norm_join_workspace_bytes(const dynamo_join_desc* desc, int32_t T, size_t* bytes) {
    if (const dynamo_status s = check_join(desc, T); s != DYNAMO_OK) return s;
    if (!bytes) return DYNAMO_ERR_NULL;
    *bytes = (size_t)grad_ctas(T, desc->d, 256) * 3 * desc->d * 4;   // up to 256 SMs are reckoned with
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
        return by_width(desc->d, [&](auto tprc, auto vc) {
            constexpr int TPR = decltype(tprc)::value, V = decltype(vc)::value;
            constexpr int THREADS = TPR < 128 ? 128 : TPR;
            return launch_pdl(norm_join_grad_kernel<TY, TR, TPR, V>, dim3((unsigned)ctas), dim3(THREADS),
                              TPR < 128 ? 3 * desc->d * sizeof(float) : 0, st, a);
        });
    });
    if (e != cudaSuccess) return DYNAMO_ERR_CUDA;
    if (columns && launch_pdl(norm_join_sums_kernel, dim3((unsigned)((desc->d + 31) / 32), 3), dim3(256), 0, st,
                              (const float*)workspace, ctas, desc->d, d_w_post, d_w_pre, channel ? d_gate : nullptr) != cudaSuccess)
        return DYNAMO_ERR_CUDA;
    return DYNAMO_OK;
}

}  // extern "C"
