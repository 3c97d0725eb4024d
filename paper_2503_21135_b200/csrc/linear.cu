// Products of few token rows with a matrix of 4-bit codes and group scales (the quantizer is the experts', quant.cuh):
//
//   y[t][n] = sum over groups g of  s[n][g] * sum_{k in g} q[n][k] x[t][k]  +  m[n][g] * sum_{k in g} x[t][k]
//
// The codes are row-major, two a byte (index 2i in the low half of byte i), so a 32-bit word holds eight consecutive ones.
// A code becomes a bf16 operand by a shift, a mask and an OR: on the four highest mantissa bits of 16.0 it reads as
// 16 + q, exactly.  The MMA therefore gives sum((16 + q) x), and 16 s goes off the zero-point:
// y += s * acc + (m - 16 s) * sum(x), with sum(x) from an MMA whose other operand is ones.  Products are exact in fp32 (bf16 by
// bf16); sums, scales and zero-points are in fp32, y is rounded once.  The order in which a warp's 16-wide steps take the
// input indices is free as long as codes and activations agree: a lane takes runs of consecutive ones from both.
#include <algorithm>
#include <type_traits>

#include "../../include/dynamo.h"
#include "common.cuh"
#include "quant.cuh"
#include "vec8.cuh"

namespace dyn {

// One warp a group: extrema, parameters and codes, in double as at the experts' packing.
__global__ void __launch_bounds__(256) linear_quantize_kernel(const __nv_bfloat16* __restrict__ w, long long n_groups, int G,
                                                              uint8_t* __restrict__ codes, __half2* __restrict__ params) {
    pdl_prologue();
    const int lane = threadIdx.x & 31;
    const long long g = ((long long)blockIdx.x * 256 + threadIdx.x) >> 5;
    if (g >= n_groups) return;
    const int per = G / 32;   // 2 or 4 consecutive values a lane
    const __nv_bfloat16* p = w + g * G + lane * per;
    double v[4], lo, hi;
    lo = hi = bf16_to_double(p[0]);
    for (int i = 0; i < per; ++i) {
        v[i] = bf16_to_double(p[i]);
        lo = v[i] < lo ? v[i] : lo;
        hi = v[i] > hi ? v[i] : hi;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const double l = __shfl_xor_sync(0xffffffffu, lo, o), h = __shfl_xor_sync(0xffffffffu, hi, o);
        lo = l < lo ? l : lo;
        hi = h > hi ? h : hi;
    }
    __half s_h, m_h;
    double s, m;
    group_params(lo, hi, 4, s_h, m_h, s, m);
    for (int i = 0; i < per; i += 2)
        codes[(g * G + lane * per + i) / 2] = (uint8_t)(quantize_code(v[i], s, m, 4) | quantize_code(v[i + 1], s, m, 4) << 4);
    if (lane == 0) params[g] = __halves2half2(s_h, m_h);
}

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Codes i and i + 4 of a word as the bf16 pair 16 + q.
template <int I>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
    const uint32_t s = I == 0 ? w << 3 : w >> (4 * I - 3);
    return (s & 0x00780078u) | 0x41804180u;
}

struct LinearArgs {
    const __nv_bfloat16* x;   // [T, K]
    const uint8_t* codes;     // [N, K / 2]
    const uint32_t* params;   // [N, K / G] half2 {scale, zero}
    void* y;                  // [T, N]
    int T, K, N;
};

constexpr int LIN_WARPS = 8;
constexpr int LIN_UNIT = 128;   // input indices a warp takes at a time

// CTA: 16 R rows of the matrix, 8 NT tokens; its warps take units of 128 input indices in turn and add up their sums at the end.
template <int NT, int R, int G, typename TO>
__global__ void __launch_bounds__(32 * LIN_WARPS) linear_kernel(LinearArgs a) {
    __shared__ float part[LIN_WARPS][R][NT][4][32];
    constexpr int GPU_ = LIN_UNIT / G;        // groups of a unit
    constexpr int WPG = 4 / GPU_;             // words of a lane and row in a group
    pdl_prologue();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tid4 = lane & 3;
    const int n0 = blockIdx.x * 16 * R, t0 = blockIdx.y * 8 * NT;
    const int ng = a.K / G;
    float acc[R][NT][4];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[r][n][i] = 0.f;
    for (int u = warp; u * LIN_UNIT < a.K; u += LIN_WARPS) {
        // codes of rows gid and gid + 8 of every atom: word j of group h covers indices 128 u + G h + (G / 4) tid4 + 8 j ..
        uint32_t cw[R][2][4];
        uint32_t pr[R][2][GPU_];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = n0 + 16 * r + gid + 8 * h;
#pragma unroll
                for (int g = 0; g < GPU_; ++g) {
                    const int k = u * LIN_UNIT + g * G;
                    const bool in = row < a.N && k < a.K;
                    const uint8_t* p = a.codes + (long long)row * (a.K / 2) + k / 2 + tid4 * (4 * WPG);
                    if constexpr (GPU_ == 1) {
                        const uint4 v = in ? ld_stream(p) : make_uint4(0u, 0u, 0u, 0u);
                        cw[r][h][0] = v.x, cw[r][h][1] = v.y, cw[r][h][2] = v.z, cw[r][h][3] = v.w;
                    } else {
                        const uint2 v = in ? __ldg(reinterpret_cast<const uint2*>(p)) : make_uint2(0u, 0u);
                        cw[r][h][2 * g] = v.x, cw[r][h][2 * g + 1] = v.y;
                    }
                    pr[r][h][g] = in ? __ldg(a.params + (long long)row * ng + k / G) : 0u;
                }
            }
#pragma unroll
        for (int g = 0; g < GPU_; ++g) {
            float c[R][NT][4], sx[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sx[n][i] = 0.f;
#pragma unroll
                    for (int r = 0; r < R; ++r) c[r][n][i] = 0.f;
                }
#pragma unroll
            for (int j = 0; j < WPG; ++j) {
                const int k = u * LIN_UNIT + g * G + tid4 * (8 * WPG) + 8 * j;
                uint32_t b[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int t = t0 + 8 * n + gid;
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (t < a.T && k < a.K) v = __ldg(reinterpret_cast<const uint4*>(a.x + (long long)t * a.K + k));
                    b[n][0] = __byte_perm(v.x, v.z, 0x5410);   // indices 0, 4
                    b[n][1] = __byte_perm(v.x, v.z, 0x7632);   // 1, 5
                    b[n][2] = __byte_perm(v.y, v.w, 0x5410);   // 2, 6
                    b[n][3] = __byte_perm(v.y, v.w, 0x7632);   // 3, 7
                    mma_bf16(sx[n], 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, b[n][0], b[n][1]);
                    mma_bf16(sx[n], 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, b[n][2], b[n][3]);
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint32_t w0 = cw[r][0][g * WPG + j], w1 = cw[r][1][g * WPG + j];
                    const uint32_t p00 = code_pair<0>(w0), p01 = code_pair<0>(w1), p10 = code_pair<1>(w0), p11 = code_pair<1>(w1);
                    const uint32_t p20 = code_pair<2>(w0), p21 = code_pair<2>(w1), p30 = code_pair<3>(w0), p31 = code_pair<3>(w1);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma_bf16(c[r][n], p00, p01, p10, p11, b[n][0], b[n][1]);
                        mma_bf16(c[r][n], p20, p21, p30, p31, b[n][2], b[n][3]);
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const __half2 pv = *reinterpret_cast<const __half2*>(&pr[r][h][g]);
                    const float s = __low2float(pv), m = fmaf(-16.f, s, __high2float(pv));
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        acc[r][n][2 * h] = fmaf(s, c[r][n][2 * h], fmaf(m, sx[n][0], acc[r][n][2 * h]));
                        acc[r][n][2 * h + 1] = fmaf(s, c[r][n][2 * h + 1], fmaf(m, sx[n][1], acc[r][n][2 * h + 1]));
                    }
                }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[warp][r][n][i][lane] = acc[r][n][i];
    __syncthreads();
    for (int o = threadIdx.x; o < R * NT * 128; o += 32 * LIN_WARPS) {
        // rows beside one another in a warp's stores: o = token (8 NT) * 16 R + row
        const int row = o % (16 * R), t = o / (16 * R);
        const int r = row >> 4, g = row & 7, h = (row >> 3) & 1, n = t >> 3, col = t & 7;
        const int l = g * 4 + (col >> 1), i = 2 * h + (col & 1);
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < LIN_WARPS; ++w) s += part[w][r][n][i][l];
        if (n0 + row < a.N && t0 + t < a.T) {
            const long long at = (long long)(t0 + t) * a.N + n0 + row;
            if constexpr (sizeof(TO) == 4) ((float*)a.y)[at] = s;
            else ((__nv_bfloat16*)a.y)[at] = __float2bfloat16_rn(s);
        }
    }
}

template <int NT, int R, int G>
static cudaError_t linear_go(const LinearArgs& a, int y_f32, cudaStream_t st) {
    const dim3 grid((unsigned)((a.N + 16 * R - 1) / (16 * R)), (unsigned)((a.T + 8 * NT - 1) / (8 * NT)));
    return y_f32 ? launch_pdl(linear_kernel<NT, R, G, float>, grid, dim3(32 * LIN_WARPS), 0, st, a)
                 : launch_pdl(linear_kernel<NT, R, G, __nv_bfloat16>, grid, dim3(32 * LIN_WARPS), 0, st, a);
}
template <int G>
static cudaError_t linear_by_tokens(const LinearArgs& a, int y_f32, cudaStream_t st) {
    if (a.T <= 8) return linear_go<1, 2, G>(a, y_f32, st);
    if (a.T <= 16) return linear_go<2, 2, G>(a, y_f32, st);
    return linear_go<4, 1, G>(a, y_f32, st);
}

}  // namespace dyn

using namespace dyn;

namespace {

dynamo_status check_linear(int32_t rows, int32_t cols, int32_t group_size) {
    if (group_size != 64 && group_size != 128) return DYNAMO_ERR_SHAPE;
    if (rows < 1 || cols < group_size || cols % group_size) return DYNAMO_ERR_SHAPE;
    return DYNAMO_OK;
}

}  // namespace

extern "C" {

dynamo_status dynamo_linear_quantize(const void* w, int32_t rows, int32_t cols, int32_t group_size, void* codes, void* params,
                                     void* stream) {
    if (const dynamo_status s = check_linear(rows, cols, group_size); s != DYNAMO_OK) return s;
    if (!w || !codes || !params) return DYNAMO_ERR_NULL;
    if (!aligned16(w, codes, params)) return DYNAMO_ERR_ALIGN;
    const long long n = (long long)rows * (cols / group_size);
    if ((n + 7) / 8 > 0x7fffffffll) return DYNAMO_ERR_SHAPE;
    return launch_pdl(linear_quantize_kernel, dim3((unsigned)((n + 7) / 8)), dim3(256), 0, (cudaStream_t)stream,
                      (const __nv_bfloat16*)w, n, group_size, (uint8_t*)codes, (__half2*)params) == cudaSuccess
               ? DYNAMO_OK
               : DYNAMO_ERR_CUDA;
}

dynamo_status dynamo_linear_forward(const void* x, int32_t T, int32_t rows, int32_t cols, int32_t group_size, const void* codes,
                                    const void* params, void* y, int32_t y_dtype, void* stream) {
    if (const dynamo_status s = check_linear(rows, cols, group_size); s != DYNAMO_OK) return s;
    if (y_dtype != DYNAMO_BF16 && y_dtype != DYNAMO_F32) return DYNAMO_ERR_SHAPE;
    if (T < 0 || T > DYNAMO_LINEAR_MAX_TOKENS) return DYNAMO_ERR_TOKENS;
    if (T == 0) return DYNAMO_OK;
    if (!x || !codes || !params || !y) return DYNAMO_ERR_NULL;
    if (!aligned16(x, codes, params, y)) return DYNAMO_ERR_ALIGN;
    LinearArgs a = {(const __nv_bfloat16*)x, (const uint8_t*)codes, (const uint32_t*)params, y, T, cols, rows};
    const cudaError_t e = group_size == 64 ? linear_by_tokens<64>(a, y_dtype == DYNAMO_F32, (cudaStream_t)stream)
                                           : linear_by_tokens<128>(a, y_dtype == DYNAMO_F32, (cudaStream_t)stream);
    return e == cudaSuccess ? DYNAMO_OK : DYNAMO_ERR_CUDA;
}

}  // extern "C"
