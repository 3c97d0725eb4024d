// Tokens sorted by expert and back: dispatch (stable counting sort of the (token, slot) pairs and copies of the tokens'
// rows in its order), combine (weighted sum of a token's rows) and combine's gradient; dispatch's gradient is a combine
// without weights.  All four walk the tokens: a token's row is read once and its k places follow from pos, so that
// nothing is added atomically and the order of every sum is the order of the token's choices.
//
// Bytes bound them all: rows in and out once each.
#include <algorithm>
#include <type_traits>

#include "../../include/dynamo.h"
#include "common.cuh"
#include "vec8.cuh"

namespace dyn {

constexpr int DISPATCH_EXPERTS = 256;
constexpr int DISPATCH_THREADS = 1024;
constexpr int DISPATCH_WARPS = DISPATCH_THREADS / 32;
constexpr int DISPATCH_CHUNK = 2048;      // pairs that a CTA ranks at a time

struct DispatchArgs {
    const int32_t* idx;    // [T * k]
    int T, k, E, seg;      // seg: tokens per CTA
    int32_t* offsets;      // [E + 1]
    int32_t* perm;         // [T * k]
    int32_t* pos;          // [T * k]
    const uint8_t* x;      // rows of row_bytes, or NULL: sort alone
    uint8_t* rows;
    long long row_bytes;
    int32_t* hist;         // [CTA][E_pad] pairs of each CTA's tokens by expert, or NULL: every CTA counts the whole array
    int E_pad;             // E rounded up to a power of two
};

// Counts of the pairs [lo, hi) by expert into shared counters, those in front of `mid` into `before`, the others into `behind`
// (integer additions: any order gives the same counts).  Sixteen bytes of indices a load where the array's address allows.
__device__ __forceinline__ void count_pairs(const int32_t* __restrict__ idx, long long lo, long long mid, long long hi, int E, int* before,
                                            int* behind) {
    auto count = [&](int v, long long i) {
        if ((uint32_t)v < (uint32_t)E) atomicAdd((i < mid ? before : behind) + v, 1);
    };
    long long done = lo;
    if ((((uintptr_t)idx + 4 * lo) & 15) == 0) {
        const long long n4 = (hi - lo) / 4;
#pragma unroll 4
        for (long long q = threadIdx.x; q < n4; q += DISPATCH_THREADS) {
            const int4 v = *reinterpret_cast<const int4*>(idx + lo + 4 * q);
            count(v.x, lo + 4 * q);
            count(v.y, lo + 4 * q + 1);
            count(v.z, lo + 4 * q + 2);
            count(v.w, lo + 4 * q + 3);
        }
        done = lo + 4 * n4;
    }
    for (long long i = done + threadIdx.x; i < hi; i += DISPATCH_THREADS) count(idx[i], i);
}

__global__ void __launch_bounds__(DISPATCH_THREADS) dispatch_count_kernel(const __grid_constant__ DispatchArgs a) {
    __shared__ int s_count[DISPATCH_EXPERTS];
    pdl_prologue();
    if (threadIdx.x < DISPATCH_EXPERTS) s_count[threadIdx.x] = 0;
    __syncthreads();
    const long long lo = (long long)blockIdx.x * a.seg * a.k, hi = min((long long)a.T * a.k, lo + (long long)a.seg * a.k);
    count_pairs(a.idx, lo, lo, hi, a.E, s_count, s_count);
    __syncthreads();
    if (threadIdx.x < a.E_pad) a.hist[blockIdx.x * a.E_pad + threadIdx.x] = s_count[threadIdx.x];
}

// One CTA per run of `seg` tokens, one an SM.  First the experts' totals and the pairs of each expert in front of the run, then
// the run's pairs are ranked (a warp per contiguous piece, lanes of the same expert found by match.any: the order is that of
// the pairs) and its tokens' rows copied, one read and k writes each, 16 bytes a thread and four of them at a time.
// Every CTA counts the whole array, so one of 1024 threads an SM: 4096 tokens of 8 KB, top-2 of 8 experts, 21.8 us (4.6 TB/s;
// some 4 us of it in front of the first copy), 24.2 with four CTAs of 256.  Asking for the rows ahead of the count (into the
// L2, 64 to 256 KB a CTA) made it 22.5, eight pieces a thread at a time 22.2.
__global__ void __launch_bounds__(DISPATCH_THREADS, 1) dispatch_kernel(const __grid_constant__ DispatchArgs a) {
    __shared__ int s_total[DISPATCH_EXPERTS], s_next[DISPATCH_EXPERTS];
    __shared__ int s_hist[DISPATCH_WARPS][DISPATCH_EXPERTS];
    __shared__ int s_pos[DISPATCH_CHUNK];
    __shared__ int s_warp[DISPATCH_EXPERTS / 32];
    pdl_prologue();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int k = a.k, E = a.E;
    const long long n_pairs = (long long)a.T * k;
    const int t0 = blockIdx.x * a.seg, t1 = t0 + min(a.seg, a.T - t0);   // (T may be 2^31 - 1)
    const long long lo = (long long)t0 * k;
    if (tid < DISPATCH_EXPERTS) {
        s_total[tid] = 0;
        s_next[tid] = 0;
    }
    __syncthreads();
    if (a.hist) {
        // a thread adds up every (threads / E_pad)-th CTA's count of one expert
        const int e = tid & (a.E_pad - 1);
        int before = 0, behind = 0;
#pragma unroll 8
        for (int r = tid / a.E_pad; r < (int)gridDim.x; r += DISPATCH_THREADS / a.E_pad) {
            const int c = a.hist[r * a.E_pad + e];
            (r < (int)blockIdx.x ? before : behind) += c;
        }
        if (before) atomicAdd(s_next + e, before);
        if (behind) atomicAdd(s_total + e, behind);
    } else {
        count_pairs(a.idx, 0, lo, n_pairs, E, s_next, s_total);
    }
    __syncthreads();
    // exclusive scan of the totals, an expert per thread
    int total = 0, sum = 0;
    if (tid < DISPATCH_EXPERTS) {
        total = sum = s_total[tid] + s_next[tid];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += u;
        }
        if (lane == 31) s_warp[warp] = sum;
    }
    __syncthreads();
    if (tid < DISPATCH_EXPERTS) {
        int first = sum - total;                 // first row of expert tid
        for (int w = 0; w < warp; ++w) first += s_warp[w];
        s_next[tid] += first;                    // its first row of this run
        if (blockIdx.x == 0) {
            if (tid < E) a.offsets[tid] = first;
            if (tid == E - 1) a.offsets[E] = first + total;
        }
    }
    const unsigned lt = (1u << lane) - 1;
    const int chunk_tokens = DISPATCH_CHUNK / k;
    for (int c0 = t0, c1; c0 < t1; c0 = c1) {
        c1 = c0 + min(chunk_tokens, t1 - c0);
        const int n = (c1 - c0) * k;
        const long long base = (long long)c0 * k;
        const int piece = ((n + 31) / 32 + DISPATCH_WARPS - 1) / DISPATCH_WARPS * 32;   // whole batches of 32 a warp
        const int pieces = (n + piece - 1) / piece;
        const int p0 = min(n, warp * piece), p1 = min(n, p0 + piece);
        for (int i = tid; i < pieces * DISPATCH_EXPERTS; i += DISPATCH_THREADS) (&s_hist[0][0])[i] = 0;
        __syncthreads();
        for (int p = p0 + lane; p - lane < p1; p += 32) {
            const uint32_t e = p < p1 ? (uint32_t)a.idx[base + p] : 0xffffffffu;
            if (e < (uint32_t)E) atomicAdd(&s_hist[warp][e], 1);
        }
        __syncthreads();
        if (tid < E) {
            int next = s_next[tid];
            for (int i = 0; i < pieces; ++i) {
                const int c = s_hist[i][tid];
                s_hist[i][tid] = next;
                next += c;
            }
            s_next[tid] = next;
        }
        __syncthreads();
        for (int p = p0 + lane; p - lane < p1; p += 32) {
            const uint32_t e0 = p < p1 ? (uint32_t)a.idx[base + p] : 0xffffffffu;
            const bool valid = e0 < (uint32_t)E;
            const int e = valid ? (int)e0 : -1;
            const unsigned same = __match_any_sync(0xffffffffu, e);
            const int start = valid ? s_hist[warp][e] : 0;
            __syncwarp();
            if (valid && (same & lt) == 0) s_hist[warp][e] = start + __popc(same);
            __syncwarp();
            if (p < p1) {
                const int at = valid ? start + __popc(same & lt) : -1;
                s_pos[p] = at;
                a.pos[base + p] = at;
                if (valid) a.perm[at] = (int32_t)(base + p);
            }
        }
        __syncthreads();
        if (a.x) {
            // thread's 16-byte piece v of token t, a CTA's width further each time
            const int n_vec = (int)(a.row_bytes >> 4), items = (c1 - c0) * n_vec;
            const int dt = DISPATCH_THREADS / n_vec, dv = DISPATCH_THREADS - dt * n_vec;
            const uint4* src = reinterpret_cast<const uint4*>(a.x + (long long)c0 * a.row_bytes);
            int t = tid / n_vec, v = tid - t * n_vec;
            for (int item = tid; item < items; item += 4 * DISPATCH_THREADS) {
                uint4 buf[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (item + u * DISPATCH_THREADS < items) buf[u] = ld_stream(src + item + u * DISPATCH_THREADS);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (item + u * DISPATCH_THREADS < items)
                        for (int j = 0; j < k; ++j) {
                            const int r = s_pos[t * k + j];
                            if (r >= 0) reinterpret_cast<uint4*>(a.rows + (long long)r * a.row_bytes)[v] = buf[u];
                        }
                    t += dt;
                    v += dv;
                    if (v >= n_vec) {
                        v -= n_vec;
                        ++t;
                    }
                }
            }
        }
        __syncthreads();
    }
}

// The row of a pair, -1 for a dropped one; nothing outside the array is touched whatever pos holds.
__device__ __forceinline__ int place_of(int p, int n_pairs) { return (uint32_t)p < (uint32_t)n_pairs ? p : -1; }

// y[t] = sum_j w[t,j] rows[pos[t,j]] (w NULL: ones).  A thread per eight columns of a token, its k loads in flight together.
template <typename TI, typename TO, int K>
__global__ void __launch_bounds__(256) combine_rows_kernel(const TI* __restrict__ rows, const int32_t* __restrict__ pos,
                                                           const float* __restrict__ w, int T, int d, TO* __restrict__ y) {
    pdl_prologue();
    const uint32_t n_vec = d / 8;
    const long long item = (long long)blockIdx.x * 256 + threadIdx.x;
    if (item >= (long long)T * n_vec) return;
    const int t = (int)(item / n_vec), c = (int)(item - (long long)t * n_vec) * 8;
    int at[K];
    float wt[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        at[j] = place_of(pos[(long long)t * K + j], T * K);
        wt[j] = w ? w[(long long)t * K + j] : 1.f;
    }
    Raw8<TI> raw[K];
#pragma unroll
    for (int j = 0; j < K; ++j) raw[j] = at[j] >= 0 ? load8(rows + (long long)at[j] * d + c) : zero8<TI>();
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < K; ++j) {
        float v[8];
        unpack8(raw[j], v);
        const float wj = at[j] >= 0 ? wt[j] : 0.f;   // the weight of a dropped pair may be anything
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = fmaf(wj, v[i], acc[i]);
    }
    store8(y + (long long)t * d + c, acc);
}

// d_rows[pos[t,j]] = w[t,j] dy[t], d_w[t,j] = <rows[pos[t,j]], dy[t]>: both from one pass over the row of dy.  `tpt` threads a
// token (a power of two up to 256).
template <typename TR, typename TY, int K>
__global__ void __launch_bounds__(256) combine_grad_kernel(const TY* __restrict__ dy, const TR* __restrict__ rows,
                                                           const int32_t* __restrict__ pos, const float* __restrict__ w,
                                                           int T, int d, int tpt, TR* __restrict__ d_rows, float* __restrict__ d_w) {
    __shared__ float s_part[8][K];
    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int t = (int)((blockIdx.x * 256ll + threadIdx.x) / tpt), tt = threadIdx.x & (tpt - 1);
    float acc[K];
#pragma unroll
    for (int j = 0; j < K; ++j) acc[j] = 0.f;
    if (t < T) {
        int at[K];
        float wt[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            at[j] = place_of(pos[(long long)t * K + j], T * K);
            wt[j] = w ? w[(long long)t * K + j] : 1.f;
        }
        for (uint32_t c = tt * 8; c < (uint32_t)d; c += tpt * 8) {   // (a step past the last of nearly 2^31 columns)
            const Raw8<TY> g = load8(dy + (long long)t * d + c);
            Raw8<TR> raw[K];
#pragma unroll
            for (int j = 0; j < K; ++j) raw[j] = at[j] >= 0 ? load8(rows + (long long)at[j] * d + c) : zero8<TR>();
            float gv[8];
            unpack8(g, gv);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if (at[j] < 0) continue;
                float v[8], o[8];
                unpack8(raw[j], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    acc[j] = fmaf(v[i], gv[i], acc[j]);
                    o[i] = wt[j] * gv[i];
                }
                store8(d_rows + (long long)at[j] * d + c, o);
            }
        }
    }
    if (!d_w) return;
    for (int o = min(tpt, 32) / 2; o; o >>= 1)
#pragma unroll
        for (int j = 0; j < K; ++j) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], o);
    if (tpt <= 32) {
        if (t < T && tt == 0)
#pragma unroll
            for (int j = 0; j < K; ++j) d_w[(long long)t * K + j] = acc[j];
        return;
    }
    if (lane == 0)
#pragma unroll
        for (int j = 0; j < K; ++j) s_part[warp][j] = acc[j];
    __syncthreads();
    if (t < T && tt < K) {
        const int w0 = threadIdx.x / tpt * (tpt / 32);
        float s = s_part[w0][tt];
        for (int i = 1; i < tpt / 32; ++i) s += s_part[w0 + i][tt];
        d_w[(long long)t * K + tt] = s;
    }
}

template <typename F>
static cudaError_t by_top_k(int k, F f) {
    switch (k) {
        case 1: return f(std::integral_constant<int, 1>{});
        case 2: return f(std::integral_constant<int, 2>{});
        case 3: return f(std::integral_constant<int, 3>{});
        case 4: return f(std::integral_constant<int, 4>{});
        case 5: return f(std::integral_constant<int, 5>{});
        case 6: return f(std::integral_constant<int, 6>{});
        case 7: return f(std::integral_constant<int, 7>{});
        default: return f(std::integral_constant<int, 8>{});
    }
}
// f(TA*, TB*) for the two element types
template <typename F>
static cudaError_t by_types(int a, int b, F f) {
    if (a == DYNAMO_BF16) return b == DYNAMO_BF16 ? f((__nv_bfloat16*)nullptr, (__nv_bfloat16*)nullptr) : f((__nv_bfloat16*)nullptr, (float*)nullptr);
    return b == DYNAMO_BF16 ? f((float*)nullptr, (__nv_bfloat16*)nullptr) : f((float*)nullptr, (float*)nullptr);
}

// Up to this many pairs every CTA counts the whole array by itself; beyond, a launch in front counts each CTA's share.
constexpr long long DISPATCH_ONE_PAIRS = 16384;

}  // namespace dyn

using namespace dyn;

namespace {

dynamo_status check_route_sizes(int32_t T, int32_t k) {
    if (k < 1 || k > 8) return DYNAMO_ERR_SHAPE;
    if (T < 0 || (long long)T * k > 0x7fffffffll) return DYNAMO_ERR_TOKENS;
    return DYNAMO_OK;
}
dynamo_status check_row(int32_t d, int32_t dtype) {
    return d < 8 || d % 8 || (dtype != DYNAMO_BF16 && dtype != DYNAMO_F32) ? DYNAMO_ERR_SHAPE : DYNAMO_OK;
}

}  // namespace

extern "C" {

dynamo_status dynamo_dispatch_workspace_bytes(int32_t T, int32_t n_experts, int32_t top_k, size_t* bytes) {
    if (!bytes) return DYNAMO_ERR_NULL;
    if (n_experts < 1 || n_experts > DISPATCH_EXPERTS || top_k > n_experts) return DYNAMO_ERR_SHAPE;
    if (const dynamo_status s = check_route_sizes(T, top_k); s != DYNAMO_OK) return s;
    // counts of every CTA, of which there is one an SM (up to 256 SMs are reckoned with)
    *bytes = (long long)T * top_k > DISPATCH_ONE_PAIRS ? (size_t)256 * DISPATCH_EXPERTS * 4 : 0;
    return DYNAMO_OK;
}

dynamo_status dynamo_dispatch(const int32_t* topk_idx, int32_t T, int32_t n_experts, int32_t top_k, const void* x, int32_t d,
                              int32_t dtype, int32_t* expert_offsets, int32_t* perm, int32_t* pos, void* rows,
                              void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    if (const dynamo_status s = dynamo_dispatch_workspace_bytes(T, n_experts, top_k, &need); s != DYNAMO_OK) return s;
    if (x || rows)
        if (const dynamo_status s = check_row(d, dtype); s != DYNAMO_OK) return s;
    if (!expert_offsets || (T > 0 && (!topk_idx || !perm || !pos || (x != nullptr) != (rows != nullptr)))) return DYNAMO_ERR_NULL;
    if (!aligned16(x, rows)) return DYNAMO_ERR_ALIGN;
    if (need && !workspace) return DYNAMO_ERR_NULL;
    if (workspace_bytes < need) return DYNAMO_ERR_ARENA_TOO_SMALL;
    if (need && ((uintptr_t)workspace & 255)) return DYNAMO_ERR_ALIGN;
    cudaStream_t st = (cudaStream_t)stream;
    int n_sms = 0;
    if (count_sms(&n_sms) != cudaSuccess) return DYNAMO_ERR_CUDA;
    DispatchArgs a = {};
    a.idx = topk_idx;
    a.T = T;
    a.k = top_k;
    a.E = n_experts;
    a.offsets = expert_offsets;
    a.perm = perm;
    a.pos = pos;
    a.x = T > 0 ? (const uint8_t*)x : nullptr;
    a.rows = (uint8_t*)rows;
    a.row_bytes = x ? (long long)d * (dtype == DYNAMO_BF16 ? 2 : 4) : 0;
    a.hist = need ? (int32_t*)workspace : nullptr;
    a.E_pad = 1;
    while (a.E_pad < n_experts) a.E_pad *= 2;
    const int most = std::min(256, n_sms);
    a.seg = std::max(1, (int)(((long long)T + most - 1) / most));
    const unsigned ctas = (unsigned)std::max(1, (int)(((long long)T + a.seg - 1) / a.seg));   // without tokens: the offsets
    if (a.hist && launch_pdl(dispatch_count_kernel, dim3(ctas), dim3(DISPATCH_THREADS), 0, st, a) != cudaSuccess)
        return DYNAMO_ERR_CUDA;
    return launch_pdl(dispatch_kernel, dim3(ctas), dim3(DISPATCH_THREADS), 0, st, a) == cudaSuccess ? DYNAMO_OK : DYNAMO_ERR_CUDA;
}

dynamo_status dynamo_combine(const void* rows, int32_t dtype, const int32_t* pos, const float* topk_w, int32_t T, int32_t top_k,
                             int32_t d, void* y, int32_t y_dtype, void* stream) {
    if (const dynamo_status s = check_route_sizes(T, top_k); s != DYNAMO_OK) return s;
    if (const dynamo_status s = check_row(d, dtype); s != DYNAMO_OK) return s;
    if (y_dtype != DYNAMO_BF16 && y_dtype != DYNAMO_F32) return DYNAMO_ERR_SHAPE;
    const long long ctas = ((long long)T * (d / 8) + 255) / 256;
    if (ctas > 0x7fffffffll) return DYNAMO_ERR_TOKENS;
    if (T == 0) return DYNAMO_OK;
    if (!rows || !pos || !y) return DYNAMO_ERR_NULL;
    if (!aligned16(rows, y)) return DYNAMO_ERR_ALIGN;
    const cudaError_t e = by_types(dtype, y_dtype, [&](auto* ti, auto* to) {
        using TI = std::remove_pointer_t<decltype(ti)>;
        using TO = std::remove_pointer_t<decltype(to)>;
        return by_top_k(top_k, [&](auto kc) {
            return launch_pdl(combine_rows_kernel<TI, TO, decltype(kc)::value>, dim3((unsigned)ctas), dim3(256), 0,
                              (cudaStream_t)stream, (const TI*)rows, pos, topk_w, T, d, (TO*)y);
        });
    });
    return e == cudaSuccess ? DYNAMO_OK : DYNAMO_ERR_CUDA;
}

dynamo_status dynamo_combine_backward(const void* dy, int32_t dy_dtype, const void* rows, int32_t dtype, const int32_t* pos,
                                      const float* topk_w, int32_t T, int32_t top_k, int32_t d, void* d_rows, float* d_w,
                                      void* stream) {
    if (const dynamo_status s = check_route_sizes(T, top_k); s != DYNAMO_OK) return s;
    if (const dynamo_status s = check_row(d, dtype); s != DYNAMO_OK) return s;
    if (dy_dtype != DYNAMO_BF16 && dy_dtype != DYNAMO_F32) return DYNAMO_ERR_SHAPE;
    if (T == 0) return DYNAMO_OK;
    if (!dy || !rows || !pos || !d_rows) return DYNAMO_ERR_NULL;
    if (!aligned16(dy, rows, d_rows)) return DYNAMO_ERR_ALIGN;
    // A run of eight columns a thread where there are few tokens, two where there are many (us with one, two and four runs; rows of
    // 2048, top-6: 64 tokens 3.3, 4.2, 6.2; 600 tokens 8.9, 8.3, 10.0).
    const int runs = (long long)T * d < 8ll * 148 * 1024 ? 1 : 2;
    int tpt = 1;
    while (tpt < 256 && tpt * 8 * runs < d) tpt *= 2;
    if (((long long)T * tpt + 255) / 256 > 0x7fffffffll) return DYNAMO_ERR_TOKENS;
    const cudaError_t e = by_types(dtype, dy_dtype, [&](auto* tr, auto* ty) {
        using TR = std::remove_pointer_t<decltype(tr)>;
        using TY = std::remove_pointer_t<decltype(ty)>;
        return by_top_k(top_k, [&](auto kc) {
            constexpr int K = decltype(kc)::value;
            return launch_pdl(combine_grad_kernel<TR, TY, K>, dim3((unsigned)(((long long)T * tpt + 255) / 256)), dim3(256), 0,
                              (cudaStream_t)stream, (const TY*)dy, (const TR*)rows, pos, topk_w, T, d, tpt, (TR*)d_rows, d_w);
        });
    });
    return e == cudaSuccess ? DYNAMO_OK : DYNAMO_ERR_CUDA;
}

}  // extern "C"
