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
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Codes i and i + 4 of a word as the bf16 pair 16 + q.  The mask (0x0078 twice) and the pattern of 16.0 come with the kernel's
// arguments: as constants that the compiler knows they became two logical instructions a pair, with an immediate each.
struct PairBits {
    uint32_t mask, sixteen;
};
template <int I>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, const PairBits& p) {
    const uint32_t s = I == 0 ? w << 3 : w >> (4 * I - 3);
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(s), "r"(p.mask), "r"(p.sixteen));   // (s & mask) | sixteen
    return r;
}

struct LinearArgs {
    const __nv_bfloat16* x;   // [T, K]
    const uint8_t* codes;     // [N, K / 2]
    const uint32_t* params;   // [N, K / G] half2 {scale, zero}
    void* y;                  // [T, N]
    int T, K, N;
    PairBits bits;
    int n_split, units;       // shares of the input indices (CTAs of a cluster), units of LIN_UNIT in a share
};

constexpr int LIN_WARPS = 8;
constexpr int LIN_UNIT = 128;   // input indices of a step of the kernels
constexpr int LIN_MAX_CLUSTER = 8;

// Where the words of codes stand: a lane has four of each of its rows a unit.  Word j of group g of a unit covers the indices
// G g + 8 (W tid4 + j) .., W = words of a lane and row in a group: consecutive in memory for the lane, the group's own for
// the four lanes of a row together.
template <int G>
struct UnitShape {
    static constexpr int GROUPS = LIN_UNIT / G, W = 4 / GROUPS;
};

// Codes and parameters of rows gid and gid + 8 of an atom (16 rows) in a unit.  A lane addresses them by two 32-bit offsets from
// its CTA's first row (AtomPlace): 64-bit address arithmetic and bounds per load were half of the kernel's instructions.  Rows
// behind the matrix are read as its last one (their results go nowhere).
template <int G>
struct AtomPlace {
    uint32_t code[2], param[2];   // bytes; code: without the unit's part

    __device__ __forceinline__ AtomPlace(const LinearArgs& a, int n0, int row0) {
        const int lane = threadIdx.x & 31, gid = lane >> 2, tid4 = lane & 3;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t row = (uint32_t)(min(row0 + gid + 8 * h, a.N - 1) - n0);
            code[h] = row * (uint32_t)(a.K / 2) + tid4 * (4 * UnitShape<G>::W);
            param[h] = row * (uint32_t)(a.K / G) * 4;
        }
    }
};
template <int G>
struct AtomUnit {
    uint32_t cw[2][4];
    uint32_t pr[2][UnitShape<G>::GROUPS];

    // codes, params: of the CTA's first row.  The second group of a last unit of 64 indices is not there and not read.
    __device__ __forceinline__ void load(const LinearArgs& a, const uint8_t* codes, const uint8_t* params, const AtomPlace<G>& at,
                                         int u) {
        using S = UnitShape<G>;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t* p = codes + (at.code[h] + (uint32_t)u * (LIN_UNIT / 2));
            const uint8_t* q = params + (at.param[h] + (uint32_t)u * (4 * S::GROUPS));
            if constexpr (S::GROUPS == 1) {
                const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
                cw[h][0] = v.x, cw[h][1] = v.y, cw[h][2] = v.z, cw[h][3] = v.w;
                pr[h][0] = __ldg(reinterpret_cast<const uint32_t*>(q));
            } else {
                const bool two = u * LIN_UNIT + G < a.K;
                const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p));
                const uint2 w = two ? __ldcs(reinterpret_cast<const uint2*>(p + G / 2)) : make_uint2(0u, 0u);
                cw[h][0] = v.x, cw[h][1] = v.y, cw[h][2] = w.x, cw[h][3] = w.y;
                pr[h][0] = __ldg(reinterpret_cast<const uint32_t*>(q));
                pr[h][1] = two ? __ldg(reinterpret_cast<const uint32_t*>(q) + 1) : 0u;
            }
        }
    }
};

// The two MMAs of word j of group g: eight of the lane's indices, 32 of the four lanes'.  b: the activations as b_operands gives them.
template <int NT>
__device__ __forceinline__ void word_mmas(float (&c)[NT][4], uint32_t w0, uint32_t w1, const PairBits& p, const uint32_t (&b)[NT][4]) {
    const uint32_t p00 = code_pair<0>(w0, p), p01 = code_pair<0>(w1, p), p10 = code_pair<1>(w0, p), p11 = code_pair<1>(w1, p);
    const uint32_t p20 = code_pair<2>(w0, p), p21 = code_pair<2>(w1, p), p30 = code_pair<3>(w0, p), p31 = code_pair<3>(w1, p);
#pragma unroll
    for (int n = 0; n < NT; ++n) mma_bf16(c[n], p00, p01, p10, p11, b[n][0], b[n][1]);
#pragma unroll
    for (int n = 0; n < NT; ++n) mma_bf16(c[n], p20, p21, p30, p31, b[n][2], b[n][3]);
}
// Eight consecutive activations as pairs (0, 4), (1, 5), (2, 6), (3, 7): the codes' order.
__device__ __forceinline__ void b_operands(uint32_t (&b)[4], const uint4& v) {
    b[0] = __byte_perm(v.x, v.z, 0x5410);
    b[1] = __byte_perm(v.x, v.z, 0x7632);
    b[2] = __byte_perm(v.y, v.w, 0x5410);
    b[3] = __byte_perm(v.y, v.w, 0x7632);
}
constexpr uint32_t BF16_ONES = 0x3f803f80u;
__device__ __forceinline__ void sum_mmas(float (&sx)[4], const uint32_t (&b)[4]) {
    mma_bf16(sx, BF16_ONES, BF16_ONES, BF16_ONES, BF16_ONES, b[0], b[1]);
    mma_bf16(sx, BF16_ONES, BF16_ONES, BF16_ONES, BF16_ONES, b[2], b[3]);
}
// A group's sums into the results: y += s * sum((16 + q) x) + (m - 16 s) * sum(x).
template <int NT>
__device__ __forceinline__ void fold_group(float (&acc)[NT][4], const float (&c)[NT][4], const float (&sx)[NT][2], uint32_t pr0,
                                           uint32_t pr1) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t pw = h ? pr1 : pr0;
        const __half2 pv = *reinterpret_cast<const __half2*>(&pw);
        const float s = __low2float(pv), m = fmaf(-16.f, s, __high2float(pv));
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[n][2 * h + i] = fmaf(s, c[n][2 * h + i], fmaf(m, sx[n][i], acc[n][2 * h + i]));
    }
}
template <int NT>
__device__ __forceinline__ void zero(float (&c)[NT][4]) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) c[n][i] = 0.f;
}

template <typename TO>
__device__ __forceinline__ void store_y(const LinearArgs& a, int t, int row, float v) {
    if (row >= a.N || t >= a.T) return;
    const long long at = (long long)t * a.N + row;
    if constexpr (sizeof(TO) == 4) ((float*)a.y)[at] = v;
    else ((__nv_bfloat16*)a.y)[at] = __float2bfloat16_rn(v);
}

// The sums of a cluster's CTAs (each a share of the input indices) from their shared memory, in the order of the CTAs:
// element i of `part` of every CTA.
__device__ __forceinline__ float cluster_sum(const float* part, int i, int n_ctas) {
    float s = 0.f;
    for (int r = 0; r < n_ctas; ++r) {
        float v;
        asm volatile("{\n\t.reg .b32 ra;\n\tmapa.shared::cluster.u32 ra, %1, %2;\n\tld.shared::cluster.f32 %0, [ra];\n\t}"
                     : "=f"(v)
                     : "r"(smem_u32(part + i)), "r"(r)
                     : "memory");
        s += v;
    }
    return s;
}

// ---- few tokens (up to 16): bound by the codes ----------------------------------------------------------------------------
// CTA: 16 R rows, 8 NT tokens, of a cluster's CTAs along the input indices the blockIdx.x % n_split-th share; its warps take the
// share's units in turn, U units' codes on their way to a warp at any time, and add up their sums at the end.
template <int NT, int R, int U, int G, typename TO>
__global__ void __launch_bounds__(32 * LIN_WARPS) linear_few_kernel(const __grid_constant__ LinearArgs a) {
    using S = UnitShape<G>;
    __shared__ float part[LIN_WARPS][NT * 8][16 * R];
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tid4 = lane & 3;
    const int split = blockIdx.x % a.n_split, n0 = blockIdx.x / a.n_split * 16 * R, t0 = blockIdx.y * 8 * NT;
    const int u0 = split * a.units, u1 = min((a.K + LIN_UNIT - 1) / LIN_UNIT, u0 + a.units);
    float acc[R][NT][4];
#pragma unroll
    for (int r = 0; r < R; ++r) zero(acc[r]);
    const uint8_t* codes = a.codes + (long long)n0 * (a.K / 2);
    const uint8_t* params = reinterpret_cast<const uint8_t*>(a.params + (long long)n0 * (a.K / G));
    AtomUnit<G> ring[U][R];
    auto fetch = [&](int i, int u) {
        if (u < u1)
#pragma unroll
            for (int r = 0; r < R; ++r) ring[i][r].load(a, codes, params, AtomPlace<G>(a, n0, n0 + 16 * r), u);
    };
#pragma unroll
    for (int i = 0; i < U; ++i) fetch(i, u0 + warp + i * LIN_WARPS);
    const uint4* xt[NT];   // tokens behind the last one are read as the last (their results go nowhere)
#pragma unroll
    for (int n = 0; n < NT; ++n)
        xt[n] = reinterpret_cast<const uint4*>(a.x + (long long)min(t0 + 8 * n + gid, a.T - 1) * a.K) + S::W * tid4;
    for (int u = u0 + warp; u < u1; u += U * LIN_WARPS) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int ui = u + i * LIN_WARPS;
            if (ui >= u1) break;
#pragma unroll
            for (int g = 0; g < S::GROUPS; ++g) {
                if (g && ui * LIN_UNIT + g * G >= a.K) break;
                float c[R][NT][4], sx4[NT][4];
                zero(sx4);
#pragma unroll
                for (int r = 0; r < R; ++r) zero(c[r]);
#pragma unroll
                for (int j = 0; j < S::W; ++j) {
                    uint32_t b[NT][4];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        b_operands(b[n], __ldg(xt[n] + (ui * (LIN_UNIT / 8) + g * (G / 8) + j)));
                        sum_mmas(sx4[n], b[n]);
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) word_mmas(c[r], ring[i][r].cw[0][g * S::W + j], ring[i][r].cw[1][g * S::W + j], a.bits, b);
                }
                float sx[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) sx[n][0] = sx4[n][0], sx[n][1] = sx4[n][1];
#pragma unroll
                for (int r = 0; r < R; ++r) fold_group(acc[r], c[r], sx, ring[i][r].pr[0][g], ring[i][r].pr[1][g]);
            }
            fetch(i, ui + U * LIN_WARPS);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[warp][8 * n + 2 * tid4 + (i & 1)][16 * r + gid + 8 * (i >> 1)] = acc[r][n][i];
    __syncthreads();
    constexpr int OUT = NT * 8 * 16 * R;
    if (a.n_split == 1) {
        for (int o = threadIdx.x; o < OUT; o += 32 * LIN_WARPS) {
            const float* p = &part[0][0][0] + o;
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < LIN_WARPS; ++w) s += p[w * OUT];
            store_y<TO>(a, t0 + o / (16 * R), n0 + o % (16 * R), s);
        }
        return;
    }
    for (int o = threadIdx.x; o < OUT; o += 32 * LIN_WARPS) {
        float* p = &part[0][0][0] + o;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < LIN_WARPS; ++w) s += p[w * OUT];
        p[0] = s;   // read and written by this thread alone
    }
    cluster_sync_all();
    for (int o = split * 32 * LIN_WARPS + threadIdx.x; o < OUT; o += a.n_split * 32 * LIN_WARPS)
        store_y<TO>(a, t0 + o / (16 * R), n0 + o % (16 * R), cluster_sum(&part[0][0][0], o, a.n_split));
    cluster_sync_all();   // nobody leaves while others read its sums
}

// ---- more tokens: bound by the MMAs -----------------------------------------------------------------------------------------
// CTA: 8 warps, 32 rows and 32 tokens each, TOK / 32 of them side by side along the tokens; a share of the input indices as
// above.  A unit's codes, parameters and activations go through a ring in shared memory.  The activations are put into the order of
// the codes' pairs on their way (load, byte permutes, store: a sixteenth of the permutes that every warp would do for itself); 16-byte
// chunk `ch` (8 indices) of token t stands at chunk_at(t, ch), which lays the chunks that the four lanes of a row read at a time side by side
// and the next token's beside them (no bank twice among eight lanes).  A warp's two atoms share each of its reads of them.
// The activations' sums per group are one more n-tile's work a warp, left in shared memory for all.
constexpr int LIN_STAGES = 3;
template <int G>
__device__ __forceinline__ int chunk_at(int t, int ch) {
    using S = UnitShape<G>;
    const int g = ch / (G / 8), in = ch % (G / 8), q = in / S::W, j = in % S::W;   // lane q's j-th chunk of group g
    return t * 16 + ((q + 4 * (S::W * g + j)) ^ (4 * (t & 1)));
}
template <int G, int TOK>
struct TileStage {
    static constexpr int ROWS = 32 * LIN_WARPS / (TOK / 32);
    uint4 x[TOK * 16];
    uint4 code[ROWS * 4];
    uint32_t param[UnitShape<G>::GROUPS][ROWS];
};
__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(void* dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
template <int TOK, int G, typename TO>
__global__ void __launch_bounds__(32 * LIN_WARPS, 2) linear_tile_kernel(const __grid_constant__ LinearArgs a) {
    using S = UnitShape<G>;
    using Stage = TileStage<G, TOK>;
    constexpr int ROWS = Stage::ROWS, THREADS = 32 * LIN_WARPS, XC = TOK * 16 / THREADS, NT = 4;
    extern __shared__ __align__(16) uint8_t smem[];
    Stage* ring = reinterpret_cast<Stage*>(smem);
    __shared__ __align__(8) float sums[2][S::GROUPS][TOK];
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tid4 = lane & 3;
    const int split = blockIdx.x % a.n_split, n0 = blockIdx.x / a.n_split * ROWS, t0 = blockIdx.y * TOK;
    const int u0 = split * a.units, u1 = min((a.K + LIN_UNIT - 1) / LIN_UNIT, u0 + a.units);
    const int row_w = 32 * (warp % (ROWS / 32)), tok_w = 32 * (warp / (ROWS / 32));
    // this thread's chunk of every token row that it brings in, and its row of the codes
    const int xch = tid & 15;
    auto load_x = [&](uint4 (&v)[XC], int u) {
        if (u >= u1) return;
#pragma unroll
        for (int i = 0; i < XC; ++i) {
            const int t = min(t0 + (tid >> 4) + i * (THREADS / 16), a.T - 1), k = u * LIN_UNIT + 8 * xch;
            v[i] = k < a.K ? __ldg(reinterpret_cast<const uint4*>(a.x + (long long)t * a.K + k)) : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    auto put_x = [&](const uint4 (&v)[XC], Stage& st) {
#pragma unroll
        for (int i = 0; i < XC; ++i) {
            uint32_t b[4];
            b_operands(b, v[i]);
            st.x[chunk_at<G>((tid >> 4) + i * (THREADS / 16), xch)] = make_uint4(b[0], b[1], b[2], b[3]);
        }
    };
    auto fetch = [&](int u, Stage& st) {   // codes and parameters; rows behind the matrix as its last one
        if (u < u1) {
#pragma unroll
            for (int i = 0; i < ROWS * 4 / THREADS; ++i) {
                const int c = tid + i * THREADS, row = min(n0 + (c >> 2), a.N - 1), k = u * LIN_UNIT + 32 * (c & 3);
                if (k < a.K) cp_async16(&st.code[c], a.codes + (long long)row * (a.K / 2) + k / 2);
            }
#pragma unroll
            for (int g = 0; g < S::GROUPS; ++g)
                if (tid < ROWS && u * LIN_UNIT + g * G < a.K)
                    cp_async4(&st.param[g][tid], a.params + (long long)min(n0 + tid, a.N - 1) * (a.K / G) + u * S::GROUPS + g);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    float acc[2][NT][4];
    zero(acc[0]);
    zero(acc[1]);
    uint4 xv[XC] = {};
    load_x(xv, u0);
    fetch(u0, ring[0]);
    fetch(u0 + 1, ring[1]);
    put_x(xv, ring[0]);
    load_x(xv, u0 + 1);
    int stage = 0;
    for (int u = u0; u < u1; ++u) {
        asm volatile("cp.async.wait_group 1;" ::: "memory");   // all but the newest: unit u has landed
        __syncthreads();                                       // for every thread; the other two stages' readers are through
        const int next = stage + 1 == LIN_STAGES ? 0 : stage + 1, after = next + 1 == LIN_STAGES ? 0 : next + 1;
        fetch(u + 2, ring[after]);
        put_x(xv, ring[next]);
        load_x(xv, u + 2);
        const Stage& st = ring[stage];
        float* sm = &sums[u & 1][0][0];
        if (warp < TOK / 8) {
#pragma unroll
            for (int g = 0; g < S::GROUPS; ++g) {
                float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < S::W; ++j) {
                    const uint4 v = st.x[chunk_at<G>(8 * warp + gid, g * (G / 8) + S::W * tid4 + j)];
                    const uint32_t b[4] = {v.x, v.y, v.z, v.w};
                    sum_mmas(s4, b);
                }
                if (gid == 0) *reinterpret_cast<float2*>(sm + g * TOK + 8 * warp + 2 * tid4) = make_float2(s4[0], s4[1]);
            }
        }
#pragma unroll
        for (int g = 0; g < S::GROUPS; ++g) {
            if (g && u * LIN_UNIT + g * G >= a.K) break;
            float c[2][NT][4];
            uint32_t cw[2][2][S::W];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                zero(c[r]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4* p = &st.code[(row_w + 16 * r + 8 * h + gid) * 4];
                    if constexpr (S::GROUPS == 1) {
                        const uint4 v = p[tid4];
                        cw[r][h][0] = v.x, cw[r][h][1] = v.y, cw[r][h][2] = v.z, cw[r][h][3] = v.w;
                    } else {
                        const uint2 v = reinterpret_cast<const uint2*>(p)[4 * g + tid4];
                        cw[r][h][0] = v.x, cw[r][h][1] = v.y;
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < S::W; ++j) {
                uint32_t b[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 v = st.x[chunk_at<G>(tok_w + 8 * n + gid, g * (G / 8) + S::W * tid4 + j)];
                    b[n][0] = v.x, b[n][1] = v.y, b[n][2] = v.z, b[n][3] = v.w;
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) word_mmas(c[r], cw[r][0][j], cw[r][1][j], a.bits, b);
            }
            if (g == 0) __syncthreads();   // the sums are there
            float sx[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float2 v = *reinterpret_cast<const float2*>(sm + g * TOK + tok_w + 8 * n + 2 * tid4);
                sx[n][0] = v.x, sx[n][1] = v.y;
            }
#pragma unroll
            for (int r = 0; r < 2; ++r)
                fold_group(acc[r], c[r], sx, st.param[g][row_w + 16 * r + gid], st.param[g][row_w + 16 * r + 8 + gid]);
        }
        stage = next;
    }
    // results to shared memory, [token][row], then out in whole rows of a token
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    float* part = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                part[(tok_w + 8 * n + 2 * tid4 + (i & 1)) * ROWS + row_w + 16 * r + gid + 8 * (i >> 1)] = acc[r][n][i];
    if (a.n_split == 1) {
        __syncthreads();
        for (int o = tid; o < TOK * ROWS; o += THREADS) store_y<TO>(a, t0 + o / ROWS, n0 + o % ROWS, part[o]);
        return;
    }
    cluster_sync_all();
    for (int o = split * THREADS + tid; o < TOK * ROWS; o += a.n_split * THREADS)
        store_y<TO>(a, t0 + o / ROWS, n0 + o % ROWS, cluster_sum(part, o, a.n_split));
    cluster_sync_all();
}

// Shares of the input indices, a CTA of a cluster each: as many as leave the fewest units to the SM with most work.
static void split_units(LinearArgs& a, long long blocks, int n_sms, int per_sm, int least) {
    const int units = (a.K + LIN_UNIT - 1) / LIN_UNIT;
    int best = 1;
    double best_cost = 1e30;
    for (int c = 1; c <= LIN_MAX_CLUSTER; ++c) {
        const int share = (units + c - 1) / c;
        if (c > 1 && share < least) break;
        const long long rounds = (blocks * c + (long long)n_sms * per_sm - 1) / ((long long)n_sms * per_sm);
        const double cost = (double)rounds * (share + 12);
        if (cost < 0.95 * best_cost) best = c, best_cost = cost;
    }
    const int share = (units + best - 1) / best;
    a.units = share;
    a.n_split = (units + share - 1) / share;   // no empty shares
}

template <int NT, int R, int U, int G>
static cudaError_t linear_few(LinearArgs a, int y_f32, int n_sms, cudaStream_t st) {
    const unsigned blocks = (unsigned)((a.N + 16 * R - 1) / (16 * R)), tiles = (unsigned)((a.T + 8 * NT - 1) / (8 * NT));
    split_units(a, (long long)blocks * tiles, n_sms, 2, LIN_WARPS);
    const dim3 grid(blocks * a.n_split, tiles);
    return y_f32 ? launch_pdl_cluster(linear_few_kernel<NT, R, U, G, float>, grid, dim3(32 * LIN_WARPS), 0, a.n_split, st, a)
                 : launch_pdl_cluster(linear_few_kernel<NT, R, U, G, __nv_bfloat16>, grid, dim3(32 * LIN_WARPS), 0, a.n_split, st, a);
}
template <int TOK, int G>
static cudaError_t linear_tile(LinearArgs a, int y_f32, int n_sms, cudaStream_t st) {
    constexpr int ROWS = TileStage<G, TOK>::ROWS;
    constexpr int SMEM = LIN_STAGES * (int)sizeof(TileStage<G, TOK>);
    static_assert(SMEM >= TOK * ROWS * 4, "the results go where the stages were");
    const unsigned blocks = (unsigned)((a.N + ROWS - 1) / ROWS), tiles = (unsigned)((a.T + TOK - 1) / TOK);
    split_units(a, (long long)blocks * tiles, n_sms, 2, 4);
    const dim3 grid(blocks * a.n_split, tiles);
    auto go = [&](auto kernel) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
        return e != cudaSuccess ? e : launch_pdl_cluster(kernel, grid, dim3(32 * LIN_WARPS), SMEM, a.n_split, st, a);
    };
    return y_f32 ? go(linear_tile_kernel<TOK, G, float>) : go(linear_tile_kernel<TOK, G, __nv_bfloat16>);
}
template <int G>
static cudaError_t linear_by_tokens(const LinearArgs& a, int y_f32, int n_sms, cudaStream_t st) {
    if (a.T <= 8) return a.N >= 64 * n_sms ? linear_few<1, 2, 2, G>(a, y_f32, n_sms, st) : linear_few<1, 1, 4, G>(a, y_f32, n_sms, st);
    if (a.T <= 16) return linear_few<2, 2, 2, G>(a, y_f32, n_sms, st);
    if (a.T <= 32) return linear_tile<32, G>(a, y_f32, n_sms, st);
    return linear_tile<64, G>(a, y_f32, n_sms, st);
}

}  // namespace dyn

using namespace dyn;

namespace {

dynamo_status check_linear(int32_t rows, int32_t cols, int32_t group_size) {
    if (group_size != 64 && group_size != 128) return DYNAMO_ERR_SHAPE;
    if (rows < 1 || cols < group_size || cols % group_size || cols > 1 << 24) return DYNAMO_ERR_SHAPE;   // (offsets of 32 bits)
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
    int n_sms = 0;
    if (count_sms(&n_sms) != cudaSuccess) return DYNAMO_ERR_CUDA;
    const LinearArgs a = {(const __nv_bfloat16*)x, (const uint8_t*)codes, (const uint32_t*)params, y, T, cols, rows, {0x00780078u, 0x41804180u}, 1, 0};
    const cudaError_t e = group_size == 64 ? linear_by_tokens<64>(a, y_dtype == DYNAMO_F32, n_sms, (cudaStream_t)stream)
                                           : linear_by_tokens<128>(a, y_dtype == DYNAMO_F32, n_sms, (cudaStream_t)stream);
    return e == cudaSuccess ? DYNAMO_OK : DYNAMO_ERR_CUDA;
}

}  // extern "C"
