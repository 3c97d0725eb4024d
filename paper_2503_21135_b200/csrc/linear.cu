// Products of few token rows with a matrix of 4-bit codes and group scales (the quantizer is the experts', quant.cuh):
//
//   y[t][n] = sum over groups g of  s[n][g] * sum_{k in g} q[n][k] x[t][k]  +  m[n][g] * sum_{k in g} x[t][k]
//
// The codes are row-major, two a byte (index 2i in the low half of byte i), so a 32-bit word holds eight consecutive ones.
// A code becomes a bf16 operand by a shift, a mask and an OR: on the four highest mantissa bits of 16.0 it reads as
// 16 + q, exactly; the 16 goes off again, either in the operand (one subtraction a pair, exact: the tcgen05 kernel) or off the
// group's sum (the few-token kernel: sum((16 + q) x) - 16 sum(x), the second from MMAs with ones in the same steps, so that
// the two cancel to 0 where the codes are 0).  Then y += s * sum(q x) + m * sum(x).  The zero-point is used as it is: a group of one value has
// scale 1 and codes 0, and m - 16 s would lose an m that is small beside 16.  Products are exact in fp32 (bf16 by
// bf16); sums, scales and zero-points are in fp32, y is rounded once.  The order in which a warp's 16-wide steps take the
// input indices is free as long as codes and activations agree: a lane takes runs of consecutive ones from both.
#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "../../include/dynamo.h"
#include "common.cuh"
#include "quant.cuh"
#include "tcgen05.cuh"
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
    uint32_t mask, sixteen;        // 0x0078 and 16.0, twice
    uint32_t low, onetwentyeight;  // 0x000f and 128.0: a code on the four lowest mantissa bits of 128.0 reads as 128 + q
};
template <int I>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, const PairBits& p) {
    const uint32_t s = I == 0 ? w << 3 : w >> (4 * I - 3);
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(s), "r"(p.mask), "r"(p.sixteen));   // (s & mask) | sixteen
    return r;
}

// The same pair as q itself, and two shifts for the four pairs of a word (w8 = w >> 8).
template <int I>
__device__ __forceinline__ uint32_t whole_pair(uint32_t w, uint32_t w8, const PairBits& p) {
    const uint32_t s = I == 0 ? w : I == 1 ? w >> 1 : I == 2 ? w8 : w8 >> 1;
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(s), "r"(I & 1 ? p.mask : p.low), "r"(I & 1 ? p.sixteen : p.onetwentyeight));
    const uint32_t off = I & 1 ? 0x41804180u : 0x43004300u;
    const __nv_bfloat162 q = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&r), *reinterpret_cast<const __nv_bfloat162*>(&off));
    return *reinterpret_cast<const uint32_t*>(&q);
}

struct LinearArgs {
    const __nv_bfloat16* x;   // [T, K]
    const uint8_t* codes;     // [N, K / 2]
    const uint32_t* params;   // [N, K / G] half2 {scale, zero}
    void* y;                  // [T, N]
    int T, K, N;
    PairBits bits;
    const uint8_t* xt;        // tcgen05 kernel: activations in its order
    float* part;              // and partial results, two tiles a CTA
    int n_split, units;       // shares of the input indices (CTAs of a cluster), units of LIN_UNIT in a share
    int withhold;             // 1 (dynamo_debug_expire_linear): the first CTA's first stage of activations is never brought
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
// A group's sums into the results: y += s * (sum((16 + q) x) - 16 sum(x)) + m * sum(x).
template <int NT>
__device__ __forceinline__ void fold_group(float (&acc)[NT][4], const float (&c)[NT][4], const float (&sx)[NT][2], uint32_t pr0,
                                           uint32_t pr1) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t pw = h ? pr1 : pr0;
        const __half2 pv = *reinterpret_cast<const __half2*>(&pw);
        const float s = __low2float(pv), m = __high2float(pv);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                acc[n][2 * h + i] = fmaf(s, fmaf(-16.f, sx[n][i], c[n][2 * h + i]), fmaf(m, sx[n][i], acc[n][2 * h + i]));
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

// ---- few tokens, small matrices: bound by the codes ----------------------------------------------------------------------------
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

// ---- tcgen05: the codes as the A operand in tensor memory -------------------------------------------------------------------
// The work is a line of stages: 256 rows (two row tiles of an MMA's 128) x 128 input indices for TOK tokens, a block's stages one behind
// another; one persistent CTA per SM takes an equal run of it.  Roles by warp:
//   0-7   expand : two groups of four (a warp per lane quarter of the tensor memory); a group takes every other stage: 16 rows x 128
//                  indices of codes at a time -> q as bf16 pairs -> A buffer (16x256b stores, so that four lanes read a
//                  row's codes; a row a lane kept the L1 busy with 32 lines a load).  The codes come by cp.async, three jobs of a warp
//                  on their way: 96 KB an SM (one job in registers left the loads' latency to bind)
//   8-    fold   : (lane quarter, row tile) each, a row a lane; per group  y += s * acc + m * sum(x); sixteen warps at 64
//                  tokens, half of the columns each (14336 x 14336, 64 tokens, groups of 64 / 128: 82 / 58 us; as 78.3 / 55.4 they were compared, before the
//                  operand's 16 went off in the expansion, with packed pairs, whose moves and registers cost more than the instructions
//                  they save, 85.1 / 54.1, and both halves of the columns on their way
//                  90.0 / 53.7, spilling; eight warps 107 / 50.6; sixteen of a quarter of the columns and both row tiles, half the reads of
//                  the sums, 109 / 54.6)
//   next  fetch  : one thread; a bulk copy a stage of the activations, which linear_x_kernel has put into the operand's order,
//                  with their sums per group behind them
//   last  MMA    : 2 * 128 / 16 tcgen05.mma of 128 x TOK x 16 a stage, a run and one commit
// Roles meet at barriers only, so that the chain of a stage (codes, expansion, MMAs, fold) overlaps its neighbours', blocks' ends
// included; the same work by eight warps that all did every part, a barrier of the CTA a stage, took 88 us at 64 tokens, 14336 x 14336.
// Bound by the fold at 64 tokens (63% of the issue slots at groups of 64), by the expansion and the hand-overs at 32 and fewer:
// 46 us at 14336 x 14336 and 32 tokens, 2.4 TB/s of codes and parameters.  The subtraction that makes 16 + q a q is 2 to 5% of the time.
// A block that lies within one CTA's run goes from the fold warps' registers to y; the pieces of the others go to the workspace, and a
// kernel behind this one adds them up in the order of the CTAs.
// Tensor memory: two A buffers of 128 columns, then BUFS accumulator buffers of 2 * TOK, one a group.
// Every wait is bounded; after an expired one the roles end (and arrive at no barrier any more: a stage that was not waited for is not
// handed on), the CTA's remaining results are NaN and the status word is set.  Copies and MMAs that are still under way then have
// a while to end before the CTA's shared and tensor memory goes away.
constexpr int TC_ROWS = 256;
constexpr int TC_SLOTS = 4;       // stages of activations on their way or in use
constexpr int TC_JOBS = 3;        // jobs (four atoms of a stage) of an expand warp whose codes are on their way or in use
constexpr int TC_COLS = 512;
constexpr int TC_MAX_CTAS = 160;  // that the workspace has room for
static __device__ int32_t g_linear_status[16];

template <int TOK, int G>
struct TcShape {
    static constexpr int GROUPS = LIN_UNIT / G, W = G / 32;     // groups of a stage; words of codes of a lane, row and group
    static constexpr int LBO = TOK * 16;                        // bytes between octets of indices
    static constexpr int XB = 16 * LBO + GROUPS * TOK * 4;      // bytes of a stage's activations and sums
    static constexpr int BUFS = TOK == 64 ? 2 : 4;
    static constexpr int FOLDS = TOK == 64 ? 16 : 8;             // fold warps: (lane quarter, row tile), and half of the tokens where there are 64
    static constexpr int NC = TOK * 8 / FOLDS;                  // columns of a fold warp
    static constexpr int W_FETCH = 8 + FOLDS, W_MMA = W_FETCH + 1, WARPS = W_MMA + 1;
    static constexpr int CODES = 8 * TC_JOBS * 4096;            // bytes of the expand warps' rings
    static constexpr int SMEM = CODES + TC_SLOTS * XB;
    static_assert(256 + BUFS * 2 * TOK <= TC_COLS, "tensor memory");
    static_assert(XB % 16 == 0, "bulk copies");
};

// Activations in the order of the B operand, K-major core matrices of 8 tokens x 8 indices: [token tile][stage][octet of indices 16]
// [token TOK][16 bytes], then the sums [group][TOK].  A warp has eight tokens of a stage.  Chunk (t, wd) of a group, the indices
// 8 (W t + wd) .., is a lane t's word wd of the codes; the 16x256b store gives the word's pairs 2 j, 2 j + 1 (j counted over
// the lane's words) the columns 8 j + 2 t, + 1: half t & 1 of octet 2 j + (t >> 1).  The sums come from MMAs with ones.
template <int TOK, int G>
__global__ void __launch_bounds__(256) linear_x_kernel(const __nv_bfloat16* __restrict__ x, int T, int K, int stages, int tiles,
                                                       uint8_t* __restrict__ out) {
    using S = TcShape<TOK, G>;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, gid = lane >> 2, tid4 = lane & 3;
    const int w = blockIdx.x * 8 + (threadIdx.x >> 5), stage = w % stages, oct = w / stages;   // octets of tokens over all tiles
    if (oct >= tiles * (TOK / 8)) return;
    const int tile = oct / (TOK / 8), tok = 8 * (oct % (TOK / 8)) + gid;
    const __nv_bfloat16* row = x + (long long)min(TOK * tile + tok, T - 1) * K + (long long)stage * LIN_UNIT;
    uint8_t* to = out + ((long long)tile * stages + stage) * S::XB;
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = 4 * i + tid4;
        v[i] = stage * LIN_UNIT + 8 * c < K ? *reinterpret_cast<const uint4*>(row + 8 * c) : make_uint4(0u, 0u, 0u, 0u);
    }
    float sum[S::GROUPS][4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mma_bf16(sum[i * S::GROUPS / 4], BF16_ONES, BF16_ONES, BF16_ONES, BF16_ONES, v[i].x, v[i].y);
        mma_bf16(sum[i * S::GROUPS / 4], BF16_ONES, BF16_ONES, BF16_ONES, BF16_ONES, v[i].z, v[i].w);
        uint32_t p[4];
        b_operands(p, v[i]);
        const int c = 4 * i + tid4, g = c / (4 * S::W), t = c % (4 * S::W) / S::W, wd = c % S::W;
        uint8_t* at = to + (G / 8 * g + 4 * wd + (t >> 1)) * S::LBO + tok * 16 + 8 * (t & 1);
        *reinterpret_cast<uint2*>(at) = make_uint2(p[0], p[1]);
        *reinterpret_cast<uint2*>(at + 2 * S::LBO) = make_uint2(p[2], p[3]);
    }
    if (lane < 4)
#pragma unroll
        for (int g = 0; g < S::GROUPS; ++g)
            *reinterpret_cast<float2*>(to + 16 * S::LBO + (g * TOK + 8 * (oct % (TOK / 8)) + 2 * lane) * 4) = make_float2(sum[g][0], sum[g][1]);
}

struct TcShared {
    uint64_t x_full[TC_SLOTS], x_empty[TC_SLOTS];   // a stage's activations have landed; the fold warps are done with the stage
    uint64_t a_full[2], a_empty[2];                 // the four expand warps of the stage have stored it; its MMAs are complete
    uint64_t acc_full[4], acc_empty[4];             // a group's MMAs are complete; the fold warps have read the accumulator buffer
    uint32_t tmem;
    volatile int poison;
};
struct TcRole {
    TcShared* S;
    uint32_t sb, ring, codes, tm;   // shared-memory addresses of the barriers, the activations and the codes; tensor memory
    int stages, blocks;             // stages of a block, blocks of a token tile
    int first, n;                   // the CTA's run: first stage (over all blocks and token tiles) and length
};
#define TC_BAR(field, i) (R.sb + (uint32_t)offsetof(TcShared, field) + 8u * (uint32_t)(i))

// Where a role is in the line of stages: token tile, first row, stage of the block.
struct TcPos {
    int tile, n0, u;
    __device__ __forceinline__ TcPos(const TcRole& R) {
        const int block = R.first / R.stages;
        u = R.first - block * R.stages;
        tile = block / R.blocks;
        n0 = (block - tile * R.blocks) * TC_ROWS;
    }
    __device__ __forceinline__ bool step(const TcRole& R, int by = 1) {   // true: to another block, its first stage
        u += by;
        if (u < R.stages) return false;
        u = 0;
        n0 += TC_ROWS;
        if (n0 == R.blocks * TC_ROWS) n0 = 0, ++tile;
        return true;
    }
};
// CTA c of n: the stages [c U / n, (c + 1) U / n) of U.
__host__ __device__ __forceinline__ int tc_first(int c, int n, int U) { return (int)((long long)c * U / n); }

// Groups that stage u has (the last may have one of two).
template <int G>
__device__ __forceinline__ int stage_groups(int u, int K) {
    return G == LIN_UNIT ? 1 : min(LIN_UNIT / G, K / G - u * (LIN_UNIT / G));
}

__device__ __forceinline__ void lds64(uint32_t a, uint32_t& x, uint32_t& y) {
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(x), "=r"(y) : "r"(a) : "memory");
}
template <int G>
__device__ __noinline__ void tc_expand_role(const LinearArgs& a, TcRole R, int warp, int lane) {
    using S = TcShape<64, G>;
    const int q = warp & 3, kh = warp >> 2, gid = lane >> 2, tid4 = lane & 3;
    // (copies: behind every asm that may write memory the arguments would be read again)
    const PairBits bits = a.bits;
    const int N = a.N, K = a.K;
    TcShared* const sh = R.S;
    const uint8_t* const base = a.codes;
    // [job][atom][row half][row 8][64 bytes]; groups of 64: rows 2, 3, 6, 7 with their halves exchanged, for the banks of the 8-byte reads
    const uint32_t ring = R.codes + warp * (TC_JOBS * 4096) + gid * 64, flip = G == LIN_UNIT ? 0 : gid & 2;
    const uint32_t put = ring + 16 * (tid4 ^ flip), take = G == LIN_UNIT ? put : ring + 16 * ((tid4 >> 1) ^ flip) + 8 * (tid4 & 1);
    TcPos ahead(R);
    if (kh) ahead.step(R);
    int s_ahead = kh;
    uint32_t rows[4][2];   // byte offsets of the lane's rows 128 (i >> 1) + 32 q + 16 (i & 1) + gid (+ 8) in the block
    const uint8_t* from;   // of the block's first row, at the lane's place
    auto block_ahead = [&]() {
        from = base + (long long)ahead.n0 * (K / 2) + tid4 * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                rows[i][e] = (uint32_t)min(128 * (i >> 1) + 32 * q + 16 * (i & 1) + gid + 8 * e, N - 1 - ahead.n0) * (uint32_t)(K / 2);
    };
    block_ahead();
    auto bring = [&](int job) {   // the four atoms of the next stage
        if (s_ahead < R.n) {
            const uint32_t k = (uint32_t)ahead.u * (LIN_UNIT / 2);
            const int ng = stage_groups<G>(ahead.u, K);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint8_t* at = from + (rows[i][e] + k);
                    if (G == LIN_UNIT || ng == 2 || tid4 < 2)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(put + job * 4096 + i * 1024 + e * 512), "l"(at) : "memory");
                }
            s_ahead += 2;
            const bool a1 = ahead.step(R), a2 = ahead.step(R);
            if (a1 || a2) block_ahead();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int j = 0; j < TC_JOBS; ++j) bring(j);
    int job = 0;
    uint32_t par = 1;   // of the round that emptied the A buffer before (passes at once the first time)
    for (int s = kh; s < R.n; s += 2, par ^= 1) {
        const uint32_t free = bar_test(TC_BAR(a_empty, kh), par);
        asm volatile("cp.async.wait_group %0;" ::"n"(TC_JOBS - 1) : "memory");   // this job's codes 
        __syncwarp();   // of all lanes
        if (!warp_saw(free) && !warp_wait(TC_BAR(a_empty, kh), par, &sh->poison, g_linear_status, 1, s)) break;
        tc_fence_after();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t to = R.tm + ((uint32_t)(32 * q + 16 * (i & 1)) << 16) + 128 * kh + 64 * (i >> 1);
            uint32_t cw[2][4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t at = take + job * 4096 + i * 1024 + e * 512;
                if constexpr (G == LIN_UNIT) {
                    const uint4 v = lds128(at);
                    cw[e][0] = v.x, cw[e][1] = v.y, cw[e][2] = v.z, cw[e][3] = v.w;
                } else {   // eight bytes of either group
                    lds64(at, cw[e][0], cw[e][1]);
                    lds64(at ^ 32, cw[e][2], cw[e][3]);
                }
            }
            uint32_t r[32];   // words in pairs of columns: register 4 j + 2 e (+ 1) is row gid + 8 e, pairs 2 j, 2 j + 1
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t w = cw[e][j >> 1], w8 = w >> 8;
                    r[4 * j + 2 * e] = j & 1 ? whole_pair<2>(w, w8, bits) : whole_pair<0>(w, w8, bits);
                    r[4 * j + 2 * e + 1] = j & 1 ? whole_pair<3>(w, w8, bits) : whole_pair<1>(w, w8, bits);
                }
            tc_st_x8(to, r);
        }
        __syncwarp();
        bring(job);   // into the place of the codes that have just been read
        job = job + 1 == TC_JOBS ? 0 : job + 1;
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(TC_BAR(a_full, kh));
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// The MMAs of a group, both row tiles: G / 16 steps of 16 indices, A columns 8 k, B octets 2 k.  The first starts from zero.
#define LIN_MMA(d, a, k, acc)                                            \
    "add.s64 bd, %4, " #k "*%6;\n\tadd.s32 aa, " a ", " #k "*8;\n\t"     \
    "@q tcgen05.mma.cta_group::1.kind::f16 [" d "], [aa], bd, %5, " acc ";\n\t"
#define LIN_MMA4(d, a, k0, k1, k2, k3, first) \
    LIN_MMA(d, a, k0, first) LIN_MMA(d, a, k1, "p1") LIN_MMA(d, a, k2, "p1") LIN_MMA(d, a, k3, "p1")
#define LIN_HEAD                                                                                                       \
    "{\n\t.reg .pred q, p0, p1;\n\t.reg .b64 bd;\n\t.reg .b32 aa;\n\telect.sync _|q, 0xffffffff;\n\t"                  \
    "setp.ne.b32 p0, 0, 0;\n\tsetp.eq.b32 p1, 0, 0;\n\t"
template <int G, int STEP>
__device__ __forceinline__ void linear_mmas(uint32_t d0, uint32_t d1, uint32_t a0, uint32_t a1, uint64_t bd, uint32_t idesc) {
    if constexpr (G == 128)
        asm volatile(LIN_HEAD LIN_MMA4("%0", "%2", 0, 1, 2, 3, "p0") LIN_MMA4("%0", "%2", 4, 5, 6, 7, "p1")
                         LIN_MMA4("%1", "%3", 0, 1, 2, 3, "p0") LIN_MMA4("%1", "%3", 4, 5, 6, 7, "p1") "}" ::"r"(d0),
                     "r"(d1), "r"(a0), "r"(a1), "l"(bd), "r"(idesc), "n"(STEP)
                     : "memory");
    else
        asm volatile(LIN_HEAD LIN_MMA4("%0", "%2", 0, 1, 2, 3, "p0") LIN_MMA4("%1", "%3", 0, 1, 2, 3, "p0") "}" ::"r"(d0), "r"(d1),
                     "r"(a0), "r"(a1), "l"(bd), "r"(idesc), "n"(STEP)
                     : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar)
        : "memory");
}
template <int TOK, int G>
__device__ __noinline__ void tc_mma_role(const LinearArgs& a, TcRole R) {
    using S = TcShape<TOK, G>;
    constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TOK / 8) << 17) | ((128u / 16) << 24);   // fp32 += bf16 x bf16
    const int K = a.K;
    TcShared* const sh = R.S;
    uint32_t buf = 0, par = 0;   // next accumulator buffer, parity of its round
    uint32_t ready = 0;          // the next stage's barriers, asked for before this stage's MMAs are issued
    TcPos pos(R);
    for (int s = 0; s < R.n; ++s, pos.step(R)) {
        const int slot = s % TC_SLOTS;
        if (!warp_saw(ready) && (!warp_wait(TC_BAR(x_full, slot), (s / TC_SLOTS) & 1, &sh->poison, g_linear_status, 2, s) ||
                                 !warp_wait(TC_BAR(a_full, s & 1), (s >> 1) & 1, &sh->poison, g_linear_status, 3, s)))
            return;
        ready = bar_test(TC_BAR(x_full, (s + 1) % TC_SLOTS), ((s + 1) / TC_SLOTS) & 1) & bar_test(TC_BAR(a_full, (s + 1) & 1), ((s + 1) >> 1) & 1);
        const int ng = stage_groups<G>(pos.u, K);
        for (int g = 0; g < ng; ++g) {
            if (!warp_wait(TC_BAR(acc_empty, buf), par ^ 1, &sh->poison, g_linear_status, 4, s)) return;
            tc_fence_after();
            // (the shuffles tell the compiler that the operands are warp-uniform)
            const uint32_t d = __shfl_sync(0xffffffffu, R.tm + 256 + buf * (2 * TOK), 0);
            const uint32_t at = __shfl_sync(0xffffffffu, R.tm + 128 * (s & 1) + (G / 2) * g, 0);
            const uint32_t xu = __shfl_sync(0xffffffffu, R.ring + slot * S::XB + g * (G / 8) * S::LBO, 0);
            linear_mmas<G, 2 * S::LBO / 16>(d, d + TOK, at, at + 64, tc_desc(xu, S::LBO, 128), IDESC);
            tc_commit(TC_BAR(acc_full, buf));
            if (++buf == S::BUFS) buf = 0, par ^= 1;
        }
        tc_commit(TC_BAR(a_empty, s & 1));
        tc_commit(TC_BAR(x_empty, slot));
    }
}

// Sixteen consecutive values that all lanes read, asked for together.
__device__ __forceinline__ void lds_values16(uint32_t a, float (&v)[16]) {
    asm volatile(
        "ld.shared.v4.f32 {%0,%1,%2,%3}, [%16];\n\tld.shared.v4.f32 {%4,%5,%6,%7}, [%16+16];\n\t"
        "ld.shared.v4.f32 {%8,%9,%10,%11}, [%16+32];\n\tld.shared.v4.f32 {%12,%13,%14,%15}, [%16+48];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
          "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(a)
        : "memory");
}
template <int TOK, int G, typename TO>
__device__ __noinline__ void tc_fold_role(const LinearArgs& a, TcRole R, int fw, int lane) {
    using S = TcShape<TOK, G>;
    constexpr int NC = S::NC;
    const int q = fw & 3, mt = (fw >> 2) & 1, col0 = (fw >> 3) * NC;
    const int K = a.K, N = a.N, groups = K / G, row_in = 128 * mt + 32 * q + lane;
    const uint32_t* const params = a.params;
    TcShared* const sh = R.S;
    float total[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) total[c] = 0.f;
    // Parameters, four groups of the lane's row at a time and one load ahead: a load takes the L1 a pass per row, and one by one these
    // were 40% of its passes.
    constexpr int QUAD = 4 / S::GROUPS;   // stages
    TcPos pos(R), ahead(R);
    const uint32_t* from;   // of the block ahead
    auto block_ahead = [&]() { from = params + (long long)min(ahead.n0 + row_in, N - 1) * groups; };
    block_ahead();
    uint4 cur, nxt;
    int left = 0;           // stages that cur has left
    auto load_quad = [&]() {
        const int g = ahead.u * S::GROUPS & ~3;
        if ((groups & 3) == 0)
            nxt = __ldg(reinterpret_cast<const uint4*>(from + g));
        else
            nxt = make_uint4(__ldg(from + g), g + 1 < groups ? __ldg(from + g + 1) : 0u, g + 2 < groups ? __ldg(from + g + 2) : 0u,
                             g + 3 < groups ? __ldg(from + g + 3) : 0u);
        if (ahead.step(R, QUAD - ahead.u % QUAD)) block_ahead();
    };
    load_quad();
    bool ok = true;
    uint32_t buf = 0, par = 0, ready = 0;
    const int u_first = pos.u;   // a first block that does not begin with its first stage is a piece
    int piece = 0;
    for (int s = 0; s < R.n; ++s) {
        const int slot = s % TC_SLOTS, ng = stage_groups<G>(pos.u, K);
        if (left == 0) {
            cur = nxt;
            const int skip = pos.u % QUAD;
            left = min(QUAD - skip, R.stages - pos.u);
            if (skip * S::GROUPS & 1) cur.x = cur.y, cur.y = cur.z, cur.z = cur.w;
            if (skip * S::GROUPS & 2) cur.x = cur.z, cur.y = cur.w;
            load_quad();
        }
        --left;
        float s1[S::GROUPS], m1[S::GROUPS];
#pragma unroll
        for (int g = 0; g < S::GROUPS; ++g) {
            const __half2 pv = *reinterpret_cast<const __half2*>(&cur.x);
            s1[g] = __low2float(pv);
            m1[g] = __high2float(pv);
            cur.x = cur.y, cur.y = cur.z, cur.z = cur.w;
        }
        if (ok) ok = warp_saw(ready) || warp_wait(TC_BAR(x_full, slot), (s / TC_SLOTS) & 1, &sh->poison, g_linear_status, 5, s);
        uint32_t full = bar_test(TC_BAR(acc_full, buf), par);
        ready = bar_test(TC_BAR(x_full, (s + 1) % TC_SLOTS), ((s + 1) / TC_SLOTS) & 1);
        // zero-points times the sums, as soon as the copies have landed (a group that is not there: m = 0, sums of zeros)
#pragma unroll
        for (int g = 0; g < S::GROUPS; ++g) {
#pragma unroll
            for (int c0 = 0; c0 < NC; c0 += 16) {
                float x[16];
                lds_values16(R.ring + slot * S::XB + 16 * S::LBO + (g * TOK + col0 + c0) * 4, x);
#pragma unroll
                for (int c = 0; c < 16; ++c) total[c0 + c] = fmaf(m1[g], x[c], total[c0 + c]);
            }
        }
        reads_done();
        __syncwarp();
        if (ok && lane == 0) bar_arrive(TC_BAR(x_empty, slot));
#pragma unroll
        for (int g = 0; g < S::GROUPS; ++g) {
            if (g >= ng) break;
            if (ok) ok = warp_saw(full) || warp_wait(TC_BAR(acc_full, buf), par, &sh->poison, g_linear_status, 6, s);
            if (!ok) break;
            tc_fence_after();
            const uint32_t acc = R.tm + ((uint32_t)(32 * q) << 16) + 256 + buf * (2 * TOK) + mt * TOK + col0;
            auto sixteen = [&](const int c0) {
                uint32_t rr[16];
                tc_ld_rows16(acc + c0, rr);
                // (with the registers: what is read of them stays behind the wait)
                asm volatile("tcgen05.wait::ld.sync.aligned;"
                             : "+r"(rr[0]), "+r"(rr[1]), "+r"(rr[2]), "+r"(rr[3]), "+r"(rr[4]), "+r"(rr[5]), "+r"(rr[6]), "+r"(rr[7]), "+r"(rr[8]),
                               "+r"(rr[9]), "+r"(rr[10]), "+r"(rr[11]), "+r"(rr[12]), "+r"(rr[13]), "+r"(rr[14]), "+r"(rr[15])
                             :
                             : "memory");
                if (c0 + 16 >= NC) {   // the buffer is read: hand it back
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(TC_BAR(acc_empty, buf));
                    if (++buf == S::BUFS) buf = 0, par ^= 1;
                    if (g + 1 < ng) full = bar_test(TC_BAR(acc_full, buf), par);
                }
#pragma unroll
                for (int c = 0; c < 16; ++c) total[c0 + c] = fmaf(s1[g], __uint_as_float(rr[c]), total[c0 + c]);
            };
#pragma unroll
            for (int c0 = 0; c0 < NC; c0 += 16) sixteen(c0);
        }
        if (pos.u + 1 == R.stages || s + 1 == R.n) {
            // the block's end, or the run's: a row a lane, so a column's stores of a warp are 32 consecutive values
            const bool whole = pos.u + 1 == R.stages && (piece || u_first == 0);
            const int t0 = pos.tile * TOK + col0, row = pos.n0 + row_in;
            float* part = a.part + ((long long)(2 * blockIdx.x + (piece ? 1 : 0)) * TOK + col0) * TC_ROWS + row_in;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const float v = !ok ? __int_as_float(0x7fffffff) : total[c];
                if (!whole) part[c * TC_ROWS] = v;
                else store_y<TO>(a, t0 + c, row, v);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) total[c] = 0.f;
            piece = 1;
        }
        pos.step(R);
    }
    if (!ok) sh->poison = 1;
}

template <int TOK, int G, typename TO>
__global__ void __launch_bounds__(32 * TcShape<TOK, G>::WARPS, 1) linear_tc_kernel(const __grid_constant__ LinearArgs a) {
    using S = TcShape<TOK, G>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ TcShared sh;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < TC_SLOTS; ++i) {
            mbar_init(&sh.x_full[i], 1);
            mbar_init(&sh.x_empty[i], S::FOLDS + 1);   // the fold warps have read the sums, and the MMAs are complete
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.a_full[i], 4);
            mbar_init(&sh.a_empty[i], 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&sh.acc_full[i], 1);
            mbar_init(&sh.acc_empty[i], S::FOLDS);
        }
        sh.poison = 0;
        fence_barrier_init();
    }
    if (warp == S::W_MMA) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "n"(TC_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // Everything above runs beside the kernel that lays the activations out (all before that one has completed).
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    TcRole R;
    R.S = &sh;
    R.sb = smem_u32(&sh);
    R.codes = smem_u32(smem);
    R.ring = R.codes + S::CODES;
    R.tm = __shfl_sync(0xffffffffu, sh.tmem, 0);
    R.stages = (a.K + LIN_UNIT - 1) / LIN_UNIT;
    R.blocks = (a.N + TC_ROWS - 1) / TC_ROWS;
    R.first = tc_first(blockIdx.x, gridDim.x, a.units);
    R.n = tc_first(blockIdx.x + 1, gridDim.x, a.units) - R.first;
    if (warp < 8) {
        tc_expand_role<G>(a, R, warp, lane);
    } else if (warp < S::W_FETCH) {
        tc_fold_role<TOK, G, TO>(a, R, warp - 8, lane);
    } else if (warp == S::W_FETCH) {
        if (lane == 0) {
            TcPos pos(R);
            bool ok = true;
            for (int s = 0; s < R.n && ok; ++s, pos.step(R)) {
                const int slot = s % TC_SLOTS;
                if (s >= TC_SLOTS)
                    ok = mbar_wait_bounded(&sh.x_empty[slot], ((s / TC_SLOTS) & 1) ^ 1, &sh.poison, g_linear_status, WAIT_LIMIT_NS, 7, s);
                if (!ok) break;
                if (a.withhold && blockIdx.x == 0 && s == 0) continue;
                mbar_arrive_expect_tx(&sh.x_full[slot], S::XB);
                bulk_g2s(smem + S::CODES + slot * S::XB, a.xt + ((long long)pos.tile * R.stages + pos.u) * S::XB, S::XB, &sh.x_full[slot]);
            }
        }
        __syncwarp();
    } else {
        tc_mma_role<TOK, G>(a, R);
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (sh.poison) {
        // what the roles that gave up had begun: bulk copies into the ring, MMAs that read it and write tensor memory
        const unsigned long long t = globaltimer_ns();
        while (globaltimer_ns() - t < 2000000ull) {
        }
        __syncthreads();
    }
    if (warp == S::W_MMA) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(R.tm), "n"(TC_COLS) : "memory");
    }
}

// The blocks whose stages several CTAs took: their pieces added up in the order of the CTAs.  grid (block over all token tiles,
// four tokens); four rows a thread.
template <int TOK, typename TO>
__global__ void __launch_bounds__(256) linear_pieces_kernel(const __grid_constant__ LinearArgs a, int ctas, int stages, int blocks) {
    pdl_wait();
    const int block = blockIdx.x, first = block * stages;
    // the CTAs whose runs hold the block's first and last stage; a block other than a CTA's first is its last piece
    int c0 = (int)((long long)first * ctas / a.units);
    while (tc_first(c0 + 1, ctas, a.units) <= first) ++c0;
    if (tc_first(c0 + 1, ctas, a.units) >= first + stages) return;   // one CTA's: written by it
    int c1 = c0 + 1;
    while (tc_first(c1 + 1, ctas, a.units) < first + stages) ++c1;
    const int slot0 = tc_first(c0, ctas, a.units) >= first ? 0 : 1;
    const int t = 4 * blockIdx.y + (threadIdx.x >> 6), row = 4 * (threadIdx.x & 63);
    const int n = block % blocks * TC_ROWS + row, t0 = block / blocks * TOK;
    if (t0 + t >= a.T) return;
    const float* part = a.part + (long long)t * TC_ROWS + row;
    float4 v = *reinterpret_cast<const float4*>(part + (long long)(2 * c0 + slot0) * (TOK * TC_ROWS));
#pragma unroll 4
    for (int c = c0 + 1; c <= c1; ++c) {
        const float4 w = *reinterpret_cast<const float4*>(part + (long long)(2 * c) * (TOK * TC_ROWS));
        v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
    }
    store_y<TO>(a, t0 + t, n, v.x);
    store_y<TO>(a, t0 + t, n + 1, v.y);
    store_y<TO>(a, t0 + t, n + 2, v.z);
    store_y<TO>(a, t0 + t, n + 3, v.w);
}

// Shares of the input indices, a CTA of a cluster each: as many as leave the fewest units to the SM with most work.
static void split_units(LinearArgs& a, int units, long long blocks, int n_sms, int per_sm, int least, int start) {
    int best = 1;
    double best_cost = 1e30;
    for (int c = 1; c <= LIN_MAX_CLUSTER; ++c) {
        const int share = (units + c - 1) / c;
        if (c > 1 && share < least) break;
        const long long rounds = (blocks * c + (long long)n_sms * per_sm - 1) / ((long long)n_sms * per_sm);
        const double cost = (double)rounds * (share + start);
        if (cost < 0.95 * best_cost) best = c, best_cost = cost;
    }
    const int share = (units + best - 1) / best;
    a.units = share;
    a.n_split = (units + share - 1) / share;   // no empty shares
}

template <int NT, int R, int U, int G>
static cudaError_t linear_few(LinearArgs a, int y_f32, int n_sms, cudaStream_t st) {
    const unsigned blocks = (unsigned)((a.N + 16 * R - 1) / (16 * R)), tiles = (unsigned)((a.T + 8 * NT - 1) / (8 * NT));
    split_units(a, (a.K + LIN_UNIT - 1) / LIN_UNIT, (long long)blocks * tiles, n_sms, 2, LIN_WARPS, 12);
    const dim3 grid(blocks * a.n_split, tiles);
    return y_f32 ? launch_pdl_cluster(linear_few_kernel<NT, R, U, G, float>, grid, dim3(32 * LIN_WARPS), 0, a.n_split, st, a)
                 : launch_pdl_cluster(linear_few_kernel<NT, R, U, G, __nv_bfloat16>, grid, dim3(32 * LIN_WARPS), 0, a.n_split, st, a);
}
// Tokens of a tile of the tcgen05 kernel; 0: the call is the few-token kernel's.
// The few-token kernel reads the matrix once a tile of 16 tokens and its warps multiply each tile anew, but it is one launch with
// nothing to set up; the tcgen05 kernel has two launches beside it and the start of its pipeline, about 10 us, and then takes
// twice the codes in the same time.  So the rule is on the weights times the tiles of 16 (us, few-token against tcgen05):
//   2^20 2.9 / 10.1,  2^24 6.4 / 12.1 (64 tokens, 2048 x 2048),  2^25 10.6 / 15.8 (64, 2048 x 4096) and 10.9 / 14.8 (32, 4096 x 4096),
//   56 * 2^20 20.0 / 20.1 (16, 14336 x 4096),  2^26 18.8 / 20.8 (16, 8192 x 8192) and 21.1 / 17.0 (64, 4096 x 4096),
//   2^27 35.9 / 20.5 (128, 4096 x 4096),  196 * 2^20 57.4 / 42.2 (16, 14336 x 14336).
// (Up to 2^25 the tcgen05 kernel's figures are from before its operand was freed of the 16: 2 to 5% more now.)  Up to 8 tokens the few-token
// kernel has half of the MMAs: 41.4 us at 14336 x 14336, 40% of the copy rate, and the tcgen05 kernel is no faster there.
static int tc_tile(int T, int rows, int cols) {
    if (T <= 8 || (T + 15) / 16 * (long long)rows * cols <= 3ll << 24) return 0;
    return T <= 16 ? 16 : T <= 32 ? 32 : 64;
}
static size_t tc_x_bytes(int T, int cols, int G, int tok) {
    const size_t n = (size_t)((T + tok - 1) / tok) * ((cols + LIN_UNIT - 1) / LIN_UNIT) * (16 * 16 * tok + LIN_UNIT / G * tok * 4);
    return (n + 255) / 256 * 256;
}
static size_t tc_workspace(int T, int rows, int cols, int G) {
    const int tok = tc_tile(T, rows, cols);
    return tok ? tc_x_bytes(T, cols, G, tok) + (size_t)TC_MAX_CTAS * 2 * tok * TC_ROWS * 4 : 0;
}
template <int TOK, int G>
static cudaError_t linear_tc(LinearArgs a, int y_f32, int n_sms, cudaStream_t st) {
    constexpr int SMEM = TcShape<TOK, G>::SMEM;
    const int stages = (a.K + LIN_UNIT - 1) / LIN_UNIT, blocks = (a.N + TC_ROWS - 1) / TC_ROWS, tiles = (a.T + TOK - 1) / TOK;
    const long long warps = (long long)tiles * (TOK / 8) * stages, units = (long long)tiles * blocks * stages;
    a.part = reinterpret_cast<float*>(const_cast<uint8_t*>(a.xt) + tc_x_bytes(a.T, a.K, G, TOK));
    a.units = (int)units;
    cudaError_t e = launch_pdl(linear_x_kernel<TOK, G>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, st, a.x, a.T, a.K, stages, tiles,
                               const_cast<uint8_t*>(a.xt));
    if (e != cudaSuccess) return e;
    // a run of two stages at least
    const int ctas = (int)std::max(1ll, std::min({(long long)n_sms, (long long)TC_MAX_CTAS, units / 2}));
    auto go = [&](auto kernel, auto pieces) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
        if (e == cudaSuccess) e = launch_pdl(kernel, dim3((unsigned)ctas), dim3(32 * TcShape<TOK, G>::WARPS), SMEM, st, a);
        if (e == cudaSuccess) e = launch_pdl(pieces, dim3((unsigned)(blocks * tiles), TOK / 4), dim3(256), 0, st, a, ctas, stages, blocks);
        return e;
    };
    return y_f32 ? go(linear_tc_kernel<TOK, G, float>, linear_pieces_kernel<TOK, float>)
                 : go(linear_tc_kernel<TOK, G, __nv_bfloat16>, linear_pieces_kernel<TOK, __nv_bfloat16>);
}
template <int G>
static cudaError_t linear_by_tokens(const LinearArgs& a, int y_f32, int n_sms, cudaStream_t st) {
    switch (tc_tile(a.T, a.N, a.K)) {
        case 16: return linear_tc<16, G>(a, y_f32, n_sms, st);
        case 32: return linear_tc<32, G>(a, y_f32, n_sms, st);
        case 64: return linear_tc<64, G>(a, y_f32, n_sms, st);
    }
    if (a.T <= 8) return a.N >= 64 * n_sms ? linear_few<1, 2, 2, G>(a, y_f32, n_sms, st) : linear_few<1, 1, 4, G>(a, y_f32, n_sms, st);
    return linear_few<2, 2, 2, G>(a, y_f32, n_sms, st);
}

}  // namespace dyn

using namespace dyn;

namespace {

dynamo_status check_linear(int32_t rows, int32_t cols, int32_t group_size) {
    if (group_size != 64 && group_size != 128) return DYNAMO_ERR_SHAPE;
    if (rows < 1 || cols < group_size || cols % group_size || cols > 1 << 24 || rows > 1 << 24) return DYNAMO_ERR_SHAPE;   // (offsets of 32 bits)
    return DYNAMO_OK;
}

dynamo_status linear_impl(const void* x, int32_t T, int32_t rows, int32_t cols, int32_t group_size, const void* codes, const void* params,
                          void* y, int32_t y_dtype, void* workspace, size_t workspace_bytes, int withhold, void* stream) {
    if (const dynamo_status s = check_linear(rows, cols, group_size); s != DYNAMO_OK) return s;
    if (y_dtype != DYNAMO_BF16 && y_dtype != DYNAMO_F32) return DYNAMO_ERR_SHAPE;
    if (T < 0 || T > DYNAMO_LINEAR_MAX_TOKENS) return DYNAMO_ERR_TOKENS;
    if (T == 0) return DYNAMO_OK;
    if (!x || !codes || !params || !y) return DYNAMO_ERR_NULL;
    if (!aligned16(x, codes, params, y)) return DYNAMO_ERR_ALIGN;
    // (the tcgen05 kernel counts its stages, a tile of tokens by 256 rows by 128 columns each, in 32 bits)
    if ((long long)(T / 16 + 1) * (rows / 256 + 1) * (cols / 128 + 1) > 0x7fffffffll) return DYNAMO_ERR_TOKENS;
    const size_t need = tc_workspace(T, rows, cols, group_size);
    if (need && !workspace) return DYNAMO_ERR_NULL;
    if (workspace_bytes < need) return DYNAMO_ERR_ARENA_TOO_SMALL;
    if (need && ((uintptr_t)workspace & 255)) return DYNAMO_ERR_ALIGN;
    int n_sms = 0;
    if (count_sms(&n_sms) != cudaSuccess) return DYNAMO_ERR_CUDA;
    const LinearArgs a = {(const __nv_bfloat16*)x, (const uint8_t*)codes, (const uint32_t*)params, y, T, cols, rows,
                          {0x00780078u, 0x41804180u, 0x000f000fu, 0x43004300u}, (const uint8_t*)workspace, nullptr, 1, 0, withhold};
    const cudaError_t e = group_size == 64 ? linear_by_tokens<64>(a, y_dtype == DYNAMO_F32, n_sms, (cudaStream_t)stream)
                                           : linear_by_tokens<128>(a, y_dtype == DYNAMO_F32, n_sms, (cudaStream_t)stream);
    return e == cudaSuccess ? DYNAMO_OK : DYNAMO_ERR_CUDA;
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

dynamo_status dynamo_linear_workspace_bytes(int32_t T, int32_t rows, int32_t cols, int32_t group_size, size_t* bytes) {
    if (const dynamo_status s = check_linear(rows, cols, group_size); s != DYNAMO_OK) return s;
    if (!bytes) return DYNAMO_ERR_NULL;
    if (T < 0 || T > DYNAMO_LINEAR_MAX_TOKENS) return DYNAMO_ERR_TOKENS;
    *bytes = tc_workspace(T, rows, cols, group_size);
    return DYNAMO_OK;
}

dynamo_status dynamo_linear_poll_status(void* stream) {
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return DYNAMO_ERR_CUDA;
    int32_t word = 0;
    if (cudaMemcpyFromSymbol(&word, g_linear_status, 4) != cudaSuccess) return DYNAMO_ERR_CUDA;
    return word == 0 ? DYNAMO_OK : DYNAMO_ERR_TIMEOUT;   // (and it stays: other users of the device ask too)
}

dynamo_status dynamo_linear_clear_status(void* stream) {
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return DYNAMO_ERR_CUDA;
    const int32_t zero[16] = {};
    return cudaMemcpyToSymbol(g_linear_status, zero, sizeof(zero)) == cudaSuccess ? DYNAMO_OK : DYNAMO_ERR_CUDA;
}

dynamo_status dynamo_linear_forward(const void* x, int32_t T, int32_t rows, int32_t cols, int32_t group_size, const void* codes,
                                    const void* params, void* y, int32_t y_dtype, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    return linear_impl(x, T, rows, cols, group_size, codes, params, y, y_dtype, workspace, workspace_bytes, 0, stream);
}

dynamo_status dynamo_debug_expire_linear(const void* x, int32_t T, int32_t rows, int32_t cols, int32_t group_size, const void* codes,
                                         const void* params, void* y, int32_t y_dtype, void* workspace, size_t workspace_bytes,
                                         void* stream) {
    if (const dynamo_status s = check_linear(rows, cols, group_size); s != DYNAMO_OK) return s;
    if (T < 0 || T > DYNAMO_LINEAR_MAX_TOKENS) return DYNAMO_ERR_TOKENS;
    if (!tc_tile(T, rows, cols)) return DYNAMO_ERR_ARG;   // the few-token kernel waits for nothing
    return linear_impl(x, T, rows, cols, group_size, codes, params, y, y_dtype, workspace, workspace_bytes, 1, stream);
}

}  // extern "C"
