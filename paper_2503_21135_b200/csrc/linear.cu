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
#include "f32x2.cuh"
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

// ---- tcgen05: the codes as the A operand in tensor memory -------------------------------------------------------------------
// CTA: 128 rows, TOK tokens, a share of the groups; eight warps that all do the same.  Warp w has the lane quarter q = w % 4 of the
// tensor memory: rows 32 q .., of which it expands 16 and folds all, half of the tokens (h = w / 4 says which).
// A stage is one group:
//   fill    codes of 16 rows -> 16 + q as bf16 pairs -> tensor memory (A, G / 2 columns; 16x256b, so that four lanes read a row's codes:
//           a row a lane kept the L1 busy with 32 lines a load); the activations -> shared memory (B, K-major core matrices of 8 tokens x
//           8 indices), in the order that this gives the indices, their sums by an mma.sync whose other operand is ones, from the
//           registers that they came in; parameters of eight groups at a time -> shared memory
//   MMAs    G / 16 tcgen05.mma of 128 x TOK x 16 into one of two accumulators, issued by one warp in one run, committed to a barrier
//   fold    y += s * acc + (m - 16 s) * sum(x), two columns an instruction
// Stage i + 1 is filled and its MMAs issued before stage i is folded: one barrier a stage, and the MMAs run under the next
// stage's filling.  Two CTAs share an SM (each 256 columns of tensor memory at most, 128 registers a thread).
// A poll of the MMAs' barrier is bounded; after an expired one the CTA's outputs are NaN and the status word is set.  The tensor
// memory is given back before the CTAs of a cluster meet: nobody waits for another CTA while it holds some.
constexpr int TC_ROWS = 128;
static __device__ int32_t g_linear_status[16];

template <int TOK, int G>
struct TcShape {
    static constexpr int OCTETS = TOK / 8, QUADS = G / 32;                       // eight tokens, 32 indices: a warp's task of the filling
    static constexpr int TPW = OCTETS * QUADS < LIN_WARPS ? 1 : OCTETS * QUADS / LIN_WARPS;
    static constexpr int SPLITS = QUADS / TPW;                                   // warps that share an octet: partial sums
    static constexpr int LBO = TOK * 16 + 16;   // bytes between octets of indices; the pad keeps the filling's stores off one another's banks
    static constexpr int XBUF = G / 8 * LBO;
    static constexpr int W = G / 32;                                             // words of codes of a lane and row: a quarter of a group
    static constexpr int A_COLS = G / 2, COLS = 2 * A_COLS + 2 * TOK <= 64 ? 64 : 2 * A_COLS + 2 * TOK <= 128 ? 128 : 256;
    static constexpr int SMEM = 2 * XBUF > TOK * TC_ROWS * 4 ? 2 * XBUF : TOK * TC_ROWS * 4;
    static_assert(2 * A_COLS + 2 * TOK <= COLS, "tensor memory");
};

// The MMAs of a stage: G / 16 steps of 16 indices, A columns 8 k, B octets 2 k.  The first starts from zero.
#define LIN_MMA(k, acc)                                                  \
    "add.s64 bd, %2, " #k "*%4;\n\tadd.s32 aa, %1, " #k "*8;\n\t"        \
    "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [aa], bd, %3, " acc ";\n\t"
template <int G, int STEP>
__device__ __forceinline__ void linear_mmas(uint32_t d, uint32_t a, uint64_t bd, uint32_t idesc, uint32_t bar) {
    if constexpr (G == 128)
        asm volatile(
            "{\n\t.reg .pred q, p0, p1;\n\t.reg .b64 bd;\n\t.reg .b32 aa;\n\telect.sync _|q, 0xffffffff;\n\t"
            "setp.ne.b32 p0, 0, 0;\n\tsetp.eq.b32 p1, 0, 0;\n\t" LIN_MMA(0, "p0") LIN_MMA(1, "p1") LIN_MMA(2, "p1") LIN_MMA(3, "p1")
                LIN_MMA(4, "p1") LIN_MMA(5, "p1") LIN_MMA(6, "p1") LIN_MMA(7, "p1")
            "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t}" ::"r"(d), "r"(a), "l"(bd), "r"(idesc),
            "n"(STEP), "r"(bar)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q, p0, p1;\n\t.reg .b64 bd;\n\t.reg .b32 aa;\n\telect.sync _|q, 0xffffffff;\n\t"
            "setp.ne.b32 p0, 0, 0;\n\tsetp.eq.b32 p1, 0, 0;\n\t" LIN_MMA(0, "p0") LIN_MMA(1, "p1") LIN_MMA(2, "p1") LIN_MMA(3, "p1")
            "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t}" ::"r"(d), "r"(a), "l"(bd), "r"(idesc),
            "n"(STEP), "r"(bar)
            : "memory");
}
__device__ __forceinline__ void cp_async4(void* dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
// Eight consecutive columns of the warp's 32 lanes, a row a lane.
__device__ __forceinline__ void tc_ld_rows8(uint32_t at, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(at)
                 : "memory");
}

template <int TOK, int G, typename TO>
__global__ void __launch_bounds__(32 * LIN_WARPS, 2) linear_tc_kernel(const __grid_constant__ LinearArgs a) {
    using S = TcShape<TOK, G>;
    constexpr int THREADS = 32 * LIN_WARPS, NC = TOK / 2, W = S::W;   // NC: columns that a warp folds
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float sums[3][S::SPLITS][TOK];
    __shared__ uint32_t params[2][8][TC_ROWS];   // of eight groups, and of the next eight
    __shared__ uint64_t bars[2];
    __shared__ uint32_t tmem_at;
    __shared__ int poison;
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, h = warp >> 2;
    const int split = blockIdx.x % a.n_split, n0 = blockIdx.x / a.n_split * TC_ROWS, t0 = blockIdx.y * TOK;
    const int groups = a.K / G, g0 = split * a.units, n = min(groups, g0 + a.units) - g0;
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_at)), "n"(S::COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) {
        mbar_init(&bars[0], 1);
        mbar_init(&bars[1], 1);
        poison = 0;
        fence_barrier_init();
    }
    // rows gid and gid + 8 of the 16 that the warp expands, and what the thread brings in of the activations: token tok, chunks
    // 4 i + tid4 of i in [i0, i0 + TPW)
    const int gid = lane >> 2, tid4 = lane & 3;
    const uint8_t* codes[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
        codes[e] = a.codes + (long long)min(n0 + 32 * q + 16 * h + gid + 8 * e, a.N - 1) * (a.K / 2) + (long long)g0 * (G / 2) + tid4 * (4 * W);
    const int oct = warp % S::OCTETS, i0 = warp / S::OCTETS * S::TPW, tok = 8 * oct + gid;
    const bool brings = warp / S::OCTETS < S::SPLITS;
    const uint4* xs = reinterpret_cast<const uint4*>(a.x + (long long)min(t0 + tok, a.T - 1) * a.K + (long long)g0 * G) + 4 * i0 + tid4;
    uint32_t cw[2][2][W];
    uint4 xv[S::TPW];
    auto load_codes = [&](uint32_t (&c)[2][W], int i) {
        if (i >= n) return;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if constexpr (W == 4) {
                const uint4 v = __ldcs(reinterpret_cast<const uint4*>(codes[e] + i * (G / 2)));
                c[e][0] = v.x, c[e][1] = v.y, c[e][2] = v.z, c[e][3] = v.w;
            } else {
                const uint2 v = __ldcs(reinterpret_cast<const uint2*>(codes[e] + i * (G / 2)));
                c[e][0] = v.x, c[e][1] = v.y;
            }
        }
    };
    // parameters of groups 8 c .. 8 c + 7: eight lanes a row
    auto bring_params = [&](int c) {
#pragma unroll
        for (int u = 0; u < 8 * TC_ROWS / THREADS; ++u) {
            const int r = (tid >> 3) + u * (THREADS / 8), g = 8 * c + (tid & 7);
            if (g < n) cp_async4(&params[c & 1][tid & 7][r], a.params + (long long)min(n0 + r, a.N - 1) * groups + g0 + g);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto load_x = [&](int i) {
        if (i >= n || !brings) return;
#pragma unroll
        for (int j = 0; j < S::TPW; ++j) xv[j] = __ldg(xs + i * (G / 8) + 4 * j);
    };
    bring_params(0);
    load_codes(cw[0], 0);
    load_x(0);
    load_codes(cw[1], 1);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tmem_at;
    const uint32_t lanes = (uint32_t)(32 * q) << 16;
    F2 acc[NC / 2];
#pragma unroll
    for (int c = 0; c < NC / 2; ++c) acc[c] = f2(0.f);
    bool dead = false;

    auto fill = [&](int i, int b) {   // stage i into buffers b; the MMAs that read them last are complete
        if (brings) {
            float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < S::TPW; ++j) {
                mma_bf16(s4, BF16_ONES, BF16_ONES, BF16_ONES, BF16_ONES, xv[j].x, xv[j].y);
                mma_bf16(s4, BF16_ONES, BF16_ONES, BF16_ONES, BF16_ONES, xv[j].z, xv[j].w);
                // chunk (t, wd): the indices 8 (W t + wd) .. of the group, a lane t's word wd of the codes.  The 16x256b store gives
                // the lane's pairs 2 j, 2 j + 1 the columns 8 j + 2 t, + 1, half t & 1 of the octet 2 j + (t >> 1).
                uint32_t p[4];
                b_operands(p, xv[j]);
                const int c = 4 * (i0 + j) + tid4, t = c / W, wd = c % W;
                const uint32_t at = smem_u32(smem) + b * S::XBUF + (4 * wd + (t >> 1)) * S::LBO + tok * 16 + 8 * (t & 1);
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(p[0]), "r"(p[1]) : "memory");
                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at + 2 * S::LBO), "r"(p[2]), "r"(p[3]) : "memory");
            }
            if (lane < 4) *reinterpret_cast<float2*>(&sums[i % 3][warp / S::OCTETS][8 * oct + 2 * lane]) = make_float2(s4[0], s4[1]);
        }
        load_x(i + 1);
        uint32_t r[8 * W];
#pragma unroll
        for (int j = 0; j < 2 * W; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t w = cw[b][e][j >> 1];
                r[4 * j + 2 * e] = j & 1 ? code_pair<2>(w, a.bits) : code_pair<0>(w, a.bits);
                r[4 * j + 2 * e + 1] = j & 1 ? code_pair<3>(w, a.bits) : code_pair<1>(w, a.bits);
            }
        if constexpr (W == 4) tc_st_x8(tm + ((uint32_t)(32 * q + 16 * h) << 16) + b * S::A_COLS, r);
        else tc_st_x4(tm + ((uint32_t)(32 * q + 16 * h) << 16) + b * S::A_COLS, r);
        load_codes(cw[b], i + 2);
        tc_wait_st();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the activations' stores, before the MMAs read them
        tc_fence_before();
    };
    auto issue = [&](int b) {
        tc_fence_after();
        const uint64_t bd = tc_desc(smem_u32(smem) + b * S::XBUF, S::LBO, 128);
        constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TOK / 8) << 17) | ((128u / 16) << 24);
        linear_mmas<G, 2 * S::LBO / 16>(__shfl_sync(0xffffffffu, tm + 2 * S::A_COLS + b * TOK, 0), __shfl_sync(0xffffffffu, tm + b * S::A_COLS, 0),
                                        bd, idesc, smem_u32(&bars[b]));
    };
    auto fold = [&](int i, int b) {
        if (!dead) dead = !warp_wait(smem_u32(&bars[b]), (i >> 1) & 1, &poison, g_linear_status, 1, i);
        tc_fence_after();
        const uint32_t from = tm + lanes + 2 * S::A_COLS + b * TOK + h * NC;
        uint32_t r[NC];
#pragma unroll
        for (int c = 0; c < NC; c += 8) tc_ld_rows8(from + c, r + c);
        const uint32_t pw = params[(i >> 3) & 1][i & 7][32 * q + lane];
        const __half2 pv = *reinterpret_cast<const __half2*>(&pw);
        const float s1 = __low2float(pv);
        const F2 s2 = f2(s1), m2 = f2(fmaf(-16.f, s1, __high2float(pv)));
#pragma unroll
        for (int c = 0; c < NC; c += 4)
#pragma unroll
            for (int sp = 0; sp < S::SPLITS; ++sp) {
                const float4 v = *reinterpret_cast<const float4*>(&sums[i % 3][sp][h * NC + c]);
                acc[c / 2] = fma2(m2, f2(v.x, v.y), acc[c / 2]);
                acc[c / 2 + 1] = fma2(m2, f2(v.z, v.w), acc[c / 2 + 1]);
            }
        tc_wait_ld();
#pragma unroll
        for (int c = 0; c < NC; c += 8)   // (what is read of them stays behind the wait)
            asm volatile("" : "+r"(r[c]), "+r"(r[c + 1]), "+r"(r[c + 2]), "+r"(r[c + 3]), "+r"(r[c + 4]), "+r"(r[c + 5]), "+r"(r[c + 6]), "+r"(r[c + 7]));
#pragma unroll
        for (int c = 0; c < NC; c += 2) acc[c / 2] = fma2(s2, f2(__uint_as_float(r[c]), __uint_as_float(r[c + 1])), acc[c / 2]);
        tc_fence_before();
    };
    fill(0, 0);
    __syncthreads();
    if (warp == 0) issue(0);
    for (int i = 0; i < n; i += 2) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (i + b >= n) break;
            // the next eight groups' parameters: asked for at the second stage of eight (every warp has folded the eight before, whose
            // place they take), there at the last
            if (((i + b) & 7) == 1 && (((i + b) >> 3) + 1) * 8 < n) bring_params(((i + b) >> 3) + 1);
            if (i + b + 1 < n) {
                fill(i + b + 1, b ^ 1);
                if (((i + b) & 7) == 7) asm volatile("cp.async.wait_group 0;" ::: "memory");
                __syncthreads();   // stage i + b + 1 is filled, stage i + b - 1 folded by every warp
                if (warp == 0) issue(b ^ 1);
            }
            fold(i + b, b);
        }
    }
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tm), "n"(S::COLS) : "memory");
    }
    // results to shared memory, [token][row], then out in whole rows of a token
    const bool bad = *(volatile int*)&poison;
    float* part = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int c = 0; c < NC; ++c)
        part[(h * NC + c) * TC_ROWS + 32 * q + lane] = bad ? __int_as_float(0x7fffffff) : (c & 1 ? hi(acc[c / 2]) : lo(acc[c / 2]));
    if (a.n_split == 1) {
        __syncthreads();
        for (int o = tid; o < TOK * TC_ROWS; o += THREADS) store_y<TO>(a, t0 + o / TC_ROWS, n0 + o % TC_ROWS, part[o]);
        return;
    }
    cluster_sync_all();
    for (int o = split * THREADS + tid; o < TOK * TC_ROWS; o += a.n_split * THREADS)
        store_y<TO>(a, t0 + o / TC_ROWS, n0 + o % TC_ROWS, cluster_sum(part, o, a.n_split));
    cluster_sync_all();
}

// Shares of the input indices, a CTA of a cluster each: as many as leave the fewest units to the SM with most work.
#ifndef LIN_OVER
#define LIN_OVER 12
#endif
#ifndef LIN_FEW
#define LIN_FEW 16
#endif
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
template <int TOK, int G>
static cudaError_t linear_tc(LinearArgs a, int y_f32, int n_sms, cudaStream_t st) {
    constexpr int SMEM = TcShape<TOK, G>::SMEM;
    const unsigned blocks = (unsigned)((a.N + TC_ROWS - 1) / TC_ROWS), tiles = (unsigned)((a.T + TOK - 1) / TOK);
    split_units(a, a.K / G, (long long)blocks * tiles, n_sms, 2, 4, LIN_OVER);
    const dim3 grid(blocks * a.n_split, tiles);
    auto go = [&](auto kernel) { return launch_pdl_cluster(kernel, grid, dim3(32 * LIN_WARPS), SMEM, a.n_split, st, a); };
    return y_f32 ? go(linear_tc_kernel<TOK, G, float>) : go(linear_tc_kernel<TOK, G, __nv_bfloat16>);
}
template <int G>
static cudaError_t linear_by_tokens(const LinearArgs& a, int y_f32, int n_sms, cudaStream_t st) {
    if (a.T <= LIN_FEW && a.T <= 8) return a.N >= 64 * n_sms ? linear_few<1, 2, 2, G>(a, y_f32, n_sms, st) : linear_few<1, 1, 4, G>(a, y_f32, n_sms, st);
    if (a.T <= LIN_FEW) return linear_few<2, 2, 2, G>(a, y_f32, n_sms, st);
    if (a.T <= 16) return linear_tc<16, G>(a, y_f32, n_sms, st);
    if (a.T <= 32) return linear_tc<32, G>(a, y_f32, n_sms, st);
    return linear_tc<64, G>(a, y_f32, n_sms, st);
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

dynamo_status dynamo_linear_poll_status(void* stream) {
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return DYNAMO_ERR_CUDA;
    int32_t word = 0;
    if (cudaMemcpyFromSymbol(&word, g_linear_status, 4) != cudaSuccess) return DYNAMO_ERR_CUDA;
    if (word == 0) return DYNAMO_OK;
    const int32_t zero[16] = {};
    if (cudaMemcpyToSymbol(g_linear_status, zero, sizeof(zero)) != cudaSuccess) return DYNAMO_ERR_CUDA;
    return DYNAMO_ERR_TIMEOUT;
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
