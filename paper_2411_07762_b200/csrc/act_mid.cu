// Activation step of 33 to a few hundred tokens in one launch without scratch memory (Sec. 4.2 smoothing, Sec. 5.1
// per-token round-to-nearest, Sec. 4.1 projection T = X~ L_A^T).
//
// At these sizes neither bytes nor products take long (101 x 8192: 2.5 MB, under 1 us of either); what bounds the step
// is its longest chain of dependent steps.  The codes need nothing of T and T nothing of the codes, so they are made
// by different CTAs of one grid, each with the shortest chain there is:
//  * a quantizing CTA takes whole rows into registers (quantize_rows): one round trip, a maximum, the codes;
//  * a projecting cluster takes 32 tokens x 32 rows of L_A, its CTAs' warps 64 columns of K at a time.  mma.sync m16n8k16:
//    an inner product does not care about the order of k, so a thread's k positions are the 8 columns that one 16-byte
//    load brings, the same for X and L_A, and neither goes through shared memory.  X is divided where the divisor is
//    not 1 (fp32), and the quotient multiplied as the sum of two fp16 numbers: rounded to one, 2 % of T's bf16 values came out a
//    step off, and in a feed-forward block a step of T moves codes of H (a few tokens' outputs by 2 %).  Code that runs once is bound by
//    the fetching of its instructions: pairs of columns are divided by a few (double-length reciprocals, and the second numbers by an mma of
//    eight columns), without divisors there is an instance of its own (96 x 8192, rank 128, 1 % of the columns / all of them divided / no divisors, us:
//    8.0 / 12.0 / 6.3; with a division and two mma of sixteen columns for each column 8.4 / 19.2 / 7.1).  The warps' sums meet in shared memory,
//    the CTAs' in distributed shared memory, both in a fixed order; the order depends on K alone, not on the number of tokens.
#include <type_traits>

#include "act_math.cuh"
#include "aser_common.cuh"
#include "sm100_ptx.cuh"

namespace aser {

namespace {

constexpr int kMThreads = 256, kMWarps = kMThreads / 32;
constexpr int kMTok = 32, kMRank = 32;              // tile of a projecting cluster
constexpr int kMAcc = kMTok * kMRank / 32;          // sums per thread

__device__ __forceinline__ void mid_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// (eight columns of k: a word of a token against a word of L_A)
__device__ __forceinline__ void mid_mma8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0) {
    asm volatile(
        "mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(b0));
}

// 32 columns of 32 tokens and of 32 rows of L_A, a thread's share: 8 columns of the tokens and rows g + 8 i.
template <bool DIV>
struct MidUnit {
    uint32_t x[4][4];
    uint4 l[4];
    unsigned tags = 0;                       // pairs of columns with a divisor

    __device__ __forceinline__ void load(const __half* xp, const __half* lp, const float* s, int K, int c, int t, const bool (&x_ok)[4], const bool (&l_ok)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = x_ok[i] ? *reinterpret_cast<const uint4*>(xp + 8 * i * K + c) : make_uint4(0, 0, 0, 0);
            x[i][0] = v.x; x[i][1] = v.y; x[i][2] = v.z; x[i][3] = v.w;
            l[i] = l_ok[i] ? __ldg(reinterpret_cast<const uint4*>(lp + 8 * i * K + c)) : make_uint4(0, 0, 0, 0);
        }
        if (DIV) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(s + c + t * 8)), b = __ldg(reinterpret_cast<const float4*>(s + c + t * 8) + 1);
            tags = (a.x != 1.f || a.y != 1.f ? 1u : 0u) | (a.z != 1.f || a.w != 1.f ? 2u : 0u) |
                   (b.x != 1.f || b.y != 1.f ? 4u : 0u) | (b.z != 1.f || b.w != 1.f ? 8u : 0u);
        }
    }
    // all: pairs where any lane has a divisor (the others divide by 1).
    __device__ __forceinline__ void multiply(float (&acc)[2][4][4], const float* sp, unsigned all) {
#pragma unroll
        for (int w = 0; DIV && w < 4; ++w) {
            if (!(all >> w & 1)) continue;
            const float2 d = __ldg(reinterpret_cast<const float2*>(sp) + w);         // (again: eight registers fewer all along)
            const Divisor d0 = divisor_parts(d.x), d1 = divisor_parts(d.y);
            const float2 first = make_float2(d0.first, d1.first), second = make_float2(d0.second, d1.second);
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                uint32_t lo[2];              // what fp16 leaves of the quotients
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t& word = x[2 * mt + i][w];
                    const float2 x2 = __half22float2(*reinterpret_cast<const __half2*>(&word));
                    const float2 q = __ffma2_rn(x2, first, __fmul2_rn(x2, second));
                    const __half2 hi = __hmin2(__hmax2(__floats2half2_rn(q.x, q.y), __float2half2_rn(-65504.f)), __float2half2_rn(65504.f));
                    const float2 h = __half22float2(hi);
                    const __half2 rest = __floats2half2_rn(q.x - h.x, q.y - h.y);
                    word = *reinterpret_cast<const uint32_t*>(&hi);
                    lo[i] = *reinterpret_cast<const uint32_t*>(&rest);
                }
#pragma unroll
                for (int nt = 0; nt < 4; ++nt)
                    mid_mma8(acc[mt][nt], lo[0], lo[1], w == 0 ? l[nt].x : w == 1 ? l[nt].y : w == 2 ? l[nt].z : l[nt].w);
            }
        }
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                mid_mma(acc[mt][nt], x[2 * mt][0], x[2 * mt + 1][0], x[2 * mt][1], x[2 * mt + 1][1], l[nt].x, l[nt].y);
                mid_mma(acc[mt][nt], x[2 * mt][2], x[2 * mt + 1][2], x[2 * mt][3], x[2 * mt + 1][3], l[nt].z, l[nt].w);
            }
    }
};

// Grid: t_tiles * CL projecting CTAs (clusters of CL along K), then the quantizing CTAs, R rows each.
// A sum (register 4 (4 mt + nt) + e of lane 4 g + t) is token 16 mt + g + 8 (e / 2), L_A row 8 nt + 2 t + e % 2.
// TH threads: 256, or 512 for rows that would fill a thread's registers; the projection takes eight warps of them either way.
// DIV: there are divisors.
template <bool DIV, int CPT, int R, int TH = kMThreads>
__global__ void __launch_bounds__(TH, 512 / TH)
quant_act_mid_kernel(const __half* __restrict__ X, const float* __restrict__ s, const __half* __restrict__ LA, int M, int K,
                     int r, int t_tiles, int CL, int8_t* __restrict__ Xq, float* __restrict__ a_scale,
                     __nv_bfloat16* __restrict__ T, int ldt, int lo_off, float qmax) {
    // As in the few-token kernel: the wait comes first, dependents may start once everything before this kernel is done.
    grid_dep_wait();
    grid_dep_launch();
    __shared__ union {
        RowsShared<R> rows;
        float red[kMWarps][kMAcc][32];
    } sh;
    __shared__ float part[kMAcc][32];
    if ((int)blockIdx.x >= t_tiles * CL) {
        const int row0 = ((int)blockIdx.x - t_tiles * CL) * R, nrows = M - row0 < R ? M - row0 : R;
        if (nrows > 0)
            quantize_rows<CPT, R>(X + (size_t)row0 * K, DIV ? s : nullptr, nrows, K, Xq + (size_t)row0 * K, a_scale + row0, qmax, sh.rows);
        return;         // clusters take one role or the other, so no peer waits for this CTA
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int tile = (int)blockIdx.x / CL, rank = (int)blockIdx.x % CL;
    const int j_tiles = (r + kMRank - 1) / kMRank, j0 = tile % j_tiles * kMRank, m0 = tile / j_tiles * kMTok;
    float acc[2][4][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[mt][nt][e] = 0.f;
    const __half* const xp = X + (size_t)(m0 + g) * K + t * 8;
    const __half* const lp = LA + (size_t)(j0 + g) * K + t * 8;
    bool x_ok[4], l_ok[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {           // token rows g + 8 i, L_A rows g + 8 i
        x_ok[i] = m0 + g + 8 * i < M;
        l_ok[i] = j0 + g + 8 * i < r;
    }
    for (int u = warp < kMWarps ? rank * kMWarps + warp : K; u < K / 64; u += CL * kMWarps) {
        MidUnit<DIV> now, next;
        now.load(xp, lp, s, K, u * 64, t, x_ok, l_ok);
        next.load(xp, lp, s, K, u * 64 + 32, t, x_ok, l_ok);
        const unsigned all = DIV ? __reduce_or_sync(0xffffffffu, now.tags | next.tags << 4) : 0u;
        now.multiply(acc, s + u * 64 + t * 8, all);
        next.multiply(acc, s + u * 64 + 32 + t * 8, all >> 4);
    }
    if (warp < kMWarps) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) sh.red[warp][(mt * 4 + nt) * 4 + e][lane] = acc[mt][nt][e];
    }
    __syncthreads();
    for (int i = tid; i < kMAcc * 32; i += TH) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kMWarps; ++w) v += sh.red[w][i >> 5][i & 31];
        part[i >> 5][i & 31] = v;
    }
    if (CL > 1) { cluster_arrive(); cluster_wait(); }
    else __syncthreads();
    const int per = kMAcc * 32 / CL;        // sums that this CTA finishes
    const uint32_t mine = smem_u32(&part[0][0]);
    for (int i = rank * per + tid; i < (rank + 1) * per; i += TH) {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = q < CL ? (CL > 1 ? ld_cluster_f32(map_to_rank(mine + 4u * i, q)) : part[i >> 5][i & 31]) : 0.f;
        float sum = v[0];
#pragma unroll
        for (int q = 1; q < 8; ++q) sum += v[q];
        const int reg = i >> 5, ln = i & 31;
        const int m = m0 + (reg >> 4) * 16 + (ln >> 2) + 8 * ((reg >> 1) & 1), j = j0 + ((reg >> 2) & 3) * 8 + (ln & 3) * 2 + (reg & 1);
        if (m < M && j < r) store_t(T + (size_t)m * ldt, j, sum, lo_off);
    }
    if (CL > 1) { cluster_arrive(); cluster_wait(); }       // nobody leaves while a peer may still read its sums
}

// CTAs of a projecting cluster: 64 columns for every warp, where K has them.
int mid_cluster(int K) { return K >= 4096 ? 8 : K >= 2048 ? 4 : K >= 1024 ? 2 : 1; }

template <typename Kernel>
int launch_mid_cfg(Kernel* kernel, int threads, int R, const __half* X, const float* s, const __half* LA, int M, int K, int r, int8_t* Xq,
                   float* a_scale, __nv_bfloat16* T, int ldt, int lo_off, float qmax, cudaStream_t st) {
    const int CL = mid_cluster(K);
    const int t_tiles = (M + kMTok - 1) / kMTok * ((r + kMRank - 1) / kMRank), rows = (M + R - 1) / R;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(t_tiles * CL + (rows + CL - 1) / CL * CL, 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CL; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, X, s, LA, M, K, r, t_tiles, CL, Xq, a_scale, T,
                                             ldt, lo_off, qmax);
    if (e != cudaSuccess) return record_cuda_error(e, "quant_act_mid_kernel");
    return check_launch("quant_act_mid_kernel");
}

}  // namespace

namespace {
// Rows of a quantizing CTA: one while the rows are few (the shortest chain), more where they would be several waves of CTAs
// (1000 x 1024, rank 32, us with one / two / four: 9.8 / 8.3 / 7.2; 333 x 8192: 11.7 / 9.0), as far as registers go.
int mid_rows(int M, int K) { return K > 8192 || M <= 128 ? 1 : M > 512 && K <= 2048 ? 4 : 2; }
}  // namespace

// The CTAs of this kernel are short and two are resident on an SM; the cluster kernel's step hardly depends on the
// number of tokens until its clusters no longer fit at once.  Measured with 1 % of the columns divided, this kernel (its CTAs) | the cluster kernel, us:
// rank 32: 64 x 4096 (80) 4.4 | 9.9, 448 x 4096 (336) 9.4 | 10.8, 101 x 8192 (133) 7.2 | 13.0, 333 x 8192 (255) 9.4 | 13.7, 448 x 8192 (336) 14.1 |
// 13.6, 333 x 14336 (421) 17.6 | 18.2; rank 64: 64 x 4096 (96) 4.5 | 10.1, 333 x 4096 (343) 9.8 | 11.2, 384 x 4096 (384) 10.9 | 10.8, 350 x 5120 (351)
// 12.6 | 18.4; rank 128: 200 x 4096 (324) 10.2 | 11.3, 333 x 4096 (519) 11.4 | 11.5, 200 x 8192 (324) 14.7 | 16.5, 333 x 8192 (519) 16.8 | 16.7,
// 200 x 14336 (424) 20.2 | 22.8; short rows: 1000 x 1024, rank 128 (506, four rows each) 10.8 | 10.7, rank 32 (314) 7.9 | 9.9, 448 x 2048,
// rank 128 (448) 9.4 | 9.8, 1000 x 2560, rank 32 (628) 12.6 | 15.6, rank 128 (1012) 17.2 | 17.1.
// two_kernels: the alternative is the step of two kernels, as in a forward pass.  Between 341 and 400 CTAs at 4096 to 5120 columns it is then faster at
// high ranks and without a projection, where rows do not have 4096 columns (105 points; a pass, this kernel | two kernels, us: 4608 columns:
// 225 tokens, rank 128, 25.1 | 22.7, 449, rank 16, 24.5 | 25.8, 681 without 31.3 | 28.4; 5120: 256, rank 128, 26.3 | 23.6, 343, rank 64, 26.1 | 26.5, 700
// without 33.2 | 30.4; 4096: 225, rank 128, 22.1 | 23.2, 343, rank 64, 22.3 | 23.6, 771 without 29.0 | 28.3).
bool quant_act_mid_prefers(int M, int K, int r, bool two_kernels) {
    const int rows = mid_rows(M, K);
    const int ctas = (M + rows - 1) / rows + mid_cluster(K) * ((M + kMTok - 1) / kMTok) * ((r + kMRank - 1) / kMRank);
    const bool high = two_kernels && (r == 0 || (r > 64 && K > 4096));
    return ctas <= (rows == 4 ? 450 : K < 4096 ? 630 : K <= 5120 && !high ? 400 : K <= 8192 ? 340 : 424);
}

int launch_quant_act_mid(const __half* X, const float* s, const __half* LA, int M, int K, int r, int8_t* Xq, float* a_scale,
                         __nv_bfloat16* T, int ldt, int lo_off, float qmax, cudaStream_t st) {
    // chunks of eight columns per thread by the row length, one, two or four rows per quantizing CTA
    const int chunks = (K / 8 + kMThreads - 1) / kMThreads, rows = mid_rows(M, K);
    auto go = [&](auto* kernel, int threads = kMThreads) { return launch_mid_cfg(kernel, threads, rows, X, s, LA, M, K, r, Xq, a_scale, T, ldt, lo_off, qmax, st); };
    auto pick = [&](auto div) {
        constexpr bool DIV = decltype(div)::value;
        if (rows == 4) return go(quant_act_mid_kernel<DIV, 1, 4>);        // up to 2048 columns
        if (chunks <= 1) return rows == 2 ? go(quant_act_mid_kernel<DIV, 1, 2>) : go(quant_act_mid_kernel<DIV, 1, 1>);
        if (chunks <= 2) return rows == 2 ? go(quant_act_mid_kernel<DIV, 2, 2>) : go(quant_act_mid_kernel<DIV, 2, 1>);
        if (chunks <= 4) return rows == 2 ? go(quant_act_mid_kernel<DIV, 4, 2>) : go(quant_act_mid_kernel<DIV, 4, 1>);
        if (chunks <= 8) return go(quant_act_mid_kernel<DIV, 8, 1>);
        return go(quant_act_mid_kernel<DIV, 8, 1, 512>, 512);
    };
    return s ? pick(std::true_type()) : pick(std::false_type());
}

}  // namespace aser
