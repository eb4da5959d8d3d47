// Low-rank adapters of many requests beside a shared projection:
//   out[m, :] = fp16( Y[m, :] + scale[a] * B_a (A_a x[m]) ),   a = the adapter of token m, or none.
//
// Two products with a small intermediate, S = A_a x (r numbers per token) and B_a S.  The bytes are those of the adapters in
// use (2 r (K + N) each), X, and Y twice; a token's 2 r (K + N) multiply-adds come to at most r of them per byte of X and Y, so
// at the ranks of adapters the tensor cores' older instruction (mma.sync m16n8k16) keeps up with HBM and its operands can
// go straight from global memory into registers.  What is left to arrange:
//  * tokens of one adapter have to meet, wherever they stand in the batch: a plan (adapters_plan_kernel), made once per batch
//    and used by all layers of a step, lists the tokens by adapter and cuts each adapter's into tiles;
//  * one launch: a tile belongs to a cluster of CTAs, which split K for the first product and N for the second.  The partial
//    sums of S meet in distributed shared memory (in a fixed order; nothing depends on the order of tokens in a tile);
//  * an inner product does not care about the order of k, so a thread's k positions are the 8 columns of one 16-byte load, the
//    same for both operands; likewise the 32 rows of B that a warp takes are dealt so that a thread's outputs are 8 neighbours.
// S is summed and exchanged in fp32.  For the second product it is rounded to fp16 (2^-11 of each number, where the output
// has 2^-11 of the whole sum) after a scaling by a power of two that brings the token's largest entry to [2^14, 2^15): exact,
// and no size of activations or adapters overflows.
#include "adapters.cuh"
#include "sm100_ptx.cuh"

namespace aser {

namespace {

constexpr int kAThreads = 256, kAWarps = kAThreads / 32;
constexpr int kChunk = 64;                  // ranks of S summed at a time
constexpr int kRedStride = kChunk + 8;      // floats: rows 8 banks apart
constexpr int kPlanThreads = 1024;

// Bytes between the fp16 rows of S: an odd multiple of 64, so that 16-byte reads of two rows do not meet in a bank.
__host__ __device__ constexpr int s_stride(int r) { return (2 * r + 63) / 128 * 128 + 64; }

struct AdapterParams {
    const __half* X;
    const __half* A;          // [slots, r, K]
    const __half* B;          // [slots, N, r]
    const int32_t* ranks;     // [slots] or NULL
    const float* scale;       // [slots] or NULL
    const int32_t* plan;
    const __half* Y;
    __half* out;
    size_t ldx, ldy, ldo;
    int M, N, K, r, n_slots;
    int parts;                // clusters per tile, each with its own part of N
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void st_cluster_u2(uint32_t addr, uint32_t a, uint32_t b) {
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void st_cluster_f32(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

// A tile of up to 16 MT TW tokens of one adapter: TW groups of warps along the tokens, KW = 8 / TW along K and along N.
template <int MT, int TW>
__global__ void __launch_bounds__(kAThreads, 2)
adapters_kernel(const AdapterParams p) {
    constexpr int TM = 16 * MT * TW, KW = kAWarps / TW;
    grid_dep_wait();
    grid_dep_launch();
    extern __shared__ __align__(16) uint8_t smem[];
    const uint32_t CL = cluster_size(), rank = cluster_rank();
    const int tile = (int)(blockIdx.x / (CL * p.parts)), part = (int)(blockIdx.x / CL % p.parts);
    const PlanView plan = plan_view(p.plan, p.M, p.n_slots);
    const int4 head = *reinterpret_cast<const int4*>(p.plan);
    if (head.x != p.M || head.y != p.n_slots || tile >= (TM == 16 ? head.z : head.w)) return;
    const int4 t4 = (TM == 16 ? plan.tiles_few : plan.tiles_many)[tile];
    const int slot = t4.x, count = t4.z;
    const int32_t* tokens = plan.tokens + t4.y;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int tw = warp % TW, kw = warp / TW;
    int rk = 0;
    if (slot >= 0) {
        rk = p.ranks ? __ldg(p.ranks + slot) : p.r;
        rk = (rk < 0 ? 0 : rk > p.r ? p.r : rk) & ~15;
    }
    const int n_units = (p.N + 31) / 32, n_step = p.parts * (int)CL * KW, n_first = (part * (int)CL + (int)rank) * KW + kw;
    size_t tok[2 * MT];
    bool ok[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
        const int row = tw * 16 * MT + 8 * i + g;
        ok[i] = row < count;
        tok[i] = ok[i] ? (size_t)tokens[row] : 0;
    }
    if (rk == 0) {              // nothing to add (the whole cluster takes this way)
        if (p.Y != p.out)
            for (int u = n_first; u < n_units; u += n_step)
#pragma unroll
                for (int i = 0; i < 2 * MT; ++i) {
                    const int n = u * 32 + 8 * t;
                    if (ok[i] && n < p.N)
                        *reinterpret_cast<uint4*>(p.out + tok[i] * p.ldo + n) = *reinterpret_cast<const uint4*>(p.Y + tok[i] * p.ldy + n);
                }
        return;
    }
    float* red = reinterpret_cast<float*>(smem);                             // [KW][TM][kRedStride]
    float* sums = red + KW * TM * kRedStride;                                // [TM][r]
    uint8_t* s16 = reinterpret_cast<uint8_t*>(sums + TM * p.r);              // [TM][s_stride(r)]
    float* row_scale = reinterpret_cast<float*>(s16 + TM * s_stride(p.r));   // [TM]

    // ---- S = A x: this CTA's part of K, the warps' parts of it ----
    const __half* A = p.A + (size_t)slot * p.r * p.K + 8 * t;
    const __half* xp[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) xp[i] = p.X + tok[i] * p.ldx + 8 * t;
    for (int r0 = 0; r0 < rk; r0 += kChunk) {
        float acc[MT][8][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[mt][nt][e] = 0.f;
        const __half* ap = A + (size_t)(r0 + g) * p.K;
        const int n_tiles = (rk - r0) / 8;
        for (int u = (int)rank * KW + kw; u < p.K / 32; u += (int)CL * KW) {
            uint4 x[2 * MT], l[8];
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) x[i] = ok[i] ? *reinterpret_cast<const uint4*>(xp[i] + u * 32) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int nt = 0; nt < 8; ++nt)
                if (nt < n_tiles) l[nt] = __ldg(reinterpret_cast<const uint4*>(ap + (size_t)nt * 8 * p.K + u * 32));
#pragma unroll
            for (int nt = 0; nt < 8; ++nt) {
                if (nt >= n_tiles) break;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    mma16816(acc[mt][nt], x[2 * mt].x, x[2 * mt + 1].x, x[2 * mt].y, x[2 * mt + 1].y, l[nt].x, l[nt].y);
                    mma16816(acc[mt][nt], x[2 * mt].z, x[2 * mt + 1].z, x[2 * mt].w, x[2 * mt + 1].w, l[nt].z, l[nt].w);
                }
            }
        }
        if (r0 > 0) __syncthreads();            // the chunk before has been summed
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float* q = red + (size_t)(kw * TM + (tw * MT + mt) * 16 + 8 * h + g) * kRedStride + nt * 8 + 2 * t;
                    if (nt < n_tiles) *reinterpret_cast<float2*>(q) = make_float2(acc[mt][nt][2 * h], acc[mt][nt][2 * h + 1]);
                }
        __syncthreads();
        const int per_row = (n_tiles < 8 ? n_tiles : 8) * 2;        // groups of four sums
        for (int i = threadIdx.x; i < count * per_row; i += kAThreads) {
            const int row = i / per_row, j = i % per_row * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float4 a = *reinterpret_cast<const float4*>(red + (size_t)(w * TM + row) * kRedStride + j);
                v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
            }
            *reinterpret_cast<float4*>(sums + row * p.r + r0 + j) = v;
        }
    }

    // the first rows of B are fetched while the cluster meets
    const __half* B = p.B + (size_t)slot * p.N * p.r;
    uint4 b[4][2];
    auto fetch = [&](int u, int r0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = u * 32 + (g >> 1) * 8 + 2 * j + (g & 1);
            const __half* row = B + (size_t)n * p.r + r0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                b[j][h] = make_uint4(0, 0, 0, 0);
                if (n >= p.N) continue;
                if (r0 + 32 * h + 32 <= rk) b[j][h] = __ldg(reinterpret_cast<const uint4*>(row + 32 * h + 8 * t));
                else if (r0 + 32 * h < rk) {            // the last 16 ranks
                    const uint2 v = __ldg(reinterpret_cast<const uint2*>(row + 32 * h + 4 * t));
                    b[j][h].x = v.x; b[j][h].y = v.y;
                }
            }
        }
    };
    if (n_first < n_units) fetch(n_first, 0);

    // ---- every CTA sums some tokens over the cluster, rounds them, and sends them to all ----
    cluster_arrive();
    cluster_wait();
    {
        const int per = (TM + (int)CL - 1) / (int)CL;
        for (int i = warp; i < per; i += kAWarps) {
            const int row = (int)rank * per + i;
            if (row >= count) continue;
            float4 v[2];
            float top = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = h * 128 + lane * 4;
                v[h] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (j >= rk) continue;
                const uint32_t at = smem_u32(sums + row * p.r + j);
                for (uint32_t q = 0; q < CL; ++q) {
                    const float4 a = ld_cluster_f32x4(map_to_rank(at, q));
                    v[h].x += a.x; v[h].y += a.y; v[h].z += a.z; v[h].w += a.w;
                }
                top = fmaxf(top, fmaxf(fmaxf(fabsf(v[h].x), fabsf(v[h].y)), fmaxf(fabsf(v[h].z), fabsf(v[h].w))));
            }
            top = warp_max(top);
            // 2^(14 - e) for top in [2^e, 2^(e+1)); an infinite or tiny top keeps a factor that is a normal number
            int e = (int)(__float_as_uint(top) >> 23) - 127;
            e = e < -100 ? -100 : e > 127 ? 127 : e;
            const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23), down = __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = h * 128 + lane * 4;
                if (j >= rk) continue;
                const __half2 lo = __floats2half2_rn(v[h].x * up, v[h].y * up), hi = __floats2half2_rn(v[h].z * up, v[h].w * up);
                const uint32_t at = smem_u32(s16 + row * s_stride(p.r) + 2 * j);
                for (uint32_t q = 0; q < CL; ++q)
                    st_cluster_u2(map_to_rank(at, q), *reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            }
            if (lane < (int)CL)
                st_cluster_f32(map_to_rank(smem_u32(row_scale + row), lane), down * (p.scale ? __ldg(p.scale + slot) : 1.f));
        }
    }
    cluster_arrive();
    cluster_wait();

    // ---- B S: this CTA's part of N ----
    float factor[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) factor[i] = ok[i] ? row_scale[tw * 16 * MT + 8 * i + g] : 0.f;
    const uint8_t* s_row = s16 + (size_t)(tw * 16 * MT + g) * s_stride(p.r);
    for (int u = n_first; u < n_units; u += n_step) {
        const int n = u * 32 + 8 * t;
        uint4 y[2 * MT];
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i)
            y[i] = ok[i] && n < p.N ? *reinterpret_cast<const uint4*>(p.Y + tok[i] * p.ldy + n) : make_uint4(0, 0, 0, 0);
        float acc[MT][4][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[mt][j][e] = 0.f;
        for (int r0 = 0; r0 < rk; r0 += kChunk) {
            if (u != n_first || r0 > 0) fetch(u, r0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k0 = r0 + 32 * h;
                if (k0 >= rk) continue;
                const bool whole = k0 + 32 <= rk;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const uint8_t* q = s_row + (size_t)mt * 16 * s_stride(p.r) + 2 * k0;
                    uint4 a, c;
                    if (whole) {
                        a = *reinterpret_cast<const uint4*>(q + 16 * t);
                        c = *reinterpret_cast<const uint4*>(q + 8 * s_stride(p.r) + 16 * t);
                    } else {
                        const uint2 a2 = *reinterpret_cast<const uint2*>(q + 8 * t), c2 = *reinterpret_cast<const uint2*>(q + 8 * s_stride(p.r) + 8 * t);
                        a = make_uint4(a2.x, a2.y, 0, 0);
                        c = make_uint4(c2.x, c2.y, 0, 0);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        mma16816(acc[mt][j], a.x, c.x, a.y, c.y, b[j][h].x, b[j][h].y);
                        if (whole) mma16816(acc[mt][j], a.z, c.z, a.w, c.w, b[j][h].z, b[j][h].w);
                    }
                }
            }
        }
        if (n >= p.N) continue;
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
            if (!ok[i]) continue;
            const uint32_t yw[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&yw[j]));
                const __half2 v = __floats2half2_rn(fmaf(acc[i >> 1][j][2 * (i & 1)], factor[i], f.x),
                                                    fmaf(acc[i >> 1][j][2 * (i & 1) + 1], factor[i], f.y));
                o[j] = *reinterpret_cast<const uint32_t*>(&v);
            }
            *reinterpret_cast<uint4*>(p.out + tok[i] * p.ldo + n) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

// Tokens by adapter (in their order within an adapter), then the tokens without one; every group cut into tiles.  One CTA.
__global__ void __launch_bounds__(kPlanThreads)
adapters_plan_kernel(const int32_t* __restrict__ slot, int M, int n_slots, int32_t* __restrict__ out) {
    extern __shared__ int32_t cursor[];            // [n_slots + 1]: tokens of a group, then where its next one goes
    __shared__ int3 warp_sum[kPlanThreads / 32];
    const PlanView plan = plan_view(out, M, n_slots);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, groups = n_slots + 1;
    auto group_of = [&](int m) {
        const int s = slot[m];
        return s >= 0 && s < n_slots ? s : n_slots;
    };
    for (int i = tid; i < groups; i += kPlanThreads) cursor[i] = 0;
    __syncthreads();
    for (int m = tid; m < M; m += kPlanThreads) atomicAdd(&cursor[group_of(m)], 1);
    __syncthreads();
    // exclusive sums over the groups: tokens, tiles of either size
    const int per = (groups + kPlanThreads - 1) / kPlanThreads, g0 = tid * per, g1 = min(groups, g0 + per);
    auto tiles_of = [](int n, int tile) { return (n + tile - 1) / tile; };
    int3 mine = make_int3(0, 0, 0);
    for (int i = g0; i < g1; ++i) {
        mine.x += cursor[i];
        mine.y += tiles_of(cursor[i], kTileFew);
        mine.z += tiles_of(cursor[i], kTileMany);
    }
    int3 at = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, at.x, o), y = __shfl_up_sync(0xffffffffu, at.y, o), z = __shfl_up_sync(0xffffffffu, at.z, o);
        if (lane >= o) { at.x += x; at.y += y; at.z += z; }
    }
    if (lane == 31) warp_sum[warp] = at;
    __syncthreads();
    at.x -= mine.x; at.y -= mine.y; at.z -= mine.z;
    for (int w = 0; w < warp; ++w) { at.x += warp_sum[w].x; at.y += warp_sum[w].y; at.z += warp_sum[w].z; }
    if (tid == kPlanThreads - 1)
        *reinterpret_cast<int4*>(out) = make_int4(M, n_slots, at.y + mine.y, at.z + mine.z);
    for (int i = g0; i < g1; ++i) {
        const int n = cursor[i], s = i < n_slots ? i : -1;
        for (int k = 0; k < n; k += kTileFew) plan.tiles_few[at.y++] = make_int4(s, at.x + k, min(kTileFew, n - k), 0);
        for (int k = 0; k < n; k += kTileMany) plan.tiles_many[at.z++] = make_int4(s, at.x + k, min(kTileMany, n - k), 0);
        cursor[i] = at.x;
        at.x += n;
    }
    __syncthreads();
    // the tokens in their order: the warps one after the other
    for (int m0 = 0; m0 < M; m0 += kPlanThreads) {
        const int m = m0 + tid, warps = min(kPlanThreads, M - m0 + 31) / 32;
        const int gr = m < M ? group_of(m) : -1;
        const unsigned same = __match_any_sync(0xffffffffu, gr);
        const int before = __popc(same & ((1u << lane) - 1));
        for (int w = 0; w < warps; ++w) {
            if (w == warp) {
                const int at0 = gr >= 0 ? cursor[gr] : 0;
                __syncwarp();
                if (gr >= 0) {
                    plan.tokens[at0 + before] = m;
                    if (before == 0) cursor[gr] = at0 + __popc(same);
                }
            }
            __syncthreads();
        }
    }
}

template <int MT, int TW>
size_t smem_bytes(int r) {
    constexpr int TM = 16 * MT * TW, KW = kAWarps / TW;
    return (size_t)KW * TM * kRedStride * 4 + (size_t)TM * r * 4 + (size_t)TM * s_stride(r) + TM * 4;
}

template <int MT, int TW>
int launch_tiles(AdapterParams p, int tiles, int CL, cudaStream_t st) {
    static bool configured[kMaxDevices] = {false};
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != ASER_OK) return rc;
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(adapters_kernel<MT, TW>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)smem_bytes<MT, TW>(256));
        if (e != cudaSuccess) return record_cuda_error(e, "adapters smem attribute");
        configured[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * p.parts * CL, 1, 1);
    cfg.blockDim = dim3(kAThreads, 1, 1);
    cfg.dynamicSmemBytes = smem_bytes<MT, TW>(p.r);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CL; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, adapters_kernel<MT, TW>, p);
    if (e != cudaSuccess) return record_cuda_error(e, "adapters_kernel");
    return check_launch("adapters_kernel");
}

}  // namespace

size_t adapters_plan_bytes(int M, int n_slots) {
    const PlanView v = plan_view(static_cast<int32_t*>(nullptr), M, n_slots);
    return (size_t)v.words * 4;
}

int launch_adapters_plan(const int32_t* slot, int M, int n_slots, void* plan, cudaStream_t st) {
    adapters_plan_kernel<<<1, kPlanThreads, (n_slots + 1) * 4, st>>>(slot, M, n_slots, static_cast<int32_t*>(plan));
    return check_launch("adapters_plan_kernel");
}

int launch_adapters(const __half* X, size_t ldx, const __half* A, const __half* B, const int32_t* ranks, const float* scale,
                    const void* plan, int M, int N, int K, int r, int n_slots, const __half* Y, size_t ldy, __half* out,
                    size_t ldo, cudaStream_t st) {
    AdapterParams p = {};
    p.X = X; p.A = A; p.B = B; p.ranks = ranks; p.scale = scale; p.plan = static_cast<const int32_t*>(plan);
    p.Y = Y; p.out = out;
    p.ldx = ldx; p.ldy = ldy; p.ldo = ldo;
    p.M = M; p.N = N; p.K = K; p.r = r; p.n_slots = n_slots;
    int num_sms = 0;
    const int rc = device_sm_count(&num_sms);
    if (rc != ASER_OK) return rc;
    const int used = n_slots < M ? n_slots : M;
    const bool few = M <= 16 * used;
    const int CL = 8;
    const int bound = plan_tiles(M, n_slots, few ? kTileFew : kTileMany);
    const int parts = 2 * num_sms / (bound * CL);
    const int want = (N + K - 1) / K;
    p.parts = parts < 1 ? 1 : parts > want ? want : parts;
    return few ? launch_tiles<1, 1>(p, bound, CL, st) : launch_tiles<2, 2>(p, bound, CL, st);
}

}  // namespace aser
