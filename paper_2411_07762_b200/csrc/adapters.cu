// Low-rank adapters of many requests beside a shared projection:
//   out[m, :] = fp16( Y[m, :] + scale[a] * B_a (A_a x[m]) ),   a = the adapter of token m, or none.
//
// Two products with a small intermediate, S = A_a x (r numbers per token) and B_a S.  The bytes are those of the adapters in
// use (2 r (K + N) each), X, and Y twice; a token's 2 r (K + N) multiply-adds come to at most r of them per byte of X and Y, so
// at the ranks of adapters mma.sync (m16n8k16) keeps up with HBM and takes tokens from anywhere in a batch.  Arranged are:
//  * tokens of one adapter have to meet, wherever they stand in the batch: a plan (adapters_plan_kernel), made once per batch
//    and used by all layers of a step, lists the tokens by adapter and cuts each adapter's into tiles of 16 and of 128;
//  * few tokens per adapter (this file): one launch, a cluster of eight CTAs per tile of 16, which split K for the first
//    product and N for the second.  What bounds it is the chain of loads, so operands go from global memory straight into
//    registers (the first rows of B to shared memory, ahead of the first product): an inner product does not care about the
//    order of k, so a thread's k positions are the 8 columns of one 16-byte load, the same for both operands; likewise the 32 rows of B that a warp takes are dealt so that a thread's outputs
//    are 8 neighbours.  Up to 64 ranks each CTA sends its sums to the others, so that one barrier is all that S waits for.  One
//    token, 4096 x 4096, rank 16: 4.5 us; 64 tokens of 32 adapters, ranks to 64: 11.4 (bytes: 3.3);
//  * many tokens per adapter: two launches (adapters_many.cu).
// S is summed and exchanged in fp32, in a fixed order; nothing depends on the order of tokens in a tile.  For the second product it
// is rounded to fp16 (2^-11 of each number, where the output has 2^-11 of the whole sum) after a scaling by a power of two that
// brings the token's largest entry to [2^14, 2^15): exact, and no size of activations or adapters overflows.
#include "adapters.cuh"
#include "sm100_ptx.cuh"

namespace aser {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kCL = 8, kTok = kTileFew;
constexpr int kChunk = 64;                  // ranks of S summed at a time
constexpr int kRedStride = kChunk + 8;      // floats: rows 8 banks apart
constexpr int kSumBytes = kCL * kTok * kChunk * 4;      // (more than 16 x 256 sums)
constexpr int kPlanThreads = 1024;

// Bytes between the fp16 rows of S: an odd multiple of 64, so that 16-byte reads of two rows do not meet in a bank.
__host__ __device__ constexpr int s_stride(int r) { return (2 * r + 63) / 128 * 128 + 64; }

__device__ __forceinline__ void st_cluster_f32x4(uint32_t addr, const float4& v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// acc += X A^T over the 32-column units u0, u0 + step, ... of K, BATCH of them in flight; NT tiles of 8 ranks, of which n_tiles are there.
template <int BATCH, int NT>
__device__ __forceinline__ void down_units(float (&acc)[8][4], const __half* (&xp)[2], const bool (&ok)[2], const __half* ap, size_t K,
                                           int n_tiles, int u0, int units, int step) {
    for (; u0 < units; u0 += BATCH * step) {
        uint4 x[BATCH][2], l[BATCH][NT];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int u = u0 + b * step;
            const bool in = BATCH == 1 || u < units;
#pragma unroll
            for (int i = 0; i < 2; ++i) x[b][i] = in && ok[i] ? *reinterpret_cast<const uint4*>(xp[i] + u * 32) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                l[b][nt] = in && nt < n_tiles ? __ldg(reinterpret_cast<const uint4*>(ap + nt * 8 * K + u * 32)) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (nt >= n_tiles) break;
                mma16816(acc[nt], x[b][0].x, x[b][1].x, x[b][0].y, x[b][1].y, l[b][nt].x, l[b][nt].y);
                mma16816(acc[nt], x[b][0].z, x[b][1].z, x[b][0].w, x[b][1].w, l[b][nt].z, l[b][nt].w);
            }
    }
}

__global__ void __launch_bounds__(kThreads, 2)
adapters_few_kernel(const AdapterParams p) {
    grid_dep_wait();
    grid_dep_launch();
    extern __shared__ __align__(128) uint8_t smem[];
    warm_ranks(p);
    const int rank = (int)cluster_rank(), cluster = (int)(blockIdx.x / kCL), tile = cluster / p.parts, part = cluster - tile * p.parts;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const PlanView plan = plan_view(p.plan, p.M, p.n_slots);
    const int32_t* record = plan.tiles_few + (size_t)tile * kFewWords;
    const int4 head = *reinterpret_cast<const int4*>(p.plan), t4 = *reinterpret_cast<const int4*>(record);
    const int tok0 = record[4 + g], tok1 = record[12 + g];
    if (head.x != p.M || head.y != p.n_slots || tile >= head.z) return;      // (the whole cluster, here and below)
    const int slot = t4.x, count = t4.z;
    const int rk = slot < 0 ? 0 : adapter_rank(p, slot);
    if (rk == 0 && p.Y == p.out) return;
    const int n_units = (p.N + 31) / 32, n_step = p.parts * kCL * kWarps, n_first = (part * kCL + rank) * kWarps + warp;
    const bool ok[2] = {g < count, 8 + g < count};
    const size_t tok[2] = {ok[0] ? (size_t)tok0 : 0, ok[1] ? (size_t)tok1 : 0};
    auto load_y = [&](int u, uint4 (&y)[2]) {
        const int n = u * 32 + 8 * t;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            y[i] = ok[i] && n < p.N ? *reinterpret_cast<const uint4*>(p.Y + tok[i] * p.ldy + n) : make_uint4(0, 0, 0, 0);
    };
    uint4 y[2];
    if (n_first < n_units) load_y(n_first, y);
    if (rk == 0) {              // nothing to add
        for (int u = n_first; u < n_units; u += n_step) {
            if (u != n_first) load_y(u, y);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (ok[i] && u * 32 + 8 * t < p.N) *reinterpret_cast<uint4*>(p.out + tok[i] * p.ldo + u * 32 + 8 * t) = y[i];
        }
        return;
    }
    // (waited for before anything is sent: every CTA of the cluster runs by then; relaxed, because a release waits for the loads)
    cluster_arrive_relaxed();
    float* red = reinterpret_cast<float*>(smem);                             // [warp][16][kRedStride]
    float* sums = red + kWarps * kTok * kRedStride;                          // up to 64 ranks: [CTA][16][64], received; else [16][r]
    uint8_t* s16 = reinterpret_cast<uint8_t*>(sums) + kSumBytes;             // [16][s_stride(r)]
    float* row_scale = reinterpret_cast<float*>(s16 + kTok * s_stride(p.r)); // [16]
    uint8_t* b_rows = reinterpret_cast<uint8_t*>(row_scale + kTok) + warp * (32 * 128);
    const __half* B = p.B + (size_t)slot * p.N * p.r;
    {   // the first 64 ranks of the warp's first rows of B: there when S is
        const int chunks = (rk < kChunk ? rk : kChunk) / 8, shift = chunks <= 2 ? 1 : chunks <= 4 ? 2 : 3, c = lane & ((1 << shift) - 1);
        for (int row = lane >> shift; row < 32; row += 32 >> shift) {
            const int n = n_first * 32 + row;
            if (c < chunks && n < p.N) cp_async16(smem_u32(b_rows) + row * 128 + ((c ^ ((row & 1) << 2)) << 4), B + (size_t)n * p.r + c * 8);
        }
        cp_async_commit();
    }

    // ---- S = A x: this CTA's part of K, the warps' parts of it ----
    const __half* A = p.A + (size_t)slot * p.r * p.K + 8 * t;
    const __half* xp[2] = {p.X + tok[0] * p.ldx + 8 * t, p.X + tok[1] * p.ldx + 8 * t};
    const bool narrow = rk <= kChunk;
    for (int r0 = 0; r0 < rk; r0 += kChunk) {
        float acc[8][4];
#pragma unroll
        for (int nt = 0; nt < 8; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[nt][e] = 0.f;
        const __half* ap = A + (size_t)(r0 + g) * p.K;
        const int n_tiles = (rk - r0) / 8, u0 = rank * kWarps + warp;
        if (n_tiles <= 4) down_units<2, 4>(acc, xp, ok, ap, p.K, n_tiles, u0, p.K / 32, kCL * kWarps);
        else down_units<1, 8>(acc, xp, ok, ap, p.K, n_tiles, u0, p.K / 32, kCL * kWarps);
        if (r0 > 0) __syncthreads();            // the chunk before has been summed
#pragma unroll
        for (int nt = 0; nt < 8; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (nt < n_tiles && ok[h])
                    *reinterpret_cast<float2*>(red + (warp * kTok + 8 * h + g) * kRedStride + nt * 8 + 2 * t) = make_float2(acc[nt][2 * h], acc[nt][2 * h + 1]);
        __syncthreads();
        if (narrow) cluster_wait();
        const int per_row = (n_tiles < 8 ? n_tiles : 8) * 2;        // groups of four sums
        for (int i = threadIdx.x; i < count * per_row; i += kThreads) {
            const int row = i / per_row, j = i % per_row * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float4 a = *reinterpret_cast<const float4*>(red + (w * kTok + row) * kRedStride + j);
                v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
            }
            if (!narrow) {
                *reinterpret_cast<float4*>(sums + row * p.r + r0 + j) = v;
                continue;
            }
            const uint32_t at = smem_u32(sums + (rank * kTok + row) * kChunk + j);
#pragma unroll
            for (int q = 0; q < kCL; ++q) st_cluster_f32x4(map_to_rank(at, q), v);
        }
    }
    if (!narrow) cluster_wait();
    cluster_arrive();
    cluster_wait();

    // ---- every CTA has the sums of all eight, adds and rounds them ----
    const float alpha = p.scale ? __ldg(p.scale + slot) : 1.f;
    if (narrow) {                           // two rows side by side
        const int row = warp * 2 + (lane >> 4), j = (lane & 15) * 4;
        const bool mine = row < count && j < rk;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mine)
#pragma unroll
            for (int q = 0; q < kCL; ++q) {
                const float4 a = *reinterpret_cast<const float4*>(sums + (q * kTok + row) * kChunk + j);
                v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
            }
        float top = max4_abs(v);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const RowFactor f = row_factor(top);
        if (mine) *reinterpret_cast<uint2*>(s16 + row * s_stride(p.r) + 2 * j) = scaled_f16(v, f.up);
        if (mine && j == 0) row_scale[row] = f.down * alpha;
    } else {
        for (int row = warp; row < count; row += kWarps) {
            float4 v[2];
            float top = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = h * 128 + lane * 4;
                v[h] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (j < rk) {
                    const uint32_t at = smem_u32(sums + row * p.r + j);
                    float4 a[kCL];
#pragma unroll
                    for (int q = 0; q < kCL; ++q) a[q] = ld_cluster_f32x4(map_to_rank(at, q));
#pragma unroll
                    for (int q = 0; q < kCL; ++q) { v[h].x += a[q].x; v[h].y += a[q].y; v[h].z += a[q].z; v[h].w += a[q].w; }
                }
                top = fmaxf(top, max4_abs(v[h]));
            }
            const RowFactor f = row_factor(warp_max(top));
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (h * 128 + lane * 4 < rk) *reinterpret_cast<uint2*>(s16 + row * s_stride(p.r) + 2 * (h * 128 + lane * 4)) = scaled_f16(v[h], f.up);
            if (lane == 0) row_scale[row] = f.down * alpha;
        }
    }
    cp_async_wait<0>();
    __syncthreads();
    if (!narrow) cluster_arrive();          // (waited for at the end: nobody leaves while a peer may still read its sums)

    // ---- B S: this CTA's part of N ----
    float factor[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) factor[i] = ok[i] ? row_scale[8 * i + g] : 0.f;
    const uint8_t* s_row = s16 + g * s_stride(p.r);
    for (int u = n_first; u < n_units; u += n_step) {
        const int n = u * 32 + 8 * t;
        float acc[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
        for (int r0 = 0; r0 < rk; r0 += kChunk) {
            // rows (g / 2) 8 + 2 j + g % 2 of the unit, 8 ranks of each 32 a thread (4 of the last 16)
            uint4 b[4][2];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = (g >> 1) * 8 + 2 * j + (g & 1), row_n = u * 32 + at;
                const __half* row = B + (size_t)row_n * p.r + r0;
                const uint8_t* kept = b_rows + at * 128;
                const int swap = (at & 1) << 6;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int left = rk - r0 - 32 * h;
                    b[j][h] = make_uint4(0, 0, 0, 0);
                    if (left <= 0 || row_n >= p.N) continue;
                    if (u == n_first && r0 == 0) {
                        if (left >= 32) b[j][h] = *reinterpret_cast<const uint4*>(kept + ((64 * h + 16 * t) ^ swap));
                        else { const uint2 v = *reinterpret_cast<const uint2*>(kept + ((64 * h + 8 * t) ^ swap)); b[j][h].x = v.x; b[j][h].y = v.y; }
                    } else if (left >= 32) b[j][h] = __ldg(reinterpret_cast<const uint4*>(row + 32 * h + 8 * t));
                    else { const uint2 v = __ldg(reinterpret_cast<const uint2*>(row + 32 * h + 4 * t)); b[j][h].x = v.x; b[j][h].y = v.y; }
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k0 = r0 + 32 * h;
                if (k0 >= rk) continue;
                const bool whole = k0 + 32 <= rk;
                const uint8_t* q = s_row + 2 * k0;
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
                    mma16816(acc[j], a.x, c.x, a.y, c.y, b[j][h].x, b[j][h].y);
                    if (whole) mma16816(acc[j], a.z, c.z, a.w, c.w, b[j][h].z, b[j][h].w);
                }
            }
        }
        const uint4 mine[2] = {y[0], y[1]};
        if (u + n_step < n_units) load_y(u + n_step, y);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (ok[i] && n < p.N) *reinterpret_cast<uint4*>(p.out + tok[i] * p.ldo + n) = add_scaled(mine[i], acc, i, factor[i]);
    }
    if (!narrow) cluster_wait();
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
    __shared__ int few, many;
    if (tid == kPlanThreads - 1) {
        few = at.y + mine.y;
        many = at.z + mine.z;
        *reinterpret_cast<int4*>(out) = make_int4(M, n_slots, few, many);
    }
    // (the last group is that of the tokens without an adapter)
    if (g0 < groups && g1 == groups) *reinterpret_cast<int4*>(out + 4) = make_int4(at.z + mine.z - tiles_of(cursor[groups - 1], kTileMany), M - cursor[groups - 1], 0, 0);
    for (int i = g0; i < g1; ++i) {
        const int n = cursor[i], s = i < n_slots ? i : -1;
        for (int k = 0; k < n; k += kTileFew) *reinterpret_cast<int4*>(plan.tiles_few + (size_t)kFewWords * at.y++) = make_int4(s, at.x + k, min(kTileFew, n - k), 0);
        for (int k = 0; k < n; k += kTileMany) plan.tiles_many[at.z++] = make_int4(s, at.x + k, min(kTileMany, n - k), -1);
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
    // the tiles of 16 carry their tokens' numbers
    for (int i = tid; i < few * kTileFew; i += kPlanThreads) {
        int32_t* record = plan.tiles_few + (size_t)kFewWords * (i / kTileFew);
        const int e = i % kTileFew;
        record[4 + e] = e < record[2] ? plan.tokens[record[1] + e] : 0;
    }
    for (int i = tid; i < many; i += kPlanThreads) {         // (a group's tokens ascend)
        const int4 r = plan.tiles_many[i];
        const int a = plan.tokens[r.y], b = plan.tokens[r.y + r.z - 1];
        if (b - a == r.z - 1) plan.tiles_many[i].w = a;
    }
}

int few_smem(int r) { return kWarps * kTok * kRedStride * 4 + kSumBytes + kTok * s_stride(r) + kTok * 4 + kWarps * 32 * 128; }

int launch_few(AdapterParams p, cudaStream_t st) {
    static bool configured[kMaxDevices] = {false};
    int dev = 0, num_sms = 0;
    int rc = current_device(&dev);
    if (rc == ASER_OK) rc = device_sm_count(&num_sms);
    if (rc != ASER_OK) return rc;
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(adapters_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, few_smem(256));
        if (e != cudaSuccess) return record_cuda_error(e, "adapters smem attribute");
        configured[dev] = true;
    }
    // several clusters to a tile where few tiles leave room, each with S of its own, until a warp has 32 channels
    const int tiles = plan_tiles(p.M, p.n_slots, kTok), want = (p.N + 32 * kCL * kWarps - 1) / (32 * kCL * kWarps), room = 2 * num_sms / (tiles * kCL);
    p.parts = room < 1 ? 1 : room > want ? want : room;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * p.parts * kCL, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = few_smem(p.r);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCL; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, adapters_few_kernel, p);
    if (e != cudaSuccess) return record_cuda_error(e, "adapters_few_kernel");
    return check_launch("adapters_few_kernel");
}

}  // namespace

size_t adapters_plan_bytes(int M, int n_slots) {
    const PlanView v = plan_view(nullptr, M, n_slots);
    return (size_t)v.words * 4;
}

int launch_adapters_plan(const int32_t* slot, int M, int n_slots, void* plan, cudaStream_t st) {
    adapters_plan_kernel<<<1, kPlanThreads, (n_slots + 1) * 4, st>>>(slot, M, n_slots, static_cast<int32_t*>(plan));
    return check_launch("adapters_plan_kernel");
}

// Estimates of both ways, in us, with half of the adapters in use, each with a short tile in two of 16 tokens and one of 128 at
// least (fitted to 90 points: 1 to 48 adapters of 8 to 128 tokens, five shapes).  Few | many, tokens to an adapter: 4096 x 4096,
// rank 64, 4 adapters: 32 9.1 | 12.0, 128 13.8 | 14.0, 16 adapters: 16 11.0 | 16.7, 32 18.3 | 17.5, 128 48.7 | 25.8; 28672 x 4096, rank 32, 4
// adapters: 32 16.3 | 19.2, 64 30.4 | 21.3; 4096 x 14336, rank 128, 16 adapters: 8 36.4 | 30.9; 1024 x 1024, rank 32, 16 adapters:
// 32 9.6 | 10.6, 64 14.0 | 10.7.
bool adapters_many(int M, int N, int K, int r, int n_slots) {
    if (M <= 32 || r == 0) return false;
    const float used = 0.5f * (n_slots < M ? n_slots : M), wide = (float)(K + N) / 8192;
    const float few_tiles = M / 16.f + 0.5f * used, many_tiles = fmaxf(used, M / 128.f + 0.5f * used);
    const float few = few_tiles * (0.07f + wide * (0.24f + 0.1f * r / 64));
    const float many = 5.f + 0.42f * many_tiles * fmaxf(0.5f, wide) + 5.6e-7f * M * (K + N);
    return many < few;
}

size_t adapters_workspace_bytes(int M, int N, int K, int r, int n_slots) {
    return adapters_many(M, N, K, r, n_slots) ? (size_t)M * (2 * r + 4) : 0;
}

int launch_adapters(AdapterParams p, void* workspace, cudaStream_t st) {
    if (!adapters_many(p.M, p.N, p.K, p.r, p.n_slots)) return launch_few(p, st);
    p.S = static_cast<__half*>(workspace);
    p.row_scale = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + (size_t)p.M * 2 * p.r);
    const int rc = launch_adapters_down(p, st);
    return rc != ASER_OK ? rc : launch_adapters_up(p, st);
}

}  // namespace aser
