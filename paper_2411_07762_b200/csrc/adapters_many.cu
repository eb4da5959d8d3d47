// Low-rank adapters of many requests (adapters.cu) where an adapter has many tokens, as in prompts: two launches.
//
//   S = A_a x      adapters_down_kernel: a cluster of CTAs per tile of 128 tokens of one adapter, split along K.  What bounds it is X
//                  from HBM and A from L2 (again for every tile: the reason for 128 tokens).  Both go to shared memory 64 columns
//                  at a time by asynchronous copies of 16 bytes, because a tile's rows lie anywhere in the batch; a ring of
//                  stages keeps 72 KB a CTA in flight, two CTAs to an SM.  Partial sums meet in distributed shared memory, in a
//                  fixed order, each CTA finishing 128 / CL tokens.
//   out = Y + B S  adapters_up_kernel: a CTA per tile and 128 channels; bound by Y, read and written once.  Nothing carries over from
//                  block to block, so enough CTAs are resident to keep the loads of Y in flight, and B and Y are asked for while
//                  the first kernel still runs.
//
// One launch for both (the kernel for few tokens with larger tiles) spent most of its time in phases that wait for one
// another: 4096 tokens of 6 adapters, rank 64, 4096 x 4096 65.7 us.
#include "adapters.cuh"
#include "sm100_ptx.cuh"

namespace aser {

namespace {

constexpr int kThreads = 256, kTok = kTileMany, kCL = 8;
constexpr int kCols = 64;                            // columns of a stage: 128 bytes a row, swizzled by row % 8
constexpr int kXBytes = kTok * kCols * 2;
constexpr int kUpCols = 128;                         // channels of a CTA of the second kernel

// Ranks side by side in a pass of the first kernel: 64, the two halves of the warps taking alternate steps of K, or 128, half each.
template <int NR>
struct DownCfg {
    static constexpr int Ranks = 64 * NR;
    static constexpr int Stage = kXBytes + Ranks * kCols * 2;
    static constexpr int Stages = NR == 1 ? 4 : 3;
    static constexpr int RowFloats = Ranks + 4;      // of the partial sums, which take the place of the stages
    static constexpr int Smem = Stage * Stages;
    static_assert(kTok * RowFloats * 4 <= Smem, "partial sums fit the ring");
    static_assert(2 * Smem + 4096 <= 227 * 1024, "two CTAs to an SM");
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldmatrix4(uint32_t (&v)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}

template <int NR>
__global__ void __launch_bounds__(kThreads, 2)
adapters_down_kernel(const AdapterParams p) {
    using C = DownCfg<NR>;
    grid_dep_wait();
    grid_dep_launch();
    extern __shared__ __align__(128) uint8_t smem[];
    const int rank = (int)cluster_rank(), tile = (int)(blockIdx.x / kCL);
    const PlanView plan = plan_view(p.plan, p.M, p.n_slots);
    const int4 head = *reinterpret_cast<const int4*>(p.plan);
    const int4 t4 = plan.tiles_many[tile];
    if (head.x != p.M || head.y != p.n_slots || tile >= head.w) return;
    const int slot = t4.x, first = t4.y, count = t4.z;
    const int rk = slot < 0 ? 0 : adapter_rank(p, slot);
    if (rk == 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int tw = warp & 3, half = warp >> 2;
    const uint32_t sb = smem_u32(smem);
    // copies: this thread's 16 bytes of rows lr, lr + 32, ...
    const int lr = threadIdx.x >> 3, lc = threadIdx.x & 7;
    const uint32_t to = (uint32_t)(lr * 128 + ((lc ^ (lr & 7)) << 4));      // (rows 32 apart have the same swizzle)
    const __half* xp[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        xp[i] = lr + 32 * i < count ? p.X + (size_t)plan.tokens[first + lr + 32 * i] * p.ldx + lc * 8 : nullptr;
    const int steps = p.K / kCols, s0 = rank * steps / kCL, s1 = (rank + 1) * steps / kCL;
    float4 sum[2][2];                     // [pass][row of this warp]: four sums a lane
    float* part = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        const int r0 = pass * C::Ranks;
        sum[pass][0] = sum[pass][1] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r0 >= rk) continue;
        const __half* ap = p.A + ((size_t)slot * p.r + r0 + lr) * p.K + lc * 8;
        auto load = [&](int s) {
            if (s < s1) {
                const uint32_t at = sb + (uint32_t)((s - s0) % C::Stages * C::Stage) + to;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (xp[i]) cp_async16(at + i * 4096, xp[i] + (size_t)s * kCols);
#pragma unroll
                for (int i = 0; i < 2 * NR; ++i)
                    if (r0 + lr + 32 * i < rk) cp_async16(at + kXBytes + i * 4096, ap + (size_t)32 * i * p.K + (size_t)s * kCols);
            }
            cp_async_commit();
        };
        float acc[2][8][4];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[mt][nt][e] = 0.f;
#pragma unroll
        for (int s = 0; s < C::Stages - 1; ++s) load(s0 + s);
        // rows behind the tile's last token and ranks behind the adapter's are whatever the ring holds: nobody reads their sums
        const int nts = NR == 2 ? (rk - r0 - 64 * half + 15) / 16 : (rk - r0 + 15) / 16;     // pairs of 8 ranks of this warp
        for (int s = s0; s < s1; ++s) {
            cp_async_wait<C::Stages - 2>();
            __syncthreads();
            load(s + C::Stages - 1);
            const uint32_t xs = sb + (uint32_t)((s - s0) % C::Stages * C::Stage), as = xs + kXBytes;
#pragma unroll
            for (int kk0 = 0; kk0 < (NR == 2 ? 4 : 2); ++kk0) {
                const int kk = NR == 2 ? kk0 : 2 * half + kk0;
                uint32_t x[2][4];
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    const int row = tw * 32 + mt * 16 + (lane & 15);
                    ldmatrix4(x[mt], xs + row * 128 + (((kk * 2 + (lane >> 4)) ^ (row & 7)) << 4));
                }
#pragma unroll
                for (int np = 0; np < 4; ++np) {
                    if (np >= nts) break;
                    uint32_t a[4];
                    const int row = (NR == 2 ? half * 64 : 0) + np * 16 + (lane & 7) + ((lane >> 4) << 3);
                    ldmatrix4(a, as + row * 128 + (((kk * 2 + ((lane >> 3) & 1)) ^ (row & 7)) << 4));
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        mma16816(acc[mt][2 * np], x[mt][0], x[mt][1], x[mt][2], x[mt][3], a[0], a[1]);
                        mma16816(acc[mt][2 * np + 1], x[mt][0], x[mt][1], x[mt][2], x[mt][3], a[2], a[3]);
                    }
                }
            }
        }
        cp_async_wait<0>();
        __syncthreads();                  // the ring is free
        // partial sums [128 tokens][ranks]; where both halves of the warps have some of the same, the second adds to the first's
        for (int turn = 0; turn < (NR == 2 ? 1 : 2); ++turn) {
            if (NR == 2 || half == turn) {
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int nt = 0; nt < 8; ++nt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (nt >= 2 * nts) continue;
                            float2* q = reinterpret_cast<float2*>(part + (tw * 32 + mt * 16 + 8 * h + g) * C::RowFloats +
                                                                  (NR == 2 ? half * 64 : 0) + nt * 8 + 2 * t);
                            float2 v = make_float2(acc[mt][nt][2 * h], acc[mt][nt][2 * h + 1]);
                            if (turn) { const float2 o = *q; v.x += o.x; v.y += o.y; }
                            *q = v;
                        }
            }
            __syncthreads();
        }
        cluster_arrive();
        cluster_wait();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = rank * (kTok / kCL) + warp * 2 + i, j = lane * 4;
            if (row >= count || j >= C::Ranks || r0 + j >= rk) continue;
            const uint32_t at = smem_u32(part + row * C::RowFloats + j);
            float4 a[kCL];
#pragma unroll
            for (int q = 0; q < kCL; ++q) a[q] = ld_cluster_f32x4(map_to_rank(at, q));
#pragma unroll
            for (int q = 0; q < kCL; ++q) { sum[pass][i].x += a[q].x; sum[pass][i].y += a[q].y; sum[pass][i].z += a[q].z; sum[pass][i].w += a[q].w; }
        }
        cluster_arrive();                 // nobody overwrites or leaves what a peer still reads
        cluster_wait();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = rank * (kTok / kCL) + warp * 2 + i;
        if (row >= count) continue;
        float top = 0.f;
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) top = fmaxf(top, max4_abs(sum[pass][i]));
        const RowFactor f = row_factor(warp_max(top));
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
            const int j = lane * 4;
            if (j < C::Ranks && pass * C::Ranks + j < rk)
                *reinterpret_cast<uint2*>(p.S + (size_t)(first + row) * p.r + pass * C::Ranks + j) = scaled_f16(sum[pass][i], f.up);
        }
        if (lane == 0) p.row_scale[first + row] = f.down * (p.scale ? __ldg(p.scale + slot) : 1.f);
    }
}

// y_ready: what wrote Y is known to be complete when this kernel starts (the first kernel waited for it).
__global__ void __launch_bounds__(kThreads, 2)
adapters_up_kernel(const AdapterParams p, int n_blocks, bool y_ready) {
    extern __shared__ __align__(128) uint8_t smem[];
    if (!y_ready) grid_dep_wait();
    const int tile = (int)blockIdx.x / n_blocks, n0 = ((int)blockIdx.x % n_blocks) * kUpCols;
    const PlanView plan = plan_view(p.plan, p.M, p.n_slots);
    const int4 head = *reinterpret_cast<const int4*>(p.plan);
    const int4 t4 = plan.tiles_many[tile];
    if (head.x != p.M || head.y != p.n_slots || tile >= head.w) return;
    const int slot = t4.x, first = t4.y, count = t4.z;
    const int rk = slot < 0 ? 0 : adapter_rank(p, slot);
    if (rk == 0 && p.Y == p.out) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int tw = warp & 3, nh = warp >> 2;
    const int stride = 2 * p.r + 16;          // bytes of a row in shared memory: an odd multiple of 16
    const uint32_t ss = smem_u32(smem), bs = ss + kTok * stride;
    const int row_chunks = rk / 8;
    for (int i = threadIdx.x; i < kUpCols * row_chunks; i += kThreads) {
        const int row = i / row_chunks, c = i % row_chunks;
        if (n0 + row < p.N) cp_async16(bs + row * stride + c * 16, p.B + ((size_t)slot * p.N + n0 + row) * p.r + c * 8);
    }
    size_t tok[4];
    bool ok[4];
    uint4 y[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = tw * 32 + 8 * i + g;
        ok[i] = row < count;
        tok[i] = ok[i] ? (size_t)plan.tokens[first + row] : 0;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int n = n0 + nh * 64 + u * 32 + 8 * t;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            y[u][i] = ok[i] && n < p.N ? *reinterpret_cast<const uint4*>(p.Y + tok[i] * p.ldy + n) : make_uint4(0, 0, 0, 0);
    }
    float factor[4] = {0.f, 0.f, 0.f, 0.f};
    if (rk > 0) {
        if (y_ready) grid_dep_wait();         // S is there
        for (int i = threadIdx.x; i < count * row_chunks; i += kThreads) {
            const int row = i / row_chunks, c = i % row_chunks;
            cp_async16(ss + row * stride + c * 16, p.S + (size_t)(first + row) * p.r + c * 8);
        }
        cp_async_commit();
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (ok[i]) factor[i] = p.row_scale[first + tw * 32 + 8 * i + g];
        cp_async_wait<0>();
        __syncthreads();
    }
    grid_dep_launch();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int n = n0 + nh * 64 + u * 32 + 8 * t;
        float acc[2][4][4];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[mt][j][e] = 0.f;
        // a tile of 8 channels takes rows (g / 2) 8 + 2 j + g % 2 of 32: a thread's outputs are then 8 neighbours
        const uint32_t a_at = ss + (uint32_t)((tw * 32 + (lane & 15)) * stride + (lane >> 4) * 16);
        const int br = nh * 64 + u * 32 + ((lane & 7) >> 1) * 8 + (lane & 1) + 2 * (lane >> 4);
        const uint32_t b_at = bs + (uint32_t)(br * stride + ((lane >> 3) & 1) * 16);
        for (int k = 0; k < rk; k += 16) {
            uint32_t a[2][4], b[2][4];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) ldmatrix4(a[mt], a_at + mt * 16 * stride + 2 * k);
#pragma unroll
            for (int jp = 0; jp < 2; ++jp) ldmatrix4(b[jp], b_at + jp * 4 * stride + 2 * k);
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    mma16816(acc[mt][j], a[mt][0], a[mt][1], a[mt][2], a[mt][3], b[j >> 1][2 * (j & 1)], b[j >> 1][2 * (j & 1) + 1]);
        }
        if (n >= p.N) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (ok[i])
                *reinterpret_cast<uint4*>(p.out + tok[i] * p.ldo + n) =
                    rk == 0 ? y[u][i] : add_scaled(y[u][i], acc[i >> 1], i & 1, factor[i]);
    }
}

template <int NR>
int launch_down(const AdapterParams& p, int tiles, cudaStream_t st) {
    static bool configured[kMaxDevices] = {false};
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != ASER_OK) return rc;
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(adapters_down_kernel<NR>, cudaFuncAttributeMaxDynamicSharedMemorySize, DownCfg<NR>::Smem);
        if (e != cudaSuccess) return record_cuda_error(e, "adapters_down smem attribute");
        configured[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * kCL, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = DownCfg<NR>::Smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCL; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, adapters_down_kernel<NR>, p);
    if (e != cudaSuccess) return record_cuda_error(e, "adapters_down_kernel");
    return check_launch("adapters_down_kernel");
}

}  // namespace

int launch_adapters_down(const AdapterParams& p, cudaStream_t st) {
    const int tiles = plan_tiles(p.M, p.n_slots, kTileMany);
    return p.r <= 64 ? launch_down<1>(p, tiles, st) : launch_down<2>(p, tiles, st);
}

int launch_adapters_up(const AdapterParams& p, bool y_ready, cudaStream_t st) {
    static bool configured[kMaxDevices] = {false};
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != ASER_OK) return rc;
    const int tiles = plan_tiles(p.M, p.n_slots, kTileMany), blocks = (p.N + kUpCols - 1) / kUpCols;
    auto smem = [](int r) { return (kTok + kUpCols) * (2 * r + 16); };
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(adapters_up_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem(256));
        if (e != cudaSuccess) return record_cuda_error(e, "adapters_up smem attribute");
        configured[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * blocks, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem(p.r);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, adapters_up_kernel, p, blocks, y_ready);
    if (e != cudaSuccess) return record_cuda_error(e, "adapters_up_kernel");
    return check_launch("adapters_up_kernel");
}

}  // namespace aser
