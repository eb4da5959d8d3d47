// Low-rank adapters of many requests (adapters.cu) where an adapter has many tokens, as in prompts: two launches, on the tensor
// cores (tcgen05, kind::f16) with everything that is large brought by tensor copies.
//
//   S = A_a x      adapters_down_kernel: a cluster of CTAs per tile of 128 tokens of one adapter, split along K; D[token, rank] in
//                  tensor memory for all ranks at once, so X is read once whatever the rank.  What bounds it is X from HBM and A from
//                  L2 (again for every tile: the reason for 128 tokens).  Partial sums meet in distributed shared memory, in a
//                  fixed order, each CTA finishing its share of the tokens.
//   out = Y + B S  adapters_up_kernel: a CTA per tile and a range of channels, 64 at a time, D[token, channel]; bound by Y, read and
//                  written once.  Y and B come through a ring; eight warps, alternately four to a block, add a block's sums to Y where
//                  it lies in shared memory, a token to a thread, and write whole 128-byte lines from there.
//
// A tile's tokens lie anywhere in the batch.  Where they follow one another (a prompt), copies take 32 rows at a time, else four
// rows by number (tile::gather4).  Threads that fetched the rows 16 bytes at a time took 15 cycles an instruction and SM, which
// bound both kernels (4096 tokens of 6 adapters, ranks to 64, 4096 x 4096: 47 us, now 31.2, where the bytes take 16.2; 2048 tokens of
// 5, ranks to 128, 14336 -> 4096: 43.9, bytes 14.9; 501 tokens of 8, ranks to 32, 4096 -> 28672: 27.6, bytes 11.3).
//
// Every wait is bounded; a warp that gives up leaves NaN in what it would have written, and its CTA sets the plan's status word.
#include "adapters.cuh"
#include "sm100_ptx.cuh"

namespace aser {

namespace {

constexpr int kTok = kTileMany, kMaxCL = 12, kGather = 8, kBox = 32;
constexpr int kCols = 64;                            // columns or channels of a stage: 128 bytes a row
constexpr int kRowsBytes = kTok * kCols * 2;
constexpr int kMaxStages = 8;
constexpr long long kWaitClocks = 400000000ll;       // about 0.2 s of SM clocks per wait

// False after the limit, or when another warp of this CTA gave up.
__device__ __forceinline__ bool bounded_wait(uint32_t bar, uint32_t parity, volatile int* stop) {
    long long t0 = 0;
    for (uint32_t spins = 0; !mbar_try_wait(bar, parity); ++spins)
        if ((spins & 255u) == 255u) {
            if (*stop) return false;
            const long long now = clock64();
            if (t0 == 0) t0 = now;
            else if (now - t0 > kWaitClocks) { *stop = 1; return false; }
        }
    return true;
}
// One lane polls.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* stop, int lane) {
    int ok = 1;
    if (lane == 0) ok = bounded_wait(bar, parity, stop) ? 1 : 0;
    return __shfl_sync(0xffffffffu, ok, 0) != 0;
}
// Copies in flight land before a CTA that gave up lets go of its shared memory.
__device__ __forceinline__ void let_copies_land() {
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000) {}
}

// A tile's rows of a matrix, 64 columns from `col`, by one warp.
struct TileRows {
    int first_token;       // >= 0: the tokens follow one another from here
    int count;
    int4 four;             // else the numbers of tokens 4 lane .. 4 lane + 3 (the first one's in the place of those that are not there)
    __device__ __forceinline__ int rows() const { return first_token >= 0 ? (count + kBox - 1) / kBox * kBox : (count + 3) / 4 * 4; }
    __device__ __forceinline__ void load(uint32_t dst, const CUtensorMap* box, const CUtensorMap* one, int col, uint32_t bar, int lane) const {
        if (first_token >= 0) {
            if (lane * kBox < count) tma_load_2d(dst + lane * kBox * 128, box, col, first_token + lane * kBox, bar);
        } else if (lane * 4 < count) {
            tma_gather4(dst + lane * 512, one, col, four.x, four.y, four.z, four.w, bar);
        }
    }
};
__device__ __forceinline__ TileRows tile_rows(const int4& t4, const int32_t* tokens, int lane) {
    TileRows r;
    r.first_token = t4.w;
    r.count = t4.z;
    r.four = make_int4(0, 0, 0, 0);
    if (t4.w < 0) {
        const int32_t* list = tokens + t4.y;
        const int i = lane * 4, zero = list[0];
        r.four = make_int4(i < t4.z ? list[i] : zero, i + 1 < t4.z ? list[i + 1] : zero, i + 2 < t4.z ? list[i + 2] : zero,
                           i + 3 < t4.z ? list[i + 3] : zero);
    }
    return r;
}

__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void tmem_alloc(uint32_t* slot, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}

// ---------------------------------------------------------------------------
// S = A x
// ---------------------------------------------------------------------------
constexpr int kDownThreads = 256, kDownWarps = 8;

struct DownMaps { CUtensorMap x, x_one, a, a_big; };

// The ring also holds the partial sums at the end, [128][rank + 4] floats.  Up to rank 128 two CTAs fit on an SM, so that clusters
// beyond those that have SMs of their own need not wait for a second turn (CTAs with an SM's shared memory each, 36 clusters of four
// where 35 fit: 41.5 us instead of 35.2 for the call above), and a CTA of the second kernel fits beside one of these.
constexpr int kDownTail = 2 * kMaxStages * 8 + 32;   // barriers, tensor memory's address, flag
__host__ __device__ constexpr int down_smem(int r) { return (r <= 128 ? 112 : 224) * 1024; }
__host__ __device__ constexpr int down_room(int r) { return down_smem(r) - kDownTail - 1024; }
static_assert(2 * (down_smem(128) + 1024) <= 228 * 1024, "two CTAs to an SM");
static_assert(down_room(128) >= 3 * (kRowsBytes + 128 * 128) && down_room(256) >= 4 * (kRowsBytes + 256 * 128), "a ring");
static_assert(down_room(128) >= kTok * 132 * 4 && down_room(256) >= kTok * 260 * 4, "partial sums");

__global__ void __launch_bounds__(kDownThreads, 2)
adapters_down_kernel(const __grid_constant__ DownMaps maps, const AdapterParams p, uint32_t tmem_cols) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + down_room(p.r));             // [stage]: filled, free
    uint64_t* done = bars + 2 * kMaxStages;                                          // all products are complete
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
    volatile int* stop = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == 0) {
        tmem_alloc(tmem_slot, tmem_cols);
    } else if (warp == 1) {
        if (lane < 2 * kMaxStages + 1) mbar_init(smem_u32(bars + lane), 1);
        if (lane == 0) *stop = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async_smem();
    } else if (warp == 2 && lane == 0) {
        prefetch_tensormap(&maps.x);
        prefetch_tensormap(&maps.a);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot, sb = smem_u32(smem), bar0 = smem_u32(bars);
    auto filled = [&](int s) { return bar0 + 16u * s; };
    auto free_ = [&](int s) { return bar0 + 16u * s + 8u; };
    grid_dep_wait();
    grid_dep_launch();
    warm_ranks(p);
    const int CL = (int)cluster_size(), rank = (int)cluster_rank(), tile = (int)blockIdx.x / CL;
    const PlanView plan = plan_view(p.plan, p.M, p.n_slots);
    const int4 head = *reinterpret_cast<const int4*>(p.plan);
    const int4 t4 = plan.tiles_many[tile];
    const bool real = head.x == p.M && head.y == p.n_slots && tile < head.w;
    const int slot = real ? t4.x : -1, first = t4.y, count = t4.z;
    const int rk = slot < 0 ? 0 : adapter_rank(p, slot);
    if (rk > 0) {                     // (the whole cluster)
        const int steps = p.K / kCols, s0 = rank * steps / CL, n = (rank + 1) * steps / CL - s0;
        // as many stages as there is room for; they are as large as the tile's tokens and the adapter's rank ask.  (The products
        // read X as 128 rows: behind the tile's tokens whatever lies there, sums that nobody reads.)
        const int row_bytes = (count + kBox - 1) / kBox * kBox * 128, stage_bytes = row_bytes + rk * 128;
        const int fit = (down_room(p.r) - (kRowsBytes - row_bytes)) / stage_bytes, stages = fit < kMaxStages ? fit : kMaxStages;
        if (warp == 0) {              // copies
            const TileRows rows = tile_rows(t4, plan.tokens, lane);
            const uint32_t bytes = (uint32_t)(rows.rows() + rk) * 128u;
            for (int i = 0, s = 0, turn = 0; i < n; ++i) {
                if (turn > 0 && !warp_wait(free_(s), (uint32_t)(turn - 1) & 1u, stop, lane)) break;
                if (lane == 0) mbar_arrive_expect_tx(filled(s), bytes);
                __syncwarp();
                const uint32_t at = sb + (uint32_t)(s * stage_bytes);
                const int col = (s0 + i) * kCols;
                rows.load(at, &maps.x, &maps.x_one, col, filled(s), lane);
                // A in boxes of 64 ranks, then of 16 (600 x 14336 x 4096, rank 256: 35.3 -> 30.0 us; of 16 alone, a stage is that many more copies)
                const int big = rk >> 6;
                if (lane < big + ((rk >> 4) & 3)) {
                    const int j = lane < big ? lane * 64 : big * 64 + (lane - big) * 16;
                    tma_load_2d(at + row_bytes + j * 128, lane < big ? &maps.a_big : &maps.a, col, slot * p.r + j, filled(s));
                }
                if (++s == stages) { s = 0; ++turn; }
            }
        } else if (warp == 1) {       // products (rows that are not there are whatever the ring holds: nobody reads their sums)
            const uint32_t idesc = make_idesc(1, 0, 128, rk);
            for (int i = 0, s = 0, turn = 0; i < n; ++i) {
                if (!warp_wait(filled(s), (uint32_t)turn & 1u, stop, lane)) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t at = sb + (uint32_t)(s * stage_bytes);
                    const uint64_t xd = smem_desc_sw128(at), ad = smem_desc_sw128(at + row_bytes);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) mma_f16_ss(tmem, xd + 2 * kk, ad + 2 * kk, idesc, (i | kk) != 0 ? 1u : 0u);
                    tc_commit(free_(s));
                    if (i == n - 1) tc_commit(smem_u32(done));
                }
                __syncwarp();
                if (++s == stages) { s = 0; ++turn; }
            }
        }
        bool ok = true;
        if (n > 0) ok = warp_wait(smem_u32(done), 0u, stop, lane);
        __syncthreads();                  // the ring is free
        if (*stop) {
            ok = false;
            if (threadIdx.x == 0) report_give_up(p);
            let_copies_land();
        }
        tc_fence_after();
        // partial sums [128 tokens][rk + 4]
        float* part = reinterpret_cast<float*>(smem);
        const int stride = rk + 4;
        for (int c = (warp >> 2) * 16; c < rk; c += 32) {
            uint32_t v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = 0u;
            if (n > 0) {
                tmem_ld16(tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)c, v);
                tmem_wait_ld(v);
            }
            uint4* q = reinterpret_cast<uint4*>(part + ((warp & 3) * 32 + lane) * stride + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t nan = 0x7fffffffu;
                q[e] = ok ? make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]) : make_uint4(nan, nan, nan, nan);
            }
        }
        tc_fence_before();
        cluster_arrive();
        cluster_wait();
        const int per = (kTok + CL - 1) / CL;
        const float alpha = p.scale ? __ldg(p.scale + slot) : 1.f;
        auto gather = [&](int row, int j) {
            const uint32_t at = smem_u32(part + row * stride + j);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int q0 = 0; q0 < CL; q0 += kGather) {
                float4 a[kGather];
#pragma unroll
                for (int q = 0; q < kGather; ++q) a[q] = q0 + q < CL ? ld_cluster_f32x4(map_to_rank(at, q0 + q)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int q = 0; q < kGather; ++q) { v.x += a[q].x; v.y += a[q].y; v.z += a[q].z; v.w += a[q].w; }
            }
            return v;
        };
        auto gather2 = [&](int row, int step, int j, const bool (&mine)[2], float4 (&v)[2]) {
            v[0] = v[1] = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int q0 = 0; q0 < CL; q0 += kGather) {
                float4 a[2][kGather];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t at = smem_u32(part + (mine[u] ? row + u * step : 0) * stride + j);
#pragma unroll
                    for (int q = 0; q < kGather; ++q)
                        a[u][q] = q0 + q < CL && mine[u] ? ld_cluster_f32x4(map_to_rank(at, q0 + q)) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int q = 0; q < kGather; ++q) { v[u].x += a[u][q].x; v[u].y += a[u][q].y; v[u].z += a[u][q].z; v[u].w += a[u][q].w; }
            }
        };
        if (rk <= 64) {                   // two tokens side by side, twice
            const int j = (lane & 15) * 4;
            for (int i0 = warp * 2; i0 < per; i0 += 4 * kDownWarps) {
                float4 v[2];
                bool mine[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int i = i0 + u * 2 * kDownWarps + (lane >> 4);
                    mine[u] = i < per && rank * per + i < count && j < rk;
                }
                gather2(rank * per + i0 + (lane >> 4), 2 * kDownWarps, j, mine, v);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int row = rank * per + i0 + u * 2 * kDownWarps + (lane >> 4);
                    float top = max4_abs(v[u]);
#pragma unroll
                    for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const RowFactor f = row_factor(top);
                    if (mine[u]) *reinterpret_cast<uint2*>(p.S + (size_t)(first + row) * p.r + j) = scaled_f16(v[u], f.up);
                    if (mine[u] && j == 0) p.row_scale[first + row] = f.down * alpha;
                }
            }
        } else {
            for (int i = warp; i < per && rank * per + i < count; i += kDownWarps) {
                const int row = rank * per + i;
                float4 v[2];
                float top = 0.f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v[h] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (h * 128 + lane * 4 < rk) v[h] = gather(row, h * 128 + lane * 4);
                    top = fmaxf(top, max4_abs(v[h]));
                }
                const RowFactor f = row_factor(warp_max(top));
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (h * 128 + lane * 4 < rk)
                        *reinterpret_cast<uint2*>(p.S + (size_t)(first + row) * p.r + h * 128 + lane * 4) = scaled_f16(v[h], f.up);
                if (lane == 0) p.row_scale[first + row] = f.down * alpha;
            }
        }
        cluster_arrive();                 // nobody leaves while a peer may still read its sums
        cluster_wait();
        tc_fence_after();
    }
    if (warp == 0) tmem_free(tmem, tmem_cols);
}

// ---------------------------------------------------------------------------
// out = Y + B S
// ---------------------------------------------------------------------------
constexpr int kUpWarps = 10, kUpThreads = kUpWarps * 32;      // copies, products, twice four that finish blocks in turn

struct UpMaps { CUtensorMap y, y_one, s, b, out; };

__host__ __device__ constexpr int up_chunks(int r) { return (r + 63) / 64; }          // blocks of 64 ranks
// Shared memory of a CTA: S, then as many stages as there is room for; they are as large as the tile's tokens and the adapter's
// rank ask (128 tokens of rank 64: four, 64 tokens: six).  Up to rank 128 two CTAs share an SM.
constexpr int kUpTail = 256;
__host__ __device__ constexpr int up_smem(int r) { return (r <= 128 ? 112 : 224) * 1024; }
static_assert(up_smem(128) - kUpTail - 1024 >= up_chunks(128) * kTok * 128 + 2 * (kRowsBytes + up_chunks(128) * kCols * 128), "two stages at least");
static_assert(up_smem(256) - kUpTail - 1024 >= up_chunks(256) * kTok * 128 + 2 * (kRowsBytes + up_chunks(256) * kCols * 128), "two stages at least");
constexpr int kUpSums = 4;                            // blocks whose sums are in tensor memory at once
constexpr uint32_t kUpTmem = kUpSums * kCols;

// Blocks of 64 channels [c n / chunks, (c + 1) n / chunks) of a tile; `resident` CTAs are dealt over the tiles that there are.  What wrote Y and the plan is known to be complete when this
// kernel starts, because the first kernel waited for it; S is waited for.  Whatever a CTA of a tile has to do, it waits for the first
// kernel before it ends: who waits for this kernel has waited for both.
__global__ void __launch_bounds__(kUpThreads, 2)
adapters_up_kernel(const __grid_constant__ UpMaps maps, const AdapterParams p, int resident) {
    extern __shared__ uint8_t smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    warm_ranks(p);
    const PlanView plan = plan_view(p.plan, p.M, p.n_slots);
    const int4 head = *reinterpret_cast<const int4*>(p.plan), more = *reinterpret_cast<const int4*>(p.plan + 4);
    const int tiles = p.Y == p.out ? more.x : head.w;        // (in place, those without an adapter, the last ones, have nothing to do)
    if (head.x != p.M || head.y != p.n_slots || tiles == 0) { grid_dep_wait(); return; }
    const int blocks = (p.N + kCols - 1) / kCols;
    int chunks = resident / tiles;                           // (two blocks and more for a CTA)
    chunks = chunks < 1 ? 1 : chunks > (blocks + 1) / 2 ? (blocks + 1) / 2 : chunks;
    const int tile = (int)blockIdx.x / chunks, chunk = (int)blockIdx.x - tile * chunks;
    if (tile >= tiles) return;
    const int4 t4 = plan.tiles_many[tile];
    const int slot = t4.x, first = t4.y, count = t4.z;
    const int32_t* tokens = plan.tokens + first;
    const int rk = slot < 0 ? 0 : adapter_rank(p, slot);
    const int b0 = (int)((long long)chunk * blocks / chunks), n = (int)((long long)(chunk + 1) * blocks / chunks) - b0;
    if (rk == 0) {                        // nothing to add
        if (p.Y != p.out)
            for (int row = warp; row < count; row += kUpWarps) {
                const size_t tok = (size_t)tokens[row];
                for (int c = b0 * kCols + lane * 8; c < (b0 + n) * kCols && c < p.N; c += 256)
                    *reinterpret_cast<uint4*>(p.out + tok * p.ldo + c) = *reinterpret_cast<const uint4*>(p.Y + tok * p.ldy + c);
            }
        grid_dep_wait();
        return;
    }
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    // (the products read S as 128 rows: behind the tile's tokens whatever lies there, sums that nobody reads)
    const int kch = up_chunks(rk), row_bytes = (count + kBox - 1) / kBox * kBox * 128, s_bytes = (kch - 1) * row_bytes + kTok * 128;
    const int stage_bytes = row_bytes + kch * kCols * 128, room = up_smem(p.r) - kUpTail - 1024;
    const int fit = (room - s_bytes) / stage_bytes, stages = fit < kMaxStages ? fit : kMaxStages;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + room);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kMaxStages + 2 * kUpSums + 1);
    volatile int* stop = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const uint32_t sb = smem_u32(smem), bar0 = smem_u32(bars);
    auto filled = [&](int s) { return bar0 + 8u * s; };                 // a stage's Y and B are there
    auto free_ = [&](int s) { return bar0 + 8u * (kMaxStages + s); };   // ... and have been read (four warps)
    auto read = [&](int h) { return bar0 + 8u * (2 * kMaxStages + h); };        // a block's sums have been read (four warps)
    auto full = [&](int h) { return bar0 + 8u * (2 * kMaxStages + kUpSums + h); };    // ... are complete
    constexpr int kBars = 2 * kMaxStages + 2 * kUpSums + 1;
    static_assert(kBars <= 32 && kBars * 8 + 8 <= kUpTail, "barriers");
    const uint32_t s_there = bar0 + 8u * (kBars - 1);
    if (warp == 0) {
        tmem_alloc(tmem_slot, kUpTmem);
    } else if (warp == 1) {
        if (lane < kBars) mbar_init(bar0 + 8u * lane, lane >= kMaxStages && lane < 2 * kMaxStages + kUpSums ? 4 : 1);
        if (lane == 0) *stop = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async_smem();
    } else if (warp == 2 && lane == 0) {
        prefetch_tensormap(&maps.y);
        prefetch_tensormap(&maps.b);
        prefetch_tensormap(&maps.s);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (warp == 0) {                      // copies
        const TileRows rows = tile_rows(t4, plan.tokens, lane);
        const uint32_t bytes = (uint32_t)rows.rows() * 128u + (uint32_t)kch * kCols * 128u;
        bool asked = false;
        auto ask_for_s = [&]() {          // once the ring is full: this waits for the first kernel
            asked = true;
            grid_dep_wait();
            if (lane == 0) mbar_arrive_expect_tx(s_there, (uint32_t)(kch * row_bytes));
            __syncwarp();
            const int boxes = row_bytes / (kBox * 128);
            if (lane < kch * boxes) tma_load_2d(sb + lane * kBox * 128, &maps.s, lane / boxes * 64, first + lane % boxes * kBox, s_there);
        };
        for (int i = 0, s = 0, turn = 0; i < n; ++i) {
            if (i == stages) ask_for_s();
            if (turn > 0 && !warp_wait(free_(s), (uint32_t)(turn - 1) & 1u, stop, lane)) break;
            if (lane == 0) mbar_arrive_expect_tx(filled(s), bytes);
            __syncwarp();
            const uint32_t at = sb + (uint32_t)(s_bytes + s * stage_bytes);
            const int ch = (b0 + i) * kCols;
            rows.load(at, &maps.y, &maps.y_one, ch, filled(s), lane);
            if (lane < kch) tma_load_2d(at + row_bytes + lane * kCols * 128, &maps.b, lane * 64, slot * p.N + ch, filled(s));
            if (++s == stages) { s = 0; ++turn; }
        }
        if (!asked) ask_for_s();
        grid_dep_launch();
    } else if (warp == 1) {               // products
        const uint32_t idesc = make_idesc(1, 0, 128, kCols);
        bool ok = warp_wait(s_there, 0u, stop, lane);
        for (int i = 0, s = 0, turn = 0; i < n && ok; ++i) {
            const int h = i % kUpSums;
            ok = warp_wait(filled(s), (uint32_t)turn & 1u, stop, lane);
            if (ok && i >= kUpSums) ok = warp_wait(read(h), (uint32_t)(i / kUpSums - 1) & 1u, stop, lane);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t at = sb + (uint32_t)(s_bytes + s * stage_bytes) + row_bytes;
                for (int k = 0; k < rk; k += 16) {
                    const uint64_t sd = smem_desc_sw128(sb + (k >> 6) * row_bytes) + 2 * ((k >> 4) & 3);
                    const uint64_t bd = smem_desc_sw128(at + (k >> 6) * kCols * 128) + 2 * ((k >> 4) & 3);
                    mma_f16_ss(tmem + h * kCols, sd, bd, idesc, k != 0 ? 1u : 0u);
                }
                tc_commit(full(h));
            }
            __syncwarp();
            if (++s == stages) { s = 0; ++turn; }
        }
    } else {
        const int q = warp & 3;           // a quarter of the tokens (of tensor memory's lanes), every other block
        const int row = q * 32 + lane;
        grid_dep_wait();                  // the factors come from the first kernel
        const float factor = row < count ? p.row_scale[first + row] : 0.f;
        // lines are written by eight lanes each: this lane's 16 bytes of rows q 32 + lane / 8, + 4, ...
        const int wr = q * 32 + (lane >> 3), wc = lane & 7;
        int out_tok[8];
        uint32_t there = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            out_tok[e] = wr + 4 * e < count ? tokens[wr + 4 * e] : 0;
            there |= wr + 4 * e < count ? 1u << e : 0u;
        }
        const bool box = t4.w >= 0 && (q + 1) * 32 <= count;
        bool ok = true;
        for (int i = (warp - 2) >> 2; i < n; i += 2) {
            const int s = i % stages, h = i % kUpSums;
            const uint32_t at = sb + (uint32_t)(s_bytes + s * stage_bytes);
            if (ok) ok = warp_wait(filled(s), (uint32_t)(i / stages) & 1u, stop, lane);
            if (ok) ok = warp_wait(full(h), (uint32_t)(i / kUpSums) & 1u, stop, lane);
            if (ok && q * 32 < count) {
                tc_fence_after();
#pragma unroll
                for (int c0 = 0; c0 < 8; c0 += 4) {
                    uint32_t v[2][16];
                    tmem_ld16(tmem + h * kCols + ((uint32_t)(q * 32) << 16) + c0 * 8, v[0]);
                    tmem_ld16(tmem + h * kCols + ((uint32_t)(q * 32) << 16) + c0 * 8 + 16, v[1]);
                    uint4 y[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        y[c] = make_uint4(0, 0, 0, 0);
                        if (row < count)
                            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(y[c].x), "=r"(y[c].y), "=r"(y[c].z), "=r"(y[c].w)
                                         : "r"(at + (uint32_t)(row * 128 + (((c0 + c) ^ (row & 7)) << 4))) : "memory");
                    }
                    tmem_wait_ld_all();
                    tmem_use(v[0]);
                    tmem_use(v[1]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (row >= count) break;
                        uint32_t yw[4] = {y[c].x, y[c].y, y[c].z, y[c].w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&yw[e]));
                            const int j = (c & 1) * 8 + 2 * e;
                            yw[e] = pack_half2(fmaf(__uint_as_float(v[c >> 1][j]), factor, f.x), fmaf(__uint_as_float(v[c >> 1][j + 1]), factor, f.y));
                        }
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at + (uint32_t)(row * 128 + (((c0 + c) ^ (row & 7)) << 4))),
                                     "r"(yw[0]), "r"(yw[1]), "r"(yw[2]), "r"(yw[3]) : "memory");
                    }
                }
                tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(read(h));
            const int ch = (b0 + i) * kCols;
            if (box && ok) {              // 32 rows that follow one another: one tensor store, which clips at N
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    tma_store_2d_tile(&maps.out, ch, t4.w + q * 32, at + (uint32_t)(q * 32 * 128));
                    bulk_store_commit();
                    // (giving the place back only with this warp's next block cost more in copies not yet asked for)
                    bulk_store_wait_read();
                    mbar_arrive(free_(s));
                }
                continue;
            }
            const bool in = ch + wc * 8 < p.N;
            uint4 o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int r = wr + 4 * e;
                o[e] = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
                if (ok && (there >> e & 1))
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(o[e].x), "=r"(o[e].y), "=r"(o[e].z), "=r"(o[e].w)
                                 : "r"(at + (uint32_t)(r * 128 + ((wc ^ (r & 7)) << 4))) : "memory");
            }
            fence_proxy_async_smem();     // the next copy into this place comes after these reads and writes
            __syncwarp();
            if (lane == 0) mbar_arrive(free_(s));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (in && (there >> e & 1)) *reinterpret_cast<uint4*>(p.out + (size_t)out_tok[e] * p.ldo + (ch + wc * 8)) = o[e];
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*stop) {
        if (threadIdx.x == 0) report_give_up(p);
        let_copies_land();
    }
    if (warp == 0) tmem_free(tmem, kUpTmem);
}

// Tiles that a call probably has (the host does not know which adapters are in use): a quarter of them leave a short one.
int likely_tiles(const AdapterParams& p) { return (p.M + kTok - 1) / kTok + (p.n_slots < p.M ? p.n_slots : p.M) / 4; }

// Boxes of `box` rows by 64 columns, 128 bytes a row, of an fp16 matrix.
int rows_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t box) {
    return encode_map_2d_ld(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, rows, cols, ld, box, kCols, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <typename Kernel>
int opt_in(Kernel* kernel, int bytes, bool (&configured)[kMaxDevices], int* num_sms) {
    int dev = 0;
    int rc = current_device(&dev);
    if (rc == ASER_OK) rc = device_sm_count(num_sms);
    if (rc != ASER_OK || configured[dev]) return rc;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return record_cuda_error(e, "adapters smem attribute");
    configured[dev] = true;
    return ASER_OK;
}

}  // namespace

int launch_adapters_down(const AdapterParams& p, cudaStream_t st) {
    static bool configured[kMaxDevices] = {false};
    int num_sms = 0;
    int rc = opt_in(adapters_down_kernel, down_smem(256), configured, &num_sms);
    if (rc != ASER_OK) return rc;
    DownMaps maps;
    rc = rows_map(&maps.x, p.X, p.M, p.K, p.ldx, kBox);
    if (rc == ASER_OK) rc = rows_map(&maps.x_one, p.X, p.M, p.K, p.ldx, 1);
    if (rc == ASER_OK) rc = rows_map(&maps.a_big, p.A, (uint64_t)p.n_slots * p.r, p.K, p.K, 64);
    if (rc == ASER_OK) rc = rows_map(&maps.a, p.A, (uint64_t)p.n_slots * p.r, p.K, p.K, 16);
    if (rc != ASER_OK) return rc;
    // CTAs for one and a half times the SMs that there are (two share one up to rank 128, and what bounds a CTA is the bytes that it
    // has in flight; more, and the last clusters of a few hundred wait for places: 4096 tokens of 6, 4096 x 4096, rank 64, 1.1 times 32.9
    // us, 1.5 30.9, 2 37.6), from 2 steps of K each; clusters above eight for long K only (2048 x 14336 x 4096, rank 128: by 8 45.4, by 12 43.6;
    // 1500 x 8192 x 1024, rank 64, 34.6 / 29.3; 1024 x 4096 x 4096 17.4 / 18.2).
    int CL = (p.r <= 128 ? num_sms * 3 / 2 : num_sms * 11 / 10) / likely_tiles(p);
    const int most = p.K >= 7680 ? kMaxCL : 8;
    CL = CL > most ? most : CL;
    CL = CL > p.K / kCols / 2 ? p.K / kCols / 2 : CL;
    CL = CL < 1 ? 1 : CL;
    uint32_t cols = 32;
    while ((int)cols < p.r) cols *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(plan_tiles(p.M, p.n_slots, kTok) * CL, 1, 1);
    cfg.blockDim = dim3(kDownThreads, 1, 1);
    cfg.dynamicSmemBytes = down_smem(p.r);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CL; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, adapters_down_kernel, maps, p, cols);
    if (e != cudaSuccess) return record_cuda_error(e, "adapters_down_kernel");
    return check_launch("adapters_down_kernel");
}

int launch_adapters_up(const AdapterParams& p, cudaStream_t st) {
    static bool configured[kMaxDevices] = {false};
    int num_sms = 0;
    int rc = opt_in(adapters_up_kernel, up_smem(256), configured, &num_sms);
    if (rc != ASER_OK) return rc;
    UpMaps maps;
    rc = rows_map(&maps.y, p.Y, p.M, p.N, p.ldy, kBox);
    if (rc == ASER_OK) rc = rows_map(&maps.y_one, p.Y, p.M, p.N, p.ldy, 1);
    if (rc == ASER_OK) rc = rows_map(&maps.s, p.S, p.M, p.r, p.r, kBox);
    if (rc == ASER_OK) rc = rows_map(&maps.b, p.B, (uint64_t)p.n_slots * p.N, p.r, p.r, kCols);
    if (rc == ASER_OK) rc = rows_map(&maps.out, p.out, p.M, p.N, p.ldo, kBox);
    if (rc != ASER_OK) return rc;
    const int resident = (p.r <= 128 ? 2 : 1) * num_sms, bound = plan_tiles(p.M, p.n_slots, kTok);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(resident > bound ? resident : bound, 1, 1);
    cfg.blockDim = dim3(kUpThreads, 1, 1);
    cfg.dynamicSmemBytes = up_smem(p.r);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, adapters_up_kernel, maps, p, resident);
    if (e != cudaSuccess) return record_cuda_error(e, "adapters_up_kernel");
    return check_launch("adapters_up_kernel");
}

}  // namespace aser
