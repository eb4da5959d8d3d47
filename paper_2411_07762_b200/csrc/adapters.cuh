// The plan of a batch's adapters (adapters.cu): tokens by adapter, cut into tiles of one adapter each.
//   words 0 .. 7   M, n_slots, tiles of kTileFew tokens, tiles of kTileMany tokens, those of the latter with an
//                  adapter, tokens with an adapter, status (not 0: a wait of a call since the plan was made gave up), 0
//   tiles of 16    {adapter or -1, first place in the list of tokens, tokens, 0, their numbers [16]}: one round of loads
//   tiles of 128   {adapter or -1, first place, tokens, the first token's number if they follow one another, else -1}
//   tokens         [M] token numbers by adapter, those without one last
#pragma once
#include "aser_common.cuh"

namespace aser {

constexpr int kTileFew = 16, kTileMany = 128;

constexpr int kFewWords = 4 + kTileFew, kPlanStatusWord = 6;

struct PlanView {
    int32_t* tiles_few;       // kFewWords each
    int4* tiles_many;
    int32_t* tokens;
    long long words;
};

// A group leaves at most one short tile of either size.
__host__ __device__ inline int plan_tiles(int M, int n_slots, int tile) { return M / tile + (n_slots + 1 < M ? n_slots + 1 : M); }

__host__ __device__ inline PlanView plan_view(const int32_t* plan, int M, int n_slots) {
    int32_t* w = const_cast<int32_t*>(plan);
    const long long few = plan_tiles(M, n_slots, kTileFew), many = plan_tiles(M, n_slots, kTileMany);
    PlanView v;
    v.tiles_few = w + 8;
    v.tiles_many = reinterpret_cast<int4*>(w + 8 + kFewWords * few);
    v.tokens = w + 8 + kFewWords * few + 4 * many;
    v.words = 8 + kFewWords * few + 4 * many + M;
    return v;
}

struct AdapterParams {
    const __half* X;
    const __half* A;          // [slots, r, K]
    const __half* B;          // [slots, N, r]
    const int32_t* ranks;     // [slots] or NULL
    const float* scale;       // [slots] or NULL
    const int32_t* plan;
    const __half* Y;
    __half* out;
    __half* S;                // between the two kernels for many tokens: [M, r] by place in the plan's list, scaled,
    float* row_scale;         // and [M] what its rows are to be multiplied by
    size_t ldx, ldy, ldo;
    int M, N, K, r, n_slots;
    int parts;                // few tokens: clusters per tile, each with its own part of N
};

size_t adapters_plan_bytes(int M, int n_slots);
int launch_adapters_plan(const int32_t* slot, int M, int n_slots, void* plan, cudaStream_t st);
// Whether a call runs the two kernels for many tokens, and the workspace that it then needs.
bool adapters_many(int M, int N, int K, int r, int n_slots);
size_t adapters_workspace_bytes(int M, int N, int K, int r, int n_slots);
// (p.S and p.row_scale are set from `workspace`.)
int launch_adapters(AdapterParams p, void* workspace, cudaStream_t st);
int launch_adapters_down(const AdapterParams& p, cudaStream_t st);
int launch_adapters_up(const AdapterParams& p, cudaStream_t st);

#ifdef __CUDACC__
// (by any number of threads: all write the same)
__device__ __forceinline__ void report_give_up(const AdapterParams& p) { const_cast<volatile int32_t*>(p.plan)[kPlanStatusWord] = 1; }
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// Which adapter a tile has is known one round trip later than where its rank stands: the list is asked for meanwhile (a
// thread per 32 bytes: the first 2048 adapters), so that the look-up finds it near.
__device__ __forceinline__ void warm_ranks(const AdapterParams& p) {
    const int i = (int)threadIdx.x * 8;
    int v;
    if (p.ranks && i < p.n_slots) asm volatile("ld.global.nc.s32 %0, [%1];" : "=r"(v) : "l"(p.ranks + i));
    float f;
    if (p.scale && i < p.n_slots) asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(f) : "l"(p.scale + i));
}
// The rank of an adapter: a multiple of 16 from 0 to r.
__device__ __forceinline__ int adapter_rank(const AdapterParams& p, int slot) {
    const int rk = p.ranks ? __ldg(p.ranks + slot) : p.r;
    return (rk < 0 ? 0 : rk > p.r ? p.r : rk) & ~15;
}
__device__ __forceinline__ float max4_abs(const float4& v) {
    return fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w)));
}
// Powers of two that bring a row whose largest magnitude is `top` to [2^14, 2^15) and back; an infinite, NaN or tiny one
// keeps factors that are normal numbers.
struct RowFactor { float up, down; };
__device__ __forceinline__ RowFactor row_factor(float top) {
    int e = (int)(__float_as_uint(top) >> 23) - 127;
    e = e < -100 ? -100 : e > 127 ? 127 : e;
    return {__uint_as_float((uint32_t)(127 + 14 - e) << 23), __uint_as_float((uint32_t)(127 - 14 + e) << 23)};
}
__device__ __forceinline__ uint2 scaled_f16(const float4& v, float f) {
    const __half2 lo = __floats2half2_rn(v.x * f, v.y * f), hi = __floats2half2_rn(v.z * f, v.w * f);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}
// Eight outputs: y + factor * the sums of row half h of four tiles.
__device__ __forceinline__ uint4 add_scaled(const uint4& y, const float (&acc)[4][4], int h, float factor) {
    const uint32_t yw[4] = {y.x, y.y, y.z, y.w};
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&yw[j]));
        const __half2 v = __floats2half2_rn(fmaf(acc[j][2 * h], factor, f.x), fmaf(acc[j][2 * h + 1], factor, f.y));
        o[j] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}
#endif

}  // namespace aser
