// The plan of a batch's adapters (adapters.cu): tokens by adapter, cut into tiles of one adapter each.
//   words 0 .. 3   M, n_slots, tiles of kTileFew tokens, tiles of kTileMany tokens
//   tiles          {adapter or -1, first place in the list of tokens, tokens, 0}, both sizes
//   tokens         [M] token numbers by adapter, those without one last
#pragma once
#include "aser_common.cuh"

namespace aser {

constexpr int kTileFew = 16, kTileMany = 64;

struct PlanView {
    int4 *tiles_few, *tiles_many;
    int32_t* tokens;
    long long words;
};

// A group leaves at most one short tile of either size.
__host__ __device__ inline int plan_tiles(int M, int n_slots, int tile) { return M / tile + (n_slots + 1 < M ? n_slots + 1 : M); }

__host__ __device__ inline PlanView plan_view(const int32_t* plan, int M, int n_slots) {
    int32_t* w = const_cast<int32_t*>(plan);
    const long long few = plan_tiles(M, n_slots, kTileFew), many = plan_tiles(M, n_slots, kTileMany);
    PlanView v;
    v.tiles_few = reinterpret_cast<int4*>(w + 4);
    v.tiles_many = reinterpret_cast<int4*>(w + 4 + 4 * few);
    v.tokens = w + 4 + 4 * (few + many);
    v.words = 4 + 4 * (few + many) + M;
    return v;
}

size_t adapters_plan_bytes(int M, int n_slots);
int launch_adapters_plan(const int32_t* slot, int M, int n_slots, void* plan, cudaStream_t st);
int launch_adapters(const __half* X, size_t ldx, const __half* A, const __half* B, const int32_t* ranks, const float* scale,
                    const void* plan, int M, int N, int K, int r, int n_slots, const __half* Y, size_t ldy, __half* out,
                    size_t ldo, cudaStream_t st);

}  // namespace aser
