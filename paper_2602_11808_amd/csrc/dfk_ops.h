// Linear layers and the mixture of experts: arguments, scratch layouts and launchers shared by their files.
#pragma once

#include "dfk_internal.h"

namespace dfk {

// What a product's epilogue does with the fp32 sums of row m and column n:
//   kEpiLinear  Y[m,n] = act(sum + bias[n]) + resid[m,n]
//   kEpiGated   two products of the same row; A_2[r,n] = SiLU(gate) * up * weight of the row
//   kEpiRows    P[slot of the row, n] = sum: fp32, or in bf16 calls half times a power of two per 64 columns
enum { kEpiLinear = 0, kEpiGated = 1, kEpiRows = 2 };

// Launches a kernel and gives that launch's own status: hipGetLastError would also report what another call in the process left behind.
template <typename... P, typename... A>
hipError_t launch_kernel(void (*kernel)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t st, A... args) {
    static_assert(sizeof...(P) == sizeof...(A), "an argument for each parameter");
    return [&](P... p) {
        void* ptrs[] = {(void*)&p...};
        return hipLaunchKernel((const void*)kernel, grid, block, ptrs, lds, st);
    }(args...);
}

// The rows of a mixture of experts, one for each (token, expert) pair of a chunk of tokens ("slot" t * top_k + k), gathered by
// expert; filled in on the device (launch_moe_plan).
constexpr int kTakenPitch = 32;       // (a cache line each)
struct MoePlan {
    int* n_tiles;     // number of row tiles
    int4* tiles;      // of a row tile: expert, first row, rows (1 to tile_rows)
    int* counts;      // [workgroup of the plan][expert] slots
    int* slot;        // [rows] slot of a row
    float* weight;    // [rows] weight of a row (an expert that a token lists twice: one row, both weights)
    int* taken;       // [16] kTakenPitch apart: tiles taken of each eighth of a product's, of gate/up and down
    int tile_rows;
    int max_tiles;    // more there cannot be
};

// Few tokens: entry y of up to kMoeFewSlots is an expert (or the expert of slot y) and the slots it has.
struct MoeFewArgs {
    const void* X;
    const int* experts;
    const float* weights;
    const void* Wg;
    const void* Wu;
    const void* Wd;        // [n_experts, d_model, d_ff]
    const void* resid;
    void* Y;
    int M, n_experts, top_k, d_model, d_ff;
    int by_slot;           // entries are the slots (the first of an expert's counts), else the experts
    int entries;
    int2* entry;           // expert, number of its slots (0: nothing)
    int* rows;             // [entries][M] its slots
    void* a2;              // [slots][d_ff]
    int down_groups;       // workgroups of the down projection that share 16 columns
    unsigned* tickets;     // [columns / 16] arrival counters, and
    float* partial;        // [down_groups][M][d_model] partial sums, where there are several
};
constexpr int kMoeFewTokens = 64, kMoeFewSlots = 256;      // at most

struct TileArgs {
    const void* A;         // activations [.., K]
    const void* B;         // weights [N, K] of a group; kEpiGated: gate rows
    const void* B2;        // kEpiGated: up rows
    void* out;
    const void* bias;      // kEpiLinear
    const void* resid;
    int M, N, K;           // M: rows of A where there is one group
    int act;               // dfk_act_t
    int vec4;              // four columns of out, bias and resid can be moved at once
    int out_fp32;          // kEpiLinear: type of out and resid is fp32, else that of the operands
    int splits;            // kEpiLinear: k splits whose partial sums a launch of its own adds up (1: none)
    float* partial;        // [split][M][pitch]
    float* scale;          // kEpiRows of bf16 calls: [slot][columns / 64, rounded up]
    size_t partial_bytes;  // what there is of it
    int pitch;             // N rounded up to a multiple of 4
    int alone;             // experts: most have one row tile, so their weights are read by one workgroup each
    int top_k;             // experts: row r of A is token slot / top_k (kEpiGated), else row r itself
    MoePlan plan;
};

// the fp32 type, any shape (dfk_tile_f32.hip)
hipError_t launch_linear_f32(const TileArgs& a, hipStream_t st);
hipError_t launch_experts_f32(const TileArgs& a, int epi, hipStream_t st);
constexpr int kTileRowsF32 = 64;

// 16-bit operands on the matrix cores, many rows (dfk_tile_linear.hip, dfk_tile_moe.hip)
hipError_t launch_linear_tile(const TileArgs& a, dfk_dtype_t dtype, int tile, hipStream_t st);
hipError_t launch_linear_sum(const TileArgs& a, dfk_dtype_t dtype, hipStream_t st);      // the k splits' partial sums, then the epilogue
hipError_t launch_experts_tile(const TileArgs& a, dfk_dtype_t dtype, int epi, hipStream_t st);

// 16-bit operands on the matrix cores, few rows (dfk_linear_stream.hip)
hipError_t launch_linear_stream(const TileArgs& a, dfk_dtype_t dtype, int nt, hipStream_t st);

// experts with few tokens (dfk_moe_few.hip)
hipError_t launch_moe_few(const MoeFewArgs& a, dfk_dtype_t dtype, hipStream_t st);

}  // namespace dfk
