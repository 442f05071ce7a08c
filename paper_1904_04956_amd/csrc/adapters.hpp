// Low-rank adapters of the sequences of a batch beside a projection that they share: launchers (adapters.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include "gemm.hpp"

namespace blstm {

constexpr int ADAPT_MAX_RANK = 128, ADAPT_MAX_COUNT = 4096;

struct AdaptShape { int T, B, K, N, rank, count; float scale; };

// Which sequences share an adapter, made on the device from ids: the sequences sorted by adapter, tiles of `rows` rows and, for the sums over rows,
// chunks of `chunk` rows, none of them of two adapters.  The rows of an adapter: its sequences in order, each one's T frames.  Keys: the adapters, count
// for sequences without one, count + 1 for ids out of range.
struct AdaptPlan {
    int rows, chunk;          // rows of a tile and of a chunk (0: no chunks)
    int max_tiles, max_chunks;
    size_t counts, perm, first, tiles, chunks, first_chunk, bytes;      // byte offsets from the plan's start
};
// Batches of few sequences need no plan for adapt_project.
inline bool adapt_finds(const AdaptShape& s) { return s.B <= 256; }
// counts: {tiles, chunks}; first [count + 3]: a key's first place in perm; first_chunk [count + 1]; tiles and chunks: {key, first row, its rows, first place in perm}
AdaptPlan adapt_plan(const AdaptShape& s, int rows, int chunk);
// Whether each launch of a call has fewer than 2^32 threads, which is what a grid holds.
bool adapt_fits(const AdaptShape& s, const AdaptPlan& p, bool backward);
// Rows of a chunk of the gradients' sums: about 64 chunks if one adapter has all rows, at most ADAPT_MAX_CHUNK rows each.
constexpr int ADAPT_MAX_CHUNK = 1024;
inline int adapter_chunk_rows(const AdaptShape& s) { const long long M = (long long)s.T * s.B, r = (M + 4095) / 4096 * 64; return (int)(r < ADAPT_MAX_CHUNK ? r : ADAPT_MAX_CHUNK); }
// Rows of a tile of y (backward: of dx): 16 where such tiles are few, 128 where the adapters' rows fill several such tiles, else 64.  16 against 64 rows, us, at W
// workgroups of 16 rows x 32 columns (K 1024 or 640, N 256), bf16: W 104 10.5 and 14.3; 544 15.0 and 18.3; 896 26.3 and 19.4; 1040 41 and 20.5; float: 104 11 and 38; 544 22 and 57;
// 1008 43 and 61; 1376 60 and 41.  The whole backward pass in float, whose contraction is short: 672 32 and 35, 840 34.7 and 33.7, 893 (of 67, no whole words) 39 and 29.
inline int adapter_tile_rows(const AdaptShape& s, bool backward, DType type) {
    const long long M = (long long)s.T * s.B, groups = s.B < s.count + 1 ? s.B : s.count + 1;
    return (M / 16 + groups) * (((backward ? s.K : s.N) + 31) / 32) <= (type == DT_BF16 || backward ? 640 : 1024) ? 16 : M >= 512 * groups && M >= 16384 ? 128 : 64;
}
hipError_t launch_adapt_plan(const AdaptShape& s, const AdaptPlan& p, const int32_t* ids, char* plan, hipStream_t st);

// y [M][N] = x [M][K] W^T + b + scale t B_a^T, t [M][rank] = x A_a^T.  W [N][K], A [count][rank][K], Bm [count][N][rank].
struct ProjectArgs {
    AdaptShape s;
    AdaptPlan p;
    const char* plan;                    // null: every workgroup finds its tile in ids itself (adapt_finds)
    const int32_t* ids;
    const void *x, *W, *b, *A, *Bm;      // b null: none
    void* y;                             // null: only t is wanted
    float* t;                            // null: not wanted
};
hipError_t launch_adapt_project(const ProjectArgs& a, DType type, hipStream_t st);

// W^T [K][N], A_a^T [K][rank], B_a^T [rank][N] of all adapters, and the plan in the same launch
struct TransposeArgs { AdaptShape s; const void *W, *A, *Bm; void *Wt, *At, *Bt; };
hipError_t launch_adapt_transpose(const TransposeArgs& a, const AdaptPlan& p, const int32_t* ids, char* plan, DType type, hipStream_t st);

// dA_a [rank][K] = scale sum q^T x, dB_a [N][rank] = scale sum dy^T t over an adapter's rows; zero for an adapter without any
struct AdaptGradArgs {
    AdaptShape s;
    AdaptPlan p;
    const char* plan;
    const void *x, *dy;
    const float *q, *t;                  // [M][rank]
    float* part;                         // [chunks][rank][K + N]
    float *dA, *dB;
};
hipError_t launch_adapt_grad(const AdaptGradArgs& a, DType type, hipStream_t st);

}  // namespace blstm
