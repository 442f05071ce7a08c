// The orthogonalised update: plan and launcher (muon.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

namespace blstm {

constexpr int MUON_MAX_GROUPS = 10;

// `count` tensors of one shape in a flat vector: tensor k starts at element at + (k / inner_count) outer + (k % inner_count) inner.
struct MuonGroup {
    long long at, outer, inner;
    int inner_count, count, rows, cols;
    bool ortho;               // its update is orthogonalised; else the tensor takes the plain momentum update
    // The rest is the plan's.  A matrix lies in scratch in halves, zero-padded to rp x cp; its Gram matrix has mp rows.  The second plane
    // of each (what the first one's rounding left over) lies xplane or splane elements behind the first.
    int rp, cp, mp, tall, splits;
    long long x[2], s, b, xplane, splane;      // elements of 2 bytes from the scratch's start
    long long diag;                            // of the diagonals of S, then of B: float elements from their start, count x mp each
    long long part;                            // float elements from the partial sums' start
    int chunks, casts;                         // the flat passes' units of a tensor
    int grams, applies;                        // product tiles of a matrix: on and above the diagonal, all
};
// Where each group's units begin in a launch (INT_MAX behind the last group): side by side, so that a workgroup finds its group with one wait.
struct MuonStarts { int chunk[MUON_MAX_GROUPS], cast[MUON_MAX_GROUPS], gram[MUON_MAX_GROUPS], square[MUON_MAX_GROUPS], apply[MUON_MAX_GROUPS], sum[MUON_MAX_GROUPS]; };
struct MuonPlan {
    MuonGroup g[MUON_MAX_GROUPS];
    MuonStarts at;
    int n;
    int tile;                 // 0: 64 x 64 tiles, 1: 128 x 128, 2: 128 x 128 and, in the last product, 256 x 128;
                              // 3: a matrix a workgroup, all in LDS (small: blocks of 16 rows of the largest Gram matrix, lds: bytes)
    int small, lds;
    int lone;                 // no more tiles of S than CUs: two sets of wavefronts a tile
    int exact;                // products of both planes
    int chunks, casts, grams, squares, applies, sums;
    size_t sums_at, diag_at, part_at, here_at, bytes;   // byte offsets in scratch: squares' sums (double), diagonals, partial Gram tiles (float), whether a matrix is in ids (int)
};
struct MuonArgs {
    float* theta; unsigned short* shadow;      // null: the update itself goes to out
    const float* grad; float* velocity;        // velocity null: grad is what is orthogonalised
    void* out; int out_bf16;
    float lr, lr_rest, momentum, decay; int nesterov;
};
struct MuonIds { const int* ids; int n; };     // ids not null: of the call's only group, the matrices that ids holds; the others stay as they are
// False: sizes beyond what the kernels index.  g[].at .. ortho are given.
bool muon_plan(const MuonGroup* g, int n, bool exact, MuonPlan* out);
hipError_t launch_muon(const MuonPlan& p, const MuonArgs& a, const MuonIds& ids, void* scratch, hipStream_t st);

}  // namespace blstm
