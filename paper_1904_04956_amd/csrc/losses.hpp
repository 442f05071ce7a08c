// Launchers of the softmax layer's operators beyond cross-entropy (losses.hip, losses_rows.hip).  All pointers are device pointers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include "gemm.hpp"

namespace blstm {

constexpr int LOSS_STRIP = 64;                       // classes of one partial sum of a row
constexpr int LOSS_MAX_TOP = 256;                    // BLSTM_MAX_TOP of the C header

// What a row's dE/du is made of: du_v = a exp2(u_v log2e - m2) + at exp2(u_v log2e / tau - mt2) - hot [v = label].
// A row that counts for nothing has a = at = hot = 0, label = -1 and m2 = mt2 = +inf.
struct LossRow {
    float m2, a, mt2, at;
    float hot;
    int label;
    float max;                                       // of the row's logits
    float pad;                                       // (two 16-byte loads)
};

// u log2e - m2 is one multiply-add, whose m2 = max log2e is rounded: the same for all classes of a row, so that it cancels, but 2^-24 of
// itself off.  From LOSS_FAR on (the type's lowest value as a bias rules a class out, and with it whole strips) it is (u - max) log2e.
constexpr float LOSS_FAR = 1e5f;

// The policy loss of one frame: present or absent old / reference log-probabilities, where the ratio is clipped, weight of the KL term.
struct PolicyArgs {
    const float* advantage;
    const float* old_logp;                           // null: the weights that sampled are the present ones, ratio 1
    const float* ref_logp;                           // null: no KL term
    float clip_low, clip_high, kl_weight;
};
// A teacher's list: [M][K]; entries with class -1 or value -inf are not used.
struct TeacherArgs {
    const float* values;
    const int32_t* classes;
    int K;
    float inv_tau, hard, soft;                       // 1/tau, weights of the two terms (soft: times tau^2 in the loss, tau in the gradient)
    float tau;
};

// Rows ahead of the products: zc = z with the rows that count for nothing set to zero, rows of ldzc elements, zeros behind Z.
// bf16 (the float rows hold their logits, see launch_loss_rows_f32): the label's logit, the entries' logits, q and the row's sum q (log q - (u - ref) / tau).
struct LossPrepArgs {
    const void* z;
    void* zc;                                        // or null: not wanted
    bool keep;                                       // rows that count for nothing are copied as they are
    int M, V, Z, ldzc;
    int twice;                                       // (bf16) zc is written a second time behind the first
    const unsigned short* W;                         // rows of ldzc elements, zeros behind Z; null: only zc is wanted
    const unsigned short* bias;
    float* bias_f;                                   // [V rounded up to 64] the bias as floats, bias_pad behind it; or null
    float bias_pad;
    const int32_t* labels;                           // or null
    float* label_logit;                              // [M]
    TeacherArgs teacher;                             // K = 0: none
    float* entry_logit;                              // [M][K]
    float* entry_q;                                  // [M][K], 0: not used; of entries with one class, the first has all
    float* soft_const;                               // [M] sum q (log q - (u - ref) / tau), then [M] ref
    int* soft_state;                                 // [M]: bit 0: some entry is used; bit 1: some class is out of range, or its value NaN or infinite (the loss is NaN)
};
hipError_t launch_loss_prep(const LossPrepArgs& a, DType type, hipStream_t st);

// bf16: the logits' tiles straight into what is wanted of them; the matrix itself is not written.
struct LossTileArgs {
    const unsigned short* z;                         // [M][ld], zeros in columns Z .. ld - 1
    const unsigned short* W;                         // [V][ld], likewise
    const unsigned short* bias;
    int M, V, ld;                                    // ld: a multiple of eight, at least Z
    float inv_tau;                                   // of the second sum (0: none)
    float* part_max;                                 // [strips][M] maximum of a strip's logits
    float* part_sum;                                 // [strips][M] sum of exp2(u log2e - max log2e)
    float* part_sum_tau;                             // [strips][M] the same at the temperature
    const LossRow* rows;                             // gradient: [M]
    unsigned short* hi;                              // [M][ldu] du rounded to bf16, zeros in columns V .. ldu - 1
    unsigned short* lo;                              // [M][ldu] what the rounding left, rounded; with third, [M][ldu] of what that left behind it
    int third;
    long long ldu;
    float* logits;                                   // [M][ldu]
};
inline int loss_strips(int V) { return (V + 2 * LOSS_STRIP - 1) / (2 * LOSS_STRIP) * 2; }
hipError_t launch_loss_stats(const LossTileArgs& a, hipStream_t st);
hipError_t launch_loss_grad(const LossTileArgs& a, hipStream_t st);
hipError_t launch_loss_logits(const LossTileArgs& a, hipStream_t st);   // logits and part_max

// z of up to 256, bf16 (losses_fused.hip).
constexpr int LOSS_FUSED_WIDTH = 256;
struct LossFusedArgs {
    const unsigned short* z;                         // [M][ld], zeros in columns Z .. ld - 1
    const unsigned short* W;                         // [V][ld], likewise
    const float* bias;                               // [V rounded up to 64], -inf beyond V
    const float* consts;                             // [6][Mp]: LossRow's m2, a, mt2, at, then minus all of du at the label, the label (as bits); rows M .. Mp - 1 count for nothing
    int M, Mp, V, Z, ld;                             // Mp: M rounded up to 64
    float k1, k;                                     // scale of the first exponential, and of the second (rows, sums not known: the only one)
    int parts;                                       // of the classes (rows kernel) or of the rows (classes kernel), a workgroup each
    float* out;                                      // rows: [parts][M][ld]; classes: [parts][V][ldo], columns 0 .. Z - 1
    const int32_t* labels;                           // [M] rows (sums not known), sums at two scales: the label's class stays out; launch_loss_dz, launch_loss_merge add it; or null
    const uint32_t* marks;                           // rows: [loss_mark_words(V)][Mr], a bit a class that stays out of the product; launch_loss_dz adds it; or null: the label's alone
    int Mr;                                          // M rounded up to 256
    float* part_ref;                                 // rows, sums not known: [parts][M] reference and sum
    float* part_sum;
    float* part_sum2;                                // sums: at the scale k
    float* out_db;                                   // classes: [parts][V]
    const float* row_loss;                           // classes: [M], whose sum goes to loss[0]
    float* loss;
    const uint2* entries;                            // classes: the teacher's, row | class << 6 within a tile and weight q, by tiles of 64 rows and 128 classes; or null
    const int* entries_from;                         // [tiles] where a tile's lie, and how many
    const int* entries_count;
    long long ldo;
    int vec;                                         // classes: rows of out take 16-byte stores
    int third;                                       // classes: a third part of du where a teacher's classes are
};
hipError_t launch_loss_fused_rows(const LossFusedArgs& a, bool known, hipStream_t st);   // known: the two distributions' sums
// The rows' sums alone at the scale k1 and, with second, k from references part_ref (a logit); or, with logits, u into out [M][ldo] (ldo a multiple
// of four; NaN behind V counts as no maximum) and the maxima of strips of 64 classes into part_ref [strips][M].
hipError_t launch_loss_fused_sums(const LossFusedArgs& a, bool second, bool logits, hipStream_t st);
hipError_t launch_loss_fused_classes(const LossFusedArgs& a, bool tau, hipStream_t st);
// dz from the parts of launch_loss_fused_rows and the label's and the teacher's classes, in float; with known false the rows' losses and
// constants too.
struct LossDzArgs {
    int M, Mp, V, Z, ld, parts;
    const float* part;
    const float* part_ref;
    const float* part_sum;
    const unsigned short* W;                         // rows of ld
    const int32_t* labels;
    const float* label_logit;
    float s;
    const PolicyArgs* policy;                        // host pointers: one of the two
    const TeacherArgs* teacher;
    const float* entry_logit;                        // [M][K], of entries with a probability
    const float* entry_q;
    const float* soft_const;
    const int* soft_state;
    float* logp;                                     // or null
    float* row_loss;
    float* consts;                                   // as in LossFusedArgs
    unsigned short* dz;                              // [M][Z]
};
hipError_t launch_loss_dz(const LossDzArgs& a, bool known, hipStream_t st);
// The teacher's entries by tiles, from the tiles' counts, and the marks of the rows kernel.  entries: room for M K, and 256 more that are read.
constexpr int LOSS_LIST_SLACK = 256;
__host__ __device__ inline int loss_mark_words(int V) { return (V + 63) / 64 * 2; }
struct LossListArgs {
    int M, V, K;
    const int32_t* classes;
    const float* q;                                  // [M][K], 0: none
    float weight;
    int* count;                                      // [tiles], the rows' tiles one after the other
    int* from;                                       // [tiles]
    uint2* entries;
    const int32_t* labels;                           // or null
    uint32_t* marks;                                 // [loss_mark_words(V)][Mr]
    int Mr;
};
hipError_t launch_loss_lists(const LossListArgs& a, hipStream_t st);
// out = sum of parts of n floats, out_b of V, in order.
hipError_t launch_loss_classes_sum(const float* p, const float* pb, int parts, long long n, int V, float* out, float* out_b, hipStream_t st);

// Joins the strips of every row, then what the call wants of a row: logp, loss term, LossRow (null: not wanted).
struct LossMergeArgs {
    int M, V, strips;
    const float* part_max;
    const float* part_sum;
    const float* part_sum_tau;                       // or null
    const int32_t* labels;
    const float* label_logit;
    float s;                                         // loss scale
    const PolicyArgs* policy;                        // host pointers: exactly one of the two, or neither (log-probabilities)
    const TeacherArgs* teacher;
    const float* soft_const;
    const int* soft_state;
    float* logp;
    float* row_loss;
    LossRow* rows;                                   // or
    float* consts;                                   // as in LossFusedArgs, rows M .. Mp - 1 too; the sums then lack the label's class
    int Mp;
};
hipError_t launch_loss_merge(const LossMergeArgs& a, hipStream_t st);

// The teacher's entries in du: each rounded to its parts from p' - q in float.
struct LossEntriesArgs {
    const LossRow* rows;
    const int32_t* classes;
    const float* entry_logit;
    const float* entry_q;
    float inv_tau, weight;                           // weight: s soft tau
    int M, V, K;
    unsigned short* hi;
    unsigned short* lo;
    long long ldu;
    int third;                                       // as in LossTileArgs
};
hipError_t launch_loss_entries(const LossEntriesArgs& a, hipStream_t st);
// dz, rounded, from the product of du's first part in float and, of the second, the label's and the teacher's classes.
struct LossDzEndArgs {
    int M, Z, ld, K;                                 // K 0: no teacher
    const float* dz_f;                               // [M][ld]
    const LossRow* rows;
    const int32_t* classes;                          // [M][K]
    const float* entry_q;                            // [M][K], 0: none
    const unsigned short* lo;
    long long ldu;
    const unsigned short* W;                         // [V][ld]
    unsigned short* dz;                              // [M][Z]
};
hipError_t launch_loss_dz_end(const LossDzEndArgs& a, hipStream_t st);

// float: everything of a row from its logits u [M][ldu], which dE/du overwrites (gradient false: they stay).
struct LossRowsArgs {
    float* u;
    long long ldu;
    int M, V;
    float s;
    const int32_t* labels;
    const PolicyArgs* policy;                        // host pointers, as above
    const TeacherArgs* teacher;
    bool gradient;
    float* logp;
    float* row_loss;
};
hipError_t launch_loss_rows_f32(const LossRowsArgs& a, hipStream_t st);

// The K largest of every row of u [M][ldu] with their columns, by falling value, equal ones by rising column, NaN last.  part_max
// [strips][M]: maxima of strips of LOSS_STRIP columns (NaN: nothing but NaN), or, with have_max false, room for them; at most LOSS_TOP_STRIPS strips.
constexpr int LOSS_TOP_STRIPS = 1024;
hipError_t launch_row_topk(const float* u, long long ldu, int M, int V, int K, float* part_max, bool have_max, float* values, int32_t* classes, hipStream_t st);
// The same without strips, for any V.
hipError_t launch_row_topk_wide(const float* u, long long ldu, int M, int V, int K, float* values, int32_t* classes, hipStream_t st);

}  // namespace blstm
