// The softmax layer's losses for z of up to 256, bf16 operands: dE/du and the logits exist in registers only.
//
//   rows      a workgroup keeps 256 rows of z in registers and walks over the classes: u = W_s z + b_s, then sum_v w_v W_v with
//             w = exp(u - reference) and their sum (the reference moves with the running maximum), or with w = dE/du itself
//             where the sums are known.  The label's and the teacher's classes, few a row, stay out and are added behind it, in float.
//   classes   a workgroup keeps 128 classes of W_s in registers and walks over the rows: dE/du from the rows' sums, then
//             dW_s = du^T z and db_s.  du goes into the product as the sum of two bf16 numbers (2^-16; of three where a label is, and
//             where a teacher's classes are and frames are few), into db_s as the float that it is.
//
// Why so: M rows of V float logits are written, read and written again by anything that keeps them (688 MB for 5376 rows of 32000, at
// 4.8 TB/s as long as the whole product takes); made twice, they cost a product of M V Z each.  In dz a weight is one bf16
// number, whose rounding (2^-8) the result's own rounding to bf16 matches.  Of a label's or a teacher's class du is a difference of probabilities: where
// the model is good, far smaller than they are and than what a rounded probability would be off.
//
// Bound by the matrix units' turns with the rest of a wavefront: two wavefronts a SIMD, each of which multiplies, takes its
// exponentials, transposes and multiplies again; the other covers part of it.  Z = 256, V = 32000, 43008 rows (705 GFLOP a unit of
// M V Z; the matrix units reach 1.66 PFLOP/s from registers): rows 1130 us (two units, 1.25 PFLOP/s), classes 1650 us (three, 1.28);
// 3633 rows: 122 and 168 us.  Two distributions (5376 rows, lists of 64): sums 112, rows 188 (176 without the marks), classes 335 us.  At 168 .. 336 rows
// the parts of dz and the loads of W_s weigh as much: rows 21 .. 29 us, classes 26 .. 34.
//
// Both read a tile [64][Z] in LDS twice: by rows for the logits (ds_read_b128) and by columns for what is made of them
// (ds_read_b64_tr_b16 transposes on the way).  16-byte chunk c of row r lies at chunk c ^ sw(r): the eight rows that a phase
// of the first reads, and the four of the second, are on different banks.  The output of the first product (lane: row or
// class, registers: the other) is the operand of the second after one exchange between the lane halves.
#include "gemm_tile.hpp"
#include "losses_terms.hpp"

namespace blstm {
namespace {

constexpr float SLACK = 8.0f;                           // powers of two by which a weight may pass one before the reference moves

__device__ __forceinline__ int sw(int r) { return ((r & 3) << 1) | ((r >> 2) & 1); }

// The lane's number, made anew: kept across a loop, or what follows from it ahead of one, it would take registers that there are not.
__device__ __forceinline__ int fresh_lane() {
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
    return l;
}

// A ring of tiles of 64 rows, NK slabs of 64 columns, loaded by eight wavefronts straight into LDS.
template <int NK>
struct Ring {
    static constexpr int CPR = 8 * NK, ROWB = 128 * NK, TILE = 64 * ROWB, STAGE = TILE + 2048, STAGES = 3;
    static constexpr int LIST = 2048;                   // bytes of a teacher's entries behind it, where there are any
    static constexpr int MARK = 2048;                   // ... and of 256 rows' marks
    static __device__ __forceinline__ void dma16(unsigned lds, const char* base, unsigned voff) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(base) : "memory");
    }
    static __device__ __forceinline__ void dma4(unsigned lds, const char* base, unsigned voff) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(base) : "memory");
    }
    // rows first .. first + 63 of p (those beyond `rows` repeat the last one, chunks beyond a row's end its last chunk)
    static __device__ __forceinline__ void tile(unsigned lds, const bf16_t* p, int first, int rows, int ld, int wv) {
        const unsigned lane = (unsigned)fresh_lane();
        const char* base = reinterpret_cast<const char*>(p + (long long)first * ld);
        const int last = rows - 1 - first, lastc = ld / 8 - 1;
#pragma unroll
        for (int j = 0; j < NK; ++j) {
            const unsigned i = (unsigned)(j * 8 + wv) * 64u + lane, x = i % CPR;
            const int r = (int)(i / CPR), c = (int)(x & ~7u) | ((int)(x & 7u) ^ sw(r));
            dma16(lds + (unsigned)((j * 8 + wv) * 1024), base, (unsigned)(__mul24(min(r, last), ld * 2) + min(c, lastc) * 16));
        }
    }
};

// A lane's reads of a tile.  By rows: chunk 2 q + half of row l32 is at row ^ 32 (q % 4), 128 (q / 4) on.  By columns: of sixteen rows,
// columns 32 zb .., the first four of each eight at col ^ 64 (zb % 2), 128 (zb / 2) on, the other four 4 rows and chunk ^ 1 on.
template <int NK>
struct Reads {
    int row, col;
    __device__ __forceinline__ Reads(int lane) {
        const int l32 = lane & 31, half = lane >> 5, li = lane & 15, g = lane >> 4;
        row = l32 * Ring<NK>::ROWB + ((half ^ sw(l32)) << 4);
        const int r = 8 * half + (li >> 2), x = (2 * (g & 1) + ((li & 3) >> 1)) ^ ((li >> 2) << 1);
        col = r * Ring<NK>::ROWB + (x << 4) + (li & 1) * 8;
    }
    __device__ __forceinline__ uint4 by_row(const char* s, int q) const { return *reinterpret_cast<const uint4*>(s + (row ^ ((q & 3) << 5)) + 128 * (q >> 2)); }
    __device__ __forceinline__ uint4 by_col(const char* s, int zb) const {
        const char* p = s + (col ^ ((zb & 1) << 6)) + 128 * (zb >> 1);
        const char* p4 = s + (col ^ ((zb & 1) << 6) ^ 16) + 128 * (zb >> 1) + 4 * Ring<NK>::ROWB;
        const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)p));
        const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)p4));
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
};

__device__ __forceinline__ f32x16_t mma32(const uint4& a, const uint4& b, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Eight values of a lane, packed, at 8 (e / 4) + 4 half + e % 4 of sixteen, as the operand of a product over the sixteen.
__device__ __forceinline__ uint4 fragment(const unsigned (&p)[4]) {
    const auto a = __builtin_amdgcn_permlane32_swap(p[0], p[2], false, false), b = __builtin_amdgcn_permlane32_swap(p[1], p[3], false, false);
    return make_uint4(a[0], b[0], a[1], b[1]);
}

// The order of a block of N operands read from LDS and multiplied: FIRST reads, then MMA products and READS reads in turn, DEPTH operands
// ahead (the compiler puts each read in front of its product, whose wait is then all of the LDS's latency).
template <int FIRST, int N, int MMA, int READS, int DEPTH>
__device__ __forceinline__ void ahead() {
    __builtin_amdgcn_sched_group_barrier(0x100, FIRST, 0);
    each<0, N - DEPTH>([](auto) { __builtin_amdgcn_sched_group_barrier(0x8, MMA, 0); __builtin_amdgcn_sched_group_barrier(0x100, READS, 0); });
    __builtin_amdgcn_sched_group_barrier(0x8, MMA * DEPTH, 0);
}
constexpr int DEPTH = 4;

// ---- rows -------------------------------------------------------------------------------------------------------------------
// KNOWN: w = a exp2(u log2e - m2) + at exp2(u k - mt2) from the rows' constants, else w = exp2(u k - reference).
// The label counts as ruled out.  MARKS: the teacher's classes stay out of the product; they are marked, a bit a class (the label's too), and the marks come
// with the tile.  They are in the sum, with the same product's logits as all others: with those of the lists, another product's, the rows' sums and the classes
// kernel, which makes p' - q of them, were 2.5e-5 apart where the two are close, and are 7e-6.
template <int NK, bool KNOWN, bool MARKS>
__global__ __launch_bounds__(512, 2) void loss_rows_kernel(LossFusedArgs a) {
    typedef Ring<NK> R;
    constexpr int STAGE = R::STAGE + (MARKS ? R::MARK : 0), LOADS = NK + 1 + (MARKS ? 1 : 0);
    extern __shared__ uint4 smem[];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int part = (int)blockIdx.x % a.parts, row0 = (int)blockIdx.x / a.parts * 256;
    const int ntv = (a.V + 63) / 64, per = (ntv + a.parts - 1) / a.parts, t0 = part * per, n = min(per, ntv - t0);
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    const Reads<NK> at(lane);
    const int m = row0 + wv * 32 + l32;
    uint4 zf[4 * NK];
#pragma unroll
    for (int q = 0; q < 4 * NK; ++q) {
        const int c = 2 * q + half;
        zf[q] = c * 8 < a.ld ? *reinterpret_cast<const uint4*>(a.z + (long long)min(m, a.M - 1) * a.ld + c * 8) : make_uint4(0, 0, 0, 0);
    }
    float m2 = 0.0f, ca = 0.0f, mt2 = 0.0f, cat = 0.0f;
    if (KNOWN && m < a.Mp) {
        m2 = a.consts[m]; ca = a.consts[a.Mp + m]; mt2 = a.consts[2 * a.Mp + m]; cat = a.consts[3 * a.Mp + m];
    }
    const int label = !KNOWN && a.labels && m < a.M ? a.labels[m] : -1;
    __builtin_amdgcn_s_waitcnt(0);                      // (known to the compiler: it would wait for these loads, and the ring's with them, in the loop)
    auto issue = [&](int it) __attribute__((always_inline)) {
        const unsigned s = lds0 + (unsigned)(it % R::STAGES * STAGE);
        R::tile(s, a.W, (t0 + it) * 64, a.V, a.ld, wv);
        R::dma4(s + R::TILE, reinterpret_cast<const char*>(a.bias + (long long)(t0 + it) * 64), (unsigned)(fresh_lane() * 4));
        if constexpr (MARKS) {                           // the wavefront's 32 rows, two words each
            const int ln = fresh_lane();
            R::dma4(s + R::STAGE + (unsigned)(wv * 256), reinterpret_cast<const char*>(a.marks + (long long)(t0 + it) * 2 * a.Mr + row0 + wv * 32), (unsigned)(((ln >> 5) * a.Mr + (ln & 31)) * 4));
        }
    };
    f32x16_t o[2 * NK];
#pragma unroll
    for (int zb = 0; zb < 2 * NK; ++zb)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[zb][e] = 0.0f;
    // (below every logit that is not ruled out)
    const float k = a.k;
    float ref = -LOSS_FAR * k, sum = 0.0f;
    if (n > 0) issue(0);
    if (n > 1) issue(1);
    for (int it = 0; it < n; ++it) {
        if (it + 1 < n) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (it + 2 < n) issue(it + 2);                  // (over tile it - 1, which every wavefront is done with)
        const char* stage = reinterpret_cast<const char*>(smem) + it % R::STAGES * STAGE;
        const float* bias = reinterpret_cast<const float*>(stage + R::TILE);
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            const char* s = stage + sub * 32 * R::ROWB;
            f32x16_t u;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 b = *reinterpret_cast<const float4*>(bias + sub * 32 + 8 * g + 4 * half);
                u[4 * g] = b.x; u[4 * g + 1] = b.y; u[4 * g + 2] = b.z; u[4 * g + 3] = b.w;
            }
#pragma unroll
            for (int q = 0; q < 4 * NK; ++q) u = mma32(at.by_row(s, q), zf[q], u);
            unsigned out = 0;                            // (bit 8 (e / 4) + e % 4: class e of the lane stays out)
            if constexpr (MARKS) out = *reinterpret_cast<const unsigned*>(stage + R::STAGE + wv * 256 + sub * 128 + (fresh_lane() & 31) * 4);
            ahead<4 + (MARKS ? 1 : 0) + DEPTH, 4 * NK, 1, 1, DEPTH>();
            unsigned ruled = out;
            if constexpr (!KNOWN) {
                const unsigned at_label = (unsigned)(label - ((t0 + it) * 64 + sub * 32));
                ruled = at_label < 32u ? 1u << at_label : 0u;
            }
            if (__any(ruled != 0)) {
                ruled >>= 4 * half;
#pragma unroll
                for (int e = 0; e < 16; ++e) u[e] = ruled & 1u << (8 * (e >> 2) + (e & 3)) ? -INFINITY : u[e];
            }
            if constexpr (!KNOWN) {
                if (MARKS) out >>= 4 * half;
                float mx = u[0];
#pragma unroll
                for (int e = 1; e < 16; ++e) mx = fmaxf(mx, u[e]);
                if (__any(mx * k > ref + SLACK)) {
                    const float now = fmaxf(ref, fmaxf(mx, __shfl_xor(mx, 32, 64)) * k), scale = __builtin_amdgcn_exp2f(ref - now);
                    ref = now;
                    sum *= scale;
#pragma unroll
                    for (int zb = 0; zb < 2 * NK; ++zb)
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[zb][e] *= scale;
                }
            }
            uint4 f[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {               // sixteen classes, a step of the second product
                unsigned p[4];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    float w[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float x = u[8 * t + e + i];
                        if constexpr (KNOWN) {
                            w[i] = ca * __builtin_amdgcn_exp2f(fmaf(x, a.k1, -m2));
                            w[i] = fmaf(cat, __builtin_amdgcn_exp2f(fmaf(x, k, -mt2)), w[i]);
                        } else {
                            w[i] = __builtin_amdgcn_exp2f(fmaf(x, k, -ref));
                            sum += w[i];
                            if (MARKS) w[i] = out & 1u << (8 * (2 * t + (e >> 2)) + (e & 3) + i) ? 0.0f : w[i];
                        }
                    }
                    p[e / 2] = pack2(w[0], w[1]);
                }
                f[t] = fragment(p);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int zb = 0; zb < 2 * NK; ++zb) o[zb] = mma32(at.by_col(s + t * 16 * R::ROWB, zb), f[t], o[zb]);
            ahead<2 * DEPTH, 4 * NK, 1, 2, DEPTH>();
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (m >= a.M) return;
    const long long to = (long long)part * a.M + m;
#pragma unroll
    for (int zb = 0; zb < 2 * NK; ++zb)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int z = zb * 32 + 8 * g + 4 * half;
            if (z < a.ld) *reinterpret_cast<float4*>(a.out + to * a.ld + z) = make_float4(o[zb][4 * g], o[zb][4 * g + 1], o[zb][4 * g + 2], o[zb][4 * g + 3]);
        }
    if (!KNOWN) {
        sum += __shfl_xor(sum, 32, 64);
        if (half == 0) { a.part_ref[to] = ref; a.part_sum[to] = sum; }
    }
}

// ---- rows, the sums alone -----------------------------------------------------------------------------------------------------
// Reference and sum of exponentials of every row and part (SUMS2: at two scales, from one reference, without the label's class), or the
// logits themselves with the maxima of strips of 64 classes (LOGITS).  5376 rows of 32000, Z = 256 (88 GFLOP): 90 us (980 TFLOP/s), SUMS2
// 112 (106 with the label in its sums), LOGITS 230, whose 688 MB are stored at 3 TB/s (past L2 or with loads that do not wait for them no faster).  Two workgroups a CU, four wavefronts a SIMD, so that some multiply while others take exponentials.
// Rows as in the rows kernel: of the 128 x 128 tiles that larger z take, both operands come from L2 for half the products.
enum { SUMS, SUMS2, LOGITS };
template <int NK, int WHAT>
__global__ __launch_bounds__(512, 4) void loss_sums_kernel(LossFusedArgs a) {
    typedef Ring<NK> R;
    extern __shared__ uint4 smem[];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int part = (int)blockIdx.x % a.parts, row0 = (int)blockIdx.x / a.parts * 256;
    const int ntv = (a.V + 63) / 64, per = (ntv + a.parts - 1) / a.parts, t0 = part * per, n = min(per, ntv - t0);
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    const Reads<NK> at(lane);
    const int m = row0 + wv * 32 + l32;
    uint4 zf[4 * NK];
#pragma unroll
    for (int q = 0; q < 4 * NK; ++q) {
        const int c = 2 * q + half;
        zf[q] = c * 8 < a.ld ? *reinterpret_cast<const uint4*>(a.z + (long long)min(m, a.M - 1) * a.ld + c * 8) : make_uint4(0, 0, 0, 0);
    }
    const int label = WHAT == SUMS2 && m < a.M ? a.labels[m] : -1;
    __builtin_amdgcn_s_waitcnt(0);
    auto issue = [&](int it) __attribute__((always_inline)) {
        const unsigned s = lds0 + (unsigned)((it & 1) * R::STAGE);
        R::tile(s, a.W, (t0 + it) * 64, a.V, a.ld, wv);
        R::dma4(s + R::TILE, reinterpret_cast<const char*>(a.bias + (long long)(t0 + it) * 64), (unsigned)(fresh_lane() * 4));
    };
    float top = -LOSS_FAR, sum = 0.0f, sum2 = 0.0f;
    const float k1 = a.k1, k = a.k, slack = SLACK / fmaxf(k1, WHAT == SUMS2 ? k : 0.0f);
    issue(0);
    for (int it = 0; it < n; ++it) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (it + 1 < n) issue(it + 1);
        const char* stage = reinterpret_cast<const char*>(smem) + (it & 1) * R::STAGE;
        const float* bias = reinterpret_cast<const float*>(stage + R::TILE);
        float strip = __builtin_nanf("");
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            const char* s = stage + sub * 32 * R::ROWB;
            f32x16_t u;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 b = *reinterpret_cast<const float4*>(bias + sub * 32 + 8 * g + 4 * half);
                u[4 * g] = b.x; u[4 * g + 1] = b.y; u[4 * g + 2] = b.z; u[4 * g + 3] = b.w;
            }
#pragma unroll
            for (int q = 0; q < 4 * NK; ++q) u = mma32(at.by_row(s, q), zf[q], u);
            ahead<4 + DEPTH, 4 * NK, 1, 1, DEPTH>();
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (WHAT == SUMS2) {
                const int at_label = label - ((t0 + it) * 64 + sub * 32);
                if (__any((unsigned)at_label < 32u)) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) u[e] = at_label == 8 * (e >> 2) + 4 * half + (e & 3) ? -INFINITY : u[e];
                }
            }
            float mx = u[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) mx = fmaxf(mx, u[e]);
            if constexpr (WHAT == LOGITS) {
                strip = fmaxf(strip, mx);
                if (m < a.M) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int v = (t0 + it) * 64 + sub * 32 + 8 * g + 4 * half;
                        if (v < a.ldo) *reinterpret_cast<float4*>(a.out + m * a.ldo + v) = make_float4(u[4 * g], u[4 * g + 1], u[4 * g + 2], u[4 * g + 3]);
                    }
                }
            } else {
                if (__any(mx > top + slack)) {
                    const float now = fmaxf(top, fmaxf(mx, __shfl_xor(mx, 32, 64)));
                    sum *= __builtin_amdgcn_exp2f(rounded_product(top, k1) - rounded_product(now, k1));
                    if (WHAT == SUMS2) sum2 *= __builtin_amdgcn_exp2f(rounded_product(top, k) - rounded_product(now, k));
                    top = now;
                }
                const float m1 = rounded_product(top, k1), m2 = rounded_product(top, k);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    sum += __builtin_amdgcn_exp2f(fmaf(u[e], k1, -m1));
                    if (WHAT == SUMS2) sum2 += __builtin_amdgcn_exp2f(fmaf(u[e], k, -m2));
                }
            }
        }
        if constexpr (WHAT == LOGITS) {
            strip = fmaxf(strip, __shfl_xor(strip, 32, 64));
            if (half == 0 && m < a.M) a.part_ref[(long long)(t0 + it) * a.M + m] = strip;
        }
    }
    if constexpr (WHAT != LOGITS) {
        sum += __shfl_xor(sum, 32, 64);
        if (WHAT == SUMS2) sum2 += __shfl_xor(sum2, 32, 64);
        if (half == 0 && m < a.M) {
            const long long to = (long long)part * a.M + m;
            a.part_ref[to] = top;
            a.part_sum[to] = sum;
            if (WHAT == SUMS2) a.part_sum2[to] = sum2;
        }
    }
}

// ---- classes ----------------------------------------------------------------------------------------------------------------
// ENTRIES: of a teacher's lists, those of a tile's 64 rows and the workgroup's 128 classes come with the tile, in any order; a wavefront puts its own
// into a block of 32 x 32 in LDS, from which du takes them, and clears them again.
// (written by an earlier launch: read with scalar loads, which the ring's waits do not count)
typedef const __attribute__((address_space(4))) int* const_int;
constexpr int SPOT = 36;                                // floats between a block's classes: eight lanes' reads on banks of their own
template <int NK, bool TAU, bool ENTRIES>
__global__ __launch_bounds__(512, 2) void loss_classes_kernel(LossFusedArgs a) {
    typedef Ring<NK> R;
    constexpr int STAGE = R::STAGE + (ENTRIES ? R::LIST : 0), LOADS = NK + 1 + (ENTRIES ? 1 : 0);
    extern __shared__ uint4 smem[];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int cg = wv & 3, rh = wv >> 2;                // the wavefront's 32 classes, and its 32 of a tile's 64 rows
    const int ntv = (a.V + 127) / 128, ct = (int)blockIdx.x % ntv, part = (int)blockIdx.x / ntv;
    const int ntm = (a.M + 63) / 64, per = (ntm + a.parts - 1) / a.parts, t0 = part * per, n = min(per, ntm - t0);
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    const Reads<NK> at(lane);
    if (blockIdx.x == 0 && a.loss) {                    // the rows' loss terms, in a fixed order (a launch less)
        float* sh = reinterpret_cast<float*>(smem);
        float s = 0.0f;
        for (int i0 = tid; i0 < a.M; i0 += 8 * 512) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = i0 + 512 * j < a.M ? a.row_loss[i0 + 512 * j] : 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += x[j];
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
        if (lane == 0) sh[wv] = s;
        __syncthreads();
        if (tid == 0) { s = sh[0]; for (int w = 1; w < 8; ++w) s += sh[w]; a.loss[0] = s; }
        __syncthreads();
    }
    const int class0 = ct * 128 + cg * 32, v = class0 + l32;
    uint4 wf[4 * NK];
#pragma unroll
    for (int q = 0; q < 4 * NK; ++q) {
        const int c = 2 * q + half;
        wf[q] = c * 8 < a.ld ? *reinterpret_cast<const uint4*>(a.W + (long long)min(v, a.V - 1) * a.ld + c * 8) : make_uint4(0, 0, 0, 0);
    }
    const float b = v < a.V ? a.bias[v] : -INFINITY, k1 = a.k1, k = a.k;
    __builtin_amdgcn_s_waitcnt(0);                      // (known to the compiler: it would wait for these loads, and the ring's with them, in the loop)
    auto issue = [&](int it) __attribute__((always_inline)) {
        const unsigned s = lds0 + (unsigned)(it % R::STAGES * STAGE);
        R::tile(s, a.z, (t0 + it) * 64, a.M, a.ld, wv);
        // the rows' constants, an array a wavefront
        R::dma4(s + R::TILE + (unsigned)(wv * 256), reinterpret_cast<const char*>(a.consts + (long long)min(wv, 5) * a.Mp + (long long)(t0 + it) * 64), (unsigned)(fresh_lane() * 4));
        if constexpr (ENTRIES) R::dma4(s + R::STAGE + (unsigned)(wv * 256), reinterpret_cast<const char*>(a.entries + ((const_int)(uintptr_t)a.entries_from)[(long long)(t0 + it) * ntv + ct]) + wv * 256, (unsigned)(fresh_lane() * 4));
    };
    f32x16_t o[2 * NK];
#pragma unroll
    for (int zb = 0; zb < 2 * NK; ++zb)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[zb][e] = 0.0f;
    float db = 0.0f, db_off = 0.0f;                     // (a long sum, with what its last addition rounded off: 43008 rows 1.2e-6 off without, 7e-7 with)
    float* spots = reinterpret_cast<float*>(reinterpret_cast<char*>(smem) + R::STAGES * STAGE) + wv * 32 * SPOT;
    if constexpr (ENTRIES) {
        for (int k = lane; k < 32 * SPOT; k += 64) spots[k] = 0.0f;
    }
    if (n > 0) issue(0);
    if (n > 1) issue(1);
    for (int it = 0; it < n; ++it) {
        if (it + 1 < n) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (it + 2 < n) issue(it + 2);
        const char* stage = reinterpret_cast<const char*>(smem) + it % R::STAGES * STAGE;
        const char* s = stage + rh * 32 * R::ROWB;
        const float* consts = reinterpret_cast<const float*>(stage + R::TILE) + rh * 32;   // [6][64]
        // the teacher's entries of these rows and classes, one a lane (and more where there are more)
        int listed = 0, spot = -1;
        auto spot_of = [&](const uint2& e) { return (int)(e.x >> 5 & 1u) == rh && (int)(e.x >> 11) == cg ? (int)(e.x >> 6 & 31u) * SPOT + (int)(e.x & 31u) : -1; };
        auto others = [&](bool clear) {
            const int from = ((const_int)(uintptr_t)a.entries_from)[(long long)(t0 + it) * ntv + ct];
            bool any = false;
            for (int k = 64 + fresh_lane(); k < listed; k += 64) {
                const uint2 e = k < R::LIST / 8 ? reinterpret_cast<const uint2*>(stage + R::STAGE)[k] : a.entries[from + k];
                const int to = spot_of(e);
                if (to >= 0) { spots[to] = clear ? 0.0f : __builtin_bit_cast(float, e.y); any = true; }
            }
            return any;
        };
        bool any_spot = false;
        if constexpr (ENTRIES) {
            listed = ((const_int)(uintptr_t)a.entries_count)[(long long)(t0 + it) * ntv + ct];
            const int ln = fresh_lane();
            if (ln < listed) {
                const uint2 e = reinterpret_cast<const uint2*>(stage + R::STAGE)[ln];
                spot = spot_of(e);
                if (spot >= 0) spots[spot] = __builtin_bit_cast(float, e.y);
            }
            any_spot = spot >= 0;
            if (listed > 64) any_spot |= others(false);
            any_spot = __any(any_spot);
        }
        f32x16_t u;                                     // (the bias first, as in the walks over the classes: the same logits, bit by bit)
        float first = b;
        asm volatile("" : "+v"(first));                 // (sixteen copies of it made ahead of the loop are sixteen registers too many)
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] = first;
#pragma unroll
        for (int q = 0; q < 4 * NK; ++q) u = mma32(at.by_row(s, q), wf[q], u);
        ahead<DEPTH, 4 * NK, 1, 1, DEPTH>();
        __builtin_amdgcn_sched_barrier(0);
        // a label among these classes: one product of 32 x 32 in V / 1024
        const int* labels = reinterpret_cast<const int*>(consts + 320);
        const bool any_hot = __any((unsigned)(labels[fresh_lane() & 31] - class0) < 32u);
#pragma unroll
        for (int t = 0; t < 2; ++t) {                   // sixteen rows, a step of the second product
            float d[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 8 * (2 * t + h) + 4 * half;
                const float4 m2 = *reinterpret_cast<const float4*>(consts + r), ca = *reinterpret_cast<const float4*>(consts + 64 + r);
                const float ms[4] = {m2.x, m2.y, m2.z, m2.w}, cs[4] = {ca.x, ca.y, ca.z, ca.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) d[4 * h + i] = cs[i] * __builtin_amdgcn_exp2f(fmaf(u[8 * t + 4 * h + i], k1, -ms[i]));
                if (TAU) {
                    const float4 mt = *reinterpret_cast<const float4*>(consts + 128 + r), ct_ = *reinterpret_cast<const float4*>(consts + 192 + r);
                    const float mts[4] = {mt.x, mt.y, mt.z, mt.w}, cts[4] = {ct_.x, ct_.y, ct_.z, ct_.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[4 * h + i] = fmaf(cts[i], __builtin_amdgcn_exp2f(fmaf(u[8 * t + 4 * h + i], k, -mts[i])), d[4 * h + i]);
                }
            }
            if (any_hot) {                              // (a label's du is one of the constants)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int r = 8 * (2 * t + (e >> 2)) + 4 * half + (e & 3);
                    if (labels[r] == class0 + (fresh_lane() & 31)) d[e] = -consts[256 + r];
                }
            }
            if (ENTRIES && any_spot) {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 x = *reinterpret_cast<const float4*>(spots + (fresh_lane() & 31) * SPOT + 8 * (2 * t + h) + 4 * half);
                    d[4 * h] -= x.x; d[4 * h + 1] -= x.y; d[4 * h + 2] -= x.z; d[4 * h + 3] -= x.w;
                }
            }
            // (with lists there is no register left for db_off: 335 us became 374)
            const float step = ((d[0] + d[1]) + (d[2] + d[3])) + ((d[4] + d[5]) + (d[6] + d[7]));
            if constexpr (ENTRIES) db += step;
            else {
                const float x = step - db_off, next = db + x;
                db_off = (next - db) - x;
                db = next;
            }
            auto split = [&] {                          // d rounded, as the operand; d: what the rounding left
                unsigned p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = pack2(d[2 * e], d[2 * e + 1]);
                    d[2 * e] -= __builtin_bit_cast(float, p[e] << 16);
                    d[2 * e + 1] -= __builtin_bit_cast(float, p[e] & 0xFFFF0000u);
                }
                return fragment(p);
            };
            const uint4 hi = split(), lo = split();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int zb = 0; zb < 2 * NK; ++zb) {
                const uint4 x = at.by_col(s + t * 16 * R::ROWB, zb);
                o[zb] = mma32(x, hi, o[zb]);
                o[zb] = mma32(x, lo, o[zb]);
            }
            ahead<2 * 2, 2 * NK, 2, 2, 2>();
            __builtin_amdgcn_sched_barrier(0);
            if (any_hot || (ENTRIES && a.third && any_spot)) {   // (where du is large: a third part of it)
                const uint4 rest = split();
#pragma unroll
                for (int zb = 0; zb < 2 * NK; ++zb) o[zb] = mma32(at.by_col(s + t * 16 * R::ROWB, zb), rest, o[zb]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (ENTRIES && any_spot) {                      // (a wavefront's LDS accesses keep their order)
            if (spot >= 0) spots[spot] = 0.0f;
            if (listed > 64) others(true);
        }
    }
    const int ln = fresh_lane(), n32 = ln & 31, hf = ln >> 5, cls = ct * 128 + cg * 32 + n32;
    // the two halves of the rows together, through LDS, and out along the rows of dW_s; register e of a lane: column 32 zb + 8 (e / 4) + 4 half + e % 4 of
    // class n32.  (Rows of LDS a 16-byte word longer: neighbouring classes on neighbouring banks.)
    db += __shfl_xor(db, 32, 64);
    constexpr int LD = 64 * NK + 4;
    float* sh = reinterpret_cast<float*>(smem);         // [128][LD], then [128]
    float* mine = sh + (cg * 32 + n32) * LD + 4 * hf;
    float* out = a.out + (long long)part * a.V * a.ldo;
    __syncthreads();
    if (rh == 1) {
#pragma unroll
        for (int zb = 0; zb < 2 * NK; ++zb)
#pragma unroll
            for (int g = 0; g < 4; ++g) *reinterpret_cast<float4*>(mine + 32 * zb + 8 * g) = make_float4(o[zb][4 * g], o[zb][4 * g + 1], o[zb][4 * g + 2], o[zb][4 * g + 3]);
        if (hf == 0) sh[128 * LD + cg * 32 + n32] = db;
    }
    __syncthreads();
    if (rh == 0) {
#pragma unroll
        for (int zb = 0; zb < 2 * NK; ++zb)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float4* p = reinterpret_cast<float4*>(mine + 32 * zb + 8 * g);
                const float4 x = *p;
                *p = make_float4(o[zb][4 * g] + x.x, o[zb][4 * g + 1] + x.y, o[zb][4 * g + 2] + x.z, o[zb][4 * g + 3] + x.w);
            }
        if (hf == 0 && cls < a.V) a.out_db[(long long)part * a.V + cls] = db + sh[128 * LD + cg * 32 + n32];
    }
    __syncthreads();
    const int rows = min(128, a.V - ct * 128);
    for (int i = wv * 64 + ln; i < rows * 16 * NK; i += 512) {
        const int r = i / (16 * NK), z = i % (16 * NK) * 4;
        const float4 x = *reinterpret_cast<const float4*>(sh + r * LD + z);
        float* to = out + (long long)(ct * 128 + r) * a.ldo + z;
        if (a.vec && z + 4 <= a.Z) *reinterpret_cast<float4*>(to) = x;
        else {
            if (z < a.Z) to[0] = x.x;
            if (z + 1 < a.Z) to[1] = x.y;
            if (z + 2 < a.Z) to[2] = x.z;
            if (z + 3 < a.Z) to[3] = x.w;
        }
    }
}

// ---- a teacher's entries by tiles of 64 rows and 128 classes, a workgroup 64 rows ------------------------------------------------
// Counts the rows' entries with a probability by tiles, gives every tile a place among the rows' own, and puts them there (in an order of no
// matter: a row's classes are different ones).  All counters in LDS: with a list of all rows together, 168 rows of 16 took three launches of
// 4 us for it and 5376 of 64 took 20 us.
// Behind those, a workgroup 32 rows and MARK_WORDS words of the marks: the entries with a probability and the label.
constexpr int LISTS_THREADS = 1024, MARK_WORDS = 512;
__global__ __launch_bounds__(LISTS_THREADS) void loss_lists_kernel(LossListArgs a, int ntv) {
    extern __shared__ uint4 smem[];
    const int lists = (a.M + 63) / 64;
    if ((int)blockIdx.x >= lists) {
        uint32_t* word = reinterpret_cast<uint32_t*>(smem);   // [words][32]
        const int all = loss_mark_words(a.V), blocks = (all + MARK_WORDS - 1) / MARK_WORDS;
        const int row0 = ((int)blockIdx.x - lists) / blocks * 32, word0 = ((int)blockIdx.x - lists) % blocks * MARK_WORDS, words = min(MARK_WORDS, all - word0);
        const int rows = min(32, a.M - row0);            // (none or less: the last rows of the last 256)
        for (int i = threadIdx.x; i < words * 32; i += LISTS_THREADS) word[i] = 0;
        __syncthreads();
        auto mark = [&](int row, int c) {
            const int w = (c >> 5) - word0;
            if (w >= 0 && w < words) atomicOr(&word[w * 32 + row], 1u << (c & 31));
        };
        for (int k = threadIdx.x; k < rows * a.K; k += LISTS_THREADS)
            if (a.q[row0 * a.K + k] > 0.0f) mark(k / a.K, a.classes[row0 * a.K + k]);
        if (a.labels && (int)threadIdx.x < rows) {
            const int lab = a.labels[row0 + threadIdx.x];
            if ((unsigned)lab < (unsigned)a.V) mark(threadIdx.x, lab);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < words * 32; i += LISTS_THREADS) a.marks[(long long)(word0 + (i >> 5)) * a.Mr + row0 + (i & 31)] = word[i];
        return;
    }
    int* at = reinterpret_cast<int*>(smem);             // [ntv], then a number a wavefront
    int* waves = at + ntv;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row0 = (int)blockIdx.x * 64;
    const int n = min(64, a.M - row0) * a.K, base = row0 * a.K;
    for (int i = tid; i < ntv; i += LISTS_THREADS) at[i] = 0;
    __syncthreads();
    for (int k = tid; k < n; k += LISTS_THREADS)
        if (a.q[base + k] > 0.0f) atomicAdd(&at[a.classes[base + k] >> 7], 1);
    __syncthreads();
    const int per = (ntv + LISTS_THREADS - 1) / LISTS_THREADS, first = min(tid * per, ntv), end = min(first + per, ntv);
    int own = 0;
    for (int i = first; i < end; ++i) own += at[i];
    int before = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int t = __shfl_up(before, o, 64); if (lane >= o) before += t; }
    if (lane == 63) waves[wave] = before;
    __syncthreads();
    before -= own;
    for (int w = 0; w < wave; ++w) before += waves[w];
    for (int i = first; i < end; ++i) {
        const int c = at[i];
        at[i] = before;
        a.count[(long long)blockIdx.x * ntv + i] = c;
        a.from[(long long)blockIdx.x * ntv + i] = base + before;
        before += c;
    }
    __syncthreads();
    for (int k = tid; k < n; k += LISTS_THREADS) {
        const float p = a.q[base + k];
        if (!(p > 0.0f)) continue;
        const int c = a.classes[base + k];
        a.entries[base + atomicAdd(&at[c >> 7], 1)] = make_uint2((unsigned)(k / a.K) | (unsigned)(c & 127) << 6, __builtin_bit_cast(unsigned, a.weight * p));
    }
}

// The parts of dW_s and db_s in order.
__global__ __launch_bounds__(256) void loss_classes_sum_kernel(const float* __restrict__ p, const float* __restrict__ pb, int parts, long long n, int V, float* __restrict__ out, float* __restrict__ out_b) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n + V; i += (long long)gridDim.x * 256) {
        const bool w = i < n;
        const float* x = w ? p + i : pb + (i - n);
        const long long step = w ? n : V;
        float s = x[0];
#pragma unroll 4
        for (int k = 1; k < parts; ++k) s += x[k * step];
        if (w) out[i] = s; else out_b[i - n] = s;
    }
}

// ---- behind the rows: a workgroup a row, four columns a lane, its wavefronts share the parts and the teacher's classes ---------
// KNOWN: the rows' constants and losses are there and the parts are sums of du W; else they are made here from the parts' references
// and sums, which are brought to the largest reference, and the label's logit, which they lack.  The parts lack the label's and the
// teacher's classes, whose dE/du is made here in float: 1 - p of a label from the sum of all others, p' - q as a difference.
// All loads of a step are independent: one by one, 128 parts and 64 classes took 49 us for 168 rows.
// SHARE: wavefronts a row, four or, where rows are many, one (43008 rows: 69 us with four, 30 with one).
template <bool KNOWN, bool POLICY, int SHARE>
__global__ __launch_bounds__(256) void loss_dz_kernel(LossDzArgs a, PolicyArgs policy, TeacherArgs teacher) {
    __shared__ float4 sh[3][64];
    const int lane = threadIdx.x & 63, wf = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = SHARE == 4 ? wf : 0;
    const long long m = SHARE == 4 ? (long long)blockIdx.x : (long long)blockIdx.x * 4 + wf;
    if (m >= a.M) {                                      // the last tile's rows that are none
        if (wave == 0 && lane < 6) a.consts[lane * (long long)a.Mp + m] = lane == 0 || lane == 2 ? INFINITY : lane == 5 ? __builtin_bit_cast(float, -1) : 0.0f;
        return;
    }
    float m2 = 0.0f, c1 = 1.0f, mt2 = 0.0f, ct = 0.0f, at_label = 0.0f;   // at_label: du there, but for the teacher's q
    int lab = a.labels ? a.labels[m] : -1;
    const float k = POLICY || KNOWN ? LOG2E : LOG2E * teacher.inv_tau, kt = LOG2E * teacher.inv_tau;
    bool some = false;                                   // entries of the teacher's that count
    // entry i's class, logit and q (nothing: class -1, q 0)
    struct Entry { int c; float u, q; };
    auto entry = [&](int i) {
        Entry e{-1, 0.0f, i < teacher.K ? a.entry_q[m * teacher.K + i] : 0.0f};
        if (e.q > 0.0f) { e.c = teacher.classes[m * teacher.K + i]; e.u = a.entry_logit[m * teacher.K + i]; }
        else e.q = 0.0f;
        return e;
    };
    if (KNOWN) {
        m2 = a.consts[m]; c1 = a.consts[a.Mp + m]; mt2 = a.consts[2 * (long long)a.Mp + m]; ct = a.consts[3 * (long long)a.Mp + m];
        at_label = -a.consts[4 * (long long)a.Mp + m];
        some = a.soft_state[m] & 1;
    } else {
        const bool lab_ok = (unsigned)lab < (unsigned)a.V;
        const float lu = lab_ok ? a.label_logit[m] : 0.0f;
        float ref = lab_ok ? lu * k : -INFINITY;
        for (int p = lane; p < a.parts; p += 64) ref = fmaxf(ref, a.part_ref[(long long)p * a.M + m]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) ref = fmaxf(ref, __shfl_xor(ref, o, 64));
        float sum = 0.0f;
        for (int p = lane; p < a.parts; p += 64) sum += a.part_sum[(long long)p * a.M + m] * __builtin_amdgcn_exp2f(a.part_ref[(long long)p * a.M + m] - ref);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        const float others = sum, w_label = lab_ok ? __builtin_amdgcn_exp2f(fmaf(lu, k, -ref)) : 0.0f;
        sum += w_label;
        m2 = ref;
        const float nan = __builtin_nanf(""), log_sum = logf(sum);
        const float lp = lab_ok ? fmaf(lu, LOG2E, -ref) * LN2 - log_sum : lab == -1 ? 0.0f : nan;
        float loss = 0.0f;
        c1 = 0.0f;
        if (POLICY) {
            if (lab_ok) {
                const PolicyTerms t = policy_terms(policy, m, lp);
                loss = a.s * t.loss; c1 = -a.s * t.g / sum; at_label = a.s * t.g * (others / sum);
            } else if (lab != -1) loss = nan;
            if (a.logp && wave == 0 && lane == 0) a.logp[m] = lp;
        } else {
            const int state = a.soft_state[m];
            some = state & 1;
            if (lab_ok) { loss = a.s * teacher.hard * -lp; c1 = a.s * teacher.hard / sum; at_label = -a.s * teacher.hard * (others / sum); }
            else if (lab != -1) loss = nan;
            if (some) {
                loss += a.s * teacher.soft * teacher.tau * teacher.tau * (a.soft_const[m] + (fmaf(-a.soft_const[a.M + m], k, ref) * LN2 + log_sum));
                c1 += a.s * teacher.soft * teacher.tau / sum;
                at_label += a.s * teacher.soft * teacher.tau / sum * w_label;
            }
            if (state & 2) loss = nan;
        }
        const bool counts = lab_ok || some;
        if (!lab_ok) lab = -1;
        if (wave == 0 && lane < 6)
            a.consts[lane * (long long)a.Mp + m] = lane == 0 ? (counts ? m2 : INFINITY) : lane == 1 ? c1 : lane == 2 ? INFINITY : lane == 3 ? 0.0f : lane == 4 ? -at_label : __builtin_bit_cast(float, lab);
        if (wave == 0 && lane == 0) a.row_loss[m] = loss;
    }
    const bool lab_ok = (unsigned)lab < (unsigned)a.V, counts = KNOWN || lab_ok || some;
    const bool in = lane * 4 < a.ld;
    const int z0 = in ? lane * 4 : 0;                    // (all lanes stay: each holds an entry of the list)
    float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (counts) {
        auto add_part = [&](int p) {
            const long long at = (long long)p * a.M + m;
            const float4 v = *reinterpret_cast<const float4*>(a.part + at * a.ld + z0);
            const float w = KNOWN ? 1.0f : __builtin_amdgcn_exp2f(a.part_ref[at] - m2);
            x[0] = fmaf(v.x, w, x[0]); x[1] = fmaf(v.y, w, x[1]); x[2] = fmaf(v.z, w, x[2]); x[3] = fmaf(v.w, w, x[3]);
        };
        int p = wave;
        for (; p + 7 * SHARE < a.parts; p += 8 * SHARE) {
#pragma unroll
            for (int k = 0; k < 8; ++k) add_part(p + SHARE * k);
        }
        for (; p < a.parts; p += SHARE) add_part(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] *= KNOWN ? 1.0f : c1;
        auto add = [&](int c, float w) {                 // w W_c
            const uint2 b = *reinterpret_cast<const uint2*>(a.W + (long long)c * a.ld + z0);
            x[0] = fmaf(w, bf2f((bf16_t)(b.x & 0xFFFFu)), x[0]); x[1] = fmaf(w, bf2f((bf16_t)(b.x >> 16)), x[1]);
            x[2] = fmaf(w, bf2f((bf16_t)(b.y & 0xFFFFu)), x[2]); x[3] = fmaf(w, bf2f((bf16_t)(b.y >> 16)), x[3]);
        };
        if (wave == 0 && lab_ok) add(lab, at_label);
        if (!POLICY && some) {
            const float weight = a.s * teacher.soft * teacher.tau;
            for (int k0 = 0; k0 < teacher.K; k0 += 64) {
                // 64 entries a lane each; the wavefront's sixteen, four at a time (one that is none: nothing times the first class)
                const Entry e = entry(k0 + lane);
                float w = -weight * e.q;
                if (e.c >= 0 && e.c != lab) {            // (the label's probability is in at_label)
                    w = fmaf(c1, __builtin_amdgcn_exp2f(fmaf(e.u, k, -m2)), w);
                    if (KNOWN) w = fmaf(ct, __builtin_amdgcn_exp2f(fmaf(e.u, kt, -mt2)), w);
                }
                const int c = max(e.c, 0);
                for (int j = wave; j < 64 && k0 + j < teacher.K; j += 4 * SHARE) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        add(__builtin_amdgcn_readlane(c, j + SHARE * i), __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), j + SHARE * i)));
                }
            }
        }
    }
    if constexpr (SHARE == 4) {
        if (wave > 0) sh[wave - 1][lane] = make_float4(x[0], x[1], x[2], x[3]);
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < 3; ++w) { const float4 y = sh[w][lane]; x[0] += y.x; x[1] += y.y; x[2] += y.z; x[3] += y.w; }
    }
    if (!in) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) if (z0 + i < a.Z) a.dz[m * a.Z + z0 + i] = f2bf(x[i]);
}

template <int NK, bool KNOWN, bool MARKS>
hipError_t rows_nk(const LossFusedArgs& a, hipStream_t st) {
    constexpr size_t lds = (size_t)Ring<NK>::STAGES * (Ring<NK>::STAGE + (MARKS ? Ring<NK>::MARK : 0));
    static thread_local bool attr_set = false;
    const hipError_t e = allow_lds(&loss_rows_kernel<NK, KNOWN, MARKS>, lds, &attr_set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((loss_rows_kernel<NK, KNOWN, MARKS>), dim3((unsigned)((a.M + 255) / 256 * a.parts)), dim3(512), lds, st, a);
    return hipGetLastError();
}
template <int NK, int WHAT>
hipError_t sums_nk(const LossFusedArgs& a, hipStream_t st) {
    constexpr size_t lds = 2 * (size_t)Ring<NK>::STAGE;
    static thread_local bool attr_set = false;
    const hipError_t e = allow_lds(&loss_sums_kernel<NK, WHAT>, lds, &attr_set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((loss_sums_kernel<NK, WHAT>), dim3((unsigned)((a.M + 255) / 256 * a.parts)), dim3(512), lds, st, a);
    return hipGetLastError();
}
template <int NK, bool TAU, bool ENTRIES>
hipError_t classes_nk(const LossFusedArgs& a, hipStream_t st) {
    constexpr size_t ring = (size_t)Ring<NK>::STAGES * (Ring<NK>::STAGE + (ENTRIES ? Ring<NK>::LIST : 0)) + (ENTRIES ? 8 * 32 * SPOT * 4 : 0), join = (128 * (64 * NK + 4) + 128) * 4, lds = ring > join ? ring : join;
    static thread_local bool attr_set = false;
    const hipError_t e = allow_lds(&loss_classes_kernel<NK, TAU, ENTRIES>, lds, &attr_set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((loss_classes_kernel<NK, TAU, ENTRIES>), dim3((unsigned)((a.V + 127) / 128 * a.parts)), dim3(512), lds, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_loss_fused_rows(const LossFusedArgs& a, bool known, hipStream_t st) {
    const int nk = (a.ld + 63) / 64;
#define BLSTM_ROWS(NK) return known ? rows_nk<NK, true, true>(a, st) : a.marks ? rows_nk<NK, false, true>(a, st) : rows_nk<NK, false, false>(a, st)
    if (nk == 1) BLSTM_ROWS(1);
    if (nk == 2) BLSTM_ROWS(2);
    if (nk == 3) BLSTM_ROWS(3);
    BLSTM_ROWS(4);
#undef BLSTM_ROWS
}
hipError_t launch_loss_fused_sums(const LossFusedArgs& a, bool second, bool logits, hipStream_t st) {
    const int nk = (a.ld + 63) / 64;
#define BLSTM_SUMS(NK) return logits ? sums_nk<NK, LOGITS>(a, st) : second ? sums_nk<NK, SUMS2>(a, st) : sums_nk<NK, SUMS>(a, st)
    if (nk == 1) BLSTM_SUMS(1);
    if (nk == 2) BLSTM_SUMS(2);
    if (nk == 3) BLSTM_SUMS(3);
    BLSTM_SUMS(4);
#undef BLSTM_SUMS
}
hipError_t launch_loss_fused_classes(const LossFusedArgs& a, bool tau, hipStream_t st) {
    const int nk = (a.ld + 63) / 64;
#define BLSTM_CLASSES(NK) return a.entries ? (tau ? classes_nk<NK, true, true>(a, st) : classes_nk<NK, false, true>(a, st)) : classes_nk<NK, false, false>(a, st)
    if (nk == 1) BLSTM_CLASSES(1);
    if (nk == 2) BLSTM_CLASSES(2);
    if (nk == 3) BLSTM_CLASSES(3);
    BLSTM_CLASSES(4);
#undef BLSTM_CLASSES
}
template <int SHARE>
static hipError_t dz_shared(const LossDzArgs& a, bool known, hipStream_t st) {
    const dim3 grid((unsigned)(SHARE == 4 ? a.Mp : a.Mp / 4));
    const PolicyArgs p = a.policy ? *a.policy : PolicyArgs{};
    const TeacherArgs t = a.teacher ? *a.teacher : TeacherArgs{};
    if (a.policy) hipLaunchKernelGGL((loss_dz_kernel<false, true, SHARE>), grid, dim3(256), 0, st, a, p, t);
    else if (known) hipLaunchKernelGGL((loss_dz_kernel<true, false, SHARE>), grid, dim3(256), 0, st, a, p, t);
    else hipLaunchKernelGGL((loss_dz_kernel<false, false, SHARE>), grid, dim3(256), 0, st, a, p, t);
    return hipGetLastError();
}
hipError_t launch_loss_dz(const LossDzArgs& a, bool known, hipStream_t st) { return a.M <= 8192 ? dz_shared<4>(a, known, st) : dz_shared<1>(a, known, st); }
hipError_t launch_loss_lists(const LossListArgs& a, hipStream_t st) {
    const int ntv = (a.V + 127) / 128;
    constexpr size_t most = ((1 << 22) / 128 + LISTS_THREADS / 64) * sizeof(int);   // (a model's most classes)
    static thread_local bool attr_set = false;
    const hipError_t e = allow_lds(&loss_lists_kernel, most, &attr_set);
    if (e != hipSuccess) return e;
    const int words = loss_mark_words(a.V);
    const size_t lists = (ntv + LISTS_THREADS / 64) * sizeof(int), marks = (size_t)(words < MARK_WORDS ? words : MARK_WORDS) * 32 * sizeof(uint32_t), lds = lists > marks ? lists : marks;
    if (lds > most) return hipErrorInvalidValue;
    const unsigned grid = (unsigned)((a.M + 63) / 64 + a.Mr / 32 * ((words + MARK_WORDS - 1) / MARK_WORDS));   // (below 2^26: T B V is below 2^44)
    hipLaunchKernelGGL(loss_lists_kernel, dim3(grid), dim3(LISTS_THREADS), lds, st, a, ntv);
    return hipGetLastError();
}
hipError_t launch_loss_classes_sum(const float* p, const float* pb, int parts, long long n, int V, float* out, float* out_b, hipStream_t st) {
    const long long blocks = (n + V + 255) / 256;
    hipLaunchKernelGGL(loss_classes_sum_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, p, pb, parts, n, V, out, out_b);
    return hipGetLastError();
}

}  // namespace blstm
