// The orthogonalised update.  Of a matrix d (a momentum) with m rows and n columns, m <= n (or the other way round: columns and rows change places):
//   X <- d / |d|_F,  then five times  S = X X^T,  B = b S + c S^2,  X <- a X + B X      (a, b, c) = (3.4445, -4.7750, 2.0315)
// which keeps the singular vectors and takes every singular value s to a s + b s^3 + c s^5: in five steps what is not tiny lands in 0.7 .. 1.2.
//
// Numbers.  Everything that a product reads is a half (the matrix cores' rate is that of bf16, with three more bits) times 2^8, which keeps the
// entries of a normalised matrix, 1/sqrt(m n), and what their rounding leaves over away from the subnormals; with singular values below 1.21 none
// exceeds 1.21 * 2^8 for X, 1.47 * 2^8 for S and 3.45 * 2^8 for B.  Products accumulate in float.  X itself is kept as the sum of two halves (22 bits): a rounding of X adds noise in all
// directions alike, and where a few directions hold most of |d| (gradients do) that noise is as large as the others; the step's other
// roundings pass through B X, which is small where the singular value is.  So mode 1 multiplies the first halves only and adds a X from both: off by
// 3e-4 to 5.4e-4 of X (4e-4, of which X's rounding in S 3.3e-4, S's 1.7e-4, B's 1.6e-4, X's in B X 1.4e-4: 301 x 602; small launches, with time to spare, multiply both halves
// for S: 2.8e-4).  Mode 0, mode 1 where matrices have few columns (muon_plan) and where the caller asks for it multiply both halves everywhere (three products): off by about 1e-6.
// The diagonals of S and B, which near the end are most of them, stay out of the halves and the products, in float: with D the diagonal and R the rest,
// S^2 = D^2 + D R + R D + R^2, and B X = D X + R X (rounded with the rest they alone put X off by 2e-3).
// The Frobenius norm is summed in double (squares of floats leave float's range) in a fixed order.
//
// S and B are symmetric: tiles on and above the diagonal are computed, and stored twice.
//
// All matrices of a call share each launch: the flat pass over v and g, the cast to halves, then S, B and the new X five times; the last X goes straight into
// the weights.  What bounds them, four layers of 512 cells (22.3 M weights in matrices and 8.2 M others, 301 GFLOP), 740 to 790 us in all, bytes as counted behind the L2: the flat pass 82 us, 449 MB
// at 5.5 TB/s; the cast 53, 255 MB; S 38 each, 35 GFLOP without the symmetry at 920 TFLOP/s, 101 MB; B 24, whose 311 tiles are 1.2 a CU, 49 MB; the new X 62, 35 GFLOP and 209 MB; the
// last 107, 407 MB.  Six of 1024: 351 (1.83 GB), 301 (1.52), 298 (448 GFLOP likewise at 1500 TFLOP/s, 0.82 GB), 151 (0.4), 512 (870 TFLOP/s, 1.75 GB), 720 (2.98 GB).
// Built and dropped: three and four buffers of a slab where a CU has one workgroup (S 41 -> 56 us: what a lone workgroup waits for are its own LDS reads and products in turn,
// 768 and 512 clocks a slab, not the loads); S in two, three or four parts of the contraction, summed by another launch (58, 66 and 77 us for 45); two steps'
// B multiplied together, so that X is written three times instead of five (error 4e-4 -> 6e-4).
#include "gemm_tile.hpp"
#include "muon.hpp"
#include <algorithm>

namespace blstm {
namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
// (a tensor may start anywhere in the flat vector, and rows need not be whole words)
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x2u_t __attribute__((ext_vector_type(2), aligned(2)));

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr int NS_STEPS = 5;
constexpr float UP = 256.0f, DOWN = 1.0f / 256.0f;      // what lies in scratch is 2^8 times its value
constexpr int FLAT = 8192;                              // elements of a unit of the flat passes
constexpr int CAST = 4096;

enum { PH_GRAM = 0, PH_SQUARE = 1, PH_APPLY = 2, PH_LAST = 3 };

// the last group that starts at or before id (empty ones share a start)
__device__ __forceinline__ int group_of(const int (&first)[MUON_MAX_GROUPS], int id) {
    int k = 0;
#pragma unroll
    for (int i = 1; i < MUON_MAX_GROUPS; ++i) k += id >= first[i] ? 1 : 0;
    return __builtin_amdgcn_readfirstlane(k);
}
// (the same in every lane: said for the scalar operand of a load)
__device__ __forceinline__ const char* uniform(const void* p) {
    const unsigned long long v = (unsigned long long)p;
    return reinterpret_cast<const char*>((unsigned long long)__builtin_amdgcn_readfirstlane((unsigned)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((unsigned)v));
}
__device__ __forceinline__ long long tensor_at(const MuonGroup& g, int k) { return g.at + (long long)(k / g.inner_count) * g.outer + (long long)(k % g.inner_count) * g.inner; }

// Whether matrix k takes part.  (Ids are a batch's: some thousand at most.  The first launch looks through them and leaves the answer for the others.)
__device__ __forceinline__ bool in_ids(const MuonIds& of, int k) {
    int found = 0;
    for (int i = threadIdx.x; i < of.n; i += blockDim.x) found |= of.ids[i] == k;
    return __syncthreads_or(found) != 0;
}

// ---- v <- momentum v + g, the squares' sums, and the whole update of what is not orthogonalised ----------------------
// 12 bytes an element of a matrix, 20 (22 with the bf16 copy) of the others.
__device__ __forceinline__ double block_sum(double v, double* lds) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}
__global__ __launch_bounds__(256) void muon_momentum_kernel(MuonPlan p, MuonArgs a, double* sums, MuonIds of, int* here) {
    __shared__ double lds[4];
    const int group = group_of(p.at.chunk, blockIdx.x);
    const MuonGroup& g = p.g[group];
    const int local = blockIdx.x - p.at.chunk[group], k = local / g.chunks, c = local % g.chunks;
    if (of.ids) {
        const bool in = in_ids(of, k);
        if (c == 0 && threadIdx.x == 0) here[k] = in;
        if (!in) return;
    }
    const long long size = (long long)g.rows * g.cols, e0 = (long long)c * FLAT, at = tensor_at(g, k) + e0;
    const int len = (int)min((long long)FLAT, size - e0);
    const float* grad = a.grad + at;
    float* vel = a.velocity ? a.velocity + at : nullptr;
    float* theta = a.theta ? a.theta + at : nullptr;
    unsigned short* shadow = a.shadow ? a.shadow + at : nullptr;
    const bool step = !g.ortho;
    double sum = 0.0;
    auto one = [&](float gr, float& v) {              // the update's direction; v becomes the new velocity
        if (!vel) return gr;
        v = a.momentum * v + gr;
        return a.nesterov ? gr + a.momentum * v : v;
    };
    const int head = (int)min((long long)((4 - (at & 3)) & 3), (long long)len), words = (len - head) / 4;
#pragma unroll 2
    for (int i = threadIdx.x; i < words; i += 256) {
        const int o = head + 4 * i;
        const f32x4_t gr = *reinterpret_cast<const f32x4_t*>(grad + o);
        f32x4_t v = vel ? *reinterpret_cast<const f32x4_t*>(vel + o) : gr, d, w;
        if (step) w = *reinterpret_cast<const f32x4_t*>(theta + o);
#pragma unroll
        for (int e = 0; e < 4; ++e) { float x = v[e]; d[e] = one(gr[e], x); v[e] = x; }
        if (vel) *reinterpret_cast<f32x4_t*>(vel + o) = v;
        if (step) {
            w = w - a.lr_rest * d;
            *reinterpret_cast<f32x4_t*>(theta + o) = w;
            if (shadow) { u32x2_t q; q[0] = pack_bf2(w[0], w[1]); q[1] = pack_bf2(w[2], w[3]); *reinterpret_cast<u32x2_t*>(shadow + o) = q; }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += (double)d[e] * d[e];
        }
    }
    // (what lies before the first and behind the last whole word)
    const int rest = len - 4 * words;
    if ((int)threadIdx.x < rest) {
        const int o = (int)threadIdx.x < head ? threadIdx.x : threadIdx.x + 4 * words;
        float v = vel ? vel[o] : 0.0f;
        const float d = one(grad[o], v);
        if (vel) vel[o] = v;
        if (step) {
            const float w = theta[o] - a.lr_rest * d;
            theta[o] = w;
            if (shadow) shadow[o] = f2bf(w);
        } else sum += (double)d * d;
    }
    if (!step) {
        const double all = block_sum(sum, lds);
        if (threadIdx.x == 0) sums[blockIdx.x] = all;
    }
}

// X where only its first halves are multiplied: the second part, times 2^10, in eight bits (e5m2, three significant bits: X to 2^-15), a quarter less to write and
// read (four layers of 512 cells 806 -> 796 us).
__device__ __forceinline__ void put_low(_Float16* hi, unsigned char* lo, const float (&v)[8]) {
    f16x8_t h;
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { h[e] = (_Float16)v[e]; r[e] = 1024.0f * (v[e] - (float)h[e]); }
    *reinterpret_cast<f16x8_t*>(hi) = h;
    u32x2_t w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int x = __builtin_amdgcn_cvt_pk_bf8_f32(r[4 * i], r[4 * i + 1], 0, false);
        w[i] = (unsigned)__builtin_amdgcn_cvt_pk_bf8_f32(r[4 * i + 2], r[4 * i + 3], x, true);
    }
    *reinterpret_cast<u32x2_t*>(lo) = w;
}
__device__ __forceinline__ f16x8_t low(u32x2_t w) {
    f16x8_t l;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        l[4 * i] = (_Float16)(__builtin_amdgcn_cvt_f32_bf8((int)w[i], 0) * (1.0f / 1024.0f));
        l[4 * i + 1] = (_Float16)(__builtin_amdgcn_cvt_f32_bf8((int)w[i], 1) * (1.0f / 1024.0f));
        l[4 * i + 2] = (_Float16)(__builtin_amdgcn_cvt_f32_bf8((int)w[i], 2) * (1.0f / 1024.0f));
        l[4 * i + 3] = (_Float16)(__builtin_amdgcn_cvt_f32_bf8((int)w[i], 3) * (1.0f / 1024.0f));
    }
    return l;
}
// the second part of matrix k of X in buffer b, in eight bits
__device__ __forceinline__ unsigned char* low_of(const MuonGroup& g, _Float16* ws, int b, int k) { return reinterpret_cast<unsigned char*>(ws + g.x[b] + g.xplane) + (long long)k * g.rp * g.cp; }

// ---- d / |d|_F as two halves, zero-padded ---------------------------------------------------------------------------
__device__ __forceinline__ void put_halves(_Float16* hi, _Float16* lo, const float (&v)[8]) {
    f16x8_t h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) { h[e] = (_Float16)v[e]; l[e] = (_Float16)(v[e] - (float)h[e]); }
    *reinterpret_cast<f16x8_t*>(hi) = h;
    if (lo) *reinterpret_cast<f16x8_t*>(lo) = l;
}
template <bool LOW>
__global__ __launch_bounds__(256) void muon_cast_kernel(MuonPlan p, MuonArgs a, const double* sums, _Float16* ws) {
    __shared__ double lds[4];
    const int group = group_of(p.at.cast, blockIdx.x);
    const MuonGroup& g = p.g[group];
    const int local = blockIdx.x - p.at.cast[group], k = local / g.casts, c = local % g.casts;
    double sum = 0.0;
    for (int i = threadIdx.x; i < g.chunks; i += 256) sum += sums[p.at.chunk[group] + k * g.chunks + i];
    const double norm2 = block_sum(sum, lds);
    // (a zero matrix stays one; an infinity or NaN anywhere makes all of it NaN)
    const double scale = norm2 == 0.0 ? 0.0 : UP / sqrt(norm2);
    const float whole = norm2 <= 1.7e308 ? 0.0f : __builtin_nanf("");
    const long long at = tensor_at(g, k);
    _Float16* x = ws + g.x[0] + (long long)k * g.rp * g.cp;
#pragma unroll
    for (int q = 0; q < CAST / 2048; ++q) {
        const long long e = (long long)c * CAST + q * 2048 + threadIdx.x * 8;
        const int r = (int)(e / g.cp), c0 = (int)(e % g.cp);
        float d[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = 0.0f;
        if (r < g.rows) {
            const long long o = at + (long long)r * g.cols + c0;
            const int n = min(8, g.cols - c0);
            float gr[8], v[8];
            if (n == 8) {
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const f32x4_t y = *reinterpret_cast<const f32x4u_t*>(a.grad + o + 4 * w);
                    const f32x4_t z = a.velocity ? (f32x4_t)*reinterpret_cast<const f32x4u_t*>(a.velocity + o + 4 * w) : y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) { gr[4 * w + j] = y[j]; v[4 * w + j] = z[j]; }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) if (j < n) { gr[j] = a.grad[o + j]; v[j] = a.velocity ? a.velocity[o + j] : 0.0f; }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) if (j < n) {
                const float f = !a.velocity ? gr[j] : a.nesterov ? gr[j] + a.momentum * v[j] : v[j];
                d[j] = (float)(f * scale) + whole;
            }
        }
        if constexpr (LOW) put_low(x + e, low_of(g, ws, 0, k) + e, d);
        else put_halves(x + e, x + g.xplane + e, d);
    }
}

// ---- the products ---------------------------------------------------------------------------------------------------
// One tile of sum_k A(row, k) B(col, k), 64 TM x 64 TN, on 2 x 2 wavefronts.  A slab of 64 k is brought to LDS by global_load_lds: an operand whose
// k is fast in memory as rows of eight 16-byte chunks, one whose k is slow as it lies in memory, to be transposed by the LDS read (layouts and
// swizzles: gemm_tile.hpp).  Two buffers: the next slab's loads run while this one is multiplied.  ONE buffer: a slab's fragments are all read into registers,
// the next slab's loads go out behind a barrier and the products run from registers; two workgroups a CU take turns.
struct NsOperand { const _Float16* p; long long ld, plane; };      // tile origin; elements to the second halves

template <int TM, int TN, bool SPLIT, bool AS, bool BS, int NST>
__device__ __forceinline__ void ns_tile(f32x16_t (&acc)[TM][TN], const NsOperand& A, const NsOperand& B, int slab0, int slab1, int trips, uint4* smem) {
    static_assert(NST == 1 || (NST == 2 && !(SPLIT && TM == 2)), "one buffer, or two");
    constexpr bool ONE = NST == 1;
    constexpr int BM = 64 * TM, BN = 64 * TN, PL = SPLIT ? 2 : 1, PA = BM * 8, PB = BN * 8, STAGE = PL * (PA + PB);   // (in 16-byte words)
    constexpr int NIA = 2 * TM, NIB = 2 * TN, CPA = BM / 8, CPB = BN / 8;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6 & 3), wm = wv >> 1, wn = wv & 1;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    unsigned voa[NIA], vob[NIB];
    auto place = [&](auto cpr, bool slow, int j, long long ld) {
        constexpr int CPR = decltype(cpr)::value;
        const int jj = 4 * j + wv, kt = (64 / CPR) * jj + lane / CPR, pos = lane % CPR, r = 8 * jj + (lane >> 3);
        const int mc = (((pos >> 1) ^ tr_swz<CPR>(kt)) << 1) | (pos & 1), kc = (lane & 7) ^ swz(r);
        return slow ? (unsigned)(kt * ld * 2 + mc * 16) : (unsigned)(r * ld * 2 + kc * 16);
    };
#pragma unroll
    for (int j = 0; j < NIA; ++j) voa[j] = place(std::integral_constant<int, (CPA < 64 ? CPA : 64)>{}, AS, j, A.ld);
#pragma unroll
    for (int j = 0; j < NIB; ++j) vob[j] = place(std::integral_constant<int, (CPB < 64 ? CPB : 64)>{}, BS, j, B.ld);
    auto dma = [](unsigned lds_addr, const char* gbase, unsigned voff) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(gbase) : "memory");
    };
    auto issue = [&](int it) __attribute__((always_inline)) {
        const char* pa = uniform(A.p + (AS ? (long long)it * 64 * A.ld : (long long)it * 64));
        const char* pb = uniform(B.p + (BS ? (long long)it * 64 * B.ld : (long long)it * 64));
        const unsigned sb = lds0 + (unsigned)(((it - slab0) % NST) * STAGE * 16);
#pragma unroll
        for (int pl = 0; pl < PL; ++pl) {
#pragma unroll
            for (int j = 0; j < NIA; ++j) dma(sb + (unsigned)(pl * PA * 16 + (4 * j + wv) * 1024), pl ? uniform(pa + A.plane * 2) : pa, voa[j]);
#pragma unroll
            for (int j = 0; j < NIB; ++j) dma(sb + (unsigned)((PL * PA + pl * PB) * 16 + (4 * j + wv) * 1024), pl ? uniform(pb + B.plane * 2) : pb, vob[j]);
        }
    };
    // fragment reads: lane l holds k = 8 (l / 32) .. of row l % 32 of its 32-row block
    const int arow = wm * 32 * TM + (lane & 31), brow = wn * 32 * TN + (lane & 31);
    int ra[4], rb[4], ta[TM], tb[TN];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        ra[q] = arow * CHUNKS + ((2 * q + (lane >> 5)) ^ swz(arow));
        rb[q] = brow * CHUNKS + ((2 * q + (lane >> 5)) ^ swz(brow));
    }
    {
        const int g = lane >> 4, li = lane & 15;
#pragma unroll
        for (int i = 0; i < TM; ++i)
            ta[i] = (8 * (g >> 1) + (li >> 2)) * (BM * 2) + (((wm * 2 * TM + 2 * i + (g & 1)) ^ tr_swz<CPA>(li >> 2)) << 5) + (li & 3) * 8;
#pragma unroll
        for (int i = 0; i < TN; ++i)
            tb[i] = (8 * (g >> 1) + (li >> 2)) * (BN * 2) + (((wn * 2 * TN + 2 * i + (g & 1)) ^ tr_swz<CPB>(li >> 2)) << 5) + (li & 3) * 8;
    }
    auto frag_a = [&](const uint4* s, int i, int q) __attribute__((always_inline)) {
        if constexpr (AS) return lfrag_tr<BM * 2>(reinterpret_cast<const char*>(s) + ta[i], 16 * q);
        else return s[ra[(i & 1) ? (q ^ 2) : q] + i * 32 * CHUNKS];
    };
    auto frag_b = [&](const uint4* s, int i, int q) __attribute__((always_inline)) {
        if constexpr (BS) return lfrag_tr<BN * 2>(reinterpret_cast<const char*>(s) + tb[i], 16 * q);
        else return s[rb[(i & 1) ? (q ^ 2) : q] + i * 32 * CHUNKS];
    };
    auto mma = [&](const uint4 (&x)[TM], const uint4 (&y)[TN]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, x[i]), __builtin_bit_cast(f16x8_t, y[j]), acc[i][j], 0, 0, 0);
    };
    if (slab0 < slab1) issue(slab0);
    if constexpr (ONE) {
        uint4 fa[4][PL][TM], fb[4][PL][TN];
        for (int it = slab0; it < slab1; ++it) {
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int pl = 0; pl < PL; ++pl) {
#pragma unroll
                    for (int i = 0; i < TM; ++i) fa[q][pl][i] = frag_a(smem + pl * PA, i, q);
#pragma unroll
                    for (int i = 0; i < TN; ++i) fb[q][pl][i] = frag_b(smem + PL * PA + pl * PB, i, q);
                }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (it + 1 < slab1) issue(it + 1);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if constexpr (SPLIT) { mma(fa[q][1], fb[q][0]); mma(fa[q][0], fb[q][1]); }
                mma(fa[q][0], fb[q][0]);
            }
        }
    } else {
        for (int it = slab0; it < slab0 + trips; ++it) {       // (every wavefront of the workgroup goes through as many barriers)
            // (the slab has landed, this wavefront's reads of the buffer that is filled next have come)
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (it + 1 < slab1) issue(it + 1);
            const uint4* sa = smem + ((it - slab0) % NST) * STAGE;
            const uint4* sb = sa + PL * PA;
            if (it >= slab1) continue;
            // (the next fragments are on their way while these are multiplied)
            uint4 af[2][PL][TM], bf[2][PL][TN];
            auto read = [&](int q, uint4 (&x)[PL][TM], uint4 (&y)[PL][TN]) __attribute__((always_inline)) {
#pragma unroll
                for (int pl = 0; pl < PL; ++pl) {
#pragma unroll
                    for (int i = 0; i < TM; ++i) x[pl][i] = frag_a(sa + pl * PA, i, q);
#pragma unroll
                    for (int i = 0; i < TN; ++i) y[pl][i] = frag_b(sb + pl * PB, i, q);
                }
            };
            read(0, af[0], bf[0]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (q < 3) read(q + 1, af[(q + 1) & 1], bf[(q + 1) & 1]);
                if constexpr (SPLIT) { mma(af[q & 1][1], bf[q & 1][0]); mma(af[q & 1][0], bf[q & 1][1]); }
                mma(af[q & 1][0], bf[q & 1][0]);
            }
        }
    }
    __syncthreads();                                        // the epilogue reuses the buffers
}

// The same by SETS sets of 2 x 2 wavefronts, each with buffers of its own and its part of the contraction; the first set is left with the sum.  For launches of
// no more tiles than CUs: a workgroup alone on a CU waits for its LDS reads and its products in turn, two sets for one another's: a step of two matrices of
// 1204 x 602 in float S 16 (in two parts and a sum) -> 13 us, B 13 -> 11; 1024 x 1024, five steps, 240 -> 217.
template <int SETS, int TM, int TN, bool SPLIT, bool AS, bool BS, int NST>
__device__ __forceinline__ void ns_tile_of_sets(f32x16_t (&acc)[TM][TN], const NsOperand& A, const NsOperand& B, int slab0, int slab1, uint4* smem) {
    if constexpr (SETS == 1) ns_tile<TM, TN, SPLIT, AS, BS, NST>(acc, A, B, slab0, slab1, slab1 - slab0, smem);
    else {
        constexpr int WORDS = NST * (SPLIT ? 2 : 1) * 64 * (TM + TN) * 8;
        const int set = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), part = (slab1 - slab0 + 1) / 2, t = threadIdx.x & 255;
        ns_tile<TM, TN, SPLIT, AS, BS, NST>(acc, A, B, slab0 + set * part, set ? slab1 : slab0 + part, part, smem + set * WORDS);
        f32x4_t* other = reinterpret_cast<f32x4_t*>(smem);
        if (set) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) other[((i * TN + j) * 4 + e) * 256 + t] = f32x4_t{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
        }
        __syncthreads();
        if (!set) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] += other[((i * TN + j) * 4 + (e >> 2)) * 256 + t][e & 3];
        }
        __syncthreads();                                    // (the epilogue reuses the place)
    }
}

// The tile's values, eight of a row at a time, each wavefront its own part through its own stretch of LDS, whose reads are conflict-free along
// rows and columns.  What an element is combined with is asked for a block of 32 rows ahead, in front of the stores of the block before (a wavefront's memory answers come in
// order, so that a load behind a store waits for it: 68 -> 63 us a product of four layers of 512 cells): load(row, column) -> aux; f(row, column, values, aux) changes the values and stores them; mirror(row, column, values) gets the same
// values of the transposed tile (`twice`).
template <int TM, int TN, typename L, typename F, typename G>
__device__ __forceinline__ void ns_values(const f32x16_t (&acc)[TM][TN], uint4* smem, bool twice, L&& load, F&& f, G&& mirror) {
    constexpr int LD = 32 * TN + 4, NQ = 2 * TN;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, wm = wv >> 1, wn = wv & 1;
    float* s = reinterpret_cast<float*>(smem) + wv * 32 * LD;
    const int col0 = wn * 32 * TN;
    decltype(load(0, 0)) aux[2][NQ];
    auto ask = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) { const int c = lane + 64 * q; aux[i & 1][q] = load(wm * 32 * TM + 32 * i + c / (4 * TN), col0 + c % (4 * TN) * 8); }
    };
    ask(0);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row0 = wm * 32 * TM + 32 * i;
        if (i + 1 < TM) ask(i + 1);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[(8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * LD + 32 * j + (lane & 31)] = acc[i][j][e];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const int c = lane + 64 * q, r = c / (4 * TN), c0 = c % (4 * TN) * 8;
            f32x4_t* at = reinterpret_cast<f32x4_t*>(s + r * LD + c0);
            const f32x4_t x = at[0], y = at[1];
            float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
            f(row0 + r, col0 + c0, v, aux[i & 1][q]);
            if (twice) { at[0] = f32x4_t{v[0], v[1], v[2], v[3]}; at[1] = f32x4_t{v[4], v[5], v[6], v[7]}; }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (twice) {
            // 32 TN columns of 32 rows, a column's eight rows a lane
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const int c = lane + 64 * q, col = c % (32 * TN), r0 = c / (32 * TN) * 8;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = s[(r0 + e) * LD + col];
                mirror(col0 + col, row0 + r0, v);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    }
}
struct Halves { f16x8_t h, l; f32x4_t d0, d1; float di; };
template <bool LOW, bool LAST> struct Applied { f16x8_t h; std::conditional_t<LOW, u32x2_t, f16x8_t> l; float di; f32x4_t w[LAST ? 2 : 1]; };

// tile number t of those on and above the diagonal, column by column: row <= column
__device__ __forceinline__ void upper(int t, int* row, int* col) {
    int c = 0;
    while (t > c) { t -= c + 1; ++c; }
    *row = t; *col = c;
}

// SPLIT: the operands' second halves are multiplied too; LO: S and B have second halves; LOW: X's second part is held in eight bits
template <int TM, int TN, bool SPLIT, bool LO, bool LOW, int PH, int NST, int SETS>
__global__ __launch_bounds__(256 * SETS, 2) void ns_product_kernel(MuonPlan p, MuonArgs a, _Float16* ws, float* diag, float* part, int from, const int* here) {
    extern __shared__ uint4 smem[];
    constexpr int BM = 64 * TM, BN = 64 * TN;
    // ids go round-robin to the eight XCDs: of each group (they differ in the length of their contractions) each XCD takes an eighth, neighbouring tiles
    const int (&starts)[MUON_MAX_GROUPS] = PH == PH_GRAM ? p.at.gram : PH == PH_SQUARE ? p.at.square : p.at.apply;
    const int group = group_of(starts, blockIdx.x);
    const MuonGroup& g = p.g[group];
    const int units = g.count * (PH == PH_GRAM ? g.grams * g.splits : PH == PH_SQUARE ? g.grams : g.applies), own = blockIdx.x - starts[group];
    const int lin = (own & 7) * ((units + 7) / 8) + (own >> 3);
    if (lin >= units) return;
    // (matrices that take no part are multiplied all the same: asked in every launch, the question costs the calls without ids 1 %)
    if (PH == PH_LAST && here && !here[lin / g.applies]) return;
    f32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    if constexpr (PH == PH_GRAM || PH == PH_SQUARE) {
        static_assert(TM == TN, "tiles on the diagonal are squares");
        int local = lin, split = 0;
        if (PH == PH_GRAM) { split = local % g.splits; local /= g.splits; }
        const int k = local / g.grams;
        int tr, tc;
        upper(local % g.grams, &tr, &tc);
        _Float16* s = ws + g.s + (long long)k * g.mp * g.mp;
        float* sd = diag + g.diag + (long long)k * g.mp;
        float* bd = sd + (long long)g.count * g.mp;
        _Float16* out = PH == PH_GRAM ? s : ws + g.b + (long long)k * g.mp * g.mp;
        auto mirror = [&](int r, int c, const float (&v)[8]) {
            const long long o = (long long)(tc * BM + r) * g.mp + tr * BM + c;
            put_halves(out + o, LO ? out + g.splane + o : nullptr, v);
        };
        if constexpr (PH == PH_GRAM) {
            const _Float16* x = ws + g.x[from] + (long long)k * g.rp * g.cp;
            const int slabs = (g.tall ? g.rp : g.cp) / 64, per = (slabs + g.splits - 1) / g.splits;
            const int s0 = min(slabs, split * per), s1 = min(slabs, s0 + per);
            if (g.tall) ns_tile_of_sets<SETS, TM, TN, SPLIT, true, true, NST>(acc, {x + tr * BM, g.cp, g.xplane}, {x + tc * BM, g.cp, g.xplane}, s0, s1, smem);
            else ns_tile_of_sets<SETS, TM, TN, SPLIT, false, false, NST>(acc, {x + (long long)tr * BM * g.cp, g.cp, g.xplane}, {x + (long long)tc * BM * g.cp, g.cp, g.xplane}, s0, s1, smem);
            if (SETS > 1 && threadIdx.x >= 256) return;
            const bool whole = g.splits == 1;
            float* sum = part + g.part + ((long long)local * g.splits + split) * BM * BM;
            ns_values(acc, smem, whole && tr != tc, [](int, int) { return 0; }, [&](int r, int c, float (&v)[8], int) {
                if (!whole) {
                    *reinterpret_cast<f32x4_t*>(sum + r * BM + c) = f32x4_t{v[0], v[1], v[2], v[3]};
                    *reinterpret_cast<f32x4_t*>(sum + r * BM + c + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
                    return;
                }
                const int row = tr * BM + r, col = tc * BM + c, on = row - col;
                const long long o = (long long)row * g.mp + col;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] *= DOWN;
                    if (on == e) { sd[row] = DOWN * v[e]; v[e] = 0.0f; }
                }
                put_halves(out + o, LO ? out + g.splane + o : nullptr, v);
            }, mirror);
        } else {
            const NsOperand A{s + (long long)tr * BM * g.mp, g.mp, g.splane}, B{s + (long long)tc * BM * g.mp, g.mp, g.splane};
            ns_tile_of_sets<SETS, TM, TN, SPLIT, false, false, NST>(acc, A, B, 0, g.mp / 64, smem);
            if (SETS > 1 && threadIdx.x >= 256) return;
            ns_values(acc, smem, tr != tc, [&](int r, int c) {
                const int row = tr * BM + r, col = tc * BM + c;
                const _Float16* at = s + (long long)row * g.mp + col;
                Halves x;
                x.h = *reinterpret_cast<const f16x8_t*>(at);
                if constexpr (LO) x.l = *reinterpret_cast<const f16x8_t*>(at + g.splane); else x.l = f16x8_t{};
                x.di = sd[row];
                x.d0 = *reinterpret_cast<const f32x4_t*>(sd + col);
                x.d1 = *reinterpret_cast<const f32x4_t*>(sd + col + 4);
                return x;
            }, [&](int r, int c, float (&v)[8], const Halves& x) {
                const int row = tr * BM + r, col = tc * BM + c, on = row - col;
                const long long o = (long long)row * g.mp + col;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = (float)x.h[e] + (float)x.l[e], full = NS_C * DOWN * v[e];
                    if (on == e) bd[row] = NS_B * x.di + NS_C * x.di * x.di + DOWN * full;
                    v[e] = on == e ? 0.0f : NS_B * y + NS_C * (x.di + (e < 4 ? x.d0[e & 3] : x.d1[e & 3])) * y + full;
                }
                put_halves(out + o, LO ? out + g.splane + o : nullptr, v);
            }, mirror);
        }
    } else {
        const int local = lin, k = local / g.applies, t = local % g.applies, nc = g.cp / BN;
        const int tr = t / nc, tc = t % nc;
        const _Float16* x = ws + g.x[from] + (long long)k * g.rp * g.cp;
        const _Float16* b = ws + g.b + (long long)k * g.mp * g.mp;
        if (g.tall) ns_tile_of_sets<SETS, TM, TN, SPLIT, false, false, NST>(acc, {x + (long long)tr * BM * g.cp, g.cp, g.xplane}, {b + (long long)tc * BN * g.mp, g.mp, g.splane}, 0, g.mp / 64, smem);
        else ns_tile_of_sets<SETS, TM, TN, SPLIT, false, true, NST>(acc, {b + (long long)tr * BM * g.mp, g.mp, g.splane}, {x + tc * BN, g.cp, g.xplane}, 0, g.mp / 64, smem);
        if (SETS > 1 && threadIdx.x >= 256) return;
        _Float16* to = ws + g.x[from ^ 1] + (long long)k * g.rp * g.cp;
        const unsigned char* xl = low_of(g, ws, from, k);
        unsigned char* tl = low_of(g, ws, from ^ 1, k);
        const long long at = tensor_at(g, k);
        const float* bd = diag + g.diag + (long long)(g.count + k) * g.mp;
        const float shrink = 1.0f - a.lr * a.decay, step = a.lr * sqrtf(fmaxf(1.0f, (float)g.rows / (float)g.cols)) * DOWN;
        // (a lane's columns are the same in all of its rows)
        f32x4_t d0{}, d1{};
        if (g.tall) {
            const float* d = bd + tc * BN + (threadIdx.x >> 6 & 1) * 32 * TN + (threadIdx.x & 63) % (4 * TN) * 8;
            d0 = *reinterpret_cast<const f32x4_t*>(d);
            d1 = *reinterpret_cast<const f32x4_t*>(d + 4);
        }
        ns_values(acc, smem, false, [&](int r, int c) {
            const int row = tr * BM + r, col = tc * BN + c;
            const long long o = (long long)row * g.cp + col;
            Applied<LOW, PH == PH_LAST> u;
            u.h = *reinterpret_cast<const f16x8_t*>(x + o);
            if constexpr (LOW) u.l = *reinterpret_cast<const u32x2_t*>(xl + o); else u.l = *reinterpret_cast<const f16x8_t*>(x + g.xplane + o);
            u.di = g.tall ? 0.0f : bd[row];
            if constexpr (PH == PH_LAST) {
                if (a.theta && row < g.rows && col + 8 <= g.cols) {
                    const f32x4u_t* w = reinterpret_cast<const f32x4u_t*>(a.theta + at + (long long)row * g.cols + col);
                    u.w[0] = w[0]; u.w[1] = w[1];
                }
            }
            return u;
        }, [&](int r, int c, float (&v)[8], const Applied<LOW, PH == PH_LAST>& u) {
            const int row = tr * BM + r, col = tc * BN + c;
            const long long o = (long long)row * g.cp + col;
            f16x8_t l;
            if constexpr (LOW) l = low(u.l); else l = u.l;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (NS_A + (g.tall ? (e < 4 ? d0[e & 3] : d1[e & 3]) : u.di)) * ((float)u.h[e] + (float)l[e]) + DOWN * v[e];
            if constexpr (PH == PH_APPLY && LOW) put_low(to + o, tl + o, v);
            else if constexpr (PH == PH_APPLY) put_halves(to + o, to + g.xplane + o, v);
            else {
                if (row >= g.rows || col >= g.cols) return;
                const long long q = at + (long long)row * g.cols + col;
                const int n = min(8, g.cols - col);
                if (a.theta) {
                    if (n == 8) {
                        f32x4_t w[2] = {u.w[0], u.w[1]};
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[i][e] = shrink * w[i][e] - step * v[4 * i + e];
                            *reinterpret_cast<f32x4u_t*>(a.theta + q + 4 * i) = w[i];
                            if (a.shadow) { u32x2_t z; z[0] = pack_bf2(w[i][0], w[i][1]); z[1] = pack_bf2(w[i][2], w[i][3]); *reinterpret_cast<u32x2u_t*>(a.shadow + q + 4 * i) = z; }
                        }
                    } else {
                        float w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = e < n ? a.theta[q + e] : 0.0f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) if (e < n) {
                            w[e] = shrink * w[e] - step * v[e];
                            a.theta[q + e] = w[e];
                            if (a.shadow) a.shadow[q + e] = f2bf(w[e]);
                        }
                    }
                } else if (n == 8) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const f32x4_t w{DOWN * v[4 * i], DOWN * v[4 * i + 1], DOWN * v[4 * i + 2], DOWN * v[4 * i + 3]};
                        if (a.out_bf16) { u32x2_t z; z[0] = pack_bf2(w[0], w[1]); z[1] = pack_bf2(w[2], w[3]); *reinterpret_cast<u32x2u_t*>(static_cast<unsigned short*>(a.out) + q + 4 * i) = z; }
                        else *reinterpret_cast<f32x4u_t*>(static_cast<float*>(a.out) + q + 4 * i) = w;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (e < n) {
                        if (a.out_bf16) static_cast<unsigned short*>(a.out)[q + e] = f2bf(DOWN * v[e]);
                        else static_cast<float*>(a.out)[q + e] = DOWN * v[e];
                    }
                }
            }
        }, [](int, int, const float (&)[8]) {});
    }
}

// The parts of split Gram tiles, in order: 64 x 64 of a tile a workgroup.
template <int T, bool LO>
__global__ __launch_bounds__(256) void ns_gram_sum_kernel(MuonPlan p, _Float16* ws, float* diag, const float* part) {
    constexpr int BM = 64 * T, LD = 65;
    __shared__ float s[64 * LD];
    const int group = group_of(p.at.sum, blockIdx.x);
    const MuonGroup& g = p.g[group];
    const int local = blockIdx.x - p.at.sum[group], tile = local / (T * T), sub = local % (T * T), k = tile / g.grams;
    int tr, tc;
    upper(tile % g.grams, &tr, &tc);
    const int sr = sub / T * 64, sc = sub % T * 64;
    const float* from = part + g.part + (long long)tile * g.splits * BM * BM;
    const int r = threadIdx.x >> 2, c0 = (threadIdx.x & 3) * 16;
    f32x4_t v[4] = {};
#pragma unroll 4
    for (int i = 0; i < g.splits; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) v[w] += *reinterpret_cast<const f32x4_t*>(from + (long long)i * BM * BM + (sr + r) * BM + sc + c0 + 4 * w);
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool own = tr == tc && sr + r == sc + c0 + 4 * w + e;
            if (own) diag[g.diag + (long long)k * g.mp + tr * BM + sr + r] = DOWN * DOWN * v[w][e];
            s[r * LD + c0 + 4 * w + e] = own ? 0.0f : DOWN * v[w][e];
        }
    __syncthreads();
    _Float16* out = ws + g.s + (long long)k * g.mp * g.mp;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float x[8];
        const long long o = (long long)(tr * BM + sr + r) * g.mp + tc * BM + sc + c0 + 8 * w;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[r * LD + c0 + 8 * w + e];
        put_halves(out + o, LO ? out + g.splane + o : nullptr, x);
        if (tr == tc) continue;
        const long long m = (long long)(tc * BM + sc + r) * g.mp + tr * BM + sr + c0 + 8 * w;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[(c0 + 8 * w + e) * LD + r];
        put_halves(out + m, LO ? out + g.splane + m : nullptr, x);
    }
}

// ---- small matrices: all steps of a matrix in one workgroup -----------------------------------------------------------------
// What the general path spends on them is twenty launches of a few microseconds.  A matrix whose short side is at most 64 and which fits LDS is read
// once, taken through the five steps there and written once, by sixteen wavefronts; the tensors that are not orthogonalised are further workgroups of the same
// launch.  48 factors of 16 x 1024 196 -> 28 us, a layer of 32 cells 94 -> 21: three to four microseconds are the launch, nine the way in and out, three a step (four barriers, and LDS, through
// which all of X goes twice).  [m][n] with m <= n in LDS as two planes of halves (rows of n + 8, so that sixteen rows' chunks spread over the banks); all products use both planes.
constexpr int SMALL_THREADS = 1024, SMALL_SIDE = 64, SMALL_LDS = 160 * 1024 - 256;
constexpr int small_parts(int mb) { return mb == 1 ? 16 : mb == 2 ? 4 : 1; }   // stretches of the columns that a tile of S is summed over
struct SmallLds { int ldn, lds, x, s, b, red, d, bytes; };      // row lengths in halves; byte offsets
__host__ __device__ inline SmallLds small_lds(int n, int mb) {
    SmallLds l{};
    const int mp = 16 * mb, kp = (mp + 31) / 32 * 32;
    l.ldn = (n + 31) / 32 * 32 + 8;
    l.lds = kp + 8;
    l.x = 0;
    l.s = l.x + 2 * mp * l.ldn * 2;
    l.b = l.s + 2 * mp * l.lds * 2;
    l.red = l.b + 2 * mp * l.lds * 2;
    l.d = l.red + (small_parts(mb) > 1 ? small_parts(mb) : 0) * mp * mp * 4;
    l.bytes = l.d + mp * 4;
    return l;
}
// (three chains, so that none waits for another's end)
__device__ __forceinline__ void mma_halves(f32x4_t (&acc)[3], const uint4 (&a)[2], const uint4 (&b)[2]) {
    auto one = [&](f32x4_t& c, const uint4& x, const uint4& y) { c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, x), __builtin_bit_cast(f16x8_t, y), c, 0, 0, 0); };
    one(acc[0], a[1], b[0]); one(acc[1], a[0], b[1]); one(acc[2], a[0], b[0]);
}
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4_t four(const _Float16* at, int plane) {
    const f16x4_t h = *reinterpret_cast<const f16x4_t*>(at), l = *reinterpret_cast<const f16x4_t*>(at + plane);
    return f32x4_t{(float)h[0] + (float)l[0], (float)h[1] + (float)l[1], (float)h[2] + (float)l[2], (float)h[3] + (float)l[3]};
}
__device__ __forceinline__ void put_four(_Float16* at, int plane, const f32x4_t& v) {
    f16x4_t h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) { h[e] = (_Float16)v[e]; l[e] = (_Float16)(v[e] - (float)h[e]); }
    *reinterpret_cast<f16x4_t*>(at) = h;
    *reinterpret_cast<f16x4_t*>(at + plane) = l;
}
template <int MB>
__global__ __launch_bounds__(SMALL_THREADS) void muon_small_kernel(MuonPlan p, MuonArgs a, MuonIds of) {
    extern __shared__ uint4 smem[];
    __shared__ double lds_sum[16];
    constexpr int MP = 16 * MB, TILES = MB * MB, PARTS = small_parts(MB), KS = (MP + 31) / 32, PLACES = MB <= 2 ? 2 : 1;
    constexpr bool KEEP = MB <= 2;          // B's fragments stay in registers
    const int group = group_of(p.at.apply, blockIdx.x);
    const MuonGroup& g = p.g[group];
    const int local = blockIdx.x - p.at.apply[group], tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto direction = [&](float gr, float v) { return !a.velocity ? gr : a.nesterov ? gr + a.momentum * v : v; };
    if (!g.ortho) {
        const int k = local / g.chunks;
        const long long size = (long long)g.rows * g.cols, e0 = (long long)(local % g.chunks) * FLAT, at = tensor_at(g, k) + e0;
        const int len = (int)min((long long)FLAT, size - e0);
        for (int i = tid; i < len; i += SMALL_THREADS) {
            const float gr = a.grad[at + i];
            float v = 0.0f;
            if (a.velocity) { v = a.momentum * a.velocity[at + i] + gr; a.velocity[at + i] = v; }
            const float w = a.theta[at + i] - a.lr_rest * direction(gr, v);
            a.theta[at + i] = w;
            if (a.shadow) a.shadow[at + i] = f2bf(w);
        }
        return;
    }
    if (of.ids && !in_ids(of, local)) return;
    const long long at = tensor_at(g, local);
    const int size = g.rows * g.cols, n = max(g.rows, g.cols);
    const bool tall = g.tall != 0;
    const SmallLds l = small_lds(n, MB);
    char* base = reinterpret_cast<char*>(smem);
    _Float16* X = reinterpret_cast<_Float16*>(base + l.x);
    _Float16* S = reinterpret_cast<_Float16*>(base + l.s);
    _Float16* Bq = reinterpret_cast<_Float16*>(base + l.b);
    float* red = reinterpret_cast<float*>(base + l.red);
    float* sd = reinterpret_cast<float*>(base + l.d);
    const int xp = MP * l.ldn, sp = MP * l.lds;             // elements of a plane
    for (int i = tid; i < (l.red - l.x) / 16; i += SMALL_THREADS) smem[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    // Eight elements a thread on their way at a time.  d waits in LDS for its norm, its bits' upper half where the first half will be and the lower
    // half where the second one will be; a thread comes back to its own elements.
    const int dr = SMALL_THREADS / g.cols, dc = SMALL_THREADS - dr * g.cols, r_first = tid / g.cols, c_first = tid - r_first * g.cols;
    const int by_row = tall ? 1 : l.ldn, by_col = tall ? l.ldn : 1;
    auto eight = [&](auto&& f) {
        int r = r_first, c = c_first;
        for (int i0 = tid; i0 < size; i0 += 8 * SMALL_THREADS) {
            int place[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                place[q] = r * by_row + c * by_col;
                r += dr; c += dc;
                if (c >= g.cols) { c -= g.cols; ++r; }
            }
            f([&](int q) { return min(i0 + q * SMALL_THREADS, size - 1); }, [&](int q) { return i0 + q * SMALL_THREADS < size; }, place);
        }
    };
    unsigned short* bits = reinterpret_cast<unsigned short*>(X);
    double sum = 0.0;
    eight([&](auto at_q, auto in, const int (&place)[8]) {
        float gr[8], v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) { gr[q] = a.grad[at + at_q(q)]; v[q] = a.velocity ? a.velocity[at + at_q(q)] : 0.0f; }
#pragma unroll
        for (int q = 0; q < 8; ++q) if (in(q)) {
            if (a.velocity) { v[q] = a.momentum * v[q] + gr[q]; a.velocity[at + at_q(q)] = v[q]; }
            const float d = direction(gr[q], v[q]);
            sum += (double)d * d;
            const unsigned w = __builtin_bit_cast(unsigned, d);
            const int o = place[q];
            bits[o] = (unsigned short)(w >> 16);
            bits[xp + o] = (unsigned short)w;
        }
    });
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) lds_sum[wave] = sum;
    __syncthreads();
    double norm2 = 0.0;
    for (int i = 0; i < 16; ++i) norm2 += lds_sum[i];
    const double scale = norm2 == 0.0 ? 0.0 : UP / sqrt(norm2);
    const float whole = norm2 <= 1.7e308 ? 0.0f : __builtin_nanf("");
    eight([&](auto, auto in, const int (&place)[8]) {
        float d[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) if (in(q)) d[q] = (float)(__builtin_bit_cast(float, (unsigned)bits[place[q]] << 16 | bits[xp + place[q]]) * scale) + whole;
#pragma unroll
        for (int q = 0; q < 8; ++q) if (in(q)) {
            const _Float16 h = (_Float16)d[q];
            X[place[q]] = h;
            X[xp + place[q]] = (_Float16)(d[q] - (float)h);
        }
    });
    __syncthreads();
    const int fr = lane & 15, fg = lane >> 4, ksteps = (n + 31) / 32, cblocks = (n + 15) / 16;
    const int tile = wave % TILES, part = wave / TILES, ti = tile / MB, tj = tile % MB;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    auto row_frag = [&](uint4 (&f)[2], const _Float16* m, int plane, int ld, int row, int k) {
#pragma unroll
        for (int q = 0; q < 2; ++q) f[q] = *reinterpret_cast<const uint4*>(m + q * plane + row * ld + k);
    };
#pragma unroll 1
    for (int step = 0; step < NS_STEPS; ++step) {
        // A lane's four results lie below one another in a column; S and B are symmetric, and X's tile is computed transposed: so they leave as four
        // neighbours of a row.
        // S = X X^T: a wavefront one tile, every PARTS-th stretch of 32 columns
        auto put_s = [&](int r, int c, f32x4_t v) {         // columns c .. c + 3
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] *= DOWN;
                if (r == c + e) { sd[r] = DOWN * v[e]; v[e] = 0.0f; }
            }
            put_four(S + r * l.lds + c, sp, v);
        };
        if (wave < TILES * PARTS) {
            f32x4_t acc[3] = {};
#pragma unroll 2
            for (int k = part; k < ksteps; k += PARTS) {
                uint4 x[2], y[2];
                row_frag(x, X, xp, l.ldn, 16 * ti + fr, 32 * k + 8 * fg);
                if constexpr (MB > 1) row_frag(y, X, xp, l.ldn, 16 * tj + fr, 32 * k + 8 * fg); else { y[0] = x[0]; y[1] = x[1]; }
                mma_halves(acc, x, y);
            }
            const f32x4_t v = acc[2] + (acc[0] + acc[1]);
            if constexpr (PARTS > 1) *reinterpret_cast<f32x4_t*>(red + part * MP * MP + (16 * tj + fr) * MP + 16 * ti + 4 * fg) = v;
            else put_s(16 * tj + fr, 16 * ti + 4 * fg, v);
        }
        __syncthreads();
        if constexpr (PARTS > 1) {
            if (tid < MP * MP / 4) {
                f32x4_t v{};
#pragma unroll
                for (int q = 0; q < PARTS; ++q) v += *reinterpret_cast<const f32x4_t*>(red + q * MP * MP + 4 * tid);
                put_s(4 * tid / MP, 4 * tid % MP, v);
            }
            __syncthreads();
        }
        if (wave < TILES) {     // B = a + b S + c S^2: both planes are multiplied, so that its diagonal may lie in them
            f32x4_t acc[3] = {};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint4 x[2], y[2];
                row_frag(x, S, sp, l.lds, 16 * ti + fr, 32 * k + 8 * fg);
                row_frag(y, S, sp, l.lds, 16 * tj + fr, 32 * k + 8 * fg);
                mma_halves(acc, x, y);
            }
            const int r = 16 * tj + fr, c = 16 * ti + 4 * fg;
            const float dr_ = sd[r];
            const f32x4_t old = four(S + r * l.lds + c, sp), dc_ = *reinterpret_cast<const f32x4_t*>(sd + c);
            f32x4_t v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float full = NS_C * DOWN * (acc[2][e] + (acc[0][e] + acc[1][e]));
                v[e] = r == c + e ? UP * (NS_A + NS_B * dr_ + NS_C * dr_ * dr_) + full : NS_B * old[e] + NS_C * (dr_ + dc_[e]) * old[e] + full;
            }
            put_four(Bq + r * l.lds + c, sp, v);
        }
        __syncthreads();
        // X = B X: a wavefront whole columns, sixteen at a time (of low matrices in two places), which nobody else reads or writes; all
        // that they need is read before the first is written
        uint4 fb[KEEP ? MB : 1][KEEP ? KS : 1][2];
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int k = 0; k < KS; ++k) row_frag(fb[i][k], Bq, sp, l.lds, 16 * i + fr, 32 * k + 8 * fg);
        }
#pragma unroll 1
        for (int cb = wave; cb < cblocks; cb += 16 * PLACES) {
            const int at_col[2] = {16 * cb, 16 * (cb + 16 < cblocks ? cb + 16 : cb)};
            f32x4_t acc[PLACES][MB][3] = {};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint4 y[PLACES][2];
                const int kr = 32 * k + 8 * fg;            // (rows beyond the matrix: zero, from a place that exists)
                const bool in = kr < MP;
#pragma unroll
                for (int j = 0; j < PLACES; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const char* from = reinterpret_cast<const char*>(X + h * xp + ((in ? kr : 0) + (fr >> 2)) * l.ldn + at_col[j] + (fr & 3) * 4);
                        const uint2 l2 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)from));
                        const uint2 h2 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(from + 4 * l.ldn * 2)));
                        y[j][h] = in ? make_uint4(l2.x, l2.y, h2.x, h2.y) : none;
                    }
#pragma unroll
                for (int i = 0; i < MB; ++i) {
                    uint4 x[2];
                    if constexpr (KEEP) { x[0] = fb[i][k][0]; x[1] = fb[i][k][1]; } else row_frag(x, Bq, sp, l.lds, 16 * i + fr, 32 * k + 8 * fg);
#pragma unroll
                    for (int j = 0; j < PLACES; ++j) mma_halves(acc[j][i], y[j], x);
                }
            }
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < PLACES; ++j)            // (the same place twice where there is one block left)
                    put_four(X + (16 * i + fr) * l.ldn + at_col[j] + 4 * fg, xp, DOWN * (acc[j][i][2] + (acc[j][i][0] + acc[j][i][1])));
        }
        __syncthreads();
    }
    const float shrink = 1.0f - a.lr * a.decay, step = a.lr * sqrtf(fmaxf(1.0f, (float)g.rows / (float)g.cols)) * DOWN;
    eight([&](auto at_q, auto in, const int (&place)[8]) {
        float w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = a.theta ? a.theta[at + at_q(q)] : 0.0f;
#pragma unroll
        for (int q = 0; q < 8; ++q) if (in(q)) {
            const int o = place[q];
            const long long to = at + at_q(q);
            const float v = (float)X[o] + (float)X[xp + o];
            if (a.theta) {
                const float x = shrink * w[q] - step * v;
                a.theta[to] = x;
                if (a.shadow) a.shadow[to] = f2bf(x);
            } else if (a.out_bf16) static_cast<unsigned short*>(a.out)[to] = f2bf(DOWN * v);
            else static_cast<float*>(a.out)[to] = DOWN * v;
        }
    });
}

constexpr int lds_bytes(int TM, int TN, bool split, int nst, int sets) {
    const int loop = sets * nst * (split ? 2 : 1) * 64 * (TM + TN) * 128, values = 4 * 32 * (32 * TN + 4) * 4;
    return loop > values ? loop : values;
}
template <int TM, int TN, bool SPLIT, bool LO, bool LOW, int PH, int NST, int SETS>
void run_product(int n, const MuonPlan& p, const MuonArgs& a, _Float16* ws, float* diag, float* part, const int* here, int from, hipStream_t st) {
    ns_product_kernel<TM, TN, SPLIT, LO, LOW, PH, NST, SETS><<<n, 256 * SETS, lds_bytes(TM, TN, SPLIT, NST, SETS), st>>>(p, a, ws, diag, part, from, here);
}

// T: edge of the Gram and square tiles; AM, AN: of the last product's
template <int T, int AM, int AN, bool FINE, bool SPLIT, int SN, int AN_ST, int SETS = 1>
hipError_t run_products(const MuonPlan& p, const MuonArgs& a, _Float16* ws, float* diag, float* part, const int* here, hipStream_t st) {
    for (int i = 0; i < NS_STEPS; ++i) {
        const int from = i & 1;
        run_product<T, T, FINE, SPLIT, !FINE, PH_GRAM, SN, SETS>(p.grams, p, a, ws, diag, part, here, from, st);
        if (p.sums) ns_gram_sum_kernel<T, SPLIT><<<p.sums, 256, 0, st>>>(p, ws, diag, part);
        run_product<T, T, SPLIT, SPLIT, !FINE, PH_SQUARE, SN, SETS>(p.squares, p, a, ws, diag, part, here, from, st);
        if (i + 1 < NS_STEPS) run_product<AM, AN, SPLIT, SPLIT, !FINE, PH_APPLY, AN_ST, 1>(p.applies, p, a, ws, diag, part, here, from, st);
        else run_product<AM, AN, SPLIT, SPLIT, !FINE, PH_LAST, AN_ST, 1>(p.applies, p, a, ws, diag, part, here, from, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

bool muon_plan(const MuonGroup* g, int n, bool exact, MuonPlan* out) {
    MuonPlan p{};
    p.n = n;
    std::copy(g, g + n, p.g);
    for (int i = 0; i < MUON_MAX_GROUPS; ++i) p.at.chunk[i] = p.at.cast[i] = p.at.gram[i] = p.at.square[i] = p.at.apply[i] = p.at.sum[i] = 0x7FFFFFFF;
    const long long index = 0x7FFFFFFF, most = 0xFFFFFFFF / 256;      // (a launch has fewer than 2^32 threads)
    auto up = [](long long v, long long m) { return (v + m - 1) / m * m; };
    // (what follows rounds sides up in 32 bits)
    for (int i = 0; i < n; ++i) if (g[i].ortho && std::max(g[i].rows, g[i].cols) > 1 << 30) return false;
    // small matrices only: a workgroup each
    int side = 0;
    for (int i = 0; i < n; ++i) if (g[i].ortho) side = std::max(side, std::min(g[i].rows, g[i].cols));
    if (side >= 1 && side <= SMALL_SIDE) {
        p.small = (side + 15) / 16;
        bool fits = true;
        for (int i = 0; i < n; ++i) if (g[i].ortho) {
            const int longer = std::max(g[i].rows, g[i].cols);
            fits = fits && longer <= 4096;
            if (fits) p.lds = std::max(p.lds, small_lds(longer, p.small).bytes);
        }
        if (fits && p.lds <= SMALL_LDS) {
            long long groups = 0;
            for (int i = 0; i < n; ++i) {
                MuonGroup& q = p.g[i];
                q.tall = q.rows > q.cols;
                q.chunks = (int)(((long long)q.rows * q.cols + FLAT - 1) / FLAT);
                p.at.apply[i] = (int)groups;
                groups += (long long)q.count * (q.ortho ? 1 : q.chunks);
                if (groups > 0xFFFFFFFF / SMALL_THREADS) return false;
            }
            p.tile = 3;
            p.applies = (int)groups;
            p.bytes = 256;
            *out = p;
            return true;
        }
    }
    // The entries of a step are lr / sqrt(cols) in size, so that O's error reaches the weights with 1 / sqrt(cols): matrices of few columns (512 a row over all of
    // them) get products of both planes in mode 1 too.  Two layers of 301 cells, gates apart, all launches: 240 -> 295 us; four of 512 would go from 790 to 1380.
    long long elements = 0, rows = 0;
    for (int i = 0; i < n; ++i) if (g[i].ortho) { rows += (long long)g[i].count * g[i].rows; elements += (long long)g[i].count * g[i].rows * g[i].cols; }
    exact = exact || elements < 512 * rows;
    p.exact = exact;
    auto tiles = [&](int high, int wide) {              // of the last product
        long long t = 0;
        for (int i = 0; i < n; ++i) if (g[i].ortho) t += (long long)g[i].count * ((g[i].rows + high - 1) / high) * ((g[i].cols + wide - 1) / wide);
        return t;
    };
    p.tile = !exact && tiles(256, 128) >= 480 ? 2 : tiles(128, 128) >= 700 ? 1 : 0;
    const int edge = p.tile ? 128 : 64, high = p.tile == 2 ? 256 : edge;
    long long halves = 0, floats = 0, diags = 0, chunks = 0, casts = 0, grams = 0, squares = 0, applies = 0, sums = 0, slabs = 0, tiles_s = 0;
    // the longest contractions first: what is left at a launch's end is short
    std::stable_sort(p.g, p.g + n, [](const MuonGroup& x, const MuonGroup& y) {
        return (x.ortho ? std::min(x.rows, x.cols) : 0) > (y.ortho ? std::min(y.rows, y.cols) : 0);
    });
    for (int i = 0; i < n; ++i) {
        MuonGroup& q = p.g[i];
        q.tall = q.rows > q.cols;
        if (!q.ortho) continue;
        q.rp = (int)up(q.rows, high); q.cp = (int)up(q.cols, edge);
        // (the side that the last product's tiles walk along B: rows padded to 256 may be more than columns padded to 128 where rows <= columns)
        q.mp = q.tall ? q.cp : q.rp;
        const long long nt = q.mp / edge;
        q.grams = (int)(nt * (nt + 1) / 2);
        tiles_s += (long long)q.count * q.grams;
        slabs += (long long)q.count * q.grams * (std::max(q.rp, q.cp) / 64);
    }
    // Gram tiles: parts along the contraction where it is long for their number, none shorter than eight slabs
    p.lone = p.tile == 0 && tiles_s <= 256;
    const long long target = std::max<long long>(8, slabs / 320);
    for (int i = 0; i < n; ++i) {
        MuonGroup& q = p.g[i];
        const long long size = (long long)q.rows * q.cols;
        p.at.chunk[i] = (int)chunks; q.chunks = (int)((size + FLAT - 1) / FLAT);
        chunks += (long long)q.count * q.chunks;
        p.at.cast[i] = (int)casts; p.at.gram[i] = (int)grams; p.at.square[i] = (int)squares; p.at.apply[i] = (int)applies; p.at.sum[i] = (int)sums;
        if (chunks > most) return false;
        if (!q.ortho) continue;
        const long long nx = (long long)q.rp * q.cp, ns = (long long)q.mp * q.mp;
        if ((long long)std::max(q.rp, q.cp) * 256 > index || nx / CAST * q.count > most) return false;
        q.casts = (int)(nx / CAST);
        casts += (long long)q.count * q.casts;
        const int length = std::max(q.rp, q.cp) / 64;
        q.splits = p.lone && length <= 24 ? 1 : std::clamp((int)((length + target / 2) / target), 1, 32);   // (the sum's launch is worth a dozen slabs, each part some more)
        auto eighths = [](long long v) { return (v + 7) / 8 * 8; };
        grams += eighths((long long)q.count * q.grams * q.splits);
        squares += eighths((long long)q.count * q.grams);
        q.applies = (int)(nx / high / edge);
        applies += eighths((long long)q.count * q.applies);
        q.xplane = nx * q.count; q.splane = ns * q.count;
        for (int b = 0; b < 2; ++b) { q.x[b] = halves; halves += 2 * q.xplane; }
        q.s = halves; halves += (exact ? 2 : 1) * q.splane;
        q.b = halves; halves += (exact ? 2 : 1) * q.splane;
        q.diag = diags; diags += 2LL * q.count * q.mp;
        q.part = floats;
        if (q.splits > 1) { floats += (long long)q.count * q.grams * q.splits * edge * edge; sums += (long long)q.count * q.grams * (p.tile ? 4 : 1); }
        if (casts > most || grams > most || applies > most || sums > most) return false;
    }
    p.chunks = (int)chunks; p.casts = (int)casts; p.grams = (int)grams; p.squares = (int)squares; p.applies = (int)applies; p.sums = (int)sums;
    auto to256 = [](size_t v) { return (v + 255) & ~size_t(255); };
    p.sums_at = to256((size_t)halves * 2);
    p.diag_at = p.sums_at + to256((size_t)chunks * 8);
    p.part_at = p.diag_at + to256((size_t)diags * 4);
    p.here_at = p.part_at + to256((size_t)floats * 4);
    p.bytes = p.here_at + to256(n == 1 ? (size_t)p.g[0].count * 4 : 0) + 256;
    *out = p;
    return true;
}

hipError_t launch_muon(const MuonPlan& p, const MuonArgs& a, const MuonIds& ids, void* scratch, hipStream_t st) {
    if (p.tile == 3) {
        if (p.small == 1) muon_small_kernel<1><<<p.applies, SMALL_THREADS, p.lds, st>>>(p, a, ids);
        else if (p.small == 2) muon_small_kernel<2><<<p.applies, SMALL_THREADS, p.lds, st>>>(p, a, ids);
        else if (p.small == 3) muon_small_kernel<3><<<p.applies, SMALL_THREADS, p.lds, st>>>(p, a, ids);
        else muon_small_kernel<4><<<p.applies, SMALL_THREADS, p.lds, st>>>(p, a, ids);
        return hipGetLastError();
    }
    _Float16* ws = static_cast<_Float16*>(scratch);
    double* sums = reinterpret_cast<double*>(static_cast<char*>(scratch) + p.sums_at);
    float* diag = reinterpret_cast<float*>(static_cast<char*>(scratch) + p.diag_at);
    float* part = reinterpret_cast<float*>(static_cast<char*>(scratch) + p.part_at);
    int* here = ids.ids ? reinterpret_cast<int*>(static_cast<char*>(scratch) + p.here_at) : nullptr;
    muon_momentum_kernel<<<p.chunks, 256, 0, st>>>(p, a, sums, ids, here);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.casts == 0) return e;
    // (second halves that are multiplied, in S at least, are halves)
    if (p.tile == 0 || p.exact) muon_cast_kernel<false><<<p.casts, 256, 0, st>>>(p, a, sums, ws);
    else muon_cast_kernel<true><<<p.casts, 256, 0, st>>>(p, a, sums, ws);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.tile == 2) return run_products<2, 4, 2, false, false, 2, 1>(p, a, ws, diag, part, here, st);
    // (both planes' fragments of a slab fit the registers too: one buffer where workgroups share CUs, 865 -> 782 us a step of two layers of 512 cells in float, 289 -> 271 for two
    // of 301 with gates apart; two buffers where they have a CU each: with one set of wavefronts 210 us against 222 for two matrices of 1204 x 602)
    if (p.tile == 0 && p.exact && !p.lone && p.applies >= 512) return run_products<1, 1, 1, true, true, 1, 1>(p, a, ws, diag, part, here, st);
    if (p.tile == 1) return p.exact ? run_products<2, 2, 2, true, true, 1, 1>(p, a, ws, diag, part, here, st) : run_products<2, 2, 2, false, false, 2, 2>(p, a, ws, diag, part, here, st);
    if (p.lone) return p.exact ? run_products<1, 1, 1, true, true, 2, 2, 2>(p, a, ws, diag, part, here, st) : run_products<1, 1, 1, true, false, 2, 2, 2>(p, a, ws, diag, part, here, st);
    return p.exact ? run_products<1, 1, 1, true, true, 2, 2>(p, a, ws, diag, part, here, st) : run_products<1, 1, 1, true, false, 2, 2>(p, a, ws, diag, part, here, st);
}

}  // namespace blstm
