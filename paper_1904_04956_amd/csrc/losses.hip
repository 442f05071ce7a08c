// The softmax layer's logits u = W_s z + b_s, bf16 operands and float sums, straight into what a loss wants of them: the sums of
// exponentials of every row (forward), or dE/du = a exp(u - max) + a' exp((u - max) / tau) - hot 1_y (backward).  The logits
// themselves stay in registers: in float they would be twice the traffic of anything else here, and rounded to bf16 they would be
// 2^-9 of their value off, which is 2 % of a probability at a logit of 5.
//
// A workgroup of four wavefronts owns 128 classes x 128 rows.  The weights are the first operand of the products, so that a
// lane holds 32 classes of one row, half of a strip of 64: maximum and sums are in its registers, and one exchange with the
// other half of the wavefront completes them.  Two workgroups a CU: one multiplies while the other takes exponentials.
//
// Bound by LDS: a wavefront's 64 x 64 tile reads four operands of 1 KB for four products of 16 cycles, twice what LDS gives.  A
// larger tile of one workgroup a CU would halve that and leave its exponentials without anything beside them.  5985 rows of 32000
// classes, z of 524 (201 GFLOP): the sums 300 us (670 TFLOP/s), du 480 us, 766 MB of stores among them; 1344 rows, z of 1024: 99 us (890).
//
// du is kept as bf16 numbers: hi, what the rounding left, and, where frames are few, what that left.  All enter dW_s and db_s; hi alone
// enters the product for dz, to which the second is added where du is large.
#include "gemm_tile.hpp"
#include "losses_terms.hpp"

namespace blstm {
namespace {

// What becomes of the logits: the strips' maxima and sums, du, or the logits themselves in float with the strips' maxima.
enum { SUMS, GRAD, LOGITS };

template <bool TAU, int WHAT>
__global__ __launch_bounds__(256, 2) void loss_tile_kernel(LossTileArgs a, int ntm, int ntv) {
    constexpr int SLAB = 128 * CHUNKS, BK = 64;
    extern __shared__ uint4 smem[];                     // [2][classes' slab, rows' slab], then the classes' bias
    float* bias_s = reinterpret_cast<float*>(smem + 4 * SLAB);
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wv >> 1, wn = wv & 1, l32 = lane & 31, half = lane >> 5;
    // each XCD takes a contiguous range of tiles, down the rows of one column of tiles after the other
    int lin = (int)blockIdx.x;
    const int nt = ntm * ntv, nt8 = nt & ~7;
    if (lin < nt8) lin = (lin & 7) * (nt8 >> 3) + (lin >> 3);
    const int col0 = lin / ntm * 128, row0 = lin % ntm * 128;
    // classes beyond the last one: their products repeat its weights, and the bias makes nothing of them
    if (tid < 128) bias_s[tid] = col0 + tid < a.V ? bf2f(a.bias[col0 + tid]) : WHAT == LOGITS ? __builtin_nanf("") : -INFINITY;   // (NaN is not a maximum)

    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    const int nslab = (a.ld + BK - 1) / BK;
    auto dma = [](unsigned lds_addr, const char* gbase, unsigned voff) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(gbase) : "memory");
    };
    const char* wbase = reinterpret_cast<const char*>(a.W + (long long)col0 * a.ld);
    const char* zbase = reinterpret_cast<const char*>(a.z + (long long)row0 * a.ld);
    auto issue = [&](int it) __attribute__((always_inline)) {
        const unsigned sb = lds0 + (unsigned)((it & 1) * 2 * SLAB * 16);
        const int chunks = min(a.ld - it * BK, BK) / 8;   // (a chunk beyond the rows' end repeats the last one, cleared below)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = 8 * (4 * j + wv) + (lane >> 3), c = min((lane & 7) ^ swz(r), chunks - 1);
            dma(sb + (unsigned)((4 * j + wv) * 1024), wbase + it * BK * 2, (unsigned)(min(r, a.V - 1 - col0) * a.ld * 2 + c * 16));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = 8 * (4 * j + wv) + (lane >> 3), c = min((lane & 7) ^ swz(r), chunks - 1);
            dma(sb + (unsigned)(SLAB * 16 + (4 * j + wv) * 1024), zbase + it * BK * 2, (unsigned)(min(r, a.M - 1 - row0) * a.ld * 2 + c * 16));
        }
    };
    int roff_w[CHUNKS / 2], roff_z[CHUNKS / 2];
    const int wrow = wn * 64 + l32, zrow = wm * 64 + l32;
#pragma unroll
    for (int q = 0; q < CHUNKS / 2; ++q) {
        roff_w[q] = wrow * CHUNKS + ((2 * q + half) ^ swz(wrow));
        roff_z[q] = zrow * CHUNKS + ((2 * q + half) ^ swz(zrow));
    }
    f32x16_t acc[2][2];                                 // [classes][rows]
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.0f;
    issue(0);
    for (int it = 0; it < nslab; ++it) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (it + 1 < nslab) issue(it + 1);              // (its buffer's products were done in front of the barrier)
        uint4* w_s = smem + (it & 1) * 2 * SLAB;
        const uint4* z_s = w_s + SLAB;
        if (a.ld - it * BK < BK) {                      // the last slab, in part
            const int chunks = (a.ld - it * BK) / 8;
            for (int c = tid; c < 2 * SLAB; c += 256) if ((c & 7) >= chunks) w_s[(c & ~7) | ((c & 7) ^ swz((c >> 3) & 127))] = make_uint4(0, 0, 0, 0);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
#pragma unroll
        for (int q = 0; q < CHUNKS / 2; ++q) {
            const uint4 w[2] = {w_s[roff_w[q]], w_s[roff_w[q ^ 2] + 32 * CHUNKS]};
            const uint4 x[2] = {z_s[roff_z[q]], z_s[roff_z[q ^ 2] + 32 * CHUNKS]};
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, w[j]), __builtin_bit_cast(bf16x8_t, x[i]), acc[j][i], 0, 0, 0);
        }
    }
    // register e of a lane: row l32 of block i, class 8 (e / 4) + 4 half + e % 4 of block j
    const float lt = LOG2E * a.inv_tau;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float b = bias_s[wn * 64 + j * 32 + 8 * (e >> 2) + 4 * half + (e & 3)];
            acc[j][0][e] += b; acc[j][1][e] += b;
        }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int m = row0 + wm * 64 + i * 32 + l32;
        if constexpr (WHAT == LOGITS) {
            float mx = acc[0][i][0];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, acc[j][i][e]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            if (m < a.M) {
                if (half == 0) a.part_max[(long long)(col0 / 64 + wn) * a.M + m] = mx;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int n = col0 + wn * 64 + j * 32 + 8 * g + 4 * half;
                        if (n < a.ldu) *reinterpret_cast<float4*>(a.logits + m * a.ldu + n) = make_float4(acc[j][i][4 * g], acc[j][i][4 * g + 1], acc[j][i][4 * g + 2], acc[j][i][4 * g + 3]);
                    }
            }
        } else if constexpr (WHAT == SUMS) {
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, acc[j][i][e]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m2 = rounded_product(mx, LOG2E), mt2 = rounded_product(mx, lt);
            float sum = 0.0f, tau = 0.0f;
            auto add = [&](auto power) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        sum += __builtin_amdgcn_exp2f(power(acc[j][i][e], LOG2E, m2));
                        if (TAU) tau += __builtin_amdgcn_exp2f(power(acc[j][i][e], lt, mt2));
                    }
            };
            // (a strip of nothing but -inf: -inf - 0 is a power of nothing, where -inf + inf would be no number)
            if (__any(fabsf(mx) > LOSS_FAR)) {           // (row by row: none depends on what the others hold)
                const bool far = fabsf(mx) > LOSS_FAR;
                const float base = mx == -INFINITY ? 0.0f : mx;
                add([&](float u, float k, float m) { return far ? (u - base) * k : fmaf(u, k, -m); });
            } else add([](float u, float k, float m) { return fmaf(u, k, -m); });
            sum += __shfl_xor(sum, 32, 64);
            if (TAU) tau += __shfl_xor(tau, 32, 64);
            if (half == 0 && m < a.M) {
                const long long at = (long long)(col0 / 64 + wn) * a.M + m;
                a.part_max[at] = mx;
                a.part_sum[at] = sum;
                if (TAU) a.part_sum_tau[at] = tau;
            }
        } else {
            const LossRow r = a.rows[min(m, a.M - 1)];
            const int rel = r.label - (col0 + wn * 64);  // the label among the wavefront's 64 classes
            const bool any_hot = __any(rel >= 0 && rel < 64), far = __any(fabsf(r.max) > LOSS_FAR && r.max < INFINITY);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float d[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    d[e] = r.a * __builtin_amdgcn_exp2f(fmaf(acc[j][i][e], LOG2E, -r.m2));
                    if (TAU) d[e] = fmaf(r.at, __builtin_amdgcn_exp2f(fmaf(acc[j][i][e], lt, -r.mt2)), d[e]);
                }
                if (far) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        if (fabsf(r.max) <= LOSS_FAR) continue;
                        d[e] = r.a * __builtin_amdgcn_exp2f((acc[j][i][e] - r.max) * LOG2E);
                        if (TAU) d[e] = fmaf(r.at, __builtin_amdgcn_exp2f((acc[j][i][e] - r.max) * lt), d[e]);
                    }
                }
                if (any_hot) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) d[e] -= rel == j * 32 + 8 * (e >> 2) + 4 * half + (e & 3) ? r.hot : 0.0f;
                }
                // d rounded, to `to`; then d is what the rounding left
                auto part = [&](unsigned short* to) __attribute__((always_inline)) {
                    unsigned p[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        p[e] = pack_bf2(d[2 * e], d[2 * e + 1]);
                        d[2 * e] -= bf2f((bf16_t)(p[e] & 0xFFFFu));
                        d[2 * e + 1] -= bf2f((bf16_t)(p[e] >> 16));
                    }
                    // an exchange between the lane halves makes four neighbouring classes eight
#pragma unroll
                    for (int g = 0; g < 4; g += 2) {
                        const int n = col0 + wn * 64 + j * 32 + 8 * (g + half);
                        const auto x = __builtin_amdgcn_permlane32_swap(p[2 * g], p[2 * g + 2], false, false), y = __builtin_amdgcn_permlane32_swap(p[2 * g + 1], p[2 * g + 3], false, false);
                        if (m < a.M && n < a.ldu) *reinterpret_cast<uint4*>(to + m * a.ldu + n) = make_uint4(x[0], y[0], x[1], y[1]);
                    }
                };
                part(a.hi);
                part(a.lo);
                if (a.third) part(a.lo + a.M * a.ldu);
            }
        }
    }
}

template <bool TAU, int WHAT>
hipError_t launch_tile(const LossTileArgs& a, hipStream_t st) {
    constexpr size_t lds = 4 * 128 * CHUNKS * 16 + 128 * sizeof(float);
    static thread_local bool attr_set = false;
    const hipError_t e = allow_lds(&loss_tile_kernel<TAU, WHAT>, lds, &attr_set);
    if (e != hipSuccess) return e;
    const int ntm = (a.M + 127) / 128, ntv = (a.V + 127) / 128;
    hipLaunchKernelGGL((loss_tile_kernel<TAU, WHAT>), dim3((unsigned)(ntm * ntv)), dim3(256), lds, st, a, ntm, ntv);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_loss_stats(const LossTileArgs& a, hipStream_t st) {
    return a.inv_tau != 0.0f ? launch_tile<true, SUMS>(a, st) : launch_tile<false, SUMS>(a, st);
}
hipError_t launch_loss_grad(const LossTileArgs& a, hipStream_t st) {
    return a.inv_tau != 0.0f ? launch_tile<true, GRAD>(a, st) : launch_tile<false, GRAD>(a, st);
}
hipError_t launch_loss_logits(const LossTileArgs& a, hipStream_t st) { return launch_tile<false, LOGITS>(a, st); }

}  // namespace blstm
