// What the softmax layer's losses do row by row: ahead of the products, behind them, on float logits, and the selection of
// the K largest.  With u the logits of a frame, y its label, q the teacher's distribution over the entries of its list:
//   log p_y = u_y - log sum_v exp u_v
//   policy:  r = exp(log p_y - old), l = -min(r A, clip(r) A) + k (exp(ref - log p_y) - (ref - log p_y) - 1)
//            g = dl/dlog p_y = -(r A, unless the clip is what the minimum takes) + k (1 - exp(ref - log p_y)),  dl/du = g (1_y - p)
//   distill: l = h (-log p_y) + w tau^2 sum_k q_k (log q_k - log p'_k), p' = softmax(u / tau)
//            dl/du = h (p - 1_y) + w tau (p' - sum_k q_k 1_k)
// All of them are bound by memory, the smallest by the latency of a few dependent loads.  bf16, z of 256, 32000 classes: ahead of the
// products 5 us (336 rows), 9 (168 rows, lists of 16: the lists' weights gathered), 35 (5376 rows, lists of 64, 176 MB from L2); the
// rows' merge 4 us; the K largest 18 us (336 rows, K = 20) and 75 (5376 rows, K = 64: 90 MB of chosen strips, then the cuts of the
// lists); float rows of 32000 logits 67 us for 1344 rows (344 MB, 5.1 TB/s).
#include "common.hpp"
#include "losses_terms.hpp"
#include <type_traits>

namespace blstm {
namespace {

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// Between a wavefront's LDS stores and its other lanes' loads of them.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

enum { LIST_USED = 1, LIST_BAD = 2 };

// A class list of one row in LDS, as its wavefront sees it.
struct ListLds { int cls[LOSS_MAX_TOP]; float q[LOSS_MAX_TOP], log_q[LOSS_MAX_TOP], logit[LOSS_MAX_TOP]; };

// q over the used entries of a row, by one wavefront.  Returns LIST_USED if there are any, and LIST_BAD if some class is out of range or its value no
// number.  An entry that is not used has class -1 and q 0.  (A value of -inf is a probability of zero: it would make a list
// of nothing else a division of zero by zero.)
__device__ int teacher_list(const TeacherArgs& t, long long m, int V, ListLds& s) {
    const int lane = threadIdx.x & 63;
    float top = -INFINITY;
    bool bad = false, some = false;
    for (int k = lane; k < t.K; k += 64) {
        const int c = t.classes[m * t.K + k];
        const float v = t.values[m * t.K + k];
        const bool in = (unsigned)c < (unsigned)V;
        bad |= in ? !(v < INFINITY) : c != -1;
        const bool used = in && v > -INFINITY && v < INFINITY;
        some |= used;
        s.cls[k] = used ? c : -1;
        s.log_q[k] = v;
        if (used) top = fmaxf(top, v);
    }
    top = wave_max(top);
    float sum = 0.0f;
    for (int k = lane; k < t.K; k += 64) {
        s.log_q[k] = (s.log_q[k] - top) * t.inv_tau;   // (the distance first: a value over the temperature may be beyond a float's range)
        const float e = s.cls[k] >= 0 ? expf(s.log_q[k]) : 0.0f;
        s.q[k] = e;
        sum += e;
    }
    sum = wave_sum(sum);
    for (int k = lane; k < t.K; k += 64) {
        const bool used = s.cls[k] >= 0;
        s.q[k] = used ? s.q[k] / sum : 0.0f;
        s.log_q[k] = used ? s.log_q[k] - logf(sum) : 0.0f;
    }
    wave_sync();
    return (__any(some) ? LIST_USED : 0) | (__any(bad) ? LIST_BAD : 0);
}

// Sum of q of the entries with entry k's class (a class may stand in a list more than once).
__device__ __forceinline__ float class_weight(const ListLds& s, int K, int k) {
    float w = 0.0f;
    for (int j = 0; j < K; ++j) w += s.cls[j] == s.cls[k] ? s.q[j] : 0.0f;
    return w;
}

// ---- ahead of the products: a wavefront a row -----------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void loss_prep_kernel(LossPrepArgs a) {
    __shared__ ListLds lists[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if constexpr (sizeof(T) == 2) {
        const int first = (a.M + 3) / 4;                 // workgroups behind the rows': the bias
        if ((int)blockIdx.x >= first) {
            const int v = ((int)blockIdx.x - first) * 256 + (int)threadIdx.x;
            if (v < ((a.V + 63) & ~63)) a.bias_f[v] = v < a.V ? bf2f(a.bias[v]) : a.bias_pad;
            return;
        }
    }
    const long long m = (long long)blockIdx.x * 4 + wave;
    if (m >= a.M) return;
    ListLds& s = lists[wave];
    const int lab = a.labels ? a.labels[m] : -1;
    const bool lab_ok = (unsigned)lab < (unsigned)a.V;
    const T* z = static_cast<const T*>(a.z) + m * a.Z;
    int state = 0;
    auto list = [&] { if (a.teacher.K > 0) state = teacher_list(a.teacher, m, a.V, s); return a.keep || lab_ok || (state & LIST_USED); };
    if constexpr (sizeof(T) == 4) {
        const bool live = list();
        if (a.zc) {
            T* zc = static_cast<T*>(a.zc) + m * a.ldzc;
            for (int k = lane; k < a.ldzc; k += 64) zc[k] = live && k < a.Z ? z[k] : (T)0;
        }
    } else {
        // sixteen lanes a product, eight elements a lane and step; the row's elements of up to PREP_STEPS steps stay in registers
        constexpr int PREP_STEPS = 4;
        const int l16 = lane & 15, g = lane >> 4;
        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
        auto row_words = [&](int k) {
            uint4 r = make_uint4(0, 0, 0, 0);
            if (k + 8 <= a.Z && a.Z % 8 == 0) r = *reinterpret_cast<const uint4*>(z + k);
            else if (k < a.Z) {
                uint32_t w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    w[q] = (k + 2 * q < a.Z ? (uint32_t)z[k + 2 * q] : 0u) | (k + 2 * q + 1 < a.Z ? (uint32_t)z[k + 2 * q + 1] << 16 : 0u);
                r = make_uint4(w[0], w[1], w[2], w[3]);
            }
            return r;
        };
        uint4 zr[PREP_STEPS];
#pragma unroll
        for (int i = 0; i < PREP_STEPS; ++i) zr[i] = row_words(l16 * 8 + 128 * i);
        const bool live = list();                       // (its loads and the row's together on their way)
        if (a.zc) {
            T* zc = static_cast<T*>(a.zc) + m * a.ldzc;
            for (int k = lane * 8; k < a.ldzc; k += 512) {
                const uint4 x = live ? row_words(k) : make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4*>(zc + k) = x;
                if (a.twice) *reinterpret_cast<uint4*>(zc + (long long)a.M * a.ldzc + k) = x;
            }
        }
        if (!a.W) return;
        auto dot = [](const uint4& x, const uint4& w, float acc) {
            acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x.x), __builtin_bit_cast(bf16x2_t, w.x), acc, false);
            acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x.y), __builtin_bit_cast(bf16x2_t, w.y), acc, false);
            acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x.z), __builtin_bit_cast(bf16x2_t, w.z), acc, false);
            return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, x.w), __builtin_bit_cast(bf16x2_t, w.w), acc, false);
        };
        // the logits of COUNT classes at once (below 0: none, 0)
        auto logits = [&](auto count, const int (&c)[4], float (&u)[4]) __attribute__((always_inline)) {
            constexpr int COUNT = decltype(count)::value;
#pragma unroll
            for (int n = 0; n < COUNT; ++n) u[n] = 0.0f;
#pragma unroll
            for (int i = 0; i < PREP_STEPS; ++i) {
                const int k = l16 * 8 + 128 * i;
                if (128 * i < a.ldzc) {
                    uint4 w[COUNT];
#pragma unroll
                    for (int n = 0; n < COUNT; ++n) w[n] = k < a.ldzc && c[n] >= 0 ? *reinterpret_cast<const uint4*>(a.W + (long long)c[n] * a.ldzc + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int n = 0; n < COUNT; ++n) u[n] = dot(zr[i], w[n], u[n]);
                }
            }
            for (int k = l16 * 8 + 128 * PREP_STEPS; k < a.ldzc; k += 128) {
                const uint4 x = row_words(k);
#pragma unroll
                for (int n = 0; n < COUNT; ++n) if (c[n] >= 0) u[n] = dot(x, *reinterpret_cast<const uint4*>(a.W + (long long)c[n] * a.ldzc + k), u[n]);
            }
#pragma unroll
            for (int n = 0; n < COUNT; ++n) {
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) u[n] += __shfl_xor(u[n], o, 64);
                if (c[n] >= 0) u[n] += bf2f(a.bias[c[n]]);
            }
        };
        {
            const int c[4] = {lab_ok ? lab : -1, -1, -1, -1};
            float u[4];
            logits(std::integral_constant<int, 1>{}, c, u);
            if (lane == 0) a.label_logit[m] = u[0];
        }
        if (a.teacher.K > 0) {
            for (int k0 = 0; k0 < a.teacher.K; k0 += 16) {
                int c[4];
                float u[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) { const int k = k0 + 4 * n + g; c[n] = k < a.teacher.K ? s.cls[k] : -1; }
                logits(std::integral_constant<int, 4>{}, c, u);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const int k = k0 + 4 * n + g;
                    if (l16 == 0 && k < a.teacher.K) { a.entry_logit[m * a.teacher.K + k] = u[n]; s.logit[k] = u[n]; }
                }
            }
            // sum q (log q - (u - ref) / tau), 0 log 0 being nothing, whatever u is; ref: the largest u, so that an offset of all logits takes no digits
            wave_sync();
            float ref = -INFINITY, part = 0.0f;
            for (int k = lane; k < a.teacher.K; k += 64) if (s.cls[k] >= 0 && s.q[k] > 0.0f) ref = fmaxf(ref, s.logit[k]);
            ref = wave_max(ref);
            if (ref == -INFINITY) ref = 0.0f;
            for (int k = lane; k < a.teacher.K; k += 64) if (s.cls[k] >= 0 && s.q[k] != 0.0f) part += s.q[k] * (s.log_q[k] - (s.logit[k] - ref) * a.teacher.inv_tau);
            part = wave_sum(part);
            // a class that stands there more than once has all of its q at the first of its entries with any
            for (int k0 = 0; k0 < a.teacher.K; k0 += 64) {
                const int k = k0 + lane;
                const int c = k < a.teacher.K ? s.cls[k] : -1;
                float q = 0.0f;
                bool first = c >= 0 && s.q[k] > 0.0f;
                for (int j0 = 0; j0 < a.teacher.K; j0 += 64) {
                    const int cj = j0 + lane < a.teacher.K ? s.cls[j0 + lane] : -1, n = min(64, a.teacher.K - j0);
                    const float qj = j0 + lane < a.teacher.K ? s.q[j0 + lane] : 0.0f;
                    for (int j = 0; j < n; ++j) {
                        const int other = __builtin_amdgcn_readlane(cj, j);
                        const float more = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, qj), j));
                        q += other == c ? more : 0.0f;
                        first &= other != c || !(more > 0.0f) || j0 + j >= k;
                    }
                }
                if (k < a.teacher.K) a.entry_q[m * a.teacher.K + k] = first ? q : 0.0f;
            }
            if (lane == 0) { a.soft_const[m] = part; a.soft_const[a.M + m] = ref; a.soft_state[m] = state; }
        }
    }
}

// The reference of a row whose sums lack the label's class: not far below that class's logit.
__device__ __forceinline__ float merge_reference(const LossMergeArgs& a, long long m, float mx) {
    return a.consts && a.labels && (unsigned)a.labels[m] < (unsigned)a.V ? fmaxf(mx, a.label_logit[m]) : mx;
}

// What a row's largest logit (or another reference) and its sums give, by one lane.  `in`: the row is none of those that fill the last tile.
template <bool TAU, bool POLICY, bool TEACHER>
__device__ __forceinline__ void merge_end(const LossMergeArgs& a, const PolicyArgs& policy, const TeacherArgs& teacher, long long m, bool in, float mx, float sum, float tau) {
    const float m2 = rounded_product(mx, LOG2E), mt2 = TAU ? rounded_product(mx, LOG2E * teacher.inv_tau) : 0.0f;
    const bool far = fabsf(mx) > LOSS_FAR;
    auto put = [&](const LossRow& r) {
        const float x[6] = {r.m2, r.a, r.mt2, r.at, r.hot, __builtin_bit_cast(float, r.label)};
#pragma unroll
        for (int i = 0; i < 6; ++i) a.consts[i * (long long)a.Mp + m] = x[i];
    };
    if (!in) {
        if (a.consts && m < a.Mp) { LossRow r{}; r.m2 = INFINITY; r.mt2 = INFINITY; r.label = -1; put(r); }
        return;
    }
    const int lab = a.labels ? a.labels[m] : -1;
    const bool lab_ok = (unsigned)lab < (unsigned)a.V;
    const float nan = __builtin_nanf("");
    // u_y - max in the scale of the sums, whose maximum is rounded once: the same number in all of them
    const float up = far ? a.label_logit[m] - mx : fmaf(a.label_logit[m], LOG2E, -m2) * LN2;
    const float others = sum;                            // (a.consts: of all but the label, so that 1 - p is a sum and no difference)
    float label_tau = 0.0f;
    if (a.consts && lab_ok) {
        sum += __builtin_amdgcn_exp2f(fmaf(a.label_logit[m], LOG2E, -m2));
        if (TAU) { label_tau = __builtin_amdgcn_exp2f(fmaf(a.label_logit[m], LOG2E * teacher.inv_tau, -mt2)); tau += label_tau; }
    }
    const float lp = lab_ok ? up - logf(sum) : lab == -1 ? 0.0f : nan;
    if (a.logp) a.logp[m] = lp;
    if (!a.rows && !a.consts) return;
    LossRow r{};
    r.m2 = INFINITY; r.mt2 = INFINITY; r.label = -1; r.max = INFINITY;
    float loss = 0.0f;
    if (POLICY) {
        if (lab_ok) {
            const PolicyTerms t = policy_terms(policy, m, lp);
            loss = a.s * t.loss;
            r.m2 = m2; r.a = -a.s * t.g / sum; r.hot = -a.s * t.g; r.label = lab;
        } else if (lab != -1) loss = nan;
    }
    if (TEACHER) {
        const int state = a.soft_state[m];
        if (lab_ok && teacher.hard != 0.0f) {
            loss = a.s * teacher.hard * -lp;
            r.m2 = m2; r.a = a.s * teacher.hard / sum; r.hot = a.s * teacher.hard; r.label = lab;
        } else if (lab != -1 && teacher.hard != 0.0f) loss = nan;
        if (state & LIST_USED) {
            // log sum exp((u - ref) / tau), ref being the terms'
            const float ref = a.soft_const[a.M + m], lt = LOG2E * teacher.inv_tau;
            const float lse = (far ? (mx - ref) * (TAU ? teacher.inv_tau : 1.0f) : (TAU ? fmaf(-ref, lt, mt2) : fmaf(-ref, LOG2E, m2)) * LN2) + logf(TAU ? tau : sum);
            loss += a.s * teacher.soft * teacher.tau * teacher.tau * (a.soft_const[m] + lse);
            const float at = a.s * teacher.soft * teacher.tau;
            if (TAU) { r.mt2 = mt2; r.at = at / tau; }
            else { r.m2 = m2; r.a += at / sum; }
        }
        if (state & LIST_BAD) loss = nan;
    }
    if (r.a != 0.0f || r.at != 0.0f) r.max = mx;         // (a NaN is not 0)
    if (a.consts && lab_ok) r.hot = r.hot * (others / sum) - r.at * label_tau;
    a.row_loss[m] = loss;
    if (a.consts) put(r); else a.rows[m] = r;
}

// ---- behind the sums of the strips: 64 rows a workgroup, its wavefronts share the strips ------------------------------
template <bool TAU, bool POLICY, bool TEACHER>
__global__ __launch_bounds__(512) void loss_merge_kernel(LossMergeArgs a, PolicyArgs policy, TeacherArgs teacher) {
    __shared__ float sh_max[8][64], sh_sum[8][64], sh_tau[8][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long m = (long long)blockIdx.x * 64 + lane;
    const bool in = m < a.M;
    float mx = -INFINITY;
    if (in) {
#pragma unroll 8
        for (int i = wave; i < a.strips; i += 8) mx = fmaxf(mx, a.part_max[(long long)i * a.M + m]);
    }
    sh_max[wave][lane] = mx;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) mx = fmaxf(mx, sh_max[w][lane]);
    if (in) mx = merge_reference(a, m, mx);
    const float m2 = rounded_product(mx, LOG2E), lt = LOG2E * teacher.inv_tau, mt2 = TAU ? rounded_product(mx, lt) : 0.0f;
    const bool far = fabsf(mx) > LOSS_FAR;
    float sum = 0.0f, tau = 0.0f;
    if (in) {
#pragma unroll 4
        for (int i = wave; i < a.strips; i += 8) {
            const float pm = a.part_max[(long long)i * a.M + m];
            const bool away = far || fabsf(pm) > LOSS_FAR;
            sum += a.part_sum[(long long)i * a.M + m] * __builtin_amdgcn_exp2f(away ? (pm - mx) * LOG2E : rounded_product(pm, LOG2E) - m2);
            if (TAU) tau += a.part_sum_tau[(long long)i * a.M + m] * __builtin_amdgcn_exp2f(away ? (pm - mx) * lt : rounded_product(pm, lt) - mt2);
        }
    }
    sh_sum[wave][lane] = sum;
    if (TAU) sh_tau[wave][lane] = tau;
    __syncthreads();
    if (wave != 0) return;
    sum = 0.0f; tau = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) { sum += sh_sum[w][lane]; if (TAU) tau += sh_tau[w][lane]; }
    merge_end<TAU, POLICY, TEACHER>(a, policy, teacher, m, in, mx, sum, tau);
}

// ---- the same, a wavefront a row: for few parts (a part a lane) ----------------------------------------------------------------
template <bool TAU>
__global__ __launch_bounds__(256) void loss_merge_row_kernel(LossMergeArgs a, TeacherArgs teacher) {
    const int lane = threadIdx.x & 63;
    const long long m = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const bool in = m < a.M;
    float mx = -INFINITY, sum = 0.0f, tau = 0.0f;
    if (in) {
        for (int i = lane; i < a.strips; i += 64) mx = fmaxf(mx, a.part_max[(long long)i * a.M + m]);
        mx = merge_reference(a, m, wave_max(mx));
        const float lt = LOG2E * teacher.inv_tau, m2 = rounded_product(mx, LOG2E), mt2 = rounded_product(mx, lt);
        for (int i = lane; i < a.strips; i += 64) {
            const float pm = a.part_max[(long long)i * a.M + m];
            const bool away = fabsf(mx) > LOSS_FAR || fabsf(pm) > LOSS_FAR;
            sum += a.part_sum[(long long)i * a.M + m] * __builtin_amdgcn_exp2f(away ? (pm - mx) * LOG2E : rounded_product(pm, LOG2E) - m2);
            if (TAU) tau += a.part_sum_tau[(long long)i * a.M + m] * __builtin_amdgcn_exp2f(away ? (pm - mx) * lt : rounded_product(pm, lt) - mt2);
        }
        sum = wave_sum(sum);
        if (TAU) tau = wave_sum(tau);
    }
    if (lane == 0) merge_end<TAU, false, TAU>(a, PolicyArgs{}, teacher, m, in, mx, sum, tau);
}

// ---- the teacher's entries of du, p' - q: a wavefront a row ------------------------------------------------------------
__global__ __launch_bounds__(256) void loss_entries_kernel(LossEntriesArgs a) {
    __shared__ ListLds lists[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long m = (long long)blockIdx.x * 4 + wave;
    if (m >= a.M) return;
    ListLds& s = lists[wave];
    for (int k = lane; k < a.K; k += 64) {
        const int c = a.classes[m * a.K + k];
        const float q = a.entry_q[m * a.K + k];
        s.cls[k] = q > 0.0f && (unsigned)c < (unsigned)a.V ? c : -1;
        s.q[k] = q;
    }
    wave_sync();
    const LossRow r = a.rows[m];
    const float lt = LOG2E * a.inv_tau;
    for (int k = lane; k < a.K; k += 64) {
        const int c = s.cls[k];
        if (c < 0) continue;
        float v;
        if (a.third) {                                   // (what the tiles made there is whole in three parts, of the very logits that the sums have seen)
            v = (bf2f(a.hi[m * a.ldu + c]) + bf2f(a.lo[m * a.ldu + c])) + bf2f(a.lo[(a.M + m) * a.ldu + c]);
        } else {                                         // (two are 2^-16 of it off: more than another product's logit in float is)
            const float u = a.entry_logit[m * a.K + k];
            const bool far = fabsf(r.max) > LOSS_FAR;
            v = r.a * __builtin_amdgcn_exp2f(far ? (u - r.max) * LOG2E : fmaf(u, LOG2E, -r.m2)) + r.at * __builtin_amdgcn_exp2f(far ? (u - r.max) * lt : fmaf(u, lt, -r.mt2));
            if (c == r.label) v -= r.hot;
        }
        v -= a.weight * s.q[k];
        const bf16_t hi = f2bf(v);
        a.hi[m * a.ldu + c] = hi;
        const bf16_t lo = f2bf(v - bf2f(hi));
        a.lo[m * a.ldu + c] = lo;
        if (a.third) a.lo[(a.M + m) * a.ldu + c] = f2bf(v - bf2f(hi) - bf2f(lo));
    }
}

// ---- the end of dz: a wavefront a row, four columns a lane ----------------------------------------------------------------
// The product took du's first part alone (2^-8 of each value).  Of the second the label's and the teacher's classes are added here, where du is large: a
// product of all of it costs a fifth of the whole loss, and without either dz was up to 1.9 times as far off as its own
// rounding makes it.  5985 rows of 528: 10 us; 1344 rows of 1024 with lists of 16: 11.
__global__ __launch_bounds__(256) void loss_dz_end_kernel(LossDzEndArgs a) {
    const int lane = threadIdx.x & 63;
    const long long m = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (m >= a.M) return;
    const int lab = a.rows[m].label;
    const bf16_t* lo = a.lo + m * a.ldu;
    const int z = (int)blockIdx.y * 256 + lane * 4;
    const bool in = z < a.ld;
    const int at = in ? z : 0;                       // (all lanes stay: each holds an entry of the list)
    const float4 d = *reinterpret_cast<const float4*>(a.dz_f + m * a.ld + at);
    float x[4] = {d.x, d.y, d.z, d.w};
    auto add = [&](int c, float w) {
        const uint2 b = *reinterpret_cast<const uint2*>(a.W + (long long)c * a.ld + at);
        x[0] = fmaf(w, bf2f((bf16_t)(b.x & 0xFFFFu)), x[0]); x[1] = fmaf(w, bf2f((bf16_t)(b.x >> 16)), x[1]);
        x[2] = fmaf(w, bf2f((bf16_t)(b.y & 0xFFFFu)), x[2]); x[3] = fmaf(w, bf2f((bf16_t)(b.y >> 16)), x[3]);
    };
    if (lab >= 0) add(lab, bf2f(lo[lab]));
    for (int k0 = 0; k0 < a.K; k0 += 64) {
        const int k = k0 + lane;
        const float q = k < a.K ? a.entry_q[m * a.K + k] : 0.0f;
        const int c = q > 0.0f ? a.classes[m * a.K + k] : 0;
        const float w = q > 0.0f && c != lab ? bf2f(lo[c]) : 0.0f;   // (what is none: nothing times the first class)
        for (int j = 0; j < 64 && k0 + j < a.K; j += 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                add(__builtin_amdgcn_readlane(c, j + i), __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), j + i)));
        }
    }
    if (!in) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) if (z + i < a.Z) a.dz[m * a.Z + z + i] = f2bf(x[i]);
}

// ---- float: a workgroup a row of logits -----------------------------------------------------------------------------------
template <bool MAX>
__device__ __forceinline__ float rows_reduce(float v, float* sh) {
    v = MAX ? wave_max(v) : wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) v = MAX ? fmaxf(v, sh[w]) : v + sh[w];
    return v;
}

// NC > 0: a row of up to 2048 NC logits stays in registers, 16-byte words, and is read and written once (of one exponential a logit, as exponentials):
// 1344 rows of 32000 101 us in three passes, 67 so.  What is beyond V in the last word counts as -inf.
template <int NC, bool TAU, bool POLICY, bool TEACHER, bool GRADIENT>
__global__ __launch_bounds__(512) void loss_rows_f32_kernel(LossRowsArgs a, PolicyArgs policy, TeacherArgs teacher) {
    __shared__ float sh[8];
    __shared__ ListLds list;
    __shared__ float consts[8];
    const long long m = blockIdx.x;
    float* row = a.u + m * a.ldu;
    const int V = a.V, words4 = (V + 3) / 4;
    auto load = [&](int c) {                             // (rows are whole 16-byte words)
        float4 x = *reinterpret_cast<const float4*>(row + 4 * c);
        if (4 * c + 4 > V) {
            if (4 * c + 1 >= V) x.y = -INFINITY;
            if (4 * c + 2 >= V) x.z = -INFINITY;
            x.w = -INFINITY;
        }
        return x;
    };
    const int lab = a.labels ? a.labels[m] : -1;
    const bool lab_ok = (unsigned)lab < (unsigned)V;
    constexpr bool KEEP = NC > 0, POWERS = KEEP && !TAU && GRADIENT;
    float4 r[KEEP ? NC : 1];
    // f(word, its number) of every word of this thread's, the row's last one with -inf behind V
    auto words = [&](auto&& f) __attribute__((always_inline)) {
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < NC; ++i) if ((int)threadIdx.x + 512 * i < words4) f(r[i], (int)threadIdx.x + 512 * i);
        } else {
            for (int c = threadIdx.x; c < words4; c += 512) { float4 x = load(c); f(x, c); }
        }
    };
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < NC; ++i) if ((int)threadIdx.x + 512 * i < words4) r[i] = load((int)threadIdx.x + 512 * i);
    }
    const float at_label = lab_ok ? row[lab] : 0.0f;
    float mx = -INFINITY;
    words([&](float4& x, int) { mx = fmaxf(fmaxf(fmaxf(mx, x.x), fmaxf(x.y, x.z)), x.w); });
    mx = rows_reduce<true>(mx, sh);
    float sum = 0.0f, tau = 0.0f;
    const float it = teacher.inv_tau;
    auto add = [&](float& x) {
        const float e = expf(x - mx);
        sum += e;
        if (TAU) tau += expf((x - mx) * it);
        if (POWERS) x = e;
    };
    words([&](float4& x, int) { add(x.x); add(x.y); add(x.z); add(x.w); });
    sum = rows_reduce<false>(sum, sh);
    if (TAU) tau = rows_reduce<false>(tau, sh);
    if (threadIdx.x < 64) {
        const float nan = __builtin_nanf("");
        const float lp = lab_ok ? at_label - mx - logf(sum) : lab == -1 ? 0.0f : nan;
        float loss = 0.0f, ca = 0.0f, cat = 0.0f, hot = 0.0f;
        if (POLICY) {
            if (lab_ok) {
                const PolicyTerms t = policy_terms(policy, m, lp);
                loss = a.s * t.loss; ca = -a.s * t.g / sum; hot = -a.s * t.g;
            } else if (lab != -1) loss = nan;
        }
        if (TEACHER) {
            const int state = teacher_list(teacher, m, V, list);
            if (lab_ok && teacher.hard != 0.0f) {
                loss = a.s * teacher.hard * -lp;
                ca = a.s * teacher.hard / sum; hot = a.s * teacher.hard;
            } else if (lab != -1 && teacher.hard != 0.0f) loss = nan;
            float part = 0.0f;
            for (int k = threadIdx.x; k < teacher.K; k += 64) {
                const int c = list.cls[k];
                const float u = c >= 0 ? row[c] : 0.0f;
                list.logit[k] = u;
                if (c >= 0 && list.q[k] != 0.0f) part += list.q[k] * (list.log_q[k] - (u - mx) * it);   // (0 log 0 is nothing, whatever u is)
            }
            part = wave_sum(part);
            if (state & LIST_USED) {
                const float total = TAU ? tau : sum;
                loss += a.s * teacher.soft * teacher.tau * teacher.tau * (part + logf(total));
                const float at = a.s * teacher.soft * teacher.tau / total;
                if (TAU) cat = at; else ca += at;
            }
            if (state & LIST_BAD) loss = nan;
        }
        if (threadIdx.x == 0) {
            if (a.logp) a.logp[m] = lp;
            if (GRADIENT) a.row_loss[m] = loss;
            consts[0] = ca; consts[1] = cat; consts[2] = hot;
        }
    }
    if (!GRADIENT) return;
    __syncthreads();                                     // (the label's and the entries' logits are read)
    const float ca = consts[0], cat = consts[1], hot = consts[2];
    const bool hard = ca != 0.0f || ca != ca, soft = TAU && (cat != 0.0f || cat != cat);
    auto grad = [&](float x, int v, bool power) {        // power: x is exp(u - max) already
        float g = hard ? ca * (power ? x : expf(x - mx)) : 0.0f;   // (a row that counts for nothing is zero whatever it holds)
        if (soft) g += cat * expf((x - mx) * it);
        return v == lab && lab_ok ? g - hot : v < V ? g : 0.0f;
    };
    words([&](float4& x, int c) {
        *reinterpret_cast<float4*>(row + 4 * c) = make_float4(grad(x.x, 4 * c, POWERS), grad(x.y, 4 * c + 1, POWERS), grad(x.z, 4 * c + 2, POWERS), grad(x.w, 4 * c + 3, POWERS));
    });
    const int pad = (int)min(a.ldu, (long long)((V + 7) & ~7));
    for (int v = 4 * words4 + threadIdx.x; v < pad; v += 512) row[v] = 0.0f;
    if (TEACHER) {
        __syncthreads();
        const float weight = a.s * teacher.soft * teacher.tau;
        for (int k = threadIdx.x; k < teacher.K; k += 512)
            if (list.cls[k] >= 0) row[list.cls[k]] = grad(list.logit[k], list.cls[k], false) - weight * class_weight(list, teacher.K, k);
    }
}

// ---- the K largest of a row ------------------------------------------------------------------------------------------------
// Values as whole numbers of the same order, NaN below all; +0 and -0 are equal.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0u;
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
// One row a wavefront.  The K largest of a row lie in the K strips whose best entries come first (K entries come before every entry of
// another strip), so that of 32000 logits 500 maxima and 64 K logits are read.  The key of the K-th best strip, found bit by bit
// with ballots over keys in registers, bounds the K largest from below; what of the chosen strips reaches it is collected in order of its column, and
// cut back to the K best whenever the list is full: what comes later then has to be larger.
constexpr int TOP_LIST = 1024;                           // entries of a list: cut back with 64 still free
struct TopLds { uint32_t key[TOP_LIST], col[TOP_LIST]; };

// Of key[0 .. N - 1] of a wavefront's lanes (entry i of lane l is number 64 i + l), the K best are those above t and, in order, the first
// `equal` of those that are t.  (K entries at least are given; what is none has key 0 and counts as the last.)
template <int N>
__device__ uint32_t kth_largest(const uint32_t (&key)[N], int K, int* equal) {
    uint32_t t = 0;
    int above = 0;                                       // entries larger than any that agrees with t so far
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t c = t | (1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__ballot((key[i] >> bit) == (c >> bit)));
        if (above + n == K) { *equal = 0; return c - 1; }   // (all of these, whatever their lower bits: about half of the bits are never looked at)
        if (above + n > K) t = c; else above += n;
    }
    *equal = K - above;
    return t;
}

// Cuts the list's n <= 64 N entries back to the K best, in order; nothing below what it returns is kept.
template <int N>
__device__ uint32_t cut_back(TopLds& s, int n, int K) {
    const int lane = threadIdx.x & 63;
    uint32_t key[N], col[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int at = 64 * i + lane;
        key[i] = at < n ? s.key[at] : 0u;
        col[i] = at < n ? s.col[at] : 0u;
    }
    int equal;
    const uint32_t t = kth_largest<N>(key, K, &equal);
    wave_sync();
    int kept = 0, seen = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool in = 64 * i + lane < n;
        const unsigned long long same = __ballot(in && key[i] == t), below = (1ull << lane) - 1;
        const bool keep = in && (key[i] > t || (key[i] == t && seen + __popcll(same & below) < equal));
        const unsigned long long k = __ballot(keep);
        if (keep) { const int to = kept + __popcll(k & below); s.key[to] = key[i]; s.col[to] = col[i]; }
        kept += __popcll(k);
        seen += __popcll(same);
    }
    wave_sync();
    return t;
}

template <int N>
__global__ __launch_bounds__(256) void row_topk_kernel(const float* u, long long ldu, int M, int V, int K, int strips, const float* part_max, float* values, int32_t* classes) {
    __shared__ TopLds lists[4];
    constexpr int AHEAD = 16;                            // strips on their way
    const int lane = threadIdx.x & 63;
    const long long m = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (m >= M) return;
    TopLds& s = lists[threadIdx.x >> 6];
    const float* row = u + m * ldu;
    const unsigned long long below = (1ull << lane) - 1;
    uint32_t key[N];
#pragma unroll
    for (int i = 0; i < N; ++i) key[i] = 64 * i + lane < strips ? order_key(part_max[(long long)(64 * i + lane) * M + m]) : 0u;
    int equal = strips;
    uint32_t t = 0;
    if (strips > K) t = kth_largest<N>(key, K, &equal);
    // the chosen strips' numbers, in order, through the list's second half
    int chosen = 0, seen = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool in = 64 * i + lane < strips;
        const unsigned long long same = __ballot(in && key[i] == t);
        const bool keep = in && (strips <= K || key[i] > t || (key[i] == t && seen + __popcll(same & below) < equal));
        const unsigned long long k = __ballot(keep);
        if (keep) s.col[TOP_LIST - LOSS_MAX_TOP + chosen + __popcll(k & below)] = (uint32_t)(64 * i + lane);
        chosen += __popcll(k);
        seen += __popcll(same);
    }
    wave_sync();
    static_assert(LOSS_MAX_TOP == 256, "four words a lane");
    uint32_t strip[LOSS_MAX_TOP / 64];                   // number 64 i + l of the chosen strips at lane l
#pragma unroll
    for (int i = 0; i < LOSS_MAX_TOP / 64; ++i) strip[i] = 64 * i + lane < chosen ? s.col[TOP_LIST - LOSS_MAX_TOP + 64 * i + lane] : 0u;
    wave_sync();
    int n = 0;
    bool beyond = false;                                 // only what is larger than t is wanted any more
    for (int part = 0; 64 * part < chosen; ++part) {
        const int here = min(64, chosen - 64 * part);
        const int strips_here = (int)(part == 0 ? strip[0] : part == 1 ? strip[1] : part == 2 ? strip[2] : strip[3]);
        for (int j0 = 0; j0 < here; j0 += AHEAD) {
            float x[AHEAD];
            int col[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                col[j] = j0 + j < here ? (int)__builtin_amdgcn_readlane(strips_here, j0 + j) * LOSS_STRIP + lane : V;
                x[j] = col[j] < V ? row[col[j]] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const uint32_t k = order_key(x[j]);
                const bool take = col[j] < V && (k > t || (k == t && !beyond));
                const unsigned long long b = __ballot(take);
                if (b == 0) continue;
                if (take) { const int to = n + __popcll(b & below); s.key[to] = k; s.col[to] = (uint32_t)col[j]; }
                n += __popcll(b);
                if (n > TOP_LIST - 64) {
                    wave_sync();
                    t = cut_back<TOP_LIST / 64>(s, n, K);
                    n = K;
                    beyond = true;                       // (of what comes with t from here on, none is in front of those kept)
                }
            }
        }
    }
    wave_sync();
    if (n > K) {
        if (n <= 128) cut_back<2>(s, n, K);
        else cut_back<TOP_LIST / 64>(s, n, K);
    }
    // places by rank: the list is in order of the columns, so that of equal keys the one in front is the better
    for (int i = lane; i < K; i += 64) {
        const uint32_t k = s.key[i], c = s.col[i];
        int rank = 0;
        for (int j = 0; j < K; ++j) rank += s.key[j] > k || (s.key[j] == k && j < i);
        values[m * K + rank] = row[c];
        classes[m * K + rank] = (int32_t)c;
    }
}

// Maxima of the strips of every row (float logits, whose product does not make them): sixteen lanes a strip.
__global__ __launch_bounds__(256) void strip_max_kernel(const float* u, long long ldu, int M, int V, int strips, float* part_max) {
    const long long m = blockIdx.x;
    const float* row = u + m * ldu;
    const int l16 = threadIdx.x & 15;
    for (int s = blockIdx.y * 64 + (threadIdx.x >> 4), k = 0; k < 4; ++k, s += 16) {
        const int c = s * LOSS_STRIP + l16 * 4;
        float mx = __builtin_nanf("");
        if (c + 4 <= V) {
            const float4 x = *reinterpret_cast<const float4*>(row + c);
            mx = fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w));
        } else {
            for (int i = c; i < V; ++i) mx = fmaxf(mx, row[i]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        if (l16 == 0 && s < strips) part_max[(long long)s * M + m] = mx;
    }
}

// Any number of columns.  Finds the K-th largest key eight bits at a time, then, where more entries have that key than are wanted, the last column of
// them that is; what is above is collected in any order and put in its place by its rank.
__global__ __launch_bounds__(512) void row_topk_wide_kernel(const float* u, long long ldu, int V, int K, float* values, int32_t* classes) {
    __shared__ unsigned hist[256];
    __shared__ unsigned found, above, equal, count;
    __shared__ unsigned long long list[LOSS_MAX_TOP];
    const long long m = blockIdx.x;
    const float* row = u + m * ldu;
    const int tid = threadIdx.x;
    // bin of the `want`-th entry from the top of hist: `found`, entries above it: `above`, in it: `equal`
    auto pick = [&](unsigned want) {
        __syncthreads();
        if (tid < 64) {
            unsigned own = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) own += hist[255 - 4 * tid - j];
            unsigned before = own;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) { const unsigned t = __shfl_up(before, o, 64); if (tid >= o) before += t; }
            before -= own;
            if (before < want && before + own >= want) {
                unsigned run = before;
                for (int j = 0; j < 4; ++j) {
                    const unsigned h = hist[255 - 4 * tid - j];
                    if (run < want && run + h >= want) { found = 255 - 4 * tid - j; above = run; equal = h; }
                    run += h;
                }
            }
        }
        __syncthreads();
    };
    auto clear = [&] { __syncthreads(); if (tid < 256) hist[tid] = 0; __syncthreads(); };
    unsigned prefix = 0, want = (unsigned)K;             // the K-th largest agrees with prefix above the present byte; want-th among those
    for (int shift = 24; shift >= 0; shift -= 8) {
        clear();
        for (int v = tid; v < V; v += 512) {
            const uint32_t k = order_key(row[v]);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        }
        pick(want);
        want -= above;
        prefix |= found << shift;
    }
    unsigned last = 0xFFFFFFFFu;                         // of the entries with the K-th key, those up to this column
    if (equal != want) {
        unsigned inv = 0, w = want;                      // (the want-th largest of the columns counted from the end)
        for (int shift = 16; shift >= 0; shift -= 8) {
            clear();
            for (int v = tid; v < V; v += 512) {
                const unsigned k = 0xFFFFFFu - (unsigned)v;
                if (order_key(row[v]) == prefix && (shift == 16 || (k >> (shift + 8)) == (inv >> (shift + 8)))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
            pick(w);
            w -= above;
            inv |= found << shift;
        }
        last = 0xFFFFFFu - inv;
    }
    if (tid == 0) count = 0;
    __syncthreads();
    for (int v = tid; v < V; v += 512) {
        const uint32_t k = order_key(row[v]);
        if (k > prefix || (k == prefix && (unsigned)v <= last)) {
            const unsigned i = atomicAdd(&count, 1u);
            if (i < (unsigned)K) list[i] = ((unsigned long long)k << 32) | (0xFFFFFFFFu - (unsigned)v);
        }
    }
    __syncthreads();
    for (int i = tid; i < K; i += 512) {
        const unsigned long long k = list[i];
        int rank = 0;
        for (int j = 0; j < K; ++j) rank += list[j] > k;
        const unsigned c = 0xFFFFFFFFu - (unsigned)(k & 0xFFFFFFFFu);
        values[m * K + rank] = row[c];
        classes[m * K + rank] = (int32_t)c;
    }
}

}  // namespace

hipError_t launch_loss_prep(const LossPrepArgs& a, DType type, hipStream_t st) {
    const dim3 grid((unsigned)((a.M + 3) / 4 + (a.bias_f ? (a.V + 255) / 256 : 0)));
    if (type == DT_BF16) hipLaunchKernelGGL(loss_prep_kernel<bf16_t>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(loss_prep_kernel<float>, grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_loss_merge(const LossMergeArgs& a, hipStream_t st) {
    // A lane a part, whose loads are a row of floats apart, where parts are few, or rows: 4 us instead of 8 for one row of 250 parts, 12.6 instead
    // of 13.8 for 1344 of 500, but 190 instead of 22 for 21504 of 500, whose lines every four rows' workgroup fetches again.
    if (!a.policy && !a.rows && (a.strips <= 64 || a.M <= 1024)) {
        const dim3 rows((unsigned)(((a.consts ? a.Mp : a.M) + 3) / 4));
        const TeacherArgs t = a.teacher ? *a.teacher : TeacherArgs{};
        if (a.teacher) hipLaunchKernelGGL(loss_merge_row_kernel<true>, rows, dim3(256), 0, st, a, t);   // (always with two sums: one ends with dz)
        else hipLaunchKernelGGL(loss_merge_row_kernel<false>, rows, dim3(256), 0, st, a, t);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)((a.M + 63) / 64));
    const PolicyArgs p = a.policy ? *a.policy : PolicyArgs{};
    const TeacherArgs t = a.teacher ? *a.teacher : TeacherArgs{};
    if (a.policy) hipLaunchKernelGGL((loss_merge_kernel<false, true, false>), grid, dim3(512), 0, st, a, p, t);
    else if (a.teacher && a.part_sum_tau) hipLaunchKernelGGL((loss_merge_kernel<true, false, true>), grid, dim3(512), 0, st, a, p, t);
    else if (a.teacher) hipLaunchKernelGGL((loss_merge_kernel<false, false, true>), grid, dim3(512), 0, st, a, p, t);
    else hipLaunchKernelGGL((loss_merge_kernel<false, false, false>), grid, dim3(512), 0, st, a, p, t);
    return hipGetLastError();
}

hipError_t launch_loss_entries(const LossEntriesArgs& a, hipStream_t st) {
    hipLaunchKernelGGL(loss_entries_kernel, dim3((unsigned)((a.M + 3) / 4)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_loss_dz_end(const LossDzEndArgs& a, hipStream_t st) {
    hipLaunchKernelGGL(loss_dz_end_kernel, dim3((unsigned)((a.M + 3) / 4), (unsigned)((a.ld + 255) / 256)), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_loss_rows_f32(const LossRowsArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)a.M), block(512);
    const PolicyArgs p = a.policy ? *a.policy : PolicyArgs{};
    const TeacherArgs t = a.teacher ? *a.teacher : TeacherArgs{};
    const int words = (a.V + 3) / 4;
#define BLSTM_LOSS_ROWS(NC) do { \
    if (a.policy) hipLaunchKernelGGL((loss_rows_f32_kernel<NC, false, true, false, true>), grid, block, 0, st, a, p, t); \
    else if (a.teacher && t.inv_tau != 1.0f) hipLaunchKernelGGL((loss_rows_f32_kernel<NC, true, false, true, true>), grid, block, 0, st, a, p, t); \
    else if (a.teacher) hipLaunchKernelGGL((loss_rows_f32_kernel<NC, false, false, true, true>), grid, block, 0, st, a, p, t); \
    else hipLaunchKernelGGL((loss_rows_f32_kernel<NC, false, false, false, false>), grid, block, 0, st, a, p, t); } while (0)
    if (words <= 2 * 512) BLSTM_LOSS_ROWS(2);
    else if (words <= 8 * 512) BLSTM_LOSS_ROWS(8);
    else if (words <= 16 * 512) BLSTM_LOSS_ROWS(16);
    else BLSTM_LOSS_ROWS(0);
#undef BLSTM_LOSS_ROWS
    return hipGetLastError();
}

hipError_t launch_row_topk(const float* u, long long ldu, int M, int V, int K, float* part_max, bool have_max, float* values, int32_t* classes, hipStream_t st) {
    const int strips = (V + LOSS_STRIP - 1) / LOSS_STRIP;
    if (strips > LOSS_TOP_STRIPS) return hipErrorInvalidValue;
    if (!have_max) {
        hipLaunchKernelGGL(strip_max_kernel, dim3((unsigned)M, (unsigned)((strips + 63) / 64)), dim3(256), 0, st, u, ldu, M, V, strips, part_max);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)((M + 3) / 4));
    if (strips <= 128) hipLaunchKernelGGL(row_topk_kernel<2>, grid, dim3(256), 0, st, u, ldu, M, V, K, strips, part_max, values, classes);
    else if (strips <= 512) hipLaunchKernelGGL(row_topk_kernel<8>, grid, dim3(256), 0, st, u, ldu, M, V, K, strips, part_max, values, classes);
    else hipLaunchKernelGGL(row_topk_kernel<LOSS_TOP_STRIPS / 64>, grid, dim3(256), 0, st, u, ldu, M, V, K, strips, part_max, values, classes);
    return hipGetLastError();
}

hipError_t launch_row_topk_wide(const float* u, long long ldu, int M, int V, int K, float* values, int32_t* classes, hipStream_t st) {
    hipLaunchKernelGGL(row_topk_wide_kernel, dim3((unsigned)M), dim3(512), 0, st, u, ldu, V, K, values, classes);
    return hipGetLastError();
}

}  // namespace blstm
