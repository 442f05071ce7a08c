// Low-rank adapters of many sequences at once beside the projection that they share:
//   y = x W^T + b + s t B_a^T,  t = x A_a^T,   a = the adapter of the row's sequence          (W [N][K], A_a [r][K], B_a [N][r])
//   dx = dy W + s q A_a,  q = dy B_a;   dA_a = s sum q^T x,   dB_a = s sum dy^T t             over the rows of a's sequences
// The sequences are sorted by adapter on the device (adapt_plan_kernel), and no tile of rows holds two adapters' rows: A_a's rows ride along as
// further rows of W in one pass over x, and s t B_a^T is one more product on the tile's accumulators before they leave.  dx is the same kernel on
// dy with the transposed weights.  (W's gradient is an ordinary product: gemm.hip.)
// Numbers: sums in float; t and q enter their products as two bf16 numbers (2^-17) for y and dx, which leave as bf16, and as three for
// the gradients, which leave as float.  Parts are no parts where something is infinite (inf - inf, 0 inf): what they make of it is always NaN,
// and an element that is NaN is made once more from its definition in float.
#include "gemm_tile.hpp"
#include "adapters.hpp"
#include <algorithm>

namespace blstm {
namespace {

// ---- which rows belong together ----------------------------------------------------------------------------------------
// One workgroup: a stable counting sort of the sequences by key (the order within an adapter is the order of its sums), then the tables of tiles and
// chunks.  64 sequences a wavefront at a time: a lane's rank among equal keys of its wavefront, and the wavefronts' counts in turn.
constexpr int PLAN_THREADS = 1024, PLAN_KEPT = 4;
constexpr int plan_lds(int count) { return (4 * (count + 3) + 3 * (PLAN_THREADS / 64)) * 4; }
__device__ __forceinline__ int key_of(int id, int count) { return id >= 0 && id < count ? id : id == -1 ? count : count + 1; }
__device__ void make_plan(const AdaptShape& s, const AdaptPlan& p, const int32_t* ids, char* plan, int* lds) {
    int *hist = lds, *first = hist + s.count + 3, *tile0 = first + s.count + 3, *chunk0 = tile0 + s.count + 3, *wave_sum = chunk0 + s.count + 3;
    int* counts = reinterpret_cast<int*>(plan + p.counts);
    int* perm = reinterpret_cast<int*>(plan + p.perm);
    const int keys = s.count + 2, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bits = 32 - __clz(keys);
    for (int i = tid; i < keys; i += PLAN_THREADS) hist[i] = 0;
    // the first sequences' keys and places stay in registers (their loads run at once), the others' places wait in perm
    int kept[PLAN_KEPT], place[PLAN_KEPT];
#pragma unroll
    for (int q = 0; q < PLAN_KEPT; ++q) { const int b = q * PLAN_THREADS + tid; kept[q] = b < s.B ? ids[b] : 0; }
#pragma unroll
    for (int q = 0; q < PLAN_KEPT; ++q) kept[q] = q * PLAN_THREADS + tid < s.B ? key_of(kept[q], s.count) : -1;
    __syncthreads();
    auto sort = [&](int b0, int key) {                      // a sequence's place among those of its key
        unsigned long long same = ~0ull;
        for (int i = 0; i < bits; ++i) { const unsigned long long v = __ballot(key >> i & 1); same &= key >> i & 1 ? v : ~v; }
        same &= __ballot(key >= 0);
        const int rank = __popcll(same & ((1ull << lane) - 1));
        const bool last = lane == 63 || same >> (lane + 1) == 0;
        int at = 0;
        for (int w = 0; w < PLAN_THREADS / 64 && b0 + 64 * w < s.B; ++w) {
            if (w == wave && key >= 0) {
                const int base = hist[key];
                at = base + rank;
                if (last) hist[key] = base + rank + 1;     // (every lane of the wavefront has read before one writes: it runs in step)
            }
            __syncthreads();
        }
        return at;
    };
#pragma unroll
    for (int q = 0; q < PLAN_KEPT; ++q) if (q * PLAN_THREADS < s.B) place[q] = sort(q * PLAN_THREADS, kept[q]);
    for (int b0 = PLAN_KEPT * PLAN_THREADS; b0 < s.B; b0 += PLAN_THREADS) {
        const int b = b0 + tid, at = sort(b0, b < s.B ? key_of(ids[b], s.count) : -1);
        if (b < s.B) perm[b] = at;
    }
    // places, tiles and chunks in front of each key
    const int per = (keys + PLAN_THREADS - 1) / PLAN_THREADS, k0 = min(keys, tid * per), k1 = min(keys, k0 + per);
    int sum[3] = {0, 0, 0};
    auto add = [&](int k) {
        const long long rows = (long long)hist[k] * s.T;
        sum[0] += hist[k];
        sum[1] += (int)((rows + p.rows - 1) / p.rows);
        if (p.chunk && k < s.count) sum[2] += (int)((rows + p.chunk - 1) / p.chunk);
    };
    for (int k = k0; k < k1; ++k) add(k);
    int before[3];
    for (int i = 0; i < 3; ++i) {
        int v = sum[i];
        for (int o = 1; o < 64; o <<= 1) { const int u = __shfl_up(v, o); if (lane >= o) v += u; }
        if (lane == 63) wave_sum[i * (PLAN_THREADS / 64) + wave] = v;
        before[i] = v - sum[i];
    }
    __syncthreads();
    if (k0 < keys) for (int w = 0; w < wave; ++w) for (int i = 0; i < 3; ++i) before[i] += wave_sum[i * (PLAN_THREADS / 64) + w];
    for (int i = 0; i < 3; ++i) sum[i] = before[i];
    for (int k = k0; k < k1; ++k) { first[k] = sum[0]; tile0[k] = sum[1]; chunk0[k] = sum[2]; add(k); }
    if (k1 == keys && k0 < keys) { first[keys] = sum[0]; tile0[keys] = sum[1]; chunk0[keys] = sum[2]; }
    __syncthreads();
    const int tiles = tile0[keys], chunks = chunk0[keys];
    if (tid == 0) { counts[0] = tiles; counts[1] = chunks; }
    for (int k = tid; k <= keys; k += PLAN_THREADS) reinterpret_cast<int*>(plan + p.first)[k] = first[k];
    if (p.chunk) for (int k = tid; k <= s.count; k += PLAN_THREADS) reinterpret_cast<int*>(plan + p.first_chunk)[k] = chunk0[k];
    auto table = [&](const int* from, int n, int rows, int4* out) {
        for (int i = tid; i < n; i += PLAN_THREADS) {
            int lo = 0, hi = keys;                              // the key whose entries hold i: the last that starts at or before it
            while (hi - lo > 1) { const int m = (lo + hi) >> 1; if (from[m] <= i) lo = m; else hi = m; }
            const long long r0 = (long long)(i - from[lo]) * rows, all = (long long)hist[lo] * s.T;
            out[i] = make_int4(lo, (int)r0, (int)min((long long)rows, all - r0), first[lo]);
        }
    };
    table(tile0, tiles, p.rows, reinterpret_cast<int4*>(plan + p.tiles));
    for (int i = tiles + tid; i < p.max_tiles; i += PLAN_THREADS) reinterpret_cast<int4*>(plan + p.tiles)[i] = make_int4(0, 0, 0, 0);
    if (p.chunk) table(chunk0, chunks, p.chunk, reinterpret_cast<int4*>(plan + p.chunks));
    // (a lane reads the place that it wrote itself, and the sorted list lies behind the places)
#pragma unroll
    for (int q = 0; q < PLAN_KEPT; ++q) { const int b = q * PLAN_THREADS + tid; if (b < s.B) perm[s.B + first[kept[q]] + place[q]] = b; }
    for (int b = PLAN_KEPT * PLAN_THREADS + tid; b < s.B; b += PLAN_THREADS) perm[s.B + first[key_of(ids[b], s.count)] + perm[b]] = b;
}
__global__ __launch_bounds__(PLAN_THREADS) void adapt_plan_kernel(AdaptShape s, AdaptPlan p, const int32_t* ids, char* plan) {
    extern __shared__ int plan_words[];
    make_plan(s, p, ids, plan, plan_words);
}

// ---- products of 16-row tiles ------------------------------------------------------------------------------------------
// A fragment is 16 bytes of a row: eight bf16 are a product's k of their lane group, four floats one k each of four products.
template <typename T>
__device__ __forceinline__ void mma16(f32x4_t& acc, const uint4& a, const uint4& b) {
    if constexpr (sizeof(T) == 2) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    else {
        const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], acc, 0, 0, 0);
    }
}
// elements [k, k + 16 bytes) of a row of n, zero beyond it.  VECTOR: rows are whole aligned 16-byte words; else words start anywhere and a row's last may be short.
typedef uint32_t u32x4e_t __attribute__((ext_vector_type(4), aligned(2)));
template <typename T, bool VECTOR>
__device__ __forceinline__ uint4 load_chunk(const T* row, int k, int n) {
    constexpr int V = Vec<T>::N;
    if constexpr (VECTOR) {
        if (k < n) { const u32x4_t v = *reinterpret_cast<const u32x4_t*>(row + k); return make_uint4(v[0], v[1], v[2], v[3]); }
        return make_uint4(0u, 0u, 0u, 0u);
    } else {
        if (k + V <= n) { const u32x4_t v = *reinterpret_cast<const u32x4e_t*>(row + k); return make_uint4(v[0], v[1], v[2], v[3]); }
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (k + e < n) {
                if constexpr (sizeof(T) == 2) w[e >> 1] |= (uint32_t)row[k + e] << (16 * (e & 1));
                else w[e] = __builtin_bit_cast(uint32_t, row[k + e]);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// A workgroup's tile: from the plan's table or, of up to FIND sequences, found in ids by every workgroup itself (a launch in front of this one costs ten
// microseconds, looking for it one).  Adapters then come in the order of their first sequences.  *cols: which of ntn column blocks.  Ids go round-robin to the
// eight XCDs: a tile's column blocks go to one, whose L2 then holds its rows.  False: no tile for this workgroup.
constexpr int FIND = 256, FIND_WORDS = 2 * FIND + 24;
__device__ __forceinline__ bool find_tile(const ProjectArgs& a, int ntn, int* lds, int4* what, const int** order, int* cols) {
    const AdaptShape& s = a.s;
    const int slot = blockIdx.x >> 3, tile = slot / ntn * 8 + (blockIdx.x & 7);
    *cols = slot % ntn;
    if (a.plan) {
        if (tile >= a.p.max_tiles) return false;
        *what = reinterpret_cast<const int4*>(a.plan + a.p.tiles)[tile];
        if (what->z == 0) return false;
        *order = reinterpret_cast<const int*>(a.plan + a.p.perm) + s.B + what->w;
        return true;
    }
    int *keys = lds, *list = lds + FIND, *sums = list + FIND, *found = sums + 8;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    const int key = tid < s.B ? key_of(a.ids[tid], s.count) : -1;
    if (tid < FIND) keys[tid] = key;
    __syncthreads();
    int rank = 0, size = 0;
    for (int j0 = 0; j0 < s.B; j0 += 32)                     // (keys beyond the batch are -1)
#pragma unroll
    for (int j = j0; j < j0 + 32; j += 4) {
        const int4 k = *reinterpret_cast<const int4*>(keys + j);
        const int e0 = k.x == key, e1 = k.y == key, e2 = k.z == key, e3 = k.w == key;
        size += e0 + e1 + e2 + e3;
        rank += (e0 & (j < tid)) + (e1 & (j + 1 < tid)) + (e2 & (j + 2 < tid)) + (e3 & (j + 3 < tid));
    }
    if (tid >= s.B) size = 0;
    const int rows = size * s.T, mine = tid < s.B && rank == 0 ? (rows + a.p.rows - 1) / a.p.rows : 0;
    int upto = mine;
    for (int o = 1; o < 64; o <<= 1) { const int u = __shfl_up(upto, o); if (lane >= o) upto += u; }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int before = upto - mine, all = 0;
    for (int w = 0; w < waves; ++w) { if (w < wave) before += sums[w]; all += sums[w]; }
    if (tile >= all) return false;
    if (tile >= before && tile < before + mine) {
        const int r0 = (tile - before) * a.p.rows;
        found[0] = key; found[1] = r0; found[2] = min(a.p.rows, rows - r0);
    }
    __syncthreads();
    *what = make_int4(found[0], found[1], found[2], 0);
    if (tid < s.B && key == what->x) list[rank] = tid;
    __syncthreads();
    *order = list;
    return true;
}
__device__ __forceinline__ long long row_at(const AdaptShape& s, const int* order, int i) { const int j = i / s.T; return (long long)(i - j * s.T) * s.B + order[j]; }
// the first V columns from c on of a row of B_a (zero beyond the rank)
template <typename T>
__device__ __forceinline__ uint4 low_chunk(const T* row, int c, int rank, bool vector) {
    return vector ? load_chunk<T, true>(row, c, rank) : load_chunk<T, false>(row, c, rank);
}

// The NaNs among a lane's V x E values, as bits (none, hardly ever: asked in pairs first).
template <int V, int E, typename F>
__device__ __forceinline__ unsigned long long nans(F&& value) {
    static_assert(V * E <= 64 && E % 2 == 0, "bits");
    bool any = false;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < E; e += 2) any |= __builtin_isunordered(value(v, e), value(v, e + 1));
    unsigned long long found = 0;
    if (__any(any)) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < E; ++e) found |= (unsigned long long)(value(v, e) != value(v, e)) << (E * v + e);
    }
    return found;
}

// Few rows (a frame, a handful of rows an adapter): 16 rows x 32 columns.  What such a tile costs is the latency of its loads, so nothing is staged: eight wavefronts share the
// contraction, each loads its fragments straight into registers, four steps at a time, and their sums meet in LDS.  s t B_a^T is then a dot product a
// thread, in float.  One frame of one sequence (K 1024, N 256, rank 16): 16 us with the staged tile and its barriers, 8 here, of which a launch that does nothing takes 3;
// 64 sequences of as many adapters 12.
constexpr int RN = 32, RWAVES = 8;
template <typename T, int RB>
__global__ __launch_bounds__(64 * RWAVES) void adapt_rows_kernel(ProjectArgs a, bool vector, bool low_vector) {
    constexpr int V = Vec<T>::N, STEP = 4 * V, RP = 16 * RB, NB = RN / 16, DEEP = RB <= 2 ? 4 : RB == 4 ? 2 : 1;
    extern __shared__ uint4 smem[];
    __shared__ __align__(16) int words[FIND_WORDS];
    const AdaptShape& s = a.s;
    int4 what;
    const int* order;
    int col0;
    if (!find_tile(a, a.y ? (s.N + RN - 1) / RN : 1, words, &what, &order, &col0)) return;
    col0 *= RN;
    const int key = what.x, nrows = what.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, fr = lane & 15, fg = lane >> 4;
    const bool low = key < s.count;
    const T* W = static_cast<const T*>(a.W);
    const T* A = static_cast<const T*>(a.A) + (long long)(low ? key : 0) * s.rank * s.K;
    const T* Bm = static_cast<const T*>(a.Bm) + (long long)(low ? key : 0) * s.rank * s.N;
    // (rows of the last tile beyond the adapter's repeat the first: nothing of them leaves)
    const T* xr = static_cast<const T*>(a.x) + row_at(s, order, what.y + (fr < nrows ? fr : 0)) * s.K;
    // this thread's element of y, and the beginning of its row of B_a
    const int orow = tid / RN, n = col0 + tid % RN;
    uint4 fb[2] = {};
    const T* br = Bm + (long long)min(n, s.N - 1) * s.rank;
    if (low && a.y) { fb[0] = low_chunk<T>(br, 0, s.rank, low_vector); fb[1] = low_chunk<T>(br, V, s.rank, low_vector); }
    f32x4_t acc[NB + RB];
#pragma unroll
    for (int i = 0; i < NB + RB; ++i) acc[i] = f32x4_t{};
    const int steps = (s.K + STEP - 1) / STEP;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    auto run = [&](auto vec) {
        constexpr bool VECTOR = decltype(vec)::value;
        for (int s0 = wave; s0 < steps; s0 += RWAVES * DEEP) {
            uint4 fx[DEEP], fw[DEEP][NB + RB];
#pragma unroll
            for (int d = 0; d < DEEP; ++d) {
                const int k = (s0 + d * RWAVES) * STEP + fg * V;      // (beyond K: zeros)
                fx[d] = load_chunk<T, VECTOR>(xr, k, s.K);
#pragma unroll
                for (int j = 0; j < NB; ++j) { const int c = col0 + 16 * j + fr; fw[d][j] = c < s.N ? load_chunk<T, VECTOR>(W + (long long)c * s.K, k, s.K) : none; }
#pragma unroll
                for (int j = 0; j < RB; ++j) { const int r = 16 * j + fr; fw[d][NB + j] = low && r < s.rank ? load_chunk<T, VECTOR>(A + (long long)r * s.K, k, s.K) : none; }
            }
#pragma unroll
            for (int d = 0; d < DEEP; ++d)
#pragma unroll
                for (int j = 0; j < NB + RB; ++j) mma16<T>(acc[j], fx[d], fw[d][j]);
        }
    };
    if (vector) run(std::true_type{}); else run(std::false_type{});
    f32x4_t* part = reinterpret_cast<f32x4_t*>(smem);
#pragma unroll
    for (int j = 0; j < NB + RB; ++j) part[(wave * (NB + RB) + j) * 64 + lane] = acc[j];
    float* ts = reinterpret_cast<float*>(part + RWAVES * (NB + RB) * 64);
    constexpr int TLD = RP + 4;
    float* os = ts + 16 * TLD;
    const float bad = key > s.count ? __builtin_nanf("") : 0.0f;
    __syncthreads();
    for (int i = tid; i < (NB + RB) * 64; i += 64 * RWAVES) {
        f32x4_t v = part[i];
#pragma unroll
        for (int w = 1; w < RWAVES; ++w) v += part[w * (NB + RB) * 64 + i];
        const int j = i >> 6, l = i & 63, r = 4 * (l >> 4), c = l & 15;
#pragma unroll
        for (int e = 0; e < 4; ++e) { if (j < NB) os[(r + e) * (RN + 1) + 16 * j + c] = v[e] + bad; else ts[(r + e) * TLD + 16 * (j - NB) + c] = (low && 16 * (j - NB) + c < s.rank ? v[e] : 0.0f) + bad; }
    }
    __syncthreads();
    if (a.t && col0 == 0) {
        for (int i = tid; i < nrows * s.rank; i += 64 * RWAVES) { const int r = i / s.rank, c = i - r * s.rank; a.t[row_at(s, order, what.y + r) * s.rank + c] = ts[r * TLD + c]; }
    }
    if (!a.y || orow >= nrows || n >= s.N) return;
    float v = os[orow * (RN + 1) + tid % RN] + (a.b ? ld_f(static_cast<const T*>(a.b) + n) : 0.0f);
    if (low) {
        float sum = 0.0f;
        auto dot = [&](const uint4& f, int c) {
            float e[V];
            if constexpr (sizeof(T) == 2) {
                const uint32_t w[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) { e[2 * q] = bf2f((bf16_t)w[q]); e[2 * q + 1] = bf2f((bf16_t)(w[q] >> 16)); }
            } else { const f32x4_t w = __builtin_bit_cast(f32x4_t, f); e[0] = w[0]; e[1] = w[1]; e[2] = w[2]; e[3] = w[3]; }
#pragma unroll
            for (int q = 0; q < V; ++q) sum += c + q < RP ? e[q] * ts[orow * TLD + c + q] : 0.0f;
        };
        dot(fb[0], 0);
        dot(fb[1], V);
        for (int c = 2 * V; c < s.rank; c += V) dot(low_chunk<T>(br, c, s.rank, low_vector), c);
        v += s.scale * sum;
    }
    st_f(static_cast<T*>(a.y) + row_at(s, order, what.y + orow) * s.N + n, v);
}

// ROWS rows x 128 columns of y and all 16 RB columns of t in one pass over x.  A slab is 128 bytes of every row (x, W, A_a) in swizzled LDS; wavefront w multiplies
// columns 32 w .. of y and rows 16 w .. (and 64 + 16 w ..) of t.  Two buffers; DIRECT (rows of whole 16-byte
// words): slabs go from memory straight to LDS, else through registers.  What bounds it is a chain of latencies: of the 23 us of 256 sequences x 21 frames (K 1024, N 256,
// rank 16: 93 tiles of 64 rows, two column blocks each) 12 are the launch, the search for the tile, t's way through LDS and the stores, 0.7 each of the sixteen slabs
// (a third of it LDS reads).  Three and five buffers: 23.5 and 29.6 us (workgroups without a tile wait for a CU then).  128 rows where the adapters have them: dx of 2048
// sequences 95 -> 83 us, of which stores 18, the low-rank part 14, slabs two to four 23.  Two workgroups a CU are asked for where they fit: the accumulators then
// share the ordinary registers (256 sequences 23.8 -> 22.2 us, dx of 2048 83 -> 79).
constexpr int PN = 128;
template <typename T, int ROWS, int RB, bool DIRECT>
__global__ __launch_bounds__(256, DIRECT && RB <= 2 ? 2 : 1) void adapt_tile_kernel(ProjectArgs a, bool low_vector) {
    constexpr int V = Vec<T>::N, SLAB = 8 * V, MR = ROWS / 16, TR = ROWS / 64, RP = 16 * RB, ES = (int)sizeof(T);
    constexpr int NX = ROWS / 32, NW = 4, NA = (RP * 8 + 255) / 256;
    constexpr int STAGE = (ROWS + PN + RP) * CHUNKS;
    extern __shared__ uint4 smem[];
    __shared__ int rows[ROWS];
    const AdaptShape& s = a.s;
    int4 what;
    const int* order;
    int col0;
    if (!find_tile(a, a.y ? (s.N + PN - 1) / PN : 1, reinterpret_cast<int*>(smem), &what, &order, &col0)) return;
    col0 *= PN;
    const int key = what.x, nrows = what.z;
    const bool low = key < s.count;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (rows beyond the adapter's repeat its first: nothing of them leaves)
    if (tid < ROWS) rows[tid] = (int)row_at(s, order, what.y + (tid < nrows ? tid : 0));
    __syncthreads();
    const T* x = static_cast<const T*>(a.x);
    const T* W = static_cast<const T*>(a.W);
    const T* A = static_cast<const T*>(a.A) + (long long)(low ? key : 0) * s.rank * s.K;
    const T* Bm = static_cast<const T*>(a.Bm) + (long long)(low ? key : 0) * s.rank * s.N;
    f32x4_t acc[MR][2] = {}, tac[TR][RB] = {};
    const int fr = lane & 15, fg = lane >> 4;
    const int slabs = (s.K + SLAB - 1) / SLAB;
    auto multiply = [&](const uint4* at) {
        auto frag = [&](int r, int q) { return at[r * CHUNKS + ((4 * q + fg) ^ swz(r))]; };
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint4 fx[MR];
#pragma unroll
            for (int i = 0; i < MR; ++i) fx[i] = frag(16 * i + fr, q);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint4 fw = frag(ROWS + 32 * wave + 16 * j + fr, q);
#pragma unroll
                for (int i = 0; i < MR; ++i) mma16<T>(acc[i][j], fw, fx[i]);
            }
            if (low) {
                uint4 ft[TR];
#pragma unroll
                for (int i = 0; i < TR; ++i) ft[i] = frag(64 * i + 16 * wave + fr, q);
#pragma unroll
                for (int j = 0; j < RB; ++j) {
                    const uint4 fa = frag(ROWS + PN + 16 * j + fr, q);
#pragma unroll
                    for (int i = 0; i < TR; ++i) mma16<T>(tac[i][j], fa, ft[i]);
                }
            }
        }
    };
    // B_a's part of the tile: asked for ahead of everything else
    constexpr int BSTEP = 4 * V, BQ = (RP + BSTEP - 1) / BSTEP;      // columns of t a step
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    uint4 fb[BQ][2];
#pragma unroll
    for (int q = 0; q < BQ; ++q)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int n = col0 + 32 * wave + 16 * j + fr;
            fb[q][j] = low && a.y && n < s.N ? low_chunk<T>(Bm + (long long)n * s.rank, q * BSTEP + fg * V, s.rank, low_vector) : none;
        }
    if constexpr (DIRECT) {
        // Instruction j of a wavefront fills eight rows: lane l fetches the chunk that belongs at slot l % 8 of row l / 8.  Rows beyond W's and A's repeat their last.
        constexpr int NAI = RB >= 2 ? RB / 2 : 1;
        const char* px[NX]; const char* pw[NW]; const char* pa[NAI];
        const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
        const int lr = lane >> 3;
        auto chunk = [&](int r) { return ((lane & 7) ^ swz(r)) * 16; };
#pragma unroll
        for (int j = 0; j < NX; ++j) { const int r = 8 * (4 * j + wave) + lr; px[j] = reinterpret_cast<const char*>(x + (long long)rows[r] * s.K) + chunk(r); }
#pragma unroll
        for (int j = 0; j < NW; ++j) { const int r = 8 * (4 * j + wave) + lr; pw[j] = reinterpret_cast<const char*>(W + (long long)min(col0 + r, s.N - 1) * s.K) + chunk(ROWS + r); }
        const bool has_a = RB >= 2 || wave < 2;              // (16 rows are two instructions)
#pragma unroll
        for (int j = 0; j < NAI; ++j) { const int r = 8 * (4 * j + wave) + lr; pa[j] = reinterpret_cast<const char*>(A + (long long)min(r, s.rank - 1) * s.K) + chunk(ROWS + PN + r); }
        auto dma = [](unsigned lds_addr, const char* from) __attribute__((always_inline)) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(from) : "memory");
        };
        const int words = s.K / V;                           // 16-byte words of a row
        auto issue = [&](int it) __attribute__((always_inline)) {
            const unsigned sb = lds0 + (unsigned)(it & 1) * (STAGE * 16);
            const long long off = (long long)it * 128;
            const int left = words - it * 8;                 // (words beyond the row's end repeat its last, and are cleared below)
            auto from = [&](const char* p, int r) { return p + off - (left < 8 ? max(((lane & 7) ^ swz(r)) - (left - 1), 0) * 16 : 0); };
#pragma unroll
            for (int j = 0; j < NX; ++j) dma(sb + (unsigned)(4 * j + wave) * 1024, from(px[j], 8 * (4 * j + wave) + lr));
#pragma unroll
            for (int j = 0; j < NW; ++j) dma(sb + ROWS * 128 + (unsigned)(4 * j + wave) * 1024, from(pw[j], ROWS + 8 * (4 * j + wave) + lr));
            if (has_a) {
#pragma unroll
                for (int j = 0; j < NAI; ++j) dma(sb + (ROWS + PN) * 128 + (unsigned)(4 * j + wave) * 1024, from(pa[j], ROWS + PN + 8 * (4 * j + wave) + lr));
            }
        };
        issue(0);
        for (int it = 0; it < slabs; ++it) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // (the slab has landed, the reads of the other buffer have come)
            if (it + 1 < slabs) issue(it + 1);
            uint4* at = smem + (it & 1) * STAGE;
            if (words - it * 8 < 8) {
                for (int i = tid; i < STAGE; i += 256) if (((i & 7) ^ swz(i >> 3)) >= words - it * 8) at[i] = none;
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
            multiply(at);
        }
        __syncthreads();
    } else {
        const int ch = tid & 7;
        uint4 rx[NX], rw[NW], ra[NA];
        auto load = [&](int k0) {
            const int k = k0 + ch * V;
#pragma unroll
            for (int i = 0; i < NX; ++i) rx[i] = load_chunk<T, false>(x + (long long)rows[(tid >> 3) + 32 * i] * s.K, k, s.K);
#pragma unroll
            for (int i = 0; i < NW; ++i) { const int n = col0 + (tid >> 3) + 32 * i; rw[i] = n < s.N ? load_chunk<T, false>(W + (long long)n * s.K, k, s.K) : none; }
#pragma unroll
            for (int i = 0; i < NA; ++i) { const int r = (tid >> 3) + 32 * i; ra[i] = low && r < s.rank ? load_chunk<T, false>(A + (long long)r * s.K, k, s.K) : none; }
        };
        auto store = [&](int buf) {
            uint4* to = smem + buf * STAGE;
            auto put = [&](int r, const uint4& v) { to[r * CHUNKS + (ch ^ swz(r))] = v; };
#pragma unroll
            for (int i = 0; i < NX; ++i) put((tid >> 3) + 32 * i, rx[i]);
#pragma unroll
            for (int i = 0; i < NW; ++i) put(ROWS + (tid >> 3) + 32 * i, rw[i]);
#pragma unroll
            for (int i = 0; i < NA; ++i) { const int r = (tid >> 3) + 32 * i; if (r < RP) put(ROWS + PN + r, ra[i]); }
        };
        load(0);
        store(0);
        __syncthreads();
        for (int it = 0; it < slabs; ++it) {
            if (it + 1 < slabs) load((it + 1) * SLAB);
            multiply(smem + (it & 1) * STAGE);
            if (it + 1 < slabs) store((it + 1) & 1);
            __syncthreads();
        }
    }
    // t, for everybody: rows of RP floats, zero beyond the rank
    float* ts = reinterpret_cast<float*>(smem);
    constexpr int TLD = RP + 4;
    const float bad = key > s.count ? __builtin_nanf("") : 0.0f;
#pragma unroll
    for (int i = 0; i < TR; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j)
        {
            f32x4_t v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = 16 * j + 4 * fg + e < s.rank ? tac[i][j][e] + bad : 0.0f;
            *reinterpret_cast<f32x4_t*>(ts + (64 * i + 16 * wave + fr) * TLD + 16 * j + 4 * fg) = v;
        }
    __syncthreads();
    if (a.t && col0 == 0) {
        for (int i = tid; i < nrows * s.rank; i += 256) { const int r = i / s.rank, c = i - r * s.rank; a.t[(long long)rows[r] * s.rank + c] = ts[r * TLD + c]; }
    }
    if (!a.y) return;
    T* y = static_cast<T*>(a.y);
    if (low) {
        // s t B_a^T: t in two bf16 parts, or as it is
#pragma unroll
        for (int q = 0; q < BQ; ++q) {
            const int c = q * BSTEP + fg * V;
#pragma unroll
            for (int i = 0; i < MR; ++i) {
                float v[V];
#pragma unroll
                for (int e = 0; e < V; e += 4) {
                    const f32x4_t w = c < RP ? *reinterpret_cast<const f32x4_t*>(ts + (16 * i + fr) * TLD + c + e) : f32x4_t{};
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[e + k] = s.scale * w[k];
                }
                uint4 hi, lo;
                if constexpr (ES == 2) {
                    uint32_t h[4], l[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        h[e] = pack_bf2(v[2 * e], v[2 * e + 1]);
                        l[e] = pack_bf2(v[2 * e] - bf2f((bf16_t)h[e]), v[2 * e + 1] - bf2f((bf16_t)(h[e] >> 16)));
                    }
                    hi = make_uint4(h[0], h[1], h[2], h[3]); lo = make_uint4(l[0], l[1], l[2], l[3]);
                } else hi = __builtin_bit_cast(uint4, f32x4_t{v[0], v[1], v[2], v[3]});
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if constexpr (ES == 2) mma16<T>(acc[i][j], fb[q][j], lo);
                    mma16<T>(acc[i][j], fb[q][j], hi);
                }
            }
        }
    }
    // (the products are computed transposed: a lane holds four neighbouring columns of a row)
    typedef uint32_t u32x2e_t __attribute__((ext_vector_type(2), aligned(2)));
    typedef float f32x4e_t __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int n = col0 + 32 * wave + 16 * j + 4 * fg;
        if (n >= s.N) continue;
        f32x4_t bias = {bad, bad, bad, bad};
        if (a.b) {
#pragma unroll
            for (int e = 0; e < 4; ++e) if (n + e < s.N) bias[e] += ld_f(static_cast<const T*>(a.b) + n + e);
        }
#pragma unroll
        for (int i = 0; i < MR; ++i) {
            if (16 * i + fr >= nrows) continue;
            T* to = y + (long long)rows[16 * i + fr] * s.N + n;
            const f32x4_t v = acc[i][j] + bias;
            if (n + 4 <= s.N) {
                if constexpr (ES == 2) { u32x2_t w; w[0] = pack_bf2(v[0], v[1]); w[1] = pack_bf2(v[2], v[3]); *reinterpret_cast<u32x2e_t*>(to) = w; }
                else *reinterpret_cast<f32x4e_t*>(to) = v;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) if (n + e < s.N) st_f(to + e, v[e]);
            }
        }
    }
    if (ES == 2 && low) {
        unsigned long long odd = nans<2 * MR, 4>([&](int v, int e) { return acc[v >> 1][v & 1][e]; });
#pragma unroll 1
        for (; odd; odd &= odd - 1) {
            const int b = __ffsll(odd) - 1, r = 16 * (b >> 3) + fr, n = col0 + 32 * wave + 16 * (b >> 2 & 1) + 4 * fg + (b & 3);
            if (r >= nrows || n >= s.N) continue;
            float part = 0.0f, sum = a.b ? ld_f(static_cast<const T*>(a.b) + n) : 0.0f;
#pragma unroll 1
            for (int c = 0; c < s.rank; ++c) part += ts[r * TLD + c] * ld_f(Bm + (long long)n * s.rank + c);
            if (part != part) continue;
#pragma unroll 4
            for (int k = 0; k < s.K; ++k) sum += ld_f(x + (long long)rows[r] * s.K + k) * ld_f(W + (long long)n * s.K + k);
            st_f(y + (long long)rows[r] * s.N + n, sum + s.scale * part);
        }
    }
}

template <typename T, int RB>
void run_rows(const ProjectArgs& a, bool vector, bool low_vector, hipStream_t st) {
    constexpr int lds = RWAVES * (RN / 16 + RB) * 1024 + 16 * (16 * RB + 4) * 4 + 16 * (RN + 1) * 4;
    const int ntn = a.y ? (a.s.N + RN - 1) / RN : 1;
    adapt_rows_kernel<T, RB><<<(a.p.max_tiles + 7) / 8 * 8 * ntn, 64 * RWAVES, lds, st>>>(a, vector, low_vector);
}
template <typename T, int ROWS, int RB, bool DIRECT>
void run_tile(const ProjectArgs& a, bool low_vector, hipStream_t st) {
    constexpr int loop = 2 * (ROWS + PN + 16 * RB) * 128, t = ROWS * (16 * RB + 4) * 4, lds = loop > t ? loop : t;
    static_assert(lds + 4 * ROWS <= 160 * 1024, "LDS of a CU");
    const int ntn = a.y ? (a.s.N + PN - 1) / PN : 1;
    adapt_tile_kernel<T, ROWS, RB, DIRECT><<<(a.p.max_tiles + 7) / 8 * 8 * ntn, 256, lds, st>>>(a, low_vector);
}
template <typename T, int RB>
void run_project(const ProjectArgs& a, bool vector, bool low_vector, hipStream_t st) {
    if (a.p.rows == 16) run_rows<T, RB>(a, vector, low_vector, st);
    else if (a.p.rows == 128) { if (vector) run_tile<T, 128, RB, true>(a, low_vector, st); else run_tile<T, 128, RB, false>(a, low_vector, st); }
    else if (vector) run_tile<T, 64, RB, true>(a, low_vector, st);
    else run_tile<T, 64, RB, false>(a, low_vector, st);
}
template <typename T>
hipError_t project(const ProjectArgs& a, hipStream_t st) {
    auto whole = [&](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const bool vector = a.s.K % Vec<T>::N == 0 && whole(a.x) && whole(a.W) && whole(a.A);
    const bool low_vector = a.s.rank % Vec<T>::N == 0 && whole(a.Bm);
    if (a.s.rank <= 16) run_project<T, 1>(a, vector, low_vector, st);
    else if (a.s.rank <= 32) run_project<T, 2>(a, vector, low_vector, st);
    else if (a.s.rank <= 64) run_project<T, 4>(a, vector, low_vector, st);
    else run_project<T, 8>(a, vector, low_vector, st);
    return hipGetLastError();
}

// ---- transposed weights ----------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(PLAN_THREADS) void adapt_transpose_kernel(TransposeArgs a, AdaptPlan p, const int32_t* ids, char* plan) {
    extern __shared__ int words[];
    const AdaptShape& s = a.s;
    // (the plan is a chain of latencies: the first workgroup makes it while the others move)
    if (blockIdx.x == 0) { make_plan(s, p, ids, plan, words); return; }
    // eight tiles of 32 x 32 a workgroup, 256 threads two of them (one: 13 us instead of 11 for 100 adapters of 16 x 1024 and 256 x 16)
    auto tiles = [](int r, int c) { return ((r + 31) / 32) * ((c + 31) / 32); };
    const int tw = tiles(s.N, s.K), ta = tiles(s.rank, s.K), tb = tiles(s.N, s.rank), sub = threadIdx.x >> 8, i = threadIdx.x >> 5 & 7, j = threadIdx.x & 31;
    const T* from[2]; T* to[2];
    int R[2], C[2], r0[2], c0[2];
    T v[2][4];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        int id = (blockIdx.x - 1) * 8 + sub * 2 + q;
        from[q] = nullptr; to[q] = nullptr; R[q] = C[q] = 0;
        if (id < tw) { from[q] = static_cast<const T*>(a.W); to[q] = static_cast<T*>(a.Wt); R[q] = s.N; C[q] = s.K; }
        else if ((id -= tw) < ta * s.count) { const long long k = id / ta; id %= ta; R[q] = s.rank; C[q] = s.K; from[q] = static_cast<const T*>(a.A) + k * R[q] * C[q]; to[q] = static_cast<T*>(a.At) + k * R[q] * C[q]; }
        else if ((id -= ta * s.count) < tb * s.count) { const long long k = id / tb; id %= tb; R[q] = s.N; C[q] = s.rank; from[q] = static_cast<const T*>(a.Bm) + k * R[q] * C[q]; to[q] = static_cast<T*>(a.Bt) + k * R[q] * C[q]; }
        else id = 0;                                        // (the last workgroup's tiles beyond the last: empty)
        const int nc = max(1, (C[q] + 31) / 32);
        r0[q] = id / nc * 32; c0[q] = id % nc * 32;
#pragma unroll
        for (int e = 0; e < 4; ++e) if (r0[q] + i + 8 * e < R[q] && c0[q] + j < C[q]) v[q][e] = from[q][(long long)(r0[q] + i + 8 * e) * C[q] + c0[q] + j];
    }
    T (*lds)[33] = reinterpret_cast<T (*)[33]>(words) + 64 * sub;
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) if (r0[q] + i + 8 * e < R[q] && c0[q] + j < C[q]) lds[32 * q + i + 8 * e][j] = v[q][e];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) if (c0[q] + i + 8 * e < C[q] && r0[q] + j < R[q]) to[q][(long long)(c0[q] + i + 8 * e) * R[q] + r0[q] + j] = lds[32 * q + j][i + 8 * e];
}

// ---- the adapters' gradients -------------------------------------------------------------------------------------------
// A lane's rows of column `col` of a chunk's product: to the parts of its sum, or, of an adapter with one chunk, straight to dA or dB (256 sequences, 100 adapters,
// most of them with one: products and sums 19 -> 16 us).
template <int RB>
__device__ __forceinline__ void grad_out(const AdaptGradArgs& a, int chunk, int key, bool only, bool second, int col, const f32x16_t (&acc)[RB]) {
    const AdaptShape& s = a.s;
    if (col >= (second ? s.N : s.K)) return;
    const int r0 = 4 * ((threadIdx.x & 63) >> 5);
    typedef float f32x4e_t __attribute__((ext_vector_type(4), aligned(4)));
    auto put = [&](float* out, long long ld, float by) __attribute__((always_inline)) {      // element r of the column lies r ld behind the first
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) { const int r = 32 * i + 8 * (e >> 2) + r0 + (e & 3); if (r < s.rank) out[r * ld] = by * acc[i][e]; }
    };
    if (!only) put(a.part + (long long)chunk * s.rank * (s.K + s.N) + (second ? s.K : 0) + col, s.K + s.N, 1.0f);
    else if (!second) put(a.dA + (long long)key * s.rank * s.K + col, s.K, s.scale);
    else if (s.rank % 4) put(a.dB + ((long long)key * s.N + col) * s.rank, 1, s.scale);
    else {
        float* out = a.dB + ((long long)key * s.N + col) * s.rank;
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = 32 * i + 8 * q + r0;
                if (r < s.rank) *reinterpret_cast<f32x4e_t*>(out + r) = f32x4e_t{s.scale * acc[i][4 * q], s.scale * acc[i][4 * q + 1], s.scale * acc[i][4 * q + 2], s.scale * acc[i][4 * q + 3]};
            }
    }
}

// The sums of a lane that are NaN, once more in float.  (The parts cleared in every product where they meet infinities: 196 us for 2048 sequences became 206; looked for afterwards: 196.
// A batch all of NaN: 2 ms.)
template <typename T, int RB, typename F>
__device__ __forceinline__ void grad_again(const AdaptGradArgs& a, int chunk, int key, bool only, bool second, int col, const f32x16_t (&acc)[RB], int nrows, F&& row_of) {
    unsigned long long odd = nans<RB, 16>([&](int v, int e) { return acc[v][e]; });
    const AdaptShape& s = a.s;
    const int width = second ? s.N : s.K;
    if (col >= width) return;
    const T* R = static_cast<const T*>(second ? a.dy : a.x);
    const float* L = second ? a.t : a.q;
#pragma unroll 1
    for (; odd; odd &= odd - 1) {
        const int b = __ffsll(odd) - 1, r = 8 * (b >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (b & 3);
        if (r >= s.rank) continue;
        float sum = 0.0f;
#pragma unroll 4
        for (int k = 0; k < nrows; ++k) { const long long row = row_of(k); sum += L[row * s.rank + r] * ld_f(R + row * width + col); }
        if (!only) a.part[((long long)chunk * s.rank + r) * (s.K + s.N) + (second ? s.K : 0) + col] = sum;
        else if (second) a.dB[((long long)key * s.N + col) * s.rank + r] = s.scale * sum;
        else a.dA[((long long)key * s.rank + r) * s.K + col] = s.scale * sum;
    }
}

// sum over a chunk's rows of L[row][i] R[row][j]: L = q with R = x, L = t with R = dy.  A workgroup: a chunk and 128 columns of x or dy, 32 a
// wavefront, 32 RB rows of the result.  64 rows at a time lie in LDS as they lie in memory; 16-bit ones are transposed by the LDS read.
template <typename T, int RB, bool VECTOR>
__global__ __launch_bounds__(256) void adapt_grad_kernel(AdaptGradArgs a) {
    constexpr int V = Vec<T>::N, PARTS = sizeof(T) == 2 ? 3 : 1, RP = 32 * RB, ES = (int)sizeof(T);
    constexpr int RLD = 128 * ES + 16, LLD = RP * ES + 16;                 // bytes of a row
    constexpr int NR = 64 * 128 / V / 256;
    extern __shared__ uint4 smem[];
    char* rs = reinterpret_cast<char*>(smem);
    char* ls = rs + 64 * RLD;
    const AdaptShape& s = a.s;
    const int nk = (s.K + 127) / 128, nn = (s.N + 127) / 128, chunk = blockIdx.x / (nk + nn), ct = blockIdx.x % (nk + nn);
    if (chunk >= reinterpret_cast<const int*>(a.plan + a.p.counts)[1]) return;
    const int4 what = reinterpret_cast<const int4*>(a.plan + a.p.chunks)[chunk];
    const int* order = reinterpret_cast<const int*>(a.plan + a.p.perm) + s.B + what.w;
    const int* first = reinterpret_cast<const int*>(a.plan + a.p.first_chunk) + what.x;
    const int chunks_of[2] = {first[0], first[1]};
    const bool second = ct >= nk;
    const int width = second ? s.N : s.K, c0 = (second ? ct - nk : ct) * 128;
    const T* R = static_cast<const T*>(second ? a.dy : a.x);
    const float* L = second ? a.t : a.q;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto row_of = [&](int r) { const int i = what.y + r, j = i / s.T; return (long long)(i - j * s.T) * s.B + order[j]; };
    f32x16_t acc[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    for (int r0 = 0; r0 < what.z; r0 += 64) {
        uint4 v[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int c = tid + 256 * i, r = c / (128 / V), k = c0 + c % (128 / V) * V;
            v[i] = r0 + r < what.z ? load_chunk<T, VECTOR>(R + row_of(r0 + r) * width, k, width) : none;
        }
        float l[64 * RP / 256];
#pragma unroll
        for (int i = 0; i < 64 * RP / 256; ++i) {
            const int c = tid + 256 * i, r = c / RP, k = c % RP;
            l[i] = r0 + r < what.z && k < s.rank ? L[row_of(r0 + r) * s.rank + k] : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NR; ++i) { const int c = tid + 256 * i; *reinterpret_cast<uint4*>(rs + c / (128 / V) * RLD + c % (128 / V) * 16) = v[i]; }
#pragma unroll
        for (int i = 0; i < 64 * RP / 256; ++i) {
            const int c = tid + 256 * i, r = c / RP, k = c % RP;
            float left = l[i];
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                if constexpr (ES == 2) { const bf16_t h = f2bf(left); *reinterpret_cast<bf16_t*>(ls + (p * 64 + r) * LLD + 2 * k) = h; left -= bf2f(h); }
                else *reinterpret_cast<float*>(ls + r * LLD + 4 * k) = left;
            }
        }
        __syncthreads();
        if constexpr (ES == 2) {
            const int g = lane >> 4, li = lane & 15, at = (8 * (g >> 1) + (li >> 2)), off = 32 * (g & 1) + (li & 3) * 8;
#pragma unroll
            for (int k = 0; k < 64; k += 16) {
                const uint4 fr = lfrag_tr<RLD>(rs + at * RLD + wave * 64 + off, k);
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int p = PARTS - 1; p >= 0; --p) {
                        const uint4 fl = lfrag_tr<LLD>(ls + (p * 64 + at) * LLD + i * 64 + off, k);
                        acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, fl), __builtin_bit_cast(bf16x8_t, fr), acc[i], 0, 0, 0);
                    }
            }
        } else {
#pragma unroll 8
            for (int k = 0; k < 64; k += 2) {
                const int r = k + (lane >> 5), c = lane & 31;
                const float fr = *reinterpret_cast<const float*>(rs + r * RLD + (32 * wave + c) * 4);
#pragma unroll
                for (int i = 0; i < RB; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(ls + r * LLD + (32 * i + c) * 4), fr, acc[i], 0, 0, 0);
            }
        }
    }
    const bool only = chunks_of[1] - chunks_of[0] == 1;
    const int col = c0 + 32 * wave + (lane & 31);
    grad_out<RB>(a, chunk, what.x, only, second, col, acc);
    if constexpr (ES == 2) grad_again<T, RB>(a, chunk, what.x, only, second, col, acc, what.z, row_of);
}

// The same in bf16 where rows are whole 16-byte words: two slabs of 64 rows of x (or dy) and of q (or t) come straight to LDS in turn, one while the other is
// multiplied; q's (t's) three bf16 parts are made of the slab that has landed.  256 sequences x 21 frames, K 1024, 100 adapters: 15 us through registers; 2048 sequences,
// 24 adapters 70 us: 11 and 36 here, 3.1 TB/s
// of x, dy and the parts of the sums.
template <int RB>
__global__ __launch_bounds__(256) void adapt_grad_direct_kernel(AdaptGradArgs a) {
    constexpr int RP = 32 * RB, LLD = RP * 2 + 16, RS = 64 * 256, LS = 64 * RP * 4, STAGE = RS + LS, LCH = RP / 4;     // bytes; 16-byte words of a row of q
    constexpr int NR = 4, NL = LS / 1024 / 4;                // load instructions of a wavefront and slab
    extern __shared__ uint4 smem[];
    __shared__ int rows[ADAPT_MAX_CHUNK];
    char* base = reinterpret_cast<char*>(smem);
    char* planes = base + 2 * STAGE;
    const AdaptShape& s = a.s;
    const int nk = (s.K + 127) / 128, nn = (s.N + 127) / 128, ncol = nk + nn;
    // (a chunk's columns on one XCD: they share q)
    const int slot = blockIdx.x >> 3, chunk = slot / ncol * 8 + (blockIdx.x & 7), ct = slot % ncol;
    if (chunk >= reinterpret_cast<const int*>(a.plan + a.p.counts)[1]) return;
    const int4 what = reinterpret_cast<const int4*>(a.plan + a.p.chunks)[chunk];
    const int* order = reinterpret_cast<const int*>(a.plan + a.p.perm) + s.B + what.w;
    const int* first = reinterpret_cast<const int*>(a.plan + a.p.first_chunk) + what.x;
    const int chunks_of[2] = {first[0], first[1]};
    const bool second = ct >= nk;
    const int width = second ? s.N : s.K, c0 = (second ? ct - nk : ct) * 128, nrows = what.z, slabs = (nrows + 63) / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int r = tid; r < nrows; r += 256) rows[r] = (int)row_at(s, order, what.y + r);
    __syncthreads();
    const char* R = static_cast<const char*>(second ? a.dy : a.x) + c0 * 2;
    const char* L = reinterpret_cast<const char*>(second ? a.t : a.q);
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
    auto dma = [](unsigned lds_addr, const char* from) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(from) : "memory");
    };
    const int last_word = (width - c0) / 8 - 1, last_low = s.rank / 4 - 1;
    // (rows behind the chunk's last repeat it and are cleared; words beyond a row's end repeat its last: those columns go nowhere)
    auto issue = [&](int it) __attribute__((always_inline)) {
        const unsigned sb = lds0 + (unsigned)(it & 1) * STAGE;
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            const int jj = 4 * j + wave, kt = 4 * jj + (lane >> 4), pos = lane & 15, mc = (((pos >> 1) ^ tr_swz<16>(kt)) << 1) | (pos & 1);
            dma(sb + jj * 1024, R + (long long)rows[min(64 * it + kt, nrows - 1)] * (2 * width) + min(mc, last_word) * 16);
        }
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int w = (4 * j + wave) * 64 + lane, r = w / LCH, c = w % LCH;
            dma(sb + RS + (4 * j + wave) * 1024, L + (long long)rows[min(64 * it + r, nrows - 1)] * (4 * s.rank) + min(c, last_low) * 16);
        }
    };
    f32x16_t acc[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
    issue(0);
    const int g = lane >> 4, li = lane & 15, at = 8 * (g >> 1) + (li >> 2), off = 32 * (g & 1) + (li & 3) * 8;
    const int tr = at * 256 + (((2 * wave + (g & 1)) ^ tr_swz<16>(li >> 2)) << 5) + (li & 3) * 8;
    for (int it = 0; it < slabs; ++it) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // (the slab has landed, the reads of the other buffer have come)
        if (it + 1 < slabs) issue(it + 1);
        char* rs = base + (it & 1) * STAGE;
        const int left = nrows - 64 * it;
        if (left < 64) for (int i = left * 16 + tid; i < 1024; i += 256) reinterpret_cast<uint4*>(rs)[i] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int w = tid + 256 * j, r = w / LCH, c = w % LCH * 4;
            f32x4_t v = *reinterpret_cast<const f32x4_t*>(rs + RS + w * 16);
            if (r >= left || c >= s.rank) v = f32x4_t{};
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                u32x2_t h;
                h[0] = pack_bf2(v[0], v[1]); h[1] = pack_bf2(v[2], v[3]);
                *reinterpret_cast<u32x2_t*>(planes + (p * 64 + r) * LLD + 2 * c) = h;
                v[0] -= bf2f((bf16_t)h[0]); v[1] -= bf2f((bf16_t)(h[0] >> 16)); v[2] -= bf2f((bf16_t)h[1]); v[3] -= bf2f((bf16_t)(h[1] >> 16));
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int k = 0; k < 64; k += 16) {
            const uint4 fr = lfrag_tr<256>(rs + tr, k);
#pragma unroll
            for (int i = 0; i < RB; ++i)
#pragma unroll
                for (int p = 2; p >= 0; --p) {
                    const uint4 fl = lfrag_tr<LLD>(planes + (p * 64 + at) * LLD + i * 64 + off, k);
                    acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, fl), __builtin_bit_cast(bf16x8_t, fr), acc[i], 0, 0, 0);
                }
        }
    }
    const bool only = chunks_of[1] - chunks_of[0] == 1;
    const int col = c0 + 32 * wave + (lane & 31);
    grad_out<RB>(a, chunk, what.x, only, second, col, acc);
    grad_again<bf16_t, RB>(a, chunk, what.x, only, second, col, acc, nrows, [&](int k) { return (long long)rows[k]; });
}

// An adapter's chunks in order, where it has none or several; dB leaves transposed (through LDS).  `groups` workgroups an adapter.
__global__ __launch_bounds__(256) void adapt_grad_sum_kernel(AdaptGradArgs a, int groups) {
    __shared__ float lds[32][33];
    const AdaptShape& s = a.s;
    const int wide = s.K + s.N, nr = (s.rank + 31) / 32, nk = (s.K + 31) / 32, nc = nk + (s.N + 31) / 32, key = blockIdx.x / groups;
    const int* first = reinterpret_cast<const int*>(a.plan + a.p.first_chunk);
    const int from = first[key], to = first[key + 1], i = threadIdx.x >> 5, j = threadIdx.x & 31;
    if (to - from == 1) return;
    for (int t = blockIdx.x % groups; t < nr * nc; t += groups) {
        const int r0 = t / nc * 32, ci = t % nc;
        const bool second = ci >= nk;
        const int c0 = second ? (ci - nk) * 32 : ci * 32, width = second ? s.N : s.K;
        const int c = c0 + j;
        float v[4] = {};
        const float* at[4];                                 // (beyond the edges: a place that exists, and goes nowhere)
#pragma unroll
        for (int e = 0; e < 4; ++e) at[e] = a.part + ((long long)from * s.rank + min(r0 + i + 8 * e, s.rank - 1)) * wide + (second ? s.K : 0) + min(c, width - 1);
#pragma unroll 2
        for (int k = 0; k < to - from; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += at[e][(long long)k * s.rank * wide];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = r0 + i + 8 * e;
            v[e] *= s.scale;
            if (second) lds[i + 8 * e][j] = v[e];
            else if (r < s.rank && c < width) a.dA[((long long)key * s.rank + r) * s.K + c] = v[e];
        }
        if (!second) continue;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int n = c0 + i + 8 * e, r = r0 + j;
            if (r < s.rank && n < s.N) a.dB[((long long)key * s.N + n) * s.rank + r] = lds[j][i + 8 * e];
        }
        __syncthreads();
    }
}

template <typename T, int RB>
void run_grad(const AdaptGradArgs& a, bool vector, hipStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (vector && a.s.rank % 4 == 0 && (reinterpret_cast<uintptr_t>(a.t) & 15) == 0) {
            constexpr int lds = 2 * (64 * 256 + 64 * 32 * RB * 4) + 3 * 64 * (64 * RB + 16);
            adapt_grad_direct_kernel<RB><<<(a.p.max_chunks + 7) / 8 * 8 * ((a.s.K + 127) / 128 + (a.s.N + 127) / 128), 256, lds, st>>>(a);
            return;
        }
    }
    constexpr int lds = 64 * (128 * (int)sizeof(T) + 16) + (sizeof(T) == 2 ? 3 : 1) * 64 * (32 * RB * (int)sizeof(T) + 16);
    const int grid = a.p.max_chunks * ((a.s.K + 127) / 128 + (a.s.N + 127) / 128);
    if (vector) adapt_grad_kernel<T, RB, true><<<grid, 256, lds, st>>>(a);
    else adapt_grad_kernel<T, RB, false><<<grid, 256, lds, st>>>(a);
}
template <typename T>
hipError_t grad(const AdaptGradArgs& a, hipStream_t st) {
    auto whole = [&](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const bool vector = a.s.K % Vec<T>::N == 0 && a.s.N % Vec<T>::N == 0 && whole(a.x) && whole(a.dy);
    if (a.s.rank <= 32) run_grad<T, 1>(a, vector, st);
    else if (a.s.rank <= 64) run_grad<T, 2>(a, vector, st);
    else run_grad<T, 4>(a, vector, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // four thousand workgroups at most, or an adapter each: most adapters may have nothing to add
    const int tiles = ((a.s.rank + 31) / 32) * ((a.s.K + 31) / 32 + (a.s.N + 31) / 32), groups = std::clamp(4096 / a.s.count, 1, tiles);
    adapt_grad_sum_kernel<<<a.s.count * groups, 256, 0, st>>>(a, groups);
    return hipGetLastError();
}

}  // namespace

AdaptPlan adapt_plan(const AdaptShape& s, int rows, int chunk) {
    AdaptPlan p{};
    auto to256 = [](size_t v) { return (v + 255) & ~size_t(255); };
    const long long M = (long long)s.T * s.B;
    const int groups = std::min(s.B, s.count + 2);
    p.rows = rows; p.chunk = chunk;
    p.max_tiles = (int)(M / rows) + groups;
    p.max_chunks = chunk ? (int)(M / chunk) + groups : 0;
    p.counts = 0;
    p.perm = 256;
    p.first = p.perm + to256((size_t)s.B * 8);
    p.first_chunk = p.first + to256(((size_t)s.count + 3) * 4);
    p.tiles = p.first_chunk + to256(((size_t)s.count + 1) * 4);
    p.chunks = p.tiles + to256((size_t)p.max_tiles * 16);
    p.bytes = p.chunks + to256((size_t)p.max_chunks * 16);
    return p;
}

bool adapt_fits(const AdaptShape& s, const AdaptPlan& p, bool backward) {
    auto up = [](long long v, long long m) { return (v + m - 1) / m; };
    auto launch = [](long long groups, int threads) { return groups <= 0xFFFFFFFFLL / threads; };
    auto project = [&](int n) { return p.rows == 16 ? launch(8 * up(p.max_tiles, 8) * up(n, RN), 64 * RWAVES) : launch(8 * up(p.max_tiles, 8) * up(n, PN), 256); };
    if (!backward) return project(s.N);
    auto tiles = [&](long long r, long long c) { return up(r, 32) * up(c, 32); };
    return project(s.K) && launch(8 * up(p.max_chunks, 8) * (up(s.K, 128) + up(s.N, 128)), 256) &&
           launch(s.count * up(s.rank, 32) * (up(s.K, 32) + up(s.N, 32)), 256) &&
           launch(1 + up(tiles(s.N, s.K) + s.count * (tiles(s.rank, s.K) + tiles(s.N, s.rank)), 8), PLAN_THREADS);
}

hipError_t launch_adapt_plan(const AdaptShape& s, const AdaptPlan& p, const int32_t* ids, char* plan, hipStream_t st) {
    adapt_plan_kernel<<<1, PLAN_THREADS, plan_lds(s.count), st>>>(s, p, ids, plan);
    return hipGetLastError();
}
hipError_t launch_adapt_project(const ProjectArgs& a, DType type, hipStream_t st) { return type == DT_BF16 ? project<bf16_t>(a, st) : project<float>(a, st); }
hipError_t launch_adapt_transpose(const TransposeArgs& a, const AdaptPlan& p, const int32_t* ids, char* plan, DType type, hipStream_t st) {
    auto tiles = [](int r, int c) { return ((r + 31) / 32) * ((c + 31) / 32); };
    const int lds = std::max(plan_lds(a.s.count), 8 * 32 * 33 * 4);
    const int n = tiles(a.s.N, a.s.K) + a.s.count * (tiles(a.s.rank, a.s.K) + tiles(a.s.N, a.s.rank));
    if (type == DT_BF16) adapt_transpose_kernel<bf16_t><<<1 + (n + 7) / 8, PLAN_THREADS, lds, st>>>(a, p, ids, plan);
    else adapt_transpose_kernel<float><<<1 + (n + 7) / 8, PLAN_THREADS, lds, st>>>(a, p, ids, plan);
    return hipGetLastError();
}
hipError_t launch_adapt_grad(const AdaptGradArgs& a, DType type, hipStream_t st) { return type == DT_BF16 ? grad<bf16_t>(a, st) : grad<float>(a, st); }

}  // namespace blstm
