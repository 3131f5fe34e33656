// Log probabilities of given labels, entropy and the k best alternatives of rows of logits, and the logits' gradient.
// With x = scale * z, m = max x, s = sum e^(x - m), w = sum e^(x - m) (x - m) over a row (one pass, running maximum):
//   lse = m + ln s,  log p_i = x_i - lse,  H = -sum p ln p = ln s - w / s      (both terms of H are positive: nothing cancels)
//   d z_i = scale * ( sum_j g_j ([i = t_j] - p_i) - g_H p_i (ln p_i + H) ),    g_j the gradient of a log probability, t_j what it belongs to.
// Sums and statistics are fp32.  Bound by HBM (the logits once; the gradient once) where rows are many.
#include <algorithm>
#include <cfloat>
#include <cooperative_groups.h>
#include "seq_common.cuh"

namespace {

using namespace sfseq;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kMaxTop = SF_MAX_TOP;

template <typename T> struct Rows {
    const T* z; size_t ld;
    const uint32_t* n_dev; uint32_t n, V;
    float scale;
    const int32_t* labels;
    float* logprob; float* entropy; float* lse;
    uint32_t k; int32_t* top_ids; float* top_lp;
    sf_dev_state* st;
};

// running statistics of a part of a row, in units of log2: w2 = w / ln 2
struct Stat { float m, s, w; };                       // m = largest z seen (-FLT_MAX at first, so that nothing is infinite minus infinite)
__device__ __forceinline__ Stat stat_none() { return {-FLT_MAX, 0.0f, 0.0f}; }
// brings (s, w) from maximum m to a larger one
__device__ __forceinline__ void stat_raise(Stat& a, float m, float c) {
    const float d = (a.m - m) * c, f = ex2(d);
    a.w = a.s == 0.0f ? 0.0f : (a.w + a.s * d) * f;
    a.s *= f; a.m = m;
}
__device__ __forceinline__ Stat stat_join(Stat a, Stat b, float c) {
    const float m = fmaxf(a.m, b.m);
    stat_raise(a, m, c); stat_raise(b, m, c);
    return {m, a.s + b.s, a.w + b.w};
}
// N values more, cm their maximum; masked ones (-infinity) add nothing, a NaN (or an infinity, minus itself) makes s a NaN
template <int N> __device__ __forceinline__ void stat_add(Stat& a, const float (&v)[N], float cm, float c) {
    if (cm > a.m) stat_raise(a, cm, c);
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float d = (v[i] - a.m) * c, e = ex2(d);
        a.s += e;
        a.w = fmaf(e, fmaxf(d, -1e4f), a.w);
    }
}
template <int N> __device__ __forceinline__ float max_of(const float (&v)[N]) {
    float m = v[0];
#pragma unroll
    for (int i = 1; i < N; i++) m = fmaxf(m, v[i]);
    return m;
}

// What is asked of a row, from its statistics.  A row with nothing but masked entries: lse and log probabilities -infinity, entropy 0.
struct Answer { float m, ln_s, lse, h; };
__device__ __forceinline__ Answer answer_of(const Stat& a, float scale) {
    Answer r;
    r.m = a.m;
    if (a.s == 0.0f) { r.ln_s = 0.0f; r.lse = -INFINITY; r.h = 0.0f; return r; }
    r.ln_s = logf(a.s);
    r.lse = __fadd_rn(__fmul_rn(scale, a.m), r.ln_s);      // (two roundings, as in the gradient: where a row has one entry its p is exactly 1)
    r.h = r.ln_s - kLn2 * (a.w / a.s);
    return r;
}
__device__ __forceinline__ float logprob_of(float z, const Answer& a, float scale) { return z == -INFINITY ? -INFINITY : (z - a.m) * scale - a.ln_s; }

template <typename T> __device__ __forceinline__ void write_row(const Rows<T>& a, uint32_t row, const Answer& r) {
    if (a.lse) a.lse[row] = r.lse;
    if (a.entropy) a.entropy[row] = r.h;
    if (a.logprob) {
        const int32_t y = a.labels[row];
        a.logprob[row] = (uint32_t)y < a.V ? logprob_of(to_f32(a.z[(size_t)row * a.ld + y]), r, a.scale) : 0.0f;
    }
}

// Order of alternatives: larger value first, of equals the lower index; 0 = none (masked entries and NaN are never picked)
__device__ __forceinline__ uint64_t key_of(float z, uint32_t i) {
    if (!(z > -INFINITY)) return 0;
    if (z == 0.0f) z = 0.0f;                               // -0 and +0 are equals
    const uint32_t b = __float_as_uint(z);
    return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (0xFFFFFFFFu - i);
}
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7FFFFFFFu : ~b);
}
template <typename T> __device__ __forceinline__ void write_top(const Rows<T>& a, uint32_t row, uint32_t j, uint64_t key, const Answer& r) {
    if (a.top_ids) a.top_ids[(size_t)row * a.k + j] = key ? (int32_t)(0xFFFFFFFFu - (uint32_t)key) : -1;
    if (a.top_lp) a.top_lp[(size_t)row * a.k + j] = key ? logprob_of(value_of(key), r, a.scale) : -INFINITY;
}

// Eight entries of a row: chunk c covers entries 8 c - shift .. 8 c - shift + 7 (shift: entries by which the row begins behind a 16-byte
// boundary, so that every chunk inside the row is loaded whole); entries outside the row read as -infinity.
template <typename T> __device__ __forceinline__ uint32_t shift_of(const T* row) { return (uint32_t)((uintptr_t)row & 15u) / sizeof(T); }
template <typename T> __device__ __forceinline__ void load_chunk(const T* __restrict__ row, int i0, uint32_t V, float (&v)[8]) {
    if (i0 >= 0 && i0 + 8 <= (int)V) load_f32<T, 8, true>(row + i0, v);
    else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (uint32_t)(i0 + e) < V ? to_f32(row[i0 + e]) : -INFINITY;
    }
}

// ---- rows of up to 1024 entries: L lanes a row, C chunks a lane, the row in registers -----------------------------------------
template <typename T, int L, int C>
__global__ void __launch_bounds__(kThreads) row_kernel(const Rows<T> a) {
    sf_chain_enter();
    uint32_t n = a.n;
    if (a.n_dev) n = sf_clamp_rows(*a.n_dev, a.n, a.st);
    const uint32_t lane = threadIdx.x % L;
    const uint64_t row = (uint64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
    const bool live = row < n;
    const T* z = a.z + (live ? row : 0) * a.ld;
    float v[C][8];
    const float c = a.scale * kLog2e;
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < C; j++) {
        const int i0 = (int)(lane + L * j) * 8;
        if (live && ((uintptr_t)z & 15u) == 0) load_chunk(z, i0, a.V, v[j]);
        else {
#pragma unroll
            for (int e = 0; e < 8; e++) v[j][e] = live && (uint32_t)(i0 + e) < a.V ? to_f32(z[i0 + e]) : -INFINITY;
        }
        m = fmaxf(m, max_of(v[j]));
    }
#pragma unroll
    for (int d = L / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    Stat q = stat_none();
    q.m = fmaxf(q.m, m);
#pragma unroll
    for (int j = 0; j < C; j++) stat_add(q, v[j], -INFINITY, c);
#pragma unroll
    for (int d = L / 2; d; d >>= 1) { q.s += __shfl_xor_sync(0xFFFFFFFFu, q.s, d); q.w += __shfl_xor_sync(0xFFFFFFFFu, q.w, d); }
    const Answer r = answer_of(q, a.scale);
    if (live && lane == 0) write_row(a, (uint32_t)row, r);
    uint64_t last = ~0ull;
    for (uint32_t t = 0; t < a.k; t++) {                   // the best behind the last one picked
        uint64_t best = 0;
#pragma unroll
        for (int j = 0; j < C; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const uint64_t key = key_of(v[j][e], (lane + L * j) * 8 + e);
                if (key < last && key > best) best = key;
            }
#pragma unroll
        for (int d = L / 2; d; d >>= 1) { const uint64_t o = __shfl_xor_sync(0xFFFFFFFFu, best, d); best = o > best ? o : best; }
        if (live && lane == 0) write_top(a, (uint32_t)row, t, best, r);
        last = best;                                       // (none left: 0, behind which there is nothing)
    }
}

// ---- longer rows: a block a row, or a cluster of blocks where rows are few ---------------------------------------------------------
constexpr uint32_t kWide = 512;                            // threads of a block
constexpr uint32_t kList = 1024;                           // candidates for the alternatives that a block collects

__device__ __forceinline__ Stat block_stat(Stat q, float c, Stat* sh) {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const Stat o = {__shfl_xor_sync(0xFFFFFFFFu, q.m, d), __shfl_xor_sync(0xFFFFFFFFu, q.s, d), __shfl_xor_sync(0xFFFFFFFFu, q.w, d)};
        q = stat_join(q, o, c);
    }
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x / 32] = q;
    __syncthreads();
    q = sh[0];
    for (uint32_t i = 1; i < kWide / 32; i++) q = stat_join(q, sh[i], c);
    return q;
}

// Alternatives of the block's part of the row.  Every thread knows the largest of its entries; the k-th largest of those is a bound that
// at least k entries reach, and only entries of threads that reach it can be among the k best: their chunks alone are read again and
// what reaches the bound is collected and ranked.  Many equals can overflow the list; then k searches over the part follow.
template <typename T>
__device__ void block_top(const T* __restrict__ z, uint32_t V, int i_first, uint32_t chunks, float mine, uint32_t k, uint64_t* list, float* tmax, uint32_t* n_list, uint64_t* out) {
    const uint32_t tid = threadIdx.x, lane = tid & 31;
    __syncthreads();
    tmax[tid] = mine;
    if (tid == 0) { n_list[0] = 0; n_list[1] = __float_as_uint(-INFINITY); }
    if (tid < kMaxTop) out[tid] = 0;
    __syncthreads();
    uint32_t before = 0;
    for (uint32_t i = 0; i < kWide; i += 4) {
        const float4 o = *reinterpret_cast<const float4*>(tmax + i);
        before += (o.x > mine || (o.x == mine && i < tid)) + (o.y > mine || (o.y == mine && i + 1 < tid)) + (o.z > mine || (o.z == mine && i + 2 < tid)) + (o.w > mine || (o.w == mine && i + 3 < tid));
    }
    if (before == k - 1) n_list[1] = __float_as_uint(mine);
    __syncthreads();
    const float bound = __uint_as_float(n_list[1]);
    for (uint32_t f = tid / 32; f < kWide; f += kWide / 32) {
        if (!(tmax[f] >= bound && tmax[f] > -INFINITY)) continue;
        for (uint32_t ch = f + lane * kWide; ch < chunks; ch += 32 * kWide) {
            float v[8];
            const int i0 = i_first + (int)ch * 8;
            load_chunk(z, i0, V, v);
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (v[e] >= bound && v[e] > -INFINITY) { const uint32_t at = atomicAdd(n_list, 1u); if (at < kList) list[at] = key_of(v[e], (uint32_t)(i0 + e)); }
        }
    }
    __syncthreads();
    const uint32_t n = n_list[0];
    if (n <= kList) {
        for (uint32_t i = tid; i < n; i += kWide) {
            const uint64_t key = list[i];
            uint32_t rank = 0;
            for (uint32_t j = 0; j < n; j++) rank += list[j] > key;
            if (rank < k) out[rank] = key;
        }
        __syncthreads();
        return;
    }
    uint64_t last = ~0ull;
    for (uint32_t t = 0; t < k; t++) {
        uint64_t best = 0;
        for (uint32_t ch = tid; ch < chunks; ch += kWide) {
            float v[8];
            const int i0 = i_first + (int)ch * 8;
            load_chunk(z, i0, V, v);
#pragma unroll
            for (int e = 0; e < 8; e++) { const uint64_t key = key_of(v[e], (uint32_t)(i0 + e)); if (key < last && key > best) best = key; }
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) { const uint64_t o = __shfl_xor_sync(0xFFFFFFFFu, best, d); best = o > best ? o : best; }
        if (lane == 0) list[tid / 32] = best;
        __syncthreads();
        best = 0;
        for (uint32_t i = 0; i < kWide / 32; i++) best = list[i] > best ? list[i] : best;
        __syncthreads();
        if (tid == 0) out[t] = best;
        last = best;
    }
    __syncthreads();
}

template <typename T, int CL>
__global__ void __launch_bounds__(kWide) long_row_kernel(const Rows<T> a) {
    sf_chain_enter();
    __shared__ Stat sh[kWide / 32];
    __shared__ Stat part;
    __shared__ uint64_t list[kList];
    __shared__ __align__(16) float tmax[kWide];
    __shared__ uint64_t best[kMaxTop];
    __shared__ uint64_t merged[kMaxTop];
    __shared__ uint32_t n_list[2];
    uint32_t n = a.n;
    if (a.n_dev) n = sf_clamp_rows(*a.n_dev, a.n, a.st);
    const float c = a.scale * kLog2e;
    const uint32_t rank = CL > 1 ? blockIdx.x % CL : 0;
    // (every block of a cluster has the same rows, so they all meet at the same barriers)
    for (uint64_t row = blockIdx.x / CL; row < n; row += gridDim.x / CL) {
        const T* z = a.z + row * a.ld;
        const uint32_t shift = shift_of(z);
        const uint32_t all = (a.V + shift + 7) / 8, per = (all + CL - 1) / CL, c0 = min(all, rank * per), chunks = min(all, c0 + per) - c0;
        const int i_first = (int)(c0 * 8) - (int)shift;
        Stat q = stat_none();
        float mine = -INFINITY;
        uint32_t ch = threadIdx.x;
        for (; ch + 3 * kWide < chunks; ch += 4 * kWide) {
            float v[4][8];
#pragma unroll
            for (int u = 0; u < 4; u++) load_chunk(z, i_first + (int)(ch + u * kWide) * 8, a.V, v[u]);
            const float cm = fmaxf(fmaxf(max_of(v[0]), max_of(v[1])), fmaxf(max_of(v[2]), max_of(v[3])));
            mine = fmaxf(mine, cm);
            if (cm > q.m) stat_raise(q, cm, c);
#pragma unroll
            for (int u = 0; u < 4; u++) stat_add(q, v[u], -INFINITY, c);
        }
        for (; ch < chunks; ch += kWide) {
            float v[8];
            load_chunk(z, i_first + (int)ch * 8, a.V, v);
            const float cm = max_of(v);
            mine = fmaxf(mine, cm);
            stat_add(q, v, cm, c);
        }
        q = block_stat(q, c, sh);
        if (a.k) block_top(z, a.V, i_first, chunks, mine, a.k, list, tmax, n_list, best);
        if constexpr (CL > 1) {
            namespace cg = cooperative_groups;
            cg::cluster_group cl = cg::this_cluster();
            if (threadIdx.x == 0) part = q;
            cl.sync();
            if (rank == 0) {
                for (int o = 1; o < CL; o++) q = stat_join(q, *cl.map_shared_rank(&part, o), c);
                if (a.k) {                                 // the k best of all blocks' k best: a key's rank is the number of larger ones
                    if (threadIdx.x < kMaxTop) merged[threadIdx.x] = 0;
                    __syncthreads();
                    for (uint32_t i = threadIdx.x; i < CL * a.k; i += kWide) {
                        const uint64_t key = *cl.map_shared_rank(best + i % a.k, i / a.k);
                        list[i] = key;
                    }
                    __syncthreads();
                    for (uint32_t i = threadIdx.x; i < CL * a.k; i += kWide) {
                        const uint64_t key = list[i];
                        uint32_t r = 0;
                        for (uint32_t j = 0; j < CL * a.k; j++) r += list[j] > key;
                        if (key && r < a.k) merged[r] = key;
                    }
                    __syncthreads();
                }
            }
            cl.sync();                                     // (no block leaves or goes on while another reads its shared memory)
        }
        if (rank == 0) {
            const Answer r = answer_of(q, a.scale);
            if (threadIdx.x == 0) write_row(a, (uint32_t)row, r);
            if (threadIdx.x < a.k) write_top(a, (uint32_t)row, threadIdx.x, CL > 1 ? merged[threadIdx.x] : best[threadIdx.x], r);
        }
        __syncthreads();
    }
}

// ---- gradient ---------------------------------------------------------------------------------------------------------------------
template <typename T> struct Back {
    const T* z; size_t ld;
    const uint32_t* n_dev; uint32_t n, V;
    float scale;
    const int32_t* labels; const float* lse; const float* entropy;
    const float* d_logprob; const float* d_entropy;
    uint32_t k; const int32_t* top_ids; const float* d_top;
    T* dz; size_t ldd;
    uint32_t chunks, groups;                               // chunks of a row, groups of C chunks a thread takes
    sf_dev_state* st;
};

// a thread takes up to C chunks of one row, lanes of a row side by side
template <typename T, int C, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) back_kernel(const Back<T> a) {
    sf_chain_enter();
    uint32_t n = a.n;
    if (a.n_dev) n = sf_clamp_rows(*a.n_dev, a.n, a.st);
    const uint64_t at = (uint64_t)blockIdx.x * kThreads + threadIdx.x, row = at / a.groups;
    const uint32_t g0 = (uint32_t)(at % a.groups);
    if (row >= n) return;
    const T* z = a.z + row * a.ld;
    T* dz = a.dz + row * a.ldd;
    const float lse = a.lse[row], ge = a.d_entropy ? a.d_entropy[row] : 0.0f, h = a.d_entropy ? a.entropy[row] : 0.0f;
    int32_t label = -1;
    float g = 0.0f, sum = 0.0f;
    if (a.d_logprob) { label = a.labels[row]; if ((uint32_t)label < a.V) g = sum = a.d_logprob[row]; else label = -1; }
    if (a.d_top) for (uint32_t j = 0; j < a.k; j++) if ((uint32_t)a.top_ids[row * a.k + j] < a.V) sum += a.d_top[row * a.k + j];
#pragma unroll
    for (int u = 0; u < C; u++) {
        const uint32_t ch = g0 + u * a.groups;
        if (ch >= a.chunks) break;
        const uint32_t i0 = ch * 8;
        float v[8];
        const bool whole = ALIGNED && i0 + 8 <= a.V;
        if (whole) load_f32<T, 8, true>(z + i0, v);
        else {
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = i0 + e < a.V ? to_f32(z[i0 + e]) : -INFINITY;
        }
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float lp = __fsub_rn(__fmul_rn(a.scale, v[e]), lse), p = ex2(lp * kLog2e);
            d[e] = -p * (sum + (ge == 0.0f ? 0.0f : ge * (fmaxf(lp, -1e4f) + h)));
            if (i0 + e == (uint32_t)label) d[e] += g;
        }
        if (a.d_top) for (uint32_t j = 0; j < a.k; j++) {
            const uint32_t id = (uint32_t)a.top_ids[row * a.k + j];
            if (id - i0 < 8u && id < a.V) {
                const float t = a.d_top[row * a.k + j];
#pragma unroll
                for (int e = 0; e < 8; e++) if (id == i0 + e) d[e] += t;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; e++) d[e] = v[e] == -INFINITY ? 0.0f : d[e] * a.scale;
        if (whole) store_f32<T, 8, true>(dz + i0, d);
        else {
#pragma unroll
            for (int e = 0; e < 8; e++) if (i0 + e < a.V) dz[i0 + e] = from_f32<T>(d[e]);
        }
    }
}

template <typename T, int L, int C> int launch_rows(const Rows<T>& a, cudaStream_t st) {
    SF_CUDA(sf_launch_chained(row_kernel<T, L, C>, (uint32_t)(((uint64_t)a.n + kThreads / L - 1) / (kThreads / L)), kThreads, 0, st, a));
    return SF_OK;
}
template <typename T, int CL> int launch_long(const Rows<T>& a, uint32_t most, cudaStream_t st) {
    cudaLaunchConfig_t lc = {};
    lc.gridDim = std::min(a.n, most) * CL; lc.blockDim = kWide; lc.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {CL, 1, 1};
    lc.attrs = at; lc.numAttrs = CL > 1 ? 2 : 1;
    SF_CUDA(cudaLaunchKernelEx(&lc, long_row_kernel<T, CL>, a));
    return SF_OK;
}

bool scale_ok(float s) { return s > 0.0f && s < INFINITY; }

}  // namespace

extern "C" int sf_label_logprobs(sf_ctx* ctx, const void* logits, int dtype, const uint32_t* n_dev, uint32_t n, uint32_t V, size_t ld, float scale,
                                 const int32_t* labels, float* logprob_out, float* entropy_out, float* lse_out, uint32_t k, int32_t* top_ids_out,
                                 float* top_logprobs_out, void* stream)
{
    if (!ctx || !type_ok(dtype) || V == 0 || V > 0x7FFFFFFFu - 64 || ld < V || n > 0x7FFFFFFFu || k > kMaxTop || k > V || !scale_ok(scale)) return SF_ERR_ARG;
    if (k == 0) { top_ids_out = nullptr; top_logprobs_out = nullptr; }
    if (!logprob_out && !entropy_out && !lse_out && !top_ids_out && !top_logprobs_out) return SF_ERR_ARG;
    if (n == 0) return SF_OK;
    if (!logits || (logprob_out && !labels) || (k && !top_ids_out && !top_logprobs_out)) return SF_ERR_ARG;
    if (!aligned(logits, type_bytes(dtype)) || !aligned(n_dev, 4) || !aligned(labels, 4) || !aligned(logprob_out, 4) || !aligned(entropy_out, 4) || !aligned(lse_out, 4) ||
        !aligned(top_ids_out, 4) || !aligned(top_logprobs_out, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    cudaStream_t st = (cudaStream_t)stream;
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const Rows<T> a = {(const T*)logits, ld, n_dev, n, V, scale, labels, logprob_out, entropy_out, lse_out, k, top_ids_out, top_logprobs_out, ctx->d_state};
        if (V <= 8) return launch_rows<T, 1, 1>(a, st);
        if (V <= 16) return launch_rows<T, 2, 1>(a, st);
        if (V <= 32) return launch_rows<T, 4, 1>(a, st);
        if (V <= 64) return launch_rows<T, 8, 1>(a, st);
        if (V <= 128) return launch_rows<T, 16, 1>(a, st);
        if (V <= 256) return launch_rows<T, 32, 1>(a, st);
        if (V <= 512) return launch_rows<T, 32, 2>(a, st);
        if (V <= 1024) return launch_rows<T, 32, 4>(a, st);
        // a cluster of eight blocks a row where the rows alone do not fill the machine and are long enough for eight blocks
        if (n < (uint32_t)ctx->num_sms && V >= 16384) return launch_long<T, 8>(a, n, st);
        return launch_long<T, 1>(a, 0x7FFFFFFFu, st);
    });
}

extern "C" int sf_label_logprobs_backward(sf_ctx* ctx, const void* logits, int dtype, const uint32_t* n_dev, uint32_t n, uint32_t V, size_t ld, float scale,
                                          const int32_t* labels, const float* lse, const float* d_logprob, const float* entropy, const float* d_entropy,
                                          uint32_t k, const int32_t* top_ids, const float* d_top_logprobs, void* d_logits_out, size_t ldd, void* stream)
{
    if (!ctx || !type_ok(dtype) || V == 0 || V > 0x7FFFFFFFu - 64 || ld < V || ldd < V || n > 0x7FFFFFFFu || k > kMaxTop || k > V || !scale_ok(scale)) return SF_ERR_ARG;
    if (k == 0) d_top_logprobs = nullptr;
    if (n == 0) return SF_OK;
    if (!logits || !lse || !d_logits_out || (d_logprob && !labels) || (d_entropy && !entropy) || (d_top_logprobs && !top_ids)) return SF_ERR_ARG;
    const uint32_t size = type_bytes(dtype);
    if (!aligned(logits, size) || !aligned(d_logits_out, size) || !aligned(n_dev, 4) || !aligned(labels, 4) || !aligned(lse, 4) || !aligned(d_logprob, 4) || !aligned(entropy, 4) ||
        !aligned(d_entropy, 4) || !aligned(top_ids, 4) || !aligned(d_top_logprobs, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        Back<T> a = {(const T*)logits, ld, n_dev, n, V, scale, labels, lse, entropy, d_logprob, d_entropy, k, top_ids, d_top_logprobs, (T*)d_logits_out, ldd, (V + 7) / 8, 0, ctx->d_state};
        const bool al = aligned(logits, 16) && aligned(d_logits_out, 16) && (ld * size) % 16 == 0 && (ldd * size) % 16 == 0;
        constexpr int C = 4;
        const bool one = a.chunks < 64;
        a.groups = one ? a.chunks : (a.chunks + C - 1) / C;
        const uint64_t blocks = ((uint64_t)n * a.groups + kThreads - 1) / kThreads;
        if (blocks > 0x7FFFFFFFu) return (int)SF_ERR_ARG;
        auto kern = one ? (al ? back_kernel<T, 1, true> : back_kernel<T, 1, false>) : (al ? back_kernel<T, C, true> : back_kernel<T, C, false>);
        SF_CUDA(sf_launch_chained(kern, (uint32_t)blocks, kThreads, 0, (cudaStream_t)stream, a));
        return (int)SF_OK;
    });
}
