// Log probabilities of given labels, entropy and the k best alternatives of rows of logits, and the logits' gradient.
// With x = scale * z, m = max x, s = sum e^(x - m), w = sum e^(x - m) (x - m) over a row (one pass, running maximum):
//   lse = m + ln s,  log p_i = x_i - lse,  H = -sum p ln p = ln s - w / s      (both terms of H are positive: nothing cancels)
//   d z_i = scale * ( sum_j g_j ([i = t_j] - p_i) - g_H p_i (ln p_i + H) ),    g_j the gradient of a log probability, t_j what it belongs to.
// Sums and statistics are fp32.  The bytes are the logits once, and for the gradient once in and once out; what bounds is the issue of instructions: a
// dozen an entry of a long row (2048 x 32,768 bf16, k = 8: 39 us forward, 20 of bytes; gradient 57, 41 of bytes), 44 an entry and thread in rows of 16, most of them lane exchanges in search of
// the alternatives (1,000,000 x 16 fp32, k = 2: 28 us, 15 of bytes; gradient 24, 20 of bytes).
#include <algorithm>
#include <cfloat>
#include <cooperative_groups.h>
#include "seq_common.cuh"

namespace {

using namespace sfseq;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kMaxTop = SF_MAX_TOP;
constexpr uint32_t kMaxV = 0x7FF00000;              // longest row
// Indexes of entries are ints: those of the chunks that a thread looks at behind a row's end (two turns of four chunks by 512 threads at most) are to fit them too.
static_assert(kMaxV + 14 + 2 * 4 * 512 * 8 <= 0x7FFFFFFFu, "entries in 31 bits");

template <typename T> struct Rows {
    const T* z; size_t ld;
    const uint32_t* n_dev; uint32_t n, V;
    float scale;
    const int32_t* labels;
    float* logprob; float* entropy; float* lse;
    uint32_t k; int32_t* top_ids; float* top_lp;
    sf_dev_state* st;
};

// Running statistics of a part of a row, in units of log2 (w / ln 2).  m = largest entry seen (-FLT_MAX at first, so that nothing is infinite minus infinite).
struct Stat { float m, s, w; };
// brings (s, w) from maximum m to a larger one
__device__ __forceinline__ void stat_raise(Stat& a, float m, float c) {
    const float d = fmaxf((a.m - m) * c, -1e4f), f = ex2(d);       // (from a maximum of -FLT_MAX it would be infinite; 2^-10000 is 0 all the same)
    a.w = (a.w + a.s * d) * f;
    a.s *= f; a.m = m;
}
// N entries more, none above m: masked ones (-infinity) add nothing, a NaN (or an infinity, minus itself) makes s a NaN
template <int N> __device__ __forceinline__ void stat_add(Stat& a, const float (&v)[N], float c) {
    const f2 m2 = dup2(-a.m), c2 = dup2(c);
    f2 s = 0, w = 0;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        float x, y;
        unpack2(mul2(add2(pack2(v[i], v[i + 1]), m2), c2), x, y);
        const f2 e = pack2(ex2(x), ex2(y));
        s = add2(s, e);
        w = fma2(e, pack2(fmaxf(x, -1e4f), fmaxf(y, -1e4f)), w);
    }
    float x, y;
    unpack2(s, x, y); a.s += x + y;
    unpack2(w, x, y); a.w += x + y;
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
// alternative j of a row: entry i of value z, or none (z -infinity)
template <typename T> __device__ __forceinline__ void write_top(const Rows<T>& a, uint32_t row, uint32_t j, float z, uint32_t i, const Answer& r) {
    const bool none = !(z > -INFINITY);
    if (a.top_ids) a.top_ids[(size_t)row * a.k + j] = none ? -1 : (int32_t)i;
    if (a.top_lp) a.top_lp[(size_t)row * a.k + j] = none ? -INFINITY : logprob_of(z, r, a.scale);
}
template <typename T> __device__ __forceinline__ void write_top(const Rows<T>& a, uint32_t row, uint32_t j, uint64_t key, const Answer& r) {
    write_top(a, row, j, key ? value_of(key) : -INFINITY, 0xFFFFFFFFu - (uint32_t)key, r);
}

// Eight entries of a row: chunk c covers entries 8 c - shift .. 8 c - shift + 7 (shift: entries by which the row begins behind a 16-byte
// boundary, so that every chunk inside the row is loaded whole); entries outside the row read as -infinity.
template <typename T> __device__ __forceinline__ uint32_t shift_of(const T* row) { return (uint32_t)((uintptr_t)row & 15u) / sizeof(T); }
template <typename T> struct Chunk {
    union { uint4 q[sizeof(T) / 2]; T e[8]; };
    __device__ __forceinline__ Chunk() {}
    __device__ __forceinline__ void fetch(const T* __restrict__ row, int i0, uint32_t V) {
        if (i0 >= 0 && i0 + 8 <= (int)V) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; i++) q[i] = __ldg(reinterpret_cast<const uint4*>(row + i0) + i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) e[i] = (uint32_t)(i0 + i) < V ? row[i0 + i] : from_f32<T>(-INFINITY);
        }
    }
    __device__ __forceinline__ void open(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = to_f32(e[i]);
    }
};
template <typename T> __device__ __forceinline__ void load_chunk(const T* __restrict__ row, int i0, uint32_t V, float (&v)[8]) {
    Chunk<T> c;
    c.fetch(row, i0, V);
    c.open(v);
}

// ---- rows of up to 2048 entries: L lanes a row, C chunks a lane, the row in registers -----------------------------------------
// Alternatives: one after the other, the largest entry that is left (of equals the lowest index); where a warp has the row and more than four are
// asked, by a bound: the k-th largest of the lanes' own maxima is reached by k entries at least, and the entries that reach it are collected and ranked.
constexpr uint32_t kWarpList = 128;                        // candidates of a warp

template <typename T, int L, int C>
__global__ void __launch_bounds__(kThreads) row_kernel(const Rows<T> a) {
    sf_chain_enter();
    __shared__ uint64_t lists[C > 1 || L == 32 ? kThreads / 32 : 1][kWarpList];
    uint32_t n = a.n;
    if (a.n_dev) n = sf_clamp_rows(*a.n_dev, a.n, a.st);
    const uint32_t lane = threadIdx.x % L;
    const uint64_t row = (uint64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
    const bool live = row < n;
    const T* z = a.z + (live ? row : 0) * a.ld;
    const int first = (int)lane * 8 - (int)shift_of(z);    // the entry that the lane's first chunk begins with
    float v[C][8];
    const float c = a.scale * kLog2e;
    float mine = -INFINITY;
#pragma unroll
    for (int j = 0; j < C; j++) {
        load_chunk(z, first + L * j * 8, live ? a.V : 0, v[j]);
        mine = fmaxf(mine, max_of(v[j]));
    }
    float m = mine;
#pragma unroll
    for (int d = L / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    Stat q = {fmaxf(m, -FLT_MAX), 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < C; j++) stat_add(q, v[j], c);
#pragma unroll
    for (int d = L / 2; d; d >>= 1) { q.s += __shfl_xor_sync(0xFFFFFFFFu, q.s, d); q.w += __shfl_xor_sync(0xFFFFFFFFu, q.w, d); }
    const Answer r = answer_of(q, a.scale);
    if (live && lane == 0) write_row(a, (uint32_t)row, r);
    if (a.k == 0) return;
    if constexpr (L == 32) if (a.k > 4) {
        uint32_t before = 0;
        for (int o = 0; o < 32; o++) { const float x = __shfl_sync(0xFFFFFFFFu, mine, o); before += x > mine || (x == mine && o < (int)lane); }
        const float bound = __shfl_sync(0xFFFFFFFFu, mine, __ffs(__ballot_sync(0xFFFFFFFFu, before == a.k - 1)) - 1);
        uint64_t* list = lists[threadIdx.x / 32];
        uint32_t found = 0;
#pragma unroll
        for (int j = 0; j < C; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const bool in = v[j][e] >= bound && v[j][e] > -INFINITY;
                const uint32_t who = __ballot_sync(0xFFFFFFFFu, in);
                if (who == 0) continue;
                const uint32_t at = found + __popc(who & ((1u << lane) - 1));
                if (in && at < kWarpList) list[at] = key_of(v[j][e], (uint32_t)(first + L * j * 8 + e));
                found += __popc(who);
            }
        __syncwarp();
        if (found <= kWarpList) {
            for (uint32_t i = lane; i < found; i += 32) {
                const uint64_t key = list[i];
                uint32_t rank = 0;
                for (uint32_t o = 0; o < found; o++) rank += list[o] > key;
                if (live && rank < a.k) write_top(a, (uint32_t)row, rank, key, r);
            }
            for (uint32_t t = found + lane; t < a.k; t += 32) if (live) write_top(a, (uint32_t)row, t, -INFINITY, 0u, r);
            return;
        }
    }
    for (uint32_t t = 0; t < a.k; t++) {
        if (t) {
            m = -INFINITY;
#pragma unroll
            for (int j = 0; j < C; j++) m = fmaxf(m, max_of(v[j]));
#pragma unroll
            for (int d = L / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
        }
        uint32_t at = 0xFFFFFFFFu;
#pragma unroll
        for (int j = C - 1; j >= 0; j--)
#pragma unroll
            for (int e = 7; e >= 0; e--) if (v[j][e] == m) at = (uint32_t)(first + L * j * 8 + e);
#pragma unroll
        for (int d = L / 2; d; d >>= 1) at = min(at, __shfl_xor_sync(0xFFFFFFFFu, at, d));
        if (live && lane == 0) write_top(a, (uint32_t)row, t, m, at, r);
#pragma unroll
        for (int j = 0; j < C; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) if ((uint32_t)(first + L * j * 8 + e) == at) v[j][e] = -INFINITY;
    }
}

// ---- longer rows: a block of TH threads a row, or a cluster of CL blocks where rows are few --------------------------------------
// One pass over the row with a running maximum.  Alternatives: every thread knows the largest of its entries; the k-th largest of 64 groups' maxima is a
// bound that at least k entries reach, and only entries of threads that reach it can be among the k best: their chunks alone are read
// again (from L2), what reaches the bound is collected and ranked.  Many equals can overflow the list; then k searches over the row follow.
constexpr uint32_t kList = 1024;                           // candidates that a block collects
constexpr uint32_t kGroups = 64;

template <int TH> struct Shared {
    float m[TH / 32], s[TH / 32], w[TH / 32];
    float group[kGroups];
    float bound;
    uint32_t n_threads, n_list;
    uint16_t thread[TH];
    uint64_t list[kList];
    uint64_t best[kMaxTop], merged[kMaxTop];
    Stat part;
};

template <typename T, int TH, int CL>
__global__ void __launch_bounds__(TH) long_row_kernel(const Rows<T> a) {
    sf_chain_enter();
    __shared__ Shared<TH> sh;
    uint32_t n = a.n;
    if (a.n_dev) n = sf_clamp_rows(*a.n_dev, a.n, a.st);
    const uint64_t row = blockIdx.x / CL;
    if (row >= n) return;                                  // (with all blocks of its cluster)
    const float c = a.scale * kLog2e;
    const uint32_t rank = CL > 1 ? blockIdx.x % CL : 0, tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
    const T* z = a.z + row * a.ld;
    const uint32_t shift = shift_of(z);
    const uint32_t all = (a.V + shift + 7) / 8, per = (all + CL - 1) / CL, c0 = min(all, rank * per), chunks = min(all, c0 + per) - c0;
    const int i_first = (int)(c0 * 8) - (int)shift;
    Stat q = {-FLT_MAX, 0.0f, 0.0f};
    float mine = -INFINITY;
    constexpr int U = 4;                                   // chunks worked on while as many are on their way
    Chunk<T> next[U];
    auto fetch = [&](uint32_t ch) {                        // (chunks behind the block's part are another block's: nothing)
#pragma unroll
        for (int u = 0; u < U; u++) next[u].fetch(z, i_first + (int)(ch + u * TH) * 8, ch + u * TH < chunks ? a.V : 0);
    };
    fetch(tid);
    for (uint32_t ch = tid; ch < chunks; ch += U * TH) {
        float v[U][8];
#pragma unroll
        for (int u = 0; u < U; u++) next[u].open(v[u]);
        if (ch + U * TH < chunks) fetch(ch + U * TH);
        mine = fmaxf(mine, fmaxf(fmaxf(max_of(v[0]), max_of(v[1])), fmaxf(max_of(v[2]), max_of(v[3]))));
        if (mine > q.m) stat_raise(q, mine, c);
#pragma unroll
        for (int u = 0; u < U; u++) stat_add(q, v[u], c);
    }
    constexpr int GL = TH / kGroups;                       // lanes of a group
    float m = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        if (d == GL && lane % GL == 0) sh.group[tid / GL] = m;
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    }
    if (lane == 0) sh.m[warp] = m;
    if (tid == 0) { sh.n_threads = sh.n_list = 0; sh.bound = -INFINITY; }
    if (tid < kMaxTop) sh.best[tid] = 0;
    __syncthreads();
    m = -FLT_MAX;
#pragma unroll
    for (int i = 0; i < TH / 32; i++) m = fmaxf(m, sh.m[i]);
    stat_raise(q, m, c);
#pragma unroll
    for (int d = 16; d; d >>= 1) { q.s += __shfl_xor_sync(0xFFFFFFFFu, q.s, d); q.w += __shfl_xor_sync(0xFFFFFFFFu, q.w, d); }
    if (lane == 0) { sh.s[warp] = q.s; sh.w[warp] = q.w; }
    if (a.k && tid < kGroups) {
        const float g = sh.group[tid];
        uint32_t before = 0;
#pragma unroll 8
        for (uint32_t i = 0; i < kGroups; i++) { const float o = sh.group[i]; before += o > g || (o == g && i < tid); }
        if (before == a.k - 1) sh.bound = g;
    }
    __syncthreads();
    q.s = q.w = 0.0f;
#pragma unroll
    for (int i = 0; i < TH / 32; i++) { q.s += sh.s[i]; q.w += sh.w[i]; }
    if (a.k) {
        const float bound = sh.bound;
        if (mine >= bound && mine > -INFINITY) sh.thread[atomicAdd(&sh.n_threads, 1u)] = (uint16_t)tid;
        __syncthreads();
        const uint32_t each = (chunks + TH - 1) / TH, F = sh.n_threads;
        for (uint32_t p = tid; p < F * each; p += TH) {
            const uint32_t k = sh.thread[p / each] + p % each * TH;
            if (k >= chunks) continue;
            float v[8];
            const int i0 = i_first + (int)k * 8;
            load_chunk(z, i0, a.V, v);
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (v[e] >= bound && v[e] > -INFINITY) { const uint32_t at = atomicAdd(&sh.n_list, 1u); if (at < kList) sh.list[at] = key_of(v[e], (uint32_t)(i0 + e)); }
        }
        __syncthreads();
        const uint32_t found = sh.n_list;
        if (found <= kList) {
            for (uint32_t i = tid; i < found; i += TH) {
                const uint64_t key = sh.list[i];
                uint32_t r = 0;
                for (uint32_t o = 0; o < found; o++) r += sh.list[o] > key;
                if (r < a.k) sh.best[r] = key;
            }
        } else {
            uint64_t last = ~0ull;
            for (uint32_t t = 0; t < a.k; t++) {
                uint64_t best = 0;
                for (uint32_t k = tid; k < chunks; k += TH) {
                    float v[8];
                    const int i0 = i_first + (int)k * 8;
                    load_chunk(z, i0, a.V, v);
#pragma unroll
                    for (int e = 0; e < 8; e++) { const uint64_t key = key_of(v[e], (uint32_t)(i0 + e)); if (key < last && key > best) best = key; }
                }
#pragma unroll
                for (int d = 16; d; d >>= 1) { const uint64_t o = __shfl_xor_sync(0xFFFFFFFFu, best, d); best = o > best ? o : best; }
                if (lane == 0) sh.list[warp] = best;
                __syncthreads();
                best = 0;
                for (uint32_t i = 0; i < TH / 32; i++) best = sh.list[i] > best ? sh.list[i] : best;
                __syncthreads();
                if (tid == 0) sh.best[t] = best;
                last = best;
            }
        }
        __syncthreads();
    }
    uint64_t* top = sh.best;
    if constexpr (CL > 1) {
        namespace cg = cooperative_groups;
        cg::cluster_group cl = cg::this_cluster();
        if (tid == 0) sh.part = {m, q.s, q.w};
        if (tid < kMaxTop) sh.merged[tid] = 0;
        cl.sync();
        if (rank == 0) {
            float top_m = m;
            for (int o = 1; o < CL; o++) top_m = fmaxf(top_m, cl.map_shared_rank(&sh.part, o)->m);
            q.m = m;
            stat_raise(q, top_m, c);
            for (int o = 1; o < CL; o++) { Stat p = *cl.map_shared_rank(&sh.part, o); stat_raise(p, top_m, c); q.s += p.s; q.w += p.w; }
            m = top_m;
            for (uint32_t i = tid; i < CL * a.k; i += TH) sh.list[i] = *cl.map_shared_rank(sh.best + i % a.k, i / a.k);
            __syncthreads();
            for (uint32_t i = tid; i < CL * a.k; i += TH) {                    // the k best of all blocks' k best
                const uint64_t key = sh.list[i];
                uint32_t r = 0;
                for (uint32_t o = 0; o < CL * a.k; o++) r += sh.list[o] > key;
                if (key && r < a.k) sh.merged[r] = key;
            }
            __syncthreads();
            top = sh.merged;
        }
        cl.sync();                                         // (no block leaves while another reads its shared memory)
        if (rank) return;
    }
    q.m = m;
    const Answer r = answer_of(q, a.scale);
    if (tid == 0) write_row(a, (uint32_t)row, r);
    if (tid < a.k) write_top(a, (uint32_t)row, tid, top[tid], r);
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
    uint32_t chunks, groups;                               // chunks of a row; threads that share them, where a thread takes several of one row
    bool few;                                              // threads in 32 bits
    sf_dev_state* st;
};

constexpr float kFar = 1024.0f;                            // from this |lse| on a row's p is worked out from its entries (p would be off by more than 2^-14)

// What a row's gradient takes besides its entries.  With t = log2 p:  d z = -p (sum + ge (t + h)) + what belongs to the label and the alternatives, everything
// times scale.
template <typename T> struct RowBack {
    float lse, ge, h, g, sum;
    uint32_t label;
    __device__ __forceinline__ void load(const Back<T>& a, size_t row) {
        lse = a.lse[row];
        ge = a.d_entropy ? a.d_entropy[row] : 0.0f;
        h = a.d_entropy ? a.entropy[row] : 0.0f;
        label = a.d_logprob ? (uint32_t)a.labels[row] : 0xFFFFFFFFu;
        g = a.d_logprob ? a.d_logprob[row] : 0.0f;
        sum = 0.0f;
        if (a.d_top) for (uint32_t j = 0; j < a.k; j++) if ((uint32_t)a.top_ids[row * a.k + j] < a.V) sum += a.d_top[row * a.k + j] * a.scale;
    }
    __device__ __forceinline__ void ready(const Back<T>& a) {
        if (lse == -INFINITY) lse = 0.0f;                  // (a row with nothing but masked entries: every p is 0)
        ge *= a.scale * kLn2; h *= kLog2e;
        if (label >= a.V) { label = 0xFFFFFFFFu; g = 0.0f; }
        g = __fmul_rn(g, a.scale);                         // (rounded here, so that g taken off and g added cancel)
        sum += g;
    }
    // lse as an fp32 number is off by half a step, up to |lse| 2^-24, and p by as much: nothing is left of ln s in the lse of a row of the type's lowest value
    __device__ __forceinline__ bool far() const { return fabsf(lse) >= kFar && (sum != 0.0f || ge != 0.0f); }
    __device__ __forceinline__ void chunk(const Back<T>& a, size_t row, int i0, const Chunk<T>& in, float (&d)[8]) const {
        const f2 e2 = dup2(kLog2e), l2 = dup2(-lse), s2 = dup2(-sum), g2 = dup2(-ge), h2 = dup2(h);
        float v[8];
        in.open(v);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float x, y;                                    // (the product is rounded before lse is taken off, as lse was, and never fused: with one entry t is exactly 0)
            const f2 t = mul2(add2(pack2(__fmul_rn(v[e], a.scale), __fmul_rn(v[e + 1], a.scale)), l2), e2);
            unpack2(t, x, y);
            const f2 p = pack2(ex2(x), ex2(y));
            f2 q = s2;
            if (ge != 0.0f) q = fma2(g2, add2(pack2(fmaxf(x, -1e4f), fmaxf(y, -1e4f)), h2), s2);
            unpack2(mul2(p, q), d[e], d[e + 1]);
        }
        if (!(lse > -INFINITY)) {                          // (a row with a NaN: its masked entries get 0 all the same)
#pragma unroll
            for (int e = 0; e < 8; e++) if (v[e] == -INFINITY) d[e] = 0.0f;
        }
        if (label - (uint32_t)i0 < 8u) {
#pragma unroll
            for (int e = 0; e < 8; e++) if (label == (uint32_t)(i0 + e)) d[e] = v[e] == -INFINITY ? 0.0f : d[e] + g;
        }
        if (a.d_top) for (uint32_t j = 0; j < a.k; j++) {
            const uint32_t id = (uint32_t)a.top_ids[row * a.k + j];
            if (id - (uint32_t)i0 < 8u && id < a.V) {
                const float t = a.d_top[row * a.k + j] * a.scale;
#pragma unroll
                for (int e = 0; e < 8; e++) if (id == (uint32_t)(i0 + e)) d[e] += t;
            }
        }
    }
};

// The gradient of a row whose lse lies far from zero, by TH threads (a warp or a block): maximum, sum and gradient from the entries themselves, differences from
// the maximum before anything is rounded.
template <typename T, int TH> __device__ __forceinline__ void far_row(const Back<T>& a, size_t row, float* sh) {
    const T* z = a.z + row * a.ld;
    T* dz = a.dz + row * a.ldd;
    const int begin = (int)(threadIdx.x % TH) * 8 - (int)shift_of(z);
    const float c = a.scale * kLog2e;
    auto join = [&](float v, auto both) {                  // over the threads, always in the same order
#pragma unroll
        for (int d = 16; d; d >>= 1) v = both(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
        if constexpr (TH > 32) {
            __syncthreads();
            if (threadIdx.x % 32 == 0) sh[threadIdx.x / 32] = v;
            __syncthreads();
            v = sh[0];
            for (int i = 1; i < TH / 32; i++) v = both(v, sh[i]);
        }
        return v;
    };
    float m = -FLT_MAX, s = 0.0f, v[8];
    for (int i0 = begin; i0 < (int)a.V; i0 += TH * 8) {
        load_chunk(z, i0, a.V, v);
        m = fmaxf(m, max_of(v));
    }
    m = join(m, [](float x, float y) { return fmaxf(x, y); });
    for (int i0 = begin; i0 < (int)a.V; i0 += TH * 8) {
        load_chunk(z, i0, a.V, v);
#pragma unroll
        for (int e = 0; e < 8; e++) s += ex2((v[e] - m) * c);
    }
    s = join(s, [](float x, float y) { return x + y; });
    const float log2_s = log2f(s);
    RowBack<T> r;
    r.load(a, row);
    r.ready(a);
    for (int i0 = begin; i0 < (int)a.V; i0 += TH * 8) {
        load_chunk(z, i0, a.V, v);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const uint32_t i = (uint32_t)(i0 + e);
            const float t = (v[e] - m) * c - log2_s;
            float d = ex2(t) * (-r.sum - r.ge * (fmaxf(t, -1e4f) + r.h));
            if (i == r.label) d += r.g;
            if (a.d_top) for (uint32_t j = 0; j < a.k; j++) if ((uint32_t)a.top_ids[row * a.k + j] == i) d += a.d_top[row * a.k + j] * a.scale;
            if (i < a.V) dz[i] = from_f32<T>(v[e] == -INFINITY ? 0.0f : d);
        }
    }
}

// Those among a thread's row and the block's other threads', one after the other, by the block
template <typename T> __device__ __forceinline__ void far_rows(const Back<T>& a, bool far, uint64_t row) {
    __shared__ float sh[kThreads / 32];
    __shared__ uint32_t rows[kThreads], n_rows;
    if (!__syncthreads_or(far)) return;
    if (threadIdx.x == 0) n_rows = 0;
    __syncthreads();
    if (far) rows[atomicAdd(&n_rows, 1u)] = (uint32_t)row;
    __syncthreads();
    for (uint32_t i = 0; i < n_rows; i++) far_row<T, kThreads>(a, rows[i], sh);
    __syncthreads();
}

// The rows that back_kernel leaves: a row a thread to look at.
template <typename T> __global__ void __launch_bounds__(kThreads) far_rows_kernel(const Back<T> a) {
    sf_chain_enter();
    uint32_t n = a.n;
    if (a.n_dev) n = sf_clamp_rows(*a.n_dev, a.n, a.st);
    for (uint64_t first = blockIdx.x; first < n; first += (uint64_t)gridDim.x * kThreads) {
        const uint64_t row = first + (uint64_t)threadIdx.x * gridDim.x;
        bool far = false;
        if (row < n && fabsf(a.lse[row]) >= kFar) {
            RowBack<T> r;
            r.load(a, row);
            r.ready(a);
            far = r.far();
        }
        far_rows(a, far, row);
    }
}

// A thread takes C chunks, everything they need on its way before the first is worked on.  SAME: of one row, `groups` apart (long rows);
// else the next ones are a whole grid's width further on.  Chunks begin on 16-byte boundaries of the logits' row; where the gradient's row lies on
// the same ones they are stored whole too.  Rows far from zero are left to the end, where the warp or (SAME) the block in which one begins does it, or (FAR false) to
// far_rows_kernel: that is a launch more (3 x 20088 with the forward call: 17.5 us without, 19.7 with it), but of many long rows the registers do not suffice for what such a row
// takes (2048 x 32768 bf16: 99 us, 110 with it in here).
template <typename T, int C, bool SAME, bool FAR>
__global__ void __launch_bounds__(kThreads) back_kernel(const Back<T> a) {
    sf_chain_enter();
    uint32_t n = a.n;
    if (a.n_dev) n = sf_clamp_rows(*a.n_dev, a.n, a.st);
    const uint32_t width = SAME ? a.groups : a.chunks;
    size_t row[C];
    int i0[C];
    bool there[C];                                         // (a thread without a row has no entries: nothing is derived from its place)
    Chunk<T> in[C];
    RowBack<T> r[SAME ? 1 : C];
#pragma unroll
    for (int u = 0; u < C; u++) {
        if (SAME && u) { row[u] = row[0]; i0[u] = i0[0] + u * (int)a.groups * 8; there[u] = there[0] && i0[u] < (int)a.V; }
        else {
            const uint64_t at = ((uint64_t)blockIdx.x + (SAME ? 0 : (uint64_t)u * gridDim.x)) * kThreads + threadIdx.x;
            if (a.few) { row[u] = (uint32_t)at / width; i0[u] = (int)((uint32_t)at % width * 8); }
            else { row[u] = at / width; i0[u] = (int)(at % width * 8); }
            there[u] = row[u] < n;
            if (there[u]) { r[u].load(a, row[u]); i0[u] -= (int)shift_of(a.z + row[u] * a.ld); there[u] = i0[u] < (int)a.V; }
        }
        if (there[u]) in[u].fetch(a.z + row[u] * a.ld, i0[u], a.V);
    }
    bool far[C];                                           // of this thread's rows
#pragma unroll
    for (int u = 0; u < C; u++) {
        far[u] = false;
        if (there[u] && (!SAME || u == 0)) { r[SAME ? 0 : u].ready(a); far[u] = r[SAME ? 0 : u].far(); }
        if (far[SAME ? 0 : u]) there[u] = false;
    }
#pragma unroll
    for (int u = 0; u < C; u++) {
        if (!there[u]) continue;
        float d[8];
        r[SAME ? 0 : u].chunk(a, row[u], i0[u], in[u], d);
        T* dz = a.dz + row[u] * a.ldd;
        if (i0[u] >= 0 && i0[u] + 8 <= (int)a.V && ((uintptr_t)(dz + i0[u]) & 15u) == 0) store_f32<T, 8, true>(dz + i0[u], d);
        else {
#pragma unroll
            for (int e = 0; e < 8; e++) if ((uint32_t)(i0[u] + e) < a.V) dz[i0[u] + e] = from_f32<T>(d[e]);
        }
    }
    // (a row's first chunk begins at entry 0 or in front of it)
    if constexpr (FAR && SAME) far_rows(a, far[0] && i0[0] <= 0, row[0]);
    if constexpr (FAR && !SAME) {
#pragma unroll
        for (int u = 0; u < C; u++)
            for (uint32_t begin = __ballot_sync(0xFFFFFFFFu, far[u] && i0[u] <= 0); begin; begin &= begin - 1)
                far_row<T, 32>(a, (size_t)__shfl_sync(0xFFFFFFFFu, (unsigned long long)row[u], __ffs(begin) - 1), nullptr);
    }
}

template <typename T, int L, int C> int launch_rows(const Rows<T>& a, cudaStream_t st) {
    SF_CUDA(sf_launch_chained(row_kernel<T, L, C>, (uint32_t)(((uint64_t)a.n + kThreads / L - 1) / (kThreads / L)), kThreads, 0, st, a));
    return SF_OK;
}
template <typename T, int TH, int CL> int launch_long(const Rows<T>& a, cudaStream_t st) {
    cudaLaunchConfig_t lc = {};
    lc.gridDim = a.n * CL; lc.blockDim = TH; lc.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {CL, 1, 1};
    lc.attrs = at; lc.numAttrs = CL > 1 ? 2 : 1;
    SF_CUDA(cudaLaunchKernelEx(&lc, long_row_kernel<T, TH, CL>, a));
    return SF_OK;
}

// entries that the chunks of a row have room for: rows that do not begin on 16-byte boundaries may reach into one chunk more
uint32_t room_of(const void* p, size_t ld, int dtype, uint32_t V) {
    return V + (aligned(p, 16) && ld * type_bytes(dtype) % 16 == 0 ? 0 : 16 / type_bytes(dtype) - 1);
}

bool scale_ok(float s) { return s > 0.0f && s <= 1e30f; }      // (a larger one times log2 e or an entry's distance of 1 would be infinite)

}  // namespace

extern "C" int sf_label_logprobs(sf_ctx* ctx, const void* logits, int dtype, const uint32_t* n_dev, uint32_t n, uint32_t V, size_t ld, float scale,
                                 const int32_t* labels, float* logprob_out, float* entropy_out, float* lse_out, uint32_t k, int32_t* top_ids_out,
                                 float* top_logprobs_out, void* stream)
{
    if (!ctx || !type_ok(dtype) || V == 0 || V > kMaxV || ld < V || n > 0x7FFFFFFFu || k > kMaxTop || k > V || !scale_ok(scale)) return SF_ERR_ARG;
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
        const uint32_t room = room_of(logits, ld, dtype, V);
        if (room <= 8) return launch_rows<T, 1, 1>(a, st);
        if (room <= 16) return launch_rows<T, 2, 1>(a, st);
        if (room <= 32) return launch_rows<T, 4, 1>(a, st);
        if (room <= 64) return launch_rows<T, 8, 1>(a, st);
        if (room <= 128) return launch_rows<T, 16, 1>(a, st);
        if (room <= 256) return launch_rows<T, 32, 1>(a, st);
        if (room <= 512) return launch_rows<T, 32, 2>(a, st);
        if (room <= 1024) return launch_rows<T, 32, 4>(a, st);
        // (20,000 rows of 2,000 fp32, k = 2: 66 us by warps, 106 by blocks; twice as long rows no longer fit a warp's registers: 246 and 98)
        if (room <= 2048) return launch_rows<T, 32, 8>(a, st);
        // Longer rows, as measured (16 bits; us):
        //   a cluster of eight blocks a row where all rows' clusters fit the machine at once: 8 x 49152 5.9, by one block 7.0; 12 x 131072 8.7 and 12.6; but 18 x 32768 6.5 and 5.9,
        //   74 x 65536 12.3 and 8.2.  Of 512 threads for the longest: 12 x 250001 9.8, of 256 10.7; but 12 x 65536 9.1 and 7.8
        //   the widest block where every row has an SM to itself: 148 x 65536 8.9 by 512 threads, 10.6 by 256; 148 x 131072 13.6 and 17.2; but 222 x 65536 16.1 and 15.5, 2048 x 131072 161 and 100
        //   256 threads or 128: 296 x 16384 6.0 and 6.9, 148 x 32768 6.2 and 8.0, 1184 x 65536 34.5 and 36.5; but 148 x 12288 5.4 and 4.9, 1184 x 16384 15.4 and 13.2, 4096 x 32768 63 and 57
        const uint32_t sms = (uint32_t)ctx->num_sms;
        if (V > 32768 && (uint64_t)n * 9 <= sms) return V >= 196608 ? launch_long<T, 512, 8>(a, st) : launch_long<T, 256, 8>(a, st);
        if (V > 32768 && n <= sms) return launch_long<T, 512, 1>(a, st);
        if (V > 32768 || (V > 12288 && n <= 2 * sms)) return launch_long<T, 256, 1>(a, st);
        return launch_long<T, 128, 1>(a, st);
    });
}

extern "C" int sf_label_logprobs_backward(sf_ctx* ctx, const void* logits, int dtype, const uint32_t* n_dev, uint32_t n, uint32_t V, size_t ld, float scale,
                                          const int32_t* labels, const float* lse, const float* d_logprob, const float* entropy, const float* d_entropy,
                                          uint32_t k, const int32_t* top_ids, const float* d_top_logprobs, void* d_logits_out, size_t ldd, void* stream)
{
    if (!ctx || !type_ok(dtype) || V == 0 || V > kMaxV || ld < V || ldd < V || n > 0x7FFFFFFFu || k > kMaxTop || k > V || !scale_ok(scale)) return SF_ERR_ARG;
    if (k == 0) d_top_logprobs = nullptr;
    if (n == 0) return SF_OK;
    if (!logits || !lse || !d_logits_out || (d_logprob && !labels) || (d_entropy && !entropy) || (d_top_logprobs && !top_ids)) return SF_ERR_ARG;
    const uint32_t size = type_bytes(dtype);
    if (!aligned(logits, size) || !aligned(d_logits_out, size) || !aligned(n_dev, 4) || !aligned(labels, 4) || !aligned(lse, 4) || !aligned(d_logprob, 4) || !aligned(entropy, 4) ||
        !aligned(d_entropy, 4) || !aligned(top_ids, 4) || !aligned(d_top_logprobs, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        Back<T> a = {(const T*)logits, ld, n_dev, n, V, scale, labels, lse, entropy, d_logprob, d_entropy, k, top_ids, d_top_logprobs, (T*)d_logits_out, ldd, 0, 0, false, ctx->d_state};
        a.chunks = (room_of(logits, ld, dtype, V) + 7) / 8;
        constexpr int C = 4, S = 2;
        const bool lng = a.chunks >= 64, two = !lng && (uint64_t)n * a.chunks >= (uint64_t)ctx->num_sms * 2048 * S;
        a.groups = (a.chunks + C - 1) / C;
        const uint64_t threads = lng ? (uint64_t)n * a.groups : ((uint64_t)n * a.chunks + (two ? S : 1) - 1) / (two ? S : 1);
        const uint64_t blocks = (threads + kThreads - 1) / kThreads;
        if (blocks > 0x7FFFFFFFu) return (int)SF_ERR_ARG;
        a.few = blocks * kThreads * S <= 0xFFFFFFFFu;
        const bool here = !lng || blocks <= (uint64_t)ctx->num_sms * 4;       // far rows too: all blocks are on the machine at once
        auto kern = lng ? (here ? back_kernel<T, C, true, true> : back_kernel<T, C, true, false>) : (two ? back_kernel<T, S, false, true> : back_kernel<T, 1, false, true>);
        SF_CUDA(sf_launch_chained(kern, (uint32_t)blocks, kThreads, 0, (cudaStream_t)stream, a));
        if (!here) SF_CUDA(sf_launch_chained(far_rows_kernel<T>, std::min(n, 2u * (uint32_t)ctx->num_sms), kThreads, 0, (cudaStream_t)stream, a));
        return (int)SF_OK;
    });
}
