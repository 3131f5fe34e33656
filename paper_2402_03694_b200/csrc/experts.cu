// A slow model made of experts: the gate (which experts a flow goes to and with what weights), the (flow, expert) pairs
// sorted by expert, the rows brought into that order and the experts' rows added back, each with its gradient.
//
// Everything is deterministic: the sort is stable (pairs of one expert keep the order of their flows), sums run in a fixed order.
#include "rows_common.cuh"
#include <algorithm>
#include <type_traits>

namespace {
using namespace sfrow;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kWarps = kThreads / 32;

// ---- gate ------------------------------------------------------------------------------------------------------
// LPR lanes share a row, V scores each (LPR * V >= E): lane l has experts l V .. l V + V - 1 where rows may be read in whole vectors
// (ALIGNED), else l, l + LPR, ... so that a row's lanes read side by side.  Bound: HBM; the scores are read once and stay in registers over
// the k rounds of "largest that is left, lowest index first".  Up to 16 experts a thread has a whole row: with four lanes a
// row the shuffles of the rounds made 1,000,000 x 16, k = 2 take 59 us.
constexpr float kNegInf = -__builtin_huge_valf();

template <int LPR, int V, bool ALIGNED> __device__ __forceinline__ uint32_t expert_of(uint32_t lane, int v) { return ALIGNED ? lane * V + v : v * LPR + lane; }
template <typename T, int LPR, int V, bool ALIGNED>
__device__ __forceinline__ void load_scores(const T* __restrict__ p, uint32_t E, uint32_t first, float (&s)[V]) {
    if (ALIGNED && first + V <= E) {
        if constexpr ((V * sizeof(T)) % 32 == 0) load_sectors<T, V>(p + first, s);
        else load_f32<T, V, (V * sizeof(T)) % 16 == 0>(p + first, s);
    } else {
#pragma unroll
        for (int v = 0; v < V; v++) { const uint32_t e = expert_of<LPR, V, ALIGNED>(first / V, v); s[v] = e < E ? to_f32(p[e]) : kNegInf; }
    }
#pragma unroll
    for (int v = 0; v < V; v++) s[v] = fmaxf(s[v], kNegInf);                      // a NaN is never picked and adds nothing
}
// exp(s - m) with the largest score m at 1 and masked ones at 0; an infinite m (nothing left, or an infinite score) has no difference
__device__ __forceinline__ float near_top(float s, float m, bool finite) {
    return finite ? expf(s - m) : (s == m && s != kNegInf ? 1.0f : 0.0f);
}

template <int LPR> __device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
    for (int o = LPR / 2; o >= 1; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
template <int LPR> __device__ __forceinline__ float max_lanes(float v) {
#pragma unroll
    for (int o = LPR / 2; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

// A lane keeps the picks of rounds j with j % LPR == lane; S of them (k <= S * LPR).
template <typename T, int LPR, int V, int S, int mode, bool ALIGNED>
__global__ void __launch_bounds__(kThreads)
gate_kernel(const T* __restrict__ scores, const uint32_t* __restrict__ n_dev, uint32_t n, uint32_t E, size_t ld, uint32_t k,
            int32_t* __restrict__ ids, float* __restrict__ weights, sf_dev_state* st)
{
    sf_chain_enter();
    const uint32_t rows = n_dev ? sf_clamp_rows(*n_dev, n, st) : n;
    const uint32_t lane = threadIdx.x & (LPR - 1);
    constexpr uint32_t kPer = kThreads / LPR;          // rows of a block at a time
    // (the loop runs the same number of times in every lane of a warp: the shuffles need them all)
    for (uint64_t base = (uint64_t)blockIdx.x * kPer; base < rows; base += (uint64_t)gridDim.x * kPer) {
        const uint64_t row = base + threadIdx.x / LPR;
        const bool live = row < rows;
        float s[V];
        load_scores<T, LPR, V, ALIGNED>(scores + (live ? row : base) * ld, E, lane * V, s);
        float left[V];
#pragma unroll
        for (int v = 0; v < V; v++) left[v] = s[v];
        float best_s[S]; int best_id[S];
        float m = 0.0f, total = 0.0f;
        bool finite = true;
#pragma unroll
        for (int v = 0; v < S; v++) { best_s[v] = kNegInf; best_id[v] = -1; }
        for (uint32_t j = 0; j < k; j++) {
            float b = left[0]; int id = 0x7FFFFFFF;
#pragma unroll
            for (int v = 1; v + 1 < V; v += 2) b = fmaxf(b, fmaxf(left[v], left[v + 1]));
            if (V % 2 == 0) b = fmaxf(b, left[V - 1]);
#pragma unroll
            for (int v = V - 1; v >= 0; v--) if (left[v] == b) id = (int)expert_of<LPR, V, ALIGNED>(lane, v);
#pragma unroll
            for (int o = LPR / 2; o >= 1; o >>= 1) {
                const float ob = __shfl_xor_sync(0xFFFFFFFFu, b, o);
                const int oid = __shfl_xor_sync(0xFFFFFFFFu, id, o);
                if (ob > b || (ob == b && oid < id)) { b = ob; id = oid; }
            }
            if (b == kNegInf) id = -1;
            if (j == 0) { m = b; finite = fabsf(m) < -kNegInf; }
#pragma unroll
            for (int v = 0; v < V; v++) if (id == (int)expert_of<LPR, V, ALIGNED>(lane, v)) left[v] = kNegInf;
#pragma unroll
            for (int v = 0; v < S; v++) if (j == (uint32_t)v * LPR + lane) { best_s[v] = b; best_id[v] = id; }
            if (mode != SF_GATE_SOFTMAX && id >= 0) total += mode == SF_GATE_SHARE ? b : near_top(b, m, finite);
        }
        if (mode == SF_GATE_SOFTMAX) {
            float t = 0.0f;
            if (finite) {
#pragma unroll
                for (int v = 0; v < V; v++) t += near_top(s[v], m, true);
            } else {
#pragma unroll
                for (int v = 0; v < V; v++) t += near_top(s[v], m, false);
            }
            total = sum_lanes<LPR>(t);
        }
        if (live) {
#pragma unroll
            for (int v = 0; v < S; v++) {
                const uint32_t j = v * LPR + lane;
                if (j < k) {
                    const float top = mode == SF_GATE_SHARE ? best_s[v] : near_top(best_s[v], m, finite);
                    ids[row * k + j] = best_id[v];
                    weights[row * k + j] = best_id[v] >= 0 && total > 0.0f ? top / total : 0.0f;
                }
            }
        }
    }
}

// With p the weights' softmax (over all experts, or over the picked ones) and g the weights' gradient at the picked experts:
// d_s = p (g - sum g p); for shares d_s = (g - sum g w) / sum s at the picked experts.  Away from the picked experts that is
// -p sum g p, or nothing (p by a reciprocal, rounded once more than the gate's quotient: 2^-24 of it), so a lane writes its part of the row without looking at the picks, and then the picked ones that are its own,
// whose scores it reads again by their ids: comparing every id with every expert in registers took twice as long (61 us at
// 1,000,000 x 16, k = 2).  P picks are fetched at a time (4 or 8).
template <typename T, int LPR, int V, int mode, int P, bool ALIGNED>
__global__ void __launch_bounds__(kThreads)
gate_backward_kernel(const T* __restrict__ scores, const uint32_t* __restrict__ n_dev, uint32_t n, uint32_t E, size_t ld, uint32_t k,
                     const int32_t* __restrict__ ids, const float* __restrict__ d_weights, T* d_scores, size_t ldd,
                     sf_dev_state* st)
{
    sf_chain_enter();
    const uint32_t rows = n_dev ? sf_clamp_rows(*n_dev, n, st) : n;
    const uint32_t lane = threadIdx.x & (LPR - 1);
    constexpr uint32_t kPer = kThreads / LPR;
    for (uint64_t base = (uint64_t)blockIdx.x * kPer; base < rows; base += (uint64_t)gridDim.x * kPer) {
        const uint64_t row = base + threadIdx.x / LPR;
        const bool live = row < rows;
        const uint64_t at = live ? row : base;
        const T* const x = scores + at * ld;
        uint32_t id[P];
        float g[P], sp[P];                             // of a pick that does not count: -inf and 0
        auto picks = [&](uint32_t j0) {
#pragma unroll
            for (int q = 0; q < P; q++) {
                id[q] = j0 + q < k ? (uint32_t)__ldg(ids + at * k + j0 + q) : 0xFFFFFFFFu;
                g[q] = j0 + q < k ? __ldg(d_weights + at * k + j0 + q) : 0.0f;
            }
#pragma unroll
            for (int q = 0; q < P; q++) {
                sp[q] = id[q] < E ? fmaxf(to_f32(x[id[q]]), kNegInf) : kNegInf;
                if (sp[q] == kNegInf) g[q] = 0.0f;
            }
        };
        float s[V], m = kNegInf;
        picks(0);
        if (mode == SF_GATE_SOFTMAX) {
            load_scores<T, LPR, V, ALIGNED>(x, E, lane * V, s);
#pragma unroll
            for (int v = 0; v < V; v++) m = fmaxf(m, s[v]);
            m = max_lanes<LPR>(m);
        } else if (mode == SF_GATE_SOFTMAX_PICKED) {
            for (uint32_t j0 = 0; j0 < k; j0 += P) {
                if (j0) picks(j0);
#pragma unroll
                for (int q = 0; q < P; q++) m = fmaxf(m, sp[q]);
            }
        }
        const bool finite = fabsf(m) < -kNegInf;
        auto part = [&](float score) { return mode == SF_GATE_SHARE ? (score == kNegInf ? 0.0f : score) : near_top(score, m, finite); };
        float t = 0.0f, dot = 0.0f;
        if (k > P && mode == SF_GATE_SOFTMAX_PICKED) picks(0);
        for (uint32_t j0 = 0; j0 < k; j0 += P) {
            if (j0) picks(j0);
#pragma unroll
            for (int q = 0; q < P; q++) { const float e = part(sp[q]); dot = fmaf(g[q], e, dot); t += e; }
        }
        if (mode == SF_GATE_SHARE) {
            // Shares by division: g - sum g w is then exactly 0 where one pick has the whole sum, and it is divided by a sum that may be small.
            dot = 0.0f;
            if (k > P) picks(0);
            for (uint32_t j0 = 0; j0 < k; j0 += P) {
                if (j0) picks(j0);
#pragma unroll
                for (int q = 0; q < P; q++) if (t > 0.0f) dot = fmaf(g[q], part(sp[q]) / t, dot);
            }
        }
        if (mode == SF_GATE_SOFTMAX) {
            t = 0.0f;
            if (finite) {
#pragma unroll
                for (int v = 0; v < V; v++) { s[v] = near_top(s[v], m, true); t += s[v]; }
            } else {
#pragma unroll
                for (int v = 0; v < V; v++) { s[v] = near_top(s[v], m, false); t += s[v]; }
            }
            t = sum_lanes<LPR>(t);
        }
        const float inv = t > 0.0f ? 1.0f / t : 0.0f;
        if (mode != SF_GATE_SHARE) dot = inv > 0.0f ? dot * inv : 0.0f;
        if (!live) continue;
        float d[V];
#pragma unroll
        for (int v = 0; v < V; v++) d[v] = mode == SF_GATE_SOFTMAX ? s[v] * inv * -dot : 0.0f;
        T* const y = d_scores + row * ldd;
        const uint32_t first = lane * V;
        if (ALIGNED && first + V <= E) {
            if constexpr ((V * sizeof(T)) % 32 == 0) store_sectors<T, V>(y + first, d);
            else store_f32<T, V, (V * sizeof(T)) % 16 == 0>(y + first, d);
        } else {
#pragma unroll
            for (int v = 0; v < V; v++) { const uint32_t e = expert_of<LPR, V, ALIGNED>(lane, v); if (e < E) y[e] = from_f32<T>(d[v]); }
        }
        for (uint32_t j0 = 0; j0 < k; j0 += P) {
            if (k > P) picks(j0);
#pragma unroll
            for (int q = 0; q < P; q++)
                if (id[q] < E && (ALIGNED ? id[q] / V : id[q] % LPR) == lane && sp[q] != kNegInf)
                    y[id[q]] = from_f32<T>(mode == SF_GATE_SHARE ? (t > 0.0f ? (g[q] - dot) / t : 0.0f) : part(sp[q]) * inv * (g[q] - dot));
        }
    }
}

// calls f with the lanes and values per row that fit E
template <typename F> int by_experts(uint32_t E, F f) {
    using std::integral_constant;
    if (E <= 4) return f(integral_constant<int, 1>(), integral_constant<int, 4>());
    if (E <= 8) return f(integral_constant<int, 1>(), integral_constant<int, 8>());
    if (E <= 16) return f(integral_constant<int, 1>(), integral_constant<int, 16>());
    if (E <= 32) return f(integral_constant<int, 2>(), integral_constant<int, 16>());
    if (E <= 64) return f(integral_constant<int, 4>(), integral_constant<int, 16>());
    if (E <= 128) return f(integral_constant<int, 8>(), integral_constant<int, 16>());
    if (E <= 256) return f(integral_constant<int, 16>(), integral_constant<int, 16>());
    return f(integral_constant<int, 32>(), integral_constant<int, 32>());
}

// ... with the weights' mode as a constant: as an argument of the kernel it made the gate 2 to 21 % and its gradient up to 58 % slower beyond 16
// experts (400,000 x 64, k = 2, shares: 30 -> 36 and 35 -> 55 us; 50,000 x 1024, k = 2: 64 -> 69 and 63 -> 100 us), up to there the gate alone 30 %
// (1,000,000 x 16, k = 2: 23 -> 30 us)
template <typename F> int by_mode(int mode, F f) {
    if (mode == SF_GATE_SOFTMAX) return f(std::integral_constant<int, SF_GATE_SOFTMAX>());
    if (mode == SF_GATE_SOFTMAX_PICKED) return f(std::integral_constant<int, SF_GATE_SOFTMAX_PICKED>());
    return f(std::integral_constant<int, SF_GATE_SHARE>());
}

// ---- sort --------------------------------------------------------------------------------------------------------
// The pairs are cut into tiles, one per block, a tile's warps take consecutive pieces of it.  Launch 1 counts each tile's pairs per
// expert; in launch 2 every block adds up the tiles before its own (tiles x E words from L2, all threads at once), turns the
// totals into aligned segment offsets and places its pairs: rank within the warp by match_any, running positions per warp and
// expert in shared memory.  A batch of one tile needs launch 2 alone.  Latency-bound: a warp has kAhead ids on their way.
struct sort_args {
    const int32_t* ids; const uint32_t* n_dev; uint32_t n, k, E, align, capacity, tiles;
    uint32_t* hist;                                       // [tiles][E]
    uint32_t* offsets; uint32_t* counts; int32_t* flow_of_row; int32_t* row_of_pair;
};
constexpr uint32_t kOneTile = 4096;                       // pairs that one block sorts alone
constexpr uint32_t kFewPairs = 1024;                      // up to here 8 warps a block, 32 beyond: fewer to meet at the barriers (4.0 instead of 4.8 us)
constexpr int kAhead = 4;

template <uint32_t WARPS>
__device__ __forceinline__ void sort_piece(const sort_args& a, uint64_t pairs, uint32_t tile, uint32_t warp, uint64_t& lo, uint64_t& hi) {
    const uint64_t per_warp = (pairs + (uint64_t)a.tiles * WARPS * 32 - 1) / ((uint64_t)a.tiles * WARPS * 32) * 32;
    lo = min(pairs, per_warp * (tile * WARPS + warp));
    hi = min(pairs, lo + per_warp);
}

// counts of this block's pairs per warp and expert -> shared memory [WARPS][E]
template <uint32_t WARPS>
__device__ __forceinline__ void sort_count(const sort_args& a, uint64_t pairs, uint32_t* mine) {
    for (uint32_t i = threadIdx.x; i < WARPS * a.E; i += WARPS * 32) mine[i] = 0;
    __syncthreads();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t lo, hi;
    sort_piece<WARPS>(a, pairs, blockIdx.x, warp, lo, hi);
    for (uint64_t i = lo + lane; i < hi; i += 32 * kAhead) {
        uint32_t e[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) e[u] = i + u * 32 < hi ? (uint32_t)__ldg(a.ids + i + u * 32) : 0xFFFFFFFFu;
#pragma unroll
        for (int u = 0; u < kAhead; u++) if (e[u] < a.E) atomicAdd(&mine[warp * a.E + e[u]], 1u);
    }
    __syncthreads();
}

template <uint32_t WARPS>
__global__ void __launch_bounds__(WARPS * 32)
sort_count_kernel(const sort_args a, sf_dev_state* st)
{
    extern __shared__ uint32_t sm[];
    sf_chain_enter();
    const uint64_t pairs = (uint64_t)(a.n_dev ? sf_clamp_rows(*a.n_dev, a.n, st) : a.n) * a.k;
    sort_count<WARPS>(a, pairs, sm);
    for (uint32_t e = threadIdx.x; e < a.E; e += WARPS * 32) {
        uint32_t t = 0;
#pragma unroll 8
        for (uint32_t w = 0; w < WARPS; w++) t += sm[w * a.E + e];
        a.hist[(size_t)blockIdx.x * a.E + e] = t;
    }
}

template <uint32_t WARPS>
__global__ void __launch_bounds__(WARPS * 32)
sort_place_kernel(const sort_args a, sf_dev_state* st)
{
    extern __shared__ uint32_t sm[];
    uint32_t* mine = sm;                                  // [WARPS][E]: counts, then the next position of each warp and expert
    uint32_t* total = sm + WARPS * a.E;                   // [E]: pairs of the whole batch
    uint32_t* before = total + a.E;                       // [E]: pairs in the tiles before this one
    uint32_t* first = before + a.E;                       // [E + 1]: segment offsets
    sf_chain_enter();
    const uint64_t pairs = (uint64_t)(a.n_dev ? sf_clamp_rows(*a.n_dev, a.n, st) : a.n) * a.k;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (uint32_t e = threadIdx.x; e < 2 * a.E; e += WARPS * 32) total[e] = 0;
    sort_count<WARPS>(a, pairs, mine);
    if (a.tiles == 1) {
        for (uint32_t e = threadIdx.x; e < a.E; e += WARPS * 32) {
            uint32_t t = 0;
#pragma unroll 8
            for (uint32_t w = 0; w < WARPS; w++) t += mine[w * a.E + e];
            total[e] = t;
        }
    } else {
        // a thread has one expert and every `rows`-th tile
        const uint32_t rows = max(1u, WARPS * 32 / a.E);
        for (uint32_t e0 = 0; e0 < a.E; e0 += WARPS * 32) {
            const uint32_t e = e0 + threadIdx.x % min(a.E, WARPS * 32), t0 = threadIdx.x / min(a.E, WARPS * 32);
            uint32_t t = 0, b = 0;
            if (e < a.E && t0 < rows) {
                for (uint32_t i0 = t0; i0 < a.tiles; i0 += rows * 8) {
                    uint32_t h[8];
#pragma unroll
                    for (int u = 0; u < 8; u++) h[u] = i0 + u * rows < a.tiles ? __ldcg(a.hist + (size_t)(i0 + u * rows) * a.E + e) : 0u;
#pragma unroll
                    for (int u = 0; u < 8; u++) { t += h[u]; if (i0 + u * rows < blockIdx.x) b += h[u]; }
                }
                if (t) atomicAdd(&total[e], t);
                if (b) atomicAdd(&before[e], b);
            }
        }
    }
    __syncthreads();
    if (warp == 0) {                                      // exclusive sum of the aligned segment sizes
        uint32_t run = 0;
        for (uint32_t e0 = 0; e0 < a.E; e0 += 32) {
            const uint32_t e = e0 + lane;
            const uint32_t size = e < a.E ? (total[e] + a.align - 1) / a.align * a.align : 0;
            uint32_t s = size;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, s, o); if (lane >= (uint32_t)o) s += u; }
            if (e < a.E) first[e] = run + s - size;
            run += __shfl_sync(0xFFFFFFFFu, s, 31);
        }
        if (lane == 0) first[a.E] = run;
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.E; e += WARPS * 32) {
        uint32_t run = first[e] + before[e];
        for (uint32_t w = 0; w < WARPS; w++) { const uint32_t c = mine[w * a.E + e]; mine[w * a.E + e] = run; run += c; }
    }
    if (blockIdx.x == 0) {
        for (uint32_t e = threadIdx.x; e <= a.E; e += WARPS * 32) {
            a.offsets[e] = min(first[e], a.capacity);
            if (e < a.E) {
                a.counts[e] = min(total[e], a.capacity - min(first[e], a.capacity));
                if (total[e] && first[e] + total[e] > a.capacity) sf_dev_set_error(st, SF_ERR_CAPACITY);
            }
        }
    }
    // rows that only fill a segment up to its aligned end
    for (uint32_t e = blockIdx.x * WARPS + warp; e < a.E; e += gridDim.x * WARPS)
        for (uint32_t r = first[e] + total[e] + lane; r < min(first[e + 1], a.capacity); r += 32) a.flow_of_row[r] = -1;
    __syncthreads();
    uint64_t lo, hi;
    sort_piece<WARPS>(a, pairs, blockIdx.x, warp, lo, hi);
    uint32_t* next = mine + warp * a.E;
    for (uint64_t i0 = lo; i0 < hi; i0 += 32 * kAhead) {
        uint32_t id[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) { const uint64_t i = i0 + u * 32 + lane; id[u] = i < hi ? (uint32_t)__ldg(a.ids + i) : 0xFFFFFFFFu; }
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            if (i0 + u * 32 >= hi) break;                 // (the same in all lanes)
            const uint64_t i = i0 + u * 32 + lane;
            const uint32_t e = id[u];
            const bool real = e < a.E;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, real ? e : 0xFFFFFFFFu);
            uint32_t row = 0xFFFFFFFFu;
            if (real) row = next[e] + __popc(same & ((1u << lane) - 1u));
            __syncwarp();
            if (real && (same >> lane) == 1u) next[e] = row + 1;      // the last lane of its expert
            __syncwarp();
            const bool kept = real && row < a.capacity;
            if (i < hi) a.row_of_pair[i] = kept ? (int32_t)row : -1;
            if (kept) a.flow_of_row[row] = (int32_t)((uint32_t)i / a.k);
        }
    }
}

// Tiles of at least 1024 pairs, at most one per SM and at most 65,536 counts in all (every block reads them).
uint32_t sort_tiles(const sf_ctx* ctx, uint32_t n, uint32_t k, uint32_t E) {
    const uint64_t pairs = (uint64_t)n * k;
    if (pairs <= kOneTile) return 1;
    return (uint32_t)std::min<uint64_t>({(uint64_t)ctx->num_sms, (pairs + 1023) / 1024, 65536 / E});
}
template <uint32_t WARPS> int launch_sort(const sf_ctx* ctx, const sort_args& a, cudaStream_t st) {
    sf_dev_state* const state = ctx->d_state;
    static bool set_dev[64] = {};                         // the shared-memory opt-in (a counter per warp and expert) is per device
    bool& set = set_dev[ctx->device & 63];
    if (!set) {
        constexpr int most = (WARPS + 3) * SF_MAX_EXPERTS * 4 + 4;
        SF_CUDA(cudaFuncSetAttribute(sort_count_kernel<WARPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
        SF_CUDA(cudaFuncSetAttribute(sort_place_kernel<WARPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
        set = true;
    }
    if (a.tiles > 1) SF_CUDA(sf_launch_chained(sort_count_kernel<WARPS>, a.tiles, WARPS * 32, WARPS * a.E * 4, st, a, state));
    SF_CUDA(sf_launch_chained(sort_place_kernel<WARPS>, a.tiles, WARPS * 32, (WARPS * a.E + 3 * a.E + 1) * 4, st, a, state));
    return SF_OK;
}

// ---- rows into the experts' order and back -------------------------------------------------------------------------------
// A group of lanes (a power of two, up to the whole block where flows are few) shares a flow.  Elements move in words of 16 bytes where
// bases, pitches and widths allow, else of 4 bytes, else one by one.  Bound: HBM.

// Every row is read once and written k times; U words a lane of F flows on their way (F > 1: a row has at most U words a lane; 325,401 rows of 17
// fp16 values, k = 2: dispatch and gradient 164 us with one flow, 79 with four).
template <typename Q, int U, int F>
__global__ void __launch_bounds__(kThreads)
gather_kernel(const Q* __restrict__ x, const uint32_t* __restrict__ n_dev, uint32_t n, uint32_t units, size_t ldx, uint32_t k,
              const int32_t* __restrict__ row_of_pair, uint32_t E, const uint32_t* __restrict__ offsets, const uint32_t* __restrict__ counts,
              uint32_t capacity, Q* __restrict__ rows, size_t ldr, uint32_t lanes, uint32_t flow_blocks, uint32_t fill_blocks, sf_dev_state* st)
{
    sf_chain_enter();
    if (blockIdx.x >= flow_blocks) {                      // the rows that only fill a segment: zeros, fill_blocks blocks an expert
        const uint32_t e = (blockIdx.x - flow_blocks) / fill_blocks, part = (blockIdx.x - flow_blocks) % fill_blocks;
        const uint32_t lo = min(offsets[e] + counts[e], capacity), hi = min(offsets[e + 1], capacity);
        const uint64_t all = lo < hi ? (uint64_t)(hi - lo) * units : 0;
        for (uint64_t i = part * kThreads + threadIdx.x; i < all; i += fill_blocks * kThreads) {
            const uint32_t r = (uint32_t)(i / units), c = (uint32_t)(i - (uint64_t)r * units);
            rows[(size_t)(lo + r) * ldr + c] = Q{};
        }
        return;
    }
    const uint32_t flows = n_dev ? sf_clamp_rows(*n_dev, n, st) : n;
    const uint32_t per = kThreads / lanes, lane = threadIdx.x & (lanes - 1);
    if constexpr (F > 1) {
        const uint64_t hop = (uint64_t)flow_blocks * per;
        for (uint64_t f0 = (uint64_t)blockIdx.x * per + threadIdx.x / lanes; f0 < flows; f0 += hop * F) {
            Q q[F][U];
#pragma unroll
            for (int i = 0; i < F; i++)
#pragma unroll
                for (int u = 0; u < U; u++) if (f0 + i * hop < flows && lane + u * lanes < units) q[i][u] = __ldg(x + (f0 + i * hop) * ldx + lane + u * lanes);
            for (uint32_t j = 0; j < k; j++) {
                uint32_t r[F];
#pragma unroll
                for (int i = 0; i < F; i++) r[i] = f0 + i * hop < flows ? (uint32_t)__ldg(row_of_pair + (f0 + i * hop) * k + j) : 0xFFFFFFFFu;
#pragma unroll
                for (int i = 0; i < F; i++)
                    if (r[i] < capacity) {
#pragma unroll
                        for (int u = 0; u < U; u++) if (lane + u * lanes < units) rows[(size_t)r[i] * ldr + lane + u * lanes] = q[i][u];
                    }
            }
        }
        return;
    }
    for (uint64_t f = (uint64_t)blockIdx.x * per + threadIdx.x / lanes; f < flows; f += (uint64_t)flow_blocks * per) {
        const Q* src = x + f * ldx;
        for (uint32_t c = lane; c < units; c += U * lanes) {
            Q q[U];
#pragma unroll
            for (int u = 0; u < U; u++) if (c + u * lanes < units) q[u] = __ldg(src + c + u * lanes);
            for (uint32_t j = 0; j < k; j++) {
                const uint32_t r = (uint32_t)__ldg(row_of_pair + f * k + j);
                if (r < capacity) {
                    Q* dst = rows + (size_t)r * ldr;
#pragma unroll
                    for (int u = 0; u < U; u++) if (c + u * lanes < units) dst[c + u * lanes] = q[u];
                }
            }
        }
    }
}

// y[f] = sum_j w[f][j] rows[row_of_pair[f][j]], j ascending, in fp32, rounded once.  A lane has U words of V elements of a row on their
// way, four rows at a time.
template <typename T, int V, int U>
__global__ void __launch_bounds__(kThreads)
combine_kernel(const T* __restrict__ rows, uint32_t capacity, uint32_t D, size_t ldr, const int32_t* __restrict__ row_of_pair,
               const float* __restrict__ weights, const uint32_t* __restrict__ n_dev, uint32_t n, uint32_t k, T* __restrict__ y, size_t ldy,
               uint32_t lanes, sf_dev_state* st)
{
    sf_chain_enter();
    const uint32_t flows = n_dev ? sf_clamp_rows(*n_dev, n, st) : n;
    const uint32_t per = kThreads / lanes, lane = threadIdx.x & (lanes - 1);
    for (uint64_t f = (uint64_t)blockIdx.x * per + threadIdx.x / lanes; f < flows; f += (uint64_t)gridDim.x * per) {
        for (uint32_t c = lane * V; c < D; c += lanes * V * U) {
            float acc[U][V];
#pragma unroll
            for (int u = 0; u < U; u++)
#pragma unroll
                for (int v = 0; v < V; v++) acc[u][v] = 0.0f;
#pragma unroll (V * U > 16 ? 2 : 4)
            for (uint32_t j = 0; j < k; j++) {
                const uint32_t r = (uint32_t)__ldg(row_of_pair + f * k + j);
                if (r < capacity) {
                    const float w = weights ? __ldg(weights + f * k + j) : 1.0f;
                    float x[U][V];
#pragma unroll
                    for (int u = 0; u < U; u++) if (u == 0 || c + u * lanes * V < D) load_word<T, V>(rows + (size_t)r * ldr + c + u * lanes * V, x[u]);
#pragma unroll
                    for (int u = 0; u < U; u++)
                        if (u == 0 || c + u * lanes * V < D) {
#pragma unroll
                            for (int v = 0; v < V; v++) acc[u][v] = fmaf(w, x[u][v], acc[u][v]);
                        }
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) if (u == 0 || c + u * lanes * V < D) store_word<T, V>(y + f * ldy + c + u * lanes * V, acc[u]);
        }
    }
}

// The same for rows of at most U words a lane: four flows at a time.
template <typename T, int V, int U>
__global__ void __launch_bounds__(kThreads)
combine_narrow_kernel(const T* __restrict__ rows, uint32_t capacity, uint32_t D, size_t ldr, const int32_t* __restrict__ row_of_pair,
                      const float* __restrict__ weights, const uint32_t* __restrict__ n_dev, uint32_t n, uint32_t k, T* __restrict__ y, size_t ldy,
                      uint32_t lanes, sf_dev_state* st)
{
    constexpr int F = 4;
    sf_chain_enter();
    const uint32_t flows = n_dev ? sf_clamp_rows(*n_dev, n, st) : n;
    const uint32_t per = kThreads / lanes, lane = threadIdx.x & (lanes - 1);
    const uint64_t hop = (uint64_t)gridDim.x * per;
    for (uint64_t f0 = (uint64_t)blockIdx.x * per + threadIdx.x / lanes; f0 < flows; f0 += hop * F) {
        float acc[F][U][V] = {};
#pragma unroll (U == 1 ? 2 : 1)
        for (uint32_t j = 0; j < k; j++) {
            uint32_t r[F];
            float w[F], x[F][U][V];
#pragma unroll
            for (int i = 0; i < F; i++) {
                const bool have = f0 + i * hop < flows;
                r[i] = have ? (uint32_t)__ldg(row_of_pair + (f0 + i * hop) * k + j) : 0xFFFFFFFFu;
                w[i] = have && weights ? __ldg(weights + (f0 + i * hop) * k + j) : 1.0f;
            }
#pragma unroll
            for (int i = 0; i < F; i++)
#pragma unroll
                for (int u = 0; u < U; u++) if (r[i] < capacity && (lane + u * lanes) * V < D) load_word<T, V>(rows + (size_t)r[i] * ldr + (lane + u * lanes) * V, x[i][u]);
#pragma unroll
            for (int i = 0; i < F; i++)
#pragma unroll
                for (int u = 0; u < U; u++)
                    if (r[i] < capacity && (lane + u * lanes) * V < D) {
#pragma unroll
                        for (int v = 0; v < V; v++) acc[i][u][v] = fmaf(w[i], x[i][u][v], acc[i][u][v]);
                    }
        }
#pragma unroll
        for (int i = 0; i < F; i++)
#pragma unroll
            for (int u = 0; u < U; u++) if (f0 + i * hop < flows && (lane + u * lanes) * V < D) store_word<T, V>(y + (f0 + i * hop) * ldy + (lane + u * lanes) * V, acc[i][u]);
    }
}

// the rows that only fill a segment: zeros, by the blocks behind the flows' ones, fill_blocks of them an expert
template <typename T, int V>
__device__ __forceinline__ void fill_rows(uint32_t D, uint32_t E, const uint32_t* __restrict__ offsets, const uint32_t* __restrict__ counts, uint32_t capacity,
                                          T* __restrict__ out, size_t ld, uint32_t flow_blocks, uint32_t fill_blocks)
{
    const uint32_t e = (blockIdx.x - flow_blocks) / fill_blocks, part = (blockIdx.x - flow_blocks) % fill_blocks;
    const uint32_t lo = min(offsets[e] + counts[e], capacity), hi = min(offsets[e + 1], capacity), units = D / V;
    const uint64_t all = e < E && lo < hi ? (uint64_t)(hi - lo) * units : 0;
    const float zero[V] = {};
    for (uint64_t i = part * kThreads + threadIdx.x; i < all; i += fill_blocks * kThreads) {
        const uint32_t r = (uint32_t)(i / units), c = (uint32_t)(i - (uint64_t)r * units);
        store_word<T, V>(out + (size_t)(lo + r) * ld + (size_t)c * V, zero);
    }
}

// d_rows[row_of_pair[f][j]] = w[f][j] dy[f], d_w[f][j] = <dy[f], rows[row_of_pair[f][j]]>; J pairs of a flow at a time, U words of V elements.
// A flow's dot products are summed over its lanes in a fixed tree (over the block's warps through shared memory).
template <typename T, int V, int U, int J>
__global__ void __launch_bounds__(kThreads)
combine_backward_kernel(const T* __restrict__ dy, size_t ldy, const T* __restrict__ rows, uint32_t capacity, uint32_t D, size_t ldr,
                        const int32_t* __restrict__ row_of_pair, const float* __restrict__ weights, const uint32_t* __restrict__ n_dev,
                        uint32_t n, uint32_t k, uint32_t E, const uint32_t* __restrict__ offsets, const uint32_t* __restrict__ counts,
                        T* __restrict__ d_rows, size_t ldd, float* __restrict__ d_weights, uint32_t lanes, uint32_t flow_blocks, uint32_t fill_blocks, sf_dev_state* st)
{
    __shared__ float part[kWarps][J];
    sf_chain_enter();
    if (blockIdx.x >= flow_blocks) { fill_rows<T, V>(D, E, offsets, counts, capacity, d_rows, ldd, flow_blocks, fill_blocks); return; }
    const uint32_t flows = n_dev ? sf_clamp_rows(*n_dev, n, st) : n;
    const uint32_t per = kThreads / lanes, lane = threadIdx.x & (lanes - 1), warp = threadIdx.x >> 5;
    for (uint64_t base = (uint64_t)blockIdx.x * per; base < flows; base += (uint64_t)flow_blocks * per) {
        const uint64_t f = base + threadIdx.x / lanes;
        const bool live = f < flows;                      // (the sums over lanes below need whole warps and blocks)
        for (uint32_t j0 = 0; j0 < k; j0 += J) {
            uint32_t r[J], any = 0xFFFFFFFFu;             // a pair without a row reads that of another (no branch among the loads)
            bool real[J];
            float w[J], dot[J];
#pragma unroll
            for (int j = 0; j < J; j++) {
                const bool have = live && j0 + j < k;
                r[j] = have ? (uint32_t)__ldg(row_of_pair + f * k + j0 + j) : 0xFFFFFFFFu;
                w[j] = have && weights ? __ldg(weights + f * k + j0 + j) : 1.0f;
                real[j] = r[j] < capacity;
                if (real[j]) any = r[j];
                dot[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < J; j++) if (!real[j]) r[j] = any;
            if (any != 0xFFFFFFFFu) for (uint32_t c0 = lane * V; c0 < D; c0 += lanes * V * U) {
                float g[U][V];
#pragma unroll
                for (int u = 0; u < U; u++) if (u == 0 || c0 + u * lanes * V < D) load_word<T, V>(dy + f * ldy + c0 + u * lanes * V, g[u]);
                if (d_weights) {
                    float x[J][U][V];
#pragma unroll
                    for (int j = 0; j < J; j++)
#pragma unroll
                        for (int u = 0; u < U; u++)
                            if (u == 0 || c0 + u * lanes * V < D) load_word<T, V>(rows + (size_t)r[j] * ldr + c0 + u * lanes * V, x[j][u]);
#pragma unroll
                    for (int j = 0; j < J; j++)
#pragma unroll
                        for (int u = 0; u < U; u++)
                            if (u == 0 || c0 + u * lanes * V < D) {
#pragma unroll
                                for (int v = 0; v < V; v++) dot[j] = fmaf(g[u][v], x[j][u][v], dot[j]);
                            }
                }
                if (d_rows) {
#pragma unroll
                    for (int j = 0; j < J; j++)
#pragma unroll
                        for (int u = 0; u < U; u++)
                            if (real[j] && (u == 0 || c0 + u * lanes * V < D)) {
                                float d[V];
#pragma unroll
                                for (int v = 0; v < V; v++) d[v] = w[j] * g[u][v];
                                store_word<T, V>(d_rows + (size_t)r[j] * ldd + c0 + u * lanes * V, d);
                            }
                }
            }
            if (!d_weights) continue;
#pragma unroll
            for (int j = 0; j < J; j++) if (!real[j]) dot[j] = 0.0f;
            const uint32_t in_warp = min(lanes, 32u);
#pragma unroll
            for (int j = 0; j < J; j++)
                for (uint32_t o = in_warp / 2; o >= 1; o >>= 1) dot[j] += __shfl_xor_sync(0xFFFFFFFFu, dot[j], o);
            if (lanes > 32) {
                if ((threadIdx.x & 31) == 0) {
#pragma unroll
                    for (int j = 0; j < J; j++) part[warp][j] = dot[j];
                }
                __syncthreads();
                if (lane == 0) {
#pragma unroll
                    for (int j = 0; j < J; j++) { dot[j] = 0.0f; for (uint32_t q = 0; q < lanes / 32; q++) dot[j] += part[warp + q][j]; }
                }
                __syncthreads();
            }
            if (live && lane == 0) {
#pragma unroll
                for (int j = 0; j < J; j++) if (j0 + j < k) d_weights[f * k + j0 + j] = dot[j];
            }
        }
    }
}

// The same for rows of at most U words a lane and up to a warp a flow: four flows at a time, their rows of dy in registers over the pairs.
template <typename T, int V, int U>
__global__ void __launch_bounds__(kThreads)
combine_backward_narrow_kernel(const T* __restrict__ dy, size_t ldy, const T* __restrict__ rows, uint32_t capacity, uint32_t D, size_t ldr,
                               const int32_t* __restrict__ row_of_pair, const float* __restrict__ weights, const uint32_t* __restrict__ n_dev,
                               uint32_t n, uint32_t k, uint32_t E, const uint32_t* __restrict__ offsets, const uint32_t* __restrict__ counts,
                               T* __restrict__ d_rows, size_t ldd, float* __restrict__ d_weights, uint32_t lanes, uint32_t flow_blocks, uint32_t fill_blocks, sf_dev_state* st)
{
    constexpr int F = 4;
    sf_chain_enter();
    if (blockIdx.x >= flow_blocks) { fill_rows<T, V>(D, E, offsets, counts, capacity, d_rows, ldd, flow_blocks, fill_blocks); return; }
    const uint32_t flows = n_dev ? sf_clamp_rows(*n_dev, n, st) : n;
    const uint32_t per = kThreads / lanes, lane = threadIdx.x & (lanes - 1);
    const uint64_t hop = (uint64_t)flow_blocks * per;
    for (uint64_t base = (uint64_t)blockIdx.x * per; base < flows; base += hop * F) {
        const uint64_t f0 = base + threadIdx.x / lanes;       // (the sums over lanes below need whole warps)
        float g[F][U][V];
#pragma unroll
        for (int i = 0; i < F; i++)
#pragma unroll
            for (int u = 0; u < U; u++) if (f0 + i * hop < flows && (lane + u * lanes) * V < D) load_word<T, V>(dy + (f0 + i * hop) * ldy + (lane + u * lanes) * V, g[i][u]);
        for (uint32_t j = 0; j < k; j++) {
            uint32_t r[F];
            float w[F], dot[F];
#pragma unroll
            for (int i = 0; i < F; i++) {
                const bool have = f0 + i * hop < flows;
                r[i] = have ? (uint32_t)__ldg(row_of_pair + (f0 + i * hop) * k + j) : 0xFFFFFFFFu;
                w[i] = have && weights ? __ldg(weights + (f0 + i * hop) * k + j) : 1.0f;
                dot[i] = 0.0f;
            }
            if (d_weights) {
                float x[F][U][V];
#pragma unroll
                for (int i = 0; i < F; i++)
#pragma unroll
                    for (int u = 0; u < U; u++) if (r[i] < capacity && (lane + u * lanes) * V < D) load_word<T, V>(rows + (size_t)r[i] * ldr + (lane + u * lanes) * V, x[i][u]);
#pragma unroll
                for (int i = 0; i < F; i++)
#pragma unroll
                    for (int u = 0; u < U; u++)
                        if (r[i] < capacity && (lane + u * lanes) * V < D) {
#pragma unroll
                            for (int v = 0; v < V; v++) dot[i] = fmaf(g[i][u][v], x[i][u][v], dot[i]);
                        }
            }
            if (d_rows) {
#pragma unroll
                for (int i = 0; i < F; i++)
#pragma unroll
                    for (int u = 0; u < U; u++)
                        if (r[i] < capacity && (lane + u * lanes) * V < D) {
                            float d[V];
#pragma unroll
                            for (int v = 0; v < V; v++) d[v] = w[i] * g[i][u][v];
                            store_word<T, V>(d_rows + (size_t)r[i] * ldd + (lane + u * lanes) * V, d);
                        }
            }
            if (d_weights) {
#pragma unroll
                for (int i = 0; i < F; i++) {
                    for (uint32_t o = lanes / 2; o >= 1; o >>= 1) dot[i] += __shfl_xor_sync(0xFFFFFFFFu, dot[i], o);
                    if (f0 + i * hop < flows && lane == 0) d_weights[(f0 + i * hop) * k + j] = dot[i];
                }
            }
        }
    }
}

// Lanes that share a flow whose row has `units` words: up to a warp, and more while the flows alone would not fill the machine (5 flows of
// 2489 values over 8 experts: 167 us with a warp a flow).
uint32_t lanes_for(const sf_ctx* ctx, uint32_t units, uint32_t n) {
    uint32_t l = 1;
    while (l < 32 && l < units) l *= 2;
    while (l >= 32 && l < kThreads && l < units && (uint64_t)n * l < (uint64_t)ctx->num_sms * 1024) l *= 2;
    return l;
}
uint32_t flow_grid(const sf_ctx* ctx, uint32_t n, uint32_t lanes) {
    const uint32_t per = kThreads / lanes;
    return std::min<uint32_t>((n + per - 1) / per, (uint32_t)ctx->num_sms * 8);
}
// Do the flows give every thread of a full grid `times` of them?  Several flows at a time pay from about one and a half a thread on (combine, us: 60,000 x 64
// bf16, k = 2: 10.1 with, 11.0 without; 30,000 x 64: 8.7 and 7.1): with fewer the lanes only wait for flows that are not there.
constexpr double kSome = 1.5;
bool many_flows(const sf_ctx* ctx, uint32_t n, uint32_t lanes, double times) { return (double)n * lanes >= (double)ctx->num_sms * 8 * kThreads * times; }
// the largest word (16, 4 or sizeof(element) bytes) in which rows at p with pitch ld can be moved
uint32_t word_of(const void* p, size_t ld, uint32_t size) {
    const size_t at = (uintptr_t)p | (ld * size);
    return at % 16 == 0 ? 16 : (at % 4 == 0 ? 4 : size);
}
// calls f with the elements per word and words per lane
template <typename T, typename F> int by_word(uint32_t bytes, F f) {
    using std::integral_constant;
    if (bytes == 16) return f(integral_constant<int, 16 / sizeof(T)>());
    if constexpr (sizeof(T) == 2) { if (bytes == 4) return f(integral_constant<int, 2>()); }
    return f(integral_constant<int, 1>());
}
// blocks that zero an expert's filling rows (up to align - 1 of them; the host knows neither their number nor `align`)
uint32_t fill_blocks(const sf_ctx* ctx, uint32_t E, uint32_t units) {
    return std::max<uint32_t>(1, std::min<uint32_t>({32, (uint32_t)ctx->num_sms * 4 / E, (units + 7) / 8}));
}
bool sizes_ok(uint32_t n, uint32_t k) { return k >= 1 && k <= SF_MAX_EXPERTS && (uint64_t)n * k <= 0x7FFFFFFFull; }
// may a lane's `count` elements be read and written as whole 16- or 32-byte pieces?
bool fits(const void* p, size_t ld, int dtype, uint32_t count) {
    const size_t piece = std::min<size_t>(32, count * type_bytes(dtype));
    return aligned(p, piece) && (ld * type_bytes(dtype)) % piece == 0;
}

}  // namespace

extern "C" int sf_expert_gate(sf_ctx* ctx, const void* scores, int dtype, const uint32_t* n_dev, uint32_t n, uint32_t E, size_t ld,
                              uint32_t k, int mode, int32_t* ids_out, float* weights_out, void* stream)
{
    if (!ctx || !type_ok(dtype) || E == 0 || E > SF_MAX_EXPERTS || k > E || ld < E || !sizes_ok(n, k)) return SF_ERR_ARG;
    if (mode != SF_GATE_SOFTMAX && mode != SF_GATE_SOFTMAX_PICKED && mode != SF_GATE_SHARE) return SF_ERR_ARG;
    if (n == 0) return SF_OK;
    if (!scores || !ids_out || !weights_out) return SF_ERR_ARG;
    if (!aligned(scores, type_bytes(dtype)) || !aligned(ids_out, 4) || !aligned(weights_out, 4) || !aligned(n_dev, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_experts(E, [&](auto lpr, auto v) {
            constexpr int L = decltype(lpr)::value, V = decltype(v)::value, S = V < 4 ? V : 4;
            const bool al = fits(scores, ld, dtype, V);
            return by_mode(mode, [&](auto m) {
                constexpr int M = decltype(m)::value;
                auto kern = k <= S * L ? (al ? gate_kernel<T, L, V, S, M, true> : gate_kernel<T, L, V, S, M, false>) : (al ? gate_kernel<T, L, V, V, M, true> : gate_kernel<T, L, V, V, M, false>);
                SF_CUDA(sf_launch_chained(kern, (n + kThreads / L - 1) / (kThreads / L), kThreads, 0, (cudaStream_t)stream, (const T*)scores, n_dev, n, E, ld, k, ids_out, weights_out, ctx->d_state));
                return SF_OK;
            });
        });
    });
}

extern "C" int sf_expert_gate_backward(sf_ctx* ctx, const void* scores, int dtype, const uint32_t* n_dev, uint32_t n, uint32_t E, size_t ld,
                                       uint32_t k, int mode, const int32_t* ids, const float* d_weights, void* d_scores_out, size_t ldd, void* stream)
{
    if (!ctx || !type_ok(dtype) || E == 0 || E > SF_MAX_EXPERTS || k > E || ld < E || ldd < E || !sizes_ok(n, k)) return SF_ERR_ARG;
    if (mode != SF_GATE_SOFTMAX && mode != SF_GATE_SOFTMAX_PICKED && mode != SF_GATE_SHARE) return SF_ERR_ARG;
    if (n == 0) return SF_OK;
    if (!scores || !ids || !d_weights || !d_scores_out) return SF_ERR_ARG;
    if (!aligned(scores, type_bytes(dtype)) || !aligned(d_scores_out, type_bytes(dtype)) || !aligned(ids, 4) || !aligned(d_weights, 4) || !aligned(n_dev, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_experts(E, [&](auto lpr, auto v) {
            constexpr int L = decltype(lpr)::value, V = decltype(v)::value;
            const bool al = fits(scores, ld, dtype, V) && fits(d_scores_out, ldd, dtype, V);
            return by_mode(mode, [&](auto m) {
                constexpr int M = decltype(m)::value;
                constexpr int P = L * V < 8 ? 4 : 8;       // (no more picks than experts)
                auto kern = k <= 4 ? (al ? gate_backward_kernel<T, L, V, M, 4, true> : gate_backward_kernel<T, L, V, M, 4, false>) :
                                     (al ? gate_backward_kernel<T, L, V, M, P, true> : gate_backward_kernel<T, L, V, M, P, false>);
                SF_CUDA(sf_launch_chained(kern, (n + kThreads / L - 1) / (kThreads / L), kThreads, 0, (cudaStream_t)stream, (const T*)scores, n_dev, n, E, ld, k, ids, d_weights,
                                          (T*)d_scores_out, ldd, ctx->d_state));
                return SF_OK;
            });
        });
    });
}

extern "C" int sf_expert_sort_workspace(uint32_t n, uint32_t k, uint32_t E, size_t* bytes_out)
{
    if (!bytes_out || E == 0 || E > SF_MAX_EXPERTS || !sizes_ok(n, k)) return SF_ERR_ARG;
    // one word per tile and expert; a tile has at least 1024 pairs
    *bytes_out = ((uint64_t)n * k + 1023) / 1024 * E * 4;
    return SF_OK;
}

extern "C" int sf_expert_sort(sf_ctx* ctx, const int32_t* ids, const uint32_t* n_dev, uint32_t n, uint32_t k, uint32_t E, uint32_t align,
                              uint32_t capacity, uint32_t* offsets_out, uint32_t* counts_out, int32_t* flow_of_row_out,
                              int32_t* row_of_pair_out, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx || E == 0 || E > SF_MAX_EXPERTS || !sizes_ok(n, k) || capacity > 0x7FFFFFFFu) return SF_ERR_ARG;
    if (align == 0 || align > 65536 || (align & (align - 1)) || (uint64_t)n * k + (uint64_t)E * (align - 1) > 0x7FFFFFFFull) return SF_ERR_ARG;
    if (!offsets_out || !counts_out || (n && (!ids || !row_of_pair_out)) || (capacity && !flow_of_row_out)) return SF_ERR_ARG;
    if (!aligned(ids, 4) || !aligned(n_dev, 4) || !aligned(offsets_out, 4) || !aligned(counts_out, 4) || !aligned(flow_of_row_out, 4) ||
        !aligned(row_of_pair_out, 4) || !aligned(workspace, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    const uint32_t tiles = sort_tiles(ctx, n, k, E);
    if (tiles > 1 && (!workspace || workspace_bytes < (size_t)tiles * E * 4)) return SF_ERR_ARG;
    const sort_args a = {ids, n_dev, n, k, E, align, capacity, tiles, (uint32_t*)workspace, offsets_out, counts_out, flow_of_row_out, row_of_pair_out};
    return (uint64_t)n * k > kFewPairs ? launch_sort<32>(ctx, a, (cudaStream_t)stream) : launch_sort<8>(ctx, a, (cudaStream_t)stream);
}

extern "C" int sf_expert_gather(sf_ctx* ctx, const void* x, int dtype, const uint32_t* n_dev, uint32_t n, uint32_t D, size_t ldx, uint32_t k,
                                const int32_t* row_of_pair, uint32_t E, const uint32_t* offsets, const uint32_t* counts, uint32_t capacity,
                                void* rows_out, size_t ldr, void* stream)
{
    if (!ctx || !type_ok(dtype) || D == 0 || D > SF_EXPERT_MAX_D || ldx < D || ldr < D || E == 0 || E > SF_MAX_EXPERTS || !sizes_ok(n, k) || capacity > 0x7FFFFFFFu) return SF_ERR_ARG;
    if (capacity == 0) return SF_OK;
    if ((n && (!x || !row_of_pair)) || !offsets || !counts || !rows_out) return SF_ERR_ARG;
    if (!aligned(x, type_bytes(dtype)) || !aligned(rows_out, type_bytes(dtype)) || !aligned(row_of_pair, 4) || !aligned(offsets, 4) || !aligned(counts, 4) || !aligned(n_dev, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    const uint32_t size = type_bytes(dtype);
    const uint32_t word = std::min({word_of(x, ldx, size), word_of(rows_out, ldr, size), word_of(nullptr, D, size)});
    auto go = [&](auto q) {
        typedef decltype(q) Q;
        constexpr int U = sizeof(Q) == 16 ? 4 : 8, S = sizeof(Q) == 16 ? 2 : 4;      // words a lane: wide rows, the most of several flows at a time
        const uint32_t per = sizeof(Q) / size, units = D / per, lanes = lanes_for(ctx, units, n), fb = flow_grid(ctx, n, lanes), zb = fill_blocks(ctx, E, units);
        // Rows of up to S words a lane: several flows at a time, 16-byte words where flows are many (30,000 x 64 bf16, k = 8: 8.5 us with, 6.6 without;
        // 150,000 x 64, k = 2: 7.4 and 9.3); narrower words gain with few flows too (3,000 x 17 fp16, k = 2: 3.1 and 3.7).
        const bool several = sizeof(Q) < 16 || many_flows(ctx, n, lanes, kSome);
        auto kern = !several ? gather_kernel<Q, U, 1> : units <= lanes ? gather_kernel<Q, 1, 4> : (units <= 2 * lanes ? gather_kernel<Q, 2, 4> : (units <= S * lanes ? gather_kernel<Q, S, 8 / S> : gather_kernel<Q, U, 1>));
        SF_CUDA(sf_launch_chained(kern, fb + E * zb, kThreads, 0, (cudaStream_t)stream, (const Q*)x, n_dev, n, units, ldx / per, k, row_of_pair, E,
                                  offsets, counts, capacity, (Q*)rows_out, ldr / per, lanes, fb, zb, ctx->d_state));
        return SF_OK;
    };
    return word == 16 ? go(uint4()) : (word == 4 ? go(uint32_t()) : go(uint16_t()));
}

static int combine(sf_ctx* ctx, const void* rows, int dtype, uint32_t capacity, uint32_t D, size_t ldr, const int32_t* row_of_pair,
                   const float* weights, const uint32_t* n_dev, uint32_t n, uint32_t k, void* y, size_t ldy, void* stream)
{
    if (!ctx || !type_ok(dtype) || D == 0 || D > SF_EXPERT_MAX_D || ldr < D || ldy < D || !sizes_ok(n, k) || capacity > 0x7FFFFFFFu) return SF_ERR_ARG;
    if (n == 0) return SF_OK;
    if ((capacity && !rows) || !row_of_pair || !y) return SF_ERR_ARG;
    if (!aligned(rows, type_bytes(dtype)) || !aligned(y, type_bytes(dtype)) || !aligned(row_of_pair, 4) || !aligned(weights, 4) || !aligned(n_dev, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    const uint32_t size = type_bytes(dtype);
    const uint32_t word = std::min({word_of(rows, ldr, size), word_of(y, ldy, size), word_of(nullptr, D, size)});
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_word<T>(word, [&](auto v) {
            constexpr int V = decltype(v)::value, U = V * sizeof(T) == 16 ? 4 : 8;
            const uint32_t units = D / V, lanes = lanes_for(ctx, units, n), grid = flow_grid(ctx, n, lanes);
            // Several flows at a time where flows are many (one word a lane, us: 150,000 x 64 bf16, k = 2: 12.5 with, 22 without).  Two words a lane: narrow words from the same number on (60,000 x 45 fp32, k = 2: 14.7 and 18.1), 16-byte words of fp32 later
            // (100,000 x 256, k = 2: 64 and 66; 30,000 x 256: 19.7 and 17.5), of 16 bits never: the sums of four flows leave the registers (150,000 x
            // 512 bf16, k = 2: 299 and 138).
            constexpr int W = V * 2 <= 8 ? 2 : 1;
            const bool one = units <= lanes && many_flows(ctx, n, lanes, kSome), two = W == 2 && units > lanes && units <= 2 * lanes && many_flows(ctx, n, lanes, V == 4 ? 8 : kSome);
            auto kern = one ? combine_narrow_kernel<T, V, 1> : (two ? combine_narrow_kernel<T, V, W> : combine_kernel<T, V, U>);
            SF_CUDA(sf_launch_chained(kern, grid, kThreads, 0, (cudaStream_t)stream, (const T*)rows, capacity, D, ldr, row_of_pair, weights, n_dev, n, k, (T*)y, ldy, lanes, ctx->d_state));
            return SF_OK;
        });
    });
}

extern "C" int sf_expert_combine(sf_ctx* ctx, const void* rows, int dtype, uint32_t capacity, uint32_t D, size_t ldr, const int32_t* row_of_pair,
                                 const float* weights, const uint32_t* n_dev, uint32_t n, uint32_t k, void* y_out, size_t ldy, void* stream)
{
    return combine(ctx, rows, dtype, capacity, D, ldr, row_of_pair, weights, n_dev, n, k, y_out, ldy, stream);
}

extern "C" int sf_expert_gather_backward(sf_ctx* ctx, const void* d_rows, int dtype, uint32_t capacity, uint32_t D, size_t ldr,
                                         const int32_t* row_of_pair, const uint32_t* n_dev, uint32_t n, uint32_t k, void* dx_out, size_t ldx, void* stream)
{
    return combine(ctx, d_rows, dtype, capacity, D, ldr, row_of_pair, nullptr, n_dev, n, k, dx_out, ldx, stream);
}

extern "C" int sf_expert_combine_backward(sf_ctx* ctx, const void* dy, int dtype, size_t ldy, const void* rows, uint32_t capacity, uint32_t D,
                                          size_t ldr, const int32_t* row_of_pair, const float* weights, const uint32_t* n_dev, uint32_t n,
                                          uint32_t k, uint32_t E, const uint32_t* offsets, const uint32_t* counts, void* d_rows_out,
                                          size_t ldd, float* d_weights_out, void* stream)
{
    if (!ctx || !type_ok(dtype) || D == 0 || D > SF_EXPERT_MAX_D || ldr < D || ldy < D || (d_rows_out && ldd < D) || E == 0 || E > SF_MAX_EXPERTS || !sizes_ok(n, k) || capacity > 0x7FFFFFFFu) return SF_ERR_ARG;
    if (!d_rows_out && !d_weights_out) return SF_ERR_ARG;
    if (n && (!dy || !row_of_pair || (d_weights_out && capacity && !rows))) return SF_ERR_ARG;
    if (d_rows_out && (!offsets || !counts)) return SF_ERR_ARG;
    if (!aligned(dy, type_bytes(dtype)) || !aligned(rows, type_bytes(dtype)) || !aligned(d_rows_out, type_bytes(dtype)) || !aligned(row_of_pair, 4) || !aligned(weights, 4) ||
        !aligned(offsets, 4) || !aligned(counts, 4) || !aligned(d_weights_out, 4) || !aligned(n_dev, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    const uint32_t size = type_bytes(dtype);
    uint32_t word = std::min(word_of(dy, ldy, size), word_of(nullptr, D, size));
    if (d_weights_out) word = std::min(word, word_of(rows, ldr, size));
    if (d_rows_out) word = std::min(word, word_of(d_rows_out, ldd, size));
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_word<T>(word, [&](auto v) {
            constexpr int V = decltype(v)::value, U = V * sizeof(T) == 16 ? 1 : 4;
            const uint32_t units = D / V, lanes = lanes_for(ctx, units, n), fb = flow_grid(ctx, n, lanes), zb = fill_blocks(ctx, E, units), grid = fb + (d_rows_out ? E * zb : 0);
            if (grid == 0) return (int)SF_OK;
            // Narrow words of rows that a warp holds: four flows at a time where flows are many, us: one word a lane (150,000 x 17 fp16, k = 2: 41 with, 60
            // to 68 without; 3,000 x 17: 6.2 and 3.8), two words (100,000 x 45 fp32, k = 2: 44 and 54; 16-bit words later: 300,000 x 90 bf16 171 and 185,
            // 100,000 x 90, k = 4: 117 and 110).  16-byte words one flow at a time: all pairs' loads of a flow on their way are enough
            // (150,000 x 64 bf16, k = 2: 24 us, four flows at a time 28; 30,000 x 512, k = 8: 102 and 372).
            // Else where flows fill the machine one pair at a time with two words on their way (120,003 x 1024 bf16, k = 2: 202 us; one word 276, two
            // pairs 226 to 239) unless a lane has one 16-byte word alone (150,000 x 256 bf16, k = 2: 112 us, 90 with two pairs), and up to four
            // pairs in flight elsewhere.
            constexpr int U2 = U == 1 ? 2 : U, W = V * sizeof(T) < 16 ? 2 : 1;
            const bool warp = W == 2 && lanes <= 32;       // (the narrow kernel's sums stay within a warp)
            const bool one = warp && units <= lanes && many_flows(ctx, n, lanes, kSome), two = warp && units > lanes && units <= 2 * lanes && many_flows(ctx, n, lanes, sizeof(T) == 4 ? kSome : 12);
            const bool one_pair = (uint64_t)n * lanes >= (uint64_t)ctx->num_sms * 2048 && (W == 2 || units > 32);
            auto kern = one_pair ? combine_backward_kernel<T, V, U2, 1> : (k == 1 ? combine_backward_kernel<T, V, U, 1> : (k == 2 ? combine_backward_kernel<T, V, U, 2> : combine_backward_kernel<T, V, U, 4>));
            if constexpr (W == 2) { if (one) kern = combine_backward_narrow_kernel<T, V, 1>; if (two) kern = combine_backward_narrow_kernel<T, V, 2>; }
            SF_CUDA(sf_launch_chained(kern, grid, kThreads, 0, (cudaStream_t)stream, (const T*)dy, ldy, (const T*)rows, capacity, D, ldr, row_of_pair, weights, n_dev, n, k, E,
                                      offsets, counts, (T*)d_rows_out, ldd, d_weights_out, lanes, fb, zb, ctx->d_state));
            return (int)SF_OK;
        });
    });
}
