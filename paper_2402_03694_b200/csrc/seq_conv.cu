// Short causal convolution over the rows of sequences, one filter of W <= 8 taps a channel, and its gradients:
//   pre_t = b + sum_k w[k] x_{t-W+1+k},  y_t = act(pre_t),   x before the sequence from a state of W - 1 rows (or zero);
//   dpre_t = dy_t act'(pre_t),  dx_j = sum_k w[k] dpre_{j+W-1-k},  dw[k] = sum_t dpre_t x_{t-W+1+k},  db = sum_t dpre_t.
// A thread owns V channels and walks down a tile of rows of one sequence with the last W rows in registers, so that every element is
// loaded once (plus W - 1 rows a tile); the filters stay in registers over all the tiles that a thread takes in turn.  Bound by HBM.
#include <algorithm>
#include "seq_common.cuh"

namespace {

using namespace sfseq;

constexpr uint32_t kThreads = 128;
constexpr uint32_t kMaxTaps = 8;
constexpr uint32_t kParts = 1024;          // partial sums of the filters' gradient at most

struct Tiling {
    uint32_t lanes;        // threads side by side on a row (a power of two), of V channels each
    uint32_t cblocks;      // blocks side by side on a row
    uint32_t tile, tiles;  // rows of a tile, tiles of a sequence
    uint32_t parts;        // blocks behind one another over the tiles
};

template <typename T> struct Conv {
    Seqs q;
    const T* x; size_t ldx;
    const float* w; const float* bias;
    uint32_t D, W;
    int silu;
    const T* state_in;
    T* state_out; T* y; size_t ldy;                                                       // forward
    const T* dy; size_t lddy; const T* d_state; T* d_state0; T* dx; size_t lddx;          // backward
    float* parts;                                                                         // [parts][D][W + 1]: filter, then bias
    Tiling t;
    sf_dev_state* st;
};

template <int V> __device__ __forceinline__ void zero(float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; i++) v[i] = 0.0f;
}
// (a pool that the same call writes is read as ordinary memory)
template <typename T, int V> __device__ __forceinline__ void load_plain(const T* p, float (&x)[V]) {
    typedef typename Word<V * sizeof(T)>::type Q;
    union { Q w; T e[V]; } u;
    u.w = *reinterpret_cast<const Q*>(p);
#pragma unroll
    for (int i = 0; i < V; i++) x[i] = to_f32(u.e[i]);
}

// Filters of the thread's channels.  Tap k of W sits at WT - W + k, so that the newest row has the last one; what lies before is not used.
template <int V, int WT>
__device__ __forceinline__ void load_taps(const float* __restrict__ w, uint32_t c, uint32_t W, float (&tap)[WT][V]) {
#pragma unroll
    for (int k = 0; k < WT; k++)
#pragma unroll
        for (int i = 0; i < V; i++) tap[k][i] = k + (int)W >= WT ? __ldg(w + (size_t)(c + i) * W + (k + (int)W - WT)) : 0.0f;
}

// Row p of a sequence; for p < 0 row W - 1 + p of the state it starts from (rows before that are never asked for by a tap that counts)
template <typename T, int V>
__device__ __forceinline__ void row_at(const Conv<T>& a, const Range& r, int p, uint32_t c, float (&v)[V]) {
    if (p >= 0) load_word<T, V>(a.x + (size_t)(r.first + p) * a.ldx + c, v);
    else if (a.state_in && r.slot >= 0 && p + (int)a.W >= 1) load_plain<T, V>(a.state_in + ((size_t)r.slot * (a.W - 1) + (a.W - 1 + p)) * a.D + c, v);
    else zero<V>(v);
}

// bias + the filter over the rows win[0] (oldest) .. win[WT - 1]
template <int V, int WT, bool EXACT>
__device__ __forceinline__ void filter(const float (&tap)[WT][V], const float (&win)[WT][V], const float (&bias)[V], uint32_t W, float (&pre)[V]) {
#pragma unroll
    for (int i = 0; i < V; i++) pre[i] = bias[i];
#pragma unroll
    for (int k = 0; k < WT; k++) {
        if (!EXACT && k + (int)W < WT) continue;
#pragma unroll
        for (int i = 0; i < V; i++) pre[i] = fmaf(tap[k][i], win[k][i], pre[i]);
    }
}

template <int V, int WT>
__device__ __forceinline__ void shift(float (&win)[WT][V]) {
#pragma unroll
    for (int k = 0; k + 1 < WT; k++)
#pragma unroll
        for (int i = 0; i < V; i++) win[k][i] = win[k + 1][i];
}

template <typename T, int V, int WT, bool EXACT>
__global__ void __launch_bounds__(kThreads) conv_kernel(const Conv<T> a) {
    sf_chain_enter();
    const Tiling& t = a.t;
    const uint32_t c = (blockIdx.x % t.cblocks * t.lanes + threadIdx.x % t.lanes) * V, per = kThreads / t.lanes;
    if (c >= a.D) return;
    const uint32_t W = EXACT ? WT : a.W;
    float tap[WT][V], bias[V];
    load_taps<V, WT>(a.w, c, W, tap);
#pragma unroll
    for (int i = 0; i < V; i++) bias[i] = a.bias ? __ldg(a.bias + c + i) : 0.0f;
    const uint64_t items = (uint64_t)a.q.n_seq * t.tiles;
    for (uint64_t it = (uint64_t)(blockIdx.x / t.cblocks) * per + threadIdx.x / t.lanes; it < items; it += (uint64_t)t.parts * per) {
        const uint32_t s = (uint32_t)(it / t.tiles), j = (uint32_t)(it % t.tiles);
        const Range r = range_of(a.q, s, a.st);
        const int p0 = (int)(j * t.tile), p1 = (int)min(r.len, (j + 1) * t.tile);
        if (p0 >= p1 && (j || !a.state_out)) continue;
        float win[WT][V];
#pragma unroll
        for (int k = 0; k + 1 < WT; k++) row_at<T, V>(a, r, p0 - (WT - 1) + k, c, win[k + 1]);
        if (j == 0 && a.state_out && r.slot >= 0) {
            // The sequence's last W - 1 rows, which where it is shorter begin with rows of the state it started from: win holds those
            // (row p < 0 at win[WT + p]).  The first tile writes them all: it alone has read the old state, so the pools may be one.
            T* so = a.state_out + (size_t)r.slot * (W - 1) * a.D + c;
            for (int i = 0; i + 1 < (int)W; i++) {
                const int p = (int)r.len - (int)(W - 1) + i;
                float o[V];
                if (p >= 0) load_word<T, V>(a.x + (size_t)(r.first + p) * a.ldx + c, o);
                else {
#pragma unroll
                    for (int k = 1; k < WT; k++) if (k == WT + p) {
#pragma unroll
                        for (int e = 0; e < V; e++) o[e] = win[k][e];
                    }
                }
                store_word<T, V>(so + (size_t)i * a.D, o);
            }
        }
        const T* x = a.x + (size_t)(r.first + p0) * a.ldx + c;
        T* y = a.y + (size_t)(r.first + p0) * a.ldy + c;
        for (int p = p0; p < p1; p++, x += a.ldx, y += a.ldy) {
            shift<V, WT>(win);
            load_word<T, V>(x, win[WT - 1]);
            float pre[V];
            filter<V, WT, EXACT>(tap, win, bias, W, pre);
            if (a.silu) {
#pragma unroll
                for (int i = 0; i < V; i++) pre[i] *= sigmoid(pre[i]);
            }
            store_word<T, V>(y, pre);
        }
    }
}

// The same walk with W - 1 rows more at a tile's end: dx_j is complete once dpre_{j+W-1} is there.
template <typename T, int V, int WT, bool EXACT>
__global__ void __launch_bounds__(kThreads) conv_backward_kernel(const Conv<T> a) {
    sf_chain_enter();
    extern __shared__ float sums[];                        // [threads][(WT + 1) * V] where the block joins its sums
    const Tiling& t = a.t;
    const uint32_t c = (blockIdx.x % t.cblocks * t.lanes + threadIdx.x % t.lanes) * V, per = kThreads / t.lanes;
    const uint32_t W = EXACT ? WT : a.W;
    float dw[WT][V], db[V];
#pragma unroll
    for (int k = 0; k < WT; k++) zero<V>(dw[k]);
    zero<V>(db);
    if (c < a.D) {
        float tap[WT][V], bias[V];
        load_taps<V, WT>(a.w, c, W, tap);
#pragma unroll
        for (int i = 0; i < V; i++) bias[i] = a.bias ? __ldg(a.bias + c + i) : 0.0f;
        const uint64_t items = (uint64_t)a.q.n_seq * t.tiles;
        for (uint64_t it = (uint64_t)(blockIdx.x / t.cblocks) * per + threadIdx.x / t.lanes; it < items; it += (uint64_t)t.parts * per) {
            const uint32_t s = (uint32_t)(it / t.tiles), j = (uint32_t)(it % t.tiles);
            const Range r = range_of(a.q, s, a.st);
            const int p0 = (int)(j * t.tile), p1 = (int)min(r.len, (j + 1) * t.tile), len = (int)r.len, H = (int)W - 1;
            const bool d0 = j == 0 && a.d_state0 && r.slot >= 0;
            if (p0 >= p1 && !d0) continue;
            float win[WT][V], dp[WT][V];                   // x_{p-WT+1} .. x_p; dpre_p, dpre_{p-1}, ..
#pragma unroll
            for (int k = 0; k + 1 < WT; k++) row_at<T, V>(a, r, p0 - (WT - 1) + k, c, win[k + 1]);
#pragma unroll
            for (int k = 0; k < WT; k++) zero<V>(dp[k]);
            for (int p = p0; p < p1 + H; p++) {
                shift<V, WT>(win);
#pragma unroll
                for (int k = WT - 1; k > 0; k--)
#pragma unroll
                    for (int i = 0; i < V; i++) dp[k][i] = dp[k - 1][i];
                zero<V>(dp[0]);
                if (p < len) {
                    row_at<T, V>(a, r, p, c, win[WT - 1]);
                    float g[V];
                    load_word<T, V>(a.dy + (size_t)(r.first + p) * a.lddy + c, g);
                    if (a.silu) {
                        float pre[V];
                        filter<V, WT, EXACT>(tap, win, bias, W, pre);
#pragma unroll
                        for (int i = 0; i < V; i++) { const float e = sigmoid(pre[i]); g[i] *= e * (1.0f + pre[i] * (1.0f - e)); }
                    }
#pragma unroll
                    for (int i = 0; i < V; i++) dp[0][i] = g[i];
                    if (p < p1) {
#pragma unroll
                        for (int i = 0; i < V; i++) db[i] += g[i];
#pragma unroll
                        for (int k = 0; k < WT; k++) {
                            if (!EXACT && k + (int)W < WT) continue;
#pragma unroll
                            for (int i = 0; i < V; i++) dw[k][i] = fmaf(g[i], win[k][i], dw[k][i]);
                        }
                    }
                } else zero<V>(win[WT - 1]);
                const int o = p - H;                       // the row whose gradient is complete now
                if (o >= p0 ? a.dx == nullptr : !d0) continue;
                float d[V];
                zero<V>(d);
#pragma unroll
                for (int k = 0; k < WT; k++) {             // tap k of W meets dpre_{o+W-1-k} = dp[k]
                    if (!EXACT && k >= (int)W) continue;
#pragma unroll
                    for (int i = 0; i < V; i++) d[i] = fmaf(EXACT ? tap[k][i] : __ldg(a.w + (size_t)(c + i) * W + k), dp[k][i], d[i]);
                }
                if (a.d_state && r.slot >= 0 && o >= len - H) {
                    float e[V];
                    load_plain<T, V>(a.d_state + ((size_t)r.slot * H + (o - (len - H))) * a.D + c, e);
#pragma unroll
                    for (int i = 0; i < V; i++) d[i] += e[i];
                }
                if (o >= 0) store_word<T, V>(a.dx + (size_t)(r.first + o) * a.lddx + c, d);
                else store_word<T, V>(a.d_state0 + ((size_t)r.slot * H + (o + H)) * a.D + c, d);
            }
        }
    }
    if (!a.parts) return;
    // the block's threads on the same channels add up their sums, in the order of the threads
    constexpr int Q = (WT + 1) * V;
    float* mine = sums + (size_t)threadIdx.x * Q;
#pragma unroll
    for (int i = 0; i < V; i++) {
#pragma unroll
        for (int k = 0; k < WT; k++) mine[i * (WT + 1) + k] = dw[k][i];
        mine[i * (WT + 1) + WT] = db[i];
    }
    __syncthreads();
    const uint32_t n = t.lanes * V * (W + 1), c0 = blockIdx.x % t.cblocks * t.lanes * V;
    for (uint32_t e = threadIdx.x; e < n; e += kThreads) {
        const uint32_t ch = e / (W + 1), k = e % (W + 1);
        if (c0 + ch >= a.D) break;
        const float* p = sums + (size_t)(ch / V) * Q + (ch % V) * (WT + 1) + (WT - W) + k;
        float v = 0.0f;
        for (uint32_t y = 0; y < per; y++) v += p[(size_t)y * t.lanes * Q];
        a.parts[((size_t)(blockIdx.x / t.cblocks) * a.D + c0 + ch) * (W + 1) + k] = v;
    }
}

// dw[c][k] and db[c] from the blocks' sums: a warp per value, lanes over the blocks
__global__ void __launch_bounds__(256) conv_join_kernel(const float* __restrict__ parts, uint32_t n_parts, uint32_t D, uint32_t W, float* dw, float* db) {
    sf_chain_enter();
    const uint32_t lane = threadIdx.x & 31, e = blockIdx.x * 8 + threadIdx.x / 32, n = D * (W + 1);
    if (e >= n) return;
    float v = 0.0f;
    for (uint32_t p = lane; p < n_parts; p += 32) v += parts[(size_t)p * n + e];
#pragma unroll
    for (int m = 16; m; m >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, m);
    if (lane) return;
    const uint32_t c = e / (W + 1), k = e % (W + 1);
    if (k < W) { if (dw) dw[(size_t)c * W + k] = v; }
    else if (db) db[c] = v;
}

// ---- host ----------------------------------------------------------------------------------------------------------
uint32_t word_of(const void* p, size_t ld, uint32_t size) {          // the widest access (16, 8, 4 or 2 bytes) on which every row begins
    const uint64_t v = (uint64_t)(uintptr_t)p | (uint64_t)ld * size;
    return v % 16 == 0 ? 16 : (v % 8 == 0 ? 8 : (v % 4 == 0 ? 4 : 2));
}

// Tiles of 32 rows (8 where the sequences are too few to fill the machine with those), threads over tiles in turn once the machine is full.
Tiling tiling(const sf_sequences* q, uint32_t D, uint32_t V, uint32_t most_parts) {
    Tiling t;
    const uint32_t units = (D + V - 1) / V;
    t.lanes = 1;
    while (t.lanes < kThreads && t.lanes < units) t.lanes *= 2;
    t.cblocks = (units + t.lanes - 1) / t.lanes;
    const uint64_t full = (uint64_t)SF_NUM_SMS_DEFAULT * 1024;
    t.tile = 32;
    while (t.tile > 8 && (uint64_t)q->n_seq * ((q->max_len + t.tile - 1) / t.tile) * units < full) t.tile /= 2;
    t.tiles = (q->max_len + t.tile - 1) / t.tile;
    const uint32_t per = kThreads / t.lanes;
    const uint64_t blocks = ((uint64_t)q->n_seq * t.tiles + per - 1) / per;
    t.parts = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>({blocks, most_parts, std::max<uint64_t>(1, (uint64_t)SF_NUM_SMS_DEFAULT * 16 / t.cblocks)}));
    return t;
}

int check(sf_ctx* ctx, const sf_sequences* seq, const void* x, int dtype, uint32_t rows, uint32_t D, size_t ldx, const float* w, const float* bias, uint32_t W, int act,
          uint32_t n_slots) {
    if (!ctx || !type_ok(dtype) || D == 0 || D > SF_EXPERT_MAX_D || ldx < D || W == 0 || W > kMaxTaps || (act != SF_ACT_NONE && act != SF_ACT_SILU)) return SF_ERR_ARG;
    if (n_slots > 0x7FFFFFFFu || !w || (rows && !x)) return SF_ERR_ARG;
    if (!aligned(x, type_bytes(dtype)) || !aligned(w, 4) || !aligned(bias, 4)) return SF_ERR_ARG;
    return check_sequences(seq, rows);
}

template <typename T, int MOST, typename F> int by_width(uint32_t word, F f) {
    constexpr int size = sizeof(T);
    if (word >= MOST) return f(std::integral_constant<int, MOST / size>());
    if (size == 2 && word >= 4) return f(std::integral_constant<int, 4 / size>());
    return f(std::integral_constant<int, 1>());
}
template <typename F> int by_taps(uint32_t W, F f) {
    if (W == 2) return f(std::integral_constant<int, 2>(), std::true_type());
    if (W == 3) return f(std::integral_constant<int, 3>(), std::true_type());
    if (W == 4) return f(std::integral_constant<int, 4>(), std::true_type());
    return f(std::integral_constant<int, (int)kMaxTaps>(), std::false_type());
}

}  // namespace

extern "C" int sf_seq_conv(sf_ctx* ctx, const sf_sequences* seq, const void* x, int dtype, uint32_t rows, uint32_t D, size_t ldx, const float* w,
                           const float* bias, uint32_t W, int act, const void* state_in, void* state_out, uint32_t n_slots, void* y_out, size_t ldy, void* stream)
{
    const int ok = check(ctx, seq, x, dtype, rows, D, ldx, w, bias, W, act, n_slots);
    if (ok != SF_OK || ldy < D || (rows && !y_out) || !aligned(y_out, type_bytes(dtype)) || !aligned(state_in, type_bytes(dtype)) || !aligned(state_out, type_bytes(dtype))) return SF_ERR_ARG;
    if (seq->n_seq == 0) return SF_OK;
    if (W == 1) state_in = state_out = nullptr;
    SF_ON_DEVICE(ctx);
    const uint32_t size = type_bytes(dtype);
    const uint32_t word = std::min({word_of(x, ldx, size), word_of(y_out, ldy, size), word_of(state_in, D, size), word_of(state_out, D, size), word_of(nullptr, D, size)});
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_width<T, 16>(word, [&](auto v) {
            return by_taps(W, [&](auto taps, auto exact) {
                constexpr int V = decltype(v)::value, WT = decltype(taps)::value;
                Conv<T> a = {};
                a.q = seqs_of(seq, rows, n_slots); a.x = (const T*)x; a.ldx = ldx; a.w = w; a.bias = bias; a.D = D; a.W = W; a.silu = act == SF_ACT_SILU;
                a.state_in = (const T*)state_in; a.state_out = (T*)state_out; a.y = (T*)y_out; a.ldy = ldy; a.st = ctx->d_state;
                a.t = tiling(seq, D, V, 0x7FFFFFFFu);
                SF_CUDA(sf_launch_chained(conv_kernel<T, V, WT, decltype(exact)::value>, a.t.cblocks * a.t.parts, kThreads, 0, (cudaStream_t)stream, a));
                return (int)SF_OK;
            });
        });
    });
}

extern "C" int sf_seq_conv_backward_workspace(uint32_t n_seq, uint32_t max_len, uint32_t D, uint32_t W, size_t* bytes_out)
{
    if (!bytes_out || max_len == 0 || D == 0 || D > SF_EXPERT_MAX_D || W == 0 || W > kMaxTaps) return SF_ERR_ARG;
    const sf_sequences q = {nullptr, nullptr, nullptr, n_seq, max_len};
    uint32_t parts = 1;
    for (uint32_t v : {1u, 2u, 4u}) parts = std::max(parts, tiling(&q, D, v, kParts).parts);
    *bytes_out = (size_t)parts * D * (W + 1) * 4;
    return SF_OK;
}

extern "C" int sf_seq_conv_backward(sf_ctx* ctx, const sf_sequences* seq, const void* x, int dtype, uint32_t rows, uint32_t D, size_t ldx, const float* w,
                                    const float* bias, uint32_t W, int act, const void* state_in, const void* dy, size_t lddy, const void* d_state,
                                    uint32_t n_slots, void* dx_out, size_t lddx, float* dw_out, float* dbias_out, void* d_state_in_out,
                                    void* workspace, size_t workspace_bytes, void* stream)
{
    const int ok = check(ctx, seq, x, dtype, rows, D, ldx, w, bias, W, act, n_slots);
    if (ok != SF_OK || lddy < D || (rows && !dy) || (dx_out && lddx < D)) return SF_ERR_ARG;
    const uint32_t size = type_bytes(dtype);
    if (!aligned(dy, size) || !aligned(dx_out, size) || !aligned(state_in, size) || !aligned(d_state, size) || !aligned(d_state_in_out, size) || !aligned(dw_out, 4) ||
        !aligned(dbias_out, 4) || !aligned(workspace, 4)) return SF_ERR_ARG;
    const bool sums = dw_out || dbias_out;
    if (!sums && !dx_out && !d_state_in_out) return SF_ERR_ARG;
    if (W == 1) { state_in = nullptr; d_state = nullptr; d_state_in_out = nullptr; }
    SF_ON_DEVICE(ctx);
    const uint32_t word = std::min({word_of(x, ldx, size), word_of(dy, lddy, size), word_of(dx_out, lddx, size), word_of(state_in, D, size), word_of(d_state, D, size),
                                    word_of(d_state_in_out, D, size), word_of(nullptr, D, size)});
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_width<T, (sizeof(T) == 2 ? 8 : 16)>(word, [&](auto v) {
            return by_taps(W, [&](auto taps, auto exact) {
                constexpr int V = decltype(v)::value, WT = decltype(taps)::value;
                Conv<T> a = {};
                a.q = seqs_of(seq, rows, n_slots); a.x = (const T*)x; a.ldx = ldx; a.w = w; a.bias = bias; a.D = D; a.W = W; a.silu = act == SF_ACT_SILU;
                a.state_in = (const T*)state_in; a.dy = (const T*)dy; a.lddy = lddy; a.d_state = (const T*)d_state; a.d_state0 = (T*)d_state_in_out;
                a.dx = (T*)dx_out; a.lddx = lddx; a.st = ctx->d_state;
                a.t = tiling(seq, D, V, kParts);
                if (sums && (!workspace || workspace_bytes < (size_t)a.t.parts * D * (W + 1) * 4)) return (int)SF_ERR_ARG;
                a.parts = sums ? (float*)workspace : nullptr;
                SF_CUDA(sf_launch_chained(conv_backward_kernel<T, V, WT, decltype(exact)::value>, a.t.cblocks * a.t.parts, kThreads, sums ? kThreads * (WT + 1) * V * 4 : 0,
                                          (cudaStream_t)stream, a));
                if (sums) SF_CUDA(sf_launch_chained(conv_join_kernel, (D * (W + 1) + 7) / 8, 256, 0, (cudaStream_t)stream, (const float*)workspace, a.t.parts, D, W, dw_out, dbias_out));
                return (int)SF_OK;
            });
        });
    });
}
