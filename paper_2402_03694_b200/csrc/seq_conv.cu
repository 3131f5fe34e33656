// Short causal convolution over the rows of sequences, one filter of W <= 8 taps a channel, and its gradients:
//   pre_t = b + sum_k w[k] x_{t-W+1+k},  y_t = act(pre_t),   x before the sequence from a state of W - 1 rows (or zero);
//   dpre_t = dy_t act'(pre_t),  dx_j = sum_k w[k] dpre_{j+W-1-k},  dw[k] = sum_t dpre_t x_{t-W+1+k},  db = sum_t dpre_t.
// A thread owns V channels and walks down a tile of rows of one sequence with the last W rows in registers, so that every element is
// loaded once (plus W - 1 rows a tile); the filters stay in registers over all the tiles that a thread takes in turn.  8192 flows of up to 128 x 256 bf16: forward 117 us
// (82 of bytes), where no unit is saturated (issue 57 %, function unit 50 %, HBM 42 %: 19 warps an SM that wait for rows); gradients 247 us (123 of bytes), where 11 warps an SM wait for
// their own instructions (166 registers; issue 46 %, HBM 33 %).
#include <algorithm>
#include "seq_common.cuh"

namespace {

using namespace sfseq;

constexpr uint32_t kThreads = 128;
constexpr uint32_t kMaxTaps = 8;
constexpr int kAheadF = 4, kAheadB = 4;     // rows on their way while others are worked on: forward, backward
constexpr int kBlocksB = 3;                // blocks of the backward kernel an SM: its registers (four with fewer rows ahead: 280 us, these 247)

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

// V channels side by side; PAIRS: two an instruction (fewer instructions, more moves: the gradients gain, 280 -> 247 us, the forward pass loses, 122 -> 129)
template <int V, bool PAIRS> struct Ch {
    float p[V];
    __device__ __forceinline__ void set(const float (&x)[V]) {
#pragma unroll
        for (int i = 0; i < V; i++) p[i] = x[i];
    }
    __device__ __forceinline__ void get(float (&x)[V]) const {
#pragma unroll
        for (int i = 0; i < V; i++) x[i] = p[i];
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < V; i++) p[i] = 0.0f;
    }
    __device__ __forceinline__ void set_product(const Ch& a, const Ch& b) {
#pragma unroll
        for (int i = 0; i < V; i++) p[i] = a.p[i] * b.p[i];
    }
    __device__ __forceinline__ void add_product(const Ch& a, const Ch& b) {
#pragma unroll
        for (int i = 0; i < V; i++) p[i] = fmaf(a.p[i], b.p[i], p[i]);
    }
    __device__ __forceinline__ void add(const Ch& a) {
#pragma unroll
        for (int i = 0; i < V; i++) p[i] += a.p[i];
    }
    template <typename T> __device__ __forceinline__ void silu() {
#pragma unroll
        for (int i = 0; i < V; i++) p[i] *= sigmoid<T>(p[i]);
    }
    template <typename T> __device__ __forceinline__ void mul_silu_slope(const Ch& x) {      // times silu'(x) = s (1 + x (1 - s))
#pragma unroll
        for (int i = 0; i < V; i++) { const float s = sigmoid<T>(x.p[i]); p[i] *= s * fmaf(x.p[i], 1.0f - s, 1.0f); }
    }
};

template <int V> struct Ch<V, true> {
    static constexpr int P = V / 2;
    f2 p[P];
    __device__ __forceinline__ void set(const float (&x)[V]) {
#pragma unroll
        for (int i = 0; i < P; i++) p[i] = pack2(x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ void get(float (&x)[V]) const {
#pragma unroll
        for (int i = 0; i < P; i++) unpack2(p[i], x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < P; i++) p[i] = 0;
    }
    __device__ __forceinline__ void set_product(const Ch& a, const Ch& b) {
#pragma unroll
        for (int i = 0; i < P; i++) p[i] = mul2(a.p[i], b.p[i]);
    }
    __device__ __forceinline__ void add_product(const Ch& a, const Ch& b) {
#pragma unroll
        for (int i = 0; i < P; i++) p[i] = fma2(a.p[i], b.p[i], p[i]);
    }
    __device__ __forceinline__ void add(const Ch& a) {
#pragma unroll
        for (int i = 0; i < P; i++) p[i] = add2(a.p[i], p[i]);
    }
    template <typename T> __device__ __forceinline__ void mul_silu_slope(const Ch& x) {
#pragma unroll
        for (int i = 0; i < P; i++) {
            const f2 s = sigmoid2<T>(x.p[i]), one = dup2(1.0f);
            p[i] = mul2(mul2(p[i], s), fma2(x.p[i], fma2(s, dup2(-1.0f), one), one));
        }
    }
};

// V elements of T as they lie in memory
template <typename T, int V> struct Raw {
    typename Word<V * sizeof(T)>::type w;
    __device__ __forceinline__ void fetch(const T* p) { w = __ldg(reinterpret_cast<const decltype(w)*>(p)); }
    __device__ __forceinline__ void fetch_plain(const T* p) { w = *reinterpret_cast<const decltype(w)*>(p); }     // (a pool that the same call writes)
    template <bool PAIRS> __device__ __forceinline__ void open(Ch<V, PAIRS>& c) const {
        union { decltype(w) q; T e[V]; } u;
        u.q = w;
        float x[V];
#pragma unroll
        for (int i = 0; i < V; i++) x[i] = to_f32(u.e[i]);
        c.set(x);
    }
};
template <typename T, int V, bool PAIRS> __device__ __forceinline__ void store(T* p, const Ch<V, PAIRS>& c) { float x[V]; c.get(x); store_word<T, V>(p, x); }

// Filters of the thread's channels by lag: tap[m] is what x_{t-m} is multiplied with, m < W; what lies behind is not used.  Four taps in one
// access where they lie on a boundary (a thread's filters are its own: narrow accesses of a warp touch as many lines each).
template <int V, int WT, bool PAIRS> __device__ __forceinline__ void load_taps(const float* __restrict__ w, uint32_t c, uint32_t W, Ch<V, PAIRS> (&tap)[WT]) {
    float x[WT][V];
    bool whole = false;
    if constexpr (WT == 4) if (((uintptr_t)w & 15u) == 0) {
        whole = true;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const float4 q = __ldg(reinterpret_cast<const float4*>(w) + c + i);
            x[3][i] = q.x; x[2][i] = q.y; x[1][i] = q.z; x[0][i] = q.w;
        }
    }
    if (!whole) {
#pragma unroll
        for (int m = 0; m < WT; m++)
#pragma unroll
            for (int i = 0; i < V; i++) x[m][i] = m < (int)W ? __ldg(w + (size_t)(c + i) * W + (W - 1 - m)) : 0.0f;
    }
#pragma unroll
    for (int m = 0; m < WT; m++) tap[m].set(x[m]);
}
template <int V, bool PAIRS> __device__ __forceinline__ void load_bias(const float* __restrict__ b, uint32_t c, Ch<V, PAIRS>& o) {
    float x[V];
#pragma unroll
    for (int i = 0; i < V; i++) x[i] = b ? __ldg(b + c + i) : 0.0f;
    o.set(x);
}

// The WT - 1 rows before row p (oldest first); row -j of a sequence is row W - 1 - j of the state it starts from, zero without one.
template <typename T, int V, int WT, int AT, bool PAIRS> __device__ __forceinline__ void rows_before(const Conv<T>& a, const Range& r, int p, uint32_t c, Ch<V, PAIRS> (&x)[AT]) {
#pragma unroll
    for (int k = 0; k + 1 < WT; k++) {
        const int q = p - (WT - 1) + k;
        Raw<T, V> v = {};
        if (q >= 0) v.fetch(a.x + (size_t)(r.first + q) * a.ldx + c);
        else if (a.state_in && r.slot >= 0 && q + (int)a.W >= 1) v.fetch_plain(a.state_in + ((size_t)r.slot * (a.W - 1) + (a.W - 1 + q)) * a.D + c);
        v.open(x[k]);
    }
}

template <typename T, int V, int WT, bool EXACT>
__global__ void __launch_bounds__(kThreads) conv_kernel(const Conv<T> a) {
    sf_chain_enter();
    const Tiling& t = a.t;
    const uint32_t c = (blockIdx.x % t.cblocks * t.lanes + threadIdx.x % t.lanes) * V, per = kThreads / t.lanes;
    if (c >= a.D) return;
    const uint32_t W = EXACT ? WT : a.W;
    Ch<V, false> tap[WT], bias;
    load_taps(a.w, c, W, tap);
    load_bias(a.bias, c, bias);
    const uint64_t items = (uint64_t)a.q.n_seq * t.tiles;
    for (uint64_t it = (uint64_t)(blockIdx.x / t.cblocks) * per + threadIdx.x / t.lanes; it < items; it += (uint64_t)t.parts * per) {
        const uint32_t j = (uint32_t)(it / a.q.n_seq), s = (uint32_t)(it % a.q.n_seq);
        const Range r = range_of(a.q, s, a.st);
        const int p0 = (int)(j * t.tile), p1 = (int)min(r.len, (j + 1) * t.tile);
        if (p0 >= p1 && (j || !a.state_out)) continue;
        const T* xr = a.x + (size_t)r.first * a.ldx + c;
        Raw<T, V> next[kAheadF] = {};                          // rows on their way
#pragma unroll
        for (int u = 0; u < kAheadF; u++) if (p0 + u < p1) next[u].fetch(xr + (size_t)(p0 + u) * a.ldx);
        Ch<V, false> x[WT + kAheadF - 1];
        rows_before<T, V, WT>(a, r, p0, c, x);
        if (j == 0 && a.state_out && r.slot >= 0) {
            // The sequence's last W - 1 rows, which where it is shorter begin with rows of the state it started from.  The first tile writes them
            // all: it alone reads the old state, and a row from a later place than it goes to, so the pools may be one.
            T* so = a.state_out + (size_t)r.slot * (W - 1) * a.D + c;
            for (int i = 0; i + 1 < (int)W; i++) {
                const int q = (int)r.len - (int)(W - 1) + i;
                Raw<T, V> v = {};
                if (q >= 0) v.fetch(xr + (size_t)q * a.ldx);
                else if (a.state_in) v.fetch_plain(a.state_in + ((size_t)r.slot * (W - 1) + (W - 1 + q)) * a.D + c);
                *reinterpret_cast<decltype(v.w)*>(so + (size_t)i * a.D) = v.w;
            }
        }
        T* y = a.y + (size_t)(r.first + p0) * a.ldy + c;
        xr += (size_t)(p0 + kAheadF) * a.ldx;              // the rows after those on their way
        // kAheadF rows; ALL: they and as many more are there, so nothing is asked row by row
        auto rows = [&](auto all, int p) {
            constexpr bool ALL = decltype(all)::value;
#pragma unroll
            for (int u = 0; u < kAheadF; u++) next[u].open(x[WT - 1 + u]);
#pragma unroll
            for (int u = 0; u < kAheadF; u++) { if (ALL || p + kAheadF + u < p1) next[u].fetch(xr); xr += a.ldx; }
#pragma unroll
            for (int u = 0; u < kAheadF; u++) {
                if (ALL || p + u < p1) {
                    Ch<V, false> pre = bias;
#pragma unroll
                    for (int m = 0; m < WT; m++) if (EXACT || m < (int)W) pre.add_product(tap[m], x[WT - 1 + u - m]);
                    if (a.silu) pre.template silu<T>();
                    store(y, pre);
                }
                y += a.ldy;
            }
#pragma unroll
            for (int k = 0; k + 1 < WT; k++) x[k] = x[k + kAheadF];
        };
        int p = p0;
        for (; p + 2 * kAheadF <= p1; p += kAheadF) rows(std::true_type(), p);
        for (; p < p1; p += kAheadF) rows(std::false_type(), p);
    }
}

// Single rows (max_len 1): the state's rows are read once, moved up by one and written; several sequences on their way at once.  65,536 x 256 bf16 with states: 104 us, 41 of bytes:
// 16 warps an SM wait for their rows and for where those lie (issue 31 %, HBM 32 %).
template <typename T, int V, int WT, bool EXACT>
__global__ void __launch_bounds__(kThreads) conv_step_kernel(const Conv<T> a) {
    sf_chain_enter();
    constexpr int U = WT <= 4 ? 4 : 2;
    const Tiling& t = a.t;
    const uint32_t c = (blockIdx.x % t.cblocks * t.lanes + threadIdx.x % t.lanes) * V, per = kThreads / t.lanes;
    if (c >= a.D) return;
    const int H = (EXACT ? WT : (int)a.W) - 1;             // rows of a state; the last is at [WT - 2]
    Ch<V, false> tap[WT], bias;
    load_taps(a.w, c, a.W, tap);
    load_bias(a.bias, c, bias);
    const uint64_t stride = (uint64_t)t.parts * per;
    for (uint64_t s0 = (uint64_t)(blockIdx.x / t.cblocks) * per + threadIdx.x / t.lanes; s0 < a.q.n_seq; s0 += U * stride) {
        Range r[U];
        Raw<T, V> x[U] = {}, st[U][WT - 1] = {};
#pragma unroll
        for (int u = 0; u < U; u++) {
            r[u].len = 0; r[u].slot = -1;
            if (s0 + u * stride < a.q.n_seq) r[u] = range_of(a.q, (uint32_t)(s0 + u * stride), a.st);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (r[u].len) x[u].fetch(a.x + (size_t)r[u].first * a.ldx + c);
            if (a.state_in && r[u].slot >= 0) {
#pragma unroll
                for (int k = 0; k + 1 < WT; k++)
                    if (EXACT || k >= WT - 1 - H) st[u][k].fetch_plain(a.state_in + ((size_t)r[u].slot * H + (k - (WT - 1 - H))) * a.D + c);
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            const bool row = r[u].len > 0;
            if (row) {
                Ch<V, false> pre = bias, v;
                x[u].open(v);
                pre.add_product(tap[0], v);
#pragma unroll
                for (int m = 1; m < WT; m++) if (EXACT || m <= H) { st[u][WT - 1 - m].open(v); pre.add_product(tap[m], v); }
                if (a.silu) pre.template silu<T>();
                store(a.y + (size_t)r[u].first * a.ldy + c, pre);
            }
            if (a.state_out && r[u].slot >= 0) {
                T* so = a.state_out + (size_t)r[u].slot * H * a.D + c;
#pragma unroll
                for (int k = 0; k + 1 < WT; k++)
                    if (EXACT || k >= WT - 1 - H) *reinterpret_cast<decltype(x[u].w)*>(so + (size_t)(k - (WT - 1 - H)) * a.D) = !row ? st[u][k].w : (k + 2 < WT ? st[u][k + 2 < WT ? k + 1 : k].w : x[u].w);
            }
        }
    }
}

// The same walk with WT - 1 rows more at a tile's end: dx_o = sum_m tap[m] dpre_{o+m} is complete once dpre_{o+WT-1} is there.
template <typename T, int V, int WT, bool EXACT>
__global__ void __launch_bounds__(kThreads, WT <= 4 ? kBlocksB : 2) conv_backward_kernel(const Conv<T> a) {
    sf_chain_enter();
    typedef Ch<V, (V > 1)> C;
    extern __shared__ float sums[];                        // [threads][V][WT + 1] where the block joins its sums
    const Tiling& t = a.t;
    const uint32_t c = (blockIdx.x % t.cblocks * t.lanes + threadIdx.x % t.lanes) * V, per = kThreads / t.lanes;
    const uint32_t W = EXACT ? WT : a.W;
    C dw[WT], db;
#pragma unroll
    for (int m = 0; m < WT; m++) dw[m].zero();
    db.zero();
    if (c < a.D) {
        C tap[WT], bias;
        load_taps(a.w, c, W, tap);
        load_bias(a.bias, c, bias);
        const uint64_t items = (uint64_t)a.q.n_seq * t.tiles;
        for (uint64_t it = (uint64_t)(blockIdx.x / t.cblocks) * per + threadIdx.x / t.lanes; it < items; it += (uint64_t)t.parts * per) {
            const uint32_t j = (uint32_t)(it / a.q.n_seq), s = (uint32_t)(it % a.q.n_seq);
            const Range r = range_of(a.q, s, a.st);
            const int len = (int)r.len, H = (int)W - 1, p0 = (int)(j * t.tile), p1 = min(len, (int)((j + 1) * t.tile)), pe = min(len, p1 + H);
            const bool d0 = j == 0 && a.d_state0 && r.slot >= 0;
            if (p0 >= p1 && !d0) continue;
            const T* xr = a.x + (size_t)r.first * a.ldx + c;
            const T* gr = a.dy + (size_t)r.first * a.lddy + c;
            Raw<T, V> nx[kAheadB] = {}, ng[kAheadB] = {};
#pragma unroll
            for (int u = 0; u < kAheadB; u++) if (p0 + u < pe) { nx[u].fetch(xr + (size_t)(p0 + u) * a.ldx); ng[u].fetch(gr + (size_t)(p0 + u) * a.lddy); }
            C x[WT + kAheadB - 1], dp[WT + kAheadB - 1];
            rows_before<T, V, WT>(a, r, p0, c, x);
#pragma unroll
            for (int k = 0; k + 1 < WT; k++) dp[k].zero();
            xr += (size_t)(p0 + kAheadB) * a.ldx;
            gr += (size_t)(p0 + kAheadB) * a.lddy;
            T* out = a.dx + ((ptrdiff_t)r.first + p0 - (WT - 1)) * (ptrdiff_t)a.lddx + c;      // (used from row 0 on)
            // kAheadB rows; ALL: they and as many more are there, and so are the rows whose gradient is complete by them
            auto rows = [&](auto all, int p) {
                constexpr bool ALL = decltype(all)::value;
#pragma unroll
                for (int u = 0; u < kAheadB; u++) { nx[u].open(x[WT - 1 + u]); ng[u].open(dp[WT - 1 + u]); }
#pragma unroll
                for (int u = 0; u < kAheadB; u++) { if (ALL || p + kAheadB + u < pe) { nx[u].fetch(xr); ng[u].fetch(gr); } xr += a.ldx; gr += a.lddy; }
#pragma unroll
                for (int u = 0; u < kAheadB; u++) {
                    C& g = dp[WT - 1 + u];
                    if (a.silu) {
                        C pre = bias;
#pragma unroll
                        for (int m = 0; m < WT; m++) if (EXACT || m < (int)W) pre.add_product(tap[m], x[WT - 1 + u - m]);
                        g.template mul_silu_slope<T>(pre);
                    }
                    if (!ALL && p + u >= pe) g.zero();
                    if (ALL || p + u < p1) {
                        db.add(g);
#pragma unroll
                        for (int m = 0; m < WT; m++) if (EXACT || m < (int)W) dw[m].add_product(g, x[WT - 1 + u - m]);
                    }
                }
#pragma unroll
                for (int u = 0; u < kAheadB; u++, out += a.lddx) {
                    const int o = p + u - (WT - 1);        // the row whose gradient is complete now
                    if (ALL ? a.dx == nullptr : o >= p1 || (o >= p0 ? a.dx == nullptr : !d0 || o < -H)) continue;
                    C d;
                    d.set_product(tap[0], dp[u]);
#pragma unroll
                    for (int m = 1; m < WT; m++) if (EXACT || m < (int)W) d.add_product(tap[m], dp[u + m]);
                    if (!ALL && a.d_state && r.slot >= 0 && o >= len - H) {
                        Raw<T, V> v;
                        C e;
                        v.fetch_plain(a.d_state + ((size_t)r.slot * H + (o - (len - H))) * a.D + c);
                        v.open(e);
                        d.add(e);
                    }
                    if (ALL || o >= 0) store(out, d);
                    else store(a.d_state0 + ((size_t)r.slot * H + (o + H)) * a.D + c, d);
                }
#pragma unroll
                for (int k = 0; k + 1 < WT; k++) { x[k] = x[k + kAheadB]; dp[k] = dp[k + kAheadB]; }
            };
            int p = p0;
            for (; p < p0 + WT - 1 && p < p1 + WT - 1; p += kAheadB) rows(std::false_type(), p);
            for (; p + 2 * kAheadB <= p1; p += kAheadB) rows(std::true_type(), p);
            for (; p < p1 + WT - 1; p += kAheadB) rows(std::false_type(), p);
        }
    }
    if (!a.parts) return;
    // the block's threads on the same channels add up their sums, in the order of the threads
    constexpr int Q = (WT + 1) * V;
    float* mine = sums + (size_t)threadIdx.x * Q;
    float v[V];
#pragma unroll
    for (int m = 0; m <= WT; m++) {
        (m < WT ? dw[m < WT ? m : 0] : db).get(v);
#pragma unroll
        for (int i = 0; i < V; i++) mine[i * (WT + 1) + m] = v[i];
    }
    __syncthreads();
    const uint32_t n = t.lanes * V * (W + 1), c0 = blockIdx.x % t.cblocks * t.lanes * V;
    for (uint32_t e = threadIdx.x; e < n; e += kThreads) {
        const uint32_t ch = e / (W + 1), k = e % (W + 1);
        if (c0 + ch >= a.D) break;
        const float* p = sums + (size_t)(ch / V) * Q + (ch % V) * (WT + 1) + (k < W ? W - 1 - k : WT);
        float q = 0.0f;
        for (uint32_t y = 0; y < per; y++) q += p[(size_t)y * t.lanes * Q];
        a.parts[((size_t)(blockIdx.x / t.cblocks) * a.D + c0 + ch) * (W + 1) + k] = q;
    }
}

// The gradient of the states written over that of the states after the call (one pool).  conv_backward_kernel reads rows of the latter at the sequences' ends, in
// other blocks too, so there the pool is only written when it is done, by this kernel: row i of a state takes row i - len of the gradient it replaces, so a thread that goes
// from the last row to the first never reads what it has written.
template <typename T, int V, int WT, bool EXACT>
__global__ void __launch_bounds__(kThreads) conv_state_backward_kernel(const Conv<T> a) {
    sf_chain_enter();
    typedef Ch<V, (V > 1)> C;
    const Tiling& t = a.t;
    const uint32_t c = (blockIdx.x % t.cblocks * t.lanes + threadIdx.x % t.lanes) * V, per = kThreads / t.lanes;
    if (c >= a.D) return;
    const uint32_t W = EXACT ? WT : a.W;
    const int H = (int)W - 1;
    C tap[WT], bias;
    load_taps(a.w, c, W, tap);
    load_bias(a.bias, c, bias);
    for (uint64_t s = (uint64_t)(blockIdx.x / t.cblocks) * per + threadIdx.x / t.lanes; s < a.q.n_seq; s += (uint64_t)t.parts * per) {
        const Range r = range_of(a.q, (uint32_t)s, a.st);
        if (r.slot < 0) continue;
        const int len = (int)r.len, rows = min(len, H);        // rows that reach back into the state
        C x[2 * WT - 2], dp[WT - 1];
        rows_before<T, V, WT>(a, r, 0, c, x);
#pragma unroll
        for (int u = 0; u + 1 < WT; u++) {
            Raw<T, V> nx = {}, ng = {};
            if (u < rows) { nx.fetch(a.x + (size_t)(r.first + u) * a.ldx + c); ng.fetch(a.dy + (size_t)(r.first + u) * a.lddy + c); }
            nx.open(x[WT - 1 + u]); ng.open(dp[u]);
        }
        if (a.silu) {
#pragma unroll
            for (int u = 0; u + 1 < WT; u++) {
                C pre = bias;
#pragma unroll
                for (int m = 0; m < WT; m++) if (EXACT || m < (int)W) pre.add_product(tap[m], x[WT - 1 + u - m]);
                dp[u].template mul_silu_slope<T>(pre);
                if (u >= rows) dp[u].zero();
            }
        }
        T* state = a.d_state0 + (size_t)r.slot * H * a.D + c;
#pragma unroll
        for (int k = WT - 2; k >= 0; k--) {
            const int o = k - (WT - 1), i = o + H;             // row -1, -2, .. of the sequence, row i of its state
            if (!EXACT && i < 0) continue;
            C d;
            d.zero();
#pragma unroll
            for (int m = 1; m < WT; m++) if (o + m >= 0 && (EXACT || m < (int)W)) d.add_product(tap[m], dp[o + m >= 0 ? o + m : 0]);
            if (i >= len) {
                Raw<T, V> v;
                C e;
                v.fetch_plain(state + (size_t)(i - len) * a.D);
                v.open(e);
                d.add(e);
            }
            store(state + (size_t)i * a.D, d);
        }
    }
}

// dw[c][k] and db[c] from the blocks' sums: 32 values a block, a warp takes every eighth sum of each
__global__ void __launch_bounds__(256) conv_join_kernel(const float* __restrict__ parts, uint32_t n_parts, uint32_t D, uint32_t W, float* dw, float* db) {
    sf_chain_enter();
    __shared__ float sh[8][32];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, e = blockIdx.x * 32 + lane, n = D * (W + 1);
    float v = 0.0f;
    if (e < n) {
#pragma unroll 8
        for (uint32_t p = warp; p < n_parts; p += 8) v += parts[(size_t)p * n + e];
    }
    sh[warp][lane] = v;
    __syncthreads();
    if (warp || e >= n) return;
#pragma unroll
    for (int i = 1; i < 8; i++) v += sh[i][lane];
    const uint32_t c = e / (W + 1), k = e % (W + 1);
    if (k < W) { if (dw) dw[(size_t)c * W + k] = v; }
    else if (db) db[c] = v;
}

// ---- host ----------------------------------------------------------------------------------------------------------
uint32_t word_of(const void* p, size_t ld, uint32_t size) {          // the widest access (16, 8, 4 or 2 bytes) on which every row begins
    const uint64_t v = (uint64_t)(uintptr_t)p | (uint64_t)ld * size;
    return v % 16 == 0 ? 16 : (v % 8 == 0 ? 8 : (v % 4 == 0 ? 4 : 2));
}

// Tiles of 128 rows, shorter (down to 8) while the sequences are too few to fill the machine with those; threads over tiles in turn once the
// machine is full (`resident` blocks an SM).
Tiling tiling(const sf_sequences* q, uint32_t D, uint32_t V, uint32_t resident) {
    Tiling t;
    const uint32_t units = (D + V - 1) / V;
    t.lanes = 1;
    while (t.lanes < kThreads && t.lanes < units) t.lanes *= 2;
    t.cblocks = (units + t.lanes - 1) / t.lanes;
    const uint64_t full = (uint64_t)SF_NUM_SMS_DEFAULT * resident;
    t.tile = 128;
    while (t.tile > 8 && (uint64_t)q->n_seq * ((q->max_len + t.tile - 1) / t.tile) * units < full * kThreads) t.tile /= 2;
    t.tiles = (q->max_len + t.tile - 1) / t.tile;
    const uint32_t per = kThreads / t.lanes;
    const uint64_t blocks = ((uint64_t)q->n_seq * t.tiles + per - 1) / per;
    t.parts = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(blocks, std::max<uint64_t>(1, full / t.cblocks)));
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
    if (size == 2 && MOST > 4 && word >= 4) return f(std::integral_constant<int, 4 / size>());
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
    const uint32_t size = type_bytes(dtype);
    if (overlap_in_part(state_in, state_out, (size_t)n_slots * (W - 1) * D * size)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    const uint32_t word = std::min({word_of(x, ldx, size), word_of(y_out, ldy, size), word_of(state_in, D, size), word_of(state_out, D, size), word_of(nullptr, D, size)});
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_width<T, (sizeof(T) == 2 ? 8 : 16)>(word, [&](auto v) {
            return by_taps(W, [&](auto taps, auto exact) {
                constexpr int V = decltype(v)::value, WT = decltype(taps)::value;
                Conv<T> a = {};
                a.q = seqs_of(seq, rows, n_slots); a.x = (const T*)x; a.ldx = ldx; a.w = w; a.bias = bias; a.D = D; a.W = W; a.silu = act == SF_ACT_SILU;
                a.state_in = (const T*)state_in; a.state_out = (T*)state_out; a.y = (T*)y_out; a.ldy = ldy; a.st = ctx->d_state;
                if (seq->max_len == 1) {
                    a.t = tiling(seq, D, V, 8);
                    SF_CUDA(sf_launch_chained(conv_step_kernel<T, V, WT, decltype(exact)::value>, a.t.cblocks * a.t.parts, kThreads, 0, (cudaStream_t)stream, a));
                    return (int)SF_OK;
                }
                a.t = tiling(seq, D, V, 32);
                SF_CUDA(sf_launch_chained(conv_kernel<T, V, WT, decltype(exact)::value>, a.t.cblocks * a.t.parts, kThreads, 0, (cudaStream_t)stream, a));
                return (int)SF_OK;
            });
        });
    });
}

extern "C" int sf_seq_conv_backward_workspace(uint32_t n_seq, uint32_t max_len, uint32_t D, uint32_t W, size_t* bytes_out)
{
    if (!bytes_out || n_seq > SF_SEQ_MAX_ROWS || max_len == 0 || max_len > SF_SEQ_MAX_ROWS || D == 0 || D > SF_EXPERT_MAX_D || W == 0 || W > kMaxTaps) return SF_ERR_ARG;
    const sf_sequences q = {nullptr, nullptr, nullptr, n_seq, max_len};
    uint32_t parts = 1;
    for (uint32_t v : {1u, 2u, 4u}) parts = std::max(parts, tiling(&q, D, v, kBlocksB).parts);
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
    const size_t pool = (size_t)n_slots * (W - 1) * D * size;
    if (overlap_in_part(d_state, d_state_in_out, pool) || overlap_in_part(state_in, d_state_in_out, pool)) return SF_ERR_ARG;
    const bool one_pool = d_state && d_state == d_state_in_out;
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
                a.state_in = (const T*)state_in; a.dy = (const T*)dy; a.lddy = lddy; a.d_state = (const T*)d_state; a.d_state0 = one_pool ? nullptr : (T*)d_state_in_out;
                a.dx = (T*)dx_out; a.lddx = lddx; a.st = ctx->d_state;
                a.t = tiling(seq, D, V, kBlocksB);
                if (sums && (!workspace || workspace_bytes < (size_t)a.t.parts * D * (W + 1) * 4)) return (int)SF_ERR_ARG;
                a.parts = sums ? (float*)workspace : nullptr;
                if (sums || dx_out || !one_pool)
                    SF_CUDA(sf_launch_chained(conv_backward_kernel<T, V, WT, decltype(exact)::value>, a.t.cblocks * a.t.parts, kThreads, sums ? kThreads * (WT + 1) * V * 4 : 0,
                                              (cudaStream_t)stream, a));
                if (sums) SF_CUDA(sf_launch_chained(conv_join_kernel, (D * (W + 1) + 31) / 32, 256, 0, (cudaStream_t)stream, (const float*)workspace, a.t.parts, D, W, dw_out, dbias_out));
                if (one_pool && seq->n_seq) {
                    sf_sequences ends = *seq;
                    ends.max_len = 1;                      // (one item a sequence)
                    a.t = tiling(&ends, D, V, kBlocksB);
                    a.d_state0 = (T*)d_state_in_out;
                    SF_CUDA(sf_launch_chained(conv_state_backward_kernel<T, V, WT, decltype(exact)::value>, a.t.cblocks * a.t.parts, kThreads, 0, (cudaStream_t)stream, a));
                }
                return (int)SF_OK;
            });
        });
    });
}
