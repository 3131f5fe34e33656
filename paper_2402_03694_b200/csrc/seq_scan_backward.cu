// Backward pass of the selective state space scan (formulas and mapping: seq_scan.cuh).
#include "seq_scan.cuh"

namespace {

using namespace sfscan;

constexpr int K = (int)kEvery;             // rows of a tile
constexpr int R = 4;                       // rows whose decays and states a thread holds at once

// What a warp keeps in shared memory.  Sums over states (s1, s2, y) and over channels (dbc) are left as one part a lane, for R rows, and joined where they are
// used; rows are spaced so that the 16-byte accesses of eight lanes meet no common bank.
template <typename T, int SL, int VV, int PB> struct __align__(16) Backward {
    typedef Shape<SL> S;
    typedef Pieces<K, S::CH, VV> P;
    typedef States<T, PB, K, S::NP> ST;
    static constexpr int PX = S::CH + 4, PY = S::CH + (SL == 1 ? 0 : (SL == 2 ? 16 : (SL == 4 ? 8 : 4))), PT = SL * PY + 4;
    static constexpr int ON_WAY = VV > 1 ? 4 * P::I + ST::I : 1;
    float step[K][PX], u[K][PX], e[K][PX];                 // delta; u; dout silu(z)
    float dstep[K][PX], dgate[K][PX];                      // d delta / d raw; dout silu'(z)
    float bc[2][K][S::NP];                                 // B, C
    float s1[R][PT], s2[R][PT], y[R][PT];                  // sum g B; sum (a g) h_{t-1} A; sum C h
    float dbc[R][2][S::CL][S::NP];                         // dB, dC
    float4 start[K / R][4][32];                            // the states before rows 0 and R by channel, every lane its own
    uint4 way[ON_WAY][32];                                 // the next tile's pieces on their way, every lane its own
    float bias[S::CH], skip[S::CH];
};

// Asks for a tile's pieces: steps, gradients of the outputs, gates, and (not ENDS) inputs.  Whole pieces only; others are read when staged.
template <typename T, int SL, int VV, int PB, bool ENDS>
__device__ __forceinline__ void ask(const Scan& a, Backward<T, SL, VV, PB>& sh, size_t row0, uint32_t ch0, uint32_t have, uint32_t g, int rows, int lane) {
    if constexpr (VV > 1) {
        typedef Backward<T, SL, VV, PB> Sh;
        typedef typename Sh::P P;
        const P pc(lane);
        const size_t at = row0 + pc.lt;
        const T* from[4] = {(const T*)a.delta, (const T*)a.dy, (const T*)a.z, (const T*)a.u};
        const size_t ld[4] = {a.lddelta, a.lddy, a.ldz, a.ldu};
#pragma unroll
        for (int k = 0; k < 4; k++) {
            if (k == 2 ? a.z == nullptr : (k == 3 && ENDS)) continue;
#pragma unroll
            for (int i = 0; i < P::I; i++) {
                const bool there = pc.t(i) < rows && pc.c(i) < (int)have;
                copy16(&sh.way[k * P::I + i][lane], there ? from[k] + at * ld[k] + ch0 + pc.lc + P::step(i, ld[k]) : from[k], there);
            }
        }
        if constexpr (Sh::ST::WHOLE) {
#pragma unroll
            for (int i = 0; i < Sh::ST::I; i++) {
                bool there;
                const T* p = Sh::ST::template piece<T>(a, i, row0, g * a.N, rows, lane, there);
                copy16(&sh.way[4 * P::I + i][lane], p, there);
            }
        }
    }
}
// The state before a tile into start[0], likewise; four by four where states lie so
template <typename T, int SL, int VV, int PB>
__device__ __forceinline__ void ask_start(const Scan& a, Backward<T, SL, VV, PB>& sh, size_t start, uint32_t ch0, uint32_t have, int lane) {
    const int cl = lane / SL, sl = lane % SL;
    const float* p = a.starts + start * a.D * a.N;
    const bool fours = Backward<T, SL, VV, PB>::ST::WHOLE || (a.n4 && ((uintptr_t)p & 15u) == 0);      // (whole pieces of states: N is a multiple of 4)
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const bool there = cl * 4 + j < (int)have;
        const float* q = p + (size_t)(ch0 + cl * 4 + j) * a.N + sl * 4;
        if (fours) copy16(&sh.start[0][j][lane], there && sl * 4 < (int)a.N ? q : p, there && sl * 4 < (int)a.N);
        else {
#pragma unroll
            for (int n = 0; n < 4; n++) copy4(&reinterpret_cast<float*>(&sh.start[0][j][lane])[n], there && sl * 4 + n < (int)a.N ? q + n : p, there && sl * 4 + n < (int)a.N);
        }
    }
}

// stages steps, inputs and gradients of the rows t0 .. t0 + K - 1 as far as there (zeros behind: they then change nothing); ENDS: what the pass for the parts' ends needs
template <typename T, int SL, int VV, int PB, bool ENDS>
__device__ __forceinline__ void stage(const Scan& a, Backward<T, SL, VV, PB>& sh, size_t row0, uint32_t ch0, uint32_t have, uint32_t g, int rows, int lane) {
    typedef Backward<T, SL, VV, PB> Sh;
    typedef typename Sh::P P;
    const P pc(lane);
    Piece<T, VV> nd[P::I], nu[P::I], nz[P::I], ng[P::I];
    typename Sh::ST ns;
    if constexpr (VV > 1 && !Sh::ST::WHOLE) ns.fetch_all(a, row0, g * a.N, rows, lane);
    copies_done();
    if constexpr (VV > 1) {
#pragma unroll
        for (int i = 0; i < P::I; i++) {
            nd[i].w = sh.way[i][lane];
            ng[i].w = sh.way[P::I + i][lane];
            if (a.z) nz[i].w = sh.way[2 * P::I + i][lane];
            if (!ENDS) nu[i].w = sh.way[3 * P::I + i][lane];
        }
        if constexpr (Sh::ST::WHOLE) {
#pragma unroll
            for (int i = 0; i < Sh::ST::I; i++) ns.take(i, sh.way[4 * P::I + i][lane]);
        }
    } else {
        const size_t at = row0 + pc.lt;
        const T* pd = (const T*)a.delta + at * a.lddelta + ch0 + pc.lc; const T* pu = (const T*)a.u + at * a.ldu + ch0 + pc.lc;
        const T* pz = (const T*)a.z + at * a.ldz + ch0 + pc.lc; const T* pg = (const T*)a.dy + at * a.lddy + ch0 + pc.lc;
#pragma unroll
        for (int i = 0; i < P::I; i++) {
            const bool there = pc.t(i) < rows && pc.c(i) < (int)have;
            nd[i] = fetch<T, VV>(pd, P::step(i, a.lddelta), there);
            if (!ENDS) nu[i] = fetch<T, VV>(pu, P::step(i, a.ldu), there);
            if (a.z) nz[i] = fetch<T, VV>(pz, P::step(i, a.ldz), there);
            ng[i] = fetch<T, VV>(pg, P::step(i, a.lddy), there);
        }
        ns.fetch_all(a, row0, g * a.N, rows, lane);
    }
    constexpr int AT = VV == 1 ? 2 : 1, W = VV * AT;       // single elements two at a time
    static_assert(P::I % AT == 0, "every lane has an even number of single elements");
#pragma unroll
    for (int i = 0; i < P::I; i += AT) {
        if (pc.t(i) >= K) continue;
        float d[W], u[W], z[W], o[W], ds[W], dg[W];
        f2 bias[W / 2];
        auto opened = [&](const Piece<T, VV>* n, float (&x)[W]) {
#pragma unroll
            for (int k = 0; k < AT; k++) {
                float v[VV];
                open<T, VV>(n[i + k], v);
#pragma unroll
                for (int e = 0; e < VV; e++) x[k * VV + e] = v[e];
            }
        };
        opened(nd, d);
        if (!ENDS) opened(nu, u);
        if (a.z) opened(nz, z);
        opened(ng, o);
        if constexpr (VV == 1) bias[0] = pack2(sh.bias[pc.c(i)], sh.bias[pc.c(i + 1)]);
        else {
#pragma unroll
            for (int e = 0; e < VV; e += 2) bias[e / 2] = *reinterpret_cast<const f2*>(&sh.bias[pc.c(i) + e]);
        }
#pragma unroll
        for (int e = 0; e < W; e += 2) {
            const f2 one = dup2(1.0f);
            f2 raw = add2(pack2(d[e], d[e + 1]), bias[e / 2]), x, v = raw, w = one;
            if (a.softplus) {                              // x is exp(-|raw|): the slope of softplus is 1 / (1 + x), or x / (1 + x) left of 0
                v = softplus2(raw, x);
                float p, q, r0, r1;
                unpack2(add2(x, one), p, q);
                unpack2(raw, r0, r1);
                if (!ENDS) { float x0, x1; unpack2(x, x0, x1); w = mul2(pack2(r0 >= 0.0f ? 1.0f : x0, r1 >= 0.0f ? 1.0f : x1), pack2(rcp(p), rcp(q))); }
            }
            unpack2(v, d[e], d[e + 1]);
            unpack2(w, ds[e], ds[e + 1]);
            if (a.z) {
                const f2 zz = pack2(z[e], z[e + 1]), oo = pack2(o[e], o[e + 1]), sg = sigmoid2<T>(zz), os = mul2(oo, sg);
                if (!ENDS) unpack2(mul2(os, fma2(zz, fma2(sg, dup2(-1.0f), one), one)), dg[e], dg[e + 1]);
                unpack2(mul2(os, zz), o[e], o[e + 1]);
            }
        }
#pragma unroll
        for (int k = 0; k < AT; k++) {
            const int t = pc.t(i + k), c = pc.c(i + k);
            const bool there = t < rows && c < (int)have;
            if (!there) {
#pragma unroll
                for (int e = 0; e < VV; e++) d[k * VV + e] = o[k * VV + e] = 0.0f;
            }
            auto put = [&](float* p, const float (&v)[W]) {
                if constexpr (VV == 1) p[0] = v[k];
                else {
#pragma unroll
                    for (int e = 0; e < VV; e += 4) *reinterpret_cast<float4*>(p + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                }
            };
            put(&sh.step[t][c], d);
            put(&sh.e[t][c], o);
            if (!ENDS) { put(&sh.u[t][c], u); put(&sh.dstep[t][c], ds); if (a.z) put(&sh.dgate[t][c], dg); }
        }
    }
    ns.stage(&sh.bc[0][0][0], lane);
}

template <typename T, int SL, int VV, int PB> __device__ __forceinline__ void channel_params(const Scan& a, Backward<T, SL, VV, PB>& sh, uint32_t ch0, uint32_t have, int lane) {
    for (int c = lane; c < Shape<SL>::CH; c += 32) {
        sh.bias[c] = c < (int)have && a.dbias ? __ldg(a.dbias + ch0 + c) : 0.0f;
        sh.skip[c] = c < (int)have && a.Dk ? __ldg(a.Dk + ch0 + c) : 0.0f;
    }
}
// the lane's 4 x 4 values of an array [channel][state], channels 2 j and 2 j + 1 side by side
__device__ __forceinline__ void load_states(f2 (&v)[2][4], const float* p, const Scan& a, uint32_t ch0, uint32_t have, int cl, int sl, float scale) {
#pragma unroll
    for (int j = 0; j < 2; j++) {
        float x[2][4];
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const uint32_t c = cl * 4 + 2 * j + k;
            const float* q = p + (size_t)(ch0 + c) * a.N + sl * 4;
#pragma unroll
            for (int n = 0; n < 4; n++) x[k][n] = 0.0f;
            if (p && c < have) {
                if (a.n4 && ((uintptr_t)q & 15u) == 0) { if (sl * 4 < (int)a.N) { const float4 w = *reinterpret_cast<const float4*>(q); x[k][0] = w.x; x[k][1] = w.y; x[k][2] = w.z; x[k][3] = w.w; } }
                else {
#pragma unroll
                    for (int n = 0; n < 4; n++) if (sl * 4 + n < (int)a.N) x[k][n] = q[n];
                }
            }
        }
#pragma unroll
        for (int n = 0; n < 4; n++) v[j][n] = pack2(x[0][n] * scale, x[1][n] * scale);
    }
}
__device__ __forceinline__ void store_states(const f2 (&v)[2][4], float* p, size_t ld, const Scan& a, uint32_t ch0, uint32_t have, int cl, int sl) {
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int n = 0; n < 4; n++) {
            float x, y;
            unpack2(v[j][n], x, y);
            const uint32_t c = cl * 4 + 2 * j;
            if (sl * 4 + n >= (int)a.N) continue;
            if (c < have) p[(size_t)(ch0 + c) * ld + sl * 4 + n] = x;
            if (c + 1 < have) p[(size_t)(ch0 + c + 1) * ld + sl * 4 + n] = y;
        }
}

// Parts: the gradient at a part's first state that the part's own rows cause, and the sum of its steps.
template <typename T, int SL, int VV, int PB>
__global__ void __launch_bounds__(32 * kWarps) back_ends_kernel(const Scan a) {
    sf_chain_enter();
    constexpr int CH = Shape<SL>::CH;
    extern __shared__ __align__(16) unsigned char shared[];
    Backward<T, SL, VV, PB>& sh = reinterpret_cast<Backward<T, SL, VV, PB>*>(shared)[threadIdx.x / 32];
    const int lane = threadIdx.x & 31, cl = lane / SL, sl = lane % SL;
    const Item it = item_of(a, CH);
    if (it.have == 0) return;
    const uint32_t s = it.s, g = it.g, ch0 = it.ch0, have = it.have;
    const Range r = range_of(a.q, s, a.st);
    const uint32_t part = blockIdx.y, t_begin = part * a.part_len, t_end = min(r.len, t_begin + a.part_len);
    if (t_begin >= r.len) return;
    f2 A[2][4], G[2][4], steps[2] = {0, 0};
    load_states(A, a.A, a, ch0, have, cl, sl, kLog2e);
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int n = 0; n < 4; n++) G[j][n] = 0;
    channel_params<T, SL, VV, PB>(a, sh, ch0, have, lane);
    __syncwarp();
    const uint32_t tiles = (t_end - t_begin + K - 1) / K;
    auto next = [&](uint32_t tile) { const uint32_t t = t_begin + tile * K; ask<T, SL, VV, PB, true>(a, sh, (size_t)r.first + t, ch0, have, g, (int)min((uint32_t)K, t_end - t), lane); };
    next(tiles - 1);
    for (uint32_t tile = tiles; tile-- > 0;) {
        const uint32_t t0 = t_begin + tile * K;
        stage<T, SL, VV, PB, true>(a, sh, (size_t)r.first + t0, ch0, have, g, (int)min((uint32_t)K, t_end - t0), lane);
        if (tile) next(tile - 1);
        __syncwarp();
#pragma unroll
        for (int t = K - 1; t >= 0; t--) {
            const ulonglong2 d2 = *reinterpret_cast<const ulonglong2*>(&sh.step[t][cl * 4]), e2 = *reinterpret_cast<const ulonglong2*>(&sh.e[t][cl * 4]);
            const float4 c4 = *reinterpret_cast<const float4*>(&sh.bc[1][t][sl * 4]);
            const f2 d[2] = {d2.x, d2.y}, e[2] = {e2.x, e2.y}, c[4] = {dup2(c4.x), dup2(c4.y), dup2(c4.z), dup2(c4.w)};
#pragma unroll
            for (int j = 0; j < 2; j++) {
                steps[j] = add2(steps[j], d[j]);
#pragma unroll
                for (int n = 0; n < 4; n++) G[j][n] = mul2(decay2(d[j], A[j][n]), fma2(e[j], c[n], G[j][n]));
            }
        }
        __syncwarp();
    }
    store_states(G, a.part_state + ((size_t)s * a.parts + part) * a.D * a.N, a.N, a, ch0, have, cl, sl);
    if (sl == 0) {
#pragma unroll
        for (int j = 0; j < 2; j++) {
            float x, y;
            unpack2(steps[j], x, y);
            float* p = a.part_step + ((size_t)s * a.parts + part) * a.D + ch0 + cl * 4 + 2 * j;
            if (cl * 4 + 2 * j < (int)have) p[0] = x;
            if (cl * 4 + 2 * j + 1 < (int)have) p[1] = y;
        }
    }
}

// One block: up to kWarps warps over neighbouring channels of a group, one part of one sequence after the other (a run), rows from last to first.
// A tile's states are stepped from the state kept before it: rows 0 to 3 to reach row 4, rows 4 to 7 with decays and states held in registers, back over
// them, then rows 0 to 3 the same way.
template <typename T, int SL, int VV, int PB>
__global__ void __launch_bounds__(32 * kWarps, 2) back_kernel(const Scan a) {
    sf_chain_enter();
    typedef Shape<SL> S;
    typedef Backward<T, SL, VV, PB> Sh;
    constexpr int CH = S::CH, CL = S::CL, VE = VV > 1 ? 4 : 1;
    typedef Pieces<R, CH, VE> P;                           // as rows are written: R at a time, 4 channels a piece
    constexpr int I = P::I;
    extern __shared__ __align__(16) unsigned char shared[];
    Sh* all = reinterpret_cast<Sh*>(shared);
    const int warp = threadIdx.x / 32, warps = blockDim.x / 32;
    Sh& sh = all[warp];
    const int lane = threadIdx.x & 31, cl = lane / SL, sl = lane % SL;
    const uint32_t gb = blockIdx.x, g = gb / a.cblocks, cb = gb % a.cblocks;
    const uint32_t c0 = min(a.per, (cb * (uint32_t)kWarps + warp) * CH);
    const uint32_t ch0 = g * a.per + c0, have = min((uint32_t)CH, a.per - c0);     // (a warp behind the group's last channel has none, but meets the others)
    const P pc(lane);
    f2 A[2][4], dA[2][4], G[2][4];
    load_states(A, a.A, a, ch0, have, cl, sl, kLog2e);
    float dD[I][VE], db[I][VE];                            // of the channels that this lane's pieces have
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int n = 0; n < 4; n++) dA[j][n] = 0;
#pragma unroll
    for (int i = 0; i < I; i++)
#pragma unroll
        for (int e = 0; e < VE; e++) dD[i][e] = db[i][e] = 0.0f;
    channel_params<T, SL, VV, PB>(a, sh, ch0, have, lane);
    __syncwarp();
    const size_t DN = (size_t)a.D * a.N;
    const uint64_t items = (uint64_t)a.q.n_seq * a.parts;
    for (uint64_t it = blockIdx.y; it < items; it += a.runs) {
        const uint32_t part = (uint32_t)(it / a.q.n_seq), s = (uint32_t)(it % a.q.n_seq);
        const Range r = range_of(a.q, s, a.st);
        const uint32_t t_begin = part * a.part_len, t_end = min(r.len, t_begin + a.part_len);
        const bool whole = a.part_state == nullptr;        // the sequence in one part: gradients of states here
        if (t_begin >= r.len && !(whole && a.d_state0 && r.slot >= 0)) continue;
        const uint32_t tiles = t_end > t_begin ? (t_end - t_begin + K - 1) / K : 0;
        auto next = [&](uint32_t tile) {
            const uint32_t t = t_begin + tile * K;
            ask<T, SL, VV, PB, false>(a, sh, (size_t)r.first + t, ch0, have, g, (int)min((uint32_t)K, t_end - t), lane);
        };
        auto next_start = [&](uint32_t tile) { ask_start<T, SL, VV, PB>(a, sh, start_index(r.first, s, t_begin + tile * K), ch0, have, lane); };
        if (tiles) { next(tiles - 1); next_start(tiles - 1); }
        load_states(G, whole ? (a.d_state && r.slot >= 0 ? a.d_state + (size_t)r.slot * DN : nullptr) : a.part_state + ((size_t)s * a.parts + part) * DN, a, ch0, have, cl, sl, 1.0f);
        for (uint32_t tile = tiles; tile-- > 0;) {
            const uint32_t t0 = t_begin + tile * K;
            const int rows = (int)min((uint32_t)K, t_end - t0);
            const size_t row0 = (size_t)r.first + t0;
            stage<T, SL, VV, PB, false>(a, sh, row0, ch0, have, g, rows, lane);
            f2 h[2][4];
            auto keep = [&](int q) {
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    float x[4], y[4];
#pragma unroll
                    for (int n = 0; n < 4; n++) unpack2(h[j][n], x[n], y[n]);
                    sh.start[q][2 * j][lane] = make_float4(x[0], x[1], x[2], x[3]);
                    sh.start[q][2 * j + 1][lane] = make_float4(y[0], y[1], y[2], y[3]);
                }
            };
            auto take = [&](f2 (&v)[2][4], int q) {
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const float4 x = sh.start[q][2 * j][lane], y = sh.start[q][2 * j + 1][lane];
                    v[j][0] = pack2(x.x, y.x); v[j][1] = pack2(x.y, y.y); v[j][2] = pack2(x.z, y.z); v[j][3] = pack2(x.w, y.w);
                }
            };
            take(h, 0);
            if (tile) next(tile - 1);                      // (what this lane had on its way it has read)
            __syncwarp();
#pragma unroll
            for (int t = 0; t < R; t++) {
                const ulonglong2 d2 = *reinterpret_cast<const ulonglong2*>(&sh.step[t][cl * 4]), u2 = *reinterpret_cast<const ulonglong2*>(&sh.u[t][cl * 4]);
                const float4 b4 = *reinterpret_cast<const float4*>(&sh.bc[0][t][sl * 4]);
                const f2 d[2] = {d2.x, d2.y}, in[2] = {mul2(d2.x, u2.x), mul2(d2.y, u2.y)}, b[4] = {dup2(b4.x), dup2(b4.y), dup2(b4.z), dup2(b4.w)};
#pragma unroll
                for (int j = 0; j < 2; j++)
#pragma unroll
                    for (int n = 0; n < 4; n++) h[j][n] = fma2(decay2(d[j], A[j][n]), h[j][n], mul2(in[j], b[n]));
            }
            keep(1);
#pragma unroll 1
            for (int q = K / R - 1; q >= 0; q--) {
                f2 al[R][2][4], hs[R + 1][2][4];           // decays; states before the rows and after them
                take(hs[0], q);
                if (q == 0 && tile) next_start(tile - 1);  // (this lane's is in registers now)
#pragma unroll
                for (int t = 0; t < R; t++) {
                    const int tt = R * q + t;
                    const ulonglong2 d2 = *reinterpret_cast<const ulonglong2*>(&sh.step[tt][cl * 4]), u2 = *reinterpret_cast<const ulonglong2*>(&sh.u[tt][cl * 4]);
                    const float4 b4 = *reinterpret_cast<const float4*>(&sh.bc[0][tt][sl * 4]);
                    const f2 d[2] = {d2.x, d2.y}, in[2] = {mul2(d2.x, u2.x), mul2(d2.y, u2.y)}, b[4] = {dup2(b4.x), dup2(b4.y), dup2(b4.z), dup2(b4.w)};
#pragma unroll
                    for (int j = 0; j < 2; j++)
#pragma unroll
                        for (int n = 0; n < 4; n++) { al[t][j][n] = decay2(d[j], A[j][n]); hs[t + 1][j][n] = fma2(al[t][j][n], hs[t][j][n], mul2(in[j], b[n])); }
                }
#pragma unroll
                for (int t = R - 1; t >= 0; t--) {
                    const int tt = R * q + t;
                    const ulonglong2 d2 = *reinterpret_cast<const ulonglong2*>(&sh.step[tt][cl * 4]), u2 = *reinterpret_cast<const ulonglong2*>(&sh.u[tt][cl * 4]), e2 = *reinterpret_cast<const ulonglong2*>(&sh.e[tt][cl * 4]);
                    const float4 b4 = *reinterpret_cast<const float4*>(&sh.bc[0][tt][sl * 4]), c4 = *reinterpret_cast<const float4*>(&sh.bc[1][tt][sl * 4]);
                    const f2 d[2] = {d2.x, d2.y}, in[2] = {mul2(d2.x, u2.x), mul2(d2.y, u2.y)}, e[2] = {e2.x, e2.y};
                    const f2 b[4] = {dup2(b4.x), dup2(b4.y), dup2(b4.z), dup2(b4.w)}, c[4] = {dup2(c4.x), dup2(c4.y), dup2(c4.z), dup2(c4.w)};
                    f2 dB[4], dC[4], s1[2], s2[2], y[2];
#pragma unroll
                    for (int j = 0; j < 2; j++)
#pragma unroll
                        for (int n = 0; n < 4; n++) {
                            const f2 gt = fma2(e[j], c[n], G[j][n]);
                            dB[n] = j ? fma2(gt, in[j], dB[n]) : mul2(gt, in[j]);
                            dC[n] = j ? fma2(e[j], hs[t + 1][j][n], dC[n]) : mul2(e[j], hs[t + 1][j][n]);
                            s1[j] = n ? fma2(gt, b[n], s1[j]) : mul2(gt, b[n]);
                            G[j][n] = mul2(gt, al[t][j][n]);
                            const f2 x = mul2(G[j][n], hs[t][j][n]);
                            s2[j] = n ? fma2(x, A[j][n], s2[j]) : mul2(x, A[j][n]);
                            dA[j][n] = fma2(x, d[j], dA[j][n]);
                            y[j] = n ? fma2(hs[t + 1][j][n], c[n], y[j]) : mul2(hs[t + 1][j][n], c[n]);
                        }
                    const int at = sl * Sh::PY + cl * 4;
                    *reinterpret_cast<ulonglong2*>(&sh.s1[t][at]) = make_ulonglong2(s1[0], s1[1]);
                    *reinterpret_cast<ulonglong2*>(&sh.s2[t][at]) = make_ulonglong2(s2[0], s2[1]);
                    if (a.z) *reinterpret_cast<ulonglong2*>(&sh.y[t][at]) = make_ulonglong2(y[0], y[1]);
                    float v[8];
#pragma unroll
                    for (int n = 0; n < 4; n++) {
                        float x, w;
                        unpack2(dB[n], x, w); v[n] = x + w;
                        unpack2(dC[n], x, w); v[4 + n] = x + w;
                    }
                    *reinterpret_cast<float4*>(&sh.dbc[t][0][cl][sl * 4]) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<float4*>(&sh.dbc[t][1][cl][sl * 4]) = make_float4(v[4], v[5], v[6], v[7]);
                }
                __syncthreads();
                const int left = rows - R * q;             // rows of the group that are there
                const size_t at = row0 + R * q + pc.lt;
#pragma unroll
                for (int i = 0; i < I; i++) {
                    const int t = pc.t(i), tt = R * q + t, c = pc.c(i);
                    if (t >= R || t >= left || c >= (int)have) continue;
                    float du[VE], dd[VE], dz[VE];
                    float s1[VE], s2[VE], y[VE];
                    auto join = [&](const float* p, float (&o)[VE]) {
                        if constexpr (VE == 1) {
                            o[0] = p[c];
#pragma unroll
                            for (int l = 1; l < SL; l++) o[0] += p[l * Sh::PY + c];
                        } else {
                            ulonglong2 x = *reinterpret_cast<const ulonglong2*>(p + c);
#pragma unroll
                            for (int l = 1; l < SL; l++) { const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(p + l * Sh::PY + c); x.x = add2(x.x, w.x); x.y = add2(x.y, w.y); }
                            unpack2(x.x, o[0], o[1]); unpack2(x.y, o[2], o[3]);
                        }
                    };
                    auto get = [&](const float* p, float (&o)[VE]) {
                        if constexpr (VE == 1) o[0] = p[c];
                        else { const float4 w = *reinterpret_cast<const float4*>(p + c); o[0] = w.x; o[1] = w.y; o[2] = w.z; o[3] = w.w; }
                    };
                    join(sh.s1[t], s1);
                    join(sh.s2[t], s2);
                    float st[VE], u[VE], o[VE], ds[VE], skip[VE];
                    get(sh.step[tt], st); get(sh.u[tt], u); get(sh.e[tt], o); get(sh.dstep[tt], ds); get(sh.skip, skip);
#pragma unroll
                    for (int e = 0; e < VE; e++) {
                        du[e] = fmaf(skip[e], o[e], st[e] * s1[e]);
                        dd[e] = fmaf(u[e], s1[e], kLn2 * s2[e]) * ds[e];
                        dD[i][e] = fmaf(o[e], u[e], dD[i][e]);
                        db[i][e] += dd[e];
                    }
                    if (a.du) store_word<T, VE>((T*)a.du + at * a.lddu + ch0 + pc.lc + P::step(i, a.lddu), du);
                    if (a.ddelta) store_word<T, VE>((T*)a.ddelta + at * a.ldddelta + ch0 + pc.lc + P::step(i, a.ldddelta), dd);
                    if (a.dz) {
                        float dg[VE];
                        join(sh.y[t], y);
                        get(sh.dgate[tt], dg);
#pragma unroll
                        for (int e = 0; e < VE; e++) dz[e] = fmaf(skip[e], u[e], y[e]) * dg[e];
                        store_word<T, VE>((T*)a.dz + at * a.lddz + ch0 + pc.lc + P::step(i, a.lddz), dz);
                    }
                }
                // dB and dC over the block's channels: a thread takes four states of a row, or four threads do, each every fourth of the lanes' parts, where
                // those are many; always in the parts' order
                auto join_part = [&](int t, int k, int n, int from, int by, f2& x, f2& y) {
                    x = y = 0;
                    for (int i = from; i < warps * CL; i += by) {
                        const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(&all[i / CL].dbc[t][k][i % CL][n]);
                        x = add2(x, w.x); y = add2(y, w.y);
                    }
                };
                auto put = [&](int t, int k, int n, float v) {
                    if (n >= (int)a.N) return;
                    const size_t row = row0 + R * q + t;
                    if (a.sum_bc) a.sum_bc[((((size_t)cb * a.q.rows + row) * a.G + g) * 2 + k) * a.N + n] = v;
                    else if (k == 0) { if (a.dB) ((T*)a.dB)[row * a.lddb + g * a.N + n] = from_f32<T>(v); }
                    else if (a.dC) ((T*)a.dC)[row * a.lddc + g * a.N + n] = from_f32<T>(v);
                };
                const int outs = min(left, R) * 2 * SL;
                if (warps * CL >= 16) {
                    for (int o = threadIdx.x / 4; o < outs; o += blockDim.x / 4) {
                        const int t = o / (2 * SL), k = o / SL % 2, n = o % SL * 4, sub = threadIdx.x & 3;
                        f2 x, y;
                        join_part(t, k, n, sub, 4, x, y);
                        const uint32_t who = 0xFu << (lane & 28);
#pragma unroll
                        for (int m = 1; m < 4; m <<= 1) { x = add2(x, __shfl_xor_sync(who, x, m)); y = add2(y, __shfl_xor_sync(who, y, m)); }
                        float v[4];
                        unpack2(x, v[0], v[1]); unpack2(y, v[2], v[3]);
                        put(t, k, n + sub, sub == 0 ? v[0] : (sub == 1 ? v[1] : (sub == 2 ? v[2] : v[3])));
                    }
                } else {
                    for (int o = threadIdx.x; o < outs; o += blockDim.x) {
                        const int t = o / (2 * SL), k = o / SL % 2, n = o % SL * 4;
                        f2 x, y;
                        join_part(t, k, n, 0, 1, x, y);
                        float v[4];
                        unpack2(x, v[0], v[1]); unpack2(y, v[2], v[3]);
#pragma unroll
                        for (int e = 0; e < 4; e++) put(t, k, n + e, v[e]);
                    }
                }
                __syncthreads();
            }
        }
        if (whole && a.d_state0 && r.slot >= 0) store_states(G, a.d_state0 + (size_t)r.slot * DN, a.N, a, ch0, have, cl, sl);
    }
    float* par = a.sum_par + (size_t)blockIdx.y * a.D * (a.N + 2);
    store_states(dA, par, a.N + 2, a, ch0, have, cl, sl);
    // a channel's sums over the lanes that have pieces of it, by way of shared memory, in the order of the rows
#pragma unroll
    for (int i = 0; i < I; i++) {
        const int t = pc.t(i), c = pc.c(i);
        if (t >= R) continue;
#pragma unroll
        for (int e = 0; e < VE; e++) { sh.u[t][c + e] = dD[i][e]; sh.e[t][c + e] = db[i][e]; }
    }
    __syncwarp();
    for (int c = lane; c < (int)have; c += 32) {
        float x = 0.0f, y = 0.0f;
#pragma unroll
        for (int t = 0; t < R; t++) { x += sh.u[t][c]; y += sh.e[t][c]; }
        par[(size_t)(ch0 + c) * (a.N + 2) + a.N] = x;
        par[(size_t)(ch0 + c) * (a.N + 2) + a.N + 1] = y;
    }
}

// dB and dC from the channel blocks' sums, in their order; rows of sequences only
template <typename T>
__global__ void __launch_bounds__(256) join_states_kernel(const Scan a) {
    sf_chain_enter();
    const Range r = range_of(a.q, blockIdx.y, a.st);
    const uint32_t width = a.G * 2 * a.N;
    const size_t plane = (size_t)a.q.rows * width;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < (uint64_t)r.len * width; i += (uint64_t)gridDim.x * 256) {
        const size_t row = r.first + i / width;
        const uint32_t col = (uint32_t)(i % width), g = col / (2 * a.N), k = col / a.N % 2, n = col % a.N;
        float v = 0.0f;
        for (uint32_t cb = 0; cb < a.cblocks; cb++) v += a.sum_bc[cb * plane + row * width + col];
        if (k == 0) { if (a.dB) ((T*)a.dB)[row * a.lddb + g * a.N + n] = from_f32<T>(v); }
        else if (a.dC) ((T*)a.dC)[row * a.lddc + g * a.N + n] = from_f32<T>(v);
    }
}

// dA, dD and dbias from the runs' sums: 32 values a block, a warp takes every eighth sum of each
__global__ void __launch_bounds__(256) join_params_kernel(const Scan a) {
    sf_chain_enter();
    __shared__ float sh[8][32];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const uint64_t e = (uint64_t)blockIdx.x * 32 + lane, n = (uint64_t)a.D * (a.N + 2);
    float v = 0.0f;
    if (e < n) {
#pragma unroll 8
        for (uint32_t p = warp; p < a.runs; p += 8) v += a.sum_par[(size_t)p * n + e];
    }
    sh[warp][lane] = v;
    __syncthreads();
    if (warp || e >= n) return;
#pragma unroll
    for (int i = 1; i < 8; i++) v += sh[i][lane];
    const uint32_t c = (uint32_t)(e / (a.N + 2)), k = (uint32_t)(e % (a.N + 2));
    if (k < a.N) { if (a.dA) a.dA[(size_t)c * a.N + k] = v; }
    else if (k == a.N) { if (a.dD) a.dD[c] = v; }
    else if (a.dbias_out) a.dbias_out[c] = v;
}

}  // namespace

extern "C" int sf_seq_scan_backward(sf_ctx* ctx, const sf_sequences* seq, const sf_scan_rows* in, uint32_t rows, const void* dy, size_t lddy, const float* starts,
                                    const float* d_state, float* d_state_in_out, uint32_t n_slots, const sf_scan_grads* out, void* workspace,
                                    size_t workspace_bytes, void* stream)
{
    const int ok = check(ctx, seq, in, rows);
    if (ok != SF_OK) return ok;
    if (!out || n_slots > 0x7FFFFFFFu || lddy < in->D || (rows && (!dy || !starts))) return SF_ERR_ARG;
    const uint32_t size = type_bytes(in->dtype);
    const size_t GN = (size_t)in->G * in->N;
    if ((out->du && out->lddu < in->D) || (out->d_delta && out->ldd_delta < in->D) || (out->dz && (out->lddz < in->D || !in->z)) || (out->dB && out->lddb < GN) || (out->dC && out->lddc < GN)) return SF_ERR_ARG;
    if (!aligned(dy, size) || !aligned(out->du, size) || !aligned(out->d_delta, size) || !aligned(out->dz, size) || !aligned(out->dB, size) || !aligned(out->dC, size) || !aligned(starts, 4) ||
        !aligned(d_state, 4) || !aligned(d_state_in_out, 4) || !aligned(out->dA, 4) || !aligned(out->dD_skip, 4) || !aligned(out->d_delta_bias, 4) || !aligned(workspace, 4) ||
        overlap_in_part(d_state, d_state_in_out, (size_t)n_slots * in->D * in->N * 4)) return SF_ERR_ARG;
    const Plan p = plan_of(seq->n_seq, seq->max_len, in->D, in->N, in->G, true);
    if (!workspace || workspace_bytes < back_bytes(p, seq->n_seq, rows, in->D, in->N, in->G)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    cudaStream_t st = (cudaStream_t)stream;
    Scan a;
    fill(a, seq, in, rows, n_slots, p, ctx);
    a.dy = dy; a.lddy = lddy; a.starts = const_cast<float*>(starts); a.d_state = d_state; a.d_state0 = d_state_in_out;
    a.du = out->du; a.ddelta = out->d_delta; a.dz = out->dz; a.dB = out->dB; a.dC = out->dC;
    a.lddu = out->lddu; a.ldddelta = out->ldd_delta; a.lddz = out->lddz; a.lddb = out->lddb; a.lddc = out->lddc;
    a.dA = out->dA; a.dD = out->dD_skip; a.dbias_out = out->d_delta_bias;
    char* ws = (char*)workspace;
    if (p.split) { a.part_state = (float*)ws; a.part_step = (float*)(ws + sf_align256((size_t)seq->n_seq * p.parts * in->D * in->N * 4)); }
    ws += part_bytes(p, seq->n_seq, in->D, in->N);
    a.sum_par = (float*)ws;
    if (p.cblocks > 1) a.sum_bc = (float*)(ws + sf_align256((size_t)p.runs * in->D * (in->N + 2) * 4));
    const uint64_t blocks = ((uint64_t)seq->n_seq * in->G * p.cwarps + kWarps - 1) / kWarps;
    if (blocks > 0x7FFFFFFFu) return SF_ERR_ARG;
    const bool vec = fits(in) && aligned(starts, 16) && fits(dy, lddy, in->dtype) && fits(out->du, out->lddu, in->dtype) && fits(out->d_delta, out->ldd_delta, in->dtype) && fits(out->dz, out->lddz, in->dtype);
    return by_type(in->dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_states(p.sl, [&](auto lanes) {
            constexpr int SL = decltype(lanes)::value;
            int e = by_width<T, SL>(vec, states_fit(in), [&](auto v, auto pb) {
                constexpr int VV = decltype(v)::value, PB = decltype(pb)::value;
                const size_t each = sizeof(Backward<T, SL, VV, PB>);
                if (p.split) {
                    int e = launch(back_ends_kernel<T, SL, VV, PB>, dim3((uint32_t)blocks, p.parts), 32 * kWarps, each * kWarps, st, a);
                    if (e == SF_OK) e = launch(parts_kernel<true>, dim3((uint32_t)(((uint64_t)in->D * in->N + 255) / 256), seq->n_seq), 256, 0, st, a);
                    if (e != SF_OK) return e;
                }
                const uint32_t w = std::min((uint32_t)kWarps, p.cwarps);
                return launch(back_kernel<T, SL, VV, PB>, dim3(in->G * p.cblocks, p.runs), 32 * w, each * w, st, a);
            });
            if (e == SF_OK && a.sum_bc && (a.dB || a.dC)) {
                for (uint32_t s = 0; s < seq->n_seq && e == SF_OK; s += 65535) {
                    Scan b = a;
                    b.q.offsets += s; b.q.n_seq = std::min(65535u, seq->n_seq - s);
                    if (b.q.counts) b.q.counts += s;
                    const uint64_t each = (uint64_t)seq->max_len * GN * 2, gx = std::max<uint64_t>(1, std::min<uint64_t>((each + 1023) / 1024, (uint64_t)SF_NUM_SMS_DEFAULT * 16 / b.q.n_seq));
                    e = launch(join_states_kernel<T>, dim3((uint32_t)gx, b.q.n_seq), 256, 0, st, b);
                }
            }
            if (e == SF_OK && (a.dA || a.dD || a.dbias_out)) e = launch(join_params_kernel, (uint32_t)(((uint64_t)in->D * (in->N + 2) + 31) / 32), 256, 0, st, a);
            return e;
        });
    });
}
