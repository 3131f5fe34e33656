// Backward pass of the selective state space scan (formulas and mapping: seq_scan.cuh).
#include "seq_scan.cuh"

namespace {

using namespace sfscan;

constexpr int K = (int)kEvery;             // rows of a tile
constexpr int R = 4;                       // rows whose decays and states a thread holds at once

// What a warp keeps in shared memory for a tile; rows of channels spaced so that 16-byte accesses of eight lanes meet no common bank
template <int SL> struct __align__(16) Backward {
    typedef Shape<SL> S;
    static constexpr int PX = S::CH + 4;
    float step[K][PX], u[K][PX], e[K][PX];                 // delta; u; dout silu(z)
    float dstep[K][PX], dgate[K][PX];                      // d delta / d raw; dout silu'(z).  A row that is done leaves du (without D e), ddelta and dz in step, dstep and dgate
    float bc[2][K][S::NP];                                 // B, C
    float sum[K][2][S::NP];                                // the warp's dB, dC
    float4 start[K / R][4][32];                            // the states before rows 0, R, .., every lane its own
    float bias[S::CH], skip[S::CH];
};

// stages steps, inputs and gradients of the rows t0 .. t0 + K - 1 as far as there (zeros behind: they then change nothing); ENDS: what the pass for the parts' ends needs
template <typename T, int SL, int VV, bool ENDS>
__device__ __forceinline__ void stage(const Scan& a, Backward<SL>& sh, size_t row0, uint32_t ch0, uint32_t have, uint32_t g, int rows, int lane) {
    typedef Shape<SL> S;
    typedef Pieces<K, S::CH, VV> P;
    const P pc(lane);
    const size_t at = row0 + pc.lt;
    const T* pd = (const T*)a.delta + at * a.lddelta + ch0 + pc.lc; const T* pu = (const T*)a.u + at * a.ldu + ch0 + pc.lc;
    const T* pz = (const T*)a.z + at * a.ldz + ch0 + pc.lc; const T* pg = (const T*)a.dy + at * a.lddy + ch0 + pc.lc;
    Piece<T, VV> nd[P::I], nu[P::I], nz[P::I], ng[P::I];
    States<T, VV, K, S::NP> ns;
#pragma unroll
    for (int i = 0; i < P::I; i++) {
        const bool there = pc.t(i) < rows && pc.c(i) < (int)have;
        nd[i] = fetch<T, VV>(pd, P::step(i, a.lddelta), there);
        if (!ENDS) nu[i] = fetch<T, VV>(pu, P::step(i, a.ldu), there);
        if (a.z) nz[i] = fetch<T, VV>(pz, P::step(i, a.ldz), there);
        ng[i] = fetch<T, VV>(pg, P::step(i, a.lddy), there);
    }
    ns.fetch_all(a, row0, g * a.N, rows, lane);
#pragma unroll
    for (int i = 0; i < P::I; i++) {
        const int t = pc.t(i), c = pc.c(i);
        if (t >= K) continue;
        const bool there = t < rows && c < (int)have;
        float d[VV], u[VV], z[VV], o[VV];
        open<T, VV>(nd[i], d);
        if (!ENDS) open<T, VV>(nu[i], u);
        if (a.z) open<T, VV>(nz[i], z);
        open<T, VV>(ng[i], o);
        float ds[VV], dg[VV];
        if constexpr (VV == 1) {
            float x;                                       // exp(-|raw|): the slope of softplus is 1 / (1 + x), or x / (1 + x) left of 0
            const float raw = d[0] + sh.bias[c], sg = a.z ? sigmoid(z[0]) : 1.0f;
            d[0] = a.softplus ? softplus_of(raw, x) : raw;
            ds[0] = a.softplus ? (raw >= 0.0f ? 1.0f : x) * rcp(1.0f + x) : 1.0f;
            dg[0] = a.z ? o[0] * sg * fmaf(z[0], 1.0f - sg, 1.0f) : 0.0f;
            if (a.z) o[0] *= z[0] * sg;
        } else {
#pragma unroll
            for (int e = 0; e < VV; e += 2) {
                const f2 one = dup2(1.0f);
                f2 raw = add2(pack2(d[e], d[e + 1]), *reinterpret_cast<const f2*>(&sh.bias[c + e])), x, v = raw, w = one;
                if (a.softplus) {
                    v = softplus2(raw, x);
                    float p, q, r0, r1;
                    unpack2(add2(x, one), p, q);
                    unpack2(raw, r0, r1);
                    if (!ENDS) { float x0, x1; unpack2(x, x0, x1); w = mul2(pack2(r0 >= 0.0f ? 1.0f : x0, r1 >= 0.0f ? 1.0f : x1), pack2(rcp(p), rcp(q))); }
                }
                unpack2(v, d[e], d[e + 1]);
                unpack2(w, ds[e], ds[e + 1]);
                if (a.z) {
                    const f2 zz = pack2(z[e], z[e + 1]), oo = pack2(o[e], o[e + 1]), sg = sigmoid2(zz), os = mul2(oo, sg);
                    if (!ENDS) unpack2(mul2(os, fma2(zz, fma2(sg, dup2(-1.0f), one), one)), dg[e], dg[e + 1]);
                    unpack2(mul2(os, zz), o[e], o[e + 1]);
                }
            }
        }
        if (!there) {
#pragma unroll
            for (int e = 0; e < VV; e++) d[e] = o[e] = 0.0f;
        }
        auto put = [&](float* p, const float (&v)[VV]) {
            if constexpr (VV == 1) p[0] = v[0];
            else {
#pragma unroll
                for (int e = 0; e < VV; e += 4) *reinterpret_cast<float4*>(p + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
            }
        };
        put(&sh.step[t][c], d);
        put(&sh.e[t][c], o);
        if (!ENDS) { put(&sh.u[t][c], u); put(&sh.dstep[t][c], ds); if (a.z) put(&sh.dgate[t][c], dg); }
    }
    ns.stage(&sh.bc[0][0][0], lane);
}

// asks for the rows of the next tile and the state before it, so that they are in L2 by then
__device__ __forceinline__ void to_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
template <typename T, int SL, int VV>
__device__ __forceinline__ void ahead(const Scan& a, size_t row0, size_t start, uint32_t ch0, uint32_t have, int lane) {
    const Pieces<K, Shape<SL>::CH, VV> pc(lane);
    if (VV > 1 && pc.lc < (int)have && pc.lt < K) {        // (the first piece of a row's line will do; narrow pieces would ask a line many times)
        const size_t at = row0 + pc.lt;
        to_l2((const T*)a.delta + at * a.lddelta + ch0 + pc.lc);
        to_l2((const T*)a.u + at * a.ldu + ch0 + pc.lc);
        to_l2((const T*)a.dy + at * a.lddy + ch0 + pc.lc);
        if (a.z) to_l2((const T*)a.z + at * a.ldz + ch0 + pc.lc);
    }
    const uint32_t floats = have * a.N;                    // (the warp's channels lie side by side)
    for (uint32_t i = lane * 32; i < floats; i += 32 * 32) to_l2(a.starts + start * a.D * a.N + (size_t)ch0 * a.N + i);
}

template <int SL> __device__ __forceinline__ void channel_params(const Scan& a, Backward<SL>& sh, uint32_t ch0, uint32_t have, int lane) {
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
template <typename T, int SL, int VV>
__global__ void __launch_bounds__(32 * kWarps) back_ends_kernel(const Scan a) {
    sf_chain_enter();
    constexpr int CH = Shape<SL>::CH;
    extern __shared__ __align__(16) unsigned char shared[];
    Backward<SL>& sh = reinterpret_cast<Backward<SL>*>(shared)[threadIdx.x / 32];
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
    channel_params<SL>(a, sh, ch0, have, lane);
    __syncwarp();
    for (uint32_t tile = (t_end - t_begin + K - 1) / K; tile-- > 0;) {
        const uint32_t t0 = t_begin + tile * K;
        stage<T, SL, VV, true>(a, sh, (size_t)r.first + t0, ch0, have, g, (int)min((uint32_t)K, t_end - t0), lane);
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

// The sums over the SL state lanes of the lane's four channels: a lane gets those of NC of them (all, two, one), from channel first(sl) on.
template <int SL> struct ByState {
    static constexpr int NC = SL == 1 ? 4 : (SL == 2 ? 2 : 1);
    __device__ __forceinline__ static int first(int sl) { return SL == 1 ? 0 : (SL == 2 ? 2 * sl : 2 * (sl & 1) + (sl >> 1 & 1)); }
    __device__ __forceinline__ static void sum(const f2 (&v)[2], int sl, float (&o)[NC]) {
        if constexpr (SL == 1) { unpack2(v[0], o[0], o[1]); unpack2(v[1], o[2], o[3]); }
        else {
            const bool hi = sl & 1;
            const f2 w = add2(hi ? v[1] : v[0], __shfl_xor_sync(0xFFFFFFFFu, hi ? v[0] : v[1], 1));
            float x, y;
            unpack2(w, x, y);
            if constexpr (SL == 2) { o[0] = x; o[1] = y; }
            else {
                const bool up = sl & 2;
                o[0] = (up ? y : x) + __shfl_xor_sync(0xFFFFFFFFu, up ? x : y, 2);
#pragma unroll
                for (int m = 4; m < SL; m <<= 1) o[0] += __shfl_xor_sync(0xFFFFFFFFu, o[0], m);
            }
        }
    }
};
// Sums of 8 values over the CL channel lanes; they end up in lane cl as the 8 / CL (at least one) values from index (cl * 8 / CL) % 8 on; put writes
// them to p[value / 4][state]
template <int SL> __device__ __forceinline__ void put_states(float* p0, float* p1, float (&v)[8], int lane, int cl, int sl) {
    int n = 8;
#pragma unroll
    for (int m = 16; m >= SL; m >>= 1) {
        if (n > 1) {
            n >>= 1;
            const bool hi = lane & m;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (i >= n) break;
                const float keep = hi ? v[i + n] : v[i], give = hi ? v[i] : v[i + n];
                v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, m);
            }
        } else v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], m);
    }
    constexpr int CL = 32 / SL, NV = CL >= 8 ? 1 : 8 / CL, SAME = CL > 8 ? CL / 8 : 1;       // values a lane has, lanes that have the same
    if (cl % SAME) return;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int k = cl / SAME * NV + i;
        (k < 4 ? p0 : p1)[sl * 4 + k % 4] = v[i];
    }
}

// One block: up to kWarps warps over neighbouring channels of a group, one part of one sequence after the other (a run), rows from last to first.
// A tile's states are stepped from the state kept before it: rows 0 to 3 to reach row 4, rows 4 to 7 with decays and states held in registers, back over
// them, then rows 0 to 3 the same way.
template <typename T, int SL, int VV>
__global__ void __launch_bounds__(32 * kWarps, 2) back_kernel(const Scan a) {
    sf_chain_enter();
    typedef Shape<SL> S;
    typedef Pieces<K, S::CH, VV> P;
    constexpr int CH = S::CH, I = P::I;
    extern __shared__ __align__(16) unsigned char shared[];
    Backward<SL>* all = reinterpret_cast<Backward<SL>*>(shared);
    const int warp = threadIdx.x / 32, warps = blockDim.x / 32;
    Backward<SL>& sh = all[warp];
    const int lane = threadIdx.x & 31, cl = lane / SL, sl = lane % SL;
    const uint32_t gb = blockIdx.x, g = gb / a.cblocks, cb = gb % a.cblocks;
    const uint32_t c0 = min(a.per, (cb * (uint32_t)kWarps + warp) * CH);
    const uint32_t ch0 = g * a.per + c0, have = min((uint32_t)CH, a.per - c0);     // (a warp behind the group's last channel has none, but meets the others)
    const P pc(lane);
    f2 A[2][4], dA[2][4], G[2][4];
    load_states(A, a.A, a, ch0, have, cl, sl, kLog2e);
    float dD[I][VV], db[I][VV];                            // of the channels that this lane's pieces have
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
        for (int n = 0; n < 4; n++) dA[j][n] = 0;
#pragma unroll
    for (int i = 0; i < I; i++)
#pragma unroll
        for (int e = 0; e < VV; e++) dD[i][e] = db[i][e] = 0.0f;
    channel_params<SL>(a, sh, ch0, have, lane);
    __syncwarp();
    const uint64_t items = (uint64_t)a.q.n_seq * a.parts;
    for (uint64_t it = blockIdx.y; it < items; it += a.runs) {
        const uint32_t part = (uint32_t)(it / a.q.n_seq), s = (uint32_t)(it % a.q.n_seq);
        const Range r = range_of(a.q, s, a.st);
        const uint32_t t_begin = part * a.part_len, t_end = min(r.len, t_begin + a.part_len);
        const bool whole = a.part_state == nullptr;        // the sequence in one part: gradients of states here
        if (t_begin >= r.len && !(whole && a.d_state0 && r.slot >= 0)) continue;
        const size_t DN = (size_t)a.D * a.N;
        load_states(G, whole ? (a.d_state && r.slot >= 0 ? a.d_state + (size_t)r.slot * DN : nullptr) : a.part_state + ((size_t)s * a.parts + part) * DN, a, ch0, have, cl, sl, 1.0f);
        const uint32_t tiles = t_end > t_begin ? (t_end - t_begin + K - 1) / K : 0;
        for (uint32_t tile = tiles; tile-- > 0;) {
            const uint32_t t0 = t_begin + tile * K;
            const int rows = (int)min((uint32_t)K, t_end - t0);
            const size_t row0 = (size_t)r.first + t0;
            f2 h[2][4];
            load_states(h, a.starts + start_index(r.first, s, t0) * DN, a, ch0, have, cl, sl, 1.0f);
            stage<T, SL, VV, false>(a, sh, row0, ch0, have, g, rows, lane);
            if (tile) ahead<T, SL, VV>(a, row0 - K, start_index(r.first, s, t0 - K), ch0, have, lane);
            __syncwarp();
            auto keep = [&](int q) {
#pragma unroll
                for (int j = 0; j < 2; j++)
#pragma unroll
                    for (int n = 0; n < 4; n += 2) *reinterpret_cast<ulonglong2*>(&sh.start[q][2 * j + n / 2][lane]) = make_ulonglong2(h[j][n], h[j][n + 1]);
            };
            auto take = [&](f2 (&v)[2][4], int q) {
#pragma unroll
                for (int j = 0; j < 2; j++)
#pragma unroll
                    for (int n = 0; n < 4; n += 2) { const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(&sh.start[q][2 * j + n / 2][lane]); v[j][n] = w.x; v[j][n + 1] = w.y; }
            };
#pragma unroll
            for (int t = 0; t < K - R; t++) {
                if (t % R == 0) keep(t / R);
                const ulonglong2 d2 = *reinterpret_cast<const ulonglong2*>(&sh.step[t][cl * 4]), u2 = *reinterpret_cast<const ulonglong2*>(&sh.u[t][cl * 4]);
                const float4 b4 = *reinterpret_cast<const float4*>(&sh.bc[0][t][sl * 4]);
                const f2 d[2] = {d2.x, d2.y}, in[2] = {mul2(d2.x, u2.x), mul2(d2.y, u2.y)}, b[4] = {dup2(b4.x), dup2(b4.y), dup2(b4.z), dup2(b4.w)};
#pragma unroll
                for (int j = 0; j < 2; j++)
#pragma unroll
                    for (int n = 0; n < 4; n++) h[j][n] = fma2(decay2(d[j], A[j][n]), h[j][n], mul2(in[j], b[n]));
            }
            keep(K / R - 1);
#pragma unroll 1
            for (int q = K / R - 1; q >= 0; q--) {
                f2 al[R][2][4], hs[R + 1][2][4];               // decays; states before the rows and after them
                take(hs[0], q);
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
                    typedef ByState<SL> Q;
                    float o1[Q::NC], o2[Q::NC], oy[Q::NC];
                    Q::sum(s1, sl, o1);
                    Q::sum(s2, sl, o2);
                    if (a.z) Q::sum(y, sl, oy);
                    float v[8];
#pragma unroll
                    for (int n = 0; n < 4; n++) {
                        float x, w;
                        unpack2(dB[n], x, w); v[n] = x + w;
                        unpack2(dC[n], x, w); v[4 + n] = x + w;
                    }
                    put_states<SL>(sh.sum[tt][0], sh.sum[tt][1], v, lane, cl, sl);
                    __syncwarp();                          // (every lane has read the row)
                    if (SL <= 4 || sl < 4) {
#pragma unroll
                        for (int i = 0; i < Q::NC; i++) {
                            const int k = cl * 4 + Q::first(sl) + i;
                            const float uu = sh.u[tt][k];
                            sh.step[tt][k] *= o1[i];
                            sh.dstep[tt][k] *= fmaf(uu, o1[i], kLn2 * o2[i]);
                            if (a.z) sh.dgate[tt][k] *= fmaf(sh.skip[k], uu, oy[i]);
                        }
                    }
                }
            }
            __syncwarp();
            const size_t at = row0 + pc.lt;
#pragma unroll
            for (int i = 0; i < I; i++) {
                const int t = pc.t(i), c = pc.c(i);
                if (t >= rows || c >= (int)have) continue;
                float du[VV], dd[VV], dz[VV];
#pragma unroll
                for (int e = 0; e < VV; e++) {
                    const float u = sh.u[t][c + e], o = sh.e[t][c + e];
                    du[e] = fmaf(sh.skip[c + e], o, sh.step[t][c + e]);
                    dd[e] = sh.dstep[t][c + e];
                    dz[e] = sh.dgate[t][c + e];
                    dD[i][e] = fmaf(o, u, dD[i][e]);
                    db[i][e] += dd[e];
                }
                if (a.du) store_word<T, VV>((T*)a.du + at * a.lddu + ch0 + pc.lc + P::step(i, a.lddu), du);
                if (a.ddelta) store_word<T, VV>((T*)a.ddelta + at * a.ldddelta + ch0 + pc.lc + P::step(i, a.ldddelta), dd);
                if (a.dz) store_word<T, VV>((T*)a.dz + at * a.lddz + ch0 + pc.lc + P::step(i, a.lddz), dz);
            }
            // dB and dC: the block's warps, in their order
            __syncthreads();
            for (int i = threadIdx.x; i < rows * 2 * S::NP; i += blockDim.x) {
                const int t = i / (2 * S::NP), k = i / S::NP % 2, n = i % S::NP;
                if (n >= (int)a.N) continue;
                float v = all[0].sum[t][k][n];
                for (int w = 1; w < warps; w++) v += all[w].sum[t][k][n];
                if (a.sum_bc) a.sum_bc[((((size_t)cb * a.q.rows + row0 + t) * a.G + g) * 2 + k) * a.N + n] = v;
                else if (k == 0) { if (a.dB) ((T*)a.dB)[(row0 + t) * a.lddb + g * a.N + n] = from_f32<T>(v); }
                else if (a.dC) ((T*)a.dC)[(row0 + t) * a.lddc + g * a.N + n] = from_f32<T>(v);
            }
            __syncthreads();
        }
        if (whole && a.d_state0 && r.slot >= 0) store_states(G, a.d_state0 + (size_t)r.slot * DN, a.N, a, ch0, have, cl, sl);
    }
    float* par = a.sum_par + (size_t)blockIdx.y * a.D * (a.N + 2);
    store_states(dA, par, a.N + 2, a, ch0, have, cl, sl);
    // a channel's sums over the lanes that have pieces of it, by way of shared memory, in the order of the rows
#pragma unroll
    for (int i = 0; i < I; i++) {
        const int t = pc.t(i), c = pc.c(i);
        if (t >= K) continue;
#pragma unroll
        for (int e = 0; e < VV; e++) { sh.u[t][c + e] = dD[i][e]; sh.e[t][c + e] = db[i][e]; }
    }
    __syncwarp();
    for (int c = lane; c < (int)have; c += 32) {
        float x = 0.0f, y = 0.0f;
#pragma unroll
        for (int t = 0; t < K; t++) { x += sh.u[t][c]; y += sh.e[t][c]; }
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

// dA, dD and dbias from the runs' sums
__global__ void __launch_bounds__(256) join_params_kernel(const Scan a) {
    sf_chain_enter();
    const uint64_t e = (uint64_t)blockIdx.x * 256 + threadIdx.x, n = (uint64_t)a.D * (a.N + 2);
    if (e >= n) return;
    float v = 0.0f;
    for (uint32_t p = 0; p < a.runs; p++) v += a.sum_par[(size_t)p * n + e];
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
        !aligned(d_state, 4) || !aligned(d_state_in_out, 4) || !aligned(out->dA, 4) || !aligned(out->dD_skip, 4) || !aligned(out->d_delta_bias, 4) || !aligned(workspace, 4)) return SF_ERR_ARG;
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
    const bool vec = fits(in) && fits(dy, lddy, in->dtype) && fits(out->du, out->lddu, in->dtype) && fits(out->d_delta, out->ldd_delta, in->dtype) && fits(out->dz, out->lddz, in->dtype);
    return by_type(in->dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_states(p.sl, [&](auto lanes) {
            constexpr int SL = decltype(lanes)::value, VV = 16 / (int)sizeof(T);
            int e = SF_OK;
            if (p.split) {
                e = launch(vec ? back_ends_kernel<T, SL, VV> : back_ends_kernel<T, SL, 1>, dim3((uint32_t)blocks, p.parts), 32 * kWarps, sizeof(Backward<SL>) * kWarps, st, a);
                if (e == SF_OK) e = launch(parts_kernel<true>, dim3((uint32_t)(((uint64_t)in->D * in->N + 255) / 256), seq->n_seq), 256, 0, st, a);
                if (e != SF_OK) return e;
            }
            const uint32_t w = std::min((uint32_t)kWarps, p.cwarps);
            e = launch(vec ? back_kernel<T, SL, VV> : back_kernel<T, SL, 1>, dim3(in->G * p.cblocks, p.runs), 32 * w, sizeof(Backward<SL>) * w, st, a);
            if (e == SF_OK && a.sum_bc && (a.dB || a.dC)) {
                for (uint32_t s = 0; s < seq->n_seq && e == SF_OK; s += 65535) {
                    Scan b = a;
                    b.q.offsets += s; b.q.n_seq = std::min(65535u, seq->n_seq - s);
                    if (b.q.counts) b.q.counts += s;
                    const uint64_t each = (uint64_t)seq->max_len * GN * 2, gx = std::max<uint64_t>(1, std::min<uint64_t>((each + 1023) / 1024, (uint64_t)SF_NUM_SMS_DEFAULT * 16 / b.q.n_seq));
                    e = launch(join_states_kernel<T>, dim3((uint32_t)gx, b.q.n_seq), 256, 0, st, b);
                }
            }
            if (e == SF_OK && (a.dA || a.dD || a.dbias_out)) e = launch(join_params_kernel, (uint32_t)(((uint64_t)in->D * (in->N + 2) + 255) / 256), 256, 0, st, a);
            return e;
        });
    });
}
