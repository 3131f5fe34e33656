// Forward pass of the selective state space scan, and its single steps (formulas and mapping: seq_scan.cuh).
#include "seq_scan.cuh"

namespace {

using namespace sfscan;

// What a warp keeps in shared memory.  Sums over states are left as one part a state lane and joined where the row is written.  Rows are spaced so that
// the 16-byte accesses of eight lanes meet no common bank: PX floats a row of channels, PY a part, PT the parts of a row.
template <typename T, int SL, int VV, int PB, int J> struct __align__(16) Forward {
    typedef Shape<SL, J> S;
    typedef Pieces<S::K, S::CH, VV> P;
    typedef States<T, PB, S::K, S::NP> ST;
    static constexpr int PX = S::CH + 4, PY = S::CH + (SL == 1 ? 0 : (SL == 2 ? 16 : (SL == 4 ? 8 : 4))), PT = SL * PY + 4;
    float step[S::K][PX], in[S::K][PX];                    // delta; delta u
    float bc[2][S::K][S::NP];                              // B, C
    float y[S::K][PT];
    uint4 way[VV > 1 ? 3 * P::I + ST::I : 1][32];          // the next tile's pieces on their way, every lane its own
    float bias[S::CH], skip[S::CH];                        // delta_bias, D of the warp's channels
};

// The scan of a sequence, or of one part of it (blockIdx.y): from the state that `part_state` holds where sequences go in parts.
// ENDS: only the state at the part's end, from zero, and the sum of the part's steps.
template <typename T, int SL, int VV, int PB, bool ENDS, int J>
__global__ void __launch_bounds__(32 * kWarps, 4) scan_kernel(const Scan a) {
    sf_chain_enter();
    typedef Shape<SL, J> S;
    typedef Pieces<S::K, S::CH, VV> P;
    constexpr int JP = J / 2;                              // pairs of channels of a lane
    constexpr int K = S::K, CH = S::CH, NP = S::NP, I = P::I;
    extern __shared__ __align__(16) unsigned char shared[];
    typedef Forward<T, SL, VV, PB, J> Sh;
    Sh& sh = reinterpret_cast<Sh*>(shared)[threadIdx.x / 32];
    const int lane = threadIdx.x & 31, cl = lane / SL, sl = lane % SL;
    const Item it = item_of(a, CH);
    if (it.have == 0) return;
    const uint32_t s = it.s, g = it.g, ch0 = it.ch0, have = it.have;
    const Range r = range_of(a.q, s, a.st);
    const uint32_t part = blockIdx.y, t_begin = part * a.part_len, t_end = min(r.len, t_begin + a.part_len);
    if (ENDS ? t_begin >= r.len : (part && t_begin >= r.len)) return;
    // rows on their way while others are worked on
    Piece<T, VV> nd[I], nu[I], nz[I];
    States<T, PB, K, NP> ns;
    const P pc(lane);
    const size_t at0 = (size_t)r.first + t_begin + pc.lt;
    const T* pd = (const T*)a.delta + at0 * a.lddelta + ch0 + pc.lc; const T* pu = (const T*)a.u + at0 * a.ldu + ch0 + pc.lc; const T* pz = (const T*)a.z + at0 * a.ldz + ch0 + pc.lc;
    T* py = (T*)a.y + at0 * a.ldy + ch0 + pc.lc;
    auto ask = [&](uint32_t t0) {                          // whole pieces go by way of shared memory, single elements through registers
        const int rows = (int)min((uint32_t)K, t_end - t0);
#pragma unroll
        for (int i = 0; i < I; i++) {
            const bool there = pc.c(i) < (int)have && pc.t(i) < rows;
            if constexpr (VV > 1) {
                copy16(&sh.way[i][lane], there ? pd + P::step(i, a.lddelta) : (const T*)a.delta, there);
                copy16(&sh.way[I + i][lane], there ? pu + P::step(i, a.ldu) : (const T*)a.u, there);
                if (!ENDS && a.z) copy16(&sh.way[2 * I + i][lane], there ? pz + P::step(i, a.ldz) : (const T*)a.z, there);
            } else {
                nd[i] = fetch<T, VV>(pd, P::step(i, a.lddelta), there);
                nu[i] = fetch<T, VV>(pu, P::step(i, a.ldu), there);
                if (!ENDS && a.z) nz[i] = fetch<T, VV>(pz, P::step(i, a.ldz), there);
            }
        }
        if constexpr (Sh::ST::WHOLE) {
#pragma unroll
            for (int i = 0; i < Sh::ST::I; i++) {
                bool there;
                const T* p = Sh::ST::template piece<T>(a, i, (size_t)r.first + t0, g * a.N, rows, lane, there);
                copy16(&sh.way[3 * I + i][lane], p, there);
            }
        } else ns.fetch_all(a, (size_t)r.first + t0, g * a.N, rows, lane);
        pd += K * a.lddelta; pu += K * a.ldu; pz += K * a.ldz;
    };
    if (t_begin < t_end) ask(t_begin);
    for (int c = lane; c < CH; c += 32) {
        sh.bias[c] = c < (int)have && a.dbias ? __ldg(a.dbias + ch0 + c) : 0.0f;
        sh.skip[c] = c < (int)have && a.Dk ? __ldg(a.Dk + ch0 + c) : 0.0f;
    }
    f2 A[JP][4], h[JP][4];                                 // channels 2 j and 2 j + 1 of the lane's side by side
#pragma unroll
    for (int j = 0; j < JP; j++)
#pragma unroll
        for (int n = 0; n < 4; n++) {
            float A_[2], h_[2];
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const uint32_t c = cl * J + 2 * j + k, st = sl * 4 + n;
                const bool there = c < have && st < a.N;
                const size_t at = (size_t)(ch0 + c) * a.N + st;
                A_[k] = there ? __ldg(a.A + at) * kLog2e : 0.0f;
                h_[k] = 0.0f;
                if (!ENDS && there) {
                    if (a.part_state) h_[k] = a.part_state[((size_t)s * a.parts + part) * a.D * a.N + at];
                    else if (a.state_in && r.slot >= 0) h_[k] = a.state_in[(size_t)r.slot * a.D * a.N + at];
                }
            }
            A[j][n] = pack2(A_[0], A_[1]); h[j][n] = pack2(h_[0], h_[1]);
        }
    // the warp's states into [channel][state]
    auto put = [&](float* p) {
#pragma unroll
        for (int j = 0; j < JP; j++) {
            float v[2][4];
#pragma unroll
            for (int n = 0; n < 4; n++) unpack2(h[j][n], v[0][n], v[1][n]);
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const uint32_t c = cl * J + 2 * j + k;
                float* o = p + (size_t)(ch0 + c) * a.N + sl * 4;
                if (c >= have) continue;
                if (a.n4 && ((uintptr_t)o & 15u) == 0) { if (sl * 4 < (int)a.N) *reinterpret_cast<float4*>(o) = make_float4(v[k][0], v[k][1], v[k][2], v[k][3]); }
                else {
#pragma unroll
                    for (int n = 0; n < 4; n++) if (sl * 4 + n < (int)a.N) o[n] = v[k][n];
                }
            }
        }
    };
    f2 steps[I][VV / 2 + 1];                               // sums of the steps that this lane stages (ENDS)
#pragma unroll
    for (int i = 0; i < I; i++)
#pragma unroll
        for (int e = 0; e <= VV / 2; e++) steps[i][e] = 0;
    __syncwarp();
    for (uint32_t t0 = t_begin; t0 < t_end; t0 += K) {
        const int rows = (int)min((uint32_t)K, t_end - t0);
        Piece<T, VV> cu[I], cz[I];
        if constexpr (VV > 1) {
            copies_done();
#pragma unroll
            for (int i = 0; i < I; i++) { nd[i].w = sh.way[i][lane]; nu[i].w = sh.way[I + i][lane]; if (!ENDS && a.z) nz[i].w = sh.way[2 * I + i][lane]; }
            if constexpr (Sh::ST::WHOLE) {
#pragma unroll
                for (int i = 0; i < Sh::ST::I; i++) ns.take(i, sh.way[3 * I + i][lane]);
            }
        }
        if constexpr (VV == 1) {                           // single elements, two at a time
            static_assert(I % 2 == 0, "every lane has an even number of single elements");
#pragma unroll
            for (int i = 0; i < I; i += 2) {
                const int t0_ = pc.t(i), c0 = pc.c(i), t1 = pc.t(i + 1), c1 = pc.c(i + 1);
                float d0[1], d1[1], u0[1], u1[1];
                open<T, 1>(nd[i], d0); open<T, 1>(nd[i + 1], d1); open<T, 1>(nu[i], u0); open<T, 1>(nu[i + 1], u1);
                cu[i] = nu[i]; cu[i + 1] = nu[i + 1];
                if (!ENDS) { cz[i] = nz[i]; cz[i + 1] = nz[i + 1]; }
                f2 x = add2(pack2(d0[0], d1[0]), pack2(sh.bias[c0], sh.bias[c1])), unused;
                if (a.softplus) x = softplus2(x, unused);
                float p, q;
                unpack2(x, p, q);
                if (ENDS) {
                    if (t0_ >= rows) p = 0.0f;
                    if (t1 >= rows) q = 0.0f;
                    steps[i][0] = add2(steps[i][0], pack2(p, 0.0f)); steps[i + 1][0] = add2(steps[i + 1][0], pack2(q, 0.0f));
                }
                sh.step[t0_][c0] = p; sh.step[t1][c1] = q;
                unpack2(mul2(pack2(p, q), pack2(u0[0], u1[0])), p, q);
                sh.in[t0_][c0] = p; sh.in[t1][c1] = q;
            }
        } else {
#pragma unroll
            for (int i = 0; i < I; i++) {
                const int t = pc.t(i), c = pc.c(i);
                if (t >= K) continue;
                float d[VV], u[VV];
                cu[i] = nu[i];
                if (!ENDS) cz[i] = nz[i];
                open<T, VV>(nd[i], d);
                open<T, VV>(nu[i], u);
#pragma unroll
                for (int e = 0; e < VV; e += 4) {
                    const float4 b4 = *reinterpret_cast<const float4*>(&sh.bias[c + e]);
                    f2 x = add2(pack2(d[e], d[e + 1]), pack2(b4.x, b4.y)), y = add2(pack2(d[e + 2], d[e + 3]), pack2(b4.z, b4.w));
                    if (a.softplus) { f2 unused; x = softplus2(x, unused); y = softplus2(y, unused); }
                    if (ENDS) {
                        if (t >= rows) x = y = 0;
                        steps[i][e / 2] = add2(steps[i][e / 2], x); steps[i][e / 2 + 1] = add2(steps[i][e / 2 + 1], y);
                    }
                    *reinterpret_cast<ulonglong2*>(&sh.step[t][c + e]) = make_ulonglong2(x, y);
                    *reinterpret_cast<ulonglong2*>(&sh.in[t][c + e]) = make_ulonglong2(mul2(x, pack2(u[e], u[e + 1])), mul2(y, pack2(u[e + 2], u[e + 3])));
                }
            }
        }
        ns.stage(&sh.bc[0][0][0], lane);
        __syncwarp();
        if (t0 + K < t_end) ask(t0 + K);
        if (!ENDS && a.starts && t0 % kEvery == 0) put(a.starts + start_index(r.first, s, t0) * a.D * a.N);
        auto row = [&](int t) {
            if (!ENDS && K > (int)kEvery && t % kEvery == 0 && t && a.starts) put(a.starts + start_index(r.first, s, t0 + t) * a.D * a.N);
            f2 d[JP], in[JP];
            if constexpr (J == 4) {
                const ulonglong2 d2 = *reinterpret_cast<const ulonglong2*>(&sh.step[t][cl * J]), i2 = *reinterpret_cast<const ulonglong2*>(&sh.in[t][cl * J]);
                d[0] = d2.x; d[1] = d2.y; in[0] = i2.x; in[1] = i2.y;
            } else { d[0] = *reinterpret_cast<const f2*>(&sh.step[t][cl * J]); in[0] = *reinterpret_cast<const f2*>(&sh.in[t][cl * J]); }
            const float4 b4 = *reinterpret_cast<const float4*>(&sh.bc[0][t][sl * 4]);
            const f2 b[4] = {dup2(b4.x), dup2(b4.y), dup2(b4.z), dup2(b4.w)};
#pragma unroll
            for (int j = 0; j < JP; j++)
#pragma unroll
                for (int n = 0; n < 4; n++) h[j][n] = fma2(decay2(d[j], A[j][n]), h[j][n], mul2(in[j], b[n]));
            if constexpr (!ENDS) {
                const float4 c4 = *reinterpret_cast<const float4*>(&sh.bc[1][t][sl * 4]);
                f2 y[JP];
#pragma unroll
                for (int j = 0; j < JP; j++) y[j] = fma2(h[j][3], dup2(c4.w), fma2(h[j][2], dup2(c4.z), fma2(h[j][1], dup2(c4.y), mul2(h[j][0], dup2(c4.x)))));
                if constexpr (J == 4) *reinterpret_cast<ulonglong2*>(&sh.y[t][sl * Sh::PY + cl * J]) = make_ulonglong2(y[0], y[1]);
                else *reinterpret_cast<f2*>(&sh.y[t][sl * Sh::PY + cl * J]) = y[0];
            }
        };
        if (rows == K) {
#pragma unroll
            for (int t = 0; t < K; t++) row(t);
        } else {
#pragma unroll 1
            for (int t = 0; t < rows; t++) row(t);
        }
        __syncwarp();
        if constexpr (!ENDS) {
            if constexpr (VV == 1) {
#pragma unroll
                for (int i = 0; i < I; i += 2) {
                    float v[2], z[2], u[1];
#pragma unroll
                    for (int k = 0; k < 2; k++) {
                        const int t = pc.t(i + k), c = pc.c(i + k);
                        open<T, 1>(cu[i + k], u);
                        if (a.z) { float w[1]; open<T, 1>(cz[i + k], w); z[k] = w[0]; }
                        v[k] = sh.skip[c] * u[0];
#pragma unroll
                        for (int l = 0; l < SL; l++) v[k] += sh.y[t][l * Sh::PY + c];
                    }
                    if (a.z) { const f2 zz = pack2(z[0], z[1]); unpack2(mul2(pack2(v[0], v[1]), mul2(zz, sigmoid2<T>(zz))), v[0], v[1]); }
#pragma unroll
                    for (int k = 0; k < 2; k++)
                        if (pc.c(i + k) < (int)have && pc.t(i + k) < rows) { const float o[1] = {v[k]}; store_word<T, 1>(py + P::step(i + k, a.ldy), o); }
                }
            } else {
#pragma unroll
                for (int i = 0; i < I; i++) {
                    const int t = pc.t(i), c = pc.c(i);
                    if (c >= (int)have || t >= rows) continue;
                    float u[VV], z[VV], y[VV];
                    open<T, VV>(cu[i], u);
                    if (a.z) open<T, VV>(cz[i], z);
#pragma unroll
                    for (int e = 0; e < VV; e += 4) {
                        const ulonglong2 k2 = *reinterpret_cast<const ulonglong2*>(&sh.skip[c + e]);
                        f2 v = mul2(k2.x, pack2(u[e], u[e + 1])), w = mul2(k2.y, pack2(u[e + 2], u[e + 3]));
#pragma unroll
                        for (int l = 0; l < SL; l++) {
                            const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(&sh.y[t][l * Sh::PY + c + e]);
                            v = add2(v, q.x); w = add2(w, q.y);
                        }
                        if (a.z) {
                            const f2 z0 = pack2(z[e], z[e + 1]), z1 = pack2(z[e + 2], z[e + 3]);
                            v = mul2(v, mul2(z0, sigmoid2<T>(z0))); w = mul2(w, mul2(z1, sigmoid2<T>(z1)));
                        }
                        unpack2(v, y[e], y[e + 1]); unpack2(w, y[e + 2], y[e + 3]);
                    }
                    store_word<T, VV>(py + P::step(i, a.ldy), y);
                }
            }
            py += K * a.ldy;
        }
        __syncwarp();
    }
    if (ENDS) put(a.part_state + ((size_t)s * a.parts + part) * a.D * a.N);
    else if (a.state_out && r.slot >= 0 && !a.part_state) put(a.state_out + (size_t)r.slot * a.D * a.N);
    if constexpr (ENDS) {                                  // a channel's steps: the lanes that staged it leave theirs, one adds them up in their order
        float* sum = &sh.y[0][0];                         // [rows of a tile][CH]
#pragma unroll
        for (int i = 0; i < I; i++) {
            const int t = pc.t(i), c = pc.c(i);
            if (t >= K) continue;
#pragma unroll
            for (int e = 0; e < VV; e += 2) {
                float x, y;
                unpack2(steps[i][e / 2], x, y);
                sum[t * CH + c + e] = x;
                if (VV > 1) sum[t * CH + c + e + 1] = y;
            }
        }
        __syncwarp();
        for (int c = lane; c < (int)have; c += 32) {
            float v = 0.0f;
#pragma unroll
            for (int t = 0; t < K; t++) v += sum[t * CH + c];
            a.part_step[((size_t)s * a.parts + part) * a.D + ch0 + c] = v;
        }
    }
}

// Single rows (max_len 1): a warp reads its channels' states once, steps them and writes them.
template <typename T, int SL, bool VEC>
__global__ void __launch_bounds__(32 * kWarps, 8) step_kernel(const Scan a) {
    sf_chain_enter();
    constexpr int CL = 32 / SL, CH = 4 * CL;
    const int lane = threadIdx.x & 31, cl = lane / SL, sl = lane % SL;
    const Item it = item_of(a, CH);
    if (it.have == 0) return;
    const uint32_t s = it.s, g = it.g, ch0 = it.ch0, have = it.have;
    const Range r = range_of(a.q, s, a.st);
    const bool row = r.len > 0;
    if (!row && !a.state_out) return;
    const size_t at = r.first;
    const bool mine = sl * 4 < (int)a.N;                   // (VEC: all four states are there or none)
    // channel j CL + cl: the warp's accesses to the states of CL channels lie side by side
    auto read = [&](const float* p, uint32_t c, float (&v)[4]) {
#pragma unroll
        for (int n = 0; n < 4; n++) v[n] = 0.0f;
        if (!p || c >= have) return;
        if constexpr (VEC) { if (mine) { const float4 q = *reinterpret_cast<const float4*>(p + c * a.N + sl * 4); v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w; } }
        else {
#pragma unroll
            for (int n = 0; n < 4; n++) if (sl * 4 + n < (int)a.N) v[n] = p[c * a.N + sl * 4 + n];
        }
    };
    float h[4][4];
    const float* si = a.state_in && r.slot >= 0 ? a.state_in + ((size_t)r.slot * a.D + ch0) * a.N : nullptr;
    float* so = a.state_out && r.slot >= 0 ? a.state_out + ((size_t)r.slot * a.D + ch0) * a.N : nullptr;
#pragma unroll
    for (int j = 0; j < 4; j++) read(si, j * CL + cl, h[j]);
    if (row) {
        // What a channel has one of (step, gate) is worked out by one of its SL lanes: a lane owns NO of its four channels
        constexpr int NO = SL == 1 ? 4 : (SL == 2 ? 2 : 1);
        auto owned = [&](int i) { return SL == 1 ? i : (SL == 2 ? 2 * sl + i : 2 * (sl & 1) + (sl >> 1 & 1)); };
        auto owner = [&](int j) { return lane - sl + (SL == 1 ? 0 : (SL == 2 ? j / 2 : j / 2 + 2 * (j % 2))); };
        float b[4], cc[4], u[NO], d[NO], z[NO], in[NO];
#pragma unroll
        for (int i = 0; i < NO; i++) {
            const uint32_t c = owned(i) * CL + cl;
            const bool there = c < have;
            u[i] = there ? to_f32(((const T*)a.u)[at * a.ldu + ch0 + c]) : 0.0f;
            d[i] = there ? to_f32(((const T*)a.delta)[at * a.lddelta + ch0 + c]) : 0.0f;
            z[i] = there && a.z ? to_f32(((const T*)a.z)[at * a.ldz + ch0 + c]) : 0.0f;
        }
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const bool there = sl * 4 + n < (int)a.N;
            b[n] = there ? to_f32(((const T*)a.B)[at * a.ldb + g * a.N + sl * 4 + n]) : 0.0f;
            cc[n] = there ? to_f32(((const T*)a.C)[at * a.ldc + g * a.N + sl * 4 + n]) : 0.0f;
        }
        float A[4][4];                                     // (asked for before the steps are worked out: 4096 x 1024 118 us, with them 124)
#pragma unroll
        for (int j = 0; j < 4; j++) read(a.A + (size_t)ch0 * a.N, j * CL + cl, A[j]);
#pragma unroll
        for (int i = 0; i < NO; i++) {
            const uint32_t c = owned(i) * CL + cl;
            if (c < have && a.dbias) d[i] += __ldg(a.dbias + ch0 + c);
            if (a.softplus) d[i] = softplus_of(d[i]);
            in[i] = d[i] * u[i];
        }
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int i = SL == 1 ? j : (SL == 2 ? j % 2 : 0);
            const float dj = SL == 1 ? d[i] : __shfl_sync(0xFFFFFFFFu, d[i], owner(j)), ij = SL == 1 ? in[i] : __shfl_sync(0xFFFFFFFFu, in[i], owner(j));
            y[j] = 0.0f;
#pragma unroll
            for (int n = 0; n < 4; n++) {
                h[j][n] = fmaf(decay(dj, A[j][n] * kLog2e), h[j][n], ij * b[n]);
                y[j] = fmaf(h[j][n], cc[n], y[j]);
            }
        }
        if constexpr (SL >= 2) {
            const bool hi = sl & 1;
            const float k0 = hi ? y[2] : y[0], k1 = hi ? y[3] : y[1], s0 = hi ? y[0] : y[2], s1 = hi ? y[1] : y[3];
            y[0] = k0 + __shfl_xor_sync(0xFFFFFFFFu, s0, 1);
            y[1] = k1 + __shfl_xor_sync(0xFFFFFFFFu, s1, 1);
        }
        if constexpr (SL >= 4) {
            const bool hi = sl & 2;
            const float k0 = hi ? y[1] : y[0], s0 = hi ? y[0] : y[1];
            y[0] = k0 + __shfl_xor_sync(0xFFFFFFFFu, s0, 2);
        }
#pragma unroll
        for (int m = 4; m < SL; m <<= 1) y[0] += __shfl_xor_sync(0xFFFFFFFFu, y[0], m);
        if (SL <= 4 || sl < 4) {
#pragma unroll
            for (int i = 0; i < NO; i++) {
                const uint32_t c = owned(i) * CL + cl;
                if (c >= have) continue;
                float v = y[i];
                if (a.Dk) v = fmaf(__ldg(a.Dk + ch0 + c), u[i], v);
                if (a.z) v *= z[i] * sigmoid<T>(z[i]);
                ((T*)a.y)[at * a.ldy + ch0 + c] = from_f32<T>(v);
            }
        }
    }
    if (so) {
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t c = j * CL + cl;
            if (c >= have) continue;
            if constexpr (VEC) { if (mine) *reinterpret_cast<float4*>(so + c * a.N + sl * 4) = make_float4(h[j][0], h[j][1], h[j][2], h[j][3]); }
            else {
#pragma unroll
                for (int n = 0; n < 4; n++) if (sl * 4 + n < (int)a.N) so[c * a.N + sl * 4 + n] = h[j][n];
            }
        }
    }
}

}  // namespace

extern "C" int sf_seq_scan_workspace(uint32_t n_seq, uint32_t max_len, uint32_t rows, uint32_t D, uint32_t N, uint32_t G, int backward, size_t* bytes_out)
{
    if (!bytes_out || !sizes_ok(rows, n_seq, max_len, D, N, G)) return SF_ERR_ARG;
    *bytes_out = part_bytes(plan_of(n_seq, max_len, D, N, G, false), n_seq, D, N);
    if (backward) *bytes_out = std::max(*bytes_out, back_bytes(plan_of(n_seq, max_len, D, N, G, true), n_seq, rows, D, N, G));
    return SF_OK;
}

extern "C" int sf_seq_scan_starts(uint32_t n_seq, uint32_t rows, uint32_t D, uint32_t N, size_t* floats_out)
{
    if (!floats_out || !sizes_ok(rows, n_seq, 1, D, N, 1)) return SF_ERR_ARG;
    *floats_out = ((size_t)rows / kEvery + n_seq) * D * N;
    return SF_OK;
}

extern "C" int sf_seq_scan(sf_ctx* ctx, const sf_sequences* seq, const sf_scan_rows* in, uint32_t rows, const float* state_in, float* state_out, uint32_t n_slots,
                           float* starts_out, void* y_out, size_t ldy, void* workspace, size_t workspace_bytes, void* stream)
{
    const int ok = check(ctx, seq, in, rows);
    if (ok != SF_OK) return ok;
    if (n_slots > 0x7FFFFFFFu || ldy < in->D || (rows && !y_out) || !aligned(y_out, type_bytes(in->dtype)) || !aligned(state_in, 4) || !aligned(state_out, 4) || !aligned(starts_out, 4) ||
        !aligned(workspace, 4) || overlap_in_part(state_in, state_out, (size_t)n_slots * in->D * in->N * 4)) return SF_ERR_ARG;
    if (seq->n_seq == 0) return SF_OK;
    const Plan p = plan_of(seq->n_seq, seq->max_len, in->D, in->N, in->G, false);
    if (p.split && (!workspace || workspace_bytes < part_bytes(p, seq->n_seq, in->D, in->N))) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    cudaStream_t st = (cudaStream_t)stream;
    Scan a;
    fill(a, seq, in, rows, n_slots, p, ctx);
    a.state_in = state_in; a.state_out = state_out; a.starts = starts_out; a.y = y_out; a.ldy = ldy;
    const uint64_t blocks = ((uint64_t)seq->n_seq * in->G * p.cwarps + kWarps - 1) / kWarps;
    if (blocks > 0x7FFFFFFFu) return SF_ERR_ARG;
    const bool vec = fits(in) && fits(y_out, ldy, in->dtype);
    return by_type(in->dtype, [&](auto zero) {
        typedef decltype(zero) T;
        return by_states(p.sl, [&](auto lanes) {
            constexpr int SL = decltype(lanes)::value;
            if (seq->max_len == 1 && !starts_out) {
                const bool v4 = in->N % 4 == 0 && aligned(state_in, 16) && aligned(state_out, 16) && aligned(in->A, 16);
                return launch(v4 ? step_kernel<T, SL, true> : step_kernel<T, SL, false>, (uint32_t)blocks, 32 * kWarps, 0, st, a);
            }
            // Where whole sequences leave much of the machine idle and are too many to go in parts: two channels a lane, twice the warps (us, with two and with four channels a lane:
            // 128 sequences of 64 rows x 256 bf16, 1024 warps with four, 20.9 and 27.9; 96 of 1024 x 512 415 and 477; but 512 of 64 x 256, 4096 warps, 66.6 and 59.2; 64 of 256 x 1024
            // fp32, 2048 warps, 141 and 130)
            const bool two = SL == 4 && vec && !p.split && (uint64_t)seq->n_seq * in->G * p.cwarps < (uint64_t)SF_NUM_SMS_DEFAULT * 10;
            return by_width<T, SL>(vec, states_fit(in), [&](auto v, auto pb) {
                constexpr int VV = decltype(v)::value, PB = decltype(pb)::value;
                if constexpr (SL == 4 && VV > 1) if (two) {
                    set_warps(a, (a.per + 15) / 16);
                    const uint64_t b = ((uint64_t)seq->n_seq * in->G * a.cwarps + kWarps - 1) / kWarps;
                    return launch(scan_kernel<T, SL, VV, PB, false, 2>, dim3((uint32_t)b, 1), 32 * kWarps, sizeof(Forward<T, SL, VV, PB, 2>) * kWarps, st, a);
                }
                const size_t smem = sizeof(Forward<T, SL, VV, PB, 4>) * kWarps;
                if (p.split) {
                    a.part_state = (float*)workspace;
                    a.part_step = (float*)((char*)workspace + sf_align256((size_t)seq->n_seq * p.parts * in->D * in->N * 4));
                    int e = launch(scan_kernel<T, SL, VV, PB, true, 4>, dim3((uint32_t)blocks, p.parts), 32 * kWarps, smem, st, a);
                    if (e == SF_OK) e = launch(parts_kernel<false>, dim3((uint32_t)(((uint64_t)in->D * in->N + 255) / 256), seq->n_seq), 256, 0, st, a);
                    if (e != SF_OK) return e;
                }
                return launch(scan_kernel<T, SL, VV, PB, false, 4>, dim3((uint32_t)blocks, p.parts), 32 * kWarps, smem, st, a);
            });
        });
    });
}
