// Backward pass of the selective state space scan (formulas and mapping: seq_scan.cuh).
#include "seq_scan.cuh"

namespace {

using namespace sfscan;

template <int SL> struct Old {
    static constexpr int CL = 32 / SL, CH = 4 * CL, NP = 4 * SL, K = 512 / CH < 16 ? 512 / CH : 16, E = K * CH / 32;
};
// B or C of a tile (rows t0 .. t0 + K - 1 as far as there) into shared memory as [K][NP], zeros elsewhere
template <typename T, int VV, int K, int NP>
__device__ __forceinline__ void stage_states(float* sh, const void* base, size_t ld, size_t row0, uint32_t col, uint32_t N, int rows, int lane) {
    constexpr int PV = NP >= VV ? VV : 1, PR = NP / PV;
#pragma unroll
    for (int i = lane; i < K * PR; i += 32) {
        const int t = i / PR, n = i % PR * PV;
        float x[PV];
        open<T, PV>(fetch<T, PV>(base, (row0 + t) * ld + col + n, t < rows && n < (int)N), x);
#pragma unroll
        for (int e = 0; e < PV; e++) sh[t * NP + n + e] = x[e];
    }
}

template <int SL> struct Forward {
    typedef Old<SL> S;
    float step[S::K][S::CH], in[S::K][S::CH];              // delta; delta u, then y
    float B[S::K][S::NP], C[S::K][S::NP];
};

// ---- backward --------------------------------------------------------------------------------------------------------------------------
// ENDS of the backward pass: the gradient at a part's first state that the part's own rows cause, and the sum of its steps.
template <typename T, int SL, int VV>
__global__ void __launch_bounds__(32 * kWarps) back_ends_kernel(const Scan a) {
    sf_chain_enter();
    typedef Old<SL> S;
    constexpr int K = S::K, CH = S::CH, NP = S::NP, VR = CH / VV, I = S::E / VV, NB = VR > 32 ? VR / 32 : 1, VL = VR < 32 ? VR : 32;
    extern __shared__ __align__(16) unsigned char shared[];
    Forward<SL>& sh = reinterpret_cast<Forward<SL>*>(shared)[threadIdx.x / 32];
    const int lane = threadIdx.x & 31, cl = lane / SL, sl = lane % SL;
    const uint64_t item = (uint64_t)blockIdx.x * kWarps + threadIdx.x / 32, warps = (uint64_t)a.G * a.cwarps;
    if (item >= warps * a.q.n_seq) return;
    const uint32_t s = (uint32_t)(item / warps), g = (uint32_t)(item % warps) / a.cwarps, c0 = (uint32_t)(item % warps) % a.cwarps * CH;
    const uint32_t ch0 = g * a.per + c0, have = min((uint32_t)CH, a.per - c0);
    const Range r = range_of(a.q, s, a.st);
    const uint32_t part = blockIdx.y, t_begin = part * a.part_len, t_end = min(r.len, t_begin + a.part_len);
    if (t_begin >= r.len) return;
    float A[4][4], h[4][4];
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const uint32_t c = cl * 4 + j, st = sl * 4 + n;
            A[j][n] = c < have && st < a.N ? __ldg(a.A + (size_t)(ch0 + c) * a.N + st) * kLog2e : 0.0f;
            h[j][n] = 0.0f;
        }
    float bias[NB][VV], steps[NB][VV];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < VV; e++) {
            const uint32_t c = (b * 32 + lane % VL) * VV + e;
            bias[b][e] = c < have && a.dbias ? __ldg(a.dbias + ch0 + c) : 0.0f;
            steps[b][e] = 0.0f;
        }
    const uint32_t tiles = (t_end - t_begin + K - 1) / K;
    for (uint32_t tile = tiles; tile-- > 0;) {
        const uint32_t t0 = t_begin + tile * K;
        const int rows = (int)min((uint32_t)K, t_end - t0);
        const size_t row0 = (size_t)r.first + t0;
#pragma unroll
        for (int i = 0; i < I; i++) {
            const int t = (i * 32 + lane) / VR, b = i % NB, vc = (b * 32 + lane % VL) * VV;
            const bool vthere = vc < (int)have;
            const bool there = vthere && t < rows;
            float d[VV], e_[VV], z[VV];
            open<T, VV>(fetch<T, VV>(a.delta, (row0 + t) * a.lddelta + ch0 + vc, there), d);
            open<T, VV>(fetch<T, VV>(a.dy, (row0 + t) * a.lddy + ch0 + vc, there), e_);
            if (a.z) open<T, VV>(fetch<T, VV>(a.z, (row0 + t) * a.ldz + ch0 + vc, there), z);
#pragma unroll
            for (int e = 0; e < VV; e++) {
                float unused;
                d[e] += bias[b][e];
                if (a.softplus) d[e] = softplus_of(d[e], unused);
                if (!there) d[e] = 0.0f;
                if (a.z) e_[e] *= z[e] * sigmoid(z[e]);
                steps[b][e] += d[e];
                sh.step[t][vc + e] = d[e];
                sh.in[t][vc + e] = there ? e_[e] : 0.0f;
            }
        }
        stage_states<T, VV, K, NP>(&sh.C[0][0], a.C, a.ldc, row0, g * a.N, a.N, rows, lane);
        __syncwarp();
        for (int t = rows - 1; t >= 0; t--) {
            const float4 d4 = *reinterpret_cast<const float4*>(&sh.step[t][cl * 4]), i4 = *reinterpret_cast<const float4*>(&sh.in[t][cl * 4]);
            const float4 c4 = *reinterpret_cast<const float4*>(&sh.C[t][sl * 4]);
            const float d[4] = {d4.x, d4.y, d4.z, d4.w}, in[4] = {i4.x, i4.y, i4.z, i4.w}, c[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int n = 0; n < 4; n++) h[j][n] = decay(d[j], A[j][n]) * fmaf(in[j], c[n], h[j][n]);
        }
        __syncwarp();
    }
    float* out = a.part_state + ((size_t)s * a.parts + part) * a.D * a.N;
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
        for (int n = 0; n < 4; n++)
            if (cl * 4 + j < (int)have && sl * 4 + n < (int)a.N) out[(size_t)(ch0 + cl * 4 + j) * a.N + sl * 4 + n] = h[j][n];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < VV; e++) {
            const uint32_t c = (b * 32 + lane % VL) * VV + e;
            for (int m = VR; m < 32; m <<= 1) steps[b][e] += __shfl_xor_sync(0xFFFFFFFFu, steps[b][e], m);
            if (lane < VR && c < have) a.part_step[((size_t)s * a.parts + part) * a.D + ch0 + c] = steps[b][e];
        }
}

template <int SL> struct Backward {
    typedef Old<SL> S;
    static constexpr int K = S::K, Q = K / 4;              // rows of a tile, groups of 4 rows
    float step[K][S::CH], u[K][S::CH], e[K][S::CH], y[K][S::CH];      // delta, u, dout silu(z); y
    float s1[K][S::CH], s2[K][S::CH];                      // sum g B; sum (a g) h_{t-1} A
    float B[K][S::NP], C[K][S::NP];
    float4 start[Q][4][32];                                // states before each group of 4 rows
    float sum[K][2][S::NP];                                // the warp's dB, dC
};

// Sums of 32 values v[i] over the CL lanes that differ in cl; lane cl ends up with the 32 / CL sums i = cl * (32 / CL) ..
template <int SL> __device__ __forceinline__ void sum_channels(float (&v)[32], int lane) {
    int n = 32;
#pragma unroll
    for (int m = 16; m >= SL; m >>= 1) {
        n >>= 1;
        const bool hi = lane & m;
#pragma unroll
        for (int i = 0; i < 16; i++) {
            if (i >= n) break;
            const float keep = hi ? v[i + n] : v[i], give = hi ? v[i] : v[i + n];
            v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, m);
        }
    }
}

// One block: up to kWarps warps over neighbouring channels of a group, one part of one sequence after the other (a run), rows from last to first.
template <typename T, int SL, int VV>
__global__ void __launch_bounds__(32 * kWarps) back_kernel(const Scan a) {
    sf_chain_enter();
    typedef Old<SL> S;
    typedef Backward<SL> Sh;
    constexpr int K = S::K, CH = S::CH, NP = S::NP, VR = CH / VV, I = S::E / VV, NB = VR > 32 ? VR / 32 : 1, VL = VR < 32 ? VR : 32, Q = Sh::Q, CL = S::CL;
    extern __shared__ __align__(16) unsigned char shared[];
    Sh* all = reinterpret_cast<Sh*>(shared);
    const int warp = threadIdx.x / 32, warps = blockDim.x / 32;
    Sh& sh = all[warp];
    const int lane = threadIdx.x & 31, cl = lane / SL, sl = lane % SL;
    const uint32_t gb = blockIdx.x, g = gb / a.cblocks, cb = gb % a.cblocks;
    const uint32_t c0 = min(a.per, (cb * (uint32_t)kWarps + warp) * CH);
    const uint32_t ch0 = g * a.per + c0, have = min((uint32_t)CH, a.per - c0);     // (a warp behind the group's last channel has none, but meets the others)
    float A[4][4], dA[4][4];
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const uint32_t c = cl * 4 + j, st = sl * 4 + n;
            A[j][n] = c < have && st < a.N ? __ldg(a.A + (size_t)(ch0 + c) * a.N + st) * kLog2e : 0.0f;
            dA[j][n] = 0.0f;
        }
    float bias[NB][VV], Dk[NB][VV], dD[NB][VV], db[NB][VV];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < VV; e++) {
            const uint32_t c = (b * 32 + lane % VL) * VV + e;
            bias[b][e] = c < have && a.dbias ? __ldg(a.dbias + ch0 + c) : 0.0f;
            Dk[b][e] = c < have && a.Dk ? __ldg(a.Dk + ch0 + c) : 0.0f;
            dD[b][e] = db[b][e] = 0.0f;
        }
    const uint64_t items = (uint64_t)a.q.n_seq * a.parts;
    for (uint64_t it = blockIdx.y; it < items; it += a.runs) {
        const uint32_t s = (uint32_t)(it / a.parts), part = (uint32_t)(it % a.parts);
        const Range r = range_of(a.q, s, a.st);
        const uint32_t t_begin = part * a.part_len, t_end = min(r.len, t_begin + a.part_len);
        const bool whole = a.part_state == nullptr;        // the sequence in one part: gradients of states here
        if (t_begin >= r.len && !(whole && a.d_state0 && r.slot >= 0)) continue;
        float G[4][4];
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int n = 0; n < 4; n++) {
                const uint32_t c = cl * 4 + j, st = sl * 4 + n;
                const size_t at = (size_t)(ch0 + c) * a.N + st;
                G[j][n] = 0.0f;
                if (c < have && st < a.N) {
                    if (!whole) G[j][n] = a.part_state[((size_t)s * a.parts + part) * a.D * a.N + at];
                    else if (a.d_state && r.slot >= 0) G[j][n] = a.d_state[(size_t)r.slot * a.D * a.N + at];
                }
            }
        const uint32_t tiles = t_end > t_begin ? (t_end - t_begin + K - 1) / K : 0;
        for (uint32_t tile = tiles; tile-- > 0;) {
            const uint32_t t0 = t_begin + tile * K;
            const int rows = (int)min((uint32_t)K, t_end - t0);
            const size_t row0 = (size_t)r.first + t0;
            // the state before the tile: kept every kEvery rows, stepped on from there where tiles are shorter
            float h[4][4];
            const uint32_t kept = t0 / kEvery * kEvery;
            {
                const float* p = a.starts + start_index(r.first, s, kept) * a.D * a.N;
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int n = 0; n < 4; n++) {
                        const uint32_t c = cl * 4 + j, st = sl * 4 + n;
                        h[j][n] = c < have && st < a.N ? p[(size_t)(ch0 + c) * a.N + st] : 0.0f;
                    }
            }
            Piece<T, VV> pz[I], pg[I];
            for (uint32_t tt = kept; tt <= t0; tt += K) {
                const bool last = tt == t0;
                const int rr = last ? rows : K;
                const size_t row = (size_t)r.first + tt;
#pragma unroll
                for (int i = 0; i < I; i++) {
                    const int t = (i * 32 + lane) / VR, b = i % NB, vc = (b * 32 + lane % VL) * VV;
                    const bool vthere = vc < (int)have;
                    const bool there = vthere && t < rr;
                    float d[VV], u[VV], e_[VV], z[VV];
                    open<T, VV>(fetch<T, VV>(a.delta, (row + t) * a.lddelta + ch0 + vc, there), d);
                    open<T, VV>(fetch<T, VV>(a.u, (row + t) * a.ldu + ch0 + vc, there), u);
                    pg[i] = fetch<T, VV>(a.dy, (row + t) * a.lddy + ch0 + vc, there);
                    open<T, VV>(pg[i], e_);
                    if (a.z) { pz[i] = fetch<T, VV>(a.z, (row + t) * a.ldz + ch0 + vc, there); open<T, VV>(pz[i], z); }
#pragma unroll
                    for (int e = 0; e < VV; e++) {
                        float unused;
                        d[e] += bias[b][e];
                        if (a.softplus) d[e] = softplus_of(d[e], unused);
                        if (a.z) e_[e] *= z[e] * sigmoid(z[e]);
                        sh.step[t][vc + e] = there ? d[e] : 0.0f;
                        sh.u[t][vc + e] = u[e];
                        sh.e[t][vc + e] = there ? e_[e] : 0.0f;
                    }
                }
                stage_states<T, VV, K, NP>(&sh.B[0][0], a.B, a.ldb, row, g * a.N, a.N, rr, lane);
                stage_states<T, VV, K, NP>(&sh.C[0][0], a.C, a.ldc, row, g * a.N, a.N, rr, lane);
                __syncwarp();
                for (int t = 0; t < K; t++) {              // (rows that are not there: step 0, nothing comes in)
                    if (t % 4 == 0) {
#pragma unroll
                        for (int j = 0; j < 4; j++) sh.start[t / 4][j][lane] = make_float4(h[j][0], h[j][1], h[j][2], h[j][3]);
                    }
                    const float4 d4 = *reinterpret_cast<const float4*>(&sh.step[t][cl * 4]), u4 = *reinterpret_cast<const float4*>(&sh.u[t][cl * 4]);
                    const float4 b4 = *reinterpret_cast<const float4*>(&sh.B[t][sl * 4]), c4 = *reinterpret_cast<const float4*>(&sh.C[t][sl * 4]);
                    const float d[4] = {d4.x, d4.y, d4.z, d4.w}, u[4] = {u4.x, u4.y, u4.z, u4.w}, b[4] = {b4.x, b4.y, b4.z, b4.w};
                    float y[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float in = d[j] * u[j];
#pragma unroll
                        for (int n = 0; n < 4; n++) h[j][n] = fmaf(decay(d[j], A[j][n]), h[j][n], in * b[n]);
                        y[j] = h[j][0] * c4.x + h[j][1] * c4.y + h[j][2] * c4.z + h[j][3] * c4.w;
                    }
                    if (a.z) { sum_states<SL>(y, sl); put_states<SL>(&sh.y[t][cl * 4], y, sl); }
                }
                __syncwarp();
            }
            // groups of 4 rows from the last to the first; within a group channel by channel
            for (int q = Q - 1; q >= 0; q--) {
                float bc[32];                              // [row][dB, dC][state]
#pragma unroll
                for (int i = 0; i < 32; i++) bc[i] = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    float ha[4][4], al[4][4], hp[4];
                    const float4 s4 = sh.start[q][j][lane];
                    hp[0] = s4.x; hp[1] = s4.y; hp[2] = s4.z; hp[3] = s4.w;
#pragma unroll
                    for (int t = 0; t < 4; t++) {
                        const float d = sh.step[4 * q + t][cl * 4 + j], in = d * sh.u[4 * q + t][cl * 4 + j];
                        const float4 b4 = *reinterpret_cast<const float4*>(&sh.B[4 * q + t][sl * 4]);
                        const float b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                        for (int n = 0; n < 4; n++) {
                            al[t][n] = decay(d, A[j][n]);
                            ha[t][n] = fmaf(al[t][n], t ? ha[t - 1][n] : hp[n], in * b[n]);
                        }
                    }
                    float s1[4], s2[4];
#pragma unroll
                    for (int t = 3; t >= 0; t--) {
                        const float d = sh.step[4 * q + t][cl * 4 + j], in = d * sh.u[4 * q + t][cl * 4 + j], e = sh.e[4 * q + t][cl * 4 + j];
                        const float4 b4 = *reinterpret_cast<const float4*>(&sh.B[4 * q + t][sl * 4]), c4 = *reinterpret_cast<const float4*>(&sh.C[4 * q + t][sl * 4]);
                        const float b[4] = {b4.x, b4.y, b4.z, b4.w}, c[4] = {c4.x, c4.y, c4.z, c4.w};
                        s1[t] = s2[t] = 0.0f;
#pragma unroll
                        for (int n = 0; n < 4; n++) {
                            const float gt = fmaf(e, c[n], G[j][n]);
                            bc[t * 8 + n] = fmaf(gt, in, bc[t * 8 + n]);
                            bc[t * 8 + 4 + n] = fmaf(e, ha[t][n], bc[t * 8 + 4 + n]);
                            s1[t] = fmaf(gt, b[n], s1[t]);
                            G[j][n] = gt * al[t][n];
                            const float x = G[j][n] * (t ? ha[t - 1][n] : hp[n]);
                            s2[t] = fmaf(x, A[j][n], s2[t]);
                            dA[j][n] = fmaf(x, d, dA[j][n]);
                        }
                    }
                    sum_states<SL>(s1, sl);
                    sum_states<SL>(s2, sl);
                    // (here the four values are rows, not channels)
                    if constexpr (SL == 1) {
#pragma unroll
                        for (int t = 0; t < 4; t++) { sh.s1[4 * q + t][cl * 4 + j] = s1[t]; sh.s2[4 * q + t][cl * 4 + j] = s2[t]; }
                    } else if constexpr (SL == 2) {
#pragma unroll
                        for (int t = 0; t < 2; t++) { sh.s1[4 * q + 2 * sl + t][cl * 4 + j] = s1[t]; sh.s2[4 * q + 2 * sl + t][cl * 4 + j] = s2[t]; }
                    } else if (sl < 4) {
                        const int t = 2 * (sl & 1) + (sl >> 1 & 1);
                        sh.s1[4 * q + t][cl * 4 + j] = s1[0]; sh.s2[4 * q + t][cl * 4 + j] = s2[0];
                    }
                }
                sum_channels<SL>(bc, lane);
                constexpr int P = 32 / CL;                 // = SL
                // sum_channels halves by the highest lane bit first, so lane cl holds values rev .. : value index = cl * P + i
#pragma unroll
                for (int i = 0; i < P; i++) {
                    const int v = cl * P + i;
                    sh.sum[4 * q + v / 8][v / 4 & 1][sl * 4 + v % 4] = bc[i];
                }
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < I; i++) {
                const int t = (i * 32 + lane) / VR, b = i % NB, vc = (b * 32 + lane % VL) * VV;
                const bool vthere = vc < (int)have;
                if (!(vthere && t < rows)) continue;
                float du[VV], dd[VV], dzv[VV], z[VV], gy[VV], raw[VV];
                open<T, VV>(pg[i], gy);
                if (a.z) open<T, VV>(pz[i], z);
                open<T, VV>(fetch<T, VV>(a.delta, (row0 + t) * a.lddelta + ch0 + vc, a.softplus), raw);
#pragma unroll
                for (int e = 0; e < VV; e++) {
                    const float step = sh.step[t][vc + e], u = sh.u[t][vc + e], ee = sh.e[t][vc + e], s1 = sh.s1[t][vc + e];
                    du[e] = fmaf(Dk[b][e], ee, step * s1);
                    dd[e] = fmaf(u, s1, kLn2 * sh.s2[t][vc + e]);
                    if (a.softplus) dd[e] *= sigmoid(raw[e] + bias[b][e]);
                    dD[b][e] = fmaf(ee, u, dD[b][e]);
                    db[b][e] += dd[e];
                    if (a.z) { const float sg = sigmoid(z[e]); dzv[e] = gy[e] * fmaf(Dk[b][e], u, sh.y[t][vc + e]) * sg * (1.0f + z[e] * (1.0f - sg)); }
                }
                if (a.du) store_word<T, VV>((T*)a.du + (row0 + t) * a.lddu + ch0 + vc, du);
                if (a.ddelta) store_word<T, VV>((T*)a.ddelta + (row0 + t) * a.ldddelta + ch0 + vc, dd);
                if (a.dz) store_word<T, VV>((T*)a.dz + (row0 + t) * a.lddz + ch0 + vc, dzv);
            }
            // dB and dC: the block's warps, in their order
            __syncthreads();
            for (int i = threadIdx.x; i < rows * 2 * (int)a.N; i += blockDim.x) {
                const int t = i / (2 * (int)a.N), k = i / (int)a.N % 2, n = i % (int)a.N;
                float v = 0.0f;
                for (int w = 0; w < warps; w++) v += all[w].sum[t][k][n];
                if (a.sum_bc) a.sum_bc[((((size_t)cb * a.q.rows + row0 + t) * a.G + g) * 2 + k) * a.N + n] = v;
                else if (k == 0) { if (a.dB) ((T*)a.dB)[(row0 + t) * a.lddb + g * a.N + n] = from_f32<T>(v); }
                else if (a.dC) ((T*)a.dC)[(row0 + t) * a.lddc + g * a.N + n] = from_f32<T>(v);
            }
            __syncthreads();
        }
        if (whole && a.d_state0 && r.slot >= 0) {
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int n = 0; n < 4; n++)
                    if (cl * 4 + j < (int)have && sl * 4 + n < (int)a.N) a.d_state0[((size_t)r.slot * a.D + ch0 + cl * 4 + j) * a.N + sl * 4 + n] = G[j][n];
        }
    }
    if (!a.sum_par) return;
    float* par = a.sum_par + (size_t)blockIdx.y * a.D * (a.N + 2);
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
        for (int n = 0; n < 4; n++)
            if (cl * 4 + j < (int)have && sl * 4 + n < (int)a.N) par[(size_t)(ch0 + cl * 4 + j) * (a.N + 2) + sl * 4 + n] = dA[j][n];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < VV; e++) {
            const uint32_t c = (b * 32 + lane % VL) * VV + e;
            for (int m = VR; m < 32; m <<= 1) { dD[b][e] += __shfl_xor_sync(0xFFFFFFFFu, dD[b][e], m); db[b][e] += __shfl_xor_sync(0xFFFFFFFFu, db[b][e], m); }
            if (lane < VR && c < have) { par[(size_t)(ch0 + c) * (a.N + 2) + a.N] = dD[b][e]; par[(size_t)(ch0 + c) * (a.N + 2) + a.N + 1] = db[b][e]; }
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
            constexpr int SL = decltype(lanes)::value, VV = std::min(16 / (int)sizeof(T), Old<SL>::E);
            int e = SF_OK;
            if (p.split) {
                e = launch(vec ? back_ends_kernel<T, SL, VV> : back_ends_kernel<T, SL, 1>, dim3((uint32_t)blocks, p.parts), 32 * kWarps, sizeof(Forward<SL>) * kWarps, st, a);
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
