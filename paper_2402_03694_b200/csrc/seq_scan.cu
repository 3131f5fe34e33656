// Selective state space scan over the rows of sequences, and its gradients.  Per channel d (group g of channels) and state n:
//   delta_t = softplus(raw_t + bias) (or raw_t),  a_t = exp(delta_t A[n]),  h_t[n] = a_t[n] h_{t-1}[n] + delta_t u_t B_t[g][n],
//   y_t = sum_n C_t[g][n] h_t[n] + D u_t,  out_t = y_t silu(z_t) (or y_t).
// Backward, from the last row to the first, with e_t = dout_t silu(z_t) and G the gradient of h_t that later rows leave:
//   g_t = G + e_t C_t,  dC_t = sum_d e_t h_t,  dB_t = sum_d g_t delta_t u_t,  G <- a_t g_t,
//   du_t = D e_t + delta_t sum_n g_t B_t,  ddelta_t = u_t sum_n g_t B_t + sum_n (a_t g_t) h_{t-1} A,  dA = sum_t (a_t g_t) h_{t-1} delta_t,
//   dD = sum_t e_t u_t,  dz_t = dout_t y_t silu'(z_t),  draw_t = ddelta_t sigmoid(raw_t + bias) = dbias_t.
// States, decays and sums are fp32.
//
// Mapping: a warp owns CH = 128 / SL channels of one sequence; its lanes are CL = 32 / SL groups of 4 channels times SL groups of 4 states
// (SL the power of two with 4 SL >= N), so a thread holds 4 x 4 states and the sums over states and over channels are both half done in registers.  Rows go by tiles:
// steps, inputs times steps and B, C are staged in shared memory of the warp's own (softplus once an element), nothing waits for another warp.
#include <algorithm>
#include "seq_common.cuh"

namespace {

using namespace sfseq;

constexpr int kWarps = 4;                  // warps of a block
constexpr uint32_t kEvery = 16;            // rows between two states that are kept for the backward pass
constexpr uint32_t kMaxStates = SF_SCAN_MAX_STATES;

struct Scan {
    Seqs q;
    const void* u; const void* delta; const void* z; const void* B; const void* C;
    size_t ldu, lddelta, ldz, ldb, ldc;
    const float* A; const float* Dk; const float* dbias;
    uint32_t D, N, G, per;                 // per: channels of a group
    int softplus;
    const float* state_in; float* state_out;
    float* starts;
    void* y; size_t ldy;
    // sequences in parts
    uint32_t part_len, parts;              // rows of a part (a multiple of kEvery), parts of the longest sequence
    float* part_state; float* part_step;   // [n_seq][parts][D][N] state at a part's end from zero, then at its start; [n_seq][parts][D] sum of its steps
    // backward
    const void* dy; size_t lddy;
    const float* d_state; float* d_state0;
    void* du; void* ddelta; void* dz; void* dB; void* dC;
    size_t lddu, ldddelta, lddz, lddb, lddc;
    float* dA; float* dD; float* dbias_out;
    float* sum_bc;                         // [blocks of channels of a group][rows][G][2][N] where a group takes several blocks
    float* sum_par;                        // [runs][D][N + 2]: dA, dD, dbias
    uint32_t runs;                         // blocks behind one another over the sequences' parts
    uint32_t cwarps;                       // warps over the channels of a group
    uint32_t cblocks;                      // blocks over them
    sf_dev_state* st;
};

// index of the state kept before row t (a multiple of kEvery) of sequence s, which begins at row `first`: sequences do not overlap
__device__ __forceinline__ size_t start_index(uint32_t first, uint32_t s, uint32_t t) { return (size_t)first / kEvery + s + t / kEvery; }

// softplus(x) = max(x, 0) + ln(1 + e), e = exp(-|x|) <= 1; ln(1 + e) = 2 artanh(e / (2 + e)) by its series in q = e / (2 + e) <= 1/3 (the first
// term left out is q^14 / 15 < 2e-8 of the sum).  Keeps its relative accuracy where e is small, which ln(1 + e) by a logarithm does not.
__device__ __forceinline__ float softplus_of(float x, float& e) {
    e = ex2(-kLog2e * fabsf(x));
    const float q = e * rcp(2.0f + e), q2 = q * q;
    float p = fmaf(q2, 1.0f / 13, 1.0f / 11);
    p = fmaf(q2, p, 1.0f / 9); p = fmaf(q2, p, 1.0f / 7); p = fmaf(q2, p, 1.0f / 5); p = fmaf(q2, p, 1.0f / 3); p = fmaf(q2, p, 1.0f);
    return fmaf(2.0f * q, p, fmaxf(x, 0.0f));
}

// a = exp(delta A) with A in units of log2.  ex2.approx is low by 0.35 to 0.8 of 2^-24 on average (measured; by a thousand steps of 0.001 the state would be off by
// 2e-5): the argument is raised by as much as takes that out near 0, where states live long.
constexpr float kCentre = 3.2e-8f;
__device__ __forceinline__ float decay(float delta, float A) { return ex2(fmaf(delta, A, kCentre)); }

template <int SL> struct Shape {
    static constexpr int CL = 32 / SL, CH = 4 * CL, NP = 4 * SL;               // channel lanes, channels of a warp, states with those that fill up
    static constexpr int K = 512 / CH < 16 ? 512 / CH : 16;                    // rows of a tile
    static constexpr int E = K * CH / 32;                                      // elements of a tile a lane stages
};

// one value a lane from four a lane: lane sl of SL gets the sum over the SL lanes of value j = 2 (sl & 1) + (sl >> 1 & 1) (SL = 1: none)
template <int SL> __device__ __forceinline__ void sum_states(float (&v)[4], int sl) {
    if constexpr (SL >= 2) {
        const bool hi = sl & 1;
        const float k0 = hi ? v[2] : v[0], k1 = hi ? v[3] : v[1], s0 = hi ? v[0] : v[2], s1 = hi ? v[1] : v[3];
        v[0] = k0 + __shfl_xor_sync(0xFFFFFFFFu, s0, 1);
        v[1] = k1 + __shfl_xor_sync(0xFFFFFFFFu, s1, 1);
    }
    if constexpr (SL >= 4) {
        const bool hi = sl & 2;
        const float k0 = hi ? v[1] : v[0], s0 = hi ? v[0] : v[1];
        v[0] = k0 + __shfl_xor_sync(0xFFFFFFFFu, s0, 2);
    }
#pragma unroll
    for (int m = 4; m < SL; m <<= 1) v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], m);
}
// writes what sum_states left to p[0..3] of the lane's channels
template <int SL> __device__ __forceinline__ void put_states(float* p, const float (&v)[4], int sl) {
    if constexpr (SL == 1) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else if constexpr (SL == 2) *reinterpret_cast<float2*>(p + 2 * sl) = make_float2(v[0], v[1]);
    else if (sl < 4) p[2 * (sl & 1) + (sl >> 1 & 1)] = v[0];
}

// VV elements at once: 16 bytes of T, or one element
template <typename T, int VV> struct Piece { typename Word<VV * sizeof(T)>::type w; };
template <typename T, int VV> __device__ __forceinline__ void open(const Piece<T, VV>& p, float (&x)[VV]) {
    union { typename Word<VV * sizeof(T)>::type w; T e[VV]; } u;
    u.w = p.w;
#pragma unroll
    for (int i = 0; i < VV; i++) x[i] = to_f32(u.e[i]);
}
template <typename T, int VV> __device__ __forceinline__ Piece<T, VV> fetch(const void* base, size_t at, bool there) {
    Piece<T, VV> p = {};
    if (there) p.w = __ldg(reinterpret_cast<const typename Word<VV * sizeof(T)>::type*>(reinterpret_cast<const T*>(base) + at));
    return p;
}

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
    typedef Shape<SL> S;
    float step[S::K][S::CH], in[S::K][S::CH];              // delta; delta u, then y
    float B[S::K][S::NP], C[S::K][S::NP];
};

// The scan of a sequence, or of one part of it (blockIdx.y): from the state that `part_state` holds where sequences go in parts.
// ENDS: only the state at the part's end, from zero, and the sum of the part's steps.
template <typename T, int SL, int VV, bool ENDS>
__global__ void __launch_bounds__(32 * kWarps) scan_kernel(const Scan a) {
    sf_chain_enter();
    typedef Shape<SL> S;
    constexpr int K = S::K, CH = S::CH, NP = S::NP, VR = CH / VV, I = S::E / VV, NB = VR > 32 ? VR / 32 : 1, VL = VR < 32 ? VR : 32;
    extern __shared__ __align__(16) unsigned char shared[];
    Forward<SL>& sh = reinterpret_cast<Forward<SL>*>(shared)[threadIdx.x / 32];
    const int lane = threadIdx.x & 31, cl = lane / SL, sl = lane % SL;
    const uint64_t item = (uint64_t)blockIdx.x * kWarps + threadIdx.x / 32, warps = (uint64_t)a.G * a.cwarps;
    if (item >= warps * a.q.n_seq) return;
    const uint32_t s = (uint32_t)(item / warps), g = (uint32_t)(item % warps) / a.cwarps, c0 = (uint32_t)(item % warps) % a.cwarps * CH;
    const uint32_t ch0 = g * a.per + c0, have = min((uint32_t)CH, a.per - c0);      // the warp's first channel, its channels
    const Range r = range_of(a.q, s, a.st);
    const uint32_t part = blockIdx.y, t_begin = part * a.part_len, t_end = min(r.len, t_begin + a.part_len);
    if (ENDS ? t_begin >= r.len : (part && t_begin >= r.len)) return;
    float A[4][4], h[4][4];
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const uint32_t c = cl * 4 + j, st = sl * 4 + n;
            const bool there = c < have && st < a.N;
            const size_t at = (size_t)(ch0 + c) * a.N + st;
            A[j][n] = there ? __ldg(a.A + at) * kLog2e : 0.0f;
            h[j][n] = 0.0f;
            if (!ENDS && there) {
                if (a.part_state) h[j][n] = a.part_state[((size_t)s * a.parts + part) * a.D * a.N + at];
                else if (a.state_in && r.slot >= 0) h[j][n] = a.state_in[(size_t)r.slot * a.D * a.N + at];
            }
        }
    float bias[NB][VV], Dk[NB][VV], steps[NB][VV];         // of the channels that this lane stages
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < VV; e++) {
            const uint32_t c = (b * 32 + lane % VL) * VV + e;
            bias[b][e] = c < have && a.dbias ? __ldg(a.dbias + ch0 + c) : 0.0f;
            Dk[b][e] = c < have && a.Dk ? __ldg(a.Dk + ch0 + c) : 0.0f;
            steps[b][e] = 0.0f;
        }
    for (uint32_t t0 = t_begin; t0 < t_end; t0 += K) {
        const int rows = (int)min((uint32_t)K, t_end - t0);
        const size_t row0 = (size_t)r.first + t0;
        Piece<T, VV> pu[I], pz[I];
#pragma unroll
        for (int i = 0; i < I; i++) {
            const int t = (i * 32 + lane) / VR, b = i % NB, vc = (b * 32 + lane % VL) * VV;
            const bool vthere = vc < (int)have;
            const bool there = vthere && t < rows;
            pu[i] = fetch<T, VV>(a.u, (row0 + t) * a.ldu + ch0 + vc, there);
            if (!ENDS && a.z) pz[i] = fetch<T, VV>(a.z, (row0 + t) * a.ldz + ch0 + vc, there);
            float d[VV], u[VV];
            open<T, VV>(fetch<T, VV>(a.delta, (row0 + t) * a.lddelta + ch0 + vc, there), d);
            open<T, VV>(pu[i], u);
#pragma unroll
            for (int e = 0; e < VV; e++) {
                float unused;
                d[e] += bias[b][e];
                if (a.softplus) d[e] = softplus_of(d[e], unused);
                if (!there) d[e] = 0.0f;                   // (a row that is not there leaves the state as it is)
                steps[b][e] += d[e];
                sh.step[t][vc + e] = d[e];
                sh.in[t][vc + e] = d[e] * u[e];
            }
        }
        stage_states<T, VV, K, NP>(&sh.B[0][0], a.B, a.ldb, row0, g * a.N, a.N, rows, lane);
        if (!ENDS) stage_states<T, VV, K, NP>(&sh.C[0][0], a.C, a.ldc, row0, g * a.N, a.N, rows, lane);
        __syncwarp();
        for (int t = 0; t < rows; t++) {
            if (!ENDS && a.starts && (t0 + t) % kEvery == 0) {
                float* p = a.starts + start_index(r.first, s, t0 + t) * a.D * a.N;
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int n = 0; n < 4; n++)
                        if (cl * 4 + j < (int)have && sl * 4 + n < (int)a.N) p[(size_t)(ch0 + cl * 4 + j) * a.N + sl * 4 + n] = h[j][n];
            }
            const float4 d4 = *reinterpret_cast<const float4*>(&sh.step[t][cl * 4]), i4 = *reinterpret_cast<const float4*>(&sh.in[t][cl * 4]);
            const float4 b4 = *reinterpret_cast<const float4*>(&sh.B[t][sl * 4]);
            const float d[4] = {d4.x, d4.y, d4.z, d4.w}, in[4] = {i4.x, i4.y, i4.z, i4.w}, b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int n = 0; n < 4; n++) h[j][n] = fmaf(decay(d[j], A[j][n]), h[j][n], in[j] * b[n]);
            if constexpr (!ENDS) {
                const float4 c4 = *reinterpret_cast<const float4*>(&sh.C[t][sl * 4]);
                float y[4];
#pragma unroll
                for (int j = 0; j < 4; j++) y[j] = h[j][0] * c4.x + h[j][1] * c4.y + h[j][2] * c4.z + h[j][3] * c4.w;
                sum_states<SL>(y, sl);
                __syncwarp();
                put_states<SL>(&sh.in[t][cl * 4], y, sl);
            }
        }
        __syncwarp();
        if constexpr (!ENDS) {
#pragma unroll
            for (int i = 0; i < I; i++) {
                const int t = (i * 32 + lane) / VR, b = i % NB, vc = (b * 32 + lane % VL) * VV;
                const bool vthere = vc < (int)have;
                if (!(vthere && t < rows)) continue;
                float u[VV], z[VV], y[VV];
                open<T, VV>(pu[i], u);
                if (a.z) open<T, VV>(pz[i], z);
#pragma unroll
                for (int e = 0; e < VV; e++) {
                    y[e] = fmaf(Dk[b][e], u[e], sh.in[t][vc + e]);
                    if (a.z) y[e] *= z[e] * sigmoid(z[e]);
                }
                store_word<T, VV>(reinterpret_cast<T*>(a.y) + (row0 + t) * a.ldy + ch0 + vc, y);
            }
            __syncwarp();
        }
    }
    float* out = nullptr;
    if (ENDS) out = a.part_state + ((size_t)s * a.parts + part) * a.D * a.N;
    else if (a.state_out && r.slot >= 0 && !a.part_state) out = a.state_out + (size_t)r.slot * a.D * a.N;
    if (out) {
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int n = 0; n < 4; n++)
                if (cl * 4 + j < (int)have && sl * 4 + n < (int)a.N) out[(size_t)(ch0 + cl * 4 + j) * a.N + sl * 4 + n] = h[j][n];
    }
    if constexpr (ENDS) {                                  // lanes on the same channels: lane, lane + VR, ..
#pragma unroll
        for (int b = 0; b < NB; b++)
#pragma unroll
            for (int e = 0; e < VV; e++) {
                const uint32_t c = (b * 32 + lane % VL) * VV + e;
                for (int m = VR; m < 32; m <<= 1) steps[b][e] += __shfl_xor_sync(0xFFFFFFFFu, steps[b][e], m);
                if (lane < VR && c < have) a.part_step[((size_t)s * a.parts + part) * a.D + ch0 + c] = steps[b][e];
            }
    }
}

// States at the parts' starts from those at their ends: h <- exp(A sum of steps) h + end, a thread per channel and state.  BACK: the same for the
// gradients, from the last part to the first (what a part holds then is the gradient at its start that its own rows cause).
template <bool BACK>
__global__ void __launch_bounds__(256) parts_kernel(const Scan a) {
    sf_chain_enter();
    const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint32_t s = blockIdx.y;
    const uint64_t DN = (uint64_t)a.D * a.N;
    if (at >= DN) return;
    const Range r = range_of(a.q, s, a.st);
    const uint32_t parts = (r.len + a.part_len - 1) / a.part_len;
    const float A = __ldg(a.A + at) * kLog2e;
    const float* in = BACK ? a.d_state : a.state_in;
    float* out = BACK ? a.d_state0 : a.state_out;
    float h = in && r.slot >= 0 ? in[(size_t)r.slot * DN + at] : 0.0f;
    float* ps = a.part_state + (size_t)s * a.parts * DN + at;
    const float* steps = a.part_step + (size_t)s * a.parts * a.D + at / a.N;
    for (uint32_t i = 0; i < parts; i++) {
        const uint32_t p = BACK ? parts - 1 - i : i;
        const float end = ps[(size_t)p * DN];
        ps[(size_t)p * DN] = h;
        h = fmaf(decay(steps[(size_t)p * a.D], A), h, end);
    }
    if (!BACK && parts == 0) ps[0] = h;
    if (out && r.slot >= 0) out[(size_t)r.slot * DN + at] = h;
}

// Single rows (max_len 1): a warp reads its channels' states once, steps them and writes them.
template <typename T, int SL, bool VEC>
__global__ void __launch_bounds__(32 * kWarps) step_kernel(const Scan a) {
    sf_chain_enter();
    constexpr int CL = 32 / SL, CH = 4 * CL;
    const int lane = threadIdx.x & 31, cl = lane / SL, sl = lane % SL;
    const uint64_t item = (uint64_t)blockIdx.x * kWarps + threadIdx.x / 32, warps = (uint64_t)a.G * a.cwarps;
    if (item >= warps * a.q.n_seq) return;
    const uint32_t s = (uint32_t)(item / warps), g = (uint32_t)(item % warps) / a.cwarps, c0 = (uint32_t)(item % warps) % a.cwarps * CH;
    const uint32_t ch0 = g * a.per + c0, have = min((uint32_t)CH, a.per - c0);
    const Range r = range_of(a.q, s, a.st);
    const bool row = r.len > 0;
    if (!row && !a.state_out) return;
    const size_t at = r.first;
    const T* u_ = (const T*)a.u + at * a.ldu + ch0; const T* d_ = (const T*)a.delta + at * a.lddelta + ch0; const T* z_ = (const T*)a.z + at * a.ldz + ch0;
    const T* B_ = (const T*)a.B + at * a.ldb + g * a.N; const T* C_ = (const T*)a.C + at * a.ldc + g * a.N;
    float h[4][4];
    // channel j CL + cl: the warp's accesses to the states of CL channels lie side by side
    const float* si = a.state_in && r.slot >= 0 ? a.state_in + ((size_t)r.slot * a.D + ch0) * a.N : nullptr;
    float* so = a.state_out && r.slot >= 0 ? a.state_out + ((size_t)r.slot * a.D + ch0) * a.N : nullptr;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const uint32_t c = j * CL + cl;
#pragma unroll
        for (int n = 0; n < 4; n++) h[j][n] = 0.0f;
        if (si && c < have) {
            if constexpr (VEC) {
                if (sl * 4 < (int)a.N) { const float4 v = *reinterpret_cast<const float4*>(si + c * a.N + sl * 4); h[j][0] = v.x; h[j][1] = v.y; h[j][2] = v.z; h[j][3] = v.w; }
            } else {
#pragma unroll
                for (int n = 0; n < 4; n++) if (sl * 4 + n < (int)a.N) h[j][n] = si[c * a.N + sl * 4 + n];
            }
        }
    }
    if (row) {
        float b[4], cc[4];
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const bool there = sl * 4 + n < (int)a.N;
            b[n] = there ? to_f32(B_[sl * 4 + n]) : 0.0f;
            cc[n] = there ? to_f32(C_[sl * 4 + n]) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t c = j * CL + cl;
            const bool there = c < have;
            const float u = there ? to_f32(u_[c]) : 0.0f;
            float d = there ? to_f32(d_[c]) : 0.0f, unused;
            if (there && a.dbias) d += __ldg(a.dbias + ch0 + c);
            if (a.softplus) d = softplus_of(d, unused);
            float y = 0.0f;
#pragma unroll
            for (int n = 0; n < 4; n++) {
                const float A = there && sl * 4 + n < (int)a.N ? __ldg(a.A + (size_t)(ch0 + c) * a.N + sl * 4 + n) * kLog2e : 0.0f;
                h[j][n] = fmaf(decay(d, A), h[j][n], d * u * b[n]);
                y = fmaf(h[j][n], cc[n], y);
            }
#pragma unroll
            for (int m = 1; m < SL; m <<= 1) y += __shfl_xor_sync(0xFFFFFFFFu, y, m);
            if (there && sl == 0) {
                if (a.Dk) y = fmaf(__ldg(a.Dk + ch0 + c), u, y);
                if (a.z) { const float z = to_f32(z_[c]); y *= z * sigmoid(z); }
                ((T*)a.y)[at * a.ldy + ch0 + c] = from_f32<T>(y);
            }
        }
    }
    if (so) {
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t c = j * CL + cl;
            if (c >= have) continue;
            if constexpr (VEC) {
                if (sl * 4 < (int)a.N) *reinterpret_cast<float4*>(so + c * a.N + sl * 4) = make_float4(h[j][0], h[j][1], h[j][2], h[j][3]);
            } else {
#pragma unroll
                for (int n = 0; n < 4; n++) if (sl * 4 + n < (int)a.N) so[c * a.N + sl * 4 + n] = h[j][n];
            }
        }
    }
}

// ---- backward --------------------------------------------------------------------------------------------------------------------------
// ENDS of the backward pass: the gradient at a part's first state that the part's own rows cause, and the sum of its steps.
template <typename T, int SL, int VV>
__global__ void __launch_bounds__(32 * kWarps) back_ends_kernel(const Scan a) {
    sf_chain_enter();
    typedef Shape<SL> S;
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
    typedef Shape<SL> S;
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
    typedef Shape<SL> S;
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

// ---- host ----------------------------------------------------------------------------------------------------------------------------
int state_lanes(uint32_t N) { int sl = 1; while ((uint32_t)(4 * sl) < N) sl *= 2; return sl; }

struct Plan { uint32_t sl, cwarps, cblocks, part_len, parts, runs; bool split; };

// Sequences go in parts where the warps of whole sequences would leave most of the machine idle: two passes over the inputs then, so only
// where parts make three times as many warps.
Plan plan_of(uint32_t n_seq, uint32_t max_len, uint32_t D, uint32_t N, uint32_t G, bool backward) {
    Plan p;
    p.sl = state_lanes(N);
    const uint32_t CH = 128 / p.sl, per = D / G;
    p.cwarps = (per + CH - 1) / CH;
    p.cblocks = (p.cwarps + kWarps - 1) / kWarps;
    const uint64_t warps = std::max<uint64_t>(1, (uint64_t)n_seq * G * p.cwarps), full = (uint64_t)SF_NUM_SMS_DEFAULT * (backward ? 8 : 16);
    uint64_t want = full / warps;
    p.part_len = (max_len + kEvery - 1) / kEvery * kEvery;
    if (want >= 3 && max_len > 2 * 64) p.part_len = (uint32_t)std::max<uint64_t>(64, ((max_len + want - 1) / want + kEvery - 1) / kEvery * kEvery);
    p.parts = (max_len + p.part_len - 1) / p.part_len;
    p.split = p.parts > 1;
    const uint64_t blocks = (uint64_t)G * p.cblocks, items = std::max<uint64_t>(1, (uint64_t)n_seq * p.parts);
    p.runs = (uint32_t)std::min<uint64_t>({items, 65535, std::max<uint64_t>(1, (uint64_t)SF_NUM_SMS_DEFAULT * 4 / blocks)});
    return p;
}
size_t part_bytes(const Plan& p, uint32_t n_seq, uint32_t D, uint32_t N) { return p.split ? sf_align256((size_t)n_seq * p.parts * D * N * 4) + sf_align256((size_t)n_seq * p.parts * D * 4) : 0; }
size_t back_bytes(const Plan& p, uint32_t n_seq, uint32_t rows, uint32_t D, uint32_t N, uint32_t G) {
    return part_bytes(p, n_seq, D, N) + sf_align256((size_t)p.runs * D * (N + 2) * 4) + (p.cblocks > 1 ? sf_align256((size_t)p.cblocks * rows * G * 2 * N * 4) : 0);
}

bool sizes_ok(uint32_t rows, uint32_t n_seq, uint32_t max_len, uint32_t D, uint32_t N, uint32_t G) {
    return rows <= 0x7FFFFFFFu && n_seq <= 0x7FFFFFFFu && max_len && max_len <= 0x7FFFFFFFu && D && D <= SF_EXPERT_MAX_D && N && N <= kMaxStates && G && D % G == 0;
}

template <typename F> int by_states(uint32_t sl, F f) {
    switch (sl) {
        case 1: return f(std::integral_constant<int, 1>());
        case 2: return f(std::integral_constant<int, 2>());
        case 4: return f(std::integral_constant<int, 4>());
        case 8: return f(std::integral_constant<int, 8>());
        default: return f(std::integral_constant<int, 16>());
    }
}

int check(sf_ctx* ctx, const sf_sequences* seq, const sf_scan_rows* in, uint32_t rows) {
    if (!ctx || !in || !type_ok(in->dtype)) return SF_ERR_ARG;
    const int ok = check_sequences(seq, rows);
    if (ok != SF_OK) return ok;
    if (!sizes_ok(rows, seq->n_seq, seq->max_len, in->D, in->N, in->G)) return SF_ERR_ARG;
    const size_t GN = (size_t)in->G * in->N;
    if (in->ldu < in->D || in->ld_delta < in->D || (in->z && in->ldz < in->D) || in->ldb < GN || in->ldc < GN || !in->A) return SF_ERR_ARG;
    if (rows && (!in->u || !in->delta || !in->B || !in->C)) return SF_ERR_ARG;
    const uint32_t size = type_bytes(in->dtype);
    if (!aligned(in->u, size) || !aligned(in->delta, size) || !aligned(in->z, size) || !aligned(in->B, size) || !aligned(in->C, size)) return SF_ERR_ARG;
    return aligned(in->A, 4) && aligned(in->D_skip, 4) && aligned(in->delta_bias, 4) ? SF_OK : SF_ERR_ARG;
}
void fill(Scan& a, const sf_sequences* seq, const sf_scan_rows* in, uint32_t rows, uint32_t n_slots, const Plan& p, sf_ctx* ctx) {
    a = {};
    a.q = seqs_of(seq, rows, n_slots);
    a.u = in->u; a.delta = in->delta; a.z = in->z; a.B = in->B; a.C = in->C;
    a.ldu = in->ldu; a.lddelta = in->ld_delta; a.ldz = in->ldz; a.ldb = in->ldb; a.ldc = in->ldc;
    a.A = in->A; a.Dk = in->D_skip; a.dbias = in->delta_bias;
    a.D = in->D; a.N = in->N; a.G = in->G; a.per = in->D / in->G; a.softplus = in->softplus != 0;
    a.part_len = p.part_len; a.parts = p.parts; a.runs = p.runs; a.cwarps = p.cwarps; a.cblocks = p.cblocks;
    a.st = ctx->d_state;
}
// rows begin on 16-byte boundaries, and so does every group's first channel and state
bool fits(const sf_scan_rows* in) {
    const uint32_t size = type_bytes(in->dtype), v = 16 / size;
    auto row = [&](const void* p, size_t ld) { return !p || (aligned(p, 16) && ld % v == 0); };
    return row(in->u, in->ldu) && row(in->delta, in->ld_delta) && row(in->z, in->ldz) && row(in->B, in->ldb) && row(in->C, in->ldc) && in->D / in->G % v == 0 && in->N % v == 0;
}
bool fits(const void* p, size_t ld, int dtype) { return !p || (aligned(p, 16) && ld % (16 / type_bytes(dtype)) == 0); }

template <typename K> int launch(K kernel, dim3 grid, uint32_t block, size_t smem, cudaStream_t st, const Scan& a) {
    if (smem > 48 * 1024) SF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    SF_CUDA(sf_launch_chained(kernel, grid, block, smem, st, a));
    return SF_OK;
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
        !aligned(workspace, 4)) return SF_ERR_ARG;
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
            constexpr int SL = decltype(lanes)::value, VV = std::min(16 / (int)sizeof(T), Shape<SL>::E);
            if (seq->max_len == 1 && !starts_out) {
                const bool v4 = in->N % 4 == 0 && aligned(state_in, 16) && aligned(state_out, 16);
                return launch(v4 ? step_kernel<T, SL, true> : step_kernel<T, SL, false>, (uint32_t)blocks, 32 * kWarps, 0, st, a);
            }
            const size_t smem = sizeof(Forward<SL>) * kWarps;
            if (p.split) {
                a.part_state = (float*)workspace;
                a.part_step = (float*)((char*)workspace + sf_align256((size_t)seq->n_seq * p.parts * in->D * in->N * 4));
                int e = launch(vec ? scan_kernel<T, SL, VV, true> : scan_kernel<T, SL, 1, true>, dim3((uint32_t)blocks, p.parts), 32 * kWarps, smem, st, a);
                if (e == SF_OK) e = launch(parts_kernel<false>, dim3((uint32_t)(((uint64_t)in->D * in->N + 255) / 256), seq->n_seq), 256, 0, st, a);
                if (e != SF_OK) return e;
            }
            return launch(vec ? scan_kernel<T, SL, VV, false> : scan_kernel<T, SL, 1, false>, dim3((uint32_t)blocks, p.parts), 32 * kWarps, smem, st, a);
        });
    });
}

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
            constexpr int SL = decltype(lanes)::value, VV = std::min(16 / (int)sizeof(T), Shape<SL>::E);
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
