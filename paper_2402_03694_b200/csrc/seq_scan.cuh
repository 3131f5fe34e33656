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
// (SL a power of two with 4 SL >= N), so a thread holds 4 x 4 states, the sums over states and over channels are both half done in registers, and what a lane
// reads of a row (steps, inputs, B, C) serves 16 states.  Rows go by tiles that the warp stages in shared memory of its own (softplus once an element) while the
// next tile's pieces are copied ahead.  In the forward pass nothing waits for another warp; the backward pass joins dB and dC over a block.
// Bound: an exponential a state, 16 a clock and SM, at N = 16 three times the time of the bytes.  4096 flows of up to 128 x 256 bf16 take 411 us (function unit 301),
// 64 x 512 x 512 with gradients 584 us, three quarters of them backward (325 instructions a row and warp, eight warps an SM).  A thread per channel would read B and C 16 states at
// a time for one channel and need 31 exchanges a row for dB and dC; 8 x 2 or 2 x 8 states a thread read as much and exchange more.
#pragma once
#include <algorithm>
#include "seq_common.cuh"

namespace sfscan {

using namespace sfseq;

constexpr int kWarps = 4;                  // warps of a block
constexpr uint32_t kEvery = SF_SCAN_EVERY; // rows between two states that are kept for the backward pass
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
    int n4;                                // states lie four by four on 16-byte boundaries
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
    bool few;                              // warps of all sequences in 32 bits
    uint32_t cblocks;                      // blocks over them
    sf_dev_state* st;
};

// index of the state kept before row t (a multiple of kEvery) of sequence s, which begins at row `first`: sequences do not overlap
__device__ __forceinline__ size_t start_index(uint32_t first, uint32_t s, uint32_t t) { return (size_t)first / kEvery + s + t / kEvery; }

// softplus(x) = max(x, 0) + ln(1 + e), e = exp(-|x|) <= 1; ln(1 + e) = 2 artanh(e / (2 + e)) by its series in q = e / (2 + e) <= 1/3 (the first
// term left out is q^14 / 15 < 2e-8 of the sum).  Keeps its relative accuracy where e is small, which ln(1 + e) by a logarithm does not.
__device__ __forceinline__ float softplus_of(float x) {
    const float e = exp_minus_abs(x), q = e * rcp(2.0f + e), q2 = q * q;
    float p = fmaf(q2, 1.0f / 13, 1.0f / 11);
    p = fmaf(q2, p, 1.0f / 9); p = fmaf(q2, p, 1.0f / 7); p = fmaf(q2, p, 1.0f / 5); p = fmaf(q2, p, 1.0f / 3); p = fmaf(q2, p, 1.0f);
    return fmaf(2.0f * q, p, fmaxf(x, 0.0f));
}

// the same for two values; ee: their exp(-|x|)
__device__ __forceinline__ f2 softplus2(f2 x, f2& ee) {
    float a, b, e, f;
    unpack2(x, a, b);
    ee = exp_minus_abs2(x);
    unpack2(add2(ee, dup2(2.0f)), e, f);
    const f2 q = mul2(ee, pack2(rcp(e), rcp(f))), q2 = mul2(q, q);
    f2 p = fma2(q2, dup2(1.0f / 13), dup2(1.0f / 11));
    p = fma2(q2, p, dup2(1.0f / 9)); p = fma2(q2, p, dup2(1.0f / 7)); p = fma2(q2, p, dup2(1.0f / 5)); p = fma2(q2, p, dup2(1.0f / 3)); p = fma2(q2, p, dup2(1.0f));
    return fma2(add2(q, q), p, pack2(fmaxf(a, 0.0f), fmaxf(b, 0.0f)));
}

// a = exp(delta A) with A in units of log2.  ex2.approx is low by 0.26 to 0.45 of 2^-24 on average for exponents from -1/2 to -2^-8 (by 0.1 for smaller ones, measured),
// which a state that lives a hundred rows adds up a hundred times: the argument is raised by as much as takes that out.  (On the CUDA cores by a polynomial for
// a quarter or half of the states, to relieve the function unit: 471 and 514 us where this takes 436.)
constexpr float kCentre = 3.2e-8f;
__device__ __forceinline__ float decay(float delta, float A) { return ex2(fmaf(delta, A, kCentre)); }
__device__ __forceinline__ f2 decay2(f2 delta, f2 A) {
    float a, b;
    unpack2(fma2(delta, A, dup2(kCentre)), a, b);
    return pack2(ex2(a), ex2(b));
}

// J: channels of a lane (4; the forward pass also 2, where warps are few)
template <int SL, int J = 4> struct Shape {
    static constexpr int CL = 32 / SL, CH = J * CL, NP = 4 * SL;               // channel lanes, channels of a warp, states with those that fill up
    static constexpr int K = J == 2 ? 16 : (SL == 1 ? 4 : 8);                  // rows of a tile of the forward pass (kEvery divides them, or they divide it)
};

// What a warp works on: sequence, group, first of its channels within the group and of all, and how many it has (none: nothing to do)
struct Item { uint32_t s, g, c0, ch0, have; };
__device__ __forceinline__ Item item_of(const Scan& a, uint32_t CH) {
    const uint32_t warps = a.G * a.cwarps, w = threadIdx.x / 32;
    Item i;
    uint32_t k;
    if (a.few) { const uint32_t at = blockIdx.x * kWarps + w; i.s = at / warps; k = at % warps; }
    else { const uint64_t at = (uint64_t)blockIdx.x * kWarps + w; i.s = (uint32_t)(at / warps); k = (uint32_t)(at % warps); }
    i.g = a.G == 1 ? 0 : k / a.cwarps;
    i.c0 = (k - i.g * a.cwarps) * CH;
    i.ch0 = i.g * a.per + i.c0;
    i.have = i.s < a.q.n_seq ? min(CH, a.per - i.c0) : 0;
    return i;
}

// How a warp stages a tile of K rows of CH channels: pieces of VV channels, piece i of a lane at row t(i), channel c(i).  Lanes without a piece have rows from K on.
template <int K, int CH, int VV> struct Pieces {
    static constexpr int VR = CH / VV, I = (K * VR + 31) / 32, RI = VR <= 32 ? 32 / VR : 1, CI = VR <= 32 ? 1 : VR / 32;
    int lt, lc;
    __device__ __forceinline__ explicit Pieces(int lane) : lt(VR <= 32 ? lane / VR : 0), lc((VR <= 32 ? lane % VR : lane) * VV) {}
    __device__ __forceinline__ int t(int i) const { return lt + i / CI * RI; }
    __device__ __forceinline__ int c(int i) const { return lc + i % CI * 32 * VV; }
    // what piece i lies beyond piece 0 in rows of pitch ld
    __device__ __forceinline__ static size_t step(int i, size_t ld) { return (size_t)(i / CI * RI) * ld + i % CI * 32 * VV; }
};

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

// 16 bytes into shared memory while the thread goes on; zeros where there is nothing
__device__ __forceinline__ void copy16(void* to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(void* to, const void* from, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// B and C of a tile on their way (PV states at once, pieces of B first); stage writes them as [2][K][NP], zeros where there is nothing.
// (PB: how many elements at once may be read.)
template <typename T, int PB, int K, int NP> struct States {
    static constexpr int PV = NP >= PB ? PB : 1, PR = NP / PV, I = (2 * K * PR + 31) / 32;
    static constexpr bool WHOLE = PV * sizeof(T) == 16;
    Piece<T, PV> p[I];
    // where piece i of a lane lies, and whether it is there
    template <typename U> __device__ __forceinline__ static const U* piece(const Scan& a, int i, size_t row0, uint32_t col, int rows, int lane, bool& there) {
        const int k = i * 32 + lane, t = k / PR % K, n = k % PR * PV;
        const bool second = k >= K * PR;
        there = k < 2 * K * PR && t < rows && n < (int)a.N;
        const U* p = (const U*)(second ? a.C : a.B);
        return there ? p + (row0 + t) * (second ? a.ldc : a.ldb) + col + n : p;
    }
    __device__ __forceinline__ void fetch_all(const Scan& a, size_t row0, uint32_t col, int rows, int lane) {
#pragma unroll
        for (int i = 0; i < I; i++) {
            bool there;
            const T* q = piece<T>(a, i, row0, col, rows, lane, there);
            p[i] = fetch<T, PV>(q, 0, there);
        }
    }
    __device__ __forceinline__ void take(int i, uint4 w) { if constexpr (WHOLE) p[i].w = w; }
    __device__ __forceinline__ void stage(float* sh, int lane) const {
#pragma unroll
        for (int i = 0; i < I; i++) {
            const int k = i * 32 + lane;
            if (k >= 2 * K * PR) continue;
            float x[PV];
            open<T, PV>(p[i], x);
            if constexpr (PV == 1) sh[k] = x[0];
            else {
#pragma unroll
                for (int e = 0; e < PV; e += 4) *reinterpret_cast<float4*>(sh + k * PV + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
            }
        }
    }
};

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
    constexpr uint32_t U = 8;                              // parts on their way at once: only h goes from one to the next
    for (uint32_t i0 = 0; i0 < parts; i0 += U) {
        float end[U], step[U];
#pragma unroll
        for (uint32_t u = 0; u < U; u++) {
            const uint32_t p = BACK ? parts - 1 - (i0 + u) : i0 + u;
            if (i0 + u < parts) { end[u] = ps[(size_t)p * DN]; step[u] = steps[(size_t)p * a.D]; }
        }
#pragma unroll
        for (uint32_t u = 0; u < U; u++) {
            const uint32_t p = BACK ? parts - 1 - (i0 + u) : i0 + u;
            if (i0 + u >= parts) continue;
            ps[(size_t)p * DN] = h;
            h = fmaf(decay(step[u], A), h, end[u]);
        }
    }
    if (!BACK && parts == 0) ps[0] = h;
    if (out && r.slot >= 0) out[(size_t)r.slot * DN + at] = h;
}

// ---- host ----------------------------------------------------------------------------------------------------------------------------
inline int state_lanes(uint32_t N) { int sl = 1; while ((uint32_t)(4 * sl) < N) sl *= 2; return sl; }

struct Plan { uint32_t sl, cwarps, cblocks, part_len, parts, runs; bool split; };

// Where warps or channels are few a warp takes fewer channels (more state lanes than states need: lanes stay idle, but a tile is staged and walked by more warps),
// and where they would still leave most of the machine idle, sequences go in parts.
inline Plan plan_of(uint32_t n_seq, uint32_t max_len, uint32_t D, uint32_t N, uint32_t G, bool backward) {
    Plan p;
    p.sl = state_lanes(N);
    const uint32_t per = D / G;
    const uint64_t full = (uint64_t)SF_NUM_SMS_DEFAULT * (backward ? 8 : 16);
    auto warps = [&]() { p.cwarps = (per + 128 / p.sl - 1) / (128 / p.sl); return std::max<uint64_t>(1, (uint64_t)n_seq * G * p.cwarps); };
    while (max_len > 1 && p.sl < 16 && (64 / p.sl >= per || warps() * ((max_len + 63) / 64) < full / 4)) p.sl *= 2;
    const uint64_t want = full / warps();
    p.cblocks = (p.cwarps + kWarps - 1) / kWarps;
    p.part_len = (max_len + kEvery - 1) / kEvery * kEvery;
    // Parts are two passes over the inputs and a kernel between them.  Forward they pay from six times as many warps on, and of short sequences from more (256 channels bf16, us, in parts
    // and not: 32 x 256 rows 39 and 41, 48 x 256 53 and 45; 48 x 1024 160 and 170, 64 x 1024 228 and 213; 4 x 96 22 and 29, 32 x 96 38 and 30); backward, where a warp waits for itself,
    // from twice as many (64 x 256 146 and 206, 64 x 1024 543 and 807).
    const bool parts = backward ? want >= 2 : want >= 6 && want * max_len >= 1700;
    if (n_seq && parts && max_len > 2 * 32) p.part_len = (uint32_t)std::max<uint64_t>(32, ((max_len + want - 1) / want + kEvery - 1) / kEvery * kEvery);
    p.parts = (max_len + p.part_len - 1) / p.part_len;
    p.split = p.parts > 1;
    const uint64_t blocks = (uint64_t)G * p.cblocks, items = std::max<uint64_t>(1, (uint64_t)n_seq * p.parts);
    p.runs = (uint32_t)std::min<uint64_t>({items, 65535, std::max<uint64_t>(1, (uint64_t)SF_NUM_SMS_DEFAULT * 2 / blocks)});
    return p;
}
inline size_t part_bytes(const Plan& p, uint32_t n_seq, uint32_t D, uint32_t N) { return p.split ? sf_align256((size_t)n_seq * p.parts * D * N * 4) + sf_align256((size_t)n_seq * p.parts * D * 4) : 0; }
inline size_t back_bytes(const Plan& p, uint32_t n_seq, uint32_t rows, uint32_t D, uint32_t N, uint32_t G) {
    return part_bytes(p, n_seq, D, N) + sf_align256((size_t)p.runs * D * (N + 2) * 4) + (p.cblocks > 1 ? sf_align256((size_t)p.cblocks * rows * G * 2 * N * 4) : 0);
}

inline bool sizes_ok(uint32_t rows, uint32_t n_seq, uint32_t max_len, uint32_t D, uint32_t N, uint32_t G) {
    return rows <= SF_SEQ_MAX_ROWS && n_seq <= SF_SEQ_MAX_ROWS && max_len && max_len <= SF_SEQ_MAX_ROWS && D && D <= SF_EXPERT_MAX_D && N && N <= kMaxStates && G && D % G == 0;
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

inline int check(sf_ctx* ctx, const sf_sequences* seq, const sf_scan_rows* in, uint32_t rows) {
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
inline void set_warps(Scan& a, uint32_t cwarps) {
    a.cwarps = cwarps;
    a.few = ((uint64_t)a.q.n_seq + 1) * a.G * cwarps + kWarps <= 0xFFFFFFFFu;
}
inline void fill(Scan& a, const sf_sequences* seq, const sf_scan_rows* in, uint32_t rows, uint32_t n_slots, const Plan& p, sf_ctx* ctx) {
    a = {};
    a.q = seqs_of(seq, rows, n_slots);
    a.u = in->u; a.delta = in->delta; a.z = in->z; a.B = in->B; a.C = in->C;
    a.ldu = in->ldu; a.lddelta = in->ld_delta; a.ldz = in->ldz; a.ldb = in->ldb; a.ldc = in->ldc;
    a.A = in->A; a.Dk = in->D_skip; a.dbias = in->delta_bias;
    a.D = in->D; a.N = in->N; a.G = in->G; a.per = in->D / in->G; a.softplus = in->softplus != 0;
    a.n4 = in->N % 4 == 0;
    a.part_len = p.part_len; a.parts = p.parts; a.runs = p.runs; a.cblocks = p.cblocks;
    set_warps(a, p.cwarps);
    a.st = ctx->d_state;
}
// rows of channels begin on 16-byte boundaries, and so does every group's first channel
inline bool fits(const sf_scan_rows* in) {
    const uint32_t size = type_bytes(in->dtype), v = 16 / size;
    auto row = [&](const void* p, size_t ld) { return !p || (aligned(p, 16) && ld % v == 0); };
    return row(in->u, in->ldu) && row(in->delta, in->ld_delta) && row(in->z, in->ldz) && in->D / in->G % v == 0;
}
// rows of B and C do, and every group's first state.  They are asked for apart: rows of a few states seldom fit where rows of channels do
// (N = 3, 64 sequences of 512 rows x 512 with gradients: 1052 us with single elements for all, 550 with them for B and C alone).
inline bool states_fit(const sf_scan_rows* in) {
    const uint32_t v = 16 / type_bytes(in->dtype);
    return in->N % v == 0 && aligned(in->B, 16) && in->ldb % v == 0 && aligned(in->C, 16) && in->ldc % v == 0;
}
inline bool fits(const void* p, size_t ld, int dtype) { return !p || (aligned(p, 16) && ld % (16 / type_bytes(dtype)) == 0); }

// elements at once of rows of channels, and of rows of states
template <typename T, int SL, typename F> int by_width(bool rows, bool states, F f) {
    constexpr int V = 16 / (int)sizeof(T), P = 4 * SL >= V ? V : 1;
    typedef std::integral_constant<int, 1> One;
    if (!rows) return f(One(), One());
    return states && P > 1 ? f(std::integral_constant<int, V>(), std::integral_constant<int, P>()) : f(std::integral_constant<int, V>(), One());
}

template <typename K> int launch(K kernel, dim3 grid, uint32_t block, size_t smem, cudaStream_t st, const Scan& a) {
    if (smem > 48 * 1024) SF_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    SF_CUDA(sf_launch_chained(kernel, grid, block, smem, st, a));
    return SF_OK;
}

}  // namespace sfscan
