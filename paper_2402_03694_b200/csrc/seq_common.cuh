// Pieces shared by the kernels that work on sequences of rows (seq_conv.cu, seq_scan.cu).
#pragma once
#include "rows_common.cuh"

namespace sfseq {

using namespace sfrow;

// What the kernels need of the sequences: sf_sequences, the rows that the arrays hold, the states that the pools hold.
struct Seqs {
    const uint32_t* offsets; const uint32_t* counts; const int32_t* slots;
    uint32_t n_seq, max_len, rows, n_slots;
};
struct Range { uint32_t first, len; int32_t slot; };

// Sequence s as far as the arrays hold it: offsets beyond the rows, counts beyond the offsets and lengths beyond max_len are cut
// (SF_ERR_CAPACITY), offsets that fall give no rows (SF_ERR_ARG), so no kernel reads or writes beyond what the caller named.
__device__ __forceinline__ Range range_of(const Seqs& q, uint32_t s, sf_dev_state* st) {
    Range r;
    const uint32_t a = __ldg(q.offsets + s);
    uint32_t b = __ldg(q.offsets + s + 1);
    int err = 0;
    if (b > q.rows) { b = q.rows; err = SF_ERR_CAPACITY; }
    if (b < a) { err = a > q.rows && err ? SF_ERR_CAPACITY : SF_ERR_ARG; b = a; }
    r.first = a; r.len = b - a;
    if (q.counts) { const uint32_t c = __ldg(q.counts + s); if (c > r.len) err = err ? err : SF_ERR_CAPACITY; else r.len = c; }
    if (r.len > q.max_len) { r.len = q.max_len; err = err ? err : SF_ERR_CAPACITY; }
    if (err) sf_dev_set_error(st, err);
    const int32_t slot = q.slots ? __ldg(q.slots + s) : (int32_t)s;
    r.slot = (uint32_t)slot < q.n_slots ? slot : -1;
    return r;
}

// ---- elementary functions in fp32 -----------------------------------------------------------------------------------
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr float kLog2eRest = 1.92596299e-8f;               // log2 e less kLog2e as a float
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// two fp32 values in a 64-bit register: one instruction for both
typedef unsigned long long f2;
__device__ __forceinline__ f2 pack2(float a, float b) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

__device__ __forceinline__ f2 dup2(float a) { return pack2(a, a); }
// exp(-|x|) with a relative error of 4 2^-24 at any x: what the product with log2 e loses, by its rounding and by log2 e's own, is worked out with fused multiply-adds and taken off
// the exponential by its slope.  (From |x| = 10^4 on, infinity included, the result is 0; a NaN stays one.)
__device__ __forceinline__ float abs_to_1e4(float x) { float y; asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(fabsf(x)), "f"(1e4f)); return y; }
__device__ __forceinline__ float exp_minus_abs(float x) {
    const float y = abs_to_1e4(x), t = -kLog2e * y, lost = fmaf(y, kLog2eRest, fmaf(y, kLog2e, t)), e = ex2(t);
    return fmaf(-kLn2 * e, lost, e);
}
__device__ __forceinline__ f2 exp_minus_abs2(f2 x) {
    float a, b;
    unpack2(x, a, b);
    const f2 y = pack2(abs_to_1e4(a), abs_to_1e4(b)), t = mul2(y, dup2(-kLog2e)), lost = fma2(y, dup2(kLog2eRest), fma2(y, dup2(kLog2e), t));
    unpack2(t, a, b);
    const f2 e = pack2(ex2(a), ex2(b));
    return fma2(mul2(e, dup2(-kLn2)), lost, e);
}

// Sigmoid of what is rounded to T in the end.  ex2 of a rounded product is off by |x| 2^-24, at most 2^-17.5 where the result is a normal number: a sixteenth of a rounding to 16 bits
// at most, but float rows would show it.  (By exp_minus_abs for 16 bits too: 8192 flows of up to 128 x 256 bf16 with gradients 405 us instead of 356.)
template <typename T> __device__ __forceinline__ float sigmoid(float x) {
    if constexpr (sizeof(T) == 4) { const float e = exp_minus_abs(x); return (x >= 0.0f ? 1.0f : e) * rcp(1.0f + e); }
    else return rcp(1.0f + ex2(-kLog2e * x));
}
template <typename T> __device__ __forceinline__ f2 sigmoid2(f2 x) {
    float a, b;
    if constexpr (sizeof(T) == 4) {
        const f2 e = exp_minus_abs2(x);
        float c, d, p, q;
        unpack2(x, a, b);
        unpack2(e, c, d);
        unpack2(add2(e, dup2(1.0f)), p, q);
        return mul2(pack2(a >= 0.0f ? 1.0f : c, b >= 0.0f ? 1.0f : d), pack2(rcp(p), rcp(q)));
    } else {
        unpack2(mul2(x, dup2(-kLog2e)), a, b);
        unpack2(add2(pack2(ex2(a), ex2(b)), dup2(1.0f)), a, b);
        return pack2(rcp(a), rcp(b));
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
inline int check_sequences(const sf_sequences* q, uint32_t rows) {
    if (!q || q->max_len == 0 || rows > SF_SEQ_MAX_ROWS || q->n_seq > SF_SEQ_MAX_ROWS || q->max_len > SF_SEQ_MAX_ROWS) return SF_ERR_ARG;
    if (q->n_seq && !q->offsets) return SF_ERR_ARG;
    return aligned(q->offsets, 4) && aligned(q->counts, 4) && aligned(q->slots, 4) ? SF_OK : SF_ERR_ARG;
}
// Two pools of `bytes` bytes that are neither one pool nor apart: what is read of the one would be what the call writes to another slot of the other.
inline bool overlap_in_part(const void* p, const void* q, size_t bytes) {
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    return p && q && a != b && (a < b ? b - a : a - b) < bytes;
}
inline Seqs seqs_of(const sf_sequences* q, uint32_t rows, uint32_t n_slots) {
    return {q->offsets, q->counts, q->slots, q->n_seq, q->max_len, rows, n_slots};
}

}  // namespace sfseq
