// The packed 4-bit format's layout and its conversions (mx4.cu, mx4_gemm.cu).
//   data    uint8 [rows][row_bytes(K)]: two values a byte, the first in the low half; rows padded to whole blocks of 32
//   scales  one byte per block (exponent + 127; 255 = NaN) in tiles of 128 rows x 4 blocks = 512 bytes, tiles row block by row
//           block: the order in which the tensor cores' scale copies take them, so a tile goes to shared memory as it is
#pragma once
#include "common.cuh"

#define SF_MX4_MAX_K (1u << 24)

namespace sfmx {

__host__ __device__ __forceinline__ uint32_t row_bytes(uint32_t K) { return (K + 31) / 32 * 16; }
__host__ __device__ __forceinline__ uint32_t k_tiles(uint32_t K) { return (K + 127) / 128; }
__host__ __device__ __forceinline__ size_t scale_bytes(uint32_t rows, uint32_t K) { return ((size_t)rows + 127) / 128 * k_tiles(K) * 512; }
__device__ __forceinline__ size_t scale_at(uint32_t row, uint32_t block, uint32_t kt) {
    return ((size_t)(row / 128) * kt + block / 4) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// scale byte of a block whose largest magnitude has these bits
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}
__device__ __forceinline__ float scale_f32(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : (byte ? byte << 23 : 0x00400000u));
}

// eight values -> eight codes (value j in bits 4j..4j+3); RELU: negative ones become 0.  1 / scale = 2^(127 - byte) is a normal number for
// every byte <= 252, the largest that occurs.  A block that stands for NaN has codes 0.
template <bool RELU = false>
__device__ __forceinline__ uint32_t encode8(const float (&v)[8], uint32_t byte) {
    const float inv = __uint_as_float((254u - min(byte, 253u)) << 23);
    float q[8];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        uint64_t a, b;
        asm("mov.b64 %0, {%1, %2};" : "=l"(a) : "f"(v[j]), "f"(v[j + 1]));
        asm("mov.b64 %0, {%1, %1};" : "=l"(b) : "f"(inv));
        asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(a) : "l"(b));
        asm("mov.b64 {%0, %1}, %2;" : "=f"(q[j]), "=f"(q[j + 1]) : "l"(a));
    }
    uint32_t r;
    if constexpr (RELU)
        asm("{\n"
            ".reg .b8 b0, b1, b2, b3;\n"
            "cvt.rn.satfinite.relu.e2m1x2.f32 b0, %2, %1;\n"
            "cvt.rn.satfinite.relu.e2m1x2.f32 b1, %4, %3;\n"
            "cvt.rn.satfinite.relu.e2m1x2.f32 b2, %6, %5;\n"
            "cvt.rn.satfinite.relu.e2m1x2.f32 b3, %8, %7;\n"
            "mov.b32 %0, {b0, b1, b2, b3};\n"
            "}\n"
            : "=r"(r) : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    else
        asm("{\n"
            ".reg .b8 b0, b1, b2, b3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
            "mov.b32 %0, {b0, b1, b2, b3};\n"
            "}\n"
            : "=r"(r) : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    return byte == 255u ? 0u : r;
}
__device__ __forceinline__ void decode8(uint32_t codes, float scale, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n"
        ".reg .b8 b0, b1, b2, b3;\n"
        "mov.b32 {b0, b1, b2, b3}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n"
        "}\n"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[j]));
        v[2 * j] = f.x * scale;
        v[2 * j + 1] = f.y * scale;
    }
}

}  // namespace sfmx

int sf_launch_mx4_quantise(sf_ctx* ctx, const void* x, int dtype, uint32_t n_src, uint32_t K, size_t ld, const int32_t* row_ids,
                           const uint32_t* n_rows_dev, uint32_t capacity, uint8_t* data, uint8_t* scales, cudaStream_t st);
// the product's launch: offsets != nullptr: E weight matrices, expert e's rows are [offsets[e], offsets[e + 1]) (device)
struct sf_mx4_product {
    const uint8_t* a; const uint8_t* a_scales; const uint32_t* n_rows_dev; const uint32_t* offsets; uint32_t E, capacity;
    const uint8_t* w; const uint8_t* w_scales; uint32_t N, K; const float* bias; int relu, out_dtype;
    void* out; size_t ld; uint8_t* out_scales;
    // a head folded in (out unused): bf16 weights [16][N] with rows past C zero, bias, logits fp32 [capacity][C], labels (nullable)
    const void* head_w; const float* head_b; uint32_t C; float* logits; uint8_t* label;
};
int sf_launch_mx4_product(sf_ctx* ctx, const sf_mx4_product& p, cudaStream_t st);
bool sf_mx4_product_takes_head(sf_ctx* ctx, const sf_mx4_product& p);       // would the launch fold p's head in?
