// Product of packed 4-bit rows with packed 4-bit weights: out[r][n] = act(sum_k A[r][k] W[n][k] + bias[n]), one weight matrix
// or one per expert over rows sorted by expert.
#include "rows_common.cuh"
#include "mx4.cuh"

namespace {
using namespace sfrow;
using namespace sfmx;

// 64 x 64 outputs per block, one scale block (32 values) of K at a time: both operands are widened to fp32 into shared memory,
// products accumulate in fp32.
__global__ void __launch_bounds__(256)
mx4_product_kernel(const sf_mx4_product p, sf_dev_state* st)
{
    __shared__ float As[32][64 + 4], Ws[32][64 + 4];
    sf_chain_enter();
    const uint32_t r0 = blockIdx.x * 64, n0 = blockIdx.y * 64;
    uint32_t end, e = 0;
    if (p.offsets) {
        // the expert whose rows these are: every expert's first row is a multiple of 128
        while (e < p.E && min(p.offsets[e + 1], p.capacity) <= r0) e++;
        if (e == p.E) return;
        end = min(p.offsets[e + 1], p.capacity);
        const uint32_t first = p.offsets[e];
        if (first > r0 || (first & 127u)) { if (threadIdx.x == 0) sf_dev_set_error(st, SF_ERR_ARG); return; }
    } else {
        end = p.n_rows_dev ? sf_clamp_rows(*p.n_rows_dev, p.capacity, st) : p.capacity;
        if (r0 >= end) return;
    }
    const uint32_t pitch = row_bytes(p.K), blocks = pitch / 16, kt = k_tiles(p.K);
    const uint8_t* w = p.w + (size_t)e * p.N * pitch;
    const uint8_t* ws = p.w_scales + (size_t)e * scale_bytes(p.N, p.K);
    const float* bias = p.bias ? p.bias + (size_t)e * p.N : nullptr;
    const uint32_t tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const uint32_t lr = threadIdx.x >> 2, lk = (threadIdx.x & 3) * 8;
    float acc[4][4] = {};
    for (uint32_t b = 0; b < blocks; b++) {
        float v[8] = {};
        if (r0 + lr < end) decode8(*reinterpret_cast<const uint32_t*>(p.a + (size_t)(r0 + lr) * pitch + b * 16 + lk / 2), scale_f32(p.a_scales[scale_at(r0 + lr, b, kt)]), v);
#pragma unroll
        for (int j = 0; j < 8; j++) As[lk + j][lr] = v[j];
        float u[8] = {};
        if (n0 + lr < p.N) decode8(*reinterpret_cast<const uint32_t*>(w + (size_t)(n0 + lr) * pitch + b * 16 + lk / 2), scale_f32(ws[scale_at(n0 + lr, b, kt)]), u);
#pragma unroll
        for (int j = 0; j < 8; j++) Ws[lk + j][lr] = u[j];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 32; k++)
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = fmaf(As[k][ty * 4 + i], Ws[k][tx * 4 + j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t r = r0 + ty * 4 + i;
        if (r >= end) continue;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t n = n0 + tx * 4 + j;
            if (n >= p.N) continue;
            float v = acc[i][j] + (bias ? bias[n] : 0.0f);
            if (p.relu) v = v < 0.0f ? 0.0f : v;           // keeps a NaN
            const size_t at = (size_t)r * p.ld + n;
            if (p.out_dtype == SF_F32) reinterpret_cast<float*>(p.out)[at] = v;
            else if (p.out_dtype == SF_BF16) reinterpret_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
            else reinterpret_cast<__half*>(p.out)[at] = __float2half_rn(v);
        }
    }
}

int check(const sf_ctx* ctx, const sf_mx4_product& p)
{
    if (!ctx || !type_ok(p.out_dtype) || p.N == 0 || p.K == 0 || p.K > SF_MX4_MAX_K || p.N > SF_MX4_MAX_K || p.ld < p.N) return SF_ERR_ARG;
    if (p.capacity == 0) return SF_OK;
    if (!p.a || !p.a_scales || !p.w || !p.w_scales || !p.out) return SF_ERR_ARG;
    if (!aligned(p.a, 16) || !aligned(p.a_scales, 16) || !aligned(p.w, 16) || !aligned(p.w_scales, 16)) return SF_ERR_ARG;
    if (!aligned(p.out, type_bytes(p.out_dtype)) || !aligned(p.bias, 4) || !aligned(p.n_rows_dev, 4) || !aligned(p.offsets, 4)) return SF_ERR_ARG;
    return SF_OK;
}

}  // namespace

int sf_launch_mx4_product(sf_ctx* ctx, const sf_mx4_product& p, cudaStream_t st)
{
    const dim3 grid((p.capacity + 63) / 64, (p.N + 63) / 64);
    SF_CUDA(sf_launch_chained(mx4_product_kernel, grid, 256, 0, st, p, ctx->d_state));
    return SF_OK;
}

extern "C" int sf_mx4_matmul(sf_ctx* ctx, const uint8_t* a, const uint8_t* a_scales, const uint32_t* n_rows_dev, uint32_t capacity,
                             const uint8_t* w, const uint8_t* w_scales, uint32_t N, uint32_t K, const float* bias, int relu,
                             int out_dtype, void* out, size_t ld, void* stream)
{
    const sf_mx4_product p = {a, a_scales, n_rows_dev, nullptr, 1, capacity, w, w_scales, N, K, bias, relu, out_dtype, out, ld, nullptr};
    const int rc = check(ctx, p);
    if (rc != SF_OK || capacity == 0) return rc;
    SF_ON_DEVICE(ctx);
    return sf_launch_mx4_product(ctx, p, (cudaStream_t)stream);
}

extern "C" int sf_mx4_matmul_experts(sf_ctx* ctx, const uint8_t* a, const uint8_t* a_scales, const uint32_t* offsets, uint32_t E,
                                     uint32_t capacity, const uint8_t* w, const uint8_t* w_scales, uint32_t N, uint32_t K,
                                     const float* bias, int relu, int out_dtype, void* out, size_t ld, void* stream)
{
    if (E == 0 || E > SF_MAX_EXPERTS || (capacity && !offsets)) return SF_ERR_ARG;
    const sf_mx4_product p = {a, a_scales, nullptr, offsets, E, capacity, w, w_scales, N, K, bias, relu, out_dtype, out, ld, nullptr};
    const int rc = check(ctx, p);
    if (rc != SF_OK || capacity == 0) return rc;
    SF_ON_DEVICE(ctx);
    return sf_launch_mx4_product(ctx, p, (cudaStream_t)stream);
}
