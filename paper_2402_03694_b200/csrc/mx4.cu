// Microscaled 4-bit floating point: rows of bf16, fp16 or fp32 into packed 4-bit values with one power-of-two scale per
// 32 values, back, and the product of packed rows with packed weights.
//
// A block of 32 values x_i becomes 2^e * q_i with e = max(floor(log2(max |x_i|)) - 2, -127) (the largest 4-bit magnitude, 6,
// lies in [2^2, 2^3)) and q_i = x_i * 2^-e rounded to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even code, beyond
// 6 to 6).  Scaling by a power of two is exact and e is read off the exponent bits, so the one rounding is the 4-bit one: the
// kernel and any other evaluation of the formula agree bit for bit.  A block that holds an infinity or a NaN stands for NaN
// (scale byte 255, codes 0).
#include "rows_common.cuh"
#include <algorithm>
#include "mx4.cuh"

namespace {
using namespace sfrow;
using namespace sfmx;

constexpr uint32_t kQThreads = 256;
constexpr uint32_t kQCols = 256;                   // columns a warp takes at once: 8 per lane, 4 lanes to a scale block

// x[rows][ld] -> data[rows][pitch], scales (tiles).  Bound: HBM (reads 2 or 4 bytes a value, writes 17/32).  A warp takes 256
// consecutive values of one row (one 16-byte load per lane for 16-bit types, 8 four-bit codes = one 4-byte store per lane);
// the block's maximum is taken over 4 lanes.  Items are (row, 256 columns), kUnroll of them in flight per warp.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kQThreads)
mx4_quantise_kernel(const T* __restrict__ x, uint32_t n_src, uint32_t K, size_t ld, const int32_t* __restrict__ row_ids,
                    const uint32_t* __restrict__ n_rows_dev, uint32_t capacity, uint8_t* __restrict__ data,
                    uint8_t* __restrict__ scales, sf_dev_state* st)
{
    sf_chain_enter();
    const uint32_t rows = n_rows_dev ? sf_clamp_rows(*n_rows_dev, capacity, st) : capacity;
    const uint32_t pitch = row_bytes(K), blocks = pitch / 16, kt = k_tiles(K);
    const uint32_t chunks = (kt * 128 + kQCols - 1) / kQCols;
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t items = (uint64_t)rows * chunks;
    const uint64_t step = (uint64_t)gridDim.x * (kQThreads / 32);
    for (uint64_t i = (uint64_t)blockIdx.x * (kQThreads / 32) + (threadIdx.x >> 5); i < items; i += step) {
        const uint32_t row = (uint32_t)(i / chunks), c = (uint32_t)(i - (uint64_t)row * chunks);
        const uint32_t k = c * kQCols + lane * 8;
        int64_t src = row;
        if (row_ids) { const int32_t id = row_ids[row]; src = (id >= 0 && (uint32_t)id < n_src) ? id : -1; }
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = 0.0f;
        if (src >= 0 && k < K) {
            const T* p = x + (size_t)src * ld + k;
            if (ALIGNED && k + 8 <= K) load_f32<T, 8, ALIGNED>(p, v);
            else {
#pragma unroll
                for (int j = 0; j < 8; j++) if (k + j < K) v[j] = to_f32(p[j]);
            }
        }
        uint32_t top = 0;                          // bits of the block's largest magnitude: they order as the values do
#pragma unroll
        for (int j = 0; j < 8; j++) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const uint32_t byte = scale_byte(top);
        const uint32_t codes = encode8(v, byte);
        if (k < pitch * 2) *reinterpret_cast<uint32_t*>(data + (size_t)row * pitch + k / 2) = codes;
        if ((lane & 3) == 0) {
            const uint32_t b = k / 32;
            if (b < kt * 4) scales[scale_at(row, b, kt)] = b < blocks ? (uint8_t)byte : (uint8_t)127;
        }
    }
}

// data, scales -> out[rows][ld].  The same split as above, the other way round.  Bound: HBM.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kQThreads)
mx4_unpack_kernel(const uint8_t* __restrict__ data, const uint8_t* __restrict__ scales, const uint32_t* __restrict__ n_rows_dev,
                  uint32_t capacity, uint32_t K, T* __restrict__ out, size_t ld, sf_dev_state* st)
{
    sf_chain_enter();
    const uint32_t rows = n_rows_dev ? sf_clamp_rows(*n_rows_dev, capacity, st) : capacity;
    const uint32_t pitch = row_bytes(K), kt = k_tiles(K);
    const uint32_t chunks = (K + kQCols - 1) / kQCols;
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t items = (uint64_t)rows * chunks;
    const uint64_t step = (uint64_t)gridDim.x * (kQThreads / 32);
    for (uint64_t i = (uint64_t)blockIdx.x * (kQThreads / 32) + (threadIdx.x >> 5); i < items; i += step) {
        const uint32_t row = (uint32_t)(i / chunks), c = (uint32_t)(i - (uint64_t)row * chunks);
        const uint32_t k = c * kQCols + lane * 8;
        if (k >= K) continue;
        float v[8];
        decode8(*reinterpret_cast<const uint32_t*>(data + (size_t)row * pitch + k / 2), scale_f32(scales[scale_at(row, k / 32, kt)]), v);
        T* p = out + (size_t)row * ld + k;
        if (ALIGNED && k + 8 <= K) store_f32<T, 8, ALIGNED>(p, v);
        else {
#pragma unroll
            for (int j = 0; j < 8; j++) if (k + j < K) p[j] = from_f32<T>(v[j]);
        }
    }
}

// A grid that fills the machine but gives no warp an empty turn.
uint32_t row_grid(const sf_ctx* ctx, uint64_t items, uint32_t blocks_per_sm) {
    const uint64_t want = (items + kQThreads / 32 - 1) / (kQThreads / 32);
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(want, (uint64_t)ctx->num_sms * blocks_per_sm));
}

}  // namespace

extern "C" int sf_mx4_sizes(uint32_t rows, uint32_t K, size_t* data_bytes_out, size_t* scale_bytes_out)
{
    if (K == 0 || K > SF_MX4_MAX_K || (!data_bytes_out && !scale_bytes_out)) return SF_ERR_ARG;
    if (data_bytes_out) *data_bytes_out = (size_t)rows * row_bytes(K);
    if (scale_bytes_out) *scale_bytes_out = scale_bytes(rows, K);
    return SF_OK;
}

extern "C" int sf_mx4_quantise(sf_ctx* ctx, const void* x, int dtype, uint32_t n_src, uint32_t K, size_t ld, const int32_t* row_ids,
                               const uint32_t* n_rows_dev, uint32_t capacity, uint8_t* data_out, uint8_t* scales_out, void* stream)
{
    if (!ctx || !type_ok(dtype) || K == 0 || K > SF_MX4_MAX_K || ld < K) return SF_ERR_ARG;
    if (!row_ids && capacity > n_src) return SF_ERR_ARG;
    if (capacity == 0) return SF_OK;
    if ((!x && n_src) || !data_out || !scales_out) return SF_ERR_ARG;
    if (!aligned(x, type_bytes(dtype)) || !aligned(data_out, 16) || !aligned(scales_out, 16) || !aligned(row_ids, 4) || !aligned(n_rows_dev, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    return sf_launch_mx4_quantise(ctx, x, dtype, n_src, K, ld, row_ids, n_rows_dev, capacity, data_out, scales_out, (cudaStream_t)stream);
}

int sf_launch_mx4_quantise(sf_ctx* ctx, const void* x, int dtype, uint32_t n_src, uint32_t K, size_t ld, const int32_t* row_ids,
                           const uint32_t* n_rows_dev, uint32_t capacity, uint8_t* data, uint8_t* scales, cudaStream_t st)
{
    const uint32_t grid = row_grid(ctx, (uint64_t)capacity * ((k_tiles(K) * 128 + kQCols - 1) / kQCols), 8);
    const bool al = aligned(x, 16) && (ld * type_bytes(dtype)) % 16 == 0;
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        auto k = al ? mx4_quantise_kernel<T, true> : mx4_quantise_kernel<T, false>;
        SF_CUDA(sf_launch_chained(k, grid, kQThreads, 0, st, (const T*)x, n_src, K, ld, row_ids, n_rows_dev, capacity, data, scales, ctx->d_state));
        return SF_OK;
    });
}

extern "C" int sf_mx4_unpack(sf_ctx* ctx, const uint8_t* data, const uint8_t* scales, const uint32_t* n_rows_dev, uint32_t capacity,
                             uint32_t K, int dtype, void* out, size_t ld, void* stream)
{
    if (!ctx || !type_ok(dtype) || K == 0 || K > SF_MX4_MAX_K || ld < K) return SF_ERR_ARG;
    if (capacity == 0) return SF_OK;
    if (!data || !scales || !out) return SF_ERR_ARG;
    if (!aligned(out, type_bytes(dtype)) || !aligned(data, 16) || !aligned(scales, 16) || !aligned(n_rows_dev, 4)) return SF_ERR_ARG;
    SF_ON_DEVICE(ctx);
    const uint32_t grid = row_grid(ctx, (uint64_t)capacity * ((K + kQCols - 1) / kQCols), 8);
    const bool al = aligned(out, 16) && (ld * type_bytes(dtype)) % 16 == 0;
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        auto k = al ? mx4_unpack_kernel<T, true> : mx4_unpack_kernel<T, false>;
        SF_CUDA(sf_launch_chained(k, grid, kQThreads, 0, (cudaStream_t)stream, data, scales, n_rows_dev, capacity, K, (T*)out, ld, ctx->d_state));
        return SF_OK;
    });
}
