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
constexpr uint32_t kPCols = 512;                   // columns a warp packs or unpacks at once: 16 per lane, 2 lanes to a scale block

// item i of rows of `chunks` pieces -> row and piece (a 64-bit division only where 32 bits do not hold i)
__device__ __forceinline__ void row_and_piece(uint64_t i, uint32_t chunks, uint32_t& row, uint32_t& c) {
    if (i >> 32) { row = (uint32_t)(i / chunks); c = (uint32_t)(i - (uint64_t)row * chunks); }
    else { row = (uint32_t)i / chunks; c = (uint32_t)i - row * chunks; }
}

// bits of the largest magnitude of 16 values, as fp32: magnitudes order as their bits do, so 16-bit values are compared in pairs
// as they are
__device__ __forceinline__ uint32_t top_bits(const uint4 (&q)[4], float) {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        t = max(max(t, q[i].x & 0x7FFFFFFFu), q[i].y & 0x7FFFFFFFu);
        t = max(max(t, q[i].z & 0x7FFFFFFFu), q[i].w & 0x7FFFFFFFu);
    }
    return t;
}
__device__ __forceinline__ uint32_t top_16(const uint4 (&q)[2]) {
    uint32_t t = __vimax3_u16x2(q[0].x & 0x7FFF7FFFu, q[0].y & 0x7FFF7FFFu, q[0].z & 0x7FFF7FFFu);
    t = __vimax3_u16x2(t, q[0].w & 0x7FFF7FFFu, q[1].x & 0x7FFF7FFFu);
    t = __vimax3_u16x2(t, q[1].y & 0x7FFF7FFFu, q[1].z & 0x7FFF7FFFu);
    t = __vimax3_u16x2(t, q[1].w & 0x7FFF7FFFu, 0u);
    return max(t & 0xFFFFu, t >> 16);
}
__device__ __forceinline__ uint32_t top_bits(const uint4 (&q)[2], __nv_bfloat16) { return top_16(q) << 16; }
__device__ __forceinline__ uint32_t top_bits(const uint4 (&q)[2], __half) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)top_16(q)))); }

// x[rows][ld] -> data[rows][pitch], scales (tiles).  Bound: HBM (reads 2 or 4 bytes a value, writes 17/32).  A warp takes 512
// consecutive values of one row (16 per lane: two or four 16-byte loads, one 8-byte store), a block's maximum is taken over two
// lanes, and U such pieces are on their way before the first is packed.  Smaller pieces one at a time (8 values a lane) ran
// at 2.9 TB/s at 240,001 x 2048 bf16.
template <typename T, int U>
__global__ void __launch_bounds__(kQThreads)
mx4_quantise_kernel(const T* __restrict__ x, uint32_t n_src, uint32_t K, size_t ld, const int32_t* __restrict__ row_ids,
                    const uint32_t* __restrict__ n_rows_dev, uint32_t capacity, uint8_t* __restrict__ data,
                    uint8_t* __restrict__ scales, sf_dev_state* st)
{
    constexpr int Q = sizeof(T);                       // 16-byte words of 16 values
    sf_chain_enter();
    const uint32_t rows = n_rows_dev ? sf_clamp_rows(*n_rows_dev, capacity, st) : capacity;
    const uint32_t pitch = row_bytes(K), blocks = pitch / 16, kt = k_tiles(K);
    const uint32_t chunks = (kt * 128 + kPCols - 1) / kPCols;
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t items = (uint64_t)rows * chunks;
    const uint64_t step = (uint64_t)gridDim.x * (kQThreads / 32) * U;
    for (uint64_t i0 = ((uint64_t)blockIdx.x * (kQThreads / 32) + (threadIdx.x >> 5)) * U; i0 < items; i0 += step) {
        union Words { uint4 q[Q]; T e[16]; } w[U];
        uint32_t row[U], k[U];
        uint32_t r, c;
        row_and_piece(i0, chunks, r, c);
#pragma unroll
        for (int u = 0; u < U; u++) {
            row[u] = r;
            k[u] = c * kPCols + lane * 16;
            if (++c == chunks) { c = 0; r++; }
            int64_t src = i0 + u < items ? (int64_t)row[u] : -1;
            if (row_ids && src >= 0) { const int32_t id = row_ids[row[u]]; src = (id >= 0 && (uint32_t)id < n_src) ? id : -1; }
#pragma unroll
            for (int q = 0; q < Q; q++) w[u].q[q] = make_uint4(0, 0, 0, 0);
            if (src >= 0 && k[u] < K) {
                const T* p = x + (size_t)src * ld + k[u];
                if (k[u] + 16 <= K) {
#pragma unroll
                    for (int q = 0; q < Q; q++) w[u].q[q] = __ldg(reinterpret_cast<const uint4*>(p) + q);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; j++) if (k[u] + j < K) w[u].e[j] = p[j];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (i0 + u >= items) break;                // (the same in all lanes)
            uint32_t top = top_bits(w[u].q, T());
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            const uint32_t byte = scale_byte(top);
            float v[8];
            uint2 codes;
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = to_f32(w[u].e[j]);
            codes.x = encode8(v, byte);
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = to_f32(w[u].e[8 + j]);
            codes.y = encode8(v, byte);
            if (k[u] < pitch * 2) *reinterpret_cast<uint2*>(data + (size_t)row[u] * pitch + k[u] / 2) = codes;
            if ((lane & 1) == 0) {
                const uint32_t b = k[u] / 32;
                if (b < kt * 4) scales[scale_at(row[u], b, kt)] = b < blocks ? (uint8_t)byte : (uint8_t)127;
            }
        }
    }
}

// Place of element e in the buffer that turns 512 elements round: written and read without bank conflicts, by lanes that have consecutive
// elements (or pairs) and by lanes that have 16 consecutive ones as four 16-byte pieces.
__device__ __forceinline__ uint32_t turned(uint32_t e) { return (e & ~15u) | ((((e >> 2) ^ (e >> 5)) & 3u) << 2) | (e & 3u); }

// The same for rows on any boundary and for narrow ones: pieces of 128 columns (a row's share of a scale tile), four of them per warp, loaded
// W elements at a time (two 16-bit ones where rows are on 4-byte boundaries), coalesced, up to 16 loads a lane on their way, and turned round in shared memory so that a lane has 16 consecutive
// values of a piece (lanes that load their own 16 values element by element ran at 0.6 TB/s at 141,031 x 1065 bf16).
template <typename T, int W>
__global__ void __launch_bounds__(kQThreads)
mx4_quantise_any_kernel(const T* __restrict__ x, uint32_t n_src, uint32_t K, size_t ld, const int32_t* __restrict__ row_ids,
                        const uint32_t* __restrict__ n_rows_dev, uint32_t capacity, uint8_t* __restrict__ data,
                        uint8_t* __restrict__ scales, sf_dev_state* st)
{
    __shared__ float4 turn[kQThreads / 32][4 * 32];
    sf_chain_enter();
    const uint32_t rows = n_rows_dev ? sf_clamp_rows(*n_rows_dev, capacity, st) : capacity;
    const uint32_t pitch = row_bytes(K), blocks = pitch / 16, kt = k_tiles(K);
    const uint32_t lane = threadIdx.x & 31;
    float* const mine = reinterpret_cast<float*>(turn[threadIdx.x >> 5]);
    const uint64_t items = (uint64_t)rows * kt;
    const uint64_t step = (uint64_t)gridDim.x * (kQThreads / 32) * 4;
    for (uint64_t i0 = ((uint64_t)blockIdx.x * (kQThreads / 32) + (threadIdx.x >> 5)) * 4; i0 < items; i0 += step) {
        uint32_t r, c;
        row_and_piece(i0, kt, r, c);
        const uint32_t r0 = r, c0 = c;
        float v[4][4 / W][W];
#pragma unroll
        for (int u = 0; u < 4; u++) {
            int64_t src = i0 + u < items ? (int64_t)r : -1;
            if (row_ids && src >= 0) { const int32_t id = row_ids[r]; src = (id >= 0 && (uint32_t)id < n_src) ? id : -1; }
            const T* const p = x + (size_t)max(src, (int64_t)0) * ld + c * 128;
            const uint32_t left = src >= 0 ? K - c * 128 : 0u;               // values of the row from this piece on
#pragma unroll
            for (int j = 0; j < 4 / W; j++) {
                const uint32_t k = (j * 32 + lane) * W;
                if (k < left) load_word<T, W>(p + k, v[u][j]);               // (W = 2: K is even)
                else {
#pragma unroll
                    for (int w = 0; w < W; w++) v[u][j][w] = 0.0f;
                }
            }
            if (++c == kt) { c = 0; r++; }
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < 4; u++)
#pragma unroll
            for (int j = 0; j < 4 / W; j++) {
                float* const q = mine + turned(u * 128 + (j * 32 + lane) * W);
                if constexpr (W == 2) *reinterpret_cast<float2*>(q) = make_float2(v[u][j][0], v[u][j][1]); else *q = v[u][j][0];
            }
        __syncwarp();
        float y[2][8];
        uint32_t top = 0;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const float4 a = *reinterpret_cast<const float4*>(mine + turned(16 * lane + 8 * h)), b = *reinterpret_cast<const float4*>(mine + turned(16 * lane + 8 * h + 4));
            y[h][0] = a.x; y[h][1] = a.y; y[h][2] = a.z; y[h][3] = a.w;
            y[h][4] = b.x; y[h][5] = b.y; y[h][6] = b.z; y[h][7] = b.w;
#pragma unroll
            for (int j = 0; j < 8; j++) top = max(top, __float_as_uint(y[h][j]) & 0x7FFFFFFFu);
        }
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        const uint32_t byte = scale_byte(top), u = lane / 8;
        const uint2 codes = make_uint2(encode8(y[0], byte), encode8(y[1], byte));
        if (i0 + u >= items) continue;
        const uint32_t piece = c0 + u, row = r0 + piece / kt, k = (piece % kt) * 128 + (lane & 7) * 16;
        if (k < pitch * 2) *reinterpret_cast<uint2*>(data + (size_t)row * pitch + k / 2) = codes;
        if ((lane & 1) == 0) scales[scale_at(row, k / 32, kt)] = k / 32 < blocks ? (uint8_t)byte : (uint8_t)127;
    }
}

// data, scales -> out[rows][ld].  The same split the other way round: 16 values a lane, whole 32-byte sectors where rows are on
// 32-byte boundaries.  Bound: HBM writes (240,001 x 2048 bf16: 231 us, 4.3 TB/s written beside 1.2 read; a kernel that only fills memory reaches 3.9
// on this card, where a copy moves 6.5).
template <typename T>
__global__ void __launch_bounds__(kQThreads)
mx4_unpack_kernel(const uint8_t* __restrict__ data, const uint8_t* __restrict__ scales, const uint32_t* __restrict__ n_rows_dev,
                  uint32_t capacity, uint32_t K, T* __restrict__ out, size_t ld, sf_dev_state* st)
{
    constexpr int U = 2;
    sf_chain_enter();
    const uint32_t rows = n_rows_dev ? sf_clamp_rows(*n_rows_dev, capacity, st) : capacity;
    const uint32_t pitch = row_bytes(K), kt = k_tiles(K);
    const uint32_t chunks = (K + kPCols - 1) / kPCols;
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t items = (uint64_t)rows * chunks;
    const uint64_t step = (uint64_t)gridDim.x * (kQThreads / 32) * U;
    for (uint64_t i0 = ((uint64_t)blockIdx.x * (kQThreads / 32) + (threadIdx.x >> 5)) * U; i0 < items; i0 += step) {
        uint32_t r, c;
        row_and_piece(i0, chunks, r, c);
        uint2 codes[U];
        uint32_t byte[U], row[U], k[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            row[u] = r;
            k[u] = c * kPCols + lane * 16;
            if (++c == chunks) { c = 0; r++; }
            if (i0 + u < items && k[u] < K) {
                codes[u] = __ldg(reinterpret_cast<const uint2*>(data + (size_t)row[u] * pitch + k[u] / 2));
                byte[u] = __ldg(scales + scale_at(row[u], k[u] / 32, kt));
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (i0 + u >= items || k[u] >= K) continue;
            const float scale = scale_f32(byte[u]);
            float a[8], b[8], v[16];
            decode8(codes[u].x, scale, a);
            decode8(codes[u].y, scale, b);
#pragma unroll
            for (int j = 0; j < 8; j++) { v[j] = a[j]; v[8 + j] = b[j]; }
            T* p = out + (size_t)row[u] * ld + k[u];
            if (k[u] + 16 <= K) store_sectors<T, 16>(p, v);
            else {
#pragma unroll
                for (int j = 0; j < 16; j++) if (k[u] + j < K) p[j] = from_f32<T>(v[j]);
            }
        }
    }
}

// The same for rows on any boundary and for narrow ones: turned round in shared memory, stored element by element, coalesced.
template <typename T, int W>
__global__ void __launch_bounds__(kQThreads)
mx4_unpack_any_kernel(const uint8_t* __restrict__ data, const uint8_t* __restrict__ scales, const uint32_t* __restrict__ n_rows_dev,
                      uint32_t capacity, uint32_t K, T* __restrict__ out, size_t ld, sf_dev_state* st)
{
    __shared__ float4 turn[kQThreads / 32][4 * 32];
    sf_chain_enter();
    const uint32_t rows = n_rows_dev ? sf_clamp_rows(*n_rows_dev, capacity, st) : capacity;
    const uint32_t pitch = row_bytes(K), kt = k_tiles(K);
    const uint32_t lane = threadIdx.x & 31;
    float* const mine = reinterpret_cast<float*>(turn[threadIdx.x >> 5]);
    const uint64_t items = (uint64_t)rows * kt;
    const uint64_t step = (uint64_t)gridDim.x * (kQThreads / 32) * 4;
    for (uint64_t i0 = ((uint64_t)blockIdx.x * (kQThreads / 32) + (threadIdx.x >> 5)) * 4; i0 < items; i0 += step) {
        uint32_t r, c;
        row_and_piece(i0, kt, r, c);
        const uint32_t q = lane / 8, piece = c + q, row = r + piece / kt, k = (piece % kt) * 128 + (lane & 7) * 16;
        float a[8] = {}, b[8] = {};
        if (i0 + q < items && k < K) {
            const uint2 codes = __ldg(reinterpret_cast<const uint2*>(data + (size_t)row * pitch + k / 2));
            const float scale = scale_f32(__ldg(scales + scale_at(row, k / 32, kt)));
            decode8(codes.x, scale, a);
            decode8(codes.y, scale, b);
        }
        __syncwarp();
        *reinterpret_cast<float4*>(mine + turned(16 * lane)) = make_float4(a[0], a[1], a[2], a[3]);
        *reinterpret_cast<float4*>(mine + turned(16 * lane + 4)) = make_float4(a[4], a[5], a[6], a[7]);
        *reinterpret_cast<float4*>(mine + turned(16 * lane + 8)) = make_float4(b[0], b[1], b[2], b[3]);
        *reinterpret_cast<float4*>(mine + turned(16 * lane + 12)) = make_float4(b[4], b[5], b[6], b[7]);
        __syncwarp();
#pragma unroll
        for (int u = 0; u < 4; u++) {
            T* const p = out + (size_t)r * ld + c * 128;
            const uint32_t left = i0 + u < items ? K - c * 128 : 0u;
#pragma unroll
            for (int j = 0; j < 4 / W; j++) {
                const uint32_t k = (j * 32 + lane) * W;
                if (k < left) {
                    const float* const q = mine + turned(u * 128 + k);
                    float y[W];
#pragma unroll
                    for (int w = 0; w < W; w++) y[w] = q[w];
                    store_word<T, W>(p + k, y);
                }
            }
            if (++c == kt) { c = 0; r++; }
        }
    }
}

// may 16-bit elements be moved in pairs?
bool pairs_ok(const void* p, size_t ld, uint32_t K, size_t size) { return size == 2 && aligned(p, 4) && ld % 2 == 0 && K % 2 == 0; }
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
    // (rows up to 128 columns wide leave three quarters of the other kernel's lanes idle)
    const bool al = aligned(x, 16) && (ld * type_bytes(dtype)) % 16 == 0 && K > 128;
    const uint64_t items = al ? (uint64_t)capacity * ((k_tiles(K) * 128 + kPCols - 1) / kPCols) : ((uint64_t)capacity * k_tiles(K) + 3) / 4;
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        constexpr int U = 8 / sizeof(T);               // 8 16-byte words a lane on their way, where there are pieces enough for all warps
        const bool many = al && items >= (uint64_t)ctx->num_sms * 64 * U;
        auto k = al ? (many ? mx4_quantise_kernel<T, U> : mx4_quantise_kernel<T, 1>) : (pairs_ok(x, ld, K, sizeof(T)) ? mx4_quantise_any_kernel<T, sizeof(T) == 2 ? 2 : 1> : mx4_quantise_any_kernel<T, 1>);
        SF_CUDA(sf_launch_chained(k, row_grid(ctx, many ? (items + U - 1) / U : items, 32), kQThreads, 0, st, (const T*)x, n_src, K, ld, row_ids, n_rows_dev, capacity, data, scales, ctx->d_state));
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
    const bool al = aligned(out, 32) && (ld * type_bytes(dtype)) % 32 == 0 && K > 128;
    const uint32_t grid = al ? row_grid(ctx, ((uint64_t)capacity * ((K + kPCols - 1) / kPCols) + 1) / 2, 8) : row_grid(ctx, ((uint64_t)capacity * k_tiles(K) + 3) / 4, 32);
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        auto k = al ? mx4_unpack_kernel<T> : (pairs_ok(out, ld, K, sizeof(T)) ? mx4_unpack_any_kernel<T, sizeof(T) == 2 ? 2 : 1> : mx4_unpack_any_kernel<T, 1>);
        SF_CUDA(sf_launch_chained(k, grid, kQThreads, 0, (cudaStream_t)stream, data, scales, n_rows_dev, capacity, K, (T*)out, ld, ctx->d_state));
        return SF_OK;
    });
}
