// Product of packed 4-bit rows with packed 4-bit weights on the tensor cores: out[r][n] = act(sum_k A[r][k] W[n][k] + bias[n]),
// one weight matrix or one per expert over rows sorted by expert.
//
// tcgen05.mma kind::mxf4 multiplies 4-bit values with one power-of-two scale per 32 of them and sums in fp32: both
// operands go to shared memory as they are packed (TMA, 256 values = one 128-byte swizzled row per matrix row and stage), their
// scale bytes as 512-byte tiles that tcgen05.cp spreads over the TMEM lanes in front of the MMAs (64 values of K each).
// Persistent kernel, one CTA per SM.  Warp roles:
//   warp 0      producer: the A, W and scale tiles of a ring of stages, all by TMA (boxes beyond an array read zeros)
//   warp 1      allocates TMEM; one lane copies scales and issues MMAs
//   warps 2..9  epilogue: tcgen05.ld (lane quarter = warp % 4, column half = (warp - 2) / 4), bias, ReLU, rounding, 128-byte row
//               pieces through shared memory
// Every wait is bounded as in gemm_tc.cu: on a timeout the block records SF_ERR_DEVICE_TIMEOUT, lets its copies land, frees TMEM
// and returns.
//
// PAIR: two CTAs share every MMA (256 x 256 tiles, each CTA loads its 128 rows of A and of W; both need all 256 columns' scales).
// Two 256-column fp32 accumulators would fill the TMEM and leave no room for scales, so they overlap by 64 columns
// (0..255 and 192..447, scales from 448): the epilogue reads the shared columns first and the next tile's MMAs start then.
#include "rows_common.cuh"
#include "tc_common.cuh"
#include "mx4.cuh"
#include <algorithm>

namespace {
using namespace sfrow;
using namespace sfmx;
using namespace sftc;

constexpr uint32_t kEpiWarps = 8;
constexpr uint32_t kThreads = 64 + kEpiWarps * 32;
constexpr uint32_t kBK = 256;                        // values of K per stage: 128 bytes a row
constexpr uint32_t kSfCol = 448;                     // first TMEM column of the scales (two buffers)

template <uint32_t BN, bool PAIR> struct Cfg {
    static constexpr uint32_t kRows = PAIR ? 256 : 128;                   // rows of a tile
    static constexpr uint32_t kNT = (BN + 127) / 128;                     // scale row tiles of W per stage
    static constexpr uint32_t kA = 128 * 128, kB = (PAIR ? BN / 2 : BN) * 128, kSA = 1024, kSB = kNT * 1024;
    static constexpr uint32_t kStage = kA + kB + kSA + kSB;
    static constexpr uint32_t kStages = BN == 64 ? 6 : 5;
    static constexpr uint32_t kStaging = kEpiWarps * (4096 + 512);        // per epilogue warp: 32 rows x 128 bytes, 128 biases
    static constexpr uint32_t kOverlap = BN == 256 ? 64 : 0;              // columns that the two accumulators share
    static constexpr uint32_t kSecond = BN - kOverlap;                    // first column of the second accumulator
    static constexpr uint32_t kSfCols = 8 + 8 * kNT;
    static_assert(kSecond + BN <= kSfCol && kSfCol + 2 * kSfCols <= 512, "TMEM");
    static_assert(kStage % 1024 == 0, "swizzled tiles start on 1024-byte boundaries");
    static uint32_t smem(uint32_t E) { return 1024 + kStages * kStage + kStaging + 512 + (2 * E + 2) * 4; }
};

struct Bars {
    uint64_t full[8], empty[8], acc_full[2], acc_free[2];
    uint32_t tmem_base, abort_flag;
};

// 4-bit operands, fp32 accumulators, power-of-two scales per 32 values; sf = 0 or 2: which pair of a scale word's bytes
__host__ __device__ constexpr uint32_t make_idesc(uint32_t M, uint32_t N, uint32_t sf) {
    return (sf << 4) | (1u << 7) | (1u << 10) | ((N >> 3) << 17) | (1u << 23) | ((M >> 4) << 24) | (sf << 29);
}
template <bool PAIR>
__device__ __forceinline__ void mma4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    if constexpr (PAIR)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// a 512-byte scale tile (32 rows of 16 bytes) -> 4 TMEM columns, the same in all four lane quarters (of both CTAs of a pair)
template <bool PAIR> __device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t saddr) {
    const uint64_t desc = make_smem_desc(saddr, 16, 128, 0);
    if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

__device__ __forceinline__ float relu_keep_nan(float v) {
    float r;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(v));
    return r;
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    uint32_t h;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
    return h;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    uint32_t h;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
    return h;
}

// What a CTA (pair) works through: tiles of kRows x BN outputs, every n_units-th one, expert by expert, a row panel's column tiles
// one after the other.
struct Segments {
    const uint32_t* begin;           // [E] first row
    const uint32_t* tile;            // [E + 1] first tile
    uint32_t E, tiles_n;
    uint32_t e = 0;                  // cursor: tiles come in rising order
    __device__ __forceinline__ void find(uint32_t t, uint32_t rows_per_tile, uint32_t& row, uint32_t& tn) {
        while (e + 1 < E && t >= tile[e + 1]) e++;
        const uint32_t local = t - tile[e], tm = local / tiles_n;
        tn = local - tm * tiles_n;
        row = begin[e] + tm * rows_per_tile;
    }
};

template <uint32_t BN, bool PAIR, typename T>
__global__ void __launch_bounds__(kThreads, 1)
mx4_product_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmSA,
                   const __grid_constant__ CUtensorMap tmSW, const sf_mx4_product p, sf_dev_state* st)
{
    using C = Cfg<BN, PAIR>;
    extern __shared__ uint8_t smem_raw[];
    sf_chain_enter();
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const tiles = smem_raw + (base - smem_u32(smem_raw));
    uint8_t* const staging = tiles + C::kStages * C::kStage;
    Bars* const bars = reinterpret_cast<Bars*>(staging + C::kStaging);
    uint32_t* const seg_begin = reinterpret_cast<uint32_t*>(staging + C::kStaging + 512);
    uint32_t* const seg_tile = seg_begin + p.E;
    volatile uint32_t* const abort_flag = &bars->abort_flag;

    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tiles_n = (p.N + BN - 1) / BN;
    const uint32_t k_blocks = (p.K + kBK - 1) / kBK;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const uint32_t unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, n_units = PAIR ? gridDim.x >> 1 : gridDim.x;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < C::kStages; s++) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], 1); }
        for (uint32_t b = 0; b < 2; b++) { mbar_init(&bars->acc_full[b], 1); mbar_init(&bars->acc_free[b], (PAIR ? 2 : 1) * kEpiWarps); }
        bars->abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 0) {                                  // the experts' first tiles (one "expert" of all rows without offsets)
        uint32_t run = 0;
        for (uint32_t e0 = 0; e0 < p.E; e0 += 32) {
            const uint32_t e = e0 + lane;
            uint32_t lo = 0, hi = 0;
            if (e < p.E) {
                if (p.offsets) { lo = p.offsets[e]; hi = min(p.offsets[e + 1], p.capacity); }
                else hi = p.n_rows_dev ? sf_clamp_rows(*p.n_rows_dev, p.capacity, nullptr) : p.capacity;
                if (lo < hi && (lo & 127u)) { if (blockIdx.x == 0) sf_dev_set_error(st, SF_ERR_ARG); hi = lo; }      // not on a tile
            }
            const uint32_t mine = lo < hi ? (hi - lo + C::kRows - 1) / C::kRows * tiles_n : 0u;
            uint32_t sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, sum, o); if (lane >= (uint32_t)o) sum += u; }
            if (e < p.E) { seg_begin[e] = lo; seg_tile[e] = run + sum - mine; }
            run += __shfl_sync(0xFFFFFFFFu, sum, 31);
        }
        if (lane == 0) {
            seg_tile[p.E] = run;
            if (!p.offsets && p.n_rows_dev && blockIdx.x == 0 && *p.n_rows_dev > p.capacity) sf_dev_set_error(st, SF_ERR_CAPACITY);
        }
    }
    if (warp == 1) { if constexpr (PAIR) tmem_alloc_pair(&bars->tmem_base, 512); else tmem_alloc(&bars->tmem_base, 512); }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;
    const uint32_t n_tiles = seg_tile[p.E];
    Segments seg = {seg_begin, seg_tile, p.E, tiles_n};

    if (warp == 0) {
        if (lane == 0) {
            tma_prefetch_desc(&tmA); tma_prefetch_desc(&tmW); tma_prefetch_desc(&tmSA); tma_prefetch_desc(&tmSW);
            const uint32_t nt = (p.N + 127) / 128;   // scale row tiles of one expert's weights
            uint32_t stage = 0, phase = 0;
            bool ok = true;
            for (uint32_t t = unit; t < n_tiles && ok; t += n_units) {
                uint32_t row, tn;
                seg.find(t, C::kRows, row, tn);
                const int32_t ra = (int32_t)(row + rank * 128), rw = (int32_t)(seg.e * p.N + tn * BN + rank * (BN / 2));
                const int32_t sw = (int32_t)(seg.e * nt + tn * BN / 128);
                for (uint32_t kb = 0; kb < k_blocks; kb++) {
                    if (!mbar_wait(&bars->empty[stage], phase ^ 1u, abort_flag)) { ok = false; break; }
                    uint8_t* const s = tiles + stage * C::kStage;
                    if constexpr (PAIR) {
                        const uint32_t bar = map_to_cta(smem_u32(&bars->full[stage]), 0);
                        if (rank == 0) mbar_expect_tx(&bars->full[stage], 2 * C::kStage);
                        tma_load_2d_pair(s, &tmA, (int32_t)(kb * 128), ra, bar);
                        tma_load_2d_pair(s + C::kA, &tmW, (int32_t)(kb * 128), rw, bar);
                        tma_load_2d_pair(s + C::kA + C::kB, &tmSA, (int32_t)(kb * 256), ra / 128, bar);
                        tma_load_2d_pair(s + C::kA + C::kB + C::kSA, &tmSW, (int32_t)(kb * 256), sw, bar);
                    } else {
                        mbar_expect_tx(&bars->full[stage], C::kStage);
                        tma_load_2d(s, &tmA, (int32_t)(kb * 128), ra, &bars->full[stage]);
                        tma_load_2d(s + C::kA, &tmW, (int32_t)(kb * 128), rw, &bars->full[stage]);
                        tma_load_2d(s + C::kA + C::kB, &tmSA, (int32_t)(kb * 256), ra / 128, &bars->full[stage]);
                        tma_load_2d(s + C::kA + C::kB + C::kSA, &tmSW, (int32_t)(kb * 256), sw, &bars->full[stage]);
                    }
                    if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
                }
            }
            // every stage's last use released: no copy is in flight, no arrival on its way to this CTA's barriers
            for (uint32_t s = 0; s < C::kStages && ok; s++) {
                if (!mbar_wait(&bars->empty[stage], phase ^ 1u, abort_flag)) ok = false;
                if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            uint32_t stage = 0, phase = 0, i = 0, sbuf = 0;
            bool ok = true;
            for (uint32_t t = unit; t < n_tiles && ok; t += n_units, i++) {
                uint32_t row, tn;
                seg.find(t, C::kRows, row, tn);
                // overlapping accumulators: the shared columns of the tile before have been read; else: the tile before that
                constexpr uint32_t kBack = C::kOverlap ? 1 : 2;
                if (i >= kBack && !mbar_wait(&bars->acc_free[(i - kBack) & 1u], ((i - kBack) >> 1) & 1u, abort_flag)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d = tmem + (i & 1u) * C::kSecond;
                const uint32_t half = BN == 64 ? (tn & 1u) * 2u : 0u;      // 64 columns: half of a scale tile
                for (uint32_t kb = 0; kb < k_blocks; kb++) {
                    if (!mbar_wait(&bars->full[stage], phase, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a = base + stage * C::kStage, b = a + C::kA, sa = b + C::kB, sb = sa + C::kSA;
                    const uint32_t sf = tmem + kSfCol + sbuf * C::kSfCols;
#pragma unroll
                    for (uint32_t j = 0; j < 2; j++) {
                        copy_scales<PAIR>(sf + j * 4, sa + j * 512);
#pragma unroll
                        for (uint32_t r = 0; r < C::kNT; r++) copy_scales<PAIR>(sf + 8 + (j * C::kNT + r) * 4, sb + r * 1024 + j * 512);
                    }
                    const uint32_t steps = min(4u, (p.K - kb * kBK + 63) / 64);
                    for (uint32_t k = 0; k < steps; k++) {
                        const uint64_t ad = make_smem_desc(a + k * 32, 16, 1024, 2), bd = make_smem_desc(b + k * 32, 16, 1024, 2);
                        mma4<PAIR>(d, ad, bd, make_idesc(C::kRows, BN, 0) + (k & 1u) * ((2u << 4) + (2u << 29)), sf + (k / 2) * 4,
                                   sf + 8 + (k / 2) * 4 * C::kNT + half, (kb | k) != 0 ? 1u : 0u);
                    }
                    if constexpr (PAIR) umma_commit_pair(&bars->empty[stage]); else umma_commit(&bars->empty[stage]);
                    sbuf ^= 1u;
                    if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                if constexpr (PAIR) umma_commit_pair(&bars->acc_full[i & 1u]); else umma_commit(&bars->acc_full[i & 1u]);
            }
        }
    } else {
        constexpr uint32_t kHalf = BN / 2;                                   // columns of this warp
        constexpr uint32_t kCols = sizeof(T) == 4 ? 32 : (kHalf < 64 ? kHalf : 64);      // columns taken at once: 128 bytes of a row (64 for a narrow tile)
        constexpr uint32_t kPieces = kCols * sizeof(T) / 16;                 // 16-byte pieces of a staged row
        const uint32_t quarter = warp & 3u, half = (warp - 2u) >> 2;
        uint8_t* const stg = staging + (warp - 2u) * 4608u;
        float* const bias_s = reinterpret_cast<float*>(stg + 4096);
        const bool vec = (p.ld * sizeof(T)) % 16 == 0 && ((uintptr_t)p.out & 15) == 0;
        uint32_t i = 0;
        bool ok = true;
        for (uint32_t t = unit; t < n_tiles && ok; t += n_units, i++) {
            uint32_t row, tn;
            seg.find(t, C::kRows, row, tn);
            const uint32_t end = p.offsets ? min(p.offsets[seg.e + 1], p.capacity) : (p.n_rows_dev ? min(*p.n_rows_dev, p.capacity) : p.capacity);
            const uint32_t row0 = row + rank * 128 + quarter * 32, col0 = tn * BN + half * kHalf;
            const float* const bias = p.bias ? p.bias + (size_t)seg.e * p.N : nullptr;
            for (uint32_t c = lane; c < kHalf; c += 32) bias_s[c] = bias && col0 + c < p.N ? __ldg(bias + col0 + c) : 0.0f;
            __syncwarp();
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_full[i & 1u], (i >> 1) & 1u, abort_flag));
            if (!ok) break;
            tc_fence_after();
            const uint32_t taddr = tmem + ((quarter * 32u) << 16) + (i & 1u) * C::kSecond + half * kHalf;
            auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) mbar_arrive_cluster(map_to_cta(smem_u32(&bars->acc_free[i & 1u]), 0));
                    else mbar_arrive(&bars->acc_free[i & 1u]);
                }
            };
            // the columns shared with the next tile's accumulator: the first one's last 64, the second one's first 64
            const bool shares = C::kOverlap && half != (i & 1u);
            if (C::kOverlap && !shares) release();
#pragma unroll 1
            for (uint32_t n = 0; n < kHalf / kCols; n++) {
                // the first accumulator's upper half begins with its last columns
                const uint32_t c = (shares && (i & 1u) == 0 ? (kHalf / kCols - 1 - n) : n) * kCols;
                uint32_t v[kCols];
#pragma unroll
                for (uint32_t g = 0; g < kCols; g += 32) tmem_ld32(taddr + c + g, *reinterpret_cast<uint32_t(*)[32]>(v + g));
                tmem_ld_wait();
                if (shares && (n + 1) * kCols == C::kOverlap) release();
#pragma unroll
                for (uint32_t g = 0; g < kCols; g += 4) {
                    const float4 b = *reinterpret_cast<const float4*>(bias_s + c + g);
                    float x[4] = {__uint_as_float(v[g]) + b.x, __uint_as_float(v[g + 1]) + b.y, __uint_as_float(v[g + 2]) + b.z, __uint_as_float(v[g + 3]) + b.w};
                    if (p.relu) {
#pragma unroll
                        for (int q = 0; q < 4; q++) x[q] = relu_keep_nan(x[q]);
                    }
                    if constexpr (sizeof(T) == 4) {
#pragma unroll
                        for (int q = 0; q < 4; q++) v[g + q] = __float_as_uint(x[q]);
                    } else {
                        v[g / 2] = pack2<T>(x[0], x[1]);
                        v[g / 2 + 1] = pack2<T>(x[2], x[3]);
                    }
                }
#pragma unroll
                for (uint32_t q = 0; q < kPieces; q++)
                    *reinterpret_cast<uint4*>(stg + lane * 128u + ((q ^ (lane & 7u)) << 4)) = make_uint4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                __syncwarp();
                constexpr uint32_t kRowsAt = 32 / kPieces;                   // rows per store instruction
                const uint32_t q = lane % kPieces;
#pragma unroll
                for (uint32_t r0 = 0; r0 < 32; r0 += kRowsAt) {
                    const uint32_t r = r0 + lane / kPieces;
                    const uint4 val = *reinterpret_cast<const uint4*>(stg + r * 128u + ((q ^ (r & 7u)) << 4));
                    const uint32_t col = col0 + c + q * (16 / sizeof(T));
                    if (row0 + r < end && col < p.N) {
                        T* const o = reinterpret_cast<T*>(p.out) + (size_t)(row0 + r) * p.ld + col;
                        if (vec && col + 16 / sizeof(T) <= p.N) *reinterpret_cast<uint4*>(o) = val;
                        else {
                            const T* const e = reinterpret_cast<const T*>(&val);
#pragma unroll
                            for (uint32_t x = 0; x < 16 / sizeof(T); x++) if (col + x < p.N) o[x] = e[x];
                        }
                    }
                }
                __syncwarp();
            }
            if (!C::kOverlap) release();
        }
    }

    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) sf_dev_set_error(st, SF_ERR_DEVICE_TIMEOUT);
        __nanosleep(200000);
        __syncthreads();
    }
    if constexpr (PAIR) cluster_sync_all();          // the partner is done with this CTA's shared memory and barriers
    tc_fence_after();
    if (warp == 1) {
        __syncwarp();
        if constexpr (PAIR) tmem_dealloc_pair(tmem, 512); else tmem_dealloc(tmem, 512);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------
template <uint32_t BN, bool PAIR, typename T>
int launch(sf_ctx* ctx, const sf_mx4_product& p, cudaStream_t st)
{
    using C = Cfg<BN, PAIR>;
    const uint32_t pitch = row_bytes(p.K), kt = k_tiles(p.K);
    CUtensorMap tmA, tmW, tmSA, tmSW;
    int rc = encode_tmap_2d(&tmA, CU_TENSOR_MAP_DATA_TYPE_UINT8, p.a, p.capacity, pitch, pitch, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc == SF_OK) rc = encode_tmap_2d(&tmW, CU_TENSOR_MAP_DATA_TYPE_UINT8, p.w, (uint64_t)p.E * p.N, pitch, pitch, PAIR ? BN / 2 : BN, 128, CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc == SF_OK) rc = encode_tmap_2d(&tmSA, CU_TENSOR_MAP_DATA_TYPE_UINT32, p.a_scales, (p.capacity + 127) / 128, kt * 128, kt * 512, 1, 256, CU_TENSOR_MAP_SWIZZLE_NONE);
    if (rc == SF_OK) rc = encode_tmap_2d(&tmSW, CU_TENSOR_MAP_DATA_TYPE_UINT32, p.w_scales, (uint64_t)p.E * ((p.N + 127) / 128), kt * 128, kt * 512, C::kNT, 256, CU_TENSOR_MAP_SWIZZLE_NONE);
    if (rc != SF_OK) return rc;
    auto kern = mx4_product_kernel<BN, PAIR, T>;
    static bool set_dev[64] = {};                      // the opt-in is per device
    bool& set = set_dev[ctx->device & 63];
    if (!set) { SF_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::smem(SF_MAX_EXPERTS))); set = true; }
    // the most tiles there can be: every expert's last tile may be a part of one
    const uint64_t most = ((uint64_t)p.capacity / C::kRows + p.E) * ((p.N + BN - 1) / BN);
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((PAIR ? 2u : 1u) * (uint32_t)std::min<uint64_t>((uint64_t)ctx->num_sms / (PAIR ? 2 : 1), most));
    lc.blockDim = dim3(kThreads); lc.dynamicSmemBytes = C::smem(p.E); lc.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    lc.attrs = at; lc.numAttrs = PAIR ? 2 : 1;
    SF_CUDA(cudaLaunchKernelEx(&lc, kern, tmA, tmW, tmSA, tmSW, p, ctx->d_state));
    return SF_OK;
}

// can the device run two-CTA clusters of the kernel? (asked once per type and device; else the single-CTA kernel serves)
template <typename T> bool pairs_supported(const sf_ctx* ctx) {
    using C = Cfg<256, true>;
    static int cache[64] = {};                         // 0 unknown, 1 yes, -1 no
    int& c = cache[ctx->device & 63];
    if (c == 0) {
        auto kern = mx4_product_kernel<256, true, T>;
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3(2); lc.blockDim = dim3(kThreads); lc.dynamicSmemBytes = C::smem(SF_MAX_EXPERTS);
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
        lc.attrs = at; lc.numAttrs = 1;
        int n = 0;
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::smem(SF_MAX_EXPERTS));
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&n, kern, &lc);
        if (e != cudaSuccess) (void)cudaGetLastError();
        c = e == cudaSuccess && n > 0 ? 1 : -1;
    }
    return c > 0;
}

int check(const sf_ctx* ctx, const sf_mx4_product& p)
{
    if (!ctx || !type_ok(p.out_dtype) || p.N == 0 || p.K == 0 || p.K > SF_MX4_MAX_K || p.N > SF_MX4_MAX_K || p.ld < p.N) return SF_ERR_ARG;
    if (p.capacity > 0x7FFFFF00u || (uint64_t)p.E * p.N > 0x7FFFFFFFull) return SF_ERR_ARG;      // tile coordinates are 32-bit signed
    if (p.capacity == 0) return SF_OK;
    if (!p.a || !p.a_scales || !p.w || !p.w_scales || !p.out) return SF_ERR_ARG;
    if (!aligned(p.a, 16) || !aligned(p.a_scales, 16) || !aligned(p.w, 16) || !aligned(p.w_scales, 16)) return SF_ERR_ARG;
    if (!aligned(p.out, type_bytes(p.out_dtype)) || !aligned(p.bias, 4) || !aligned(p.n_rows_dev, 4) || !aligned(p.offsets, 4)) return SF_ERR_ARG;
    return SF_OK;
}

}  // namespace

int sf_launch_mx4_product(sf_ctx* ctx, const sf_mx4_product& p, cudaStream_t st)
{
    // rows and tiles as far as the host knows them (the counts live on the device)
    const uint64_t rows = std::max<uint64_t>(1, p.capacity / p.E);
    const bool pairs = p.N > 128 && rows >= 256 && (rows + 255) / 256 * p.E * ((p.N + 255) / 256) >= (uint64_t)ctx->num_sms / 2;
    const bool narrow = (rows + 127) / 128 * p.E * ((p.N + 127) / 128) < (uint64_t)ctx->num_sms;
    return by_type(p.out_dtype, [&](auto zero) {
        typedef decltype(zero) T;
        if (pairs && pairs_supported<T>(ctx)) return launch<256, true, T>(ctx, p, st);
        return narrow ? launch<64, false, T>(ctx, p, st) : launch<128, false, T>(ctx, p, st);
    });
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
