// Product of packed 4-bit rows with packed 4-bit weights on the tensor cores: out[r][n] = act(sum_k A[r][k] W[n][k] + bias[n]),
// one weight matrix or one per expert over rows sorted by expert.
//
// tcgen05.mma kind::mxf4 multiplies 4-bit values with one power-of-two scale per 32 of them and sums in fp32: both
// operands go to shared memory as they are packed (TMA, 256 values = one 128-byte swizzled row per matrix row and stage), their
// scale bytes as 512-byte tiles that tcgen05.cp spreads over the TMEM lanes in front of the MMAs (64 values of K each).
// Persistent kernel, one CTA per SM, each with a run of consecutive tiles (a row panel's column tiles one after the other).  While
// K <= 1280 a panel's slices of A stay in shared memory (a ring of five) for all its column tiles and only W is streamed: 2 % at
// 120,000 x 1024 x 1024 (a longer ring, with fewer stages of W or without the 128-byte staging below, gains nothing: 240,001 x
// 2048 x 1024 in 0.215 ms with eight slots and 64-byte stores, 0.217 ms this way).  Warp roles:
//   warp 0      producer: slices of A and W with their scales, all by TMA (boxes beyond an array read zeros)
//   warp 1      allocates TMEM; copies scales and issues MMAs.  The whole warp walks the loop and one elected lane issues: descriptors
//               and addresses then stay in uniform registers.  With a loop of one lane every copy and MMA first moves its operands
//               there (about 57 cycles each), and the six copies and four MMAs of a stage took 870 cycles to issue instead of
//               the 512 that the MMAs run
//   warps 2..9  epilogue: tcgen05.ld (lane quarter = warp % 4, column half = (warp - 2) / 4), bias, ReLU, rounding, then 32 rows x 128
//               bytes through shared memory and out by TMA (plain 64-byte row pieces: 76 instead of 67 us at 120,000 x 1024 x
//               1024), or by plain stores where rows are not on 16-byte boundaries or a tile ends inside
// Every wait is bounded as in gemm_tc.cu: on a timeout the block records SF_ERR_DEVICE_TIMEOUT, lets its copies land, frees TMEM
// and returns.
//
// Head<CH> (pairs only): a pair has whole panels, and a lane multiplies its row's bf16 outputs with the head's weights (shared memory,
// the same address in all lanes) and keeps the logits: the activations are neither written nor read again.  The four column groups
// of a row are summed apart and added in a fixed order.
//
// PAIR: two CTAs share every MMA (256 x 256 tiles, each CTA loads its 128 rows of A and of W; both need all 256 columns' scales).
// Two 256-column fp32 accumulators would fill the TMEM and leave no room for scales, so they overlap by 64 columns
// (0..255 and 192..447, scales from 448): the epilogue reads the shared columns first and the next tile's MMAs start then.
#include "rows_common.cuh"
#include "tc_common.cuh"
#include "mx4.cuh"
#include <algorithm>
#include <type_traits>

namespace {
using namespace sfrow;
using namespace sfmx;
using namespace sftc;

constexpr uint32_t kEpiWarps = 8;
constexpr uint32_t kThreads = 64 + kEpiWarps * 32;
constexpr uint32_t kBK = 256;                        // values of K per stage: 128 bytes a row
constexpr uint32_t kSfCol = 448;                     // first TMEM column of the scales (two buffers)

struct Bars {
    uint64_t a_full[5], a_empty[5], w_full[5], w_empty[5], acc_full[2], acc_free[2];
    uint32_t tmem_base, abort_flag;
};
struct Mx4 {};                                       // output type: packed again
// output type: the logits of a head of up to CH classes over the bf16 outputs, which are not written
template <uint32_t CH> struct Head {};
template <typename T> struct HeadOf { static constexpr uint32_t kCh = 0; };
template <uint32_t CH> struct HeadOf<Head<CH>> { static constexpr uint32_t kCh = CH; };
constexpr uint32_t kHeadMaxN = 1024;                 // widest hidden layer whose head weights fit where outputs are staged
template <typename T> constexpr uint32_t head_bytes() { return 128 * HeadOf<T>::kCh * 4; }      // one half's partial logits

template <uint32_t BN, bool PAIR> struct Cfg {
    static constexpr uint32_t kRows = PAIR ? 256 : 128;                   // rows of a tile
    static constexpr uint32_t kNT = (BN + 127) / 128;                     // scale row tiles of W per stage
    static constexpr uint32_t kA = 128 * 128, kSlot = kA + 1024;          // a slice of A: 128 rows x 256 values and their scales
    static constexpr uint32_t kB = (PAIR ? BN / 2 : BN) * 128, kStage = kB + kNT * 1024;      // a slice of W
    static constexpr uint32_t kSlots = 5, kStages = 5;
    static constexpr uint32_t kStaging = kEpiWarps * 4096 + BN * 4;       // per epilogue warp: 32 rows x 128 bytes; a tile's biases
    static constexpr uint32_t kOverlap = BN == 256 ? 64 : 0;              // columns that the two accumulators share
    static constexpr uint32_t kSecond = BN - kOverlap;                    // first column of the second accumulator
    static constexpr uint32_t kSfCols = 8 + 8 * kNT;
    static_assert(kSecond + BN <= kSfCol && kSfCol + 2 * kSfCols <= 512, "TMEM");
    static_assert(kSlot % 1024 == 0 && kStage % 1024 == 0, "swizzled tiles start on 1024-byte boundaries");
    template <typename T = float> static constexpr uint32_t smem(uint32_t E) { return 1024 + kSlots * kSlot + kStages * kStage + kStaging + sizeof(Bars) + (2 * E + 2) * 4 + (head_bytes<T>() ? 16 + head_bytes<T>() : 0); }
};

static_assert(Cfg<256, true>::smem<Head<8>>(SF_MAX_EXPERTS) <= 232448 && kHeadMaxN * 32 <= kEpiWarps * 4096 && Cfg<128, false>::smem(SF_MAX_EXPERTS) <= 232448 &&
              Cfg<64, false>::smem(SF_MAX_EXPERTS) <= 232448, "shared memory of a block");

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

// one lane of a converged warp
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
    return p != 0;
}

// Arrival on a barrier of the leader CTA that releases TMEM only: the tcgen05 fence orders that.  A releasing arrival at cluster scope
// would first wait for the thread's stores of the tile before.
__device__ __forceinline__ void mbar_arrive_relaxed(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// `threads` threads meet at named barrier `id`: true in all of them if it is in each
__device__ __forceinline__ bool all_agree(uint32_t id, uint32_t threads, bool mine) {
    uint32_t r;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %3, 0;\nbar.red.and.pred q, %1, %2, p;\nselp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"(id), "r"(threads), "r"((uint32_t)mine) : "memory");
    return r != 0;
}

__device__ __forceinline__ float relu_keep_nan(float v) {
    float r;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(v));
    return r;
}
// two outputs in one word, the first in the low half; the conversion itself clamps at zero and keeps a NaN
template <typename T, bool RELU> __device__ __forceinline__ uint32_t pack2(float a, float b) {
    uint32_t h;
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        if constexpr (RELU) asm("cvt.rn.relu.bf16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
        else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
    } else {
        if constexpr (RELU) asm("cvt.rn.relu.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
        else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
    }
    return h;
}
// (a0, a1) + (b0, b1): two fp32 additions in one instruction
__device__ __forceinline__ void add_pair(float& x0, float& x1, uint32_t a0, uint32_t a1, float b0, float b1) {
    uint64_t a, b;
    asm("mov.b64 %0, {%1, %2};" : "=l"(a) : "r"(a0), "r"(a1));
    asm("mov.b64 %0, {%1, %2};" : "=l"(b) : "f"(b0), "f"(b1));
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(a) : "l"(b));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x0), "=f"(x1) : "l"(a));
}
// accumulators + biases, ReLU, rounding: v[0..COLS) -> the row's words (fp32 values for T = float and for rows packed again)
template <typename T, uint32_t COLS, bool RELU> __device__ __forceinline__ void finish(uint32_t (&v)[COLS], const float* bias_s) {
#pragma unroll
    for (uint32_t g = 0; g < COLS; g += 4) {
        const float4 b = *reinterpret_cast<const float4*>(bias_s + g);
        float x[4];
        add_pair(x[0], x[1], v[g], v[g + 1], b.x, b.y);
        add_pair(x[2], x[3], v[g + 2], v[g + 3], b.z, b.w);
        if constexpr (sizeof(T) == 2) {
            v[g / 2] = pack2<T, RELU>(x[0], x[1]);
            v[g / 2 + 1] = pack2<T, RELU>(x[2], x[3]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; q++) v[g + q] = __float_as_uint(RELU ? relu_keep_nan(x[q]) : x[q]);
        }
    }
}

// logits += bf16 outputs (two a word, column col and the next first) x the head's weights
template <uint32_t CH, uint32_t WORDS, uint32_t COLS> __device__ __forceinline__ void add_head(float (&lg)[CH], const uint32_t (&v)[COLS], const uint8_t* weights, uint32_t col) {
#pragma unroll
    for (uint32_t q = 0; q < WORDS; q++) {
        const float a[2] = {__uint_as_float(v[q] << 16), __uint_as_float(v[q] & 0xFFFF0000u)};
#pragma unroll
        for (uint32_t h = 0; h < 2; h++) {
            const float* const w = reinterpret_cast<const float*>(weights) + (size_t)(col + 2 * q + h) * CH;
            float x[CH];
            if constexpr (CH == 2) { const float2 y = *reinterpret_cast<const float2*>(w); x[0] = y.x; x[1] = y.y; }
            else {
#pragma unroll
                for (uint32_t c = 0; c < CH; c += 4) {
                    const float4 y = *reinterpret_cast<const float4*>(w + c);
                    x[c] = y.x; x[c + 1] = y.y; x[c + 2] = y.z; x[c + 3] = y.w;
                }
            }
#pragma unroll
            for (uint32_t c = 0; c < CH; c += 2) {
                uint64_t d, aa, ww;                  // two fused multiply-adds in one instruction
                asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lg[c]), "f"(lg[c + 1]));
                asm("mov.b64 %0, {%1, %1};" : "=l"(aa) : "f"(a[h]));
                asm("mov.b64 %0, {%1, %2};" : "=l"(ww) : "f"(x[c]), "f"(x[c + 1]));
                asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(d) : "l"(aa), "l"(ww));
                asm("mov.b64 {%0, %1}, %2;" : "=f"(lg[c]), "=f"(lg[c + 1]) : "l"(d));
            }
        }
    }
}

// 32-column blocks of a row's fp32 values -> words of codes and scale bytes.  With ReLU a negative value orders below 0 as a signed
// integer and the conversion clamps it; a NaN that an addition made is positive and orders above infinity.
template <uint32_t COLS, bool RELU> __device__ __forceinline__ void pack_blocks(const uint32_t (&v)[COLS], uint32_t (&w)[COLS / 8], uint32_t& bytes) {
#pragma unroll
    for (uint32_t g = 0; g < COLS; g += 32) {
        int top = 0;
#pragma unroll
        for (uint32_t q = 0; q < 32; q += 2) {
            if (RELU) top = __vimax3_s32(top, (int)v[g + q], (int)v[g + q + 1]);
            else top = __vimax3_s32(top, (int)(v[g + q] & 0x7FFFFFFFu), (int)(v[g + q + 1] & 0x7FFFFFFFu));
        }
        const uint32_t byte = scale_byte((uint32_t)top);
        bytes |= byte << (g / 4);
#pragma unroll
        for (uint32_t q = 0; q < 4; q++) {
            float x[8];
#pragma unroll
            for (uint32_t r = 0; r < 8; r++) x[r] = __uint_as_float(v[g + q * 8 + r]);
            w[g / 8 + q] = encode8<RELU>(x, byte);
        }
    }
}

// A value that is the same in all lanes, told to the compiler as such: loop bounds and addresses that come out of shared memory
// would otherwise keep the issuing warps' operands out of the uniform registers.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }

// What a CTA (pair) works through: tiles of kRows x BN outputs, expert by expert, panel by panel; unit u of U takes tiles
// [n u / U, n (u + 1) / U).
struct Segments {
    const uint32_t* begin;           // [E] first row
    const uint32_t* tile;            // [E + 1] first tile
    uint32_t E, tiles_n;
    uint32_t e = 0;                  // cursor: tiles come in rising order
    __device__ __forceinline__ void find(uint32_t t, uint32_t rows_per_tile, uint32_t& row, uint32_t& tn) {
        while (e + 1 < E && t >= tile[e + 1]) e++;
        e = uniform(e);
        const uint32_t local = uniform(t - tile[e]), tm = local / tiles_n;
        tn = local - tm * tiles_n;
        row = uniform(begin[e]) + tm * rows_per_tile;
    }
};

template <uint32_t BN, bool PAIR, typename T>
__global__ void __launch_bounds__(kThreads, 1)
mx4_product_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmSA,
                   const __grid_constant__ CUtensorMap tmSW, const __grid_constant__ CUtensorMap tmO,
                   const uint32_t tma_out, const sf_mx4_product p, sf_dev_state* st)
{
    using C = Cfg<BN, PAIR>;
    extern __shared__ uint8_t smem_raw[];
    sf_chain_enter();
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const tiles = smem_raw + (base - smem_u32(smem_raw));
    uint8_t* const w_ring = tiles + C::kSlots * C::kSlot;
    uint8_t* const staging = w_ring + C::kStages * C::kStage;
    Bars* const bars = reinterpret_cast<Bars*>(staging + C::kStaging);
    uint32_t* const seg_begin = reinterpret_cast<uint32_t*>(bars + 1);
    uint32_t* const seg_tile = seg_begin + p.E;
    volatile uint32_t* const abort_flag = &bars->abort_flag;

    const uint32_t warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    constexpr bool kPacked = std::is_same<T, Mx4>::value;
    constexpr uint32_t kCh = HeadOf<T>::kCh;
    static_assert(kCh == 0 || PAIR, "the head is folded into pairs only");
    const uint32_t tiles_n = ((kPacked ? k_tiles(p.N) * 128 : p.N) + BN - 1) / BN;      // packed rows: up to the last scale tile's end
    const uint32_t k_blocks = (p.K + kBK - 1) / kBK;
    const bool keep = k_blocks <= C::kSlots;          // a panel of A fits in the ring
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const uint32_t unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, n_units = PAIR ? gridDim.x >> 1 : gridDim.x;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < C::kStages; s++) { mbar_init(&bars->w_full[s], 1); mbar_init(&bars->w_empty[s], 1); }
        for (uint32_t s = 0; s < C::kSlots; s++) { mbar_init(&bars->a_full[s], 1); mbar_init(&bars->a_empty[s], 1); }
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
    float* const partial = reinterpret_cast<float*>(((uintptr_t)(seg_tile + p.E + 1) + 15) & ~(uintptr_t)15);      // [128][kCh]
    if constexpr (kCh != 0) {                         // head weights: fp32 [column][kCh]
        const __nv_bfloat16* const hw = reinterpret_cast<const __nv_bfloat16*>(p.head_w);
        for (uint32_t i = threadIdx.x; i < p.N * kCh; i += kThreads) {
            reinterpret_cast<float*>(staging)[i] = __bfloat162float(hw[(size_t)(i % kCh) * p.N + i / kCh]);
        }
    }
    if (warp == 1) { if constexpr (PAIR) tmem_alloc_pair(&bars->tmem_base, 512); else tmem_alloc(&bars->tmem_base, 512); }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = uniform(bars->tmem_base);
    const uint32_t n_tiles = uniform(seg_tile[p.E]);
    const uint32_t grain = kCh ? tiles_n : 1u;        // (whole panels with a head)
    const uint32_t t_begin = (uint32_t)((uint64_t)(n_tiles / grain) * unit / n_units) * grain, t_end = (uint32_t)((uint64_t)(n_tiles / grain) * (unit + 1) / n_units) * grain;
    Segments seg = {seg_begin, seg_tile, p.E, tiles_n};

    if (warp == 0) {
        if (elect_one()) { tma_prefetch_desc(&tmA); tma_prefetch_desc(&tmW); tma_prefetch_desc(&tmSA); tma_prefetch_desc(&tmSW); }
        const uint32_t nt = (p.N + 127) / 128;       // scale row tiles of one expert's weights
        uint32_t stage = 0, phase = 0, slot = 0, sphase = 0;
        bool ok = true;
        for (uint32_t t = t_begin; t < t_end && ok; t++) {
            uint32_t row, tn;
            seg.find(t, C::kRows, row, tn);
            const bool fresh = !keep || tn == 0 || t == t_begin;           // A's slices have to be loaded
            const int32_t ra = (int32_t)(row + rank * 128), rw = (int32_t)(seg.e * p.N + tn * BN + rank * (BN / 2));
            const int32_t sw = (int32_t)(seg.e * nt + tn * BN / 128);
            for (uint32_t kb = 0; kb < k_blocks; kb++) {
                if (fresh) {
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->a_empty[slot], sphase ^ 1u, abort_flag));
                    if (!ok) break;
                    if (elect_one()) {
                        uint8_t* const s = tiles + slot * C::kSlot;
                        if constexpr (PAIR) {
                            const uint32_t bar = map_to_cta(smem_u32(&bars->a_full[slot]), 0);
                            if (rank == 0) mbar_expect_tx(&bars->a_full[slot], 2 * C::kSlot);
                            tma_load_2d_pair(s, &tmA, (int32_t)(kb * 128), ra, bar);
                            tma_load_2d_pair(s + C::kA, &tmSA, (int32_t)(kb * 256), ra / 128, bar);
                        } else {
                            mbar_expect_tx(&bars->a_full[slot], C::kSlot);
                            tma_load_2d(s, &tmA, (int32_t)(kb * 128), ra, &bars->a_full[slot]);
                            tma_load_2d(s + C::kA, &tmSA, (int32_t)(kb * 256), ra / 128, &bars->a_full[slot]);
                        }
                    }
                    __syncwarp();
                    if (++slot == C::kSlots) { slot = 0; sphase ^= 1u; }
                }
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->w_empty[stage], phase ^ 1u, abort_flag));
                if (!ok) break;
                if (elect_one()) {
                    uint8_t* const s = w_ring + stage * C::kStage;
                    if constexpr (PAIR) {
                        const uint32_t bar = map_to_cta(smem_u32(&bars->w_full[stage]), 0);
                        if (rank == 0) mbar_expect_tx(&bars->w_full[stage], 2 * C::kStage);
                        tma_load_2d_pair(s, &tmW, (int32_t)(kb * 128), rw, bar);
                        tma_load_2d_pair(s + C::kB, &tmSW, (int32_t)(kb * 256), sw, bar);
                    } else {
                        mbar_expect_tx(&bars->w_full[stage], C::kStage);
                        tma_load_2d(s, &tmW, (int32_t)(kb * 128), rw, &bars->w_full[stage]);
                        tma_load_2d(s + C::kB, &tmSW, (int32_t)(kb * 256), sw, &bars->w_full[stage]);
                    }
                }
                __syncwarp();
                if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
            }
        }
        // every stage's and slot's last use released: no copy is in flight, no arrival on its way to this CTA's barriers
        for (uint32_t s = 0; s < C::kStages && ok; s++) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->w_empty[stage], phase ^ 1u, abort_flag));
            if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
        }
        for (uint32_t s = 0; s < C::kSlots && ok; s++) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->a_empty[slot], sphase ^ 1u, abort_flag));
            if (++slot == C::kSlots) { slot = 0; sphase ^= 1u; }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            uint32_t stage = 0, phase = 0, i = 0, sbuf = 0;
            uint32_t panel = 0, pphase = 0;           // first slot of the current panel and its phase
            bool ok = true;
            for (uint32_t t = t_begin; t < t_end && ok; t++, i++) {
                uint32_t row, tn;
                seg.find(t, C::kRows, row, tn);
                const bool fresh = !keep || tn == 0 || t == t_begin;
                const bool last = !keep || tn + 1 == tiles_n || t + 1 == t_end;       // the panel's last tile here
                // overlapping accumulators: the shared columns of the tile before have been read; else: the tile before that
                // (waited for with the first slices and their scales already on their way)
                constexpr uint32_t kBack = C::kOverlap ? 1 : 2;
                const uint32_t d = tmem + (i & 1u) * C::kSecond;
                const uint32_t half = BN == 64 ? (tn & 1u) * 2u : 0u;      // 64 columns: half of a scale tile
                uint32_t slot = panel, sphase = pphase;
                for (uint32_t kb = 0; kb < k_blocks; kb++) {
                    if (fresh) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->a_full[slot], sphase, abort_flag));
                    if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->w_full[stage], phase, abort_flag));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t a = base + slot * C::kSlot, sa = a + C::kA;
                    const uint32_t b = base + C::kSlots * C::kSlot + stage * C::kStage, sb = b + C::kB;
                    const uint32_t sf = tmem + kSfCol + sbuf * C::kSfCols;
                    const uint32_t left = p.K - kb * kBK;                  // values of K from here on
                    const bool issue = elect_one();
                    if (issue) {
#pragma unroll
                        for (uint32_t j = 0; j < 2; j++) {
                            copy_scales<PAIR>(sf + j * 4, sa + j * 512);
#pragma unroll
                            for (uint32_t r = 0; r < C::kNT; r++) copy_scales<PAIR>(sf + 8 + (j * C::kNT + r) * 4, sb + r * 1024 + j * 512);
                        }
                    }
                    if (kb == 0 && i >= kBack) {
                        ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_free[(i - kBack) & 1u], ((i - kBack) >> 1) & 1u, abort_flag));
                        if (!ok) break;
                        tc_fence_after();
                    }
                    if (issue) {
#pragma unroll
                        for (uint32_t k = 0; k < 4; k++) {
                            if (k == 0 || k * 64 < left)
                                mma4<PAIR>(d, make_smem_desc(a + k * 32, 16, 1024, 2), make_smem_desc(b + k * 32, 16, 1024, 2), make_idesc(C::kRows, BN, (k & 1u) * 2u),
                                           sf + (k / 2) * 4, sf + 8 + (k / 2) * 4 * C::kNT + half, (kb | k) != 0 ? 1u : 0u);
                        }
                        if constexpr (PAIR) umma_commit_pair(&bars->w_empty[stage]); else umma_commit(&bars->w_empty[stage]);
                        if (last) { if constexpr (PAIR) umma_commit_pair(&bars->a_empty[slot]); else umma_commit(&bars->a_empty[slot]); }
                        if (kb + 1 == k_blocks) { if constexpr (PAIR) umma_commit_pair(&bars->acc_full[i & 1u]); else umma_commit(&bars->acc_full[i & 1u]); }
                    }
                    __syncwarp();
                    sbuf ^= 1u;
                    if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
                    if (++slot == C::kSlots) { slot = 0; sphase ^= 1u; }
                }
                if (last) { panel = slot; pphase = sphase; }
            }
        }
    } else {
        constexpr uint32_t kHalf = BN / 2;                                   // columns of this warp
        constexpr uint32_t kCols = kHalf < 64 ? kHalf : 64;                  // columns read at once
        const uint32_t quarter = warp & 3u, half = (warp - 2u) >> 2;
        uint8_t* const stg = staging + (warp - 2u) * 4096u;
        float lg[2][kCh ? kCh : 1] = {};                                     // this row's logits over the warp's first and second 64 columns
        const bool vec = !kPacked && (p.ld * sizeof(T)) % 16 == 0 && ((uintptr_t)p.out & 15) == 0;
        float* const bias_s = reinterpret_cast<float*>(staging + kEpiWarps * 4096) + half * kHalf;       // shared by the half's four warps
        uint32_t i = 0;
        bool ok = true;
        for (uint32_t t = t_begin; t < t_end && ok; t++, i++) {
            uint32_t row, tn;
            seg.find(t, C::kRows, row, tn);
            const uint32_t end = p.offsets ? min(p.offsets[seg.e + 1], p.capacity) : (p.n_rows_dev ? min(*p.n_rows_dev, p.capacity) : p.capacity);
            const uint32_t row0 = row + rank * 128 + quarter * 32, col0 = tn * BN + half * kHalf;
            // (columns quarter * 32 ... of the half, fetched while the tile is multiplied)
            const uint32_t bias_c = quarter * (kHalf / 4) + lane;
            const float bias_v = p.bias && lane < kHalf / 4 && col0 + bias_c < p.N ? __ldg(p.bias + (size_t)seg.e * p.N + col0 + bias_c) : 0.0f;
            // (the half's four warps go on, or leave, together: they meet again below.  All have written the tile before by now)
            // (with a head all eight meet: the halves exchange logits)
            ok = mbar_wait(&bars->acc_full[i & 1u], (i >> 1) & 1u, abort_flag);
            ok = kCh ? all_agree(3, 256, ok) : all_agree(1u + half, 128, ok);
            if (!ok) break;
            tc_fence_after();
            const uint32_t taddr = tmem + ((quarter * 32u) << 16) + (i & 1u) * C::kSecond + half * kHalf;
            auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) mbar_arrive_relaxed(map_to_cta(smem_u32(&bars->acc_free[i & 1u]), 0));
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
                if ((shares && n == 0) || (!C::kOverlap && n + 1 == kHalf / kCols)) release();
                if (n == 0) {
                    if (lane < kHalf / 4) bias_s[bias_c] = bias_v;
                    asm volatile("bar.sync %0, 128;" ::"r"(1u + half) : "memory");
                }
                if (col0 + c >= (kPacked ? k_tiles(p.N) * 128 : p.N)) continue;
                if constexpr (kCh != 0) finish<__nv_bfloat16, kCols, true>(v, bias_s + c);
                else if (!kPacked && p.relu) finish<T, kCols, true>(v, bias_s + c);
                else finish<T, kCols, false>(v, bias_s + c);
                if constexpr (kCh != 0) {
                    if (c == 0) add_head<kCh, kCols / 2>(lg[0], v, staging, col0);
                    else add_head<kCh, kCols / 2>(lg[1], v, staging, col0 + c);
                } else if constexpr (kPacked) {
                    // a lane's 32 consecutive columns are one scale block
                    const uint32_t col = col0 + c, pitch = row_bytes(p.N), kt = k_tiles(p.N);
                    if (col + kCols > p.N) {                                 // columns that fill the last block, and blocks behind it
#pragma unroll
                        for (uint32_t q = 0; q < kCols; q++) if (col + q >= p.N) v[q] = 0;
                    }
                    uint32_t w[kCols / 8], bytes = 0;
                    if (p.relu) pack_blocks<kCols, true>(v, w, bytes); else pack_blocks<kCols, false>(v, w, bytes);
#pragma unroll
                    for (uint32_t g = 0; g < kCols; g += 32) if (col + g >= p.N) bytes = (bytes & ~(0xFFu << (g / 4))) | 127u << (g / 4);
                    if (row0 + lane < end) {
                        uint8_t* const o = reinterpret_cast<uint8_t*>(p.out) + (size_t)(row0 + lane) * pitch + col / 2;
                        uint8_t* const so = p.out_scales + scale_at(row0 + lane, col / 32, kt);
                        if constexpr (kCols == 64) {
                            if (col + 32 < p.N && (((uintptr_t)p.out | pitch) & 31u) == 0)         // whole 32-byte sectors
                                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                                             ::"l"(o), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
                            else {
                                if (col < p.N) *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
                                if (col + 32 < p.N) *reinterpret_cast<uint4*>(o + 16) = make_uint4(w[4], w[5], w[6], w[7]);
                            }
                            *reinterpret_cast<uint16_t*>(so) = (uint16_t)bytes;              // (col < k_tiles * 128: both blocks have a place)
                        } else {
                            if (col < p.N) *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
                            *so = (uint8_t)bytes;
                        }
                    }
                } else {
                    constexpr uint32_t kWords = kCols * sizeof(T) / 4;       // a row's words,
                    constexpr uint32_t kAt = kWords < 32 ? kWords : 32;      // ... 32 of them (128 bytes) staged at a time, 16-byte pieces
                    constexpr uint32_t kPieces = kAt / 4;                    // XOR-swizzled by row as a 128-byte swizzled TMA box has them
                    constexpr uint32_t kPer = 16 / sizeof(T);                // values of a piece
                    const bool inside = row0 + 32 <= end;
#pragma unroll
                    for (uint32_t g = 0; g < kWords; g += kAt) {
                        const uint32_t col = col0 + c + g / 4 * kPer;
                        if (tma_out) {                                       // the last box has been read
                            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                            __syncwarp();
                        }
#pragma unroll
                        for (uint32_t j = 0; j < kPieces; j++)
                            *reinterpret_cast<uint4*>(stg + lane * 128u + ((j ^ (lane & 7u)) << 4)) = make_uint4(v[g + 4 * j], v[g + 4 * j + 1], v[g + 4 * j + 2], v[g + 4 * j + 3]);
                        if (tma_out && inside) {                             // (columns beyond N are left out by the map)
                            fence_proxy_async();
                            __syncwarp();
                            if (lane == 0 && col < p.N) {
                                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                                             ::"l"(reinterpret_cast<uint64_t>(&tmO)), "r"(col), "r"(row0), "r"(smem_u32(stg)) : "memory");
                                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                            }
                            continue;
                        }
                        __syncwarp();
                        if (!vec) {                                          // rows on any boundary: consecutive columns, element by element
                            constexpr uint32_t kLane = kAt * 4 / sizeof(T) / 32;             // columns of a row per lane
                            T* const o = reinterpret_cast<T*>(p.out) + (size_t)row0 * p.ld + col;
                            const uint32_t rows_in = end > row0 ? min(32u, end - row0) : 0u;
#pragma unroll 8
                            for (uint32_t r = 0; r < rows_in; r++) {
#pragma unroll
                                for (uint32_t h = 0; h < kLane; h++) {
                                    const uint32_t x = h * 32 + lane;        // its 16-byte piece is swizzled by row
                                    const T val = *reinterpret_cast<const T*>(stg + r * 128u + (((x / kPer) ^ (r & 7u)) << 4) + (x % kPer) * sizeof(T));
                                    if (col + x < p.N) o[(size_t)r * p.ld + x] = val;
                                }
                            }
                            __syncwarp();
                            continue;
                        }
                        constexpr uint32_t kRowsAt = 32 / kPieces;           // rows per store instruction
                        const uint32_t q = lane % kPieces, r = lane / kPieces, at = col + q * kPer;
                        T* const o = reinterpret_cast<T*>(p.out) + (size_t)(row0 + r) * p.ld + at;
#pragma unroll
                        for (uint32_t k = 0; k < 32; k += kRowsAt) {
                            if (row0 + k + r >= end || at >= p.N) continue;
                            const uint4 val = *reinterpret_cast<const uint4*>(stg + (k + r) * 128u + ((q ^ ((k + r) & 7u)) << 4));
                            T* const d = o + (size_t)k * p.ld;
                            if (vec && at + kPer <= p.N) { *reinterpret_cast<uint4*>(d) = val; continue; }
                            const T* const e = reinterpret_cast<const T*>(&val);
#pragma unroll
                            for (uint32_t x = 0; x < kPer; x++) if (at + x < p.N) d[x] = e[x];
                        }
                        __syncwarp();
                    }
                }
            }
            if constexpr (kCh != 0) {
                if (tn + 1 == tiles_n) {                                     // the panel's end: the halves meet
                    if (half == 1) {
#pragma unroll
                        for (uint32_t q = 0; q < kCh; q++) partial[(quarter * 32 + lane) * kCh + q] = lg[0][q] + lg[1][q];
                    }
                    asm volatile("bar.sync 4, 256;" ::: "memory");
                    if (half == 0 && row0 + lane < end) {
                        float best = 0.0f;
                        uint32_t arg = 0;
#pragma unroll
                        for (uint32_t q = 0; q < kCh; q++) {
                            if (q < p.C) {
                                const float x = ((lg[0][q] + lg[1][q]) + partial[(quarter * 32 + lane) * kCh + q]) + __ldg(p.head_b + q);
                                p.logits[(size_t)(row0 + lane) * p.C + q] = x;
                                if (q == 0 || x > best) { best = x; arg = q; }
                            }
                        }
                        if (p.label) p.label[row0 + lane] = (uint8_t)arg;
                    }
#pragma unroll
                    for (uint32_t q = 0; q < kCh; q++) lg[0][q] = lg[1][q] = 0.0f;
                }
            }
        }
        // Every way out of the loop ends here: the block's shared memory is not given up before its last boxes have been read out of it.
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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
    // the most tiles there can be: every expert's last tile may be a part of one
    const uint64_t most = ((uint64_t)p.capacity / C::kRows + p.E) * (((std::is_same<T, Mx4>::value ? k_tiles(p.N) * 128 : p.N) + BN - 1) / BN);
    if (most > 0x7FFFFFFFull) return SF_ERR_UNSUPPORTED;
    CUtensorMap tmA, tmW, tmSA, tmSW, tmO;
    int rc = encode_tmap_2d(&tmA, CU_TENSOR_MAP_DATA_TYPE_UINT8, p.a, p.capacity, pitch, pitch, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc == SF_OK) rc = encode_tmap_2d(&tmW, CU_TENSOR_MAP_DATA_TYPE_UINT8, p.w, (uint64_t)p.E * p.N, pitch, pitch, PAIR ? BN / 2 : BN, 128, CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc == SF_OK) rc = encode_tmap_2d(&tmSA, CU_TENSOR_MAP_DATA_TYPE_UINT32, p.a_scales, (p.capacity + 127) / 128, kt * 128, kt * 512, 1, 256, CU_TENSOR_MAP_SWIZZLE_NONE);
    if (rc == SF_OK) rc = encode_tmap_2d(&tmSW, CU_TENSOR_MAP_DATA_TYPE_UINT32, p.w_scales, (uint64_t)p.E * ((p.N + 127) / 128), kt * 128, kt * 512, C::kNT, 256, CU_TENSOR_MAP_SWIZZLE_NONE);
    bool tma_out = false;
    if constexpr (!std::is_same<T, Mx4>::value && HeadOf<T>::kCh == 0) {
        tma_out = aligned(p.out, 16) && (p.ld * sizeof(T)) % 16 == 0 && (p.N * sizeof(T)) % 16 == 0 && !(BN == 64 && sizeof(T) == 2);      // (64 16-bit columns: a warp has 64 bytes of a row)
        if (rc == SF_OK && tma_out) rc = encode_tmap_2d(&tmO, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, p.out,
                                                        p.capacity, p.N, p.ld * sizeof(T), 32, 128 / sizeof(T), CU_TENSOR_MAP_SWIZZLE_128B);
    }
    if (!tma_out) tmO = tmA;                           // not read
    if (rc != SF_OK) return rc;
    auto kern = mx4_product_kernel<BN, PAIR, T>;
    static bool set_dev[64] = {};                      // the opt-in is per device
    bool& set = set_dev[ctx->device & 63];
    if (!set) { SF_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::template smem<T>(SF_MAX_EXPERTS))); set = true; }
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((PAIR ? 2u : 1u) * (uint32_t)std::min<uint64_t>((uint64_t)ctx->num_sms / (PAIR ? 2 : 1), most));
    lc.blockDim = dim3(kThreads); lc.dynamicSmemBytes = C::template smem<T>(p.E); lc.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    lc.attrs = at; lc.numAttrs = PAIR ? 2 : 1;
    SF_CUDA(cudaLaunchKernelEx(&lc, kern, tmA, tmW, tmSA, tmSW, tmO, (uint32_t)tma_out, p, ctx->d_state));
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
        lc.gridDim = dim3(2); lc.blockDim = dim3(kThreads); lc.dynamicSmemBytes = C::template smem<T>(SF_MAX_EXPERTS);
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
        lc.attrs = at; lc.numAttrs = 1;
        int n = 0;
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::template smem<T>(SF_MAX_EXPERTS));
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&n, kern, &lc);
        if (e != cudaSuccess) (void)cudaGetLastError();
        c = e == cudaSuccess && n > 0 ? 1 : -1;
    }
    return c > 0;
}

int check(const sf_ctx* ctx, const sf_mx4_product& p)
{
    const bool packed = p.out_dtype == SF_MX4;
    if (!ctx || (!packed && !type_ok(p.out_dtype)) || p.N == 0 || p.K == 0 || p.K > SF_MX4_MAX_K || p.N > SF_MX4_MAX_K || (!packed && p.ld < p.N)) return SF_ERR_ARG;
    if (p.capacity > 0x7FFFFF00u || (uint64_t)p.E * p.N > 0x7FFFFFFFull) return SF_ERR_ARG;      // tile coordinates are 32-bit signed
    if (p.capacity == 0) return SF_OK;
    if (!p.a || !p.a_scales || !p.w || !p.w_scales || !p.out) return SF_ERR_ARG;
    if (!aligned(p.a, 16) || !aligned(p.a_scales, 16) || !aligned(p.w, 16) || !aligned(p.w_scales, 16)) return SF_ERR_ARG;
    if (packed != (p.out_scales != nullptr) || !aligned(p.out_scales, 16)) return SF_ERR_ARG;
    if (!aligned(p.out, packed ? 16 : type_bytes(p.out_dtype)) || !aligned(p.bias, 4) || !aligned(p.n_rows_dev, 4) || !aligned(p.offsets, 4)) return SF_ERR_ARG;
    return SF_OK;
}

}  // namespace

// Pairs where their tiles give every pair of SMs one (rows and tiles as far as the host knows them: the counts live on the device); 64-column
// tiles where 128-column ones would not give every SM one.
static bool use_pairs(const sf_ctx* ctx, const sf_mx4_product& p) {
    const uint64_t rows = std::max<uint64_t>(1, p.capacity / p.E);
    return p.N > 128 && rows >= 256 && (rows + 255) / 256 * p.E * ((p.N + 255) / 256) >= (uint64_t)ctx->num_sms / 2;
}

bool sf_mx4_product_takes_head(sf_ctx* ctx, const sf_mx4_product& p) {
    // A pair has whole panels: from a panel for every pair on.  Up to eight classes: 240,000 rows, 1024 -> 1024 and the head take 113, 147 and 212
    // us with 2, 4 and 8 classes folded in, about 220 in two launches; with 16 the epilogue's products take 600.
    return use_pairs(ctx, p) && p.E == 1 && p.N <= kHeadMaxN && p.N % 64 == 0 && p.C >= 1 && p.C <= 8 && p.relu &&
           (p.capacity + 255) / 256 >= (uint32_t)ctx->num_sms / 2 && pairs_supported<Head<8>>(ctx);
}

int sf_launch_mx4_product(sf_ctx* ctx, const sf_mx4_product& p, cudaStream_t st)
{
    if (p.head_w) {
        if (p.C <= 2) return launch<256, true, Head<2>>(ctx, p, st);
        if (p.C <= 4) return launch<256, true, Head<4>>(ctx, p, st);
        return launch<256, true, Head<8>>(ctx, p, st);
    }
    const bool pairs = use_pairs(ctx, p);
    const uint64_t rows = std::max<uint64_t>(1, p.capacity / p.E);
    const bool narrow = (rows + 127) / 128 * p.E * ((p.N + 127) / 128) < (uint64_t)ctx->num_sms;
    auto go = [&](auto zero) {
        typedef decltype(zero) T;
        if (pairs && pairs_supported<T>(ctx)) return launch<256, true, T>(ctx, p, st);
        return narrow ? launch<64, false, T>(ctx, p, st) : launch<128, false, T>(ctx, p, st);
    };
    return p.out_scales ? go(Mx4()) : by_type(p.out_dtype, go);
}

// ---- the slow model's hidden layers in 4 bits ------------------------------------------------------------------
// The wide rows (bf16) are packed once; every hidden layer but the last packs its own output in its epilogue (from the fp32 sums: no
// activations in 16 bits in between); the head stays in bf16 (its logits decide labels) and takes the last layer's outputs rounded to
// bf16, in that layer's epilogue for large batches, else by a launch of its own.
namespace {
struct MlpScratch { size_t data, scales, half, bytes; };      // two packed buffers, then the bf16 rows of the last hidden layer
MlpScratch mlp_scratch(const sf_slow* s, uint32_t capacity) {
    uint32_t widest = 0;
    for (uint32_t l = 0; l + 1 < s->n_layers; l++) widest = std::max(widest, s->dims[l]);
    MlpScratch m;
    m.data = sf_align256((size_t)capacity * row_bytes(widest));
    m.scales = sf_align256(scale_bytes(capacity, widest));
    m.half = 2 * (m.data + m.scales);
    m.bytes = m.half + sf_align256((size_t)capacity * s->dims[s->n_layers - 1] * 2) + 256;
    return m;
}
}  // namespace

size_t sf_mlp_mx4_scratch_bytes(const sf_slow* s, uint32_t capacity) { return mlp_scratch(s, capacity).bytes; }

int sf_mlp_mx4_forward(sf_ctx* ctx, const sf_slow* s, const void* rows, const uint32_t* n_rows_dev, uint32_t capacity,
                       float* logits, uint8_t* label, void* scratch, cudaStream_t st)
{
    const MlpScratch m = mlp_scratch(s, capacity);
    uint8_t* const w = reinterpret_cast<uint8_t*>(scratch);
    uint8_t* const data[2] = {w, w + m.data + m.scales};
    uint8_t* const scales[2] = {data[0] + m.data, data[1] + m.data};
    const uint32_t L = s->n_layers - 1;                  // the head
    sf_time_begin(ctx, SF_T_GEMM, st);
    int rc = sf_launch_mx4_quantise(ctx, rows, SF_BF16, capacity, s->dims[0], s->dims[0], nullptr, n_rows_dev, capacity, data[0], scales[0], st);
    bool folded = false;
    for (uint32_t l = 0; l < L && rc == SF_OK; l++) {
        const bool last = l + 1 == L;
        const uint32_t i = l & 1u;
        sf_mx4_product p = {data[i], scales[i], n_rows_dev, nullptr, 1, capacity, (const uint8_t*)s->d_W[l], (const uint8_t*)s->d_S[l], s->dims[l + 1], s->dims[l],
                            s->d_b[l], 1, SF_BF16, w + m.half, s->dims[l + 1], nullptr, nullptr, nullptr, 0, nullptr, nullptr};
        if (last) {
            p.C = s->dims[L + 1];
            if (sf_mx4_product_takes_head(ctx, p)) { p.head_w = s->d_W[L]; p.head_b = s->d_b[L]; p.logits = logits; p.label = label; }
            folded = p.head_w != nullptr;
        }
        if (!last) { p.out_dtype = SF_MX4; p.out = data[i ^ 1u]; p.out_scales = scales[i ^ 1u]; }
        rc = sf_launch_mx4_product(ctx, p, st);
    }
    sf_time_end(ctx, SF_T_GEMM, st);
    if (rc != SF_OK || folded) return rc;
    sf_time_begin(ctx, SF_T_HEAD, st);
    rc = sf_mlp_head_bf16(ctx, w + m.half, s->d_W[L], s->d_b[L], n_rows_dev, capacity, s->dims[L], s->dims[L + 1], logits, label, st);
    sf_time_end(ctx, SF_T_HEAD, st);
    return rc;
}

extern "C" int sf_mx4_matmul(sf_ctx* ctx, const uint8_t* a, const uint8_t* a_scales, const uint32_t* n_rows_dev, uint32_t capacity,
                             const uint8_t* w, const uint8_t* w_scales, uint32_t N, uint32_t K, const float* bias, int relu,
                             int out_dtype, void* out, size_t ld, uint8_t* out_scales, void* stream)
{
    const sf_mx4_product p = {a, a_scales, n_rows_dev, nullptr, 1, capacity, w, w_scales, N, K, bias, relu, out_dtype, out, ld, out_scales, nullptr, nullptr, 0, nullptr, nullptr};
    const int rc = check(ctx, p);
    if (rc != SF_OK || capacity == 0) return rc;
    SF_ON_DEVICE(ctx);
    return sf_launch_mx4_product(ctx, p, (cudaStream_t)stream);
}

extern "C" int sf_mx4_matmul_experts(sf_ctx* ctx, const uint8_t* a, const uint8_t* a_scales, const uint32_t* offsets, uint32_t E,
                                     uint32_t capacity, const uint8_t* w, const uint8_t* w_scales, uint32_t N, uint32_t K,
                                     const float* bias, int relu, int out_dtype, void* out, size_t ld, uint8_t* out_scales, void* stream)
{
    if (E == 0 || E > SF_MAX_EXPERTS || (capacity && !offsets)) return SF_ERR_ARG;
    const sf_mx4_product p = {a, a_scales, nullptr, offsets, E, capacity, w, w_scales, N, K, bias, relu, out_dtype, out, ld, out_scales, nullptr, nullptr, 0, nullptr, nullptr};
    const int rc = check(ctx, p);
    if (rc != SF_OK || capacity == 0) return rc;
    SF_ON_DEVICE(ctx);
    return sf_launch_mx4_product(ctx, p, (cudaStream_t)stream);
}
