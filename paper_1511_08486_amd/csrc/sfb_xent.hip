// Softmax cross entropy of a linear head, z_i = W a_i, without the N x J scores in memory, and its gradients.
//
//   lse_i = log sum_j exp(z_ij)       loss_i = lse_i - z_i,y(i)
//   u_ij  = w_i (exp(z_ij - lse_i) - [j = y(i)])         dA = f U W       dW = f U^T A      (w: the rows' weights, f: the scale)
// Rows whose label is outside [0, J) take no part: the others are packed to the front (by their labels, on the device), so a padded batch
// costs what its real rows cost, and what stands in the padding is never multiplied.
//
// Pieces of the vocabulary: the loss needs of the scores only a maximum and a sum per row and tile of 256 words, taken from the
// accumulators.  The gradients form one piece of the scores again, turn it into a piece of U in the accumulators as well (16-bit terms, the
// only thing kept of it), and multiply that with W's piece (dA, added up over the pieces in fp32) and with A (dW's rows, done at once).
//
// One kernel multiplies: out[n][m] = sum_k Y[n][k] X[m][k], operands in bf16 terms, m contiguous in memory; X and Y each lie with k
// contiguous or with k as their slow index (gfx950's transposing LDS read takes those as they are).
//   scores  X = W[j][d], Y = A[i][d]      dA  X = W[j][d] (k = j slow), Y = U[i][j]      dW  X = A[i][d], Y = U[i][j] (k = i slow, both)
// fp32 operands go in terms of 16 bits, a longer k to the kernel, the small products first:
//   scores and dA  two fp16 terms of every row divided by its own power of two, x = 2^e (h + l / 2048): 22 bits of every value above 2^-29 of its
//                  row's largest, and three products (two with one bf16 operand, which is one fp16 term).  Of dA's contraction W's exponents
//                  are in U, and U's rows are divided by what their weight bounds them by.  A bf16 dA takes one term of each (2^-12).
//   dW             three bf16 terms (exact) and six products (three with bf16 features): along its contraction, the rows, the factors of a
//                  rare word may all be below 2^-40 of a label's, and must not be rounded by that.
//   fp32 W, up to 64 rows   three bf16 terms of W, split where they are used, in scores and dA too (a bf16 dA: two)
// Small problems keep their scores (256 MB at most, their slices of D included) where forming them again would take longer than reading them.
//
// Bound by: many rows, the matrix cores at the clock that they hold (131072 words, 4096 rows and features, bf16: scores 1.20 PFLOP/s, with U
// 1.10, dA 1.30, dW 1.18, the clock at 1.63 GHz, 64 to 75 % of its cycles in matrix instructions, LDS a fifth, no bank conflicts); few rows, W's
// way from memory (65536 x 4096 in bf16, 24 rows: 109 us, 4.9 TB/s).
#include "sfb_kernels.h"
#include "sfb_split.h"

namespace sfb {

typedef uint32_t xe_u32x4u __attribute__((ext_vector_type(4), aligned(2)));   // a 16-byte access at any bf16's address

constexpr int kXeK = 64;           // k of a stage: 128 bytes of a row
enum XentEnd { kXeStats = 0, kXeU = 1, kXeStore = 2 };

struct XentProduct {
    const bf16_t *x, *y;
    int64_t ldx, ldy, x_plane, y_plane;      // in elements
    int x_rows, y_rows;                      // rows in memory (reads are clamped to them)
    int x_cols, y_cols;                      // k slow: columns that may be read, a multiple of 8
    int M, N;
    int k_tiles, last_x, last_y;             // stages of one pair of terms; where the last one begins (k contiguous)
    int pairs;
    uint32_t pair_x, pair_y;                 // four bits a pair: the terms of X and Y, in order
    const int *exp_m, *exp_n, *exp_top;      // fp16 terms: results are times 2^(exp_m[m] + exp_n[n] + *exp_top); null: 0
    int m_tiles, n_tiles, total, splits, per_split;
    const int* count;                        // rows that take part; null: all N
    bool n_is_rows, k_is_rows;               // what `count` bounds
    // kXeStats, kXeU
    const int* label;
    int first_word;                          // word of m = 0
    float2* partial;                         // [rows][ld_partial], from this product's first tile on
    float* z_label;
    int ld_partial;
    const float *lse, *g;
    bf16_t *u, *u16;                         // [terms][..][ldu], in bf16 and fp16
    int64_t ldu, u_plane;
    int u_terms, u16_terms;
    const int *exp_g, *exp_words;            // U's fp16 terms are of u 2^(exp_m[m] - exp_g[n] - *exp_words)
    // kXeStore
    void* out;
    int64_t ldo, out_plane;                  // out_plane: between splits
    const float* factor;                     // of the results
    const float* add;                        // fp32, or nullptr
    int64_t ld_add;
    const int* row_map;                      // row of out for n, or nullptr
    const float *loss_packed, *weights;      // of the total, if the first workgroup is to form that
    float* loss_total;
};

__device__ __forceinline__ uint32_t xe_lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// 64 lanes x 16 bytes from base + off to LDS, lane l's at lds + 16 l (not seen by the compiler: waits are the caller's)
__device__ __forceinline__ void xe_dma(const void* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}

// exp(x), x <= 0 or little more, off by |x| 2^-23 of itself: what x's own rounding, of a difference of two scores, is worth as well
__device__ __forceinline__ float xe_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// How one operand goes to LDS and comes from there.  ROWS: of m (n) in the tile.  Not TR: LDS rows of 64 k, 16-byte piece p of row r at
// p ^ (r & 7) ^ (r >> 3 & 1): sixteen consecutive rows on sixteen different bank groups (without the last bit half of all reads waited).  TR: LDS rows of ROWS m, 32-byte piece p of k-row r at p ^ turn(r), so that the four rows of a transposing read, and its
// neighbour's sixteen columns, fall on different banks.
template <bool TR, int ROWS, int WAVES, int TILES>
struct XentSide {
    static constexpr int LOADS = ROWS / 8 / WAVES, BYTES = ROWS * 128;
    static_assert(LOADS * 8 * WAVES == ROWS && WAVES % 2 == 0, "whole accesses");
    uint32_t off[LOADS];
    int at[TR ? TILES : 4];
    __device__ __forceinline__ static int turn(int r) { return ROWS >= 128 ? 2 * (r & 3) : r & 3; }
    // k_most: the last k-row that may be read, counted from the stage's first
    __device__ __forceinline__ void offsets(int wave, int lane, int row0, int rows, int cols, int64_t ld, int k_most) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            if constexpr (!TR) {
                const int r = min(row0 + (i * WAVES + wave) * 8 + (lane >> 3), rows - 1) - row0;
                off[i] = (uint32_t)r * (uint32_t)ld * 2u + (uint32_t)(((lane & 7) ^ ((lane >> 3) & 7) ^ (wave & 1)) * 16);
            } else {
                constexpr int PER = ROWS / 8;
                const int q = (i * WAVES + wave) * 64 + lane, r = q / PER, p = q % PER;
                const int c = min(row0 + 8 * (2 * ((p >> 1) ^ turn(r)) + (p & 1)), cols - 8) - row0;
                off[i] = (uint32_t)min(r, k_most) * (uint32_t)ld * 2u + (uint32_t)c * 2u;
            }
        }
    }
    // first: the wavefront's first row (column) in the tile
    __device__ __forceinline__ void places(int lane, int first) {
        const int l32 = lane & 31, half = lane >> 5;
        if constexpr (!TR) {
#pragma unroll
            for (int s = 0; s < 4; ++s) at[s] = (first + l32) * 128 + (((2 * s + half) ^ (l32 & 7) ^ ((l32 >> 3) & 1)) << 4);
        } else {
            // sixteen lanes read four k of sixteen columns and are handed a column each; the next sixteen the other columns, the next k eight on
            const int g = lane >> 4, l16 = lane & 15, k = 8 * (g >> 1) + (l16 >> 2);
#pragma unroll
            for (int i = 0; i < TILES; ++i) at[i] = k * (ROWS * 2) + 32 * (((first >> 4) + 2 * i + (g & 1)) ^ turn(k)) + 8 * (l16 & 3);
        }
    }
    template <int S, int I>
    __device__ __forceinline__ sp_u32x4 read(const unsigned char* lds) const {
        if constexpr (!TR) {
            return *reinterpret_cast<const sp_u32x4*>(lds + at[S] + I * 4096);
        } else {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4* lds_ptr;
            const unsigned char* p = lds + at[I] + S * 16 * ROWS * 2;
            const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p));
            const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * ROWS * 2)));
            return sp_u32x4{lo.x, lo.y, hi.x, hi.y};
        }
    }
};

__device__ __forceinline__ void xe_wait_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void xe_stage_barrier() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory"); }

// fp16 terms of x[0..3], the second 2^11 times as large; x becomes what they leave
__device__ __forceinline__ uint2 xe_half4(float (&x)[4]) {
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    const h4 h = {(_Float16)x[0], (_Float16)x[1], (_Float16)x[2], (_Float16)x[3]};
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (x[e] - (float)h[e]) * 2048.f;
    return __builtin_bit_cast(uint2, h);
}
__device__ __forceinline__ uint2 xe_bf4(float (&x)[4]) {
    const uint2 w = make_uint2(cvt_pk_bf16(x[0], x[1]), cvt_pk_bf16(x[2], x[3]));
    x[0] -= __uint_as_float(w.x << 16);
    x[1] -= __uint_as_float(w.x & 0xffff0000u);
    x[2] -= __uint_as_float(w.y << 16);
    x[3] -= __uint_as_float(w.y & 0xffff0000u);
    return w;
}

template <bool F16>
__device__ __forceinline__ f32x16 xe_mfma(sp_u32x4 a, sp_u32x4 b, f32x16 c) {
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(sp_f16x8, a), __builtin_bit_cast(sp_f16x8, b), c, 0, 0, 0);
    else return split_mfma(a, b, c);
}

// A tile's maxima and sums of exponentials by rows, and the scores of labels among its words.  Entry e of acc[i][j]: word
// m0 + 32 (wm MT + i) + 8 (e / 4) + 4 (lane / 32) + e % 4 of row n0 + 32 (wn NT + j) + lane % 32.
template <int WGM, int MT, int NT, int BN>
__device__ __forceinline__ void xe_stats_end(const XentProduct& a, f32x16 (&acc)[MT][NT], int m0, int n0, int wm, int wn, int lane, int count) {
    constexpr int BM = WGM * MT * 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char xe_lds[];
    const int tid = threadIdx.x, l32 = lane & 31, half = lane >> 5;
    const int mw = m0 + wm * MT * 32 + 4 * half, nw = n0 + wn * NT * 32 + l32;
            float2* const red = reinterpret_cast<float2*>(xe_lds);
            const bool inside = m0 + BM <= a.M;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int n = nw + 32 * j;
                const int hit = n < count ? a.label[n] - a.first_word - mw : -1;         // this lane's offset of the label's word
                float top = -__builtin_inff(), sum = 0.f, z_hit = 0.f;
                bool got = false;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int m = 32 * i + 8 * (e / 4) + e % 4;
                        if (!inside && mw + m >= a.M) acc[i][j][e] = -__builtin_inff();
                        top = fmaxf(top, acc[i][j][e]);
                        if (hit == m) { z_hit = acc[i][j][e]; got = true; }
                    }
                const float base = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum += xe_exp(acc[i][j][e] - base);
                if (got) a.z_label[n] = z_hit;
                const float top2 = __shfl_xor(top, 32, kWave), sum2 = __shfl_xor(sum, 32, kWave);
                const float t = fmaxf(top, top2), b = t == -__builtin_inff() ? 0.f : t;
                sum = sum * xe_exp(top - b) + sum2 * xe_exp(top2 - b);
                if (half == 0) red[wm * BN + wn * NT * 32 + 32 * j + l32] = make_float2(t, sum);
            }
            __syncthreads();
            for (int n = tid; n < BN; n += blockDim.x) {
                float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
                for (int w = 0; w < WGM; ++w) top = fmaxf(top, red[w * BN + n].x);
                const float base = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
                for (int w = 0; w < WGM; ++w) sum += red[w * BN + n].y * xe_exp(red[w * BN + n].x - base);
                if (n0 + n < count) a.partial[(int64_t)(n0 + n) * a.ld_partial + m0 / BM] = make_float2(top, sum);
            }
}

// total = f sum of g loss in a fixed order, in 64 bits, by one workgroup; `part`: 8 bytes of LDS a wavefront
__device__ __forceinline__ void xe_total(const float* loss, const float* g, int n, const float* factor, float* total, double* part) {
    double s = 0.0;
    for (int k = threadIdx.x; k < n; k += blockDim.x) s += (double)loss[k] * (double)g[k];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int w = 0; w < (int)blockDim.x / 64; ++w) s += part[w];
        *total = (float)(s * (double)*factor);
    }
    __syncthreads();
}

// F16: operands in fp16 terms, exponents beside them; the products of a second term come first and are 2^11 times as large
template <int WGM, int WGN, int MT, int NT, int ST, int OCC, bool XT, bool YT, bool F16, int END, class Out>
__global__ __launch_bounds__(WGM * WGN * 64, OCC) void xent_product_kernel(const XentProduct a) {
    constexpr int WAVES = WGM * WGN, BM = WGM * MT * 32, BN = WGN * NT * 32;
    typedef XentSide<XT, BM, WAVES, MT> SideX;
    typedef XentSide<YT, BN, WAVES, NT> SideY;
    constexpr int STAGE = SideX::BYTES + SideY::BYTES, LOADS = SideX::LOADS + SideY::LOADS;
    extern __shared__ __attribute__((aligned(16))) unsigned char xe_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5, wm = wave / WGN, wn = wave % WGN;

    int id = xcd_contiguous_id(blockIdx.x, a.total);
    const int split = id / (a.m_tiles * a.n_tiles);
    id -= split * (a.m_tiles * a.n_tiles);
    // eight tiles of m beside each other for every n: what a die works on at once shares operands
    const int band = id / (8 * a.n_tiles), in_band = id - band * (8 * a.n_tiles), wide = min(8, a.m_tiles - 8 * band);
    const int m0 = (8 * band + in_band % wide) * BM, n0 = in_band / wide * BN;

    const int count = a.count ? *a.count : a.N;
    if constexpr (END == kXeStore) {
        if (a.loss_total && blockIdx.x == 0) xe_total(a.loss_packed, a.weights, count, a.factor, a.loss_total, reinterpret_cast<double*>(xe_lds));
    }
    if (a.n_is_rows && n0 >= count) return;
    const int k_tiles = a.k_is_rows ? (count + kXeK - 1) / kXeK : a.k_tiles;
    const int k_begin = min(split * a.per_split, k_tiles), k_end = min(k_begin + a.per_split, k_tiles);
    const int stages = (k_end - k_begin) * a.pairs;

    SideX sx;
    SideY sy;
    sx.places(lane, wm * MT * 32);
    sy.places(lane, wn * NT * 32);
    sx.offsets(wave, lane, m0, a.x_rows, a.x_cols, a.ldx, 63);
    sy.offsets(wave, lane, n0, a.y_rows, a.y_cols, a.ldy, 63);
    const uint32_t lds0 = xe_lds_address(xe_lds);

    // the stage being requested
    int q_pair = 0, q_k = k_begin;
    uint32_t q_lds = lds0;
    const bf16_t *q_x, *q_y;
    bool q_short = false;
    auto aim = [&]() {
        const bool last = q_k == k_tiles - 1;
        const bf16_t* x = a.x + (int64_t)((a.pair_x >> (4 * q_pair)) & 15u) * a.x_plane;
        const bf16_t* y = a.y + (int64_t)((a.pair_y >> (4 * q_pair)) & 15u) * a.y_plane;
        q_x = XT ? x + (int64_t)q_k * kXeK * a.ldx + m0 : x + (int64_t)m0 * a.ldx + (last ? a.last_x : q_k * kXeK);
        q_y = YT ? y + (int64_t)q_k * kXeK * a.ldy + n0 : y + (int64_t)n0 * a.ldy + (last ? a.last_y : q_k * kXeK);
        if constexpr (XT) {                                              // rows of k beyond the last: W's own piece may end inside a stage
            const int most = a.x_rows - 1 - q_k * kXeK;
            if (most < 63 || q_short) sx.offsets(wave, lane, m0, a.x_rows, a.x_cols, a.ldx, min(most, 63));
            q_short = most < 63;
        }
    };
    auto next = [&]() {
        if (++q_k == k_end) {
            q_k = k_begin;
            ++q_pair;
        }
        q_lds += STAGE;
        if (q_lds == lds0 + ST * STAGE) q_lds = lds0;
    };
    auto request = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
        if constexpr (i < SideX::LOADS) xe_dma(q_x, sx.off[i], q_lds + (i * WAVES + wave) * 1024);
        else xe_dma(q_y, sy.off[i - SideX::LOADS], q_lds + SideX::BYTES + ((i - SideX::LOADS) * WAVES + wave) * 1024);
    };

    f32x16 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    // Tiles for few rows, whose vector units have time, add up blocks of 256 k: a score of 2048 k is rounded 16 times at an eighth of its
    // size and 8 times at its whole, not 128 times (a single token's loss of 0.05 at scores of 20 was 6.1e-6 off, 6.5e-7 so)
    constexpr bool BLOCKS = BN <= 64;
    f32x16 sum[BLOCKS ? MT : 1][BLOCKS ? NT : 1];
    if constexpr (BLOCKS) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) sum[i][j] = acc[i][j];
    }

    struct Frag { sp_u32x4 x[MT], y[NT]; };
    Frag f0, f1;
    auto read = [&](auto sc, auto rc, Frag& f, const unsigned char* lds) {
        constexpr int s = decltype(sc)::value, r = decltype(rc)::value;
        if constexpr (r < MT) f.x[r] = sx.template read<s, r>(lds);
        else f.y[r - MT] = sy.template read<s, r - MT>(lds + SideX::BYTES);
    };
    constexpr int READS = MT + NT, MFMAS = MT * NT, SPREAD = MFMAS > 1 ? MFMAS / 2 : 1;
    // multiplies `now`; meanwhile reads step S of `from` into `then` and requests loads FIRST .. LAST - 1 of the aimed stage
    auto phase = [&](auto sc, auto reads, auto first, auto last, const Frag& now, Frag& then, const unsigned char* from) {
        constexpr int READ = decltype(reads)::value, FIRST = decltype(first)::value, COUNT = decltype(last)::value - FIRST;
        split_for<0, MFMAS>([&](auto qc) {
            constexpr int q = decltype(qc)::value;
            if constexpr (READ) {
                constexpr int R0 = q * READS / SPREAD, R1 = (q + 1) * READS / SPREAD;
                split_for<(R0 < READS ? R0 : READS), (R1 < READS ? R1 : READS)>([&](auto r) { read(sc, r, then, from); });
            }
            __builtin_amdgcn_sched_barrier(0);
            acc[q / NT][q % NT] = xe_mfma<F16>(now.x[q / NT], now.y[q % NT], acc[q / NT][q % NT]);
            __builtin_amdgcn_sched_barrier(0);
            split_for<FIRST + q * COUNT / MFMAS, FIRST + (q + 1) * COUNT / MFMAS>([&](auto i) { request(i); });
        });
    };
    constexpr std::integral_constant<int, 0> I0{};
    constexpr std::integral_constant<int, 1> I1{};
    constexpr std::integral_constant<int, 2> I2{};
    constexpr std::integral_constant<int, 3> I3{};
    constexpr std::integral_constant<int, LOADS / 2> MID{};
    constexpr std::integral_constant<int, LOADS> ALL{};

    if (stages > 0) {
        const int ahead = min(ST, stages);
        for (int s = 0; s < ahead; ++s) {
            aim();
            split_for<0, LOADS>([&](auto i) { request(i); });
            next();
        }
        if (stages >= ST) xe_stage_barrier<(ST - 1) * LOADS>();
        else xe_wait_barrier();
        const unsigned char* now = xe_lds;
        split_for<0, READS>([&](auto r) { read(I0, r, f0, now); });
        // the last step of a stage is multiplied behind the barrier that frees its buffer, while the first of the next is read; the stage
        // ST ahead is requested during that and the next step
        phase(I1, I1, I0, I0, f0, f1, now);
        phase(I2, I1, I0, I0, f1, f0, now);
        phase(I3, I1, I0, I0, f0, f1, now);
        const int shrink_at = F16 && a.pairs > 1 ? (k_end - k_begin) * (a.pairs - 1) - 1 : -1;
        auto settle = [&](int s) {
            if constexpr (BLOCKS) {
                if ((s & 3) == 3) {
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            sum[i][j] += acc[i][j];
#pragma unroll
                            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
                        }
                }
            }
            if constexpr (F16) {
                if (s == shrink_at) {                                    // behind the last product of a second term
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            acc[i][j] *= 1.f / 2048.f;
                            if constexpr (BLOCKS) sum[i][j] *= 1.f / 2048.f;
                        }
                }
            }
        };
        auto follow = [&]() { now = now + STAGE == xe_lds + ST * STAGE ? xe_lds : now + STAGE; };
        int s = 0;
        for (; s + ST < stages; ++s) {
            xe_stage_barrier<(ST - 2) * LOADS>();                        // the ST - 2 stages after the next may still be on their way
            follow();
            aim();
            phase(I0, I1, I0, MID, f1, f0, now);
            settle(s);
            phase(I1, I1, MID, ALL, f0, f1, now);
            next();
            phase(I2, I1, I0, I0, f1, f0, now);
            phase(I3, I1, I0, I0, f0, f1, now);
        }
        for (; s + 1 < stages; ++s) {
            xe_wait_barrier();
            follow();
            phase(I0, I1, I0, I0, f1, f0, now);
            settle(s);
            phase(I1, I1, I0, I0, f0, f1, now);
            phase(I2, I1, I0, I0, f1, f0, now);
            phase(I3, I1, I0, I0, f0, f1, now);
        }
        phase(I0, I0, I0, I0, f1, f0, now);
    }
    xe_wait_barrier();                                                   // LDS is free
    if constexpr (BLOCKS) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] += sum[i][j];
    }

    const int mw = m0 + wm * MT * 32 + 4 * half, nw = n0 + wn * NT * 32 + l32;      // entry e of (i, j): m = mw + 32 i + 8 (e / 4) + e % 4
    // exponents of four m from mw + 32 i + 8 q on (the arrays reach to the end of the last tile)
    auto exps_of = [&](int i, int q) { return *reinterpret_cast<const int4*>(a.exp_m + mw + 32 * i + 8 * q); };
    if constexpr (F16) {
        const int top = a.exp_top ? *a.exp_top : 0;
        int en[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) en[j] = top + (a.exp_n && nw + 32 * j < count ? a.exp_n[nw + 32 * j] : 0);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int4 em = a.exp_m ? exps_of(i, q) : make_int4(0, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    acc[i][j][4 * q] = __builtin_ldexpf(acc[i][j][4 * q], en[j] + em.x);
                    acc[i][j][4 * q + 1] = __builtin_ldexpf(acc[i][j][4 * q + 1], en[j] + em.y);
                    acc[i][j][4 * q + 2] = __builtin_ldexpf(acc[i][j][4 * q + 2], en[j] + em.z);
                    acc[i][j][4 * q + 3] = __builtin_ldexpf(acc[i][j][4 * q + 3], en[j] + em.w);
                }
            }
    }
    if constexpr (END == kXeStats) {
        xe_stats_end<WGM, MT, NT, BN>(a, acc, m0, n0, wm, wn, lane, count);
    } else if constexpr (END == kXeU) {
        constexpr int PER = BM / 8;                                      // 16-byte pieces of an LDS row
        static_assert(BN * BM * 2 <= ST * STAGE, "the tile of U in one go");
        const bool inside = m0 + BM <= a.M;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = nw + 32 * j;
            const bool real = n < count;
            const float lse = real ? a.lse[n] : 0.f, g = real ? a.g[n] : 0.f;
            const int hit = real ? a.label[n] - a.first_word - mw : -1;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int m = 32 * i + 8 * (e / 4) + e % 4;
                    float u = xe_exp(acc[i][j][e] - lse);
                    if (hit == m) u -= 1.f;
                    u *= g;
                    acc[i][j][e] = real && (inside || mw + m < a.M) ? u : 0.f;
                }
        }
        // the tile of one term: to LDS by columns of m, to memory by rows of n.  term_of(x, i, j, q): its bits of the four values x
        auto pass_on = [&](bf16_t* to, auto term_of) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int4 em = F16 ? exps_of(i, q) : make_int4(0, 0, 0, 0);
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        const int row = wn * NT * 32 + 32 * j + l32;
                        float x[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = acc[i][j][4 * q + e];
                        const uint2 w = term_of(x, em, j);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = x[e];
                        const int piece = (wm * MT * 32 + 32 * i + 8 * q) / 8;
                        *reinterpret_cast<uint2*>(xe_lds + row * (BM * 2) + ((piece ^ (row & 15)) << 4) + 8 * half) = w;
                    }
                }
            __syncthreads();
            to += m0;
            for (int c = tid; c < BN * PER; c += WAVES * 64) {
                const int row = c / PER, piece = c % PER;
                *reinterpret_cast<sp_u32x4*>(to + (int64_t)(n0 + row) * a.ldu + piece * 8) =
                    *reinterpret_cast<const sp_u32x4*>(xe_lds + row * (BM * 2) + ((piece ^ (row & 15)) << 4));
                // dW takes whole stages of 64 rows
                if constexpr (BN == 32) *reinterpret_cast<sp_u32x4*>(to + (int64_t)(n0 + 32 + row) * a.ldu + piece * 8) = sp_u32x4{0u, 0u, 0u, 0u};
            }
            __syncthreads();
        };
        if constexpr (F16) {
            if (a.u16_terms > 0) {
                int en[NT];
#pragma unroll
                for (int j = 0; j < NT; ++j) en[j] = nw + 32 * j < count ? -a.exp_g[nw + 32 * j] - *a.exp_words : 0;
                for (int term = 0; term < a.u16_terms; ++term)
                    pass_on(a.u16 + term * a.u_plane, [&](float(&x)[4], int4 em, int j) {
                        float y[4] = {__builtin_ldexpf(x[0], en[j] + em.x), __builtin_ldexpf(x[1], en[j] + em.y), __builtin_ldexpf(x[2], en[j] + em.z),
                                      __builtin_ldexpf(x[3], en[j] + em.w)};
                        const uint2 h = xe_half4(y);
                        return term == 0 ? h : xe_half4(y);
                    });
            }
        }
        for (int term = 0; term < a.u_terms; ++term) pass_on(a.u + term * a.u_plane, [](float(&x)[4], int4, int) { return xe_bf4(x); });
    } else {
        // rows of n, as many 32-row blocks of every wavefront at a time as LDS holds in fp32
        constexpr int FIT = ST * STAGE / (WGN * 32 * BM * 4), JR = FIT < NT ? FIT : NT;
        static_assert(FIT >= 1 && NT % JR == 0, "whole rounds");
        constexpr int PER = BM / 4;
        const int n_most = a.n_is_rows ? min(a.N, count) : a.N;
        Out* const out = reinterpret_cast<Out*>(a.out) + split * a.out_plane;
        const float factor = a.factor ? *a.factor : 1.f;
        const float* const add = a.add ? a.add + split * a.out_plane : nullptr;
#pragma unroll
        for (int j0 = 0; j0 < NT; j0 += JR) {
            if (j0 > 0) __syncthreads();
#pragma unroll
            for (int jj = 0; jj < JR; ++jj) {
                const int row = (wn * JR + jj) * 32 + l32;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int piece = (wm * MT * 32 + 32 * i + 8 * q) / 4 + half;
                        f32x4 v;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = acc[i][j0 + jj][4 * q + e];
                        *reinterpret_cast<f32x4*>(xe_lds + row * (BM * 4) + ((piece ^ (row & 15)) << 4)) = v;
                    }
            }
            __syncthreads();
            // eight m a thread: two pieces of LDS, 16 bytes of bf16 or 32 of fp32
            for (int c = tid; c < WGN * JR * 32 * (PER / 2); c += WAVES * 64) {
                const int row = c / (PER / 2), p8 = c % (PER / 2);
                const int n = n0 + (row / (JR * 32)) * NT * 32 + j0 * 32 + row % (JR * 32), m = m0 + 8 * p8;
                if (n >= n_most || m >= a.M) continue;
                f32x4 lo = *reinterpret_cast<const f32x4*>(xe_lds + row * (BM * 4) + (((2 * p8) ^ (row & 15)) << 4));
                f32x4 hi = *reinterpret_cast<const f32x4*>(xe_lds + row * (BM * 4) + (((2 * p8 + 1) ^ (row & 15)) << 4));
                lo *= factor;
                hi *= factor;
                if (add) {
                    const float* p = add + (int64_t)n * a.ld_add + m;    // (rows of the accumulators are whole multiples of 8)
                    lo += *reinterpret_cast<const f32x4*>(p);
                    hi += *reinterpret_cast<const f32x4*>(p + 4);
                }
                Out* const o = out + (int64_t)(a.row_map ? a.row_map[n] : n) * a.ldo + m;
                if (m + 8 <= a.M) {                                      // (at the elements' own alignment)
                    if constexpr (sizeof(Out) == 4) {
                        *reinterpret_cast<sp_f32x4u*>(o) = lo;
                        *reinterpret_cast<sp_f32x4u*>(o + 4) = hi;
                    } else {
                        *reinterpret_cast<xe_u32x4u*>(o) = xe_u32x4u{cvt_pk_bf16(lo[0], lo[1]), cvt_pk_bf16(lo[2], lo[3]), cvt_pk_bf16(hi[0], hi[1]), cvt_pk_bf16(hi[2], hi[3])};
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (m + e < a.M) {
                            const float v = e < 4 ? lo[e & 3] : hi[e & 3];
                            if constexpr (sizeof(Out) == 4) o[e] = v;
                            else o[e] = f32_to_bf16(v);
                        }
                }
            }
        }
    }
}

// Scores of up to 64 rows with W in fp32 as it is: W goes to LDS raw and is split into three bf16 terms on its way to the matrix cores
// (exact; six products with fp32 features, three with bf16 ones), so that it crosses memory once.  By the general way its terms are
// written and read again.  128 words a workgroup, a stage of 64 k with all of the features' terms; two
// stages, so that two workgroups fit a compute unit (65536 x 4096, one row of bf16: 190 us, 5.7 TB/s; its terms packed first 607), three where only
// one fits anyway (fp32 features: 200; packed 700).  The leading products and the others have sums of their own, the former in blocks of 256 k.
// LDS rows of W: 256 bytes, 16-byte piece p of row r at p ^ (r & 15).
// ANY: rows of W at any 4-byte place and of any length.  They come through registers, two stages ahead, since LDS-DMA wants whole pieces at
// 16-byte places; what lies behind a row is not read (65536 x 4096, rows 4097 apart: one row of bf16 199 us, 64 of fp32 289; their terms packed
// first 607 and 733).
constexpr int kXeRawWords = 128;
template <int NT, int TERMS, bool ANY> constexpr int kXeRawStages = TERMS == 3 && NT == 1 && !ANY ? 3 : 2;

template <int NT, int TERMS, bool ANY>
__global__ __launch_bounds__(256, ANY && TERMS == 1 ? 2 : 1) void xent_raw_scores_kernel(const XentProduct a) {
    constexpr int X_BYTES = kXeRawWords * 256, Y_BYTES = NT * 32 * 128, STAGE = X_BYTES + TERMS * Y_BYTES, LOADS = 8 + TERMS * NT, ST = kXeRawStages<NT, TERMS, ANY>;
    extern __shared__ __attribute__((aligned(16))) unsigned char xe_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5, m0 = blockIdx.x * kXeRawWords, count = *a.count;
    if (count == 0) return;
    const float* const W = reinterpret_cast<const float*>(a.x) + (int64_t)m0 * a.ldx;
    const int in16 = wave * 4 + (lane >> 4);                             // 16 rows of W an access of the four wavefronts
    uint32_t y_off[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
        y_off[i] = (uint32_t)((i * 4 + wave) * 8 + (lane >> 3)) * (uint32_t)a.ldy * 2u + (uint32_t)(((lane & 7) ^ ((lane >> 3) & 7) ^ (wave & 1)) * 16);
    const uint32_t lds0 = xe_lds_address(xe_lds);
    const int stages = a.k_tiles;
    auto request_y = [&](int s, int k) __attribute__((always_inline)) {
        const uint32_t to = lds0 + (s % ST) * STAGE + X_BYTES;
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            const bf16_t* const y = a.y + t * a.y_plane + (k == stages - 1 ? a.last_y : k * kXeK);
#pragma unroll
            for (int i = 0; i < NT; ++i) xe_dma(y, y_off[i], to + t * Y_BYTES + (i * 4 + wave) * 1024);
        }
    };
    f32x16 acc[1][NT], sum[NT], small[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[0][j][e] = sum[j][e] = small[j][e] = 0.f;
    // the products of stage s, which is in LDS
    auto multiply = [&](int s) __attribute__((always_inline)) {
        const unsigned char* const now = xe_lds + (s % ST) * STAGE;
        const unsigned char* const w_row = now + (wave * 32 + l32) * 256;
        split_for<0, 4>([&](auto sc) {
            constexpr int ks = decltype(sc)::value;
            f32x4 v[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) v[q] = *reinterpret_cast<const f32x4*>(w_row + (((4 * ks + 2 * half + q) ^ (l32 & 15)) << 4));
            sp_u32x4 w[3];
#pragma unroll
            for (int t = 0; t < 3; ++t)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float x[4] = {v[q][0], v[q][1], v[q][2], v[q][3]};
                    const uint2 b = xe_bf4(x);
                    w[t][2 * q] = b.x;
                    w[t][2 * q + 1] = b.y;
                    v[q] = f32x4{x[0], x[1], x[2], x[3]};
                }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                sp_u32x4 y[TERMS];
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
                    y[t] = *reinterpret_cast<const sp_u32x4*>(now + X_BYTES + t * Y_BYTES + (j * 32 + l32) * 128 +
                                                              (((2 * ks + half) ^ (l32 & 7) ^ ((l32 >> 3) & 1)) << 4));
                small[j] = split_mfma(w[2], y[0], small[j]);
                if constexpr (TERMS == 3) {
                    small[j] = split_mfma(w[0], y[2], small[j]);
                    small[j] = split_mfma(w[1], y[1], small[j]);
                    small[j] = split_mfma(w[0], y[1], small[j]);
                }
                small[j] = split_mfma(w[1], y[0], small[j]);
                acc[0][j] = split_mfma(w[0], y[0], acc[0][j]);
            }
        });
        if ((s & 3) == 3) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                sum[j] += acc[0][j];
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[0][j][e] = 0.f;
            }
        }
    };
    if constexpr (ANY) {
        const int k = 4 * (lane & 15), features = a.x_cols, full = stages - 1;
        const float* row[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) row[i] = W + (int64_t)(min(m0 + i * 16 + in16, a.x_rows - 1) - m0) * a.ldx + k;
        f32x4 even[8], odd[8];                                           // stages on their way
        auto load = [&](int s, f32x4 (&w)[8]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const sp_f32x4u*>(row[i] + s * kXeK);
        };
        auto put = [&](int s, const f32x4 (&w)[8]) __attribute__((always_inline)) {
            unsigned char* const to = xe_lds + (s % ST) * STAGE;
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<f32x4*>(to + (i * 16 + in16) * 256 + (((lane & 15) ^ in16) << 4)) = w[i];
        };
        // The eight loads of stage s + 1 were requested after stage s and its features: eight on their way leave nothing of that.  A stage's buffer is
        // free at the barrier: everybody is through with the stage before
        auto step = [&](int s, f32x4 (&w)[8]) __attribute__((always_inline)) {
            put(s, w);
            xe_stage_barrier<8>();
            request_y(s + 1, s + 1);
            load(s + 2, w);
            asm volatile("" ::: "memory");                               // (the loads stay in front)
            multiply(s);
        };
        request_y(0, 0);
        int s = 0;
        if (full > 3) {                                                  // (no branch among the loads: waits are counted)
            load(0, even);
            asm volatile("" ::: "memory");                               // in this order
            load(1, odd);
            do {
                step(s, even);
                step(s + 1, odd);
                s += 2;
            } while (s + 3 < full);
        } else {
            if (full > 0) load(0, even);
            if (full > 1) load(1, odd);
        }
        for (; s < full; ++s) {                                          // the last three at most
            put(s, even);
            xe_wait_barrier();
            request_y(s + 1, s + 1);
            multiply(s);
#pragma unroll
            for (int i = 0; i < 8; ++i) even[i] = odd[i];
            if (s + 2 < full) load(s + 2, odd);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)                                      // a row may end anywhere in the last stage
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = full * kXeK + e, inside = min(at + k, features - 1) - k;
                even[i][e] = row[i][inside];
                if (at + k >= features) even[i][e] = 0.f;
            }
        put(full, even);
        xe_wait_barrier();
        multiply(full);
    } else {
        uint32_t x_off[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x_off[i] = (uint32_t)(min(m0 + i * 16 + in16, a.x_rows - 1) - m0) * (uint32_t)a.ldx * 4u + (uint32_t)(((lane & 15) ^ in16) * 16);
        // Every workgroup begins a stage on from its neighbour and goes round: rows 2^14 bytes apart are on the same few memory channels where all
        // workgroups read the same columns (65536 x 4096, one row of bf16 242 -> 190 us, of fp32 301 -> 200; 32768 x 4096 163 -> 110)
        const int turn = (int)(blockIdx.x % (unsigned)stages);
        auto request = [&](int s) {
            const int k = s + turn < stages ? s + turn : s + turn - stages;
            const uint32_t to = lds0 + (s % ST) * STAGE;
            const float* const x = W + (k == stages - 1 ? a.last_x : k * kXeK);
#pragma unroll
            for (int i = 0; i < 8; ++i) xe_dma(x, x_off[i], to + (i * 4 + wave) * 1024);
            request_y(s, k);
        };
        for (int s = 0; s < min(ST - 1, stages); ++s) request(s);
        for (int s = 0; s < stages; ++s) {
            if (s + 1 < stages) xe_stage_barrier<(ST - 2) * LOADS>();    // this stage is there, the next of three may be on its way
            else xe_wait_barrier();
            if (s + ST - 1 < stages) request(s + ST - 1);                // into the buffer that everybody is through with
            multiply(s);
        }
    }
    xe_wait_barrier();
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[0][j] += sum[j] + small[j];
    if (a.out) {                                                         // rows are padded to whole tiles
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            float* const z = reinterpret_cast<float*>(a.out) + (int64_t)(32 * j + l32) * a.ldo + m0 + wave * 32 + 4 * half;
            if (32 * j + l32 < count)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4*>(z + 8 * q) = f32x4{acc[0][j][4 * q], acc[0][j][4 * q + 1], acc[0][j][4 * q + 2], acc[0][j][4 * q + 3]};
        }
        return;
    }
    xe_stats_end<4, 1, NT, NT * 32>(a, acc, m0, 0, wave, 0, lane, count);
}

// dA of up to 64 rows with W in fp32 as it is, so that W's terms are never written: out[n][d] += sum_j U[n][j] W[j][d], U in its bf16 terms, W split into
// terms in registers.  A wavefront has 128 d and all rows; a lane loads four d of a word at once, at any 4-byte place, and they belong to four
// tiles of the matrix cores: tile c has d0 + 4 r + c for r = 0 .. 31, so that a lane also stores four d at once.  A row's last lanes load its last four
// d again, and store what is their own.  Words go through registers, 32 ahead, U through LDS, 64 words a stage.  Blocks of 32 words are added up by
// themselves.  MOST: pairs of terms whose numbers add up to so much at most.  65536 x 4096, 24 rows: 186 us, 5.8 TB/s; 64 of fp32 260.  (From terms
// written before, 91 and 277, but writing them takes 400.)
constexpr int kXeRawFeatures = 512;                                      // of a workgroup
template <int NT, int MOST>
__global__ __launch_bounds__(256, 1) void xent_raw_features_kernel(const XentProduct a) {
    constexpr int TERMS = MOST + 1, Y_BYTES = NT * 32 * 128, STAGE = TERMS * Y_BYTES;
    extern __shared__ __attribute__((aligned(16))) unsigned char xe_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5, count = *a.count;
    if (count == 0) return;
    const int split = blockIdx.x / a.m_tiles, d0 = (blockIdx.x % a.m_tiles) * kXeRawFeatures + wave * 128;
    const int k_begin = min(split * a.per_split, a.k_tiles), k_end = min(k_begin + a.per_split, a.k_tiles);
    const float* const W = reinterpret_cast<const float*>(a.x) + min(d0 + 4 * l32, a.M - 4);
    uint32_t y_off[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
        y_off[i] = (uint32_t)((i * 4 + wave) * 8 + (lane >> 3)) * (uint32_t)a.ldy * 2u + (uint32_t)(((lane & 7) ^ ((lane >> 3) & 7) ^ (wave & 1)) * 16);
    const uint32_t lds0 = xe_lds_address(xe_lds);
    auto request_y = [&](int s) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
#pragma unroll
            for (int i = 0; i < NT; ++i)
                xe_dma(a.y + t * a.y_plane + (int64_t)s * kXeK, y_off[i], lds0 + (s & 1) * STAGE + t * Y_BYTES + (i * 4 + wave) * 1024);
    };
    f32x16 acc[4][NT];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[c][j][e] = 0.f;
    f32x4 first[16], second[16];                                         // the halves of a stage, on their way
    auto load = [&](int s, int h, f32x4 (&w)[16]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int j = min(s * kXeK + 32 * h + 16 * (i >> 3) + 8 * half + (i & 7), a.x_rows - 1);   // (U is 0 from there on)
            w[i] = *reinterpret_cast<const sp_f32x4u*>(W + (int64_t)j * a.ldx);
        }
    };
    auto multiply = [&](int s, int h, const f32x4 (&w)[16]) __attribute__((always_inline)) {
        const unsigned char* const now = xe_lds + (s & 1) * STAGE;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            sp_u32x4 x[2][TERMS];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float v[4] = {w[8 * i + 4 * q][c], w[8 * i + 4 * q + 1][c], w[8 * i + 4 * q + 2][c], w[8 * i + 4 * q + 3][c]};
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) {
                        const uint2 b = xe_bf4(v);
                        x[i][t][2 * q] = b.x;
                        x[i][t][2 * q + 1] = b.y;
                    }
                }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                sp_u32x4 y[2][TERMS];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t)
                        y[i][t] = *reinterpret_cast<const sp_u32x4*>(now + t * Y_BYTES + (j * 32 + l32) * 128 +
                                                                     (((4 * h + 2 * i + half) ^ (l32 & 7) ^ ((l32 >> 3) & 1)) << 4));
                f32x16 block;
#pragma unroll
                for (int e = 0; e < 16; ++e) block[e] = 0.f;
#pragma unroll
                for (int sum = MOST; sum >= 0; --sum)
#pragma unroll
                    for (int t = 0; t <= sum; ++t)
#pragma unroll
                        for (int i = 0; i < 2; ++i) block = split_mfma(x[i][t], y[i][sum - t], block);
                acc[c][j] += block;
            }
        }
    };
    if (k_begin < k_end) {
        request_y(k_begin);
        __builtin_amdgcn_sched_barrier(0);
        load(k_begin, 0, first);
        for (int s = k_begin; s < k_end; ++s) {
            __builtin_amdgcn_sched_barrier(0);
            xe_stage_barrier<16>();                                      // U of this stage was requested before the sixteen loads on their way
            if (s + 1 < k_end) request_y(s + 1);                         // into the buffer that everybody is through with
            load(s, 1, second);
            __builtin_amdgcn_sched_barrier(0);                           // (nothing that waits goes in front of the loads)
            multiply(s, 0, first);
            __builtin_amdgcn_sched_barrier(0);
            load(s + 1, 0, first);
            __builtin_amdgcn_sched_barrier(0);
            multiply(s, 1, second);
        }
    }
    float* const out = reinterpret_cast<float*>(a.out) + split * a.out_plane;
    const float* const add = a.add ? a.add + split * a.out_plane : nullptr;
    const float factor = *a.factor;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = 32 * j + l32;
        if (n >= min(a.N, count)) continue;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int d = d0 + 4 * (8 * (e / 4) + 4 * half + e % 4), base = min(d, a.M - 4);
            if (d >= a.M) continue;
            f32x4 v = f32x4{acc[0][j][e], acc[1][j][e], acc[2][j][e], acc[3][j][e]} * factor;
            float* const o = out + (int64_t)n * a.ldo + base;
            if (base == d) {                                             // (rows of the accumulators are whole multiples of 8)
                if (add) v += *reinterpret_cast<const f32x4*>(add + (int64_t)n * a.ld_add + d);
                *reinterpret_cast<f32x4*>(o) = v;
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (base + c >= d) o[c] = v[c] + (add ? add[(int64_t)n * a.ld_add + base + c] : 0.f);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------
// What stands around the products

constexpr int kXeFewRows = 1024;   // up to so many every workgroup that packs finds the rows that take part by itself

struct XentPack {
    const void* a;
    int64_t lda;
    int n, J, D, n_padded;
    const int32_t* y;
    const float* weight;
    float scale;
    int mean;
    int *rows, *label, *exp_g, *count;       // what the later kernels read
    float *g, *lse_packed, *factor;          // g: the rows' weights; factor: scale, or scale / count
    const float* lse_given;                  // or nullptr
    bf16_t *to, *to16;                       // bf16 and fp16 terms, [terms][n_padded][ld]
    int64_t ld, plane, ld16, plane16;
    int terms, terms16, window;
    int* exps;
    void* zero;                              // dA, loss, lse of the rows that take no part; or nullptr
    int64_t ld_zero;
    float *loss, *lse;
};

// The rows that take part in front, in order, then the others; label, weight and its exponent, and a given lse, of each of the former.  All threads of a
// workgroup of 64 `waves`; what is found of row `mine` of the packed order is returned (source row, or -1 behind n), and the count.
__device__ __forceinline__ int xe_find_rows(const XentPack& p, int mine, bool write, int waves, int* found_count) {
    __shared__ int before[16], total, source;
    int taken = 0;                                                       // so far, the same in every thread
    if (threadIdx.x == 0) source = -1;
    const int threads = 64 * waves;
    for (int base = 0; base < p.n; base += threads) {
        const int i = base + (int)threadIdx.x, lab = i < p.n ? p.y[i] : -1;
        const bool real = lab >= 0 && lab < p.J;
        const uint64_t votes = __ballot(real);
        if ((threadIdx.x & 63) == 0) before[threadIdx.x >> 6] = __popcll(votes);
        __syncthreads();
        if (threadIdx.x == 0) {
            int s = taken;
            for (int w = 0; w < waves; ++w) {
                const int c = before[w];
                before[w] = s;
                s += c;
            }
            total = s;
        }
        __syncthreads();
        const int k = before[threadIdx.x >> 6] + __popcll(votes & ((1ull << (threadIdx.x & 63)) - 1ull));
        const int at = real ? k : p.n - 1 - (i - k);                     // i - k rows before this one take no part
        if (i < p.n) {
            if (at == mine) source = i;
            if (write) {
                p.rows[at] = i;
                if (real) {
                    p.label[k] = lab;
                    p.g[k] = p.weight ? p.weight[i] : 1.f;
                    if (p.lse_given) p.lse_packed[k] = p.lse_given[i];
                }
            }
        }
        taken = total;
        __syncthreads();
    }
    if (write) {
        for (int k = threadIdx.x; k < taken; k += threads) {             // (written before the last barrier)
            p.exp_g[k] = (int)(__float_as_uint(p.g[k]) >> 23 & 255u) - 127 - 14;   // |u| <= |g| is below 2^15 of it
        }
        if (threadIdx.x == 0) {
            *p.count = taken;
            *p.factor = p.mean && taken > 0 ? p.scale / (float)taken : p.scale;
        }
    }
    if (p.n == 0) __syncthreads();
    *found_count = taken;
    return source;
}

__global__ __launch_bounds__(1024) void xent_rows_kernel(const XentPack p) {
    int count;
    xe_find_rows(p, -1, true, 16, &count);
}

// A row of D elements by a workgroup of 256 threads, or by a wavefront of it (LANES = 64, rows of up to 2048): the first 4 HELD a thread stay
// in registers between what looks them over and what takes them (long rows of a large W, all on their way at once, are out of the
// caches by then: 10000 x 21504 in fp32 452 us with 16 elements a thread, 371 with 96).
template <class T, int LANES, int HELD = 4>
struct XentRow {
    f32x4 held[HELD];
    const T* row;
    int D, lane;
    __device__ __forceinline__ XentRow(const T* r, int d) : row(r), D(d), lane(threadIdx.x & (LANES - 1)) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) held[i] = load4(row, lane * 4 + 4 * LANES * i, D);
    }
    // f(d, four elements from d on), d < whole; zeros from D on
    template <class F>
    __device__ __forceinline__ void each(int64_t whole, F f) const {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int d = lane * 4 + 4 * LANES * i;
            if (d < whole) f(d, held[i]);
        }
#pragma unroll 4
        for (int d = lane * 4 + 4 * HELD * LANES; d < whole; d += 4 * LANES) f(d, load4(row, d, D));
    }
    // exponent that brings the largest finite magnitude into [2^14, 2^15) (2^-126 for all below)
    __device__ __forceinline__ int exponent() const {
        float top = 0.f;
        each(D, [&](int, f32x4 x) {
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(x[e]) < __builtin_inff() ? fabsf(x[e]) : 0.f);
        });
        top = wave_max(top);
        if constexpr (LANES == 256) {
            __shared__ float part[4];
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
            __syncthreads();
            top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
        }
        return (int)(__float_as_uint(top) >> 23) - 127 - 14;
    }
};
__device__ __forceinline__ void xe_put16(bf16_t* to, int64_t plane, int terms, f32x4 v, int e0) {
    float x[4] = {__builtin_ldexpf(v[0], -e0), __builtin_ldexpf(v[1], -e0), __builtin_ldexpf(v[2], -e0), __builtin_ldexpf(v[3], -e0)};
    for (int t = 0; t < terms; ++t) *reinterpret_cast<uint2*>(to + t * plane) = xe_half4(x);
}
__device__ __forceinline__ void xe_put(bf16_t* to, int64_t plane, int terms, f32x4 v) {
    float x[4] = {v[0], v[1], v[2], v[3]};
    for (int t = 0; t < terms; ++t) *reinterpret_cast<uint2*>(to + t * plane) = xe_bf4(x);
}

// Packed row k of the features: bf16 terms and fp16 terms (divided by 2^exps[k]), zeros to whole stages and for rows behind those that take part; a
// row that takes none gets its results' zeros here.  window: one stage more of the bf16 terms that repeats the last 64 columns, with zeros where
// they are in the stage before: it meets W's last 64 columns where W is read as it is.
template <class T>
__device__ __forceinline__ void xe_pack_row(const XentPack& p, int k) {
    const int tid = threadIdx.x;
    int real, i;
    if (p.n <= kXeFewRows) {
        i = xe_find_rows(p, k, k == 0, 4, &real);
    } else {
        real = *p.count;
        i = k < p.n ? p.rows[k] : -1;
    }
    bf16_t* const to = p.to + (int64_t)k * p.ld;
    bf16_t* const to16 = p.to16 + (int64_t)k * p.ld16;
    if (k >= real) {
        const f32x4 none{0.f, 0.f, 0.f, 0.f};
        for (int d = tid * 4; d < p.ld; d += 1024) xe_put(to + d, p.plane, p.terms, none);
        for (int d = tid * 4; d < p.ld16; d += 1024) xe_put(to16 + d, p.plane16, p.terms16, none);
        if (p.terms16 && tid == 0) p.exps[k] = 0;
        if (k >= p.n) return;
        if (p.zero)
            for (int d = tid; d < p.D; d += 256) ((T*)p.zero)[(int64_t)i * p.ld_zero + d] = T(0);
        if (tid == 0 && p.loss) p.loss[i] = 0.f;
        if (tid == 0 && p.lse) p.lse[i] = 0.f;
        return;
    }
    const T* const src = (const T*)p.a + (int64_t)i * p.lda;
    const XentRow<T, 256> row(src, p.D);
    int e0 = 0;
    if (p.terms16) {
        e0 = row.exponent();
        if (tid == 0) p.exps[k] = e0;
    }
    row.each(p.window ? p.window : p.terms ? p.ld : p.ld16, [&](int d, f32x4 v) {
        xe_put16(to16 + d, p.plane16, p.terms16, v, e0);
        xe_put(to + d, p.plane, p.terms, v);
    });
    if (p.window && tid < 16) {
        const int d = p.D - 64 + tid * 4;                                // D is a multiple of 4 here
        f32x4 v = load4(src, d, p.D);
        if (d < p.window - 64) v = f32x4{0.f, 0.f, 0.f, 0.f};
        xe_put(to + p.window + tid * 4, p.plane, p.terms, v);
    }
}

struct XentWords {
    const void* w;
    int64_t ld;
    int D, n;
    bf16_t* to;
    int64_t ldd, plane;
    int terms;
    int* exps;
};
// Row k of W's piece in one bf16 term or (F16) fp16 terms and its exponent; zeros to whole stages and for rows from n on.
template <class T, bool F16, int LANES, int HELD>
__device__ __forceinline__ void xe_pack_word(const XentWords& p, int k) {
    bf16_t* const out = p.to + (int64_t)k * p.ldd;
    const int lane = threadIdx.x & (LANES - 1);
    if (k >= p.n) {
        for (int d = lane * 4; d < p.ldd; d += 4 * LANES) xe_put(out + d, p.plane, p.terms, f32x4{0.f, 0.f, 0.f, 0.f});
        if (F16 && lane == 0) p.exps[k] = -200;                          // below any other: has no say in the largest
        return;
    }
    const XentRow<T, LANES, HELD> row((const T*)p.w + (int64_t)k * p.ld, p.D);
    if constexpr (F16) {
        const int e0 = row.exponent();
        if (lane == 0) p.exps[k] = e0;
        row.each(p.ldd, [&](int d, f32x4 v) { xe_put16(out + d, p.plane, p.terms, v, e0); });
    } else {
        row.each(p.ldd, [&](int d, f32x4 v) { xe_put(out + d, p.plane, 1, v); });
    }
}
// Workgroup b's rows: four short ones (a wavefront each) or one.  The rows are padded to whole multiples of 64.
constexpr int kXeShortRow = 2048, kXeLongRow = 4096;
template <class T, bool F16, bool LONG>
__device__ __forceinline__ void xe_pack_words(const XentWords& p, int b) {
    if constexpr (LONG) xe_pack_word<T, F16, 256, 24>(p, b);
    else if (p.D <= kXeShortRow / 2) xe_pack_word<T, F16, 64, 4>(p, 4 * b + (threadIdx.x >> 6));
    else if (p.D <= kXeShortRow) xe_pack_word<T, F16, 64, 8>(p, 4 * b + (threadIdx.x >> 6));
    else xe_pack_word<T, F16, 256, 4>(p, b);
}

template <class T>
__global__ __launch_bounds__(256) void xent_pack_rows_kernel(const XentPack p) { xe_pack_row<T>(p, blockIdx.x); }
template <class T, bool F16, bool LONG>
__global__ __launch_bounds__(256) void xent_pack_words_kernel(const XentWords w) { xe_pack_words<T, F16, LONG>(w, blockIdx.x); }
// The rows and the first piece's words in one launch
template <class TA, class TW, bool F16, bool LONG>
__global__ __launch_bounds__(256) void xent_pack_both_kernel(const XentPack p, const XentWords w) {
    if ((int)blockIdx.x < p.n_padded) xe_pack_row<TA>(p, blockIdx.x);
    else xe_pack_words<TW, F16, LONG>(w, (int)blockIdx.x - p.n_padded);
}
template <bool LONG>
static void launch_pack_words(const XentWords& w, bool w_bf16, bool f16, uint32_t groups, hipStream_t s) {
    if (!f16) hipLaunchKernelGGL((xent_pack_words_kernel<bf16_t, false, LONG>), dim3(groups), dim3(256), 0, s, w);
    else if (w_bf16) hipLaunchKernelGGL((xent_pack_words_kernel<bf16_t, true, LONG>), dim3(groups), dim3(256), 0, s, w);
    else hipLaunchKernelGGL((xent_pack_words_kernel<float, true, LONG>), dim3(groups), dim3(256), 0, s, w);
}
template <bool LONG>
static void launch_pack_both(const XentPack& p, const XentWords& w, bool a_bf16, bool w_bf16, uint32_t groups, hipStream_t s) {
    const dim3 grid((uint32_t)p.n_padded + groups), block(256);
    if (a_bf16 && w_bf16) hipLaunchKernelGGL((xent_pack_both_kernel<bf16_t, bf16_t, false, LONG>), grid, block, 0, s, p, w);
    else if (w_bf16) hipLaunchKernelGGL((xent_pack_both_kernel<float, bf16_t, true, LONG>), grid, block, 0, s, p, w);
    else if (a_bf16) hipLaunchKernelGGL((xent_pack_both_kernel<bf16_t, float, true, LONG>), grid, block, 0, s, p, w);
    else hipLaunchKernelGGL((xent_pack_both_kernel<float, float, true, LONG>), grid, block, 0, s, p, w);
}

// The largest of a piece's exponents
__global__ __launch_bounds__(1024) void xent_top_kernel(const int* __restrict__ exps, int n, int* __restrict__ top) {
    __shared__ int part[16];
    int m = -200;
    for (int i = threadIdx.x; i < n; i += 8192)                          // eight on their way at a time
#pragma unroll
        for (int k = 0; k < 8; ++k) m = max(m, exps[min(i + 1024 * k, n - 1)]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, __shfl_xor(m, o, kWave));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) m = max(m, part[w]);
        *top = m;
    }
}

struct XentRows {
    const float* z;                          // [splits][..][ldz] scores of all words
    int64_t ldz, z_plane;
    int splits, words;
    int first, columns;                      // U's words: from `first` on, `columns` of them with the padding of its rows (0: none)
    const int *rows, *label, *count;
    const float* g;
    float *loss, *lse;
    float* loss_packed;
    float* lse_packed;
    bf16_t *u, *u16;
    int64_t ldu, u_plane;
    int u_terms, u16_terms;
    const int *exp_m, *exp_g;                // of all words; of the rows
    int* exp_words;                          // out: the largest of exp_m
    bool given;                              // lse_packed is there already
};
constexpr int kXeRowThreads = 512;

// Kept scores: a workgroup a row, loss and a piece of U from one row of scores (read again for U: it is in the die's cache by then)
__global__ __launch_bounds__(kXeRowThreads) void xent_row_kernel(const XentRows a) {
    __shared__ float red[2][kXeRowThreads / 64], z_label;
    __shared__ int red_exp[kXeRowThreads / 64];
    const int k = blockIdx.x, tid = threadIdx.x, count = *a.count;
    bf16_t* const u = a.u + (int64_t)k * a.ldu;
    bf16_t* const u16 = a.u16 + (int64_t)k * a.ldu;
    if (k >= count) {                                                    // dW takes whole stages of 64 rows
        if (k < (count + 63) / 64 * 64)
            for (int j = tid * 4; j < a.columns; j += kXeRowThreads * 4)
                for (int t = 0; t < a.u_terms; ++t) *reinterpret_cast<uint2*>(u + t * a.u_plane + j) = make_uint2(0u, 0u);
        return;
    }
    const float* const z = a.z + (int64_t)k * a.ldz;
    auto scores = [&](int j) {                                           // four from j on; rows are padded to whole accesses
        f32x4 s = *reinterpret_cast<const f32x4*>(z + j);
        for (int p = 1; p < a.splits; ++p) s += *reinterpret_cast<const f32x4*>(z + p * a.z_plane + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = j + e < a.words ? s[e] : -__builtin_inff();
        return s;
    };
    const int label = a.label[k];
    float lse;
    if (a.given) {
        lse = a.lse_packed[k];
    } else {
        float top = -__builtin_inff(), sum = 0.f;
        for (int j = tid * 4; j < a.words; j += kXeRowThreads * 4) {
            const f32x4 s = scores(j);
            const float m = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), top), base = m == -__builtin_inff() ? 0.f : m;
            sum *= xe_exp(top - base);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum += xe_exp(s[e] - base);
                if (j + e == label) z_label = s[e];
            }
            top = m;
        }
        const float m = wave_max(top);
        sum = wave_sum(sum * xe_exp(top - (m == -__builtin_inff() ? 0.f : m)));
        if ((tid & 63) == 0) {
            red[0][tid >> 6] = m;
            red[1][tid >> 6] = sum;
        }
        __syncthreads();
        float most = red[0][0];
#pragma unroll
        for (int w = 1; w < kXeRowThreads / 64; ++w) most = fmaxf(most, red[0][w]);
        const float base = most == -__builtin_inff() ? 0.f : most;
        sum = 0.f;
#pragma unroll
        for (int w = 0; w < kXeRowThreads / 64; ++w) sum += red[1][w] * xe_exp(red[0][w] - base);
        const float l = logf(sum);
        lse = most + l;
        if (tid == 0) {
            const float f = l + (most - z_label);
            const int i = a.rows[k];
            if (a.lse) a.lse[i] = lse;
            if (a.loss) a.loss[i] = f;
            a.loss_packed[k] = f;
            a.lse_packed[k] = lse;                                       // (for the other pieces)
        }
    }
    if (a.columns == 0) return;
    const float g = a.g[k];
    int en = 0;
    if (a.u16_terms > 0) {                                               // (every row finds it: a word's exponent is a third of its scores' bytes or less)
        int m = -200;
        for (int j = tid; j < a.words; j += kXeRowThreads) m = max(m, a.exp_m[j]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m = max(m, __shfl_xor(m, o, kWave));
        if ((tid & 63) == 0) red_exp[tid >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kXeRowThreads / 64; ++w) m = max(m, red_exp[w]);
        if (k == 0 && tid == 0) *a.exp_words = m;
        en = -a.exp_g[k] - m;
    }
    for (int c = tid * 4; c < a.columns; c += kXeRowThreads * 4) {
        const int j = a.first + c;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (j < a.words) {
            const f32x4 s = scores(j);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = xe_exp(s[e] - lse);
                if (j + e == label) x[e] -= 1.f;
                x[e] = j + e < a.words ? x[e] * g : 0.f;
            }
        }
        if (a.u16_terms > 0) {
            const int4 em = j < a.words ? *reinterpret_cast<const int4*>(a.exp_m + j) : make_int4(0, 0, 0, 0);
            float y[4] = {__builtin_ldexpf(x[0], en + em.x), __builtin_ldexpf(x[1], en + em.y), __builtin_ldexpf(x[2], en + em.z), __builtin_ldexpf(x[3], en + em.w)};
            for (int t = 0; t < a.u16_terms; ++t) *reinterpret_cast<uint2*>(u16 + t * a.u_plane + c) = xe_half4(y);
        }
        for (int t = 0; t < a.u_terms; ++t) *reinterpret_cast<uint2*>(u + t * a.u_plane + c) = xe_bf4(x);
    }
}

// Maximum of a row's scores and sum of their exponentials under it from its tiles', in a fixed order, by a wavefront
__device__ __forceinline__ float2 xe_join(const float2* __restrict__ partial, int tiles, int lane) {
    float top = -__builtin_inff(), sum = 0.f;
    for (int t = lane; t < tiles; t += 512) {                            // eight on their way at a time
        float2 p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = t + 64 * i < tiles ? partial[t + 64 * i] : make_float2(-__builtin_inff(), 0.f);
        float m = top;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, p[i].x);
        const float base = m == -__builtin_inff() ? 0.f : m;
        sum *= xe_exp(top - base);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += p[i].y * xe_exp(p[i].x - base);
        top = m;
    }
    const float most = wave_max(top), base = most == -__builtin_inff() ? 0.f : most;
    return make_float2(most, wave_sum(sum * xe_exp(top - base)));
}

// The same of up to 64 rows that were read where they lie, by one workgroup: row k of the partial sums is row k of the call, and what those
// that take no part left there (it may be NaN) is dropped here.
__global__ __launch_bounds__(1024) void xent_in_place_loss_kernel(const XentPack p, const float2* __restrict__ partial, int tiles, int ld_partial,
                                                                  const float* __restrict__ z_label, float* __restrict__ loss, float* __restrict__ lse,
                                                                  float* __restrict__ total) {
    __shared__ float found[64];
    const int lane = threadIdx.x & 63;
    for (int k = threadIdx.x >> 6; k < p.n; k += 16) {
        const int label = p.y[k];
        const bool real = label >= 0 && label < p.J;
        const float2 s = xe_join(partial + (int64_t)k * ld_partial, tiles, lane);
        if (lane == 0) {
            const float l = logf(s.y), f = real ? l + (s.x - z_label[k]) : 0.f;
            if (lse) lse[k] = real ? s.x + l : 0.f;
            if (loss) loss[k] = f;
            found[k] = f;
        }
    }
    __syncthreads();
    if (!total || threadIdx.x >= 64) return;
    const int label = lane < p.n ? p.y[lane] : -1;
    const bool real = label >= 0 && label < p.J;
    const int count = __popcll(__ballot(real));
    double s = real ? (double)found[lane] * (double)(p.weight ? p.weight[lane] : 1.f) : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
    if (lane == 0) *total = (float)(s * (double)(p.mean && count > 0 ? p.scale / (float)count : p.scale));
}

// lse and loss of a row from its tiles' maxima and sums: a wavefront a row, tiles in a fixed order.  One workgroup alone adds up the total
// as well (total not null).
__global__ __launch_bounds__(1024) void xent_loss_kernel(const float2* __restrict__ partial, int tiles, int ld_partial, const int* __restrict__ rows,
                                                         const int* __restrict__ counted, const float* __restrict__ z_label, const float* __restrict__ g,
                                                         float* __restrict__ loss, float* __restrict__ lse, float* lse_packed, float* loss_packed,
                                                         const float* __restrict__ factor, float* __restrict__ total) {
    const int lane = threadIdx.x & 63, count = *counted;
    for (int k = blockIdx.x * 16 + (threadIdx.x >> 6); k < count; k += gridDim.x * 16) {
        const float2 s = xe_join(partial + (int64_t)k * ld_partial, tiles, lane);
        if (lane == 0) {
            const float l = logf(s.y), v = s.x + l, f = l + (s.x - z_label[k]);
            const int i = rows[k];
            if (lse) lse[i] = v;
            if (loss) loss[i] = f;
            lse_packed[k] = v;
            loss_packed[k] = f;
        }
    }
    if (total) {
        __shared__ double part[16];
        __syncthreads();
        xe_total(loss_packed, g, count, factor, total, part);
    }
}

__global__ __launch_bounds__(1024) void xent_total_kernel(const float* __restrict__ loss, const float* __restrict__ g, const int* __restrict__ count,
                                                          const float* __restrict__ factor, float* __restrict__ total) {
    __shared__ double part[16];
    xe_total(loss, g, *count, factor, total, part);
}

// dA's rows from the accumulators' planes
template <class Out>
__global__ __launch_bounds__(256) void xent_rows_out_kernel(const float* __restrict__ acc, int64_t ld, int64_t plane, int planes,
                                                            const int* __restrict__ rows, const int* __restrict__ count, int D, Out* __restrict__ out,
                                                            int64_t ldo) {
    const int per = (D + 3) / 4;
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int k = (int)(c / per), d = (int)(c % per) * 4;
    if (k >= *count) return;
    f32x4 s{0.f, 0.f, 0.f, 0.f};
    const float* const at = acc + (int64_t)k * ld + d;
    for (int p = 0; p < planes; p += 8) {                                // eight on their way at a time
        f32x4 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const f32x4*>(at + min(p + i, planes - 1) * plane);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (p + i < planes) s += x[i];
    }
    store4(out + (int64_t)rows[k] * ldo, d, D, s);
}

// ---------------------------------------------------------------------------------------------------------------
// Plans and launches

template <int WGM, int WGN, int MT, int NT, int ST, int OCC, bool XT, bool YT, bool F16, int END, class Out>
static hipError_t launch_tiles(XentProduct a, hipStream_t s) {
    constexpr int BM = WGM * MT * 32, BN = WGN * NT * 32;
    constexpr size_t lds = (size_t)ST * (BM + BN) * 128;
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    auto* const kernel = &xent_product_kernel<WGM, WGN, MT, NT, ST, OCC, XT, YT, F16, END, Out>;
    if constexpr (lds > 64 * 1024) {
        static std::atomic<uint64_t> raised{0};
        const hipError_t e = raise_lds(kernel, lds, raised);
        if (e != hipSuccess) return e;
    }
    a.m_tiles = (a.M + BM - 1) / BM;
    a.n_tiles = (a.N + BN - 1) / BN;
    a.total = a.m_tiles * a.n_tiles * a.splits;
    a.per_split = (a.k_tiles + a.splits - 1) / a.splits;
    SFB_LAUNCH((xent_product_kernel<WGM, WGN, MT, NT, ST, OCC, XT, YT, F16, END, Out>), dim3(a.total), dim3(WGM * WGN * 64), lds, s, a);
    return hipGetLastError();
}

// Largest dynamic LDS of a kernel beyond 64 KB, told to the runtime once for every GPU.
template <class K>
static hipError_t raise_lds(K* kernel, size_t lds, std::atomic<uint64_t>& raised) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev > 63 || !(raised.load() >> dev & 1)) {
        e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        if (dev <= 63) raised |= 1ull << dev;
    }
    return hipSuccess;
}

template <int NT, int TERMS, bool ANY>
static hipError_t launch_raw_scores(const XentProduct& a, hipStream_t s) {
    constexpr size_t lds = (size_t)kXeRawStages<NT, TERMS, ANY> * (kXeRawWords * 256 + TERMS * NT * 32 * 128);
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    static std::atomic<uint64_t> raised{0};
    const hipError_t e = raise_lds(&xent_raw_scores_kernel<NT, TERMS, ANY>, lds, raised);
    if (e != hipSuccess) return e;
    SFB_LAUNCH((xent_raw_scores_kernel<NT, TERMS, ANY>), dim3((uint32_t)((a.M + kXeRawWords - 1) / kXeRawWords)), dim3(256), lds, s, a);
    return hipGetLastError();
}
template <int NT, int MOST>
static hipError_t launch_raw_features(XentProduct a, hipStream_t s) {
    constexpr size_t lds = 2 * (size_t)(MOST + 1) * NT * 32 * 128;
    static_assert(lds <= 64 * 1024, "without being told to the runtime");
    a.m_tiles = (a.M + kXeRawFeatures - 1) / kXeRawFeatures;
    a.per_split = (a.k_tiles + a.splits - 1) / a.splits;
    SFB_LAUNCH((xent_raw_features_kernel<NT, MOST>), dim3((uint32_t)(a.m_tiles * a.splits)), dim3(256), lds, s, a);
    return hipGetLastError();
}
template <bool ANY>
static hipError_t launch_raw_scores(const XentProduct& a, bool a_bf16, int rows, hipStream_t s) {
    if (a_bf16) return rows > 32 ? launch_raw_scores<2, 1, ANY>(a, s) : launch_raw_scores<1, 1, ANY>(a, s);
    return rows > 32 ? launch_raw_scores<2, 3, ANY>(a, s) : launch_raw_scores<1, 3, ANY>(a, s);
}

// Tiles, m x n; kXe128x128Lone: four stages on their way instead of two, a compute unit to itself.
enum XentTile { kXe256x256, kXe128x128, kXe128x128Lone, kXe256x64, kXe256x32, kXe128x32 };
static const int kXeTileM[] = {256, 128, 128, 256, 256, 128}, kXeTileN[] = {256, 128, 128, 64, 32, 32};

template <bool XT, bool YT, bool F16, int END, class Out>
static hipError_t launch_product(const XentProduct& a, XentTile tile, hipStream_t s) {
    switch (tile) {
        // four wavefronts of 128 x 128 read a third less of LDS than eight of 128 x 64 (16384 x 4096, k 4096: 1174 against 1080 TFLOP/s, W's
        // k slow 1208 against 1125); what U's end and the scaling between fp16 terms take in registers goes with the eight only (U, 4096 x 4096: 1147
        // against 1045)
        case kXe256x256:
            if constexpr (END == kXeU || F16) return launch_tiles<2, 4, 4, 2, 2, 2, XT, YT, F16, END, Out>(a, s);
            else return launch_tiles<2, 2, 4, 4, 2, 1, XT, YT, F16, END, Out>(a, s);
        case kXe128x128: return launch_tiles<2, 2, 2, 2, 2, 2, XT, YT, F16, END, Out>(a, s);
        case kXe128x128Lone: return launch_tiles<2, 2, 2, 2, 4, 1, XT, YT, F16, END, Out>(a, s);
        default: break;
    }
    if constexpr (!YT) {
        if (tile == kXe256x64) return launch_tiles<4, 1, 2, 2, 3, 1, XT, YT, F16, END, Out>(a, s);
        if (tile == kXe256x32) return launch_tiles<4, 1, 2, 1, 4, 1, XT, YT, F16, END, Out>(a, s);
        if (tile == kXe128x32) return launch_tiles<4, 1, 1, 1, 4, 2, XT, YT, F16, END, Out>(a, s);
    }
    return hipErrorInvalidValue;
}

struct Tiling {
    XentTile tile;
    int splits;
};

// Tile and splits of k for an M x N product of `stages` stages (all pairs of terms), by microseconds: a launch's own, a round of workgroups',
// a stage's in a lone workgroup (latency) and on a full card (at whose rate the matrix cores' clock falls), and the way of `out` bytes a result
// to memory, splits (at most `most`) with planes of their own that are read again.  Fitted to 2100 products (D 256 to 20000, J 500 to
// 60000, n 100 to 5000; each within 3 to 5 % for tiles of 256 and lone ones of 128, 8 to 14 % for pairs of them; the choice is within 1.1 % of
// the best measured one on average).  Up to 64 rows take tiles of their own, bound by W's way from memory: 65536 x 4096, 32 rows:
// scores in 128 x 32 113 us, 256 x 32 121; dA (k slow) 100 and 89.
static Tiling tiling_for(int64_t M, int64_t N, int64_t stages, int64_t most, bool rows_are_n, bool k_slow, XentEnd end, double out) {
    static const struct { XentTile tile; int resident; double own_us, round_us[2], lone_us, full_us; } kinds[] = {
        {kXe256x256, 1, 8.0, {11.0, 2.0}, 1.07, 1.58},    {kXe128x128, 2, 4.0, {0.5, 0.0}, 0.64, 0.97}, {kXe128x128Lone, 1, 3.5, {4.0, 1.0}, 0.41, 0.53},
        {kXe256x64, 1, 4.0, {2.0, 1.0}, 0.40, 0.55}, {kXe256x32, 1, 4.0, {2.0, 1.0}, 0.30, 0.45}, {kXe128x32, 2, 4.0, {2.0, 1.0}, 0.30, 0.45}};
    Tiling best{kXe128x128, 1};
    double best_us = 1e300;
    for (const auto& t : kinds) {
        if (rows_are_n && N <= 64) {
            if (t.tile != (N > 32 ? kXe256x64 : k_slow ? kXe256x32 : kXe128x32)) continue;
        } else if (kXeTileN[t.tile] < 128 || (rows_are_n && N <= 128 && kXeTileN[t.tile] > 128)) {
            continue;
        }
        const int64_t tiles = ((M + kXeTileM[t.tile] - 1) / kXeTileM[t.tile]) * ((N + kXeTileN[t.tile] - 1) / kXeTileN[t.tile]);
        const int64_t room = 256 * t.resident;
        for (int64_t s = 1; s <= most && (s == 1 || s * 4 <= stages); ++s) {
            const int64_t n = tiles * s, rest = n % room;
            const double part = t.full_us * (double)rest / (double)room;
            const double stage = t.full_us * (double)(n / room) + (rest == 0 ? 0.0 : part > t.lone_us ? part : t.lone_us);
            const double plane = (double)M * (double)N * 1e-6;
            const double us = t.own_us + t.round_us[end == kXeStore] * (double)((n + room - 1) / room) + (double)((stages + s - 1) / s) * stage +
                              plane * out * (double)s / 4.0 + (s > 1 ? 2.0 + plane * 4.0 * (double)s / 4.0 : 0.0);
            if (us < best_us * 0.999) {
                best_us = us;
                best = Tiling{t.tile, (int)s};
            }
        }
    }
    return best;
}

// Pairs of terms of a product, the small ones first: those whose numbers (0, 1, 2) add up to `most` at most
static int pair_list(int x_terms, int y_terms, int most, uint32_t* px, uint32_t* py) {
    int n = 0;
    *px = *py = 0;
    for (int sum = most; sum >= 0; --sum)
        for (int i = 0; i <= sum; ++i) {
            const int j = sum - i;
            if (i >= x_terms || j >= y_terms) continue;
            *px |= (uint32_t)i << (4 * n);
            *py |= (uint32_t)j << (4 * n);
            ++n;
        }
    return n;
}
static int pair_count(int x_terms, int y_terms, int most) {
    uint32_t x, y;
    return pair_list(x_terms, y_terms, most, &x, &y);
}

namespace {
constexpr int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
constexpr size_t kXePieceBytes = (size_t)512 << 20, kXeScoreBytes = (size_t)256 << 20, kXeWordBytes = (size_t)1 << 30;   // of U, kept scores and W's terms
constexpr size_t kXePackedBytes = (size_t)768 << 20;                     // of a workspace, for the sake of W's terms where W may be read as it is

// What a call does and where it keeps it.
struct Layout {
    int64_t n_padded, piece, ld_k, ld_a, ld_acc, ld_z, ld_partial; // piece: words; ld_k: features to whole stages
    bool f16, direct, kept, raw, raw_any;              // fp16 terms (either operand fp32); W read as it is; scores of all words kept; fp32 W as it
                                                       // is, and at any place
    int k_tiles, window;
    int a_terms, a16_terms, w16_terms, u_terms, u16_terms;
    int score_most, dA_most, dW_most;                  // pairs of terms
    Tiling scores, dA, dW;
    size_t rows, label, g, exp_g, factor, lse, loss, z_label, count, top, exp_a, exp_w, partial, acc, a, a16, w, z, u, u16, bytes;
};
}  // namespace

// Whether fp32 words read as they are give the loss of few rows sooner than their terms do.  Reading them takes a stage's latency after another, its
// workgroups have all of D; terms cost W two more passes at 5.4 TB/s and 4 us, and their product is cut into slices of D.  One row of
// bf16, as they are and as terms: 1000 x 1024 27 us and 16, 1000 x 8192 146 and 41, 4000 x 2048 44 and 34, 8000 x 4096 78 and 78, 16000 x 2048 45
// and 72, 16000 x 8192 164 and 371; 64 rows of fp32: 1000 x 4096 120 and 33, 16000 x 4096 134 and 250, 10000 x 21504 670 and 1104.  The choice
// loses 16 % at most there.
// With gradients terms are written once for scores and dA, and the scores' product is sliced at any number of words: one row of bf16, as they are
// and as terms: 500 x 512 34 and 45 (scores formed twice), 1000 x 4096 100 and 46, 8000 x 8192 297 and 289, 32000 x 512 85 and 95, 65536 x 4096 819 and 1129;
// 64 rows of fp32: 4000 x 2048 114 and 73, 8000 x 8192 435 and 376, 32000 x 2048 287 and 382, 65536 x 4096 1033 and 1516.  It loses a twentieth.
static bool raw_pays(const XentCall& c, bool grads) {
    const double stage_us = c.a_bf16 ? (c.n > 32 ? 1.20 : 1.06) : (c.n > 32 ? 1.63 : 1.23), own_us = stage_us * (double)((c.D + 63) / 64);
    if (grads) {
        if (c.D < 64 || (size_t)64 * up(c.J, 256) * 4 > kXeScoreBytes) return false;
        const double more_us = c.D * (c.a_bf16 ? 2 : 3) < 1500 ? 12.0 : -2.0;
        return own_us <= more_us + (c.a_bf16 ? 1.9e-6 : 2.7e-6) * (double)c.J * (double)c.D;
    }
    if (c.J > 63 * 128) return true;                                     // 64 tiles and more are not sliced
    return own_us <= 4.0 + 2.2e-6 * (double)c.J * (double)c.D;
}

// Rows of W that LDS-DMA takes: pieces of 16 bytes, 32-bit offsets
static bool words_in_pieces(const XentCall& c) {
    const int per = c.w_bf16 ? 8 : 4;
    return c.D >= 64 && c.D % per == 0 && c.ldw % per == 0 && ((uintptr_t)c.W % 16) == 0 && c.ldw < (1 << 22);
}
// Rows of W that a product reads as they are: in bf16 with bf16 features, in pieces; in fp32 for the loss of few rows.
static bool reads_w_directly(const XentCall& c, bool grads) {
    if (c.w_bf16) return c.a_bf16 && words_in_pieces(c);
    return c.n <= 64 && raw_pays(c, grads);
}

// piece: words of a piece, a multiple of 256
static Layout layout_of(const XentCall& c, bool direct, bool grads, bool kept, int64_t piece) {
    Layout l{};
    const int64_t n = c.n > 0 ? c.n : 1, words = piece < c.J ? piece : c.J;
    l.raw = direct && !c.w_bf16;
    l.raw_any = l.raw && !words_in_pieces(c);
    l.f16 = !l.raw && !(c.a_bf16 && c.w_bf16);
    l.direct = direct;
    l.kept = kept;
    l.piece = piece;
    l.n_padded = n <= 64 ? 64 : n <= 128 ? 128 : up(n, 256);             // whole tiles, and whole stages of dW's k
    l.k_tiles = (int)((c.D + 63) / 64);
    l.ld_k = 64 * (int64_t)l.k_tiles;
    l.window = direct && !l.raw_any && c.D % 64 != 0 ? (int)l.ld_k : 0;
    l.ld_a = l.ld_k + (l.window ? 64 : 0);
    l.ld_acc = up(c.D, 8);
    if (l.f16) {
        l.a16_terms = c.a_bf16 ? 1 : 2;
        l.w16_terms = c.w_bf16 ? 1 : 2;
        l.score_most = 1;
        l.dA_most = c.a_bf16 ? 0 : 1;
        l.dW_most = c.w_bf16 ? 1 : 2;
        l.u16_terms = grads ? (c.a_bf16 ? 1 : 2) : 0;
        l.u_terms = grads ? l.dW_most + 1 : 0;
        l.a_terms = grads ? (c.a_bf16 ? 1 : l.dW_most + 1) : 0;
    } else {
        l.a_terms = l.raw && !c.a_bf16 ? 3 : 1;
        l.u_terms = !grads ? 0 : l.raw ? 3 : 1;
        l.dW_most = l.raw ? 2 : 0;
    }
    const int score_pairs = l.f16 ? pair_count(l.w16_terms, l.a16_terms, 1) : 1;
    const int64_t row_tiles = (n + 63) / 64, word_tiles = (words + 63) / 64;
    l.ld_z = up(c.J, 256);
    const int64_t planes = (int64_t)(kXeScoreBytes / ((size_t)l.n_padded * l.ld_z * 4)), slices = !kept || l.raw || planes < 1 ? 1 : planes < 16 ? planes : 16;
    l.scores = tiling_for(words, n, (int64_t)l.k_tiles * score_pairs, slices, true, false,
                          kept ? kXeStore : grads ? kXeU : kXeStats, kept ? 4.0 : 2.0 * (l.u_terms + l.u16_terms));
    if (grads) {
        l.dA = tiling_for(c.D, n, word_tiles * (l.f16 ? pair_count(l.w16_terms, l.u16_terms, l.dA_most) : 1), 64, true, true, kXeStore, 4.0);
        if (l.raw) {                                                     // a workgroup a compute unit
            const int64_t tiles = (c.D + kXeRawFeatures - 1) / kXeRawFeatures;
            l.dA.splits = tiles < 2 ? 128 : tiles < 256 ? (int)(256 / tiles) : 1;
        }
        if (l.dA.splits > word_tiles) l.dA.splits = (int)word_tiles;
        l.dW = tiling_for(c.D, words, row_tiles * pair_count(l.a_terms, l.u_terms, l.dW_most), 1, false, true, kXeStore, c.w_bf16 ? 2.0 : 4.0);
    }
    if (l.scores.splits > l.k_tiles) l.scores.splits = l.k_tiles;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += up(bytes, 256);
        return p;
    };
    l.rows = take((size_t)n * 4);
    l.label = take((size_t)l.n_padded * 4);
    l.g = take((size_t)l.n_padded * 4);
    l.exp_g = take((size_t)l.n_padded * 4);
    l.lse = take((size_t)l.n_padded * 4);
    l.loss = take((size_t)l.n_padded * 4);
    l.z_label = take((size_t)l.n_padded * 4);
    l.count = take(4);
    l.factor = take(4);
    l.top = take(4);
    if (l.f16) {
        l.exp_a = take((size_t)l.n_padded * 4);
        l.exp_w = take((size_t)up(c.J, 256) * 4);
        l.a16 = take((size_t)l.a16_terms * l.n_padded * l.ld_k * 2);
    }
    if (l.a_terms) l.a = take((size_t)l.a_terms * l.n_padded * l.ld_a * 2);
    if (kept) l.z = take((size_t)l.scores.splits * l.n_padded * l.ld_z * 4);
    l.ld_partial = up(c.J, 256) / 128;
    if (!kept) l.partial = take((size_t)l.ld_partial * n * 8);
    if (grads) {
        l.acc = take((size_t)l.dA.splits * n * l.ld_acc * 4);
        l.u = take((size_t)l.u_terms * l.n_padded * piece * 2);
        l.u16 = take((size_t)l.u16_terms * l.n_padded * piece * 2);
    }
    if (!direct) l.w = take((size_t)(l.f16 ? l.w16_terms : 1) * piece * l.ld_k * 2);
    l.bytes = at;
    return l;
}

// Whether a call keeps its scores: they fit, and forming them again (or leaving most compute units idle) would take longer than their
// way to memory and back.  A score costs 2 D flops a pair of terms again, at about 1.1 PFLOP/s, or some 12 bytes at 4 TB/s.
// Measured, kept and not, bf16: both directions, 32 rows, 65536 x 4096: 450 us and 532; 64 rows, 1000 x 2048: 35 and 71; one, 32000 x 1504:
// 88 and 95.  The loss alone splits k over idle units, so that its stages (0.33 to 0.45 us each, one after another) are fewer, and pays a
// launch, the slices' planes and less of a tile's reuse for it: 7 us (3 where a packing launch goes before either way) and W's terms at 4.2 TB/s
// fit what was measured up to 64 rows.  One row, 1000 x 4096: 16 and 27, 4000 x 2048 16 and 17, 4000 x 1504 15 and 18, 8000 x 1504 20 and 18, 8000 x
// 4096 31 and 28, 8000 x 8192 41 and 48; 64 rows, 8000 x 1536 24 and 24, 8000 x 4096 32 and 44.  The choice loses a tenth at most there.
static bool keeps_scores(const XentCall& c, bool direct, bool forward, bool grads) {
    const int64_t n = c.n > 0 ? c.n : 1, whole = up(c.J, 256);
    if ((size_t)up(n, 256) * whole * 4 > kXeScoreBytes) return false;
    const int pairs = c.a_bf16 && c.w_bf16 ? 1 : c.a_bf16 || c.w_bf16 ? 2 : 3;
    const int64_t tiles = ((c.J + 127) / 128) * ((n + 127) / 128);
    if (c.D * pairs < 1500) return false;
    if (!grads && n <= 64) {
        const double stages = (double)((c.D + 63) / 64) * pairs, w_bytes = (double)c.J * (double)c.D * (c.w_bf16 ? 2.0 : 4.0);
        const double gain = stages * (n > 32 ? 0.45 : pairs == 1 ? 0.33 : 0.39), cost = (direct && c.D % 64 == 0 ? 7.0 : 3.0) - (n > 32 ? 2.0 : 0.0) + w_bytes / 4.2e6;
        return tiles < 64 && gain > cost;
    }
    return (forward && grads) || tiles < (n > 64 ? 200 : 64);
}

// The layout that a call on c's sizes takes within `bytes`; .bytes > bytes: there is none
static Layout plan_call(const XentCall& c, bool direct, bool forward, bool grads, size_t bytes) {
    const int64_t whole = up(c.J, 256) / 256;
    const bool raw = direct && !c.w_bf16;                                // keeps its scores if gradients follow, and has no other way
    for (int kept = raw ? grads : keeps_scores(c, direct, forward, grads); kept >= 0; --kept) {
        // a launch has fewer than 2^32 threads, 256 for 128 x 128 results: fewer than 2^38 scores a piece
        const int64_t launch_most = (((int64_t)1 << 37) / up(c.n > 0 ? c.n : 1, 256)) / 256;
        if (!grads && direct) {
            const Layout l = layout_of(c, true, false, kept != 0, (whole < launch_most ? whole : launch_most) * 256);
            if (l.bytes <= bytes || !kept) return l;
            continue;
        }
        // the most words whose U and whose W's terms stay within their bounds, and the whole within `bytes`
        const Layout one = layout_of(c, direct, grads, kept != 0, 256);
        const size_t u_bytes = (size_t)(one.u_terms + one.u16_terms) * one.n_padded * 512, w_bytes = direct ? 0 : (size_t)(one.f16 ? one.w16_terms : 1) * one.ld_k * 512;
        int64_t lo = 1, hi = whole < (1 << 14) ? whole : (1 << 14);      // 32-bit offsets inside a tile: 2^22 words at most
        if (u_bytes > 0 && hi > (int64_t)(kXePieceBytes / u_bytes)) hi = (int64_t)(kXePieceBytes / u_bytes);
        if (w_bytes > 0 && hi > (int64_t)(kXeWordBytes / w_bytes)) hi = (int64_t)(kXeWordBytes / w_bytes);
        if (hi > launch_most) hi = launch_most;
        if (hi < 1) hi = 1;
        if (layout_of(c, direct, grads, kept != 0, hi * 256).bytes <= bytes) lo = hi;    // (bytes may fall as pieces grow: fewer splits of dA)
        while (lo < hi) {
            const int64_t mid = (lo + hi + 1) / 2;
            if (layout_of(c, direct, grads, kept != 0, mid * 256).bytes <= bytes) lo = mid; else hi = mid - 1;
        }
        const int64_t pieces = (whole + lo - 1) / lo;                    // evened out
        Layout l = layout_of(c, direct, grads, kept != 0, (whole + pieces - 1) / pieces * 256);
        if (l.bytes > bytes) l = layout_of(c, direct, grads, kept != 0, lo * 256);
        if (l.bytes <= bytes || !kept || raw) return l;
    }
    return Layout{};                                                     // (not reached)
}

size_t xent_workspace(const XentCall& c, bool grads, bool least) {
    const bool direct = c.w_bf16 && c.a_bf16 && c.D % 8 == 0 && c.D >= 64;
    size_t m = 0;
    // fewer rows can take more splits: the least is what the smallest piece takes at the most splits
    for (int d = 0; d < 2; ++d) {
        if (d && !direct) break;
        Layout l = layout_of(c, d != 0, grads, false, 256);
        size_t b = l.bytes;
        if (grads) b += (size_t)(4 - l.dA.splits > 0 ? 4 - l.dA.splits : 0) * (size_t)(c.n > 0 ? c.n : 1) * l.ld_acc * 4;
        if (b > m) m = b;
    }
    if (least) return m;
    // Whether W can be read as it is its address and leading dimension say, call by call: room for both ways.  Packed rows of it take as much as W
    // itself where they are all there at once, so this way's room ends at kXePackedBytes (65536 x 4096, rows at odd places, 24 rows: loss 764
    // us with what the other way takes, 19 pieces, and 326 in one; with gradients 2305 and 636).
    for (int g = 0; g <= (grads ? 1 : 0); ++g) {
        const bool as_is = direct || (!c.w_bf16 && c.n <= 64 && raw_pays(c, g != 0));
        for (int f = g ? 0 : 1; f < 2; ++f) {
            if (as_is) {
                const size_t b = plan_call(c, true, f != 0, g != 0, ~(size_t)0).bytes;
                if (b > m) m = b;
            }
            const size_t b = plan_call(c, false, f != 0, g != 0, as_is ? (m > kXePackedBytes ? m : kXePackedBytes) : ~(size_t)0).bytes;
            if (b > m) m = b;
        }
    }
    return m;
}

hipError_t launch_xent(const XentCall& c, bool forward, bool grads, hipStream_t s) {
    bool direct = reads_w_directly(c, grads);
    Layout l = plan_call(c, direct, forward, grads, c.ws_bytes);
    if (l.raw && l.bytes > c.ws_bytes) l = plan_call(c, direct = false, forward, grads, c.ws_bytes);
    if (l.bytes > c.ws_bytes) return hipErrorInvalidValue;
    char* const ws = (char*)c.ws;
    int* const rows = (int*)(ws + l.rows);
    int* const label = (int*)(ws + l.label);
    int* const count = (int*)(ws + l.count);
    int* const top = (int*)(ws + l.top);
    float* const g = (float*)(ws + l.g);
    int* const exp_g = (int*)(ws + l.exp_g);
    float* const factor = (float*)(ws + l.factor);
    float* const lse = (float*)(ws + l.lse);
    float* const loss = (float*)(ws + l.loss);
    bf16_t* const A = (bf16_t*)(ws + l.a);
    bf16_t* const A16 = (bf16_t*)(ws + l.a16);
    bf16_t* const Wp = (bf16_t*)(ws + l.w);
    int* const exp_a = (int*)(ws + l.exp_a);
    int* const exp_w = (int*)(ws + l.exp_w);
    const int64_t a_plane = l.n_padded * l.ld_a, a16_plane = l.n_padded * l.ld_k, w_plane = l.piece * l.ld_k;
    const int64_t n_some = c.n > 0 ? c.n : 1;                            // an empty batch: nothing takes part, dW is 0
    hipError_t e;

    XentPack pack;
    {
        XentPack p{};
        p.a = c.a; p.lda = c.lda; p.n = (int)c.n; p.J = (int)c.J; p.D = (int)c.D; p.n_padded = (int)l.n_padded;
        p.y = c.y; p.weight = c.weight; p.scale = c.scale; p.mean = c.mean;
        p.rows = rows; p.label = label; p.exp_g = exp_g; p.count = count; p.g = g;
        p.lse_packed = lse; p.factor = factor; p.lse_given = forward ? nullptr : c.lse;
        p.to = A; p.ld = l.ld_a; p.plane = a_plane; p.terms = l.a_terms; p.window = l.window;
        p.to16 = A16; p.ld16 = l.f16 ? l.ld_k : 0; p.plane16 = a16_plane; p.terms16 = l.a16_terms; p.exps = exp_a;
        p.zero = grads ? c.dA : nullptr; p.ld_zero = c.ldda;
        p.loss = forward ? c.loss : nullptr; p.lse = forward ? c.lse : nullptr;
        pack = p;
    }
    // A loss of few bf16 rows in whole stages at 16-byte places is bound by W's read and by its launches: its product reads the features
    // where they lie, every row's, and no launch packs them first (one row, 32000 x 2048: 24.5 us, 29.0 packed; 24, 65536 x 4096: 109 and 116;
    // 64, 32000 x 1024: 23.2 and 27.0; one, 1000 x 512: 10.9 and 14.2)
    const bool in_place = !grads && direct && c.w_bf16 && !l.kept && c.n > 0 && c.n <= 64 && c.D % 64 == 0 && ((uintptr_t)c.a % 16) == 0 &&
                          c.lda % 8 == 0 && c.lda < (1 << 22);
    if (c.n > kXeFewRows) hipLaunchKernelGGL(xent_rows_kernel, dim3(1), dim3(1024), 0, s, pack);

    // W's rows first .. first + n - 1 as an operand; the first call packs the features as well
    struct Words { const bf16_t* p; int64_t ld, plane; int rows; };
    int64_t there = -1;                                                  // the piece whose terms are in the workspace
    auto words = [&](int64_t first, int64_t n, Words* w) -> hipError_t {
        const bool rows_too = there < 0;
        if (direct) {
            *w = Words{(const bf16_t*)((const char*)c.W + (size_t)first * c.ldw * (c.w_bf16 ? 2 : 4)), c.ldw, 0, (int)n};
            if (in_place) return hipSuccess;
            if (rows_too && c.a_bf16) hipLaunchKernelGGL(xent_pack_rows_kernel<bf16_t>, dim3((uint32_t)l.n_padded), dim3(256), 0, s, pack);
            if (rows_too && !c.a_bf16) hipLaunchKernelGGL(xent_pack_rows_kernel<float>, dim3((uint32_t)l.n_padded), dim3(256), 0, s, pack);
            there = 0;
            return rows_too ? hipGetLastError() : hipSuccess;
        }
        const int64_t padded = up(n, 64), groups = c.D <= kXeShortRow ? padded / 4 : padded;
        *w = Words{Wp, l.ld_k, w_plane, (int)padded};
        if (there == first) return hipSuccess;
        there = first;
        const XentWords x{(const char*)c.W + (size_t)first * c.ldw * (c.w_bf16 ? 2 : 4), c.ldw, (int)c.D, (int)n, Wp, l.ld_k, w_plane, l.f16 ? l.w16_terms : 1,
                          l.f16 ? exp_w + first : nullptr};
        const bool long_rows = c.D > kXeLongRow;
        if (rows_too) {
            if (long_rows) launch_pack_both<true>(pack, x, c.a_bf16, c.w_bf16, (uint32_t)groups, s);
            else launch_pack_both<false>(pack, x, c.a_bf16, c.w_bf16, (uint32_t)groups, s);
        } else {
            if (long_rows) launch_pack_words<true>(x, c.w_bf16, l.f16, (uint32_t)groups, s);
            else launch_pack_words<false>(x, c.w_bf16, l.f16, (uint32_t)groups, s);
        }
        if (l.f16 && grads && !l.kept) hipLaunchKernelGGL(xent_top_kernel, dim3(1), dim3(1024), 0, s, (const int*)(exp_w + first), (int)n, top);
        return hipGetLastError();
    };
    XentProduct scores{};
    scores.y = l.f16 ? A16 : A; scores.ldy = l.f16 ? l.ld_k : l.ld_a; scores.y_plane = l.f16 ? a16_plane : a_plane; scores.y_rows = (int)l.n_padded;
    scores.N = (int)n_some; scores.k_tiles = l.k_tiles; scores.x_cols = (int)c.D;
    scores.last_x = l.window ? (int)c.D - 64 : 64 * (l.k_tiles - 1);
    scores.last_y = l.window ? l.window : 64 * (l.k_tiles - 1);
    scores.pairs = l.f16 ? pair_list(l.w16_terms, l.a16_terms, l.score_most, &scores.pair_x, &scores.pair_y) : 1;
    scores.exp_n = exp_a;
    scores.splits = 1;
    scores.count = count; scores.n_is_rows = true;
    scores.label = label; scores.ld_partial = (int)l.ld_partial;
    scores.z_label = (float*)(ws + l.z_label);
    scores.lse = lse; scores.g = g;
    if (in_place) {
        scores.y = (const bf16_t*)c.a; scores.ldy = c.lda; scores.y_rows = (int)c.n;
        scores.count = nullptr; scores.label = c.y;
    }
    auto scores_of = [&](int64_t first, int64_t n, const Words& w) {
        scores.x = w.p; scores.ldx = w.ld; scores.x_plane = w.plane; scores.x_rows = w.rows;
        scores.M = (int)n; scores.first_word = (int)first;
        scores.exp_m = exp_w + first;
    };
    bf16_t* const U = (bf16_t*)(ws + l.u);
    bf16_t* const U16 = (bf16_t*)(ws + l.u16);
    const int64_t u_plane = l.n_padded * l.piece, acc_plane = n_some * l.ld_acc;

    bool total_done = false;
    const int64_t pieces = (c.J + l.piece - 1) / l.piece;
    // kept scores: the loss, and U's words from `first` on
    auto rows_of = [&](int64_t first, bool given) {
        XentRows r{};
        r.z = (const float*)(ws + l.z); r.ldz = l.ld_z; r.z_plane = l.n_padded * l.ld_z; r.splits = l.scores.splits;
        r.words = (int)c.J; r.first = (int)first; r.columns = grads ? (int)l.piece : 0;
        r.rows = rows; r.label = label; r.count = count; r.g = g;
        r.loss = c.loss; r.lse = c.lse; r.loss_packed = loss; r.lse_packed = lse;
        r.u = U; r.u16 = U16; r.ldu = l.piece; r.u_plane = u_plane; r.u_terms = l.u_terms; r.u16_terms = l.u16_terms;
        r.exp_m = exp_w; r.exp_g = exp_g; r.exp_words = top;
        r.given = given;
        hipLaunchKernelGGL(xent_row_kernel, dim3((uint32_t)up(n_some, 64)), dim3(kXeRowThreads), 0, s, r);
        return hipGetLastError();
    };
    if (l.kept) {
        for (int64_t first = 0; first < c.J; first += l.piece) {
            const int64_t n = c.J - first < l.piece ? c.J - first : l.piece;
            Words w;
            e = words(first, n, &w);
            if (e != hipSuccess) return e;
            scores_of(first, n, w);
            XentProduct p = scores;
            p.splits = l.scores.splits;
            p.out = (float*)(ws + l.z) + first; p.ldo = l.ld_z; p.out_plane = l.n_padded * l.ld_z;
            if (l.raw) e = l.raw_any ? launch_raw_scores<true>(p, c.a_bf16, (int)n_some, s) : launch_raw_scores<false>(p, c.a_bf16, (int)n_some, s);
            else if (l.f16) e = launch_product<false, false, true, kXeStore, float>(p, l.scores.tile, s);
            else e = launch_product<false, false, false, kXeStore, float>(p, l.scores.tile, s);
            if (e != hipSuccess) return e;
        }
        e = rows_of((pieces - 1) * l.piece, !forward);
        if (e != hipSuccess) return e;
    } else if (forward) {
        int tiles = 0;
        for (int64_t first = 0; first < c.J; first += l.piece) {
            const int64_t n = c.J - first < l.piece ? c.J - first : l.piece;
            Words w;
            e = words(first, n, &w);
            if (e != hipSuccess) return e;
            scores_of(first, n, w);
            scores.partial = (float2*)(ws + l.partial) + tiles;
            if (l.raw) {
                e = l.raw_any ? launch_raw_scores<true>(scores, c.a_bf16, (int)n_some, s) : launch_raw_scores<false>(scores, c.a_bf16, (int)n_some, s);
            } else {
                e = l.f16 ? launch_product<false, false, true, kXeStats, float>(scores, l.scores.tile, s)
                          : launch_product<false, false, false, kXeStats, float>(scores, l.scores.tile, s);
            }
            if (e != hipSuccess) return e;
            const int tile_m = l.raw ? kXeRawWords : kXeTileM[l.scores.tile];
            tiles += (int)((n + tile_m - 1) / tile_m);
        }
        if (in_place) {
            hipLaunchKernelGGL(xent_in_place_loss_kernel, dim3(1), dim3(1024), 0, s, pack, (const float2*)(ws + l.partial), tiles, (int)l.ld_partial,
                               (const float*)(ws + l.z_label), c.loss, c.lse, c.total);
            return hipGetLastError();
        }
        // (64 rows are four a wavefront of one workgroup, which then needs no launch behind it for the total)
        const bool alone = n_some <= 64;
        hipLaunchKernelGGL(xent_loss_kernel, dim3(alone ? 1u : (uint32_t)((n_some + 15) / 16)), dim3(1024), 0, s, (const float2*)(ws + l.partial), tiles,
                           (int)l.ld_partial, (const int*)rows, (const int*)count, (const float*)(ws + l.z_label), (const float*)g, c.loss, c.lse, lse, loss,
                           (const float*)factor, alone ? c.total : nullptr);
        total_done = alone;
    }
    // with gradients the first workgroup of their first product does it
    float* total_left = forward && !total_done && grads ? c.total : nullptr;
    if (l.raw && !c.dW) total_left = nullptr;
    if (forward && c.total && !total_done && !total_left)
        hipLaunchKernelGGL(xent_total_kernel, dim3(1), dim3(1024), 0, s, (const float*)loss, (const float*)g, (const int*)count, (const float*)factor, c.total);
    e = hipGetLastError();
    if (e != hipSuccess || !grads) return e;

    // from the last piece back: its terms of W are still there
    for (int64_t i = pieces - 1; i >= 0; --i) {
        const int64_t first = i * l.piece, n = c.J - first < l.piece ? c.J - first : l.piece;
        Words w;
        e = words(first, n, &w);
        if (e != hipSuccess) return e;
        if (l.kept) {
            if (i < pieces - 1) e = rows_of(first, true);
            if (e != hipSuccess) return e;
        } else {
            scores_of(first, n, w);
            scores.u = U; scores.u16 = U16; scores.ldu = l.piece; scores.u_plane = u_plane; scores.u_terms = l.u_terms; scores.u16_terms = l.u16_terms;
            scores.exp_g = exp_g; scores.exp_words = top;
            e = l.f16 ? launch_product<false, false, true, kXeU, float>(scores, l.scores.tile, s) : launch_product<false, false, false, kXeU, float>(scores, l.scores.tile, s);
            if (e != hipSuccess) return e;
        }
        if (c.dA && l.raw) {
            XentProduct p{};
            p.x = w.p; p.ldx = w.ld; p.x_rows = w.rows;
            p.y = U; p.ldy = l.piece; p.y_plane = u_plane;
            p.M = (int)c.D; p.N = (int)n_some;
            p.k_tiles = (int)((n + 63) / 64);
            p.factor = factor;
            p.splits = l.dA.splits;
            p.count = count;
            p.out = ws + l.acc; p.ldo = l.ld_acc; p.out_plane = acc_plane;
            p.add = i < pieces - 1 ? (const float*)(ws + l.acc) : nullptr; p.ld_add = l.ld_acc;
            if (c.a_bf16) e = n_some > 32 ? launch_raw_features<2, 1>(p, s) : launch_raw_features<1, 1>(p, s);
            else e = n_some > 32 ? launch_raw_features<2, 2>(p, s) : launch_raw_features<1, 2>(p, s);
            if (e != hipSuccess) return e;
        } else if (c.dA) {
            XentProduct p{};
            p.x = w.p; p.ldx = w.ld; p.x_plane = w.plane; p.x_rows = w.rows; p.x_cols = direct ? (int)c.D : (int)l.ld_k;
            p.y = l.f16 ? U16 : U; p.ldy = l.piece; p.y_plane = u_plane; p.y_rows = (int)l.n_padded;
            p.M = (int)c.D; p.N = (int)n_some;
            p.k_tiles = (int)((n + 63) / 64); p.last_y = 64 * (p.k_tiles - 1);
            p.pairs = l.f16 ? pair_list(l.w16_terms, l.u16_terms, l.dA_most, &p.pair_x, &p.pair_y) : 1;
            p.exp_n = exp_g; p.exp_top = top;
            p.factor = factor;
            p.splits = l.dA.splits;
            p.count = count; p.n_is_rows = true;
            if (l.dA.splits == 1 && i == 0) {                            // the last sum goes straight to its row
                p.out = c.dA; p.ldo = c.ldda; p.row_map = rows;
            } else {
                p.out = ws + l.acc; p.ldo = l.ld_acc; p.out_plane = acc_plane;
            }
            p.add = i < pieces - 1 ? (const float*)(ws + l.acc) : nullptr; p.ld_add = l.ld_acc;
            p.loss_packed = loss; p.weights = g; p.loss_total = total_left;
            total_left = nullptr;
            if (p.row_map && c.a_bf16)
                e = l.f16 ? launch_product<true, false, true, kXeStore, bf16_t>(p, l.dA.tile, s) : launch_product<true, false, false, kXeStore, bf16_t>(p, l.dA.tile, s);
            else
                e = l.f16 ? launch_product<true, false, true, kXeStore, float>(p, l.dA.tile, s) : launch_product<true, false, false, kXeStore, float>(p, l.dA.tile, s);
            if (e != hipSuccess) return e;
        }
        if (c.dW) {
            XentProduct p{};
            p.x = A; p.ldx = l.ld_a; p.x_plane = a_plane; p.x_rows = (int)l.n_padded; p.x_cols = (int)l.ld_k;
            p.y = U; p.ldy = l.piece; p.y_plane = u_plane; p.y_rows = (int)l.n_padded; p.y_cols = (int)l.piece;
            p.M = (int)c.D; p.N = (int)n;
            p.k_tiles = (int)((n_some + 63) / 64);
            p.pairs = pair_list(l.a_terms, l.u_terms, l.dW_most, &p.pair_x, &p.pair_y);
            p.splits = 1;
            p.count = count; p.k_is_rows = true;
            p.factor = factor;
            p.ldo = c.lddw;
            p.loss_packed = loss; p.weights = g; p.loss_total = total_left;
            total_left = nullptr;
            if (c.w_bf16) {
                p.out = (bf16_t*)c.dW + first * c.lddw;
                e = launch_product<true, true, false, kXeStore, bf16_t>(p, l.dW.tile, s);
            } else {
                p.out = (float*)c.dW + first * c.lddw;
                e = launch_product<true, true, false, kXeStore, float>(p, l.dW.tile, s);
            }
            if (e != hipSuccess) return e;
        }
    }
    if (c.dA && (l.dA.splits > 1 || l.raw)) {
        const uint32_t grid = (uint32_t)((n_some * ((c.D + 3) / 4) + 255) / 256);
        if (c.a_bf16)
            hipLaunchKernelGGL(xent_rows_out_kernel<bf16_t>, dim3(grid), dim3(256), 0, s, (const float*)(ws + l.acc), l.ld_acc, acc_plane, l.dA.splits,
                               (const int*)rows, (const int*)count, (int)c.D, (bf16_t*)c.dA, c.ldda);
        else
            hipLaunchKernelGGL(xent_rows_out_kernel<float>, dim3(grid), dim3(256), 0, s, (const float*)(ws + l.acc), l.ld_acc, acc_plane, l.dA.splits,
                               (const int*)rows, (const int*)count, (int)c.D, (float*)c.dA, c.ldda);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace sfb
