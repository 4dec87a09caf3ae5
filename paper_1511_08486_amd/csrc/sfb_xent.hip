// Softmax cross entropy of a linear head, z_i = W a_i, without the N x J scores in memory, and its gradients.
//
//   lse_i = log sum_j exp(z_ij)       loss_i = lse_i - z_i,y(i)
//   u_ij  = g_i (exp(z_ij - lse_i) - [j = y(i)])         dA = U W         dW = U^T A
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
// fp32 operands are three bf16 terms each (exact), a product six of theirs; with one bf16 operand three.  They are a longer k to the
// kernel: the small products first, so that the sum is rounded at its full size only along the last one.
#include "sfb_kernels.h"
#include "sfb_split.h"

namespace sfb {

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
    int m_tiles, n_tiles, total, splits, per_split;
    const int* count;                        // rows that take part
    bool n_is_rows, k_is_rows;               // what `count` bounds
    // kXeStats, kXeU
    const int* label;
    int first_word;                          // word of m = 0
    float2* partial;                         // [m_tiles][ld_rows]
    float* z_label;
    int ld_rows;
    const float *lse, *g;
    bf16_t* u;                               // [terms][..][ldu]
    int64_t ldu, u_plane;
    int u_terms;
    // kXeStore
    void* out;
    int64_t ldo, out_plane;                  // out_plane: between splits
    const float* add;                        // fp32, or nullptr
    int64_t ld_add;
    const int* row_map;                      // row of out for n, or nullptr
    bool wide;                               // out takes 16 bytes at a time
};

__device__ __forceinline__ uint32_t xe_lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// 64 lanes x 16 bytes from base + off to LDS, lane l's at lds + 16 l (not seen by the compiler: waits are the caller's)
__device__ __forceinline__ void xe_dma(const void* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}

// exp(x) with x's whole part taken off in two products, so that its error is that of exp2 of a number below 1/2; NaN stays
__device__ __forceinline__ float xe_exp(float x) {
    x = x < -104.f ? -104.f : x;
    const float n = rintf(x * 1.44269504f);
    const float r = __builtin_fmaf(x, 1.44269504f, -n) + x * 1.92596299e-8f;
    return __builtin_ldexpf(__builtin_amdgcn_exp2f(r), (int)n);
}

// How one operand goes to LDS and comes from there.  ROWS: of m (n) in the tile.  Not TR: LDS rows of 64 k, 16-byte piece p of row r at
// p ^ (r & 7).  TR: LDS rows of ROWS m, 32-byte piece p of k-row r at p ^ turn(r), so that the four rows of a transposing read, and its
// neighbour's sixteen columns, fall on different banks.
template <bool TR, int ROWS, int WAVES, int TILES>
struct XentSide {
    static constexpr int LOADS = ROWS / 8 / WAVES, BYTES = ROWS * 128;
    static_assert(LOADS * 8 * WAVES == ROWS, "whole accesses");
    uint32_t off[LOADS];
    int at[TR ? TILES : 4];
    __device__ __forceinline__ static int turn(int r) { return ROWS >= 128 ? 2 * (r & 3) : r & 3; }
    // k_most: the last k-row that may be read, counted from the stage's first
    __device__ __forceinline__ void offsets(int wave, int lane, int row0, int rows, int cols, int64_t ld, int k_most) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            if constexpr (!TR) {
                const int r = min(row0 + (i * WAVES + wave) * 8 + (lane >> 3), rows - 1) - row0;
                off[i] = (uint32_t)r * (uint32_t)ld * 2u + (uint32_t)(((lane & 7) ^ ((lane >> 3) & 7)) * 16);
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
            for (int s = 0; s < 4; ++s) at[s] = (first + l32) * 128 + (((2 * s + half) ^ (l32 & 7)) << 4);
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

template <int WGM, int WGN, int MT, int NT, int ST, int OCC, bool XT, bool YT, int END, class Out>
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

    const int count = *a.count;
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
            acc[q / NT][q % NT] = split_mfma(now.x[q / NT], now.y[q % NT], acc[q / NT][q % NT]);
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
        auto follow = [&]() { now = now + STAGE == xe_lds + ST * STAGE ? xe_lds : now + STAGE; };
        int s = 0;
        for (; s + ST < stages; ++s) {
            xe_stage_barrier<(ST - 2) * LOADS>();                        // the ST - 2 stages after the next may still be on their way
            follow();
            aim();
            phase(I0, I1, I0, MID, f1, f0, now);
            phase(I1, I1, MID, ALL, f0, f1, now);
            next();
            phase(I2, I1, I0, I0, f1, f0, now);
            phase(I3, I1, I0, I0, f0, f1, now);
        }
        for (; s + 1 < stages; ++s) {
            xe_wait_barrier();
            follow();
            phase(I0, I1, I0, I0, f1, f0, now);
            phase(I1, I1, I0, I0, f0, f1, now);
            phase(I2, I1, I0, I0, f1, f0, now);
            phase(I3, I1, I0, I0, f0, f1, now);
        }
        phase(I0, I0, I0, I0, f1, f0, now);
    }
    xe_wait_barrier();                                                   // LDS is free

    const int mw = m0 + wm * MT * 32 + 4 * half, nw = n0 + wn * NT * 32 + l32;      // entry e of (i, j): m = mw + 32 i + 8 (e / 4) + e % 4
    if constexpr (END == kXeStats) {
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
        for (int n = tid; n < BN; n += WAVES * 64) {
            float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
            for (int w = 0; w < WGM; ++w) top = fmaxf(top, red[w * BN + n].x);
            const float base = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
            for (int w = 0; w < WGM; ++w) sum += red[w * BN + n].y * xe_exp(red[w * BN + n].x - base);
            a.partial[(int64_t)(m0 / BM) * a.ld_rows + n0 + n] = make_float2(top, sum);
        }
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
        for (int term = 0; term < a.u_terms; ++term) {
            if (term > 0) __syncthreads();
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int row = wn * NT * 32 + 32 * j + l32;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint2 w;
                        w.x = cvt_pk_bf16(acc[i][j][4 * q], acc[i][j][4 * q + 1]);
                        w.y = cvt_pk_bf16(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                        // what the term leaves over, exact
                        acc[i][j][4 * q] -= __uint_as_float(w.x << 16);
                        acc[i][j][4 * q + 1] -= __uint_as_float(w.x & 0xffff0000u);
                        acc[i][j][4 * q + 2] -= __uint_as_float(w.y << 16);
                        acc[i][j][4 * q + 3] -= __uint_as_float(w.y & 0xffff0000u);
                        const int piece = (wm * MT * 32 + 32 * i + 8 * q) / 8;
                        *reinterpret_cast<uint2*>(xe_lds + row * (BM * 2) + ((piece ^ (row & 15)) << 4) + 8 * half) = w;
                    }
            }
            __syncthreads();
            bf16_t* const u = a.u + term * a.u_plane + m0;
            for (int c = tid; c < BN * PER; c += WAVES * 64) {
                const int row = c / PER, piece = c % PER;
                *reinterpret_cast<sp_u32x4*>(u + (int64_t)(n0 + row) * a.ldu + piece * 8) =
                    *reinterpret_cast<const sp_u32x4*>(xe_lds + row * (BM * 2) + ((piece ^ (row & 15)) << 4));
                // dW takes whole stages of 64 rows
                if constexpr (BN == 32) *reinterpret_cast<sp_u32x4*>(u + (int64_t)(n0 + 32 + row) * a.ldu + piece * 8) = sp_u32x4{0u, 0u, 0u, 0u};
            }
        }
    } else {
        // rows of n, as many 32-row blocks of every wavefront at a time as LDS holds in fp32
        constexpr int FIT = ST * STAGE / (WGN * 32 * BM * 4), JR = FIT < NT ? FIT : NT;
        static_assert(FIT >= 1 && NT % JR == 0, "whole rounds");
        constexpr int PER = BM / 4;
        const int n_most = a.n_is_rows ? min(a.N, count) : a.N;
        Out* const out = reinterpret_cast<Out*>(a.out) + split * a.out_plane;
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
                if (add) {
                    const float* p = add + (int64_t)n * a.ld_add + m;    // (rows of the accumulators are whole multiples of 8)
                    lo += *reinterpret_cast<const f32x4*>(p);
                    hi += *reinterpret_cast<const f32x4*>(p + 4);
                }
                Out* const o = out + (int64_t)(a.row_map ? a.row_map[n] : n) * a.ldo + m;
                if (a.wide && m + 8 <= a.M) {
                    if constexpr (sizeof(Out) == 4) {
                        *reinterpret_cast<f32x4*>(o) = lo;
                        *reinterpret_cast<f32x4*>(o + 4) = hi;
                    } else {
                        *reinterpret_cast<sp_u32x4*>(o) = sp_u32x4{cvt_pk_bf16(lo[0], lo[1]), cvt_pk_bf16(lo[2], lo[3]), cvt_pk_bf16(hi[0], hi[1]), cvt_pk_bf16(hi[2], hi[3])};
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

// ---------------------------------------------------------------------------------------------------------------
// What stands around the products

// One workgroup: the rows that take part, in order, then the others; label and factor of each of the former.
__global__ __launch_bounds__(1024) void xent_rows_kernel(const int32_t* __restrict__ y, int n, int J, const float* __restrict__ weight, float scale,
                                                         int mean, int* __restrict__ rows, int* __restrict__ label, float* __restrict__ g,
                                                         int* __restrict__ count) {
    __shared__ int before[16], total;
    int taken = 0;                                                       // so far, the same in every thread
    for (int base = 0; base < n; base += 1024) {
        const int i = base + (int)threadIdx.x, lab = i < n ? y[i] : -1;
        const bool real = lab >= 0 && lab < J;
        const uint64_t votes = __ballot(real);
        if ((threadIdx.x & 63) == 0) before[threadIdx.x >> 6] = __popcll(votes);
        __syncthreads();
        if (threadIdx.x == 0) {
            int s = taken;
            for (int w = 0; w < 16; ++w) {
                const int c = before[w];
                before[w] = s;
                s += c;
            }
            total = s;
        }
        __syncthreads();
        const int k = before[threadIdx.x >> 6] + __popcll(votes & ((1ull << (threadIdx.x & 63)) - 1ull));
        if (real) {
            rows[k] = i;
            label[k] = lab;
            g[k] = scale * (weight ? weight[i] : 1.f);
        } else if (i < n) {
            rows[n - 1 - (i - k)] = i;                                   // i - k rows before this one take no part
        }
        taken = total;
        __syncthreads();
    }
    if (mean && taken > 0)
        for (int k = threadIdx.x; k < taken; k += 1024) g[k] = g[k] / (float)taken;      // (written before the last barrier)
    if (threadIdx.x == 0) *count = taken;
}

// Rows of `src` in bf16 terms, k padded with zeros to whole stages.  rows: row of src for every packed row (the first *count of them; a row
// behind those takes its results' zeros here), or nullptr: rows first .. first + n - 1.  window: one stage more that repeats the last 64
// columns of src, with zeros where they are in the stage before: it meets W's last 64 columns where W is read as it is.
template <class T>
__global__ __launch_bounds__(256) void xent_pack_kernel(const T* __restrict__ src, int64_t ld, int D, const int* __restrict__ rows,
                                                        const int* __restrict__ count, int n, int n_padded, bf16_t* __restrict__ dst, int64_t ldd,
                                                        int64_t plane, int terms, int window, T* __restrict__ zero, int64_t ld_zero,
                                                        float* __restrict__ loss, float* __restrict__ lse) {
    const int per = (int)(ldd / 8);
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int k = (int)(c / per), p = (int)(c % per);
    if (k >= n_padded) return;
    const int real = rows ? min(*count, n) : n;
    if (rows && k >= real && k < n) {
        const int i = rows[k];
        if (zero)
            for (int d = p * 8; d < min(D, p * 8 + 8); ++d) zero[(int64_t)i * ld_zero + d] = T(0);
        if (p == 0 && loss) loss[i] = 0.f;
        if (p == 0 && lse) lse[i] = 0.f;
    }
    float x[8];
    const int at = window && p * 8 >= window ? D - 64 + (p * 8 - window) : p * 8;
    const int least = window && p * 8 >= window ? window - 64 : 0;
    const T* row = src + (int64_t)(rows && k < real ? rows[k] : min(k, n - 1)) * ld;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = at + e;
        const bool in = k < real && d < D && d >= least;
        if constexpr (sizeof(T) == 4) x[e] = in ? row[d] : 0.f;
        else x[e] = in ? bf16_to_f32(row[d]) : 0.f;
    }
    for (int t = 0; t < terms; ++t) {
        sp_u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = cvt_pk_bf16(x[2 * e], x[2 * e + 1]);
            x[2 * e] -= __uint_as_float(w[e] << 16);
            x[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
        }
        *reinterpret_cast<sp_u32x4*>(dst + t * plane + (int64_t)k * ldd + p * 8) = w;
    }
}

// lse and loss of a row from its tiles' maxima and sums: a wavefront a row, tiles in a fixed order
__global__ __launch_bounds__(256) void xent_loss_kernel(const float2* __restrict__ partial, int tiles, int ld_rows, const int* __restrict__ rows,
                                                        const int* __restrict__ count, const float* __restrict__ z_label, float* __restrict__ loss,
                                                        float* __restrict__ lse, float* __restrict__ lse_packed, float* __restrict__ loss_packed) {
    const int k = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (k >= *count) return;
    float top = -__builtin_inff(), sum = 0.f;
    for (int t = lane; t < tiles; t += 64) {
        const float2 p = partial[(int64_t)t * ld_rows + k];
        const float m = fmaxf(top, p.x), base = m == -__builtin_inff() ? 0.f : m;
        sum = sum * xe_exp(top - base) + p.y * xe_exp(p.x - base);
        top = m;
    }
    const float most = wave_max(top), base = most == -__builtin_inff() ? 0.f : most;
    sum = wave_sum(sum * xe_exp(top - base));
    if (lane == 0) {
        const float l = logf(sum), v = most + l, f = l + (most - z_label[k]);
        const int i = rows[k];
        if (lse) lse[i] = v;
        if (loss) loss[i] = f;
        lse_packed[k] = v;
        loss_packed[k] = f;
    }
}

__global__ __launch_bounds__(256) void xent_gather_kernel(const float* __restrict__ lse, const int* __restrict__ rows, const int* __restrict__ count,
                                                          float* __restrict__ lse_packed) {
    const int k = blockIdx.x * 256 + threadIdx.x;
    if (k < *count) lse_packed[k] = lse[rows[k]];
}

// total = sum of g loss in a fixed order, in 64 bits
__global__ __launch_bounds__(1024) void xent_total_kernel(const float* __restrict__ loss, const float* __restrict__ g, const int* __restrict__ count,
                                                          float* __restrict__ total) {
    __shared__ double part[16];
    const int n = *count;
    double s = 0.0;
    for (int k = threadIdx.x; k < n; k += 1024) s += (double)loss[k] * (double)g[k];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, kWave);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int w = 0; w < 16; ++w) s += part[w];
        *total = (float)s;
    }
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
    for (int p = 0; p < planes; ++p) s += *reinterpret_cast<const f32x4*>(acc + p * plane + (int64_t)k * ld + d);
    store4(out + (int64_t)rows[k] * ldo, d, D, s);
}

// ---------------------------------------------------------------------------------------------------------------
// Plans and launches

template <int WGM, int WGN, int MT, int NT, int ST, int OCC, bool XT, bool YT, int END, class Out>
static hipError_t launch_product(XentProduct a, hipStream_t s) {
    constexpr int BM = WGM * MT * 32, BN = WGN * NT * 32;
    constexpr size_t lds = (size_t)ST * (BM + BN) * 128;
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    auto* const kernel = &xent_product_kernel<WGM, WGN, MT, NT, ST, OCC, XT, YT, END, Out>;
    if constexpr (lds > 64 * 1024) {
        static std::atomic<uint64_t> raised{0};                          // GPUs that know
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        if (dev > 63 || !(raised.load() >> dev & 1)) {
            e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) return e;
            if (dev <= 63) raised |= 1ull << dev;
        }
    }
    a.m_tiles = (a.M + BM - 1) / BM;
    a.n_tiles = (a.N + BN - 1) / BN;
    a.total = a.m_tiles * a.n_tiles * a.splits;
    a.per_split = (a.k_tiles + a.splits - 1) / a.splits;
    SFB_LAUNCH((xent_product_kernel<WGM, WGN, MT, NT, ST, OCC, XT, YT, END, Out>), dim3(a.total), dim3(WGM * WGN * 64), lds, s, a);
    return hipGetLastError();
}

// Tiles by the number of n (rows): m x n.
enum XentTile { kXe256x256, kXe128x128, kXe256x64, kXe256x32 };
static const int kXeTileM[] = {256, 128, 256, 256}, kXeTileN[] = {256, 128, 64, 32};

template <bool XT, bool YT, int END, class Out>
static hipError_t launch_product(const XentProduct& a, XentTile tile, hipStream_t s) {
    switch (tile) {
        case kXe256x256: return launch_product<2, 4, 4, 2, 2, 2, XT, YT, END, Out>(a, s);
        case kXe128x128: return launch_product<2, 2, 2, 2, 2, 2, XT, YT, END, Out>(a, s);
        default: break;
    }
    if constexpr (!YT) {
        if (tile == kXe256x64) return launch_product<4, 1, 2, 2, 3, 1, XT, YT, END, Out>(a, s);
        if (tile == kXe256x32) return launch_product<4, 1, 2, 1, 4, 1, XT, YT, END, Out>(a, s);
    }
    return hipErrorInvalidValue;
}

static XentTile tile_for(int64_t M, int64_t N) {
    if (N <= 32) return kXe256x32;
    if (N <= 64) return kXe256x64;
    return ((M + 255) / 256) * ((N + 255) / 256) >= 192 ? kXe256x256 : kXe128x128;
}

// Pairs of terms of a product, the small ones first; `most`: the sum of their numbers (0, 1, 2) goes up to it
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

namespace {
constexpr int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
struct Layout {
    int64_t n_padded, ld_a, ld_w, piece, ld_acc;
    int a_terms, w_terms, u_terms, k_tiles, window, splits;
    size_t rows, label, g, lse, loss, z, count, partial, acc, a, w, u, bytes;
};
}  // namespace

// direct: W is read as it is.  piece: words of a piece, a multiple of 256
static Layout layout_of(const XentCall& c, bool direct, bool grads, int64_t piece) {
    Layout l{};
    const int64_t n_some = c.n > 0 ? c.n : 1;
    l.n_padded = up(n_some, 256);
    l.k_tiles = (int)((c.D + 63) / 64);
    l.window = direct && c.D % 64 != 0 ? 64 * l.k_tiles : 0;
    l.ld_a = 64 * l.k_tiles + (l.window ? 64 : 0);
    l.ld_w = 64 * l.k_tiles;
    l.ld_acc = up(c.D, 8);
    l.a_terms = c.a_bf16 ? 1 : 3;
    l.w_terms = c.w_bf16 ? 1 : 3;
    l.u_terms = grads ? (c.a_bf16 && c.w_bf16 ? 1 : 3) : 0;
    l.piece = piece;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += up(bytes, 256);
        return p;
    };
    l.rows = take((size_t)n_some * 4);
    l.label = take((size_t)l.n_padded * 4);
    l.g = take((size_t)l.n_padded * 4);
    l.lse = take((size_t)l.n_padded * 4);
    l.loss = take((size_t)l.n_padded * 4);
    l.z = take((size_t)l.n_padded * 4);
    l.count = take(4);
    l.partial = take((size_t)(up(c.J, 256) / 128) * l.n_padded * 8);
    l.a = take((size_t)l.a_terms * l.n_padded * l.ld_a * 2);
    if (grads) {
        // few rows leave few tiles of dA: the words are cut into splits with sums of their own
        const XentTile t = tile_for(c.D, n_some);
        const int64_t tiles = ((c.D + kXeTileM[t] - 1) / kXeTileM[t]) * ((n_some + kXeTileN[t] - 1) / kXeTileN[t]), most = up(piece, 64) / 64 / 8;
        int64_t s = tiles >= 192 ? 1 : (256 + tiles - 1) / tiles;
        if (s > most) s = most;
        l.splits = s < 1 ? 1 : (int)s;
        l.acc = take((size_t)l.splits * l.n_padded * l.ld_acc * 4);
        l.u = take((size_t)l.u_terms * l.n_padded * piece * 2);
    }
    if (!direct) l.w = take((size_t)l.w_terms * up(piece, 64) * l.ld_w * 2);
    l.bytes = at;
    return l;
}

static bool reads_w_directly(const XentCall& c) {
    return c.w_bf16 && c.D % 8 == 0 && c.D >= 64 && c.ldw % 8 == 0 && ((uintptr_t)c.W % 16) == 0 && c.ldw < (1 << 23);
}

size_t xent_workspace(const XentCall& c, bool grads, bool least) {
    const int64_t whole = up(c.J, 256);
    if (least) return layout_of(c, false, grads, 256).bytes > layout_of(c, true, grads, 256).bytes ? layout_of(c, false, grads, 256).bytes
                                                                                                  : layout_of(c, true, grads, 256).bytes;
    // pieces of 256 MB of U and W together
    const bool direct = c.w_bf16 && c.D % 8 == 0 && c.D >= 64;
    const Layout one = layout_of(c, direct, grads, 256), two = layout_of(c, direct, grads, 512);
    int64_t pieces = (int64_t)(((size_t)256 << 20) / (two.bytes - one.bytes + 1));
    if (pieces < 4) pieces = 4;
    const size_t b = layout_of(c, direct, grads, pieces * 256 < whole ? pieces * 256 : whole).bytes, m = xent_workspace(c, grads, true);
    return b > m ? b : m;
}

// The largest piece that the workspace holds, evened out over the pieces; 0: none.
static int64_t piece_for(const XentCall& c, bool direct, bool grads, size_t bytes) {
    const int64_t whole = up(c.J, 256) / 256;
    if (!grads && direct) return layout_of(c, true, false, 256).bytes <= bytes ? whole * 256 : 0;
    int64_t lo = 0, hi = whole < (1 << 14) ? whole : (1 << 14);          // 32-bit offsets inside a tile: 2^22 words at most
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (layout_of(c, direct, grads, mid * 256).bytes <= bytes) lo = mid; else hi = mid - 1;
    }
    if (lo == 0) return 0;
    const int64_t pieces = (whole + lo - 1) / lo;
    return (whole + pieces - 1) / pieces * 256;
}

hipError_t launch_xent(const XentCall& c, bool forward, bool grads, hipStream_t s) {
    const bool direct = reads_w_directly(c);
    const int64_t piece = piece_for(c, direct, grads, c.ws_bytes);
    if (piece == 0) return hipErrorInvalidValue;
    const Layout l = layout_of(c, direct, grads, piece);
    char* const ws = (char*)c.ws;
    int* const rows = (int*)(ws + l.rows);
    int* const label = (int*)(ws + l.label);
    int* const count = (int*)(ws + l.count);
    float* const g = (float*)(ws + l.g);
    float* const lse = (float*)(ws + l.lse);
    float* const loss = (float*)(ws + l.loss);
    bf16_t* const A = (bf16_t*)(ws + l.a);
    bf16_t* const Wp = (bf16_t*)(ws + l.w);
    const int64_t a_plane = l.n_padded * l.ld_a;
    const int64_t n_some = c.n > 0 ? c.n : 1;                            // an empty batch: nothing takes part, dW is 0
    hipError_t e;

    hipLaunchKernelGGL(xent_rows_kernel, dim3(1), dim3(1024), 0, s, c.y, (int)c.n, (int)c.J, c.weight, c.scale, c.mean, rows, label, g, count);
    const uint32_t pack_grid = (uint32_t)((l.n_padded * (l.ld_a / 8) + 255) / 256);
    float* const loss0 = forward ? c.loss : nullptr;
    float* const lse0 = forward ? c.lse : nullptr;
    if (c.a_bf16)
        hipLaunchKernelGGL(xent_pack_kernel<bf16_t>, dim3(pack_grid), dim3(256), 0, s, (const bf16_t*)c.a, c.lda, (int)c.D, (const int*)rows, (const int*)count,
                           (int)c.n, (int)l.n_padded, A, l.ld_a, a_plane, l.a_terms, l.window, (bf16_t*)(grads ? c.dA : nullptr), c.ldda, loss0, lse0);
    else
        hipLaunchKernelGGL(xent_pack_kernel<float>, dim3(pack_grid), dim3(256), 0, s, (const float*)c.a, c.lda, (int)c.D, (const int*)rows, (const int*)count,
                           (int)c.n, (int)l.n_padded, A, l.ld_a, a_plane, l.a_terms, l.window, (float*)(grads ? c.dA : nullptr), c.ldda, loss0, lse0);
    e = hipGetLastError();
    if (e != hipSuccess) return e;

    // X = W's rows first .. first + words - 1 in terms
    struct Words { const bf16_t* p; int64_t ld, plane; int rows; };
    auto words = [&](int64_t first, int64_t n, Words* w) -> hipError_t {
        if (direct) {
            *w = Words{(const bf16_t*)c.W + first * c.ldw, c.ldw, 0, (int)n};
            return hipSuccess;
        }
        const int64_t padded = up(n, 64), plane = up(piece, 64) * l.ld_w;
        const uint32_t grid = (uint32_t)((padded * (l.ld_w / 8) + 255) / 256);
        if (c.w_bf16)
            hipLaunchKernelGGL(xent_pack_kernel<bf16_t>, dim3(grid), dim3(256), 0, s, (const bf16_t*)c.W + first * c.ldw, c.ldw, (int)c.D, (const int*)nullptr,
                               (const int*)nullptr, (int)n, (int)padded, Wp, l.ld_w, plane, 1, 0, (bf16_t*)nullptr, (int64_t)0, (float*)nullptr, (float*)nullptr);
        else
            hipLaunchKernelGGL(xent_pack_kernel<float>, dim3(grid), dim3(256), 0, s, (const float*)c.W + first * c.ldw, c.ldw, (int)c.D, (const int*)nullptr,
                               (const int*)nullptr, (int)n, (int)padded, Wp, l.ld_w, plane, 3, 0, (float*)nullptr, (int64_t)0, (float*)nullptr, (float*)nullptr);
        *w = Words{Wp, l.ld_w, plane, (int)padded};
        return hipGetLastError();
    };
    XentProduct scores{};
    scores.y = A; scores.ldy = l.ld_a; scores.y_plane = a_plane; scores.y_rows = (int)l.n_padded;
    scores.N = (int)n_some; scores.k_tiles = l.k_tiles;
    scores.last_x = l.window ? (int)c.D - 64 : 64 * (l.k_tiles - 1);
    scores.last_y = l.window ? l.window : 64 * (l.k_tiles - 1);
    scores.pairs = pair_list(l.w_terms, l.a_terms, 2, &scores.pair_x, &scores.pair_y);
    scores.splits = 1;
    scores.count = count; scores.n_is_rows = true;
    scores.label = label; scores.ld_rows = (int)l.n_padded;
    scores.z_label = (float*)(ws + l.z);
    scores.lse = lse; scores.g = g;
    auto scores_of = [&](int64_t first, int64_t n, const Words& w) {
        scores.x = w.p; scores.ldx = w.ld; scores.x_plane = w.plane; scores.x_rows = w.rows;
        scores.M = (int)n; scores.first_word = (int)first;
    };

    if (forward) {
        int tiles = 0;
        for (int64_t first = 0; first < c.J; first += piece) {
            const int64_t n = c.J - first < piece ? c.J - first : piece;
            Words w;
            e = words(first, n, &w);
            if (e != hipSuccess) return e;
            scores_of(first, n, w);
            const XentTile t = tile_for(n, n_some);
            scores.partial = (float2*)(ws + l.partial) + (int64_t)tiles * l.n_padded;
            e = launch_product<false, false, kXeStats, float>(scores, t, s);
            if (e != hipSuccess) return e;
            tiles += (int)((n + kXeTileM[t] - 1) / kXeTileM[t]);
        }
        hipLaunchKernelGGL(xent_loss_kernel, dim3((uint32_t)((n_some + 3) / 4)), dim3(256), 0, s, (const float2*)(ws + l.partial), tiles, (int)l.n_padded,
                           (const int*)rows, (const int*)count, (const float*)(ws + l.z), c.loss, c.lse, lse, loss);
        if (c.total)
            hipLaunchKernelGGL(xent_total_kernel, dim3(1), dim3(1024), 0, s, (const float*)loss, (const float*)g, (const int*)count, c.total);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    } else {
        hipLaunchKernelGGL(xent_gather_kernel, dim3((uint32_t)((n_some + 255) / 256)), dim3(256), 0, s, (const float*)c.lse, (const int*)rows, (const int*)count, lse);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!grads) return hipSuccess;

    bf16_t* const U = (bf16_t*)(ws + l.u);
    const int64_t u_plane = l.n_padded * piece, acc_plane = l.n_padded * l.ld_acc;
    for (int64_t first = 0; first < c.J; first += piece) {
        const int64_t n = c.J - first < piece ? c.J - first : piece;
        Words w;
        e = words(first, n, &w);
        if (e != hipSuccess) return e;
        scores_of(first, n, w);
        scores.u = U; scores.ldu = piece; scores.u_plane = u_plane; scores.u_terms = l.u_terms;
        e = launch_product<false, false, kXeU, float>(scores, tile_for(n, n_some), s);
        if (e != hipSuccess) return e;
        if (c.dA) {
            XentProduct p{};
            p.x = w.p; p.ldx = w.ld; p.x_plane = w.plane; p.x_rows = w.rows; p.x_cols = direct ? (int)c.D : (int)l.ld_w;
            p.y = U; p.ldy = piece; p.y_plane = u_plane; p.y_rows = (int)l.n_padded;
            p.M = (int)c.D; p.N = (int)n_some;
            p.k_tiles = (int)((n + 63) / 64); p.last_y = 64 * (p.k_tiles - 1);
            // a bf16 dA is rounded to 2^-9 itself: the second terms' own products are beside it
            p.pairs = pair_list(l.w_terms, l.u_terms, c.a_bf16 ? (l.w_terms > 1 ? 1 : 0) : 2, &p.pair_x, &p.pair_y);
            p.splits = l.splits;
            p.count = count; p.n_is_rows = true;
            p.out = ws + l.acc; p.ldo = l.ld_acc; p.out_plane = acc_plane; p.wide = true;
            p.add = first > 0 ? (const float*)(ws + l.acc) : nullptr; p.ld_add = l.ld_acc;
            e = launch_product<true, false, kXeStore, float>(p, tile_for(c.D, n_some), s);
            if (e != hipSuccess) return e;
        }
        if (c.dW) {
            XentProduct p{};
            p.x = A; p.ldx = l.ld_a; p.x_plane = a_plane; p.x_rows = (int)l.n_padded; p.x_cols = (int)l.ld_w;
            p.y = U; p.ldy = piece; p.y_plane = u_plane; p.y_rows = (int)l.n_padded; p.y_cols = (int)piece;
            p.M = (int)c.D; p.N = (int)n;
            p.k_tiles = (int)((n_some + 63) / 64);
            p.pairs = pair_list(l.a_terms, l.u_terms, c.w_bf16 ? (l.a_terms > 1 ? 1 : 0) : 2, &p.pair_x, &p.pair_y);
            p.splits = 1;
            p.count = count; p.k_is_rows = true;
            p.ldo = c.lddw;
            if (c.w_bf16) {
                p.out = (bf16_t*)c.dW + first * c.lddw;
                p.wide = c.lddw % 8 == 0 && ((uintptr_t)c.dW % 16) == 0;
                const XentTile t = ((c.D + 255) / 256) * ((n + 255) / 256) >= 192 ? kXe256x256 : kXe128x128;
                e = launch_product<true, true, kXeStore, bf16_t>(p, t, s);
            } else {
                p.out = (float*)c.dW + first * c.lddw;
                p.wide = c.lddw % 4 == 0 && ((uintptr_t)c.dW % 16) == 0;
                const XentTile t = ((c.D + 255) / 256) * ((n + 255) / 256) >= 192 ? kXe256x256 : kXe128x128;
                e = launch_product<true, true, kXeStore, float>(p, t, s);
            }
            if (e != hipSuccess) return e;
        }
    }
    if (c.dA) {
        const uint32_t grid = (uint32_t)((n_some * ((c.D + 3) / 4) + 255) / 256);
        if (c.a_bf16)
            hipLaunchKernelGGL(xent_rows_out_kernel<bf16_t>, dim3(grid), dim3(256), 0, s, (const float*)(ws + l.acc), l.ld_acc, acc_plane, l.splits,
                               (const int*)rows, (const int*)count, (int)c.D, (bf16_t*)c.dA, c.ldda);
        else
            hipLaunchKernelGGL(xent_rows_out_kernel<float>, dim3(grid), dim3(256), 0, s, (const float*)(ws + l.acc), l.ld_acc, acc_plane, l.splits,
                               (const int*)rows, (const int*)count, (int)c.D, (float*)c.dA, c.ldda);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace sfb
