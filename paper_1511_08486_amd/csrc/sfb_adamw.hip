// AdamW over many tensors in one pass, with moments in fp32 or in 8 bits, and the norm of many gradients.
//
// With g' = s g (s: the clip factor, or 1), t the step being taken:
//   m <- b1 m + (1 - b1) g'          v <- b2 v + (1 - b2) g'^2
//   p <- p - lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay p)
// Every element is read and written once, so the traffic is all of it: 28 bytes an element with fp32 gradients and moments,
// 16.03 with 8-bit ones.  p is moved by the moments before these are rounded to 8 bits.
//
// Moments in 8 bits, blocks of 128 elements, a power of two for each (its exponent + 127 in a byte):
//   m   sign, 4 exponent bits of bias 7, 3 mantissa bits; the block's largest magnitude lands in [2^7, 2^8)
//   v   5 exponent bits of bias 15, 3 mantissa bits, the upper half of an fp16 number without its sign; largest in [2^14, 2^15)
// A step moves v by a thousandth or so (1 - b2) and the codes are an eighth apart: rounding to the nearest would leave v where it is for
// ever, so both are rounded up with the probability of the part that is cut off (16 random bits each, from the seed, the step and the
// element's number).  v keeps its smallest code rather than becoming 0: a 0 under a moment that is not would throw p by m / eps.
// What is not finite takes the codes 0x7f and 0xff, NaN in both formats, and no part in the scale.
//
// Eight consecutive elements a thread: 16 lanes are one block, its largest value found by four DPP steps, no LDS.  The tensors' table
// travels in the launch's arguments (nothing is uploaded, a captured launch keeps its own copy), 44 tensors a launch.
#include "sfb_device.h"
#include "sfb_kernels.h"

namespace sfb {

constexpr int kAwThreads = 256, kAwPer = 8, kAwChunk = 4096;             // elements a workgroup takes
constexpr int kAwRounds = kAwChunk / (kAwThreads * kAwPer);
constexpr int kAwLaunch = (1 << 24) - 1;                                 // workgroups of a launch: it has fewer than 2^32 threads

struct AdamwTable {
    AdamwTensor t[kAdamwTensors];
    int32_t first_chunk[kAdamwTensors + 1];                              // workgroups before each tensor's
    int32_t count;
};

// the last i with first[i] <= x: uniform
template <class Table>
__device__ __forceinline__ int aw_tensor_of(const Table& table, int x) {
    int lo = 0, hi = table.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (table.first_chunk[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ uint32_t aw_mix(uint32_t x) {                 // the fractions of sqrt(2) and sqrt(3), made odd, as multipliers
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

// largest of the 16 lanes of a row, in all of them
template <int CTRL>
__device__ __forceinline__ float aw_dpp_max(float x) {
    return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, 0xf, 0xf, true)));
}
__device__ __forceinline__ float aw_row_max(float x) {
    x = aw_dpp_max<0xB1>(x);                                             // lanes 1, 0, 3, 2
    x = aw_dpp_max<0x4E>(x);                                             // lanes 2, 3, 0, 1
    x = aw_dpp_max<0x141>(x);                                            // the other four of eight
    return aw_dpp_max<0x140>(x);                                         // the other eight
}

// exponent of a block's scale
template <int BELOW>
__device__ __forceinline__ int aw_scale(float largest) {
    const int k = (int)(__float_as_uint(largest) >> 23) - 127 - BELOW;
    return min(max(k, -100), 120);
}
__device__ __forceinline__ float aw_pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// code of x >= 0 (already divided by its scale); r: 16 random bits
template <int BIAS, int NAN_CODE>
__device__ __forceinline__ uint32_t aw_code(float x, uint32_t r) {
#pragma clang fp contract(off)
    constexpr float step = BIAS == 7 ? 512.f : 131072.f;                 // one over the smallest code
    const uint32_t normal = ((__float_as_uint(x) + (r << 4)) >> 20) - ((127 - BIAS) << 3);
    const float s = x * step;
    const uint32_t low = (uint32_t)floorf(s + (float)r * 0x1p-16f);
    const uint32_t code = s < 8.f ? low : normal;
    return x < __builtin_inff() ? code : (uint32_t)NAN_CODE;             // (false for NaN as well)
}
__device__ __forceinline__ float aw_finite(float x) { return fabsf(x) < __builtin_inff() ? fabsf(x) : 0.f; }

__device__ __forceinline__ float aw_second(uint32_t code) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(code << 7));
}
// values of eight codes
__device__ __forceinline__ void aw_firsts(uint2 c, float scale, float (&x)[8]) {
    x[0] = __builtin_amdgcn_cvt_f32_fp8(c.x, 0); x[1] = __builtin_amdgcn_cvt_f32_fp8(c.x, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8(c.x, 2); x[3] = __builtin_amdgcn_cvt_f32_fp8(c.x, 3);
    x[4] = __builtin_amdgcn_cvt_f32_fp8(c.y, 0); x[5] = __builtin_amdgcn_cvt_f32_fp8(c.y, 1);
    x[6] = __builtin_amdgcn_cvt_f32_fp8(c.y, 2); x[7] = __builtin_amdgcn_cvt_f32_fp8(c.y, 3);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= scale;
}
__device__ __forceinline__ void aw_seconds(uint2 c, float scale, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = aw_second((c.x >> (8 * e)) & 0xff) * scale;
        x[4 + e] = aw_second((c.y >> (8 * e)) & 0xff) * scale;
    }
}

// Eight elements: at once (`wide`), or one by one at any address, those at and beyond `left` read as 0 and not written
template <class T>
__device__ __forceinline__ void aw_load(const T* p, bool wide, int left, float (&x)[8]) {
    if (wide) {
        if constexpr (sizeof(T) == 4) {
            const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
        } else {
            const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(a[e] << 16); x[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u); }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (sizeof(T) == 4) x[e] = e < left ? p[e] : 0.f;
            else x[e] = e < left ? bf16_to_f32(p[e]) : 0.f;
        }
    }
}
__device__ __forceinline__ uint2 aw_codes(const uint8_t* p, bool wide, int left) {
    if (wide) return *reinterpret_cast<const uint2*>(p);
    uint2 x = make_uint2(0u, 0u);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x.x |= e < left ? (uint32_t)p[e] << (8 * e) : 0u;
        x.y |= 4 + e < left ? (uint32_t)p[4 + e] << (8 * e) : 0u;
    }
    return x;
}
template <class T>
__device__ __forceinline__ void aw_store(T* p, bool wide, int left, const float (&x)[8]) {
    if (wide) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
        } else {
            *reinterpret_cast<u32x4*>(p) = u32x4{cvt_pk_bf16(x[0], x[1]), cvt_pk_bf16(x[2], x[3]), cvt_pk_bf16(x[4], x[5]), cvt_pk_bf16(x[6], x[7])};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) {
                if constexpr (sizeof(T) == 4) p[e] = x[e];
                else p[e] = f32_to_bf16(x[e]);
            }
    }
}
__device__ __forceinline__ void aw_store_codes(uint8_t* p, bool wide, int left, uint2 x) {
    if (wide) {
        *reinterpret_cast<uint2*>(p) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e < left) p[e] = (uint8_t)(x.x >> (8 * e));
            if (4 + e < left) p[4 + e] = (uint8_t)(x.y >> (8 * e));
        }
    }
}

struct AwNow {
    float scale, lr, by_c1, by_c2;                                       // of the gradient, the rate, 1 / (1 - b1^t) and 1 / (1 - b2^t)
    uint32_t key;
};

// left < 8: the tensor ends among the thread's elements, or before them (left = 0; the thread goes along for its block's maximum)
template <class G, int BITS, bool WHOLE>
__device__ __forceinline__ void aw_elements(const AdamwTensor& t, const AdamwRates& r, const AwNow& now, int64_t at, int left) {
#pragma clang fp contract(off)
    const bool wide = WHOLE || (t.wide && left == 8);
    float p[8], g[8], m[8], v[8];
    aw_load((const G*)t.g + at, wide, left, g);
    aw_load(t.p + at, wide, left, p);
    if constexpr (BITS == 32) {
        aw_load((const float*)t.m + at, wide, left, m);
        aw_load((const float*)t.v + at, wide, left, v);
    } else {
        const uint2 mc = aw_codes((const uint8_t*)t.m + at, wide, left), vc = aw_codes((const uint8_t*)t.v + at, wide, left);
        aw_firsts(mc, aw_pow2((int)t.m_scale[at >> 7] - 127), m);
        aw_seconds(vc, aw_pow2((int)t.v_scale[at >> 7] - 127), v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = g[e] * now.scale;
        m[e] = m[e] * r.beta1 + x * r.one_beta1;
        v[e] = v[e] * r.beta2 + x * x * r.one_beta2;
        // square root and reciprocal to one unit in the last place: p moves by lr of this, and is rounded itself
        const float move = (m[e] * now.by_c1) * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[e] * now.by_c2) + r.eps);
        p[e] = p[e] - now.lr * (move + r.decay * p[e]);
    }
    aw_store(t.p + at, wide, left, p);
    if (t.copy) aw_store((bf16_t*)t.copy + at, wide, left, p);
    if constexpr (BITS == 32) {
        aw_store((float*)t.m + at, wide, left, m);
        aw_store((float*)t.v + at, wide, left, v);
    } else {
        float top_m = 0.f, top_v = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            top_m = fmaxf(top_m, aw_finite(m[e]));                       // (elements that are not there are 0)
            top_v = fmaxf(top_v, aw_finite(v[e]));
        }
        const int km = aw_scale<7>(aw_row_max(top_m)), kv = aw_scale<14>(aw_row_max(top_v));
        const float dm = aw_pow2(-km), dv = aw_pow2(-kv);
        const uint64_t number = (uint64_t)t.first * 128u + (uint64_t)at;
        const uint32_t key = now.key ^ ((uint32_t)(number >> 32) * 0x9E3779B9u);
        uint32_t mo[2] = {0u, 0u}, vo[2] = {0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t h = aw_mix((uint32_t)(number + e) ^ key);
            const uint32_t a = aw_code<7, 0x7f>(fabsf(m[e]) * dm, h & 0xffffu) | (__float_as_uint(m[e]) >> 31 << 7);
            uint32_t b = aw_code<15, 0xff>(v[e] * dv, h >> 16);
            if (v[e] > 0.f) b = max(b, 1u);
            mo[e / 4] |= a << (8 * (e % 4));
            vo[e / 4] |= b << (8 * (e % 4));
        }
        aw_store_codes((uint8_t*)t.m + at, wide, left, make_uint2(mo[0], mo[1]));
        aw_store_codes((uint8_t*)t.v + at, wide, left, make_uint2(vo[0], vo[1]));
        if ((threadIdx.x & 15) == 0 && left > 0) {
            t.m_scale[at >> 7] = (uint8_t)(km + 127);
            t.v_scale[at >> 7] = (uint8_t)(kv + 127);
        }
    }
}

template <class G, int BITS>
__global__ __launch_bounds__(kAwThreads) void adamw_kernel(const AdamwTable table, const AdamwRates r) {
    AwNow now;
    now.scale = r.grad_scale ? *r.grad_scale : 1.f;
    if (now.scale != now.scale) return;                                  // a gradient that is not finite: no step
    const int step = *r.step + 1;
    now.lr = r.lr_scale ? r.lr * *r.lr_scale : r.lr;
    // 1 - b^t, log b in 64 bits from the host: the exponent's own rounding is 2^-24 of it, and so is that of the result at most
    now.by_c1 = -1.f / expm1f((float)((double)step * r.log_beta1));
    now.by_c2 = -1.f / expm1f((float)((double)step * r.log_beta2));
    now.key = aw_mix(r.seed + (uint32_t)step * 0x9E3779B9u);
    const int i = aw_tensor_of(table, blockIdx.x);
    const AdamwTensor t = table.t[i];
    const int64_t begin = (int64_t)(blockIdx.x - table.first_chunk[i]) * kAwChunk;
    if (t.wide && begin + kAwChunk <= t.n) {
#pragma unroll
        for (int k = 0; k < kAwRounds; ++k) aw_elements<G, BITS, true>(t, r, now, begin + (k * kAwThreads + threadIdx.x) * kAwPer, 8);
        return;
    }
#pragma unroll 1
    for (int k = 0; k < kAwRounds; ++k) {
        const int64_t at = begin + (k * kAwThreads + threadIdx.x) * kAwPer, left = t.n - at;
        // (a thread behind the end reads its block's scale at the tensor's last element)
        aw_elements<G, BITS, false>(t, r, now, left > 0 ? at : ((t.n - 1) & ~(int64_t)7), left >= 8 ? 8 : left > 0 ? (int)left : 0);
    }
}

__global__ void adamw_advance_kernel(int32_t* step, const float* grad_scale) {
    const float s = grad_scale ? *grad_scale : 1.f;
    if (s == s) *step += 1;
}

// fp32 moments as bf16 numbers: four significant bits and a power of two, exact
__global__ __launch_bounds__(kAwThreads) void adamw_unpack_kernel(const AdamwTable table) {
    const int i = aw_tensor_of(table, blockIdx.x);
    const AdamwTensor t = table.t[i];
    const int64_t begin = (int64_t)(blockIdx.x - table.first_chunk[i]) * kAwChunk;
    for (int k = 0; k < kAwRounds; ++k) {
        const int64_t at = begin + (k * kAwThreads + threadIdx.x) * kAwPer;
        if (at >= t.n) return;
        const int left = t.n - at > 8 ? 8 : (int)(t.n - at);
        const bool wide = t.wide && left == 8;
        float m[8], v[8];
        aw_firsts(aw_codes((const uint8_t*)t.m + at, wide, left), aw_pow2((int)t.m_scale[at >> 7] - 127), m);
        aw_seconds(aw_codes((const uint8_t*)t.v + at, wide, left), aw_pow2((int)t.v_scale[at >> 7] - 127), v);
        aw_store((bf16_t*)t.p + at, wide, left, m);                      // (outputs travel in p and copy)
        aw_store((bf16_t*)t.copy + at, wide, left, v);
    }
}

// Splits the list into launches of at most kAdamwTensors tensors and kAwLaunch workgroups (2^36 elements).
template <class Launch>
static hipError_t aw_each_table(const AdamwTensor* t, int count, Launch launch) {
    AdamwTable table;
    int64_t first = 0;                                                   // 128-element blocks before the tensor
    int i = 0;
    while (i < count) {
        table.count = 0;
        int64_t chunks = 0;
        for (; i < count && table.count < kAdamwTensors; ++i) {
            const int64_t c = (t[i].n + kAwChunk - 1) / kAwChunk;
            if (chunks + c > kAwLaunch && table.count > 0) break;
            if (t[i].n > 0) {
                table.t[table.count] = t[i];
                table.t[table.count].first = first;
                table.first_chunk[table.count++] = (int32_t)chunks;
                chunks += c;
            }
            first += (t[i].n + 127) / 128;
        }
        if (table.count == 0) continue;
        table.first_chunk[table.count] = (int32_t)chunks;
        const hipError_t e = launch(table, (int)chunks);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_adamw(const AdamwTensor* t, int count, const AdamwRates& r, bool bf16_grads, int bits, hipStream_t s) {
    const hipError_t e = aw_each_table(t, count, [&](const AdamwTable& table, int chunks) {
        if (bits == 32) {
            if (bf16_grads) SFB_LAUNCH((adamw_kernel<bf16_t, 32>), dim3(chunks), dim3(kAwThreads), 0, s, table, r);
            else SFB_LAUNCH((adamw_kernel<float, 32>), dim3(chunks), dim3(kAwThreads), 0, s, table, r);
        } else {
            if (bf16_grads) SFB_LAUNCH((adamw_kernel<bf16_t, 8>), dim3(chunks), dim3(kAwThreads), 0, s, table, r);
            else SFB_LAUNCH((adamw_kernel<float, 8>), dim3(chunks), dim3(kAwThreads), 0, s, table, r);
        }
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(adamw_advance_kernel, dim3(1), dim3(1), 0, s, r.step, r.grad_scale);
    return hipGetLastError();
}

hipError_t launch_adamw_unpack(const AdamwTensor* t, int count, hipStream_t s) {
    return aw_each_table(t, count, [&](const AdamwTable& table, int chunks) {
        hipLaunchKernelGGL(adamw_unpack_kernel, dim3(chunks), dim3(kAwThreads), 0, s, table);
        return hipGetLastError();
    });
}

// ---------------------------------------------------------------------------------------------------------------
// norm = sqrt(sum of all g^2) in 64 bits (squares of fp32 numbers overflow fp32; the units have 64-bit products to spare beside
// the reads), added per workgroup, then by one workgroup in a fixed order.  factor = min(1, max_norm / norm), NaN if the norm is not finite.
constexpr int kGnChunk = 8192;

struct GradTable {
    GradTensor t[kGradTensors];
    int32_t first_chunk[kGradTensors + 1];
    int32_t count;
};

__device__ __forceinline__ double gn_wave_sum(double x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    return x;
}
template <int WAVES>
__device__ __forceinline__ double gn_block_sum(double x) {               // in thread 0
    __shared__ double part[WAVES];
    x = gn_wave_sum(x);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = part[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) x += part[w];
    return x;
}

template <class G>
__global__ __launch_bounds__(kAwThreads) void grad_norm_kernel(const GradTable table, double* __restrict__ partial) {
    const int i = aw_tensor_of(table, blockIdx.x);
    const GradTensor t = table.t[i];
    const G* const g = (const G*)t.g;
    const int64_t begin = (int64_t)(blockIdx.x - table.first_chunk[i]) * kGnChunk;
    double s[8] = {};
    auto add = [&](const float(&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = __builtin_fma((double)x[e], (double)x[e], s[e]);
    };
    constexpr int ROUNDS = kGnChunk / (kAwThreads * 8);
    if (t.wide && begin + kGnChunk <= t.n) {                             // a whole chunk: all of it on its way at once
        float x[ROUNDS][8];
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) aw_load(g + begin + (k * kAwThreads + threadIdx.x) * 8, true, 8, x[k]);
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) add(x[k]);
    } else {
        for (int k = 0; k < ROUNDS; ++k) {
            const int64_t at = begin + (k * kAwThreads + threadIdx.x) * 8, left = t.n - at;
            if (left <= 0) break;
            float x[8];
            aw_load(g + at, t.wide && left >= 8, left >= 8 ? 8 : (int)left, x);
            add(x);
        }
    }
    const double sum = gn_block_sum<kAwThreads / 64>(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void grad_norm_sum_kernel(const double* __restrict__ partial, int64_t n, float max_norm, float* __restrict__ out) {
    double s[8] = {};
    for (int64_t i = threadIdx.x; i < n; i += 8192)                      // eight on their way at a time
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += i + 1024 * k < n ? partial[i + 1024 * k] : 0.0;
    const double sum = gn_block_sum<16>(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum), f = (double)max_norm / norm;
        out[0] = (float)norm;
        out[1] = !(norm < __builtin_inf()) ? __builtin_nanf("") : f < 1.0 ? (float)f : 1.f;
    }
}

int64_t grad_norm_chunks(const GradTensor* t, int count) {
    int64_t n = 0;
    for (int i = 0; i < count; ++i) n += (t[i].n + kGnChunk - 1) / kGnChunk;
    return n;
}

hipError_t launch_grad_norm(const GradTensor* t, int count, bool bf16, float max_norm, float* out, double* partial, hipStream_t s) {
    GradTable table;
    int64_t before = 0;
    int i = 0;
    while (i < count) {
        table.count = 0;
        int64_t chunks = 0;
        for (; i < count && table.count < kGradTensors; ++i) {
            const int64_t c = (t[i].n + kGnChunk - 1) / kGnChunk;
            if (c == 0) continue;
            if (chunks + c > kAwLaunch && table.count > 0) break;
            table.t[table.count] = t[i];
            table.first_chunk[table.count++] = (int32_t)chunks;
            chunks += c;
        }
        if (table.count == 0) continue;
        table.first_chunk[table.count] = (int32_t)chunks;
        if (bf16) SFB_LAUNCH(grad_norm_kernel<bf16_t>, dim3((uint32_t)chunks), dim3(kAwThreads), 0, s, table, partial + before);
        else SFB_LAUNCH(grad_norm_kernel<float>, dim3((uint32_t)chunks), dim3(kAwThreads), 0, s, table, partial + before);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        before += chunks;
    }
    hipLaunchKernelGGL(grad_norm_sum_kernel, dim3(1), dim3(1024), 0, s, (const double*)partial, before, max_norm, out);
    return hipGetLastError();
}

}  // namespace sfb
