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

__device__ __forceinline__ float aw_first(uint32_t code) {               // sign, e4m3
    const uint32_t mag = code & 0x7f;
    float x = mag < 8 ? (float)mag * 0x1p-9f : __uint_as_float((mag << 20) + (120u << 23));
    if (mag == 0x7f) x = __builtin_nanf("");
    return code & 0x80 ? -x : x;
}
__device__ __forceinline__ float aw_second(uint32_t code) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(code << 7));
}

// eight elements at any address; those at and beyond `left` read as 0
template <class T, bool WIDE>
__device__ __forceinline__ void aw_load(const T* p, int left, float (&x)[8]) {
    if constexpr (WIDE) {
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
template <bool WIDE>
__device__ __forceinline__ uint64_t aw_codes(const uint8_t* p, int left) {
    if constexpr (WIDE) return *reinterpret_cast<const uint64_t*>(p);
    uint64_t x = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) x |= e < left ? (uint64_t)p[e] << (8 * e) : 0ull;
    return x;
}
template <class T, bool WIDE>
__device__ __forceinline__ void aw_store(T* p, int left, const float (&x)[8]) {
    if constexpr (WIDE) {
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
template <bool WIDE>
__device__ __forceinline__ void aw_store_codes(uint8_t* p, int left, uint64_t x) {
    if constexpr (WIDE) {
        *reinterpret_cast<uint64_t*>(p) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = (uint8_t)(x >> (8 * e));
    }
}

struct AwNow {
    float scale, lr, c1, c2;                                             // of the gradient, the rate, 1 - b1^t and 1 - b2^t
    uint32_t key;
};

template <class G, int BITS, bool WIDE>
__device__ __forceinline__ void aw_elements(const AdamwTensor& t, const AdamwRates& r, const AwNow& now, int64_t at, int left) {
#pragma clang fp contract(off)
    float p[8], g[8], m[8], v[8];
    aw_load<G, WIDE>((const G*)t.g + at, left, g);
    aw_load<float, WIDE>(t.p + at, left, p);
    uint64_t mc = 0, vc = 0;
    if constexpr (BITS == 32) {
        aw_load<float, WIDE>((const float*)t.m + at, left, m);
        aw_load<float, WIDE>((const float*)t.v + at, left, v);
    } else {
        mc = aw_codes<WIDE>((const uint8_t*)t.m + at, left);
        vc = aw_codes<WIDE>((const uint8_t*)t.v + at, left);
        const float ms = aw_pow2((int)t.m_scale[at >> 7] - 127), vs = aw_pow2((int)t.v_scale[at >> 7] - 127);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = aw_first((uint32_t)(mc >> (8 * e)) & 0xff) * ms;
            v[e] = aw_second((uint32_t)(vc >> (8 * e)) & 0xff) * vs;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = g[e] * now.scale;
        m[e] = m[e] * r.beta1 + x * r.one_beta1;
        v[e] = v[e] * r.beta2 + x * x * r.one_beta2;
        const float move = (m[e] / now.c1) / (sqrtf(v[e] / now.c2) + r.eps);
        p[e] = p[e] - now.lr * (move + r.decay * p[e]);
    }
    aw_store<float, WIDE>(t.p + at, left, p);
    if (t.copy) aw_store<bf16_t, WIDE>((bf16_t*)t.copy + at, left, p);
    if constexpr (BITS == 32) {
        aw_store<float, WIDE>((float*)t.m + at, left, m);
        aw_store<float, WIDE>((float*)t.v + at, left, v);
    } else {
        float top_m = 0.f, top_v = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            top_m = fmaxf(top_m, e < left ? aw_finite(m[e]) : 0.f);
            top_v = fmaxf(top_v, e < left ? aw_finite(v[e]) : 0.f);
        }
        const int km = aw_scale<7>(aw_row_max(top_m)), kv = aw_scale<14>(aw_row_max(top_v));
        const float dm = aw_pow2(-km), dv = aw_pow2(-kv);
        const uint64_t number = (uint64_t)t.first * 128u + (uint64_t)at;
        uint32_t key = now.key ^ ((uint32_t)(number >> 32) * 0x9E3779B9u);
        uint64_t mo = 0, vo = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t h = aw_mix((uint32_t)(number + e) ^ key);
            const uint32_t a = aw_code<7, 0x7f>(fabsf(m[e]) * dm, h & 0xffffu) | (__float_as_uint(m[e]) >> 31 << 7);
            uint32_t b = aw_code<15, 0xff>(v[e] * dv, h >> 16);
            if (v[e] > 0.f) b = max(b, 1u);
            mo |= (uint64_t)a << (8 * e);
            vo |= (uint64_t)b << (8 * e);
        }
        aw_store_codes<WIDE>((uint8_t*)t.m + at, left, mo);
        aw_store_codes<WIDE>((uint8_t*)t.v + at, left, vo);
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
    // 1 - b^t; log b in 64 bits from the host
    now.c1 = (float)-expm1((double)step * r.log_beta1);
    now.c2 = (float)-expm1((double)step * r.log_beta2);
    now.key = aw_mix(r.seed + (uint32_t)step * 0x9E3779B9u);
    const int i = aw_tensor_of(table, blockIdx.x);
    const AdamwTensor t = table.t[i];
    const int64_t begin = (int64_t)(blockIdx.x - table.first_chunk[i]) * kAwChunk;
    if (t.wide && begin + kAwChunk <= t.n) {
#pragma unroll
        for (int k = 0; k < kAwRounds; ++k) aw_elements<G, BITS, true>(t, r, now, begin + (k * kAwThreads + threadIdx.x) * kAwPer, 8);
    } else {
#pragma unroll 1
        for (int k = 0; k < kAwRounds; ++k) {
            const int64_t at = begin + (k * kAwThreads + threadIdx.x) * kAwPer;
            const int64_t left = t.n - at;
            // threads behind the end go along (the block's maximum is over all 16 lanes), at the tensor's last element, storing nothing
            aw_elements<G, BITS, false>(t, r, now, left > 0 ? at : ((t.n - 1) & ~(int64_t)7), left > 8 ? 8 : left > 0 ? (int)left : 0);
        }
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
    const bool wide = t.wide && begin + kAwChunk <= t.n;
    for (int k = 0; k < kAwRounds; ++k) {
        const int64_t at = begin + (k * kAwThreads + threadIdx.x) * kAwPer;
        if (at >= t.n) return;
        const int left = t.n - at > 8 ? 8 : (int)(t.n - at);
        const uint64_t mc = wide ? aw_codes<true>((const uint8_t*)t.m + at, 8) : aw_codes<false>((const uint8_t*)t.m + at, left);
        const uint64_t vc = wide ? aw_codes<true>((const uint8_t*)t.v + at, 8) : aw_codes<false>((const uint8_t*)t.v + at, left);
        const float ms = aw_pow2((int)t.m_scale[at >> 7] - 127), vs = aw_pow2((int)t.v_scale[at >> 7] - 127);
        float m[8], v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = aw_first((uint32_t)(mc >> (8 * e)) & 0xff) * ms;
            v[e] = aw_second((uint32_t)(vc >> (8 * e)) & 0xff) * vs;
        }
        if (wide) {
            aw_store<bf16_t, true>((bf16_t*)t.p + at, 8, m);             // (outputs travel in p and copy)
            aw_store<bf16_t, true>((bf16_t*)t.copy + at, 8, v);
        } else {
            aw_store<bf16_t, false>((bf16_t*)t.p + at, left, m);
            aw_store<bf16_t, false>((bf16_t*)t.copy + at, left, v);
        }
    }
}

// Splits the list into launches of at most kAdamwTensors tensors and 2^30 workgroups.
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
            if (chunks + c > (1 << 30) && table.count > 0) break;
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
constexpr int kGnChunk = 16384;

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
__device__ __forceinline__ double gn_block_sum(double x) {               // four wavefronts; in thread 0
    __shared__ double part[4];
    x = gn_wave_sum(x);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

template <class G>
__global__ __launch_bounds__(kAwThreads) void grad_norm_kernel(const GradTable table, double* __restrict__ partial) {
    const int i = aw_tensor_of(table, blockIdx.x);
    const GradTensor t = table.t[i];
    const G* const g = (const G*)t.g;
    const int64_t begin = (int64_t)(blockIdx.x - table.first_chunk[i]) * kGnChunk;
    double s[8] = {};
    if (t.wide && begin + kGnChunk <= t.n) {
#pragma unroll
        for (int k = 0; k < kGnChunk / (kAwThreads * 8); ++k) {
            float x[8];
            aw_load<G, true>(g + begin + (k * kAwThreads + threadIdx.x) * 8, 8, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = __builtin_fma((double)x[e], (double)x[e], s[e]);
        }
    } else {
        for (int64_t at = begin + threadIdx.x; at < t.n && at < begin + kGnChunk; at += kAwThreads) {
            float x;
            if constexpr (sizeof(G) == 4) x = g[at];
            else x = bf16_to_f32(g[at]);
            s[0] = __builtin_fma((double)x, (double)x, s[0]);
        }
    }
    const double sum = gn_block_sum(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kAwThreads) void grad_norm_sum_kernel(const double* __restrict__ partial, int64_t n, float max_norm,
                                                                   float* __restrict__ out) {
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kAwThreads) s += partial[i];
    s = gn_block_sum(s);
    if (threadIdx.x == 0) {
        const double norm = sqrt(s), f = (double)max_norm / norm;
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
            if (chunks + c > (1 << 30) && table.count > 0) break;
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
    hipLaunchKernelGGL(grad_norm_sum_kernel, dim3(1), dim3(kAwThreads), 0, s, (const double*)partial, before, max_norm, out);
    return hipGetLastError();
}

}  // namespace sfb
