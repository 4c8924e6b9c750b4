// One AdamW step over many tensors: the descriptors of up to 48 tensors travel as kernel arguments, a workgroup finds its tensor
// from its number and takes kAdamwChunk values of it, four to a lane.
// Bound by HBM: 16.06 bytes a value with states in 8 bits, bfloat16 parameters and a master (400 M values: 1.08 to 1.11 ms from card to
// card, 5.8 to 5.95 TB/s), 28 with fp32 all through (100 M: 0.44 ms, 6.3 TB/s); a large copy reaches 6.2.  Nothing is read or written
// twice, so loads and stores are told not to keep their lines (without: 1.12 where it took 1.06, and 0.51), and every workgroup has one
// set of loads (with two: 1.25 and 0.52 ms).
#include "groot_dense_device.h"

namespace groot {

namespace {

constexpr int kAdamwTensors = 48;            // 72 bytes each: the arguments stay below 4 KB
constexpr int kAdamwPerLane = 4;             // neighbouring values of a lane: a wavefront takes one block of 256
constexpr int kAdamwChunk = kBlock * kAdamwPerLane;
constexpr float kCodeTop = 448.f, kCodeLeast = 0x1p-9f;
static_assert(kWave * kAdamwPerLane == kAdamwBlock, "a wavefront's values share a scale");

struct AdamwTensor {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    int64_t n;
    uint32_t key;                            // of its random numbers
    uint32_t chunks_to;                      // chunks of this and the tensors before it; the top bit: not every array begins on 16 bytes
};

struct AdamwBatch {
    AdamwTensor t[kAdamwTensors];
    AdamwFactors f;
    const float *grad_scale;
    int32_t count;
};
static_assert(sizeof(AdamwBatch) <= 4096, "kernel arguments");

constexpr uint32_t kUnaligned = 0x80000000u;

__host__ __device__ __forceinline__ uint32_t mixed(uint32_t h)
{
    h ^= h >> 16;
    h *= 0x85EBCA6Bu;
    h ^= h >> 13;
    h *= 0xC2B2AE35u;
    return h ^ (h >> 16);
}

// four neighbouring values as floats; `left` of them exist
template <typename T, bool kWhole>
__device__ __forceinline__ v4f load4(const T *p, int left)
{
    typedef T v4t __attribute__((ext_vector_type(4)));
    v4f r = {0.f, 0.f, 0.f, 0.f};
    if (kWhole) {
        const v4t x = __builtin_nontemporal_load((const v4t *)p);
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = (float)x[k];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < left) r[k] = (float)p[k];
    }
    return r;
}

template <typename T, bool kWhole>
__device__ __forceinline__ void store4(T *p, v4f x, int left)
{
    typedef T v4t __attribute__((ext_vector_type(4)));
    if (kWhole) {
        v4t r;
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = (T)x[k];      // rounded to nearest, once
        __builtin_nontemporal_store(r, (v4t *)p);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < left) p[k] = (T)x[k];
    }
}

template <bool kWhole>
__device__ __forceinline__ v4f load_codes(const uint8_t *p, float scale, int left)
{
    uint32_t c = 0;
    if (kWhole) {
        c = __builtin_nontemporal_load((const uint32_t *)p);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < left) c |= (uint32_t)p[k] << (8 * k);
    }
    v4f r;
    r[0] = __builtin_amdgcn_cvt_f32_fp8(c, 0) * scale;
    r[1] = __builtin_amdgcn_cvt_f32_fp8(c, 1) * scale;
    r[2] = __builtin_amdgcn_cvt_f32_fp8(c, 2) * scale;
    r[3] = __builtin_amdgcn_cvt_f32_fp8(c, 3) * scale;
    return r;
}

// Square roots and quotients of 8-bit states, rounded as the mathematical library's and the division's, from three and six instructions
// each where all values of the wavefront are of an ordinary size.  (Where a value takes 16 bytes, the library's bound the kernel: 115
// instructions a value in all.)  The instructions behind them were compared with fp64, rounded, for every value of their ranges: a
// reciprocal is off in a ninth of the cases by itself and in none with one step of Newton's, a root with its remainder in none.
// ordinary: |m| in (2^-80, 2^60), v in (2^-96, 2^32), none of them NaN, in the whole wavefront
__device__ __forceinline__ bool ordinary(v4f m, v4f v)
{
    float least = __builtin_fabsf(m[0]), most = least, low = v[0], high = low;
#pragma unroll
    for (int k = 1; k < 4; ++k) {
        const float a = __builtin_fabsf(m[k]);
        least = fminf(least, a);
        most = __builtin_elementwise_maximum(most, a);       // NaN if one of them is
        low = fminf(low, v[k]);
        high = __builtin_elementwise_maximum(high, v[k]);
    }
    return __all(low > 0x1p-96f && high < 0x1p32f && least > 0x1p-80f && most < 0x1p60f);
}

__device__ __forceinline__ v4f roots(v4f v, bool usual)
{
    v4f r;
    if (usual) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float y = __builtin_amdgcn_rsqf(v[k]), g = v[k] * y;
            r[k] = __builtin_fmaf(__builtin_fmaf(-g, g, v[k]), 0.5f * y, g);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = sqrtf(v[k]);
    }
    return r;
}

// m / d for d of 2^-64 to 2^80 where `usual`
__device__ __forceinline__ v4f quotients(v4f m, v4f d, bool usual)
{
    v4f q;
    if (usual) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float r = __builtin_amdgcn_rcpf(d[k]);
            q[k] = quotient(m[k], d[k], __builtin_fmaf(__builtin_fmaf(-d[k], r, 1.f), r, r));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = m[k] / d[k];
    }
    return q;
}

// Codes and scale of the wavefront's 256 values: the scale takes the largest finite magnitude to the largest code.  The instruction
// adds its random number's upper 20 bits behind the three that a code keeps and cuts the rest off (below 2^-6: behind steps of 2^-9).
// `never0`: a positive value is held as the smallest code at least (a root of 0 beside a first moment above 0 is a step of m / eps).
// `usual`: the values are known to be finite.
template <bool kWhole>
__device__ __forceinline__ void store_codes(uint8_t *p, float *scale_at, v4f x, const uint32_t (&random)[4], bool never0, int left, bool usual)
{
    // one look at four values: their sum is not finite if one of them is not
    const bool finite = usual || __all(__builtin_isfinite((x[0] + x[1]) + (x[2] + x[3])));
    float top = 0.f;                                         // values that do not exist are zeros
    if (finite) {
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, __builtin_fabsf(x[k]));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, __builtin_isfinite(x[k]) ? __builtin_fabsf(x[k]) : 0.f);
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float scale = top * (1.f / kCodeTop);
    v4f r;
    if (scale > 0x1p-96f) {                                  // the same for the whole wavefront
        const float inverse = 1.f / scale;
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = quotient(x[k], scale, inverse);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = scale > 0.f ? x[k] / scale : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        r[k] = __builtin_amdgcn_fmed3f(r[k], -kCodeTop, kCodeTop);
        if (never0 && x[k] > 0.f) r[k] = fmaxf(r[k], kCodeLeast);
    }
    uint32_t c = __builtin_amdgcn_cvt_sr_fp8_f32(r[0], random[0], 0, 0);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(r[1], random[1], c, 1);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(r[2], random[2], c, 2);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(r[3], random[3], c, 3);
    if (!finite) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (!__builtin_isfinite(x[k])) c |= 0x7Fu << (8 * k);
    }
    if (kWhole) {
        __builtin_nontemporal_store(c, (uint32_t *)p);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < left) p[k] = (uint8_t)(c >> (8 * k));
    }
    if (threadIdx.x % kWave == 0) *scale_at = scale;
}

// the values [at, at + 4) of a tensor, by one lane; all lanes of the wavefront come here
template <typename P, typename G, bool kMaster, int kBits, bool kWhole>
__device__ __forceinline__ void adamw_values(const AdamwTensor &t, const AdamwFactors &f, float gs, bool scaled, int64_t at)
{
#pragma clang fp contract(off)
    const int64_t rest = t.n - at;
    const int left = rest > 4 ? 4 : rest < 0 ? 0 : (int)rest;
    P *const param = (P *)t.param + at;
    float *const master = t.master + at;
    const int64_t block = at / kAdamwBlock;
    v4f w = kMaster ? load4<float, kWhole>(master, left) : load4<P, kWhole>(param, left);
    v4f g = load4<G, kWhole>((const G *)t.grad + at, left), m, v;
    if (kBits == 8) {
        m = load_codes<kWhole>((const uint8_t *)t.m + at, t.m_scale[block], left);
        const v4f r = load_codes<kWhole>((const uint8_t *)t.v + at, t.v_scale[block], left);
        v = r * r;
    } else {
        m = load4<float, kWhole>((const float *)t.m + at, left);
        v = load4<float, kWhole>((const float *)t.v + at, left);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float gk = scaled ? g[k] * gs : g[k];
        m[k] = m[k] * f.beta1 + gk * f.one_minus_beta1;
        v[k] = v[k] * f.beta2 + (gk * gk) * f.one_minus_beta2;
    }
    v4f root, denom, step;
    bool usual = false;
    if (kBits == 8) {
        usual = ordinary(m, v);
        root = roots(v, usual);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) root[k] = sqrtf(v[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) denom[k] = root[k] * f.root_factor + f.eps;
    if (kBits == 8) {
        step = quotients(m, denom, usual && f.eps > 0x1p-60f && f.eps < 0x1p36f && f.root_factor < 0x1p30f);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) step[k] = m[k] / denom[k];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = w[k] * f.decay - f.step_size * step[k];
    if (kMaster) store4<float, kWhole>(master, w, left);
    store4<P, kWhole>(param, w, left);
    if (kBits == 8) {
        const uint32_t key = t.key + (uint32_t)(at >> 32) * 0x9E3779B9u;
        uint32_t low[4], high[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t h = mixed((uint32_t)(at + k) ^ key);
            low[k] = h << 16;
            high[k] = h & 0xFFFF0000u;
        }
        store_codes<kWhole>((uint8_t *)t.m + at, t.m_scale + block, m, low, false, left, usual);
        store_codes<kWhole>((uint8_t *)t.v + at, t.v_scale + block, root, high, true, left, usual);
    } else {
        store4<float, kWhole>((float *)t.m + at, m, left);
        store4<float, kWhole>((float *)t.v + at, v, left);
    }
}

template <typename P, typename G, bool kMaster, int kBits>
__global__ __launch_bounds__(kBlock) void adamw_kernel(const AdamwBatch b)
{
    const uint32_t chunk = blockIdx.x;
    const int lane = threadIdx.x % kWave;
    const uint32_t to = b.t[lane < kAdamwTensors ? lane : 0].chunks_to & ~kUnaligned;
    const int which = __popcll(__ballot(lane < b.count && to <= chunk));
    if (which >= b.count) return;
    const AdamwTensor t = b.t[which];
    const uint32_t before = which ? b.t[which - 1].chunks_to & ~kUnaligned : 0;
    const bool scaled = b.grad_scale != nullptr;
    const float gs = scaled ? *b.grad_scale : 1.f;
    const int64_t wave = (int64_t)(chunk - before) * kAdamwChunk + threadIdx.x / kWave * kAdamwBlock;   // the same for the whole wavefront
    if (wave >= t.n) return;
    if (!(t.chunks_to & kUnaligned) && wave + kAdamwBlock <= t.n) adamw_values<P, G, kMaster, kBits, true>(t, b.f, gs, scaled, wave + lane * kAdamwPerLane);
    else adamw_values<P, G, kMaster, kBits, false>(t, b.f, gs, scaled, wave + lane * kAdamwPerLane);
}

template <typename P, typename G, bool kMaster>
void adamw_launch(const AdamwBatch &b, int bits, uint32_t chunks, hipStream_t stream)
{
    if (bits == 8) adamw_kernel<P, G, kMaster, 8><<<chunks, kBlock, 0, stream>>>(b);
    else adamw_kernel<P, G, kMaster, 32><<<chunks, kBlock, 0, stream>>>(b);
}

template <typename P, bool kMaster>
void adamw_launch(const AdamwBatch &b, int32_t grad_dtype, int bits, uint32_t chunks, hipStream_t stream)
{
    if (grad_dtype == GROOT_F32) adamw_launch<P, float, kMaster>(b, bits, chunks, stream);
    else if (grad_dtype == GROOT_BF16) adamw_launch<P, bf16_t, kMaster>(b, bits, chunks, stream);
    else adamw_launch<P, f16_t, kMaster>(b, bits, chunks, stream);
}

}  // namespace

int launch_adamw(const groot_adamw_tensor *tensors, int64_t n_tensors, int32_t param_dtype, int32_t grad_dtype, int32_t state_bits,
                 const AdamwFactors &f, const float *grad_scale, uint32_t step, uint32_t seed, void *stream)
{
    constexpr uint32_t kMostChunks = 1u << 23;               // a launch holds 2^32 lanes, twice as many
    AdamwBatch b;
    b.f = f;
    b.grad_scale = grad_scale;
    b.count = 0;
    uint32_t chunks = 0;
    bool master = false;
    auto flush = [&]() -> int {
        if (!b.count) return 0;
        hipStream_t s = (hipStream_t)stream;
        if (param_dtype == GROOT_F32) master ? adamw_launch<float, true>(b, grad_dtype, state_bits, chunks, s) : adamw_launch<float, false>(b, grad_dtype, state_bits, chunks, s);
        else if (param_dtype == GROOT_BF16) master ? adamw_launch<bf16_t, true>(b, grad_dtype, state_bits, chunks, s) : adamw_launch<bf16_t, false>(b, grad_dtype, state_bits, chunks, s);
        else master ? adamw_launch<f16_t, true>(b, grad_dtype, state_bits, chunks, s) : adamw_launch<f16_t, false>(b, grad_dtype, state_bits, chunks, s);
        b.count = 0;
        chunks = 0;
        return (int)hipGetLastError();
    };
    for (int64_t i = 0; i < n_tensors; ++i) {
        const groot_adamw_tensor &x = tensors[i];
        if (x.n == 0) continue;
        master = x.master != nullptr;
        const int64_t mine = (x.n + kAdamwChunk - 1) / kAdamwChunk;              // at most 2^23 for n below 2^33
        if (b.count == kAdamwTensors || mine > (int64_t)(kMostChunks - chunks))
            if (const int err = flush()) return err;
        chunks += (uint32_t)mine;
        uintptr_t any = (uintptr_t)x.param | (uintptr_t)x.grad | (uintptr_t)x.master | (uintptr_t)x.m | (uintptr_t)x.v;
        AdamwTensor &t = b.t[b.count++];
        t = AdamwTensor{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.master, x.n,
                        mixed(mixed(mixed((uint32_t)i + 0x9E3779B9u) ^ step) ^ seed), chunks | ((any & 15) ? kUnaligned : 0u)};
    }
    return flush();
}

}  // namespace groot
