// One AdamW step over many tensors: the descriptors of up to 48 tensors travel as kernel arguments, a workgroup finds its tensor
// from its number and takes kAdamwChunk values of it.
#include "groot_dense_device.h"

namespace groot {

namespace {

constexpr int kAdamwTensors = 48;            // 72 bytes each: the arguments stay below 4 KB
constexpr int kAdamwPerLane = 4;             // neighbouring values of a lane: a wavefront takes one block of 256
constexpr int kAdamwChunk = 2 * kBlock * kAdamwPerLane;
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
        const v4t x = *(const v4t *)p;
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
        *(v4t *)p = r;
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
        c = *(const uint32_t *)p;
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

// x on the grid of the codes: |x| / step + u rounded down.  step is a power of two and |x| / step below 16, so both are exact and
// the sum is rounded once, at 2^-20.
__device__ __forceinline__ float on_grid(float x, float u)
{
    const float a = __builtin_fabsf(x);
    int e = (int)(__float_as_uint(a) >> 23) - 127;
    e = e < -6 ? -6 : e;
    const float inverse = __uint_as_float((uint32_t)(127 + 3 - e) << 23), step = __uint_as_float((uint32_t)(127 - 3 + e) << 23);
    const float r = fminf(floorf(a * inverse + u) * step, kCodeTop);
    return __builtin_copysignf(r, x);
}

// Codes and scale of the wavefront's 256 values: the scale takes the largest finite magnitude to the largest code.  `never0`: a
// positive value is held as the smallest code at least (a root of 0 beside a first moment above 0 is a step of m / eps).
template <bool kWhole>
__device__ __forceinline__ void store_codes(uint8_t *p, float *scale_at, v4f x, const uint32_t (&u16)[4], bool never0, int left)
{
#pragma clang fp contract(off)
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float a = __builtin_fabsf(x[k]);
        if (__builtin_isfinite(a) && (kWhole || k < left)) top = fmaxf(top, a);
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float scale = top * (1.f / kCodeTop);
    v4f r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float over = scale > 0.f ? x[k] / scale : 0.f;
        r[k] = on_grid(over, (float)u16[k] * 0x1p-16f);
        if (never0 && x[k] > 0.f && r[k] == 0.f) r[k] = kCodeLeast;
        if (!__builtin_isfinite(x[k])) r[k] = __builtin_nanf("");
    }
    uint32_t c = __builtin_amdgcn_cvt_pk_fp8_f32(r[0], r[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(r[2], r[3], c, true);
    if (kWhole) {
        *(uint32_t *)p = c;
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
    v4f root;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float gk = scaled ? g[k] * gs : g[k];
        m[k] = m[k] * f.beta1 + gk * f.one_minus_beta1;
        v[k] = v[k] * f.beta2 + (gk * gk) * f.one_minus_beta2;
        root[k] = sqrtf(v[k]);
        w[k] = w[k] * f.decay - f.step_size * (m[k] / (root[k] * f.root_factor + f.eps));
    }
    if (kMaster) store4<float, kWhole>(master, w, left);
    store4<P, kWhole>(param, w, left);
    if (kBits == 8) {
        const uint32_t key = t.key + (uint32_t)(at >> 32) * 0x9E3779B9u;
        uint32_t low[4], high[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t h = mixed((uint32_t)(at + k) ^ key);
            low[k] = h & 0xFFFFu;
            high[k] = h >> 16;
        }
        store_codes<kWhole>((uint8_t *)t.m + at, t.m_scale + block, m, low, false, left);
        store_codes<kWhole>((uint8_t *)t.v + at, t.v_scale + block, root, high, true, left);
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
    const int64_t from = (int64_t)(chunk - before) * kAdamwChunk;
    if (!(t.chunks_to & kUnaligned) && from + kAdamwChunk <= t.n) {
#pragma unroll
        for (int i = 0; i < kAdamwChunk; i += kBlock * kAdamwPerLane)
            adamw_values<P, G, kMaster, kBits, true>(t, b.f, gs, scaled, from + i + threadIdx.x * kAdamwPerLane);
        return;
    }
    for (int i = 0; i < kAdamwChunk; i += kBlock * kAdamwPerLane) {
        const int64_t wave = from + i + threadIdx.x / kWave * kAdamwBlock;      // the same for the whole wavefront
        if (wave < t.n) adamw_values<P, G, kMaster, kBits, false>(t, b.f, gs, scaled, wave + lane * kAdamwPerLane);
    }
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
    constexpr uint32_t kMostChunks = (1u << 24) - 1;      // a launch holds 2^32 lanes
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
        const int64_t mine = (x.n + kAdamwChunk - 1) / kAdamwChunk;              // at most 2^23 for n below 2^34
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
