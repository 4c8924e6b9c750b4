// The choice of experts for every row, their weights, and every choice's place in the order of the experts.
//   value c of an expert: its score where that orders as the probability does, otherwise softmax or sigmoid of the score, plus a bias
//   top k of c (ties to the lowest expert) among the sets whose best members' sum is largest; weights factor x p, renormalised or not
// A call cannot do without n E scores and 12 n k bytes of results.  Values that decide are compared in 64 bits, as an expert's number is
// a whole one whatever lies next to it.
//
// Places: workgroups take kRouteRows rows each.  A row chooses an expert once, so the rows of a workgroup that chose an expert are the bits
// of one 64-bit word, and a choice's rank is the number of bits below its row's: nothing depends on the order of atomics.  The ranks
// wait in `places` until the counts of all workgroups are known.
#include <cfloat>

#include "groot_dense_device.h"

namespace groot {

namespace {

constexpr int kRouteRows = 64;               // rows of a workgroup: bits of a word
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float score_at(const void *row, int32_t dtype, int32_t e)
{
    if (dtype == GROOT_F32) return ((const float *)row)[e];
    if (dtype == GROOT_BF16) return (float)((const bf16_t *)row)[e];
    return (float)((const f16_t *)row)[e];
}

template <int kLanes>
__device__ __forceinline__ double top_of(double x)
{
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) x = fmax(x, __shfl_xor(x, d));
    return x;
}
template <int kLanes>
__device__ __forceinline__ double sum_of(double x)
{
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) x += __shfl_xor(x, d);
    return x;
}
template <int kLanes>
__device__ __forceinline__ int32_t least_of(int32_t x)
{
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) {
        const int32_t o = __shfl_xor(x, d);
        x = o < x ? o : x;
    }
    return x;
}
// whether any of the row's lanes says so
template <int kLanes>
__device__ __forceinline__ bool any_of(bool x)
{
    const uint64_t all = __ballot(x);
    const int first = threadIdx.x % kWave / kLanes * kLanes;
    return (all >> first & (kLanes == kWave ? ~0ull : (1ull << (kLanes % kWave)) - 1)) != 0;
}

__device__ __forceinline__ double log_sigmoid(double x) { return fmin(x, 0.0) - log1p(exp(-fabs(x))); }

// Exclusive sums of the workgroup's first E words of LDS, in place; the sum of all goes to word E.
__device__ __forceinline__ void exclusive_sums(int32_t *x, int32_t E, int32_t *waves)
{
    const int tid = threadIdx.x, lane = tid % kWave, per = (E + kBlock - 1) / kBlock;
    int32_t mine = 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < E) mine += x[tid * per + i];
    int32_t upto = mine;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int32_t o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == kWave - 1) waves[tid / kWave] = upto;
    __syncthreads();
    int32_t before = upto - mine;
    for (int w = 0; w < tid / kWave; ++w) before += waves[w];
    for (int i = 0; i < per; ++i)
        if (tid * per + i < E) {
            const int32_t here = x[tid * per + i];
            x[tid * per + i] = before;
            before += here;
        }
    if (tid == kBlock - 1) x[E] = before;
    __syncthreads();
}

// kLanes lanes to a row, kEach experts a lane (expert v kLanes + lane)
template <int kLanes, int kEach>
__global__ __launch_bounds__(kBlock) void route_kernel(RouteArgs a, int32_t *__restrict__ counts)
{
    constexpr int kAtOnce = kBlock / kLanes;
    extern __shared__ char lds[];
    uint64_t *const mask = (uint64_t *)lds;                               // [E] the rows that chose an expert
    int32_t *const prefix = (int32_t *)(mask + a.E);                      // [E + 1]
    int32_t *const waves = prefix + a.E + 1;                              // [kWavesPerBlock]
    int16_t *const chosen = (int16_t *)(waves + kWavesPerBlock);          // [kRouteRows, k]
    double *const values = (double *)(lds + a.values_at) + threadIdx.x / kLanes * a.E;    // [E] of the row, where sets are ranked
    const int lane = threadIdx.x % kLanes;
    for (int e = threadIdx.x; e < a.E; e += kBlock) mask[e] = 0;
    __syncthreads();
    for (int local = threadIdx.x / kLanes; local < kRouteRows; local += kAtOnce) {
        const int64_t row = (int64_t)blockIdx.x * kRouteRows + local;
        const bool real = row < a.n;                                      // the lanes of a row go together, rows beyond the last idle
        const char *const scores = (const char *)a.scores + (real ? row : 0) * a.score_bytes;
        double x[kEach];
        bool broken = false;
        double top = -kInf;
#pragma unroll
        for (int v = 0; v < kEach; ++v) {
            const int32_t e = v * kLanes + lane;
            const float s = real && e < a.E ? score_at(scores, a.dtype, e) : -kInf;
            broken |= s != s || (a.gate == GROOT_SOFTMAX && s == kInf);
            x[v] = s;
            top = fmax(top, x[v]);                                        // a NaN is passed over: the row is broken
        }
        broken = any_of<kLanes>(broken);
        top = top_of<kLanes>(top);
        const double base = top == -kInf ? 0.0 : top;
        double sum = 0;
        if (a.gate == GROOT_SOFTMAX && (a.by_value || !a.renormalise)) {
#pragma unroll
            for (int v = 0; v < kEach; ++v) sum += exp(x[v] - base);
            sum = sum_of<kLanes>(sum);
        }
        auto probability = [&](double s) { return a.gate == GROOT_SOFTMAX ? exp(s - base) / sum : 1.0 / (1.0 + exp(-s)); };
        if (a.by_value) {
#pragma unroll
            for (int v = 0; v < kEach; ++v) {
                const int32_t e = v * kLanes + lane;
                double c = probability(x[v]);
                if (a.bias && e < a.E) c += (double)a.bias[e];
                x[v] = x[v] == -kInf || !(c > -kInf) ? -(double)kInf : c;  // closed
            }
        }
        if (broken) {
#pragma unroll
            for (int v = 0; v < kEach; ++v) x[v] = -kInf;
        }
        if (a.open_sets < a.sets) {                                       // the same for all rows
            const int32_t size = a.E / a.sets;
#pragma unroll
            for (int v = 0; v < kEach; ++v)
                if (v * kLanes + lane < a.E) values[v * kLanes + lane] = x[v];
            wave_sync();
            uint64_t open = 0;
            double value = -kInf;                                         // of set `lane` (rows of 16 lanes: up to four sets a lane)
            double held[kWave / kLanes];
#pragma unroll
            for (int h = 0; h < kWave / kLanes; ++h) {
                const int32_t set = h * kLanes + lane;
                double first = -kInf, second = -kInf;
                if (set < a.sets)
                    for (int32_t i = 0; i < size; ++i) {
                        const double c = values[set * size + i];
                        if (c > first) {
                            second = first;
                            first = c;
                        } else if (c > second) {
                            second = c;
                        }
                    }
                held[h] = a.set_best == 2 && second > -kInf ? first + second : first;
            }
            for (int32_t r = 0; r < a.open_sets; ++r) {
                value = -kInf;
                int32_t at = a.sets;
#pragma unroll
                for (int h = 0; h < kWave / kLanes; ++h) {
                    const int32_t set = h * kLanes + lane;
                    if (set < a.sets && !(open >> set & 1) && (at == a.sets || held[h] > value)) {
                        value = held[h];
                        at = set;
                    }
                }
                const double best = top_of<kLanes>(value);
                open |= 1ull << least_of<kLanes>(value == best ? at : a.sets);   // open_sets < sets: there is one left
            }
            wave_sync();
#pragma unroll
            for (int v = 0; v < kEach; ++v) {
                const int32_t e = v * kLanes + lane;
                if (e < a.E && !(open >> (e / size) & 1)) x[v] = -kInf;
            }
        }
        int32_t mine = -1;                                                // expert of slot `lane`
        for (int32_t slot = 0; slot < a.k; ++slot) {
            double value = x[0];
            int32_t at = 0;
#pragma unroll
            for (int v = 1; v < kEach; ++v)
                if (x[v] > value) {
                    value = x[v];
                    at = v;
                }
            const double best = top_of<kLanes>(value);
            const int32_t e = least_of<kLanes>(value == best ? at * kLanes + lane : a.E);
            const bool taken = best > -kInf;                              // none is left otherwise
#pragma unroll
            for (int v = 0; v < kEach; ++v)
                if (taken && v * kLanes + lane == e) x[v] = -kInf;
            if (lane == slot) mine = taken ? e : -1;
        }
        // weights: lane = slot
        const double s = mine >= 0 ? (double)score_at(scores, a.dtype, mine) : 0.0;
        double w;
        if (a.renormalise) {
            const double u = mine < 0 ? -kInf : a.gate == GROOT_SOFTMAX ? s : log_sigmoid(s);
            const double most = top_of<kLanes>(u);
            const double q = mine < 0 ? 0.0 : exp(u - most);
            w = q / sum_of<kLanes>(q);
        } else {
            w = probability(s);
        }
        w = broken ? (double)__builtin_nanf("") : mine < 0 ? 0.0 : (double)a.factor * w;
        if (real && lane < a.k) {
            a.experts[row * a.k + lane] = mine;
            a.weights[row * a.k + lane] = (float)w;
        }
        if (lane < a.k) chosen[local * a.k + lane] = real ? mine : -1;
        if (real && mine >= 0) atomicOr((unsigned long long *)&mask[mine], 1ull << local);
    }
    __syncthreads();
    const bool alone = gridDim.x == 1;
    for (int e = threadIdx.x; e < a.E; e += kBlock) {
        const int32_t count = __popcll(mask[e]);
        if (alone) prefix[e] = count;
        else counts[(int64_t)blockIdx.x * a.E + e] = count;
    }
    __syncthreads();
    if (alone) {
        exclusive_sums(prefix, a.E, waves);
        for (int e = threadIdx.x; e <= a.E; e += kBlock) a.offsets[e] = prefix[e];
    }
    const int64_t first = (int64_t)blockIdx.x * kRouteRows;
    const int32_t entries = (int32_t)(a.n - first < kRouteRows ? a.n - first : kRouteRows) * a.k;
    for (int32_t i = threadIdx.x; i < entries; i += kBlock) {
        const int32_t e = chosen[i];
        const int32_t rank = e < 0 ? -1 : __popcll(mask[e] & ((1ull << (i / a.k)) - 1));
        a.places[first * a.k + i] = alone && e >= 0 ? prefix[e] + rank : rank;
    }
}

// counts of the workgroups before each, expert by expert, in place, and every expert's sum in the row behind the last
__global__ __launch_bounds__(1024) void route_scan_kernel(int32_t *__restrict__ counts, int32_t groups, int32_t E)
{
    __shared__ int32_t sums[16][kWave];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int32_t e = blockIdx.x * kWave + lane, each = (groups + 15) / 16;
    const int32_t begin = wave * each, end = begin + each < groups ? begin + each : groups;
    int32_t sum = 0;
    if (e < E)
        for (int32_t g = begin; g < end; ++g) sum += counts[(int64_t)g * E + e];
    sums[wave][lane] = sum;
    __syncthreads();
    int32_t before = 0, all = 0;
    for (int w = 0; w < 16; ++w) {
        before += w < wave ? sums[w][lane] : 0;
        all += sums[w][lane];
    }
    if (e >= E) return;
    for (int32_t g = begin; g < end; ++g) {
        const int32_t here = counts[(int64_t)g * E + e];
        counts[(int64_t)g * E + e] = before;
        before += here;
    }
    if (wave == 0) counts[(int64_t)groups * E + e] = all;
}

// ranks -> places
__global__ __launch_bounds__(kBlock) void route_place_kernel(RouteArgs a, const int32_t *__restrict__ counts, int32_t groups)
{
    extern __shared__ char lds[];
    int32_t *const prefix = (int32_t *)lds, *const waves = prefix + a.E + 1;
    const int32_t *const mine = counts + (int64_t)blockIdx.x * a.E, *const all = counts + (int64_t)groups * a.E;
    for (int e = threadIdx.x; e < a.E; e += kBlock) prefix[e] = all[e];
    __syncthreads();
    exclusive_sums(prefix, a.E, waves);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= a.E; e += kBlock) a.offsets[e] = prefix[e];
    const int64_t first = (int64_t)blockIdx.x * kRouteRows;
    const int32_t entries = (int32_t)(a.n - first < kRouteRows ? a.n - first : kRouteRows) * a.k;
    for (int32_t i = threadIdx.x; i < entries; i += kBlock) {
        const int32_t e = a.experts[first * a.k + i];
        if (e >= 0) a.places[first * a.k + i] += prefix[e] + mine[e];
    }
}

// ds of a row.  softmax: l = log p, p_j (g_j - sum g p) with g the gradients at the chosen weights; renormalised over the chosen ones.
// sigmoid: the gradient at log p times 1 - p.
template <int kLanes, int kEach>
__global__ __launch_bounds__(kBlock) void route_backward_kernel(RouteBackwardArgs a)
{
    const int lane = threadIdx.x % kLanes;
    for (int64_t row = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kLanes; row < a.n; row += (int64_t)gridDim.x * (kBlock / kLanes)) {
        const char *const scores = (const char *)a.scores + row * a.score_bytes;
        float x[kEach], d[kEach];
        bool broken = false;
        float top = -kInf;
#pragma unroll
        for (int v = 0; v < kEach; ++v) {
            const int32_t e = v * kLanes + lane;
            x[v] = e < a.E ? score_at(scores, a.dtype, e) : -kInf;
            broken |= x[v] != x[v] || (a.gate == GROOT_SOFTMAX && x[v] == kInf);
            top = fmaxf(top, x[v]);
            d[v] = 0.f;
        }
        broken = any_of<kLanes>(broken);
        top = (float)top_of<kLanes>(top);
        const float base = top == -kInf ? 0.f : top;
        // slots: lane = slot
        int32_t mine = -1;
        float dw = 0.f;
        if (lane < a.k) {
            mine = a.experts[row * a.k + lane];
            mine = mine >= 0 && mine < a.E ? mine : -1;
            if (mine >= 0) dw = a.dweights[row * a.k + lane];
        }
        const float s = mine >= 0 ? score_at(scores, a.dtype, mine) : -kInf;
        float at_log = 0.f;                                   // the gradient at the slot's log p, or at its score
        if (a.renormalise) {
            const float u = mine < 0 ? -kInf : a.gate == GROOT_SOFTMAX ? s : fminf(s, 0.f) - log1pf(expf(-fabsf(s)));
            const float most = (float)top_of<kLanes>(u);
            const float q = mine < 0 ? 0.f : expf(u - most);
            const float all = (float)sum_of<kLanes>(q);       // every lane takes part
            const float w = mine < 0 ? 0.f : q / all;
            const float mean = (float)sum_of<kLanes>((double)w * dw);
            at_log = mine < 0 ? 0.f : a.factor * w * (dw - mean);
        }
        double sum = 0;
        if (a.gate == GROOT_SOFTMAX && !a.renormalise) {
#pragma unroll
            for (int v = 0; v < kEach; ++v) sum += (double)expf(x[v] - base);
            sum = sum_of<kLanes>(sum);
            const float p = mine < 0 ? 0.f : expf(s - base) / (float)sum;
            at_log = a.factor * p * dw;
        } else if (!a.renormalise && mine >= 0) {
            at_log = a.factor * dw / (1.f + expf(-s));
        }
        const float total = a.gate == GROOT_SOFTMAX && !a.renormalise ? (float)sum_of<kLanes>(at_log) : 0.f;
        for (int32_t slot = 0; slot < a.k; ++slot) {
            const int32_t e = __shfl(mine, slot, kLanes);
            const float g = __shfl(at_log, slot, kLanes);
#pragma unroll
            for (int v = 0; v < kEach; ++v)
                if (e == v * kLanes + lane) d[v] += g;
        }
#pragma unroll
        for (int v = 0; v < kEach; ++v) {
            const int32_t e = v * kLanes + lane;
            float r = d[v];
            if (a.gate == GROOT_SIGMOID) r *= 1.f / (1.f + expf(x[v]));
            else if (!a.renormalise && top > -kInf) r -= expf(x[v] - base) / (float)sum * total;
            if (x[v] == -kInf) r = 0.f;
            if (broken) r = __builtin_nanf("");
            if (e < a.E) {
                char *const to = (char *)a.dscores + row * a.ds_bytes;
                if (a.dtype == GROOT_F32) ((float *)to)[e] = r;
                else if (a.dtype == GROOT_BF16) ((bf16_t *)to)[e] = (bf16_t)r;
                else ((f16_t *)to)[e] = (f16_t)r;
            }
        }
    }
}

int64_t route_groups(int64_t n) { return n <= kRouteRows ? 1 : (n + kRouteRows - 1) / kRouteRows; }

template <int kLanes, int kEach>
int route_launch(RouteArgs a, int32_t *counts, hipStream_t stream)
{
    const int64_t groups = route_groups(a.n);
    size_t lds = a.E * sizeof(uint64_t) + (a.E + 1 + kWavesPerBlock) * sizeof(int32_t) + kRouteRows * a.k * sizeof(int16_t);
    lds = (lds + 7) / 8 * 8;
    a.values_at = (int32_t)lds;
    if (a.open_sets < a.sets) lds += (size_t)(kBlock / kLanes) * a.E * sizeof(double);
    route_kernel<kLanes, kEach><<<(uint32_t)groups, kBlock, lds, stream>>>(a, counts);
    if (groups > 1) {
        route_scan_kernel<<<(a.E + kWave - 1) / kWave, 1024, 0, stream>>>(counts, (int32_t)groups, a.E);
        route_place_kernel<<<(uint32_t)groups, kBlock, (a.E + 1 + kWavesPerBlock) * sizeof(int32_t), stream>>>(a, counts, (int32_t)groups);
    }
    return (int)hipGetLastError();
}

template <int kLanes, int kEach>
int backward_launch(const RouteBackwardArgs &a, hipStream_t stream)
{
    const int64_t blocks = (a.n * kLanes + kBlock - 1) / kBlock;
    route_backward_kernel<kLanes, kEach><<<(uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20), kBlock, 0, stream>>>(a);
    return (int)hipGetLastError();
}

}  // namespace

size_t route_workspace(int64_t n, int32_t E)
{
    const int64_t groups = route_groups(n);
    return groups == 1 ? 0 : (size_t)(groups + 1) * E * sizeof(int32_t);
}

// 16 lanes a row while they hold its experts and slots, a wavefront otherwise
#define GROOT_BY_EXPERTS(call)                                                                                                           \
    if (a.E > 256 || a.k > 16) {                                                                                                         \
        if (a.E <= 512) return call<64, 8>;                                                                                              \
        return call<64, 16>;                                                                                                             \
    }                                                                                                                                    \
    if (a.E <= 16) return call<16, 1>;                                                                                                   \
    if (a.E <= 32) return call<16, 2>;                                                                                                   \
    if (a.E <= 64) return call<16, 4>;                                                                                                   \
    if (a.E <= 128) return call<16, 8>;                                                                                                  \
    return call<16, 16>;

typedef int (*RouteLaunch)(RouteArgs, int32_t *, hipStream_t);
typedef int (*BackwardLaunch)(const RouteBackwardArgs &, hipStream_t);
static RouteLaunch route_for(const RouteArgs &a) { GROOT_BY_EXPERTS(route_launch) }
static BackwardLaunch backward_for(const RouteBackwardArgs &a) { GROOT_BY_EXPERTS(backward_launch) }

int launch_route(const RouteArgs &a, void *workspace, void *stream) { return route_for(a)(a, (int32_t *)workspace, (hipStream_t)stream); }
int launch_route_backward(const RouteBackwardArgs &a, void *stream) { return backward_for(a)(a, (hipStream_t)stream); }

}  // namespace groot
