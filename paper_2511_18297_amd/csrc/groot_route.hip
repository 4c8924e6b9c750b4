// The choice of experts for every row, their weights, and every choice's place in the order of the experts.
//   value c of an expert: its score where that orders as the probability does, otherwise softmax or sigmoid of the score, plus a bias
//   top k of c (ties to the lowest expert) among the sets whose best members' sum is largest; weights factor x p, renormalised or not
// A call cannot do without n E scores and 12 n k bytes of results.  The scores are read once; what bounds the kernel is the search, in
// instructions where there are many rows (65536 rows of 128 scores in fp32, top 8: 14.4 us, 2.8 TB/s; 666 vector instructions a wavefront
// of 8 rows, the vector units busy in 60 % of the time) and in latency where there are few (one row of 64: 3.4 us; 16384 rows of 64, one
// wavefront to a SIMD: 7).  Probabilities in 64 bits are a third of the instructions where they decide (16384 rows of 256 in
// bfloat16, sigmoid with a bias, 4 of 8 sets: 20 us).  Taken one by one, k maxima over a row's lanes took 31 us where the lists took 13.5.
//
// The search: a key is a number of 64 bits, the value with the expert's number in its last ten bits, so that one comparison decides and
// breaks ties (a score of fp32 leaves 29 bits free; a probability computed in 64 bits keeps 42, and what agrees in these counts as tied).
// A lane has kEach = 16 neighbouring experts and sorts them by a network of minima and maxima; lists of the kList best then meet between
// lanes: the larger of a list and the other one's reverse are the best of both, and a merging network sorts them.  Every lane of a row ends
// with the row's list.
//
// Places: a workgroup takes up to 64 rows.  A row chooses an expert once, so the rows of a workgroup that chose an expert are the bits of
// one 64-bit word, and a choice's rank is the number of bits below its row's: nothing depends on the order of atomics.  The ranks wait
// in `places` until the counts of all workgroups are known: every workgroup of a second launch adds them up (4 to 6 us), beyond 256
// workgroups a launch between the two does (256 counts of 256 experts in bytes are 64 KB to read for each workgroup).  That one takes 5 us for the 1024
// counts of 65536 rows and grows with them, 16 experts to a workgroup: 60 us for 1 M rows, 0.8 and 1.4 ms of 1.05 and 2.05 for 8.4 M of 8 and 64.
#include "groot_tile.h"

namespace groot {

namespace {

constexpr int kRouteRows = 64;               // rows of a workgroup at most: bits of a word
constexpr int kNumberBits = 10;              // of an expert in a key
constexpr uint32_t kNumbers = (1u << kNumberBits) - 1;
// Workgroups whose counts every workgroup of the second launch adds up by itself: 16384 rows of 64, 256 and 512 scores 8.9, 12.6 and 21.7 us, with
// a launch between for the sums 11.2, 14.8 and 23.1; 1024 workgroups of 128 scores gained nothing (21.5, with the launch 20.9).
constexpr int kSumGroups = 256;
typedef v4i piece_t __attribute__((aligned(1)));
constexpr float kInf = __builtin_inff();
constexpr double kClosed = -0x1p1023, kLeastOpen = -0x1p1022, kMostOpen = 0x1p1022;

__device__ __forceinline__ float score_at(const void *row, int32_t dtype, int32_t e)
{
    if (dtype == GROOT_F32) return ((const float *)row)[e];
    if (dtype == GROOT_BF16) return (float)((const bf16_t *)row)[e];
    return (float)((const f16_t *)row)[e];
}

template <int kLanes, typename T>
__device__ __forceinline__ T top_of(T x)
{
    return over_lanes<kLanes>(x, [](T a, T b) { return a > b ? a : b; });
}
template <int kLanes, typename T>
__device__ __forceinline__ T sum_of(T x)
{
    return over_lanes<kLanes>(x, [](T a, T b) { return a + b; });
}
template <int kLanes>
__device__ __forceinline__ bool any_of(bool x)
{
    return over_lanes<kLanes>((uint32_t)x, [](uint32_t a, uint32_t b) { return a | b; }) != 0;
}

// The scores of a lane's kEach experts from `begin` on; -inf beyond the last.
template <int kEach, typename T>
__device__ __forceinline__ void load_scores_of(const char *row, int32_t E, int32_t begin, float (&s)[kEach])
{
    constexpr int kPer = 16 / sizeof(T);
    v4i v[kEach / kPer];
    if (E % kPer == 0) {                                     // whole pieces of 16 bytes
#pragma unroll
        for (int i = 0; i < kEach / kPer; ++i) v[i] = *(const piece_t *)(row + (begin + i * kPer < E ? begin + i * kPer : 0) * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < kEach / kPer; ++i) {
            const RowValues<T> x = row_values<T>(v[i]);
            const bool there = begin + i * kPer < E;
#pragma unroll
            for (int j = 0; j < kPer; ++j) s[i * kPer + j] = there ? x.x[j] : -kInf;
        }
    } else {
        const bool short_row = E < kPer;
        asm("" : "+v"(begin));                               // what follows is computed here and not, for all calls, in front
#pragma unroll
        for (int i = 0; i < kEach / kPer; ++i) {
            const int32_t e = begin + i * kPer, at = e + kPer <= E ? e : E - kPer;   // the row's last piece in place of what there is not
            v[i] = short_row ? short16<T>(row + e * (int)sizeof(T), (E - e) * (int)sizeof(T)) : *(const piece_t *)(row + at * (int)sizeof(T));
        }
#pragma unroll
        for (int i = 0; i < kEach / kPer; ++i) {
            const int32_t left = E - (begin + i * kPer);
            if (!short_row && left < kPer) v[i] = cut16(v[i], left * (int)sizeof(T));
            const RowValues<T> x = row_values<T>(v[i]);
#pragma unroll
            for (int j = 0; j < kPer; ++j) s[i * kPer + j] = j < left ? x.x[j] : -kInf;
        }
    }
}
template <int kEach>
__device__ __forceinline__ void load_scores(const char *row, const RouteArgs &a, int32_t begin, float (&s)[kEach])
{
    if (a.dtype == GROOT_F32) load_scores_of<kEach, float>(row, a.E, begin, s);
    else if (a.dtype == GROOT_BF16) load_scores_of<kEach, bf16_t>(row, a.E, begin, s);
    else load_scores_of<kEach, f16_t>(row, a.E, begin, s);
}

// e^x for x <= 0 to 2^-50 of itself: x = i log 2 + r, |r| <= log 2 / 2, and r's series up to r^12 / 12! (the next term is 2^-52)
__device__ __forceinline__ double exp64(double x)
{
    x = fmax(x, -760.0);                                     // e^x is 0 there
    const double i = __builtin_rint(x * 0x1.71547652b82fep+0);
    double r = __builtin_fma(-i, 0x1.62e42fefa2000p-1, x);     // log 2 in two parts, i times the first is exact
    r = __builtin_fma(-i, 0x1.9ef35793c7673p-41, r);
    double p = 1.0 / 479001600;
    p = __builtin_fma(p, r, 1.0 / 39916800);
    p = __builtin_fma(p, r, 1.0 / 3628800);
    p = __builtin_fma(p, r, 1.0 / 362880);
    p = __builtin_fma(p, r, 1.0 / 40320);
    p = __builtin_fma(p, r, 1.0 / 5040);
    p = __builtin_fma(p, r, 1.0 / 720);
    p = __builtin_fma(p, r, 1.0 / 120);
    p = __builtin_fma(p, r, 1.0 / 24);
    p = __builtin_fma(p, r, 1.0 / 6);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return ldexp(p, (int)i);
}

// e^x for x <= 0 to 2^-31 of itself, for what fp32 holds in the end (e^-700 below -700): the same with r's series up to r^8 / 8!.  i comes out of an addition
// that leaves it in the last bits, and is added to the exponent's: conversions and ldexp take four times an addition's cycles.
__device__ __forceinline__ double exp31(double x)
{
    constexpr double kRound = 0x1.8p52;
    x = fmax(x, -700.0);
    const double shifted = __builtin_fma(x, 0x1.71547652b82fep+0, kRound), r = __builtin_fma(kRound - shifted, 0x1.62e42fefa39efp-1, x);
    double p = 1.0 / 40320;
    p = __builtin_fma(p, r, 1.0 / 5040);
    p = __builtin_fma(p, r, 1.0 / 720);
    p = __builtin_fma(p, r, 1.0 / 120);
    p = __builtin_fma(p, r, 1.0 / 24);
    p = __builtin_fma(p, r, 1.0 / 6);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, p) + (__builtin_bit_cast(uint64_t, shifted) << 52));
}

// 1 / x to 2^-51: the instruction's approximation and two of Newton's steps, which square its error of 2^-14 at most
__device__ __forceinline__ double reciprocal64(double x)
{
    double y = __builtin_amdgcn_rcp(x);
    y = __builtin_fma(__builtin_fma(-x, y, 1.0), y, y);
    return __builtin_fma(__builtin_fma(-x, y, 1.0), y, y);
}

// The weight of a score up to a factor that the row shares.  softmax: e^(s - m), m the largest score.  sigmoid: e^min(s, 0) / (1 + e^-|s|),
// with e^(min(s, 0) - m) in its place where weights are renormalised, so that low scores keep their ratios.  In 64 bits, as the sums of them
// are, and a weight is rounded once: in fp32 the difference and its product with log2(e) alone cost |s - m| half steps (55 were seen).
__device__ __forceinline__ double weight_of(float s, float m, bool sigmoid)
{
    const double e = exp31((double)(sigmoid ? fminf(s, 0.f) : s) - (double)m);
    return sigmoid ? e * reciprocal64(1.0 + exp31(-__builtin_fabs((double)s))) : e;
}
// The softmax's sum over all experts is of terms in fp32, in pairs: a term p that is |x| below the largest is off by 2.5 |x| + 2 half steps, and p |x| adds
// up to 4.4 of the sum at the most (1024 experts).  In 64 bits: 65536 rows of 128, top 8: 23.9 us in place of 20.6.
template <int kCount>
__device__ __forceinline__ float tree_sum(float (&x)[kCount])
{
#pragma unroll
    for (int d = 1; d < kCount; d *= 2)
#pragma unroll
        for (int i = 0; i + d < kCount; i += 2 * d) x[i] += x[i + d];
    return x[0];
}
// 1 - sigmoid(s)
__device__ __forceinline__ double rest_of(float s)
{
    const double e = exp31(-__builtin_fabs((double)s));
    return (s > 0.f ? e : 1.0) * reciprocal64(1.0 + e);
}

// The value with the number in its last bits, so that of equal values the lower number is the larger key: its complement where the value
// is positive, the number where it is negative.
__device__ __forceinline__ double key_of(double c, uint32_t number, uint32_t numbers)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, c);
    const uint32_t high = (uint32_t)(b >> 32), low = ((uint32_t)b & ~numbers) | (number ^ numbers ^ (uint32_t)((int32_t)high >> 31 & (int32_t)numbers));
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
__device__ __forceinline__ uint32_t number_of(double key, uint32_t numbers)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, key);
    return ((uint32_t)b ^ ~(uint32_t)((int64_t)b >> 63)) & numbers;
}
__device__ __forceinline__ float score_of(double key)        // a key of a score
{
    return (float)__builtin_bit_cast(double, __builtin_bit_cast(uint64_t, key) & ~(uint64_t)kNumbers);
}

// The instructions themselves: keys are no NaN, and the language's maximum puts another one in front of it to be sure.
__device__ __forceinline__ double larger(double a, double b)
{
    double r;
    asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ double smaller(double a, double b)
{
    double r;
    asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ void order(double &a, double &b)  // descending
{
    const double most = larger(a, b), least = smaller(a, b);
    a = most;
    b = least;
}
// x[i] for an i that differs from lane to lane
template <int kCount>
__device__ __forceinline__ double picked(const double *x, int i)
{
    if constexpr (kCount == 1) return x[0];
    else {
        const double low = picked<kCount / 2>(x, i), high = picked<kCount / 2>(x + kCount / 2, i);
        return i & (kCount / 2) ? high : low;
    }
}

// Batcher's odd-even merge sort of kCount neighbouring keys, descending
template <int kCount>
__device__ __forceinline__ void sort_keys(double *x)
{
#pragma unroll
    for (int p = 1; p < kCount; p *= 2)
#pragma unroll
        for (int d = p; d >= 1; d /= 2)
#pragma unroll
            for (int j = d % p; j + d < kCount; j += 2 * d)
#pragma unroll
                for (int i = 0; i < d; ++i)
                    if (i + j + d < kCount && (i + j) / (2 * p) == (i + j + d) / (2 * p)) order(x[i + j], x[i + j + d]);
}
// x: the kCount largest of two descending lists, descending
template <int kCount>
__device__ __forceinline__ void merge_keys(double *x, const double *y)
{
#pragma unroll
    for (int i = 0; i < kCount; ++i) x[i] = larger(x[i], y[kCount - 1 - i]);
#pragma unroll
    for (int d = kCount / 2; d >= 1; d /= 2)
#pragma unroll
        for (int i = 0; i < kCount; ++i)
            if (!(i & d)) order(x[i], x[i + d]);
}
template <int kLanes, int kCount, int kAway = 1>
__device__ __forceinline__ void merge_lanes(double *x)
{
    if constexpr (kAway < kLanes) {
        double y[kCount];
#pragma unroll
        for (int i = 0; i < kCount; ++i) pair_lanes<kAway>(x[i], &x[i], &y[i]);
        merge_keys<kCount>(x, y);
        merge_lanes<kLanes, kCount, kAway * 2>(x);
    }
}

// Exclusive sums of E words of LDS, in place; the sum of all goes to word E.  `waves`: a word for every wavefront.
__device__ __forceinline__ void exclusive_sums(int32_t *x, int32_t E, int32_t *waves)
{
    const int tid = threadIdx.x, lane = tid % kWave, threads = blockDim.x, per = (E + threads - 1) / threads;
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
    if (tid == threads - 1) x[E] = before;
    __syncthreads();
}

// the two largest of a set, of what lanes kAway apart hold of it
template <int kAway>
__device__ __forceinline__ void meet_sets(double &most, double &second)
{
    double m1, m2, s1, s2;
    pair_lanes<kAway>(most, &m1, &m2);
    pair_lanes<kAway>(second, &s1, &s2);
    most = larger(m1, m2);
    second = larger(larger(s1, s2), smaller(m1, m2));
}

// Sets of kSize neighbouring experts, several in a lane: `values` of the row's sets, and those that are not among the open ones closed.
template <int kSize, int kEach>
__device__ __forceinline__ void close_small_sets(double (&x)[kEach], double *values, const RouteArgs &a, int lane)
{
    constexpr int kOwn = kEach / kSize;
    double mine[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
        double most = x[j * kSize], second = kClosed;
#pragma unroll
        for (int v = 1; v < kSize; ++v) {
            second = larger(second, smaller(most, x[j * kSize + v]));
            most = larger(most, x[j * kSize + v]);
        }
        const int32_t set = lane * kOwn + j;
        mine[j] = key_of(a.set_best == 2 && second > kLeastOpen ? smaller(most + second, kMostOpen) : most, (uint32_t)set, 63);
        if (set < a.sets) values[set] = mine[j];
    }
    wave_sync();
    int32_t above[kOwn] = {};
    for (int32_t i = 0; i < a.sets; ++i) {
        const double v = values[i];
#pragma unroll
        for (int j = 0; j < kOwn; ++j) above[j] += v > mine[j];
    }
    wave_sync();                                             // before the next rows' values
#pragma unroll
    for (int v = 0; v < kEach; ++v) x[v] = above[v / kSize] >= a.open_sets ? kClosed : x[v];
}

// Sets of 16 experts or more that begin anywhere: a lane's experts belong to two at the most, those up to `border` to its first one.
// `values`: what the row's sets come to, behind them the two largest that each lane holds of each of its two sets.
template <int kLanes, int kEach>
__device__ __forceinline__ void close_wide_sets(double (&x)[kEach], double *values, const RouteArgs &a, int lane, int32_t size)
{
    double *const held = values + a.sets;                    // [kLanes, 2 sets, 2 values]
    const int32_t begin = lane * kEach, set = begin / size, border = (set + 1) * size - begin;
    double most[2] = {kClosed, kClosed}, second[2] = {kClosed, kClosed};
#pragma unroll
    for (int v = 0; v < kEach; ++v) {
        const double c[2] = {v < border ? x[v] : kClosed, v < border ? kClosed : x[v]};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            second[j] = larger(second[j], smaller(most[j], c[j]));
            most[j] = larger(most[j], c[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        held[lane * 4 + j * 2] = most[j];
        held[lane * 4 + j * 2 + 1] = second[j];
    }
    wave_sync();
    for (int32_t s = lane; s < a.sets; s += kLanes) {
        double m = kClosed, n = kClosed;
        for (int32_t l = s * size / kEach; l <= ((s + 1) * size - 1) / kEach; ++l) {
            const double *const h = held + l * 4 + (s - l * kEach / size) * 2;
            n = larger(larger(n, h[1]), smaller(m, h[0]));
            m = larger(m, h[0]);
        }
        values[s] = key_of(a.set_best == 2 && n > kLeastOpen ? smaller(m + n, kMostOpen) : m, (uint32_t)s, 63);
    }
    wave_sync();
    const double own[2] = {values[set < a.sets ? set : 0], values[set + 1 < a.sets ? set + 1 : 0]};
    int32_t above[2] = {};
    for (int32_t i = 0; i < a.sets; ++i) {
        const double v = values[i];
#pragma unroll
        for (int j = 0; j < 2; ++j) above[j] += v > own[j];
    }
    wave_sync();                                             // before the next rows'
#pragma unroll
    for (int v = 0; v < kEach; ++v) x[v] = above[v < border ? 0 : 1] >= a.open_sets ? kClosed : x[v];
}

// words of a workgroup's counts: a byte for each expert
__host__ __device__ constexpr int32_t count_words(int32_t E) { return (E + 3) / 4; }

constexpr int kRouteThreads = 512;           // of a workgroup at most
constexpr int kMaxWaves = 16;

// the workgroup's LDS, in bytes
struct RouteLds {
    int32_t mask, prefix, waves, weights, chosen, values, total;
    __host__ __device__ RouteLds(int32_t E, int32_t rows, int32_t k, int32_t value_bytes)
    {
        mask = 0;                                            // uint64 [E]: the rows that chose an expert
        values = mask + E * 8;                               // double: values of sets, or of experts
        prefix = values + value_bytes;                       // int32 [E + 1]
        waves = prefix + (E + 1) * 4;                        // int32 [kMaxWaves]
        weights = waves + kMaxWaves * 4;                     // float [rows, k]
        chosen = weights + rows * k * 4;                     // int16 [rows, k]
        total = chosen + rows * k * 2;
    }
};

// i / k for i below 2^11 and k up to 32, from 2^16 / k rounded up: the error of i / 2^16 stays below 1 / k
__device__ __forceinline__ int32_t over(int32_t i, uint32_t inverse) { return (int32_t)((uint32_t)i * inverse >> 16); }
uint32_t inverse_of(int32_t k) { return ((1u << 16) + k - 1) / k; }

// kLanes lanes to a row, kEach neighbouring experts a lane, lists of kList keys (top_k of up to that many; beyond 16 they are taken one by one)
template <int kLanes, int kEach, int kList, bool kByValue, bool kSets>
__global__ __launch_bounds__(kRouteThreads, 4) void route_kernel(RouteArgs a, uint32_t *__restrict__ counts)
{
    extern __shared__ char lds[];
    const RouteLds at(a.E, a.rows, a.k, a.value_bytes);
    unsigned long long *const mask = (unsigned long long *)(lds + at.mask);
    int32_t *const prefix = (int32_t *)(lds + at.prefix), *const waves = (int32_t *)(lds + at.waves);
    float *const weights = (float *)(lds + at.weights);
    int16_t *const chosen = (int16_t *)(lds + at.chosen);
    const int threads = blockDim.x, at_once = threads / kLanes;
    const bool sigmoid = a.gate == GROOT_SIGMOID;
    for (int e = threadIdx.x; e < a.E; e += threads) mask[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * a.rows;
    const int here = (int)(a.n - first < a.rows ? a.n - first : a.rows);  // rows of this workgroup
    for (int pass = 0; pass < here; pass += at_once) {
        int lane = threadIdx.x % kLanes;
        asm("" : "+v"(lane));                                             // nothing that goes by it is computed in front of the loop and held
        const int32_t begin = lane * kEach;
        const int local = pass + threadIdx.x / kLanes;
        const bool real = local < here;                                   // rows beyond the last go along
        const char *const scores = (const char *)a.scores + (first + (real ? local : here - 1)) * a.score_bytes;
        float bias[kByValue ? kEach : 1] = {};
        if constexpr (kByValue) {
            if (a.bias) load_scores_of<kEach, float>((const char *)a.bias, a.E, begin, bias);
        }
        float s[kEach];
        load_scores<kEach>(scores, a, begin, s);
        float top = s[0];                                                 // NaN if one of them is
#pragma unroll
        for (int v = 1; v < kEach; ++v) top = __builtin_elementwise_maximum(top, s[v]);
        top = over_lanes<kLanes>(top, [](float x, float y) { return __builtin_elementwise_maximum(x, y); });
        const bool broken = top != top || (!sigmoid && top == kInf);
        const float base = sigmoid || top == -kInf ? 0.f : top;
        double sum = 1.0;                                                 // of e^(s - base), where weights go by it
        double x[kEach];
        if constexpr (!kByValue) {
            if (!sigmoid && !a.renormalise) {
                float term[kEach];
#pragma unroll
                for (int v = 0; v < kEach; ++v) term[v] = __expf(s[v] - base);
                sum = (double)sum_of<kLanes>(tree_sum(term));
            }
#pragma unroll
            for (int v = 0; v < kEach; ++v) {
                x[v] = fmax((double)(s[v] + 0.f), kClosed);               // -0 is 0, -inf is closed
            }
            if (sigmoid) {
#pragma unroll
                for (int v = 0; v < kEach; ++v) x[v] = fmin(x[v], kMostOpen);   // +inf
            }
        } else {
            double all = 0;
#pragma unroll
            for (int v = 0; v < kEach; ++v) {
                x[v] = exp64(sigmoid ? -__builtin_fabs((double)s[v]) : (double)s[v] - (double)base);
                all += x[v];
            }
            if (!sigmoid) {
                all = sum_of<kLanes>(all);
                sum = all;
                all = 1.0 / all;
            }
#pragma unroll
            for (int v = 0; v < kEach; ++v) {
                const double p = sigmoid ? (s[v] < 0.f ? x[v] : 1.0) * reciprocal64(1.0 + x[v]) : x[v] * all;
                const double c = p + (double)bias[v];
                x[v] = s[v] > -kInf && c > -__builtin_inf() ? fmin(c, kMostOpen) : kClosed;
            }
        }
        if constexpr (kSets) {
            const int32_t size = a.E / a.sets;
            // the values that a row's sets come to, the set's number in each; a set counts as many others as are above it
            if (a.set_lanes) {                                            // a set is all of a few lanes' experts
                double *const values = (double *)(lds + at.values) + threadIdx.x / kLanes * a.sets;
                double most = kClosed, second = kClosed;
#pragma unroll
                for (int v = 0; v < kEach; ++v) {
                    second = larger(second, smaller(most, x[v]));
                    most = larger(most, x[v]);
                }
                if (a.set_lanes > 1) meet_sets<1>(most, second);
                if (a.set_lanes > 2) meet_sets<2>(most, second);
                if (a.set_lanes > 4) meet_sets<4>(most, second);
                if (a.set_lanes > 8) meet_sets<8>(most, second);
                if (a.set_lanes > 16) meet_sets<16>(most, second);
                const int32_t set = lane / a.set_lanes;
                const double mine = key_of(a.set_best == 2 && second > kLeastOpen ? fmin(most + second, kMostOpen) : most, (uint32_t)set, 63);
                if (set < a.sets && lane % a.set_lanes == 0) values[set] = mine;
                wave_sync();
                int32_t above = 0;
                for (int32_t i = 0; i < a.sets; ++i) above += values[i] > mine;
                wave_sync();                                              // before the next rows' values
                if (above >= a.open_sets) {
#pragma unroll
                    for (int v = 0; v < kEach; ++v) x[v] = kClosed;
                }
            } else if (a.wide_sets) {
                close_wide_sets<kLanes, kEach>(x, (double *)(lds + at.values) + threadIdx.x / kLanes * (a.sets + 4 * kLanes), a, lane, size);
            } else if (a.small_sets) {
                double *const values = (double *)(lds + at.values) + threadIdx.x / kLanes * a.sets;
                if (size == 1) close_small_sets<1>(x, values, a, lane);
                else if (size == 2) close_small_sets<2>(x, values, a, lane);
                else if (size == 4) close_small_sets<4>(x, values, a, lane);
                else close_small_sets<8>(x, values, a, lane);
            } else {
                double *const values = (double *)(lds + at.values) + (int64_t)(threadIdx.x / kLanes) * (kLanes * kEach + a.sets), *const row = values + a.sets;
#pragma unroll
                for (int v = 0; v < kEach; ++v) row[begin + v] = x[v];
                wave_sync();
                for (int32_t set = lane; set < a.sets; set += kLanes) {
                    double most = kClosed, second = kClosed;
                    for (int32_t i = 0; i < size; ++i) {
                        const double c = row[set * size + i];
                        second = larger(second, smaller(most, c));
                        most = larger(most, c);
                    }
                    values[set] = key_of(a.set_best == 2 && second > kLeastOpen ? fmin(most + second, kMostOpen) : most, (uint32_t)set, 63);
                }
                wave_sync();
                for (int32_t set = lane; set < a.sets; set += kLanes) {
                    const double mine = values[set];
                    int32_t above = 0;
                    for (int32_t i = 0; i < a.sets; ++i) above += values[i] > mine;
                    if (above >= a.open_sets)
                        for (int32_t i = 0; i < size; ++i) row[set * size + i] = kClosed;
                }
                wave_sync();
#pragma unroll
                for (int v = 0; v < kEach; ++v) x[v] = begin + v < a.E ? row[begin + v] : kClosed;
                wave_sync();
            }
        }
#pragma unroll
        for (int v = 0; v < kEach; ++v) x[v] = key_of(x[v], (uint32_t)(begin + v), kNumbers);
        // the lane's lists, the lane's list, the row's
#pragma unroll
        for (int v = 0; v < kEach; v += kList) sort_keys<kList>(x + v);
#pragma unroll
        for (int half = kEach / 2; half >= kList; half /= 2)
#pragma unroll
            for (int v = 0; v < half; v += kList) merge_keys<kList>(x + v, x + v + half);
        const float nan = __builtin_nanf("");
        if (kList < 16 || a.k <= 16) {
            merge_lanes<kLanes, kList>(x);
            // every lane takes its share of the slots: slot j kWide + lane
            constexpr int kWide = kLanes < kList ? kLanes : kList, kSlots = kList / kWide;
            const int here_lane = lane % kWide;
            float at_slot[kSlots];
            int32_t expert[kSlots];
            float m = -kInf;
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                const double key = picked<kWide>(x + j * kWide, here_lane);
                const bool taken = key > kLeastOpen && !broken && j * kWide + lane < a.k && (kWide == kLanes || lane < kWide);
                expert[j] = taken ? (int32_t)number_of(key, kNumbers) : -1;
                at_slot[j] = !taken ? -kInf : kByValue ? score_at(scores, a.dtype, expert[j]) : score_of(key);
                m = fmaxf(m, sigmoid ? fminf(at_slot[j], 0.f) : at_slot[j]);
            }
            if (a.renormalise) {
                m = top_of<kLanes>(m);
                m = m == -kInf ? 0.f : m;
            } else {
                m = base;
            }
            double w[kSlots], all = 0.0;
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                w[j] = expert[j] < 0 ? 0.0 : weight_of(at_slot[j], m, sigmoid);
                all += w[j];
            }
            const double scale = a.factor * reciprocal64(a.renormalise ? sum_of<kLanes>(all) : sum);
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                const int slot = j * kWide + lane;
                if (real && slot < a.k && (kWide == kLanes || lane < kWide)) {
                    weights[local * a.k + slot] = broken ? nan : expert[j] < 0 ? 0.f : (float)(w[j] * scale);
                    chosen[local * a.k + slot] = (int16_t)expert[j];
                    if (expert[j] >= 0) atomicOr(&mask[expert[j]], 1ull << local);
                }
            }
        } else if constexpr (kList == 16 && kEach == 16) {                // the lists hold all of a lane's experts
            for (int32_t slot = 0; slot < a.k; ++slot) {
                const double best = top_of<kLanes>(x[0]);
                const bool mine = x[0] == best;
#pragma unroll
                for (int v = 0; v + 1 < kEach; ++v) x[v] = mine ? x[v + 1] : x[v];
                if (mine) x[kEach - 1] = kClosed;
                const bool taken = best > kLeastOpen && !broken;
                const int32_t expert = taken ? (int32_t)number_of(best, kNumbers) : -1;
                if (real && lane == 0) {
                    weights[local * a.k + slot] = taken ? score_at(scores, a.dtype, expert) : -kInf;
                    chosen[local * a.k + slot] = (int16_t)expert;
                    if (taken) atomicOr(&mask[expert], 1ull << local);
                }
            }
            wave_sync();
            // every lane takes its share of the slots: slot j kLanes + lane
            const int32_t slots = real ? a.k : 0;
            float m = -kInf;
            for (int32_t slot = lane; slot < slots; slot += kLanes) m = fmaxf(m, sigmoid ? fminf(weights[local * a.k + slot], 0.f) : weights[local * a.k + slot]);
            if (a.renormalise) {
                m = top_of<kLanes>(m);
                m = m == -kInf ? 0.f : m;
            } else {
                m = base;
            }
            double all = 0.0;
            if (a.renormalise)
                for (int32_t slot = lane; slot < slots; slot += kLanes) all += weight_of(weights[local * a.k + slot], m, sigmoid);
            const double scale = a.factor * reciprocal64(a.renormalise ? sum_of<kLanes>(all) : sum);
            for (int32_t slot = lane; slot < slots; slot += kLanes) {
                const float at_slot = weights[local * a.k + slot];
                weights[local * a.k + slot] = broken ? nan : at_slot == -kInf ? 0.f : (float)(weight_of(at_slot, m, sigmoid) * scale);
            }
            wave_sync();
        }
    }
    __syncthreads();
    const bool alone = gridDim.x == 1;
    if (!alone) {
        const int32_t words = count_words(a.E);
        for (int w = threadIdx.x; w < words; w += threads) {
            uint32_t four = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) four |= (uint32_t)__popcll(mask[4 * w + i < a.E ? 4 * w + i : a.E - 1]) << (8 * i);   // beyond the last: nobody's
            counts[(int64_t)blockIdx.x * words + w] = four;
        }
    } else {
        for (int e = threadIdx.x; e < a.E; e += threads) prefix[e] = __popcll(mask[e]);
        __syncthreads();
        exclusive_sums(prefix, a.E, waves);
        for (int e = threadIdx.x; e <= a.E; e += threads) a.offsets[e] = prefix[e];
    }
    for (int32_t i = threadIdx.x; i < here * a.k; i += threads) {
        const int32_t e = chosen[i];
        int32_t place = -1;
        if (e >= 0) place = __popcll(mask[e] & ((1ull << over(i, a.inverse_k)) - 1)) + (alone ? prefix[e] : 0);
        a.experts[first * a.k + i] = e;
        a.weights[first * a.k + i] = weights[i];
        a.places[first * a.k + i] = place;
    }
}

// before[g, e]: the counts of the workgroups before g; the row behind the last: every expert's sum
constexpr int kScanExperts = 16, kScanParts = 64;
__global__ __launch_bounds__(kScanExperts * kScanParts) void route_scan_kernel(const uint32_t *__restrict__ counts, int32_t *__restrict__ before_at, int32_t groups,
                                                                               int32_t E)
{
    __shared__ int32_t sums[kScanParts][kScanExperts];
    const int part = threadIdx.x / kScanExperts, at = threadIdx.x % kScanExperts;
    const int32_t e = blockIdx.x * kScanExperts + at, each = (groups + kScanParts - 1) / kScanParts, pitch = count_words(E) * 4;
    const int32_t begin = part * each, end = begin + each < groups ? begin + each : groups;
    auto count = [&](int32_t g) { return (int32_t)((const uint8_t *)counts)[(int64_t)g * pitch + e]; };
    constexpr int kHeld = 16;                                // of a part in registers: 1024 workgroups' counts are read once
    int32_t held[kHeld], sum = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        held[i] = e < E && begin + i < end ? count(begin + i) : 0;
        sum += held[i];
    }
    if (e < E)
        for (int32_t g = begin + kHeld; g < end; ++g) sum += count(g);
    sums[part][at] = sum;
    __syncthreads();
    int32_t before = 0, all = 0;
#pragma unroll 16
    for (int p = 0; p < kScanParts; ++p) {
        const int32_t s = sums[p][at];
        before += p < part ? s : 0;
        all += s;
    }
    if (e >= E) return;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        if (begin + i < end) before_at[(int64_t)(begin + i) * E + e] = before;
        before += held[i];
    }
    for (int32_t g = begin + kHeld; g < end; ++g) {
        before_at[(int64_t)g * E + e] = before;
        before += count(g);
    }
    if (part == 0) before_at[(int64_t)groups * E + e] = all;
}

// ranks -> places.  kScanned: with the sums of route_scan_kernel; otherwise this workgroup adds the counts up, four experts a thread
// and its threads in as many parts as there are for these (the sums of 256 counts of up to 64 stay below 2^16: two to a word).
template <bool kScanned>
__global__ __launch_bounds__(1024) void route_place_kernel(RouteArgs a, const uint32_t *__restrict__ counts, const int32_t *__restrict__ before_at, int32_t groups)
{
    extern __shared__ char lds[];
    int32_t *const prefix = (int32_t *)lds, *const before = prefix + a.E + 1, *const waves = before + a.E;
    const int threads = blockDim.x;
    if constexpr (kScanned) {
        for (int e = threadIdx.x; e < a.E; e += threads) {
            prefix[e] = before_at[(int64_t)groups * a.E + e];
            before[e] = before_at[(int64_t)blockIdx.x * a.E + e];
        }
    } else {
        static_assert(kSumGroups * kRouteRows < 65536, "sums of 16 bits");
        for (int e = threadIdx.x; e < a.E; e += threads) prefix[e] = before[e] = 0;
        __syncthreads();
        const int words = count_words(a.E), parts = threads / words;        // 1024 threads, 256 words at the most
        const int part = threadIdx.x / words, w = threadIdx.x - part * words;
        if (part < parts) {
            uint32_t all_even = 0, all_odd = 0, mine_even = 0, mine_odd = 0;
#pragma unroll 8
            for (int32_t g = part; g < groups; g += parts) {
                const uint32_t c = counts[(int64_t)g * words + w], even = c & 0x00FF00FFu, odd = c >> 8 & 0x00FF00FFu;
                const bool earlier = g < (int32_t)blockIdx.x;
                all_even += even;
                all_odd += odd;
                mine_even += earlier ? even : 0;
                mine_odd += earlier ? odd : 0;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 4 * w + i;
                if (e >= a.E) break;
                atomicAdd(&prefix[e], (int32_t)((i % 2 ? all_odd : all_even) >> (i / 2 * 16) & 0xFFFF));
                atomicAdd(&before[e], (int32_t)((i % 2 ? mine_odd : mine_even) >> (i / 2 * 16) & 0xFFFF));
            }
        }
    }
    __syncthreads();
    exclusive_sums(prefix, a.E, waves);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= a.E; e += threads) a.offsets[e] = prefix[e];
    const int64_t first = (int64_t)blockIdx.x * a.rows;
    const int32_t entries = (int32_t)(a.n - first < a.rows ? a.n - first : a.rows) * a.k;
    for (int32_t i = threadIdx.x; i < entries; i += threads) {
        const int32_t e = a.experts[first * a.k + i];
        if (e >= 0) a.places[first * a.k + i] += prefix[e] + before[e];
    }
}

// kEach neighbouring scores of a row; where they begin beyond E none of them exist
template <int kEach, typename T>
__device__ __forceinline__ void row_scores(const char *row, int32_t E, int32_t begin, bool whole, float (&x)[kEach])
{
    typedef T vt __attribute__((ext_vector_type(kEach)));
    typedef vt at_any __attribute__((aligned(sizeof(T) == 4 ? 4 : 2)));
    if (whole) {
        const vt v = *(const at_any *)(row + (begin < E ? begin : 0) * (int)sizeof(T));
#pragma unroll
        for (int k = 0; k < kEach; ++k) x[k] = begin < E ? (float)v[k] : -kInf;
    } else {
#pragma unroll
        for (int k = 0; k < kEach; ++k) x[k] = begin + k < E ? (float)((const T *)row)[begin + k] : -kInf;
    }
}
template <int kEach, typename T>
__device__ __forceinline__ void put_scores(char *row, int32_t E, int32_t begin, bool whole, const float (&x)[kEach])
{
    typedef T vt __attribute__((ext_vector_type(kEach)));
    typedef vt at_any __attribute__((aligned(sizeof(T) == 4 ? 4 : 2)));
    if (whole) {
        vt v;
#pragma unroll
        for (int k = 0; k < kEach; ++k) v[k] = (T)x[k];      // the one rounding
        if (begin < E) *(at_any *)(row + begin * (int)sizeof(T)) = v;
    } else {
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (begin + k < E) ((T *)row)[begin + k] = (T)x[k];
    }
}

// ds of a row.  softmax: l = log p, p_j (g_j - sum g p) with g the gradients at the chosen weights; renormalised over the chosen ones.
// sigmoid: the gradient at log p times 1 - p.  In 64 bits up to the products that are rounded to wait in LDS and registers.  kLanes lanes to a row with kEach neighbouring experts each, and a slot.
template <int kLanes, int kEach>
__global__ __launch_bounds__(kBlock) void route_backward_kernel(RouteBackwardArgs a)
{
    __shared__ float chosen_at[kBlock * kEach];              // the gradients at the chosen experts of the workgroup's rows
    const int lane = threadIdx.x % kLanes;
    const int32_t begin = lane * kEach;
    float *const at = chosen_at + threadIdx.x / kLanes * (kLanes * kEach);
    const bool whole = a.E % kEach == 0, sigmoid = a.gate == GROOT_SIGMOID;
    for (int64_t row = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kLanes; row < a.n; row += (int64_t)gridDim.x * (kBlock / kLanes)) {
        const char *const scores = (const char *)a.scores + row * a.score_bytes;
        // slots: lane = slot
        int32_t mine = -1;
        float dw = 0.f, s = -kInf;
        if (lane < a.k) {
            mine = a.experts[row * a.k + lane];
            mine = mine >= 0 && mine < a.E ? mine : -1;
            if (mine >= 0) {
                dw = a.dweights[row * a.k + lane];
                s = score_at(scores, a.dtype, mine);
            }
        }
        float x[kEach];
        if (a.dtype == GROOT_F32) row_scores<kEach, float>(scores, a.E, begin, whole, x);
        else if (a.dtype == GROOT_BF16) row_scores<kEach, bf16_t>(scores, a.E, begin, whole, x);
        else row_scores<kEach, f16_t>(scores, a.E, begin, whole, x);
        float top = x[0];                                    // NaN if one of them is
#pragma unroll
        for (int v = 1; v < kEach; ++v) top = __builtin_elementwise_maximum(top, x[v]);
        top = over_lanes<kLanes>(top, [](float a, float b) { return __builtin_elementwise_maximum(a, b); });
        const bool broken = top != top || (!sigmoid && top == kInf);
        const float base = top == -kInf ? 0.f : top;
        double at_log = 0.0;                                 // the gradient at the slot's log p, under a sigmoid times 1 - p
        float e[kEach], shared = 0.f;                        // without renormalisation under a softmax: an expert's e^(x - base), and what all have for each
        constexpr int kSlots = kLanes < 32 ? kLanes : 32;    // lanes that can have one
        if (a.renormalise) {
            const float most = top_of<kSlots>(sigmoid ? fminf(s, 0.f) : s);
            const double q = mine < 0 || s == -kInf ? 0.0 : weight_of(s, most, sigmoid);
            const double all = sum_of<kSlots>(q), with_dw = sum_of<kSlots>(q * (double)dw);   // every lane takes part
            const double over_all = reciprocal64(all);
            at_log = mine < 0 ? 0.0 : a.factor * (q * over_all) * ((double)dw - with_dw * over_all);
        } else if (!sigmoid) {
            float term[kEach];
#pragma unroll
            for (int v = 0; v < kEach; ++v) {
                term[v] = e[v] = __expf(x[v] - base);
            }
            const double over_sum = reciprocal64((double)sum_of<kLanes>(tree_sum(term)));
            at_log = mine < 0 ? 0.0 : a.factor * (double)dw * (exp31((double)s - (double)base) * over_sum);
            shared = (float)(sum_of<kLanes>(at_log) * over_sum);
        } else if (mine >= 0) {
            at_log = a.factor * (double)dw * weight_of(s, 0.f, true);
        }
        if (sigmoid && mine >= 0) at_log *= rest_of(s);
        const float at_slot = (float)at_log;
        // an expert that is named twice (not by groot_route) gets both, in the order of the slots
        if (mine >= 0) at[mine] = __int_as_float(lane);
        wave_sync();
        const bool twice = any_of<kLanes>(mine >= 0 && __float_as_int(at[mine]) != lane);
        wave_sync();
#pragma unroll
        for (int v = 0; v < kEach; ++v) at[begin + v] = 0.f;
        wave_sync();
        if (!twice) {
            if (mine >= 0) at[mine] = at_slot;
        } else {
            for (int32_t slot = 0; slot < a.k; ++slot) {
                if (lane == slot && mine >= 0) at[mine] += at_slot;
                wave_sync();
            }
        }
        wave_sync();
        float r[kEach];
#pragma unroll
        for (int v = 0; v < kEach; ++v) {
            r[v] = at[begin + v];
            if (!sigmoid && !a.renormalise) r[v] -= e[v] * shared;
            if (x[v] == -kInf) r[v] = 0.f;
            if (broken) r[v] = __builtin_nanf("");
        }
        wave_sync();                                         // before the next row's
        char *const to = (char *)a.dscores + row * a.ds_bytes;
        if (a.dtype == GROOT_F32) put_scores<kEach, float>(to, a.E, begin, whole, r);
        else if (a.dtype == GROOT_BF16) put_scores<kEach, bf16_t>(to, a.E, begin, whole, r);
        else put_scores<kEach, f16_t>(to, a.E, begin, whole, r);
    }
}

// lanes of a row
int32_t route_lanes(int32_t E)
{
    int32_t lanes = 1;
    while (lanes * 16 < E) lanes *= 2;
    return lanes;
}
// Rows of a workgroup.  All of them where its threads hold them at once: one launch (64 rows of 128 scores in bfloat16: 4.5 us, 6.8 in two
// launches).  Otherwise few, down to a wavefront's, while the workgroups are no more than the second launch adds up by itself (128 rows of 256: 7.9
// us, 10.4 with 64 rows a workgroup; 2000 rows of 64: 7.5 and 7.1).
int32_t route_rows(int64_t n, int32_t E)
{
    const int32_t lanes = route_lanes(E);
    if (n <= kRouteRows && n * lanes <= kRouteThreads) return kRouteRows;
    int32_t rows = kWave / lanes;
    while (rows < kRouteRows && (n + rows - 1) / rows > kSumGroups) rows *= 2;
    return rows;
}
size_t count_bytes(int64_t groups, int32_t E) { return ((size_t)groups * count_words(E) * 4 + 15) / 16 * 16; }
int64_t route_groups(int64_t n, int32_t rows) { return n <= 0 ? 1 : (n + rows - 1) / rows; }

template <int kLanes, int kEach, int kList, bool kByValue, bool kSets>
int route_launch(RouteArgs a, uint32_t *counts, hipStream_t stream)
{
    a.rows = route_rows(a.n, a.E);
    a.inverse_k = inverse_of(a.k);
    const int64_t groups = route_groups(a.n, a.rows);
    int threads = (int)(a.n < a.rows ? (a.n < 1 ? 1 : a.n) : a.rows) * kLanes;
    threads = threads >= kRouteThreads ? kRouteThreads : (threads + kWave - 1) / kWave * kWave;
    a.set_lanes = 0;
    a.small_sets = a.wide_sets = false;
    a.value_bytes = 0;
    if (kSets) {
        const int32_t size = a.E / a.sets, lanes = size / kEach;
        if (size % kEach == 0 && (lanes & (lanes - 1)) == 0 && lanes <= 32) {
            a.set_lanes = lanes;
            a.value_bytes = threads / kLanes * a.sets * 8;
        } else if (size >= kEach) {
            a.wide_sets = true;
            a.value_bytes = threads / kLanes * (a.sets + 4 * kLanes) * 8;
        } else if (size == 1 || size == 2 || size == 4 || size == 8) {
            a.small_sets = true;
            a.value_bytes = threads / kLanes * a.sets * 8;
        } else {
            auto bytes = [&] { return threads / kLanes * (kLanes * kEach + a.sets) * 8; };
            while (threads > kWave && bytes() > 32 * 1024) threads = (threads / 2 + kWave - 1) / kWave * kWave;
            a.value_bytes = bytes();
        }
    }
    if (!fits_launch(groups, threads)) return kErrTooManyTiles;
    route_kernel<kLanes, kEach, kList, kByValue, kSets><<<(uint32_t)groups, threads, RouteLds(a.E, a.rows, a.k, a.value_bytes).total, stream>>>(a, counts);
    if (groups > 1) {
        const size_t lds = (2 * a.E + 1 + kMaxWaves) * sizeof(int32_t);
        int32_t *const before = (int32_t *)((char *)counts + count_bytes(groups, a.E));
        if (groups > kSumGroups) {
            route_scan_kernel<<<(a.E + kScanExperts - 1) / kScanExperts, kScanExperts * kScanParts, 0, stream>>>(counts, before, (int32_t)groups, a.E);
            const int fit = fits_launch(groups, kBlock) ? kBlock : threads;   // from 2^30 rows on a launch holds no more lanes than the search's
            route_place_kernel<true><<<(uint32_t)groups, fit, lds, stream>>>(a, counts, before, (int32_t)groups);
        } else {
            route_place_kernel<false><<<(uint32_t)groups, 1024, lds, stream>>>(a, counts, before, (int32_t)groups);
        }
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
    const int64_t groups = route_groups(n, route_rows(n, E));
    return groups == 1 ? 0 : count_bytes(groups, E) + (groups > kSumGroups ? (size_t)(groups + 1) * E * sizeof(int32_t) : 0);
}

// 16 experts a lane (8 where there are no more), lists as long as top_k needs
typedef int (*RouteLaunch)(RouteArgs, uint32_t *, hipStream_t);
template <int kLanes, bool kByValue, bool kSets>
static RouteLaunch route_of_lanes(const RouteArgs &a)
{
    return a.k <= 4   ? route_launch<kLanes, 16, 4, kByValue, kSets>
           : a.k <= 8 ? route_launch<kLanes, 16, 8, kByValue, kSets>
                      : route_launch<kLanes, 16, 16, kByValue, kSets>;
}
template <bool kByValue, bool kSets>
static RouteLaunch route_for(const RouteArgs &a)
{
    if (a.E <= 8) return a.k <= 4 ? route_launch<1, 8, 4, kByValue, kSets> : route_launch<1, 8, 8, kByValue, kSets>;
    if (a.E <= 16) return route_of_lanes<1, kByValue, kSets>(a);
    if (a.E <= 32) return route_of_lanes<2, kByValue, kSets>(a);
    if (a.E <= 64) return route_of_lanes<4, kByValue, kSets>(a);
    if (a.E <= 128) return route_of_lanes<8, kByValue, kSets>(a);
    if (a.E <= 256) return route_of_lanes<16, kByValue, kSets>(a);
    if (a.E <= 512) return route_of_lanes<32, kByValue, kSets>(a);
    return route_of_lanes<64, kByValue, kSets>(a);
}

// 16 lanes a row while they hold its experts and slots, a wavefront otherwise
typedef int (*BackwardLaunch)(const RouteBackwardArgs &, hipStream_t);
static BackwardLaunch backward_for(const RouteBackwardArgs &a)
{
    if (a.E > 256 || a.k > 16) return a.E <= 512 ? backward_launch<64, 8> : backward_launch<64, 16>;
    if (a.E <= 16) return backward_launch<16, 1>;
    if (a.E <= 32) return backward_launch<16, 2>;
    if (a.E <= 64) return backward_launch<16, 4>;
    if (a.E <= 128) return backward_launch<16, 8>;
    return backward_launch<16, 16>;
}

int launch_route(const RouteArgs &a, void *workspace, void *stream)
{
    const bool sets = a.open_sets < a.sets;
    const RouteLaunch launch = a.by_value ? (sets ? route_for<true, true>(a) : route_for<true, false>(a)) : (sets ? route_for<false, true>(a) : route_for<false, false>(a));
    return launch(a, (uint32_t *)workspace, (hipStream_t)stream);
}
int launch_route_backward(const RouteBackwardArgs &a, void *stream) { return backward_for(a)(a, (hipStream_t)stream); }

}  // namespace groot
