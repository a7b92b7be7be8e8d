// One token from each row of logits: temperature, top-k, top-p and min-p, from given uniform numbers.
//
// The tokens of a row are ordered by falling logit, the lower index first among equals; each of the filters keeps a first part of
// that order, so all of them together are one border: a logit, and how many of the tokens that have just it.  Weights are
// exp((logit - largest) / temperature) as whole multiples of 2^-43, computed in 64 bits: their sums are exact and in no order, and
// a token is decided by which side of a border a sum of up to a million of them lies on.
#include "kv8.h"

namespace mq {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr double kUnit = (double)(1ll << 43);

// Logits as unsigned numbers of the same order: NaN as -infinity, the two zeros as one
static __device__ __forceinline__ uint32_t key_of(float x)
{
    x = x != x ? -__builtin_inff() : x + 0.0f;
    const uint32_t u = __float_as_uint(x);
    return u >> 31 ? ~u : u | 0x80000000u;
}
static __device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }

template <class T>
static __device__ __forceinline__ float load_logit(const T *p, int64_t i)
{
    if constexpr (sizeof(T) == 2)
        return __uint_as_float((uint32_t)p[i] << 16);
    else
        return p[i];
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_kernel(Sample a)
{
    __shared__ unsigned long long mass[256];
    __shared__ uint32_t count[256];
    __shared__ unsigned long long parts[kWaves];
    __shared__ int counts[kWaves];
    __shared__ unsigned long long found_mass;
    __shared__ int found_digit, found_at;
    __shared__ uint32_t found_count;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = (int)a.V;
    const int64_t r = blockIdx.x;
    const T *const row = reinterpret_cast<const T *>(a.logits) + r * a.ld;

    // the first of the order: the largest key, the lowest index
    unsigned long long best = 0;
    for (int i = tid; i < V; i += kThreads) best = max(best, ((unsigned long long)key_of(load_logit(row, i)) << 32) | (uint32_t)~i);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) best = max(best, (unsigned long long)__shfl_xor((long long)best, d));
    if (lane == 0) parts[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = max(best, parts[w]);
    __syncthreads();
    const uint32_t top_key = (uint32_t)(best >> 32);
    const float top = value_of(top_key);
    const float t = a.temperature ? a.temperature[r] : 1.0f, p = a.top_p ? a.top_p[r] : 1.0f, mp = a.min_p ? a.min_p[r] : 0.0f;
    const int k = a.top_k ? a.top_k[r] : 0;
    if (top == -__builtin_inff() || !(t > 0.0f) || k == 1 || !(p > 0.0f) || mp != mp || mp > 1.0f) {
        if (tid == 0) a.tokens[r] = top == -__builtin_inff() ? -1 : (int)~(uint32_t)best;
        return;
    }
    auto weight = [&](uint32_t key) -> double {
        const float x = value_of(key);
        if (x == top) return 1.0;
        return x == -__builtin_inff() || top == __builtin_inff() ? 0.0 : exp(((double)x - (double)top) / (double)t);
    };
    auto whole = [&](double w) { return (unsigned long long)(w * kUnit + 0.5); };

    // The border: the first element of the order with which the count, or the mass, reaches the limit.  `ties` of the elements with
    // border_key are kept, `before` is the mass in front of them.
    uint32_t border_key = 0;
    long long ties = V;
    auto find = [&](bool by_mass, double limit, unsigned long long &before) {
        uint32_t prefix = 0, n_before = 0;
        before = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) mass[tid] = 0, count[tid] = 0;
            __syncthreads();
            for (int i = tid; i < V; i += kThreads) {
                const uint32_t key = key_of(load_logit(row, i));
                if (shift < 24 && (key >> (shift + 8)) != prefix) continue;
                atomicAdd(&count[key >> shift & 255], 1u);
                atomicAdd(&mass[key >> shift & 255], whole(weight(key)));
            }
            __syncthreads();
            if (tid == 0) {
                int d = 255, last = 0;
                for (; d >= 0; --d) {
                    if (!count[d]) continue;
                    last = d;
                    if (by_mass ? (double)(before + mass[d]) >= limit : (double)(n_before + count[d]) >= limit) break;
                    before += mass[d], n_before += count[d];
                }
                if (d < 0) before -= mass[last], n_before -= count[last], d = last;  // (the limit is beyond all of them)
                found_digit = d, found_mass = before, found_count = n_before;
            }
            __syncthreads();
            prefix = prefix << 8 | (uint32_t)found_digit, before = found_mass, n_before = found_count;
            __syncthreads();
        }
        border_key = prefix;
        const unsigned long long w = whole(weight(prefix));
        if (!by_mass)
            ties = (long long)(limit - n_before);
        else
            ties = w == 0 ? 1 : max((long long)ceil((limit - (double)before) / (double)w), 1ll);
    };
    unsigned long long before = 0, all = 0;
    auto sum_of = [&](auto &&of) {
        unsigned long long s = 0;
        for (int i = tid; i < V; i += kThreads) s += of(key_of(load_logit(row, i)));
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) s += (unsigned long long)__shfl_xor((long long)s, d);
        if (lane == 0) parts[wave] = s;
        __syncthreads();
        s = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += parts[w];
        __syncthreads();
        return s;
    };
    if (k > 0 && k < V) find(false, k, before);
    if (p < 1.0f) {
        const unsigned long long w = whole(weight(border_key));
        all = border_key ? before + (unsigned long long)ties * w : sum_of([&](uint32_t key) { return whole(weight(key)); });
        find(true, (double)p * (double)all, before);
    }
    auto kept = [&](uint32_t key) { return key >= border_key && (key == top_key || weight(key) >= (double)mp); };

    // the kept tokens in the order of their indices, a thousand at a time, twice: their mass, then where it passes the draw
    unsigned long long total = 0, aim = 0;
    for (int pass = 0; pass < 2; ++pass) {
        unsigned long long sum = 0;
        long long seen = 0;
        if (tid == 0) found_at = -1;
        for (int base = 0; base < V; base += kThreads) {
            const int i = base + tid;
            const uint32_t key = i < V ? key_of(load_logit(row, i)) : 0;
            const bool tie = i < V && key == border_key;
            const unsigned long long tied = __ballot(tie);
            if (lane == 0) counts[wave] = __popcll(tied);
            __syncthreads();
            long long rank = seen + __popcll(tied & ((1ull << lane) - 1));
            for (int w = 0; w < kWaves; ++w) {
                if (w < wave) rank += counts[w];
                seen += counts[w];
            }
            unsigned long long m = i < V && kept(key) && (!tie || rank < ties) ? whole(weight(key)) : 0, upto = m;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const unsigned long long u = (unsigned long long)__shfl_up((long long)upto, d);
                if (lane >= d) upto += u;
            }
            if (lane == 63) parts[wave] = upto;
            __syncthreads();
            unsigned long long front = sum;
            for (int w = 0; w < kWaves; ++w) {
                if (w < wave) front += parts[w];
                sum += parts[w];
            }
            if (pass && m && front <= aim && front + upto > aim && front + upto - m <= aim) found_at = i;
            __syncthreads();
        }
        total = sum;
        const double u = (double)a.uniform[r] * (double)total;
        aim = u > 0.0 ? (u < (double)total ? (unsigned long long)u : total - 1) : 0;
        aim = min(aim, total - 1);
    }
    if (tid == 0) a.tokens[r] = found_at;
}

int64_t sample_workspace(int64_t rows, int64_t V)
{
    (void)rows, (void)V;
    return 0;
}

int launch_sample(const Sample &a, bool fp32, hipStream_t s)
{
    return fp32 ? enqueue(sample_kernel<float>, dim3((unsigned)a.rows), dim3(kThreads), 0, s, a)
                : enqueue(sample_kernel<uint16_t>, dim3((unsigned)a.rows), dim3(kThreads), 0, s, a);
}

}  // namespace mq
