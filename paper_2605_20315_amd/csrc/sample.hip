// One token from each row of logits: temperature, top-k, top-p and min-p, from given uniform numbers.
//
// The tokens of a row are ordered by falling logit, the lower index first among equals; each of the filters keeps a first part of
// that order, so all of them together are one border in it.  Nothing is sorted: the logits are counted into bins, and only
// the tokens of the border's own bin are looked at one by one.
//
// With pos = 8 log2(e) logit / temperature, in binary64, a token's weight is 2^(pos / 8) over a common factor, and its bin is
// floor(pos): the same for every part of a row, whatever the largest logit there, so that parts are counted by themselves and put
// together by shifting.  Weights in a bin lie between 2^-1/8 and 1 of its top, and a bin's mass is its count less
// what its weights fall short of one: 64 bits hold both, 2^-34 of a weight fine, and one addition in LDS counts a token.
// Such masses tell where a border or a draw is to about 2^-30 of them.  Where it falls exactly between two tokens the answer goes by whole
// numbers: of tokens for top_p (only equal weights have such borders), of one weight a token for the draw.
//
// Three kernels.  sample_chunks reads the logits once, a chunk of a row by a workgroup: the largest, the mass, and where the row has
// filters the count and mass up to each of the 512 bins below the chunk's largest (weights down to 2^-64).  sample_border, several workgroups a row:
// the row's own sums from those, the bins that the borders are in, and their tokens.  sample_rows, a workgroup a row: the borders among those
// tokens, the chunk that the draw falls into, the token.  Without filters the first and the last are all; a row of one chunk needs only the last.
// 64 rows of 151673 with all filters, BF16: 44 to 46 us (16, 13 and 15 and what lies between); a large copy would read them in 4.  Counting in 64 bits bounds
// the first (22 vector instructions and an addition in LDS a logit), trips to memory and to a barrier one after another the others, as they do
// all of one row's 22 us.  500 rows of 100003 in FP32 by temperature alone: 53 to 69 us by card, 41 by a large copy; reading takes as long as the 20
// instructions of each weight's power of two, and the two overlap in part.
#include "kv8.h"

namespace mq {

typedef unsigned long long u64;
constexpr int kBins = 512;
constexpr int kCountBit = 47;  // a bin of a chunk: count << 47 | shortfall in 2^-34, at most 2^14 * 2^30.4
constexpr double kFine = (double)(1ll << 34);
constexpr int kChunkThreads = 256, kBorderThreads = 1024, kRowThreads = 512;
constexpr int kChunk = 8192;  // logits
constexpr int kChunksMost = (int)(kSampleTokens / kChunk);  // of a row

struct Chunk {
    float top;    // the largest logit
    int first;    // its lowest index (of a row that takes the largest)
    double mass;  // over that of the top of the largest logit's bin
};

// Count and mass of a chunk up to a bin in one word: count << 50 | mass in 2^-36 of the weight at the end of the octave that the largest logit is
// in (an octave is eight bins, the ends at multiples of eight), so that one chunk's masses become another's by shifts
struct Upto {
    u64 word;
};
constexpr int kUptoCount = 50;
constexpr double kUptoUnit = 0x1p36;
static __device__ __forceinline__ u64 mass_of(Upto u) { return u.word & ((1ull << kUptoCount) - 1); }
static __device__ __forceinline__ int count_of(Upto u) { return (int)(u.word >> kUptoCount); }
// the octave's end over eight, and the bins from the end of bin `edge` to it, 0 to 7
static __device__ __forceinline__ double octave_of(double edge) { return ceil((edge + 1.0) * 0.125); }
static __device__ __forceinline__ int bins_to_octave(double edge) { return (int)fmin(fmax(8.0 * octave_of(edge) - (edge + 1.0), 0.0), 7.0); }

// What of a row's borders goes by the bins alone: the bins of the three borders, those of the mass's between what it is at least
// and at most (what the first k have is only known to a bin)
struct Borders {
    int k, m, p0, p1;
    bool part_k;     // whether the first k end inside their bin
    double limit_m;  // the pos of min_p's
};

// What is known of a row with filters: the masses and counts up to each bin below its largest logit's, and the tokens, as numbers, of the
// bins that a border may be in (listed may be more than there is room for: then sample_rows reads the row again for each of its passes, by
// itself.  64 rows of 262144 with logits of deviation 2.2 and top_p of 0.95 62 us at a temperature of 1, 491 at 1.3, where a bin
// holds more; 64 of 151673 54 us at 1.5, 306 at 2; of equal logits 1810)
constexpr int kList = 4096;
struct Row {
    double masses[kBins];
    int counts[kBins];
    double min_bits;  // bins from the largest logit's pos to the min_p border's, less than zero
    Borders borders;
    int listed;
    u64 list[kList];
};

// The workspace: a Chunk for each chunk of a launch's rows, and for rows with filters the masses and counts up to each bin, and a Row
struct Tables {
    Chunk *chunks;
    Upto *upto;
    Row *rows;
};
constexpr int64_t kChunkBytes = sizeof(Chunk) + kBins * sizeof(Upto);

struct Setting {
    double scale, inverse;  // pos over logit, and logit over pos
    // The share of the mass in front of which tokens are kept: top_p, taken down by what the bins' masses and the border's may be apart, so that a
    // token that has it in front of it in binary64 (temperatures beyond the logits' differences make weights of one) is not kept
    double share;
    int k;
    float p, min_p;
    bool largest, filters;
};

static __device__ __forceinline__ Setting setting_of(const Sample &a, int64_t r)
{
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    Setting s;
    s.k = a.top_k ? a.top_k[r] : 0;
    s.p = a.top_p ? a.top_p[r] : 1.0f;
    s.min_p = a.min_p ? a.min_p[r] : 0.0f;
    s.share = (double)s.p * (1.0 - 0x1p-33);
    s.largest = !(t > 0.0f) || s.k == 1 || !(s.p > 0.0f) || s.min_p != s.min_p || s.min_p > 1.0f;
    if (s.k <= 0 || s.k >= a.V) s.k = 0;
    s.filters = s.k > 0 || s.p < 1.0f || s.min_p > 0.0f;
    s.scale = 8.0 * 1.4426950408889634074 / (double)t;
    s.inverse = (double)t * (0.69314718055994530942 / 8.0);
    return s;
}

// Where a logit lies, given the largest: +infinity leaves weight to nothing else, and nothing is above it
static __device__ __forceinline__ double pos_of(float x, float top, double scale) { return top == __builtin_inff() ? 0.0 : (double)x * scale; }
static __device__ __forceinline__ bool weighs(float x, float top) { return top == __builtin_inff() ? x == top : x != -__builtin_inff(); }

// 2^((f - 1) / 8) for f in 0 .. 1: the sixth-order Taylor polynomial about 1/2, within 6e-14
static __device__ __forceinline__ double in_bin(double f)
{
    constexpr double h = 0.086643397569993163677, s = 0.95760328069857364694;  // ln(2) / 8, 2^(-1/16)
    const double z = f - 0.5;
    double w = s * h * h * h * h * h * h / 720;
    w = __builtin_fma(w, z, s * h * h * h * h * h / 120);
    w = __builtin_fma(w, z, s * h * h * h * h / 24);
    w = __builtin_fma(w, z, s * h * h * h / 6);
    w = __builtin_fma(w, z, s * h * h / 2);
    w = __builtin_fma(w, z, s * h);
    return __builtin_fma(w, z, s);
}

// 2^y for y <= 0: the Taylor polynomial of order 11 about the nearest whole number, within 7e-15; nothing below 2^-1000
static __device__ __forceinline__ double power(double y)
{
    constexpr double h = 0.69314718055994530942;
    constexpr double c[12] = {1, h, h * h / 2, h * h * h / 6, h * h * h * h / 24, h * h * h * h * h / 120, h * h * h * h * h * h / 720,
                              h * h * h * h * h * h * h / 5040, h * h * h * h * h * h * h * h / 40320, h * h * h * h * h * h * h * h * h / 362880,
                              h * h * h * h * h * h * h * h * h * h / 3628800, h * h * h * h * h * h * h * h * h * h * h / 39916800};
    y = fmax(y, -1000.0);
    const double shifted = y + 0x1.8p52, z = y - (shifted - 0x1.8p52);
    double w = c[11];
#pragma unroll
    for (int i = 10; i >= 0; --i) w = __builtin_fma(w, z, c[i]);
    return __builtin_bit_cast(double, __builtin_bit_cast(u64, w) + (__builtin_bit_cast(u64, shifted) << 52));
}

// 2^(v / 32) from 2^(i / 32), i < 32, and a polynomial of order 4 about the nearest whole v, within 2e-12; nothing below 2^-1000
static __device__ __forceinline__ double power32(double v, const double *powers)
{
    constexpr double h = 0.021660849392498290919;  // ln(2) / 32
    v = fmax(v, -32000.0);
    const double shifted = v + 0x1.8p52, z = v - (shifted - 0x1.8p52);
    double w = h * h * h * h / 24;
    w = __builtin_fma(w, z, h * h * h / 6);
    w = __builtin_fma(w, z, h * h / 2);
    w = __builtin_fma(w, z, h);
    w = __builtin_fma(w, z, 1.0);
    const int n = (int)(uint32_t)__builtin_bit_cast(u64, shifted);
    return __builtin_ldexp(w * powers[n & 31], n >> 5);
}

// 2^(-b / 8)
static __device__ __forceinline__ double eighth(int b)
{
    constexpr double e1 = 0.91700404320467123175, e2 = 0.84089641525371454303, e4 = 0.70710678118654752440;  // of one, two and four eighths
    return __builtin_ldexp((b & 1 ? e1 : 1.0) * (b & 2 ? e2 : 1.0) * (b & 4 ? e4 : 1.0), -(b >> 3));
}

// u times a total of less than 2^63, rounded down: exact, so that a sum that is u times the total is not below it.  For u <= 0
// and NaN 0, for u >= 1 what 1 - 2^-40 gives.
static __device__ __forceinline__ u64 share_of(float u, u64 total)
{
    if (!(u > 0.0f)) return 0;
    if (!(u < 1.0f)) return total - ((total + ((1ull << 40) - 1)) >> 40);
    const uint32_t bits = __float_as_uint(u), exponent = bits >> 23, by = 150 - max(exponent, 1u);  // u is m / 2^by
    const u64 m = (bits & 0x7fffffu) | (exponent > 0 ? 0x800000u : 0u), lo = m * total, hi = __umul64hi(m, total);
    return by < 64 ? lo >> by | hi << (64 - by) : by < 128 ? hi >> (by - 64) : 0;
}

// Logits as unsigned numbers of the same order, the two zeros as one
static __device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
static __device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }

// The lowest logit (as a key) with a pos of at least `limit` that has weight: pos is monotonous in it, and the quotient less than a step off,
// so a lane tries each of the four around it.  (Of the whole wave.)
static __device__ __forceinline__ uint32_t lowest(const Setting &s, float top, double limit)
{
    if (top == __builtin_inff()) return 0xff800000u;
    if (s.scale == 0.0) return 0x00800000u;
    const float y = (float)fmin(fmax(limit * s.inverse, -3.4028234663852886e38), 3.4028234663852886e38);
    const uint32_t key = max(key_of(y) - 2, 0x00800000u);  // (what is in front of it is no number)
    return key + __popcll(__ballot((double)value_of(key + (threadIdx.x & 3)) * s.scale < limit) & 15);
}

typedef uint32_t words2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(4)));

// 16 bytes of a row from element i on (aligned to an element); what lies behind the row as -infinity
template <class T>
static __device__ __forceinline__ u32x4 load16(const T *row, int i, int V)
{
    constexpr int N = 16 / sizeof(T);
    if (i + N <= V) return *reinterpret_cast<const std::conditional_t<sizeof(T) == 2, words2, words4> *>(row + i);
    uint32_t e[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if constexpr (sizeof(T) == 2)
            e[j] = i + j < V ? row[i + j] : 0xff80u;
        else
            e[j] = i + j < V ? __float_as_uint(row[i + j]) : 0xff800000u;
    }
    if constexpr (sizeof(T) == 2)
        return u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
    else
        return u32x4{e[0], e[1], e[2], e[3]};
}

// the j-th of them
template <class T>
static __device__ __forceinline__ float bits_of(u32x4 w, int j)
{
    if constexpr (sizeof(T) == 2)
        return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    else
        return __uint_as_float(w[j]);
}

// NaN as -infinity
template <class T>
static __device__ __forceinline__ float logit_of(u32x4 w, int j)
{
    const float x = bits_of<T>(w, j);
    return x == x ? x : -__builtin_inff();
}

// bits_of for a j that is not known to the compiler
template <class T>
static __device__ __forceinline__ float pick(u32x4 w, int j)
{
    const int k = sizeof(T) == 2 ? j >> 1 : j;
    uint32_t v = w[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) v = k == i ? w[i] : v;
    if constexpr (sizeof(T) == 2) v = j & 1 ? v & 0xffff0000u : v << 16;
    return __uint_as_float(v);
}

// v of the lane that a cross-lane control names, `none` where it names none.  (In registers: a step of a scan through LDS waits 100 cycles, and
// these kernels have little else to do meanwhile.)
template <int CONTROL, int ROWS, class T>
static __device__ __forceinline__ T moved(T v, T none)
{
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) / 4)));
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CONTROL, ROWS, 0xf, false));
    } else {
        words x = __builtin_bit_cast(words, v);
        const words y = __builtin_bit_cast(words, none);
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = (uint32_t)__builtin_amdgcn_update_dpp((int)y[i], (int)x[i], CONTROL, ROWS, 0xf, false);
        return __builtin_bit_cast(T, x);
    }
}

// Of each lane what f makes of it and the lanes in front: rows of 16 lanes by shifts of 1, 2, 4 and 8, then each row's last to the next
// row, and the lower half's last to the upper.  none: what f leaves all values as they are with.
template <class T, class F>
static __device__ __forceinline__ T wave_scan(T v, T none, F &&f)
{
    v = f(v, moved<0x111, 0xf>(v, none));
    v = f(v, moved<0x112, 0xf>(v, none));
    v = f(v, moved<0x114, 0xf>(v, none));
    v = f(v, moved<0x118, 0xf>(v, none));
    v = f(v, moved<0x142, 0xa>(v, none));
    return f(v, moved<0x143, 0xc>(v, none));
}

template <class T>
static __device__ __forceinline__ T lane_of(T v, int lane)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else {
        typedef uint32_t words __attribute__((ext_vector_type(2)));
        words x = __builtin_bit_cast(words, v);
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = (uint32_t)__builtin_amdgcn_readlane((int)x[i], lane);
        return __builtin_bit_cast(T, x);
    }
}

static __device__ __forceinline__ float wave_max(float v) { return lane_of(wave_scan(v, -__builtin_inff(), [](float x, float y) { return fmaxf(x, y); }), 63); }
static __device__ __forceinline__ int wave_min(int v) { return lane_of(wave_scan(v, 0x7fffffff, [](int x, int y) { return min(x, y); }), 63); }
// the sum of a lane's and those in front
template <class T>
static __device__ __forceinline__ T sum_to(T v) { return wave_scan(v, T(0), [](T x, T y) { return x + y; }); }

// One more token, and what its weight falls short of one
static __device__ __forceinline__ void count_in_bin(float y, float top, double scale, double edge, u64 *bins)
{
    const double pos = pos_of(y, top, scale), q = floor(pos);
    // 2^52 more than the shortfall, whose bits are then the low ones
    const double d = __builtin_fma(in_bin(pos - q), -kFine, kFine + 0x1p52);
    atomicAdd(&bins[(int)(edge - q)], (1ull << kCountBit) + (__builtin_bit_cast(u64, d) - 0x4330000000000000ull));
}
// the mass of bin b over that of the first bin's top
static __device__ __forceinline__ double mass_in_bin(u64 bin, int b)
{
    return ((double)((bin >> kCountBit) << 34) - (double)(bin & ((1ull << kCountBit) - 1))) * (1.0 / kFine) * eighth(b);
}

// One chunk of kChunk logits.  They stay in LDS, so that the loop over them is no longer than its body: unrolled, the
// code alone (12 KB read once by each compute unit) takes longer than the logits.
template <class T>
__global__ __launch_bounds__(kChunkThreads) void sample_chunks(Sample a, Tables t, int64_t row0, int chunks)
{
    constexpr int N = 16 / sizeof(T), NV = kChunk / kChunkThreads / N, NW = kChunkThreads / 64;
    __shared__ u32x4 stage[NV][kChunkThreads];
    __shared__ u64 bins[kBins];
    __shared__ int largest[kBins];
    __shared__ float tops[NW];
    __shared__ int firsts[NW];
    __shared__ double sums[NW], powers[32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = (int)a.V;
    const int local = blockIdx.x / chunks, c = blockIdx.x - local * chunks, base = c * kChunk;
    const int64_t r = row0 + local;
    const T *const row = reinterpret_cast<const T *>(a.logits) + r * a.ld;
    const Setting s = setting_of(a, r);
    float top = -__builtin_inff();
    {
        u32x4 x[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) x[j] = load16(row, base + (j * kChunkThreads + tid) * N, V);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            stage[j][tid] = x[j];
#pragma unroll
            for (int i = 0; i < N; i += 2) top = fmaxf(top, fmaxf(bits_of<T>(x[j], i), bits_of<T>(x[j], i + 1)));  // (the maximum of a number and NaN is the number)
        }
    }
    const float mine = top;
    top = wave_max(top);
    if (lane == 0) tops[wave] = top;
    bins[2 * tid] = bins[2 * tid + 1] = 0, largest[2 * tid] = largest[2 * tid + 1] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, tops[w]);
    Chunk *const out = t.chunks + blockIdx.x;
    if (s.largest) {
        int first = 0x7fffffff;
#pragma unroll 1
        for (int j = NV - 1; j >= 0; --j) {
            const u32x4 x = stage[j][tid];
#pragma unroll
            for (int i = N - 1; i >= 0; --i)
                if (logit_of<T>(x, i) == top) first = base + (j * kChunkThreads + tid) * N + i;
        }
        first = wave_min(first);
        if (lane == 0) firsts[wave] = first;
        __syncthreads();
        if (tid == 0) {
#pragma unroll
            for (int w = 0; w < NW; ++w) first = min(first, firsts[w]);
            *out = Chunk{top, first, 0.0};
        }
        return;
    }
    const double edge = floor(pos_of(top, top, s.scale));  // the largest logit's bin
    const double min_bits = s.min_p > 0.0f && (c == 0 || s.p >= 1.0f) ? 8.0 * log2((double)s.min_p) : 0.0;
    if (s.filters && tid == 0 && c == 0) t.rows[local].listed = 0, t.rows[local].min_bits = min_bits;
    if (!s.filters || top == -__builtin_inff()) {
        // (in 64 bits these few instructions take as long as the loads; NaN and -infinity come out as 2^-1000)
        if (tid < 32) powers[tid] = power(0.03125 * tid);
        __syncthreads();
        double sum = 0.0;
        const double from = -(edge + 1.0) * 4;
        if (top == __builtin_inff()) {
#pragma unroll 1
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) sum += bits_of<T>(stage[j][tid], i) == top ? powers[28] * 0.5 : 0.0;  // (2^(-1/8), the bottom of its bin)
        } else {
#pragma unroll 1
            for (int j = 0; j < NV; ++j) {
                const u32x4 x = stage[j][tid];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    sum += power32(__builtin_fma((double)bits_of<T>(x, i) * s.scale, 4.0, from), powers);
                }
            }
        }
        sum = sum_to(sum);
        if (lane == 63) sums[wave] = sum;
        __syncthreads();
        if (tid == 0) {
            sum = 0.0;
#pragma unroll
            for (int w = 0; w < NW; ++w) sum += sums[w];
            *out = Chunk{top, 0, sum};
        }
        return;
    }
    // Bins behind which nothing counts: behind those of the largest k of the threads' largest, and behind what min_p leaves where the
    // mass of the others is not asked for.  An addition in LDS
    // to a bin that lanes share waits for them (64 rows of 151673 with all filters: sample_chunks 18 us, 22 without).  What is behind is found by its logit.
    double last = kBins - 1;
    if (s.k > 0 && s.k <= kChunkThreads) {
        const double below = edge - floor(pos_of(mine, top, s.scale));
        if (weighs(mine, top) && below < kBins) atomicAdd(&largest[(int)below], 1);
        __syncthreads();
        const int n0 = largest[2 * tid], n1 = n0 + largest[2 * tid + 1];
        int n = sum_to(n1);
        if (lane == 63) firsts[wave] = n;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w)
            if (w < wave) n += firsts[w];
        const int before = n - n1;
        last = fmin(last, (double)(__syncthreads_count(n < s.k) + __syncthreads_count(before + n0 < s.k)));
    }
    if (s.min_p > 0.0f && s.p >= 1.0f) last = fmin(last, 1.0 - floor(min_bits));
    const float least = value_of(lowest(s, top, edge - last));
#pragma unroll 1
    for (int j = 0; j < NV; ++j) {
        const u32x4 x = stage[j][tid];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = bits_of<T>(x, i);
            if (y >= least) {  // (not for NaN and -infinity)
                count_in_bin(y, top, s.scale, edge, bins);
            }
        }
    }
    __syncthreads();
    // counts and masses up to each bin, two to a thread
    int count[2];
    double mass[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u64 bin = bins[2 * tid + i];
        count[i] = (int)(bin >> kCountBit);
        mass[i] = mass_in_bin(bin, 2 * tid + i);
    }
    int n = sum_to(count[0] + count[1]);
    double m = sum_to(mass[0] + mass[1]);
    if (lane == 63) firsts[wave] = n, sums[wave] = m;
    n -= count[0] + count[1], m -= mass[0] + mass[1];
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w)
        if (w < wave) n += firsts[w], m += sums[w];
    Upto out2[2];
    const double unit = kUptoUnit * eighth(bins_to_octave(edge));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        n += count[i], m += mass[i];
        out2[i] = Upto{(u64)n << kUptoCount | (u64)(m * unit + 0.5)};
    }
    *reinterpret_cast<u32x4 *>(t.upto + (int64_t)blockIdx.x * kBins + 2 * tid) = __builtin_bit_cast(u32x4, out2);
    if (tid == kChunkThreads - 1) *out = Chunk{top, 0, m};
}
static_assert(2 * kChunkThreads == kBins, "two bins a thread");

constexpr int kFew = 128;  // tokens that are compared each with each

struct Token {
    u64 number, weight;  // its place in the order (the first the largest), its weight in 2^-40 of its bin's top
};

// Tokens as numbers in their order: 36 bits, or 52
static_assert(kSampleTokens == 1 << 20, "the bits of an index");
template <class T>
static __device__ __forceinline__ u64 number_of(uint32_t key, int i)
{
    return (u64)(sizeof(T) == 2 ? key >> 16 : key) << 20 | (0xfffff - i);
}

// How many of the sums up to each bin (which rise) are below a limit: each wave looks at all of them, which takes no barrier
template <class T>
static __device__ __forceinline__ int bins_below(const T *upto, T limit, int lane)
{
    int n = 0;
#pragma unroll
    for (int i = 0; i < kBins; i += 64) n += __popcll(__ballot(upto[i + lane] < limit));
    return n;
}
static __device__ __forceinline__ Borders borders_of(const Setting &s, double peak, double edge, double min_bits, const double *masses, const int *counts, int lane)
{
    Borders b{kBins, kBins, kBins, kBins, false, -__builtin_inf()};
    if (s.min_p > 0.0f) {
        b.limit_m = peak + min_bits;
        b.m = (int)fmin(edge - floor(b.limit_m), (double)kBins);
    }
    if (s.k > 0) b.k = bins_below(counts, s.k, lane);
    double most = masses[kBins - 1], least = most;
    if (b.k < kBins) {
        most = least = masses[b.k];
        b.part_k = counts[b.k] > s.k;
        if (b.part_k) least = b.k > 0 ? masses[b.k - 1] : 0.0;
    }
    if (s.p < 1.0f) {
        b.p0 = min(bins_below(masses, s.share * least, lane), b.k);
        b.p1 = min(bins_below(masses, s.share * most, lane), b.k);
    }
    return b;
}

// The bins that a border is in (-1: none), the first and the last of them
struct Wanted {
    int k, m, p0, p1, from, to;
    __device__ __forceinline__ bool has(int bin) const { return bin == k || bin == m || (bin >= p0 && bin <= p1); }
};
static __device__ __forceinline__ Wanted wanted_of(const Setting &s, const Borders &b)
{
    Wanted w;
    w.k = b.k < kBins && b.part_k && (s.p < 1.0f || b.k <= b.m) ? b.k : -1;
    w.m = b.m < kBins && b.m <= b.k && b.m <= b.p1 ? b.m : -1;
    w.p0 = b.p0, w.p1 = min(min(b.p1, b.m), kBins - 1);
    const bool p = w.p0 <= w.p1;
    w.from = min(min(w.k >= 0 ? w.k : kBins, w.m >= 0 ? w.m : kBins), p ? w.p0 : kBins);
    w.to = max(max(w.k, w.m), p ? w.p1 : -1);
    return w;
}

// Tokens into a list of numbers.  The logits between the first bin that is wanted and the last, `least` to `most`, are few as a rule: two
// comparisons in 32 bits find them (-0 may count as in front of 0 there), and what has bins is asked of them alone.
template <class T>
static __device__ __forceinline__ void list_wanted(u32x4 x, int i0, float least, float most, const Setting &s, float top, double edge, const Wanted &w, u64 *list, int *listed)
{
    constexpr int N = 16 / sizeof(T);
    uint32_t some = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float y = bits_of<T>(x, i);
        some |= (uint32_t)(y >= least && y <= most) << i;
    }
#pragma unroll 1
    for (; some; some &= some - 1) {
        const int i = __builtin_ctz(some);
        const float y = pick<T>(x, i);
        if (w.has((int)(edge - floor(pos_of(y, top, s.scale))))) {
            const int slot = atomicAdd(listed, 1);
            if (slot < kList) list[slot] = number_of<T>(key_of(y), i0 + i);
        }
    }
}

// A row's counts and masses up to each bin, and the tokens of the bins that a border is in, a part of the row's chunks by each
// workgroup: as many in all as there are compute units, since each adds up all chunks' sums first (64 rows in 256 workgroups 13 us, in 512
// 15.5; the additions as integers, which 64-bit ones of floating numbers took 1.2 us more for).
template <class T>
__global__ __launch_bounds__(kBorderThreads) void sample_border(Sample a, Tables t, int64_t row0, int chunks, int parts)
{
    constexpr int NT = kBorderThreads, N = 16 / sizeof(T);
    constexpr float kInf = __builtin_inff();
    __shared__ float tops[kChunksMost];
    __shared__ int2 shifts[kChunksMost];  // bins below the row's largest logit's, and octaves
    __shared__ double masses[kBins];
    __shared__ u64 sums[kBins];
    __shared__ int counts[kBins];
    __shared__ u64 list[kList];
    __shared__ int listed, at;
    const int tid = threadIdx.x, lane = tid & 63, V = (int)a.V, local = blockIdx.x / parts, part = blockIdx.x - local * parts;
    const int64_t r = row0 + local;
    const Setting s = setting_of(a, r);
    if (!s.filters || s.largest) return;
    const Chunk *const heads = t.chunks + (int64_t)local * chunks;
    const Upto *const upto = t.upto + (int64_t)local * chunks * kBins;
    Row &out = t.rows[local];
    const double min_bits = out.min_bits;
    float own = -kInf;
    if (tid < chunks) tops[tid] = own = heads[tid].top;
    __syncthreads();
    float top = -kInf;
    for (int c = lane; c < chunks; c += 64) top = fmaxf(top, tops[c]);
    top = wave_max(top);
    if (top == -kInf) return;
    const double peak = pos_of(top, top, s.scale), edge = floor(peak);
    if (tid < chunks) {
        const double below = own == top ? 0.0 : !weighs(own, top) ? kBins : fmin(edge - floor(own * s.scale), (double)kBins);
        shifts[tid] = int2{(int)below, (int)fmin(octave_of(edge) - octave_of(edge - below), 63.0)};
    }
    if (tid == 0) listed = 0;
    __syncthreads();
    {  // half of the chunks by each half of the threads
        const int b = tid & (kBins - 1), half = tid / kBins;
        u64 m = 0;
        int n = 0;
#pragma unroll 8
        for (int c = half; c < chunks; c += NT / kBins) {
            const int2 shift = shifts[c];
            const Upto u{shift.x > b ? 0 : upto[c * kBins + b - min(shift.x, b)].word};
            m += ((mass_of(u) << 1 >> shift.y) + 1) >> 1, n += count_of(u);
        }
        if (half) sums[b] = m, counts[b] = n;
        __syncthreads();
        if (!half) masses[b] = (double)(m + sums[b]) * (1.0 / kUptoUnit) * eighth(-bins_to_octave(edge)), counts[b] += n;
        __syncthreads();
        if (part == 0 && !half) out.masses[b] = masses[b], out.counts[b] = counts[b];
    }
    static_assert(NT == 2 * kBins, "two halves");
    const Borders b = borders_of(s, peak, edge, min_bits, masses, counts, lane);
    if (part == 0 && tid == 0) out.borders = b;
    const Wanted w = wanted_of(s, b);
    if (w.to < 0) return;
    const float least = value_of(lowest(s, top, edge - w.to)), most = w.from > 0 ? value_of(lowest(s, top, edge - w.from + 1) - 1) : kInf;
    const T *const row = reinterpret_cast<const T *>(a.logits) + r * a.ld;
    const int first = (int)((int64_t)chunks * part / parts) * kChunk, end = min(V, (int)((int64_t)chunks * (part + 1) / parts) * kChunk);
#pragma unroll 1
    for (int i0 = first + tid * N; i0 < end; i0 += NT * N) list_wanted<T>(load16(row, i0, V), i0, least, most, s, top, edge, w, list, &listed);
    __syncthreads();
    if (tid == 0) at = listed > 0 ? atomicAdd(&out.listed, listed) : 0;
    __syncthreads();
    for (int i = tid; i < min(listed, kList - at); i += NT) out.list[at + i] = list[i];
}

template <bool F, bool ONE>
struct RowLds {
    float tops[kChunksMost];
    int shift[kChunksMost];  // bins between the row's largest logit and the chunk's; kBins: its weights are none
    double scale[kChunksMost], kept[kChunksMost];
    u64 part[kChunksMost];  // what the border's bin adds to a chunk
    double masses[F ? kBins : 1];  // of the bins up to each
    int counts[F ? kBins : 1];
    u64 list[F ? kList : 1];
    Token few[F ? kFew : 1];
    int listed;
    int digit_counts[F ? 256 : 1];
    u64 digit_masses[F ? 256 : 1];
    u64 found_mass;
    int found, found_n;
    u64 cut;
    u64 fronts[kRowThreads / 64];
    double powers[32];
    int chosen;
    double rest, total;
    bool near;
    u64 bins[F && ONE ? kBins : 1];
    float wave_tops[kRowThreads / 64];
    int wave_counts[kRowThreads / 64];
    double wave_masses[kRowThreads / 64];
};

// One row by one workgroup.  What takes it is one trip to memory after another, and its own code, which each compute unit reads
// once, from memory: so everything that looks at tokens stands here once, in loops.  512 threads, since much of it is done by every wave alike and four
// waves a SIMD wait for each other there (a pass over a border's tokens 1.2 us, 1.7 with 1024).  F: rows may have filters.
// ONE: rows of one chunk, of which it does all in one launch (sample_chunks' counts and sample_border's tokens included): a
// row of 8192 with all filters 11 to 12.4 us by card, 24.1 by three kernels; 500 of 8000 20.2 to 23.5 and 36.5.  (Rows of two chunks the same way gain little, 22 and 24:
// a compute unit's own instructions bound it.)
template <class T, bool F, bool ONE>
__global__ __launch_bounds__(kRowThreads) void sample_rows(Sample a, Tables t, int64_t row0, int chunks)
{
    constexpr int NT = kRowThreads, N = 16 / sizeof(T);
    constexpr float kInf = __builtin_inff();
    __shared__ RowLds<F, ONE> l;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = (int)a.V;
    const int64_t r = row0 + blockIdx.x;
    const T *const row = reinterpret_cast<const T *>(a.logits) + r * a.ld;
    [[maybe_unused]] const Chunk *const parts = t.chunks + (int64_t)blockIdx.x * chunks;
    [[maybe_unused]] const Upto *const upto = t.upto + (int64_t)blockIdx.x * chunks * kBins;
    [[maybe_unused]] const Row &known = t.rows[blockIdx.x];
    const Setting s = setting_of(a, r);
    constexpr int kEach = kChunk / NT, kVectors = kEach / N;  // logits of a chunk side by side to a thread
    const bool filters = F && s.filters && !s.largest;
    [[maybe_unused]] int listed = 0;
    [[maybe_unused]] Borders known_to{};
    u32x4 x[kVectors];
    // the next of them: the first, which goes to the end (registers have no numbers that a loop could go by)
    auto next_vector = [&] {
        const u32x4 v = x[0];
#pragma unroll
        for (int q = 1; q < kVectors; ++q) x[q - 1] = x[q];
        return x[kVectors - 1] = v;
    };
    float top = -kInf;
    double peak, edge;
    if (tid < 32) l.powers[tid] = power(0.03125 * tid);
    if constexpr (ONE) {
        constexpr int NW = NT / 64;
        static_assert(NT == kBins, "a bin a thread");
#pragma unroll
        for (int j = 0; j < kVectors; ++j) x[j] = load16(row, min(tid * kEach + j * N, V), V);
#pragma unroll
        for (int j = 0; j < kVectors; ++j)
#pragma unroll
            for (int i = 0; i < N; i += 2) top = fmaxf(top, fmaxf(bits_of<T>(x[j], i), bits_of<T>(x[j], i + 1)));
        const float mine = top;
        top = wave_max(top);
        if (lane == 0) l.wave_tops[wave] = top;
        if (F) l.bins[tid] = 0;
        if (tid == 0) l.listed = 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, l.wave_tops[w]);
        if (s.largest || top == -kInf) {
            // (threads and waves have their logits in the order of the row)
            const u64 hits = __ballot(mine == top);
            if (lane == 0) l.wave_counts[wave] = hits ? __ffsll(hits) - 1 : -1;
            __syncthreads();
            int from = 0;
            while (from < NW - 1 && l.wave_counts[from] < 0) ++from;
            if (wave == from && lane == l.wave_counts[from]) {
                int first = 0;
#pragma unroll
                for (int j = kVectors - 1; j >= 0; --j)
#pragma unroll
                    for (int i = N - 1; i >= 0; --i)
                        if (bits_of<T>(x[j], i) == top) first = tid * kEach + j * N + i;
                a.tokens[r] = top == -kInf ? -1 : first;
            }
            return;
        }
        peak = pos_of(top, top, s.scale), edge = floor(peak);
        if constexpr (F) if (filters) {
            {
                const float least = value_of(lowest(s, top, edge - (kBins - 1)));
#pragma unroll 1
                for (int j = 0; j < kVectors; ++j) {
                    const u32x4 v = next_vector();
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (bits_of<T>(v, i) >= least) count_in_bin(bits_of<T>(v, i), top, s.scale, edge, l.bins);
                }
            }
            __syncthreads();
            const u64 bin = l.bins[tid];
            int n = sum_to((int)(bin >> kCountBit));
            double m = sum_to(mass_in_bin(bin, tid));
            if (lane == 63) l.wave_counts[wave] = n, l.wave_masses[wave] = m;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NW; ++w)
                if (w < wave) n += l.wave_counts[w], m += l.wave_masses[w];
            l.counts[tid] = n, l.masses[tid] = m;
            __syncthreads();
            known_to = borders_of(s, peak, edge, s.min_p > 0.0f ? 8.0 * log2((double)s.min_p) : 0.0, l.masses, l.counts, lane);
            const Wanted w = wanted_of(s, known_to);
            if (w.to >= 0) {
                const float least = value_of(lowest(s, top, edge - w.to)), most = w.from > 0 ? value_of(lowest(s, top, edge - w.from + 1) - 1) : kInf;
#pragma unroll 1
                for (int j = 0; j < kVectors; ++j) list_wanted<T>(next_vector(), tid * kEach + j * N, least, most, s, top, edge, w, l.list, &l.listed);
            }
            __syncthreads();
            listed = l.listed;
            __syncthreads();
        }
    } else {
        Chunk own{-kInf, 0, 0.0};
        if (tid < chunks) own = parts[tid], l.tops[tid] = own.top;
        if (F && filters) {
            listed = known.listed, known_to = known.borders;
            if (tid < kBins) l.masses[tid] = known.masses[tid], l.counts[tid] = known.counts[tid];
#pragma unroll
            for (int i = 0; i < kList / NT; ++i)
                if (i * NT + tid < listed) l.list[i * NT + tid] = known.list[i * NT + tid];
        }
        __syncthreads();
        for (int c = lane; c < chunks; c += 64) top = fmaxf(top, l.tops[c]);
        top = wave_max(top);
        if (s.largest || top == -kInf) {
            if (wave == 0) {
                int first = 0x7fffffff;
                for (int c = lane; c < chunks; c += 64)
                    if (l.tops[c] == top) first = min(first, parts[c].first);
                first = wave_min(first);
                if (lane == 0) a.tokens[r] = top == -kInf ? -1 : first;
            }
            return;
        }
        peak = pos_of(top, top, s.scale), edge = floor(peak);
        if (tid < chunks) {
            const double below = own.top == top ? 0.0 : !weighs(own.top, top) ? kBins : fmin(edge - floor(own.top * s.scale), (double)kBins);
            l.shift[tid] = (int)below;
            l.scale[tid] = below < kBins ? eighth((int)below) : 0.0;
            l.kept[tid] = own.mass * l.scale[tid];
            l.part[tid] = 0;
        }
        __syncthreads();
    }

    auto value_of_number = [](u64 number) {
        const uint32_t key = (uint32_t)(number >> 20);
        return value_of(sizeof(T) == 4 ? key : key << 16 | (key >> 15 ? 0u : 0xffffu));
    };
    // the lowest number of a logit from `key` on (16 bits of a key stand for the first of 65536 above zero, below for the last)
    auto number_from = [&](uint32_t key) { return number_of<T>(sizeof(T) == 2 && key >> 31 ? key + 0xffffu : key, 0xfffff); };
    auto first_of = [&](int b) { return lowest(s, top, edge - b); };                       // of bin b's logits

    // The least number that is kept, and its bin: the filters' borders are such numbers, and the highest of them counts
    u64 cut = number_of<T>(top == kInf ? 0xff800000u : 0x00800000u, 0xfffff);
    if constexpr (F) if (filters) {
        auto mass_to = [&](int b) { return b > 0 ? l.masses[b - 1] : 0.0; };  // of the bins in front of b
        auto count_in = [&](int b) { return l.counts[b] - (b > 0 ? l.counts[b - 1] : 0); };
        const int bin_m = known_to.m, bin_k = known_to.k;
        int bin_p = kBins;
        if (s.min_p > 0.0f) cut = max(cut, number_from(lowest(s, top, known_to.limit_m)));
        double all = l.masses[min(bin_k, kBins - 1)], limit_p = 0.0;

        // The border of the first k in its bin, that of the mass in its, and what is kept of the last bin, each where it is needed.
        // A pass reads the tokens of a bin, from the list or, where that is not whole, from the row: into 256 classes by eight bits of
        // their numbers, the few left ones into a list of their own, or what is kept of them into the chunks' masses.
        enum { kNew = 8, kCount = 0, kMass, kRest };
        enum { kToDigits, kToFew, kToParts };
        int count = 0, n = 0;          // tokens between lo and hi, and above hi
        u64 lo = 0, hi = 0, mass = 0;  // and the mass above hi
        bool whole = false;            // whether all of the last bin is kept
        bool by_mass = false;          // whether a border is where a mass is reached, or a number of tokens
        double limit = 0.0;
        // How many tokens weigh as much as the largest logit (of the tokens of the first bin, if those are listed)
        auto count_largest = [&] {
            const uint32_t key = lowest(s, top, peak);
            const u64 least = number_from(key);
            const float least_logit = value_of(key);
            int c = 0;
            if (listed <= kList) {
#pragma unroll 1
                for (int i = tid; i < listed; i += NT) c += l.list[i] >= least;
            } else {
#pragma unroll 1
                for (int i0 = tid * N; i0 < V; i0 += NT * N) {
                    const u32x4 x = load16(row, i0, V);
#pragma unroll
                    for (int i = 0; i < N; ++i) c += bits_of<T>(x, i) >= least_logit;
                }
            }
            c = sum_to(c);
            if (lane == 63) l.wave_counts[wave] = c;
            __syncthreads();
            c = 0;
#pragma unroll
            for (int w = 0; w < NT / 64; ++w) c += l.wave_counts[w];
            return c;
        };
        auto look_at = [&](int b) {
            n = 0, mass = 0, count = count_in(b);
            lo = number_from(first_of(b)), hi = b > 0 ? number_from(first_of(b - 1)) - 1 : number_of<T>(~0u, 0);
        };
#pragma unroll 1
        for (int task = kNew + kCount;;) {
            if (task == kNew + kCount) {
                task = kNew + kMass;
                if (bin_k < kBins) {
                    if (!known_to.part_k) {
                        cut = max(cut, number_from(first_of(bin_k)));
                    } else if (s.p < 1.0f || bin_k <= bin_m) {
                        task = kCount;
                        look_at(bin_k);
                        limit = (double)(s.k - l.counts[bin_k] + count);
                    }
                }
            }
            if (task == kNew + kMass) {
                task = kNew + kRest;
                if (s.p < 1.0f) {
                    limit_p = s.share * all;
                    bin_p = min(bins_below(l.masses, limit_p, lane), bin_k);
                    if (bin_p < kBins && bin_p <= bin_m) {
                        task = kMass;
                        look_at(bin_p);
                        limit = (limit_p - mass_to(bin_p)) * (0x1p40 * eighth(-bin_p));
                        by_mass = true;
                        // Sums of different weights are never equal (the exponential of a difference of logits is no fraction), but where
                        // all that count weigh the same the border may fall exactly between two of them, which rounded masses do not
                        // tell: a number of tokens does, top_p times theirs (24 bits by 20, exact).
                        if (bin_p == 0 && count > 1 && all <= l.masses[0] * (1.0 + 0x1p-33)) {
                            const int same = count_largest();
                            if (same == count || (s.k > 0 && same >= s.k)) by_mass = false, limit = ceil((double)s.p * (s.k > 0 ? min(s.k, same) : same));
                        }
                    }
                }
            }
            if (task == kNew + kRest) {
                if (ONE) break;
                task = kRest;
                const int b = min(min(bin_k, bin_p), bin_m);
                if (b == kBins) break;
                look_at(b);
                if (cut <= lo) {
                    whole = true;
                    break;
                }
            }
            // one pass
            const int what = task == kRest ? kToParts : count > kFew ? kToDigits : kToFew;
            const int shift = max(64 - __clzll((long long)(lo ^ hi)) - 8, 0);
            const u64 from = what == kToParts ? max(lo, cut) : lo;
            if (tid < 256) l.digit_counts[tid] = 0, l.digit_masses[tid] = 0;
            if (tid == 0) l.listed = 0;
            __syncthreads();
            auto take = [&](u64 number) {
                if (number < from || number > hi) return;
                const double pos = pos_of(value_of_number(number), top, s.scale);
                const u64 weight = (u64)(in_bin(pos - floor(pos)) * 0x1p40 + 0.5);
                if (what == kToParts) {
                    atomicAdd(&l.part[(0xfffff - (int)(number & 0xfffff)) / kChunk], weight);
                } else if (what == kToDigits) {
                    const int d = (int)(number >> shift) & 255;
                    atomicAdd(&l.digit_counts[d], 1);
                    atomicAdd(&l.digit_masses[d], weight);
                } else {
                    const int slot = atomicAdd(&l.listed, 1);
                    if (slot < kFew) l.few[slot] = Token{number, weight};
                }
            };
            if (listed <= kList) {
#pragma unroll 1
                for (int i = tid; i < listed; i += NT) take(l.list[i]);
            } else {
#pragma unroll 1
                for (int i0 = tid * N; i0 < V; i0 += NT * N) {
                    const u32x4 x = load16(row, i0, V);
#pragma unroll 1
                    for (int i = 0; i < N; ++i) {
                        const float y = pick<T>(x, i);
                        if (y == y) take(number_of<T>(key_of(y), i0 + i));
                    }
                }
            }
            __syncthreads();
            if (what == kToParts) break;
            if (what == kToDigits) {
                if (wave == 0) {  // a lane takes four classes, the highest first
                    int dn[4], sn = 0;
                    u64 dm[4], sm = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) dn[i] = l.digit_counts[255 - 4 * lane - i], dm[i] = l.digit_masses[255 - 4 * lane - i], sn += dn[i], sm += dm[i];
                    int fn = sum_to(sn);
                    u64 fm = sum_to(sm);
                    auto reaches = [&](int number, u64 sum) { return (by_mass ? (double)sum : (double)number) >= limit; };
                    const u64 hits = __ballot(reaches(n + fn, mass + fm));
                    if (lane == (hits ? __ffsll(hits) - 1 : 63)) {  // (rounding may leave the limit behind all of them)
                        fn = n + fn - sn, fm = mass + fm - sm;
                        bool done = false;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (done) continue;
                            done = i == 3 || reaches(fn + dn[i], fm + dm[i]);
                            if (done)
                                l.found = 255 - 4 * lane - i;
                            else
                                fn += dn[i], fm += dm[i];
                        }
                        l.found_n = fn, l.found_mass = fm;
                    }
                }
                __syncthreads();
                n = l.found_n, mass = l.found_mass, count = l.digit_counts[l.found];
                const u64 above = shift + 8 >= 64 ? 0 : hi >> (shift + 8) << (shift + 8), least = above | (u64)l.found << shift;
                lo = max(lo, least), hi = min(hi, least | ((1ull << shift) - 1));  // (the first and last class may begin and end outside)
                __syncthreads();
                if (count > 0) continue;  // (none: the limit is behind all, so all are kept)
            }
            // the few left: how many are in front of each, and their mass; the one with which the limit is reached
            if (tid == 0) l.cut = lo, l.found_mass = mass;
            __syncthreads();
            {
                constexpr int kLanes = NT / kFew;  // that share a token's comparisons
                const int own = min(tid / kLanes, max(count - 1, 0));
                const Token x = l.few[own];
                int fn = 0;
                u64 fm = 0;
#pragma unroll 4
                for (int i = tid % kLanes; i < count; i += kLanes) {
                    const Token y = l.few[i];
                    const bool front = y.number > x.number;
                    fn += front, fm += front ? y.weight : 0;
                }
#pragma unroll
                for (int d = 1; d < kLanes; d <<= 1) fn += __shfl_xor(fn, d), fm += (u64)__shfl_xor((long long)fm, d);
                fn += n, fm += mass;
                const bool reached = by_mass ? (double)fm < limit && (double)(fm + x.weight) >= limit : (double)(fn + 1) == limit;
                if (reached && tid / kLanes < count && tid % kLanes == 0) l.cut = x.number, l.found_mass = fm + x.weight;
            }
            __syncthreads();
            cut = max(cut, l.cut);
            if (task == kCount) all = mass_to(bin_k) + (double)l.found_mass * 0x1p-40 * eighth(bin_k);
            task = kNew + task + 1;
        }
        const int border = min(min(bin_k, bin_p), bin_m);
        if (!ONE && border < kBins && tid < chunks) {
            const int b = border - l.shift[tid] + whole;
            const double m = b > 0 && l.shift[tid] < kBins ? (double)mass_of(upto[tid * kBins + b - 1]) * (1.0 / kUptoUnit) * eighth(-bins_to_octave(edge - l.shift[tid])) : 0.0;
            l.kept[tid] = m * l.scale[tid] + (double)l.part[tid] * 0x1p-40 * eighth(border);
        }
        __syncthreads();
    }

    // The chunk that the draw falls into: sums over two chunks a lane
    static_assert(kChunksMost == 128, "two a lane");
    const float u = a.uniform[r];
    if (!ONE && wave == 0) {
        const double m0 = 2 * lane < chunks ? l.kept[2 * lane] : 0.0, m1 = 2 * lane + 1 < chunks ? l.kept[2 * lane + 1] : 0.0, sum = m0 + m1;
        const double front = sum_to(sum), total = lane_of(front, 63);
        const double aim = u > 0.0f ? fmin((double)u, 1.0 - 0x1p-40) * total : 0.0;
        const u64 hits = __ballot(front > aim && sum > 0.0), some = __ballot(sum > 0.0);
        if (lane == (hits ? __ffsll(hits) - 1 : 63 - __clzll((long long)some))) {  // (rounding may leave the draw behind the last)
            const double before = front - sum;
            const bool second = !(m0 > 0.0) || (m1 > 0.0 && before + m0 <= aim);
            l.chosen = 2 * lane + second;
            l.rest = aim - (second ? before + m0 : before);
            l.total = total;
            l.near = false;
        }
    }
    if (!ONE) __syncthreads();

    // The token in it, sixteen side by side to a thread: weights in whole 2^-50 of the top of the chunk's first bin, so that all sums
    // agree (what is kept of a chunk has its largest logit in it).  The chunks' masses are made of other roundings, so a draw that comes
    // near either end of its token, as one does that falls exactly between equal logits, is made again with one weight for
    // a token everywhere: kAdding takes the sums of the chunks that have tokens with weight, in 2^-43 of the top of the row's first bin, one chunk
    // after the other, kAgain the token.  Near: by what the roundings may add up to, 2^-51 for each of 8192 tokens here and as much once more where
    // their sums become binary64; with filters 2^-36 for each chunk (half a unit of an octave's end) and 2^-34 of the row's mass (the bins'
    // shortfalls), without 2^-43 of it (sums of the same weights in binary64).
    enum { kFirst, kAdding, kAgain };
    int state = ONE ? kAgain : kFirst, chosen = ONE ? 0 : l.chosen;
    u64 goal = 0;  // what of the draw is left in the chosen chunk, of kAgain
    auto is_kept = [&](float y, int i) { return F ? y == y && number_of<T>(key_of(y), i) >= cut : top != kInf || y == top; };
    // the first chunk from c on that has tokens with weight
    auto chunk_from = [&](int c) {
        while (c < chunks && (l.shift[c] == kBins || !is_kept(l.tops[c], c * kChunk))) ++c;
        return c;
    };
#pragma unroll 1
    for (;;) {
        const int first = chosen * kChunk + tid * kEach;
        if constexpr (!ONE) {
#pragma unroll
            for (int j = 0; j < kVectors; ++j) x[j] = load16(row, min(first + j * N, V), V);
        }
        const double chosen_edge = state == kFirst ? floor(pos_of(l.tops[chosen], top, s.scale)) : edge, from = (chosen_edge + 1.0) * -4.0;
        const double units = state == kFirst ? 0x1p50 : 0x1p43;
        // (2^52 more than the weight, which is then in the low bits; NaN and -infinity weigh nothing)
        auto weight = [&](float y) {
            const double w = power32(__builtin_fma(pos_of(y, top, s.scale), 4.0, from), l.powers);
            return __builtin_bit_cast(u64, __builtin_fma(w, units, 0x1p52)) - 0x4330000000000000ull;
        };
        u64 sum = 0;
#pragma unroll 1
        for (int j = 0; j < kVectors; ++j) {
            const u32x4 v = next_vector();
            uint32_t kept = 0;  // a bit each
#pragma unroll
            for (int i = 0; i < N; ++i) kept |= (uint32_t)is_kept(bits_of<T>(v, i), first + j * N + i) << i;
            if (F && !__any(kept)) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const u64 w = weight(bits_of<T>(v, i));
                sum += kept >> i & 1 ? w : 0;
            }
        }
        const u64 front = sum_to(sum);
        if (lane == 63) l.fronts[wave] = front;
        __syncthreads();
        u64 total = 0, before = front - sum;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) {
            const u64 f = l.fronts[w];
            if (w < wave) before += f;
            total += f;
        }
        if (!ONE && state == kAdding) {
            if (tid == 0) l.part[chosen] = total;
            chosen = chunk_from(chosen + 1);
            __syncthreads();
            if (chosen < chunks) continue;
            const u64 m0 = l.part[2 * lane], m1 = l.part[2 * lane + 1], end = sum_to(m0 + m1), aim = share_of(u, lane_of(end, 63));
            const int at = __ffsll(__ballot(end > aim)) - 1;
            const u64 start = lane_of(end - m0 - m1, at), middle = start + lane_of(m0, at);
            const bool second = middle <= aim;
            chosen = 2 * at + second, goal = aim - (second ? middle : start);
            state = kAgain;
            continue;
        }
        double rest = 0.0;
        u64 aim = goal;
        if constexpr (ONE) {
            aim = share_of(u, total);
        } else if (state == kFirst) {
            rest = l.rest / l.scale[chosen] * units;
            // (the weights here are those of the bins but where a pos of 2^53 and more leaves the one of its bin's top no bit)
            if (filters) rest *= eighth((int)(chosen_edge + 1.0 - chosen_edge) - 1);
            aim = min(rest > 0.0 ? (u64)fmin(rest, 0x1p63) : 0ull, total - 1);
        }
        const u64 owner = __ballot(sum > 0 && before <= aim && aim < before + sum);  // one thread of all
        if (owner) {
            // its logits again, a lane each
            const int own = __ffsll(owner) - 1, at = lane_of(first, own), i = at + lane;
            const u64 start = lane_of(before, own);
            static_assert(kEach <= 64, "a lane each");
            float y = -kInf;
            if (lane < kEach && i < V) y = sizeof(T) == 2 ? __uint_as_float((uint32_t)row[i] << 16) : (float)row[i];
            const u64 w = is_kept(y, i) ? weight(y) : 0, end = start + sum_to(w);
            const int token = __ffsll(__ballot(end > aim)) - 1;
            bool near = false;
            if (!ONE && state == kFirst && u > 0.0f) {
                // (nothing lies in front of a draw of 0)
                const double high = (double)lane_of(end, token), low = high - (double)lane_of(w, token);
                near = fmin(rest - low, high - rest) * l.scale[chosen] * 0x1p-7 < 0x1p6 + (filters ? chunks * 0x1p7 + l.total * 0x1p9 : l.total);
            }
            if (lane == 0) {
                if (near)
                    l.near = true;
                else
                    a.tokens[r] = at + token;
            }
        }
        if (ONE || state == kAgain) return;
        __syncthreads();
        if (!l.near) return;
        if (tid < kChunksMost) l.part[tid] = 0;
        __syncthreads();
        state = kAdding, chosen = chunk_from(0);
    }
}

// Rows of a launch: those of 64 MiB of workspace
constexpr int64_t kSampleSpace = (int64_t)64 << 20;
static int64_t chunks_of(int64_t V) { return (V + kChunk - 1) / kChunk; }
static int64_t row_bytes(int64_t chunks) { return chunks * kChunkBytes + sizeof(Row); }
static int64_t rows_of(int64_t rows, int64_t chunks) { return std::min(rows, std::max<int64_t>(kSampleSpace / row_bytes(chunks), 1)); }
// (a launch whose rows have no filters needs the Chunks alone: as many rows as the same space holds)
static int64_t plain_rows_of(int64_t rows, int64_t chunks) { return std::min(rows, rows_of(rows, chunks) * row_bytes(chunks) / (chunks * (int64_t)sizeof(Chunk))); }

int64_t sample_workspace(int64_t rows, int64_t V)
{
    const int64_t chunks = chunks_of(V);
    return chunks == 1 ? 0 : rows_of(rows, chunks) * row_bytes(chunks);
}

template <class T>
static int sample_typed(const Sample &a, hipStream_t s)
{
    const bool filters = a.top_k || a.top_p || a.min_p;
    const int64_t chunks = chunks_of(a.V);
    if (chunks == 1) {  // (no workspace)
        auto go = [&](auto kernel) { return enqueue(kernel, dim3((unsigned)a.rows), dim3(kRowThreads), 0, s, a, Tables{}, (int64_t)0, 1); };
        return filters ? go(sample_rows<T, true, true>) : go(sample_rows<T, false, true>);
    }
    const int64_t most = filters ? rows_of(a.rows, chunks) : plain_rows_of(a.rows, chunks);
    Chunk *const first = static_cast<Chunk *>(a.ws);
    Upto *const upto = reinterpret_cast<Upto *>(first + most * chunks);
    const Tables t{first, upto, reinterpret_cast<Row *>(upto + most * chunks * kBins)};
    for (int64_t r = 0; r < a.rows; r += most) {
        const int64_t n = std::min(most, a.rows - r);
        auto go = [&](auto kernel, int64_t groups, int threads, auto... more) {
            return enqueue(kernel, dim3((unsigned)groups), dim3(threads), 0, s, a, t, r, (int)chunks, more...);
        };
        if (int rc = go(sample_chunks<T>, n * chunks, kChunkThreads)) return rc;
        if (filters) {
            const int64_t parts = std::min(chunks, std::max<int64_t>(256 / n, 1));
            if (int rc = go(sample_border<T>, n * parts, kBorderThreads, (int)parts)) return rc;
        }
        if (int rc = filters ? go(sample_rows<T, true, false>, n, kRowThreads) : go(sample_rows<T, false, false>, n, kRowThreads)) return rc;
    }
    return MQ_OK;
}

int launch_sample(const Sample &a, bool fp32, hipStream_t s) { return fp32 ? sample_typed<float>(a, s) : sample_typed<uint16_t>(a, s); }

}  // namespace mq
