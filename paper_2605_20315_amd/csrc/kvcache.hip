// Position rotation of queries and keys, and keys and values into the paged FP8 cache.
//
// The cache of one layer is k_codes, v_codes [pages, Hkv, P, D] (E4M3) and k_scales, v_scales [pages, Hkv] (the exponent byte
// e + 127 of a power of two): a page's scale is 2^e with the smallest e that brings the page's largest finite magnitude to 448
// or below.  A power of two because the page's scale has to grow when a later token is larger than all before it: the codes
// already there then move by whole binades, which is exact but where they become subnormal, instead of being rounded again; and
// because reading multiplies by it for nothing, in the conversion to BF16 itself.  It costs at most one binade of range at the
// lower end (E4M3 holds 18 binades), no precision.
#include "kv8.h"

namespace mq {

__global__ __launch_bounds__(256) void rope_table_kernel(RopeTable r)
{
    const int half = r.rot / 2;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= r.max_pos * half) return;
    const int64_t pos = i / half;
    const int f = (int)(i - pos * half);
    // the angle in 64 bits: at position 131071 a 32-bit angle is off by up to 2^-8 radians
    double s, c;
    sincos((double)pos * r.freq[f], &s, &c);
    r.table[pos * r.rot + f] = (float)c * r.gain;
    r.table[pos * r.rot + half + f] = (float)s * r.gain;
}

int launch_rope_table(const RopeTable &r, hipStream_t s)
{
    const int64_t n = r.max_pos * (r.rot / 2);
    if (n == 0) return MQ_OK;
    return enqueue(rope_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, r);
}

// cosines and sines for the eight elements 8 * sub .. of a head (four pairs of them where interleaved)
struct Turn {
    float c[8], s[8];
    int kind;  // 0: not rotated, 1: first half, 2: second half, 3: interleaved
};

static __device__ __forceinline__ Turn turn_of(const Kv8Append &a, int pos, int sub)
{
    Turn t;
    const int e = 8 * sub, half = a.rot / 2;
    t.kind = e >= a.rot ? 0 : a.interleaved ? 3 : e < half ? 1 : 2;
    if (t.kind == 0) return t;
    const bool known = (unsigned)pos < (uint64_t)a.max_pos;
    const float *row = a.table + (int64_t)(known ? pos : 0) * a.rot + (t.kind == 3 ? e / 2 : t.kind == 1 ? e : e - half);
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
        if (i == 4 && t.kind == 3) break;
        const f32x4 c = *reinterpret_cast<const f32x4 *>(row + i), s = *reinterpret_cast<const f32x4 *>(row + half + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) t.c[i + j] = known ? c[j] : __builtin_nanf(""), t.s[i + j] = known ? s[j] : __builtin_nanf("");
    }
    return t;
}

static __device__ __forceinline__ float lo_of(uint32_t w) { return __uint_as_float(w << 16); }
static __device__ __forceinline__ float hi_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
static __device__ __forceinline__ uint32_t pack(float lo, float hi)  // both rounded to BF16, nearest even
{
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

// The rotation of eight BF16 elements; in the half layout the other element of each pair is `sub` +- rot / 16 lanes away.
// Products and sums are separate binary32 steps, so that the plain evaluation gives the same bits.
static __device__ __forceinline__ u32x4 rotate(const Kv8Append &a, u32x4 x, const Turn &t, int lane)
{
    if (a.rot == 0) return x;
    u32x4 r = x;
    if (a.interleaved) {
        if (t.kind == 3)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = lo_of(x[i]), q = hi_of(x[i]);
                r[i] = pack(p * t.c[i] - q * t.s[i], q * t.c[i] + p * t.s[i]);
            }
        return r;
    }
    const int other = t.kind == 1 ? lane + a.rot / 16 : t.kind == 2 ? lane - a.rot / 16 : lane;
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (uint32_t)__shfl((int)x[i], other);
    if (t.kind) {
        // first half: a c - b s; second: b c + a s
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float l = lo_of(x[i]) * t.c[2 * i], h = hi_of(x[i]) * t.c[2 * i + 1];
            const float ol = lo_of(o[i]) * t.s[2 * i], oh = hi_of(o[i]) * t.s[2 * i + 1];
            r[i] = t.kind == 1 ? pack(l - ol, h - oh) : pack(l + ol, h + oh);
        }
    }
    return r;
}

// largest finite |x| of eight BF16 elements, as bits
static __device__ __forceinline__ uint32_t amax_of(u32x4 x, uint32_t m)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t l = x[i] & 0x7fffu, h = (x[i] >> 16) & 0x7fffu;
        m = max(m, l < 0x7f80u ? l : 0u);
        m = max(m, h < 0x7f80u ? h : 0u);
    }
    return m;
}

// smallest e with amax <= 448 * 2^e = 1.75 * 2^(8 + e), for the bits of a BF16 number
static __device__ __forceinline__ int exponent_of(uint32_t amax)
{
    const int e = (int)(amax >> 7) - 127 - ((amax & 0x7fu) <= 96u ? 8 : 7);
    return amax == 0 ? kExpLowest : min(max(e, kExpLowest), kExpHighest);
}

static __device__ __forceinline__ u32x2 quantize8(u32x4 x, float inv)
{
    return u32x2{e4m3_of(lo_of(x[0]) * inv, hi_of(x[0]) * inv, lo_of(x[1]) * inv, hi_of(x[1]) * inv),
                 e4m3_of(lo_of(x[2]) * inv, hi_of(x[2]) * inv, lo_of(x[3]) * inv, hi_of(x[3]) * inv)};
}

// the sequence and page of the idx-th of all (sequence, page that its new tokens touch)
struct Run {
    bool found;
    int b, page, q0, start, end;  // `page` in the sequence; places start .. end are new
};

static __device__ Run run_of(const Kv8Seqs &s, int idx, int lane)
{
    Run r{};
    const int most = s.width << s.page_shift;
    int before = 0;
    for (int base = 0; base < s.B; base += 64) {
        const int b = base + lane;
        int count = 0, lo = 0, hi = 0;
        Span sp{};
        if (b < s.B) {
            sp = span_of(s, b);
            lo = max(sp.start, 0);
            hi = min(sp.start + sp.n, most);
            count = hi > lo ? ((hi - 1) >> s.page_shift) - (lo >> s.page_shift) + 1 : 0;
        }
        const int sum = wave_scan(count, lane);
        const int total = __shfl(sum, 63);
        if (idx < before + total) {
            const int at = __ffsll((unsigned long long)__ballot(before + sum > idx)) - 1;
            r.found = true;
            r.b = __builtin_amdgcn_readlane(b, at);
            r.q0 = __builtin_amdgcn_readlane(sp.q0, at);
            r.start = __builtin_amdgcn_readlane(sp.start, at);
            r.end = __builtin_amdgcn_readlane(hi, at);
            r.page = (max(r.start, 0) >> s.page_shift) + idx - before - __builtin_amdgcn_readlane(sum - count, at);
            return r;
        }
        before += total;
    }
    return r;
}

// One (page, head) of keys or values by NW waves, in one pass over the new tokens where registers hold them (kKeep loads a
// thread), in two otherwise: their largest magnitude, the scale, their codes, and the codes of
// the tokens that were there before where the scale has grown.
template <int D, int NW>
static __device__ void store_unit(const Kv8Append &a, const Run &r, bool key, int head, int tid, uint32_t *part)
{
    constexpr int kSubs = D / 8, kRows = 64 * NW / kSubs, kKeep = 8;
    const int lane = tid & 63, sub = tid % kSubs, row = tid / kSubs, P = 1 << a.s.page_shift;
    if ((unsigned)r.page >= (unsigned)a.s.width) return;
    const int id = a.s.page_table[r.b * a.s.pt_ld + r.page];
    if ((unsigned)id >= (uint64_t)a.s.pages) return;  // (the same for every wave of the unit)
    const int first = r.page << a.s.page_shift, s0 = max(r.start - first, 0), s1 = min(r.end - first, P);
    const int64_t unit = (int64_t)id * a.Hkv + head;
    uint8_t *const codes = (key ? a.k_codes : a.v_codes) + unit * P * D + 8 * sub;
    uint8_t *const scale = (key ? a.k_scales : a.v_scales) + unit;
    const int old = s0 > 0 ? min(max((int)*scale - 127, kExpLowest), kExpHighest) : kExpLowest;
    const uint16_t *const src = (key ? a.k + (int64_t)head * D : a.v + (int64_t)head * D) + 8 * sub;
    const int64_t ld = key ? a.ldk : a.ldv;
    const int steps = (s1 - s0 + kRows - 1) / kRows;

    auto load = [&](int step, u32x4 &x) {  // (every lane takes part: the rotation passes values between lanes)
        const int place = s0 + step * kRows + row;
        const bool live = place < s1;
        const int64_t t = r.q0 + (first + (live ? place : s0) - r.start);
        x = *reinterpret_cast<const u32x4 *>(src + t * ld);
        if (key && a.rot) x = rotate(a, x, turn_of(a, a.positions ? a.positions[t] : first + (live ? place : s0), sub), lane);
    };
    u32x4 kept[kKeep];
    uint32_t m = 0;
    const bool keep = steps <= kKeep;
    if (keep) {
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
            if (i < steps) load(i, kept[i]), m = amax_of(kept[i], m);
    } else {
        for (int i = 0; i < steps; ++i) load(i, kept[0]), m = amax_of(kept[0], m);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    if constexpr (NW > 1) {
        if (lane == 0) part[tid >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) m = max(m, part[w]);
    }
    const int e = max(exponent_of(m), old);
    const float inv = exp2_of(-e);
    auto write = [&](int step, u32x4 x) {
        const int place = s0 + step * kRows + row;
        if (place < s1) *reinterpret_cast<u32x2 *>(codes + (int64_t)place * D) = quantize8(x, inv);
    };
    if (keep) {
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
            if (i < steps) write(i, kept[i]);
    } else {
        for (int i = 0; i < steps; ++i) load(i, kept[0]), write(i, kept[0]);
    }
    if (s0 > 0 && e > old) {
        const float shrink = exp2_of(max(old - e, -126));  // (from 2^-19 on every code becomes zero)
        for (int place = row; place < s0; place += kRows) {
            u32x2 *const p = reinterpret_cast<u32x2 *>(codes + (int64_t)place * D);
            u32x2 c = *p;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const f32x2 l = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), h = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
                c[i] = e4m3_of(l[0] * shrink, l[1] * shrink, h[0] * shrink, h[1] * shrink);
            }
            *p = c;
        }
    }
    // behind the reads of the other waves
    if constexpr (NW > 1) __syncthreads();
    if (tid == 0) *scale = (uint8_t)(e + 127);
}

// rotated queries of one token: the heads h0 .. h0 + kHeads
template <int D>
static __device__ void rotate_queries(const Kv8Append &a, int t, int h0, int lane)
{
    constexpr int kSubs = D / 8, kPer = 64 / kSubs, kSteps = 4;
    const int sub = lane % kSubs, row = lane / kSubs;
    u32x4 x[kSteps];
    const uint16_t *const src = a.q + (int64_t)t * a.ldq + 8 * sub;
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
        x[i] = *reinterpret_cast<const u32x4 *>(src + (int64_t)min(h0 + i * kPer + row, a.Hq - 1) * D);
    Turn turn;
    turn.kind = 0;
    if (a.rot) {
        int pos;
        if (a.positions) {
            pos = a.positions[t];
        } else {
            int b = 0;  // sequences that end at or before t
            for (int base = 0; base < a.s.B; base += 64) {
                const int i = base + lane;
                const unsigned long long done = __ballot(i < a.s.B && a.s.cu_q[min(i, a.s.B - 1) + 1] <= t);
                b += __popcll(done);
                if (done != ~0ull) break;
            }
            if (b >= a.s.B) return;  // a row that belongs to no sequence
            const Span sp = span_of(a.s, b);
            pos = sp.start + (t - sp.q0);
        }
        turn = turn_of(a, pos, sub);
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int h = h0 + i * kPer + row;
        const u32x4 r = rotate(a, x[i], turn, lane);
        if (h < a.Hq) *reinterpret_cast<u32x4 *>(a.q_out + ((int64_t)t * a.Hq + h) * D + 8 * sub) = r;
    }
}

// One launch for keys, values and queries.  Bound by HBM for prompts (8111 tokens of 32 query and 8 key heads of 128: 187 MB in
// 45.5 us = 4.1 TB/s, a large copy reaches 4.8), by three dependent trips to memory (lengths, page number, codes' scale) for
// single tokens: 200 of them 7.1 us.
// Workgroups below `stores` take (page, head) units of keys and values, the others four waves of queries each.
template <int D, int NW>
__global__ __launch_bounds__(256) void kv8_append_kernel(Kv8Append a, int stores, int units)
{
    __shared__ uint32_t part[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if ((int)blockIdx.x < stores) {
        const int unit = NW == 1 ? (int)blockIdx.x * 4 + wave : (int)blockIdx.x;
        if (unit >= units) return;
        const int heads = 2 * a.Hkv, run = unit / heads, h = unit - run * heads;
        const Run r = run_of(a.s, run, lane);
        if (!r.found) return;
        store_unit<D, NW>(a, r, h < a.Hkv, h < a.Hkv ? h : h - a.Hkv, NW == 1 ? lane : tid, part);
        return;
    }
    constexpr int kHeads = 4 * 512 / D;
    const int per = (a.Hq + kHeads - 1) / kHeads;
    const int64_t unit = (int64_t)(blockIdx.x - stores) * 4 + wave;
    const int64_t t = unit / per;
    if (t < a.s.T) rotate_queries<D>(a, (int)t, (int)(unit - t * per) * kHeads, lane);
}

int launch_kv8_append(const Kv8Append &a, hipStream_t s)
{
    if (a.s.T == 0 || a.s.B == 0) return MQ_OK;
    // pages touched: at most one for each new token, and n / P + 2 for a sequence of n
    const int64_t T = a.s.T, runs = std::min<int64_t>(T, (T >> a.s.page_shift) + 2 * (int64_t)a.s.B);
    const int64_t units = runs * 2 * a.Hkv;
    // One wave a unit for a few tokens a sequence, and for pages of which it can keep all in registers (8 loads of 512 elements:
    // a mixed batch with pages of 16 x 64 takes 14.5 us so, 22.5 with four waves); else four waves share a unit (pages of
    // 64 x 128, 8111 tokens: 45.5 us, 58.9 with one wave, which would read them twice).
    const bool few = T <= 4 * (int64_t)a.s.B || (a.D << a.s.page_shift) <= 4096;
    const int64_t stores = few ? (units + 3) / 4 : units;
    const int heads = 4 * 512 / a.D;
    const int64_t queries = (T * ((a.Hq + heads - 1) / heads) + 3) / 4;
    if (stores + queries > 0x7fffffff || units > 0x7fffffff) return MQ_ERR_SHAPE;
    auto go = [&](auto kernel) { return enqueue(kernel, dim3((unsigned)(stores + queries)), dim3(256), 0, s, a, (int)stores, (int)units); };
    if (a.D == 64) return few ? go(kv8_append_kernel<64, 1>) : go(kv8_append_kernel<64, 4>);
    if (a.D == 128) return few ? go(kv8_append_kernel<128, 1>) : go(kv8_append_kernel<128, 4>);
    return few ? go(kv8_append_kernel<256, 1>) : go(kv8_append_kernel<256, 4>);
}

}  // namespace mq
