// What the kernels of the 8-bit paged cache share: its layout, the sequences of a call, and the codes' arithmetic.
#pragma once
#include "mq_common.h"

namespace mq {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Page scales are 2^e, e within these bounds: a code's value code * 2^e is then a normal BF16 number (2^-9 * 2^-112 at
// least, 448 * 2^119 at most), which is what the attention expands it to.
constexpr int kExpLowest = -112, kExpHighest = 119;

// The sequences of a call: new tokens cu_q[b] .. cu_q[b + 1] of T, the last ones of the kv_lens[b] tokens in the pages
// page_table[b * pt_ld + i], i < width.
struct Kv8Seqs {
    const int32_t *page_table, *cu_q, *kv_lens;
    int64_t pt_ld, pages;
    int width, B, T, page_shift;
};

struct Kv8Append {
    const uint16_t *q, *k, *v;
    int64_t ldq, ldk, ldv;  // token strides in elements
    uint16_t *q_out;        // [T, Hq, D], dense
    uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    const float *table;        // [max_pos, rot], cosines then sines, or NULL
    const int32_t *positions;  // [T], or NULL: the token's place in its sequence
    int64_t max_pos;
    int rot, interleaved, Hq, Hkv, D;
    Kv8Seqs s;
};

struct Kv8Attend {
    const uint16_t *q;
    int64_t ldq;
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    uint16_t *y;
    int64_t ldy;
    int Hq, Hkv, D, window;
    float scale;  // of the scores, times log2(e)
    float *ws;
    int64_t ws_bytes;
    Kv8Seqs s;
};

struct RopeTable {
    double freq[128];
    float *table;
    int64_t max_pos;
    int rot;
    float gain;
};

int launch_rope_table(const RopeTable &r, hipStream_t s);
int launch_kv8_append(const Kv8Append &a, hipStream_t s);
int launch_kv8_attention(const Kv8Attend &a, hipStream_t s);
int describe_kv8_attention(const Kv8Attend &a, mq_kv8_launch *out);  // what the above launches (mixquant_diag.h)
int64_t kv8_attention_workspace(int64_t T, int64_t B, int Hq, int Hkv, int D);
int launch_nvfp4_matvec(const uint16_t *x, int64_t ldx, const uint8_t *codes, const uint8_t *scales, const float *alpha, int64_t M,
                        int64_t N, int64_t K, void *y, int64_t ldy, int out, int layout, void *ws, hipStream_t s);
int describe_nvfp4_matvec(int64_t M, int64_t N, int64_t K, mq_launch *out);
int64_t matvec_workspace(int64_t M, int64_t N, int64_t K);
int configure_matvec_kernels();

#if defined(__HIPCC__)
// One sequence as the kernels see it: its new tokens q0 .. q0 + n, the place `start` of the first of them (negative where the
// stated length is shorter than that), and how many of its places the page table covers.
struct Span {
    int q0, n, start, len;
};

static __device__ __forceinline__ Span span_of(const Kv8Seqs &s, int b)
{
    Span r;
    int q1 = s.cu_q[b + 1];
    r.q0 = s.cu_q[b];
    const int len = s.kv_lens[b];
    q1 = min(q1, s.T);
    r.n = r.q0 >= 0 && q1 > r.q0 ? q1 - r.q0 : 0;
    r.start = max(len, 0) - r.n;
    r.len = min(max(len, 0), s.width << s.page_shift);
    return r;
}

static __device__ __forceinline__ int wave_scan(int v, int lane)  // inclusive sum over the wave
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(v, d);
        if (lane >= d) v += u;
    }
    return v;
}

static __device__ __forceinline__ float exp2_of(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// nearest E4M3 codes of four values, ties to even, clipped to +-448 (the conversion itself turns larger values into NaN)
static __device__ __forceinline__ uint32_t e4m3_of(float a, float b, float c, float d)
{
    auto clip = [](float x) {  // keeps a NaN
        x = x > 448.0f ? 448.0f : x;
        return x < -448.0f ? -448.0f : x;
    };
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(clip(a), clip(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clip(c), clip(d), r, true);
}
#endif

}  // namespace mq
