// BF16 activations of a few tokens times NVFP4 weights: y[m, n] = alpha * sum_k x[m, k] * sigma[n, k/16] * q[n, k].
//
// Bound by reading the weights, 9/16 byte each.  sigma * q has at most six significant bits, so it is a BF16 number exactly
// and the products are exact on the BF16 matrix pipe with x as it is: no conversion of x, whose range FP16 would not hold.
// Two codes become two FP32 numbers in one conversion, two multiplications by sigma and one byte permute that takes the upper
// halves (exact: the lower ones are zero): two instructions a weight, of the 3.7 that a compute unit has time for while its
// share of the memory stream brings one.
//
// A wave owns S strips of 16 rows of W and a range of K, and all tokens: of each 128 elements of K a lane (row = lane % 16,
// g = lane / 16) loads the 16 bytes of codes at element 32 g, which are its own slots of four matrix instructions.  The waves
// of a workgroup share the strips and split K; their sums are added in LDS in the order of the waves.
#include "kv8.h"

namespace mq {

struct MatvecArgs {
    const uint16_t *x;
    int64_t ldx;
    const uint8_t *codes, *scales;
    const float *alpha;
    int64_t c_row, c_step, s_row, s_step;  // bytes from row to row, and from one 64 elements of K to the next
    int64_t M, N, K;
    void *y;
    int64_t ldy;
    int out;
};

static __device__ __forceinline__ float e4m3_value(uint32_t byte) { return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0); }

// eight codes times sigma, as BF16
static __device__ __forceinline__ bf16x8 expand_codes(uint32_t w, float sigma)
{
    auto two = [&](f32x2 v) {
        const uint32_t lo = __float_as_uint(v[0] * sigma), hi = __float_as_uint(v[1] * sigma);
        return __builtin_amdgcn_perm(hi, lo, 0x07060302);
    };
    return __builtin_bit_cast(bf16x8, u32x4{two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0)), two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1)),
                                            two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2)), two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3))});
}

static __device__ __forceinline__ void store_one(const MatvecArgs &a, int64_t m, int64_t n, float v)
{
    if (a.out == MQ_OUT_BF16)
        reinterpret_cast<uint16_t *>(a.y)[m * a.ldy + n] = __builtin_bit_cast(uint16_t, (__bf16)v);
    else
        reinterpret_cast<float *>(a.y)[m * a.ldy + n] = v;
}

// MT tiles of 16 tokens, S strips of 16 rows, NW waves along K, U iterations of 128 elements loaded together
template <int MT, int S, int NW, int U>
__global__ __launch_bounds__(64 * NW) void matvec_kernel(MatvecArgs a)
{
    __shared__ f32x4 part[NW][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
    const int64_t row0 = (int64_t)blockIdx.x * 16 * S, m0 = (int64_t)blockIdx.y * 16 * MT;
    const int steps = (int)(a.K / 64), iters = (steps + 1) / 2;
    const int begin = (int)((int64_t)iters * wave / NW), end = (int)((int64_t)iters * (wave + 1) / NW);

    const uint8_t *code[S], *scale[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t r = min(row0 + 16 * s + col, a.N - 1);  // rows beyond the last are computed again and not stored
        code[s] = a.codes + r * a.c_row + 16 * (g & 1);
        scale[s] = a.scales + r * a.s_row + 2 * (g & 1);
    }
    const uint16_t *x[MT];
    bool live[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t m = m0 + 16 * t + col;
        live[t] = m < a.M;
        x[t] = a.x + (live[t] ? m : 0) * a.ldx + 32 * g;
    }
    f32x4 acc[S][MT];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[s][t] = f32x4{0, 0, 0, 0};

    for (int i0 = begin; i0 < end; i0 += U) {
        u32x4 c[U][S], xv[U][MT][4];
        uint32_t sc[U][S];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int step = min(2 * (i0 + u) + (g >> 1), steps - 1);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                c[u][s] = *reinterpret_cast<const u32x4 *>(code[s] + step * a.c_step);
                sc[u][s] = *reinterpret_cast<const uint16_t *>(scale[s] + step * a.s_step);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // beyond the wave's range, or K's end in the second half of the last iteration: zeros for x
            const bool in = i0 + u < end && 2 * (i0 + u) + (g >> 1) < steps;
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    xv[u][t][j] = u32x4{0, 0, 0, 0};
                    if (live[t] && in) xv[u][t][j] = *reinterpret_cast<const u32x4 *>(x[t] + (int64_t)(i0 + u) * 128 + 8 * j);
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const float sigma[2] = {e4m3_value(sc[u][s] & 0xff), e4m3_value(sc[u][s] >> 8)};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x8 w = expand_codes(c[u][s][j], sigma[j / 2]);
#pragma unroll
                    for (int t = 0; t < MT; ++t)
                        acc[s][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, xv[u][t][j]), acc[s][t], 0, 0, 0);
                }
            }
    }

    const float alpha = *a.alpha;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            part[wave][lane] = acc[s][t];
            __syncthreads();
            if (wave == (s * MT + t) % NW) {
                f32x4 sum = part[0][lane];
#pragma unroll
                for (int w = 1; w < NW; ++w) sum += part[w][lane];
                const int64_t m = m0 + 16 * t + col, n = row0 + 16 * s + 4 * g;
                if (m < a.M)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (n + i < a.N) store_one(a, m, n + i, sum[i] * alpha);
            }
            __syncthreads();
        }
}

// K that is no multiple of 64: one wave a row of W and token, a block of 16 elements per lane and step
__global__ __launch_bounds__(64) void matvec_simple_kernel(MatvecArgs a)
{
    const int lane = threadIdx.x;
    const int64_t n = blockIdx.x;
    const uint16_t *const x = a.x + (int64_t)blockIdx.y * a.ldx;
    float sum = 0.0f;
    for (int64_t b = lane; b < a.K / 16; b += 64) {
        const float sigma = e4m3_value(a.scales[n * a.s_row + b]);
        const uint8_t *const c = a.codes + n * a.c_row + 8 * b;
        float dot = 0.0f;
        for (int i = 0; i < 8; ++i) {
            const f32x2 q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)c[i], 1.0f, 0);
            dot += q[0] * __uint_as_float((uint32_t)x[16 * b + 2 * i] << 16);
            dot += q[1] * __uint_as_float((uint32_t)x[16 * b + 2 * i + 1] << 16);
        }
        sum += sigma * dot;
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) store_one(a, blockIdx.y, n, sum * *a.alpha);
}

template <int MT, int S, int NW, int U>
static int launch(const MatvecArgs &a, hipStream_t s)
{
    const int64_t strips = (a.N + 16 * S - 1) / (16 * S), tokens = (a.M + 16 * MT - 1) / (16 * MT);
    return enqueue(matvec_kernel<MT, S, NW, U>, dim3((unsigned)strips, (unsigned)tokens), dim3(64 * NW), 0, s, a);
}

int launch_nvfp4_matvec(const uint16_t *x, int64_t ldx, const uint8_t *codes, const uint8_t *scales, const float *alpha, int64_t M,
                        int64_t N, int64_t K, void *y, int64_t ldy, int out, int layout, hipStream_t s)
{
    MatvecArgs a{x, ldx, codes, scales, alpha, K / 2, 32, K / 16, 4, M, N, K, y, ldy, out};
    if (layout == MQ_LAYOUT_KTILE) a.c_row = 32, a.c_step = 32 * N, a.s_row = 4, a.s_step = 4 * N;
    if (K % 64) return enqueue(matvec_simple_kernel, dim3((unsigned)N, (unsigned)M), dim3(64), 0, s, a);
    if (M <= 16) return launch<1, 1, 8, 2>(a, s);
    if (M <= 32) return launch<2, 2, 8, 1>(a, s);
    if (M <= 48) return launch<3, 2, 8, 1>(a, s);
    return launch<4, 2, 8, 1>(a, s);
}

}  // namespace mq
