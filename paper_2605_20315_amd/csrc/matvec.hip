// BF16 activations of a few tokens times NVFP4 weights: y[m, n] = alpha * sum_k x[m, k] * sigma[n, k/16] * q[n, k].
//
// Bound by reading the weights, 9/16 byte each, if little enough is done per weight: a compute unit has time for 3.7 vector
// instructions while its share of the memory stream brings one.  sigma * q is an FP16 number exactly (six significant bits,
// 2^-10 .. 2688), and two codes become two of them in one conversion and one packed multiply: one instruction a weight.
// (As BF16, which takes x as it is, there is no packed multiply: 2.6 a weight, and 95 us instead of 38 for 64 tokens
// [4096 -> 28672].)  So x becomes FP16 as well, each token times the power of two that brings its largest magnitude
// to 2^14 .. 2^15: exact for every element down to 2^-29 of that one, below that off by at most 2^-38 of it.  Sums are FP32.
//
// The activations are laid out once in the order in which the matrix instructions take them, so that an operand is 1 KB of
// contiguous memory or LDS: up to kLdsTokens tokens by every workgroup in its LDS (in_lds), more of them by a kernel in front
// into the workspace.  (Read in rows, 40 tokens of 25600 took 36 us of 68 for themselves.)
//
// A wave owns S strips of 16 rows of W and a range of K, and up to 16 MT tokens: of each 128 elements of K (an iteration) a
// lane (row = lane % 16, g = lane / 16) loads the 16 bytes of codes at element 32 g, its slots of four 16x16x32 products.
// The waves of a workgroup share the strips and split K; their sums are added in LDS in the order of the waves.
#include <algorithm>

#include "kv8.h"

namespace mq {

constexpr int kLdsTokens = 4;
constexpr int64_t kLdsBytes = 64 << 10;

struct MatvecArgs {
    const uint16_t *x;
    int64_t ldx;
    const uint8_t *codes, *scales;
    const float *alpha;
    int64_t c_row, c_step, s_row, s_step;  // bytes from row to row, and from one 64 elements of K to the next
    int64_t M, N, K;
    void *y;
    int64_t ldy;
    int out, tiles;       // tiles: of 16 tokens, in `packed`
    const u32x4 *packed;  // [iteration][tile][4][64 lanes], eight FP16 elements each
    const int *exps;      // [M]: x * 2^exps is what is packed
    float *sums;          // [slabs][M][N], where K is cut into slabs across workgroups
    int slabs;
};

static __device__ __forceinline__ uint32_t bf16_amax(u32x4 v, uint32_t m)  // largest finite magnitude, as bits
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t l = v[i] & 0x7fffu, h = (v[i] >> 16) & 0x7fffu;
        m = max(m, max(l < 0x7f80u ? l : 0u, h < 0x7f80u ? h : 0u));
    }
    return m;
}

static __device__ __forceinline__ int shift_of(uint32_t amax) { return amax == 0 ? 0 : 14 + 127 - (int)max(amax >> 7, 1u); }

static __device__ __forceinline__ u32x4 to_f16(u32x4 v, int e)  // eight BF16 elements times 2^e
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(ldexpf(__uint_as_float(v[i] << 16), e), ldexpf(__uint_as_float(v[i] & 0xffff0000u), e)));
    return r;
}

// One workgroup a token: its largest magnitude, then its elements in their places
__global__ __launch_bounds__(1024) void matvec_pack_kernel(MatvecArgs a)
{
    __shared__ uint32_t part[16];
    const int64_t m = blockIdx.x;
    const int tid = threadIdx.x, pieces = (int)(a.K / 8), all = (pieces + 15) / 16 * 16;
    const u32x4 *const x = reinterpret_cast<const u32x4 *>(a.x + m * a.ldx);
    constexpr int kKeep = 4;  // pieces that a thread keeps from the first pass
    u32x4 kept[kKeep];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < kKeep; ++k) kept[k] = tid + 1024 * k < pieces ? x[tid + 1024 * k] : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < kKeep; ++k) top = bf16_amax(kept[k], top);
    for (int i = tid + 1024 * kKeep; i < pieces; i += 1024) top = bf16_amax(x[i], top);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if ((tid & 63) == 0) part[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) top = max(top, part[w]);
    const int e = shift_of(top);
    if (tid == 0) const_cast<int *>(a.exps)[m] = e;
    // piece i: iteration i / 16, lane group i / 4 % 4, operand i % 4; zeros where K ends in the middle of an iteration
    auto put = [&](int i, u32x4 v) {
        if (i < all) const_cast<u32x4 *>(a.packed)[((int64_t)(i / 16 * a.tiles + m / 16) * 4 + i % 4) * 64 + i / 4 % 4 * 16 + m % 16] = to_f16(v, e);
    };
#pragma unroll
    for (int k = 0; k < kKeep; ++k) put(tid + 1024 * k, kept[k]);
    for (int i = tid + 1024 * kKeep; i < all; i += 1024) put(i, i < pieces ? x[i] : u32x4{0, 0, 0, 0});
}

static __device__ __forceinline__ void swap32(uint32_t &a, uint32_t &b)  // the upper half of a with the lower half of b
{
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(a, b, false, false));
    a = r[0], b = r[1];
}
static __device__ __forceinline__ void swap16(uint32_t &a, uint32_t &b)  // the odd 16 lanes of a with the even 16 lanes of b
{
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a, b, false, false));
    a = r[0], b = r[1];
}
// v of the four lanes of a row, in all of them
static __device__ __forceinline__ void gather4(uint32_t v, uint32_t (&out)[4])
{
    out[0] = out[2] = v;
    swap32(out[0], out[2]);
    out[1] = out[0], out[3] = out[2];
    swap16(out[0], out[1]);
    swap16(out[2], out[3]);
}

// Eight codes times sigma.  `sigma` holds sigma * 2^-8 twice: an E4M3 byte shifted left by 7 is that FP16 number.
static __device__ __forceinline__ f16x8 expand_codes(uint32_t w, uint32_t sigma)
{
    const f16x2 by = __builtin_bit_cast(f16x2, sigma);
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 256.0f, 0) * by, b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 256.0f, 1) * by;
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 256.0f, 2) * by, d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 256.0f, 3) * by;
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

static __device__ __forceinline__ void store_one(const MatvecArgs &a, int64_t m, int64_t n, float v)
{
    if (a.out == MQ_OUT_BF16)
        reinterpret_cast<uint16_t *>(a.y)[m * a.ldy + n] = __builtin_bit_cast(uint16_t, (__bf16)v);
    else
        reinterpret_cast<float *>(a.y)[m * a.ldy + n] = v;
}

// LDS: activations from the workgroup's own LDS (at most kLdsTokens), else from `packed`.  Codes are loaded four iterations
// ahead, activations one, and the scales of four iterations at once: lane group g loads iteration g's.  No load is conditional:
// a branch around one makes the compiler wait for all of them.
template <bool LDS, int MT, int S, int NW>
__global__ __launch_bounds__(64 * NW) void matvec_kernel(MatvecArgs a)
{
    __shared__ f32x4 part[S * MT < NW ? S * MT : NW][NW][64];
    __shared__ int lds_exps[NW][kLdsTokens];
    extern __shared__ __attribute__((aligned(16))) u32x4 lds_x[];  // [iteration][16 pieces][tokens]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
    const int64_t row0 = (int64_t)blockIdx.x * 16 * S;
    const int tile0 = blockIdx.y * MT, M = (int)a.M, slab = blockIdx.z;
    const int steps = (int)(a.K / 64), iters = (steps + 1) / 2, parts = a.slabs * NW;
    const int begin = (int)((int64_t)iters * (slab * NW + wave) / parts), end = (int)((int64_t)iters * (slab * NW + wave + 1) / parts);

    const uint8_t *code[S], *scale[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t r = min(row0 + 16 * s + col, a.N - 1);  // rows beyond the last are computed again and not stored
        code[s] = a.codes + r * a.c_row + 16 * (g & 1);
        scale[s] = a.scales + r * a.s_row;
    }
    u32x4 c[4][S], xv[2][MT][4];
    uint32_t sc[S][2];
    auto load_codes = [&](int u, int i) {  // (an iteration beyond the last reads the last again)
        const int64_t step = min(2 * i + (g >> 1), steps - 1);
#pragma unroll
        for (int s = 0; s < S; ++s) c[u][s] = *reinterpret_cast<const u32x4 *>(code[s] + step * a.c_step);
    };
    auto load_scales = [&](int i) {
        const int64_t one = min(2 * (i + g), steps - 1), two = min(2 * (i + g) + 1, steps - 1);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            sc[s][0] = *reinterpret_cast<const uint32_t *>(scale[s] + one * a.s_step);
            sc[s][1] = *reinterpret_cast<const uint32_t *>(scale[s] + two * a.s_step);
        }
    };
    load_scales(begin);
#pragma unroll
    for (int u = 0; u < 4; ++u) load_codes(u, begin + u);

    if constexpr (LDS) {
        // a wave's own part of K, with an exponent of its own: nothing to wait for but the wave itself
        const int pieces = (int)(a.K / 8);
        for (int m = 0; m < M; ++m) {
            const u32x4 *const from = reinterpret_cast<const u32x4 *>(a.x + m * a.ldx);
            uint32_t top = 0;
            for (int i = begin * 16 + lane; i < min(end * 16, pieces); i += 64) top = bf16_amax(from[i], top);
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
            const int e = shift_of(top);
            if (lane == 0) lds_exps[wave][m] = e;
            for (int i = begin * 16 + lane; i < end * 16; i += 64) lds_x[i * M + m] = i < pieces ? to_f16(from[i], e) : u32x4{0, 0, 0, 0};
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    const int own = min(col, M - 1);  // (columns beyond the last token are not stored either)
    auto load_x = [&](int b, int i) {
        const int at = min(i, (LDS ? max(end, 1) : iters) - 1);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (LDS)
                    xv[b][t][j] = lds_x[(at * 16 + 4 * g + j) * M + own];
                else
                    xv[b][t][j] = a.packed[((int64_t)at * a.tiles + min(tile0 + t, a.tiles - 1)) * 256 + 64 * j + lane];
            }
    };
    f32x4 acc[S][MT];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[s][t] = f32x4{0, 0, 0, 0};

    load_x(0, begin);
    // lane group g needs blocks 2g and 2g + 1 of an iteration's eight: of the first four scales' dword or of the second
    const uint32_t low = g & 1 ? 0x0c020c02u : 0x0c000c00u, high = g & 1 ? 0x0c030c03u : 0x0c010c01u;
    auto four = [&](int i0, auto more) {  // iterations i0 .. i0 + 3; more: and loads for the next four
        uint32_t sb[S][4];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            uint32_t one[4], two[4];
            gather4(sc[s][0], one);
            gather4(sc[s][1], two);
#pragma unroll
            for (int u = 0; u < 4; ++u) sb[s][u] = g < 2 ? one[u] : two[u];
        }
        if (more) load_scales(i0 + 4);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (!more && i0 + u >= end) break;
            if (more || u < 3) load_x((u + 1) & 1, i0 + u + 1);
            __builtin_amdgcn_sched_barrier(0);  // (the compiler would move the loads down to where they are needed)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const uint32_t sigma[2] = {__builtin_amdgcn_perm(0u, sb[s][u], low) << 7, __builtin_amdgcn_perm(0u, sb[s][u], high) << 7};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f16x8 w = expand_codes(c[u][s][j], sigma[j / 2]);
#pragma unroll
                    for (int t = 0; t < MT; ++t)
                        acc[s][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w, __builtin_bit_cast(f16x8, xv[u & 1][t][j]), acc[s][t], 0, 0, 0);
                }
            }
            // (two iterations' codes together: of a canonical row they share lines)
            __builtin_amdgcn_sched_barrier(0);
            if (more && (u & 1)) load_codes(u - 1, i0 + u + 3), load_codes(u, i0 + u + 4);
        }
    };
    int i0 = begin;
    for (; i0 + 4 < end; i0 += 4) four(i0, std::true_type());
    four(i0, std::false_type());

    const float alpha = *a.alpha;
    if constexpr (LDS)
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[s][0][i] = ldexpf(acc[s][0][i], -lds_exps[wave][own]);
    // NW of the S * MT tiles at a time, wave w adds the waves' sums of the w-th
#pragma unroll
    for (int base = 0; base < S * MT; base += NW) {
        if (base > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < NW; ++i)
            if (base + i < S * MT) part[i][wave][lane] = acc[(base + i) / MT][(base + i) % MT];
        __syncthreads();
        const int tile = base + wave, s = tile / MT, t = tile % MT;
        if (tile < S * MT) {
            f32x4 sum = part[wave][0][lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) sum += part[wave][w][lane];
            const int64_t n = row0 + 16 * s + 4 * g;
            const int m = 16 * (tile0 + t) + col;
            if (m < M) {
                const int e = LDS ? 0 : a.exps[m];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (n + i >= a.N) continue;
                    if (!LDS && a.slabs > 1)
                        a.sums[((int64_t)slab * M + m) * a.N + n + i] = sum[i];
                    else
                        store_one(a, m, n + i, ldexpf(sum[i], -e) * alpha);
                }
            }
        }
    }
}

// The slabs' sums in ascending order
__global__ __launch_bounds__(256) void matvec_join_kernel(MatvecArgs a)
{
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x, m = blockIdx.y;
    if (n >= a.N) return;
    float sum = 0.0f;
#pragma unroll 8
    for (int i = 0; i < a.slabs; ++i) sum += a.sums[((int64_t)i * a.M + m) * a.N + n];
    store_one(a, m, n, ldexpf(sum, -a.exps[m]) * *a.alpha);
}

// K that is no multiple of 64: one wave a row of W and token, a block of 16 elements per lane and step
__global__ __launch_bounds__(64) void matvec_simple_kernel(MatvecArgs a)
{
    const int lane = threadIdx.x;
    const int64_t n = blockIdx.x;
    const uint16_t *const x = a.x + (int64_t)blockIdx.y * a.ldx;
    float sum = 0.0f;
    for (int64_t b = lane; b < a.K / 16; b += 64) {
        const float sigma = __builtin_amdgcn_cvt_f32_fp8((int)a.scales[n * a.s_row + b], 0);
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

// Activations in every workgroup's LDS instead of a launch in front: for so few workgroups that each can afford it
// ([2, 14336 -> 4096] 14.5 us, packed 20.5; [4, 5120 -> 51200] 46 and 40; nine tokens of 4096 would be 39 instead of 21).  Four
// strips share a wide layer's; a narrow one has a strip and eight waves a workgroup ([1, 4096 -> 6144] 7.0 us, four strips 9.0;
// [1, 14336 -> 4096] 12 and 22).
static bool is_wide(int64_t N) { return N >= 8192; }
static bool in_lds(int64_t M, int64_t N, int64_t K)
{
    return M <= (is_wide(N) ? kLdsTokens / 2 : kLdsTokens) && M * ((K + 127) / 128) * 256 <= kLdsBytes;
}
static int64_t packed_bytes(int64_t M, int64_t K) { return (K + 127) / 128 * ((M + 15) / 16) * 4096; }

// Strips of a workgroup that share the packed activations, and slabs of K, by the time of the busiest of 256 compute units: the
// iterations of a slab times the workgroups that it gets.  Writing the slabs' sums and joining them costs about what 24 two-strip
// iterations do, and 4 for each slab and 64 tokens; an iteration of four strips 1.6 of two.
//   two strips:   [40, 25600 -> 5120], 160 workgroups a slab: no slabs 52 us, two (most units have one, some two) 56, three 44
//                 [5, 4096 -> 6144], 192: no slabs 9.5, two 12
//   four strips:  [40, 25600 -> 5120], 80: three slabs 37; [40, 12288 -> 8192], 128: no slabs 35, two 30, four 34;
//                 [64, 4096 -> 28672]: 38, two strips 46; [16, 4096 -> 4096] 11 and 9.6
struct Split {
    int strips, slabs;
};
static Split split_of(int64_t M, int64_t N, int64_t K)
{
    const int64_t iters = (K + 127) / 128, blocks = (M + 63) / 64;
    Split best{2, 1};
    double least = 1e300;
    for (int strips = 2; strips <= 4; strips += 2) {
        const int64_t groups = (N + 16 * strips - 1) / (16 * strips) * blocks;
        for (int slabs = 1; slabs == 1 || (slabs <= 8 && iters >= 16 * slabs); ++slabs) {
            const int64_t rounds = (groups * slabs + 255) / 256;
            const double cost = (double)(rounds * iters) / slabs * (strips == 4 ? 1.6 : 1.0) + (slabs > 1 ? 24 + 4 * slabs * blocks : 0);
            if (cost < least) least = cost, best = Split{strips, slabs};
        }
    }
    return best;
}

int64_t matvec_workspace(int64_t M, int64_t N, int64_t K)
{
    if (K % 64 || in_lds(M, N, K)) return 0;
    const int slabs = split_of(M, N, K).slabs;
    return packed_bytes(M, K) + 16 * ((M + 3) / 4) + (slabs > 1 ? 4 * slabs * M * N : 0);
}

int describe_nvfp4_matvec(int64_t M, int64_t N, int64_t K, mq_launch *out)
{
    if (K % 64) {
        *out = mq_launch{MQ_KERNEL_SIMPLE, 1, 1, 1, 1, M, N};
    } else if (in_lds(M, N, K)) {
        *out = mq_launch{MQ_KERNEL_MATVEC_LDS, 16, is_wide(N) ? 64 : 16, is_wide(N) ? 4 : 8, 1, M, N};
    } else {
        const Split split = split_of(M, N, K);
        *out = mq_launch{MQ_KERNEL_MATVEC, 16 * (int)std::min<int64_t>((M + 15) / 16, 4), 16 * split.strips, 4, split.slabs, M, N};
    }
    return 1;
}

template <bool LDS, int MT, int S, int NW>
static int launch(const MatvecArgs &a, hipStream_t s)
{
    const int64_t strips = (a.N + 16 * S - 1) / (16 * S), tokens = LDS ? 1 : (a.tiles + MT - 1) / MT;
    const int64_t lds = LDS ? a.M * ((a.K + 127) / 128) * 256 : 0;
    return enqueue(matvec_kernel<LDS, MT, S, NW>, dim3((unsigned)strips, (unsigned)tokens, (unsigned)a.slabs), dim3(64 * NW), (size_t)lds, s, a);
}

int configure_matvec_kernels()
{
    for (const void *k : {reinterpret_cast<const void *>(matvec_kernel<true, 1, 1, 8>), reinterpret_cast<const void *>(matvec_kernel<true, 1, 4, 4>)}) {
        const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLdsBytes);
        if (e != hipSuccess) return note_launch(e);
    }
    return MQ_OK;
}

int launch_nvfp4_matvec(const uint16_t *x, int64_t ldx, const uint8_t *codes, const uint8_t *scales, const float *alpha, int64_t M,
                        int64_t N, int64_t K, void *y, int64_t ldy, int out, int layout, void *ws, hipStream_t s)
{
    MatvecArgs a{x, ldx, codes, scales, alpha, K / 2, 32, K / 16, 4, M, N, K, y, ldy, out, (int)((M + 15) / 16), nullptr, nullptr, nullptr, 1};
    if (layout == MQ_LAYOUT_KTILE) a.c_row = 32, a.c_step = 32 * N, a.s_row = 4, a.s_step = 4 * N;
    if (K % 64) return enqueue(matvec_simple_kernel, dim3((unsigned)N, (unsigned)M), dim3(64), 0, s, a);
    if (in_lds(M, N, K)) return is_wide(N) ? launch<true, 1, 4, 4>(a, s) : launch<true, 1, 1, 8>(a, s);
    a.packed = static_cast<const u32x4 *>(ws);
    a.exps = reinterpret_cast<const int *>(static_cast<const char *>(ws) + packed_bytes(M, K));
    if (int rc = enqueue(matvec_pack_kernel, dim3((unsigned)M), dim3(1024), 0, s, a)) return rc;
    const Split split = split_of(M, N, K);
    a.slabs = split.slabs;
    a.sums = reinterpret_cast<float *>(static_cast<char *>(ws) + packed_bytes(M, K) + 16 * ((M + 3) / 4));
    auto go = [&](auto tiles) {
        constexpr int MT = decltype(tiles)::value;
        return split.strips == 4 ? launch<false, MT, 4, 4>(a, s) : launch<false, MT, 2, 4>(a, s);
    };
    const int rc = a.tiles == 1 ? go(std::integral_constant<int, 1>()) : a.tiles == 2 ? go(std::integral_constant<int, 2>())
                 : a.tiles == 3 ? go(std::integral_constant<int, 3>()) : go(std::integral_constant<int, 4>());
    if (rc || a.slabs == 1) return rc;
    return enqueue(matvec_join_kernel, dim3((unsigned)((N + 255) / 256), (unsigned)M), dim3(256), 0, s, a);
}

}  // namespace mq
