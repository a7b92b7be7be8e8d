// Attention over the paged FP8 cache: y = softmax(scale * q K^T) V per query head, causal, with an optional window.
//
// Queries of one sequence and one key head are rows: row r is head r % G of the group, token r / G, so the G query heads that
// share a key head read its cache once.  One pass over the keys with a running maximum and sum.  Two kernels:
//   attend_few    tiles of 16 rows, no LDS in its loop: bound by reading the cache
//   attend_many   tiles of 256 rows, the cache's tiles expanded once per workgroup into LDS: bound by the matrix pipe
// Both compute the transposes S^T = K Q^T and O^T = V^T P^T: a lane then holds, of one row, the very scores that it has to
// supply as its slots of P^T in the second product, so the probabilities never move between lanes.  MFMA slots are matched
// to tokens and head elements by whatever order the loads have; both operands of a product only have to agree.
//
// Work is cut in the same way in both: (sequence, tile of rows, chunk of tokens, key head) is an item, one workgroup each,
// chunk lengths chosen on the device from the sequences' own lengths so that the items are about `target` (a batch of uneven
// lengths is cut evenly, and the host needs to know no lengths).  A sequence with several chunks leaves its partial sums in
// the workspace, and attend_join adds them in ascending order.
#include "kv8.h"

namespace mq {

constexpr int kTile = 64;       // tokens: chunks are whole tiles
constexpr int kFewRows = 16, kManyRows = 256;
constexpr int kFewMost = 64;    // sequences of more rows than this go to attend_many where that is launched
constexpr float kNone = -__builtin_inff();

// How a call is cut: rows per item, number of items aimed at, tiles a chunk has at least, sequences of more than `above` and
// at most `most` rows
struct Cut {
    int rows, target, least, above, most;
    bool split;
    float *ws;
    int slots;
};

struct Item {
    bool found;
    Span sp;
    int b, tile, head, chunk, chunks, lo, hi;  // tokens lo .. hi of the sequence for this chunk; lo is a multiple of kTile
    int slot;                                  // of the partial sums; the first one of the sequence for attend_join
    int tiles;                                 // of rows
};

struct Extent {
    int row_tiles, lo, tiles;  // first token (a multiple of kTile) and tiles of tokens that any query sees
};

static __device__ __forceinline__ Extent extent_of(const Kv8Attend &a, const Cut &c, const Span &sp)
{
    Extent e{0, 0, 0};
    const int64_t rows = (int64_t)sp.n * (a.Hq / a.Hkv);
    if (rows <= c.above || rows > c.most) return e;
    e.row_tiles = (int)((rows + c.rows - 1) / c.rows);
    e.lo = a.window > 0 ? max(sp.start - a.window + 1, 0) & ~(kTile - 1) : 0;
    e.tiles = sp.len > e.lo ? (sp.len - e.lo + kTile - 1) / kTile : 0;
    return e;
}

template <int NT>
static __device__ __forceinline__ int64_t block_sum(int64_t v, int64_t *lds, int tid)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    if ((tid & 63) == 0) lds[tid >> 6] = v;
    __syncthreads();
    int64_t sum = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) sum += lds[w];
    __syncthreads();
    return sum;
}

struct PlanLds {
    int64_t sums[16];
    int items[16], slots[16];
    Item found;
};

// tokens per chunk, in tiles, that make the call about c.target items
template <int NT>
static __device__ int chunk_tiles(const Kv8Attend &a, const Cut &c, PlanLds &lds, int tid)
{
    if (!c.split) return INT32_MAX;
    int64_t work = 0;
    if (a.s.B == 1) {
        const Extent e = extent_of(a, c, span_of(a.s, 0));
        work = (int64_t)e.row_tiles * e.tiles;
    } else {
        for (int b = tid; b < a.s.B; b += NT) {
            const Extent e = extent_of(a, c, span_of(a.s, b));
            work += (int64_t)e.row_tiles * e.tiles;
        }
        work = block_sum<NT>(work, lds.sums, tid);
    }
    const int64_t per = (work * a.Hkv + c.target - 1) / c.target;
    return (int)min(max(per, (int64_t)c.least), (int64_t)INT32_MAX);
}

static __device__ __forceinline__ void cut_sequence(const Kv8Attend &a, const Extent &e, int per, int &chunks, int &items, int &slots)
{
    // (a sequence whose queries see nothing still writes zeros)
    chunks = e.row_tiles == 0 ? 0 : e.tiles <= per ? 1 : (e.tiles - 1) / per + 1;
    items = e.row_tiles * chunks * a.Hkv;
    slots = chunks > 1 ? items : 0;
}

// The item `idx` (or, where `of` is not negative, the sequence `of` with its first slot).  Every thread of the workgroup calls it.
template <int NT>
static __device__ Item item_of(const Kv8Attend &a, const Cut &c, int idx, int of, PlanLds &lds, int tid)
{
    const int per = chunk_tiles<NT>(a, c, lds, tid), lane = tid & 63, wave = tid >> 6;
    if (tid == 0) lds.found.found = false;
    int items_before = 0, slots_before = 0;
    for (int base = 0; base < a.s.B; base += NT) {
        const int b = base + tid;
        Span sp{};
        Extent e{};
        int chunks = 0, items = 0, slots = 0;
        if (b < a.s.B) {
            sp = span_of(a.s, b);
            e = extent_of(a, c, sp);
            cut_sequence(a, e, per, chunks, items, slots);
        }
        const int item_sum = wave_scan(items, lane), slot_sum = wave_scan(slots, lane);
        __syncthreads();
        if (lane == 63) lds.items[wave] = item_sum, lds.slots[wave] = slot_sum;
        __syncthreads();
        int ib = items_before, sb = slots_before;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) {
            if (w < wave) ib += lds.items[w], sb += lds.slots[w];
            items_before += lds.items[w], slots_before += lds.slots[w];
        }
        const int first = ib + item_sum - items, first_slot = sb + slot_sum - slots;
        if (of >= 0 ? b == of : idx >= first && idx < first + items) {
            Item it;
            it.found = of < 0 || items > 0;
            it.sp = sp;
            it.b = b;
            it.chunks = chunks;
            it.tiles = e.row_tiles;
            it.slot = first_slot;
            it.lo = e.lo;
            it.hi = sp.len;
            it.head = it.chunk = it.tile = 0;
            if (of < 0) {
                // head fastest: with eight key heads the workgroups of one head share an XCD and its L2; then the chunk; the
                // tiles of rows from the last, which sees the most, to the first
                const int local = idx - first, rest = local / a.Hkv;
                it.head = local - rest * a.Hkv;
                it.chunk = rest % chunks;
                it.tile = e.row_tiles - 1 - rest / chunks;
                it.slot += local;
                const int size = (e.tiles + chunks - 1) / chunks;
                it.lo = e.lo + it.chunk * size * kTile;
                it.hi = (int)min((int64_t)sp.len, (int64_t)e.lo + (int64_t)(it.chunk + 1) * size * kTile);
            }
            lds.found = it;
        }
        __syncthreads();
        if (of >= 0 ? of < base + NT : idx < items_before) break;
    }
    __syncthreads();
    return lds.found;
}

// one partial result: sums [rows][D], then maxima and sums of the rows' exponentials
static __device__ __forceinline__ float *slot_at(const Cut &c, int D, int slot) { return c.ws + (int64_t)slot * c.rows * (D + 2); }

static __device__ __forceinline__ uint32_t pack2(float lo, float hi) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi}); }

static __device__ __forceinline__ bf16x8 four(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d});
}

// eight E4M3 codes times a power of two as BF16: exact
static __device__ __forceinline__ bf16x8 expand8(uint32_t lo, uint32_t hi, float scale)
{
    return four(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true)));
}

// What a part of a row with maximum m and sum l counts for beside the row's maximum.  No maximum: the part has seen nothing
// (l is 0) or NaN alone (l is NaN), and l says which.
static __device__ __forceinline__ float weight_of(float m, float l, float top, float scale)
{
    return m == kNone ? l : __builtin_amdgcn_exp2f((m - top) * scale);
}

// 0x01 in the bytes that are NaN codes
static __device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u; }

// 1.0 or 0.0 in BF16 for the lowest two bits
static __device__ __forceinline__ uint32_t ones(uint32_t bits) { return (bits & 1 ? 0x3f80u : 0u) | (bits & 2 ? 0x3f800000u : 0u); }

// Four bytes of each of eight tokens' rows (the same four head elements), turned round: out[d] = element d of the eight tokens
static __device__ __forceinline__ void turn8(const uint32_t (&w)[8], const float (&scale)[2], bf16x8 (&out)[4])
{
    uint32_t r[4][4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t lo = __builtin_amdgcn_perm(w[2 * p + 1], w[2 * p], 0x05010400), hi = __builtin_amdgcn_perm(w[2 * p + 1], w[2 * p], 0x07030602);
        const float s = scale[p / 2];
        r[0][p] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false));
        r[1][p] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true));
        r[2][p] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false));
        r[3][p] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true));
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) out[d] = four(r[d][0], r[d][1], r[d][2], r[d][3]);
}

// ------------------------------------------------------------------------------------------------ few rows

constexpr int kFewWaves = 4, kFewThreads = 64 * kFewWaves;

// One item by four waves, each with every fourth group of 32 tokens.  Lane (c = lane % 16, g = lane / 16) of a wave reads, of
// the keys, bytes g * D / 4 .. of token c of each half; of the values, bytes c * D / 16 .. of tokens 4g .. 4g + 3 of each half:
// whole rows of the page in one instruction, operands without any exchange between lanes.
template <int D>
__global__ __launch_bounds__(kFewThreads) void attend_few(Kv8Attend a, Cut c)
{
    constexpr int KW = D / 16;  // dwords of a key row's quarter, and MFMA steps over the head elements per 2 of them
    constexpr int VW = D / 64;  // dwords of a value row's sixteenth
    __shared__ PlanLds plan;
    __shared__ float stat[kFewWaves][2][16];
    __shared__ float sums[kFewWaves][16][D + 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
    const Item it = item_of<kFewThreads>(a, c, blockIdx.x, -1, plan, tid);
    if (!it.found) return;
    const int G = a.Hq / a.Hkv, rows = it.sp.n * G, r = it.tile * kFewRows + col;
    const int row = min(r, rows - 1), token = row / G, head = it.head * G + row - token * G;
    const int pos = it.sp.start + token;  // the last place that this row sees
    const int first = a.window > 0 ? pos - a.window + 1 : 0;
    // what every row of the tile, and what any of them sees
    const int last_token = (min((it.tile + 1) * kFewRows, rows) - 1) / G;
    const int pos_lo = it.sp.start + it.tile * kFewRows / G, pos_hi = it.sp.start + last_token;
    const int hi = min(it.hi, pos_hi + 1), lo = max(it.lo, a.window > 0 ? pos_lo - a.window + 1 : 0);
    const int all_lo = a.window > 0 ? pos_hi - a.window + 1 : 0, all_hi = min(it.hi, pos_lo + 1);

    u32x4 q[D / 32];
    {
        const uint16_t *const p = a.q + (int64_t)(it.sp.q0 + token) * a.ldq + (int64_t)head * D + g * (D / 4);
#pragma unroll
        for (int s = 0; s < D / 32; ++s) q[s] = *reinterpret_cast<const u32x4 *>(p + 8 * s);
    }
    f32x4 acc[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) acc[d] = f32x4{0, 0, 0, 0};
    float m = kNone, l = 0.0f;

    const int P = 1 << a.s.page_shift;
    const int64_t unit = (int64_t)P * D;
    const int32_t *const table = a.s.page_table + it.b * a.s.pt_ld;
    const int begin = (lo & ~31) + 32 * wave;

    struct Tokens {
        u32x4 k[2][KW / 4 ? KW / 4 : 1];
        uint32_t v[8][VW];
    };
    // pages of the wave's next 32 groups: lane 2i + h holds half h of group i
    int ids = 0;
    float ks = 0.0f, vs = 0.0f;
    auto look_up = [&](int t) {
        const int at = t + (lane >> 1) * 32 * kFewWaves + (lane & 1) * 16;
        const int page = at >> a.s.page_shift;
        ids = at < hi && page < a.s.width ? table[page] : -1;
        if ((unsigned)ids >= (uint64_t)a.s.pages) ids = -1;
        const int64_t u = (int64_t)max(ids, 0) * a.Hkv + it.head;
        ks = exp2_of(min((int)a.k_scales[u], 254) - 127);
        vs = exp2_of(min((int)a.v_scales[u], 254) - 127);
    };
    auto load = [&](int t, int i, Tokens &x) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int id = max(__builtin_amdgcn_readlane(ids, 2 * i + h), 0), place = (t + 16 * h) & (P - 1);
            const int64_t at = ((int64_t)id * a.Hkv + it.head) * unit + (int64_t)place * D;
            const uint8_t *const kp = a.k_codes + at + col * D + g * (D / 4);
#pragma unroll
            for (int w = 0; w < KW / 4; ++w) x.k[h][w] = *reinterpret_cast<const u32x4 *>(kp + 16 * w);
            const uint8_t *const vp = a.v_codes + at + 4 * g * D + col * (D / 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (VW == 1) x.v[4 * h + j][0] = *reinterpret_cast<const uint32_t *>(vp + j * D);
                if constexpr (VW == 2) {
                    const u32x2 v = *reinterpret_cast<const u32x2 *>(vp + j * D);
                    x.v[4 * h + j][0] = v[0], x.v[4 * h + j][1] = v[1];
                }
                if constexpr (VW == 4) {
                    const u32x4 v = *reinterpret_cast<const u32x4 *>(vp + j * D);
#pragma unroll
                    for (int w = 0; w < 4; ++w) x.v[4 * h + j][w] = v[w];
                }
            }
        }
    };
    auto compute = [&](int t, int i, Tokens &x) {
        const int id0 = __builtin_amdgcn_readlane(ids, 2 * i), id1 = __builtin_amdgcn_readlane(ids, 2 * i + 1);
        const float k_scale[2] = {__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), 2 * i)),
                                  __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), 2 * i + 1))};
        const float v_scale[2] = {__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), 2 * i)),
                                  __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), 2 * i + 1))};
        f32x4 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < D / 32; ++w)
                s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(expand8(x.k[h][w / 2][2 * (w % 2)], x.k[h][w / 2][2 * (w % 2) + 1], k_scale[h]),
                                                               __builtin_bit_cast(bf16x8, q[w]), s[h], 0, 0, 0);
        }
        const bool edge = t < all_lo || t + 32 > all_hi || id0 < 0 || id1 < 0;
        uint32_t seen = 0;
        bool odd = false;
        if (edge) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = t + 16 * h + 4 * g + j;
                    const bool there = at >= lo && at < hi && (h ? id1 : id0) >= 0;
                    if (there && at >= first && at <= pos)
                        seen |= 1u << (4 * h + j);
                    else
                        s[h][j] = kNone;
                    // places that no row sees may hold anything, NaN codes among it: a zero probability would not hide those
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        x.v[4 * h + j][w] = there ? x.v[4 * h + j][w] : 0u;
                        odd |= nan_bytes(x.v[4 * h + j][w]) != 0;
                    }
                }
            odd = __any(odd);
        }
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > m)) {
            const float next = fmaxf(m, top), by = next == kNone ? 1.0f : __builtin_amdgcn_exp2f((m - next) * a.scale);
            m = next;
            l *= by;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) acc[d] *= by;
        }
        const float base = m == kNone ? 0.0f : m * a.scale;
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(s[j / 4][j % 4], a.scale, -base)), l += p[j];
        const bf16x8 pb = four(pack2(p[0], p[1]), pack2(p[2], p[3]), pack2(p[4], p[5]), pack2(p[6], p[7]));
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = x.v[j][w];
            bf16x8 turned[4];
            if (odd) {
                // NaN values that some rows see and others do not: out of the product, and into the rows that see them by
                // the product of where they are with who sees them
                const bf16x8 who = four(ones(seen), ones(seen >> 2), ones(seen >> 4), ones(seen >> 6));
                const float one[2] = {1.0f, 1.0f};
                uint32_t where[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t n = nan_bytes(v[j]);
                    where[j] = n * 0x38u;  // 1.0
                    v[j] &= ~(n * 0xffu);
                }
                turn8(where, one, turned);
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(turned[d], who, f32x4{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[4 * w + d][i] = hit[i] > 0.0f ? __builtin_nanf("") : acc[4 * w + d][i];
                }
            }
            turn8(v, v_scale, turned);
#pragma unroll
            for (int d = 0; d < 4; ++d) acc[4 * w + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(turned[d], pb, acc[4 * w + d], 0, 0, 0);
        }
    };

    constexpr int kStride = 32 * kFewWaves;
    for (int t0 = begin; t0 < hi; t0 += 32 * kStride) {
        look_up(t0);
        const int count = min(32, (hi - t0 + kStride - 1) / kStride);
        Tokens x[2];
        load(t0, 0, x[0]);
        for (int i = 0; i < count; i += 2) {
            if (i + 1 < count) load(t0 + (i + 1) * kStride, i + 1, x[1]);
            compute(t0 + i * kStride, i, x[0]);
            if (i + 2 < count) load(t0 + (i + 2) * kStride, i + 2, x[0]);
            if (i + 1 < count) compute(t0 + (i + 1) * kStride, i + 1, x[1]);
        }
    }

    // the four waves' results: lane (col, g) holds, of row col, the elements (4g + i) * D / 16 + d for i < 4, d < D / 16
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) stat[wave][0][col] = m, stat[wave][1][col] = l;
    __syncthreads();
    float top = kNone;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, stat[w][0][col]);
    const float by = weight_of(m, l, top, a.scale);
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[wave][col][(4 * g + i) * (D / 16) + d] = acc[d][i] * by;
    __syncthreads();
    // 16 threads a row, D / 16 elements each
    const int orow = tid >> 4, e0 = (tid & 15) * (D / 16), out = it.tile * kFewRows + orow;
    if (out >= rows) return;
    float best = kNone, total = 0.0f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) best = fmaxf(best, stat[w][0][orow]);
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) total += stat[w][1][orow] * weight_of(stat[w][0][orow], stat[w][1][orow], best, a.scale);
    float o[D / 16];
#pragma unroll
    for (int e = 0; e < D / 16; ++e) o[e] = ((sums[0][orow][e0 + e] + sums[1][orow][e0 + e]) + sums[2][orow][e0 + e]) + sums[3][orow][e0 + e];
    if (it.chunks > 1) {
        float *const p = slot_at(c, D, it.slot);
#pragma unroll
        for (int e = 0; e < D / 16; e += 4) *reinterpret_cast<f32x4 *>(p + orow * D + e0 + e) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
        if ((tid & 15) == 0) p[kFewRows * D + orow] = best, p[kFewRows * D + kFewRows + orow] = total;
        return;
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const int t = out / G;
    uint32_t *const y = reinterpret_cast<uint32_t *>(a.y + (int64_t)(it.sp.q0 + t) * a.ldy + (int64_t)(it.head * G + out - t * G) * D + e0);
#pragma unroll
    for (int e = 0; e < D / 16; e += 2) y[e / 2] = pack2(o[e] * inv, o[e + 1] * inv);
}

// ------------------------------------------------------------------------------------------------ partial sums

// One wave a row (token, head) of the sequences with several chunks.
template <int D>
__global__ __launch_bounds__(256) void attend_join(Kv8Attend a, Cut c)
{
    __shared__ PlanLds plan;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int groups = (a.Hq + 3) / 4, t = blockIdx.x / groups, h = (blockIdx.x - t * groups) * 4 + wave;
    int b = 0;
    for (int base = 0; base < a.s.B; base += 64) {
        const int i = base + lane;
        const unsigned long long done = __ballot(i < a.s.B && a.s.cu_q[min(i, a.s.B - 1) + 1] <= t);
        b += __popcll(done);
        if (done != ~0ull) break;
    }
    if (b >= a.s.B) return;
    const Item it = item_of<256>(a, c, 0, b, plan, tid);
    if (!it.found || it.chunks < 2 || h >= a.Hq || t < it.sp.q0 || t >= it.sp.q0 + it.sp.n) return;
    const int G = a.Hq / a.Hkv, kv = h / G, row = (t - it.sp.q0) * G + h - kv * G, tile = row / c.rows, r = row - tile * c.rows;
    const int first = it.slot + (it.tiles - 1 - tile) * it.chunks * a.Hkv + kv;
    constexpr int E = D / 64;
    float best = kNone, total = 0.0f, o[E] = {};
    for (int i0 = 0; i0 < it.chunks; i0 += 64) {
        // a lane's own chunk gives the maximum; then the chunks in ascending order
        const int n = min(64, it.chunks - i0);
        const float *const mine = slot_at(c, D, first + (i0 + min(lane, n - 1)) * a.Hkv) + c.rows * D + r;
        const float m = lane < n ? mine[0] : kNone, l = lane < n ? mine[c.rows] : 0.0f;
        float top = m;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        top = fmaxf(top, best);
        const float past = weight_of(best, total, top, a.scale), by = weight_of(m, l, top, a.scale);
        best = top;
        float sum = l * by;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
        total = total * past + sum;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= past;
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(by), i));
            const float *const p = slot_at(c, D, first + (i0 + i) * a.Hkv) + r * D + lane * E;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] += w * p[e];
        }
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    uint16_t *const y = a.y + (int64_t)t * a.ldy + (int64_t)h * D + lane * E;
    if constexpr (E == 1) {
        y[0] = (uint16_t)pack2(o[0] * inv, 0.0f);
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 2) reinterpret_cast<uint32_t *>(y)[e / 2] = pack2(o[e] * inv, o[e + 1] * inv);
    }
}

// ------------------------------------------------------------------------------------------------ launches

constexpr int kFewTarget = 1024, kManyTarget = 512;

int64_t kv8_attention_workspace(int64_t T, int64_t B, int Hq, int Hkv, int D)
{
    (void)B, (void)Hq, (void)Hkv;
    if (T <= 0) return 0;
    // a sequence in n > 1 chunks has at most 2 (n - 1) of them for n - 1 whole targets' worth: no more than twice the target in all
    return (int64_t)2 * kFewTarget * kFewRows * (D + 2) * 4;
}

template <int D>
static int launch_attention(const Kv8Attend &a, hipStream_t s)
{
    const int G = a.Hq / a.Hkv;
    const int64_t T = a.s.T, B = a.s.B;
    Cut few{kFewRows, kFewTarget, 2, 0, INT32_MAX, false, nullptr, 0};
    const int64_t row_tiles = T * G / kFewRows + B;
    few.split = a.ws && a.ws_bytes >= kv8_attention_workspace(T, B, a.Hq, a.Hkv, D);
    few.ws = a.ws;
    // an item for each tile of rows and key head, and as many chunks more as the target has
    const int64_t items = row_tiles * a.Hkv + (few.split ? 2 * kFewTarget : 0);
    if (items > 0x7fffffff) return MQ_ERR_SHAPE;
    if (int rc = enqueue(attend_few<D>, dim3((unsigned)items), dim3(kFewThreads), 0, s, a, few)) return rc;
    if (!few.split) return MQ_OK;
    return enqueue(attend_join<D>, dim3((unsigned)(T * ((a.Hq + 3) / 4))), dim3(256), 0, s, a, few);
}

int launch_kv8_attention(const Kv8Attend &a, hipStream_t s)
{
    if (a.s.T == 0 || a.s.B == 0) return MQ_OK;
    return a.D == 64 ? launch_attention<64>(a, s) : a.D == 128 ? launch_attention<128>(a, s) : launch_attention<256>(a, s);
}

int configure_kv8_kernels() { return MQ_OK; }

}  // namespace mq
