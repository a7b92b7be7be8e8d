// Attention over the paged FP8 cache: y = softmax(scale * q K^T) V per query head, causal, with an optional window.
//
// Queries of one sequence and one key head are rows: row r is head r % G of the group, token r / G, so the G query heads that
// share a key head read its cache once.  One pass over the keys with a running maximum and sum.  Two kernels:
//   attend_few    tiles of 16 rows, no LDS in its loop: bound by reading the cache
//   attend_many   tiles of 256 rows (128 of 256 elements), the cache's tiles expanded once per workgroup into LDS: bound by the matrix pipe
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
constexpr int kFewRows = 16;
constexpr int kFewMost = 64;    // sequences of more rows go to attend_many where that is launched
constexpr float kNone = -__builtin_inff();

// How a call is cut: rows per item, number of items aimed at, tiles a chunk has at least, sequences of more than `above` and
// at most `most` rows
struct Cut {
    int rows, target, least, above, most;
    bool split;
    float *ws;
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
static __device__ __forceinline__ float weight_of(float m, float l, float top)
{
    return m == kNone ? l : __builtin_amdgcn_exp2f(m - top);
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
    float mb = kNone, l = 0.0f;  // the running maximum times the scale

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
        top = fmaxf(top, __shfl_xor(top, 32)) * a.scale;
        if (__any(top > mb)) {
            const float next = fmaxf(mb, top), by = next == kNone ? 1.0f : __builtin_amdgcn_exp2f(mb - next);
            mb = next;
            l *= by;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) acc[d] *= by;
        }
        const float base = mb == kNone ? 0.0f : mb;
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
    if (g == 0) stat[wave][0][col] = mb, stat[wave][1][col] = l;
    __syncthreads();
    float top = kNone;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, stat[w][0][col]);
    const float by = weight_of(mb, l, top);
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
    for (int w = 0; w < kFewWaves; ++w) total += stat[w][1][orow] * weight_of(stat[w][0][orow], stat[w][1][orow], best);
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

// ------------------------------------------------------------------------------------------------ many rows

// One item by NW waves of 32 rows each, a tile of 64 tokens at a time.  The threads expand a tile's codes to BF16 in LDS once
// for all waves, in the order in which the matrix instructions take them: a block of 1 KB is one operand of one 32x32x16
// product, lane l's 16 bytes at 16 l, so that reading is free of bank conflicts and needs no address arithmetic.  Two buffers:
// tile i + 1 is loaded while tile i is multiplied, expanded behind that, and one barrier a tile is enough.
//    keys    block (half of the tile, 16 elements): lane (token % 32, k = 8 elements)
//    values  block (16 tokens s, 32 elements): lane (element, tokens 16s + 4h .. + 3 and 16s + 8 + 4h .. + 3), h = lane / 32:
//            the tokens whose scores that lane holds after S^T = K Q^T
template <int D, int NW>
__global__ __launch_bounds__(64 * NW) void attend_many(Kv8Attend a, Cut c)
{
    constexpr int NT = 64 * NW, kTasks = 4 * D, TN = (kTasks + NT - 1) / NT;  // a task: 32 bytes of codes
    constexpr int kBlock16 = 1024 + 16;  // the padding spreads a key token's four writes over the banks
    constexpr int kKeys = 2 * (D / 16), kBlocks = 2 * kKeys;
    __shared__ PlanLds plan;
    __shared__ int flags[3];
    __shared__ __attribute__((aligned(16))) unsigned char tile[2][kBlocks * kBlock16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    const Item it = item_of<NT>(a, c, blockIdx.x, -1, plan, tid);
    if (!it.found) return;
    const int G = a.Hq / a.Hkv, rows = it.sp.n * G, tile0 = it.tile * 32 * NW, wave0 = tile0 + 32 * wave;
    const int r = wave0 + col, row = min(r, rows - 1), token = row / G, head = it.head * G + row - token * G;
    const int pos = it.sp.start + token;
    const int first = a.window > 0 ? pos - a.window + 1 : 0;
    // places that any row of the workgroup sees, that any and that every row of the wave sees
    const int group_hi = min(it.hi, it.sp.start + (min(tile0 + 32 * NW, rows) - 1) / G + 1);
    const int group_lo = max(it.lo, a.window > 0 ? it.sp.start + tile0 / G - a.window + 1 : 0);
    const bool live = wave0 < rows;
    const int pos_lo = it.sp.start + min(wave0, rows - 1) / G, pos_hi = it.sp.start + (min(wave0 + 32, rows) - 1) / G;
    const int hi = live ? min(it.hi, pos_hi + 1) : 0, lo = max(it.lo, a.window > 0 ? pos_lo - a.window + 1 : 0);
    const int all_lo = a.window > 0 ? pos_hi - a.window + 1 : 0, all_hi = min(it.hi, pos_lo + 1);

    bf16x8 q[D / 16];
    {
        const uint16_t *const p = a.q + (int64_t)(it.sp.q0 + token) * a.ldq + (int64_t)head * D + 8 * h;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) q[s] = *reinterpret_cast<const bf16x8 *>(p + 16 * s);
    }
    f32x16 acc[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
    float mb = kNone, l = 0.0f;  // the running maximum times the scale

    const int P = 1 << a.s.page_shift;
    const int64_t unit = (int64_t)P * D;
    const int32_t *const table = a.s.page_table + it.b * a.s.pt_ld;

    // of a thread's tasks: keys (token, 32 elements) below 2 D, values (16 tokens s and half h, 4 elements) from there
    auto is_key = [&](int n) { return tid + n * NT < 2 * D; };
    auto sub_of = [&](int n) { return is_key(n) ? (tid + n * NT) / (D / 32) / 16 : (tid + n * NT - 2 * D) / (D / 4) / 2; };
    auto page_of = [&](int t, int n) -> int {  // page of the task's 16 tokens in the tile at t, -1 if there is none
        const int at = t + 16 * sub_of(n);
        const int page = at >> a.s.page_shift;
        if (tid + n * NT >= kTasks || at >= group_hi || page >= a.s.width) return -1;
        const int id = table[page];
        return (unsigned)id < (uint64_t)a.s.pages ? id : -1;
    };
    uint32_t raw[TN][8];
    int exps[TN], ids[TN], next_ids[TN];
    auto load = [&](int t) {
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            const int task = tid + n * NT;
            exps[n] = 127;
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[n][i] = 0;
            if (ids[n] < 0) continue;
            const int64_t u = (int64_t)ids[n] * a.Hkv + it.head;
            if (is_key(n)) {
                const int tok = task / (D / 32), part = task % (D / 32);
                exps[n] = a.k_scales[u];
                const u32x4 *const p = reinterpret_cast<const u32x4 *>(a.k_codes + u * unit + (int64_t)((t + tok) & (P - 1)) * D + 32 * part);
                const u32x4 x = p[0], y = p[1];
#pragma unroll
                for (int i = 0; i < 4; ++i) raw[n][i] = x[i], raw[n][4 + i] = y[i];
            } else {
                const int group = (task - 2 * D) / (D / 4), el = (task - 2 * D) % (D / 4), tok = 16 * (group >> 1) + 4 * (group & 1);
                exps[n] = a.v_scales[u];
                const uint8_t *const p = a.v_codes + u * unit + (int64_t)((t + tok) & (P - 1)) * D + 4 * el;
#pragma unroll
                for (int i = 0; i < 8; ++i) raw[n][i] = *reinterpret_cast<const uint32_t *>(p + ((i & 3) + 8 * (i >> 2)) * D);
            }
        }
    };
    auto expand = [&](int t, unsigned char *to, int *flag) {
        int found = 0;
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            const int task = tid + n * NT;
            if (task >= kTasks) continue;
            const float scale = exp2_of(min(exps[n], 254) - 127);
            if (is_key(n)) {
                const int tok = task / (D / 32), part = task % (D / 32);
                if (ids[n] < 0) found |= 1 << (tok / 16);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<bf16x8 *>(to + ((tok / 32) * (D / 16) + 2 * part + j / 2) * kBlock16 + (j & 1) * 512 + (tok & 31) * 16) =
                        expand8(raw[n][2 * j], raw[n][2 * j + 1], scale);
            } else {
                const int group = (task - 2 * D) / (D / 4), el = (task - 2 * D) % (D / 4), tok = 16 * (group >> 1) + 4 * (group & 1);
                // places that no row sees may hold anything, NaN codes among it: a zero probability would not hide those
                if (t < group_lo || t + kTile > group_hi)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int at = t + tok + (i & 3) + 8 * (i >> 2);
                        raw[n][i] = at >= group_lo && at < group_hi ? raw[n][i] : 0u;
                    }
                uint32_t odd = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) odd |= nan_bytes(raw[n][i]);
                if (odd) found |= 16;
                const float both[2] = {scale, scale};
                bf16x8 turned[4];
                turn8(raw[n], both, turned);
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const int block = D == 64 ? d & 1 : d + 4 * (el / 32), slot = D == 64 ? el + 16 * (d >> 1) : el & 31;
                    *reinterpret_cast<bf16x8 *>(to + (kKeys + (group >> 1) * (D / 32) + block) * kBlock16 + ((group & 1) * 32 + slot) * 16) = turned[d];
                }
            }
        }
        if (found) atomicOr(flag, found);
    };
    auto compute = [&](int t, const unsigned char *from, int flag) {
        const unsigned char *const mine = from + lane * 16;
        f32x16 s[2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[tt][i] = 0.0f;
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(mine + (tt * (D / 16) + k) * kBlock16), q[k], s[tt], 0, 0, 0);
        }
        const bool edge = t < all_lo || t + kTile > all_hi || (flag & 15);
        uint32_t seen = ~0u;
        if (edge) {
            seen = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int off = 32 * (i / 16) + 8 * (i % 16 / 4) + 4 * h + i % 4, at = t + off;
                if (at >= max(first, lo) && at <= pos && at < hi && !(flag >> (off / 16) & 1))
                    seen |= 1u << i;
                else
                    s[i / 16][i % 16] = kNone;
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i / 16][i % 16]);
        top = fmaxf(top, __shfl_xor(top, 32)) * a.scale;
        // The maximum only follows where a row's scores have outgrown it by 2^8: sums and products hold that in 32 bits, a
        // probability of BF16 has the same relative rounding, and most tiles need no pass over the sums.
        if (__any(top > mb + 8.0f)) {
            const float next = fmaxf(mb, top), by = next == kNone ? 1.0f : __builtin_amdgcn_exp2f(mb - next);
            mb = next;
            l *= by;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= by;
        }
        const float base = mb == kNone ? 0.0f : mb;
        bf16x8 p[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(s[k / 2][8 * (k % 2) + i], a.scale, -base));
            l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
            p[k] = four(pack2(e[0], e[1]), pack2(e[2], e[3]), pack2(e[4], e[5]), pack2(e[6], e[7]));
        }
        const unsigned char *const values = mine + kKeys * kBlock16;
        if (edge && (flag & 16)) {
            // NaN values that some rows see and others do not: out of the product, and into the rows that see them by the
            // product of where they are with who sees them
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t w = seen >> (8 * k);
                const bf16x8 who = four(ones(w), ones(w >> 2), ones(w >> 4), ones(w >> 6));
                for (int d = 0; d < D / 32; ++d) {
                    u32x4 v = *reinterpret_cast<const u32x4 *>(values + (k * (D / 32) + d) * kBlock16), where;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t n = ((v[i] & 0x7fffu) > 0x7f80u ? 0xffffu : 0u) | ((v[i] & 0x7fff0000u) > 0x7f800000u ? 0xffff0000u : 0u);
                        where[i] = n & 0x3f803f80u;
                        v[i] &= ~n;
                    }
                    f32x16 hit;
#pragma unroll
                    for (int i = 0; i < 16; ++i) hit[i] = 0.0f;
                    hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, where), who, hit, 0, 0, 0);
#pragma unroll
                    for (int dd = 0; dd < D / 32; ++dd)
                        if (dd == d) {
                            acc[dd] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), p[k], acc[dd], 0, 0, 0);
#pragma unroll
                            for (int i = 0; i < 16; ++i) acc[dd][i] = hit[i] > 0.0f ? __builtin_nanf("") : acc[dd][i];
                        }
                }
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(values + (k * (D / 32) + d) * kBlock16), p[k], acc[d], 0, 0, 0);
    };

    const int begin = group_lo & ~(kTile - 1), tiles = group_hi > begin ? (group_hi - begin + kTile - 1) / kTile : 0;
    if (tid < 3) flags[tid] = 0;
    if (tiles > 0) {
#pragma unroll
        for (int n = 0; n < TN; ++n) ids[n] = page_of(begin, n);
        load(begin);
        __syncthreads();
        expand(begin, tile[0], &flags[0]);
#pragma unroll
        for (int n = 0; n < TN; ++n) next_ids[n] = tiles > 1 ? page_of(begin + kTile, n) : -1;
    }
    for (int i = 0; i < tiles; ++i) {
        const int t = begin + i * kTile;
        __syncthreads();
        if (tid == 0) flags[(i + 2) % 3] = 0;
        if (i + 1 < tiles) {
#pragma unroll
            for (int n = 0; n < TN; ++n) {
                ids[n] = next_ids[n];
                next_ids[n] = i + 2 < tiles ? page_of(t + 2 * kTile, n) : -1;
            }
            load(t + kTile);
        }
        if (t < hi && t + kTile > lo) compute(t, tile[i & 1], __builtin_amdgcn_readfirstlane(flags[i % 3]));
        if (i + 1 < tiles) expand(t + kTile, tile[(i + 1) & 1], &flags[(i + 1) % 3]);
    }

    l += __shfl_xor(l, 32);
    if (r >= rows) return;
    const bool split = it.chunks > 1;
    float *const part = slot_at(c, D, it.slot);
    const int local = 32 * wave + col;
    if (split && h == 0) part[c.rows * D + local] = mb, part[c.rows * D + c.rows + local] = l;
    const float inv = split ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t *const y = a.y + (int64_t)(it.sp.q0 + token) * a.ldy + (int64_t)head * D;
    // acc[d][i] of the lane is element 4 * e + d % 4 of its row, e = (8 (i / 4) + 4 h + i % 4) + 32 (d / 4); with 64 elements
    // the rows from 16 on of the product hold the upper two of each four
#pragma unroll
    for (int b = 0; b < (D + 127) / 128; ++b)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            if constexpr (D == 64) {
                const int e = 4 * ((8 * i4 + 4 * h) & 15) + (i4 >= 2 ? 2 : 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = acc[0][4 * i4 + i] * inv, z = acc[1][4 * i4 + i] * inv;
                    if (split)
                        *reinterpret_cast<f32x2 *>(part + local * D + e + 4 * i) = f32x2{x, z};
                    else
                        *reinterpret_cast<uint32_t *>(y + e + 4 * i) = pack2(x, z);
                }
            } else {
                const int e = 4 * (8 * i4 + 4 * h) + 128 * b;
                if (split) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4 *>(part + local * D + e + 4 * i) = f32x4{acc[4 * b][4 * i4 + i], acc[4 * b + 1][4 * i4 + i],
                                                                                         acc[4 * b + 2][4 * i4 + i], acc[4 * b + 3][4 * i4 + i]};
                } else {
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        u32x4 w;
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            w[2 * k] = pack2(acc[4 * b][4 * i4 + i + k] * inv, acc[4 * b + 1][4 * i4 + i + k] * inv),
                            w[2 * k + 1] = pack2(acc[4 * b + 2][4 * i4 + i + k] * inv, acc[4 * b + 3][4 * i4 + i + k] * inv);
                        *reinterpret_cast<u32x4 *>(y + e + 4 * i) = w;
                    }
                }
            }
        }
}

// ------------------------------------------------------------------------------------------------ partial sums

// Rows (token, head) of the sequences with several chunks, `heads` of one token by a workgroup: D / 4 threads cover a row's
// elements, the workgroup's other threads every so-many-th chunk.
template <int D>
__global__ __launch_bounds__(256) void attend_join(Kv8Attend a, Cut c, int heads)
{
    constexpr int kCols = D / 4, kParts = 256 / kCols;
    __shared__ PlanLds plan;
    __shared__ float tops[4], totals[kParts];
    __shared__ f32x4 sums[kParts][kCols];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = tid % kCols, part = tid / kCols;
    const int groups = (a.Hq + heads - 1) / heads, t = blockIdx.x / groups, h0 = (blockIdx.x - t * groups) * heads;
    int b = 0;
    for (int base = 0; base < a.s.B; base += 64) {
        const int i = base + lane;
        const unsigned long long done = __ballot(i < a.s.B && a.s.cu_q[min(i, a.s.B - 1) + 1] <= t);
        b += __popcll(done);
        if (done != ~0ull) break;
    }
    if (b >= a.s.B) return;
    const Item it = item_of<256>(a, c, 0, b, plan, tid);
    if (!it.found || it.chunks < 2 || t < it.sp.q0 || t >= it.sp.q0 + it.sp.n) return;
    const int G = a.Hq / a.Hkv;
    for (int h = h0; h < min(h0 + heads, a.Hq); ++h) {
        const int kv = h / G, row = (t - it.sp.q0) * G + h - kv * G, tile = row / c.rows, r = row - tile * c.rows;
        const int first = it.slot + (it.tiles - 1 - tile) * it.chunks * a.Hkv + kv;
        float top = kNone;
        for (int i = tid; i < it.chunks; i += 256) top = fmaxf(top, slot_at(c, D, first + i * a.Hkv)[c.rows * D + r]);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        float total = 0.0f;
        f32x4 o{0, 0, 0, 0};
#pragma unroll 4
        for (int i = part; i < it.chunks; i += kParts) {
            const float *const p = slot_at(c, D, first + i * a.Hkv), *const stat = p + c.rows * D + r;
            const f32x4 x = *reinterpret_cast<const f32x4 *>(p + r * D + 4 * col);
            const float w = weight_of(stat[0], stat[c.rows], top);
            total += w * stat[c.rows];
            o += w * x;
        }
        sums[part][col] = o;
        if (col == 0) totals[part] = total;
        __syncthreads();
        if (part == 0) {
#pragma unroll
            for (int i = 1; i < kParts; ++i) o += sums[i][col], total += totals[i];
            const float inv = total == 0.0f ? 0.0f : 1.0f / total;
            *reinterpret_cast<u32x2 *>(a.y + (int64_t)t * a.ldy + (int64_t)h * D + 4 * col) = u32x2{pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv)};
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------ launches

constexpr int kFewTarget = 1024;
constexpr int64_t kWorkspace = (int64_t)64 << 20;

static int64_t slot_bytes(int rows, int D) { return (int64_t)rows * (D + 2) * 4; }
// A sequence in several chunks has fewer than twice as many of them as whole targets' worth: the items of all that are cut
// are at most twice the target, and the slots of the workspace have to hold them.
static int many_target(int rows, int D) { return (int)std::min<int64_t>(kWorkspace / slot_bytes(rows, D) / 2, 512); }

int64_t kv8_attention_workspace(int64_t T, int64_t B, int Hq, int Hkv, int D)
{
    (void)T, (void)B, (void)Hq, (void)Hkv, (void)D;
    return kWorkspace;
}

template <int D>
static int launch_attention(const Kv8Attend &a, hipStream_t s)
{
    constexpr int kWaves = D == 256 ? 4 : 8, kRows = 32 * kWaves;
    const int64_t G = a.Hq / a.Hkv, T = a.s.T, B = a.s.B;
    const bool ws = a.ws && a.ws_bytes >= kWorkspace;
    // If every sequence has a token, none has more than T - B + 1 of them.  (Where some have none, one may have more: attend_few
    // is then slower than it need be, and as right.)
    const bool many = (T - B + 1) * G > kFewMost;
    auto go = [&](auto kernel, Cut cut, int threads) {
        // an item for each tile of rows and key head, and as many more as the target has
        cut.split = cut.split && ws;
        const int64_t items = (T * G / cut.rows + B) * a.Hkv + (cut.split ? 2 * cut.target : 0);
        if (items > 0x7fffffff) return (int)MQ_ERR_SHAPE;
        if (int rc = enqueue(kernel, dim3((unsigned)items), dim3(threads), 0, s, a, cut)) return rc;
        if (!cut.split) return (int)MQ_OK;
        // (a workgroup first finds its sequence's chunks: many rows share that)
        const int heads = (int)std::min<int64_t>(std::max<int64_t>(T * a.Hq / 2048, 1), a.Hq);
        return enqueue(attend_join<D>, dim3((unsigned)(T * ((a.Hq + heads - 1) / heads))), dim3(256), 0, s, a, cut, heads);
    };
    if (!many || B > 1)
        if (int rc = go(attend_few<D>, Cut{kFewRows, kFewTarget, 2, 0, many ? kFewMost : INT32_MAX, true, a.ws}, kFewThreads)) return rc;
    if (!many) return MQ_OK;
    const int target = many_target(kRows, D);
    return go(attend_many<D, kWaves>, Cut{kRows, target, 4, B > 1 ? kFewMost : 0, INT32_MAX, T * G / kRows * a.Hkv < 2 * target, a.ws}, 64 * kWaves);
}

int launch_kv8_attention(const Kv8Attend &a, hipStream_t s)
{
    if (a.s.T == 0 || a.s.B == 0) return MQ_OK;
    return a.D == 64 ? launch_attention<64>(a, s) : a.D == 128 ? launch_attention<128>(a, s) : launch_attention<256>(a, s);
}

}  // namespace mq
