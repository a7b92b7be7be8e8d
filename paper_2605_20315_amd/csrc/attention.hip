// Attention over the paged FP8 cache: y = softmax(scale * q K^T) V per query head, causal, with an optional window.
//
// Queries of one sequence and one key head are rows: row r is head r % G of the group, token r / G, so the G query heads that
// share a key head read its cache once.  One pass over the keys with a running maximum and sum.  Three kernels:
//   attend_few    tiles of 16 or 32 rows, no LDS in its loop: bound by reading the cache
//   attend_many   tiles of 128 rows, the cache's tiles expanded once per workgroup into LDS: bound by the matrix and vector pipes
//   attend_tree   tiles of 16 or 32 rows of drafted tokens, which see of each other what a mask of bits says
// All compute the transposes S^T = K Q^T and O^T = V^T P^T: a lane then holds, of one row, the very scores that it has to
// supply as its slots of P^T in the second product, so the probabilities never move between lanes.  MFMA slots are matched
// to tokens and head elements by whatever order the loads have; both operands of a product only have to agree.
//
// Work is cut in the same way in all: (sequence, tile of rows, chunk of tokens, key head) is an item, one workgroup each,
// chunk lengths chosen on the device from the sequences' own lengths so that the items are about `target` (a batch of uneven
// lengths is cut evenly, and the host needs to know no lengths).  A sequence with several chunks leaves its partial sums in
// the workspace, and attend_join adds them in ascending order.
//
// Roundings.  Codes times page scales are BF16 numbers exactly, and scores, maxima, sums and the output's sums are binary32.  The
// probabilities are rounded to BF16 for the product with the values, 2^-8 of each at most, since a value with its page's
// exponent (-112 .. 119) fits no 16-bit operand but BF16, and both operands of a product are of one type: a prompt of 8192 is
// 0.0020 from 64 bits so, where a result whose only rounding is its own is 0.0016 (single tokens: 0.0017 and 0.0017).  The sum they are divided
// by is of the unrounded ones, but in attend_tree of the rounded ones.
// Ranges.  The output's sums are not divided before the end: with values of 2^119 over the number of places seen and more they may
// overflow.  Scores beyond 2^30 leave less of the exponential of a row's own maximum than 32 bits hold.
#include "kv8.h"

namespace mq {

constexpr int kTile = 64;       // tokens: chunks are whole tiles
constexpr int kFewRows = 16;
constexpr int kFewMost = 64;    // sequences of more rows go to attend_many where that is launched
constexpr int kAllMany = 8, kManyWaves = 4;
constexpr float kNone = -__builtin_inff();

// How a call is cut: rows per item, number of items aimed at, tiles a chunk has at least, sequences of more than `above` and
// at most `most` rows
struct Cut {
    int rows, target, least, above, most;
    bool split, fit;
    float *ws;
    int slots;   // that the workspace holds
    int tokens;  // attend_join goes by sequences of at most so many tokens; 0: by the call's tokens
};

struct Item {
    bool found;
    Span sp;
    int b, tile, head, chunks, lo, hi;  // tokens lo .. hi of the sequence for this chunk; lo is a multiple of kTile
    int slot;                           // of the partial sums
};

// What attend_join needs to know of a sequence, at the start of the workspace
struct Parts {
    int chunks, slot, row_tiles;  // slot: the sequence's first
};
constexpr int64_t kPartsBytes = 1 << 20;
constexpr int kPartsMost = (int)(kPartsBytes / sizeof(Parts));

struct Extent {
    int row_tiles, lo, tiles;  // first token (a multiple of kTile) and tiles of tokens that any query sees
};

// The first place that a token at `pos` sees (at least 0: it may lie before the first place, and its window is any int32)
static __device__ __forceinline__ int first_seen(const Kv8Attend &a, int pos)
{
    return a.window > 0 ? max(pos, a.window - 1) - (a.window - 1) : 0;
}

static __device__ __forceinline__ Extent extent_of(const Kv8Attend &a, const Cut &c, const Span &sp)
{
    Extent e{0, 0, 0};
    const int64_t rows = (int64_t)sp.n * (a.Hq / a.Hkv);
    if (rows <= c.above || rows > c.most) return e;
    e.row_tiles = (int)((rows + c.rows - 1) / c.rows);
    e.lo = first_seen(a, sp.start) & ~(kTile - 1);
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

static __device__ __forceinline__ void cut_sequence(const Kv8Attend &a, const Extent &e, int per, int &chunks, int &items, int &slots)
{
    // (a sequence whose queries see nothing still writes zeros; a last quarter of a chunk is worth one)
    chunks = e.row_tiles == 0 ? 0 : max((int)(((int64_t)e.tiles + (per == INT32_MAX ? 0 : (int64_t)per * 3 / 4)) / per), 1);
    items = e.row_tiles * chunks * a.Hkv;
    slots = chunks > 1 ? items : 0;
}

// sum over the sequences of what `of` makes of their extents
template <int NT, class F>
static __device__ __forceinline__ int64_t sum_of(const Kv8Attend &a, const Cut &c, PlanLds &lds, int tid, F &&of)
{
    if (a.s.B == 1) return of(extent_of(a, c, span_of(a.s, 0)));
    int64_t sum = 0;
    for (int b = tid; b < a.s.B; b += NT) sum += of(extent_of(a, c, span_of(a.s, b)));
    return block_sum<NT>(sum, lds.sums, tid);
}

// Tokens per chunk, in tiles, that make the call about c.target items; no more than that where c.fit: one workgroup too many
// is a second round of all (39 sequences in 530 items for 512 places 30 % longer than in fewer and longer ones, 218 us).
template <int NT>
static __device__ int chunk_tiles(const Kv8Attend &a, const Cut &c, PlanLds &lds, int tid)
{
    if (!c.split) return INT32_MAX;
    const int64_t work = sum_of<NT>(a, c, lds, tid, [](const Extent &e) { return (int64_t)e.row_tiles * e.tiles; });
    int per = (int)min(max((work * a.Hkv + c.target - 1) / c.target, (int64_t)c.least), (int64_t)1 << 28);
    if (c.fit)
        for (int i = 0; i < 8; ++i) {
            const int64_t items = sum_of<NT>(a, c, lds, tid, [&](const Extent &e) {
                int chunks, n, slots;
                cut_sequence(a, e, per, chunks, n, slots);
                return (int64_t)n;
            });
            if (items <= c.target) break;
            per += per / 8 + 1;
        }
    return per;
}

// The item `idx`; every thread of the workgroup calls it.  Workgroup 0 also writes down the sequences' parts.
template <int NT>
static __device__ Item item_of(const Kv8Attend &a, const Cut &c, int idx, PlanLds &lds, int tid)
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
        if (c.split && blockIdx.x == 0 && b < a.s.B) reinterpret_cast<Parts *>(c.ws)[b] = Parts{chunks, first_slot, e.row_tiles};
        if (idx >= first && idx < first + items) {
            // head fastest: with eight key heads the workgroups of one head share an XCD and its L2; then the tiles of rows that
            // read the same tokens, from the last, which sees the most, to the first
            const int local = idx - first, rest = local / a.Hkv, chunk = rest / e.row_tiles;
            // the chunks' shares of the tiles, even to within one
            const int t0 = (int)((int64_t)e.tiles * chunk / chunks), t1 = (int)((int64_t)e.tiles * (chunk + 1) / chunks);
            // (ranges of tokens that overlap, which cu_q must not have, could ask for more slots than there are)
            const int slot = first_slot + local;
            lds.found = Item{chunks == 1 || (unsigned)slot < (unsigned)c.slots, sp, b, e.row_tiles - 1 - rest % e.row_tiles, local - rest * a.Hkv, chunks, e.lo + t0 * kTile,
                             (int)min((int64_t)sp.len, (int64_t)e.lo + (int64_t)t1 * kTile), slot};
        }
        __syncthreads();
        if (idx < items_before && !(c.split && blockIdx.x == 0)) break;
    }
    __syncthreads();
    return lds.found;
}

// one partial result: sums [rows][D], then maxima and sums of the rows' exponentials
static __device__ __forceinline__ float *slot_at(const Cut &c, int D, int slot) 
{
    return c.ws + kPartsBytes / 4 + (int64_t)slot * c.rows * (D + 2);
}

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

// What a row's sums are multiplied by.  A sum of exponentials of zero: the row sees no place, and gives zeros, or no score above
// -infinity, and gives NaN as the definition does.
static __device__ __forceinline__ float inverse_of(const Kv8Attend &a, int b, const Span &sp, int pos, float total)
{
    if (total != 0.0f) return 1.0f / total;
    const int32_t *const table = a.s.page_table + b * a.s.pt_ld;
#pragma unroll 1
    for (int place = first_seen(a, pos); place <= min(pos, sp.len - 1); place = ((place >> a.s.page_shift) + 1) << a.s.page_shift)
        if ((unsigned)table[place >> a.s.page_shift] < (uint64_t)a.s.pages) return __builtin_nanf("");
    return 0.0f;
}

// Drafted tokens.  A token sees the places before the sequence's new tokens, and of those its own mask's: the new ones are in the
// last places, so only the last tiles differ from those of a chain, and there a row's 32 places are one word of bits.
template <bool TREE>
using Attend = std::conditional_t<TREE, Kv8TreeAttend, Kv8Attend>;

// The position that a window is measured from; it is no less than that of the sequence's first new token
static __device__ __forceinline__ int position_of(const Kv8TreeAttend &a, const Span &sp, int token)
{
    return a.positions ? max(a.positions[sp.q0 + token], sp.start) : sp.start + token;
}

static __device__ __forceinline__ uint32_t bits_below(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1; }

// Which of the places t .. t + 31 a token sees, as bits; `first` is the first that its window leaves.
static __device__ __forceinline__ uint32_t seen_word(const Kv8TreeAttend &a, int start, const uint32_t *mask, int first, int t)
{
    const int64_t at = (int64_t)t - start;  // the number of place t among the new tokens
    uint32_t seen = 0;
    if (at < 0) seen = bits_below((int)min(-at, (int64_t)32)) & ~bits_below((int)max(min((int64_t)first - t, (int64_t)32), (int64_t)0));
    if (at > -32 && at < 32 * a.words) {
        const int w = (int)(at >> 5), s = (int)(at & 31);
        const uint32_t lo = w >= 0 ? mask[w] : 0u, hi = s > 0 && w + 1 < a.words ? mask[w + 1] : 0u;
        seen |= (uint32_t)((((uint64_t)hi << 32) | lo) >> s);
    }
    return seen;
}

// As inverse_of, for the sequence's new token `token`
static __device__ __forceinline__ float tree_inverse_of(const Kv8TreeAttend &a, int b, const Span &sp, int token, float total)
{
    if (total != 0.0f) return 1.0f / total;
    const int32_t *const table = a.s.page_table + b * a.s.pt_ld;
    auto has_page = [&](int place) { return (unsigned)table[place >> a.s.page_shift] < (uint64_t)a.s.pages; };
#pragma unroll 1
    for (int place = first_seen(a, position_of(a, sp, token)); place < min(sp.start, sp.len); place = ((place >> a.s.page_shift) + 1) << a.s.page_shift)
        if (has_page(place)) return __builtin_nanf("");
    const uint32_t *const mask = a.tree + (int64_t)(sp.q0 + token) * a.words;
#pragma unroll 1
    for (int i = 0; i < min(sp.n, 32 * a.words); ++i) {
        const int place = sp.start + i;
        if ((mask[i >> 5] >> (i & 31) & 1) && place >= 0 && place < sp.len && has_page(place)) return __builtin_nanf("");
    }
    return 0.0f;
}

// 0x01 in the bytes that are NaN codes
static __device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u; }

// The order of instructions: N matrix instructions, behind each V vector instructions and T transcendental ones, and an LDS
// read.
template <int N, int V, int T>
static __device__ __forceinline__ void interleave()
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        if (V > 0) __builtin_amdgcn_sched_group_barrier(0x002, V, 0);
        if (T > 0) __builtin_amdgcn_sched_group_barrier(0x400, T, 0);
    }
}

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
// Measured, heads of 128, 32 on 8: 64 tokens after 100 to 8000 each, 600 MB, 116 us = 5.2 TB/s (a large copy 4.8), all of it
// waiting for memory (vector instructions 15 % of the time); two sequences of 105000, 435 MB, 83 us.  A branch around the loads
// ahead would make every wait one for all of them (125 and 92 us with the join, so 120.5 and 89).
// RT tiles of 16 rows: what a wave has expanded serves all of them (109 sequences of 23000, 52 rows each: 365 us with one, 233 with two).
template <int D, int RT>
__global__ __launch_bounds__(kFewThreads) void attend_few(Kv8Attend a, Cut c)
{
    constexpr int KW = D / 16;  // dwords of a key row's quarter, and MFMA steps over the head elements per 2 of them
    constexpr int VW = D / 64;  // dwords of a value row's sixteenth
    __shared__ PlanLds plan;
    constexpr int kRows = 16 * RT;
    __shared__ float stat[kFewWaves][2][kRows];
    __shared__ float sums[kFewWaves][kRows][D + 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
    const Item it = item_of<kFewThreads>(a, c, blockIdx.x, plan, tid);
    if (!it.found) return;
    const int G = a.Hq / a.Hkv, rows = it.sp.n * G, row0 = it.tile * kRows;
    int pos[RT], first[RT];  // the places that the lane's row of each tile sees: from first to pos
    u32x4 q[RT][D / 32];
    f32x4 acc[RT][D / 16];
    float mb[RT], l[RT];  // the running maximum times the scale, and the lane's share of the sum
#pragma unroll
    for (int f = 0; f < RT; ++f) {
        const int row = min(row0 + 16 * f + col, rows - 1), token = row / G, head = it.head * G + row - token * G;
        pos[f] = it.sp.start + token;
        first[f] = first_seen(a, pos[f]);
        const uint16_t *const p = a.q + (int64_t)(it.sp.q0 + token) * a.ldq + (int64_t)head * D + g * (D / 4);
#pragma unroll
        for (int s = 0; s < D / 32; ++s) q[f][s] = *reinterpret_cast<const u32x4 *>(p + 8 * s);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) acc[f][d] = f32x4{0, 0, 0, 0};
        mb[f] = kNone, l[f] = 0.0f;
    }
    // what every row of the item, and what any of them sees
    const int pos_lo = it.sp.start + row0 / G, pos_hi = it.sp.start + (min(row0 + kRows, rows) - 1) / G;
    const int hi = min(it.hi, pos_hi + 1), lo = max(it.lo, first_seen(a, pos_lo));
    const int all_lo = first_seen(a, pos_hi), all_hi = min(it.hi, pos_lo + 1);
    bool marked = false;  // whether the wave's part of `sums` holds NaN for what rows have seen

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
        f32x4 s[RT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int f = 0; f < RT; ++f) s[f][h] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < D / 32; ++w) {
                const bf16x8 k = expand8(x.k[h][w / 2][2 * (w % 2)], x.k[h][w / 2][2 * (w % 2) + 1], k_scale[h]);
#pragma unroll
                for (int f = 0; f < RT; ++f)
                    s[f][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, __builtin_bit_cast(bf16x8, q[f][w]), s[f][h], 0, 0, 0);
            }
        }
        const bool edge = t < all_lo || t + 32 > all_hi || id0 < 0 || id1 < 0;
        if (edge) {
            uint32_t seen[RT];
            bool odd = false;
#pragma unroll
            for (int f = 0; f < RT; ++f) seen[f] = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = t + 16 * h + 4 * g + j;
                    const bool there = at >= lo && at < hi && (h ? id1 : id0) >= 0;
#pragma unroll
                    for (int f = 0; f < RT; ++f) {
                        if (there && at >= first[f] && at <= pos[f])
                            seen[f] |= 1u << (4 * h + j);
                        else
                            s[f][h][j] = kNone;
                    }
                    // places that no row sees may hold anything, NaN codes among it: a zero probability would not hide those
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        x.v[4 * h + j][w] = there ? x.v[4 * h + j][w] : 0u;
                        odd |= nan_bytes(x.v[4 * h + j][w]) != 0;
                    }
                }
            if (__any(odd)) {
                // NaN values that some rows see and others do not: out of the product, and kept for the rows that see them
                if (!marked)
                    for (int i = lane; i < kRows * (D + 4); i += 64) (&sums[wave][0][0])[i] = 0.0f;
                marked = true;
#pragma unroll 1
                for (int r = 0; r < kRows; ++r) {
                    const uint32_t own = RT == 1 || r < 16 ? seen[0] : seen[RT - 1], sees = (uint32_t)__shfl((int)own, (r & 15) + 16 * g);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int w = 0; w < VW; ++w)
                            if (const uint32_t n = nan_bytes(x.v[j][w]); n && (sees >> j & 1))
#pragma unroll 1
                                for (int b = 0; b < 4; ++b)
                                    if (n >> (8 * b) & 1) sums[wave][r][col * (D / 16) + 4 * w + b] = __builtin_nanf("");
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int w = 0; w < VW; ++w) x.v[j][w] &= ~(nan_bytes(x.v[j][w]) * 0xffu);
            }
        }
        float top[RT];
        bool grown = false;
#pragma unroll
        for (int f = 0; f < RT; ++f) {
            const f32x4 u = s[f][0], v = s[f][1];
            top[f] = fmaxf(fmaxf(fmaxf(u[0], u[1]), fmaxf(u[2], u[3])), fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])));
            top[f] = fmaxf(top[f], __shfl_xor(top[f], 16));
            top[f] = fmaxf(top[f], __shfl_xor(top[f], 32)) * a.scale;
            grown |= top[f] > mb[f];
        }
        if (__any(grown))
#pragma unroll
            for (int f = 0; f < RT; ++f) {
                const float next = fmaxf(mb[f], top[f]), by = next == kNone ? 1.0f : __builtin_amdgcn_exp2f(mb[f] - next);
                mb[f] = next;
                l[f] *= by;
#pragma unroll
                for (int d = 0; d < D / 16; ++d) acc[f][d] *= by;
            }
        bf16x8 pb[RT];
#pragma unroll
        for (int f = 0; f < RT; ++f) {
            const float base = mb[f] == kNone ? 0.0f : mb[f];
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(s[f][j / 4][j % 4], a.scale, -base)), l[f] += p[j];
            pb[f] = four(pack2(p[0], p[1]), pack2(p[2], p[3]), pack2(p[4], p[5]), pack2(p[6], p[7]));
        }
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = x.v[j][w];
            bf16x8 turned[4];
            turn8(v, v_scale, turned);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int f = 0; f < RT; ++f) acc[f][4 * w + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(turned[d], pb[f], acc[f][4 * w + d], 0, 0, 0);
        }
    };

    constexpr int kStride = 32 * kFewWaves;
    for (int t0 = begin; t0 < hi; t0 += 32 * kStride) {
        look_up(t0);
        const int count = min(32, (hi - t0 + kStride - 1) / kStride);
        Tokens x[2];
        if constexpr (D * RT >= 256) {  // two sets of registers would leave one wave a SIMD (146 sequences of 200 tokens 77 us, 45 so)
            for (int i = 0; i < count; ++i) {
                load(t0 + i * kStride, i, x[0]);
                compute(t0 + i * kStride, i, x[0]);
            }
            continue;
        }
        // (no load is conditional: where one may have been left out the compiler waits for all of them)
        load(t0, 0, x[0]);
        int i = 0;
        for (; i + 2 < count; i += 2) {
            load(t0 + (i + 1) * kStride, i + 1, x[1]);
            compute(t0 + i * kStride, i, x[0]);
            load(t0 + (i + 2) * kStride, i + 2, x[0]);
            compute(t0 + (i + 1) * kStride, i + 1, x[1]);
        }
        if (i + 1 < count) {
            load(t0 + (i + 1) * kStride, i + 1, x[1]);
            compute(t0 + i * kStride, i, x[0]);
            compute(t0 + (i + 1) * kStride, i + 1, x[1]);
        } else {
            compute(t0 + i * kStride, i, x[0]);
        }
    }

    // the four waves' results: lane (col, g) holds, of row col, the elements (4g + i) * D / 16 + d for i < 4, d < D / 16
#pragma unroll
    for (int f = 0; f < RT; ++f) {
        l[f] += __shfl_xor(l[f], 16);
        l[f] += __shfl_xor(l[f], 32);
        if (g == 0) stat[wave][0][16 * f + col] = mb[f], stat[wave][1][16 * f + col] = l[f];
    }
    __syncthreads();
#pragma unroll
    for (int f = 0; f < RT; ++f) {
        const int r = 16 * f + col;
        float top = kNone;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, stat[w][0][r]);
        const float by = weight_of(mb[f], l[f], top);
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float &to = sums[wave][r][(4 * g + i) * (D / 16) + d];
                to = marked ? fmaf(acc[f][d][i], by, to) : acc[f][d][i] * by;
            }
    }
    __syncthreads();
    // 16 threads a row, D / 16 elements each
#pragma unroll
    for (int f = 0; f < RT; ++f) {
        const int r = 16 * f + (tid >> 4), e0 = (tid & 15) * (D / 16), row = row0 + r;
        if (row >= rows) return;
        float best = kNone, total = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) best = fmaxf(best, stat[w][0][r]);
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) total += stat[w][1][r] * weight_of(stat[w][0][r], stat[w][1][r], best);
        float o[D / 16];
#pragma unroll
        for (int e = 0; e < D / 16; ++e) o[e] = ((sums[0][r][e0 + e] + sums[1][r][e0 + e]) + sums[2][r][e0 + e]) + sums[3][r][e0 + e];
        if (it.chunks > 1) {
            float *const p = slot_at(c, D, it.slot);
#pragma unroll
            for (int e = 0; e < D / 16; e += 4) *reinterpret_cast<f32x4 *>(p + r * D + e0 + e) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
            if ((tid & 15) == 0) p[kRows * D + r] = best, p[kRows * D + kRows + r] = total;
            continue;
        }
        const int token = row / G;
        const float inv = inverse_of(a, it.b, it.sp, it.sp.start + token, total);
        uint32_t *const y = reinterpret_cast<uint32_t *>(a.y + (int64_t)(it.sp.q0 + token) * a.ldy + (int64_t)(it.head * G + row - token * G) * D + e0);
#pragma unroll
        for (int e = 0; e < D / 16; e += 2) y[e / 2] = pack2(o[e] * inv, o[e + 1] * inv);
    }
}

// ------------------------------------------------------------------------------------------------ many rows

// One item by four waves of 32 rows each, a tile of 64 tokens at a time.  The threads expand a tile's codes to BF16 in LDS once
// for all waves, in the order in which the matrix instructions take them: a block of 1 KB is one operand of one 32x32x16
// product, lane l's 16 bytes at 16 l, so that reading is free of bank conflicts and needs no address arithmetic.
//    keys    block (half of the tile, 16 elements): lane (token % 32, k = 8 elements)
//    values  block (16 tokens s, 32 elements): lane (element, tokens 16s + 4h .. + 3 and 16s + 8 + 4h .. + 3), h = lane / 32:
//            the tokens whose scores that lane holds after S^T = K Q^T
// The exponentials and what goes with them are as much vector work as the two products are matrix work, so the two have to run
// side by side: in a wave the keys of the next 32 tokens are multiplied between the exponentials of these, and their values
// between those and the next ones' maxima; and two workgroups share a compute unit, which their barriers hold up in turn.  So tile i
// of keys is 32 tokens ahead of tile i of values: tokens t + 32 .. t + 95 and t .. t + 63.  Both of tile i + 1 are loaded when
// tile i begins and expanded at its end; with two buffers one barrier a tile is enough.
// Measured, a prompt of 8192 tokens, 32 query and 8 key heads of 128: 595 us = 924 TFLOP/s of 1364 that a library product of
// 8192^3 reaches here.  Compared while it took 635 (its page numbers were looked at where they were read): without the keys
// ahead 747; one wave a SIMD with 64 rows, which reads LDS half as often, 945 (it has no second wave to fill its waits);
// eight waves in one workgroup 635, and less even shares of short work.
template <int D>
__global__ __launch_bounds__(64 * kManyWaves) void attend_many(Kv8Attend a, Cut c)
{
    constexpr int NW = kManyWaves, NT = 64 * NW, TN = 4 * D / NT;  // tasks of a thread: 32 bytes of codes each
    static_assert(TN * NT == 4 * D && (TN > 1 || NT == 2 * 2 * D), "every thread has the same tasks, or half of the waves those of keys");
    constexpr int kRows = 32 * NW;
    constexpr int kBlock16 = 1024 + 16;  // the padding spreads a key token's four writes over the banks
    constexpr int kHalf = 2 * (D / 16);  // blocks of a tile's keys, and of its values
    __shared__ PlanLds plan;
    __shared__ int flags[4];
    __shared__ uint32_t nans[kTile][D / 32], marks[D / 32][NT];  // what set_nan_aside finds, and the rows' elements that see it
    __shared__ __attribute__((aligned(16))) unsigned char keys[2][kHalf * kBlock16], values[2][kHalf * kBlock16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    const Item it = item_of<NT>(a, c, blockIdx.x, plan, tid);
    if (!it.found) return;
    const int G = a.Hq / a.Hkv, rows = it.sp.n * G, tile0 = it.tile * kRows, wave0 = tile0 + 32 * wave;
    // the lane's row (rows beyond the last are computed again and not stored) and the places that it sees
    const int row = min(wave0 + col, rows - 1), token = row / G, head = it.head * G + row - token * G;
    const int pos = it.sp.start + token, first = first_seen(a, pos);
    // places that any row of the workgroup sees, that any and that every row of the wave sees
    const int group_hi = min(it.hi, it.sp.start + (min(tile0 + kRows, rows) - 1) / G + 1);
    const int group_lo = max(it.lo, first_seen(a, it.sp.start + tile0 / G));
    const int pos_lo = it.sp.start + min(wave0, rows - 1) / G, pos_hi = it.sp.start + (min(wave0 + 32, rows) - 1) / G;
    const int all_lo = max(group_lo, first_seen(a, pos_hi)), all_hi = min(group_hi, pos_lo + 1);
    // places that every row of the workgroup sees
    const int rows_lo = max(group_lo, first_seen(a, it.sp.start + (min(tile0 + kRows, rows) - 1) / G));
    const int rows_hi = min(group_hi, it.sp.start + tile0 / G + 1);

    bf16x8 q[D / 16];
    {
        const uint16_t *const p = a.q + (int64_t)(it.sp.q0 + token) * a.ldq + (int64_t)head * D + 8 * h;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) q[s] = *reinterpret_cast<const bf16x8 *>(p + 16 * s);
    }
    f32x16 acc[D / 32];
    float mb = kNone, l = 0.0f;  // the running maximum times the scale, and the lane's share of the sum
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;

    const int P = 1 << a.s.page_shift;
    const int64_t unit = (int64_t)P * D;
    const int32_t *const table = a.s.page_table + it.b * a.s.pt_ld;
    const int begin = group_lo & ~(kTile - 1), tiles = group_hi > begin && a.s.pages > 0 ? (group_hi - begin + kTile - 1) / kTile : 0;

    // A thread's tasks: first of keys (token, 32 elements), then of values (16 tokens and a half of them, 4 elements); with one
    // task a thread the first waves take the keys.
    auto is_key = [&](int n) { return TN > 1 ? n < TN / 2 : wave < NW / 2; };
    auto task_of = [&](int n) { return TN > 1 ? tid + n % (TN / 2 ? TN / 2 : 1) * NT : tid % (NT / 2); };
    auto key_token = [&](int n) { return task_of(n) / (D / 32); };
    auto key_part = [&](int n) { return task_of(n) % (D / 32); };
    auto group_of = [&](int n) { return task_of(n) / (D / 4); };  // 16 tokens s and half h, as 2 s + h
    auto element_of = [&](int n) { return task_of(n) % (D / 4); };
    auto value_token = [&](int n) { return 16 * (group_of(n) >> 1) + 4 * (group_of(n) & 1); };
    auto place_of = [&](int i, int n) { return begin + i * kTile + (is_key(n) ? 32 + (key_token(n) & ~15) : 16 * (group_of(n) >> 1)); };
    struct Codes {
        uint32_t w[TN][8];
        int e[TN];      // the exponent byte
        bool there[TN];  // whether there is a page (else these are page 0's, to be taken for nothing)
    };
    // Page numbers are read an iteration before they are needed, and looked at only then; and no load is conditional: a comparison
    // at once, or a branch around a load, would wait for everything that is on its way (a prompt of 8192 took 9 % longer).
    // The index is clamped, as the place may lie beyond the history.
    int ids[TN];
    Codes x;
    auto pages_of = [&](int i) {
#pragma unroll
        for (int n = 0; n < TN; ++n) ids[n] = table[min(max(place_of(i, n), 0) >> a.s.page_shift, a.s.width - 1)];
    };
    auto load = [&](int i) {  // tile i, whose pages are in `ids`
        int64_t u[TN];
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            const int at = place_of(i, n);
            x.there[n] = at >= begin && at < group_hi && (unsigned)ids[n] < (uint64_t)a.s.pages;
            u[n] = (int64_t)(x.there[n] ? ids[n] : 0) * a.Hkv + it.head;
        }
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            if (is_key(n)) {
                x.e[n] = a.k_scales[u[n]];
                const u32x4 *const p = reinterpret_cast<const u32x4 *>(a.k_codes + u[n] * unit + (int64_t)((begin + i * kTile + 32 + key_token(n)) & (P - 1)) * D + 32 * key_part(n));
                const u32x4 y = p[0], z = p[1];
#pragma unroll
                for (int j = 0; j < 4; ++j) x.w[n][j] = y[j], x.w[n][4 + j] = z[j];
            } else {
                x.e[n] = a.v_scales[u[n]];
                const uint8_t *const p = a.v_codes + u[n] * unit + (int64_t)((begin + i * kTile + value_token(n)) & (P - 1)) * D + 4 * element_of(n);
#pragma unroll
                for (int j = 0; j < 8; ++j) x.w[n][j] = *reinterpret_cast<const uint32_t *>(p + ((j & 3) + 8 * (j >> 2)) * D);
            }
        }
    };
    auto expand = [&](int i) {
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            const float scale = exp2_of(min(max(x.e[n], 1), 254) - 127);
            if (is_key(n)) {
                const int tok = key_token(n);
                if (!x.there[n]) atomicOr(&flags[(i + tok / 32) & 3], 1 << ((tok / 16) ^ 2));
                unsigned char *const to = keys[i & 1] + ((tok / 32) * (D / 16) + 2 * key_part(n)) * kBlock16 + (tok & 31) * 16;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<bf16x8 *>(to + (j / 2) * kBlock16 + (j & 1) * 512) = expand8(x.w[n][2 * j], x.w[n][2 * j + 1], scale);
            } else {
                const int group = group_of(n), el = element_of(n), t = begin + i * kTile;
                // places that no row sees may hold anything, NaN codes among it: a zero probability would not hide those
                if (t < group_lo || t + kTile > group_hi || !x.there[n])
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int at = t + value_token(n) + (j & 3) + 8 * (j >> 2);
                        x.w[n][j] = x.there[n] && at >= group_lo && at < group_hi ? x.w[n][j] : 0u;
                    }
                if (t < rows_lo || t + kTile > rows_hi) {  // some rows of the workgroup do not see all of it
                    uint32_t odd = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) odd |= nan_bytes(x.w[n][j]);
                    if (odd) atomicOr(&flags[i & 3], 16);
                }
                const float both[2] = {scale, scale};
                bf16x8 turned[4];
                turn8(x.w[n], both, turned);
                unsigned char *const to = values[i & 1] + (group >> 1) * (D / 32) * kBlock16 + (group & 1) * 512;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const int block = D == 64 ? d & 1 : d + 4 * (el / 32), slot = D == 64 ? el + 16 * (d >> 1) : el & 31;
                    *reinterpret_cast<bf16x8 *>(to + block * kBlock16 + slot * 16) = turned[d];
                }
            }
        }
    };
    f32x16 s[2];  // of the tile's first and second 32 tokens
    float top;
    constexpr int kAhead = 2;  // LDS reads ahead of their products (3 or 4 are no faster)
    bf16x8 first_keys[kAhead];
    auto read_keys = [&](const unsigned char *from) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) first_keys[k] = *reinterpret_cast<const bf16x8 *>(from + k * kBlock16);
    };
    auto scores = [&](const unsigned char *from, int to) {
#pragma unroll
        for (int j = 0; j < 16; ++j) s[to][j] = 0.0f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const bf16x8 y = k < kAhead ? first_keys[k] : *reinterpret_cast<const bf16x8 *>(from + k * kBlock16);
            s[to] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, q[k], s[to], 0, 0, 0);
        }
    };
    auto maxima = [&](int of) {
        float m = s[of][0];
#pragma unroll
        for (int j = 1; j < 16; ++j) m = fmaxf(m, s[of][j]);
        const u32x2 both = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false));
        top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * a.scale;
    };
    auto sees = [&](int at, int no_page) { return at >= max(first, group_lo) && at <= pos && at < group_hi && !no_page; };
    const unsigned char *key_at, *value_at;
    auto half_step = [&](int i, int half, int flag) {
        const unsigned char *const next = key_at + half * (D / 16) * kBlock16, *const from = value_at + 2 * half * (D / 32) * kBlock16;
        read_keys(next);
        const int t = begin + i * kTile + 32 * half, bad = flag >> (2 * half) & 3;
        const bool edge = t < all_lo || t + 32 > all_hi || bad;
        if (edge) {
#pragma unroll
            for (int j = 0; j < 16; ++j) s[half][j] = sees(t + 8 * (j / 4) + 4 * h + j % 4, bad >> (j / 8) & 1) ? s[half][j] : kNone;
            maxima(half);
        }
        // The maximum only follows where a row's scores have outgrown it by 2^8: sums and products hold that in 32 bits, a
        // probability of BF16 has the same relative rounding, and most tiles need no pass over the sums.
        if (__any(top > mb + 8.0f)) {
            const float next = fmaxf(mb, top), by = next == kNone ? 1.0f : __builtin_amdgcn_exp2f(mb - next);
            mb = next;
            l *= by;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[d][j] *= by;
        }
        bf16x8 p[2];
        auto exponentials = [&](int k) {
            const float base = mb == kNone ? 0.0f : mb;
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(fmaf(s[half][8 * k + j], a.scale, -base));
            l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
            p[k] = four(pack2(e[0], e[1]), pack2(e[2], e[3]), pack2(e[4], e[5]), pack2(e[6], e[7]));
        };
        auto products = [&](int k) {
#pragma unroll
            for (int d = 0; d < D / 32; ++d) {
                const bf16x8 v = *reinterpret_cast<const bf16x8 *>(from + (k * (D / 32) + d) * kBlock16);
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[k], acc[d], 0, 0, 0);
            }
        };
        __builtin_amdgcn_sched_barrier(0);
        scores(next, half ^ 1);
        exponentials(0);
        interleave<D / 16, 320 / D, 128 / D>();
        products(0);
        exponentials(1);
        interleave<D / 32, 640 / D, 256 / D>();
        products(1);
        maxima(half ^ 1);
        interleave<D / 32, 4, 0>();
        if (half) expand(i + 1);
    };

    // Values of tile i that are NaN and that some rows of the workgroup see and others do not: out of the product, and a bit for
    // each row and element that sees one.
    auto set_nan_aside = [&](int i, int flag) {
        for (int j = tid; j < kTile * (D / 32); j += NT) (&nans[0][0])[j] = 0;
        __syncthreads();
        for (int block = wave; block < kHalf; block += NW) {
            uint16_t *const v = reinterpret_cast<uint16_t *>(values[i & 1] + block * kBlock16 + lane * 16);
            for (int j = 0; j < 8; ++j)
                if ((v[j] & 0x7fff) > 0x7f80) {
                    v[j] = 0;
                    atomicOr(&nans[16 * (block / (D / 32)) + 4 * h + (j & 3) + 8 * (j >> 2)][block % (D / 32)], 1u << col);
                }
        }
        __syncthreads();
        for (int j = 0; j < kTile; ++j)
            if (sees(begin + i * kTile + j, flag >> (j / 16) & 1))
                for (int d = 0; d < D / 32; ++d) marks[d][tid] |= nans[j][d];
        __syncthreads();
    };

    if (tid < 4) flags[tid] = 0;
    for (int j = 0; j < D / 32; ++j) marks[j][tid] = 0;
    if (tiles > 0) {
        pages_of(-1);
        load(-1);
        pages_of(0);
        __syncthreads();
        expand(-1);
        load(0);
        pages_of(1);
        __syncthreads();
        read_keys(keys[1] + lane * 16 + (D / 16) * kBlock16);
        scores(keys[1] + lane * 16 + (D / 16) * kBlock16, 0);
        maxima(0);
        expand(0);
        for (int i = 0; i < tiles; ++i) {
            __syncthreads();
            const int own_flag = flags[i & 3];
            if (tid == 0) flags[(i + 3) & 3] = 0;
            load(i + 1);
            pages_of(i + 2);
            const int flag = __builtin_amdgcn_readfirstlane(own_flag);
            if (flag & 16) set_nan_aside(i, flag);
            key_at = keys[i & 1] + lane * 16, value_at = values[i & 1] + lane * 16;
            half_step(i, 0, flag);
            half_step(i, 1, flag);
        }
    }

    l += __shfl_xor(l, 32);
    const int local = 32 * wave + col;
    if (tile0 + local >= rows) return;
    const bool split = it.chunks > 1;
    float *const part = slot_at(c, D, it.slot);
    if (split && h == 0) part[c.rows * D + local] = mb, part[c.rows * D + c.rows + local] = l;
    // (the item is read from LDS again: kept through the loop it spills 16 more scalar registers, 595 us for the long prompt's 591)
    const float inv = split ? 1.0f : inverse_of(a, plan.found.b, plan.found.sp, pos, l);
    uint16_t *const y = a.y + (int64_t)(it.sp.q0 + token) * a.ldy + (int64_t)head * D;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
        if (const uint32_t mark = marks[d][tid] >> (4 * h))
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (mark >> (8 * (i / 4) + i % 4) & 1) acc[d][i] = __builtin_nanf("");
    // acc[d][i] of the lane is element 4 e + d % 4 of its row, e = (8 (i / 4) + 4 h + i % 4) + 32 (d / 4); with 64 elements
    // the product's rows from 16 on hold the upper two of each four
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

// ------------------------------------------------------------------------------------------------ rows of drafted tokens

// N KB from memory into LDS at `to`, 16 bytes a lane and KB from `lane_at` bytes behind `from` on (the instruction's offset counts for
// both).  In inline assembly because the compiler holds every LDS read until all such loads have landed; the waits for them are
// written where they are read.
template <int N>
static __device__ __forceinline__ void lds_load(uint32_t to, uint32_t lane_at, const uint8_t *from)
{
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    static_assert(N == 1 || N == 2, "");
    if constexpr (N == 1)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(lane_at), "s"(from) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:1024"
                     :
                     : "s"(to), "v"(lane_at), "s"(from)
                     : "memory", "m0");
#pragma clang diagnostic pop
}

// As item_of, where no sequence is cut and there are at most NT: those with the longest histories first, so that no long item begins when the
// others end (64 trees after 100 to 8000: 173 us, 203 in the order of the call; 32 of 30 to 60 tokens with heads of 256 175 and 212; equal lengths lose
// nothing).  Each thread compares its sequence with all others, 0.5 us for 64.
template <int NT>
static __device__ Item longest_first(const Kv8Attend &a, const Cut &c, int idx, PlanLds &lds, uint2 *lengths, int tid)
{
    Span sp{};
    Extent e{};
    if (tid < a.s.B) sp = span_of(a.s, tid), e = extent_of(a, c, sp);
    const int items = e.row_tiles * a.Hkv;
    static_assert(NT <= 256, "a sequence's number in eight bits, the lowest first among equals");
    const uint32_t own = (uint32_t)min(e.tiles, 0xffffff) << 8 | (255 - tid);
    lengths[tid] = uint2{own, (uint32_t)items};
    if (tid == 0) lds.found.found = false;
    __syncthreads();
    int first = 0;
    if ((tid & ~63) < a.s.B)
#pragma unroll 1
        for (int i = 0; i < a.s.B; i += 16)  // (those behind the last have no items)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const uint2 other = lengths[i + k];
                first += other.x > own ? (int)other.y : 0;
            }
    if (idx >= first && idx < first + items) {
        const int local = idx - first, tile = local / a.Hkv;
        lds.found = Item{true, sp, tid, e.row_tiles - 1 - tile, local - tile * a.Hkv, 1, e.lo, (int)min((int64_t)sp.len, (int64_t)e.lo + (int64_t)e.tiles * kTile), 0};
    }
    __syncthreads();
    return lds.found;
}

// As attend_few, for drafted tokens, which have tens of rows a key head where single ones have a few: a tile's arithmetic counts as
// much as its memory, and a wave by itself issues a vector instruction only every other time that its SIMD could.  So registers are
// spared for a third wave a SIMD: the queries stand in LDS, and keys and values come through it (from memory straight into LDS, the next
// group's on their way while this one's are multiplied), into the same registers one after the other.  32 heads of 128 on 8:
// 64 sequences of 8 to 26 tokens after 100 to 8000 take 173 us, 237 by the kernels for single tokens and prompts; 60 tokens after 2000
// in one 22 and 26.9; two of 64 after 100000 to 131000 285 to 303 and 288; 32 of 30 to 60 after 500 to 6000, 16 heads of 256 on 4, 175 and 338.
// Of the 173, reading the cache (530 MB) is 108 at a large copy's rate.  In the long one the vector instructions, which expand and turn round the codes and
// take the exponentials, are 58 % of the time and the matrix pipes 37 %; LDS is busy 37 %, nearly half of it by bank conflicts, but an order without those of
// keys and values takes no less time.
template <int D, int RT>
__global__ __launch_bounds__(kFewThreads, D <= 128 ? 3 : 2) void attend_tree(Kv8TreeAttend a, Cut c, bool longest)
{
    constexpr int KW = D / 16;  // dwords of a key row's quarter
    constexpr int VW = D / 64;  // dwords of a value row's sixteenth
    constexpr int kRows = 16 * RT, kHalf = 32 * D, kPieces = D / 16, kLoads = D / 32;  // bytes, 16-byte pieces of a row, and loads of a group's keys or values
    constexpr int kSums = 2 * kRows * (D + 4) * 4, kRing = kFewWaves * 2 * kHalf;
    __shared__ PlanLds plan;
    __shared__ float stat[kFewWaves][2][kRows];
    __shared__ uint32_t marks[kFewWaves][kRows][D / 32];  // the rows' elements that have seen NaN, a bit each
    constexpr int kTurn = D == 64 ? 7 : 15;
    __shared__ u32x4 queries[kRows][D / 8];               // piece p of row r in place p ^ (r & kTurn)
    __shared__ int firsts[kRows], tokens[kRows];          // the first place that a row sees, and its token's number in the call
    __shared__ __attribute__((aligned(16))) unsigned char pool[kRing > kSums ? kRing : kSums];  // keys and values of each wave's group, then sums
    float(*const sums)[kRows][D + 4] = reinterpret_cast<float(*)[kRows][D + 4]>(pool);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
    const Item it = longest ? longest_first<kFewThreads>(a, c, blockIdx.x, plan, reinterpret_cast<uint2 *>(pool), tid) : item_of<kFewThreads>(a, c, blockIdx.x, plan, tid);
    if (!it.found) return;
    const int G = a.Hq / a.Hkv, rows = it.sp.n * G, row0 = it.tile * kRows;
    // (rows beyond the last are computed again and not stored)
    for (int i = tid; i < kRows * (D / 8); i += kFewThreads) {
        const int r = i / (D / 8), p = i % (D / 8), row = min(row0 + r, rows - 1), token = row / G;
        queries[r][p ^ (r & kTurn)] = *reinterpret_cast<const u32x4 *>(a.q + (int64_t)(it.sp.q0 + token) * a.ldq + (int64_t)(it.head * G + row - token * G) * D + 8 * p);
    }
    f32x4 acc[RT][D / 16];
    // the running maximum times the scale, and the sum of the probabilities as the product takes them: that of ones in the values' place
    // (kLow: none yet.  It is the lowest number: any other score is 2^8 above it, and one that is it has a probability of one)
    constexpr float kLow = -0x1.fffffep127f;
    float mb[RT];
    f32x4 sum[RT];
    const bf16x8 ones = four(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
    int all_lo = 0;  // what every row of the item sees
#pragma unroll
    for (int f = 0; f < RT; ++f) {
        const int token = min(row0 + 16 * f + col, rows - 1) / G, first = first_seen(a, position_of(a, it.sp, token));
        if (wave == 0 && g == 0) firsts[16 * f + col] = first, tokens[16 * f + col] = it.sp.q0 + token;
        all_lo = max(all_lo, first);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) acc[f][d] = f32x4{0, 0, 0, 0};
        mb[f] = kLow, sum[f] = f32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) all_lo = max(all_lo, __shfl_xor(all_lo, d));
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    // (uniform, and in scalar registers only if the compiler is told so)
    const int start = __builtin_amdgcn_readfirstlane(it.sp.start), head = __builtin_amdgcn_readfirstlane(it.head);
    const int hi = __builtin_amdgcn_readfirstlane(min(it.hi, it.sp.start + it.sp.n)), lo = __builtin_amdgcn_readfirstlane(max(it.lo, first_seen(a, it.sp.start)));
    const int all_hi = min(hi, start);
    bool marked = false;

    const int P = 1 << a.s.page_shift, unit_shift = a.s.page_shift + (D == 64 ? 6 : D == 128 ? 7 : 8);
    const int32_t *const table = a.s.page_table + it.b * a.s.pt_ld;
    const int begin = (lo & ~31) + 32 * wave;
    __syncthreads();

    // pages of the wave's next 32 groups: lane 2i + h holds half h of group i, as its (page, head), whose bytes memory has room for; -1: none
    int units = 0;
    float ks = 0.0f, vs = 0.0f;
    auto look_up = [&](int t) {
        const int at = t + (lane >> 1) * 32 * kFewWaves + (lane & 1) * 16, page = at >> a.s.page_shift;
        int id = at < hi && page < a.s.width ? table[page] : -1;
        if ((unsigned)id >= (uint64_t)a.s.pages) id = -1;
        const int64_t u = (int64_t)max(id, 0) * a.Hkv + head;
        units = id < 0 ? -1 : (int)u;
        ks = exp2_of(min((int)a.k_scales[u], 254) - 127);
        vs = exp2_of(min((int)a.v_scales[u], 254) - 127);
    };
    // A group is 32 tokens' keys and then their values, a row as it is in the page but for its pieces, which stand in an order that spreads
    // the reads over the banks: piece c of token t in place c ^ t.
    unsigned char *const ring = pool + wave * 2 * kHalf;
    const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)ring;
    const uint32_t lane_at = (lane / kPieces) * D + ((lane % kPieces) ^ (lane / kPieces % kPieces)) * 16;
    // where group i's tokens t .. t + 31 are, in bytes of either array
    auto where = [&](int t, int i, int64_t (&at)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int own = max(__builtin_amdgcn_readlane(units, 2 * i + h), 0), place = (t + 16 * h) & (P - 1);
            at[h] = ((int64_t)own << unit_shift) + place * D;
        }
    };
    auto fetch = [&](const int64_t (&at)[2], bool value) {
        const uint8_t *const codes = value ? a.v_codes : a.k_codes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t to = ring_at + (value ? kHalf : 0) + 16 * h * D;
            if constexpr (D <= 128) {
                lds_load<D / 64>(to, lane_at, codes + at[h]);
            } else {
                // (a load of heads of 256 holds four tokens: the pieces' order goes on with the fifth)
#pragma unroll
                for (int u = 0; u < 4; ++u) lds_load<1>(to + 1024 * u, lane_at ^ (64 * u), codes + at[h] + 1024 * u);
            }
        }
    };
    auto wait = [](int left) {  // until at most so many loads are on their way
        if (left)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    auto scales_of = [&](float x, int i, float (&to)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) to[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 2 * i + h));
    };

    auto group = [&](int t, int i, bool more) {
        const int unit0 = __builtin_amdgcn_readlane(units, 2 * i), unit1 = __builtin_amdgcn_readlane(units, 2 * i + 1);
        float scale[2];
        scales_of(ks, i, scale);
        int64_t next[2];
        where(t + 32 * kFewWaves, more ? i + 1 : i, next);
        f32x4 s[RT][2];
#pragma unroll
        for (int f = 0; f < RT; ++f) s[f][0] = s[f][1] = f32x4{0, 0, 0, 0};
        wait(1);  // (its values may still be on their way)
        {
            u32x4 k[2][KW / 4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int w = 0; w < KW / 4; ++w)
                    k[h][w] = *reinterpret_cast<const u32x4 *>(ring + (16 * h + col) * D + ((g * (KW / 4) + w) ^ (col % kPieces)) * 16);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read: their place is filled again
            if (more) fetch(next, false);
#pragma unroll
            for (int w = 0; w < D / 32; ++w)
#pragma unroll
                for (int f = 0; f < RT; ++f) {
                    const bf16x8 q = __builtin_bit_cast(bf16x8, queries[16 * f + col][(g * (D / 32) + w) ^ (col & kTurn)]);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        s[f][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(expand8(k[h][w / 2][2 * (w % 2)], k[h][w / 2][2 * (w % 2) + 1], scale[h]), q, s[f][h], 0, 0, 0);
                }
        }
        const bool edge = t < all_lo || t + 32 > all_hi || unit0 < 0 || unit1 < 0;
        uint32_t seen[RT], there = 0;  // of the lane's eight tokens: those that its row sees, and those that are any row's
        if (edge) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = t + 16 * h + 4 * g + j;
                    there |= (uint32_t)(at >= lo && at < hi && (h ? unit1 : unit0) >= 0) << (4 * h + j);
                }
#pragma unroll
            for (int f = 0; f < RT; ++f) {
                const int r = 16 * f + col;
                const uint32_t word = seen_word(a, start, a.tree + (int64_t)tokens[r] * a.words, firsts[r], t) >> (4 * g);
                seen[f] = ((word & 15) | (word >> 12 & 0xf0)) & there;
#pragma unroll
                for (int j = 0; j < 8; ++j) s[f][j / 4][j % 4] = seen[f] >> j & 1 ? s[f][j / 4][j % 4] : kNone;
            }
        }
        // The exponents above the maximum in use.  That only follows where a lane finds one of its row's scores to have outgrown it by 2^8,
        // as in attend_many (a chunk's early groups raise one of 32 rows' nearly always), and only then do lanes have to exchange theirs.
        bool grown = false;
#pragma unroll
        for (int f = 0; f < RT; ++f) {
            float top = kLow;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fmaf(s[f][j / 4][j % 4], a.scale, -mb[f]));
            grown |= top > 8.0f;
        }
        if (__any(grown))
#pragma unroll
            for (int f = 0; f < RT; ++f) {
                float top = kNone;
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, s[f][j / 4][j % 4]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32)) * a.scale;
                const float next_mb = fmaxf(mb[f], top), by = __builtin_amdgcn_exp2f(mb[f] - next_mb);
                mb[f] = next_mb;
                sum[f] *= by;
#pragma unroll
                for (int d = 0; d < D / 16; ++d) acc[f][d] *= by;
            }
        bf16x8 pb[RT];
#pragma unroll
        for (int f = 0; f < RT; ++f) {
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(s[f][j / 4][j % 4], a.scale, -mb[f]));
            pb[f] = four(pack2(p[0], p[1]), pack2(p[2], p[3]), pack2(p[4], p[5]), pack2(p[6], p[7]));
            sum[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[f], sum[f], 0, 0, 0);
        }
        scales_of(vs, i, scale);
        wait(more);
        uint32_t v[VW][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int token = 16 * (j / 4) + 4 * g + j % 4;
            const unsigned char *const p = ring + kHalf + token * D + ((col * VW / 4) ^ (token % kPieces)) * 16 + col * VW % 4 * 4;
            if constexpr (VW == 1) v[0][j] = *reinterpret_cast<const uint32_t *>(p);
            if constexpr (VW == 2) {
                const u32x2 y = *reinterpret_cast<const u32x2 *>(p);
                v[0][j] = y[0], v[1][j] = y[1];
            }
            if constexpr (VW == 4) {
                const u32x4 y = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
                for (int w = 0; w < 4; ++w) v[w][j] = y[w];
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) fetch(next, true);
        if (edge) {
            // places that no row sees may hold anything, NaN codes among it: a zero probability would not hide those
            bool odd = false;
#pragma unroll
            for (int w = 0; w < VW; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[w][j] = there >> j & 1 ? v[w][j] : 0u;
                    odd |= nan_bytes(v[w][j]) != 0;
                }
            if (__any(odd)) {
                // NaN values that some rows see and others do not: out of the product, and a mark for the rows that see them
                if (!marked)
                    for (int n = lane; n < kRows * (D / 32); n += 64) (&marks[wave][0][0])[n] = 0;
                marked = true;
#pragma unroll 1
                for (int r = 0; r < kRows; ++r) {
                    const uint32_t own = RT == 1 || r < 16 ? seen[0] : seen[RT - 1], sees = (uint32_t)__shfl((int)own, (r & 15) + 16 * g);
#pragma unroll
                    for (int w = 0; w < VW; ++w)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (const uint32_t n = nan_bytes(v[w][j]); n && (sees >> j & 1))
#pragma unroll 1
                                for (int b = 0; b < 4; ++b)
                                    if (n >> (8 * b) & 1) {
                                        const int e = col * (D / 16) + 4 * w + b;
                                        atomicOr(&marks[wave][r][e / 32], 1u << (e % 32));
                                    }
                }
#pragma unroll
                for (int w = 0; w < VW; ++w)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[w][j] &= ~(nan_bytes(v[w][j]) * 0xffu);
            }
        }
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            bf16x8 turned[4];
            turn8(v[w], scale, turned);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int f = 0; f < RT; ++f) acc[f][4 * w + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(turned[d], pb[f], acc[f][4 * w + d], 0, 0, 0);
        }
    };

    constexpr int kStride = 32 * kFewWaves;
    for (int t0 = begin; t0 < hi; t0 += 32 * kStride) {
        look_up(t0);
        const int count = min(32, (hi - t0 + kStride - 1) / kStride);
        int64_t at[2];
        where(t0, 0, at);
        fetch(at, false);
        fetch(at, true);
#pragma unroll 1
        for (int i = 0; i < count; ++i) group(t0 + i * kStride, i, i + 1 < count);
    }

    // The four waves' results, two and two: lane (col, g) holds, of row col, the elements (4g + i) * D / 16 + d for i < 4, d < D / 16
#pragma unroll
    for (int f = 0; f < RT; ++f) {
        mb[f] = mb[f] == kLow && !(sum[f][0] > 0.0f) ? kNone : mb[f];
        if (g == 0) stat[wave][0][16 * f + col] = mb[f], stat[wave][1][16 * f + col] = sum[f][0];
    }
    __syncthreads();
#pragma unroll 1
    for (int turn = 1; turn >= 0; --turn) {
        if (wave >> 1 == turn)
#pragma unroll
            for (int f = 0; f < RT; ++f) {
                const int r = 16 * f + col;
                float top = kNone;
#pragma unroll
                for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, stat[w][0][r]);
                const float by = weight_of(mb[f], sum[f][0], top);
#pragma unroll
                for (int d = 0; d < D / 16; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int e = (4 * g + i) * (D / 16) + d;
                        float &to = sums[wave & 1][r][e];
                        float x = acc[f][d][i] * by;
                        if (marked && (marks[wave][r][e / 32] >> (e % 32) & 1)) x = __builtin_nanf("");
                        to = turn ? x : x + to;
                    }
            }
        __syncthreads();
    }
    // 16 threads a row, D / 16 elements each (the item from LDS again, which spares its registers in the loop)
    const Item &own = plan.found;
    const int own_row0 = own.tile * kRows, own_rows = own.sp.n * G;
#pragma unroll
    for (int f = 0; f < RT; ++f) {
        const int r = 16 * f + (tid >> 4), e0 = (tid & 15) * (D / 16), row = own_row0 + r;
        if (row >= own_rows) return;
        float best = kNone, total = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) best = fmaxf(best, stat[w][0][r]);
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) total += stat[w][1][r] * weight_of(stat[w][0][r], stat[w][1][r], best);
        float o[D / 16];
#pragma unroll
        for (int e = 0; e < D / 16; ++e) o[e] = sums[0][r][e0 + e] + sums[1][r][e0 + e];
        if (own.chunks > 1) {
            float *const p = slot_at(c, D, own.slot);
#pragma unroll
            for (int e = 0; e < D / 16; e += 4) *reinterpret_cast<f32x4 *>(p + r * D + e0 + e) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
            if ((tid & 15) == 0) p[kRows * D + r] = best, p[kRows * D + kRows + r] = total;
            continue;
        }
        const int token = row / G;
        const float inv = tree_inverse_of(a, own.b, own.sp, token, total);
        uint32_t *const y = reinterpret_cast<uint32_t *>(a.y + (int64_t)(own.sp.q0 + token) * a.ldy + (int64_t)(own.head * G + row - token * G) * D + e0);
#pragma unroll
        for (int e = 0; e < D / 16; e += 2) y[e / 2] = pack2(o[e] * inv, o[e + 1] * inv);
    }
}

// ------------------------------------------------------------------------------------------------ partial sums

// Rows (token, head) of the sequences with several chunks.  D / 4 threads cover a row's elements; a workgroup's 1024 / D such
// groups take a row each (ROWS: many rows), or every so-many-th chunk of one row.
template <int D, bool ROWS, bool TREE>
__global__ __launch_bounds__(256) void attend_join(Attend<TREE> a, Cut c)
{
    constexpr int kCols = D / 4, kParts = 256 / kCols;
    __shared__ float tops[4], totals[kParts];
    __shared__ f32x4 sums[kParts][kCols];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = tid % kCols, part = tid / kCols;
    const int per = ROWS ? kParts : 1, groups = (a.Hq + per - 1) / per, unit = blockIdx.x / groups, h0 = (blockIdx.x - unit * groups) * per;
    int b = 0, t = unit;
    if (c.tokens > 0) {
        b = unit / c.tokens;
    } else {
        // sequences that end at or before t
        for (int base = 0; base < a.s.B; base += 256) {
            int done = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = base + 64 * k + lane;
                done += __popcll(__ballot(i < a.s.B && a.s.cu_q[min(i, a.s.B - 1) + 1] <= t));
            }
            b += done;
            if (done < 256) break;
        }
        if (b >= a.s.B) return;
    }
    const Parts parts = reinterpret_cast<const Parts *>(c.ws)[b];
    if (parts.chunks < 2 || parts.slot < 0 || (int64_t)parts.slot + (int64_t)parts.chunks * parts.row_tiles * a.Hkv > c.slots) return;
    const Span sp = span_of(a.s, b);
    if (c.tokens > 0) t = sp.q0 + unit - b * c.tokens;
    if (t < sp.q0 || t >= sp.q0 + sp.n) return;
    const int G = a.Hq / a.Hkv, h = ROWS ? min(h0 + part, a.Hq - 1) : h0;
    const int kv = h / G, row = (t - sp.q0) * G + h - kv * G, tile = row / c.rows, r = row - tile * c.rows;
    const int first = parts.slot + (parts.row_tiles - 1 - tile) * a.Hkv + kv, next = parts.row_tiles * a.Hkv;
    auto stats = [&](int i) { return slot_at(c, D, first + i * next) + c.rows * D + r; };
    float top = kNone, total = 0.0f;
    f32x4 o{0, 0, 0, 0};
    if constexpr (ROWS) {
#pragma unroll 8
        for (int i = 0; i < parts.chunks; ++i) top = fmaxf(top, stats(i)[0]);
    } else {
        for (int i = tid; i < parts.chunks; i += 256) top = fmaxf(top, stats(i)[0]);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    }
#pragma unroll 4
    for (int i = ROWS ? 0 : part; i < parts.chunks; i += ROWS ? 1 : kParts) {
        const float *const s = stats(i);
        const f32x4 x = *reinterpret_cast<const f32x4 *>(slot_at(c, D, first + i * next) + r * D + 4 * col);
        const float l = s[c.rows], w = weight_of(s[0], l, top);
        total += w * l;
        o += w * x;
    }
    if constexpr (!ROWS) {
        sums[part][col] = o;
        if (col == 0) totals[part] = total;
        __syncthreads();
        if (part > 0) return;
#pragma unroll
        for (int i = 1; i < kParts; ++i) o += sums[i][col], total += totals[i];
    } else if (h0 + part >= a.Hq) {
        return;
    }
    float inv;
    if constexpr (TREE)
        inv = tree_inverse_of(a, b, sp, t - sp.q0, total);
    else
        inv = inverse_of(a, b, sp, sp.start + t - sp.q0, total);
    *reinterpret_cast<u32x2 *>(a.y + (int64_t)t * a.ldy + (int64_t)h * D + 4 * col) = u32x2{pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv)};
}

// ------------------------------------------------------------------------------------------------ launches

constexpr int64_t kWorkspace = (int64_t)64 << 20;
// Items aimed at: as many workgroups as the GPU holds at a time (attend_few, which is bound by memory, half as many more: when a
// batch of uneven lengths took 124 us so, it took 136 with one round; two long sequences 92 and 89), but no more than half of the slots that
// the workspace holds, since the items of the sequences that are cut are less than twice as many.  For attend_many that is less than the
// GPU's places: 496 of 512 with heads of 128, 250 of 256 with heads of 256 (with heads of 64 the places, 768).
constexpr int kFewTarget = 768;
// workgroups of attend_many that a compute unit holds, by registers and LDS: three, two and one
static int many_target(int D) { return 256 * (D == 64 ? 3 : D == 128 ? 2 : 1); }
// workgroups of attend_tree with two tiles of rows that the GPU holds, by registers and LDS
static int tree_places(int D) { return 256 * (D == 64 ? 4 : 3); }
// (query row, place) pairs above which attend_tree takes two tiles of rows
constexpr int64_t kTreeRowPlaces = (int64_t)48 << 20;
static int slots_of(int rows, int D) { return (int)((kWorkspace - kPartsBytes) / ((int64_t)rows * (D + 2) * 4)); }
static int target_of(int most, int rows, int D) { return std::min(slots_of(rows, D) / 2, most); }

int64_t kv8_attention_workspace(int64_t T, int64_t B, int Hq, int Hkv, int D)
{
    (void)T, (void)B, (void)Hq, (void)Hkv, (void)D;
    return kWorkspace;
}

// One launch of a call: which kernel, how it cuts, and its workgroups
struct Launch {
    bool many;
    Cut cut;
    int64_t items;
};

constexpr int kManyRows = 32 * kManyWaves;

// Tiles of rows at most, over sequences of more than cut.above and at most cut.most rows with T tokens in all: the host knows no
// sequence's own length.  A tile begun by every sequence; where sequences of more rows are another kernel's, what their own rows fill; and
// where those of fewer are, the most that a row can count for, two tiles of kManyRows + 1 rows.  (2048 tokens beside 8
// single ones after 100000: 1056 us when the prompt's rows counted for attend_few and kept it from cutting, 405 so.)
static int64_t row_tiles_most(const Cut &cut, int64_t T, int64_t B, int64_t G)
{
    static_assert(2 * (kFewMost + 1) >= kManyRows + 1, "one tile of kFewMost + 1 rows counts for less");
    int64_t most = T * G / cut.rows + B;
    if (cut.most < INT32_MAX) most = std::min(most, B * ((cut.most + cut.rows - 1) / cut.rows));
    if (cut.above > 0) most = std::min(most, 2 * T * G / (kManyRows + 1));
    return most;
}

static int plan_attention(const Kv8Attend &a, Launch *out)
{
    const int D = a.D;
    const int64_t G = a.Hq / a.Hkv, T = a.s.T, B = a.s.B;
    const bool ws = a.ws && a.ws_bytes >= kWorkspace && B <= kPartsMost;
    int n = 0;
    // If every sequence has a token, none has more than T - B + 1 of them, and where there are few tokens a sequence (a decode
    // batch, drafted tokens among it) a second kernel that finds nothing to do costs more than a longer prompt loses in
    // attend_few.  (Every split of the work is right: it is only slower than it need be.  A batch on that side of the line with one
    // chunk of 512 after 100000 among 200 single tokens takes 2.1 ms.)  Up to kAllMany sequences attend_many takes all if it takes any: with
    // short histories that saves two launches (300 tokens beside 7 single ones after 500 to 2000: 32 us, 50 by two kernels; two
    // prompts of 100 beside 6 after 500 to 1000: 22 and 36; 512 beside one after 20000: 43 and 67), deep ones pay for tiles of 128 rows with few
    // in them (1024 beside 7 after 100000: 630 us, 330 by two kernels; 512 beside 3 after 50000: 140 and 110).  All with heads of 128, 32 on 8.
    const bool many = T > 4 * B && (T - B + 1) * G > kFewMost, few = !many || B > kAllMany;
    auto add = [&](bool is_many, int rows, int most_items, int least, int above, int most) {
        Cut cut{rows, target_of(most_items, rows, D), least, above, most, true, is_many, a.ws, slots_of(rows, D), 0};
        // Beside attend_many the sequences of attend_few have few tokens each, and most of the call's are not theirs (2048 beside 20
        // single ones after 300: 106 us, 108 with a join over all tokens)
        const int64_t tokens = std::max<int64_t>(kFewMost / G, 1);
        if (most < INT32_MAX && B * tokens < T) cut.tokens = (int)tokens;
        // An item for each tile of rows and key head; where sequences are cut, as many more as the target has, or as their
        // longest possible history has chunks.  None are cut where there are twice as many items as the GPU has places: looking for
        // them and the join cost more than they give in a batch without very uneven lengths (170 single tokens after 200 to 300, 8 key
        // heads: 27 us, 37 if they may be cut; after 2000 126 and 130; but 190 with one after 131000 803 and 197).
        const int64_t whole = row_tiles_most(cut, T, B, G) * a.Hkv, tiles = ((int64_t)a.s.width << a.s.page_shift) / kTile + 1;
        cut.split = ws && whole < 2 * cut.target && tiles >= 2 * cut.least;
        out[n++] = Launch{is_many, cut, cut.split ? std::min(whole + 2 * cut.target, whole * (tiles / cut.least + 1)) : whole};
    };
    // Two tiles of rows from one expansion where the average sequence has more than one: 64 times 5 drafted tokens after 100 to 8000
    // 150 us, 178 with one tile; 40 times 13 after 10000 255 and 312; but 64 times 4 129 and 121.  A prompt in the batch raises the average
    // for the single tokens beside it, which then lose by it what drafted ones would gain: 2048 beside 8 after 100000 412 and 381, 512
    // beside 40 times 13 296 and 324.  Heads of 256 have no registers for two.
    const bool two = D <= 128 && T * G > B * kFewRows;
    // Chunks of 8 tiles at least beside attend_many, whose own time hides longer ones (600 beside 40 after 200: 47 us, 62 with 2 tiles; 1000
    // beside 12 after 1000: 60 and 68; the same with deep histories; uncut these two take 66 and 74)
    if (few) add(false, two ? 2 * kFewRows : kFewRows, kFewTarget, many ? 8 : 2, 0, many ? kFewMost : INT32_MAX);
    if (many) add(true, kManyRows, many_target(D), 4, few ? kFewMost : 0, INT32_MAX);
    return n;
}

// Drafted tokens.  All of a call's sequences go to one kernel: they have about as many tokens each, and a second kernel that finds
// nothing to do costs 14 us.  Two tiles of rows from one expansion where there is enough work that arithmetic bounds it (32 heads of
// 128 on 8: two sequences of 64 tokens after 100000 to 131000 294 us, 406 with one tile; 64 of 16 after 4000 134 and 165), not where the latency of an
// item does (4 of 60 after 500 to 1000, cut: 29.6, 21.3 with one; one of 60 after 2000 28 and 23.4; 8 of 30 to 60 after 1000 to 4000 50 and 47).
// Few items of two tiles are cut into as many as the GPU holds at a time, others into 512: what comes after a first round then is short.
// Chunks of 8 tiles at least and histories of three of them, since a join costs 6 us (30 tokens after 300 in one sequence 11.5 us, 17.7 with chunks of two
// tiles; 5 of 60 to 120 after 100 to 900, heads of 256, 27.7 and 41.3; longer histories the same; with chunks of 12 16 tokens after 8000 21.8 and 20.7).
// All of this goes by the page table's width, the longest history that the host knows of: with a table for 131072 places the short ones are
// cut and joined after all (30 tokens after 300 18.9 us, 11.0 with a table as wide as the history; one of 60 after 2000 26.1 and 22.7; 5 of 60 to 120 with
// heads of 256 41.2 and 27.5; long ones the same).
static Launch plan_tree(const Kv8TreeAttend &a)
{
    const int D = a.D;
    const int64_t G = a.Hq / a.Hkv, T = a.s.T, B = a.s.B, places = (int64_t)a.s.width << a.s.page_shift;
    const bool ws = a.ws && a.ws_bytes >= kWorkspace && B <= kPartsMost;
    const bool two = D <= 128 && T * G > B * kFewRows && T * G * a.Hkv * places > kTreeRowPlaces;
    const int rows = two ? 2 * kFewRows : kFewRows;
    Launch p{false, Cut{rows, 0, 8, 0, INT32_MAX, true, false, a.ws, slots_of(rows, D), 0}, 0};
    const int64_t whole = row_tiles_most(p.cut, T, B, G) * a.Hkv, tiles = places / kTile + 1;
    p.cut.target = target_of(two && whole <= 256 ? tree_places(D) : 512, rows, D);
    p.cut.split = ws && whole < 2 * p.cut.target && tiles >= 3 * p.cut.least;
    p.items = p.cut.split ? std::min(whole + 2 * p.cut.target, whole * (tiles / p.cut.least + 1)) : whole;
    return p;
}

template <int D, bool TREE>
static int launch_join(const Attend<TREE> &a, const Cut &cut, hipStream_t s)
{
    constexpr int kPer = 1024 / D;
    const int64_t T = cut.tokens ? (int64_t)a.s.B * cut.tokens : a.s.T;
    return T * a.Hq >= 2048 ? enqueue(attend_join<D, true, TREE>, dim3((unsigned)(T * ((a.Hq + kPer - 1) / kPer))), dim3(256), 0, s, a, cut)
                            : enqueue(attend_join<D, false, TREE>, dim3((unsigned)(T * a.Hq)), dim3(256), 0, s, a, cut);
}

template <int D>
static int launch_tree(const Kv8TreeAttend &a, hipStream_t s)
{
    const Launch p = plan_tree(a);
    if (p.items > 0x7fffffff) return MQ_ERR_SHAPE;
    const bool longest = !p.cut.split && a.s.B > 1 && a.s.B <= kFewThreads && p.items > tree_places(D);
    auto go = [&](auto kernel) { return enqueue(kernel, dim3((unsigned)p.items), dim3(kFewThreads), 0, s, a, p.cut, longest); };
    const int rc = p.cut.rows == kFewRows ? go(attend_tree<D, 1>) : go(attend_tree<D, D <= 128 ? 2 : 1>);
    return rc || !p.cut.split ? rc : launch_join<D, true>(a, p.cut, s);
}

template <int D>
static int launch_attention(const Kv8Attend &a, hipStream_t s)
{
    Launch plan[2];
    const int n = plan_attention(a, plan);
    for (int i = 0; i < n; ++i) {
        const Launch &p = plan[i];
        if (p.items > 0x7fffffff) return MQ_ERR_SHAPE;
        auto go = [&](auto kernel, int threads) { return enqueue(kernel, dim3((unsigned)p.items), dim3(threads), 0, s, a, p.cut); };
        int rc;
        if (p.many)
            rc = go(attend_many<D>, 64 * kManyWaves);
        else if (p.cut.rows == kFewRows)
            rc = go(attend_few<D, 1>, kFewThreads);
        else
            rc = go(attend_few<D, D <= 128 ? 2 : 1>, kFewThreads);
        if (rc) return rc;
        if (!p.cut.split) continue;
        rc = launch_join<D, false>(a, p.cut, s);
        if (rc) return rc;
    }
    return MQ_OK;
}

int describe_kv8_attention(const Kv8Attend &a, mq_kv8_launch *out)
{
    Launch plan[2];
    const int n = plan_attention(a, plan);
    for (int i = 0; i < n; ++i)
        out[i] = mq_kv8_launch{plan[i].many ? MQ_KV8_MANY : MQ_KV8_FEW, plan[i].cut.rows, plan[i].cut.split, plan[i].items,
                               (int64_t)a.s.width << a.s.page_shift};
    return n;
}

int launch_kv8_attention(const Kv8Attend &a, hipStream_t s)
{
    if (a.s.T == 0 || a.s.B == 0) return MQ_OK;
    return a.D == 64 ? launch_attention<64>(a, s) : a.D == 128 ? launch_attention<128>(a, s) : launch_attention<256>(a, s);
}

int launch_kv8_tree_attention(const Kv8TreeAttend &a, hipStream_t s)
{
    if (a.s.T == 0 || a.s.B == 0) return MQ_OK;
    return a.D == 64 ? launch_tree<64>(a, s) : a.D == 128 ? launch_tree<128>(a, s) : launch_tree<256>(a, s);
}

}  // namespace mq
