// Drafted tokens: their trees, which of them the sampled tokens confirm, and the confirmed ones brought together in the cache.
//
// All three are a few dependent trips to memory for each sequence and no more: lengths, then parents (or the path), then, in the
// cache, page numbers, scales and codes.
#include "kv8.h"

namespace mq {

// One workgroup for each sequence: the parents in LDS, a thread walks up from its token and writes its words from the last to the
// first.
constexpr int kTreeThreads = 256;
__global__ __launch_bounds__(kTreeThreads) void draft_tree_kernel(DraftTree a)
{
    __shared__ int above[kDraftMost];
    const Span sp = span_of(a.s, blockIdx.x);
    const int tid = threadIdx.x, most = min(sp.n, 32 * a.words);
    for (int i = tid; i < most; i += kTreeThreads) {
        const int p = a.parents[sp.q0 + i];
        above[i] = p >= 0 && p < i ? p : -1;
    }
    __syncthreads();
    for (int i = tid; i < sp.n; i += kTreeThreads) {
        uint32_t *const row = a.tree + (int64_t)(sp.q0 + i) * a.words;
        int w = a.words - 1, levels = 0;
        uint32_t bits = 0;
        for (int at = i < most ? i : -1; at >= 0; at = above[at], ++levels) {
            for (; w > at >> 5; --w) row[w] = bits, bits = 0;
            if (a.window == 0 || levels < a.window) bits |= 1u << (at & 31);
        }
        for (; w >= 0; --w) row[w] = bits, bits = 0;
        a.positions[sp.q0 + i] = sp.start + (i < most ? levels - 1 : i);
    }
}

// One wave for each sequence.  A child has a higher number than its parent, so the search only goes on: a step looks at 64 tokens,
// which stay in registers while the path is among them.
__global__ __launch_bounds__(256) void draft_accept_kernel(DraftAccept a)
{
    const int lane = threadIdx.x & 63, b = (int)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= a.s.B) return;
    const Span sp = span_of(a.s, b);
    int count = 0, want = -1;
    if (sp.n > 0) {
        int parent = 0, token = 0, sampled = 0, at = 0;
        auto load = [&](int base) {
            const int i = min(base + lane, sp.n - 1);
            parent = a.parents[sp.q0 + i], token = a.tokens[sp.q0 + i], sampled = a.sampled[sp.q0 + i];
        };
        load(0);
        want = __builtin_amdgcn_readfirstlane(sampled);
        if (lane == 0) a.path[sp.q0] = 0;
        count = 1;
        for (int base = 0; base < sp.n;) {
            const int i = base + lane;
            const unsigned long long fits = __ballot(i > at && i < sp.n && parent == at && token == want);
            if (fits) {
                const int child = __ffsll(fits) - 1;
                at = base + child;
                want = __builtin_amdgcn_readlane(sampled, child);
                if (lane == 0) a.path[sp.q0 + count] = at;
                ++count;
            } else if ((base += 64) < sp.n) {
                load(base);
            }
        }
    }
    for (int i = count + lane; i < sp.n; i += 64) a.path[sp.q0 + i] = -1;
    if (lane == 0) {
        a.counts[b] = count;
        a.next[b] = want;
        a.lens[b] = max(sp.start + count, 0);
    }
}

// The smallest e with |code| * 2^from <= 448 * 2^e, for the largest finite code (its seven lower bits)
static __device__ __forceinline__ int exponent_for(uint32_t code, int from)
{
    if (code == 0) return kExpLowest;
    const uint32_t bits = __float_as_uint(__builtin_amdgcn_cvt_f32_fp8((int)code, 0));
    const int e = (int)(bits >> 23) - 127 - ((bits & 0x7fffffu) <= 0x600000u ? 8 : 7);
    return min(max(e + from, kExpLowest), kExpHighest);
}

// codes times a power of two, each rounded once
static __device__ __forceinline__ u32x4 rescale(u32x4 c, float by)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 l = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), h = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
        c[i] = e4m3_of(l[0] * by, l[1] * by, h[0] * by, h[1] * by);
    }
    return c;
}

// One wave for each sequence, head, and keys or values; a lane has 16 codes of a token.  Pages are completed one after the other in
// ascending order.  A token only moves to a lower place than its own, and those behind it come from higher ones still: what a step
// writes is read by no later one, and a page's scale changes only when every token that leaves it has been read.
template <int D>
__global__ __launch_bounds__(256) void compact_kernel(Kv8Compact a, int units)
{
    constexpr int kSubs = D / 16, kPer = 64 / kSubs;  // lanes a token, tokens a step
    const int lane = threadIdx.x & 63, sub = lane % kSubs, row = lane / kSubs;
    const int unit = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= units) return;
    const int b = unit / (2 * a.Hkv), which = unit - b * 2 * a.Hkv, head = which >> 1;
    uint8_t *const codes = which & 1 ? a.v_codes : a.k_codes, *const scales = which & 1 ? a.v_scales : a.k_scales;
    const Span sp = span_of(a.s, b);
    const int count = min(max(a.counts[b], 0), sp.n), shift = a.s.page_shift, P = 1 << shift;
    const int32_t *const path = a.path + sp.q0, *const table = a.s.page_table + b * a.s.pt_ld;
    // the first token that moves
    int i = count;
    for (int base = 0; base < count; base += 64) {
        const unsigned long long other = __ballot(base + lane < count && path[min(base + lane, count - 1)] != base + lane);
        if (other) {
            i = base + __ffsll(other) - 1;
            break;
        }
    }
    i = max(i, -sp.start);  // (a length below the number of new tokens leaves the first ones no place)
    auto page_of = [&](int place) {  // -1: none
        const int id = place >= 0 && place < a.s.width << shift ? table[place >> shift] : -1;
        return (unsigned)id < (uint64_t)a.s.pages ? id : -1;
    };
    auto scale_of = [&](int id) { return min(max((int)scales[(int64_t)id * a.Hkv + head] - 127, kExpLowest), kExpHighest); };
    auto codes_at = [&](int id, int place) {
        return reinterpret_cast<u32x4 *>(codes + (((int64_t)id * a.Hkv + head) * P + (place & (P - 1))) * D + 16 * sub);
    };
    while (i < count) {
        const int first = ((sp.start + i) >> shift) << shift, end = (int)min((int64_t)count, (int64_t)first + P - sp.start);
        const int to = page_of(first);
        if (to < 0) {
            i = end;
            continue;
        }
        const int old = scale_of(to);
        // where the row's token of a step comes from: its page (-1: it does not move), its place, the page's exponent
        struct From {
            int id, place, e;
        };
        auto from = [&](int j) {
            From f{-1, 0, 0};
            const int number = path[min(j + row, end - 1)];
            if (j + row < end && number >= 0 && number < sp.n) {
                f.place = sp.start + number;
                f.id = page_of(f.place);
                f.e = f.id == to ? old : f.id >= 0 ? scale_of(f.id) : 0;
            }
            return f;
        };
        int e = old;
        for (int j = i; j < end; j += kPer) {
            const From f = from(j);
            if (f.id < 0 || f.e <= old) continue;
            const u32x4 c = *codes_at(f.id, f.place);
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const uint32_t v = (c[k / 4] >> (8 * (k % 4))) & 0x7f;
                m = max(m, v == 0x7f ? 0u : v);
            }
            e = max(e, exponent_for(m, f.e));
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) e = max(e, __shfl_xor(e, d));
        if (e > old) {  // the tokens in front of the first that moves
            const float by = exp2_of(max(old - e, -126));
            for (int place = first + row; place < sp.start + i; place += kPer) *codes_at(to, place) = rescale(*codes_at(to, place), by);
        }
        for (int j = i; j < end; j += kPer) {
            const From f = from(j);
            if (f.id < 0) continue;
            u32x4 c = *codes_at(f.id, f.place);
            if (f.e != e) c = rescale(c, exp2_of(min(max(f.e - e, -126), 127)));
            *codes_at(to, sp.start + j + row) = c;
        }
        if (e > old && lane == 0) scales[(int64_t)to * a.Hkv + head] = (uint8_t)(e + 127);
        i = end;
    }
}

int launch_draft_tree(const DraftTree &a, hipStream_t s)
{
    return enqueue(draft_tree_kernel, dim3(a.s.B), dim3(kTreeThreads), 0, s, a);
}

int launch_draft_accept(const DraftAccept &a, hipStream_t s)
{
    return enqueue(draft_accept_kernel, dim3((unsigned)((a.s.B + 3) / 4)), dim3(256), 0, s, a);
}

int launch_kv8_compact(const Kv8Compact &a, hipStream_t s)
{
    const int64_t units = (int64_t)a.s.B * 2 * a.Hkv;
    if (units > 0x7fffffff - 4) return MQ_ERR_SHAPE;
    auto go = [&](auto kernel) { return enqueue(kernel, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, a, (int)units); };
    return a.D == 64 ? go(compact_kernel<64>) : a.D == 128 ? go(compact_kernel<128>) : go(compact_kernel<256>);
}

}  // namespace mq
