// Shared by the kernels of chunks of new tokens over a paged cache: the sequences of a packed batch, tiles of 32 rows
// in LDS, and small wavefront helpers.
#pragma once

#include "attn_common.h"

namespace mcsd {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef const int32_t __attribute__((address_space(4))) *const_i32_ptr;      // wave-uniform reads through it are scalar loads

constexpr float LN2_F = 0.69314718055994530942f;

// x / d for 0 <= x < 2^31: with 2^(b-1) < d <= 2^b, m = floor(2^(31+b) / d) + 1 exceeds 2^(31+b) / d by at most 1, so that
// x m / 2^(31+b) is too large by less than 1 / d and its whole part right.
struct FastDiv {
    uint32_t magic;
    int shift;            // -1: d = 1
    FastDiv() = default;
    explicit FastDiv(int d)
    {
        int bits = 0;
        while ((1LL << bits) < d) ++bits;
        shift = bits - 1;
        magic = d > 1 ? (uint32_t)((1ULL << (31 + bits)) / (unsigned)d + 1) : 0;
    }
    __device__ __forceinline__ int of(int x) const { return shift < 0 ? x : (int)(__umulhi((uint32_t)x, magic) >> shift); }
};

struct ChunkParams {
    const void *q, *k_pool, *v_pool;
    const int32_t *chunk_start, *prefix_len, *block_table;
    void *out;
    float *lse, *part_o, *part_ml;
    struct ChunkNotes *notes;
    int B, T, H_q, H_kv, G, d, L_stride, page_size, n_pages, max_pages;
    FastDiv group;        // by G
    int many, by_work;    // rows beyond which a sequence belongs to the wide kernel; 1: where those have enough of the work
    int rows_few;         // ROWS_FEW, or ROWS_SPLIT
    int min_seg, max_parts, max_parts_many;
    float at_once, at_once_many;    // workgroups per KV head that the chip takes at once, of either kernel
    size_t q_row;         // bytes from a row of q to the next one's
    float scale_log2;     // scale * log2(e)
};

inline ChunkParams chunk_params(const mcsd_chunk_desc &d, const mcsd_paged_kv &kv)
{
    ChunkParams p = {};
    p.B = d.B; p.T = d.T; p.H_q = d.H_q; p.H_kv = d.H_kv; p.G = d.H_q / d.H_kv; p.d = d.d; p.L_stride = d.L_stride;
    p.page_size = kv.page_size; p.n_pages = kv.n_pages; p.max_pages = kv.max_pages_per_seq; p.block_table = kv.block_table;
    p.q_row = (size_t)d.q_stride * (d.dtype == MCSD_DTYPE_FP32 ? 4 : 2);
    p.scale_log2 = d.scale * LOG2E_F;
    p.group = FastDiv(p.G);
    return p;
}

__device__ __forceinline__ int by_group(const ChunkParams &p, int row) { return p.group.of(row); }

// New tokens s0 .. s0 + n - 1 of a sequence stand at positions L .. L + n - 1; `keys` positions are there (below the capacity).
// Whatever the caller's arrays hold, s0 + n <= T and keys <= L_stride.
struct ChunkSeq { int s0, n, L, keys; };

__device__ __forceinline__ ChunkSeq chunk_sequence(const ChunkParams &p, int b)
{
    ChunkSeq s;
    s.s0 = max(0, min(p.chunk_start[b], p.T));
    s.n = max(s.s0, min(p.chunk_start[b + 1], p.T)) - s.s0;
    s.L = max(0, min(p.prefix_len[b], p.L_stride));
    s.keys = min(s.L + s.n, p.L_stride);
    return s;
}

// A value that is the same in all lanes, back in a scalar register: divisions are vector arithmetic, and what stands behind one in a loop
// would follow it.
// (the statement keeps the compiler from following the value back)
__device__ __forceinline__ int uniform(int x)
{
    int r = __builtin_amdgcn_readfirstlane(x);
    asm("" : "+s"(r));
    return r;
}

// running sum over the lanes of a wavefront
__device__ __forceinline__ int wave_running_sum(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // inside the rows of 16
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // rows 0, 2 into 1, 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // and into 2, 3
    return v;
}

// sum and maximum (of values >= 0) over the lanes of a wavefront, in all of them
template <bool MAX>
__device__ __forceinline__ float wave_reduce(float v)
{
    auto join = [&](int x) { const float y = __int_as_float(x); v = MAX ? fmaxf(v, y) : v + y; };
    join(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x111, 0xf, 0xf, false));
    join(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x112, 0xf, 0xf, false));
    join(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x114, 0xf, 0xf, false));
    join(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x118, 0xf, 0xf, false));
    join(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x142, 0xa, 0xf, false));
    join(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x143, 0xc, 0xf, false));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_sum(float v) { return wave_reduce<false>(v); }
__device__ __forceinline__ float wave_max(float v) { return wave_reduce<true>(v); }

// ---- the work of a launch
// Rows r = token * G + head in group of a (sequence, KV head) go in tiles, of ROWS_MANY for sequences of more than p.many rows and
// of ROWS_FEW for others (one kernel each), the keys of a tile in equal segments of at least min_seg key tiles: a sequence is cut into
// kt / length of them, rounded up (few rows: a partial result is small) or to nearest.
// Every workgroup works out the same list, a sequence a lane; the length of segments of many rows takes longer and is left by the kernel for few
// (worked out by all workgroups: 10 to 40 us a launch).  Partial results are numbered in blocks of 32 rows, row tile by row tile, segment by segment.
// MANY: us with the kernel for many rows and with that for few: 32/8 heads, 80 rows of 32 sequences on 4000 tokens 151, 139, of 4 on 8000 58, 63; 128 rows 150, 153
// and 59, 71; 192 rows of 32 162, 217.  (Between 64 and 128 rows the border loses 8 % with many sequences and gains as much with few.)
constexpr int ROWS_SPLIT = 32, ROWS_FEW = 128, ROWS_MANY = 256, MANY = 64, NEVER_MANY = 0x7fffffff;
// Key tiles of many rows a workgroup at once, below which they do not pay for a kernel of their own (each item 8 tiles' time, the launch 4 us):
// us with the kernel for many rows and without it, work in tiles: one prompt of 512 tokens, 32/8 heads (4) 36.8, 30.2; 8 of 128 to 256, 32/32
// heads (6) 36.5, 35.0; 32 of 32 to 64 on 0 to 512, 32/8 heads (10) 68.9, 62.7; one of 256 on 4096, 32/8 heads (17) 50, 70; 8 of 64 to 128
// on 64 to 4096 (24) 78, 97.
constexpr float SMALL_WORK = 12.f;
// segments aimed at, times the workgroups at once
constexpr int CUTS = 4;
__host__ __device__ constexpr float cut_at(int j) { return j == 0 ? 1.f : j == 1 ? 1.5f : j == 2 ? 2.f : 3.f; }
enum ItemKind { FEW_ROWS, MANY_ROWS, MERGE };
struct Item { int b, rt, rows, seg, n_seg, part; ChunkSeq s; };

// what the kernel for few rows, which comes first, leaves to those behind it: items of the wide kernel that were taken; rows beyond which a
// sequence belongs to that; key tiles of a segment of either kernel
struct ChunkNotes { int taken, many, len, len_many; };

template <bool MANY_ROW_TILES> __device__ __forceinline__ int segments(int kt, int len) { return max(1, (kt + (MANY_ROW_TILES ? len / 2 : len - 1)) / len); }

// The sequences' row tiles and key tiles, one of the first 64 a lane, further ones read again by every search.
struct ChunkWork {
    ChunkSeq s = {0, 0, 0, 0};
    int many;           // rows beyond which a sequence belongs to the wide kernel

    __device__ __forceinline__ bool has_many(const ChunkParams &p, const ChunkSeq &q) const { return q.n * p.G > many; }
    __device__ __forceinline__ int row_tiles(const ChunkParams &p, const ChunkSeq &q) const
    {
        return has_many(p, q) ? (q.n * p.G + ROWS_MANY - 1) / ROWS_MANY : (q.n * p.G + p.rows_few - 1) / p.rows_few;
    }
    // f(many rows?, row tiles, key tiles) of every sequence
    template <class F>
    __device__ __forceinline__ void each(const ChunkParams &p, int lane, F &&f) const
    {
        f(has_many(p, s), row_tiles(p, s), (s.keys + KT - 1) / KT);
        for (int b = lane + 64; b < p.B; b += 64) {
            const ChunkSeq q = chunk_sequence(p, b);
            f(has_many(p, q), row_tiles(p, q), (q.keys + KT - 1) / KT);
        }
    }
    // Key tiles of a segment.  Few rows: so that there are about twice as many segments as the chip takes at once, which evens the lengths out
    // (a search among lengths, as for many rows, gains nothing: 32 sequences of 100 to 8000 tokens 131 us, 133 with it).
    __device__ __forceinline__ int few_segment(const ChunkParams &p, int lane)
    {
        float work, work_many;
        auto sum = [&]() {
            work = work_many = 0.f;
            each(p, lane, [&](bool m, int rt, int kt) {
                work += m ? 0.f : (float)rt * (float)kt;
                work_many += m ? (float)rt * (float)kt : 0.f;
            });
            work = wave_sum(work);
        };
        sum();
        if (p.by_work && many != NEVER_MANY && wave_sum(work_many) < fmaxf(work, SMALL_WORK * p.at_once_many)) {
            many = NEVER_MANY;
            sum();
        }
        return uniform(max(p.min_seg, (int)ceilf(work / (2.f * p.at_once))));
    }
    // Many rows: of CUTS lengths the one with which the kernel should end first.  An item costs 8 tiles' time beside its own, one that leaves
    // partial results 16 (32 sequences of 32 to 64 tokens on 64 to 4096, 32/8 heads: 182 us with one length, 143 so).  Items are taken in rounds, or all work goes over the workgroups and half the longest item is left over.
    __device__ __forceinline__ int many_segment(const ChunkParams &p, int lane) const
    {
        float work = 0.f, least = INFINITY;
        each(p, lane, [&](bool m, int rt, int kt) { work += m ? (float)rt * (float)kt : 0.f; });
        work = wave_sum(work);
        int best = p.min_seg;
        for (int j = 0; j < CUTS; ++j) {
            const int len = max(p.min_seg, (int)ceilf(work / (p.at_once_many * cut_at(j))));
            float items = 0.f, total = 0.f, longest = 0.f;
            each(p, lane, [&](bool m, int rt, int kt) {
                const int n = segments<true>(kt, len);
                const float own = (float)((kt + n - 1) / n) + (n > 1 ? 16.f : 8.f);
                items += m ? (float)(rt * n) : 0.f;
                total += m ? (float)(rt * n) * own : 0.f;
                longest = fmaxf(longest, m ? own : 0.f);
            });
            items = wave_sum(items), total = wave_sum(total), longest = wave_max(longest);
            const float end = fminf(ceilf(items / p.at_once_many) * longest, fmaxf(longest, total / p.at_once_many + 0.5f * longest));
            if (end < least) { least = end; best = len; }
        }
        return uniform(best);
    }
};

template <ItemKind KIND>
struct ItemList : ChunkWork {
    int len = 0, len_many = 0;              // key tiles of a segment of either kernel
    int rt = 0, n_seg = 1, blocks = 1, mine = 0, part = 0;      // of sequence `lane`
    struct Parts { int few, many; } parts;

    __device__ __forceinline__ ItemList(const ChunkParams &p, int lane)
    {
        if (lane < p.B) s = chunk_sequence(p, lane);
        many = p.many;
        if (KIND == FEW_ROWS) {
            if (p.notes) len = few_segment(p, lane);
        } else {
            many = uniform(p.notes->many);
            len = uniform(p.notes->len);
            len_many = uniform(p.notes->len_many);
        }
        parts = count(p, {0, p.max_parts});
    }
    // items and partial results of the lane's sequence, behind those of `before`; returns the partial results up to lane 63
    __device__ __forceinline__ Parts count(const ChunkParams &p, Parts before)
    {
        const bool many = has_many(p, s);
        const int kt = (s.keys + KT - 1) / KT;
        rt = row_tiles(p, s);
        blocks = (many ? ROWS_MANY : p.rows_few) / 32;
        n_seg = 1;
        if (many && p.max_parts_many && KIND != FEW_ROWS) n_seg = segments<true>(kt, len_many);
        if (!many && p.max_parts && KIND != MANY_ROWS) n_seg = segments<false>(kt, len);
        const int my_parts = n_seg > 1 ? rt * n_seg * blocks : 0;
        Parts to = before;
        if (KIND != MANY_ROWS) to.few += wave_running_sum(many ? 0 : my_parts);
        if (KIND != FEW_ROWS) to.many += wave_running_sum(many ? my_parts : 0);
        if (many ? to.many > p.max_parts + p.max_parts_many : to.few > p.max_parts) n_seg = 1;      // (cannot be, but by arrays that contradict themselves)
        part = (many ? to.many : to.few) - my_parts;
        mine = KIND == MERGE ? n_seg > 1 : many == (KIND == MANY_ROWS);
        return {__builtin_amdgcn_readlane(to.few, 63), __builtin_amdgcn_readlane(to.many, 63)};
    }
    __device__ __forceinline__ void fill(int o, int b, int from_end, int seg, Item *it) const
    {
        auto of = [&](int v) { return __builtin_amdgcn_readlane(v, o); };
        it->b = b;
        it->s = {of(s.s0), of(s.n), of(s.L), of(s.keys)};
        it->n_seg = of(n_seg);
        it->rows = 32 * of(blocks);
        it->rt = of(rt) - 1 - from_end;
        it->seg = seg;
        it->part = of(part) + (it->rt * it->n_seg + seg) * of(blocks);
    }
    // Item number idx; false: there are fewer.  Sequence by sequence (their row tiles share keys and values), the last rows, which see the most keys, first.
    __device__ __forceinline__ bool find(const ChunkParams &p, int idx, int lane, Item *it) const
    {
        ItemList l = *this;
        int items = 0;
        Parts behind = parts;
        for (int b0 = 0;;) {
            const int per = KIND == MERGE ? 1 : l.n_seg, my_items = l.mine ? l.rt * per : 0, items_to = items + wave_running_sum(my_items);
            const unsigned long long found = __ballot(items_to > idx);
            if (found) {
                const int o = __ffsll((long long)found) - 1, local = idx - __builtin_amdgcn_readlane(items_to - my_items, o), n = __builtin_amdgcn_readlane(per, o);
                const int from_end = uniform(local / n);
                l.fill(o, b0 + o, from_end, local - from_end * n, it);
                return true;
            }
            items = __builtin_amdgcn_readlane(items_to, 63);
            b0 += 64;
            if (b0 >= p.B) return false;
            l.s = {0, 0, 0, 0};
            if (b0 + lane < p.B) l.s = chunk_sequence(p, b0 + lane);
            behind = l.count(p, behind);
        }
    }
};

template <ItemKind KIND>
__device__ __forceinline__ bool find_item(const ChunkParams &p, int idx, int lane, Item *it)
{
    return ItemList<KIND>(p, lane).find(p, idx, lane, it);
}

__device__ __forceinline__ u32x4 finite_or_zero(u32x4 v, bool f32, bool *bad)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t e_lo = f32 ? 0u : 0x00007f80u, e_hi = 0x7f800000u;
        const bool hi = (v[i] & e_hi) == e_hi, lo = !f32 && (v[i] & e_lo) == e_lo;
        *bad |= hi | lo;
        if (f32) v[i] = hi ? 0u : v[i];
        else v[i] = (hi ? 0u : v[i] & 0xffff0000u) | (lo ? 0u : v[i] & 0xffffu);
    }
    return v;
}

// bf16, d = 128, sequences of more than p.many rows (chunk_wide.hip)
void launch_chunk_wide(const ChunkParams &p, int max_items, hipStream_t stream);

// A tile of 32 rows of DP (padded head dimension) values in LDS, pitches in words.
//   K  read 16 bytes a lane, lanes 0..31 in 32 rows: a pitch of 4 x an odd number spreads 16 lanes over the 64 banks.
//   V  bf16, transposing reads of 4 rows x 16 words: a pitch of 16 or 48 modulo 64 keeps the rows apart.
//      fp32, rows 4 apart read 32 words each: a pitch of 8 modulo 16 puts them 32 banks apart.
template <int DP, bool F32>
struct TileShape {
    static constexpr int ES = F32 ? 4 : 2, ROW_WORDS = DP * ES / 4, GRANULES = ROW_WORDS / 4;
    static constexpr int PK = ROW_WORDS + 4;
    static constexpr int PV = F32 ? ROW_WORDS + 8 : ROW_WORDS + (ROW_WORDS % 64 == 16 || ROW_WORDS % 64 == 48 ? 0 : 16);
    static constexpr int PER_THREAD = (KT * GRANULES + 255) / 256;       // 16-byte pieces of a tile per thread of 256
    static constexpr int KK = DP / (F32 ? 8 : 16);                       // 16-byte operand pieces a lane holds of a row
};

// scores of 32 keys x 32 rows, of KK 16-byte pieces of them: s = K Q^T, K from LDS rows at `k` (this lane's row and half), q this lane's row in registers.
// Score i of a lane is key 8 (i / 4) + 4 h + i % 4 of row lane % 32, h = lane / 32.  (bf16: the pieces of a lane are the operands of
// v_mfma_f32_32x32x16_bf16; fp32: v_mfma_f32_32x32x2_f32 takes the contraction four values of a piece after the other)
template <int KK, bool F32>
__device__ __forceinline__ f32x16 tile_scores(const uint32_t *k, const u32x4 *q)
{
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        const u32x4 a = *reinterpret_cast<const u32x4 *>(k + 8 * kk);
        if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(q[kk][j]), s, 0, 0, 0);
        } else {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, q[kk]), s, 0, 0, 0);
        }
    }
    return s;
}

// key of score i inside a tile, without the lane's 4 h
__device__ __forceinline__ constexpr int key_of_score(int i) { return 8 * (i >> 2) + (i & 3); }

}  // namespace mcsd
