// Tree attention (Sec. 3.3 of the paper) over a paged prefix cache held in 4 bits, on the matrix cores
// of gfx950.
//
//   attn_fourbit_kernel          up to 32 query rows per KV head (16 for d > 128; more of them in tiles): a (sequence, KV head, row tile, segment of the keys) per workgroup
//   attn_fourbit_shared_kernel   d = 128, more rows: tiles of 64 or 128 that share their keys
//   attn_fourbit_combine_kernel  merges the segments of a sequence by log-sum-exp
//
// Keys in tiles of 32.  S^T = K Q^T leaves a lane with 8 scores of one query row, which is the B operand
// of O^T += V^T P^T, so that the weights never leave their lane (as in tree_attn_any.hip).  A lane loads
// a quarter of a key's row, which for d = 128 is one block, 16 bytes and one scale: in the order of the
// layout a wavefront's load is 1 KB without a gap.  The contraction over d runs in the order in
// which the lanes then hold it (Q is read to match), so that K goes from memory to the
// matrix cores through the converters alone, without LDS.  V has to be transposed: converted, stored to
// LDS as rows and read back with the transposing load.
//
// Measured (inputs that take turns, d = 128, by the tracer): single tokens, 32 sequences of 100 to 8000 keys, 32 heads over 8: 39.4 us for 146 MB, 3.7 TB/s (32 us and
// 4.5 TB/s where part of it is still in a cache; 6.2 per further byte), bound by memory and the launch's ends: segments of 10 to 90 tiles, by sequence.  16 sequences of 256
// to 4096 keys, 32 heads, 60 nodes: 74 us for 197 MB, 2.7 TB/s and 0.51 PFLOP/s.  4 sequences of 16384, 64 heads over 8, 84 nodes: 226 us, 0.80 PFLOP/s.  These
// two are bound by the instructions between the products: matrix instructions 29 and 37 % of the cycles, vector ones 49 and 48 %, and a wavefront's are not
// free of each other (products of a step without softmax, conversions or V's reads: 47 to 50 of 53 us for 4096 keys more).
#include <algorithm>
#include <type_traits>

#include "attn_common.h"
#include "fourbit.h"

namespace mcsd {
namespace {

struct FourbitParams : AttnParams {
    const uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
    int n_blocks;           // d / 32
    int n_seg_max;
    int min_seg, whole;     // tiles of a segment at least; of a sequence that stays whole at most
    int units;              // row tiles x KV heads: workgroups of a segment
    float units_per_target, bias;   // units / workgroups aimed at; see find_segment
    uint32_t G_magic;       // r / G = r G_magic >> 32 for the rows there are
};

// How the tiles of all sequences are cut: a sequence of T tiles into max(1, T / chunk + bias) segments, with chunk so that there are
// as many workgroups as aimed at, by the real lengths (a cache's capacity says little about them).  Where the sequences are enough by themselves
// (bias 0), at most 64, and their segments more than one per CU, these are numbered longest first, and if all of them fit the chip at once (two per CU) the second 256
// shortest first: the hardware deals them out one per CU in order, so that a long one shares its CU with a short one.  Otherwise they go by sequence.
// A wavefront works this out for itself, its lanes take a sequence each.
struct Segment { int b, L, n, first, i; };       // sequence, its length, its segments, the number of its first one, which of them

__device__ __forceinline__ int lane_sum(int v, int lane, int *all)
{
    const int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    *all = __builtin_amdgcn_readlane(v, 63);
    return v - x;
}

__device__ __forceinline__ int length_of(const FourbitParams &p, int b) { return b < p.B ? max(0, min(p.prefix_len[b], p.L_stride)) : 0; }

__device__ __forceinline__ int tiles_of(const FourbitParams &p, int b, int L) { return b < p.B ? (L + KT - 1) / KT + p.tiles_tree : 0; }

// 1 / chunk; L0: the length of sequence `lane`.  (In floating point: a rounding moves a cut by a tile.)
__device__ __forceinline__ float cuts_per_tile(const FourbitParams &p, int L0, int lane)
{
    int total = 0, all;
    lane_sum(tiles_of(p, lane, L0), lane, &total);
    for (int b0 = 64; b0 < p.B; b0 += 64) {
        lane_sum(tiles_of(p, b0 + lane, length_of(p, b0 + lane)), lane, &all);
        total += all;
    }
    const int chunk = max(p.min_seg, (int)fminf(ceilf((float)total * p.units_per_target), 1e9f));
    return 1.0f / (float)chunk;
}

// Segments of sequence b, of T tiles.
__device__ __forceinline__ int segments_of(const FourbitParams &p, int b, int T, float per_tile)
{
    return b < p.B ? (T <= p.whole ? 1 : max(1, min(p.n_seg_max, (int)((float)T * per_tile + p.bias)))) : 0;
}

// Where segments are numbered by length: the number of the first of this lane's n, of T tiles together.  (The condition stands where it is asked: as a
// function's it becomes another schedule of the loops behind it, d 64 3 % slower.)
__device__ __forceinline__ int first_by_length(const FourbitParams &p, int T, int n, int lane)
{
    // tiles of a segment and the lane, as one number: the segments of all sequences with a larger one come before this one's
    const int key = (T / max(n, 1) << 6) | (63 - lane);
    int at = 0;
    for (int j = 0; j < p.B; ++j) at += __builtin_amdgcn_readlane(key, j) > key ? __builtin_amdgcn_readlane(n, j) : 0;
    return at;
}

// The segment of number `index`; numbers past the last one: none.
__device__ __forceinline__ Segment find_segment(const FourbitParams &p, int index, int lane)
{
    Segment s = {-1, 0, 0, 0, 0};
    if (p.n_seg_max == 1 && (p.B > 64 || p.bias != 0.f || p.B * p.units <= 256)) {
        s.b = index; s.L = length_of(p, index); s.n = 1; s.first = index;
        return s;
    }
    int L = length_of(p, lane), before = 0, all;
    const float per_tile = cuts_per_tile(p, L, lane);
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        if (b0 > 0) L = length_of(p, b0 + lane);
        const int T = tiles_of(p, b0 + lane, L), n = segments_of(p, b0 + lane, T, per_tile);
        int at = before + lane_sum(n, lane, &all);
        int wanted = index;
        if (p.B <= 64 && p.bias == 0.f && all * p.units > 256) {
            at = first_by_length(p, T, n, lane);
            const int half = 256 / p.units;
            if (all * p.units <= 512 && index >= half) wanted = all - 1 - (index - half);
            if (index >= all) wanted = -1;
        }
        const unsigned long long hit = __ballot(n > 0 && wanted >= at && wanted < at + n);
        if (hit) {
            const int l = __ffsll((long long)hit) - 1;
            s.b = b0 + l;
            s.L = __builtin_amdgcn_readlane(L, l);
            s.n = __builtin_amdgcn_readlane(n, l);
            s.first = __builtin_amdgcn_readlane(at, l);
            s.i = wanted - s.first;
            return s;
        }
        before += all;
    }
    return s;
}

// Node of query row r of a KV head, and where that row's output lies.
__device__ __forceinline__ int row_node(const FourbitParams &p, int r) { return p.G == 1 ? r : (int)__umulhi((uint32_t)r, p.G_magic); }

__device__ __forceinline__ uint16_t *row_out(const FourbitParams &p, int b, int g, int r)
{
    const int node = row_node(p, r);
    return static_cast<uint16_t *>(p.out) + (((size_t)b * p.N + node) * p.H_q + (size_t)g * p.G + (r - node * p.G)) * (size_t)p.d;
}

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef v4i16 __attribute__((address_space(3))) *lds_v4i16_ptr;

// Eight codes of a block -> eight bf16.
__device__ __forceinline__ u32x4 decode8(uint32_t c, float s)
{
    return (u32x4){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3))};
}

// All bits set, or none, as bit i of `keys` is (a comparison per key would be a mask in two scalar registers, and there are none left).
__device__ __forceinline__ uint32_t all_of(uint32_t keys, int i) { return (uint32_t)((int)(keys << (31 - i)) >> 31); }

// Weights of NS parts of 16 keys with the running maximum as it stands, tested by their sum: only where that is large (or the first
// scores come) the maximum is looked for and raised.  keys_of(mt, s): the keys of part s that count for the lane's row, the
// lowest four bits (MASKED; a masked score can not be told by its value where scale is 0).  Weights enter PV as TERMS bf16 terms each, their
// sum is of the unrounded ones.  As in the framework's attention over caches of full precision: one at d = 128, at most 2^-8 of the weight off, two at
// other d (the nearest bf16 and the nearest to what it leaves; what is not a number never meets them, see finite_of), at most 2^-17 off.  What the second
// costs, us with one (more than 32 rows: 128 together) / two (32 together, see variant_of): d 64, one token, 32 x 8 heads of 100-8000 keys 27.2 / 28.8; 16 x 8
// of 28 rows 20.2 / 22.3; 16 x 32 of 60 55.5 / 59.2; 8 x 8 of 84 27.9 / 24.7; 4 x 8 of 336 rows and 8000 keys 48.2 / 58.9, 2 x 8 of 672 and 16000 73.7 / 96.0; d 96,
// one token 18.5 / 19.5, 16 x 16 of 60 48.0 / 48.5, 4 x 8 of 336 76.0 / 92.4.  At d = 128 16 x 32 of 60 rows would be 70.5 / 87.1.
template <int DP, int RT, int NS, int TERMS, bool MASKED, typename KeysOf>
__device__ __forceinline__ void fourbit_softmax(float c2, const f32x4 (&sacc)[NS][RT], u32x2 (&pw)[TERMS][NS][RT], f32x4 (&oacc)[DP / 16][RT], float (&m_used)[RT],
                                                float (&l_part)[RT], KeysOf keys_of)
{
    float sum[RT];
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int mt = 0; mt < RT; ++mt) {
            sum[mt] = 0.f;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                float pv[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) pv[i] = fast_exp2(fmaf(sacc[s][mt][i], c2, -m_used[mt]));
                if (MASKED) {
                    const uint32_t keys = keys_of(mt, s);
#pragma unroll
                    for (int i = 0; i < 4; ++i) pv[i] = __uint_as_float(__float_as_uint(pv[i]) & all_of(keys, i));
                }
                sum[mt] += (pv[0] + pv[1]) + (pv[2] + pv[3]);
                const u32x2 hi = {pack_bf16(pv[0], pv[1]), pack_bf16(pv[2], pv[3])};
                pw[0][s][mt] = hi;
                if constexpr (TERMS == 2) {
                    float lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) lo[i] = pv[i] - __uint_as_float(i & 1 ? hi[i / 2] & 0xffff0000u : hi[i / 2] << 16);
                    pw[1][s][mt] = (u32x2){pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3])};
                }
            }
        }
    };
    weights();
    bool raise = false;
#pragma unroll
    for (int mt = 0; mt < RT; ++mt) raise |= sum[mt] > 4096.f;
    if (__any(raise)) {
#pragma unroll
        for (int mt = 0; mt < RT; ++mt) {
            float rm = -INFINITY;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const uint32_t keys = MASKED ? keys_of(mt, s) : 15u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t of = MASKED ? all_of(keys, i) : ~0u;
                    rm = fmaxf(rm, __uint_as_float((__float_as_uint(sacc[s][mt][i]) & of) | (0xff800000u & ~of)));
                }
            }
            rm = rm == -INFINITY ? rm : rm * c2;
            rm = fmaxf(rm, __shfl_xor(rm, 16));
            rm = fmaxf(rm, __shfl_xor(rm, 32));
            const float m_new = fmaxf(m_used[mt], rm);
            const float alpha = fast_exp2(m_used[mt] - m_new);
            m_used[mt] = m_new;
            l_part[mt] *= alpha;
#pragma unroll
            for (int nt = 0; nt < DP / 16; ++nt) oacc[nt][mt] *= alpha;
        }
        weights();
    }
#pragma unroll
    for (int mt = 0; mt < RT; ++mt) l_part[mt] += sum[mt];
}

// O^T += V^T P^T of a tile: V as rows in LDS, read back transposed; the weights of its two parts are 2 j and 2 j + 1 of pw.
template <int DP, int RT, int NS, int TERMS>
__device__ __forceinline__ void fourbit_values(const uint32_t *v, int lj, int lc, const u32x2 (&pw)[TERMS][NS][RT], int j, f32x4 (&oacc)[DP / 16][RT])
{
    constexpr int PV = DP / 2 + 8;
    const uint32_t *vl = v + (4 * lj + (lc >> 2)) * PV + (lc & 3) * 2;
#pragma unroll
    for (int nt = 0; nt < DP / 16; ++nt) {
        const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(vl + nt * 8));
        const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(vl + 16 * PV + nt * 8));
        const bf16x8 vop = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int term = 0; term < TERMS; ++term)
#pragma unroll
            for (int mt = 0; mt < RT; ++mt) {
                const u32x2 w0 = pw[term][2 * j][mt], w1 = pw[term][2 * j + 1][mt];
                const u32x4 w = {w0[0], w0[1], w1[0], w1[1]};
                oacc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, __builtin_bit_cast(bf16x8, w), oacc[nt][mt], 0, 0, 0);
            }
    }
}

// Values of a node that are no numbers (padding of a tree may hold them) would reach, as 0 times NaN, the rows that may not see the
// node: they enter the products as zeros, and finish adds them to the rows that see it, whatever its weight.  Bit 16 h + 15 of `odd`: half
// h of a word was one.  (In whole words: an exponent of all ones carries into its half's top bit.)
__device__ __forceinline__ u32x4 finite_of(u32x4 x, uint32_t *odd)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t top = ((x[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
        x[i] &= ~(top | (top - (top >> 15)));
        *odd |= top;
    }
    return x;
}

// Rows of the lanes with a bit set, a lane's row being its number % 16.
__device__ __forceinline__ uint32_t rows_with(uint32_t bits)
{
    const unsigned long long b = __ballot(bits != 0u);
    const uint32_t h = (uint32_t)b | (uint32_t)(b >> 32);
    return (h | h >> 16) & 0xffffu;
}

// The end of both kernels, 16 rows of every row group at a time: the key streams leave (m, l) and O in LDS (4 x 16 rows) and are added up
// behind a barrier; a sequence in one segment is written out, others leave their partials in the workspace.  s_odd: nodes of this
// segment's tree tiles with values that are no numbers.
template <int DP, int RT, int RG>
__device__ __forceinline__ void finish(const FourbitParams &p, const Segment &my, int g, int row_tile0, int tid, uint32_t *words, float (*s_m)[16], float (*s_l)[16],
                                       const uint32_t (*s_anc)[4], const uint32_t *s_odd, const f32x4 (&oacc)[DP / 16][RT], const float (&m_used)[RT], const float (&l_part)[RT])
{
    constexpr int KS = 4 / RG, NNT = DP / 16, PO = DP + 4;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lj = lane >> 4, lc = lane & 15, b = my.b;
    float *area = reinterpret_cast<float *>(words);
#pragma unroll
    for (int mt = 0; mt < RT; ++mt) {
        float lt = l_part[mt];
        lt += __shfl_xor(lt, 16);
        lt += __shfl_xor(lt, 32);
        __syncthreads();
        if (lj == 0) { s_m[wave][lc] = m_used[mt]; s_l[wave][lc] = lt; }
#pragma unroll
        for (int nt = 0; nt < NNT; ++nt) *reinterpret_cast<f32x4 *>(area + (wave * 16 + lc) * PO + 16 * nt + 4 * lj) = oacc[nt][mt];
        __syncthreads();
        const uint32_t any_odd = s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3];
        const uint16_t *v_tree = static_cast<const uint16_t *>(p.v_tree) + ((size_t)b * p.H_kv + g) * p.N * p.d;
        // (a thread has the same four columns of several rows)
        constexpr int D4 = DP / 4, RSTEP = 256 / D4;
        const int d4 = tid % D4;
#pragma unroll 2
        for (int r0 = 0; r0 < 16 * RG; r0 += RSTEP) {
            const int r16 = r0 + tid / D4, grp = r16 >> 4, r = r16 & 15;
            const int gr = row_tile0 + 16 * RT * grp + 16 * mt + r;
            if (gr >= p.M || 4 * d4 >= p.d) continue;
            float ms = s_m[grp][r], ls = 0.f;
#pragma unroll
            for (int k = 1; k < KS; ++k) ms = fmaxf(ms, s_m[k * RG + grp][r]);
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int w = k * RG + grp;
                const float f = fast_exp2(s_m[w][r] - ms);
                ls += f * s_l[w][r];
                acc += f * *reinterpret_cast<const f32x4 *>(area + (w * 16 + r) * PO + 4 * d4);
            }
            if (__builtin_amdgcn_readfirstlane(any_odd) != 0u)
#pragma unroll 1
                for (int i = 0; i < MCSD_MAX_NODES / KT; ++i)
                    for (uint32_t seen = s_odd[i] & s_anc[row_node(p, gr)][i]; seen != 0u; seen &= seen - 1u) {
                        const int node = i * KT + __ffs((int)seen) - 1;
                        const u32x2 v = *reinterpret_cast<const u32x2 *>(v_tree + (uint32_t)(node * p.d + 4 * d4));
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t x = c & 1 ? v[c / 2] & 0xffff0000u : v[c / 2] << 16;
                            acc[c] += __uint_as_float(x & (uint32_t)((int)((x & 0x7f800000u) + 0x00800000u) >> 31));
                        }
                    }
            if (my.n == 1) {
                const float inv = 1.0f / ls;
                __builtin_nontemporal_store((u32x2){pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)}, reinterpret_cast<u32x2 *>(row_out(p, b, g, gr) + 4 * d4));
            } else {
                const size_t u = ((size_t)(my.first + my.i) * p.H_kv + g) * (size_t)p.R + gr;
                __builtin_nontemporal_store(acc, reinterpret_cast<f32x4 *>(p.part_o + u * p.d + 4 * d4));
                if (d4 == 0) { p.part_m[u] = ms; p.part_l[u] = ls; }
            }
        }
    }
}

// DP: d padded to 64, 128 or 256.  Up to 16 RT query rows (d != 128: a row tile of as many), all of them by every wavefront, which takes every fourth tile
// and needs no barrier in its loop.
template <int DP, int RT, int TERMS>
__global__ __launch_bounds__(256, 2)
void attn_fourbit_kernel(FourbitParams p)
{
    constexpr int KS = 4, STEP = KS;                // key streams, tiles per step
    constexpr int NST = DP == 256 ? 1 : 2;          // steps asked for ahead
    constexpr int NR = DP == 256 ? 2 : 1;           // runs of columns a lane holds of a key's row
    constexpr int RUN = DP / 4 / NR;                // columns per run: 16, 32, 32
    constexpr int NKK = DP / 32, NNT = DP / 16;
    constexpr int W = RUN / 8;                      // words of codes per run
    typedef uint32_t u32xW __attribute__((ext_vector_type(W)));
    constexpr int PV = DP / 2 + 8;                  // row pitch of V in LDS, words
    constexpr int TILE_WORDS = KT * PV, OUT_WORDS = 4 * 16 * (DP + 4);

    __shared__ __attribute__((aligned(16))) uint32_t s_big[KS * TILE_WORDS > OUT_WORDS ? KS * TILE_WORDS : OUT_WORDS];
    __shared__ uint32_t s_anc[MCSD_MAX_NODES][4];
    __shared__ int s_parent[MCSD_MAX_NODES];
    __shared__ float s_m[4][16], s_l[4][16];
    __shared__ uint32_t s_odd[MCSD_MAX_NODES / KT + 1];

    const int tid = threadIdx.x, lane = tid & 63;
    const int ks = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lj = lane >> 4, lc = lane & 15;
    const int g = blockIdx.x, row0 = TERMS == 2 ? 16 * RT * (int)blockIdx.y : 0;
    const Segment my = find_segment(p, blockIdx.z, lane);
    const int b = my.b, L = my.L;
    if (b < 0) return;
    const int tiles_prefix = (L + KT - 1) / KT, T = tiles_prefix + p.tiles_tree;
    // (whole steps, so that the last segments may have no tile: their partials are without weight)
    const int seg = (int)(((uint32_t)(T + my.n - 1) / (uint32_t)my.n + STEP - 1) / STEP * STEP);
    const int t_begin = min(T, my.i * seg), t_end = min(T, t_begin + seg);

    const int my_parent = parent_of_thread(p, b);

    // First of the eight columns that a lane holds in part kk of the contraction: its runs are [RUN lj, RUN lj + RUN) (DP = 256:
    // of each half of the row).
    auto run_col = [&](int kk) __attribute__((always_inline)) { return NR == 2 ? 128 * (kk / 4) + 32 * lj + 8 * (kk % 4) : RUN * lj + 8 * kk; };
    bf16x8 qreg[RT][NKK];
#pragma unroll
    for (int mt = 0; mt < RT; ++mt) {
        const int r = row0 + 16 * mt + lc;
        const int rr = min(r, p.M - 1), node = row_node(p, rr), hh = rr - node * p.G;
        const uint16_t *src = static_cast<const uint16_t *>(p.q) + (((size_t)b * p.N + node) * p.H_q + (size_t)g * p.G + hh) * (size_t)p.d;
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
            u32x4 v = {0u, 0u, 0u, 0u};
            if (r < p.M && run_col(kk & ~3) < p.d) v = *reinterpret_cast<const u32x4 *>(src + run_col(kk));     // (d ends with a run)
            qreg[mt][kk] = __builtin_bit_cast(bf16x8, v);
        }
    }
    if (tid <= MCSD_MAX_NODES / KT) s_odd[tid] = 0u;
    build_ancestor_masks(p, my_parent, s_anc, s_parent);
    __syncthreads();

    f32x4 oacc[NNT][RT];
    float m_used[RT], l_part[RT];
#pragma unroll
    for (int mt = 0; mt < RT; ++mt) {
        m_used[mt] = M_INIT;
        l_part[mt] = 0.f;
#pragma unroll
        for (int nt = 0; nt < NNT; ++nt) oacc[nt][mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const float c2 = p.scale_log2;

    u32x2 pw[TERMS][2][RT];
    f32x4 sacc[2][RT];
    uint32_t *const vt = s_big + ks * TILE_WORDS;
    auto scores = [&](int s, auto k_of) __attribute__((always_inline)) {
#pragma unroll
        for (int mt = 0; mt < RT; ++mt) sacc[s][mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
            const bf16x8 k = k_of(kk);
#pragma unroll
            for (int mt = 0; mt < RT; ++mt) sacc[s][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qreg[mt][kk], sacc[s][mt], 0, 0, 0);
        }
    };
    auto softmax = [&](auto masked, auto keys_of) __attribute__((always_inline)) {
        fourbit_softmax<DP, RT, 2, TERMS, decltype(masked)::value>(c2, sacc, pw, oacc, m_used, l_part, keys_of);
    };
    auto values = [&]() __attribute__((always_inline)) { fourbit_values<DP, RT>(vt, lj, lc, pw, 0, oacc); };

    // Codes and scales of a wavefront's tiles of the next NST steps are on their way while it works on the present one.  The
    // block-table entries of 64 of them are read at once, a lane each (an entry read by itself ahead of its use was
    // sunk down to it, a trip to memory per step).  A column past d reads the last block (Q is zero there, and V's
    // columns are not written).
    const int32_t *table = p.block_table + (size_t)b * p.max_pages;
    u32xW kraw[NST][2][NR], vraw[NST][2][NR];
    uint32_t ksc[NST][2][NR], vsc[NST][2][NR];
    int blk[NST];
    uint32_t block_of[NR];
#pragma unroll
    for (int run = 0; run < NR; ++run) block_of[run] = min(DP == 64 ? lj >> 1 : 4 * run + lj, p.n_blocks - 1) * FB_TILE + lc;
    const int t_prefix = min(t_end, tiles_prefix);
    int t = t_begin + ks, t_ask = t;                // the tile worked on next, and the one asked for next
    int row_ask = t_ask * KT % p.page_size;
    const int row_step = STEP * KT % p.page_size;
    auto look_up = [&]() __attribute__((always_inline)) { return table[min((t_ask + lane * STEP) * KT / p.page_size, p.max_pages - 1)]; };
    int entries = look_up(), n_asked = 0;
    // (Unconditional: behind a branch the compiler would wait for everything that is on its way.  Past the end, and for a page that
    // is none, page 0 is read and not used.)
    auto request = [&](auto stage) __attribute__((always_inline)) {
        constexpr int S = decltype(stage)::value;
        const int e = __builtin_amdgcn_readlane(entries, n_asked);
        blk[S] = e;
        const size_t first = (((size_t)(t_ask < t_prefix && (unsigned)e < (unsigned)p.n_pages ? e : 0) * p.H_kv + g) * p.page_size + row_ask) * p.n_blocks;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int run = 0; run < NR; ++run) {
                const uint32_t block = block_of[run] + s * p.n_blocks * FB_TILE, byte = block * 16 + (DP == 64 ? 8 * (lj & 1) : 0);
                kraw[S][s][run] = *reinterpret_cast<const u32xW *>(p.k_codes + first * 16 + byte);
                ksc[S][s][run] = (p.k_scales + first)[block];
                vraw[S][s][run] = *reinterpret_cast<const u32xW *>(p.v_codes + first * 16 + byte);
                vsc[S][s][run] = (p.v_scales + first)[block];
            }
        t_ask += STEP;
        row_ask += row_step;
        if (row_ask >= p.page_size) row_ask -= p.page_size;
        if (++n_asked == 64) {
            n_asked = 0;
            entries = look_up();
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(entries));
        }
    };
    // rows from `keep` on hold anything, and those of a page that is none were read from another: they take part as zeros
    auto zero_from = [&](int keep, auto stage) __attribute__((always_inline)) {
        constexpr int S = decltype(stage)::value;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int run = 0; run < NR; ++run)
                if (16 * s + lc >= keep) {
                    kraw[S][s][run] = (u32xW)(0u);
                    vraw[S][s][run] = (u32xW)(0u);
                    ksc[S][s][run] = vsc[S][s][run] = 127u;
                }
    };
    // K into the products, V as rows into LDS
    auto convert = [&](auto stage) __attribute__((always_inline)) {
        constexpr int S = decltype(stage)::value;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int run = 0; run < NR; ++run)
#pragma unroll
                for (int w = 0; w < W; ++w)
                    *reinterpret_cast<u32x4 *>(vt + (16 * s + lc) * PV + run_col(run * 4 + w) / 2) = decode8(vraw[S][s][run][w], fourbit_scale(vsc[S][s][run]));
#pragma unroll
        for (int s = 0; s < 2; ++s)
            scores(s, [&](int kk) __attribute__((always_inline)) { return __builtin_bit_cast(bf16x8, decode8(kraw[S][s][kk / 4][kk % 4], fourbit_scale(ksc[S][s][kk / 4]))); });
    };
    // ---- whole prefix tiles
    const int t_plain = min(t_end, L / KT);
    auto plain = [&](auto stage) __attribute__((always_inline)) {
        if ((unsigned)blk[decltype(stage)::value] >= (unsigned)p.n_pages) zero_from(0, stage);
        convert(stage);
        request(stage);
        softmax(std::false_type(), [](int, int) __attribute__((always_inline)) { return 15u; });
        values();
        t += STEP;
    };
    // ---- the others: the end of the prefix and the tree block, bf16
    auto any = [&](auto stage) __attribute__((always_inline)) {
        const int left = L - t * KT;
        uint32_t vis[RT];               // keys that count for the lane's rows
        if (t < t_prefix) {
            zero_from((unsigned)blk[decltype(stage)::value] < (unsigned)p.n_pages ? left : 0, stage);
            convert(stage);
            request(stage);
#pragma unroll
            for (int mt = 0; mt < RT; ++mt) vis[mt] = left >= KT ? ~0u : (1u << (left & 31)) - 1u;
        } else {
            const size_t head = ((size_t)b * p.H_kv + g) * p.N;
            uint32_t odd = 0u;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int node = (t - tiles_prefix) * KT + 16 * s + lc;
                auto of_tree = [&](const void *from, int kk) __attribute__((always_inline)) {
                    u32x4 x = {0u, 0u, 0u, 0u};
                    if (node < p.N && run_col(kk & ~3) < p.d) x = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(from) + (head + node) * p.d + run_col(kk));
                    return x;
                };
                uint32_t bits = 0u;
#pragma unroll
                for (int kk = 0; kk < NKK; ++kk) *reinterpret_cast<u32x4 *>(vt + (16 * s + lc) * PV + run_col(kk) / 2) = finite_of(of_tree(p.v_tree, kk), &bits);
                odd |= rows_with(bits) << (16 * s);
                scores(s, [&](int kk) __attribute__((always_inline)) { return __builtin_bit_cast(bf16x8, of_tree(p.k_tree, kk)); });
            }
            s_odd[t - tiles_prefix] = odd;              // (all lanes the same)
#pragma unroll
            for (int mt = 0; mt < RT; ++mt) vis[mt] = s_anc[row_node(p, min(row0 + 16 * mt + lc, p.M - 1))][t - tiles_prefix];
        }
        softmax(std::true_type(), [&](int mt, int s) __attribute__((always_inline)) { return vis[mt] >> (16 * s + 4 * lj); });
        values();
        t += STEP;
    };
    typedef std::integral_constant<int, 0> stage0;
    typedef std::integral_constant<int, NST - 1> stage1;
    request(stage0());
    __builtin_amdgcn_sched_barrier(0);          // (the order in which they are waited for)
    if (NST > 1) request(stage1());
    __builtin_amdgcn_sched_barrier(0);
    while (t + (NST - 1) * STEP < t_plain) {
        plain(stage0());
        if (NST > 1) plain(stage1());
    }
    while (t < t_end) {
        any(stage0());
        if (NST > 1 && t < t_end) any(stage1());
    }
    finish<DP, RT, 1>(p, my, g, row0, tid, s_big, s_m, s_l, s_anc, s_odd, oacc, m_used, l_part);
}

// 16 or 4 bytes per lane from base + offset straight into LDS, lane after lane from byte `to` on.  No register is written.  Written as text
// because behind the builtin the compiler waits for everything on its way ahead of every read of LDS; who reads what arrives has counted
// down vmcnt to it and passed a barrier (the counts are at begin_step).
__device__ __forceinline__ void fetch16(uint32_t to, const uint8_t *base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(to), "v"(offset), "s"(base) : "memory", "m0");
}

__device__ __forceinline__ void fetch4(uint32_t to, const uint8_t *base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(to), "v"(offset), "s"(base) : "memory", "m0");
}

// d = 128, more than 32 query rows: RG row groups of 16 RT rows share their keys.  Wavefront (rg, ks) of the four owns rows [16 RT rg, 16 RT (rg + 1)) of
// the workgroup's and, RG = 2, key stream ks (one tile of the two of a step) or, RG = 4, both tiles.
//   - Codes and scales go from memory straight into a ring of DEPTH steps in LDS (a wavefront asks for K or V of one of the two tiles), so
//     that three steps are on their way without a register: with two steps in registers a launch that reads from memory took the
//     sum of its loads and its arithmetic.
//   - A wavefront converts the K that it multiplies by itself (conversions run beside matrix instructions), and a quarter of the step's V, as
//     rows in LDS for the transposing load.
//   - PV runs a step behind the scores: the one barrier of a step then stands between both the codes' arrival and their
//     readers, and the V of the last step and its readers.
template <int RT, int RG>
__global__ __launch_bounds__(256, 2)
void attn_fourbit_shared_kernel(FourbitParams p)
{
    constexpr int DP = 128, ROWS = 16 * RT * RG, STEP = 2, DEPTH = 4;
    constexpr int TPS = RG / 2, SUBK = 2 * TPS;     // tiles, and 16-key parts, that a wavefront multiplies per step
    constexpr int RUN = DP / 4, W = RUN / 8;        // columns a lane holds of a key's row, words of their codes
    constexpr int NB = DP / FB_BLOCK, NKK = DP / 32, NNT = DP / 16;
    typedef uint32_t u32xW __attribute__((ext_vector_type(W)));
    constexpr int PV = DP / 2 + 8, PO = DP + 4;     // row pitches of V in LDS and of the epilogue, words
    constexpr int NLOAD = DP / 64;                  // 1 KB pieces of a tile's codes
    constexpr int CODE_WORDS = KT * DP / 8, SCALE_WORDS = 64;       // of a tile's K or V in the ring
    constexpr int SIDE_WORDS = CODE_WORDS + SCALE_WORDS, RING_WORDS = 4 * SIDE_WORDS;
    constexpr int TILE_WORDS = KT * PV, VBUF_WORDS = STEP * TILE_WORDS;
    constexpr int MAIN_WORDS = DEPTH * RING_WORDS + 2 * VBUF_WORDS, OUT_WORDS = 4 * 16 * PO;
    static_assert(RG == 2 || RG == 4, "row groups");

    __shared__ __attribute__((aligned(16))) uint32_t s_big[MAIN_WORDS > OUT_WORDS ? MAIN_WORDS : OUT_WORDS];
    __shared__ uint32_t s_anc[MCSD_MAX_NODES][4];
    __shared__ int s_parent[MCSD_MAX_NODES];
    __shared__ float s_m[4][16], s_l[4][16];
    __shared__ uint32_t s_odd[MCSD_MAX_NODES / KT + 1];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rg = wave % RG, ks = wave / RG;
    const int lj = lane >> 4, lc = lane & 15;
    const int g = blockIdx.x, row_tile0 = blockIdx.y * ROWS, row0 = row_tile0 + 16 * RT * rg;
    const Segment my = find_segment(p, blockIdx.z, lane);
    const int b = my.b, L = my.L;
    if (b < 0) return;
    const int tiles_prefix = (L + KT - 1) / KT, T = tiles_prefix + p.tiles_tree;
    // (whole steps, so that the last segments may have no tile: their partials are without weight)
    const int seg = (int)(((uint32_t)(T + my.n - 1) / (uint32_t)my.n + STEP - 1) / STEP * STEP);
    const int t_begin = min(T, my.i * seg), t_end = min(T, t_begin + seg), t_prefix = min(t_end, tiles_prefix);
    const int my_parent = parent_of_thread(p, b);

    // ---- requests.  This wavefront's: K (even) or V (odd) of tile wave / 2 of a step.  The block-table entries of 64 steps are read at once, a
    // lane each.  Past the end, and for a page that is none, page 0 is read and not used: every step asks for as much, so that what is
    // waited for can be counted.
    const int32_t *table = p.block_table + (size_t)b * p.max_pages;
    const uint8_t *const my_codes = wave & 1 ? p.v_codes : p.k_codes, *const my_scales = wave & 1 ? p.v_scales : p.k_scales;
    int t_ask = t_begin + (wave >> 1), row_ask = t_ask * KT % p.page_size, n_asked = 0, slot_ask = 0;
    const int row_step = STEP * KT % p.page_size;
    auto look_up = [&]() __attribute__((always_inline)) { return table[min((t_ask + lane * STEP) * KT / p.page_size, p.max_pages - 1)]; };
    int entries = look_up();
    uint32_t code_off[NLOAD];
#pragma unroll
    for (int i = 0; i < NLOAD; ++i) code_off[i] = 16u * (64 * i + lane);
    const uint32_t scale_off = 4u * min(lane, 8 * NB - 1);
    const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint32_t *)s_big;
    auto request = [&]() __attribute__((always_inline)) {
        const int e = __builtin_amdgcn_readlane(entries, n_asked);
        const size_t first = (((size_t)(t_ask < t_prefix && (unsigned)e < (unsigned)p.n_pages ? e : 0) * p.H_kv + g) * p.page_size + row_ask) * NB;
        const uint8_t *codes = my_codes + first * 16, *scales = my_scales + first;
        const uint32_t to = ring_at + 4u * (slot_ask * RING_WORDS + wave * SIDE_WORDS);
#pragma unroll
        for (int i = 0; i < NLOAD; ++i) fetch16(to + 1024 * i, codes, code_off[i]);
        fetch4(to + 4 * CODE_WORDS, scales, scale_off);
        t_ask += STEP;
        row_ask += row_step;
        if (row_ask >= p.page_size) row_ask -= p.page_size;
        slot_ask = (slot_ask + 1) % DEPTH;
        if (++n_asked == 64) {
            n_asked = 0;
            entries = look_up();
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(entries) :: "memory");
        }
    };
    // a page that is none among the segment's: all of its steps then look at every entry
    bool bad_pages = false;
    for (int e = t_begin * KT / p.page_size + lane; e * p.page_size < t_prefix * KT; e += 64) bad_pages |= (unsigned)table[e] >= (unsigned)p.n_pages;
    const bool any_bad = __any(bad_pages);
    const int t_plain = any_bad ? t_begin : min(t_end, L / KT);
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(entries) :: "memory");
#pragma unroll
    for (int s = 0; s < DEPTH - 1; ++s) request();

    // First of the eight columns that a lane holds in part kk of the contraction.
    auto run_col = [&](int kk) __attribute__((always_inline)) { return RUN * lj + 8 * kk; };
    bf16x8 qreg[RT][NKK];
#pragma unroll
    for (int mt = 0; mt < RT; ++mt) {
        const int r = row0 + 16 * mt + lc;
        const int rr = min(r, p.M - 1), node = row_node(p, rr), hh = rr - node * p.G;
        const uint16_t *src = static_cast<const uint16_t *>(p.q) + (((size_t)b * p.N + node) * p.H_q + (size_t)g * p.G + hh) * (size_t)DP;
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
            u32x4 v = {0u, 0u, 0u, 0u};
            if (r < p.M) v = *reinterpret_cast<const u32x4 *>(src + run_col(kk));
            qreg[mt][kk] = __builtin_bit_cast(bf16x8, v);
        }
    }
    if (tid <= MCSD_MAX_NODES / KT) s_odd[tid] = 0u;
    build_ancestor_masks(p, my_parent, s_anc, s_parent);

    f32x4 oacc[NNT][RT];
    float m_used[RT], l_part[RT];
#pragma unroll
    for (int mt = 0; mt < RT; ++mt) {
        m_used[mt] = M_INIT;
        l_part[mt] = 0.f;
#pragma unroll
        for (int nt = 0; nt < NNT; ++nt) oacc[nt][mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const float c2 = p.scale_log2;
    const bool active = row0 < p.M;
    // where the lane's codes of part `s` (of a tile's K or V) lie in the ring, in words behind that side; its scale byte behind CODE_WORDS
    int code_at[2], scale_at[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int block = (s * NB + lj) * FB_TILE + lc;
        code_at[s] = block * 4;
        scale_at[s] = CODE_WORDS * 4 + block;
    }
    auto codes_in = [&](const uint32_t *side, int s) __attribute__((always_inline)) { return *reinterpret_cast<const u32xW *>(side + code_at[s]); };
    auto scale_in = [&](const uint32_t *side, int s) __attribute__((always_inline)) {
        return fourbit_scale(reinterpret_cast<const uint8_t *>(side)[scale_at[s]]);
    };
    uint32_t *const vbuf = s_big + DEPTH * RING_WORDS;
    const int my_tile = RG == 4 ? 0 : ks;                   // the wavefront's first tile of a step
    const int v_row = 16 * (wave & 1) + lc;                 // its row of V in tile wave / 2

    // (the first step has none before it: weights and V of zeros)
    u32x2 pw[1][SUBK][RT];
#pragma unroll
    for (int term = 0; term < 1; ++term)
#pragma unroll
        for (int s = 0; s < SUBK; ++s)
#pragma unroll
            for (int mt = 0; mt < RT; ++mt) pw[term][s][mt] = (u32x2){0u, 0u};
    for (int i = tid; i < VBUF_WORDS / 4; i += 256) reinterpret_cast<u32x4 *>(vbuf + VBUF_WORDS)[i] = (u32x4){0u, 0u, 0u, 0u};
    f32x4 sacc[SUBK][RT];
    // O^T += V^T P^T of the last step
    auto values = [&](const uint32_t *v) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < TPS; ++j) fourbit_values<DP, RT>(v + (my_tile + j) * TILE_WORDS, lj, lc, pw, j, oacc);
    };
    auto scores = [&](int s, auto k_of) __attribute__((always_inline)) {
#pragma unroll
        for (int mt = 0; mt < RT; ++mt) sacc[s][mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
            const bf16x8 k = k_of(kk);
#pragma unroll
            for (int mt = 0; mt < RT; ++mt) sacc[s][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qreg[mt][kk], sacc[s][mt], 0, 0, 0);
        }
    };
    auto softmax = [&](auto masked, auto keys_of) __attribute__((always_inline)) {
        fourbit_softmax<DP, RT, SUBK, 1, decltype(masked)::value>(c2, sacc, pw, oacc, m_used, l_part, keys_of);
    };

    // (Everything asked for so far is there; said through the builtin, so that the compiler knows it of its own loads and puts no wait for
    // them, which would be one for the ring as well, into the loops.)
    __builtin_amdgcn_s_waitcnt(0x0f70);         // vmcnt(0)
    int t0 = t_begin, slot = 0, buf = 0;
    // the codes of this step are there for all wavefronts, and the V rows of the last one; the ring's oldest place is free again
    auto begin_step = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0)" :: "n"((DEPTH - 2) * (NLOAD + 1)) : "memory");
        __syncthreads();
        request();
    };
    auto end_step = [&]() __attribute__((always_inline)) {
        t0 += STEP;
        slot = (slot + 1) % DEPTH;
        buf ^= 1;
    };
    for (; t0 + STEP <= t_plain; end_step()) {
        begin_step();
        const uint32_t *ring = s_big + slot * RING_WORDS;
        const uint32_t *vside = ring + (wave | 1) * SIDE_WORDS;
        uint32_t *const vrow = vbuf + buf * VBUF_WORDS + (wave >> 1) * TILE_WORDS + v_row * PV;
        // (One run of instructions, everything read from LDS ahead of what is written to it: the products of the last step beside the
        // conversions of this one.)
        u32xW kc[SUBK];
        float ksc[SUBK];
        const u32xW vc = codes_in(vside, wave & 1);
        const float vsc = scale_in(vside, wave & 1);
        auto convert_v = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int w = 0; w < W; ++w) *reinterpret_cast<u32x4 *>(vrow + run_col(w) / 2) = decode8(vc[w], vsc);
        };
        if (!active) {
            convert_v();
            continue;
        }
#pragma unroll
        for (int s = 0; s < SUBK; ++s) {
            const uint32_t *kside = ring + 2 * (my_tile + s / 2) * SIDE_WORDS;
            kc[s] = codes_in(kside, s & 1);
            ksc[s] = scale_in(kside, s & 1);
        }
        values(vbuf + (buf ^ 1) * VBUF_WORDS);
        convert_v();
#pragma unroll
        for (int s = 0; s < SUBK; ++s)
            scores(s, [&](int kk) __attribute__((always_inline)) { return __builtin_bit_cast(bf16x8, decode8(kc[s][kk], ksc[s])); });
        softmax(std::false_type(), [](int, int) __attribute__((always_inline)) { return 15u; });
    }
    // ---- the other steps: the end of the prefix and the tree block, bf16
    for (; t0 < t_end; end_step()) {
        begin_step();
        int t1 = t0;            // (hidden from the compiler: it would keep what depends on it in scalar registers from step to step, and there are none)
        asm volatile("" : "+s"(t1));
        const uint32_t *ring = s_big + slot * RING_WORDS;
        if (active) values(vbuf + (buf ^ 1) * VBUF_WORDS);
        const size_t head = ((size_t)b * p.H_kv + g) * p.N;
        auto of_tree = [&](const void *from, int node, int kk) __attribute__((always_inline)) {
            u32x4 x = {0u, 0u, 0u, 0u};
            if (node < p.N) x = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(from) + (head + node) * DP + run_col(kk));
            return x;
        };
        // rows of a prefix tile that there are (none of a page that is none); the others hold anything and take part as zeros
        auto rows_of = [&](int t) __attribute__((always_inline)) {
            if (any_bad && (unsigned)__builtin_amdgcn_readfirstlane(table[t * KT / p.page_size]) >= (unsigned)p.n_pages) return 0;
            return L - t * KT;
        };
        const int tv = t1 + (wave >> 1);
        uint32_t *vrow = vbuf + buf * VBUF_WORDS + (wave >> 1) * TILE_WORDS + v_row * PV;
        if (tv < t_prefix) {
            const uint32_t *vside = ring + (wave | 1) * SIDE_WORDS;
            const bool off = v_row >= rows_of(tv);
            const u32xW c = codes_in(vside, wave & 1);
            const float sc = scale_in(vside, wave & 1);
#pragma unroll
            for (int w = 0; w < W; ++w) *reinterpret_cast<u32x4 *>(vrow + run_col(w) / 2) = decode8(off ? 0u : c[w], off ? 1.f : sc);
        } else {
            const int node = tv < t_end ? (tv - tiles_prefix) * KT + v_row : p.N;
            uint32_t bits = 0u;
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) *reinterpret_cast<u32x4 *>(vrow + run_col(kk) / 2) = finite_of(of_tree(p.v_tree, node, kk), &bits);
            const uint32_t odd = rows_with(bits);
            reinterpret_cast<uint16_t *>(s_odd)[2 * (tv - tiles_prefix) + (wave & 1)] = (uint16_t)odd;        // (all lanes the same; past t_end: one tile, zeros)
        }
        if (active) {
#pragma unroll
            for (int s = 0; s < SUBK; ++s) {
                const int t = t1 + my_tile + s / 2;
                bf16x8 k[NKK];
                if (t < t_prefix) {
                    const uint32_t *kside = ring + 2 * (my_tile + s / 2) * SIDE_WORDS;
                    const bool off = 16 * (s & 1) + lc >= rows_of(t);
#pragma unroll
                    for (int kk = 0; kk < NKK; ++kk)
                        k[kk] = __builtin_bit_cast(bf16x8, decode8(off ? 0u : codes_in(kside, s & 1)[kk], off ? 1.f : scale_in(kside, s & 1)));
                } else {
#pragma unroll
                    for (int kk = 0; kk < NKK; ++kk) k[kk] = __builtin_bit_cast(bf16x8, of_tree(p.k_tree, t < t_end ? (t - tiles_prefix) * KT + 16 * (s & 1) + lc : p.N, kk));
                }
                scores(s, [&](int kk) __attribute__((always_inline)) { return k[kk]; });
            }
            uint32_t vis[TPS][RT];          // keys of a tile that count for the lane's rows
#pragma unroll
            for (int j = 0; j < TPS; ++j)
#pragma unroll
                for (int mt = 0; mt < RT; ++mt) {
                    const int t = t1 + my_tile + j, left = L - t * KT;
                    vis[j][mt] = t >= t_end ? 0u : (t < t_prefix ? (left >= KT ? ~0u : (1u << (left & 31)) - 1u)
                                                                 : s_anc[row_node(p, min(row0 + 16 * mt + lc, p.M - 1))][t - tiles_prefix]);
                }
            softmax(std::true_type(), [&](int mt, int s) __attribute__((always_inline)) { return vis[s / 2][mt] >> (16 * (s & 1) + 4 * lj); });
        }
    }
    __syncthreads();
    if (active) values(vbuf + (buf ^ 1) * VBUF_WORDS);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // (nothing may still be on its way into what follows)

    finish<DP, RT, RG>(p, my, g, row_tile0, tid, s_big, s_m, s_l, s_anc, s_odd, oacc, m_used, l_part);
}

// out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  Bound by the launch and two trips to memory: 4.0 us for the single tokens above, 3.9 where nothing is
// cut and 12.4 for 45 MB of partials.  A thread per four columns of a row, ROWS rows of a (sequence, KV head) at a time per workgroup.
template <int DP>
__device__ __forceinline__ void merge_row(const FourbitParams &p, int b, int n_seg, int first, int g, int r, int d4)
{
    const size_t u0 = ((size_t)first * p.H_kv + g) * (size_t)p.R + r, step = (size_t)p.H_kv * p.R;
    float ms = M_INIT, ls = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    // eight segments at a time, all of them requested before the first is used (those past the end are the first again, without weight)
    for (int s0 = 0; s0 < n_seg; s0 += 8) {
        float m[8], l[8];
        f32x4 o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool on = s0 + i < n_seg;
            const size_t u = u0 + (on ? s0 + i : 0) * step;
            m[i] = on ? p.part_m[u] : M_INIT;
            l[i] = on ? p.part_l[u] : 0.f;
            o[i] = *reinterpret_cast<const f32x4 *>(p.part_o + u * p.d + 4 * d4);
        }
        float m_new = ms;
#pragma unroll
        for (int i = 0; i < 8; ++i) m_new = fmaxf(m_new, m[i]);
        const float keep = fast_exp2(ms - m_new);
        ls *= keep;
        acc *= keep;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float f = s0 + i < n_seg ? fast_exp2(m[i] - m_new) : 0.f;
            ls += f * l[i];
            acc += f * o[i];
        }
        ms = m_new;
    }
    const float inv = 1.0f / ls;
    __builtin_nontemporal_store((u32x2){pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)}, reinterpret_cast<u32x2 *>(row_out(p, b, g, r) + 4 * d4));
}

// Units of ROWS rows of a KV head of the sequences that are cut: a workgroup each or, LOOP, dealt out among fewer (the loop around it takes registers: 672 rows
// of 8 KV heads and 4 sequences in eight parts 12.1 us, 13.0 with it).
template <int DP, bool LOOP>
__global__ __launch_bounds__(256) void attn_fourbit_combine_kernel(FourbitParams p)
{
    constexpr int D4 = DP / 4, ROWS = 256 / D4;
    const int lane = threadIdx.x & 63, d4 = threadIdx.x % D4;
    const int groups = (p.M + ROWS - 1) / ROWS, per_sequence = groups * p.H_kv;
    int unit = blockIdx.x, before = 0, all;         // unit: counted from the first cut sequence of the 64 that are looked at
    const float per_tile = cuts_per_tile(p, length_of(p, lane), lane);
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int T = tiles_of(p, b0 + lane, length_of(p, b0 + lane)), n = segments_of(p, b0 + lane, T, per_tile);
        int at = before + lane_sum(n, lane, &all);
        if (p.B <= 64 && p.bias == 0.f && all * p.units > 256) at = first_by_length(p, T, n, lane);
        before += all;
        unsigned long long cut = __ballot(n > 1);
        int passed = 0;                             // cut sequences ahead of the first that `cut` still holds
        const int units = __popcll(cut) * per_sequence;
        while (unit < units) {
            const int k = unit / per_sequence, in = unit % per_sequence;
            for (; passed < k; ++passed) cut &= cut - 1;
            const int l = __ffsll((long long)cut) - 1, r = in % groups * ROWS + threadIdx.x / D4;
            const int n_seg = __builtin_amdgcn_readlane(n, l), first = __builtin_amdgcn_readlane(at, l);
            if (r < p.M && 4 * d4 < p.d) merge_row<DP>(p, b0 + l, n_seg, first, in / groups, r, d4);
            if (!LOOP) return;
            unit += gridDim.x;
        }
        unit -= units;
    }
}

size_t round_256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

// Variants of the kernel: 16-row tiles per wavefront and row groups (1: rows do not share keys in LDS).
// d = 128: 32 rows together / shared: 16 x 32 heads of 60 rows 77.8 / 71.4 us, 64 x 32 of 60 243 / 188, 4 x 8 of 672 rows and 16384 keys 249 / 222 and with 64 rows
// together 251, 4 x 32 of 1024 221 / 171; not so where there are few workgroups: 32 x 8 of 60 46.4 / 56.9, 16 x 8 of 128 43.8 / 66.9, short ones of 60 12.4 / 15.9.
// Other d, with two terms per weight: the shared forms have no registers for them (128 rows together: a wavefront per SIMD fewer at d = 64, spills at d = 96;
// one workgroup per CU at d > 128) and were behind tiles of 32 (16 for d > 128) whose workgroups read one behind the other from cache, d 64, 64 rows together / 32: 8 x 8 of 60
// rows 30.6 / 29.1, 16 x 32 of 60 64.5 / 59.2, 4 x 8 of 336 and 8000 keys 60.4 / 58.9, 4 x 32 of 1024 148 / 153; d 96, 16 x 16 of 60 57.3 / 48.5; d 256, 64 rows together /
// 16: 8 x 16 of 60 91.7 / 66.3, 8 x 4 of 112 59.7 / 40.5, 4 x 8 of 336 220 / 208, 4 x 32 of 1024 643 / 640; 32 rows together / 16: 16 x 4 of 28 41.4 / 31.8.
struct FourbitVariant { int rt, rg; };

static FourbitVariant variant_of(int rows, int d)
{
    if (rows <= 16 || d > 128) return {1, 1};
    if (rows <= 32 || d != 128) return {2, 1};
    return rows <= 64 ? FourbitVariant{2, 2} : FourbitVariant{2, 4};
}

bool make_fourbit_plan(const mcsd_attn_desc &d, FourbitPlan *plan)
{
    FourbitPlan f = {};
    const int rows = d.N + d.root_row;
    if (d.H_kv > 65535 || (long)rows * (d.H_q / d.H_kv) > (1 << 20)) return false;      // (grids and row counts)
    f.rows_per_kv = rows * (d.H_q / d.H_kv);
    const FourbitVariant v = variant_of(f.rows_per_kv, d.d);
    f.row_tile = 16 * v.rt * v.rg;
    f.n_row_tiles = (f.rows_per_kv + f.row_tile - 1) / f.row_tile;
    if ((long)f.rows_per_kv * (d.H_q / d.H_kv) >= 0x7fffffffL || f.n_row_tiles > 65535) return false;
    const long units = (long)d.H_kv * f.n_row_tiles;
    const int tiles = (d.L_stride + KT - 1) / KT + (rows + KT - 1) / KT;
    // Workgroups aimed at.  Enough sequences for two workgroups per CU: cut only what is twice as long as the average.  Fewer: two, three or four
    // per CU, whichever leaves the fullest CU with the fewest tiles if the sequences are alike, ceil(workgroups / 256) / segments of
    // each (4 sequences of 16384 keys, 48 workgroups a segment: 256, 512, 768, 1024 aimed at 369, 294, 229, 233 us; one of 16000, 32 a segment:
    // 512 39, 768 46 us with the merge).  The line between the two, fewer / enough: 8 heads of 60 rows, 32 sequences of 2000 keys each 61.8 / 71.0, 40 66.4 / 61.7,
    // 55 59.6 / 63.9; of 100 to 4000 keys 32 55.7 / 49.7, 55 87 / 72, 60 86 / 74, 80 110 / 108, 128 158 / 149; one row, of 2000 each 56 31.8 / 38.1, 80 52.6 / 45.3; of
    // 100 to 4000 32 26.5 / 29.4, 48 36.9 / 40.0, 64 46.8 / 46.7.
    const long base = units * d.B;
    const bool enough = base >= 448;
    f.target = 512;
    f.bias = enough ? 0.f : 0.5f;
    double least = 1e30;
    for (long k = 2; k <= 4 && !enough; ++k) {
        const long n = std::max(1L, (256 * k + base / 2) / base);
        const double cost = (double)((base * n + 255) / 256) / (double)n;
        if (cost < least * 0.999) { least = cost; f.target = (int)(256 * k); }
    }
    // A merge is a launch of 4 us, which a sequence of few steps does not earn: 1 x 12 heads of 64, one row, whole / in two: 517 keys 5.9 / 8.9, 1000
    // 7.7 / 9.3, 2000 11.4 / 9.1; 32 heads, 60 rows: 517 17.4 / 17.7, 1000 20.5 / 16.8.  2 x 8 heads of 128, one row: 700 8.7 / 11.4, 1500 12.3 / 11.4.  A
    // tile of d > 128 takes twice as long: 2 x 4 heads of 256, one row, 400 keys 10.8 whole; 1000 17.4 whole, 14.6 in two; 2000 16.1 in pieces of 16 tiles, 14.1 in pieces of 8.
    f.min_seg = (v.rg == 1 ? 16 : 8) / (d.d > 128 ? 2 : 1);
    f.whole = (v.rg == 1 ? 40 : 20) / (d.d > 128 ? 2 : 1);
    // (beyond 512 sequences they fill the chip by themselves, and every workgroup would look through all lengths)
    if (tiles <= f.whole || d.B > 512) f.target = 1;
    f.n_segments_max = (int)std::max(1L, std::min((long)(tiles / f.min_seg), f.target / units));
    // Segments of all sequences: n = max(1, T / chunk + bias), with chunk >= all tiles units / target
    f.n_segments = f.n_segments_max == 1 ? d.B : (int)std::min((long)d.B * f.n_segments_max, f.target / units + 1 + d.B);
    if (f.n_segments > 65535) return false;
    if (f.n_segments_max > 1) {
        const size_t partials = (size_t)f.n_segments * d.H_kv * f.n_row_tiles * f.row_tile;
        f.ws_bytes = round_256(partials * d.d * 4) + 2 * round_256(partials * 4);
    }
    *plan = f;
    return true;
}

int32_t launch_attn_fourbit(const mcsd_attn_desc &d, const mcsd_attn_bufs &b, const mcsd_fourbit_kv &kv, const FourbitPlan &plan, hipStream_t stream)
{
    FourbitParams p = {};
    p.q = b.q; p.k_tree = b.k_tree; p.v_tree = b.v_tree; p.prefix_len = b.prefix_len; p.parent = b.parent; p.out = b.out;
    p.B = d.B; p.N = d.N + d.root_row; p.H_q = d.H_q; p.H_kv = d.H_kv; p.G = d.H_q / d.H_kv; p.d = d.d; p.L_stride = d.L_stride;
    p.M = plan.rows_per_kv; p.n_row_tiles = plan.n_row_tiles; p.parent_per_seq = d.parent_per_seq; p.root_row = d.root_row;
    p.tiles_tree = (p.N + KT - 1) / KT;
    p.scale_log2 = d.scale * LOG2E_F;
    p.block_table = kv.block_table; p.page_size = kv.page_size; p.n_pages = kv.n_pages; p.max_pages = kv.max_pages_per_seq;
    p.k_codes = static_cast<const uint8_t *>(kv.k_codes); p.v_codes = static_cast<const uint8_t *>(kv.v_codes);
    p.k_scales = static_cast<const uint8_t *>(kv.k_scales); p.v_scales = static_cast<const uint8_t *>(kv.v_scales);
    p.n_blocks = d.d / FB_BLOCK;
    p.R = plan.n_row_tiles * plan.row_tile;
    p.n_seg_max = plan.n_segments_max; p.min_seg = plan.min_seg; p.whole = plan.whole; p.bias = plan.bias; p.units = d.H_kv * plan.n_row_tiles; p.units_per_target = (float)((double)d.H_kv * plan.n_row_tiles / plan.target);
    p.G_magic = p.G > 1 ? (uint32_t)((0x100000000ull + p.G - 1) / p.G) : 0u;
    if (plan.ws_bytes > 0) {
        const size_t partials = (size_t)plan.n_segments * d.H_kv * p.R;
        char *ws = static_cast<char *>(b.workspace);
        p.part_o = reinterpret_cast<float *>(ws);
        p.part_m = reinterpret_cast<float *>(ws + round_256(partials * d.d * 4));
        p.part_l = reinterpret_cast<float *>(ws + round_256(partials * d.d * 4) + round_256(partials * 4));
    }
    const dim3 grid(d.H_kv, plan.n_row_tiles, plan.n_segments);
    auto go = [&](auto kernel) { launch_kernel(K_ATTN_FOURBIT, kernel, grid, dim3(256), stream, p); };
    const FourbitVariant v = variant_of(plan.rows_per_kv, d.d);
    if (d.d > 128) {
        go(attn_fourbit_kernel<256, 1, 2>);
    } else if (d.d == 128) {
        if (v.rg == 4) go(attn_fourbit_shared_kernel<2, 4>);
        else if (v.rg == 2) go(attn_fourbit_shared_kernel<2, 2>);
        else if (v.rt == 2) go(attn_fourbit_kernel<128, 2, 1>);
        else go(attn_fourbit_kernel<128, 1, 1>);
    } else if (d.d > 64) {
        if (v.rt == 2) go(attn_fourbit_kernel<128, 2, 2>);
        else go(attn_fourbit_kernel<128, 1, 2>);
    } else {
        if (v.rt == 2) go(attn_fourbit_kernel<64, 2, 2>);
        else go(attn_fourbit_kernel<64, 1, 2>);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("attn_fourbit launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    if (plan.n_segments_max == 1) return MCSD_OK;
    // (Where sequences are cut only far beyond the average most or all are whole: no more workgroups than start at once, among which the rows of those that are
    // cut are dealt out.  16 x 32 heads of 60 rows, none cut: 3.9 us, with a workgroup per eight rows 7.6; one of 16000 keys among 15 of 300: 5.9, 9.4; 6
    // of 8000 among 54 of 500, 8 heads of 84 rows: 8.0; with the workgroups dealt to sequences instead, whole or not, 12.9 and 13.3.)
    auto merge = [&](auto whole, auto dealt, int rows) {
        const long units = (long)((p.M + rows - 1) / rows) * d.H_kv * d.B;
        const bool deal = plan.bias == 0.f && units > 1024;
        launch_kernel(K_ATTN_FOURBIT_COMBINE, deal ? dealt : whole, dim3((unsigned)(deal ? 1024 : units)), dim3(256), stream, p);
    };
    if (d.d > 128) merge(attn_fourbit_combine_kernel<256, false>, attn_fourbit_combine_kernel<256, true>, 4);
    else if (d.d > 64) merge(attn_fourbit_combine_kernel<128, false>, attn_fourbit_combine_kernel<128, true>, 8);
    else merge(attn_fourbit_combine_kernel<64, false>, attn_fourbit_combine_kernel<64, true>, 16);
    e = hipGetLastError();
    if (e != hipSuccess) { set_error("attn_fourbit_combine launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
