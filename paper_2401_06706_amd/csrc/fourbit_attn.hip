// Tree attention (Sec. 3.3 of the paper) over a paged prefix cache held in 4 bits, on the matrix cores
// of gfx950.
//
//   attn_fourbit_kernel          a (sequence, KV head, row tile, segment of the keys) per workgroup
//   attn_fourbit_combine_kernel  merges the segments of a sequence by log-sum-exp
//
// Keys in tiles of 32.  S^T = K Q^T leaves a lane with 8 scores of one query row, which is the B operand
// of O^T += V^T P^T, so that the weights never leave their lane (as in tree_attn_any.hip).  A lane loads
// a quarter of a key's row, which for d = 128 is one block, 16 bytes and one scale: in the order of the
// layout a wavefront's load is 1 KB without a gap.  The contraction over d runs in the order in
// which the lanes then hold it (Q is read to match), so that K goes from memory to the
// matrix cores through the converters alone, without LDS.  V has to be transposed: converted, stored to
// LDS as rows and read back with the transposing load.
#include <algorithm>

#include "attn_common.h"
#include "fourbit.h"

namespace mcsd {
namespace {

struct FourbitParams : AttnParams {
    const uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
    int n_blocks;           // d / 32
    int n_seg_max;
    int units;              // row tiles x KV heads
    int target;             // workgroups aimed at
};

constexpr int MIN_SEG = 8;      // tiles of a segment at least: two steps of four wavefronts

// Segments of a sequence of T tiles where all sequences have `total`: as many workgroups as aimed at, each a whole number
// of steps of the four wavefronts.
__device__ __forceinline__ void fourbit_segments(const FourbitParams &p, int T, long total, int *n, int *seg)
{
    const long chunk = max((long)MIN_SEG, (total * p.units + p.target - 1) / p.target);
    const int want = (int)min((long)p.n_seg_max, max(1L, (T + chunk / 2) / chunk));
    *seg = ((T + want - 1) / want + 3) & ~3;
    *n = (T + *seg - 1) / *seg;
}

// Tiles of all sequences, by every wavefront for itself.
__device__ __forceinline__ long total_tiles(const FourbitParams &p, int lane)
{
    long t = 0;
    for (int b = lane; b < p.B; b += 64) t += (max(0, min(p.prefix_len[b], p.L_stride)) + KT - 1) / KT + p.tiles_tree;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) t += __shfl_xor(t, o);
    return t;
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

// DP: d padded to 64, 128 or 256.  RT: 16-row tiles of query rows per wavefront; all four wavefronts have the same rows
// and every fourth tile.
template <int DP, int RT>
__global__ __launch_bounds__(256, 2)
void attn_fourbit_kernel(FourbitParams p)
{
    constexpr int ROWS = 16 * RT, KS = 4;
    constexpr int NR = DP == 256 ? 2 : 1;           // runs of columns a lane holds of a key's row
    constexpr int RUN = DP / 4 / NR;                // columns per run: 16, 32, 32
    constexpr int NKK = DP / 32, NNT = DP / 16;
    constexpr int W = RUN / 8;                      // words of codes per run
    typedef uint32_t u32xW __attribute__((ext_vector_type(W)));
    constexpr int PV = DP / 2 + 8;                  // row pitch of V in LDS, words
    constexpr int PO = DP + 4;                      // row pitch of the epilogue
    constexpr int TILE_WORDS = KT * PV;
    constexpr int AREA = TILE_WORDS > 16 * PO ? TILE_WORDS : 16 * PO;

    __shared__ __attribute__((aligned(16))) uint32_t s_big[KS * AREA];
    __shared__ uint32_t s_anc[MCSD_MAX_NODES][4];
    __shared__ int s_parent[MCSD_MAX_NODES];
    __shared__ float s_m[KS][16], s_l[KS][16];

    const int tid = threadIdx.x, lane = tid & 63;
    const int ks = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lj = lane >> 4, lc = lane & 15;
    const int g = blockIdx.x, b = blockIdx.z;
    const int segment = blockIdx.y / p.n_row_tiles, row0 = blockIdx.y % p.n_row_tiles * ROWS;

    const int L = max(0, min(p.prefix_len[b], p.L_stride));
    const int tiles_prefix = (L + KT - 1) / KT, T = tiles_prefix + p.tiles_tree;
    int n_seg = 1, seg = T;
    if (p.n_seg_max > 1) fourbit_segments(p, T, total_tiles(p, lane), &n_seg, &seg);
    n_seg = __builtin_amdgcn_readfirstlane(n_seg);
    seg = __builtin_amdgcn_readfirstlane(seg);
    if (segment >= n_seg) return;
    const int t_begin = segment * seg, t_end = min(T, t_begin + seg);

    const int my_parent = parent_of_thread(p, b);

    // column of word-run element (kk, i): lane lj holds runs [RUN lj, RUN lj + RUN) (DP = 256: of each half of the row)
    auto col0 = [&](int kk) __attribute__((always_inline)) { return NR == 2 ? 128 * (kk / 4) + 32 * lj + 8 * (kk % 4) : RUN * lj + 8 * kk; };
    bf16x8 qreg[RT][NKK];
#pragma unroll
    for (int mt = 0; mt < RT; ++mt) {
        const int r = row0 + 16 * mt + lc;
        const int rr = min(r, p.M - 1), node = rr / p.G, hh = rr % p.G;
        const uint16_t *src = static_cast<const uint16_t *>(p.q) + (((size_t)b * p.N + node) * p.H_q + (size_t)g * p.G + hh) * (size_t)p.d;
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
            u32x4 v = {0u, 0u, 0u, 0u};
            if (r < p.M && col0(kk) < p.d) v = *reinterpret_cast<const u32x4 *>(src + col0(kk));
            qreg[mt][kk] = __builtin_bit_cast(bf16x8, v);
        }
    }
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
    uint32_t *const vt = s_big + ks * AREA;

    // One tile whose operands are there: K in kop, V as rows in LDS.  vis_of(mt): the keys of the tile that count for the lane's row of
    // row tile mt, where `masked`.
    bf16x8 kop[2][NKK];
    auto tile_step = [&](const bool masked, auto vis_of) __attribute__((always_inline)) {
        f32x4 sacc[2][RT];
#pragma unroll
        for (int mt = 0; mt < RT; ++mt)
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
                sacc[sub][mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < NKK; ++kk)
                    sacc[sub][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[sub][kk], qreg[mt][kk], sacc[sub][mt], 0, 0, 0);
            }
        uint32_t vis[RT];
        float lmax[RT];
        bool raise = false;
#pragma unroll
        for (int mt = 0; mt < RT; ++mt) {
            settle_scores(sacc[0][mt], sacc[1][mt]);
            if (masked) {
                vis[mt] = vis_of(mt) >> (4 * lj);
#pragma unroll
                for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((vis[mt] >> (16 * sub + i)) & 1u)) sacc[sub][mt][i] = -INFINITY;
            }
            const float mr = max_of_scores(sacc[0][mt], sacc[1][mt]);
            lmax[mt] = (mr == -INFINITY) ? -INFINITY : mr * c2;
            raise |= lmax[mt] > m_used[mt] + RESCALE_GAP;
        }
        if (__any(raise)) {
#pragma unroll
            for (int mt = 0; mt < RT; ++mt) {
                float rm = lmax[mt];
                rm = fmaxf(rm, __shfl_xor(rm, 16));
                rm = fmaxf(rm, __shfl_xor(rm, 32));
                const float m_new = fmaxf(m_used[mt], rm);
                const float alpha = fast_exp2(m_used[mt] - m_new);
                m_used[mt] = m_new;
                l_part[mt] *= alpha;
#pragma unroll
                for (int nt = 0; nt < NNT; ++nt) oacc[nt][mt] *= alpha;
            }
        }
        bf16x8 pop[RT];
#pragma unroll
        for (int mt = 0; mt < RT; ++mt) {
            float pv[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) pv[e] = fast_exp2(fmaf(sacc[e >> 2][mt][e & 3], c2, -m_used[mt]));
            if (masked) {
                // (with scale == 0 a masked score can not be told apart by its value)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!((vis[mt] >> (16 * (e >> 2) + (e & 3))) & 1u)) pv[e] = 0.f;
            }
            l_part[mt] += ((pv[0] + pv[1]) + (pv[2] + pv[3])) + ((pv[4] + pv[5]) + (pv[6] + pv[7]));
            u32x4 ph;
#pragma unroll
            for (int j = 0; j < 4; ++j) ph[j] = pack_bf16(pv[2 * j], pv[2 * j + 1]);
            pop[mt] = __builtin_bit_cast(bf16x8, ph);
        }
        const uint32_t *vl = vt + (4 * lj + (lc >> 2)) * PV + (lc & 3) * 2;
#pragma unroll
        for (int nt = 0; nt < NNT; ++nt) {
            const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(vl + nt * 8));
            const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(vl + 16 * PV + nt * 8));
            const bf16x8 vop = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int mt = 0; mt < RT; ++mt) oacc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, pop[mt], oacc[nt][mt], 0, 0, 0);
        }
    };

    // ---- the prefix.  The codes of a wavefront's next tile are asked for before its present one is worked on, and the
    // block-table entry of the one behind that; page and row of it advance without a division.
    int t = t_begin + ks;
    const int t_prefix = min(t_end, tiles_prefix);
    if (t < t_prefix) {
        const int32_t *table = p.block_table + (size_t)b * p.max_pages;
        int page = (t * KT) / p.page_size, page_row = (t * KT) % p.page_size;
        const int page_step = KS * KT / p.page_size, row_step = KS * KT % p.page_size;
        auto entry = [&]() __attribute__((always_inline)) { return table[page]; };
        // codes and scales of the tile that starts at row page_row of page blk; a column past d reads the last block (Q is zero
        // there, and V's columns are not written)
        u32xW kraw[2][NR], vraw[2][NR];
        uint32_t ksc[2][NR], vsc[2][NR];
        uint32_t block_of[NR];
#pragma unroll
        for (int run = 0; run < NR; ++run) block_of[run] = min(DP == 64 ? lj >> 1 : 4 * run + lj, p.n_blocks - 1) * FB_TILE + lc;
        auto request = [&](int blk, int row) __attribute__((always_inline)) {
            const size_t tile0 = (((size_t)((unsigned)blk < (unsigned)p.n_pages ? blk : 0) * p.H_kv + g) * p.page_size + row) / FB_TILE;
            const size_t at = tile0 * p.n_blocks * FB_TILE;
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                for (int run = 0; run < NR; ++run) {
                    const uint32_t block = block_of[run] + sub * p.n_blocks * FB_TILE, byte = block * 16 + (DP == 64 ? 8 * (lj & 1) : 0);
                    kraw[sub][run] = *reinterpret_cast<const u32xW *>(p.k_codes + at * 16 + byte);
                    ksc[sub][run] = (p.k_scales + at)[block];
                    vraw[sub][run] = *reinterpret_cast<const u32xW *>(p.v_codes + at * 16 + byte);
                    vsc[sub][run] = (p.v_scales + at)[block];
                }
        };
        int blk = __builtin_amdgcn_readfirstlane(entry());
        request(blk, page_row);
        int next = 0, next_row = 0;
        auto look_up = [&](int t_next) __attribute__((always_inline)) {
            page += page_step;
            page_row += row_step;
            if (page_row >= p.page_size) { page_row -= p.page_size; ++page; }
            if (t_next < t_prefix) next = entry();
            next_row = page_row;
        };
        look_up(t + KS);
        for (; t < t_prefix; t += KS) {
            const int nvalid = L - t * KT;
            if (nvalid < KT || (unsigned)blk >= (unsigned)p.n_pages) {
                // rows past the end hold anything, and those of a page that is none were read from another: they take part as zeros
                const int keep = (unsigned)blk < (unsigned)p.n_pages ? nvalid : 0;
#pragma unroll
                for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                    for (int run = 0; run < NR; ++run)
                        if (16 * sub + lc >= keep) {
                            kraw[sub][run] = (u32xW)(0u);
                            vraw[sub][run] = (u32xW)(0u);
                            ksc[sub][run] = vsc[sub][run] = 127u;
                        }
            }
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                for (int run = 0; run < NR; ++run)
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        kop[sub][run * 4 + w] = __builtin_bit_cast(bf16x8, decode8(kraw[sub][run][w], fourbit_scale(ksc[sub][run])));
                        *reinterpret_cast<u32x4 *>(vt + (16 * sub + lc) * PV + col0(run * 4 + w) / 2) = decode8(vraw[sub][run][w], fourbit_scale(vsc[sub][run]));
                    }
            if (t + KS < t_prefix) {
                blk = __builtin_amdgcn_readfirstlane(next);
                request(blk, next_row);
                look_up(t + 2 * KS);
            }
            tile_step(nvalid < KT, [&](int) __attribute__((always_inline)) { return (1u << (nvalid & 31)) - 1u; });
        }
    }
    // ---- the tree block, bf16
    for (; t < t_end; t += KS) {
        const int node0 = (t - tiles_prefix) * KT;
        const size_t head = ((size_t)b * p.H_kv + g) * p.N;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            const int node = node0 + 16 * sub + lc;
            const size_t at = (head + min(node, p.N - 1)) * p.d;
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) {
                u32x4 ko = {0u, 0u, 0u, 0u}, vo = {0u, 0u, 0u, 0u};
                if (node < p.N && col0(kk) < p.d) {
                    ko = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p.k_tree) + at + col0(kk));
                    vo = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p.v_tree) + at + col0(kk));
                }
                kop[sub][kk] = __builtin_bit_cast(bf16x8, ko);
                *reinterpret_cast<u32x4 *>(vt + (16 * sub + lc) * PV + col0(kk) / 2) = vo;
            }
        }
        tile_step(true, [&](int mt) __attribute__((always_inline)) { return s_anc[min(row0 + 16 * mt + lc, p.M - 1) / p.G][t - tiles_prefix]; });
    }

    // ---- epilogue, 16 rows at a time: the wavefronts leave (m, l) and O in LDS and are added up behind a barrier
    float *area = reinterpret_cast<float *>(s_big);
    const int d4n = p.d / 4;
#pragma unroll
    for (int mt = 0; mt < RT; ++mt) {
        float lt = l_part[mt];
        lt += __shfl_xor(lt, 16);
        lt += __shfl_xor(lt, 32);
        __syncthreads();
        if (lj == 0) { s_m[ks][lc] = m_used[mt]; s_l[ks][lc] = lt; }
#pragma unroll
        for (int nt = 0; nt < NNT; ++nt) *reinterpret_cast<f32x4 *>(area + ks * AREA + lc * PO + 16 * nt + 4 * lj) = oacc[nt][mt];
        __syncthreads();
        const int first = row0 + 16 * mt, valid = min(16, p.M - first);
        for (int idx = tid; idx < valid * d4n; idx += 256) {
            const int r = idx / d4n, d4 = idx - r * d4n;
            float ms = s_m[0][r], ls = 0.f;
#pragma unroll
            for (int k = 1; k < KS; ++k) ms = fmaxf(ms, s_m[k][r]);
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const float f = fast_exp2(s_m[k][r] - ms);
                ls += f * s_l[k][r];
                acc += f * *reinterpret_cast<const f32x4 *>(area + k * AREA + r * PO + 4 * d4);
            }
            const int gr = first + r;
            if (n_seg == 1) {
                const float inv = 1.0f / ls;
                const int node = gr / p.G, hh = gr % p.G;
                uint16_t *ob = static_cast<uint16_t *>(p.out) + (((size_t)b * p.N + node) * p.H_q + (size_t)g * p.G + hh) * (size_t)p.d + 4 * d4;
                __builtin_nontemporal_store((u32x2){pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)}, reinterpret_cast<u32x2 *>(ob));
            } else {
                const size_t u = (((size_t)b * p.H_kv + g) * p.n_seg_max + segment) * (size_t)p.R + gr;
                __builtin_nontemporal_store(acc, reinterpret_cast<f32x4 *>(p.part_o + u * p.d + 4 * d4));
                if (d4 == 0) { p.part_m[u] = ms; p.part_l[u] = ls; }
            }
        }
    }
}

// A thread per four columns of a row.
__global__ __launch_bounds__(256) void attn_fourbit_combine_kernel(FourbitParams p)
{
    const int g = blockIdx.y, b = blockIdx.z;
    const int L = max(0, min(p.prefix_len[b], p.L_stride));
    int n_seg, seg;
    fourbit_segments(p, (L + KT - 1) / KT + p.tiles_tree, total_tiles(p, threadIdx.x & 63), &n_seg, &seg);
    if (n_seg == 1) return;
    const int d4n = p.d / 4, idx = blockIdx.x * 256 + threadIdx.x, r = idx / d4n, d4 = idx - r * d4n;
    if (r >= p.M) return;
    const size_t u0 = ((size_t)b * p.H_kv + g) * p.n_seg_max * (size_t)p.R + r;
    float ms = M_INIT, ls = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < n_seg; ++s) {
        const size_t u = u0 + (size_t)s * p.R;
        const float m = p.part_m[u], m_new = fmaxf(ms, m), keep = fast_exp2(ms - m_new), f = fast_exp2(m - m_new);
        ls = keep * ls + f * p.part_l[u];
        acc = keep * acc + f * *reinterpret_cast<const f32x4 *>(p.part_o + u * p.d + 4 * d4);
        ms = m_new;
    }
    const float inv = 1.0f / ls;
    const int node = r / p.G, hh = r % p.G;
    uint16_t *ob = static_cast<uint16_t *>(p.out) + (((size_t)b * p.N + node) * p.H_q + (size_t)g * p.G + hh) * (size_t)p.d + 4 * d4;
    __builtin_nontemporal_store((u32x2){pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)}, reinterpret_cast<u32x2 *>(ob));
}

size_t round_256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

bool make_fourbit_plan(const mcsd_attn_desc &d, FourbitPlan *plan)
{
    FourbitPlan f = {};
    const int rows = d.N + d.root_row;
    if (d.H_kv > 65535 || (long)rows * (d.H_q / d.H_kv) > (1 << 20)) return false;      // (grids and row counts)
    f.rows_per_kv = rows * (d.H_q / d.H_kv);
    f.row_tile = f.rows_per_kv <= 16 || d.d > 128 ? 16 : 32;      // (32 rows of 256 columns do not fit the registers)
    f.n_row_tiles = (f.rows_per_kv + f.row_tile - 1) / f.row_tile;
    const long units = (long)d.H_kv * f.n_row_tiles;
    const int tiles = (d.L_stride + KT - 1) / KT + (rows + KT - 1) / KT;
    long n = std::max(1L, std::min((long)(tiles + MIN_SEG - 1) / MIN_SEG, 1024 / units + 1));
    n = std::max(1L, std::min(n, 4096 / (units * d.B)));
    f.n_segments_max = (int)n;
    if (n * f.n_row_tiles > 65535) return false;
    if (n > 1) {
        const size_t partials = (size_t)d.B * d.H_kv * n * f.n_row_tiles * f.row_tile;
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
    p.n_seg_max = plan.n_segments_max; p.units = d.H_kv * plan.n_row_tiles; p.target = 1024;
    if (plan.ws_bytes > 0) {
        const size_t partials = (size_t)d.B * d.H_kv * plan.n_segments_max * p.R;
        char *ws = static_cast<char *>(b.workspace);
        p.part_o = reinterpret_cast<float *>(ws);
        p.part_m = reinterpret_cast<float *>(ws + round_256(partials * d.d * 4));
        p.part_l = reinterpret_cast<float *>(ws + round_256(partials * d.d * 4) + round_256(partials * 4));
    }
    const dim3 grid(d.H_kv, plan.n_segments_max * plan.n_row_tiles, d.B);
    auto go = [&](auto kernel) { launch_kernel(K_ATTN_FOURBIT, kernel, grid, dim3(256), stream, p); };
    const bool one = plan.row_tile == 16;
    if (d.d <= 64) { if (one) go(attn_fourbit_kernel<64, 1>); else go(attn_fourbit_kernel<64, 2>); }
    else if (d.d <= 128) { if (one) go(attn_fourbit_kernel<128, 1>); else go(attn_fourbit_kernel<128, 2>); }
    else go(attn_fourbit_kernel<256, 1>);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("attn_fourbit launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    if (plan.n_segments_max == 1) return MCSD_OK;
    launch_kernel(K_ATTN_FOURBIT_COMBINE, attn_fourbit_combine_kernel, dim3((p.M * (d.d / 4) + 255) / 256, d.H_kv, d.B), dim3(256), stream, p);
    e = hipGetLastError();
    if (e != hipSuccess) { set_error("attn_fourbit_combine launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
