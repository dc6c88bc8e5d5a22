// Attention of a chunk of new tokens over a paged cache (a prompt, a piece of one, a lone token; a batch mixes them), and the
// store of their keys and values into its pages.
#include <type_traits>

#include "chunk_common.h"

namespace mcsd {
namespace {

constexpr int OFF_NOWHERE = 0x7fff0000; // an offset beyond every buffer's extent: reads as zero

// softmax(scale Q K^T) V of a tile of rows over a segment of its keys, one pass: with a running maximum m, weights 2^(s c - m) and their
// sum l, o = sum w V; out = o / l, lse = (m + log2 l) ln 2, or (o, m, l) as a partial result.
// 32 keys at a time stand in LDS, two tiles more are on their way in registers.  Four wavefronts take 32 rows each; or (SPLIT) all take the same
// 32, form the scores together (fp32: a quarter of the contraction each, summed in a fixed order through LDS; bf16: all of them, which is
// cheaper) and the output a quarter of the columns each: a lone token's few rows then keep four matrix units busy, and its tiles leave
// registers for three workgroups a compute unit.
// A decoding batch is bound by the reading of its keys and values: 32 sequences of 100 to 8000 tokens, 32/8 heads, d = 128: 111 to 116 us, 4.7 to 4.9 TB/s.
template <int DP, bool F32, bool SPLIT, bool TWO_TERMS>      // TWO_TERMS: of the weights in PV, as in tree attention
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(F32 && DP == 256 ? 1 : 2)))
void chunk_attn_kernel(ChunkParams p)
{
    using S = TileShape<DP, F32>;
    constexpr int ROWS = SPLIT ? ROWS_SPLIT : ROWS_FEW, BUF_WORDS = KT * (S::PK + S::PV);
    constexpr int NT = SPLIT ? (DP / 32 + 3) / 4 : DP / 32;             // column tiles of a wavefront
    constexpr bool SHARE = SPLIT && F32;                                // the products of the scores are shared out too
    constexpr int KK = SHARE ? S::KK / 4 : S::KK;
    __shared__ __attribute__((aligned(16))) uint32_t s_tiles[(SHARE ? 1 : 2) * BUF_WORDS];
    __shared__ __attribute__((aligned(16))) float s_share[SHARE ? 4 : 1][4][64][4];
    __shared__ int s_bad;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, l32 = lane & 31, lj = lane >> 4, lc = lane & 15;
    const int in_head = uniform(blockIdx.x / p.H_kv), g = blockIdx.x - in_head * p.H_kv;        // (KV head fastest: the row tiles of one meet in one XCD's L2 where their number is a multiple of 8)
    Item it;
    const ItemList<FEW_ROWS> list(p, lane);
    if (p.notes && blockIdx.x == gridDim.x - 1) {           // (as a rule it has no item)
        const int len_many = p.max_parts_many ? list.many_segment(p, lane) : 0;
        if (tid == 0) *p.notes = {0, list.many, list.len, len_many};
    }
    if (!list.find(p, in_head, lane, &it)) return;
    const int M = it.s.n * p.G, row0 = it.rt * ROWS + (SPLIT ? 0 : 32 * wave);
    const int nt0 = SPLIT && NT * wave < DP / 32 ? NT * wave : 0, kk0 = SHARE ? KK * wave : 0;
    const bool writes = !SPLIT || NT * wave < DP / 32;          // (96 columns are three tiles)
    auto position = [&](int row) { return min(it.s.L + by_group(p, row), it.s.keys - 1); };
    const int kt = uniform(position(min(it.rt * ROWS + ROWS, M) - 1)) / KT + 1;           // key tiles that some row of this tile sees
    const int seg = uniform((kt + it.n_seg - 1) / it.n_seg), t_begin = it.seg * seg, t_end = min(kt, t_begin + seg);
    const int diagonal = (uniform(position(it.rt * ROWS)) + 1) / KT;                    // from this tile on there are keys that some row does not see
    const bool active = row0 < M;
    const int my_row = min(row0 + l32, M - 1), my_pos = position(my_row);
    // tiles that every row of this wavefront sees whole; tiles that any of them sees
    const int t_plain = active ? min(t_end, (uniform(position(row0)) + 1) / KT) : t_begin;
    const int t_seen = active ? min(t_end, uniform(position(min(row0 + 32, M) - 1)) / KT + 1) : t_begin;
    if (tid == 0) s_bad = 0;

    u32x4 q[KK];
    {
        const int token = by_group(p, my_row), head = g * p.G + my_row - token * p.G;
        const char *src = static_cast<const char *>(p.q) + (size_t)(it.s.s0 + token) * p.q_row + (size_t)head * p.d * S::ES;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            const int at = 32 * (kk0 + kk) + 16 * h;
            const u32x4 zero = {0, 0, 0, 0};
            q[kk] = DP * S::ES == 256 && p.d == DP ? *reinterpret_cast<const u32x4 *>(src + at)
                                                   : (at < p.d * S::ES ? *reinterpret_cast<const u32x4 *>(src + at) : zero);
        }
    }
    f32x16 o[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[nt][i] = 0.f;
    float m_used = M_INIT, l_part = 0.f;
    const float c2 = p.scale_log2;

    // ---- tiles: global -> registers -> LDS
    const int row_bytes = p.d * S::ES;
    uint32_t load_at[S::PER_THREAD], k_st[S::PER_THREAD], v_st[S::PER_THREAD];
#pragma unroll
    for (int j = 0; j < S::PER_THREAD; ++j) {
        const int e = tid + 256 * j, row = e / S::GRANULES, c = e % S::GRANULES;
        load_at[j] = e < KT * S::GRANULES && 16 * c < row_bytes ? row * row_bytes + 16 * c : OFF_NOWHERE;
        if (j && 256 % S::GRANULES == 0) load_at[j] = load_at[0] + j * (256 / S::GRANULES) * row_bytes;         // (the same column: one register holds them)
        k_st[j] = row * S::PK + 4 * c;
        v_st[j] = KT * S::PK + row * S::PV + 4 * c;
    }
    const const_i32_ptr table = (const_i32_ptr)(uintptr_t)(p.block_table + (size_t)it.b * p.max_pages);
    u32x4 kr[2][S::PER_THREAD], vr[2][S::PER_THREAD];
    // tiles are asked for one after the other, from t_begin on
    const int page_size = uniform(p.page_size);
    int entry = uniform(t_begin * KT / page_size), in_page = t_begin * KT - entry * page_size;
    auto load_kv = [&](int t, int st) __attribute__((always_inline)) {
        const int page = t < t_end ? (int)table[entry] : -1;
        const bool in = (unsigned)page < (unsigned)p.n_pages;
        const size_t off = in ? (((size_t)page * p.H_kv + g) * page_size + in_page) * row_bytes : 0;
        const uint32_t extent = in ? (uint32_t)max(0, min(KT, it.s.keys - t * KT)) * row_bytes : 0u;
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(static_cast<const char *>(p.k_pool) + off, extent);
        const __amdgpu_buffer_rsrc_t rv = make_rsrc(static_cast<const char *>(p.v_pool) + off, extent);
#pragma unroll
        for (int j = 0; j < S::PER_THREAD; ++j) {
            kr[st][j] = __builtin_amdgcn_raw_buffer_load_b128(rk, load_at[j], 0, 0);
            vr[st][j] = __builtin_amdgcn_raw_buffer_load_b128(rv, load_at[j], 0, 0);
        }
        in_page += KT;
        if (in_page == page_size) { in_page = 0; ++entry; }
    };
    bool bad = false;
    auto store_kv = [&](int t, uint32_t *buf, int st) __attribute__((always_inline)) {
        if (t >= diagonal && t < t_end) {
            // A weight of 0 times a value that is no number is none either: here, where rows do not see all keys, such values
            // enter the products as zeros and are added in the epilogue to the rows that see them.
#pragma unroll
            for (int j = 0; j < S::PER_THREAD; ++j) vr[st][j] = finite_or_zero(vr[st][j], F32, &bad);
        }
#pragma unroll
        for (int j = 0; j < S::PER_THREAD; ++j)
            if (KT * S::GRANULES % 256 == 0 || tid + 256 * j < KT * S::GRANULES) {
                *reinterpret_cast<u32x4 *>(buf + k_st[j]) = kr[st][j];
                *reinterpret_cast<u32x4 *>(buf + v_st[j]) = vr[st][j];
            }
    };
    const uint32_t k_ld = l32 * S::PK + 4 * h + 8 * kk0;
    const uint32_t v_ld = F32 ? KT * S::PK + 4 * h * S::PV + l32 + 32 * nt0
                              : KT * S::PK + (4 * h + (lc >> 2)) * S::PV + 8 * (lj & 1) + 2 * (lc & 3) + 16 * nt0;
    typedef short v4i16 __attribute__((ext_vector_type(4)));
    typedef v4i16 __attribute__((address_space(3))) *lds_v4i16_ptr;

    auto compute = [&](int t, const uint32_t *cb, auto masked_tag) __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(masked_tag)::value;
        f32x16 s = tile_scores<KK, F32>(cb + k_ld, q);
        if constexpr (SHARE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(s_share[wave][i][lane]) = make_float4(s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]);
            __syncthreads();            // (what is read here has been read by all before the next step's first barrier)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float4 x = *reinterpret_cast<const float4 *>(s_share[0][i][lane]);
#pragma unroll
                for (int w = 1; w < 4; ++w) {
                    const float4 y = *reinterpret_cast<const float4 *>(s_share[w][i][lane]);
                    x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
                }
                s[4 * i] = x.x; s[4 * i + 1] = x.y; s[4 * i + 2] = x.z; s[4 * i + 3] = x.w;
            }
        }
        const int seen = my_pos - t * KT - 4 * h;       // key_of_score(i) <= seen: row sees it
        float w[16], sum;
        auto weights = [&]() __attribute__((always_inline)) {
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                w[i] = fast_exp2(fmaf(s[i], c2, -m_used));
                if (MASKED && key_of_score(i) > seen) w[i] = 0.f;
                sum += w[i];
            }
        };
        weights();
        // The maximum is raised only where the weights outgrow it: their sum, which is formed anyway, tells.
        if (__builtin_expect(__any(!(sum <= 4096.f)), 0)) {
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!MASKED || key_of_score(i) <= seen) mx = fmaxf(mx, s[i] * c2);
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            // (row by row, so that no row's bits depend on its neighbours')
            const bool raise = __shfl_xor((int)!(sum <= 4096.f), 32) | (int)!(sum <= 4096.f);
            const float m_new = raise ? fmaxf(m_used, mx) : m_used, alpha = fast_exp2(m_used - m_new);
            m_used = m_new;
            l_part *= alpha;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[nt][i] *= alpha;
            weights();
        }
        l_part += sum;
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    o[nt] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(cb[v_ld + key_of_score(i) * S::PV + 32 * nt]), w[i], o[nt], 0, 0, 0);
        } else {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                u32x4 hi, lo;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w0 = w[8 * m + 2 * i], w1 = w[8 * m + 2 * i + 1];
                    if constexpr (TWO_TERMS) {
                        // The first term is cut, so that the second is never negative, nor, by the 2^-23 added, zero for a weight
                        // that is not: with an infinite value both terms then agree.
                        hi[i] = __builtin_amdgcn_perm(__float_as_uint(w1), __float_as_uint(w0), 0x07060302);
                        lo[i] = pack_bf16(fmaf(w0, 1.0f + 0x1p-23f, -__uint_as_float(hi[i] << 16)), fmaf(w1, 1.0f + 0x1p-23f, -__uint_as_float(hi[i] & 0xffff0000u)));
                    } else {
                        hi[i] = pack_bf16(w0, w1);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(cb + v_ld + 16 * m * S::PV + 16 * nt));
                    const v4i16 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(cb + v_ld + (16 * m + 8) * S::PV + 16 * nt));
                    const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7));
                    o[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, hi), o[nt], 0, 0, 0);
                    if constexpr (TWO_TERMS) o[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, lo), o[nt], 0, 0, 0);
                }
            }
        }
    };

    // Tile t is in buffer t % 2 of LDS behind the barrier of its step; t + 1 is stored and t + 3 asked for during it.
    auto step = [&](int t, auto stage) __attribute__((always_inline)) {
        constexpr int ST = decltype(stage)::value, BUF = SHARE ? 0 : ST;
        __syncthreads();
        if constexpr (SHARE) {
            store_kv(t, s_tiles, ST);
            load_kv(t + 2, ST);
            __syncthreads();
        } else {
            store_kv(t + 1, s_tiles + (ST ^ 1) * BUF_WORDS, ST ^ 1);
            load_kv(t + 3, ST ^ 1);
        }
        if (t < t_plain) compute(t, s_tiles + BUF * BUF_WORDS, std::false_type());
        else if (t < t_seen) compute(t, s_tiles + BUF * BUF_WORDS, std::true_type());
    };
    int t = t_begin;
    load_kv(t, 0);
    load_kv(t + 1, 1);
    if constexpr (!SHARE) {
        store_kv(t, s_tiles, 0);
        load_kv(t + 2, 0);
    }
    for (; t + 1 < t_end; t += 2) {
        step(t, std::integral_constant<int, 0>());
        step(t + 1, std::integral_constant<int, 1>());
    }
    if (t < t_end) step(t, std::integral_constant<int, 0>());
    if (__any(bad) && lane == 0) s_bad = 1;
    __syncthreads();
    if (!active || !writes) return;

    // ---- epilogue: a lane holds columns 32 nt + 8 a + 4 h .. + 3 of its row, nt from its wavefront's first tile on
    const float l_row = l_part + __shfl_xor(l_part, 32);
    if (row0 + l32 >= M) return;
    const int in_seq = by_group(p, my_row), token = it.s.s0 + in_seq, head = g * p.G + my_row - in_seq * p.G;
    const bool direct = it.n_seg == 1;
    // row of out and lse, or of the partial results
    const size_t at = direct ? (size_t)token * p.H_q + head : ((size_t)(it.part + (SPLIT ? 0 : wave)) * p.H_kv + g) * 32 + l32;
    const float f = direct ? 1.0f / l_row : 1.0f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int c = 32 * (nt0 + nt) + 8 * a + 4 * h;
            const float4 x = make_float4(o[nt][4 * a] * f, o[nt][4 * a + 1] * f, o[nt][4 * a + 2] * f, o[nt][4 * a + 3] * f);
            if (!direct) *reinterpret_cast<float4 *>(p.part_o + at * DP + c) = x;
            else if (c >= p.d) continue;
            else if (F32) *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at * p.d + c) = x;
            else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + at * p.d + c) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
        }
    if (h == 0 && (!SPLIT || wave == 0)) {
        if (!direct) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(m_used, l_row);
        else if (p.lse) p.lse[at] = (m_used + __builtin_amdgcn_logf(l_row)) * LN2_F;
    }
    if (__builtin_expect(s_bad, 0)) {
        // what is no number joins what was written, by the lane that wrote it
        for (int key = max(diagonal, t_begin) * KT; key <= min(my_pos, t_end * KT - 1); ++key) {
            const int page = p.block_table[(size_t)it.b * p.max_pages + key / p.page_size];
            if ((unsigned)page >= (unsigned)p.n_pages) continue;
            const char *v = static_cast<const char *>(p.v_pool) + (((size_t)page * p.H_kv + g) * p.page_size + key % p.page_size) * row_bytes;
            for (int c = 32 * nt0 + 4 * h; c < min(p.d, 32 * (nt0 + NT)); c += (c & 3) == 3 ? 5 : 1) {
                const float y = F32 ? reinterpret_cast<const float *>(v)[c] : bf16_bits_to_float(reinterpret_cast<const uint16_t *>(v)[c]);
                if (fabsf(y) < INFINITY) continue;
                if (!direct) {
                    volatile float *z = p.part_o + at * DP + c;
                    *z = *z + y;
                } else if (F32) {
                    volatile float *z = static_cast<float *>(p.out) + at * p.d + c;
                    *z = *z + y;
                } else {
                    volatile uint16_t *z = static_cast<uint16_t *>(p.out) + at * p.d + c;
                    *z = (uint16_t)pack_bf16(bf16_bits_to_float(*z) + y, 0.f);
                }
            }
        }
    }
}

// A row's segments, one partial result after the other with a running maximum: columns c, c + 32 .. of a row.
template <int DP, int COLS>
struct Merged {
    float m = M_INIT, l = 0.f;
    float4 acc[COLS];
    __device__ __forceinline__ void add(float m2, float l2, const float4 *x)
    {
        const float m_new = fmaxf(m, m2), old = fast_exp2(m - m_new), f = l2 == 0.f ? 0.f : fast_exp2(m2 - m_new);     // (no weight: a segment that the row sees nothing of)
        m = m_new;
        l = l * old + f * l2;
#pragma unroll
        for (int k = 0; k < COLS; ++k) {
            acc[k].x = acc[k].x * old + f * x[k].x; acc[k].y = acc[k].y * old + f * x[k].y;
            acc[k].z = acc[k].z * old + f * x[k].z; acc[k].w = acc[k].w * old + f * x[k].w;
        }
    }
};

// The segments of the rows whose keys are cut.  grid (KV heads x tiles of rows, 4 or 8).  Few segments: eight lanes a row, four columns of every
// 32 each.  Many, as a lone long sequence has: eight groups of 32 lanes take every eighth segment of a row, and meet in LDS
// (one sequence of 16000 keys, 128 segments of 4 rows: 15.3 us in the first way).
template <int DP, bool F32>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkParams p)
{
    constexpr int GROUPS = 8, WIDE = (DP + 127) / 128;
    __shared__ float s_ml[GROUPS][2], s_acc[GROUPS][WIDE * 128];
    const int tid = threadIdx.x, lane = tid & 63, g = blockIdx.x % p.H_kv;
    Item it;
    if (!find_item<MERGE>(p, blockIdx.x / p.H_kv, lane, &it)) return;
    const int M = it.s.n * p.G;
    const size_t step = (size_t)(it.rows / 32) * p.H_kv * 32;
    auto write = [&](size_t at, int c, const float4 &x, float f) {
        if (F32) *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at * p.d + c) = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
        else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + at * p.d + c) = make_uint2(pack_bf16(x.x * f, x.y * f), pack_bf16(x.z * f, x.w * f));
    };
    auto row_of_out = [&](int row) {
        const int token = by_group(p, row);
        return (size_t)(it.s.s0 + token) * p.H_q + (g * p.G + row - token * p.G);
    };
    const bool by_segments = it.n_seg >= 2 * GROUPS;        // then the grid's y are rows, otherwise blocks of 32
    if (!by_segments) {
        for (int block = blockIdx.y; block < it.rows / 32; block += gridDim.y) {
            const int row0 = it.rt * it.rows + 32 * block;
            const size_t first = ((size_t)(it.part + block) * p.H_kv + g) * 32;
            constexpr int COLS = DP / 32;
            const int row = row0 + tid / 8;
            if (row >= M) break;
            Merged<DP, COLS> a;
#pragma unroll
            for (int k = 0; k < COLS; ++k) a.acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
            for (int s = 0; s < it.n_seg; ++s) {
                const size_t at = first + tid / 8 + s * step;
                const float2 ml = *reinterpret_cast<const float2 *>(p.part_ml + 2 * at);
                float4 x[COLS];
#pragma unroll
                for (int k = 0; k < COLS; ++k) x[k] = *reinterpret_cast<const float4 *>(p.part_o + at * DP + 32 * k + 4 * (tid & 7));
                a.add(ml.x, ml.y, x);
            }
            const size_t at = row_of_out(row);
#pragma unroll
            for (int k = 0; k < COLS; ++k)
                if (32 * k + 4 * (tid & 7) < p.d) write(at, 32 * k + 4 * (tid & 7), a.acc[k], 1.0f / a.l);
            if (p.lse && (tid & 7) == 0) p.lse[at] = (a.m + __builtin_amdgcn_logf(a.l)) * LN2_F;
        }
        return;
    }
    const int group = tid >> 5, l32 = tid & 31;
    for (int r = blockIdx.y; r < it.rows && it.rt * it.rows + r < M; r += gridDim.y) {
        const size_t first = ((size_t)(it.part + r / 32) * p.H_kv + g) * 32 + r % 32;
        Merged<DP, WIDE> a;
#pragma unroll
        for (int k = 0; k < WIDE; ++k) a.acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int s = group; s < it.n_seg; s += GROUPS) {
            const size_t at = first + s * step;
            const float2 ml = *reinterpret_cast<const float2 *>(p.part_ml + 2 * at);
            float4 x[WIDE];
#pragma unroll
            for (int k = 0; k < WIDE; ++k) x[k] = 128 * k + 4 * l32 < DP ? *reinterpret_cast<const float4 *>(p.part_o + at * DP + 128 * k + 4 * l32) : make_float4(0.f, 0.f, 0.f, 0.f);
            a.add(ml.x, ml.y, x);
        }
        __syncthreads();                // (the row before has been read)
        if (l32 == 0) { s_ml[group][0] = a.m; s_ml[group][1] = a.l; }
#pragma unroll
        for (int k = 0; k < WIDE; ++k) *reinterpret_cast<float4 *>(&s_acc[group][128 * k + 4 * l32]) = a.acc[k];
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int j = 1; j < GROUPS; ++j) {
                float4 x[WIDE];
#pragma unroll
                for (int k = 0; k < WIDE; ++k) x[k] = *reinterpret_cast<const float4 *>(&s_acc[j][128 * k + 4 * l32]);
                a.add(s_ml[j][0], s_ml[j][1], x);
            }
            const size_t at = row_of_out(it.rt * it.rows + r);
#pragma unroll
            for (int k = 0; k < WIDE; ++k)
                if (128 * k + 4 * l32 < p.d) write(at, 128 * k + 4 * l32, a.acc[k], 1.0f / a.l);
            if (p.lse && l32 == 0) p.lse[at] = (a.m + __builtin_amdgcn_logf(a.l)) * LN2_F;
        }
    }
}

// ---- rows of new tokens into their pages: 16 bytes of K and of V a thread
struct StoreParams {
    size_t pieces;                      // T * pieces of a row
    int row_pieces, head_pieces, page_size, n_slots, H_kv;
    const char *k, *v;
    char *k_pool, *v_pool;
    size_t k_stride, v_stride, k_layer, v_layer, pool_layer;        // bytes
    const int32_t *slot_map;
};

__global__ __launch_bounds__(256) void kv_store_paged_kernel(StoreParams p)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.pieces) return;
    const int t = (int)(i / p.row_pieces), c = (int)(i % p.row_pieces), head = c / p.head_pieces, in_head = c % p.head_pieces;
    const u32x4 k = *reinterpret_cast<const u32x4 *>(p.k + blockIdx.y * p.k_layer + t * p.k_stride + 16 * (size_t)c);
    const u32x4 v = *reinterpret_cast<const u32x4 *>(p.v + blockIdx.y * p.v_layer + t * p.v_stride + 16 * (size_t)c);
    const int slot = p.slot_map[t];
    if ((unsigned)slot >= (unsigned)p.n_slots) return;
    const size_t at = blockIdx.y * p.pool_layer +
                      ((((size_t)(slot / p.page_size) * p.H_kv + head) * p.page_size + slot % p.page_size) * p.head_pieces + in_head) * 16;
    *reinterpret_cast<u32x4 *>(p.k_pool + at) = k;
    *reinterpret_cast<u32x4 *>(p.v_pool + at) = v;
}

// Where a workgroup takes 32 rows and shares out the columns, instead of 128 rows.  32 sequences on 100 to 8000 tokens, 32/8 heads, us of the
// attention with 128 rows and with 32:
//   bf16, d = 128, 4 rows each 133, 115; 32 rows 133, 117; 48 rows 138, 169.  d = 80, 4 rows 111, 92; d = 96, 48 rows 120, 168.
//   d = 64, 4 rows 68, 77: two wavefronts of the four would have columns.
//   fp32, where a wavefront's products take longer than its tiles to come: d = 128, 4 rows 735, 297; 8 prompts of 200 to 500 tokens 181, 157;
//   d = 96, 573, 247 and 143, 135; d = 64, 259, 198 and 90, 118.
//   d = 256, where 128 rows need more registers than there are: bf16, 4 rows 676, 233; 8 prompts of 500 to 1000 tokens 425, 374; fp32 523, 121.
enum Split { NO_SPLIT, SPLIT_FEW, ALWAYS_SPLIT };
constexpr Split split_rule(int DP, bool f32)
{
    return DP == 256 || (f32 && DP >= 96) ? ALWAYS_SPLIT : (f32 ? DP == 64 : DP >= 96) ? SPLIT_FEW : NO_SPLIT;
}

int padded_dim(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : 256; }

// Weights in PV.  fp32 as they are; bf16 as two terms (2^-16 of a weight), at d = 128 as one (2^-8), the convention of the framework's tree attention, so that a
// token's result has the same error whichever of the two computes it.  One term and two at d = 128: root-mean-square error of a result against 64 bits 2.3e-3 and
// 1.7e-3 (the latter is the rounding of the result); 32 sequences of 100 to 8000 tokens, 32/8 heads, one new token 111 and 116 us, four of them with 200 to 512
// on up to 4096 113 and 128.
template <int DP, bool F32>
void launch_shape(const ChunkParams &p, const ChunkPlan &plan, hipStream_t stream)
{
    constexpr Split rule = split_rule(DP, F32);
    constexpr bool FEW = rule != NO_SPLIT, MORE = rule == ALWAYS_SPLIT;         // SPLIT of either number of rows
    const bool few = plan.rows_few == ROWS_SPLIT;
    auto kernel = few ? chunk_attn_kernel<DP, F32, FEW, !F32> : chunk_attn_kernel<DP, F32, MORE, !F32>;
    if constexpr (!F32 && DP == 128)
        if (p.d == DP) kernel = few ? chunk_attn_kernel<DP, F32, FEW, false> : chunk_attn_kernel<DP, F32, MORE, false>;
    launch_kernel(K_CHUNK_ATTN, kernel, dim3(p.H_kv * plan.max_items), dim3(256), stream, p);
    if (plan.max_items_many) launch_chunk_wide(p, plan.max_items_many, stream);
    if (plan.max_parts + plan.max_parts_many)
        launch_kernel(K_CHUNK_MERGE, chunk_merge_kernel<DP, F32>, dim3(p.H_kv * plan.max_cut, plan.merge_y), dim3(256), stream, p);
}

template <bool F32>
void launch_type(const ChunkParams &p, const ChunkPlan &plan, hipStream_t stream)
{
    switch (padded_dim(p.d)) {
    case 32: return launch_shape<32, F32>(p, plan, stream);
    case 64: return launch_shape<64, F32>(p, plan, stream);
    case 96: return launch_shape<96, F32>(p, plan, stream);
    case 128: return launch_shape<128, F32>(p, plan, stream);
    default: return launch_shape<256, F32>(p, plan, stream);
    }
}

}  // namespace

// Row tiles of `rows` of one KV head at most, where T tokens make sequences of any length.
static long most_tiles(long T, long B, long G, long rows)
{
    const long by_rows = T * G / rows + (T < B ? T : B), by_token = T * ((G + rows - 1) / rows);
    return by_rows < by_token ? by_rows : by_token;
}

bool make_chunk_plan(const mcsd_chunk_desc &d, ChunkPlan *plan)
{
    const long G = d.H_q / d.H_kv, T = d.T, kt = (d.L_stride + KT - 1) / KT;
    // bf16, d = 128: sequences of more than MANY rows have a kernel of their own where a launch has so many on average (it would find
    // nothing to do in a batch that decodes, for 4 us).  Up to one of its row tiles on average the arrays decide, on the device: sequences of few
    // rows that have most of the work are bound by memory, and those of many run beside them (32 sequences, four with 200 to 512 tokens, 32/8 heads:
    // 137 us, 159 in two kernels one after the other); otherwise the kernel for many is faster (8 sequences of 128 to 256 tokens on 2000 to 4000,
    // 32/32 heads: 158 us, 204 in one kernel).
    // Little work of many rows stays with the kernel for few, too.  What the sizes say of the work: at least `least` (sequences of one length
    // without cached tokens), at most all row tiles by the capacity.
    // Two workgroups of few rows run on a compute unit, one of many.
    plan->at_once = d.H_kv < 512 ? 512 / d.H_kv : 1;
    plan->at_once_many = d.H_kv < 256 ? 256 / d.H_kv : 1;
    const double small = SMALL_WORK * plan->at_once_many, least = (double)T * T * G / ((double)ROWS_MANY * KT * d.B);
    const bool many = d.dtype == MCSD_DTYPE_BF16 && d.d == 128 && T * G > (long)MANY * d.B && (double)most_tiles(T, d.B, G, ROWS_MANY) * kt >= small;
    plan->many = many ? MANY : NEVER_MANY;
    plan->by_work = many && (T * G <= (long)ROWS_MANY * d.B || least < small);
    const Split rule = split_rule(padded_dim(d.d), d.dtype == MCSD_DTYPE_FP32);
    const bool split = rule == ALWAYS_SPLIT || (rule == SPLIT_FEW && T * G <= (long)ROWS_SPLIT * d.B);
    plan->rows_few = split ? ROWS_SPLIT : ROWS_FEW;
    // Segments of 8 tiles at least.  A sequence that is cut has kt / len of them, of few rows rounded up, 2 kt / len at most, of many to nearest,
    // 4/3 kt / len at most.
    plan->min_seg = 8;
    const long target = 2L * plan->at_once, target_many = (long)(cut_at(CUTS - 1) * plan->at_once_many);
    const long n_seg = (kt + plan->min_seg - 1) / plan->min_seg;
    // (a sequence of few rows is one row tile where those of many are not here)
    const long tiles = many && !plan->by_work ? (T < d.B ? T : d.B) : most_tiles(T, d.B, G, plan->rows_few), tiles_many = many ? most_tiles(T, d.B, G, ROWS_MANY) : 0;
    // a sequence of n segments has its keys cut where n >= 2
    auto parts_of = [&](long most, long row_tiles) { return n_seg < 2 ? 0 : most < row_tiles * n_seg ? most : row_tiles * n_seg; };
    auto less = [](long x, long y) { return x < y ? x : y; };
    const long parts = parts_of(less(2 * target, target + tiles) + 2, tiles);
    const long parts_many = parts_of(less((4 * target_many + 2) / 3, target_many + tiles_many / 2) + 2, tiles_many);
    // kt / len and one more of every row tile
    auto items_of = [&](long target, long row_tiles) { return n_seg < 2 ? row_tiles : target + row_tiles < row_tiles * n_seg ? target + row_tiles : row_tiles * n_seg; };
    const long items = items_of(target, tiles), items_many = tiles_many ? items_of(target_many, tiles_many) : 0;
    const long cut = parts / 2 < tiles ? parts / 2 : tiles, cut_many = parts_many / 2 < tiles_many ? parts_many / 2 : tiles_many;
    const long rows = many ? ROWS_MANY : plan->rows_few, cells = 2048 / (d.H_kv * (cut + cut_many) + 1);
    plan->merge_y = (int)(cells < rows / 32 ? rows / 32 : cells < rows ? cells : rows);
    plan->max_items = (int)items;
    plan->max_items_many = (int)items_many;
    plan->max_cut = (int)(cut + cut_many);
    plan->max_parts = (int)(parts * (plan->rows_few / 32));
    plan->max_parts_many = (int)(parts_many * (ROWS_MANY / 32));
    const size_t rows_cut = (size_t)(plan->max_parts + plan->max_parts_many) * d.H_kv * 32;
    plan->ws_bytes = rows_cut || many ? (rows_cut * (padded_dim(d.d) + 2) * 4 + 255) / 256 * 256 + 256 : 0;
    return items * d.H_kv < 1L << 24 && items_many * d.H_kv < 1L << 24;     // (a launch has fewer than 2^32 threads)
}

int32_t launch_chunk_attn(const mcsd_chunk_desc &d, const mcsd_chunk_bufs &b, const mcsd_paged_kv &kv, const ChunkPlan &plan, hipStream_t stream)
{
    ChunkParams p = chunk_params(d, kv);
    p.q = b.q; p.k_pool = b.k_pool; p.v_pool = b.v_pool; p.chunk_start = b.chunk_start; p.prefix_len = b.prefix_len; p.out = b.out; p.lse = b.lse;
    p.min_seg = plan.min_seg; p.max_parts = plan.max_parts; p.max_parts_many = plan.max_parts_many; p.many = plan.many; p.by_work = plan.by_work; p.rows_few = plan.rows_few;
    p.at_once = (float)plan.at_once; p.at_once_many = (float)plan.at_once_many;
    p.part_o = static_cast<float *>(b.workspace);
    const size_t parts = (size_t)(plan.max_parts + plan.max_parts_many) * d.H_kv * 32;
    p.part_ml = p.part_o + parts * padded_dim(d.d);
    p.notes = plan.ws_bytes ? reinterpret_cast<ChunkNotes *>(static_cast<char *>(b.workspace) + plan.ws_bytes - 256) : nullptr;
    if (d.dtype == MCSD_DTYPE_FP32) launch_type<true>(p, plan, stream);
    else launch_type<false>(p, plan, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("chunk attention launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

int32_t launch_kv_store_paged(const mcsd_rows_desc &d, const mcsd_store_bufs &b, const mcsd_paged_kv &kv, hipStream_t stream)
{
    if (d.T == 0) return MCSD_OK;
    const size_t esize = d.dtype == MCSD_DTYPE_FP32 ? 4 : 2;
    StoreParams p;
    p.head_pieces = (int)(d.d * esize / 16); p.row_pieces = p.head_pieces * d.H_kv; p.pieces = (size_t)d.T * p.row_pieces;
    p.page_size = kv.page_size; p.n_slots = kv.n_pages * kv.page_size; p.H_kv = d.H_kv;
    p.k = static_cast<const char *>(b.k); p.v = static_cast<const char *>(b.v);
    p.k_pool = static_cast<char *>(b.k_pool); p.v_pool = static_cast<char *>(b.v_pool);
    p.k_stride = d.k_stride * esize; p.v_stride = d.v_stride * esize;
    p.k_layer = d.n_layers > 1 ? d.k_layer_stride * esize : 0; p.v_layer = d.n_layers > 1 ? d.v_layer_stride * esize : 0;
    p.pool_layer = (size_t)p.n_slots * p.row_pieces * 16;
    p.slot_map = b.slot_map;
    launch_kernel(K_KV_STORE_PAGED, kv_store_paged_kernel, dim3((unsigned)((p.pieces + 255) / 256), d.n_layers), dim3(256), stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("kv store (pages) launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
