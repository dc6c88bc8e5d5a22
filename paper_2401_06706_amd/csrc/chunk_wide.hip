// Attention of a chunk of new tokens over a paged cache: bf16, d = 128, sequences with more rows than one wavefront holds.
#include <type_traits>

#include "chunk_common.h"

namespace mcsd {
namespace {

constexpr int ROWS = ROWS_MANY, D = 128, ROW_BYTES = 2 * D, DEPTH = 4;
constexpr int SIDE_BYTES = KT * ROW_BYTES, TILE_BYTES = 2 * SIDE_BYTES;      // K, then V

// what a page outside the pool reads as: four rows, a load's worth
__device__ __attribute__((aligned(16))) uint32_t zero_rows[ROW_BYTES] = {0};

// 64 lanes x 16 bytes from base + offset straight into LDS at `to` (lane after lane); arrived once the wavefront has counted vmcnt down to it
__device__ __forceinline__ void fetch16(uint32_t to, const void *base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(to), "v"(offset), "s"(base) : "memory", "m0");
}

// A workgroup of four wavefronts, one per SIMD, owns 256 rows of a (sequence, KV head) and a segment of its key tiles; a wavefront owns
// 64 rows in two blocks of 32, A and B, and shares every K and V operand between them.  S^T = K Q^T and O^T += V^T P^T
// with v_mfma_f32_32x32x16_bf16 as in tree attention (a weight never leaves its lane).
//   - One block's softmax runs beside the other's matrix instructions, tile after tile:
//        phase A(t): weights of A from S_A(t)     beside   O_B += V(t-1) P_B(t-1),  S_B(t) = K(t) Q_B
//        phase B(t): weights of B from S_B(t)     beside   O_A += V(t) P_A(t),      S_A(t+1) = K(t+1) Q_A
//     so that 16 matrix instructions (512 cycles) and some 60 vector ones that do not depend on them stand in one stretch of code.
//   - K and V go from memory straight into a ring of four tiles in LDS, asked for three tiles ahead.  16-byte pieces lie permuted: K piece c of row r
//     at c ^ (r % 16), V piece c at c ^ 4 (r % 4), which keeps the 16 rows of an operand read, and the four rows
//     of a transposing read, in banks of their own.
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1)))
void chunk_wide_kernel(ChunkParams p)
{
    __shared__ __attribute__((aligned(1024))) uint32_t s_ring[DEPTH * TILE_BYTES / 4];
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, l32 = lane & 31, lj = lane >> 4, lc = lane & 15;
    const int g = blockIdx.x % p.H_kv;
    Item it;
    if (!find_item<MANY_ROWS>(p, blockIdx.x / p.H_kv, lane, &it)) return;
    const int M = it.s.n * p.G, tile0 = it.rt * ROWS, row0 = tile0 + 64 * wave;
    auto position = [&](int row) { return min(it.s.L + row / p.G, it.s.keys - 1); };
    const int kt = position(min(tile0 + ROWS, M) - 1) / KT + 1;                  // key tiles that some row of this tile sees
    const int seg = (kt + it.n_seg - 1) / it.n_seg, t_begin = it.seg * seg, t_end = min(kt, t_begin + seg);
    const int diagonal = (position(tile0) + 1) / KT;                             // from here on there are keys that some row does not see
    const bool active = row0 < M;
    // tiles that every row of this wavefront sees whole; tiles that any of them sees
    const int t_plain = active ? max(t_begin, min(t_end, (position(row0) + 1) / KT)) : t_begin;
    const int t_seen = active ? max(t_begin, min(t_end, position(min(row0 + 64, M) - 1) / KT + 1)) : t_begin;
    if (tid == 0) s_bad = 0;

    // ---- requests: this wavefront's 8 rows of K and of V of a tile.  Past the end the last tile is asked for again, so that what is
    // waited for can be counted.
    const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint32_t *)s_ring;
    const uint32_t row_off = (uint32_t)lj * ROW_BYTES;
    const uint32_t k_off0 = row_off + 16 * (lc ^ ((8 * wave + lj) & 15)), k_off1 = row_off + 16 * (lc ^ ((8 * wave + 4 + lj) & 15));
    const uint32_t v_off = row_off + 16 * (lc ^ (4 * lj));
    const const_i32_ptr table = (const_i32_ptr)(uintptr_t)(p.block_table + (size_t)it.b * p.max_pages);
    const int t_last = max(t_begin, t_end - 1);
    // (advance() works out, among the matrix instructions, where the next tile lies)
    int ask = t_begin - 1, ask_page = t_begin * KT / p.page_size, ask_row = t_begin * KT % p.page_size - KT;
    int entry = t_begin < t_end ? (int)table[ask_page] : -1, next;
    const size_t page_bytes = (size_t)p.H_kv * p.page_size * ROW_BYTES, head_at = ((size_t)g * p.page_size + 8 * wave) * ROW_BYTES;
    const char *const k_head = static_cast<const char *>(p.k_pool) + head_at, *const v_head = static_cast<const char *>(p.v_pool) + head_at;
    const char *zeros = reinterpret_cast<const char *>(zero_rows);
    asm volatile("" : "+s"(zeros));
    const char *k_at, *v_at;
    uint32_t to;
    auto advance = [&]() __attribute__((always_inline)) {
        ++ask;
        to = ring_at + (ask & (DEPTH - 1)) * TILE_BYTES + wave * (8 * ROW_BYTES);
        if (ask <= t_last) {
            ask_row += KT;
            if (ask_row >= p.page_size) {
                ask_row = 0;
                entry = table[++ask_page];
            }
        }
        const bool in = (unsigned)entry < (unsigned)p.n_pages;
        const size_t at = (size_t)(uint32_t)entry * page_bytes + (uint32_t)ask_row * ROW_BYTES;
        k_at = in ? k_head + at : zeros;
        v_at = in ? v_head + at : zeros;
        next = in ? 4 * ROW_BYTES : 0;
    };
    auto request = [&]() __attribute__((always_inline)) {
        fetch16(to, k_at, k_off0);
        fetch16(to + 4 * ROW_BYTES, k_at + next, k_off1);
        fetch16(to + SIDE_BYTES, v_at, v_off);
        fetch16(to + SIDE_BYTES + 4 * ROW_BYTES, v_at + next, v_off);
    };
    advance();
    if (t_begin < t_end) {
#pragma unroll
        for (int i = 0; i < DEPTH - 1; ++i) { request(); advance(); }
    }

    // ---- Q: lane holds Q[row][16 kk + 8 h .. + 7] of a row of each block (lanes past the last row repeat it)
    int my_row[2], my_pos[2];
    bf16x8 q[2][8];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        my_row[x] = min(row0 + 32 * x + l32, M - 1);
        my_pos[x] = position(my_row[x]);
        const char *src = static_cast<const char *>(p.q) + (size_t)(it.s.s0 + my_row[x] / p.G) * p.q_row + (size_t)(g * p.G + my_row[x] % p.G) * ROW_BYTES + 16 * h;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) q[x][kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(src + 32 * kk));
    }
    f32x16 o[2][4], s[2];
    float m_used[2] = {M_INIT, M_INIT}, l_part[2] = {0.f, 0.f};
    bf16x8 w[2][2];             // packed weights
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[x][nt][i] = 0.f;
        const u32x4 zero = {0, 0, 0, 0};
        w[x][0] = w[x][1] = __builtin_bit_cast(bf16x8, zero);
    }
    const float c2 = p.scale_log2;

    // ---- operands out of LDS
    const uint32_t k_ld = l32 * ROW_BYTES + 16 * (h ^ (l32 & 15));              // ^ 32 kk
    uint32_t v_ld[4];
#pragma unroll
    for (int nt = 0; nt < 4; ++nt)
        v_ld[nt] = SIDE_BYTES + (4 * h + (lc >> 2)) * ROW_BYTES + 16 * ((4 * nt + 2 * (lj & 1) + ((lc & 3) >> 1)) ^ (4 * (lc >> 2))) + 8 * (lc & 1);
    const char *const ring = reinterpret_cast<const char *>(s_ring);
    typedef short v4i16 __attribute__((ext_vector_type(4)));
    typedef v4i16 __attribute__((address_space(3))) *lds_v4i16_ptr;
    auto read_k = [&](int t, bf16x8 *k) __attribute__((always_inline)) {
        const char *at = ring + (t & (DEPTH - 1)) * TILE_BYTES;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) k[kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(at + (k_ld ^ (32 * kk))));
    };
    auto read_v = [&](int t, bf16x8 (*v)[4]) __attribute__((always_inline)) {
        const char *at = ring + (t & (DEPTH - 1)) * TILE_BYTES;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int nt = 0; nt < 4; ++nt) {
                const v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(at + v_ld[nt] + 16 * m * ROW_BYTES));
                const v4i16 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(at + v_ld[nt] + (16 * m + 8) * ROW_BYTES));
                v[m][nt] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7));
            }
    };
    // weights of block x from its scores of tile t
    auto weights = [&](const int x, int t, auto masked, u32x4 *pk) __attribute__((always_inline)) {
        const int seen = my_pos[x] - t * KT - 4 * h;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            float w0 = fast_exp2(fmaf(s[x][i], c2, -m_used[x])), w1 = fast_exp2(fmaf(s[x][i + 1], c2, -m_used[x]));
            if constexpr (decltype(masked)::value) {
                if (key_of_score(i) > seen) w0 = 0.f;
                if (key_of_score(i + 1) > seen) w1 = 0.f;
            }
            sum += w0 + w1;
            pk[i / 8][i / 2 % 4] = pack_bf16(w0, w1);
        }
        return sum;
    };
    // The maximum is raised only where the weights outgrow it (their sum, which is formed anyway, tells), row by row.
    auto settle = [&](const int x, int t, auto masked, float sum, u32x4 *pk) __attribute__((always_inline)) {
        if (__builtin_expect(__any(!(sum <= 4096.f)), 0)) {
            const int seen = my_pos[x] - t * KT - 4 * h;
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!decltype(masked)::value || key_of_score(i) <= seen) mx = fmaxf(mx, s[x][i] * c2);
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const bool raise = __shfl_xor((int)!(sum <= 4096.f), 32) | (int)!(sum <= 4096.f);
            const float m_new = raise ? fmaxf(m_used[x], mx) : m_used[x], alpha = fast_exp2(m_used[x] - m_new);
            m_used[x] = m_new;
            l_part[x] *= alpha;
#pragma unroll
            for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[x][nt][i] *= alpha;
            sum = weights(x, t, masked, pk);
        }
        l_part[x] += sum;
        w[x][0] = __builtin_bit_cast(bf16x8, pk[0]);
        w[x][1] = __builtin_bit_cast(bf16x8, pk[1]);
    };
    auto pv = [&](const int x, const int m, const int nt, const bf16x8 (*v)[4]) __attribute__((always_inline)) {
        o[x][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[m][nt], w[x][m], o[x][nt], 0, 0, 0);
    };
    auto zero_scores = [&](const int x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = 0.f;
    };
    auto qk = [&](const int x, const int kk, const bf16x8 *k) __attribute__((always_inline)) {
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kk], q[x][kk], s[x], 0, 0, 0);
    };

    // ---- steps
    bool bad = false;
    // Where rows do not see all keys, values that are no numbers enter the products as zeros (0 times such a value is none either)
    // and are added in the epilogue to the rows that see them.  This wavefront's own rows of the tile.
    auto clean = [&](int t) __attribute__((always_inline)) {
        char *at = const_cast<char *>(ring) + (t & (DEPTH - 1)) * TILE_BYTES + SIDE_BYTES + wave * (8 * ROW_BYTES) + 16 * lane;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(at + 4 * j * ROW_BYTES);
            bool here = false;
            const u32x4 y = finite_or_zero(x, false, &here);
            if (here) *reinterpret_cast<u32x4 *>(at + 4 * j * ROW_BYTES) = y;
            bad |= here;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    // Tile t + 1 has arrived (4 requests per tile, those of t + 2 may still be on their way) and, behind the barrier, everybody's part of it; what
    // lay where t + 3 goes, t - 1, was last read ahead of it.
    auto begin_step = [&](int t) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
        if (t + 1 >= diagonal && t + 1 < t_end) clean(t + 1);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        request();
    };
    // One tile: k, v hold K(t) and V(t - 1), afterwards k_next, v_now hold K(t + 1) and V(t).
    auto step = [&](int t, auto masked, const bf16x8 (&k)[8], const bf16x8 (&v)[2][4], bf16x8 (&k_next)[8], bf16x8 (&v_now)[2][4]) __attribute__((always_inline)) {
        begin_step(t);
        u32x4 pk[2];
        float sum;
        read_v(t, v_now);
        read_k(t + 1, k_next);
        sum = weights(0, t, masked, pk);
        zero_scores(1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            pv(1, i / 4, i % 4, v);
            qk(1, i, k);
        }
        if (!decltype(masked)::value) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x402, 4, 0);
            }
        }
        settle(0, t, masked, sum, pk);
        advance();
        sum = weights(1, t, masked, pk);
        zero_scores(0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            pv(0, i / 4, i % 4, v_now);
            qk(0, i, k_next);
        }
        if (!decltype(masked)::value) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x402, 4, 0);
            }
        }
        settle(1, t, masked, sum, pk);
    };
    if (t_begin < t_end) {
        int t = t_begin;
        // the first tiles and Q (the compiler waits for what it knows of, Q, ahead of this: not in the loop, where it would wait for all requests)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+a"(q[x][kk]));
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (t >= diagonal) clean(t);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t < t_seen) {
            const u32x4 zero = {0, 0, 0, 0};
            bf16x8 k0[8], v0[2][4], k1[8], v1[2][4];        // (two sets that take turns)
#pragma unroll
            for (int i = 0; i < 8; ++i) v0[i / 4][i % 4] = __builtin_bit_cast(bf16x8, zero);
            read_k(t, k0);
            zero_scores(0);
#pragma unroll
            for (int i = 0; i < 8; ++i) qk(0, i, k0);
            for (; t + 1 < t_plain; t += 2) {
                step(t, std::false_type(), k0, v0, k1, v1);
                step(t + 1, std::false_type(), k1, v1, k0, v0);
            }
            for (; t + 1 < t_seen; t += 2) {
                step(t, std::true_type(), k0, v0, k1, v1);
                step(t + 1, std::true_type(), k1, v1, k0, v0);
            }
            if (t < t_seen) {
                step(t, std::true_type(), k0, v0, k1, v1);
                ++t;
#pragma unroll
                for (int i = 0; i < 8; ++i) pv(1, i / 4, i % 4, v1);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) pv(1, i / 4, i % 4, v0);
            }
        }
        for (; t < t_end; ++t) { begin_step(t); advance(); }                   // (this wavefront only helps to load)
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // nothing may be on its way into LDS when the workgroup ends
    if (__any(bad) && lane == 0) s_bad = 1;
    __syncthreads();
    if (!active) return;

    // ---- epilogue: a lane holds columns 32 nt + 8 a + 4 h .. + 3 of its row in each block
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        if (__builtin_expect(s_bad, 0)) {
            for (int key = max(diagonal, t_begin) * KT; key <= min(my_pos[x], t_end * KT - 1); ++key) {
                const int page = p.block_table[(size_t)it.b * p.max_pages + key / p.page_size];
                if ((unsigned)page >= (unsigned)p.n_pages) continue;
                const uint16_t *v = static_cast<const uint16_t *>(p.v_pool) + (((size_t)page * p.H_kv + g) * p.page_size + key % p.page_size) * D;
#pragma unroll
                for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float y = bf16_bits_to_float(v[32 * nt + 8 * (i >> 2) + 4 * h + (i & 3)]);
                        if (!(fabsf(y) < INFINITY)) o[x][nt][i] += y;
                    }
            }
        }
        const float l_row = l_part[x] + __shfl_xor(l_part[x], 32);
        const bool mine = row0 + 32 * x + l32 < M;
        const int token = it.s.s0 + my_row[x] / p.G, head = g * p.G + my_row[x] % p.G;
        if (it.n_seg == 1) {
            const float f = 1.0f / l_row;
            char *dst = static_cast<char *>(p.out) + ((size_t)token * p.H_q + head) * ROW_BYTES + 16 * h;
#pragma unroll
            for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                for (int a = 0; a < 4; a += 2) {
                    // lanes l32 and l32 + 32 exchange so that each holds eight neighbouring columns
                    u32x4 y;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t even = pack_bf16(o[x][nt][4 * a + 2 * k] * f, o[x][nt][4 * a + 2 * k + 1] * f);
                        const uint32_t odd = pack_bf16(o[x][nt][4 * a + 4 + 2 * k] * f, o[x][nt][4 * a + 5 + 2 * k] * f);
                        const auto both = __builtin_amdgcn_permlane32_swap(even, odd, false, false);
                        y[k] = both[0];
                        y[2 + k] = both[1];
                    }
                    if (mine) *reinterpret_cast<u32x4 *>(dst + 2 * (32 * nt + 8 * a)) = y;
                }
            if (p.lse && h == 0 && mine) p.lse[(size_t)token * p.H_q + head] = (m_used[x] + __builtin_amdgcn_logf(l_row)) * LN2_F;
        } else if (mine) {
            const size_t prow = ((size_t)(it.part + 2 * wave + x) * p.H_kv + g) * 32 + l32;
            if (h == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * prow) = make_float2(m_used[x], l_row);
            float *dst = p.part_o + prow * D;
#pragma unroll
            for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                for (int a = 0; a < 4; ++a)
                    *reinterpret_cast<float4 *>(dst + 32 * nt + 8 * a + 4 * h) = make_float4(o[x][nt][4 * a], o[x][nt][4 * a + 1], o[x][nt][4 * a + 2], o[x][nt][4 * a + 3]);
        }
    }
}

}  // namespace

void launch_chunk_wide(const ChunkParams &p, int max_items, hipStream_t stream)
{
    launch_kernel(K_CHUNK_WIDE, chunk_wide_kernel, dim3(p.H_kv * max_items), dim3(256), stream, p);
}

}  // namespace mcsd
