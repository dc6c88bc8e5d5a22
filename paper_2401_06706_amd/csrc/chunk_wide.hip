// Attention of a chunk of new tokens over a paged cache: bf16, d = 128, sequences with more rows than one wavefront holds.
#include <type_traits>

#include "chunk_common.h"

namespace mcsd {
namespace {

constexpr int ROWS = ROWS_MANY, D = 128, ROW_BYTES = 2 * D, DEPTH = 4;
constexpr int SIDE_BYTES = KT * ROW_BYTES, TILE_BYTES = 2 * SIDE_BYTES;      // K, then V

// what a page outside the pool reads as: a wavefront's rows of a tile
__device__ __attribute__((aligned(16))) uint32_t zero_rows[8 * ROW_BYTES / 4] = {0};

// 2 x 64 lanes x 16 bytes from base + offset, and from 1 KB behind, straight into LDS at `to` (lane after lane) and 1 KB behind (the
// instruction's offset counts on both sides); arrived once the wavefront has counted vmcnt down to them
__device__ __forceinline__ void fetch(uint32_t to, const void *base, uint32_t offset, uint32_t offset_behind)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024"
                 :: "s"(to), "v"(offset), "v"(offset_behind), "s"(base) : "memory", "m0");
}

// the same from an address of each lane's own
__device__ __forceinline__ void fetch_from(uint32_t to, const void *from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(uniform((int)to)), "v"(from) : "memory", "m0");
}

// A workgroup of four wavefronts, one per SIMD, owns 256 rows of a (sequence, KV head) and a segment of its key tiles; a wavefront owns
// 64 rows in two blocks of 32, A and B, and shares every K and V operand between them.  S^T = K Q^T and O^T += V^T P^T
// with v_mfma_f32_32x32x16_bf16 as in tree attention (a weight never leaves its lane).  Weights are rounded to one bf16 term for PV, their sum is taken of the
// unrounded ones: a second term would be 8 more matrix instructions on the 16 of a block and tile, and these bind.  (see launch_shape for what either costs)
//   - One block's softmax runs beside the other's matrix instructions, tile after tile:
//        phase A(t): weights of A from S_A(t)     beside   O_B += V(t-1) P_B(t-1),  S_B(t) = K(t) Q_B
//        phase B(t): weights of B from S_B(t)     beside   O_A += V(t) P_A(t),      S_A(t+1) = K(t+1) Q_A
//     so that 16 matrix instructions (512 cycles) and some 60 vector ones that do not depend on them stand in one stretch of code.
//   - K and V go from memory straight into a ring of four tiles in LDS, asked for three tiles ahead.  16-byte pieces lie permuted: K piece c of row r
//     at c ^ (r % 16), V piece c at c ^ 4 (r % 4), which keeps the 16 rows of an operand read, and the four rows
//     of a transposing read, in banks of their own.
//   - A workgroup goes through several row tiles, and asks for the next one's first tiles and Q ahead of the present one's epilogue:
//     there is no other workgroup on its CU that would run meanwhile.  Items are taken
//     as workgroups come to them, the heavy row tiles of a sequence first: dealt out beforehand, forth and back, eight prompts
//     of 1000 to 2048 tokens, 32 heads, gave the busiest workgroup 18 % more than the mean.
// Bound by the chip's power behind a long prefix: 2048 tokens on 16384, 64/8 heads 963 to 1050 us (1.17 to 1.27 PFLOP/s; matrix instructions busy 54 % of
// the cycles at about 2.0 GHz), 1398 with 32 rows a wavefront in the kernel for few.  Short prompts by what an item costs beside its tiles, some 8 us: 8 of 1000 to
// 2048 tokens, 32/32 heads 261 to 309 us, 278 on average (0.58 PFLOP/s).  Operands are replaced in place and the loop makes one step a turn: with two sets of operand registers, or
// scores in accumulator registers, the compiler copied them between the halves of the register file (1060 us).
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1)))
void chunk_wide_kernel(ChunkParams p)
{
    __shared__ __attribute__((aligned(1024))) uint32_t s_ring[DEPTH * TILE_BYTES / 4];
    __shared__ __attribute__((aligned(1024))) uint32_t s_rows[4][64 * ROW_BYTES / 4];       // Q of the next item, a wavefront's rows; results on their way out
    __shared__ int s_odd[2], s_next;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, l32 = lane & 31, lj = lane >> 4, lc = lane & 15;
    const int page_size = uniform(p.page_size), H_kv = uniform(p.H_kv);         // (scalars beside the vector copies that divisions make of them)
    const ItemList<MANY_ROWS> list(p, lane);
    // The first item of a workgroup is its own, each further one the next that nobody has (the counter starts from 0: the kernel for few rows clears
    // it).  Which workgroup takes an item changes nothing in its results.
    int next = blockIdx.x;
    auto next_item = [&](Item *it, int *g) __attribute__((always_inline)) {
        const int in_head = uniform(next / H_kv);
        *g = next - in_head * H_kv;           // (KV head fastest: the row tiles of one meet in one XCD's L2 where their number is a multiple of 8)
        return list.find(p, in_head, lane, it);
    };

    // ---- an item, worked out ahead of its turn
    struct Plan {
        int b, g, n_seg, part, s0;
        int M, row0, t_begin, t_end;
        int diagonal;           // from this tile on there are keys that some row does not see
        int t_plain, t_seen;    // tiles that every row of this wavefront sees whole; tiles that any of them sees
        int page;               // of the first tile
        int row[2], pos[2];     // of this lane's row in each block (lanes past the last row repeat it)
        int entries;            // block table from that page on, a lane each
    } now, ahead;
    auto plan_item = [&](Plan *n) __attribute__((always_inline)) {
        Item it;
        if (!next_item(&it, &n->g)) return false;
        n->b = it.b;
        n->n_seg = it.n_seg;
        n->part = it.part;
        n->s0 = it.s.s0;
        n->M = it.s.n * p.G;
        const int tile0 = it.rt * ROWS;
        n->row0 = tile0 + 64 * wave;
        auto position = [&](int row) { return min(it.s.L + by_group(p, row), it.s.keys - 1); };
        const int kt = uniform(position(min(tile0 + ROWS, n->M) - 1)) / KT + 1;          // key tiles that some row of this tile sees
        const int seg = uniform((kt + it.n_seg - 1) / it.n_seg);
        n->t_begin = uniform(min(kt, it.seg * seg));
        n->t_end = uniform(min(kt, n->t_begin + seg));
        n->diagonal = (uniform(position(tile0)) + 1) / KT;
        const bool active = n->row0 < n->M;
        n->t_plain = active ? max(n->t_begin, min(n->t_end, (uniform(position(n->row0)) + 1) / KT)) : n->t_begin;
        n->t_seen = active ? max(n->t_begin, min(n->t_end, uniform(position(min(n->row0 + 64, n->M) - 1)) / KT + 1)) : n->t_begin;
        n->page = uniform(n->t_begin * KT / page_size);
        n->entries = p.block_table[(size_t)it.b * p.max_pages + min(n->page + lane, (p.L_stride - 1) / page_size)];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            n->row[x] = max(0, min(n->row0 + 32 * x + l32, n->M - 1));
            n->pos[x] = position(n->row[x]);
        }
        return true;
    };

    // ---- requests: this wavefront's 8 rows of K and of V of a tile, four loads.  Past the end the last tile is asked for again, so that what
    // is waited for can be counted.
    const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint32_t *)s_ring;
    const uint32_t row_off = (uint32_t)lj * ROW_BYTES;
    const uint32_t k_off0 = row_off + 16 * (lc ^ ((8 * wave + lj) & 15)), k_off1 = row_off + 16 * (lc ^ ((8 * wave + 4 + lj) & 15));
    const uint32_t v_off = row_off + 16 * (lc ^ (4 * lj));
    const size_t page_bytes = (size_t)H_kv * page_size * ROW_BYTES;
    const char *zeros = reinterpret_cast<const char *>(zero_rows);
    asm volatile("" : "+s"(zeros));
    const char *k_head = nullptr, *v_head = nullptr, *k_at = nullptr, *v_at = nullptr;
    int ask = 0, ask_page = 0, ask_row = 0, entries = -1, n_entry = 0, entry = -1;
    // works out, among the matrix instructions, where the next tile lies
    auto advance = [&]() __attribute__((always_inline)) {
        ++ask;
        if (ask < now.t_end) {
            ask_row += KT;
            if (ask_row >= page_size) {
                ask_row = 0;
                if (++n_entry == 64) {
                    n_entry = 0;
                    ask_page += 64;
                    entries = p.block_table[(size_t)now.b * p.max_pages + min(ask_page + lane, (p.L_stride - 1) / page_size)];
                    asm volatile("s_waitcnt vmcnt(0)" : "+v"(entries) :: "memory");     // (here, not in the loop)
                }
                entry = uniform(__builtin_amdgcn_readlane(entries, n_entry));
            }
        }
        const bool in = (unsigned)entry < (unsigned)p.n_pages;
        const size_t at = (size_t)(uint32_t)entry * page_bytes + (uint32_t)ask_row * ROW_BYTES;
        k_at = in ? k_head + at : zeros;
        v_at = in ? v_head + at : zeros;
    };
    auto request = [&]() __attribute__((always_inline)) {
        const uint32_t to = ring_at + (ask & (DEPTH - 1)) * TILE_BYTES + wave * (8 * ROW_BYTES);
        fetch(to, k_at, k_off0, k_off1);
        fetch(to + SIDE_BYTES, v_at, v_off, v_off);
    };
    auto begin_item = [&]() __attribute__((always_inline)) {
        // (scalars again: what the compiler keeps between items in vector registers would bring vector arithmetic into the loops)
        now.b = uniform(now.b);
        now.g = uniform(now.g);
        now.t_begin = uniform(now.t_begin);
        now.t_end = uniform(now.t_end);
        now.t_plain = uniform(now.t_plain);
        now.t_seen = uniform(now.t_seen);
        now.diagonal = uniform(now.diagonal);
        now.page = uniform(now.page);
        entries = now.entries;
        asm volatile("" : "+v"(entries));
        if (now.t_begin < now.t_end) {
            const size_t head_at = ((size_t)now.g * page_size + 8 * wave) * ROW_BYTES;
            k_head = static_cast<const char *>(p.k_pool) + head_at;
            v_head = static_cast<const char *>(p.v_pool) + head_at;
            ask = uniform(now.t_begin) - 1;
            ask_row = now.t_begin * KT - now.page * page_size - KT;
            ask_page = now.page;
            n_entry = 0;
            entry = uniform(__builtin_amdgcn_readlane(entries, 0));
            advance();
#pragma unroll
            for (int i = 0; i < DEPTH - 1; ++i) { request(); advance(); }
        }
    };
    // ---- Q of an item: into this wavefront's part of LDS (16 loads of four rows each, permuted as K is), then as operands: lane holds
    // Q[row][16 kk + 8 h .. + 7] of a row of each block.  (Loaded as operands, 32 bytes of each of 32 rows at a time, the 64 KB of a
    // workgroup took 2.4 us.)  Rows past the last one repeat it.
    constexpr int Q_LOADS = 16;
    char *const my_rows = reinterpret_cast<char *>(s_rows[wave]);
    const uint32_t rows_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint32_t *)s_rows[wave];
    bf16x8 q[2][8];
    auto fetch_q = [&](const Plan &n) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < Q_LOADS; ++i) {
            const int r = max(0, min(n.row0 + 4 * i + lj, n.M - 1)), token = by_group(p, r);
            const char *src = static_cast<const char *>(p.q) + (size_t)(n.s0 + token) * p.q_row + (size_t)(n.g * p.G + r - token * p.G) * ROW_BYTES + 16 * (lc ^ ((4 * i + lj) & 15));
            fetch_from(rows_at + 4 * i * ROW_BYTES, src);
            __builtin_amdgcn_sched_barrier(0);      // (or all addresses are held at once)
        }
    };
    auto read_q = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {
                q[x][kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(my_rows + (32 * x + l32) * ROW_BYTES + ((16 * (h ^ (l32 & 15))) ^ (32 * kk))));
            }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+a"(q[x][kk]));
    };

    f32x16 o[2][4], s[2];
    float m_used[2], l_part[2];
    bf16x8 w[2][2];             // packed weights
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
    bf16x8 k[8], v[2][4];       // operands of a tile of K, of a tile of V
    auto read_k = [&](const int kk, int t) __attribute__((always_inline)) {
        k[kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(ring + (t & (DEPTH - 1)) * TILE_BYTES + (k_ld ^ (32 * kk))));
    };
    auto read_v = [&](const int m, const int nt, int t) __attribute__((always_inline)) {
        const char *from = ring + (t & (DEPTH - 1)) * TILE_BYTES + v_ld[nt] + 16 * m * ROW_BYTES;
        const v4i16 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)from);
        const v4i16 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(from + 8 * ROW_BYTES));
        v[m][nt] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // Weights of block x from its scores of tile t: two at a time (pair), which join the sum and are packed a step later (fold), so that nothing
    // waits for an exponential.
    float we[16];
    auto pair = [&](const int x, const int j, int t, auto masked) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 2 * j; i < 2 * j + 2; ++i) {
            we[i] = fast_exp2(fmaf(s[x][i], c2, -m_used[x]));
            if (decltype(masked)::value && key_of_score(i) > now.pos[x] - t * KT - 4 * h) we[i] = 0.f;
        }
    };
    auto fold = [&](const int j, float &sum, u32x4 *pk) __attribute__((always_inline)) {
        sum += we[2 * j] + we[2 * j + 1];
        pk[j / 4][j % 4] = pack_bf16(we[2 * j], we[2 * j + 1]);
    };
    auto weights = [&](const int x, int t, auto masked, u32x4 *pk) __attribute__((always_inline)) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) { pair(x, j, t, masked); fold(j, sum, pk); }
        return sum;
    };
    // The maximum is raised only where the weights outgrow it (their sum, which is formed anyway, tells), row by row.
    auto settle = [&](const int x, int t, auto masked, float sum, u32x4 *pk) __attribute__((always_inline)) {
        if (__builtin_expect(__any(!(sum <= 4096.f)), 0)) {
            const int seen = now.pos[x] - t * KT - 4 * h;
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
    auto pv = [&](const int x, const int m, const int nt) __attribute__((always_inline)) {
        o[x][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[m][nt], w[x][m], o[x][nt], 0, 0, 0);
    };
    auto zero_scores = [&](const int x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = 0.f;
    };
    auto qk = [&](const int x, const int kk) __attribute__((always_inline)) {
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kk], q[x][kk], s[x], 0, 0, 0);
    };

    // ---- steps
    // Where rows do not see all keys, a value that is no number would reach them: 0 times it is none either.  An item whose results hold
    // such a value is done again, with such values of these tiles as zeros, and the epilogue adds them to the rows that see
    // them.  A wavefront looks at its own rows of a tile; an exponent of all ones carries into the bit above it.
    auto mine_of = [&](int t) __attribute__((always_inline)) { return const_cast<char *>(ring) + (t & (DEPTH - 1)) * TILE_BYTES + SIDE_BYTES + wave * (8 * ROW_BYTES) + 16 * lane; };
    auto clean = [&](int t) __attribute__((always_inline)) {
        if (t < now.diagonal || t >= now.t_end) return;
        const u32x4 x[2] = {*reinterpret_cast<const u32x4 *>(mine_of(t)), *reinterpret_cast<const u32x4 *>(mine_of(t) + 4 * ROW_BYTES)};
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) any |= (x[i / 4][i % 4] & 0x7f807f80u) + 0x00800080u;
        if (__builtin_expect((any & 0x80008000u) != 0, 0)) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u32x4 y;
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = x[j][i] & ~(((((x[j][i] & 0x7f807f80u) + 0x00800080u) >> 15) & 0x00010001u) * 0xffffu);
                *reinterpret_cast<u32x4 *>(mine_of(t) + 4 * j * ROW_BYTES) = y;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    // Ahead of it: tile t + 1 has arrived (4 loads per tile, those of t + 2 may still be on their way); behind the barrier: everybody's part of
    // it.  What lay where t + 3 goes, t - 1, was last read ahead of it.
    int behind_q = 0;
    auto arrival = [&]() __attribute__((always_inline)) {
        if (behind_q > 0) {         // (the next item's Q was asked for behind t + 2)
            --behind_q;
            asm volatile("s_waitcnt vmcnt(%0)" :: "n"(4 + Q_LOADS) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
        }
        __builtin_amdgcn_s_barrier();
        request();
    };
    // One tile: k, v hold K(t) and V(t - 1), afterwards K(t + 1) and V(t); each operand is replaced as soon as block B has used it.
    // partial: some row may not see all of its keys.
    auto step = [&](int t, auto partial) __attribute__((always_inline)) {
        u32x4 pk[2];
        float sum = 0.f;
        zero_scores(1);
        // (products that need nothing of what the barrier stands for run while it is waited at)
#pragma unroll
        for (int i = 0; i < 2; ++i) { pv(1, 0, i); qk(1, i); }
        __builtin_amdgcn_sched_barrier(0);
        arrival();
        __builtin_amdgcn_sched_barrier(0);
        // A matrix instruction, the operands that take the place of an earlier one's, two weights: in this order, which the compiler would not find
        // by itself.
#pragma unroll
        for (int n = 4; n < 16; ++n) {
            const int i = n / 2;
            if (n % 2 == 0) pv(1, i / 4, i % 4);
            else qk(1, i);
            if (n < 12) {
                const int r = (n - 4) / 2;          // 0 .. 3
                if (n % 2 == 0) read_v(r / 4, r % 4, t);
                else read_k(r, t + 1);
            } else {
                const int r = n - 8;                // 4 .. 7
                read_v(r / 4, r % 4, t);
                if (n > 12) read_k(r - 1, t + 1);
                if (n == 15) read_k(7, t + 1);
            }
            if (n < 12) pair(0, n - 4, t, partial);
            if (n > 4 && n < 13) fold(n - 5, sum, pk);
            __builtin_amdgcn_sched_barrier(0);
        }
        settle(0, t, partial, sum, pk);
        advance();
        sum = 0.f;
        zero_scores(0);
#pragma unroll
        for (int n = 0; n < 16; ++n) {
            const int i = n / 2;
            if (n % 2 == 0) pv(0, i / 4, i % 4);
            else qk(0, i);
            if (n > 1 && n < 10) pair(1, n - 2, t, partial);
            if (n > 2 && n < 11) fold(n - 3, sum, pk);
            __builtin_amdgcn_sched_barrier(0);
        }
        settle(1, t, partial, sum, pk);
    };
    if (tid < 2) s_odd[tid] = 0;
    bool more = plan_item(&ahead), done = false, direct = false, poisoned = false, mine[2] = {false, false};    // an item is done, and what its epilogue needs
    int done_b = 0, done_g = 0, done_s0 = 0, done_row0 = 0, done_M = 0, key_from = 0, key_end = 0, done_pos[2] = {0, 0};
    size_t at[2] = {0, 0};      // row of out and lse, or of the partial results
    // ---- epilogue: a lane holds columns 32 nt + 8 a + 4 h .. + 3 of its row in each block
    auto epilogue = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float l_row = l_part[x] + __shfl_xor(l_part[x], 32);
            if (direct) {
                // through LDS, so that whole rows go out (16-byte pieces permuted as K's are)
                const float f = 1.0f / l_row;
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
                        *reinterpret_cast<u32x4 *>(my_rows + (32 * x + l32) * ROW_BYTES + 16 * ((4 * nt + a + h) ^ (l32 & 15))) = y;
                    }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 4 * i + lj;
                    const int row = done_row0 + 32 * x + r, token = by_group(p, row);
                    const u32x4 y = *reinterpret_cast<const u32x4 *>(my_rows + (32 * x + r) * ROW_BYTES + 16 * (lc ^ (r & 15)));
                    if (row < done_M)
                        *reinterpret_cast<u32x4 *>(static_cast<char *>(p.out) + ((size_t)(done_s0 + token) * p.H_q + (done_g * p.G + row - token * p.G)) * ROW_BYTES + 16 * lc) = y;
                }
                if (p.lse && h == 0 && mine[x]) p.lse[at[x]] = (m_used[x] + __builtin_amdgcn_logf(l_row)) * LN2_F;
            } else if (mine[x]) {
                if (h == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at[x]) = make_float2(m_used[x], l_row);
                float *dst = p.part_o + at[x] * D;
#pragma unroll
                for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                    for (int a = 0; a < 4; ++a)
                        *reinterpret_cast<float4 *>(dst + 32 * nt + 8 * a + 4 * h) = make_float4(o[x][nt][4 * a], o[x][nt][4 * a + 1], o[x][nt][4 * a + 2], o[x][nt][4 * a + 3]);
            }
            if (__builtin_expect(poisoned, 0) && mine[x]) {
                // what is no number joins what was written, lane l32 + 32 h takes columns 64 h .. 64 h + 63
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                for (int key = key_from; key <= min(done_pos[x], key_end); ++key) {
                    const int page = p.block_table[(size_t)done_b * p.max_pages + key / page_size];
                    if ((unsigned)page >= (unsigned)p.n_pages) continue;
                    const uint16_t *v = static_cast<const uint16_t *>(p.v_pool) + (((size_t)page * H_kv + done_g) * page_size + key % page_size) * D;
                    for (int c = 64 * h; c < 64 * h + 64; ++c) {
                        const float y = bf16_bits_to_float(v[c]);
                        if (fabsf(y) < INFINITY) continue;
                        if (direct) {
                            volatile uint16_t *z = static_cast<uint16_t *>(p.out) + at[x] * D + c;
                            *z = (uint16_t)pack_bf16(bf16_bits_to_float(*z) + y, 0.f);
                        } else {
                            volatile float *z = p.part_o + at[x] * D + c;
                            *z = *z + y;
                        }
                    }
                }
            }
        }
    };
    if (more) {
        now = ahead;
        fetch_q(now);
        if (tid == 0) s_next = (int)gridDim.x + atomicAdd(&p.notes->taken, 1);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
    for (int pass = 0;; ++pass) {
        const bool here = uniform(more) != 0;
        if (here) {
            begin_item();
            read_q();           // (arrived during the item before)
        }
        if (done) epilogue();
        if (!here) break;
        // the next item and its Q, while the first tiles are on their way
        next = uniform(s_next);
        more = plan_item(&ahead);
        if (more) fetch_q(ahead);
        behind_q = uniform(more ? 2 : 0);
        int careful = 0;            // (the item is done a second time)
        for (;; ++pass) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[x][nt][i] = 0.f;
                const u32x4 zero = {0, 0, 0, 0};
                w[x][0] = w[x][1] = __builtin_bit_cast(bf16x8, zero);
                m_used[x] = M_INIT;
                l_part[x] = 0.f;
            }
            if (behind_q) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(Q_LOADS) : "memory");       // (the first tiles)
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            int t = now.t_begin;
            if (careful) clean(t);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (tid == 0) s_odd[(pass + 1) & 1] = 0;            // (whoever read it is past this barrier)
            if (t < now.t_seen) {
                const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i / 4][i % 4] = __builtin_bit_cast(bf16x8, zero);
#pragma unroll
                for (int i = 0; i < 8; ++i) read_k(i, t);
                zero_scores(0);
#pragma unroll
                for (int i = 0; i < 8; ++i) qk(0, i);
                asm volatile(".p2align 6");             // (the loop starts on an instruction-cache line)
                if (!careful)
                    for (; t < now.t_plain; ++t) step(t, std::false_type());
                for (; t < now.t_seen; ++t) {
                    step(t, std::true_type());
                    if (careful) clean(t + 1);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) pv(1, i / 4, i % 4);
            }
            int taken = 0;
            if (!careful)
                if (tid == 0) taken = atomicAdd(&p.notes->taken, 1);
            for (; t < now.t_end; ++t) {                        // (this wavefront only helps to load)
                arrival();
                advance();
                if (careful) clean(t + 1);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // (nothing is on its way into LDS any more)
            if (!careful) {
                if (tid == 0) s_next = (int)gridDim.x + taken;
                float sum = 0.f;
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int nt = 0; nt < 4; ++nt)
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum = fmaf(o[x][nt][i], 0.f, sum);         // (0 times it is 0, or no number)
                if (__any(sum != 0.f) && lane == 0) s_odd[pass & 1] = 1;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (careful || !uniform(s_odd[pass & 1])) break;
            careful = 1;
            behind_q = 0;
            begin_item();
        }

        done = true;
        direct = now.n_seg == 1;
        poisoned = careful != 0;
        done_b = now.b;
        done_g = now.g;
        done_s0 = now.s0;
        done_row0 = now.row0;
        done_M = now.M;
        key_from = max(now.diagonal, now.t_begin) * KT;
        key_end = now.t_end * KT - 1;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            mine[x] = now.row0 + 32 * x + l32 < now.M;
            done_pos[x] = now.pos[x];
            const int token = by_group(p, now.row[x]);
            at[x] = direct ? (size_t)(now.s0 + token) * p.H_q + (now.g * p.G + now.row[x] - token * p.G)
                           : ((size_t)(now.part + 2 * wave + x) * H_kv + now.g) * 32 + l32;
        }
        if (more) now = ahead;
    }
}

}  // namespace

void launch_chunk_wide(const ChunkParams &p, int max_items, hipStream_t stream)
{
    launch_kernel(K_CHUNK_WIDE, chunk_wide_kernel, dim3(min(p.H_kv * max_items, 256)), dim3(256), stream, p);
}

}  // namespace mcsd
