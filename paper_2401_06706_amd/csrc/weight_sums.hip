// What every cached position was given by the softmax of new rows, added up (the measure by which a cache is cut).
#include "chunk_common.h"

namespace mcsd {
namespace {

struct SumsParams { ChunkParams c; const float *lse; float *sums; int last_rows, blocks; };

// A workgroup owns 128 positions of a (sequence, KV head) at a time, 32 a wavefront with their keys in registers, and goes through the rows
// that see them in tiles of 32 (through LDS): S = K Q^T as in attention, weights 2^(s c2 - lse), added up in the
// lane that holds them.  No other workgroup adds to these positions, so the order of the sum is fixed.  A partial sum of 64 tiles is
// added to the whole at a time: over n tiles the error stays below (64 + n / 64) 2^-24 of the sum.
// Few rows: a workgroup goes through `blocks` of 128 positions, the next one's keys asked for ahead, so that lengths, table and rows are
// waited for once.  Bound by the reading of the keys: 32 sequences of 100 to 8000 tokens, 32/8 heads, d = 128, one new token 70 us (278 MB, 4.0 TB/s);
// many rows by launch, trips to memory, exponentials and products in turn: 64 tokens on 4 x 3000 to 8000 29 to 33 us (1.1 times 10^10 products' operations), all rows
// of 8 prompts of 1000 to 2048 244 us.  Workgroups are those of the capacity, and find nothing behind a sequence's end: the first of these with room for 8000, 32768 and
// 131072 tokens a sequence 69, 70, 77 us.
template <int DP, bool F32, bool MULTI>
__global__ __launch_bounds__(256, DP * (F32 ? 4 : 2) <= 256 ? 3 : 1) void weight_sums_kernel(SumsParams sp)
{
    using S = TileShape<DP, F32>;
    const ChunkParams &p = sp.c;
    __shared__ __attribute__((aligned(16))) uint32_t s_q[2][KT * S::PK];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, l32 = lane & 31;
    const int g = blockIdx.x, b = blockIdx.z, blocks = MULTI ? sp.blocks : 1, key0 = blockIdx.y * 128 * blocks;
    const ChunkSeq sq = chunk_sequence(p, b);
    if (sq.n == 0 || key0 >= sq.keys) return;
    const int M = sq.n * p.G, row_bytes = p.d * S::ES;
    const int first_token = max(sp.last_rows ? sq.n - min(sp.last_rows, sq.n) : 0, key0 - sq.L);
    const int row_first = first_token * p.G, tiles = (M - row_first + KT - 1) / KT;

    // ---- keys of a block
    auto load_keys = [&](int wkey, u32x4 *k) __attribute__((always_inline)) {
        const int page = wkey < sq.keys ? p.block_table[(size_t)b * p.max_pages + wkey / p.page_size] : -1;
        const bool in = (unsigned)page < (unsigned)p.n_pages;
        const size_t off = in ? (((size_t)page * p.H_kv + g) * p.page_size + wkey % p.page_size) * row_bytes : 0;
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(static_cast<const char *>(p.k_pool) + off, in ? (uint32_t)min(KT, sq.keys - wkey) * row_bytes : 0u);
#pragma unroll
        for (int kk = 0; kk < S::KK; ++kk) {
            const int at = 32 * kk + 16 * h;
            k[kk] = __builtin_amdgcn_raw_buffer_load_b128(rk, at < row_bytes ? l32 * row_bytes + at : 0x7fff0000, 0, 0);
        }
    };
    // ---- tiles of rows: global -> registers -> LDS, two tiles ahead
    u32x4 qr[2][S::PER_THREAD];
    float lse_of[2];
    auto load_q = [&](int tile, int st) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < S::PER_THREAD; ++j) {
            const int e = tid + 256 * j, r = row_first + tile * KT + e / S::GRANULES, c = e % S::GRANULES;
            const u32x4 zero = {0, 0, 0, 0};
            qr[st][j] = zero;
            if (e < KT * S::GRANULES && r < M && 16 * c < row_bytes) {
                const int token = by_group(p, r);
                qr[st][j] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(p.q) + (size_t)(sq.s0 + token) * p.q_row +
                                                             (size_t)(g * p.G + r - token * p.G) * row_bytes + 16 * c);
            }
        }
        const int r = row_first + tile * KT + l32;
        lse_of[st] = 0.f;
        if (r < M) {
            const int token = by_group(p, r);
            lse_of[st] = sp.lse[(size_t)(sq.s0 + token) * p.H_q + g * p.G + r - token * p.G] * LOG2E_F;
        }
    };
    auto store_q = [&](int st) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < S::PER_THREAD; ++j) {
            const int e = tid + 256 * j;
            if (KT * S::GRANULES % 256 == 0 || e < KT * S::GRANULES)
                *reinterpret_cast<u32x4 *>(s_q[st] + e / S::GRANULES * S::PK + 4 * (e % S::GRANULES)) = qr[st][j];
        }
    };
    u32x4 k[S::KK], k_next[S::KK];
    load_keys(key0 + 32 * wave, k);
    load_q(0, 0);
    float first_lse = lse_of[0];
    store_q(0);
    for (int block = 0; block < blocks && key0 + 128 * block < sq.keys; ++block) {
        const int wkey = key0 + 128 * block + 32 * wave;
        if (MULTI && block + 1 < blocks) load_keys(wkey + 128, k_next);
        // (lane l32 < 16 ends up with this position, see below; what it held is asked for now)
        const int mine = 8 * (l32 & 1) + 4 * ((l32 >> 1) & 1) + 2 * ((l32 >> 2) & 1) + ((l32 >> 3) & 1);
        const int key = wkey + key_of_score(mine) + 4 * h;
        float *const at = sp.sums + ((size_t)b * p.H_kv + g) * p.L_stride + key;
        const bool writes = l32 < 16 && key < sq.keys;
        const float old = writes && key < sq.L ? *at : 0.f;
        float part[16], total[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) part[i] = total[i] = 0.f;
        auto step = [&](int tile, const int st, float lse) __attribute__((always_inline)) {
            if (wkey < sq.keys) {
                const uint32_t *qb = s_q[st] + l32 * S::PK + 4 * h;
                f32x16 s;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
                for (int kk = 0; kk < S::KK; ++kk) {
                    const u32x4 a = *reinterpret_cast<const u32x4 *>(qb + 8 * kk);
                    if constexpr (F32) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[kk][j]), __uint_as_float(a[j]), s, 0, 0, 0);
                    } else {
                        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[kk]), __builtin_bit_cast(bf16x8, a), s, 0, 0, 0);
                    }
                }
                const int row0 = row_first + tile * KT;
                // Some row does not see some of these keys, or stands past the last one: that sees none (its zeros times an infinity in a key would be
                // no number).
                if (min(sq.L + by_group(p, row0), sq.keys - 1) < wkey + KT - 1 || row0 + KT > M) {
                    const int seen = row0 + l32 < M ? min(sq.L + by_group(p, row0 + l32), sq.keys - 1) - wkey - 4 * h : -1;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (key_of_score(i) <= seen) part[i] += fast_exp2(fmaf(s[i], p.scale_log2, -lse));
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) part[i] += fast_exp2(fmaf(s[i], p.scale_log2, -lse));
                }
                if ((tile & 63) == 63) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) { total[i] += part[i]; part[i] = 0.f; }
                }
            }
        };
        if (tiles == 1) {
            if (block == 0) __syncthreads();
            step(0, 0, first_lse);
        } else if (MULTI) {
            // (a sequence with more rows than most: without look-ahead)
            for (int tile = 0; tile < tiles; ++tile) {
                if (block + tile > 0) { load_q(tile, 0); store_q(0); }
                const float lse = lse_of[0];
                __syncthreads();
                step(tile, 0, lse);
                __syncthreads();
            }
        } else {
            load_q(1, 1);
            float lse = lse_of[0];
            __syncthreads();
            // tile t in buffer t % 2; t + 1 is stored, and t + 2 asked for, while it is worked on
            for (int tile = 0; tile < tiles; tile += 2) {
                float lse1 = lse_of[1];
                store_q(1);
                if (tile + 2 < tiles) load_q(tile + 2, 0);
                step(tile, 0, lse);
                __syncthreads();
                if (tile + 1 >= tiles) break;
                lse = lse_of[0];
                if (tile + 2 < tiles) store_q(0);
                if (tile + 3 < tiles) load_q(tile + 3, 1);
                step(tile + 1, 1, lse1);
                __syncthreads();
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) total[i] += part[i];
        // sum over the 32 rows of a tile: every exchange halves what a lane holds, so that lane l32 ends up with score
        // 8 (l32 & 1) + 4 (l32 >> 1 & 1) + 2 (l32 >> 2 & 1) + (l32 >> 3 & 1) of its half
#pragma unroll
        for (int bit = 0; bit < 4; ++bit) {
            const int n = 8 >> bit;
            const bool up = (lane >> bit) & 1;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) {
                    const float keep = up ? total[j + n] : total[j], give = up ? total[j] : total[j + n];
                    total[j] = keep + __shfl_xor(give, 1 << bit);
                }
        }
        total[0] += __shfl_xor(total[0], 16);
        if (writes) *at = old + total[0];
        if (MULTI)
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk) k[kk] = k_next[kk];
    }
}

template <bool F32, bool MULTI>
void launch_type(const SumsParams &sp, hipStream_t stream)
{
    const dim3 grid(sp.c.H_kv, (sp.c.L_stride + 128 * sp.blocks - 1) / (128 * sp.blocks), sp.c.B), block(256);
    const int d = sp.c.d;
    if (d <= 32) launch_kernel(K_WEIGHT_SUMS, weight_sums_kernel<32, F32, MULTI>, grid, block, stream, sp);
    else if (d <= 64) launch_kernel(K_WEIGHT_SUMS, weight_sums_kernel<64, F32, MULTI>, grid, block, stream, sp);
    else if (d <= 96) launch_kernel(K_WEIGHT_SUMS, weight_sums_kernel<96, F32, MULTI>, grid, block, stream, sp);
    else if (d <= 128) launch_kernel(K_WEIGHT_SUMS, weight_sums_kernel<128, F32, MULTI>, grid, block, stream, sp);
    else launch_kernel(K_WEIGHT_SUMS, weight_sums_kernel<256, F32, MULTI>, grid, block, stream, sp);
}

}  // namespace

int32_t launch_weight_sums(const mcsd_chunk_desc &d, const mcsd_sums_bufs &b, const mcsd_paged_kv &kv, hipStream_t stream)
{
    SumsParams sp;
    sp.c = chunk_params(d, kv);
    sp.c.q = b.q; sp.c.k_pool = b.k_pool; sp.c.chunk_start = b.chunk_start; sp.c.prefix_len = b.prefix_len;
    sp.lse = b.lse; sp.sums = b.sums; sp.last_rows = b.last_rows;
    // Several blocks a workgroup where sequences bring up to two tiles of rows on average and workgroups are plenty, us with them and without: 32 sequences of
    // 100 to 8000 tokens, one new, 32/8 heads 73.3, 75.0; 16 of 2000 to 8000 46.2, 49.2; 8 new tokens on 32 x 8000 125, 138; 64 of 100 to 4000, which the rule
    // takes too, 78.3, 75.9.
    const long rows = (long)d.T * (d.H_q / d.H_kv), groups = (long)d.H_kv * d.B * ((d.L_stride + 127) / 128);
    sp.blocks = rows <= 64L * d.B ? (groups >= 8192 ? 4 : groups >= 4096 ? 2 : 1) : 1;
    if (d.dtype == MCSD_DTYPE_FP32) sp.blocks > 1 ? launch_type<true, true>(sp, stream) : launch_type<true, false>(sp, stream);
    else sp.blocks > 1 ? launch_type<false, true>(sp, stream) : launch_type<false, false>(sp, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("weight sums launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
