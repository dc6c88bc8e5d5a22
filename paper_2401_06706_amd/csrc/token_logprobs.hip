// Log probability, rank and entropy for given tokens, with the most probable alternatives.
#include <float.h>
#include <algorithm>
#include <type_traits>

#include "attn_common.h"
#include "vocab_row.h"

namespace mcsd {
namespace {

struct LogprobParams {
    int rows, R, V, n_top;
    size_t row_stride;              // elements
    const void *logits;
    const int32_t *row_map, *tokens;
    const float *temperature;
    float *logprob, *entropy, *top_logprob;
    int32_t *rank, *top_tok;
    uint32_t *flags;
    int bf16;
    int parts;                      // workgroups of a row; more than one: their results go to
    struct RowPart *part;           // [rows][parts]
    float *part_logit;              // [rows][parts][n_top], in order
    int32_t *part_tok;
};

// what a workgroup found in its part of a row: the largest logit, sums relative to it, tokens that come before the given one
struct RowPart { double s, u; float m; int before; };

constexpr int MAX_PARTS = 16;
constexpr int CAP = 1024;         // candidates for the top that fit; those equal to the smallest of them
constexpr float LOWEST = -200.0f;           // 2^-200 is 0: a bound that keeps 0 * infinity out of the entropy

// log2(e) / T; finite, so that 0 times it is 0, and not 0, so that -infinity times it is -infinity (an infinite temperature: what is not masked is alike)
__device__ __forceinline__ float scale_of(float T) { return fmaxf(fminf(LOG2E_F / (T > 0.f ? T : 1.f), FLT_MAX), FLT_TRUE_MIN); }

template <bool BF16>
__device__ __forceinline__ float logit_at(const void *row, int i)
{
    return BF16 ? bf16_bits_to_float(static_cast<const uint16_t *>(row)[i]) : static_cast<const float *>(row)[i];
}

// Where 16-byte pieces begin and end in a row that starts anywhere: elements [0, head), pieces, elements [tail, V).
template <bool BF16>
struct Pieces {
    static constexpr int W = BF16 ? 8 : 4;
    int head, n, tail;
    __device__ __forceinline__ Pieces(const void *row, int V)
    {
        const int es = BF16 ? 2 : 4, off = (int)((16 - ((uintptr_t)row & 15u)) & 15u) / es;
        head = min(off, V);
        n = (V - head) / W;
        tail = head + n * W;
    }
    __device__ __forceinline__ u32x4 raw(const void *row, int piece) const
    {
        return *reinterpret_cast<const u32x4 *>(static_cast<const char *>(row) + (size_t)(head + piece * W) * (BF16 ? 2 : 4));
    }
    __device__ __forceinline__ void values(const u32x4 &x, float *z) const
    {
#pragma unroll
        for (int i = 0; i < W; ++i)
            z[i] = BF16 ? ((i & 1) ? __uint_as_float(x[i >> 1] & 0xffff0000u) : __uint_as_float(x[i >> 1] << 16)) : __uint_as_float(x[i & 3]);
    }
    __device__ __forceinline__ void load(const void *row, int piece, float *z) const { values(raw(row, piece), z); }
};

// Sums of a row relative to the largest logit seen: s = sum 2^t, u = sum t 2^t with t = (z - m) c, c = log2(e) / T.
struct Sums {
    float m = -FLT_MAX, s = 0.f, u = 0.f;
    __device__ __forceinline__ void raise(float to, float c)
    {
        const float t = fmaxf((m - to) * c, LOWEST), f = fast_exp2(t);
        u = f * (u + t * s);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void add(float z, float c)
    {
        const float t = (z - m) * c, e = fast_exp2(t);
        s += e;
        u = fmaf(e, fmaxf(t, LOWEST), u);
    }
};

// A workgroup per row, which is read once: every thread keeps running sums, its largest logit and how many tokens come before the given
// one.  For the top, the n-th largest of 64 maxima (of groups of threads) bounds it from below: only the few threads whose
// largest logit reaches that bound have the piece that holds it read again, or all of theirs where another reaches it too, by all threads together.
// PART: of few long rows a workgroup takes a part, as if it were the row, and token_logprobs_merge_kernel joins what they found.
template <bool BF16, int NT, int AHEAD, bool PART>
__global__ __launch_bounds__(NT) void token_logprobs_kernel(LogprobParams p)
{
    constexpr int W = Pieces<BF16>::W, WAVES = NT / 64;
    __shared__ float s_max[NT];
    __shared__ double s_sum[2][WAVES];
    __shared__ int s_rank[WAVES], s_hot[NT], s_one[NT], s_n_hot, s_n_one, s_n_above, s_n_equal;
    __shared__ float s_val[CAP];
    __shared__ int s_id[CAP], s_eq[CAP];
    static_assert(WAVES <= CAP, "");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i_row = blockIdx.x;
    const int map = p.row_map ? p.row_map[i_row] : i_row;
    auto refuse = [&](uint32_t flag) {
        if (tid == 0) {
            p.logprob[i_row] = NAN;
            if (p.entropy) p.entropy[i_row] = NAN;
            if (p.rank) p.rank[i_row] = -1;
            p.flags[i_row] = flag;
        }
        if (tid < p.n_top) {
            p.top_tok[(size_t)i_row * p.n_top + tid] = -1;
            p.top_logprob[(size_t)i_row * p.n_top + tid] = NAN;
        }
    };
    if ((unsigned)map >= (unsigned)p.R) return refuse(MCSD_FLAG_BAD_TREE);
    const void *row = static_cast<const char *>(p.logits) + (size_t)map * p.row_stride * (BF16 ? 2 : 4);
    const void *const whole_row = row;
    int V = p.V, from = 0;
    if (PART) {
        const Pieces<BF16> whole(row, V);
        auto begin = [&](int y) { return y == 0 ? 0 : y == p.parts ? V : whole.head + (int)((long)whole.n * y / p.parts) * W; };
        from = begin(blockIdx.y);
        V = begin(blockIdx.y + 1) - from;
        row = static_cast<const char *>(row) + (size_t)from * (BF16 ? 2 : 4);
    }
    const Pieces<BF16> pc(row, V);
    if (tid == 0) s_n_hot = s_n_one = s_n_above = s_n_equal = 0;

    Sums sums;
    float top = -INFINITY, second = -INFINITY;          // the largest logit of this thread's pieces, and of all of them but that one's
    int before = 0, top_piece = -1;
    // AHEAD pieces are under way at a time
    int piece = tid;
    u32x4 raw[AHEAD];
    auto ask = [&](int k, int piece) {
        if (piece < pc.n) raw[k] = pc.raw(row, piece);
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) raw[k] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) ask(k, piece + k * NT);         // (ahead of the token's logit)
    const int token = p.tokens[i_row], x = token - from;            // (in terms of the part)
    const bool known = (unsigned)token < (unsigned)p.V;
    const float zx = known ? logit_at<BF16>(whole_row, token) : INFINITY;
    const float zx_next = nextafterf(zx, INFINITY);         // z > zx is z >= zx_next
    const float T = p.temperature ? p.temperature[i_row] : 1.f, c = scale_of(T);
    auto most_of = [&](const float *z) {
        float most = z[0];
#pragma unroll
        for (int i = 1; i < W; ++i) most = fmaxf(most, z[i]);
        return most;
    };
    auto keep = [&](float most, int piece) {
        second = fmaxf(second, fminf(top, most));
        top_piece = most > top ? piece : top_piece;
        top = fmaxf(top, most);
    };
    // of a piece the logits from `least` on come before x; beside that, in the piece that holds x, those equal to it that stand before it
    auto least_of = [&](int piece) { return x - (pc.head + piece * W) >= W ? zx : zx_next; };
    auto own_piece = [&](const float *z, int piece) {
        const int d = x - (pc.head + piece * W);
        if (d > 0 && d < W) {
#pragma unroll
            for (int i = 0; i < W; ++i) before += z[i] == zx && i < d ? 1 : 0;
        }
    };
    // while all lanes have AHEAD pieces: the largest of them all first, so that the sums are raised once; tokens that come before x are counted for the wavefront
    int before_all = 0;
    for (int first = __builtin_amdgcn_readfirstlane(piece); first + 63 + (AHEAD - 1) * NT < pc.n; first += AHEAD * NT) {
        float z[AHEAD][W], most[AHEAD], all = -INFINITY;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            pc.values(raw[k], z[k]);
            ask(k, piece + (AHEAD + k) * NT);       // (the place of a piece that is taken is free for one of the next)
            most[k] = most_of(z[k]);
            all = fmaxf(all, most[k]);
        }
        if (all > sums.m) sums.raise(all, c);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int at = piece + k * NT;
            const float least = least_of(at);
            keep(most[k], at);
#pragma unroll
            for (int i = 0; i < W; ++i) {
                sums.add(z[k][i], c);
                before_all += __popcll(__ballot(z[k][i] >= least));
            }
            own_piece(z[k], at);
        }
        piece += AHEAD * NT;
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
        const int at = piece + k * NT;
        if (at < pc.n) {
            float z[W];
            pc.values(raw[k], z);
            const float most = most_of(z), least = least_of(at);
            if (most > sums.m) sums.raise(most, c);
            keep(most, at);
#pragma unroll
            for (int i = 0; i < W; ++i) {
                sums.add(z[i], c);
                before += z[i] >= least ? 1 : 0;
            }
            own_piece(z, at);
        }
    }
    float edge = -INFINITY;
    auto take = [&](float z, int id) {
        if (z > sums.m) sums.raise(z, c);
        edge = fmaxf(edge, z);
        sums.add(z, c);
        before += (z > zx || (z == zx && id < x)) ? 1 : 0;
    };
    // (elements outside the pieces: fewer than 16)
    if (tid < pc.head) take(logit_at<BF16>(row, tid), tid);
    if (pc.tail + tid < V) take(logit_at<BF16>(row, pc.tail + tid), pc.tail + tid);

    // ---- the row's sums
    s_max[tid] = fmaxf(top, edge);
    __syncthreads();
    float group = s_max[lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) group = fmaxf(group, s_max[64 * w + lane]);
    const float m = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vocab::wave_max(group)), 63));
    sums.raise(fmaxf(m, -FLT_MAX), c);
    double s = vocab::wave_sum(sums.s), u = vocab::wave_sum(sums.u);        // (in lane 63, as the count)
    before += __builtin_amdgcn_update_dpp(0, before, 0xB1, 0xf, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x4E, 0xf, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x141, 0xf, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x140, 0xf, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x142, 0xa, 0xf, false);
    before += __builtin_amdgcn_update_dpp(0, before, 0x143, 0xc, 0xf, false);
    if (lane == 63) { s_sum[0][wave] = s; s_sum[1][wave] = u; s_rank[wave] = before + before_all; }
    // ---- the bound of the top: n_top-th largest of the 64 maxima
    float bound = INFINITY;
    if (p.n_top) {
        int ahead = 0;
#pragma unroll
        for (int k = 0; k < 64; ++k) {
            const float other = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(group), k));
            ahead += (other > group || (other == group && k < lane)) ? 1 : 0;
        }
        const unsigned long long at = __ballot(ahead == p.n_top - 1);
        bound = __shfl(group, at ? __ffsll((long long)at) - 1 : 0);
        const float from_here = bound > -INFINITY ? bound : -FLT_MAX;        // (of masked tokens, where they are wanted, the first ones are looked for)
        if (second >= from_here) s_hot[atomicAdd(&s_n_hot, 1)] = tid;
        else if (top >= from_here) s_one[atomicAdd(&s_n_one, 1)] = top_piece;
    }
    __syncthreads();
    s = u = 0.0;
    before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { s += s_sum[0][w]; u += s_sum[1][w]; before += s_rank[w]; }
    // a NaN anywhere is in s; an infinity is the maximum
    const size_t part = (size_t)i_row * p.parts + blockIdx.y;
    if (PART) {
        if (tid == 0) p.part[part] = {s, u, m, before};
    } else if (!(s > 0.0 && s < (double)INFINITY) || !(m < INFINITY) || !(m > -INFINITY)) {
        return refuse(MCSD_FLAG_NONFINITE);
    }
    const double lse = log(s), to_ln = 1.0 / 1.44269504088896340736;
    const double inv_T = (double)c * to_ln;
    auto logprob_of = [&](float z) { return z == -INFINITY ? -INFINITY : (float)(((double)z - (double)m) * inv_T - lse); };
    if (!PART && tid == 0) {
        p.logprob[i_row] = known ? logprob_of(zx) : NAN;
        if (p.entropy) p.entropy[i_row] = (float)fmax(lse - u / s * to_ln, 0.0);
        if (p.rank) p.rank[i_row] = known ? before : -1;
        p.flags[i_row] = known ? 0u : (uint32_t)MCSD_FLAG_BAD_TOKEN;
    }
    if (!p.n_top) return;

    // ---- candidates: all that reach the bound
    auto candidate = [&](float z, int id) {
        if (z > bound) {
            const int at = atomicAdd(&s_n_above, 1);
            if (at < CAP) { s_val[at] = z; s_id[at] = id; }
        } else if (z == bound && bound > -INFINITY) {
            const int at = atomicAdd(&s_n_equal, 1);
            if (at < CAP) s_eq[at] = id;
        }
    };
    const int per = (pc.n + NT - 1) / NT, n_one = s_n_one, n_hot = s_n_hot;
    for (int k = tid; k < n_one + n_hot * per; k += NT) {
        const int j = k - n_one, piece = j < 0 ? s_one[k] : s_hot[j / per] + j % per * NT;
        if (piece >= pc.n) continue;
        float z[W];
        pc.load(row, piece, z);
#pragma unroll
        for (int i = 0; i < W; ++i) candidate(z[i], pc.head + piece * W + i);
    }
    if (tid < pc.head) candidate(logit_at<BF16>(row, tid), tid);
    if (pc.tail + tid < V) candidate(logit_at<BF16>(row, pc.tail + tid), pc.tail + tid);
    __syncthreads();
    int32_t *tok = PART ? p.part_tok + part * p.n_top : p.top_tok + (size_t)i_row * p.n_top;
    float *lp = PART ? p.part_logit + part * p.n_top : p.top_logprob + (size_t)i_row * p.n_top;
    auto put = [&](int place, int id, float z) { tok[place] = from + id; lp[place] = PART ? z : logprob_of(z); };
    const int above = s_n_above, equal = bound > -INFINITY ? s_n_equal : CAP + 1;
    if (above <= CAP) {
        // the place of each among them; up to 64 by one wavefront, from registers
        if (above <= 64) {
            if (wave == 0) {
                const float z = lane < above ? s_val[lane] : 0.f;
                const int id = lane < above ? s_id[lane] : 0;
                int place = 0;
                for (int j = 0; j < above; ++j) {
                    const float zj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(z), j));
                    const int idj = __builtin_amdgcn_readlane(id, j);
                    place += (zj > z || (zj == z && idj < id)) ? 1 : 0;
                }
                if (lane < above && place < p.n_top) put(place, id, z);
            }
        } else {
            for (int k = tid; k < above; k += NT) {
                const float z = s_val[k];
                const int id = s_id[k];
                int place = 0;
                for (int j = 0; j < above; ++j) place += (s_val[j] > z || (s_val[j] == z && s_id[j] < id)) ? 1 : 0;
                if (place < p.n_top) put(place, id, z);
            }
        }
        const int missing = p.n_top - above;            // of those equal to the bound, the lowest ids
        if (missing > 0 && equal <= CAP) {
            for (int k = tid; k < equal; k += NT) {
                const int id = s_eq[k];
                int place = 0;
                for (int j = 0; j < equal; ++j) place += s_eq[j] < id ? 1 : 0;
                if (place < missing) put(above + place, id, bound);
            }
        } else if (missing > 0 && wave == 0) {          // very many: looked for in the row, in order
            int found = 0;
            for (int base = 0; base < V && found < missing; base += 64) {
                const bool is = base + lane < V && logit_at<BF16>(row, base + lane) == bound;
                const unsigned long long who = __ballot(is);
                const int place = found + __popcll(who & ((1ull << lane) - 1));
                if (is && place < missing) put(above + place, base + lane, bound);
                found += __popcll(who);
            }
        }
        return;
    }
    // More than CAP above the bound (one thread's pieces hold them all): the top one by one, each the first behind the one before it.
    float last = INFINITY;
    int last_id = -1;
    for (int k = 0; k < p.n_top; ++k) {
        float best = -INFINITY;
        int best_id = 0x7fffffff;
        for (int i = tid; i < V; i += NT) {
            const float z = logit_at<BF16>(row, i);
            const bool behind = z < last || (z == last && i > last_id);
            if (behind && (z > best || (z == best && i < best_id))) { best = z; best_id = i; }
        }
#pragma unroll
        for (int q = 32; q > 0; q >>= 1) {
            const float z = __shfl_xor(best, q);
            const int id = __shfl_xor(best_id, q);
            if (z > best || (z == best && id < best_id)) { best = z; best_id = id; }
        }
        __syncthreads();
        if (lane == 0) { s_val[wave] = best; s_id[wave] = best_id; }
        __syncthreads();
        for (int w = 0; w < WAVES; ++w)
            if (s_val[w] > best || (s_val[w] == best && s_id[w] < best_id)) { best = s_val[w]; best_id = s_id[w]; }
        last = best;
        last_id = best_id;
        if (tid == 0) put(k, best_id, best);
    }
}

// The parts of a row: a workgroup a row.  A token's place among all lists is its place in its own and, in each other one (they are in order), how many
// come before it.
__global__ __launch_bounds__(256) void token_logprobs_merge_kernel(LogprobParams p)
{
    __shared__ float s_logit[MAX_PARTS * MCSD_MAX_TOP];
    __shared__ int s_tok[MAX_PARTS * MCSD_MAX_TOP];
    const int tid = threadIdx.x, i_row = blockIdx.x, map = p.row_map ? p.row_map[i_row] : i_row, n = p.parts * p.n_top;
    if ((unsigned)map >= (unsigned)p.R) return;         // (refused by the parts)
    const RowPart *part = p.part + (size_t)i_row * p.parts;
    for (int k = tid; k < n; k += 256) {
        s_logit[k] = p.part_logit[(size_t)i_row * n + k];
        s_tok[k] = p.part_tok[(size_t)i_row * n + k];
    }
    const int x = p.tokens[i_row];
    const bool known = (unsigned)x < (unsigned)p.V;
    const float T = p.temperature ? p.temperature[i_row] : 1.f, c = scale_of(T);
    // a part a lane, in every row of MAX_PARTS lanes alike
    const int y = tid % MAX_PARTS;
    const RowPart q = y < p.parts ? part[y] : RowPart{0.0, 0.0, -INFINITY, 0};
    float m = q.m;
#pragma unroll
    for (int k = 1; k < MAX_PARTS; k *= 2) m = fmaxf(m, __shfl_xor(m, k));
    double s = q.s, u = q.u;
    if (s != 0.0) {                 // (0: nothing but -infinity)
        const double t = ((double)q.m - (double)m) * (double)c, f = exp2(t);
        u = f > 0.0 ? f * (u + t * s) : 0.0;
        s *= f;
    }
    int before = q.before;
#pragma unroll
    for (int k = 1; k < MAX_PARTS; k *= 2) { s += __shfl_xor(s, k); u += __shfl_xor(u, k); before += __shfl_xor(before, k); }
    const bool bad = !(s > 0.0 && s < (double)INFINITY) || !(m < INFINITY) || !(m > -INFINITY);
    const double lse = log(s), to_ln = 1.0 / 1.44269504088896340736, inv_T = (double)c * to_ln;
    auto logprob_of = [&](float z) { return z == -INFINITY ? -INFINITY : (float)(((double)z - (double)m) * inv_T - lse); };
    if (tid == 0) {
        const float zx = !known ? 0.f : p.bf16 ? logit_at<true>(static_cast<const uint16_t *>(p.logits) + (size_t)map * p.row_stride, x)
                                               : logit_at<false>(static_cast<const float *>(p.logits) + (size_t)map * p.row_stride, x);
        p.logprob[i_row] = known && !bad ? logprob_of(zx) : NAN;
        if (p.entropy) p.entropy[i_row] = bad ? NAN : (float)fmax(lse - u / s * to_ln, 0.0);
        if (p.rank) p.rank[i_row] = known && !bad ? before : -1;
        p.flags[i_row] = bad ? (uint32_t)MCSD_FLAG_NONFINITE : known ? 0u : (uint32_t)MCSD_FLAG_BAD_TOKEN;
    }
    __syncthreads();
    int32_t *tok = p.top_tok + (size_t)i_row * p.n_top;
    float *lp = p.top_logprob + (size_t)i_row * p.n_top;
    if (bad) {
        if (tid < p.n_top) { tok[tid] = -1; lp[tid] = NAN; }
        return;
    }
    for (int k = tid; k < n; k += 256) {
        const int own = k / p.n_top;
        const float z = s_logit[k];
        int place = k - own * p.n_top;
        for (int y = 0; y < p.parts && place < p.n_top; ++y) {
            if (y == own) continue;
            int lo = 0, hi = p.n_top;       // (parts are in the order of their tokens: an equal logit of an earlier part comes before)
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                const float other = s_logit[y * p.n_top + mid];
                if (other > z || (other == z && y < own)) lo = mid + 1;
                else hi = mid;
            }
            place += lo;
        }
        if (place < p.n_top) { tok[place] = s_tok[k]; lp[place] = logprob_of(z); }
    }
}

// Parts of a row of 48 KB at least, where few long rows leave most of the chip idle.  us of a call with one workgroup a row and with parts: 1 row of
// 208 KB 14.2, 12.7; 64 of 208 KB 15.6, 14.2; 1 of 608 KB 24.2, 15.3; 64 of 608 KB 25.8, 18.6; 1 of 1 MB 35.0, 17.0; 128 of 1 MB 40.7, 36.1; 6 of 128 KB are
// as fast in one (11.8), the second launch takes 4.
int parts_of(const mcsd_logprob_desc &d)
{
    const long bytes = (long)d.V * (d.dtype == MCSD_DTYPE_BF16 ? 2 : 4);
    if (d.rows < 1 || d.rows > 128 || bytes < 200 << 10) return 1;
    const long by_rows = 256 / d.rows, by_bytes = bytes / (48 << 10);
    return (int)std::min((long)MAX_PARTS, std::min(by_rows, by_bytes));
}

size_t lists_at(const mcsd_logprob_desc &d, int parts) { return ((size_t)d.rows * parts * sizeof(RowPart) + 255) / 256 * 256; }

}  // namespace

size_t logprob_workspace(const mcsd_logprob_desc &d)
{
    const int parts = parts_of(d);
    return parts < 2 ? 0 : lists_at(d, parts) + (size_t)d.rows * parts * d.n_top * 8;
}

int32_t launch_token_logprobs(const mcsd_logprob_desc &d, const mcsd_logprob_bufs &b, hipStream_t stream)
{
    LogprobParams p;
    p.rows = d.rows; p.R = d.R; p.V = d.V; p.n_top = d.n_top; p.row_stride = (size_t)d.row_stride;
    p.logits = b.logits; p.row_map = b.row_map; p.tokens = b.tokens; p.temperature = b.temperature;
    p.logprob = b.logprob; p.entropy = b.entropy; p.rank = b.rank; p.top_tok = b.top_tok; p.top_logprob = b.top_logprob; p.flags = b.flags;
    // Threads of a row, us of a call: many rows leave a CU several at a time.  3580 rows of 1 KB with 512 threads 39.0, 128 15.4; 16 KB 39.5, 23.7; 32 KB
    // 53.1, 40.1; 64 KB 512 threads 68, 256 61.6, 128 75.9; 2000 of 100 KB 64.5 and 59.9 with 256; 4096 of 128 KB 121.9 and 125.4; 300 of 600 KB 51, 60.
    // Up to a row a CU: 6 rows of 4 KB with 1024 threads 8.2, 128 6.6; of 8 KB 8.3, 8.8.
    p.bf16 = d.dtype == MCSD_DTYPE_BF16;
    p.parts = parts_of(d);
    p.part = static_cast<RowPart *>(b.workspace);
    p.part_logit = p.parts > 1 ? reinterpret_cast<float *>(static_cast<char *>(b.workspace) + lists_at(d, p.parts)) : nullptr;
    p.part_tok = reinterpret_cast<int32_t *>(p.part_logit + (size_t)d.rows * p.parts * d.n_top);
    const size_t row_bytes = (size_t)d.V * (d.dtype == MCSD_DTYPE_BF16 ? 2 : 4);
    auto launch = [&](auto bf16_tag) {
        constexpr bool BF16 = decltype(bf16_tag)::value;
        auto threads = [&](auto kernel, int n) { launch_kernel(K_TOKEN_LOGPROBS, kernel, dim3(d.rows), dim3(n), stream, p); };
        const bool many = d.rows > 256;
        if (row_bytes <= (many ? 32 << 10 : 4 << 10)) threads(token_logprobs_kernel<BF16, 128, 4, false>, 128);
        else if (many && row_bytes <= 112 << 10) threads(token_logprobs_kernel<BF16, 256, 4, false>, 256);
        else if (many) threads(token_logprobs_kernel<BF16, 512, 4, false>, 512);
        else if (p.parts == 1) threads(token_logprobs_kernel<BF16, 1024, BF16 ? 4 : 8, false>, 1024);       // (fewer rows: registers for more pieces under way)
        else {
            launch_kernel(K_TOKEN_LOGPROBS, token_logprobs_kernel<BF16, 512, 4, true>, dim3(d.rows, p.parts), dim3(512), stream, p);
            launch_kernel(K_LOGPROBS_MERGE, token_logprobs_merge_kernel, dim3(d.rows), dim3(256), stream, p);
        }
    };
    if (d.dtype == MCSD_DTYPE_BF16) launch(std::true_type());
    else launch(std::false_type());
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("token log probabilities launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
