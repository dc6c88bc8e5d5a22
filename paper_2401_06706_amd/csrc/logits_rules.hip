// Penalties, biases and grammar masks on the logit rows of the candidate trees.
#include <algorithm>

#include "mcsd_internal.h"

namespace mcsd {
namespace {

constexpr int RULE_THREADS = 256, RULE_SLICE = 4 * RULE_THREADS;       // tokens per workgroup
constexpr uint32_t IN_PROMPT = 0x80000000u;
// Workgroups aimed at by dealing the rows out: all that the chip holds at once (eight per CU).  More of them count the history more often, fewer wait for memory:
// 512, 1024, 2048, 4096 workgroups, 976 rows of 32000 in fp32 124, 84, 61, 64 us; 232 of 65536 in bf16 47, 32, 25, 27; 129 of 32000 18, 14.2, 12.5, 14.3; 32 sequences of
// 7 rows and 4096 tokens of history 20.7, 20.8, 19.0, 22.5; one of 29 rows of 50001 7.0, 6.5, 7.2, 7.1.  Not so with two rows and 16384 tokens of history, which every
// workgroup reads for 1024 tokens of the vocabulary (32 sequences, 50001): 17.4, 17.5, 24.2, 24.3.
constexpr long RULE_GROUPS = 2048;

struct RuleParams {
    int B, N, V, R, parent_per_seq, row_begin, row_end, hist_stride, n_bias, rows_per_group, mask_words;
    const void *logits;
    float *out;
    const int32_t *row_map, *parent, *cand_tok, *history, *hist_len, *prompt_len;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_tok;
    const float *bias_val;
    const uint32_t *mask;
};

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));          // four values that start anywhere
typedef uint16_t u16x4u __attribute__((ext_vector_type(4), aligned(2)));

// Bound by memory: 976 rows of 32000 in fp32, one token in 50 allowed: 61 us for 209 MB (84 read, 125 written), 3.4 TB/s; 254 MB
// if all were read, 4.2.  One sequence, 29 rows of 50001 in bf16: 7 us, launch and the history's count.
// grid (slices of the vocabulary, groups of tree rows, sequences).  A workgroup counts the sequence's history once, in
// LDS, for the 1024 tokens of its slice, keeps what the rules ask of a thread's four tokens in registers and then goes through
// its tree rows, AHEAD of them at a time: their mask words, then those logits that are not masked throughout, then the rules.  The
// candidates on a row's path are counted on top of the history, found by a ballot over the at most 128 nodes.
template <bool BF16, bool INPLACE>
__global__ __launch_bounds__(RULE_THREADS) void logits_rules_kernel(RuleParams p)
{
    constexpr int AHEAD = 4;
    __shared__ uint32_t s_count[RULE_SLICE];
    __shared__ int s_bias[RULE_SLICE];
    __shared__ int s_parent[MCSD_MAX_NODES];
    __shared__ uint32_t s_anc[MCSD_MAX_NODES + 1][4];       // by tree row
    __shared__ int s_row[MCSD_MAX_NODES + 1];               // logit row of every tree row, or -1
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.z;
    const int s0 = blockIdx.x * RULE_SLICE;
    const int r0 = p.row_begin + blockIdx.y * p.rows_per_group, r1 = min(p.row_end, r0 + p.rows_per_group);

    if (tid < p.N) s_parent[tid] = p.parent[(p.parent_per_seq ? (size_t)b * p.N : 0) + tid];
    if (tid <= p.N) {
        int row = tid;
        if (p.row_map) row = p.row_map[(p.parent_per_seq ? (size_t)b * (1 + p.N) : 0) + tid];
        s_row[tid] = (unsigned)row < (unsigned)p.R ? row : -1;
    }
    // candidates of this lane: nodes lane and 64 + lane
    const int tok0 = lane < p.N ? p.cand_tok[(size_t)b * p.N + lane] : -1, tok1 = 64 + lane < p.N ? p.cand_tok[(size_t)b * p.N + 64 + lane] : -1;
    for (int i = tid; i < RULE_SLICE; i += RULE_THREADS) { s_count[i] = 0u; s_bias[i] = -1; }
    __syncthreads();
    if (tid >= r0 && tid < r1) {
        uint32_t m[4] = {0u, 0u, 0u, 0u};
        int a = tid - 1;
        for (int step = 0; step < MCSD_MAX_NODES && a >= 0; ++step) {
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if ((a >> 5) == w) m[w] |= 1u << (a & 31);
            const int pa = s_parent[a];
            a = pa < a ? pa : -1;       // a malformed array can not loop or index out of range
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) s_anc[tid][w] = m[w];
    }
    if (p.hist_stride > 0) {
        const int n = min(max(p.hist_len[b], 0), p.hist_stride);
        const int prompt = p.prompt_len ? p.prompt_len[b] : 0;
        const int32_t *h = p.history + (size_t)b * p.hist_stride;
        // eight tokens a thread at a time, all requested before the first is counted
        for (int i0 = tid; i0 < n; i0 += 8 * RULE_THREADS) {
            int tok[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) tok[k] = i0 + k * RULE_THREADS < n ? h[i0 + k * RULE_THREADS] : -1;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const unsigned t = (unsigned)(tok[k] - s0);
                if (tok[k] >= 0 && t < (unsigned)RULE_SLICE && tok[k] < p.V) {
                    if (i0 + k * RULE_THREADS < prompt) atomicOr(&s_count[t], IN_PROMPT);
                    else atomicAdd(&s_count[t], 1u);
                }
            }
        }
    }
    for (int i = tid; i < p.n_bias; i += RULE_THREADS) {
        const int tok = p.bias_tok[(size_t)b * p.n_bias + i];
        if (tok >= 0 && (unsigned)(tok - s0) < (unsigned)RULE_SLICE) atomicMax(&s_bias[tok - s0], i);        // the last entry counts
    }
    __syncthreads();

    const float R = p.repetition ? p.repetition[b] : 1.f, P = p.presence ? p.presence[b] : 0.f, F = p.frequency ? p.frequency[b] : 0.f;
    uint32_t count[4];
    float bias[4];
    bool biased = false;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        count[c] = s_count[4 * tid + c];
        const int e = s_bias[4 * tid + c];
        bias[c] = e >= 0 ? p.bias_val[(size_t)b * p.n_bias + e] : 0.f;
        biased |= e >= 0;
    }
    const bool counted = (count[0] | count[1]) | (count[2] | count[3]);
    const int t = s0 + 4 * tid, left = p.V - t;         // the thread's tokens: t and on, `left` of them (more than three: all)
    for (int rb = r0; rb < r1; rb += AHEAD) {
        int row[AHEAD];
        uint32_t allowed[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            row[u] = rb + u < r1 ? __builtin_amdgcn_readfirstlane(s_row[rb + u]) : -1;
            allowed[u] = 15u;
            if (p.mask && row[u] >= 0 && left > 0) allowed[u] = p.mask[((size_t)b * p.R + row[u]) * p.mask_words + (t >> 5)] >> (t & 31) & 15u;
        }
        uint64_t extra[AHEAD];          // times that the thread's tokens stand on the row's path, 16 bits each
        float z[AHEAD][4];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            extra[u] = 0;
            if (row[u] < 0) continue;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t word = s_anc[rb + u][2 * half + (lane >> 5)];
                const int tok = half ? tok1 : tok0;
                unsigned long long hits = __ballot(((word >> (lane & 31)) & 1u) && tok >= s0 && (unsigned)(tok - s0) < (unsigned)RULE_SLICE);
                while (hits) {
                    const int l = __ffsll((long long)hits) - 1;
                    hits &= hits - 1;
                    const int c = __builtin_amdgcn_readlane(tok, l) - t;
                    if ((unsigned)c < 4u) extra[u] += 1ull << (16 * c);
                }
            }
            // what is masked throughout is not read, and in place what no rule touches
            const size_t at = ((size_t)b * p.R + row[u]) * (size_t)p.V + t;
            const bool want = allowed[u] != 0u && (!INPLACE || biased || counted || extra[u] != 0 || allowed[u] != 15u);
#pragma unroll
            for (int c = 0; c < 4; ++c) z[u][c] = 0.f;
            if (want && left > 3) {
                if (BF16) {
                    const u16x4u w = *reinterpret_cast<const u16x4u *>(static_cast<const uint16_t *>(p.logits) + at);
#pragma unroll
                    for (int c = 0; c < 4; ++c) z[u][c] = __uint_as_float((uint32_t)w[c] << 16);
                } else {
                    const f32x4u w = *reinterpret_cast<const f32x4u *>(static_cast<const float *>(p.logits) + at);
#pragma unroll
                    for (int c = 0; c < 4; ++c) z[u][c] = w[c];
                }
            } else if (want) {
#pragma unroll
                for (int c = 0; c < 3; ++c)
                    if (c < left) z[u][c] = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(p.logits)[at + c] << 16) : static_cast<const float *>(p.logits)[at + c];
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (row[u] < 0 || left <= 0) continue;
            const bool touched = biased || counted || extra[u] != 0 || allowed[u] != 15u;
            if (INPLACE && !touched) continue;
            if (touched) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t n = count[c] + (uint32_t)(extra[u] >> (16 * c) & 0xffffu), after = n & ~IN_PROMPT;
                    if (n) z[u][c] = z[u][c] > 0.f ? z[u][c] / R : z[u][c] * R;
                    if (after) z[u][c] = (z[u][c] - F * (float)after) - P;
                    z[u][c] += bias[c];
                    if (!((allowed[u] >> c) & 1u)) z[u][c] = -INFINITY;
                }
            }
            float *to = p.out + ((size_t)b * p.R + row[u]) * (size_t)p.V + t;
            if (left > 3) {
                *reinterpret_cast<f32x4u *>(to) = (f32x4u){z[u][0], z[u][1], z[u][2], z[u][3]};
            } else {
#pragma unroll
                for (int c = 0; c < 3; ++c)
                    if (c < left) to[c] = z[u][c];
            }
        }
    }
}

}  // namespace

int32_t launch_logits_rules(const mcsd_logits_desc &d, const mcsd_logits_bufs &b, hipStream_t stream)
{
    RuleParams p;
    p.B = d.B; p.N = d.N; p.V = d.V; p.R = d.R; p.parent_per_seq = d.parent_per_seq; p.row_begin = d.row_begin; p.row_end = d.row_end;
    p.hist_stride = d.hist_stride; p.n_bias = d.n_bias; p.mask_words = (d.V + 31) / 32;
    p.logits = b.logits; p.out = b.out; p.row_map = b.row_map; p.parent = b.parent; p.cand_tok = b.cand_tok;
    p.history = b.history; p.hist_len = b.hist_len; p.prompt_len = b.prompt_len;
    p.repetition = b.repetition; p.presence = b.presence; p.frequency = b.frequency;
    p.bias_tok = b.bias_tok; p.bias_val = b.bias_val; p.mask = b.mask;
    const int rows = d.row_end - d.row_begin;
    if (rows == 0) return MCSD_OK;
    const int slices = (d.V + RULE_SLICE - 1) / RULE_SLICE;
    const long base = (long)slices * d.B;
    const int groups = (int)std::max(1L, std::min((long)rows, (RULE_GROUPS + base - 1) / base));
    p.rows_per_group = (rows + groups - 1) / groups;
    const dim3 grid(slices, (rows + p.rows_per_group - 1) / p.rows_per_group, d.B);
    auto go = [&](auto kernel) { launch_kernel(K_LOGITS_RULES, kernel, grid, dim3(RULE_THREADS), stream, p); };
    if (d.dtype == MCSD_DTYPE_BF16) go(logits_rules_kernel<true, false>);
    else if (static_cast<const void *>(b.out) == b.logits) go(logits_rules_kernel<false, true>);
    else go(logits_rules_kernel<false, false>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("logits_rules launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
