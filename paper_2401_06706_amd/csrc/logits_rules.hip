// Penalties, biases and grammar masks on the logit rows of the candidate trees.
#include "mcsd_internal.h"

namespace mcsd {
namespace {

constexpr int RULE_THREADS = 256, RULE_SLICE = 4 * RULE_THREADS;       // tokens per workgroup
constexpr uint32_t IN_PROMPT = 0x80000000u;

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

// grid (slices of the vocabulary, groups of tree rows, sequences).  A workgroup counts the sequence's history once, in
// LDS, for the tokens of its slice, keeps what the rules ask of a token in registers and then
// goes through its tree rows; of those the candidates on a row's path are counted on top, found by a
// ballot over the at most 128 nodes.  VEC: rows that start 16-byte aligned, four neighbouring tokens a thread;
// otherwise every 256th.
template <bool BF16, bool VEC, bool INPLACE>
__global__ __launch_bounds__(RULE_THREADS) void logits_rules_kernel(RuleParams p)
{
    __shared__ uint32_t s_count[RULE_SLICE];
    __shared__ int s_bias[RULE_SLICE];
    __shared__ int s_parent[MCSD_MAX_NODES];
    __shared__ uint32_t s_anc[MCSD_MAX_NODES + 1][4];       // by tree row
    __shared__ int s_row[MCSD_MAX_NODES + 1];               // logit row of every tree row, or -1
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.z;
    const int s0 = blockIdx.x * RULE_SLICE;
    const int r0 = p.row_begin + blockIdx.y * p.rows_per_group, r1 = min(p.row_end, r0 + p.rows_per_group);

    for (int i = tid; i < RULE_SLICE; i += RULE_THREADS) { s_count[i] = 0u; s_bias[i] = -1; }
    if (tid < p.N) s_parent[tid] = p.parent[(p.parent_per_seq ? (size_t)b * p.N : 0) + tid];
    if (tid <= p.N) {
        int row = tid;
        if (p.row_map) row = p.row_map[(p.parent_per_seq ? (size_t)b * (1 + p.N) : 0) + tid];
        s_row[tid] = (unsigned)row < (unsigned)p.R ? row : -1;
    }
    // candidates of this lane: nodes lane and 64 + lane
    const int tok0 = lane < p.N ? p.cand_tok[(size_t)b * p.N + lane] : -1, tok1 = 64 + lane < p.N ? p.cand_tok[(size_t)b * p.N + 64 + lane] : -1;
    __syncthreads();
    if (tid <= p.N) {
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
        for (int i = tid; i < n; i += RULE_THREADS) {
            const unsigned t = (unsigned)(h[i] - s0);
            if (t < (unsigned)RULE_SLICE && (int)t < p.V - s0) {
                if (i < prompt) atomicOr(&s_count[t], IN_PROMPT);
                else atomicAdd(&s_count[t], 1u);
            }
        }
    }
    for (int i = tid; i < p.n_bias; i += RULE_THREADS) {
        const unsigned t = (unsigned)(p.bias_tok[(size_t)b * p.n_bias + i] - s0);
        if (t < (unsigned)RULE_SLICE) atomicMax(&s_bias[t], i);        // the last entry counts
    }
    __syncthreads();

    const float R = p.repetition ? p.repetition[b] : 1.f, P = p.presence ? p.presence[b] : 0.f, F = p.frequency ? p.frequency[b] : 0.f;
    uint32_t count[4];
    float bias[4];
    bool biased = false;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int t = VEC ? 4 * tid + c : tid + RULE_THREADS * c;
        count[c] = s_count[t];
        const int e = s_bias[t];
        bias[c] = e >= 0 ? p.bias_val[(size_t)b * p.n_bias + e] : 0.f;
        biased |= e >= 0;
    }
    for (int r = r0; r < r1; ++r) {
        const int row = __builtin_amdgcn_readfirstlane(s_row[r]);
        if (row < 0) continue;
        const size_t base = ((size_t)b * p.R + row) * (size_t)p.V + s0;
        // the candidates on this row's path, added to the counts of their tokens
        uint32_t n[4] = {count[0], count[1], count[2], count[3]};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t word = s_anc[r][2 * half + (lane >> 5)];
            const int tok = half ? tok1 : tok0;
            unsigned long long hits = __ballot(((word >> (lane & 31)) & 1u) && (unsigned)(tok - s0) < (unsigned)RULE_SLICE);
            while (hits) {
                const int l = __ffsll((long long)hits) - 1;
                hits &= hits - 1;
                const int t = __builtin_amdgcn_readlane(tok, l) - s0;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if ((VEC ? 4 * tid + c : tid + RULE_THREADS * c) == t) ++n[c];
            }
        }
        uint32_t allowed = 15u;
        if (p.mask) {
            const uint32_t *m = p.mask + ((size_t)b * p.R + row) * p.mask_words;
            if (VEC) {
                const int t = s0 + 4 * tid;
                allowed = t < p.V ? (m[t >> 5] >> (t & 31)) & 15u : 15u;
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int t = s0 + tid + RULE_THREADS * c;
                    if (t < p.V && !((m[t >> 5] >> (t & 31)) & 1u)) allowed &= ~(1u << c);
                }
            }
        }
        const bool touched = biased || allowed != 15u || ((n[0] | n[1]) | (n[2] | n[3]));
        if (INPLACE && !touched) continue;
        float z[4];
        if (VEC) {
            const int t = 4 * tid;
            if (s0 + t >= p.V) continue;
            if (BF16) {
                const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p.logits) + base + t);
                z[0] = __uint_as_float(w.x << 16); z[1] = __uint_as_float(w.x & 0xffff0000u);
                z[2] = __uint_as_float(w.y << 16); z[3] = __uint_as_float(w.y & 0xffff0000u);
            } else {
                const float4 w = *reinterpret_cast<const float4 *>(static_cast<const float *>(p.logits) + base + t);
                z[0] = w.x; z[1] = w.y; z[2] = w.z; z[3] = w.w;
            }
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int t = tid + RULE_THREADS * c;
                z[c] = 0.f;
                if (s0 + t < p.V) z[c] = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(p.logits)[base + t] << 16) : static_cast<const float *>(p.logits)[base + t];
            }
        }
        if (touched) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t after = n[c] & ~IN_PROMPT;
                if (n[c]) z[c] = z[c] > 0.f ? z[c] / R : z[c] * R;
                if (after) z[c] = (z[c] - F * (float)after) - P;
                z[c] += bias[c];
                if (!((allowed >> c) & 1u)) z[c] = -INFINITY;
            }
        }
        if (VEC) {
            *reinterpret_cast<float4 *>(p.out + base + 4 * tid) = make_float4(z[0], z[1], z[2], z[3]);
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int t = tid + RULE_THREADS * c;
                if (s0 + t < p.V) p.out[base + t] = z[c];
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
    p.rows_per_group = rows;
    const dim3 grid(slices, 1, d.B);
    const bool bf16 = d.dtype == MCSD_DTYPE_BF16;
    const uintptr_t in = (uintptr_t)b.logits, out = (uintptr_t)b.out;
    const bool vec = d.V % 4 == 0 && out % 16 == 0 && in % (bf16 ? 8 : 16) == 0, inplace = in == out;
    auto go = [&](auto kernel) { launch_kernel(K_LOGITS_RULES, kernel, grid, dim3(RULE_THREADS), stream, p); };
    if (bf16) { if (vec) go(logits_rules_kernel<true, true, false>); else go(logits_rules_kernel<true, false, false>); }
    else if (inplace) { if (vec) go(logits_rules_kernel<false, true, true>); else go(logits_rules_kernel<false, false, true>); }
    else { if (vec) go(logits_rules_kernel<false, true, false>); else go(logits_rules_kernel<false, false, false>); }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("logits_rules launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
