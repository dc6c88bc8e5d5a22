// C ABI of libmcsd: argument validation, error reporting, optional per-kernel
// event timing.  All compute happens in the other .hip files.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <mutex>
#include <vector>

#include "mcsd_internal.h"

namespace mcsd {

static thread_local char g_err[512] = "";

void set_error(const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
}

// ------------------------------------------------------------------ event timing
// Off by default.  When on, every kernel launch carries a start and a stop event of its own
// dispatch; mcsd_kernel_timing_read waits for them and adds up the durations.
namespace {
struct EventPair { hipEvent_t a, b; int id; };
std::mutex g_tmutex;
bool g_timing = false;
std::vector<EventPair> g_pending;
double g_total_ms[K_COUNT];
long long g_count[K_COUNT];
const char *const g_names[K_COUNT] = {"tree_attn_mfma", "tree_attn_generic", "tree_attn_combine",
                                      "verify_rows", "walk", "draft_rows", "tree_build", "kv_copy", "kv_finish",
                                      "kv_store_fourbit", "kv_load_fourbit", "attn_fourbit", "attn_fourbit_combine",
                                      "page_assign", "page_slots", "logits_rules",
                                      "kv_store_paged", "chunk_attn", "chunk_merge", "weight_sums", "evict_select", "evict_move", "token_logprobs", "chunk_wide", "logprobs_merge"};
}  // namespace

bool timing_new_events(hipEvent_t *start, hipEvent_t *stop)
{
    if (!g_timing) return false;
    if (hipEventCreate(start) != hipSuccess) return false;
    if (hipEventCreate(stop) != hipSuccess) { (void)hipEventDestroy(*start); return false; }
    return true;
}

void timing_commit(int id, hipEvent_t start, hipEvent_t stop)
{
    std::lock_guard<std::mutex> lk(g_tmutex);
    g_pending.push_back({start, stop, id});
}

}  // namespace mcsd

using namespace mcsd;

extern "C" {

const char *mcsd_last_error(void) { return g_err; }
const char *mcsd_version(void) { return "libmcsd 0.1 (gfx950)"; }

// Profiling aid (not part of the verification step): enable != 0 starts bracketing
// every kernel launch with HIP events; 0 stops.  Totals are reset when enabled.
int32_t mcsd_kernel_timing(int32_t enable)
{
    std::lock_guard<std::mutex> lk(g_tmutex);
    g_timing = enable != 0;
    if (g_timing) {
        for (auto &p : g_pending) { (void)hipEventDestroy(p.a); (void)hipEventDestroy(p.b); }
        g_pending.clear();
        for (int i = 0; i < K_COUNT; ++i) { g_total_ms[i] = 0.0; g_count[i] = 0; }
    }
    return MCSD_OK;
}

int32_t mcsd_kernel_count(void) { return K_COUNT; }
const char *mcsd_kernel_name(int32_t id) { return (id >= 0 && id < K_COUNT) ? g_names[id] : ""; }

// Waits for the recorded events (synchronises with them) and returns the summed
// duration in ms and the number of launches of kernel `id` since timing was enabled.
int32_t mcsd_kernel_timing_read(int32_t id, double *total_ms, int64_t *launches)
{
    if (id < 0 || id >= K_COUNT || !total_ms || !launches) return MCSD_E_SHAPE;
    std::lock_guard<std::mutex> lk(g_tmutex);
    for (auto &p : g_pending) {
        float ms = 0.f;
        if (hipEventSynchronize(p.b) == hipSuccess && hipEventElapsedTime(&ms, p.a, p.b) == hipSuccess) {
            g_total_ms[p.id] += ms;
            g_count[p.id] += 1;
        }
        (void)hipEventDestroy(p.a);
        (void)hipEventDestroy(p.b);
    }
    g_pending.clear();
    *total_ms = g_total_ms[id];
    *launches = g_count[id];
    return MCSD_OK;
}

int32_t mcsd_tree_validate(const int32_t *parent, int32_t n)
{
    if (!parent) { set_error("parent is NULL"); return MCSD_E_NULL; }
    if (n < 1 || n > MCSD_MAX_NODES) { set_error("n_nodes %d outside 1..%d", n, MCSD_MAX_NODES); return MCSD_E_TREE; }
    for (int i = 0; i < n; ++i)
        if (parent[i] < -1 || parent[i] >= i) {
            set_error("parent[%d] = %d violates -1 <= parent[i] < i", i, parent[i]);
            return MCSD_E_TREE;
        }
    return MCSD_OK;
}

static int32_t check_attn(const mcsd_attn_desc *d, const mcsd_attn_bufs *b, AttnPlan *plan)
{
    if (!d) { set_error("attn desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_attn_desc)) { set_error("attn desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_attn_desc)); return MCSD_E_SHAPE; }
    if (d->B < 1 || d->H_q < 1 || d->H_kv < 1 || d->d < 1 || d->L_stride < 0) { set_error("attn: non-positive size"); return MCSD_E_SHAPE; }
    if (d->L_stride > (1 << 22)) { set_error("attn: L_stride %d > %d", d->L_stride, 1 << 22); return MCSD_E_UNSUPPORTED; }
    if (d->root_row != 0 && d->root_row != 1) { set_error("attn: root_row must be 0 or 1"); return MCSD_E_SHAPE; }
    if (d->N < 1 || d->N + d->root_row > MCSD_MAX_NODES) { set_error("attn: N %d (+ root row) outside 1..%d", d->N, MCSD_MAX_NODES); return MCSD_E_TREE; }
    if (d->H_q % d->H_kv != 0) { set_error("attn: H_q %d not a multiple of H_kv %d", d->H_q, d->H_kv); return MCSD_E_SHAPE; }
    if (d->dtype != MCSD_DTYPE_FP32 && d->dtype != MCSD_DTYPE_BF16) { set_error("attn: unknown dtype %d", d->dtype); return MCSD_E_UNSUPPORTED; }
    if (d->d > MCSD_MAX_HEAD_DIM || d->d % (d->dtype == MCSD_DTYPE_BF16 ? 8 : 4) != 0) { set_error("attn: head dim %d unsupported", d->d); return MCSD_E_UNSUPPORTED; }
    if (!(d->scale >= 0.f) || !(d->scale < 1e30f)) { set_error("attn: scale must be finite and >= 0"); return MCSD_E_SHAPE; }
    if (!make_attn_plan(*d, plan)) { set_error("attn: no kernel for this shape"); return MCSD_E_UNSUPPORTED; }
    if (!b) return MCSD_OK;
    if (b->struct_size != sizeof(mcsd_attn_bufs)) { set_error("attn bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_attn_bufs)); return MCSD_E_SHAPE; }
    if (!b->q || !b->k_tree || !b->v_tree || !b->prefix_len || !b->parent || !b->out) { set_error("attn: NULL buffer"); return MCSD_E_NULL; }
    if (d->L_stride > 0 && (!b->k_prefix || !b->v_prefix)) { set_error("attn: NULL prefix cache"); return MCSD_E_NULL; }
    if (plan->ws_bytes > 0) {
        if (!b->workspace) { set_error("attn: workspace is NULL, %zu bytes needed", plan->ws_bytes); return MCSD_E_WORKSPACE; }
        if (b->workspace_bytes < plan->ws_bytes) { set_error("attn: workspace %zu < %zu bytes", b->workspace_bytes, plan->ws_bytes); return MCSD_E_WORKSPACE; }
        if (((uintptr_t)b->workspace & 255u) != 0) { set_error("attn: workspace not 256-byte aligned"); return MCSD_E_WORKSPACE; }
    }
    const uintptr_t al = (uintptr_t)b->q | (uintptr_t)b->k_prefix | (uintptr_t)b->v_prefix | (uintptr_t)b->k_tree |
                         (uintptr_t)b->v_tree | (uintptr_t)b->out;
    if (al & 15u) { set_error("attn: tensors must be 16-byte aligned"); return MCSD_E_SHAPE; }
    return MCSD_OK;
}

static int32_t check_verify(const mcsd_verify_desc *d, const mcsd_verify_bufs *b)
{
    if (!d) { set_error("verify desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_verify_desc)) { set_error("verify desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_verify_desc)); return MCSD_E_SHAPE; }
    if (d->B < 1 || d->V < 1 || d->P < 1 || d->gamma_max < 1) { set_error("verify: non-positive size"); return MCSD_E_SHAPE; }
    if (d->N < 1 || d->N > MCSD_MAX_NODES) { set_error("verify: N %d outside 1..%d", d->N, MCSD_MAX_NODES); return MCSD_E_TREE; }
    if (d->P > 1 + d->N) { set_error("verify: P %d > 1+N", d->P); return MCSD_E_SHAPE; }
    if (d->B > 65535) { set_error("verify: B %d > 65535", d->B); return MCSD_E_UNSUPPORTED; }
    if (d->V > MCSD_MAX_VOCAB) { set_error("verify: V %d > %d", d->V, MCSD_MAX_VOCAB); return MCSD_E_UNSUPPORTED; }
    if (d->variant != MCSD_WITH_REPLACEMENT && d->variant != MCSD_WITHOUT_REPLACEMENT && d->variant != MCSD_NAIVE) { set_error("verify: unknown variant %d", d->variant); return MCSD_E_UNSUPPORTED; }
    if (!(d->near_tie_eps >= 0.f)) { set_error("verify: near_tie_eps must be >= 0"); return MCSD_E_SHAPE; }
    if (d->parent_per_seq != 0 && d->parent_per_seq != 1) { set_error("verify: parent_per_seq must be 0 or 1"); return MCSD_E_SHAPE; }
    if (!b) return MCSD_OK;
    if (b->struct_size != sizeof(mcsd_verify_bufs)) { set_error("verify bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_verify_bufs)); return MCSD_E_SHAPE; }
    if (!b->target_logits || !b->draft_logits || !b->q_row || !b->parent || !b->cand_tok || !b->u_accept ||
        !b->u_endpoint || !b->temperature || !b->n_accepted || !b->accepted_path || !b->out_tokens ||
        !b->acc_child || !b->endpoint || !b->flags) { set_error("verify: NULL buffer"); return MCSD_E_NULL; }
    if (d->V % 4 == 0 && (((uintptr_t)b->target_logits | (uintptr_t)b->draft_logits | (uintptr_t)b->residual_out) & 15u)) {
        set_error("verify: logit arrays must be 16-byte aligned");
        return MCSD_E_SHAPE;
    }
    return MCSD_OK;
}

static int32_t check_draft(const mcsd_draft_desc *d, const mcsd_draft_bufs *b)
{
    if (!d) { set_error("draft desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_draft_desc)) { set_error("draft desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_draft_desc)); return MCSD_E_SHAPE; }
    if (d->B < 1 || d->V < 1 || d->P < 1) { set_error("draft: non-positive size"); return MCSD_E_SHAPE; }
    if (d->N < 1 || d->N > MCSD_MAX_NODES) { set_error("draft: N %d outside 1..%d", d->N, MCSD_MAX_NODES); return MCSD_E_TREE; }
    if (d->P > 1 + d->N) { set_error("draft: P %d > 1+N", d->P); return MCSD_E_SHAPE; }
    if (d->B > 65535) { set_error("draft: B %d > 65535", d->B); return MCSD_E_UNSUPPORTED; }
    if (d->V > MCSD_MAX_VOCAB) { set_error("draft: V %d > %d", d->V, MCSD_MAX_VOCAB); return MCSD_E_UNSUPPORTED; }
    if (d->variant != MCSD_WITH_REPLACEMENT && d->variant != MCSD_WITHOUT_REPLACEMENT) { set_error("draft: unknown variant %d", d->variant); return MCSD_E_UNSUPPORTED; }
    if (!(d->near_tie_eps >= 0.f)) { set_error("draft: near_tie_eps must be >= 0"); return MCSD_E_SHAPE; }
    if (d->parent_per_seq != 0 && d->parent_per_seq != 1) { set_error("draft: parent_per_seq must be 0 or 1"); return MCSD_E_SHAPE; }
    if (!b) { set_error("draft bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_draft_bufs)) { set_error("draft bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_draft_bufs)); return MCSD_E_SHAPE; }
    if (!b->draft_logits || !b->q_row || !b->parent || !b->u_draw || !b->temperature || !b->cand_tok || !b->flags) {
        set_error("draft: NULL buffer");
        return MCSD_E_NULL;
    }
    if (d->V % 4 == 0 && ((uintptr_t)b->draft_logits & 15u)) { set_error("draft: draft_logits must be 16-byte aligned"); return MCSD_E_SHAPE; }
    return MCSD_OK;
}

size_t mcsd_attn_workspace_bytes(const mcsd_attn_desc *desc)
{
    AttnPlan plan;
    if (check_attn(desc, nullptr, &plan) != MCSD_OK) return 0;
    return plan.ws_bytes;
}

size_t mcsd_verify_workspace_bytes(const mcsd_verify_desc *desc)
{
    (void)desc;
    return 0;
}

int32_t mcsd_tree_attn(const mcsd_attn_desc *desc, const mcsd_attn_bufs *bufs, void *stream)
{
    AttnPlan plan;
    if (!bufs) { set_error("attn bufs is NULL"); return MCSD_E_NULL; }
    int32_t rc = check_attn(desc, bufs, &plan);
    if (rc != MCSD_OK) return rc;
    return launch_tree_attn(*desc, *bufs, plan, (hipStream_t)stream);
}

// ---------------------------------------------------------- allocation-free attention
// The scratch of mcsd_tree_attn_static lives in the device image of this library: no
// allocation at any call.  In host code the array's name is only a handle for
// hipGetSymbolAddress; the device address it returns (one per GPU) is what kernels get.
static __device__ __align__(256) unsigned char scratch[MCSD_STATIC_SCRATCH_BYTES];

namespace {
constexpr int MAX_DEVICES = 64;
std::mutex g_scratch_mutex;
void *g_scratch_ptr[MAX_DEVICES];     // device address of `scratch` on each GPU, looked up once

int32_t static_scratch_of_current_device(void **out)
{
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) { set_error("attn(static): hipGetDevice failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    if (dev < 0 || dev >= MAX_DEVICES) { set_error("attn(static): device %d outside 0..%d", dev, MAX_DEVICES - 1); return MCSD_E_UNSUPPORTED; }
    std::lock_guard<std::mutex> lk(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void *ptr = nullptr;
        e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !ptr) {
            set_error("attn(static): hipGetSymbolAddress failed on device %d: %s", dev, hipGetErrorString(e));
            return MCSD_E_HIP;
        }
        g_scratch_ptr[dev] = ptr;
    }
    *out = g_scratch_ptr[dev];
    return MCSD_OK;
}
}  // namespace

int32_t mcsd_tree_attn_static(const mcsd_attn_desc *desc, const mcsd_attn_bufs *bufs, void *stream)
{
    AttnPlan plan;
    if (!bufs) { set_error("attn bufs is NULL"); return MCSD_E_NULL; }
    int32_t rc = check_attn(desc, nullptr, &plan);       // the descriptor alone fixes the scratch size
    if (rc != MCSD_OK) return rc;
    if (plan.ws_bytes > MCSD_STATIC_SCRATCH_BYTES) {
        set_error("attn(static): this shape needs %zu bytes of scratch, the static buffer holds %zu; use mcsd_tree_attn with a workspace",
                  plan.ws_bytes, (size_t)MCSD_STATIC_SCRATCH_BYTES);
        return MCSD_E_WORKSPACE;
    }
    if (bufs->struct_size != sizeof(mcsd_attn_bufs)) { set_error("attn bufs struct_size %u != %zu", bufs->struct_size, sizeof(mcsd_attn_bufs)); return MCSD_E_SHAPE; }
    mcsd_attn_bufs b = *bufs;
    void *ptr = nullptr;
    rc = static_scratch_of_current_device(&ptr);
    if (rc != MCSD_OK) return rc;
    b.workspace = ptr;
    b.workspace_bytes = MCSD_STATIC_SCRATCH_BYTES;
    rc = check_attn(desc, &b, &plan);
    if (rc != MCSD_OK) return rc;
    return launch_tree_attn(*desc, b, plan, (hipStream_t)stream);
}

int32_t mcsd_tree_attn_paged(const mcsd_attn_desc *desc, const mcsd_attn_bufs *bufs, const mcsd_paged_kv *paged,
                             void *stream)
{
    AttnPlan plan;
    if (!bufs) { set_error("attn bufs is NULL"); return MCSD_E_NULL; }
    if (!paged) { set_error("paged descriptor is NULL"); return MCSD_E_NULL; }
    int32_t rc = check_attn(desc, bufs, &plan);
    if (rc != MCSD_OK) return rc;
    if (paged->struct_size != sizeof(mcsd_paged_kv)) { set_error("paged struct_size %u != %zu", paged->struct_size, sizeof(mcsd_paged_kv)); return MCSD_E_SHAPE; }
    if (!paged->block_table) { set_error("paged: block_table is NULL"); return MCSD_E_NULL; }
    if (paged->page_size < 32 || paged->page_size % 32 != 0) { set_error("paged: page_size %d is not a positive multiple of 32", paged->page_size); return MCSD_E_SHAPE; }
    if (paged->n_pages < 1 || paged->max_pages_per_seq < 1) { set_error("paged: non-positive size"); return MCSD_E_SHAPE; }
    if ((long)paged->max_pages_per_seq * paged->page_size < (long)desc->L_stride) { set_error("paged: L_stride %d exceeds max_pages_per_seq * page_size", desc->L_stride); return MCSD_E_SHAPE; }
    return launch_tree_attn(*desc, *bufs, plan, (hipStream_t)stream, paged);
}

int32_t mcsd_verify_sample(const mcsd_verify_desc *desc, const mcsd_verify_bufs *bufs, void *stream)
{
    if (!bufs) { set_error("verify bufs is NULL"); return MCSD_E_NULL; }
    int32_t rc = check_verify(desc, bufs);
    if (rc != MCSD_OK) return rc;
    return launch_verify(*desc, *bufs, (hipStream_t)stream);
}

int32_t mcsd_draft_sample(const mcsd_draft_desc *desc, const mcsd_draft_bufs *bufs, void *stream)
{
    int32_t rc = check_draft(desc, bufs);
    if (rc != MCSD_OK) return rc;
    return launch_draft_sample(*desc, *bufs, (hipStream_t)stream);
}

int32_t mcsd_tree_size(const int32_t *kconfig, int32_t gamma, int32_t *n_nodes, int32_t *n_draft_rows)
{
    if (!kconfig) { set_error("tree: kconfig is NULL"); return MCSD_E_NULL; }
    if (gamma < 1 || gamma > MAX_GAMMA) { set_error("tree: gamma %d outside 1..%d", gamma, MAX_GAMMA); return MCSD_E_SHAPE; }
    long level = 1, n = 0, internal = 1;
    for (int i = 0; i < gamma; ++i) {
        if (kconfig[i] < 1) { set_error("tree: k_%d = %d < 1", i + 1, kconfig[i]); return MCSD_E_SHAPE; }
        level *= kconfig[i];
        n += level;
        if (n > MCSD_MAX_NODES) { set_error("tree: more than %d nodes", MCSD_MAX_NODES); return MCSD_E_TREE; }
        if (i + 1 < gamma) internal += level;
    }
    if (n_nodes) *n_nodes = (int32_t)n;
    if (n_draft_rows) *n_draft_rows = (int32_t)internal;
    return MCSD_OK;
}

int32_t mcsd_tree_build(const int32_t *kconfig, int32_t gamma, int32_t B, const int32_t *prefix_len, int32_t *parent,
                        int32_t *depth, int32_t *q_row, int32_t *position_ids, int32_t root_row, void *stream)
{
    if (root_row != 0 && root_row != 1) { set_error("tree: root_row must be 0 or 1"); return MCSD_E_SHAPE; }
    int32_t n = 0;
    int32_t rc = mcsd_tree_size(kconfig, gamma, &n, nullptr);
    if (rc != MCSD_OK) return rc;
    if (!parent || !depth || !q_row) { set_error("tree: NULL output"); return MCSD_E_NULL; }
    if (position_ids && !prefix_len) { set_error("tree: position_ids needs prefix_len"); return MCSD_E_NULL; }
    if (position_ids && (B < 1 || B > 65535)) { set_error("tree: B %d outside 1..65535", B); return MCSD_E_SHAPE; }
    return launch_tree_build(kconfig, gamma, n, B, prefix_len, parent, depth, q_row, position_ids, root_row, (hipStream_t)stream);
}

static int32_t check_commit(const mcsd_commit_desc *d, const mcsd_commit_bufs *b, bool prefix_in_bufs = true)
{
    if (!d) { set_error("commit desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_commit_desc)) { set_error("commit desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_commit_desc)); return MCSD_E_SHAPE; }
    if (d->B < 1 || d->H_kv < 1 || d->d < 1 || d->L_stride < 1 || d->gamma_max < 1 || d->n_layers < 1) { set_error("commit: non-positive size"); return MCSD_E_SHAPE; }
    if (d->root_row != 0 && d->root_row != 1) { set_error("commit: root_row must be 0 or 1"); return MCSD_E_SHAPE; }
    if (d->N < 1 || d->N + d->root_row > MCSD_MAX_NODES) { set_error("commit: N %d (+ root row) outside 1..%d", d->N, MCSD_MAX_NODES); return MCSD_E_TREE; }
    if (d->dtype != MCSD_DTYPE_FP32 && d->dtype != MCSD_DTYPE_BF16) { set_error("commit: unknown dtype %d", d->dtype); return MCSD_E_UNSUPPORTED; }
    const int esize = d->dtype == MCSD_DTYPE_FP32 ? 4 : 2;
    if ((d->d * esize) % 16 != 0) { set_error("commit: d * element size must be a multiple of 16 bytes"); return MCSD_E_SHAPE; }
    if (d->B > 65535 || d->gamma_max > 65535 || d->n_layers > 65535) { set_error("commit: grid too large"); return MCSD_E_UNSUPPORTED; }
    if (!b) { set_error("commit bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_commit_bufs)) { set_error("commit bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_commit_bufs)); return MCSD_E_SHAPE; }
    if ((prefix_in_bufs && (!b->k_prefix || !b->v_prefix)) || !b->k_tree || !b->v_tree || !b->n_accepted || !b->accepted_path ||
        !b->out_tokens || !b->prefix_len || !b->next_root || !b->flags) { set_error("commit: NULL buffer"); return MCSD_E_NULL; }
    const uintptr_t prefix = prefix_in_bufs ? (uintptr_t)b->k_prefix | (uintptr_t)b->v_prefix : 0;
    if ((prefix | (uintptr_t)b->k_tree | (uintptr_t)b->v_tree) & 15u) {
        set_error("commit: caches must be 16-byte aligned");
        return MCSD_E_SHAPE;
    }
    return MCSD_OK;
}

int32_t mcsd_kv_commit(const mcsd_commit_desc *d, const mcsd_commit_bufs *b, void *stream)
{
    const int32_t rc = check_commit(d, b);
    if (rc != MCSD_OK) return rc;
    return launch_kv_commit(*d, *b, (hipStream_t)stream);
}

int32_t mcsd_kv_commit_paged(const mcsd_commit_desc *d, const mcsd_commit_bufs *b, const mcsd_paged_kv *paged, void *stream)
{
    int32_t rc = check_commit(d, b);
    if (rc != MCSD_OK) return rc;
    if (!paged) { set_error("paged descriptor is NULL"); return MCSD_E_NULL; }
    if (paged->struct_size != sizeof(mcsd_paged_kv)) { set_error("paged struct_size %u != %zu", paged->struct_size, sizeof(mcsd_paged_kv)); return MCSD_E_SHAPE; }
    if (!paged->block_table) { set_error("paged: block_table is NULL"); return MCSD_E_NULL; }
    if (paged->page_size < 32 || paged->page_size % 32 != 0) { set_error("paged: page_size %d is not a positive multiple of 32", paged->page_size); return MCSD_E_SHAPE; }
    if (paged->n_pages < 1 || paged->max_pages_per_seq < 1) { set_error("paged: non-positive size"); return MCSD_E_SHAPE; }
    if ((long)paged->max_pages_per_seq * paged->page_size < (long)d->L_stride) { set_error("paged: L_stride %d exceeds max_pages_per_seq * page_size", d->L_stride); return MCSD_E_SHAPE; }
    return launch_kv_commit(*d, *b, (hipStream_t)stream, paged);
}

// ------------------------------------------------------------ prefix cache in 4 bits
// L_stride >= 0: the logical capacity that the block table has to hold (rows in and out by slot have none: -1)
static int32_t check_fourbit(const mcsd_fourbit_kv *kv, int d, long L_stride)
{
    if (!kv) { set_error("fourbit: cache descriptor is NULL"); return MCSD_E_NULL; }
    if (kv->struct_size != sizeof(mcsd_fourbit_kv)) { set_error("fourbit: struct_size %u != %zu", kv->struct_size, sizeof(mcsd_fourbit_kv)); return MCSD_E_SHAPE; }
    if (d < 32 || d % 32 != 0 || d > MCSD_MAX_HEAD_DIM) { set_error("fourbit: head dim %d is not a multiple of 32 up to %d", d, MCSD_MAX_HEAD_DIM); return MCSD_E_UNSUPPORTED; }
    if (kv->page_size < 32 || kv->page_size % 32 != 0) { set_error("fourbit: page_size %d is not a positive multiple of 32", kv->page_size); return MCSD_E_SHAPE; }
    if (kv->n_pages < 1 || (L_stride >= 0 && kv->max_pages_per_seq < 1)) { set_error("fourbit: non-positive size"); return MCSD_E_SHAPE; }
    if ((long)kv->n_pages * kv->page_size > 0x7fffffffL) { set_error("fourbit: n_pages * page_size does not fit a slot"); return MCSD_E_UNSUPPORTED; }
    if (L_stride >= 0 && (long)kv->max_pages_per_seq * kv->page_size < L_stride) { set_error("fourbit: L_stride %ld exceeds max_pages_per_seq * page_size", L_stride); return MCSD_E_SHAPE; }
    if (!kv->k_codes || !kv->v_codes || !kv->k_scales || !kv->v_scales) { set_error("fourbit: NULL pool"); return MCSD_E_NULL; }
    if (L_stride >= 0 && !kv->block_table) { set_error("fourbit: block_table is NULL"); return MCSD_E_NULL; }
    if (((uintptr_t)kv->k_codes | (uintptr_t)kv->v_codes | (uintptr_t)kv->k_scales | (uintptr_t)kv->v_scales) & 15u) {
        set_error("fourbit: pools must be 16-byte aligned");
        return MCSD_E_SHAPE;
    }
    return MCSD_OK;
}

static int32_t check_attn_fourbit(const mcsd_attn_desc *d, const mcsd_attn_bufs *b, FourbitPlan *plan)
{
    AttnPlan unused;
    int32_t rc = check_attn(d, nullptr, &unused);
    if (rc != MCSD_OK) return rc;
    if (d->dtype != MCSD_DTYPE_BF16) { set_error("attn(fourbit): bf16 queries only"); return MCSD_E_UNSUPPORTED; }
    if (d->d % 32 != 0) { set_error("attn(fourbit): head dim %d is not a multiple of 32", d->d); return MCSD_E_UNSUPPORTED; }
    if (d->B > 65535) { set_error("attn(fourbit): B %d > 65535", d->B); return MCSD_E_UNSUPPORTED; }
    if (!make_fourbit_plan(*d, plan)) { set_error("attn(fourbit): no kernel for this shape"); return MCSD_E_UNSUPPORTED; }
    if (!b) return MCSD_OK;
    if (b->struct_size != sizeof(mcsd_attn_bufs)) { set_error("attn bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_attn_bufs)); return MCSD_E_SHAPE; }
    if (!b->q || !b->k_tree || !b->v_tree || !b->prefix_len || !b->parent || !b->out) { set_error("attn(fourbit): NULL buffer"); return MCSD_E_NULL; }
    if (plan->ws_bytes > 0) {
        if (!b->workspace) { set_error("attn(fourbit): workspace is NULL, %zu bytes needed", plan->ws_bytes); return MCSD_E_WORKSPACE; }
        if (b->workspace_bytes < plan->ws_bytes) { set_error("attn(fourbit): workspace %zu < %zu bytes", b->workspace_bytes, plan->ws_bytes); return MCSD_E_WORKSPACE; }
        if (((uintptr_t)b->workspace & 255u) != 0) { set_error("attn(fourbit): workspace not 256-byte aligned"); return MCSD_E_WORKSPACE; }
    }
    if (((uintptr_t)b->q | (uintptr_t)b->k_tree | (uintptr_t)b->v_tree | (uintptr_t)b->out) & 15u) { set_error("attn(fourbit): tensors must be 16-byte aligned"); return MCSD_E_SHAPE; }
    return MCSD_OK;
}

size_t mcsd_attn_fourbit_workspace_bytes(const mcsd_attn_desc *desc)
{
    FourbitPlan plan;
    return check_attn_fourbit(desc, nullptr, &plan) == MCSD_OK ? plan.ws_bytes : 0;
}

int32_t mcsd_tree_attn_fourbit(const mcsd_attn_desc *desc, const mcsd_attn_bufs *bufs, const mcsd_fourbit_kv *kv, void *stream)
{
    FourbitPlan plan;
    if (!bufs) { set_error("attn bufs is NULL"); return MCSD_E_NULL; }
    int32_t rc = check_attn_fourbit(desc, bufs, &plan);
    if (rc != MCSD_OK) return rc;
    rc = check_fourbit(kv, desc->d, desc->L_stride);
    if (rc != MCSD_OK) return rc;
    return launch_attn_fourbit(*desc, *bufs, *kv, plan, (hipStream_t)stream);
}

int32_t mcsd_kv_commit_fourbit(const mcsd_commit_desc *d, const mcsd_commit_bufs *b, const mcsd_fourbit_kv *kv, void *stream)
{
    int32_t rc = check_commit(d, b, false);
    if (rc != MCSD_OK) return rc;
    rc = check_fourbit(kv, d->d, d->L_stride);
    if (rc != MCSD_OK) return rc;
    return launch_kv_commit(*d, *b, (hipStream_t)stream, nullptr, kv);
}

static int32_t check_rows(const mcsd_rows_desc *d, const mcsd_rows_bufs *b, const mcsd_fourbit_kv *kv)
{
    if (!d) { set_error("rows desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_rows_desc)) { set_error("rows desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_rows_desc)); return MCSD_E_SHAPE; }
    if (d->T < 0 || d->H_kv < 1 || d->n_layers < 1) { set_error("rows: non-positive size"); return MCSD_E_SHAPE; }
    if (d->dtype != MCSD_DTYPE_FP32 && d->dtype != MCSD_DTYPE_BF16) { set_error("rows: unknown dtype %d", d->dtype); return MCSD_E_UNSUPPORTED; }
    const int32_t rc = check_fourbit(kv, d->d, -1);
    if (rc != MCSD_OK) return rc;
    // (a launch has fewer than 2^32 threads)
    if (d->n_layers > 65535 || d->T > (1 << 30) || d->H_kv > 65535 || ((long)d->T + 15) / 16 * d->H_kv * (d->d / 32) >= 1L << 26) { set_error("rows: grid too large"); return MCSD_E_UNSUPPORTED; }
    const int64_t row = (int64_t)d->H_kv * d->d, per16 = d->dtype == MCSD_DTYPE_FP32 ? 4 : 8;
    if (d->k_stride < row || d->v_stride < row) { set_error("rows: a stride is less than a row"); return MCSD_E_SHAPE; }
    if (d->k_stride % per16 != 0 || d->v_stride % per16 != 0) { set_error("rows: strides must be multiples of 16 bytes"); return MCSD_E_SHAPE; }
    if (d->n_layers > 1 && (d->k_layer_stride % per16 != 0 || d->v_layer_stride % per16 != 0 || d->k_layer_stride < 0 || d->v_layer_stride < 0)) {
        set_error("rows: layer strides must be multiples of 16 bytes");
        return MCSD_E_SHAPE;
    }
    if (!b) { set_error("rows bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_rows_bufs)) { set_error("rows bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_rows_bufs)); return MCSD_E_SHAPE; }
    if (d->T == 0) return MCSD_OK;
    if (!b->k || !b->v || !b->slot_map) { set_error("rows: NULL buffer"); return MCSD_E_NULL; }
    if (((uintptr_t)b->k | (uintptr_t)b->v) & 15u) { set_error("rows: k and v must be 16-byte aligned"); return MCSD_E_SHAPE; }
    return MCSD_OK;
}

int32_t mcsd_kv_store_fourbit(const mcsd_rows_desc *d, const mcsd_rows_bufs *b, const mcsd_fourbit_kv *kv, void *stream)
{
    const int32_t rc = check_rows(d, b, kv);
    return rc != MCSD_OK ? rc : launch_fourbit_rows(*d, *b, *kv, true, (hipStream_t)stream);
}

int32_t mcsd_kv_load_fourbit(const mcsd_rows_desc *d, const mcsd_rows_bufs *b, const mcsd_fourbit_kv *kv, void *stream)
{
    const int32_t rc = check_rows(d, b, kv);
    return rc != MCSD_OK ? rc : launch_fourbit_rows(*d, *b, *kv, false, (hipStream_t)stream);
}

// ------------------------------------------------- prompts in chunks over a paged cache, eviction
// L_stride > 0: the logical capacity that the block table has to hold (a store by slot has none: 0)
static int32_t check_pages(const char *what, const mcsd_paged_kv *kv, long L_stride)
{
    if (!kv) { set_error("%s: paged descriptor is NULL", what); return MCSD_E_NULL; }
    if (kv->struct_size != sizeof(mcsd_paged_kv)) { set_error("%s: paged struct_size %u != %zu", what, kv->struct_size, sizeof(mcsd_paged_kv)); return MCSD_E_SHAPE; }
    if (kv->page_size < 32 || kv->page_size % 32 != 0) { set_error("%s: page_size %d is not a positive multiple of 32", what, kv->page_size); return MCSD_E_SHAPE; }
    if (kv->n_pages < 1 || (L_stride > 0 && kv->max_pages_per_seq < 1)) { set_error("%s: non-positive size", what); return MCSD_E_SHAPE; }
    if ((long)kv->n_pages * kv->page_size > 0x7fffffffL) { set_error("%s: n_pages * page_size does not fit a slot", what); return MCSD_E_UNSUPPORTED; }
    if (L_stride > 0 && !kv->block_table) { set_error("%s: block_table is NULL", what); return MCSD_E_NULL; }
    if (L_stride > 0 && (long)kv->max_pages_per_seq * kv->page_size < L_stride) { set_error("%s: L_stride %ld exceeds max_pages_per_seq * page_size", what, L_stride); return MCSD_E_SHAPE; }
    return MCSD_OK;
}

static int32_t check_head_dim(const char *what, int d, int dtype)
{
    if (dtype != MCSD_DTYPE_FP32 && dtype != MCSD_DTYPE_BF16) { set_error("%s: unknown dtype %d", what, dtype); return MCSD_E_UNSUPPORTED; }
    if (d < 1 || d > MCSD_MAX_HEAD_DIM || d % (dtype == MCSD_DTYPE_BF16 ? 8 : 4) != 0) { set_error("%s: head dim %d unsupported", what, d); return MCSD_E_UNSUPPORTED; }
    return MCSD_OK;
}

int32_t mcsd_kv_store_paged(const mcsd_rows_desc *d, const mcsd_store_bufs *b, const mcsd_paged_kv *kv, void *stream)
{
    if (!d) { set_error("rows desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_rows_desc)) { set_error("rows desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_rows_desc)); return MCSD_E_SHAPE; }
    if (d->T < 0 || d->H_kv < 1 || d->n_layers < 1) { set_error("rows: non-positive size"); return MCSD_E_SHAPE; }
    int32_t rc = check_head_dim("rows", d->d, d->dtype);
    if (rc != MCSD_OK) return rc;
    rc = check_pages("rows", kv, 0);
    if (rc != MCSD_OK) return rc;
    const int64_t row = (int64_t)d->H_kv * d->d, per16 = d->dtype == MCSD_DTYPE_FP32 ? 4 : 8;
    // (a launch has fewer than 2^32 threads)
    if (d->n_layers > 65535 || d->T > (1 << 30) || d->H_kv > 65535 || d->T * (row / per16) >= 1L << 31) { set_error("rows: grid too large"); return MCSD_E_UNSUPPORTED; }
    if (d->k_stride < row || d->v_stride < row) { set_error("rows: a stride is less than a row"); return MCSD_E_SHAPE; }
    if (d->k_stride % per16 != 0 || d->v_stride % per16 != 0) { set_error("rows: strides must be multiples of 16 bytes"); return MCSD_E_SHAPE; }
    if (d->n_layers > 1 && (d->k_layer_stride % per16 != 0 || d->v_layer_stride % per16 != 0 || d->k_layer_stride < 0 || d->v_layer_stride < 0)) {
        set_error("rows: layer strides must be multiples of 16 bytes");
        return MCSD_E_SHAPE;
    }
    if (!b) { set_error("rows bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_store_bufs)) { set_error("rows bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_store_bufs)); return MCSD_E_SHAPE; }
    if (d->T == 0) return MCSD_OK;
    if (!b->k || !b->v || !b->slot_map || !b->k_pool || !b->v_pool) { set_error("rows: NULL buffer"); return MCSD_E_NULL; }
    if (((uintptr_t)b->k | (uintptr_t)b->v | (uintptr_t)b->k_pool | (uintptr_t)b->v_pool) & 15u) { set_error("rows: k, v and the pools must be 16-byte aligned"); return MCSD_E_SHAPE; }
    return launch_kv_store_paged(*d, *b, *kv, (hipStream_t)stream);
}

static int32_t check_chunk(const mcsd_chunk_desc *d)
{
    if (!d) { set_error("chunk desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_chunk_desc)) { set_error("chunk desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_chunk_desc)); return MCSD_E_SHAPE; }
    if (d->B < 1 || d->T < 0 || d->H_q < 1 || d->H_kv < 1 || d->L_stride < 1) { set_error("chunk: non-positive size"); return MCSD_E_SHAPE; }
    if (d->H_q % d->H_kv != 0) { set_error("chunk: H_q %d not a multiple of H_kv %d", d->H_q, d->H_kv); return MCSD_E_SHAPE; }
    const int32_t rc = check_head_dim("chunk", d->d, d->dtype);
    if (rc != MCSD_OK) return rc;
    if (d->B > 65535 || d->H_kv > 65535) { set_error("chunk: B %d or H_kv %d > 65535", d->B, d->H_kv); return MCSD_E_UNSUPPORTED; }
    if (d->L_stride > (1 << 22)) { set_error("chunk: L_stride %d > %d", d->L_stride, 1 << 22); return MCSD_E_UNSUPPORTED; }
    if ((long)d->T * d->H_q >= 1L << 30) { set_error("chunk: T * H_q %ld >= 2^30", (long)d->T * d->H_q); return MCSD_E_UNSUPPORTED; }
    if (!(d->scale >= 0.f) || !(d->scale < 1e30f)) { set_error("chunk: scale must be finite and >= 0"); return MCSD_E_SHAPE; }
    if (d->q_stride < (int64_t)d->H_q * d->d || d->q_stride % (d->dtype == MCSD_DTYPE_FP32 ? 4 : 8) != 0) { set_error("chunk: q_stride is less than a row or no multiple of 16 bytes"); return MCSD_E_SHAPE; }
    return MCSD_OK;
}

size_t mcsd_chunk_workspace_bytes(const mcsd_chunk_desc *d)
{
    ChunkPlan plan;
    return check_chunk(d) == MCSD_OK && make_chunk_plan(*d, &plan) ? plan.ws_bytes : 0;
}

int32_t mcsd_chunk_attn_paged(const mcsd_chunk_desc *d, const mcsd_chunk_bufs *b, const mcsd_paged_kv *kv, void *stream)
{
    int32_t rc = check_chunk(d);
    if (rc != MCSD_OK) return rc;
    ChunkPlan plan;
    if (!make_chunk_plan(*d, &plan)) { set_error("chunk: no kernel for this shape"); return MCSD_E_UNSUPPORTED; }
    rc = check_pages("chunk", kv, d->L_stride);
    if (rc != MCSD_OK) return rc;
    if (!b) { set_error("chunk bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_chunk_bufs)) { set_error("chunk bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_chunk_bufs)); return MCSD_E_SHAPE; }
    if (d->T == 0) return MCSD_OK;
    if (!b->q || !b->k_pool || !b->v_pool || !b->chunk_start || !b->prefix_len || !b->out) { set_error("chunk: NULL buffer"); return MCSD_E_NULL; }
    if (((uintptr_t)b->q | (uintptr_t)b->k_pool | (uintptr_t)b->v_pool | (uintptr_t)b->out) & 15u) { set_error("chunk: tensors must be 16-byte aligned"); return MCSD_E_SHAPE; }
    if (plan.ws_bytes > 0) {
        if (!b->workspace) { set_error("chunk: workspace is NULL, %zu bytes needed", plan.ws_bytes); return MCSD_E_WORKSPACE; }
        if (b->workspace_bytes < plan.ws_bytes) { set_error("chunk: workspace %zu < %zu bytes", b->workspace_bytes, plan.ws_bytes); return MCSD_E_WORKSPACE; }
        if (((uintptr_t)b->workspace & 255u) != 0) { set_error("chunk: workspace not 256-byte aligned"); return MCSD_E_WORKSPACE; }
    }
    return launch_chunk_attn(*d, *b, *kv, plan, (hipStream_t)stream);
}

int32_t mcsd_attn_weight_sums(const mcsd_chunk_desc *d, const mcsd_sums_bufs *b, const mcsd_paged_kv *kv, void *stream)
{
    int32_t rc = check_chunk(d);
    if (rc != MCSD_OK) return rc;
    rc = check_pages("sums", kv, d->L_stride);
    if (rc != MCSD_OK) return rc;
    if (!b) { set_error("sums bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_sums_bufs)) { set_error("sums bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_sums_bufs)); return MCSD_E_SHAPE; }
    if (b->last_rows < 0) { set_error("sums: last_rows %d < 0", b->last_rows); return MCSD_E_SHAPE; }
    if (d->T == 0) return MCSD_OK;
    if (!b->q || !b->k_pool || !b->chunk_start || !b->prefix_len || !b->lse || !b->sums) { set_error("sums: NULL buffer"); return MCSD_E_NULL; }
    if (((uintptr_t)b->q | (uintptr_t)b->k_pool) & 15u) { set_error("sums: q and the pool must be 16-byte aligned"); return MCSD_E_SHAPE; }
    return launch_weight_sums(*d, *b, *kv, (hipStream_t)stream);
}

int32_t mcsd_kv_evict_paged(const mcsd_evict_desc *d, const mcsd_evict_bufs *b, const mcsd_paged_kv *kv, void *stream)
{
    if (!d) { set_error("evict desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_evict_desc)) { set_error("evict desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_evict_desc)); return MCSD_E_SHAPE; }
    if (d->B < 1 || d->H_kv < 1 || d->L_stride < 1 || d->n_layers < 1 || d->n_first < 0 || d->n_recent < 0) { set_error("evict: non-positive size"); return MCSD_E_SHAPE; }
    int32_t rc = check_head_dim("evict", d->d, d->dtype);
    if (rc != MCSD_OK) return rc;
    if (d->B > 65535 || d->L_stride > (1 << 22) || (__int128)d->n_layers * d->B * d->H_kv >= 1 << 22) { set_error("evict: B, L_stride or n_layers * B * H_kv too large"); return MCSD_E_UNSUPPORTED; }
    rc = check_pages("evict", kv, d->L_stride);
    if (rc != MCSD_OK) return rc;
    if (!b) { set_error("evict bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_evict_bufs)) { set_error("evict bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_evict_bufs)); return MCSD_E_SHAPE; }
    if (!b->k_pool || !b->v_pool || !b->sums || !b->prefix_len || !b->keep_len || !b->kept || !b->flags) { set_error("evict: NULL buffer"); return MCSD_E_NULL; }
    if (((uintptr_t)b->k_pool | (uintptr_t)b->v_pool) & 15u) { set_error("evict: pools must be 16-byte aligned"); return MCSD_E_SHAPE; }
    if (b->out_table == kv->block_table) { set_error("evict: out_table is the block table (NULL moves in place)"); return MCSD_E_SHAPE; }
    return launch_kv_evict(*d, *b, *kv, (hipStream_t)stream);
}

// --------------------------------------------------------- log probabilities of tokens
static int32_t check_logprob(const mcsd_logprob_desc *d)
{
    if (!d) { set_error("logprob desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_logprob_desc)) { set_error("logprob desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_logprob_desc)); return MCSD_E_SHAPE; }
    if (d->rows < 0 || d->R < 1 || d->V < 1 || d->n_top < 0) { set_error("logprob: non-positive size"); return MCSD_E_SHAPE; }
    if (d->V > (1 << 30) || d->rows > (1 << 22)) { set_error("logprob: V %d > 2^30 or rows %d > 2^22", d->V, d->rows); return MCSD_E_UNSUPPORTED; }
    if (d->dtype != MCSD_DTYPE_FP32 && d->dtype != MCSD_DTYPE_BF16) { set_error("logprob: unknown dtype %d", d->dtype); return MCSD_E_UNSUPPORTED; }
    if (d->n_top > MCSD_MAX_TOP || d->n_top > d->V) { set_error("logprob: n_top %d > %d or V", d->n_top, MCSD_MAX_TOP); return MCSD_E_UNSUPPORTED; }
    if (d->row_stride < d->V) { set_error("logprob: row_stride is less than V"); return MCSD_E_SHAPE; }
    return MCSD_OK;
}

size_t mcsd_logprob_workspace_bytes(const mcsd_logprob_desc *d) { return check_logprob(d) == MCSD_OK ? logprob_workspace(*d) : 0; }

int32_t mcsd_token_logprobs(const mcsd_logprob_desc *d, const mcsd_logprob_bufs *b, void *stream)
{
    const int32_t rc = check_logprob(d);
    if (rc != MCSD_OK) return rc;
    if (!b) { set_error("logprob bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_logprob_bufs)) { set_error("logprob bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_logprob_bufs)); return MCSD_E_SHAPE; }
    if (!b->row_map && d->rows > d->R) { set_error("logprob: %d rows of %d without a row_map", d->rows, d->R); return MCSD_E_SHAPE; }
    if (d->rows == 0) return MCSD_OK;
    if (!b->logits || !b->tokens || !b->logprob || !b->flags || (d->n_top > 0 && (!b->top_tok || !b->top_logprob))) { set_error("logprob: NULL buffer"); return MCSD_E_NULL; }
    if ((uintptr_t)b->logits % (d->dtype == MCSD_DTYPE_FP32 ? 4 : 2) != 0) { set_error("logprob: misaligned logits"); return MCSD_E_SHAPE; }
    const size_t need = logprob_workspace(*d);
    if (need > 0) {
        if (!b->workspace) { set_error("logprob: workspace is NULL, %zu bytes needed", need); return MCSD_E_WORKSPACE; }
        if (b->workspace_bytes < need) { set_error("logprob: workspace %zu < %zu bytes", b->workspace_bytes, need); return MCSD_E_WORKSPACE; }
        if (((uintptr_t)b->workspace & 255u) != 0) { set_error("logprob: workspace not 256-byte aligned"); return MCSD_E_WORKSPACE; }
    }
    return launch_token_logprobs(*d, *b, (hipStream_t)stream);
}

// ------------------------------------------------------- pages from lengths, rules on logits
int32_t mcsd_page_assign(const mcsd_page_desc *d, const mcsd_page_bufs *b, void *stream)
{
    if (!d) { set_error("page desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_page_desc)) { set_error("page desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_page_desc)); return MCSD_E_SHAPE; }
    if (d->B < 1 || d->page_size < 1 || d->n_pages < 1 || d->max_pages_per_seq < 1 || d->max_slots < 0) { set_error("pages: non-positive size"); return MCSD_E_SHAPE; }
    if (d->B > 65535 || d->max_slots > (1 << 30)) { set_error("pages: B %d > 65535 or max_slots %d > %d", d->B, d->max_slots, 1 << 30); return MCSD_E_UNSUPPORTED; }
    // (a wavefront goes through a sequence's pages 64 at a time)
    if (d->max_pages_per_seq > (1 << 30)) { set_error("pages: max_pages_per_seq %d > 2^30", d->max_pages_per_seq); return MCSD_E_UNSUPPORTED; }
    if ((long)d->n_pages * d->page_size > 0x7fffffffL) { set_error("pages: n_pages * page_size does not fit a slot"); return MCSD_E_UNSUPPORTED; }
    if (!b) { set_error("page bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_page_bufs)) { set_error("page bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_page_bufs)); return MCSD_E_SHAPE; }
    if (!b->prefix_len || !b->want_len || !b->n_held || !b->block_table || !b->free_pages || !b->n_free || !b->flags) { set_error("pages: NULL buffer"); return MCSD_E_NULL; }
    if (!b->slot_map != !b->slot_start) { set_error("pages: slot_map and slot_start come together"); return MCSD_E_NULL; }
    if (!b->slot_map && d->max_slots > 0) { set_error("pages: max_slots without a slot_map"); return MCSD_E_NULL; }
    return launch_page_assign(*d, *b, (hipStream_t)stream);
}

int32_t mcsd_logits_rules(const mcsd_logits_desc *d, const mcsd_logits_bufs *b, void *stream)
{
    if (!d) { set_error("logits desc is NULL"); return MCSD_E_NULL; }
    if (d->struct_size != sizeof(mcsd_logits_desc)) { set_error("logits desc struct_size %u != %zu", d->struct_size, sizeof(mcsd_logits_desc)); return MCSD_E_SHAPE; }
    if (d->B < 1 || d->V < 1 || d->R < 1 || d->hist_stride < 0 || d->n_bias < 0) { set_error("logits: non-positive size"); return MCSD_E_SHAPE; }
    if (d->N < 0 || d->N > MCSD_MAX_NODES) { set_error("logits: N %d outside 0..%d", d->N, MCSD_MAX_NODES); return MCSD_E_TREE; }
    if (d->B > 65535 || d->V > (1 << 30)) { set_error("logits: B %d > 65535 or V %d > %d", d->B, d->V, 1 << 30); return MCSD_E_UNSUPPORTED; }
    // (a thread's place in them goes on by 2048, and a token's count has 31 bits)
    if (d->hist_stride > (1 << 30) || d->n_bias > (1 << 30)) { set_error("logits: hist_stride %d or n_bias %d > 2^30", d->hist_stride, d->n_bias); return MCSD_E_UNSUPPORTED; }
    if (d->dtype != MCSD_DTYPE_FP32 && d->dtype != MCSD_DTYPE_BF16) { set_error("logits: unknown dtype %d", d->dtype); return MCSD_E_UNSUPPORTED; }
    if (d->parent_per_seq != 0 && d->parent_per_seq != 1) { set_error("logits: parent_per_seq must be 0 or 1"); return MCSD_E_SHAPE; }
    if (d->row_begin < 0 || d->row_begin > d->row_end || d->row_end > 1 + d->N) { set_error("logits: rows %d..%d outside the tree's 0..%d", d->row_begin, d->row_end, 1 + d->N); return MCSD_E_SHAPE; }
    if (!b) { set_error("logits bufs is NULL"); return MCSD_E_NULL; }
    if (b->struct_size != sizeof(mcsd_logits_bufs)) { set_error("logits bufs struct_size %u != %zu", b->struct_size, sizeof(mcsd_logits_bufs)); return MCSD_E_SHAPE; }
    if (!b->logits || !b->out || (d->N > 0 && (!b->parent || !b->cand_tok)) || (d->hist_stride > 0 && (!b->history || !b->hist_len)) ||
        (d->n_bias > 0 && (!b->bias_tok || !b->bias_val))) { set_error("logits: NULL buffer"); return MCSD_E_NULL; }
    if (!b->row_map && d->R != 1 + d->N) { set_error("logits: R %d != 1 + N without a row_map", d->R); return MCSD_E_SHAPE; }
    const uintptr_t esize = d->dtype == MCSD_DTYPE_FP32 ? 4 : 2, in = (uintptr_t)b->logits, out = (uintptr_t)b->out;
    if (in % esize != 0 || out % 4 != 0) { set_error("logits: misaligned"); return MCSD_E_SHAPE; }
    const uintptr_t n = (uintptr_t)d->B * d->R * d->V;
    if (in < out + 4 * n && out < in + esize * n && !(in == out && esize == 4)) { set_error("logits: out overlaps the logits without being them"); return MCSD_E_SHAPE; }
    return launch_logits_rules(*d, *b, (hipStream_t)stream);
}

int32_t mcsd_verify_step(const mcsd_attn_desc *ad, const mcsd_attn_bufs *ab, const mcsd_verify_desc *vd,
                         const mcsd_verify_bufs *vb, void *stream)
{
    AttnPlan plan;
    if (!ab || !vb) { set_error("bufs is NULL"); return MCSD_E_NULL; }
    int32_t rc = check_attn(ad, ab, &plan);
    if (rc != MCSD_OK) return rc;
    rc = check_verify(vd, vb);
    if (rc != MCSD_OK) return rc;
    // The merge of the attention partials and the walk are the two small tail kernels of the step;
    // when the attention is split they go out as one launch after the verification rows, and when
    // it is not, the walk rides on the attention launch, which then follows the verification rows.
    if (plan.use_mfma && plan.n_chunks_max > 1) {
        rc = launch_tree_attn(*ad, *ab, plan, (hipStream_t)stream, nullptr, ATTN_PHASE_MAIN);
        if (rc != MCSD_OK) return rc;
        rc = launch_verify(*vd, *vb, (hipStream_t)stream, false);
        if (rc != MCSD_OK) return rc;
        const WalkParams w = make_walk_params(*vd, *vb);
        return launch_tree_attn(*ad, *ab, plan, (hipStream_t)stream, nullptr, ATTN_PHASE_COMBINE, &w);
    }
    if (plan.use_mfma) {
        // no merge launch: the verification rows go first and the attention launch carries the walk
        rc = launch_verify(*vd, *vb, (hipStream_t)stream, false);
        if (rc != MCSD_OK) return rc;
        const WalkParams w = make_walk_params(*vd, *vb);
        return launch_tree_attn(*ad, *ab, plan, (hipStream_t)stream, nullptr, ATTN_PHASE_MAIN, &w);
    }
    rc = launch_tree_attn(*ad, *ab, plan, (hipStream_t)stream);
    if (rc != MCSD_OK) return rc;
    return launch_verify(*vd, *vb, (hipStream_t)stream);
}

int32_t mcsd_attn_plan_override(int32_t variant, int32_t chunk_tiles, int32_t target_items)
{
    const int32_t rc = attn_plan_override(variant, chunk_tiles, target_items);
    if (rc != MCSD_OK) set_error("plan override: variant must be 0..3, chunk_tiles and target_items >= 0");
    return rc;
}

}  // extern "C"
