// Block tables, slot map and free list of a paged cache from the lengths that requests are to have.
#include "mcsd_internal.h"

namespace mcsd {
namespace {

constexpr int PAGE_THREADS = 1024;

struct PageParams {
    int B, page_size, n_pages, max_pages, max_slots;
    const int32_t *prefix_len, *want_len;
    int32_t *n_held, *block_table, *free_pages, *n_free, *slot_start, *slot_map;
    uint32_t *flags;
};

// What sequence b asks for: pages that go back (surplus) or are lacking, new tokens.
struct Request { int held, need, surplus, lack, tokens; uint32_t flags; };

__device__ __forceinline__ Request request_of(const PageParams &p, int b)
{
    Request r = {0, 0, 0, 0, 0, 0u};
    if (b >= p.B) return r;
    const int want = p.want_len[b], prefix = p.prefix_len[b];
    r.held = p.n_held[b];
    r.need = r.held;
    if (want < 0 || prefix < 0 || r.held < 0 || r.held > p.max_pages) {
        r.flags = MCSD_FLAG_BAD_PAGES;
        return r;
    }
    const int need = want / p.page_size + (want % p.page_size != 0);
    if (need > p.max_pages) {
        r.flags = MCSD_FLAG_CACHE_FULL;
        return r;
    }
    r.need = need;
    r.surplus = max(0, r.held - need);
    r.lack = max(0, need - r.held);
    r.tokens = max(0, want - prefix);
    return r;
}

// Sum over the threads before this one, and of all threads.  (64 bits: lengths of 2^31 tokens and 65535 sequences)
__device__ __forceinline__ long long scan_block(long long x, long long *s_wave, long long *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    long long v = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = v;
    __syncthreads();
    long long w = s_wave[lane & (PAGE_THREADS / 64 - 1)];
#pragma unroll
    for (int o = 1; o < PAGE_THREADS / 64; o <<= 1) {
        const long long u = __shfl_up(w, o);
        if (lane >= o) w += u;
    }
    *total = __shfl(w, PAGE_THREADS / 64 - 1);
    const long long before = __shfl(w, max(wave - 1, 0));
    return (wave > 0 ? before : 0) + v - x;
}

__device__ __forceinline__ int slot_of(const PageParams &p, int b, int pos)
{
    const int page = p.block_table[(size_t)b * p.max_pages + pos / p.page_size];
    return (unsigned)page < (unsigned)p.n_pages ? page * p.page_size + pos % p.page_size : -1;
}

// One workgroup: the stack's bookkeeping is two running sums over the sequences.
__global__ __launch_bounds__(PAGE_THREADS) void page_assign_kernel(PageParams p)
{
    __shared__ long long s_wave[PAGE_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int free0 = min(max(*p.n_free, 0), p.n_pages);
    // 1. what comes back: all of it is known before anything is stacked, because the first page lies on top
    long long back = 0, all;
    for (int b0 = 0; b0 < p.B; b0 += PAGE_THREADS) {
        const Request r = request_of(p, b0 + tid);
        scan_block(r.surplus, s_wave, &all);
        back += all;
    }
    long long before = 0;
    for (int b0 = 0; b0 < p.B; b0 += PAGE_THREADS) {
        const int b = b0 + tid;
        const Request r = request_of(p, b);
        const long long at = before + scan_block(r.surplus, s_wave, &all);
        before += all;
        // a wavefront gives back the pages of its sequences one sequence after the other
        unsigned long long todo = __ballot(r.surplus > 0);
        while (todo) {
            const int l = __ffsll((long long)todo) - 1;
            todo &= todo - 1;
            const int n = __shfl(r.surplus, l), need = __shfl(r.need, l), seq = __shfl(b, l);
            const long long top = (long long)free0 + back - 1 - __shfl(at, l);
            int32_t *row = p.block_table + (size_t)seq * p.max_pages + need;
            for (int i = lane; i < n; i += 64) {
                if (top - i < p.n_pages) p.free_pages[top - i] = row[i];
                row[i] = -1;
            }
        }
        // (a page past the end of the stack is lost)
        if (b < p.B) p.flags[b] = r.flags | (r.surplus > 0 && (long long)free0 + back - 1 - at >= p.n_pages ? MCSD_FLAG_BAD_PAGES : 0u);
    }
    const int stacked = (int)min((long long)free0 + back, (long long)p.n_pages);
    __syncthreads();
    // 2. what is lacking, in order while it lasts; 3. where the slots of a sequence begin
    long long asked = 0, given = 0, slots = 0;
    for (int b0 = 0; b0 < p.B; b0 += PAGE_THREADS) {
        const int b = b0 + tid;
        const Request r = request_of(p, b);
        const long long at = asked + scan_block(r.lack, s_wave, &all);
        asked += all;
        const bool served = r.flags == 0u && (r.lack == 0 || at + r.lack <= stacked);
        scan_block(served ? r.lack : 0, s_wave, &all);
        given += all;
        const long long first = slots + scan_block(served ? r.tokens : 0, s_wave, &all);
        slots += all;
        unsigned long long todo = __ballot(served && r.lack > 0);
        while (todo) {
            const int l = __ffsll((long long)todo) - 1;
            todo &= todo - 1;
            const int n = __shfl(r.lack, l), held = __shfl(r.held, l), seq = __shfl(b, l);
            const int top = stacked - 1 - (int)__shfl(at, l);
            int32_t *row = p.block_table + (size_t)seq * p.max_pages + held;
            for (int i = lane; i < n; i += 64) row[i] = p.free_pages[top - i];
        }
        if (b < p.B) {
            uint32_t more = served || r.flags ? 0u : (uint32_t)MCSD_FLAG_CACHE_FULL;
            if (served) p.n_held[b] = r.need;
            if (p.slot_start) {
                if (b == 0) p.slot_start[0] = 0;
                const long long end = first + (served ? r.tokens : 0);
                if (served && r.tokens > 0 && end > p.max_slots) more |= MCSD_FLAG_SLOTS_FULL;
                p.slot_start[b + 1] = (int)min(end, (long long)p.max_slots);
            }
            if (more) p.flags[b] |= more;
        }
    }
    if (tid == 0) *p.n_free = stacked - (int)given;
}

// A thread per slot: its sequence by halving slot_start.
__global__ __launch_bounds__(256) void page_slots_kernel(PageParams p)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= p.max_slots) return;
    int slot = -1;
    if (i < p.slot_start[p.B]) {
        int lo = 0, hi = p.B - 1;          // the last sequence whose slots begin at or before i
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.slot_start[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        slot = slot_of(p, lo, p.prefix_len[lo] + i - p.slot_start[lo]);
    }
    p.slot_map[i] = slot;
}

}  // namespace

int32_t launch_page_assign(const mcsd_page_desc &d, const mcsd_page_bufs &b, hipStream_t stream)
{
    PageParams p;
    p.B = d.B; p.page_size = d.page_size; p.n_pages = d.n_pages; p.max_pages = d.max_pages_per_seq; p.max_slots = d.max_slots;
    p.prefix_len = b.prefix_len; p.want_len = b.want_len; p.n_held = b.n_held; p.block_table = b.block_table;
    p.free_pages = b.free_pages; p.n_free = b.n_free; p.slot_start = b.slot_start; p.slot_map = b.slot_map; p.flags = b.flags;
    launch_kernel(K_PAGE_ASSIGN, page_assign_kernel, dim3(1), dim3(PAGE_THREADS), stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("page_assign launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    if (d.max_slots == 0) return MCSD_OK;
    launch_kernel(K_PAGE_SLOTS, page_slots_kernel, dim3((d.max_slots + 255) / 256), dim3(256), stream, p);
    e = hipGetLastError();
    if (e != hipSuccess) { set_error("page_slots launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
