// Block tables, slot map and free list of a paged cache from the lengths that requests are to have.
#include "mcsd_internal.h"

namespace mcsd {
namespace {

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

// Sums of x and y over the threads before this one, and of all threads.  (64 bits: lengths of 2^31 tokens and 65535 sequences)
struct Sums { long long x, y, all_x, all_y; };

template <int NT>
__device__ __forceinline__ Sums scan_block(long long x, long long y, long long (*s_wave)[2])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    long long vx = x, vy = y;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long ux = __shfl_up(vx, o), uy = __shfl_up(vy, o);
        if (lane >= o) { vx += ux; vy += uy; }
    }
    if (NT == 64) return {vx - x, vy - y, __shfl(vx, 63), __shfl(vy, 63)};
    __syncthreads();
    if (lane == 63) { s_wave[wave][0] = vx; s_wave[wave][1] = vy; }
    __syncthreads();
    long long wx = s_wave[lane & (NT / 64 - 1)][0], wy = s_wave[lane & (NT / 64 - 1)][1];
#pragma unroll
    for (int o = 1; o < NT / 64; o <<= 1) {
        const long long ux = __shfl_up(wx, o), uy = __shfl_up(wy, o);
        if (lane >= o) { wx += ux; wy += uy; }
    }
    const long long bx = __shfl(wx, max(wave - 1, 0)), by = __shfl(wy, max(wave - 1, 0));
    return {(wave > 0 ? bx : 0) + vx - x, (wave > 0 ? by : 0) + vy - y, __shfl(wx, NT / 64 - 1), __shfl(wy, NT / 64 - 1)};
}

__device__ __forceinline__ int slot_of(const PageParams &p, int b, int pos)
{
    const int page = p.block_table[(size_t)b * p.max_pages + pos / p.page_size];
    return (unsigned)page < (unsigned)p.n_pages ? page * p.page_size + pos % p.page_size : -1;
}

// What page_assign_kernel does with a sequence's pages, by the wavefront it lies in: a few by the sequence's own lane (most requests go on by a
// page or none: all of them at once), many by all lanes, one sequence after the other.
constexpr int FEW_PAGES = 4;

__device__ __forceinline__ void give_back(const PageParams &p, const Request &r, int b, long long top_of_mine, int lane)
{
    if (r.surplus > 0 && r.surplus <= FEW_PAGES) {
        int32_t *row = p.block_table + (size_t)b * p.max_pages + r.need;
        int page[FEW_PAGES];
#pragma unroll
        for (int i = 0; i < FEW_PAGES; ++i) page[i] = i < r.surplus ? row[i] : 0;
#pragma unroll
        for (int i = 0; i < FEW_PAGES; ++i)
            if (i < r.surplus) {
                if (top_of_mine - i < p.n_pages) p.free_pages[top_of_mine - i] = page[i];
                row[i] = -1;
            }
    }
    unsigned long long todo = __ballot(r.surplus > FEW_PAGES);
    while (todo) {
        const int l = __ffsll((long long)todo) - 1;
        todo &= todo - 1;
        const int n = __shfl(r.surplus, l), need = __shfl(r.need, l), seq = __shfl(b, l);
        const long long top = __shfl(top_of_mine, l);
        int32_t *row = p.block_table + (size_t)seq * p.max_pages + need;
        for (int i = lane; i < n; i += 64) {
            if (top - i < p.n_pages) p.free_pages[top - i] = row[i];
            row[i] = -1;
        }
    }
}

__device__ __forceinline__ void take(const PageParams &p, const Request &r, bool served, int b, int top_of_mine, int lane)
{
    if (served && r.lack > 0 && r.lack <= FEW_PAGES) {
        int32_t *row = p.block_table + (size_t)b * p.max_pages + r.held;
        int page[FEW_PAGES];
#pragma unroll
        for (int i = 0; i < FEW_PAGES; ++i) page[i] = i < r.lack ? p.free_pages[top_of_mine - i] : 0;
#pragma unroll
        for (int i = 0; i < FEW_PAGES; ++i)
            if (i < r.lack) row[i] = page[i];
    }
    unsigned long long todo = __ballot(served && r.lack > FEW_PAGES);
    while (todo) {
        const int l = __ffsll((long long)todo) - 1;
        todo &= todo - 1;
        const int n = __shfl(r.lack, l), held = __shfl(r.held, l), seq = __shfl(b, l), top = __shfl(top_of_mine, l);
        int32_t *row = p.block_table + (size_t)seq * p.max_pages + held;
        for (int i = lane; i < n; i += 64) row[i] = p.free_pages[top - i];
    }
}

// One workgroup: the stack's bookkeeping is running sums over the sequences.  NT threads, one sequence each where they are enough, which then costs a trip to
// memory for the lengths, two pairs of sums, and a trip each for pages that come back and that go out (1024
// sequences, 16 wavefronts: 11 us; a form that went over the sequences three times, a sum at a time, 15; 16 sequences in one
// wavefront, no barrier, 4.1).  SLOTS: the slot map too, where it is short: a launch of its own is 4 us.
template <int NT, bool SLOTS>
__global__ __launch_bounds__(NT) void page_assign_kernel(PageParams p)
{
    __shared__ long long s_wave[NT / 64][2];
    __shared__ int s_first[SLOTS ? NT + 1 : 1], s_prefix[SLOTS ? NT : 1];
    const int tid = threadIdx.x, lane = tid & 63;
    const int free0 = min(max(*p.n_free, 0), p.n_pages);
    if (p.B <= NT) {
        const int b = tid;
        const Request r = request_of(p, b);
        const Sums s = scan_block<NT>(r.surplus, r.lack, s_wave);
        const int stacked = (int)min((long long)free0 + s.all_x, (long long)p.n_pages);
        const bool served = b < p.B && r.flags == 0u && (r.lack == 0 || s.y + r.lack <= stacked);
        give_back(p, r, b, (long long)free0 + s.all_x - 1 - s.x, lane);
        const Sums t = scan_block<NT>(served ? r.lack : 0, served ? r.tokens : 0, s_wave);
        if (NT > 64) __syncthreads();
        else __threadfence_block();
        take(p, r, served, b, stacked - 1 - (int)min(s.y, (long long)stacked), lane);
        const long long end = t.y + (served ? r.tokens : 0);
        if (b < p.B) {
            uint32_t flags = r.flags;
            if (r.surplus > 0 && (long long)free0 + s.all_x - 1 - s.x >= p.n_pages) flags |= MCSD_FLAG_BAD_PAGES;      // (a page past the end of the stack is lost)
            if (!served && r.flags == 0u) flags |= MCSD_FLAG_CACHE_FULL;
            if (p.slot_start) {
                if (b == 0) p.slot_start[0] = 0;
                if (served && r.tokens > 0 && end > p.max_slots) flags |= MCSD_FLAG_SLOTS_FULL;
                p.slot_start[b + 1] = (int)min(end, (long long)p.max_slots);
            }
            p.flags[b] = flags;
            if (served) p.n_held[b] = r.need;
        }
        if (tid == 0) *p.n_free = stacked - (int)t.all_x;
        if (!SLOTS) return;
        if (b < p.B) {
            s_first[b] = (int)min(t.y, (long long)p.max_slots);
            s_prefix[b] = p.prefix_len[b];
        }
        __syncthreads();
        const int used = (int)min(t.all_y, (long long)p.max_slots);
        for (int i = tid; i < p.max_slots; i += NT) {
            int slot = -1;
            if (i < used) {
                int lo = 0, hi = p.B - 1;          // the last sequence whose slots begin at or before i
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (s_first[mid] <= i) lo = mid;
                    else hi = mid - 1;
                }
                slot = slot_of(p, lo, s_prefix[lo] + i - s_first[lo]);
            }
            p.slot_map[i] = slot;
        }
        return;
    }
    // More sequences than threads.  What comes back first: all of it is known before anything is stacked, because the first page lies on top.
    long long back = 0;
    for (int b0 = 0; b0 < p.B; b0 += NT) back += scan_block<NT>(request_of(p, b0 + tid).surplus, 0, s_wave).all_x;
    const int stacked = (int)min((long long)free0 + back, (long long)p.n_pages);
    long long before = 0;
    for (int b0 = 0; b0 < p.B; b0 += NT) {
        const int b = b0 + tid;
        const Request r = request_of(p, b);
        const Sums s = scan_block<NT>(r.surplus, 0, s_wave);
        const long long top = (long long)free0 + back - 1 - before - s.x;
        before += s.all_x;
        give_back(p, r, b, top, lane);
        if (b < p.B) p.flags[b] = r.flags | (r.surplus > 0 && top >= p.n_pages ? MCSD_FLAG_BAD_PAGES : 0u);
    }
    __syncthreads();
    long long asked = 0, given = 0, slots = 0;
    for (int b0 = 0; b0 < p.B; b0 += NT) {
        const int b = b0 + tid;
        const Request r = request_of(p, b);
        const Sums s = scan_block<NT>(r.lack, 0, s_wave);
        const long long at = asked + s.x;
        asked += s.all_x;
        const bool served = b < p.B && r.flags == 0u && (r.lack == 0 || at + r.lack <= stacked);
        const Sums t = scan_block<NT>(served ? r.lack : 0, served ? r.tokens : 0, s_wave);
        given += t.all_x;
        const long long end = slots + t.y + (served ? r.tokens : 0);
        slots += t.all_y;
        take(p, r, served, b, stacked - 1 - (int)min(at, (long long)stacked), lane);
        if (b < p.B) {
            uint32_t more = served || r.flags ? 0u : (uint32_t)MCSD_FLAG_CACHE_FULL;
            if (served) p.n_held[b] = r.need;
            if (p.slot_start) {
                if (b == 0) p.slot_start[0] = 0;
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

// Slots that the one workgroup lists itself: 1000 take it 1.5 us more, a launch of their own is 4.7.
constexpr int SLOTS_TOGETHER = 2048;

}  // namespace

int32_t launch_page_assign(const mcsd_page_desc &d, const mcsd_page_bufs &b, hipStream_t stream)
{
    PageParams p;
    p.B = d.B; p.page_size = d.page_size; p.n_pages = d.n_pages; p.max_pages = d.max_pages_per_seq; p.max_slots = d.max_slots;
    p.prefix_len = b.prefix_len; p.want_len = b.want_len; p.n_held = b.n_held; p.block_table = b.block_table;
    p.free_pages = b.free_pages; p.n_free = b.n_free; p.slot_start = b.slot_start; p.slot_map = b.slot_map; p.flags = b.flags;
    // The slot map in the same launch while one workgroup is not longer at it than a launch takes
    const bool together = d.max_slots > 0 && d.B <= 1024 && d.max_slots <= SLOTS_TOGETHER;
    auto go = [&](auto kernel, int threads) { launch_kernel(K_PAGE_ASSIGN, kernel, dim3(1), dim3(threads), stream, p); };
    if (d.B <= 64 && d.max_slots <= 256) { if (together) go(page_assign_kernel<64, true>, 64); else go(page_assign_kernel<64, false>, 64); }
    else if (d.B <= 256 && together) go(page_assign_kernel<256, true>, 256);
    else if (d.B <= 256) go(page_assign_kernel<256, false>, 256);
    else if (together) go(page_assign_kernel<1024, true>, 1024);
    else go(page_assign_kernel<1024, false>, 1024);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("page_assign launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    if (d.max_slots == 0 || together) return MCSD_OK;
    launch_kernel(K_PAGE_SLOTS, page_slots_kernel, dim3((d.max_slots + 255) / 256), dim3(256), stream, p);
    e = hipGetLastError();
    if (e != hipSuccess) { set_error("page_slots launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
