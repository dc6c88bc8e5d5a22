// A paged cache cut to a budget: what every (layer, sequence, KV head) keeps, by the sums of its attention weights, and
// the move of what is kept.
#include "chunk_common.h"

namespace mcsd {
namespace {

struct EvictParams {
    int B, H_kv, L_stride, n_layers, n_first, n_recent, page_size, n_pages, max_pages, row_bytes, row_lanes;
    FastDiv page;                   // by the page size
    size_t pool_layer;              // bytes of one layer's pool
    char *k_pool, *v_pool;
    float *sums;
    int32_t *prefix_len, *kept;
    const int32_t *keep_len, *block_table, *out_table;
    uint32_t *flags;
};

constexpr int SEL_PER = 16;

// order of sums as whole numbers: no number first, then -infinity .. infinity, both zeros alike
__device__ __forceinline__ uint32_t order_key(float x)
{
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}

// A workgroup per (layer, sequence, KV head).  The sum that decides is found digit by digit (of 11, 11 and 10 bits, counts of all digits
// in LDS), then what is kept is written down in ascending order: positions are dealt out in rows of NT, so that the counts per row and
// wavefront, summed up, give every position its place.  Up to 16 NT positions stay in registers (NT by the caches' capacity: barriers of few wavefronts are
// cheap, and more workgroups share a CU); longer ones are read again by every pass.
template <int SEL_NT>
__global__ __launch_bounds__(SEL_NT) void evict_select_kernel(EvictParams p)
{
    constexpr int SEL_CHUNK = SEL_NT * SEL_PER, SEL_WAVES = SEL_NT / 64, BINS = 2048 / SEL_NT;
    __shared__ uint32_t s_count[2048], s_scan[SEL_PER * SEL_WAVES], s_wave[SEL_WAVES], s_pick[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int head = blockIdx.x, b = head / p.H_kv % p.B;
    const int n = max(0, min(p.prefix_len[b], p.L_stride)), m = min(n, max(0, p.keep_len[b]));
    const int f = min(p.n_first, m), r = min(p.n_recent, m - f);
    float *sums = p.sums + (size_t)head * p.L_stride;
    int32_t *kept = p.kept + (size_t)head * p.L_stride;
    if (head < p.B * p.H_kv && head % p.H_kv == 0 && tid == 0) p.flags[b] = 0;      // (the move's workgroups add to it)
    if (m == n) {
        for (int j = tid; j < n; j += SEL_NT) kept[j] = j;
        return;
    }
    const int chunks = (n + SEL_CHUNK - 1) / SEL_CHUNK, to = n - r;                 // between f and `to` the sums decide
    float val[SEL_PER];
    auto load = [&](int chunk) {
#pragma unroll
        for (int i = 0; i < SEL_PER; ++i) {
            const int at = chunk * SEL_CHUNK + i * SEL_NT + tid;
            val[i] = at < n ? sums[at] : 0.f;
        }
    };
    load(0);
    uint32_t prefix = 0, left = m - f - r;      // digits so far; how many of those that begin with them are kept
    if (left > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, above = pass == 1 ? 21 : 10;
            const uint32_t digits = pass == 2 ? 1023u : 2047u;
#pragma unroll
            for (int k = 0; k < BINS; ++k) s_count[k * SEL_NT + tid] = 0;
            __syncthreads();
            for (int c = 0; c < chunks; ++c) {
                if (chunks > 1) load(c);
#pragma unroll
                for (int i = 0; i < SEL_PER; ++i) {
                    if (c * SEL_CHUNK + i * SEL_NT >= n) break;
                    const int at = c * SEL_CHUNK + i * SEL_NT + tid;
                    const uint32_t key = order_key(val[i]);
                    const bool on = at >= f && at < to && (pass == 0 || (key >> above) == prefix);
                    const uint32_t digit = (key >> shift) & digits;
                    const unsigned long long all = __ballot(on);
                    if (!all) continue;
                    // one addition for the lanes that agree with the first of them (sums of 0 are many)
                    const uint32_t d0 = __builtin_amdgcn_readlane(digit, __ffsll((long long)all) - 1);
                    const unsigned long long same = __ballot(on && digit == d0);
                    if (lane == 0) atomicAdd(&s_count[d0], (uint32_t)__popcll(same));
                    if (on && digit != d0) atomicAdd(&s_count[digit], 1u);
                }
            }
            __syncthreads();
            // the digit at which the counts from the top reach `left`: BINS digits a thread
            uint32_t bins[BINS], mine = 0;
#pragma unroll
            for (int k = 0; k < BINS; ++k) { bins[k] = s_count[2047 - BINS * tid - k]; mine += bins[k]; }
            uint32_t upto = wave_running_sum(mine);
            if (lane == 63) s_wave[wave] = upto;
            __syncthreads();
            for (int w = 0; w < wave; ++w) upto += s_wave[w];
            uint32_t before = upto - mine;
            if (upto >= left && before < left) {
#pragma unroll
                for (int k = 0; k < BINS; ++k) {
                    if (before < left && before + bins[k] >= left) { s_pick[0] = 2047 - BINS * tid - k; s_pick[1] = left - before; }
                    before += bins[k];
                }
            }
            __syncthreads();
            prefix = (prefix << (pass == 2 ? 10 : 11)) | s_pick[0];
            left = s_pick[1];
        }
    }
    const bool some = m - f - r > 0;            // keys above `prefix` are kept, and the first `left` of those that are equal
    int equal_before = 0, kept_before = 0;
    // running sum of the counts of (row, wavefront), in place; returns their total
    constexpr int COUNTS = SEL_PER * SEL_WAVES, COUNT_WAVES = COUNTS / 64;
    static_assert(COUNT_WAVES <= SEL_WAVES && COUNTS % 64 == 0, "a count a thread");
    auto scan_counts = [&]() -> int {
        uint32_t mine = 0, upto = 0;
        __syncthreads();
        if (tid < COUNTS) {
            mine = s_scan[tid];
            upto = wave_running_sum(mine);
            if (lane == 63) s_wave[wave] = upto;
        }
        __syncthreads();
        if (tid < COUNTS) {
            for (int w = 0; w < wave; ++w) upto += s_wave[w];
            s_scan[tid] = upto - mine;
        }
        int total = 0;
#pragma unroll
        for (int w = 0; w < COUNT_WAVES; ++w) total += s_wave[w];
        __syncthreads();
        return total;
    };
    const unsigned long long below = (1ull << lane) - 1;
    for (int c = 0; c < chunks; ++c) {
        if (chunks > 1) load(c);
        uint32_t take = 0, equal = 0;
#pragma unroll
        for (int i = 0; i < SEL_PER; ++i) {
            const int at = c * SEL_CHUNK + i * SEL_NT + tid;
            if (c * SEL_CHUNK + i * SEL_NT >= n) {
                if (lane == 0) s_scan[i * SEL_WAVES + wave] = 0;
                continue;
            }
            const uint32_t key = order_key(val[i]);
            const bool between = at >= f && at < to;
            if (at < n && (!between || (some && key > prefix))) take |= 1u << i;
            const bool eq = between && some && key == prefix;
            if (eq) equal |= 1u << i;
            const int cnt = __popcll(__ballot(eq));
            if (lane == 0) s_scan[i * SEL_WAVES + wave] = cnt;
        }
        const int equals = scan_counts();
#pragma unroll
        for (int i = 0; i < SEL_PER; ++i) {
            if (c * SEL_CHUNK + i * SEL_NT >= n) break;
            const unsigned long long eq = __ballot((equal >> i) & 1u);
            const uint32_t rank = equal_before + s_scan[i * SEL_WAVES + wave] + __popcll(eq & below);
            if (((equal >> i) & 1u) && rank < left) take |= 1u << i;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < SEL_PER; ++i) {
            const int cnt = __popcll(__ballot((take >> i) & 1u));
            if (lane == 0) s_scan[i * SEL_WAVES + wave] = cnt;
        }
        const int takes = scan_counts();
        // (all sums of this chunk have been read; those kept go no farther back than they stood)
#pragma unroll
        for (int i = 0; i < SEL_PER; ++i) {
            if (c * SEL_CHUNK + i * SEL_NT >= n) break;
            const unsigned long long on = __ballot((take >> i) & 1u);
            if ((take >> i) & 1u) {
                const int place = kept_before + s_scan[i * SEL_WAVES + wave] + __popcll(on & below);
                kept[place] = c * SEL_CHUNK + i * SEL_NT + tid;
                sums[place] = val[i];
            }
        }
        equal_before += equals;
        kept_before += takes;
        __syncthreads();
    }
}

// Rows of K or V to their new places, 8 pieces of 16 bytes a thread: kept position, page entries, row, three trips to memory behind each
// other, so that many rows are under way at a time.
// In place a workgroup takes 128 bytes of all rows of a (layer, sequence, KV head), a row for each of its threads a step in ascending order, everything of a step read
// before any of it is written: a row moves to a lower position or stays, so that a step writes only what itself and the
// steps before it have read.  To pages of their own, a workgroup of 256 takes a step of whole rows.  grid (heads, 2 x slices, steps or 1)
// Bound by memory where much is kept: 1024 rows of 256 bytes of 1024 heads, keys and values, 228 us (1.07 GB read and written, 4.7 TB/s).
template <bool IN_PLACE, int NT>
__global__ __launch_bounds__(NT) void evict_move_kernel(EvictParams p)
{
    constexpr int U = 8;
    const int tid = threadIdx.x, head = blockIdx.x, g = head % p.H_kv, b = head / p.H_kv % p.B, layer = head / p.H_kv / p.B;
    const int len = max(0, min(p.prefix_len[b], p.L_stride)), keep = max(0, p.keep_len[b]), m = min(len, keep);
    const int moved = IN_PLACE && len < keep ? 0 : m;           // (all is kept where it stands)
    const bool value = blockIdx.y & 1;
    // (to other pages: as many lanes a row as it has pieces, rounded up to a power of two)
    const int lanes = IN_PLACE ? 8 : p.row_lanes, rows = NT / lanes;
    const int col = IN_PLACE ? (blockIdx.y >> 1) * 128 + 16 * (tid & 7) : 16 * (tid & (lanes - 1)), my_row = IN_PLACE ? tid >> 3 : tid / lanes;
    char *pool = (value ? p.v_pool : p.k_pool) + (size_t)layer * p.pool_layer;
    const int32_t *kept = p.kept + (size_t)head * p.L_stride;
    const int32_t *from = p.block_table + (size_t)b * p.max_pages;
    const int32_t *to = IN_PLACE ? from : p.out_table + (size_t)b * p.max_pages;
    bool bad = false;
    for (int base = blockIdx.z * rows * U; base < moved; base += gridDim.z * rows * U) {
        u32x4 x[U];
        int i[U], src[U], dst[U];
        uint32_t on = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = base + rows * u + my_row;
            i[u] = j < m && col < p.row_bytes ? kept[j] : -1;
            if (IN_PLACE && i[u] == j) i[u] = -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = base + rows * u + my_row;
            src[u] = dst[u] = 0;
            if (i[u] >= 0) {
                src[u] = from[p.page.of(i[u])];
                dst[u] = to[p.page.of(j)];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i[u] < 0) continue;
            if ((unsigned)src[u] >= (unsigned)p.n_pages || (unsigned)dst[u] >= (unsigned)p.n_pages) { bad = true; continue; }
            x[u] = *reinterpret_cast<const u32x4 *>(pool + (((size_t)src[u] * p.H_kv + g) * p.page_size + (i[u] - p.page.of(i[u]) * p.page_size)) * p.row_bytes + col);
            on |= 1u << u;
        }
        if (IN_PLACE) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // (the rows have arrived before others write)
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = base + rows * u + my_row;
            if ((on >> u) & 1u)
                *reinterpret_cast<u32x4 *>(pool + (((size_t)dst[u] * p.H_kv + g) * p.page_size + (j - p.page.of(j) * p.page_size)) * p.row_bytes + col) = x[u];
        }
    }
    if (bad) atomicOr(&p.flags[b], (uint32_t)MCSD_FLAG_BAD_PAGES);
    // (every workgroup reads the smaller of this and keep_len, which is m before and after)
    if (head < p.B * p.H_kv && g == 0 && blockIdx.y == 0 && blockIdx.z == 0 && tid == 0) p.prefix_len[b] = m;
}

}  // namespace

int32_t launch_kv_evict(const mcsd_evict_desc &d, const mcsd_evict_bufs &b, const mcsd_paged_kv &kv, hipStream_t stream)
{
    EvictParams p;
    p.B = d.B; p.H_kv = d.H_kv; p.L_stride = d.L_stride; p.n_layers = d.n_layers; p.n_first = d.n_first; p.n_recent = d.n_recent;
    p.page_size = kv.page_size; p.n_pages = kv.n_pages; p.max_pages = kv.max_pages_per_seq;
    p.page = FastDiv(kv.page_size);
    p.row_bytes = d.d * (d.dtype == MCSD_DTYPE_FP32 ? 4 : 2);
    p.row_lanes = 1;
    while (p.row_lanes * 16 < p.row_bytes) p.row_lanes *= 2;
    p.pool_layer = (size_t)kv.n_pages * kv.page_size * d.H_kv * p.row_bytes;
    p.k_pool = static_cast<char *>(b.k_pool); p.v_pool = static_cast<char *>(b.v_pool);
    p.sums = b.sums; p.prefix_len = b.prefix_len; p.kept = b.kept; p.keep_len = b.keep_len;
    p.block_table = kv.block_table; p.out_table = b.out_table; p.flags = b.flags;
    const unsigned heads = (unsigned)(d.n_layers * d.B * d.H_kv);
    // us of the selection with 256, 512 and 1024 threads by capacity and with 1024: 8 heads of 1200 11.2, 11.5; 512 of 1000 to 4000 19.9, 23.3; 1024 of
    // 2048 to 8192 36.8, 58.7
    if (d.L_stride <= 256 * SEL_PER) launch_kernel(K_EVICT_SELECT, evict_select_kernel<256>, dim3(heads), dim3(256), stream, p);
    else if (d.L_stride <= 512 * SEL_PER) launch_kernel(K_EVICT_SELECT, evict_select_kernel<512>, dim3(heads), dim3(512), stream, p);
    else launch_kernel(K_EVICT_SELECT, evict_select_kernel<1024>, dim3(heads), dim3(1024), stream, p);
    if (!b.out_table) {
        const dim3 grid(heads, 2 * ((p.row_bytes + 127) / 128));
        // Steps of 1024 rows where the chip has room for them, of 256 where there are more workgroups: 2304 heads with 13 of up to 375 rows of 128 bytes kept
        // 40.7 and 10.7 us, 512 heads with 512 of 1000 rows of 256 bytes 69 and 61; 128 heads with 2048 of 4096 60 and 91.
        if (grid.x * grid.y >= 1024) launch_kernel(K_EVICT_MOVE, evict_move_kernel<true, 256>, grid, dim3(256), stream, p);
        else launch_kernel(K_EVICT_MOVE, evict_move_kernel<true, 1024>, grid, dim3(1024), stream, p);
    } else {
        // (workgroups that find nothing to move are many where the caches are longer than what is kept: a few per CU go through all steps)
        const unsigned step = 8 * 256 / p.row_lanes, steps = (d.L_stride + step - 1) / step, wanted = (8192 + 2 * heads - 1) / (2 * heads);
        launch_kernel(K_EVICT_MOVE, evict_move_kernel<false, 256>, dim3(heads, 2, steps < wanted ? steps : wanted), dim3(256), stream, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("evict launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
