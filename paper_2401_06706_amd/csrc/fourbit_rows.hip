// Rows of tokens into a prefix cache held in 4 bits and back, by slot (the commit of an accepted path
// is in tree_commit.hip, attention over the cache in fourbit_attn.hip).
#include "fourbit.h"

namespace mcsd {
namespace {

struct RowsParams {
    int T, H_kv, n_blocks, n_slots, page_size, is_f32;
    size_t pool_blocks;                 // blocks of one layer's pool
    char *k, *v;
    size_t k_stride, v_stride, k_layer, v_layer;        // bytes
    uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
    const int32_t *slot_map;
};

// Bound by memory.  Four lanes a block, eight values each; a wavefront takes TOKENS tokens x 2 blocks of a head: 128-byte
// pieces of a bf16 row, and 128-byte runs of codes where the tokens' slots follow each other.  16384 tokens of 8 heads of 128 (85 MB a
// call): 4 tokens store 17.9, load 16.7 us; 8: 17.6, 14.3; 16: 17.4, 14.3 (from caches; with inputs that take turns 25.0 and 15.4, and
// 27.5 and 32.4 where a thread of the store takes two or four blocks, all of their loads ahead).
// grid (units / 64 per workgroup of 256, 1, layers); unit = ((token / TOKENS) H_kv n_blocks + head n_blocks + block) TOKENS + token % TOKENS.
constexpr int TOKENS = 8;

struct Unit { int t, blk, quarter; size_t row_at; size_t block; bool on; };

__device__ __forceinline__ Unit unit_of(const RowsParams &p)
{
    Unit u;
    const size_t unit = (size_t)blockIdx.x * 64 + (threadIdx.x >> 2);
    const int per = p.H_kv * p.n_blocks;
    const size_t group = unit / TOKENS;
    u.t = (int)(group / per) * TOKENS + (int)(unit % TOKENS);
    const int hb = (int)(group % per), head = hb / p.n_blocks;
    u.blk = hb % p.n_blocks;
    u.quarter = threadIdx.x & 3;
    const int slot = u.t < p.T ? p.slot_map[u.t] : -1;
    u.on = (unsigned)slot < (unsigned)p.n_slots;
    const int page = u.on ? slot / p.page_size : 0, r = u.on ? slot % p.page_size : 0;
    u.block = (size_t)blockIdx.z * p.pool_blocks + fourbit_block(((size_t)page * p.H_kv + head) * p.page_size + r, p.n_blocks, u.blk);
    u.row_at = ((size_t)head * p.n_blocks + u.blk) * FB_BLOCK + 8 * u.quarter;
    return u;
}

__global__ __launch_bounds__(256) void kv_store_fourbit_kernel(RowsParams p)
{
    const Unit u = unit_of(p);
    if (!u.on) return;              // (all four lanes of a block)
    const size_t at = u.row_at * (p.is_f32 ? 4 : 2);
    float k[8], v[8];
    load8(p.k + blockIdx.z * p.k_layer + u.t * p.k_stride + at, p.is_f32, k);
    load8(p.v + blockIdx.z * p.v_layer + u.t * p.v_stride + at, p.is_f32, v);
    const uint32_t ks = fourbit_scale_byte(fourbit_amax_bits(k)), vs = fourbit_scale_byte(fourbit_amax_bits(v));
    reinterpret_cast<uint32_t *>(p.k_codes)[u.block * 4 + u.quarter] = fourbit_encode8(k, ks);
    reinterpret_cast<uint32_t *>(p.v_codes)[u.block * 4 + u.quarter] = fourbit_encode8(v, vs);
    if (u.quarter == 0) {
        p.k_scales[u.block] = (uint8_t)ks;
        p.v_scales[u.block] = (uint8_t)vs;
    }
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void decode8_to(char *at, bool is_f32, uint32_t c, uint32_t scale_byte)
{
    const float s = fourbit_scale(scale_byte);
    if (is_f32) {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
        const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2), f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
        *reinterpret_cast<float4 *>(at) = make_float4(a[0], a[1], b[0], b[1]);
        *reinterpret_cast<float4 *>(at + 16) = make_float4(e[0], e[1], f[0], f[1]);
    } else {
        uint4 o;
        o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
        o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
        o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
        o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
        *reinterpret_cast<uint4 *>(at) = o;
    }
}

__global__ __launch_bounds__(256) void kv_load_fourbit_kernel(RowsParams p)
{
    const Unit u = unit_of(p);
    if (!u.on) return;
    const size_t at = u.row_at * (p.is_f32 ? 4 : 2);
    const uint32_t kc = reinterpret_cast<const uint32_t *>(p.k_codes)[u.block * 4 + u.quarter];
    const uint32_t vc = reinterpret_cast<const uint32_t *>(p.v_codes)[u.block * 4 + u.quarter];
    const uint32_t ks = p.k_scales[u.block], vs = p.v_scales[u.block];
    decode8_to(p.k + blockIdx.z * p.k_layer + u.t * p.k_stride + at, p.is_f32, kc, ks);
    decode8_to(p.v + blockIdx.z * p.v_layer + u.t * p.v_stride + at, p.is_f32, vc, vs);
}

}  // namespace

int32_t launch_fourbit_rows(const mcsd_rows_desc &d, const mcsd_rows_bufs &b, const mcsd_fourbit_kv &kv, bool store, hipStream_t stream)
{
    if (d.T == 0) return MCSD_OK;
    RowsParams p;
    const size_t esize = d.dtype == MCSD_DTYPE_FP32 ? 4 : 2;
    p.T = d.T; p.H_kv = d.H_kv; p.n_blocks = d.d / FB_BLOCK; p.page_size = kv.page_size; p.n_slots = kv.n_pages * kv.page_size;
    p.is_f32 = d.dtype == MCSD_DTYPE_FP32;
    p.pool_blocks = (size_t)p.n_slots * d.H_kv * p.n_blocks;
    p.k = static_cast<char *>(b.k); p.v = static_cast<char *>(b.v);
    p.k_stride = (size_t)d.k_stride * esize; p.v_stride = (size_t)d.v_stride * esize;
    p.k_layer = (size_t)d.k_layer_stride * esize; p.v_layer = (size_t)d.v_layer_stride * esize;
    if (d.n_layers == 1) p.k_layer = p.v_layer = 0;
    p.k_codes = static_cast<uint8_t *>(kv.k_codes); p.v_codes = static_cast<uint8_t *>(kv.v_codes);
    p.k_scales = static_cast<uint8_t *>(kv.k_scales); p.v_scales = static_cast<uint8_t *>(kv.v_scales);
    p.slot_map = b.slot_map;
    const size_t units = ((size_t)d.T + TOKENS - 1) / TOKENS * TOKENS * d.H_kv * p.n_blocks;
    const dim3 grid((unsigned)((units + 63) / 64), 1, d.n_layers);
    if (store) launch_kernel(K_KV_STORE, kv_store_fourbit_kernel, grid, dim3(256), stream, p);
    else launch_kernel(K_KV_LOAD, kv_load_fourbit_kernel, grid, dim3(256), stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("kv rows (4 bits) launch failed: %s", hipGetErrorString(e)); return MCSD_E_HIP; }
    return MCSD_OK;
}

}  // namespace mcsd
