// Pages of a cache in 4 bits to 16-bit pages (decode_attn_expand_kv).
//
// Bound by memory: 4.5 bits read and 16 written a value.  A warp takes tiles of one KV head (2,304 contiguous bytes at head_dim
// 128): it copies them to a ring of its own (cp.async, two tiles ahead), and 16 lanes (8 at head_dim 64) write a row of K or V
// whole, 16 bytes a lane, from one word of codes each.  (96,000 tokens of 8 heads of 128: 502 MB in 90 us, 5.56 TB/s; a plain
// copy's rate would be 77 us.  With the tiles in registers instead, 128 of them, the same.)
#include <cstring>

#include "common.cuh"
#include "opt_in.h"
#include "packed.cuh"
#include "planner.h"

using namespace da;

namespace {

constexpr int kExpandThreads = 256;
constexpr int kExpandTiles = 8;        // tiles of a sequence that a block takes, all KV heads of them
constexpr int kExpandRing = 3;         // tiles in a warp's ring

struct ExpandParams {
    const char* pool;
    const int32_t *block_table, *seq_lens, *dst_table;
    uint16_t *k, *v;
    int32_t* status;
    int64_t src_stride_page, src_stride_head, src_pages, num_pages;
    int64_t k_stride_page, k_stride_token, k_stride_head;
    int64_t v_stride_page, v_stride_token, v_stride_head;
    int32_t num_kv_heads, src_width, dst_width, page_shift;
};

template <bool F16>
__device__ __forceinline__ uint32_t round_pair(float lo, float hi)
{
    if (F16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <bool F16>
__device__ __forceinline__ uint4 expand_word(uint32_t w, __half scale)
{
    uint32_t c[4], r[4];
    packed_unpack(w, c);
    const __half2 s2 = __half2half2(scale);
    const float s = __half2float(scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 x = *reinterpret_cast<const __half2*>(&c[i]);
        if (F16) {
            const __half2 y = __hmul2(x, s2);
            r[i] = *reinterpret_cast<const uint32_t*>(&y);
        } else {
            const float2 f = __half22float2(x);
            r[i] = round_pair<F16>(f.x * s, f.y * s);         // (the products are exact: 2 and 11 significant bits)
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

template <int D, bool F16>
__global__ void __launch_bounds__(kExpandThreads) decode_attn_expand_kernel(const ExpandParams p)
{
    constexpr int L = D / 8;                                  // lanes of a row
    constexpr int STEP = 32 / L;                              // rows at a time
    constexpr int N = 16 / STEP;
    constexpr int TILE = packed_tile_bytes(D);
    extern __shared__ __align__(128) uint8_t smem[];
    pdl_launch_dependents();
    pdl_wait_primary();
    const int b = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int len = p.seq_lens[b];
    const int64_t fits = (int64_t)(p.src_width < p.dst_width ? p.src_width : p.dst_width) << p.page_shift;
    if (len < 0 || len > fits) {
        if (blockIdx.x == 0 && threadIdx.x == 0 && p.status != nullptr) record_status(p.status, DA_ERR_STALE_PLAN);
        return;
    }
    const int tile0 = blockIdx.x * kExpandTiles, here = min(kExpandTiles, ((len + 15) >> 4) - tile0);
    if (here <= 0) return;
    // lane i: the pages of the block's tile i
    int src_id = 0, dst_id = -1;
    if (lane < here) {
        const int at = (tile0 + lane) >> (p.page_shift - 4);
        src_id = p.block_table[(int64_t)b * p.src_width + at];
        dst_id = p.dst_table[(int64_t)b * p.dst_width + at];
        if ((unsigned)src_id >= (unsigned)p.src_pages || (unsigned)dst_id >= (unsigned)p.num_pages) {
            if (p.status != nullptr) record_status(p.status, DA_ERR_BAD_PAGE);
            src_id = 0;                                       // (nothing outside the pool is read)
            dst_id = -1;
        }
    }
    const uint32_t ring = smem_u32(smem) + warp * (kExpandRing * TILE);
    // this warp's tasks: head h of tile i, every eighth one
    int i_tile = 0, i_head = warp;
    uint32_t i_at = ring;
    auto settle = [&](int& tile, int& head) {
        while (head >= p.num_kv_heads) {
            head -= p.num_kv_heads;
            ++tile;
        }
    };
    settle(i_tile, i_head);
    auto ask = [&]() {
        if (i_tile < here) {
            const int page = __shfl_sync(0xffffffffu, src_id, i_tile);
            const int in_page = (tile0 + i_tile) & ((1 << (p.page_shift - 4)) - 1);
            const char* const src = p.pool + page * p.src_stride_page + i_head * p.src_stride_head + in_page * TILE + lane * 16;
#pragma unroll
            for (int c = 0; c <= TILE / 512; ++c)
                if (c < TILE / 512 || lane * 16 < TILE % 512)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(i_at + lane * 16 + c * 512), "l"(src + c * 512) : "memory");
            i_head += kExpandThreads / 32;
            settle(i_tile, i_head);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");  // (a group for every call: the waits below count them)
        i_at = i_at + TILE == ring + kExpandRing * TILE ? ring : i_at + TILE;
    };
    for (int s = 0; s < kExpandRing - 1; ++s) ask();

    const int l = lane % L, r0 = lane / L;
    const int64_t k_step = STEP * p.k_stride_token, v_step = STEP * p.v_stride_token;
    int tile = 0, head = warp;
    settle(tile, head);
    uint32_t at = ring;
    while (tile < here) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kExpandRing - 2) : "memory");
        __syncwarp();                                         // every lane's copies are there, and the tile before is read
        ask();
        const int page = __shfl_sync(0xffffffffu, dst_id, tile);
        if (page >= 0) {
            const int in_page = (tile0 + tile) & ((1 << (p.page_shift - 4)) - 1);
            const int rows = min(16, len - (tile0 + tile) * 16);
            const uint8_t* const from = smem + (at - smem_u32(smem));
            const uint32_t* const kc = reinterpret_cast<const uint32_t*>(from) + packed_k_word(D, r0, l);
            const uint32_t* const vc = reinterpret_cast<const uint32_t*>(from + packed_v_codes(D));
            const __half* const ks = reinterpret_cast<const __half*>(from + packed_k_scales(D)) + packed_k_scale(D, r0, l >> 2);
            const __half* const vs = reinterpret_cast<const __half*>(from + packed_v_scales(D));
            uint16_t* kt = p.k + page * p.k_stride_page + (in_page * 16 + r0) * p.k_stride_token + head * p.k_stride_head + 8 * l;
            uint16_t* vt = p.v + page * p.v_stride_page + (in_page * 16 + r0) * p.v_stride_token + head * p.v_stride_head + 8 * l;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (j * STEP + r0 < rows) {
                    *reinterpret_cast<uint4*>(kt) = expand_word<F16>(kc[packed_k_word(D, j * STEP, 0)], ks[packed_k_scale(D, j * STEP, 0)]);
                    *reinterpret_cast<uint4*>(vt) =
                        expand_word<F16>(vc[packed_v_word(D, j * STEP + r0, l)], vs[packed_v_scale(j * STEP + r0, l >> 2)]);
                }
                kt += k_step;
                vt += v_step;
            }
        }
        at = at + TILE == ring + kExpandRing * TILE ? ring : at + TILE;
        head += kExpandThreads / 32;
        settle(tile, head);
    }
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

}  // namespace

extern "C" int64_t decode_attn_packed_head_bytes(int32_t head_dim, int32_t page_size)
{
    if (head_dim != 64 && head_dim != 128) return 0;
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return 0;
    return (int64_t)(page_size / 16) * packed_tile_bytes(head_dim);
}

extern "C" int decode_attn_expand_kv(const decode_attn_shape_t* shape, const decode_attn_shape_t* from, const void* pool,
                                     const int32_t* block_table, const int32_t* seq_lens, const int32_t* dst_block_table,
                                     void* k_cache, void* v_cache, int32_t* status_or_null, cudaStream_t stream)
{
    if (!shape || !from) return DA_ERR_INVALID_ARG;
    int rc = validate_shape(*shape);
    if (rc != DA_OK) return rc;
    decode_attn_shape_t f;
    rc = packed_shape(*from, &f);
    if (rc == DA_OK) rc = validate_shape(f);
    if (rc != DA_OK) return rc;
    const decode_attn_shape_t& s = *shape;
    if (f.batch != s.batch || f.num_kv_heads != s.num_kv_heads || f.head_dim != s.head_dim || f.page_size != s.page_size)
        return DA_ERR_INVALID_ARG;
    const int width = s.max_pages_per_seq < f.max_pages_per_seq ? s.max_pages_per_seq : f.max_pages_per_seq;
    if (s.batch == 0 || width == 0) return DA_OK;
    if (!pool || !block_table || !seq_lens || !dst_block_table || !k_cache || !v_cache) return DA_ERR_INVALID_ARG;
    if (!aligned(pool, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(block_table, 4) || !aligned(seq_lens, 4) ||
        !aligned(dst_block_table, 4) || !aligned(status_or_null, 4))
        return DA_ERR_INVALID_ARG;
    if (s.batch > 65535) return DA_ERR_UNSUPPORTED;
    ExpandParams p;
    std::memset(&p, 0, sizeof p);
    p.pool = static_cast<const char*>(pool);
    p.block_table = block_table;
    p.seq_lens = seq_lens;
    p.dst_table = dst_block_table;
    p.k = static_cast<uint16_t*>(k_cache);
    p.v = static_cast<uint16_t*>(v_cache);
    p.status = status_or_null;
    p.src_stride_page = f.k_stride_page;
    p.src_stride_head = f.k_stride_head;
    p.src_pages = f.num_pages;
    p.num_pages = s.num_pages;
    p.k_stride_page = s.k_stride_page; p.k_stride_token = s.k_stride_token; p.k_stride_head = s.k_stride_head;
    p.v_stride_page = s.v_stride_page; p.v_stride_token = s.v_stride_token; p.v_stride_head = s.v_stride_head;
    p.num_kv_heads = s.num_kv_heads;
    p.src_width = f.max_pages_per_seq;
    p.dst_width = s.max_pages_per_seq;
    while ((1 << p.page_shift) < s.page_size) ++p.page_shift;
    const int64_t tiles = (int64_t)width * (s.page_size / 16);
    const int64_t blocks = (tiles + kExpandTiles - 1) / kExpandTiles;
    if (blocks > 0x7fffffffLL || tiles * 16 > INT32_MAX) return DA_ERR_UNSUPPORTED;
    const bool f16 = s.kv_dtype == DA_DTYPE_FP16;
    auto fn = s.head_dim == 128 ? (f16 ? decode_attn_expand_kernel<128, true> : decode_attn_expand_kernel<128, false>)
                                : (f16 ? decode_attn_expand_kernel<64, true> : decode_attn_expand_kernel<64, false>);
    const int smem = kExpandThreads / 32 * kExpandRing * packed_tile_bytes(s.head_dim);
    rc = opt_in_shared_memory((const void*)fn, smem);
    if (rc != DA_OK) return rc;
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3((unsigned)blocks, (unsigned)s.batch, 1);
    cfg.blockDim = dim3(kExpandThreads, 1, 1);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, fn, p) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}
