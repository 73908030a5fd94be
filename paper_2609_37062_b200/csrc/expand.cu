// Pages of a cache in 4 bits to 16-bit pages (decode_attn_expand_kv).
//
// Bound by memory: 4.5 bits read and 16 written a value.  A task is a tile of one KV head (2,304 contiguous bytes at head_dim
// 128).  A warp copies its tasks to a ring of its own (cp.async, one task ahead), and 16 lanes (8 at head_dim 64) write a row of
// K or V whole, 16 bytes a lane, from one word of codes each.
//
// The lengths are on the device, so the grid cannot follow them: it is bounded by the machine, every block makes the
// sums of the sequences' tiles, and the grid's warps go through the tasks together.  96,000 tokens of 8 heads of 128, 502 MB: 85 us,
// 5.9 TB/s (a plain copy's rate would be 77), with 24 blocks launched for every SM.  Blocks over the width of the tables, eight tiles
// each, took 90 on lengths of 8,000 to 30,000, since their SMs were not equally full, and had thousands of empty blocks where
// tables are wide; 3, 6, 12, 20 and 48 blocks for every SM took 96, 89, 88, 88 and 84.6: warps that start together also read and write
// together.
#include <cstring>

#include "common.cuh"
#include "opt_in.h"
#include "packed.cuh"
#include "planner.h"

using namespace da;

namespace {

constexpr int kExpandThreads = 256;
constexpr int kExpandRing = 2;         // tasks in a warp's ring
constexpr int kExpandGrid = 148 * 24;  // blocks at most, for a B200's 148 SMs (the results do not depend on it)
// Blocks that registers leave room for on an SM, 40 a thread.  At head_dim 64 six are resident, at 128 five: 41,024 bytes of shared
// memory each, the system's 1 KB included.  (With the 48 registers of five: the same, 3.7 us instead of 3.6 for 500 tokens.)
constexpr int kExpandBlocks = 6;
constexpr int kExpandBatch = kExpandThreads;         // sequences that the sums are made for at a time

struct ExpandParams {
    const char* pool;
    const int32_t *block_table, *seq_lens, *dst_table;
    uint16_t *k, *v;
    int32_t* status;
    int64_t src_stride_page, src_stride_head, src_pages, num_pages;
    int64_t k_stride_page, k_stride_token, k_stride_head;
    int64_t v_stride_page, v_stride_token, v_stride_head;
    int32_t batch, num_kv_heads, src_width, dst_width, page_shift;
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
__global__ void __launch_bounds__(kExpandThreads, kExpandBlocks) decode_attn_expand_kernel(const ExpandParams p)
{
    constexpr int L = D / 8;                                  // lanes of a row
    constexpr int STEP = 32 / L;                              // rows at a time
    constexpr int N = 16 / STEP;
    constexpr int TILE = packed_tile_bytes(D);
    constexpr int W = kExpandThreads / 32;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t sm_upto[kExpandBatch];                 // tiles of the sequences up to and with this one
    __shared__ int32_t sm_len[kExpandBatch];
    __shared__ int64_t sm_warp[W];
    pdl_launch_dependents();
    pdl_wait_primary();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t fits = (int64_t)min(p.src_width, p.dst_width) << p.page_shift;
    const int tile_mask = (1 << (p.page_shift - 4)) - 1;
    const uint32_t ring = smem_u32(smem) + warp * (kExpandRing * TILE);
    const int l = lane % L, r0 = lane / L;
    const int64_t k_step = STEP * p.k_stride_token, v_step = STEP * p.v_stride_token;
    const int64_t stride = (int64_t)gridDim.x * W;            // warps of the grid

    for (int b0 = 0; b0 < p.batch; b0 += kExpandBatch) {
        const int here = min(kExpandBatch, p.batch - b0);
        // ---- sums of the tiles
        if (b0 > 0) __syncthreads();                          // the sums before are read
        int len = (int)threadIdx.x < here ? p.seq_lens[b0 + threadIdx.x] : 0;
        if (len < 0 || len > fits) {
            if (blockIdx.x == 0 && p.status != nullptr) record_status(p.status, DA_ERR_STALE_PLAN);
            len = 0;
        }
        sm_len[threadIdx.x] = len;
        int64_t upto = ((int64_t)len + 15) >> 4;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t x = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += x;
        }
        if (lane == 31) sm_warp[warp] = upto;
        __syncthreads();
        for (int w = 0; w < warp; ++w) upto += sm_warp[w];
        sm_upto[threadIdx.x] = upto;
        __syncthreads();
        const int64_t tasks = sm_upto[here - 1] * p.num_kv_heads;

        for (int64_t first = (int64_t)blockIdx.x * W + warp; first < tasks; first += 32 * stride) {
            // ---- lane i: where this warp's task i lies
            const int64_t task = first + lane * stride;
            const int n = __popc(__ballot_sync(0xffffffffu, task < tasks));
            int64_t src_at = 0;
            int dst_id = -1, place = 0;                       // place: tile of the page * 16 + rows - 1
            int head = 0;
            if (task < tasks) {
                const int64_t flat = task / p.num_kv_heads;
                head = (int)(task - flat * p.num_kv_heads);
                int lo = 0, hi = here - 1;                    // the first sequence whose sum is larger
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (sm_upto[mid] > flat) hi = mid;
                    else lo = mid + 1;
                }
                const int tile = (int)(flat - (lo > 0 ? sm_upto[lo - 1] : 0)), page = tile >> (p.page_shift - 4);
                int src_id = p.block_table[(int64_t)(b0 + lo) * p.src_width + page];
                dst_id = p.dst_table[(int64_t)(b0 + lo) * p.dst_width + page];
                if ((unsigned)src_id >= (unsigned)p.src_pages || (unsigned)dst_id >= (unsigned)p.num_pages) {
                    if (p.status != nullptr) record_status(p.status, DA_ERR_BAD_PAGE);
                    src_id = 0;                               // (nothing outside the pool is read)
                    dst_id = -1;
                }
                place = (tile & tile_mask) * 16 + min(16, sm_len[lo] - tile * 16) - 1;
                src_at = src_id * p.src_stride_page + head * p.src_stride_head + (tile & tile_mask) * TILE;
            }
            __syncwarp();                                     // the tasks before are read
            int asked = 0;
            uint32_t ask_at = ring, at = ring;
            auto ask = [&]() {
                if (asked < n) {
                    const char* const src = p.pool + __shfl_sync(0xffffffffu, src_at, asked) + lane * 16;
#pragma unroll
                    for (int c = 0; c <= TILE / 512; ++c)
                        if (c < TILE / 512 || lane * 16 < TILE % 512)
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ask_at + lane * 16 + c * 512), "l"(src + c * 512) : "memory");
                    ++asked;
                }
                asm volatile("cp.async.commit_group;" ::: "memory");          // (a group for every call: the waits below count them)
                ask_at = ask_at + TILE == ring + kExpandRing * TILE ? ring : ask_at + TILE;
            };
            for (int s = 0; s < kExpandRing - 1; ++s) ask();
            for (int i = 0; i < n; ++i) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kExpandRing - 2) : "memory");
                __syncwarp();                                 // every lane's copies are there, and the task before is read
                ask();
                const int page = __shfl_sync(0xffffffffu, dst_id, i), where = __shfl_sync(0xffffffffu, place, i);
                const int h = __shfl_sync(0xffffffffu, head, i);
                if (page >= 0) {
                    const int rows = (where & 15) + 1, row = (where & ~15) + r0;
                    const uint8_t* const from = smem + (at - smem_u32(smem));
                    const uint32_t* const kc = reinterpret_cast<const uint32_t*>(from) + packed_k_word(D, r0, l);
                    const uint32_t* const vc = reinterpret_cast<const uint32_t*>(from + packed_v_codes(D));
                    const __half* const ks = reinterpret_cast<const __half*>(from + packed_k_scales(D)) + packed_k_scale(D, r0, l >> 2);
                    const __half* const vs = reinterpret_cast<const __half*>(from + packed_v_scales(D));
                    uint16_t* kt = p.k + page * p.k_stride_page + row * p.k_stride_token + h * p.k_stride_head + 8 * l;
                    uint16_t* vt = p.v + page * p.v_stride_page + row * p.v_stride_token + h * p.v_stride_head + 8 * l;
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        if (j * STEP + r0 < rows) {
                            *reinterpret_cast<uint4*>(kt) =
                                expand_word<F16>(kc[packed_k_word(D, j * STEP, 0)], ks[packed_k_scale(D, j * STEP, 0)]);
                            *reinterpret_cast<uint4*>(vt) =
                                expand_word<F16>(vc[packed_v_word(D, j * STEP + r0, l)], vs[packed_v_scale(j * STEP + r0, l >> 2)]);
                        }
                        kt += k_step;
                        vt += v_step;
                    }
                }
                at = at + TILE == ring + kExpandRing * TILE ? ring : at + TILE;
            }
        }
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
    p.batch = s.batch;
    p.num_kv_heads = s.num_kv_heads;
    p.src_width = f.max_pages_per_seq;
    p.dst_width = s.max_pages_per_seq;
    while ((1 << p.page_shift) < s.page_size) ++p.page_shift;
    constexpr int64_t kWarps = kExpandThreads / 32;
    const int64_t tiles = (int64_t)width * (s.page_size / 16) * s.batch;
    const int64_t most = tiles > INT32_MAX ? INT32_MAX : tiles * s.num_kv_heads, needed = (most + kWarps - 1) / kWarps;
    const int64_t blocks = needed < kExpandGrid ? needed : kExpandGrid;    // (no more than the tables have room for)
    const bool f16 = s.kv_dtype == DA_DTYPE_FP16;
    auto fn = s.head_dim == 128 ? (f16 ? decode_attn_expand_kernel<128, true> : decode_attn_expand_kernel<128, false>)
                                : (f16 ? decode_attn_expand_kernel<64, true> : decode_attn_expand_kernel<64, false>);
    const int smem = kExpandThreads / 32 * kExpandRing * packed_tile_bytes(s.head_dim);
    rc = opt_in_shared_memory((const void*)fn, smem);
    if (rc != DA_OK) return rc;
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3((unsigned)blocks, 1, 1);
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
