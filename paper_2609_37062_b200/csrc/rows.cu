// Host side of decode_attn_prepare_rows.
#include <cmath>
#include <cstring>

#include "opt_in.h"
#include "planner.h"
#include "rows.cuh"

using namespace da;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// A row-wise operand: given, 16-byte aligned, its rows of `heads` heads apart.
bool rows_ok(const void* p, int64_t stride, int64_t heads, int64_t D)
{
    return aligned(p, 16) && stride >= heads * D && stride % 8 == 0;
}

typedef void (*rows_kernel_t)(const RowsParams);

template <int D, bool F16, bool PACKED>
rows_kernel_t for_turn(bool halves, bool all)
{
    if (halves) return all ? decode_attn_rows_kernel<D, F16, PACKED, true, true> : decode_attn_rows_kernel<D, F16, PACKED, true, false>;
    return all ? decode_attn_rows_kernel<D, F16, PACKED, false, true> : decode_attn_rows_kernel<D, F16, PACKED, false, false>;
}

// halves: pairs are (i, i + rotary_dim / 2); all: every dim turns.
template <int D>
rows_kernel_t kernel_for(bool f16, bool packed, bool halves, bool all)
{
    if (packed) return f16 ? for_turn<D, true, true>(halves, all) : for_turn<D, false, true>(halves, all);
    return f16 ? for_turn<D, true, false>(halves, all) : for_turn<D, false, false>(halves, all);
}

// Shares of a row's tasks: as many as 148 SMs have resident warps for, so that every warp has one; a share costs its tasks and
// about one and a half to begin.  Where rows are more than half of the warps, another number may fill the last round of warps
// better.  (32 + 8 + 8 heads of 128, us: 256 rows 5.3 with shares for a little more than the resident warps, 4.0 so; 600 rows 7.2
// and 5.2; 1,777 rows 12.8 and 11.2; 1,200 rows 10.1 whole and 9.1 in three shares, 3,000 rows 19.5 whole and 18.0 in two.)
// (Of a B200's 148 SMs; on another number the results are the same.)
constexpr int kRowsWarps = 148 * kRowsBlocks * (kRowsThreads / 32);

int split_of(int rows, int tasks)
{
    auto cost = [&](int split) {
        const int64_t rounds = ((int64_t)rows * split + kRowsWarps - 1) / kRowsWarps;
        return rounds * (2 * ((tasks + split - 1) / split) + 3);
    };
    int best = rows < kRowsWarps ? kRowsWarps / rows : 1;
    if (best > tasks) best = tasks;
    if (best > 2) return best;
    int64_t least = cost(best);
    for (int split = 1; split <= tasks && split <= 4; ++split) {
        const int64_t c = cost(split);
        if (c * 100 < least * 95) {
            best = split;
            least = c;
        }
    }
    return best;
}

}  // namespace

extern "C" int decode_attn_prepare_rows(const decode_attn_shape_t* shape, const decode_attn_rows_args_t* a, cudaStream_t stream)
{
    if (!shape || !a) return DA_ERR_INVALID_ARG;
    if (a->struct_size != sizeof(decode_attn_rows_args_t) || a->flags != 0) return DA_ERR_INVALID_ARG;
    if (a->cache_bits != 0 && a->cache_bits != 16 && a->cache_bits != 4) return DA_ERR_INVALID_ARG;
    const bool packed = a->cache_bits == 4;
    decode_attn_shape_t s;
    int rc = packed ? packed_shape(*shape, &s) : (s = *shape, DA_OK);
    if (rc != DA_OK) return rc;
    s.batch = s.max_pages_per_seq = 0;
    rc = validate_shape(s);
    if (rc != DA_OK) return rc;
    const int D = s.head_dim;
    if (a->rows < 0 || !(a->eps >= 0.f) || std::isinf(a->eps) || (a->interleaved != 0 && a->interleaved != 1)) return DA_ERR_INVALID_ARG;
    if (a->cos_sin != nullptr) {
        if (a->rotary_dim < 8 || a->rotary_dim > D || a->rotary_dim % 8 != 0 || a->max_positions < 1 || !aligned(a->cos_sin, 16))
            return DA_ERR_INVALID_ARG;
    } else if (a->rotary_dim != 0) {
        return DA_ERR_INVALID_ARG;
    }
    if (a->rows == 0) return DA_OK;
    const bool cache = a->k_cache != nullptr;
    if (!packed && cache != (a->v_cache != nullptr)) return DA_ERR_INVALID_ARG;
    if (packed && (!cache || a->v_cache != nullptr)) return DA_ERR_INVALID_ARG;
    // what is read has somewhere to go, and what is written comes from somewhere
    if ((a->q != nullptr) != (a->q_out != nullptr)) return DA_ERR_INVALID_ARG;
    if ((a->k != nullptr) != (a->k_out != nullptr || cache) || (a->v != nullptr) != cache) return DA_ERR_INVALID_ARG;
    if (!a->q && !a->k) return DA_ERR_INVALID_ARG;
    if ((a->cos_sin && !a->positions) || (cache && !a->slots)) return DA_ERR_INVALID_ARG;
    if ((a->q && (!rows_ok(a->q, a->q_stride, s.num_q_heads, D) || !rows_ok(a->q_out, a->q_out_stride, s.num_q_heads, D))) ||
        (a->k && !rows_ok(a->k, a->k_stride, s.num_kv_heads, D)) || (a->v && !rows_ok(a->v, a->v_stride, s.num_kv_heads, D)) ||
        (a->k_out && !rows_ok(a->k_out, a->k_out_stride, s.num_kv_heads, D)))
        return DA_ERR_INVALID_ARG;
    if ((a->q_weight && !a->q) || (a->k_weight && !a->k)) return DA_ERR_INVALID_ARG;
    if (!aligned(a->q_weight, 16) || !aligned(a->k_weight, 16) || (a->q_weight && a->q_weight_stride != 0 && a->q_weight_stride != D) ||
        (a->k_weight && a->k_weight_stride != 0 && a->k_weight_stride != D))
        return DA_ERR_INVALID_ARG;
    if (!aligned(a->positions, 4) || !aligned(a->slots, 8) || !aligned(a->status, 4) || !aligned(a->k_cache, 16) || !aligned(a->v_cache, 16))
        return DA_ERR_INVALID_ARG;

    RowsParams rp;
    std::memset(&rp, 0, sizeof rp);
    rp.q = static_cast<const uint16_t*>(a->q);
    rp.k = static_cast<const uint16_t*>(a->k);
    rp.v = static_cast<const uint16_t*>(a->v);
    rp.q_stride = a->q_stride; rp.k_stride = a->k_stride; rp.v_stride = a->v_stride;
    rp.q_weight = static_cast<const uint16_t*>(a->q_weight);
    rp.k_weight = static_cast<const uint16_t*>(a->k_weight);
    rp.q_weight_stride = a->q_weight_stride; rp.k_weight_stride = a->k_weight_stride;
    rp.cos_sin = a->cos_sin;
    rp.positions = a->positions;
    rp.slots = a->slots;
    rp.q_out = static_cast<uint16_t*>(a->q_out);
    rp.k_out = static_cast<uint16_t*>(a->k_out);
    rp.q_out_stride = a->q_out_stride; rp.k_out_stride = a->k_out_stride;
    rp.k_cache = a->k_cache;
    rp.v_cache = a->v_cache;
    rp.status = a->status;
    rp.num_pages = s.num_pages;
    rp.k_stride_page = s.k_stride_page; rp.k_stride_token = s.k_stride_token; rp.k_stride_head = s.k_stride_head;
    rp.v_stride_page = s.v_stride_page; rp.v_stride_token = s.v_stride_token; rp.v_stride_head = s.v_stride_head;
    rp.rows = a->rows;
    rp.n_q = a->q ? s.num_q_heads : 0;
    rp.n_k = a->k ? s.num_kv_heads : 0;
    rp.n_v = a->v ? s.num_kv_heads : 0;
    rp.rotary_dim = a->rotary_dim;
    rp.max_positions = a->max_positions;
    while ((1 << rp.page_shift) < s.page_size) ++rp.page_shift;
    rp.eps = a->eps;

    const bool f16 = s.kv_dtype == DA_DTYPE_FP16, halves = a->cos_sin != nullptr && !a->interleaved, all = a->rotary_dim == D;
    rows_kernel_t fn = D == 128 ? kernel_for<128>(f16, packed, halves, all) : kernel_for<64>(f16, packed, halves, all);
    const int per_task = 512 / D, tasks = (rp.n_q + per_task - 1) / per_task + (rp.n_k + per_task - 1) / per_task + (rp.n_v + per_task - 1) / per_task;
    rp.split = split_of(a->rows, tasks);
    // (numbers of work items stay below 2^31, two rounds of all warps included)
    if ((int64_t)a->rows * rp.split > INT32_MAX - 4 * kRowsWarps) return DA_ERR_UNSUPPORTED;
    const int64_t warps = (int64_t)a->rows * rp.split, needed = (warps + kRowsThreads / 32 - 1) / (kRowsThreads / 32);
    const int64_t blocks = needed < 148 * kRowsBlocks ? needed : 148 * kRowsBlocks;
    rc = opt_in_shared_memory((const void*)fn, kRowsSmem);
    if (rc != DA_OK) return rc;
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3((unsigned)blocks, 1, 1);
    cfg.blockDim = dim3(kRowsThreads, 1, 1);
    cfg.dynamicSmemBytes = kRowsSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, fn, rp) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}
