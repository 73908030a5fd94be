// Step tables: block tables, slots and positions of a step from what every sequence gains (decode_attn_step_tables).
//
// Lengths, the list of free pages and the tables live on the device, so nothing of it waits for the host.  The order is
// fixed by prefix sums over the sequences: pages given back, pages lacked, new rows.  One block makes them (a batch is
// some hundred sequences: a few words a thread) and everything that is counted in sequences; what is counted in tokens
// (slots, positions, block-table entries of fresh pages) follows from the sums for every row by itself: row -> sequence
// by a binary search in row_starts, position -> page by the table or, for a fresh page, by its place in the list of free
// pages.  The row whose token is a fresh page's first writes the table entry.
#include <cstring>

#include "common.cuh"
#include "planner.h"

using namespace da;

namespace {

struct TablesParams {
    const int32_t* seq_lens;
    const int32_t* gains;
    int32_t* seq_lens_out;
    int32_t* block_table;
    int32_t* free_pages;
    const int32_t* free_count;
    int32_t* free_count_out;
    int32_t* row_starts;
    int32_t* page_starts;
    int64_t* slots;
    int32_t* positions;
    int32_t* row_seq;
    int32_t* status;
    int64_t num_pages, most_tokens;   // most_tokens: what a row of the block table has pages for
    int32_t batch, max_pages_per_seq, max_rows, free_capacity, page_shift;
    int32_t vec;                      // slots, positions and row_seq may be written 16 bytes at a time
};

constexpr int kScanThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int kRowsPerThread = 4;

// Exclusive prefix sums of two values over the block's threads; the totals in `all`.
__device__ __forceinline__ void block_scan2(int64_t& x, int64_t& y, int64_t (&all)[2], int64_t (*sm)[2])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int64_t a = x, b = y;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, a, off), v = __shfl_up_sync(0xffffffffu, b, off);
        if (lane >= off) {
            a += u;
            b += v;
        }
    }
    __syncthreads();                                          // the scratch of the scan before is free
    if (lane == 31) {
        sm[warp][0] = a;
        sm[warp][1] = b;
    }
    __syncthreads();
    int64_t u = lane < warps ? sm[lane][0] : 0, v = lane < warps ? sm[lane][1] : 0;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t s = __shfl_up_sync(0xffffffffu, u, off), t = __shfl_up_sync(0xffffffffu, v, off);
        if (lane >= off) {
            u += s;
            v += t;
        }
    }
    all[0] = __shfl_sync(0xffffffffu, u, 31);
    all[1] = __shfl_sync(0xffffffffu, v, 31);
    const int64_t u0 = __shfl_sync(0xffffffffu, u, warp ? warp - 1 : 0), v0 = __shfl_sync(0xffffffffu, v, warp ? warp - 1 : 0);
    x = a - x + (warp ? u0 : 0);
    y = b - y + (warp ? v0 : 0);
}

__device__ __forceinline__ void report(const TablesParams& p, int code)
{
    if (p.status != nullptr) record_status(p.status, code);
}

// What sequence b asks for.  back / lack: pages given back / lacked; rows: tokens gained.  old < 0: it is left alone.
struct Ask {
    int64_t old, fresh, back, lack, rows;
};

__device__ __forceinline__ Ask ask_of(const TablesParams& p, int b, bool loud)
{
    Ask a = {-1, -1, 0, 0, 0};
    if (b >= p.batch) return a;
    const int64_t old = p.seq_lens[b], gain = p.gains[b];
    const int64_t fresh = old + gain > 0 ? old + gain : 0;
    if (old < 0 || old > p.most_tokens || fresh > p.most_tokens) {
        if (loud) report(p, DA_ERR_STALE_PLAN);
        return a;
    }
    const int64_t round = ((int64_t)1 << p.page_shift) - 1;
    const int64_t held = (old + round) >> p.page_shift, holds = (fresh + round) >> p.page_shift;
    a.old = old;
    a.fresh = fresh;
    a.back = held > holds ? held - holds : 0;
    a.lack = holds > held ? holds - held : 0;
    a.rows = gain > 0 ? gain : 0;
    return a;
}

// Rows first .. first + 3 of the step.
__device__ __forceinline__ void fill_rows(const TablesParams& p, int64_t first, int64_t avail)
{
    const int total = p.row_starts[p.batch];
    const int mask = (1 << p.page_shift) - 1;
    int64_t slot[kRowsPerThread];
    int pos[kRowsPerThread], seq[kRowsPerThread];
    int b = -1, start = 0, end = 0, old = 0, page_at = 0, held = 0, last_page = -1, id = 0;
#pragma unroll
    for (int i = 0; i < kRowsPerThread; ++i) {
        const int64_t row = first + i;
        slot[i] = -1;
        pos[i] = seq[i] = -1;
        if (row >= total) continue;
        if (b < 0) {
            int lo = 0, hi = p.batch;                         // row_starts[lo] <= row < row_starts[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.row_starts[mid] <= row) lo = mid;
                else hi = mid;
            }
            b = lo;
        } else if (row >= end) {
            do ++b;                                           // (sequences without rows in between)
            while (p.row_starts[b + 1] <= row);
        }
        if (row >= end) {
            start = p.row_starts[b];
            end = p.row_starts[b + 1];
            old = p.seq_lens_out[b] - (end - start);
            held = (old + mask) >> p.page_shift;
            page_at = p.page_starts[b];
            last_page = -1;
        }
        const int at = old + (int)(row - start);
        const int page = at >> p.page_shift;
        int32_t* const entry = p.block_table + (int64_t)b * p.max_pages_per_seq + page;
        if (page != last_page) {
            id = page < held ? *entry : p.free_pages[avail - 1 - page_at - (page - held)];
            last_page = page;
            if ((unsigned)id >= (unsigned)p.num_pages) report(p, DA_ERR_BAD_PAGE);
        }
        if (page >= held && (at & mask) == 0) *entry = id;
        if ((unsigned)id < (unsigned)p.num_pages) slot[i] = ((int64_t)id << p.page_shift) + (at & mask);
        pos[i] = at;
        seq[i] = b;
    }
    if (p.vec && first + kRowsPerThread <= p.max_rows) {
        reinterpret_cast<longlong2*>(p.slots + first)[0] = make_longlong2(slot[0], slot[1]);
        reinterpret_cast<longlong2*>(p.slots + first)[1] = make_longlong2(slot[2], slot[3]);
        *reinterpret_cast<int4*>(p.positions + first) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        if (p.row_seq != nullptr) *reinterpret_cast<int4*>(p.row_seq + first) = make_int4(seq[0], seq[1], seq[2], seq[3]);
        return;
    }
#pragma unroll
    for (int i = 0; i < kRowsPerThread; ++i) {
        if (first + i >= p.max_rows) break;
        p.slots[first + i] = slot[i];
        p.positions[first + i] = pos[i];
        if (p.row_seq != nullptr) p.row_seq[first + i] = seq[i];
    }
}

// The sums and all that is counted in sequences; with FILL the rows too.
template <bool FILL>
__global__ void __launch_bounds__(kScanThreads) decode_attn_tables_kernel(const TablesParams p)
{
    __shared__ int64_t sm[kScanThreads / 32][2];
    pdl_launch_dependents();
    pdl_wait_primary();
    const int tid = threadIdx.x, lane = tid & 31;
    const int64_t count = *p.free_count;
    const bool sane = count >= 0 && count <= p.free_capacity;
    if (!sane && tid == 0) report(p, DA_ERR_STALE_PLAN);
    // 1. pages given back: their places in the list, and how many fit
    int64_t pushed = 0, all[2];
    for (int b0 = 0; b0 < p.batch; b0 += kScanThreads) {
        const Ask a = sane ? ask_of(p, b0 + tid, false) : Ask{-1, -1, 0, 0, 0};
        int64_t at = a.back, none = 0;
        block_scan2(at, none, all, sm);
        at += pushed;
        const bool fits = count + at + a.back <= p.free_capacity;
        if (a.back > 0 && !fits) report(p, DA_ERR_NO_PAGES);
        // a few pages by their own thread, many by the warp
        const int64_t pages = fits ? a.back : 0;
        const int64_t from = (a.fresh + ((int64_t)1 << p.page_shift) - 1) >> p.page_shift;
        const int32_t* const row = p.block_table + (int64_t)(b0 + tid) * p.max_pages_per_seq + from;
        if (pages <= 4)
            for (int i = 0; i < (int)pages; ++i) p.free_pages[count + at + i] = row[i];
        for (unsigned many = __ballot_sync(0xffffffffu, pages > 4); many != 0; many &= many - 1) {
            const int l = __ffs(many) - 1;
            const int64_t n = __shfl_sync(0xffffffffu, pages, l), to = __shfl_sync(0xffffffffu, count + at, l);
            const int32_t* const src = reinterpret_cast<const int32_t*>(__shfl_sync(0xffffffffu, (unsigned long long)row, l));
            for (int64_t i = lane; i < n; i += 32) p.free_pages[to + i] = src[i];
        }
        // (what does not fit is behind what does: the sums only grow)
        int64_t ok = pages, none2 = 0;
        block_scan2(ok, none2, all, sm);
        pushed += all[0];
        if (__syncthreads_or(a.back > 0 && !fits)) {
            // one that does not fit: of those behind it none fits either
            for (int b = b0 + kScanThreads + tid; b < p.batch; b += kScanThreads)
                if (ask_of(p, b, false).back > 0) report(p, DA_ERR_NO_PAGES);
            break;
        }
    }
    const int64_t avail = count + pushed;
    // 2. pages and rows of those that grow; lengths
    int64_t lacked = 0, asked = 0, taken = 0, rows = 0, gave = 0;
    for (int b0 = 0; b0 < p.batch; b0 += kScanThreads) {
        const int b = b0 + tid;
        const Ask a = sane ? ask_of(p, b, true) : Ask{-1, -1, 0, 0, 0};
        int64_t lack = a.lack, row = a.rows;
        block_scan2(lack, row, all, sm);
        const bool pages_ok = a.lack == 0 || lacked + lack + a.lack <= avail;
        const bool rows_ok = a.rows == 0 || asked + row + a.rows <= p.max_rows;
        lacked += all[0];
        asked += all[1];
        if (!pages_ok) report(p, DA_ERR_NO_PAGES);
        if (!rows_ok) report(p, DA_ERR_WORKSPACE_TOO_SMALL);
        // giving back is granted by the same sums as above
        int64_t back = a.back, got_rows = pages_ok && rows_ok ? a.rows : 0;
        const int64_t own_rows = got_rows;
        block_scan2(back, got_rows, all, sm);
        const bool back_ok = a.back == 0 || count + gave + back + a.back <= p.free_capacity;
        gave += all[0];
        const int64_t row_at = rows + got_rows;
        rows += all[1];
        int64_t got = pages_ok && rows_ok ? a.lack : 0, none = 0;
        block_scan2(got, none, all, sm);
        const int64_t page_at = taken + got;
        taken += all[0];
        if (b < p.batch) {
            p.row_starts[b] = (int32_t)row_at;
            p.page_starts[b] = (int32_t)page_at;
            // (a length that is left alone is copied: the two arrays may be one)
            const bool granted = a.old >= 0 && (a.rows > 0 ? own_rows > 0 : back_ok);
            const int32_t len = granted ? (int32_t)a.fresh : p.seq_lens[b];
            p.seq_lens_out[b] = len;
        }
    }
    if (tid == 0) {
        p.row_starts[p.batch] = (int32_t)rows;
        p.page_starts[p.batch] = (int32_t)taken;
        *p.free_count_out = (int32_t)(avail - taken);
    }
    if (FILL) {
        __syncthreads();
        for (int64_t first = (int64_t)tid * kRowsPerThread; first < p.max_rows; first += (int64_t)kScanThreads * kRowsPerThread)
            fill_rows(p, first, avail);
    }
}

__global__ void __launch_bounds__(kFillThreads) decode_attn_tables_rows_kernel(const TablesParams p)
{
    pdl_launch_dependents();
    pdl_wait_primary();
    const int64_t first = ((int64_t)blockIdx.x * kFillThreads + threadIdx.x) * kRowsPerThread;
    if (first < p.max_rows) fill_rows(p, first, (int64_t)*p.free_count_out + p.page_starts[p.batch]);
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int launch(const void* fn, unsigned grid, int threads, TablesParams& tp, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = 0;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void* args[] = {&tp};
    if (cudaLaunchKernelExC(&cfg, fn, args) != cudaSuccess) {
        (void)cudaGetLastError();
        return DA_ERR_CUDA;
    }
    return DA_OK;
}

}  // namespace

extern "C" int decode_attn_step_tables(const decode_attn_shape_t* shape, const decode_attn_tables_args_t* a, cudaStream_t stream)
{
    if (!shape || !a) return DA_ERR_INVALID_ARG;
    const decode_attn_shape_t& s = *shape;
    if (a->struct_size != sizeof(decode_attn_tables_args_t) || a->flags != 0) return DA_ERR_INVALID_ARG;
    if (s.batch < 0 || s.max_pages_per_seq < 0 || s.num_pages <= 0 || a->max_rows < 0 || a->free_capacity < 0)
        return DA_ERR_INVALID_ARG;
    if (s.page_size < 16 || s.page_size > 256 || (s.page_size & (s.page_size - 1)) != 0) return DA_ERR_UNSUPPORTED;
    if (s.num_pages > (int64_t)INT32_MAX || s.batch == INT32_MAX) return DA_ERR_UNSUPPORTED;
    if (!a->free_count || !a->free_count_out || !a->row_starts || !a->page_starts) return DA_ERR_INVALID_ARG;
    if (s.batch > 0 && (!a->seq_lens || !a->gains || !a->seq_lens_out)) return DA_ERR_INVALID_ARG;
    if (s.batch > 0 && s.max_pages_per_seq > 0 && !a->block_table) return DA_ERR_INVALID_ARG;
    if (a->free_capacity > 0 && !a->free_pages) return DA_ERR_INVALID_ARG;
    if (a->max_rows > 0 && (!a->slots || !a->positions)) return DA_ERR_INVALID_ARG;
    const void* const words[] = {a->seq_lens, a->gains, a->seq_lens_out, a->block_table, a->free_pages, a->free_count,
                                 a->free_count_out, a->row_starts, a->page_starts, a->positions, a->row_seq, a->status};
    for (const void* w : words)
        if (!aligned(w, 4)) return DA_ERR_INVALID_ARG;
    if (!aligned(a->slots, 8)) return DA_ERR_INVALID_ARG;

    TablesParams tp;
    std::memset(&tp, 0, sizeof tp);
    tp.seq_lens = a->seq_lens;
    tp.gains = a->gains;
    tp.seq_lens_out = a->seq_lens_out;
    tp.block_table = a->block_table;
    tp.free_pages = a->free_pages;
    tp.free_count = a->free_count;
    tp.free_count_out = a->free_count_out;
    tp.row_starts = a->row_starts;
    tp.page_starts = a->page_starts;
    tp.slots = a->slots;
    tp.positions = a->positions;
    tp.row_seq = a->row_seq;
    tp.status = a->status;
    tp.num_pages = s.num_pages;
    tp.batch = s.batch;
    tp.max_pages_per_seq = s.max_pages_per_seq;
    tp.max_rows = a->max_rows;
    tp.free_capacity = a->free_capacity;
    while ((1 << tp.page_shift) < s.page_size) ++tp.page_shift;
    // (positions are int32: the last page of a table too wide for that is never reached)
    const int64_t most = (int64_t)s.max_pages_per_seq * s.page_size;
    tp.most_tokens = most < INT32_MAX - 256 ? most : INT32_MAX - 256;
    tp.vec = aligned(a->slots, 16) && aligned(a->positions, 16) && aligned(a->row_seq, 16);
    // A step's rows by the block that makes the sums, as long as one launch costs less than two.
    constexpr int kOneLaunchRows = 8192;
    if (a->max_rows <= kOneLaunchRows) return launch((const void*)decode_attn_tables_kernel<true>, 1, kScanThreads, tp, stream);
    int rc = launch((const void*)decode_attn_tables_kernel<false>, 1, kScanThreads, tp, stream);
    if (rc != DA_OK) return rc;
    const int64_t per_block = (int64_t)kFillThreads * kRowsPerThread;
    return launch((const void*)decode_attn_tables_rows_kernel, (unsigned)((a->max_rows + per_block - 1) / per_block), kFillThreads,
                  tp, stream);
}
