// Step tables: block tables, slots and positions of a step from what every sequence gains (decode_attn_step_tables).
//
// Lengths, the list of free pages and the tables live on the device, so nothing of it waits for the host.  The order is
// fixed by prefix sums over the sequences: pages given back, pages lacked, new rows.  One block makes them (a batch is
// some hundred sequences: a few words a thread) and everything that is counted in sequences; what is counted in tokens
// (slots, positions, block-table entries of fresh pages) follows from the sums for every row by itself: row -> sequence
// by a binary search in row_starts, position -> page by the table or, for a fresh page, by its place in the list of free
// pages.  The row whose token is a fresh page's first writes the table entry.
//
// A step is latency: the chain of a launch, two reads of the inputs, a scan and one look at a table.  So the block is no larger
// than its work, the sums stay in shared memory for the search, and what a step without anything given back or refused
// does not need (three of four scans) is left out when a vote says so: 64 sequences decoding 8.7 -> 4.1 us, of which a launch
// that does nothing is about 2.  A prompt step's rows are a second launch (1 million rows, 17 MB, in 9.6 us).
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
    int32_t shared;                   // the batch's sums fit shared memory
};

constexpr int kScanThreads = 1024;                // at most
constexpr int kFillThreads = 256;
constexpr int kRowsPerThread = 4;
constexpr int kSharedBatch = 2048;                // sequences whose sums are kept in shared memory

// Sums saturate above every limit that they are held against (INT32_MAX rows or pages), which keeps them associative.  (Two that
// have saturated are 2^32, which 32 bits do not hold: what is added is cut off ahead of the addition.)
constexpr uint32_t kSaturated = 0x80000000u;
__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return a + min(b, kSaturated - a); }
__device__ __forceinline__ uint32_t sat(int64_t x) { return x > kSaturated ? kSaturated : (uint32_t)x; }

// Exclusive prefix sums of two values over the block's threads; the totals in `all`.
__device__ __forceinline__ void block_scan2(uint32_t& x, uint32_t& y, uint32_t (&all)[2], uint32_t (*sm)[2])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    uint32_t a = x, b = y;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, a, off), v = __shfl_up_sync(0xffffffffu, b, off);
        if (lane >= off) {
            a = sat_add(a, u);
            b = sat_add(b, v);
        }
    }
    __syncthreads();                                          // the scratch of the scan before is free
    if (lane == 31) {
        sm[warp][0] = a;
        sm[warp][1] = b;
    }
    __syncthreads();
    uint32_t u = lane < warps ? sm[lane][0] : 0, v = lane < warps ? sm[lane][1] : 0;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t s = __shfl_up_sync(0xffffffffu, u, off), t = __shfl_up_sync(0xffffffffu, v, off);
        if (lane >= off) {
            u = sat_add(u, s);
            v = sat_add(v, t);
        }
    }
    all[0] = __shfl_sync(0xffffffffu, u, 31);
    all[1] = __shfl_sync(0xffffffffu, v, 31);
    const uint32_t u0 = __shfl_sync(0xffffffffu, u, warp ? warp - 1 : 0), v0 = __shfl_sync(0xffffffffu, v, warp ? warp - 1 : 0);
    const uint32_t pa = __shfl_up_sync(0xffffffffu, a, 1), pb = __shfl_up_sync(0xffffffffu, b, 1);
    x = sat_add(lane ? pa : 0, warp ? u0 : 0);
    y = sat_add(lane ? pb : 0, warp ? v0 : 0);
}

// What the rows are found by, in shared memory or where the caller has it.
struct Sums {
    const int32_t *row_starts, *page_starts;
    const int32_t* old;               // tokens before the call (shared memory), or nullptr: from seq_lens_out
};

__device__ __forceinline__ void report(const TablesParams& p, int code)
{
    if (p.status != nullptr) record_status(p.status, code);
}

// What sequence b asks for.  back / lack: pages given back / lacked; rows: tokens gained.  old < 0: it is left alone.
struct Ask {
    int64_t old, fresh, back, lack, rows;
};

__device__ __forceinline__ Ask ask_of(const TablesParams& p, int b)
{
    Ask a = {-1, -1, 0, 0, 0};
    if (b >= p.batch) return a;
    const int64_t old = p.seq_lens[b], gain = p.gains[b];
    const int64_t fresh = old + gain > 0 ? old + gain : 0;
    if (old < 0 || old > p.most_tokens || fresh > p.most_tokens) return a;
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
__device__ __forceinline__ void fill_rows(const TablesParams& p, const Sums& sums, int64_t first, int64_t avail)
{
    const int total = sums.row_starts[p.batch];
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
                if (sums.row_starts[mid] <= row) lo = mid;
                else hi = mid;
            }
            b = lo;
        } else if (row >= end) {
            do ++b;                                           // (sequences without rows in between)
            while (sums.row_starts[b + 1] <= row);
        }
        if (row >= end) {
            start = sums.row_starts[b];
            end = sums.row_starts[b + 1];
            old = sums.old ? sums.old[b] : p.seq_lens_out[b] - (end - start);
            held = (old + mask) >> p.page_shift;
            page_at = sums.page_starts[b];
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
    extern __shared__ int32_t sm_sums[];                      // [batch + 1] rows, [batch + 1] pages, [batch] tokens before
    __shared__ uint32_t sm[kScanThreads / 32][2];
    pdl_launch_dependents();
    pdl_wait_primary();
    const int tid = threadIdx.x, lane = tid & 31, nt = blockDim.x;
    int32_t* const sm_rows = sm_sums;
    int32_t* const sm_pages = sm_rows + p.batch + 1;
    int32_t* const sm_old = sm_pages + p.batch + 1;
    const bool keep = FILL && p.shared;
    const int64_t count = *p.free_count;
    Ask ask = ask_of(p, tid);                          // of the first nt sequences, asked for beside the count
    const bool sane = count >= 0 && count <= p.free_capacity;
    if (!sane && tid == 0) report(p, DA_ERR_STALE_PLAN);
    const Ask none = {-1, -1, 0, 0, 0};
    if (!sane) ask = none;
    // 1. pages given back: their places in the list, and how many fit
    int64_t pushed = 0;
    uint32_t all[2];
    bool any_back = ask.back > 0;
    for (int b = nt + tid; b < p.batch; b += nt) any_back |= p.gains[b] < 0;
    bool full = false;                                        // some of what is given back does not fit
    if (__syncthreads_or(any_back && sane)) {
        for (int b0 = 0; b0 < p.batch && !full; b0 += nt) {
            const Ask a = b0 == 0 ? ask : sane ? ask_of(p, b0 + tid) : none;
            uint32_t at = sat(a.back), zero = 0;
            block_scan2(at, zero, all, sm);
            const bool fits = count + pushed + at + a.back <= p.free_capacity;
            // a few pages by their own thread, many by the warp
            const int64_t pages = fits ? a.back : 0, to = count + pushed + at;
            const int64_t from = (a.fresh + ((int64_t)1 << p.page_shift) - 1) >> p.page_shift;
            const int32_t* const row = p.block_table + (int64_t)(b0 + tid) * p.max_pages_per_seq + from;
            if (pages <= 4)
                for (int i = 0; i < (int)pages; ++i) p.free_pages[to + i] = row[i];
            for (unsigned many = __ballot_sync(0xffffffffu, pages > 4); many != 0; many &= many - 1) {
                const int l = __ffs(many) - 1;
                const int64_t n = __shfl_sync(0xffffffffu, pages, l), dst = __shfl_sync(0xffffffffu, to, l);
                const int32_t* const src = reinterpret_cast<const int32_t*>(__shfl_sync(0xffffffffu, (unsigned long long)row, l));
                for (int64_t i = lane; i < n; i += 32) p.free_pages[dst + i] = src[i];
            }
            full = __syncthreads_or(a.back > 0 && !fits);
            if (full) {
                // (what does not fit is behind what does: the sums only grow)
                uint32_t ok = sat(pages), zero2 = 0;
                block_scan2(ok, zero2, all, sm);
            }
            pushed += all[0];
        }
    }
    const int64_t avail = count + pushed;
    // 2. pages and rows of those that grow; lengths
    uint32_t lacked = 0, asked = 0, gave = 0;                 // by all that ask
    int64_t taken = 0, rows = 0;                              // granted
    bool refused = false;
    for (int b0 = 0; b0 < p.batch; b0 += nt) {
        const int b = b0 + tid;
        const Ask a = sane ? (b0 == 0 ? ask : ask_of(p, b)) : none;
        if (sane && b < p.batch && a.old < 0) report(p, DA_ERR_STALE_PLAN);
        uint32_t lack = sat(a.lack), row = sat(a.rows);
        block_scan2(lack, row, all, sm);
        const bool pages_ok = a.lack == 0 || (int64_t)sat_add(sat_add(lacked, lack), sat(a.lack)) <= avail;
        const bool rows_ok = a.rows == 0 || (int64_t)sat_add(sat_add(asked, row), sat(a.rows)) <= p.max_rows;
        lacked = sat_add(lacked, all[0]);
        asked = sat_add(asked, all[1]);
        if (!pages_ok) report(p, DA_ERR_NO_PAGES);
        if (!rows_ok) report(p, DA_ERR_WORKSPACE_TOO_SMALL);
        bool back_ok = true;
        int64_t row_at = rows + row, page_at = taken + lack;
        // (who has been refused something leaves gaps in the sums: those behind need sums of their own)
        refused |= __syncthreads_or(!(pages_ok && rows_ok)) != 0;
        if (refused) {
            uint32_t got_rows = pages_ok && rows_ok ? sat(a.rows) : 0, got = pages_ok && rows_ok ? sat(a.lack) : 0;
            block_scan2(got, got_rows, all, sm);
            row_at = rows + got_rows;
            page_at = taken + got;
        }
        taken += all[0];
        rows += all[1];
        if (full) {                                           // giving back is granted by the sums of 1.
            uint32_t back = sat(a.back), zero = 0;
            block_scan2(back, zero, all, sm);
            back_ok = a.back == 0 || count + (int64_t)sat_add(sat_add(gave, back), sat(a.back)) <= p.free_capacity;
            if (!back_ok) report(p, DA_ERR_NO_PAGES);
            gave = sat_add(gave, all[0]);
        }
        if (b < p.batch) {
            p.row_starts[b] = (int32_t)row_at;
            p.page_starts[b] = (int32_t)page_at;
            const bool granted = a.old >= 0 && pages_ok && rows_ok && back_ok;
            // (a length that is left alone is copied: the two arrays may be one)
            p.seq_lens_out[b] = granted ? (int32_t)a.fresh : p.seq_lens[b];
            if (keep) {
                sm_rows[b] = (int32_t)row_at;
                sm_pages[b] = (int32_t)page_at;
                sm_old[b] = (int32_t)a.old;
            }
        }
    }
    if (tid == 0) {
        p.row_starts[p.batch] = (int32_t)rows;
        p.page_starts[p.batch] = (int32_t)taken;
        *p.free_count_out = (int32_t)(avail - taken);
        if (keep) sm_rows[p.batch] = (int32_t)rows;
    }
    if (FILL) {
        __syncthreads();
        const Sums sums = keep ? Sums{sm_rows, sm_pages, sm_old} : Sums{p.row_starts, p.page_starts, nullptr};
        for (int64_t first = (int64_t)tid * kRowsPerThread; first < p.max_rows; first += (int64_t)nt * kRowsPerThread)
            fill_rows(p, sums, first, avail);
    }
}

__global__ void __launch_bounds__(kFillThreads) decode_attn_tables_rows_kernel(const TablesParams p)
{
    extern __shared__ int32_t sm_sums[];
    pdl_launch_dependents();
    pdl_wait_primary();
    const int64_t first = ((int64_t)blockIdx.x * kFillThreads + threadIdx.x) * kRowsPerThread;
    const int64_t avail = (int64_t)*p.free_count_out + p.page_starts[p.batch];
    Sums sums = {p.row_starts, p.page_starts, nullptr};
    if (p.shared) {
        int32_t* const rows = sm_sums;
        int32_t* const pages = rows + p.batch + 1;
        int32_t* const old = pages + p.batch + 1;
        for (int b = threadIdx.x; b <= p.batch; b += kFillThreads) {
            rows[b] = p.row_starts[b];
            if (b < p.batch) {
                pages[b] = p.page_starts[b];
                old[b] = p.seq_lens_out[b] - (p.row_starts[b + 1] - p.row_starts[b]);
            }
        }
        __syncthreads();
        sums = {rows, pages, old};
    }
    if (first < p.max_rows) fill_rows(p, sums, first, avail);
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int launch(const void* fn, unsigned grid, int threads, size_t smem, TablesParams& tp, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg;
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
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
    tp.shared = s.batch <= kSharedBatch;
    const size_t smem = tp.shared ? (3 * (size_t)s.batch + 2) * sizeof(int32_t) : 0;
    auto threads_for = [](int64_t n) { return (int)(n >= kScanThreads ? kScanThreads : n < 64 ? 64 : (n + 31) / 32 * 32); };
    // A step's rows by the block that makes the sums, as long as one launch costs less than two.
    constexpr int kOneLaunchRows = 8192;
    if (a->max_rows <= kOneLaunchRows) {
        const int64_t n = s.batch > a->max_rows / kRowsPerThread ? s.batch : a->max_rows / kRowsPerThread;
        return launch((const void*)decode_attn_tables_kernel<true>, 1, threads_for(n), smem, tp, stream);
    }
    int rc = launch((const void*)decode_attn_tables_kernel<false>, 1, threads_for(s.batch), 0, tp, stream);
    if (rc != DA_OK) return rc;
    const int64_t per_block = (int64_t)kFillThreads * kRowsPerThread;
    return launch((const void*)decode_attn_tables_rows_kernel, (unsigned)((a->max_rows + per_block - 1) / per_block), kFillThreads,
                  smem, tp, stream);
}
