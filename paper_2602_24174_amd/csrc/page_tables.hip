// Block tables and slots of a paged cache from the requests' lengths.
//
// One launch: every workgroup owns 8 sequences (more of a batch beyond 2048, so that 256 workgroups read all lengths), sums the pages and rows
// that all sequences ask for (those before its own give its place in the list of free pages and in the list of slots), and a wave
// writes a sequence's new pages and slots.  A few integers per sequence, page and row: bound by launch latency and three dependent
// reads.  One more workgroup adds up what was given and refused (4096 sequences of up to 600 rows 18.9 us with that at the end of the last
// one, 11.3 so).
#include "tasc_internal.h"
#include <algorithm>

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;

struct PageArgs {
    const int32_t* kv_len;
    const int32_t* new_rows;
    const int32_t* held;
    const int32_t* free_pages;
    int32_t *table, *pages, *row_off, *slots, *summary;
    int32_t batch, n_free, max_pages, slots_cap, per_wg, n_wgs;
};

struct Ask { int32_t len, rows, held, need, pages; bool fits; };   // rows: those that count in row_off; pages: new ones
__device__ __forceinline__ Ask ask_of(const PageArgs& a, int b) {
    Ask q;
    q.len = a.kv_len[b];
    const int32_t n = a.new_rows ? a.new_rows[b] : 0;
    q.held = a.held ? a.held[b] : 0;
    q.rows = max(n, 0);
    q.need = q.len > 0 ? (q.len - 1) / TASC_PAGE_TOKENS + 1 : 0;
    q.fits = n >= 0 && n <= q.len && q.need <= a.max_pages && q.held >= 0 && q.held <= a.max_pages;
    q.pages = q.fits ? max(q.need - q.held, 0) : 0;
    return q;
}
__device__ __forceinline__ int64_t wave_sum64(int64_t v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ int64_t wave_scan64(int64_t v, int lane) {      // inclusive
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t up = __shfl_up(v, o);
        if (lane >= o) v += up;
    }
    return v;
}
__device__ __forceinline__ int64_t from_lane(int64_t v, int lane) {        // a uniform lane
    return (int64_t)(u32)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (u32)__builtin_amdgcn_readlane((int)v, lane);
}

// The summary, by a workgroup of its own: a wave adds up a run of sequences, and goes over it again once it knows where it begins.
__device__ __forceinline__ void sum_up(const PageArgs& a, int tid, int lane, int wave, int64_t (&s_sum)[3][kWaves], int32_t (&s_refused)[kWaves]) {
    const int run = ((a.batch + kWaves - 1) / kWaves + 63) / 64 * 64, from = min(wave * run, a.batch), to = min(from + run, a.batch);
    int64_t pages = 0, rows = 0;
#pragma unroll 4
    for (int b = from + lane; b < to; b += 64) {
        const Ask q = ask_of(a, b);
        pages += q.pages;
        rows += q.rows;
    }
    pages = wave_sum64(pages);
    rows = wave_sum64(rows);
    if (lane == 0) {
        s_sum[0][wave] = pages;
        s_sum[1][wave] = rows;
    }
    __syncthreads();
    // pages asked for up to the last sequence that is granted: the sums only grow, so it is the largest of a granted one's
    int64_t before = 0, reach = 0;
    for (int w = 0; w < wave; ++w) before += s_sum[0][w];
    int refused = 0;
    constexpr int AHEAD = 4;
    for (int c = from; c < to; c += 64 * AHEAD) {
        Ask q[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            q[j] = Ask{};
            if (c + 64 * j + lane < to) q[j] = ask_of(a, c + 64 * j + lane);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int64_t end = wave_scan64(q[j].pages, lane) + before;
            before = from_lane(end, 63);
            if (c + 64 * j + lane >= to) continue;
            if (!q[j].fits || (q[j].pages > 0 && end > a.n_free)) ++refused;
            else reach = end;
        }
    }
    for (int o = 32; o > 0; o >>= 1) {
        reach = max(reach, (int64_t)__shfl_xor(reach, o));
        refused += __shfl_xor(refused, o);
    }
    if (lane == 0) {
        s_sum[2][wave] = reach;
        s_refused[wave] = refused;
    }
    __syncthreads();
    if (tid != 0) return;
    rows = 0;
    for (int w = 0; w < kWaves; ++w) rows += s_sum[1][w];
    for (int w = 1; w < kWaves; ++w) {
        reach = max(reach, s_sum[2][w]);
        refused += s_refused[w];
    }
    a.summary[0] = (int32_t)min(rows, (int64_t)INT32_MAX);
    a.summary[1] = (int32_t)min(reach, (int64_t)INT32_MAX);
    a.summary[2] = refused;
}

__global__ __launch_bounds__(kThreads) void k_page_tables(PageArgs a) {
    __shared__ int64_t s_sum[3][kWaves];
    __shared__ int32_t s_refused[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if ((int)blockIdx.x == a.n_wgs) return sum_up(a, tid, lane, wave, s_sum, s_refused);
    const int b0 = (int)min((int64_t)blockIdx.x * a.per_wg, (int64_t)a.batch), b1 = min(b0 + a.per_wg, a.batch);
    int64_t pages_before = 0, rows_before = 0, rows_all = 0;
#pragma unroll 4
    for (int b = tid; b < a.batch; b += kThreads) {
        const Ask q = ask_of(a, b);
        pages_before += b < b0 ? q.pages : 0;
        rows_before += b < b0 ? q.rows : 0;
        rows_all += q.rows;
    }
    pages_before = wave_sum64(pages_before);
    rows_before = wave_sum64(rows_before);
    rows_all = wave_sum64(rows_all);
    if (lane == 0) {
        s_sum[0][wave] = pages_before;
        s_sum[1][wave] = rows_before;
        s_sum[2][wave] = rows_all;
    }
    __syncthreads();
    pages_before = rows_before = rows_all = 0;
    for (int w = 0; w < kWaves; ++w) {
        pages_before += s_sum[0][w];
        rows_before += s_sum[1][w];
        rows_all += s_sum[2][w];
    }
    // the workgroup's sequences, 64 at a time: a lane each for the sums, then a wave each in turn
    for (int c = b0; c < b1; c += 64) {
        Ask mine{};
        if (c + lane < b1) mine = ask_of(a, c + lane);
        const int64_t pages_to = wave_scan64(mine.pages, lane) + pages_before, rows_to = wave_scan64(mine.rows, lane) + rows_before;
        pages_before = from_lane(pages_to, 63);
        rows_before = from_lane(rows_to, 63);
        for (int n = wave; n < min(64, b1 - c); n += kWaves) {
            const int b = c + n;
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, n); };
            const int held = of(mine.held), need = of(mine.need), pages = of(mine.pages), rows = of(mine.rows), len = of(mine.len);
            const int64_t end = from_lane(pages_to, n), first = end - pages, row = from_lane(rows_to, n) - rows;
            const bool granted = of(mine.fits) && (pages == 0 || end <= a.n_free);
            int32_t* const tab = a.table + (size_t)b * a.max_pages;
            auto given = [&](int j) { return a.free_pages ? a.free_pages[first + j] : (int32_t)(first + j); };      // the sequence's new page j
            if (granted)
                for (int j = lane; j < pages; j += 64) tab[held + j] = given(j);
            if (lane == 0) {
                if (a.pages) a.pages[b] = granted ? max(need, held) : held;
                if (a.row_off) a.row_off[b] = (int32_t)min(row, (int64_t)INT32_MAX);
            }
            if (!a.slots) continue;
            const u32 count = (u32)min((int64_t)rows, max((int64_t)a.slots_cap - row, (int64_t)0));
#pragma unroll 4
            for (u32 i = lane; i < count; i += 64) {        // (the step behind 2^31 - 1 slots is past 31 bits)
                const int pos = len - rows + (int)i, at = pos / TASC_PAGE_TOKENS;
                int32_t slot = -1;
                if (granted) {
                    const int page = at < held ? tab[at] : given(at - held);
                    if (page >= 0 && page < 1 << 27) slot = page * TASC_PAGE_TOKENS + pos % TASC_PAGE_TOKENS;      // (no cache has more pages)
                }
                a.slots[row + i] = slot;
            }
        }
    }
    if (a.slots)
        for (int64_t i = rows_all + (int64_t)blockIdx.x * kThreads + tid; i < a.slots_cap; i += (int64_t)a.n_wgs * kThreads) a.slots[i] = -1;
    if ((int)blockIdx.x == a.n_wgs - 1 && tid == 0 && a.row_off) a.row_off[a.batch] = (int32_t)min(rows_all, (int64_t)INT32_MAX);
}

}  // namespace

extern "C" tasc_status tasc_page_tables(const int32_t* kv_len, const int32_t* new_rows, const int32_t* held, int32_t batch, const int32_t* free_pages, int32_t n_free,
                                        int32_t* table, int32_t max_pages, int32_t* pages, int32_t* row_off, int32_t* slots, int32_t slots_cap, int32_t* summary,
                                        void* stream) {
    TASC_REQUIRE(kv_len && table, "page_tables: null argument");
    TASC_REQUIRE(batch >= 1 && batch <= 1 << 20, "page_tables: batch %d outside [1, 2^20]", batch);
    TASC_REQUIRE(max_pages >= 1 && max_pages < 1 << 27, "page_tables: max_pages %d outside [1, 2^27)", max_pages);
    TASC_REQUIRE(n_free >= 0 && n_free < 1 << 27, "page_tables: n_free %d outside [0, 2^27)", n_free);
    TASC_REQUIRE(slots_cap >= 0 && (slots || slots_cap == 0), "page_tables: %d slots", slots_cap);
    // (workgroups read the lengths of all sequences while others write)
    struct Array { const char* name; const int32_t* at; int64_t n; };
    const Array written[] = {{"table", table, (int64_t)batch * max_pages}, {"pages", pages, batch}, {"row_off", row_off, batch + 1}, {"slots", slots, slots_cap}, {"summary", summary, 3}};
    const Array read[] = {{"kv_len", kv_len, batch}, {"new_rows", new_rows, batch}, {"held", held, batch}, {"free_pages", free_pages, n_free}};
    auto apart = [](const Array& x, const Array& y) { return !x.at || !y.at || x.n == 0 || y.n == 0 || (uintptr_t)(x.at + x.n) <= (uintptr_t)y.at || (uintptr_t)(y.at + y.n) <= (uintptr_t)x.at; };
    for (const Array& w : written) {
        for (const Array& r : read) TASC_REQUIRE(apart(w, r), "page_tables: %s and %s overlap", w.name, r.name);
        for (const Array* v = written; v != &w; ++v) TASC_REQUIRE(apart(w, *v), "page_tables: %s and %s overlap", w.name, v->name);
    }
    // runs of at least 8 sequences (a wave each), 256 workgroups at most, for each reads all lengths (us of 64, 2048 and 4096 sequences of up to 600
    // rows 6.3, 8.0, 11.7; with up to 512 workgroups 6.4, 7.9, 12.7, and runs of 4 then 6.0, 9.1, 12.5; with runs of 16 8.6, 10.1, 11.7)
    const int per_wg = std::max(8, (batch + 255) / 256);
    const int n_wgs = (batch + per_wg - 1) / per_wg;
    const PageArgs a{kv_len, new_rows, held, free_pages, table, pages, row_off, slots, summary, batch, n_free, max_pages, slots_cap, per_wg, n_wgs};
    k_page_tables<<<dim3((unsigned)(n_wgs + (summary ? 1 : 0))), dim3(kThreads), 0, (hipStream_t)stream>>>(a);
    TASC_LAUNCH_CHECK();
    return TASC_OK;
}
