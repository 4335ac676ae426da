// Pages of a cache behind their tables: sequences that continue others, pages copied through all layers, the pages that no table lists, and the
// pages in use moved to the front of their pool.
//
// Which pages are in use follows from the tables alone (a map of the pages that any table lists), so sequences may share pages without
// counts that have to be kept beside them.
#include "tasc_internal.h"
#include <algorithm>

namespace {

constexpr int kPageLimit = 1 << 27;                        // no cache has more pages

__device__ __forceinline__ int wave_sum32(int v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// ---------------------------------------------------------------- forks
struct ForkArgs {
    const int32_t *src, *dst, *new_pages;
    int32_t *kv_len, *table, *pages, *copy_from, *copy_to, *summary;
    int32_t n, batch, max_pages;
};
struct Fork { int32_t src, dst, len, need; bool part, ok; };
// a pair by itself; whether another one names its dst is left to the caller
__device__ __forceinline__ Fork fork_of(const ForkArgs& a, int i) {
    Fork f{a.src[i], a.dst[i], 0, 0, false, false};
    if (f.src < 0 || f.src >= a.batch || f.dst < 0 || f.dst >= a.batch) return f;
    f.len = a.kv_len[f.src];
    const int held = a.pages[f.src];
    f.need = f.len > 0 ? (f.len - 1) / TASC_PAGE_TOKENS + 1 : 0;
    f.part = f.len > 0 && f.len % TASC_PAGE_TOKENS != 0;
    f.ok = f.src != f.dst && f.len >= 0 && f.need <= held && held <= a.max_pages;
    if (f.part) {
        const int fresh = a.new_pages ? a.new_pages[i] : -1;
        f.ok = f.ok && fresh >= 0 && fresh < kPageLimit;
    }
    return f;
}

// A workgroup a pair, which looks through all pairs for one that takes the same place or continues it (nothing that a granted pair reads is
// then written by another).  A few integers per page of a prompt: bound by launch and three dependent reads.  Up to kForkThreads pairs are added up by
// one more workgroup of the same launch, a lane a pair with the others' numbers out of LDS; more by a launch of its own, since that
// workgroup's look at all pairs of all pairs would take longer than the copies (480 pairs, one at a time through the scalar cache: 130 us).
constexpr int kForkThreads = 256;
__device__ __forceinline__ void sum_forks(int done, int taken, int refused, int32_t* summary, int (&s_sum)[3][kForkThreads / 64], int tid) {
    done = wave_sum32(done);
    taken = wave_sum32(taken);
    refused = wave_sum32(refused);
    if ((tid & 63) == 0) {
        s_sum[0][tid >> 6] = done;
        s_sum[1][tid >> 6] = taken;
        s_sum[2][tid >> 6] = refused;
    }
    __syncthreads();
    if (tid < 3) summary[tid] = s_sum[tid][0] + s_sum[tid][1] + s_sum[tid][2] + s_sum[tid][3];
}
__global__ __launch_bounds__(kForkThreads) void k_pages_fork(ForkArgs a) {
    __shared__ int s_clash[kForkThreads / 64], s_sum[3][kForkThreads / 64];
    __shared__ int2 s_pair[kForkThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if ((int)blockIdx.x == a.n) {
        Fork f{-1, -1, 0, 0, false, false};
        if (tid < a.n) f = fork_of(a, tid);
        s_pair[tid] = int2{f.src, f.dst};
        __syncthreads();
        for (int j = 0; j < a.n; ++j) {
            const int2 p = s_pair[j];
            if (p.x == f.dst || (j < tid && p.y == f.dst)) f.ok = false;
        }
        const bool real = tid < a.n;
        return sum_forks(real && f.ok, real && f.ok && f.part, real && !f.ok, a.summary, s_sum, tid);
    }
    const int i = blockIdx.x;
    const Fork f = fork_of(a, i);
    bool clash = false;
    for (int j = tid; j < a.n; j += kForkThreads) clash |= a.src[j] == f.dst || (j < i && a.dst[j] == f.dst);
    const bool any = __any(clash);
    if (lane == 0) s_clash[wave] = any;
    __syncthreads();
    const bool granted = f.ok && !(s_clash[0] | s_clash[1] | s_clash[2] | s_clash[3]);
    const int fresh = !granted ? -2 : f.part ? a.new_pages[i] : -1;
    if (granted) {
        const int32_t* const from = a.table + (size_t)f.src * a.max_pages;
        int32_t* const to = a.table + (size_t)f.dst * a.max_pages;
        for (int c = tid; c < f.need; c += kForkThreads) to[c] = fresh >= 0 && c == f.need - 1 ? fresh : from[c];
        if (tid == 0) {
            a.kv_len[f.dst] = f.len;
            a.pages[f.dst] = f.need;
        }
    }
    if (tid == 0) {
        a.copy_from[i] = fresh >= 0 ? a.table[(size_t)f.src * a.max_pages + f.need - 1] : fresh;
        a.copy_to[i] = fresh;
    }
}
__global__ __launch_bounds__(kForkThreads) void k_pages_fork_sum(const int32_t* copy_to, int n, int32_t* summary) {
    __shared__ int s_sum[3][kForkThreads / 64];
    int done = 0, taken = 0, refused = 0;
    for (int i = threadIdx.x; i < n; i += kForkThreads) {
        const int to = copy_to[i];
        done += to != -2;
        taken += to >= 0;
        refused += to == -2;
    }
    sum_forks(done, taken, refused, summary, s_sum, threadIdx.x);
}

// ---------------------------------------------------------------- copies
typedef u32 quad __attribute__((ext_vector_type(4)));
struct CopyArgs {
    char* pool;
    const int32_t *from, *to;
    size_t page_bytes, layer_stride;
    int64_t n_items;                   // (layer, pair, piece), a wave each
    int32_t n, n_pages, pieces, quads; // of a page: pieces, and 16-byte words of a piece
};
constexpr int kCopyThreads = 256, kCopyAhead = 8;
// Bound by the bytes: a wave has up to 8 KB under way before it writes.  480 copies of 18432-byte pages in 12 layers (106 MB written, the sources' 7 MB read once): 24 us;
// a few thousand pages of 4608 bytes in 28 layers 35.
__global__ __launch_bounds__(kCopyThreads) void k_pages_copy(CopyArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t waves = (int64_t)gridDim.x * (kCopyThreads / 64);
    for (int64_t w = (int64_t)blockIdx.x * (kCopyThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < a.n_items; w += waves) {
        const int64_t pair_of = w / a.pieces;
        const int piece = (int)(w % a.pieces), i = (int)(pair_of % a.n), layer = (int)(pair_of / a.n);
        const int from = a.from[i], to = a.to[i];
        if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages || from == to) continue;
        const int first = piece * a.quads, n = min(a.quads, (int)(a.page_bytes / 16) - first);
        const quad* const p = (const quad*)(a.pool + layer * a.layer_stride + from * a.page_bytes) + first;
        quad* const q = (quad*)(a.pool + layer * a.layer_stride + to * a.page_bytes) + first;
        quad v[kCopyAhead];
#pragma unroll
        for (int j = 0; j < kCopyAhead; ++j)
            if (64 * j + lane < n) v[j] = p[64 * j + lane];
#pragma unroll
        for (int j = 0; j < kCopyAhead; ++j)
            if (64 * j + lane < n) q[64 * j + lane] = v[j];
    }
}

// ---------------------------------------------------------------- which pages are listed
struct UseArgs {
    const int32_t *table, *pages;
    int32_t batch, max_pages, n_pages, n_words;
    uint8_t* marks;                    // [32 n_words, to a whole 64] a byte a page: some table lists it
    u32* bits;                         // the same as bits
    u32* before;                       // [n_words] listed pages in the words before (compacting)
    u32* sums;                         // [n_blocks] listed pages of a block of words
    u64* entries;                      // [n_marking] table entries that list a page of the pool, by workgroup
    int32_t n_marking;
    int32_t* free_pages;               // freeing
    int32_t *table_out, *copy_from, *copy_to;   // compacting
    int32_t cap;                       // moves
    int32_t* summary;
};
constexpr int kBlockWords = 256, kUseThreads = 256, kSmallThreads = 1024;

__device__ __forceinline__ int row_pages(const UseArgs& a, int b) { return min(max(a.pages[b], 0), a.max_pages); }

// Times below: 4096 sequences, 2.5 million entries, a pool of 3.7 million pages.  3.7 MB of marks: 2 us
__global__ __launch_bounds__(kUseThreads) void k_use_clear(UseArgs a) {
    quad* const to = (quad*)a.marks;                       // (two words' pages)
    const int n = (a.n_words + 1) / 2 * 4;
    for (int i = blockIdx.x * kUseThreads + threadIdx.x; i < n; i += gridDim.x * kUseThreads) to[i] = quad{0, 0, 0, 0};
}
// A wave a sequence (of a run of columns).  A page's mark is a byte, written by whoever lists it: with bits set by atomics, which all meet behind the dies'
// caches, a whole call over 2.5 million entries of a pool of 3.7 million pages took 248 us, with bytes 56.  Workgroups in turn take the lower and the upper half of the
// pages (the dispatcher deals them to the dies in turn, so a die's cache then holds half of the marks): 26 us of this kernel without that, 19 with two or four
// shares, 24 with eight, since every share reads all entries.
constexpr int kMarkCols = 4096, kMarkBlocks = 2048, kMarkShares = 2;
__global__ __launch_bounds__(kUseThreads) void k_use_mark(UseArgs a, int col_runs, int64_t n_items) {
    constexpr int shares = kMarkShares;
    __shared__ u64 s_n[kUseThreads / 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = blockIdx.x % shares;
    const int per = (a.n_pages - 1) / shares + 1;
    const u32 from = share * (u32)per, count = min((u32)per, (u32)a.n_pages - min(from, (u32)a.n_pages));
    u64 n = 0;
    for (int64_t item = (int64_t)(blockIdx.x / shares) * (kUseThreads / 64) + wave; item < n_items; item += (int64_t)(gridDim.x / shares) * (kUseThreads / 64)) {
        const int b = (int)(item / col_runs), run = (int)(item % col_runs);
        const int to = min(row_pages(a, b), (int)min((int64_t)(run + 1) * kMarkCols, (int64_t)a.max_pages));
        const int32_t* const row = a.table + (size_t)b * a.max_pages;
        constexpr int AHEAD = 8;
        for (int c = run * kMarkCols + lane; c < to; c += 64 * AHEAD) {
            int p[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) p[j] = c + 64 * j < to ? row[c + 64 * j] : -1;
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if ((u32)p[j] - from >= count) continue;   // (also what is no page of the pool)
                ++n;
                a.marks[p[j]] = 1;
            }
        }
    }
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
    if (lane == 0) s_n[wave] = n;
    __syncthreads();
    if (threadIdx.x == 0) a.entries[blockIdx.x] = s_n[0] + s_n[1] + s_n[2] + s_n[3];
}
__device__ __forceinline__ int block_sum(int v, int* s, int tid) {       // of 256 threads
    v = wave_sum32(v);
    if ((tid & 63) == 0) s[tid >> 6] = v;
    __syncthreads();
    v = s[0] + s[1] + s[2] + s[3];
    __syncthreads();
    return v;
}
// Marks to bits, and a block of words' sum.  Bound by the launch: 4 us
__global__ __launch_bounds__(kUseThreads) void k_use_count(UseArgs a) {
    __shared__ int s[kUseThreads / 64];
    const int tid = threadIdx.x, w0 = blockIdx.x * kBlockWords;
    int n = 0;
    for (int w = w0 + tid; w < min(w0 + kBlockWords, a.n_words); w += kUseThreads) {
        const quad* const p = (const quad*)(a.marks + 32 * (size_t)w);
        const quad lo = p[0], hi = p[1];
        // four marks to four bits: byte i's bit 0 goes to bit 21 + i of the product
        auto four = [](u32 m) { return m * 0x00204081u >> 21 & 15; };
        const u32 bits = four(lo[0]) | four(lo[1]) << 4 | four(lo[2]) << 8 | four(lo[3]) << 12 | four(hi[0]) << 16 | four(hi[1]) << 20 | four(hi[2]) << 24 | four(hi[3]) << 28;
        a.bits[w] = bits;
        n += __popc(bits);
    }
    n = block_sum(n, s, tid);
    if (tid == 0) a.sums[blockIdx.x] = n;
}
// pages of word w that exist
__device__ __forceinline__ u32 word_mask(const UseArgs& a, int w) {
    const int left = a.n_pages - 32 * w;
    return left >= 32 ? 0xFFFFFFFFu : left > 0 ? (1u << left) - 1 : 0;
}

// What the pages of one word leave where: lanes 0 .. 31 take word w, the others word w + 1; `before`: listed pages in the words before the lane's
struct Totals { int listed, moves; };
template <bool COMPACT>
__device__ __forceinline__ void place_page(const UseArgs& a, const Totals& t, int w, u32 bits, int before, int lane) {
    const int bit = lane & 31, p = 32 * w + bit;
    if (p >= a.n_pages) return;
    const bool listed = bits >> bit & 1;
    const int below = before + __popc(bits & ((1u << bit) - 1));         // listed pages below p
    if (!COMPACT) {
        if (!listed) a.free_pages[p - below] = p;
    } else if (listed && p >= t.listed) {
        const int j = t.listed - 1 - below;
        if (j < a.cap) a.copy_from[j] = p;
        if (j == a.cap && a.summary) a.summary[2] = p + 1;
    } else if (!listed && p < t.listed && p - below < a.cap) {
        a.copy_to[p - below] = p;
    }
}
// one thread: what is known without the pages
template <bool COMPACT>
__device__ __forceinline__ void sum_use(const UseArgs& a, const Totals& t, u64 entries) {
    if (!a.summary) return;
    if (!COMPACT) {
        a.summary[0] = a.n_pages - t.listed;
        a.summary[1] = t.listed;
        a.summary[2] = (int32_t)min(entries, (u64)INT32_MAX);
    } else {
        a.summary[0] = t.listed;
        a.summary[1] = min(t.moves, a.cap);
        if (t.moves <= a.cap) a.summary[2] = t.listed;
    }
}
template <bool COMPACT>
__device__ __forceinline__ void pad(const UseArgs& a, const Totals& t, int64_t first, int64_t step) {
    if (!COMPACT) {
        for (int64_t i = a.n_pages - t.listed + first; i < a.n_pages; i += step) a.free_pages[i] = -1;
    } else {
        for (int64_t i = t.moves + first; i < a.cap; i += step) a.copy_from[i] = a.copy_to[i] = -1;
    }
}
// listed pages from the first page on that is not below `listed`
__device__ __forceinline__ int listed_from(const UseArgs& a, int w, u32 bits, int listed) {
    const int lo = listed - 32 * w;
    return lo >= 32 ? 0 : __popc(lo > 0 ? bits & ~((1u << lo) - 1) : bits);
}

// Every page to its place, by the sums of all blocks before (each workgroup adds them all up itself: 447 here, 16384 in the largest pool).  Bound by its rounds, 32 a wave, of two
// shuffles and a partly filled store to consecutive places: 14 MB in 10.6 us, with blocks of 1024 words instead of 256 24.
template <bool COMPACT>
__global__ __launch_bounds__(kUseThreads) void k_use_list(UseArgs a) {
    __shared__ int s[kUseThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, blk = blockIdx.x, n_blocks = gridDim.x;
    int before = 0, all = 0;
    for (int i = tid; i < n_blocks; i += kUseThreads) {
        const int v = a.sums[i];
        all += v;
        before += i < blk ? v : 0;
    }
    before = block_sum(before, s, tid);
    Totals t{block_sum(all, s, tid), 0};
    if (COMPACT) {                                          // pages behind the last one that stays
        const int edge = t.listed / 32 / kBlockWords;       // the block that holds page `listed`
        int far = 0;
        for (int i = edge + 1 + tid; i < n_blocks; i += kUseThreads) far += a.sums[i];
        for (int w = edge * kBlockWords + tid; w < min((edge + 1) * kBlockWords, a.n_words); w += kUseThreads) far += listed_from(a, w, a.bits[w], t.listed);
        t.moves = block_sum(far, s, tid);
    }
    // a wave 64 words at a time: a lane each for the sums, then two words side by side
    __shared__ int s_wave[kBlockWords / 64];
    const int w0 = blk * kBlockWords;
    u32 mine[kBlockWords / kUseThreads];
#pragma unroll
    for (int j = 0; j < kBlockWords / kUseThreads; ++j) {
        const int w = w0 + (4 * j + wave) * 64 + lane;
        mine[j] = w < a.n_words ? a.bits[w] : 0;
        const int n = wave_sum32(__popc(mine[j]));
        if (lane == 0) s_wave[4 * j + wave] = n;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kBlockWords / kUseThreads; ++j) {
        const int run = 4 * j + wave, first = w0 + run * 64;
        if (first >= a.n_words) break;
        int at = before;
        for (int i = 0; i < run; ++i) at += s_wave[i];
        int up = __popc(mine[j]);
        const int own = up;
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(up, o);
            if (lane >= o) up += v;
        }
        const int mine_before = at + up - own;
        if (COMPACT && first + lane < a.n_words) a.before[first + lane] = mine_before;
        for (int i = 0; i < 64 && first + i < a.n_words; i += 2) {
            const int of = i + (lane >> 5);
            place_page<COMPACT>(a, t, first + of, __shfl(mine[j], of), __shfl(mine_before, of), lane);
        }
    }
    pad<COMPACT>(a, t, (int64_t)blk * kUseThreads + tid, (int64_t)n_blocks * kUseThreads);
    if (blk == 0) {
        __shared__ u64 s_entries[kUseThreads / 64];
        u64 n = 0;
        if (!COMPACT)
            for (int i = tid; i < a.n_marking; i += kUseThreads) n += a.entries[i];
        for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
        if (lane == 0) s_entries[wave] = n;
        __syncthreads();
        if (tid == 0) sum_use<COMPACT>(a, t, s_entries[0] + s_entries[1] + s_entries[2] + s_entries[3]);
    }
    if (COMPACT && blk == 0 && tid == 0) a.sums[n_blocks] = t.listed;
}
// the page that holds page p's contents after the moves
__device__ __forceinline__ int moved(const UseArgs& a, int p, u32 bits, int before, int listed) {
    if (p < listed) return p;
    const int j = listed - 1 - (before + __popc(bits & ((1u << (p & 31)) - 1)));
    return j < a.cap ? a.copy_to[j] : p;
}
// A wave a sequence: an entry read, its page's bits and sum, for one that moves the move, and the entry written; bound by these dependent reads.
__global__ __launch_bounds__(kUseThreads) void k_use_rewrite(UseArgs a, int n_blocks) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.x * (kUseThreads / 64) + wave;
    if (b >= a.batch) return;
    const int listed = a.sums[n_blocks], to = min(row_pages(a, b), (int)min((int64_t)(blockIdx.y + 1) * kMarkCols, (int64_t)a.max_pages));
    const size_t row = (size_t)b * a.max_pages;
    constexpr int AHEAD = 4;
    for (int c = blockIdx.y * kMarkCols + lane; c < to; c += 64 * AHEAD) {
        int p[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) p[j] = c + 64 * j < to ? a.table[row + c + 64 * j] : -1;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (c + 64 * j >= to) continue;
            const bool known = p[j] >= listed && p[j] < a.n_pages;
            a.table_out[row + c + 64 * j] = known ? moved(a, p[j], a.bits[p[j] >> 5], a.before[p[j] >> 5], listed) : p[j];
        }
    }
}

// All of it by one workgroup, the bitmap and its running sums in LDS: one launch where there is little to read
template <bool COMPACT>
__global__ __launch_bounds__(kSmallThreads) void k_use_small(UseArgs a) {
    extern __shared__ u32 s_bits[];                         // n_words, then their running sums
    u32* const s_before = s_bits + a.n_words;
    __shared__ int s_wave[16], s_count[16];
    constexpr int kWaves = kSmallThreads / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int w = tid; w < a.n_words; w += kSmallThreads) s_bits[w] = 0;
    __syncthreads();
    int n = 0;
    for (int b = wave; b < a.batch; b += kWaves) {
        const int to = row_pages(a, b);
        const int32_t* const row = a.table + (size_t)b * a.max_pages;
#pragma unroll 4
        for (int c = lane; c < to; c += 64) {
            const int p = row[c];
            if (p < 0 || p >= a.n_pages) continue;
            ++n;
            atomicOr(&s_bits[p >> 5], 1u << (p & 31));
        }
    }
    n = wave_sum32(n);
    if (lane == 0) s_count[wave] = n;
    __syncthreads();
    // running sums: a wave a run of words
    const int per = ((a.n_words + kWaves - 1) / kWaves + 63) / 64 * 64, w0 = min(wave * per, a.n_words), w1 = min(w0 + per, a.n_words);
    int at = 0;
    for (int w = w0; w < w1; w += 64) {
        const int own = w + lane < w1 ? __popc(s_bits[w + lane]) : 0;
        int up = own;
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(up, o);
            if (lane >= o) up += v;
        }
        if (w + lane < w1) s_before[w + lane] = at + up - own;
        at += __shfl(up, 63);
    }
    if (lane == 0) s_wave[wave] = at;
    __syncthreads();
    Totals t{0, 0};
    int before = 0;
    u64 entries = 0;
    for (int i = 0; i < kWaves; ++i) {
        before += i < wave ? s_wave[i] : 0;
        t.listed += s_wave[i];
        entries += (u64)s_count[i];
    }
    for (int w = w0 + lane; w < w1; w += 64) s_before[w] += before;
    __syncthreads();
    if (COMPACT) {
        const int w = t.listed >> 5;
        t.moves = w < a.n_words ? t.listed - (int)s_before[w] - __popc(s_bits[w] & ((1u << (t.listed & 31)) - 1)) : 0;
    }
    for (int w = 2 * wave; w < a.n_words; w += 2 * kWaves) {
        const int of = w + (lane >> 5);
        if (of < a.n_words) place_page<COMPACT>(a, t, of, s_bits[of], (int)s_before[of], lane);
    }
    pad<COMPACT>(a, t, tid, kSmallThreads);
    if (tid == 0) sum_use<COMPACT>(a, t, entries);
    if (!COMPACT) return;
    __threadfence_block();
    __syncthreads();                                        // (copy_to is read again)
    for (int b = wave; b < a.batch; b += kWaves) {
        const int to = row_pages(a, b);
        const size_t row = (size_t)b * a.max_pages;
#pragma unroll 4
        for (int c = lane; c < to; c += 64) {
            const int p = a.table[row + c];
            a.table_out[row + c] = p >= t.listed && p < a.n_pages ? moved(a, p, s_bits[p >> 5], (int)s_before[p >> 5], t.listed) : p;
        }
    }
}

// the workspace: entries, marks, bits, running sums, sums of blocks and how many are listed
int words_of(int n_pages) { return (n_pages - 1) / 32 + 1; }
size_t mark_bytes(int n_words) { return (size_t)((n_words + 1) / 2) * 64; }
int blocks_of(int n_words) { return (n_words - 1) / kBlockWords + 1; }
// Up to these bounds one workgroup does it all.  That | the four launches, us, free (compact): 64 sequences of 64 pages 5.3 | 12.7 (7.8 | 17.7); of 256 9.9 | 13.7 (17.7 | 20.1), in a
// pool of 32768 11.0 | 13.5 (20.1 | 20.5), of 65536 15.6 | 13.3 (29.5 | 20.9); 256 sequences of 64 12.4 | 13.7 (23.0 | 18.6); 64 of 680 20.6 | 14.4 (41.4 | 25.0).
constexpr int kSmallWords = 1024, kSmallBatch = 64, kSmallEntries = 1 << 14;

struct Array { const char* name; const int32_t* at; int64_t n; };
bool apart(const Array& x, const Array& y) {
    return !x.at || !y.at || x.n == 0 || y.n == 0 || (uintptr_t)(x.at + x.n) <= (uintptr_t)y.at || (uintptr_t)(y.at + y.n) <= (uintptr_t)x.at;
}

template <bool COMPACT>
tasc_status enqueue_use(const char* who, UseArgs a, void* workspace, size_t ws_bytes, hipStream_t st) {
    a.n_words = words_of(a.n_pages);
    const int n_blocks = blocks_of(a.n_words);
    const size_t need = tasc_pages_workspace_bytes(a.n_pages);
    if (!workspace || ws_bytes < need) {
        tasc_set_error("%s: workspace of %zu of %zu bytes", who, workspace ? ws_bytes : 0, need);
        return TASC_ENOMEM;
    }
    TASC_REQUIRE(((uintptr_t)workspace & 15) == 0, "%s: the workspace must be 16-byte aligned", who);
    if (a.n_words <= kSmallWords && a.batch <= kSmallBatch && (int64_t)a.batch * a.max_pages <= kSmallEntries) {
        k_use_small<COMPACT><<<dim3(1), dim3(kSmallThreads), (size_t)a.n_words * 8, st>>>(a);
        TASC_LAUNCH_CHECK();
        return TASC_OK;
    }
    a.entries = (u64*)workspace;
    a.marks = (uint8_t*)(a.entries + kMarkBlocks);
    a.bits = (u32*)(a.marks + mark_bytes(a.n_words));
    a.before = a.bits + a.n_words;
    a.sums = a.before + a.n_words;
    const int col_runs = (a.max_pages - 1) / kMarkCols + 1;
    const int64_t items = (int64_t)a.batch * col_runs;
    a.n_marking = (int)std::min<int64_t>((items + kUseThreads / 64 - 1) / (kUseThreads / 64), kMarkBlocks / kMarkShares) * kMarkShares;
    const dim3 threads(kUseThreads), rows((unsigned)((a.batch + kUseThreads / 64 - 1) / (kUseThreads / 64)), (unsigned)col_runs);
    k_use_clear<<<dim3((unsigned)std::min((a.n_words / 2 * 4 + kUseThreads) / kUseThreads, 4096)), threads, 0, st>>>(a);
    k_use_mark<<<dim3((unsigned)a.n_marking), threads, 0, st>>>(a, col_runs, items);
    k_use_count<<<dim3((unsigned)n_blocks), threads, 0, st>>>(a);
    k_use_list<COMPACT><<<dim3((unsigned)n_blocks), threads, 0, st>>>(a);
    if (COMPACT) k_use_rewrite<<<rows, threads, 0, st>>>(a, n_blocks);
    TASC_LAUNCH_CHECK();
    return TASC_OK;
}

tasc_status check_tables(const char* who, const int32_t* table, const int32_t* pages, int32_t batch, int32_t max_pages, int32_t n_pages) {
    TASC_REQUIRE(table && pages, "%s: null argument", who);
    TASC_REQUIRE(batch >= 1 && batch <= 1 << 20, "%s: batch %d outside [1, 2^20]", who, batch);
    TASC_REQUIRE(max_pages >= 1 && max_pages < kPageLimit, "%s: max_pages %d outside [1, 2^27)", who, max_pages);
    TASC_REQUIRE(n_pages >= 1 && n_pages < kPageLimit, "%s: n_pages %d outside [1, 2^27)", who, n_pages);
    return TASC_OK;
}

}  // namespace

extern "C" tasc_status tasc_pages_fork(const int32_t* src, const int32_t* dst, int32_t n, const int32_t* new_pages, int32_t* kv_len, int32_t* table, int32_t* pages,
                                       int32_t batch, int32_t max_pages, int32_t* copy_from, int32_t* copy_to, int32_t* summary, void* stream) {
    TASC_REQUIRE(n >= 0 && n <= 1 << 14, "pages_fork: %d pairs outside [0, 2^14]", n);
    TASC_REQUIRE(kv_len && table && pages && (n == 0 || (src && dst && copy_from && copy_to)), "pages_fork: null argument");
    TASC_REQUIRE(batch >= 1 && batch <= 1 << 20, "pages_fork: batch %d outside [1, 2^20]", batch);
    TASC_REQUIRE(max_pages >= 1 && max_pages < kPageLimit, "pages_fork: max_pages %d outside [1, 2^27)", max_pages);
    const Array read[] = {{"src", src, n}, {"dst", dst, n}, {"new_pages", new_pages, n}};
    const Array written[] = {{"kv_len", kv_len, batch}, {"table", table, (int64_t)batch * max_pages}, {"pages", pages, batch}, {"copy_from", copy_from, n},
                             {"copy_to", copy_to, n}, {"summary", summary, 3}};
    for (const Array& w : written) {
        for (const Array& r : read) TASC_REQUIRE(apart(w, r), "pages_fork: %s and %s overlap", w.name, r.name);
        for (const Array* v = written; v != &w; ++v) TASC_REQUIRE(apart(w, *v), "pages_fork: %s and %s overlap", w.name, v->name);
    }
    if (n == 0 && !summary) return TASC_OK;
    const ForkArgs a{src, dst, new_pages, kv_len, table, pages, copy_from, copy_to, summary, n, batch, max_pages};
    const bool at_once = n <= kForkThreads;
    k_pages_fork<<<dim3((unsigned)(n + (summary && at_once ? 1 : 0))), dim3(kForkThreads), 0, (hipStream_t)stream>>>(a);
    if (summary && !at_once) k_pages_fork_sum<<<dim3(1), dim3(kForkThreads), 0, (hipStream_t)stream>>>(copy_to, n, summary);
    TASC_LAUNCH_CHECK();
    return TASC_OK;
}

extern "C" tasc_status tasc_pages_copy(void* pool, size_t page_bytes, int32_t n_pages, int32_t n_layers, size_t layer_stride, const int32_t* copy_from,
                                       const int32_t* copy_to, int32_t n, void* stream) {
    TASC_REQUIRE(n >= 0 && n_layers >= 0, "pages_copy: %d copies in %d layers", n, n_layers);
    if (n == 0 || n_layers == 0) return TASC_OK;
    TASC_REQUIRE(pool && copy_from && copy_to, "pages_copy: null argument");
    TASC_REQUIRE(n_pages >= 1 && n_pages < kPageLimit, "pages_copy: n_pages %d outside [1, 2^27)", n_pages);
    TASC_REQUIRE(page_bytes >= 16 && page_bytes % 16 == 0 && page_bytes <= (size_t)1 << 30, "pages_copy: pages of %zu bytes are not a multiple of 16 up to 2^30", page_bytes);
    TASC_REQUIRE(layer_stride % 16 == 0 && (n_layers == 1 || layer_stride / page_bytes >= (size_t)n_pages), "pages_copy: layers of %d pages of %zu bytes lie %zu bytes apart",
                 n_pages, page_bytes, layer_stride);
    TASC_REQUIRE(((uintptr_t)pool & 15) == 0, "pages_copy: the pool must be 16-byte aligned");
    const int words = (int)(page_bytes / 16), pieces = (words + 64 * kCopyAhead - 1) / (64 * kCopyAhead), quads = (words + pieces - 1) / pieces;
    const int64_t items = (int64_t)n * n_layers * pieces;
    const CopyArgs a{(char*)pool, copy_from, copy_to, page_bytes, layer_stride, items, n, n_pages, pieces, quads};
    const unsigned blocks = (unsigned)std::min<int64_t>((items + 3) / 4, 16384);
    k_pages_copy<<<dim3(blocks), dim3(kCopyThreads), 0, (hipStream_t)stream>>>(a);
    TASC_LAUNCH_CHECK();
    return TASC_OK;
}

extern "C" size_t tasc_pages_workspace_bytes(int32_t n_pages) {
    if (n_pages < 1 || n_pages >= kPageLimit) return 0;
    const int words = words_of(n_pages);
    return kMarkBlocks * sizeof(u64) + mark_bytes(words) + ((size_t)words * 2 + blocks_of(words) + 1) * 4;
}

extern "C" tasc_status tasc_pages_free(const int32_t* table, const int32_t* pages, int32_t batch, int32_t max_pages, int32_t n_pages, int32_t* free_pages,
                                       int32_t* summary, void* workspace, size_t ws_bytes, void* stream) {
    const tasc_status rc = check_tables("pages_free", table, pages, batch, max_pages, n_pages);
    if (rc != TASC_OK) return rc;
    TASC_REQUIRE(free_pages, "pages_free: null argument");
    const Array read[] = {{"table", table, (int64_t)batch * max_pages}, {"pages", pages, batch}};
    const Array written[] = {{"free_pages", free_pages, n_pages}, {"summary", summary, 3}, {"workspace", (const int32_t*)workspace, (int64_t)(ws_bytes / 4)}};
    for (const Array& w : written) {
        for (const Array& r : read) TASC_REQUIRE(apart(w, r), "pages_free: %s and %s overlap", w.name, r.name);
        for (const Array* v = written; v != &w; ++v) TASC_REQUIRE(apart(w, *v), "pages_free: %s and %s overlap", w.name, v->name);
    }
    UseArgs a{};
    a.table = table;
    a.pages = pages;
    a.batch = batch;
    a.max_pages = max_pages;
    a.n_pages = n_pages;
    a.free_pages = free_pages;
    a.summary = summary;
    return enqueue_use<false>("pages_free", a, workspace, ws_bytes, (hipStream_t)stream);
}

extern "C" tasc_status tasc_pages_compact(const int32_t* table, const int32_t* pages, int32_t batch, int32_t max_pages, int32_t n_pages, int32_t* table_out,
                                          int32_t* copy_from, int32_t* copy_to, int32_t max_moves, int32_t* summary, void* workspace, size_t ws_bytes, void* stream) {
    const tasc_status rc = check_tables("pages_compact", table, pages, batch, max_pages, n_pages);
    if (rc != TASC_OK) return rc;
    TASC_REQUIRE(max_moves >= 0 && max_moves < kPageLimit, "pages_compact: max_moves %d outside [0, 2^27)", max_moves);
    TASC_REQUIRE(table_out && (max_moves == 0 || (copy_from && copy_to)), "pages_compact: null argument");
    const Array read[] = {{"table", table, (int64_t)batch * max_pages}, {"pages", pages, batch}};
    const Array written[] = {{"table_out", table_out, (int64_t)batch * max_pages}, {"copy_from", copy_from, max_moves}, {"copy_to", copy_to, max_moves}, {"summary", summary, 3},
                             {"workspace", (const int32_t*)workspace, (int64_t)(ws_bytes / 4)}};
    for (const Array& w : written) {
        for (const Array& r : read) TASC_REQUIRE(apart(w, r) || (w.at == table && table_out == table && w.at == r.at), "pages_compact: %s and %s overlap", w.name, r.name);
        for (const Array* v = written; v != &w; ++v) TASC_REQUIRE(apart(w, *v), "pages_compact: %s and %s overlap", w.name, v->name);
    }
    UseArgs a{};
    a.table = table;
    a.pages = pages;
    a.batch = batch;
    a.max_pages = max_pages;
    a.n_pages = n_pages;
    a.table_out = table_out;
    a.copy_from = copy_from;
    a.copy_to = copy_to;
    a.cap = max_moves;
    a.summary = summary;
    return enqueue_use<true>("pages_compact", a, workspace, ws_bytes, (hipStream_t)stream);
}
