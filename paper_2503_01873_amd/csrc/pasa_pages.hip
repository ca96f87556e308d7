// Pages of a cache: copied, shared between sequences, given out, taken back and packed.  Entry points and kernels.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>
#include <type_traits>

#include "pasa.h"
#include "pasa_cache.h"

namespace {

constexpr int kPlanThreads = 1024;               // of the workgroups that look through holders
constexpr int kEach = 16;                        // holders of a thread at a time
constexpr int kSpan = kPlanThreads * kEach;      // of a workgroup
constexpr int kCopyAtOnce = 2;                   // chunks of a workgroup that are on their way together
constexpr int kCopyGroups = 8192;                // workgroups of a copy whose length only the device knows

// ---- copies ----

// A page is up to five stretches of memory, whole heads behind one another: codes, scales, the mean.  Each is cut into chunks of 4 KiB, 16 bytes a thread, the last of them
// shorter: what a chunk is goes through the scalar unit.  `ends` counts chunks up to and with each stretch, `units` its 16-byte units.
typedef unsigned u4 __attribute__((ext_vector_type(4)));
struct CopyArgs {
    const u4* from[5];
    u4* to[5];
    unsigned ends[5], units[5];
    int pages_from, pages_to;
    FastDiv chunks;                              // of a page
};

CopyArgs copy_args(const pasa_cache& to, const pasa_cache& from)
{
    CopyArgs a = {};
    const unsigned codes = (unsigned)((size_t)from.Hkv * from.page * cache_token_bytes(from) / 16), scales = (unsigned)((size_t)from.Hkv * from.page / 4);
    const unsigned mean = to.kmean != nullptr ? (unsigned)((size_t)from.Hkv * from.d / 4) : 0;
    const unsigned size[5] = {codes, codes, scales, scales, mean};
    const void* of[5] = {from.k, from.v, from.kscale, from.vscale, from.kmean};
    void* at[5] = {to.k, to.v, to.kscale, to.vscale, to.kmean};
    unsigned end = 0;
    for (int i = 0; i < 5; ++i) {
        a.from[i] = static_cast<const u4*>(of[i]);
        a.to[i] = static_cast<u4*>(at[i]);
        a.units[i] = size[i];
        a.ends[i] = end += (size[i] + kCacheThreads - 1) / kCacheThreads;
    }
    a.pages_from = from.pages;
    a.pages_to = to.pages;
    a.chunks = fast_div(end);
    return a;
}

// Chunks first .. first + kCopyAtOnce - 1 of `all`, pair_of giving the pages of a pair (a page outside its pool: nothing to be done).  All loads go out before the first store.
// Stores go past the L2s, which would have to bring what they hold to memory before the kernel ends: half of 8400 pages of 37 KB packed, 82 MB, in 39.2 us with the plan, through them
// 60.5 (one to eight chunks at once 39 to 41.6, 1024 workgroups in place of 8192 44.4).
template <class PairOf>
__device__ inline void copy_chunks(const CopyArgs& a, unsigned first, unsigned all, PairOf pair_of)
{
    u4 x[kCopyAtOnce];
    u4* dst[kCopyAtOnce];
    unsigned size[kCopyAtOnce];
#pragma unroll
    for (int j = 0; j < kCopyAtOnce; ++j) {
        const unsigned chunk = first + j < all ? first + j : all - 1;
        const unsigned pair = a.chunks.quotient(chunk), c = a.chunks.rest(chunk, pair);
        int from, to;
        pair_of(pair, from, to);
        const bool in = from >= 0 && from < a.pages_from && to >= 0 && to < a.pages_to;
        int i = 0;
        while (i < 4 && c >= a.ends[i]) ++i;
        const unsigned units = a.units[i], at = (c - (i > 0 ? a.ends[i - 1] : 0u)) * kCacheThreads;
        const unsigned left = units - at < kCacheThreads ? units - at : kCacheThreads;
        const unsigned mine = at + (threadIdx.x < left ? threadIdx.x : left - 1);
        x[j] = a.from[i][(size_t)(unsigned)(in ? from : 0) * units + mine];
        dst[j] = a.to[i] + (size_t)(unsigned)(in ? to : 0) * units + mine;
        size[j] = in && first + j < all ? left : 0u;
    }
#pragma unroll
    for (int j = 0; j < kCopyAtOnce; ++j)
        if (threadIdx.x < size[j]) __builtin_nontemporal_store(x[j], dst[j]);
}

// Pairs of two lists
__global__ __launch_bounds__(kCacheThreads)
void pasa_copy_pages_k(CopyArgs a, const int* __restrict__ from_pages, const int* __restrict__ to_pages, unsigned all)
{
    copy_chunks(a, blockIdx.x * kCopyAtOnce, all, [&](unsigned pair, int& from, int& to) { from = from_pages[pair], to = to_pages[pair]; });
}

// ---- sequences go on as others ----

struct Tables {
    int* table;
    int* length;
    int* refs;
    int S, width, pages, page_log2, page;
};
Tables tables_of(const pasa_cache& c, int* refs)
{
    return {const_cast<int*>(c.table), const_cast<int*>(c.length), refs, c.S, c.table_width, c.pages, log2_of(c.page), c.page};
}
__device__ inline bool in_pool(const Tables& t, int page) { return page >= 0 && page < t.pages; }
__device__ inline int length_of(const Tables& t, int b) { return clamp_int(t.length[b], 0, t.width << t.page_log2); }

// What a workgroup's threads have read, written and counted in memory is done before any of them goes on.
__device__ inline void memory_barrier()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// What sequences that go on as others will hold, beside the tables; they let go of what they hold.
__global__ __launch_bounds__(kCacheThreads)
void pasa_fork_out_k(Tables t, const int* __restrict__ source, int* __restrict__ table_next, int* __restrict__ length_next, FastDiv chunks)
{
    const int b = (int)chunks.quotient(blockIdx.x), p = (int)chunks.rest(blockIdx.x, (unsigned)b) * kCacheThreads + (int)threadIdx.x;
    const int from = source[b];
    if (from == b || p >= t.width) return;
    const bool ends = from < 0 || from >= t.S;
    const int length = ends ? 0 : length_of(t, from), places = (length + t.page - 1) >> t.page_log2;
    const size_t at = (size_t)b * t.width + p;
    const int old = t.table[at];
    table_next[at] = p < places ? t.table[(size_t)from * t.width + p] : -1;
    if (p == 0) length_next[b] = length;
    if (in_pool(t, old)) atomicSub(t.refs + old, 1);
}

__global__ __launch_bounds__(kCacheThreads)
void pasa_fork_in_k(Tables t, const int* __restrict__ source, const int* __restrict__ table_next, const int* __restrict__ length_next, FastDiv chunks)
{
    const int b = (int)chunks.quotient(blockIdx.x), p = (int)chunks.rest(blockIdx.x, (unsigned)b) * kCacheThreads + (int)threadIdx.x;
    if (source[b] == b || p >= t.width) return;
    const size_t at = (size_t)b * t.width + p;
    const int page = table_next[at];
    t.table[at] = page;
    if (p == 0) t.length[b] = length_next[b];
    if (in_pool(t, page)) atomicAdd(t.refs + page, 1);
}

// Both in one launch of one workgroup, for tables of few entries: 64 x 65 in 4.9 us (in two launches 2.9 and 2.5, and the host's 3.5 for one more).
constexpr long long kForkEntries = 8 * kPlanThreads;
__global__ __launch_bounds__(kPlanThreads)
void pasa_fork_small_k(Tables t, const int* __restrict__ source, FastDiv width)
{
    constexpr int EACH = (int)(kForkEntries / kPlanThreads);
    const int entries = t.S * t.width;
    int at[EACH], b[EACH], p[EACH], from[EACH], length[EACH], next[EACH], old[EACH];
    // step by step for all of a thread's entries, without branches between: what is not there stands for the last entry
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        at[i] = i * kPlanThreads + (int)threadIdx.x < entries ? i * kPlanThreads + (int)threadIdx.x : entries - 1;
        b[i] = (int)width.quotient((unsigned)at[i]);
        p[i] = (int)width.rest((unsigned)at[i], (unsigned)b[i]);
        from[i] = source[b[i]];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const bool ends = from[i] < 0 || from[i] >= t.S;
        length[i] = length_of(t, ends ? b[i] : from[i]);
        next[i] = t.table[(size_t)(ends ? b[i] : from[i]) * t.width + p[i]];
        old[i] = t.table[at[i]];
        if (ends) length[i] = 0;
    }
    memory_barrier();                            // all have read
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (i * kPlanThreads + (int)threadIdx.x >= entries || from[i] == b[i]) continue;
        if (p[i] >= (length[i] + t.page - 1) >> t.page_log2) next[i] = -1;
        t.table[at[i]] = next[i];
        if (p[i] == 0) t.length[b[i]] = length[i];
        if (old[i] == next[i]) continue;
        if (in_pool(t, old[i])) atomicSub(t.refs + old[i], 1);
        if (in_pool(t, next[i])) atomicAdd(t.refs + next[i], 1);
    }
}

// Pages behind the lengths are let go of.
__global__ __launch_bounds__(kCacheThreads)
void pasa_free_k(Tables t, FastDiv chunks)
{
    const int b = (int)chunks.quotient(blockIdx.x), p = (int)chunks.rest(blockIdx.x, (unsigned)b) * kCacheThreads + (int)threadIdx.x;
    if (p >= t.width || p < (length_of(t, b) + t.page - 1) >> t.page_log2) return;
    const size_t at = (size_t)b * t.width + p;
    const int old = t.table[at];
    t.table[at] = -1;
    if (in_pool(t, old)) atomicSub(t.refs + old, 1);
}

// ---- room for rows ----

// Bit i: whether page p + i is in use
__device__ inline unsigned in_use(const Tables& t, int p)
{
    unsigned live = 0;
#pragma unroll
    for (int i = 0; i < kEach / 4; ++i) {
        int4 x = make_int4(0, 0, 0, 0);
        if (p + 4 * i + 3 < t.pages) {
            x = *reinterpret_cast<const int4*>(t.refs + p + 4 * i);
        } else {
            if (p + 4 * i < t.pages) x.x = t.refs[p + 4 * i];
            if (p + 4 * i + 1 < t.pages) x.y = t.refs[p + 4 * i + 1];
            if (p + 4 * i + 2 < t.pages) x.z = t.refs[p + 4 * i + 2];
        }
        live |= (unsigned)((x.x != 0) | (x.y != 0) << 1 | (x.z != 0) << 2 | (x.w != 0) << 3) << (4 * i);
    }
    return live;
}

// Sum over the threads of a workgroup before one's own, and over all
template <int NT>
__device__ inline unsigned scan_workgroup(unsigned x, unsigned* sums, unsigned& all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned upto = scan64(x);
    __syncthreads();                             // the sums of the last time are read
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    unsigned before = upto - x;
    all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        if (w < wave) before += sums[w];
        all += sums[w];
    }
    return before;
}

__device__ inline int holders(const int* refs, int page) { return __hip_atomic_load(refs + page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// One workgroup.  The places that rows are written to are gone through in order of sequences: a place without a page takes a free one, and so does one whose page
// others hold too, unless they all are written to here as well and this is the last.  Who holds a page shows in its count: all places here let go first; what is
// left above 0 belongs to others; otherwise the places take the number of their sequence down to the last one's, which keeps the page.
// Free pages are looked for from the first on, 16384 at a time, and only as many as are needed: most steps need none and end before that.
struct RoomArgs {
    Tables t;
    const int* row_start;
    int* lacking;
    int* begin;                                  // [S + 1] places before each sequence's
    int* copies;                                 // [2][S] page to be copied and where to, or -1
    int* free_pages;                             // [most_free]
    int R, most_free;
};
// In most steps nobody needs a page: every place has one, whose count was 1 when it was let go of.  That is known after one trip to the counts.
// What bounds it: one trip to memory after the other.  16 sequences, none of which needs a page, 4.0 us; 64, of which 24 take one, 8.4, and 3.0 for the copies of 24 pages of 37 KB.
// Where no page is copied the workgroups of the copies still begin, read the first page and end: 16 sequences of pages of 37 KB 2.3 us, 256 of 74 KB 3.8, 256 of 270 KB 8.8.
__global__ __launch_bounds__(kPlanThreads)
void pasa_room_k(RoomArgs a)
{
    constexpr int NT = kPlanThreads;
    __shared__ unsigned sums[NT / 64];
    __shared__ int lds_begin[NT + 1], lds_first[NT], lds_free[NT];
    const int tid = threadIdx.x;
    const Tables& t = a.t;
    const int most = t.width << t.page_log2;
    const bool in_lds = t.S <= NT;               // what is kept of the sequences; otherwise in the workspace, and read again
    auto first_token = [&](const Sequence& s) { return s.length > s.rows ? s.length - s.rows : 0; };

    unsigned total = 0;
    for (int b0 = 0; b0 < t.S; b0 += NT) {
        const int b = b0 + tid;
        unsigned places = 0;
        int first = 0;
        if (b < t.S) {
            const Sequence s = sequence_at(t.length, a.row_start, b, a.R, most);
            first = first_token(s);
            if (s.rows > 0 && s.length > 0) places = (unsigned)(((s.length - 1) >> t.page_log2) - (first >> t.page_log2) + 1);
            a.copies[b] = -1;
        }
        unsigned all;
        const unsigned before = scan_workgroup<NT>(places, sums, all);
        if (in_lds) {
            if (b < t.S) lds_begin[b] = (int)before, lds_first[b] = first;
        } else if (b < t.S) {
            a.begin[b] = (int)(total + before);
        }
        total += all;
    }
    if (tid == 0) {
        if (in_lds) lds_begin[t.S] = (int)total;
        else a.begin[t.S] = (int)total;
    }
    memory_barrier();

    struct Place {
        int b, first;                            // sequence, its first new token
        size_t at;                               // in the table
        int place, page;                         // the page that is there, or -1
    };
    auto place_of = [&](unsigned i) {
        auto begin = [&](int b) { return in_lds ? lds_begin[b] : a.begin[b]; };
        int low = 0, high = t.S;                 // the last sequence whose places begin at i or before, and that has some
        while (high - low > 1) {
            const int middle = (low + high) / 2;
            if ((unsigned)begin(middle) <= i) low = middle;
            else high = middle;
        }
        Place p;
        p.b = low;
        p.first = in_lds ? lds_first[low] : first_token(sequence_at(t.length, a.row_start, low, a.R, most));
        p.place = clamp_int((p.first >> t.page_log2) + (int)(i - (unsigned)begin(low)), 0, t.width - 1);
        p.at = (size_t)low * t.width + p.place;
        const int page = t.table[p.at];
        p.page = in_pool(t, page) ? page : -1;
        return p;
    };
    const bool few = total <= NT;                // a place a thread, looked up once
    Place mine = {};
    if (few && (unsigned)tid < total) mine = place_of(tid);
    auto place_at = [&](unsigned i) { return few ? mine : place_of(i); };

    bool alone = true;
    for (unsigned i = tid; i < total; i += NT) {
        const Place p = place_at(i);
        if (p.page < 0 || atomicSub(t.refs + p.page, 1) != 1) alone = false;
    }
    // what was returned has arrived, so all of them have let go
    if (__syncthreads_and(alone)) {
        for (unsigned i = tid; i < total; i += NT) t.refs[place_at(i).page] = 1;
        if (tid == 0 && a.lacking != nullptr) *a.lacking = 0;
        return;
    }
    for (unsigned i = tid; i < total; i += NT) {
        const Place p = place_at(i);
        if (p.page >= 0 && holders(t.refs, p.page) <= 0) atomicMin(t.refs + p.page, -(p.b + 1));
    }
    memory_barrier();
    auto needs = [&](const Place& p) { return p.page < 0 || holders(t.refs, p.page) != -(p.b + 1); };
    bool my_need = false;                        // where there are few: looked up once, before anything is written
    if (few && (unsigned)tid < total) my_need = needs(mine);
    unsigned wanted = 0, my_rank = 0;
    for (unsigned i0 = 0; i0 < total; i0 += NT) {
        const unsigned i = i0 + tid;
        unsigned all;
        my_rank = scan_workgroup<NT>(i < total && (few ? my_need : needs(place_at(i))) ? 1u : 0u, sums, all);
        wanted += all;
    }
    unsigned found = 0;
    const unsigned enough = wanted < (unsigned)a.most_free ? wanted : (unsigned)a.most_free;
    const bool list_in_lds = enough <= NT;
    for (int p0 = 0; p0 < t.pages && found < enough; p0 += kSpan) {
        const int p = p0 + tid * kEach;
        const int there = t.pages - p < kEach ? t.pages - p : kEach;             // pages of this thread
        unsigned free = there > 0 ? ~in_use(t, p) & ((1u << there) - 1u) : 0u;
        unsigned all, rank = found + scan_workgroup<NT>((unsigned)__builtin_popcount(free), sums, all);
        for (; free != 0 && rank < enough; free &= free - 1, ++rank) {
            if (list_in_lds) lds_free[rank] = p + __builtin_ctz(free);
            else a.free_pages[rank] = p + __builtin_ctz(free);
        }
        found += all;
    }
    if (found > enough) found = enough;
    if (list_in_lds) __syncthreads();
    else memory_barrier();
    unsigned given = 0;
    for (unsigned i0 = 0; i0 < total; i0 += NT) {
        const unsigned i = i0 + tid;
        Place p = {};
        bool need = false;
        if (i < total) {
            p = place_at(i);
            need = few ? my_need : needs(p);
        }
        unsigned all = 0;
        const unsigned rank = few ? my_rank : given + scan_workgroup<NT>(need ? 1u : 0u, sums, all);
        given += all;
        if (i >= total) continue;
        if (!need) {
            t.refs[p.page] = 1;                  // all others have let go
            continue;
        }
        const int fresh = rank < found ? (list_in_lds ? lds_free[rank] : a.free_pages[rank]) : -1;
        t.table[p.at] = fresh;
        if (fresh < 0) continue;
        t.refs[fresh] = 1;
        if (p.page >= 0 && p.place << t.page_log2 < p.first) {       // older tokens are in it: the sequence's first place
            a.copies[p.b] = p.page;
            a.copies[t.S + p.b] = fresh;
        }
    }
    if (tid == 0 && a.lacking != nullptr) *a.lacking = (int)(wanted - found);
}

// ---- a pool is packed ----

struct PackArgs {
    Tables t;
    int* used;
    int* counts;                                 // of the workgroups
    int* header;                                 // pages in use, pages that move
    int* to;                                     // [pages / 2 + 1] free pages below the number of those in use, ascending
    int* from;                                   // pages in use from that number on, ascending
    int* rank;                                   // [pages] which of those a page is, or -1
    int groups;
};

__global__ __launch_bounds__(kPlanThreads)
void pasa_pack_count_k(PackArgs a)
{
    __shared__ unsigned sums[kPlanThreads / 64];
    unsigned all;
    scan_workgroup<kPlanThreads>((unsigned)__builtin_popcount(in_use(a.t, (int)blockIdx.x * kSpan + (int)threadIdx.x * kEach)), sums, all);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = (int)all;
}

// With n pages in use, the k-th free one below n takes the k-th used one from n on.  A workgroup has 16384 pages (8400 in 6.4 us).
__global__ __launch_bounds__(kPlanThreads)
void pasa_pack_plan_k(PackArgs a)
{
    constexpr int NT = kPlanThreads;
    __shared__ unsigned sums[NT / 64];
    const int tid = threadIdx.x, g = (int)blockIdx.x;
    const int p = g * kSpan + tid * kEach;
    const unsigned live = in_use(a.t, p);
    unsigned here;
    unsigned before = scan_workgroup<NT>((unsigned)__builtin_popcount(live), sums, here);
    unsigned n = here, others = 0;               // pages in use: of all, of the workgroups before
    if (a.groups > 1) {
        unsigned all = 0, first = 0;
        for (int i = tid; i < a.groups; i += NT) {
            const unsigned c = (unsigned)a.counts[i];
            all += c;
            if (i < g) first += c;
        }
        scan_workgroup<NT>(all, sums, n);
        scan_workgroup<NT>(first, sums, others);
    }
    before += others;
    // of the pages below n those in use: in the workgroup that n lies in, and those before
    const int at_n = n > 0 ? (int)((n - 1) / kSpan) : 0, q = at_n * kSpan + tid * kEach;
    unsigned below = q == p ? live : q < (int)n ? in_use(a.t, q) : 0u;
    if (q >= (int)n) below = 0u;
    if ((int)n - q < kEach && q < (int)n) below &= (1u << ((int)n - q)) - 1u;
    unsigned stay;
    scan_workgroup<NT>((unsigned)__builtin_popcount(below), sums, stay);
    if (a.groups > 1) {
        unsigned first = 0, all;
        for (int i = tid; i < at_n && i < a.groups; i += NT) first += (unsigned)a.counts[i];
        scan_workgroup<NT>(first, sums, all);
        stay += all;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int page = p + i;
        if (page >= a.t.pages) break;
        const bool lives = (live >> i & 1u) != 0u;
        if (page < (int)n) {
            if (!lives) a.to[page - (int)before] = page;
        } else {
            a.rank[page] = lives ? (int)(before - stay) : -1;
            if (lives) a.from[before - stay] = page;
        }
        before += lives;
    }
    if (g == 0 && tid == 0) {
        a.header[0] = (int)n;
        a.header[1] = (int)(n - stay);
        if (a.used != nullptr) *a.used = (int)n;
    }
}

// The first workgroups: table entries and holders.  The others: contents.
__global__ __launch_bounds__(kCacheThreads)
void pasa_pack_move_k(PackArgs a, CopyArgs c, unsigned entry_groups)
{
    const int n = a.header[0], moved = a.header[1];
    if (blockIdx.x < entry_groups) {
        const size_t at = (size_t)blockIdx.x * kCacheThreads + threadIdx.x;
        if (at < (size_t)a.t.S * a.t.width) {
            const int page = a.t.table[at];
            if (page >= n && page < a.t.pages) {
                const int k = a.rank[page];
                if (k >= 0) a.t.table[at] = a.to[k];
            }
        }
        for (size_t k = at; k < (size_t)moved; k += (size_t)entry_groups * kCacheThreads) {
            const int of = a.from[k];
            a.t.refs[a.to[k]] = a.t.refs[of];
            a.t.refs[of] = 0;
        }
        return;
    }
    const unsigned all = (unsigned)moved * c.chunks.d;
    for (unsigned i = (blockIdx.x - entry_groups) * kCopyAtOnce; i < all; i += kCopyGroups * kCopyAtOnce)
        copy_chunks(c, i, all, [&](unsigned pair, int& from, int& to) { from = a.from[pair], to = a.to[pair]; });
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool buffer(const void* p, uintptr_t a) { return p != nullptr && aligned(p, a); }
size_t rounded_up(size_t bytes) { return (bytes + 255) / 256 * 256; }
int check_workspace(const void* ws, size_t bytes, size_t need) { return buffer(ws, 256) && bytes >= need ? PASA_OK : PASA_EWORKSPACE; }
int launched() { return hipGetLastError() == hipSuccess ? PASA_OK : PASA_ELAUNCH; }

constexpr long long kMaxThreads = 0xffffffff;    // of a launch: the hardware counts them in 32 bits
constexpr int kMaxPages = 1 << 30;               // page numbers and those of a workgroup behind them fit 31 bits
// Workgroups of a copy by lists, and whether a launch has as many
long long copy_grid(long long chunks) { return (chunks + kCopyAtOnce - 1) / kCopyAtOnce; }
bool copy_fits(long long chunks) { return copy_grid(chunks) <= kMaxThreads / kCacheThreads; }
// units of a page are counted in 32 bits
bool page_fits(const pasa_cache& c) { return (long long)c.Hkv * c.page * c.d <= 1LL << 30 && c.pages <= kMaxPages; }
unsigned entry_chunks(const pasa_cache& c) { return (unsigned)((c.table_width + kCacheThreads - 1) / kCacheThreads); }

// The description and the holders of its pages
int check(const pasa_cache* cache, const int* refs)
{
    const int st = pasa_check_cache(cache);
    if (st != PASA_OK) return st;
    if (!buffer(refs, 16)) return PASA_EINVAL;
    if (((long long)cache->table_width + kCacheThreads) * cache->S > kMaxThreads / 2 || !page_fits(*cache)) return PASA_EUNSUPPORTED;
    return PASA_OK;
}

long long most_places(const pasa_cache& c, int R)
{
    const long long places = (long long)R / c.page + 2LL * c.S;      // a sequence of n rows is written to in (n - 1) / page + 2 places at most, and in n at most
    return places < R ? places : R;
}
int most_free(const pasa_cache& c, int R) { return (int)(most_places(c, R) < c.pages ? most_places(c, R) : c.pages); }
size_t fork_bytes(const pasa_cache& c) { return rounded_up(((size_t)c.S * c.table_width + c.S) * 4); }
size_t room_bytes(const pasa_cache& c, int R) { return rounded_up(((size_t)3 * c.S + 1 + most_free(c, R)) * 4); }
int pack_groups(const pasa_cache& c) { return (int)(((long long)c.pages + kSpan - 1) / kSpan); }
size_t pack_bytes(const pasa_cache& c) { return rounded_up(((size_t)pack_groups(c) + 2 + 2 * ((size_t)c.pages / 2 + 1) + c.pages) * 4); }

}  // namespace

extern "C" {

int pasa_cache_copy(const pasa_cache* to, const pasa_cache* from, const int* to_pages, const int* from_pages, int n, void* stream)
{
    int st = pasa_check_cache(to);
    if (st != PASA_OK) return st;
    st = pasa_check_cache(from);
    if (st != PASA_OK) return st;
    if (!buffer(to_pages, 4) || !buffer(from_pages, 4) || n <= 0) return PASA_EINVAL;
    if (to->Hkv != from->Hkv || to->d != from->d || to->page != from->page || to->format != from->format) return PASA_EINVAL;
    if (to->kmean != nullptr && from->kmean == nullptr) return PASA_EINVAL;
    if ((to->kshift != nullptr) != (from->kshift != nullptr)) return PASA_EINVAL;            // held keys would stand for others
    if (!page_fits(*to) || !page_fits(*from)) return PASA_EUNSUPPORTED;
    const CopyArgs a = copy_args(*to, *from);
    const long long all = (long long)n * a.chunks.d;
    if (!copy_fits(all)) return PASA_EUNSUPPORTED;
    pasa_copy_pages_k<<<(unsigned)copy_grid(all), kCacheThreads, 0, static_cast<hipStream_t>(stream)>>>(a, from_pages, to_pages, (unsigned)all);
    return launched();
}

size_t pasa_cache_fork_workspace(const pasa_cache* cache) { return pasa_check_cache(cache) == PASA_OK ? fork_bytes(*cache) : 0; }

int pasa_cache_fork(const pasa_cache* cache, int* refs, const int* source, void* workspace, size_t workspace_bytes, void* stream)
{
    int st = check(cache, refs);
    if (st != PASA_OK) return st;
    if (!buffer(source, 4)) return PASA_EINVAL;
    st = check_workspace(workspace, workspace_bytes, fork_bytes(*cache));
    if (st != PASA_OK) return st;
    const Tables t = tables_of(*cache, refs);
    if ((long long)cache->S * cache->table_width <= kForkEntries) {
        pasa_fork_small_k<<<1, kPlanThreads, 0, static_cast<hipStream_t>(stream)>>>(t, source, fast_div((unsigned)cache->table_width));
        return launched();
    }
    const unsigned chunks = entry_chunks(*cache), grid = chunks * (unsigned)cache->S;
    int* const table_next = static_cast<int*>(workspace);
    int* const length_next = table_next + (size_t)cache->S * cache->table_width;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    pasa_fork_out_k<<<grid, kCacheThreads, 0, s>>>(t, source, table_next, length_next, fast_div(chunks));
    if (hipGetLastError() != hipSuccess) return PASA_ELAUNCH;
    pasa_fork_in_k<<<grid, kCacheThreads, 0, s>>>(t, source, table_next, length_next, fast_div(chunks));
    return launched();
}

int pasa_cache_free(const pasa_cache* cache, int* refs, void* stream)
{
    const int st = check(cache, refs);
    if (st != PASA_OK) return st;
    const unsigned chunks = entry_chunks(*cache);
    pasa_free_k<<<chunks * (unsigned)cache->S, kCacheThreads, 0, static_cast<hipStream_t>(stream)>>>(tables_of(*cache, refs), fast_div(chunks));
    return launched();
}

size_t pasa_cache_room_workspace(const pasa_cache* cache, int R) { return pasa_check_cache(cache) == PASA_OK && R > 0 ? room_bytes(*cache, R) : 0; }

int pasa_cache_room(const pasa_cache* cache, int* refs, int R, const int* row_start, int* lacking, void* workspace, size_t workspace_bytes, void* stream)
{
    int st = check(cache, refs);
    if (st != PASA_OK) return st;
    if (R <= 0 || !buffer(row_start, 4) || !aligned(lacking, 4)) return PASA_EINVAL;
    const CopyArgs c = copy_args(*cache, *cache);
    const long long all = (long long)cache->S * c.chunks.d;
    if (!copy_fits(all)) return PASA_EUNSUPPORTED;
    st = check_workspace(workspace, workspace_bytes, room_bytes(*cache, R));
    if (st != PASA_OK) return st;
    RoomArgs a;
    a.t = tables_of(*cache, refs);
    a.row_start = row_start;
    a.lacking = lacking;
    a.begin = static_cast<int*>(workspace);
    a.copies = a.begin + cache->S + 1;
    a.free_pages = a.copies + 2 * (size_t)cache->S;
    a.R = R;
    a.most_free = most_free(*cache, R);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    pasa_room_k<<<1, kPlanThreads, 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return PASA_ELAUNCH;
    pasa_copy_pages_k<<<(unsigned)copy_grid(all), kCacheThreads, 0, s>>>(c, a.copies, a.copies + cache->S, (unsigned)all);
    return launched();
}

size_t pasa_cache_compact_workspace(const pasa_cache* cache) { return pasa_check_cache(cache) == PASA_OK ? pack_bytes(*cache) : 0; }

int pasa_cache_compact(const pasa_cache* cache, int* refs, int* used, void* workspace, size_t workspace_bytes, void* stream)
{
    int st = check(cache, refs);
    if (st != PASA_OK) return st;
    if (!aligned(used, 4)) return PASA_EINVAL;
    const CopyArgs c = copy_args(*cache, *cache);
    if ((long long)cache->pages / 2 * c.chunks.d > INT_MAX) return PASA_EUNSUPPORTED;        // half of the pages move at most
    st = check_workspace(workspace, workspace_bytes, pack_bytes(*cache));
    if (st != PASA_OK) return st;
    PackArgs a;
    a.t = tables_of(*cache, refs);
    a.used = used;
    a.groups = pack_groups(*cache);
    a.counts = static_cast<int*>(workspace);
    a.header = a.counts + a.groups;
    a.to = a.header + 2;
    a.from = a.to + (size_t)cache->pages / 2 + 1;
    a.rank = a.from + (size_t)cache->pages / 2 + 1;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (a.groups > 1) {
        pasa_pack_count_k<<<(unsigned)a.groups, kPlanThreads, 0, s>>>(a);
        if (hipGetLastError() != hipSuccess) return PASA_ELAUNCH;
    }
    pasa_pack_plan_k<<<(unsigned)a.groups, kPlanThreads, 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return PASA_ELAUNCH;
    const unsigned entry_groups = (unsigned)(((long long)cache->S * cache->table_width + kCacheThreads - 1) / kCacheThreads);
    pasa_pack_move_k<<<entry_groups + kCopyGroups, kCacheThreads, 0, s>>>(a, c, entry_groups);
    return launched();
}

}  // extern "C"
