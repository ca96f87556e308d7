// Attention of a few rows per sequence over the paged 8-bit cache: pasa_cache_rows, and the merge of what its workgroups leave.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "pasa_cache.h"

namespace {

// A row's level is set 2^7 below its largest product of score and scale, and set again when one exceeds it by 2^15: P is 2^7 to 2^15 there, inside fp16, and
// what is 2^-21 of it or more keeps all of fp16's bits (2^-14 with levels at the largest itself; many keys of little weight each are a long row's rule).
constexpr float kBelow = 7.f, kRise = 15.f;
constexpr float kNoLevel = -3.402823466e38f;     // the lowest finite number: a score of -inf against it gives 0 and no NaN, and no finite one lies below it

// The sum of a row's softmax is held times 2^-14.  A weight over a value's scale is up to 2^15 / (2^-100 / 448), and 262144 of them come to 2^142, which fp32
// holds no more; at the other end, P = 2^7 and values of 2^128, it is 2^-128 then, which fp32 still holds.
constexpr int kSumBits = 14;
constexpr float kSum = 1.f / (1 << kSumBits);

// The bytes of two keys' values, two channels a word, as fp16 pairs (key, next key) of one channel; and of a key, as pairs of channels.
// Excess-128 bytes become 1024 + byte by putting 0x64 above them, exactly, and 1152 is taken off, exactly.
template <bool E4M3, bool HIGH>
__device__ inline h2 widen2(unsigned w)
{
    if constexpr (E4M3) {
        return __builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, HIGH));
    } else {
        const unsigned x = __builtin_amdgcn_perm(0x64646464u, w, HIGH ? 0x04030402u : 0x04010400u);
        return __builtin_bit_cast(h2, x) - h2{(_Float16)1152, (_Float16)1152};
    }
}

struct RowsArgs {
    pasa_cache c;
    const unsigned short* q;
    unsigned short* o;
    const int* row_start;
    const unsigned long long* tree;
    const int* blocks;
    MergeRecord* records;
    float* slots;
    long long row_stride;
    float scale2;                                // scale * log2(e)
    int R, Hq, count, io_bf16, page_log2, never_cut;
    FastDiv G;
};

// What the workgroups share out is units of 64 keys, over sequences, KV heads and blocks of rows.  A multiple of what a workgroup sweeps at once:
__device__ inline unsigned whole_units(unsigned units) { return (units + kUnitsAtOnce - 1) / kUnitsAtOnce * kUnitsAtOnce; }

// Keys that a sequence's rows are swept over, in the order of the list where there is one; its units, at least one (rows without keys
// are written too); its blocks of rows
struct Extent {
    int keys, units, row_blocks;
};
template <int ROWS>
__device__ inline Extent extent_of(const RowsArgs& a, const Sequence& s)
{
    Extent x;
    x.keys = s.length;
    if (a.blocks != nullptr) {
        const int pages = (s.length + a.c.page - 1) >> a.page_log2;
        x.keys = (pages < a.count ? pages : a.count) << a.page_log2;
    }
    x.units = (x.keys + kUnit - 1) / kUnit;
    if (x.units < 1) x.units = 1;
    x.row_blocks = (int)(((unsigned)s.rows * a.G.d + ROWS - 1) / ROWS);
    return x;
}

// What a workgroup sweeps first: from `at` on, block of rows `pair` (of all heads) of sequence b, and how far from there on; b < 0: nothing.  Counted in
// units, with `beside` for each block before its first one.
// Then, in groups of `group` wavefronts, whole blocks of rows of short sequences: `shorts` of them in all, dealt to the workgroups in turn (none where
// there are no more blocks than workgroups).
struct Start {
    int b, at, beside;
    unsigned pair, left, per;
    Sequence s;
    unsigned shorts;
    int longest_short, group;
};

// What a workgroup keeps of the sequences for its shorts: each one, and how many blocks of rows of short sequences there are up to and with it.
template <int NT>
struct Known {
    Sequence s[NT];
    unsigned shorts[NT];
};

// What a block of rows costs a workgroup beside its keys (5 us), in units times rows.
constexpr unsigned kBeside = 640;

// units / size, rounded up; both below 2^13, where the quotient with a half added is off by far less than keeps it from the next whole number
__device__ inline unsigned ranges_of(unsigned units, unsigned size)
{
    return (unsigned)(((float)(units + size - 1) + 0.5f) * __builtin_amdgcn_rcpf((float)size));
}

// How the work is shared out.  A block of rows (of a sequence and head) costs a workgroup about 5 us beside its keys: lengths, places, queries, the first keys'
// way from memory, the wavefronts' states brought together.
// - No more blocks than workgroups: each is cut into ranges of `per` units, one a workgroup, with `per` the least of eight sizes
//   that gives no more ranges than workgroups; the largest of the eight always does: the longest sequence, or the share of the workgroups that are
//   left when every block has one range that is not full.
// - More, or where that gives larger ranges than an even share: the units of all, with what a block costs beside them, are one line that is cut evenly, and a
//   workgroup's range may end inside one block and begin inside the next, as often as it has to.  (Trees behind 8 sequences, 204 blocks of 128
//   units at most: ranges of 120 units 59.1 us; the line, an even share of 80, 49.8; 65.4 where it does not count what blocks cost beside their units.)
//   Short sequences, which would leave wavefronts idle, stay out of the line: groups of 1, 2, 4 or 8 wavefronts, as many as there are for each, take
//   their blocks whole, in 5 us and 1 us a unit and wavefront, while a workgroup would take its blocks one after the other (64 sequences of up to 500
//   keys, 8 KV heads, 14.7 us; single wavefronts 20.4).
// Never cut (where the host knows that no sequence is long): ranges are whole sequences, and there is no line.
// Up to 64 sequences a wavefront has one a lane and needs no other; up to as many as threads the wavefronts exchange their sums.  More go in launches of their own.
template <int ROWS, int NT>
__device__ inline Start find_start(const RowsArgs& a, unsigned w, unsigned grid, int most, Known<NT>& known)
{
    constexpr int NW = NT / 64, SIZES = 8;
    constexpr unsigned beside = kBeside / ROWS;
    __shared__ unsigned lds_sum[4][NW], lds_try[SIZES][NW];
    __shared__ Start found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // Place `rest` of a sequence's ranges (or units, where the line is cut)
    auto start_at = [&](int b, const Sequence& s, unsigned rest, unsigned line, unsigned per, bool ranges) {
        const Extent x = extent_of<ROWS>(a, s);
        const unsigned of_pair = ranges ? ranges_of((unsigned)x.units, per) : (unsigned)x.units + beside;
        Start st = {b, 0, ranges ? 0 : (int)beside, rest / of_pair, 0, per, s, 0, 0, 1};
        st.at = (int)((rest - st.pair * of_pair) * (ranges ? per : 1u));
        st.left = ranges ? (unsigned)(x.units - st.at) : line - w * per;
        if (st.left > per) st.left = per;
        return st;
    };
    const bool one_wave = a.c.S <= 64;
    const int b = one_wave ? lane : tid;
    unsigned units = 1, pairs = 0;
    Sequence s = {0, 0, 0};
    if (b < a.c.S) {
        s = sequence_at(a.c.length, a.row_start, b, a.R, most);
        const Extent x = extent_of<ROWS>(a, s);
        units = (unsigned)x.units;
        pairs = (unsigned)x.row_blocks * (unsigned)a.c.Hkv;
    }
    // Sums over the sequences up to and with one's own, and over all
    auto sums = [&](int n, const unsigned (&x)[2], unsigned (&upto)[2], unsigned (&all)[2]) {
        unsigned sum[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            upto[i] = scan64(x[i]);
            sum[i] = (unsigned)__builtin_amdgcn_readlane((int)upto[i], 63);
            all[i] = sum[i];
        }
        if (__builtin_expect(one_wave, 1)) return;
        if (lane == 0) lds_sum[2 * n][wave] = sum[0], lds_sum[2 * n + 1][wave] = sum[1];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            all[i] = 0;
            for (int j = 0; j < NW; ++j) {
                if (j < wave) upto[i] += lds_sum[2 * n + i][j];
                all[i] += lds_sum[2 * n + i][j];
            }
        }
    };
    unsigned upto[2], all[2];
    sums(0, {units * pairs, pairs}, upto, all);
    const unsigned total = all[0], blocks = all[1];
    bool ranges = blocks <= grid;
    unsigned group = NW;
    while (group > 1 && blocks * group > NW * grid) group /= 2;
    const unsigned longest_short = ranges ? 0u : a.never_cut ? 0x7fffffffu : min(32u, group * 5u * ((blocks - 1) / grid));
    unsigned per = 0;
    if (ranges) {
        unsigned longest = largest64(pairs > 0 ? units : 0);
        if (__builtin_expect(!one_wave, 0)) {
            __syncthreads();
            if (lane == 0) lds_sum[0][wave] = longest;
            __syncthreads();
            for (int j = 0; j < NW; ++j) longest = max(longest, lds_sum[0][j]);
        }
        per = whole_units(longest);
        if (!a.never_cut && longest > 0) {
            unsigned sure = per;
            if (blocks < grid) sure = min(sure, whole_units((total + grid - blocks - 1) / (grid - blocks)));
            const unsigned least = min(whole_units((total + grid - 1) / grid), sure);
            auto size = [&](unsigned i) { return whole_units(least + (sure - least) * i / (SIZES - 1)); };
            if (__builtin_expect(one_wave, 1)) { // the least by halving: more ranges, smaller ones
                unsigned low = 0, high = SIZES - 1;
                for (int i = 0; i < 3; ++i) {
                    const unsigned middle = (low + high) / 2;
                    const unsigned sum = (unsigned)__builtin_amdgcn_readlane((int)scan64(pairs * ranges_of(units, size(middle))), 63);
                    if (sum <= grid) high = middle;
                    else low = middle + 1;
                }
                per = size(high);
            } else {
                for (unsigned i = 0; i < SIZES; ++i) {
                    const unsigned sum = scan64(pairs * ranges_of(units, size(i)));
                    if (lane == 63) lds_try[i][wave] = sum;
                }
                __syncthreads();
                per = sure;
                for (int i = SIZES - 2; i >= 0; --i) {
                    unsigned sum = 0;
                    for (int j = 0; j < NW; ++j) sum += lds_try[i][j];
                    if (sum <= grid) per = size((unsigned)i);
                }
            }
            ranges = per <= whole_units((total + blocks * beside + grid - 1) / grid);
        }
    }
    per = (unsigned)__builtin_amdgcn_readfirstlane((int)per);
    const bool is_short = units <= longest_short;
    const unsigned mine = is_short || pairs == 0 ? 0u : ranges ? pairs * ranges_of(units, per) : (units + beside) * pairs;
    if (__builtin_expect(!one_wave, 0)) __syncthreads();         // the sums are read
    sums(1, {mine, is_short ? pairs : 0u}, upto, all);
    const unsigned line = all[0];
    if (!ranges) per = whole_units((line + grid - 1) / grid);
    if (__builtin_expect(all[1] > 0, 0)) {
        if (one_wave ? wave == 0 : true) {
            known.s[b] = s;
            known.shorts[b] = upto[1];
        }
        __syncthreads();
    }
    const unsigned want = ranges ? w : w * per, before = upto[0] - mine;
    const bool here = want >= before && want < upto[0];
    Start st = {-1, 0, 0, 0, 0, per, {0, 0, 0}, 0, 0, 1};
    if (__builtin_expect(one_wave, 1)) {
        const unsigned long long who = __builtin_amdgcn_ballot_w64(here);
        if (who != 0ull) {
            const int l = __builtin_ctzll(who);
            const Sequence of = {__builtin_amdgcn_readlane(s.length, l), __builtin_amdgcn_readlane(s.row0, l), __builtin_amdgcn_readlane(s.rows, l)};
            st = start_at(l, of, want - (unsigned)__builtin_amdgcn_readlane((int)before, l), line, per, ranges);
        }
    } else {
        if (tid == 0) found = st;
        __syncthreads();
        if (here) found = start_at(b, s, want - before, line, per, ranges);
        __syncthreads();
        st = found;
    }
    st.shorts = all[1];
    st.longest_short = (int)longest_short;
    st.group = (int)group;
    while (st.group < NW && (int)st.shorts * 2 * st.group <= (int)(NW * grid)) st.group *= 2;        // fewer shorts than blocks
    return st;
}

// Workgroups are dealt round-robin to the 8 XCDs; each XCD gets a contiguous range of the work, so that blocks of rows that read the
// same keys share an L2.
__device__ inline unsigned logical_workgroup(unsigned idx, unsigned grid)
{
    const unsigned x = idx & 7, whole = grid >> 3, rest = grid & 7;
    return x * whole + (x < rest ? x : rest) + (idx >> 3);
}

// Eight channels of a row's output, divided by the sum of its softmax: by its mantissa, then by the power of two, as fp32 may not hold what is
// between (one over a sum below 2^-126)
__device__ inline void store_row(const RowsArgs& a, int row0, int hk, int p, int D, int c8, const f4 (&acc)[2], float sum)
{
    const float f = sum == 0.f ? 0.f : 1.f / __builtin_amdgcn_frexp_mantf(sum);
    const int bits = -kSumBits - __builtin_amdgcn_frexp_expf(sum);
    const int t = (int)a.G.quotient((unsigned)p), h = (int)a.G.rest((unsigned)p, (unsigned)t);
    unsigned out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y0 = __builtin_ldexpf(acc[i >> 1][2 * (i & 1)] * f, bits), y1 = __builtin_ldexpf(acc[i >> 1][2 * (i & 1) + 1] * f, bits);
        out[i] = a.io_bf16 ? pack_bf16(y0, y1) : pack_f16(y0, y1);
    }
    *reinterpret_cast<uint4*>(a.o + ((size_t)(row0 + t) * a.Hq + hk * (int)a.G.d + h) * D + c8) = make_uint4(out[0], out[1], out[2], out[3]);
}

// One workgroup = 8 wavefronts sweeps a contiguous range of units; a range may end inside one (sequence, head, row block) and begin
// inside another, whose parts go to slots and are merged by a second kernel.  So the work is even whatever the lengths, and the host need not
// know them.  The rows are those of all query heads of a KV head: a decoding step reads its keys once.
//
// What bounds it: long sequences, memory (262144 keys on 4 heads, 277 MB, 47.8 us, 5.8 TB/s; 16 ragged sequences, 305 MB, 56.5 us); few keys, what hangs on one
// another, about 10 us whatever is done in between (lengths 1.1, the table's entries 0.9, keys and queries 2, a unit 1.5, the wavefronts' states 2, the start of
// eight XCDs 2); 32 rows, the vector unit (a unit's 495 vector instructions and 64 MFMAs of 16 clocks, two wavefronts to a SIMD: 90 % of its time).
// Widening takes 1 instruction a key's number and 1.25 a value's (which is turned too), e4m3 0.5 and 0.75, of every lane; shared by the 16 or 32 rows it is
// two thirds of the vector work with 16.
//
// GEMMs on v_mfma_f32_16x16x32_f16, transposed: S^T = K Q^T, O^T += V^T P^T.  Lane l holds query row l % 16 and, with g = l / 16, keys
// 4g .. 4g+3 of a block of 16.  Which channels a k-step of the first GEMM consists of is free, so a lane takes 16 consecutive bytes of a
// key's row; which keys a k-step of the second consists of is free, so P needs no exchange; which channel a row of V^T is, is free too, so a lane takes D / 16
// consecutive bytes of a key's value, and the 8 keys x D / 16 channels that it holds are turned while they are widened.
//
// The value's scale is not applied to values (there are 128 of them per key, and one P per row): it goes into the exponent.  With
// t = score + log2(vscale), M a level near the running maximum of t and P = 2^(t - M): O = sum P y, and the sum of the softmax is sum P / vscale (held times kSum).
// P is at most 2^15, whatever the scales, and fp16 holds what matters of it.
template <int D, int RB, bool E4M3, bool LISTED, bool FAR>
__global__ __launch_bounds__(64 * kUnitsAtOnce, 2)
void pasa_cache_rows(RowsArgs a)
{
    constexpr int ROWS = 16 * RB, KS = D / 32, CB = D / 16, NW = kUnitsAtOnce, NT = 64 * NW;
    constexpr int LD = D + 4;                    // LDS row of the merge, in floats
    constexpr int VW = CB / 4;                   // words of a key's value that a lane takes
    constexpr int ONCE = FAR ? 2 : 0;            // non-temporal
    constexpr bool QLDS = RB > 1;                // the query fragments wait in LDS: the registers are needed for RB blocks
    // A wavefront's own part: while it sweeps, per key of the unit the score's factor, log2 of the value's scale and kSum over it, and the query fragments;
    // afterwards its stored output.
    __shared__ __attribute__((aligned(16))) float lds_o[NW * ROWS * LD];
    static_assert(3 * kUnit * 4 + (QLDS ? RB * KS * 1024 : 0) <= ROWS * LD * 4, "what a wavefront keeps while it sweeps fits its part");
    __shared__ float lds_l[NW][ROWS], lds_m[NW][ROWS];
    __shared__ Known<NT> known;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 15, g = lane >> 4;
    const int G = (int)a.G.d, most = a.c.table_width << a.page_log2, lg = a.page_log2;
    const unsigned grid = gridDim.x, w = logical_workgroup(blockIdx.x, grid);
    float* const key_f = lds_o + wave * ROWS * LD;
    h8* const lds_q = reinterpret_cast<h8*>(key_f + 3 * kUnit);

    Start at = find_start<ROWS, NT>(a, w, grid, most, known);
    // the same in all lanes, which the compiler does not see on all ways to here: the buffers' descriptions would be taken lane by lane
    auto uniform = [](auto& v) { v = (std::remove_reference_t<decltype(v)>)__builtin_amdgcn_readfirstlane((int)v); };
    uniform(at.b), uniform(at.per), uniform(at.beside), uniform(at.at), uniform(at.shorts), uniform(at.longest_short), uniform(at.group);
    unsigned left = at.left, pair = at.pair;     // units of this workgroup still to be swept
    int b = at.b, pos = at.at, beside = at.beside;
    Sequence s = at.s;
    Extent x = extent_of<ROWS>(a, s);
    bool first_piece = true;
    // Shorts: neighbours go to different workgroups.  False where the workgroup has no more; a group
    // for which there is none while the first one still has one goes along with no rows and no keys.
    int group = NW, lead = wave;                 // wavefronts that share a range or a short, and one's place among them
    unsigned next_short = w;
    auto take_short = [&] {
        const unsigned groups = NW / (unsigned)at.group, first = next_short, mine = first + grid * ((unsigned)wave / (unsigned)at.group);
        group = at.group;
        lead = wave & (group - 1);
        next_short += grid * groups;
        if ((group > 1 ? first : mine) >= at.shorts) return false;
        const unsigned want = mine < at.shorts ? mine : at.shorts - 1;
        int n = 0;                               // sequences whose shorts all come before
        for (int i = 0; i < a.c.S; i += 64) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i + lane < a.c.S && known.shorts[i + lane] <= want));
        b = __builtin_amdgcn_readfirstlane(n < a.c.S ? n : a.c.S - 1);
        s.length = __builtin_amdgcn_readfirstlane(known.s[b].length);
        s.row0 = __builtin_amdgcn_readfirstlane(known.s[b].row0);
        s.rows = __builtin_amdgcn_readfirstlane(known.s[b].rows);
        x = extent_of<ROWS>(a, s);
        pair = want - (unsigned)__builtin_amdgcn_readfirstlane(b > 0 ? (int)known.shorts[b - 1] : 0);
        pos = beside = 0;
        left = mine < at.shorts ? (unsigned)x.units : 0u;
        return true;
    };
    bool whole_blocks = b < 0;                   // shorts, not ranges
    if (__builtin_expect(whole_blocks, 0)) {
        if (tid == 0) a.records[w].pieces = 0;
        if (!take_short()) return;
    }

    for (;;) {
        uniform(b), uniform(pos), uniform(left), uniform(pair);
        uniform(s.length), uniform(s.row0), uniform(s.rows);
        uniform(x.keys), uniform(x.units), uniform(x.row_blocks);
        // the piece's units, [us, ue); none where the range ends before the block's first one, which the next workgroup then has
        const int end = (int)((unsigned)(x.units + beside - pos) < left ? x.units + beside : pos + (int)left);
        const int us = pos > beside ? pos - beside : 0, ue = end > beside ? end - beside : 0;
        const int hk = (int)(pair / (unsigned)x.row_blocks), p0 = (int)(pair - (unsigned)hk * (unsigned)x.row_blocks) * ROWS;
        const int list = ue > us ? s.rows * G : 0;      // rows of the KV head's query heads, by token, then head
        const int new0 = s.length - s.rows;      // position of the sequence's first row
        uniform(group), uniform(lead);
        const int begin = us + lead, step = group;
        const int units = begin < ue ? (ue - begin + step - 1) / step : 0;       // of this wavefront

        f4 O[RB][CB];
        float M[RB], l[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            M[rb] = kNoLevel;
            l[rb] = 0.f;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) O[rb][cb] = (f4)0.f;
        }
        auto row_of = [&](int rb) { return p0 + 16 * rb + lq < list ? p0 + 16 * rb + lq : list - 1; };
        auto query = [&](int p, int ks) {
            const int t = (int)a.G.quotient((unsigned)p), h = (int)a.G.rest((unsigned)p, (unsigned)t);
            return *reinterpret_cast<const u16x8*>(a.q + (size_t)(s.row0 + t) * (size_t)a.row_stride + (size_t)(hk * G + h) * D + 16 * g +
                                                   64 * (ks / 2) + 8 * (ks & 1));
        };
        if (units > 0) {
            // Places of the blocks of 16 keys, lane group g that of block g, by way of the list where there is one.  Three steps, each an
            // iteration ahead of the next: the list's entry, the table's, the keys.  Entries are read at index 0 where there is no block, and not
            // used.  No load hangs on a branch: where ways with and without one meet, the compiler waits for all that is on its way.
            const int* const table = a.c.table + (size_t)b * a.c.table_width;
            const int* const chosen = LISTED ? a.blocks + ((size_t)b * a.c.Hkv + hk) * a.count : nullptr;
            int listed_a, place_b, entry_b;      // of the unit after the next two; of the one after the next
            int pos_next = 0, page_next = -1, pos_now = 0, page_now = -1;
            auto first_key = [&](int n) { return (begin + step * n) * kUnit + 16 * g; };
            auto read_list = [&](int n) {
                const int vk = first_key(n);
                listed_a = LISTED ? chosen[n < units && vk < x.keys ? vk >> lg : 0] : 0;
            };
            auto read_entry = [&](int n) {
                const int vk = first_key(n), place = LISTED ? listed_a : vk >> lg;
                const bool in = n < units && vk < x.keys && place >= 0 && place < a.c.table_width;
                place_b = in ? place : -1;
                entry_b = table[in ? place : 0];
            };
            auto take_entry = [&](int n) {
                const int pos = (place_b << lg) + (first_key(n) & (a.c.page - 1));
                const bool in = place_b >= 0 && pos < s.length && entry_b >= 0 && entry_b < a.c.pages;
                pos_next = in ? pos : 0;
                page_next = in ? entry_b : -1;
            };

            uint4 K[4][D / 64];
            unsigned V[2][8][VW];                // k-step of 32 keys, key, word
            float ks_raw, vs_raw;
            const int koff = lq * D + 16 * g, voff = 4 * g * D + lq * CB;
            // A block that is not there reads nothing and comes as zeros: its buffer has no bytes.
            unsigned long long at_next = 0, at_now = 0;          // bytes from the first key (value) of the pool to the block's
            auto buffer_of = [&](void* base, int blk, unsigned long long offsets, int pages) {
                const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)offsets, 16 * blk), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(offsets >> 32), 16 * blk);
                return __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(base) + ((unsigned long long)hi << 32 | lo), 0,
                                                         __builtin_amdgcn_readlane(pages, 16 * blk) < 0 ? 0 : 16 * D, 0x00020000);
            };
            auto load_k = [&] {
                const size_t slot = ((size_t)(unsigned)(page_next < 0 ? 0 : page_next) * (unsigned)a.c.Hkv + (unsigned)hk) * (unsigned)a.c.page +
                                    (unsigned)(pos_next & (a.c.page - 1));
                at_next = slot * D;
#pragma unroll
                for (int blk = 0; blk < 4; ++blk) {
                    const __amdgpu_buffer_rsrc_t from = buffer_of(a.c.k, blk, at_next, page_next);
#pragma unroll
                    for (int j = 0; j < D / 64; ++j) K[blk][j] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(from, koff + 64 * j, 0, ONCE));
                }
                // a lane a key
                ks_raw = a.c.kscale[slot + lq];
                vs_raw = a.c.vscale[slot + lq];
            };
            auto load_v = [&] {
#pragma unroll
                for (int blk = 0; blk < 4; ++blk) {
                    const __amdgpu_buffer_rsrc_t from = buffer_of(a.c.v, blk, at_now, page_now);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (VW == 2) {
                            const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(from, voff + i * D, 0, ONCE));
                            V[blk >> 1][4 * (blk & 1) + i][0] = y.x;
                            V[blk >> 1][4 * (blk & 1) + i][VW - 1] = y.y;
                        } else {
                            V[blk >> 1][4 * (blk & 1) + i][0] = __builtin_amdgcn_raw_buffer_load_b32(from, voff + i * D, 0, ONCE);
                        }
                    }
                }
            };

            // query rows, and what each sees; rows behind the last one are the last one again, and not stored
            u16x8 raw[RB][KS];
            int last[RB];
            unsigned long long bits[RB];
            read_list(0);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int p = row_of(rb), t = (int)a.G.quotient((unsigned)p);
                last[rb] = a.tree != nullptr ? new0 - 1 : new0 + t;
                bits[rb] = a.tree != nullptr ? a.tree[s.row0 + t] : 0ull;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) raw[rb][ks] = query(p, ks);
            }
            read_entry(0);
            read_list(1);
            take_entry(0);
            read_entry(1);
            read_list(2);
            load_k();
            page_now = page_next, pos_now = pos_next, at_now = at_next;
            load_v();
            PASA_FENCE();
            h8 Qr[RB][KS];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) Qr[rb][ks] = __builtin_bit_cast(h8, raw[rb][ks]);
            if (a.io_bf16) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) Qr[rb][ks] = bf16x8_to_h8(raw[rb][ks]);
            }
            if (QLDS) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) lds_q[(rb * KS + ks) * 64 + lane] = Qr[rb][ks];
            }
            auto Q = [&](int rb, int ks) { return QLDS ? lds_q[(rb * KS + ks) * 64 + lane] : Qr[rb][ks]; };

            int n = 0;
            do {
                const bool whole = __builtin_amdgcn_ballot_w64(page_now >= 0 && pos_now + 16 <= new0) == ~0ull;      // all rows see all keys of the unit
                const bool vs_one = vs_raw == 1.f;
                // per key: what its score is multiplied by, log2 of the value's scale and kSum over it; in the lanes' order of keys
                key_f[lane] = ks_raw * a.scale2;
                key_f[kUnit + lane] = __builtin_amdgcn_logf(vs_raw);
                // finite, so that 0 times it is 0: a key that is not there may have any scale, and a NaN shows in the score of the rows that see it
                key_f[2 * kUnit + lane] = kSum * __builtin_fminf(__builtin_fmaxf(__builtin_amdgcn_rcpf(vs_raw), 0.f), 3e38f);
                __builtin_amdgcn_wave_barrier();                 // a wavefront's LDS accesses are done in order
                asm volatile("" ::: "memory");

                f4 S[RB][4];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int blk = 0; blk < 4; ++blk) S[rb][blk] = (f4)0.f;
                h8 q[RB][KS];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) q[rb][ks] = Q(rb, ks);
                if (QLDS) PASA_FENCE();          // all asked for before the first is used
#pragma unroll
                for (int j = 0; j < D / 64; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int blk = 0; blk < 4; ++blk) {
                            const unsigned kw[2] = {h == 0 ? K[blk][j].x : K[blk][j].z, h == 0 ? K[blk][j].y : K[blk][j].w};
                            h8 f;
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const h2 lo = widen2<E4M3, false>(kw[e]), hi = widen2<E4M3, true>(kw[e]);
                                f[4 * e] = lo[0]; f[4 * e + 1] = lo[1]; f[4 * e + 2] = hi[0]; f[4 * e + 3] = hi[1];
                            }
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb) S[rb][blk] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, q[rb][2 * j + h], S[rb][blk], 0, 0, 0);
                        }
                PASA_FENCE();
                take_entry(n + 1);
                read_entry(n + 2);
                read_list(n + 3);
                load_k();
                PASA_FENCE();

                f4 inv[4];
#pragma unroll
                for (int blk = 0; blk < 4; ++blk) {
                    const f4 factor = *reinterpret_cast<const f4*>(key_f + 16 * blk + 4 * g);
                    const f4 lv = *reinterpret_cast<const f4*>(key_f + kUnit + 16 * blk + 4 * g);
                    inv[blk] = *reinterpret_cast<const f4*>(key_f + 2 * kUnit + 16 * blk + 4 * g);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) S[rb][blk][i] = __builtin_fmaf(S[rb][blk][i], factor[i], lv[i]);
                }
                // A token whose value is all zeros has the scale 1, which may be far above the others', and adds nothing to O: it is not to raise the
                // level that P is rounded at (a first token with most of the weight would take the others below what fp16 holds).  Any scale
                // stands for its value; 2^-60 is below those of fp16 values, and far above where its share of the sum would be lost.
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(vs_one) != 0ull, 0)) {
#pragma unroll
                    for (int blk = 0; blk < 4; ++blk)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            unsigned any = 0;
#pragma unroll
                            for (int d = 0; d < VW; ++d) {
                                const unsigned y = V[blk >> 1][4 * (blk & 1) + i][d];
                                any |= E4M3 ? y & 0x7f7f7f7fu : y ^ 0x80808080u;
                            }
                            const unsigned long long who = __builtin_amdgcn_ballot_w64(any != 0u);       // lanes 16 g .. 16 g + 15 have a key
                            const bool zeros = ((unsigned)(who >> (16 * g)) & 0xffffu) == 0u && inv[blk][i] == kSum;
                            inv[blk][i] = zeros ? kSum * 0x1p60f : inv[blk][i];
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb) S[rb][blk][i] = zeros ? S[rb][blk][i] - 60.f : S[rb][blk][i];
                        }
                }
                if (__builtin_expect(!whole, 0)) {
#pragma unroll
                    for (int blk = 0; blk < 4; ++blk) {
                        const int pos0 = __builtin_amdgcn_readlane(pos_now, 16 * blk), page = __builtin_amdgcn_readlane(page_now, 16 * blk);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // selections, no ways: hipcc 7.2 drops the -inf of a way that && and || make
                            const int pos = pos0 + 4 * g + i, nth = pos - new0;
                            const unsigned there = (unsigned)(page >= 0) & (unsigned)(pos < s.length), proposed = (unsigned)((unsigned)nth < 64u);
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb) {
                                const unsigned see = there & ((unsigned)(pos <= last[rb]) | (proposed & (unsigned)(bits[rb] >> (nth & 63))));
                                S[rb][blk][i] = (see & 1u) != 0u ? S[rb][blk][i] : -__builtin_inff();
                            }
                            // what is no key may hold anything, NaN among it, and 0 times that is not 0
#pragma unroll
                            for (int d = 0; d < VW; ++d) V[blk >> 1][4 * (blk & 1) + i][d] = there != 0u ? V[blk >> 1][4 * (blk & 1) + i][d] : 0u;
                        }
                    }
                }

                h8 P[RB][2];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    float top = S[rb][0][0];
#pragma unroll
                    for (int blk = 0; blk < 4; ++blk)
#pragma unroll
                        for (int i = 0; i < 4; ++i) top = __builtin_fmaxf(top, S[rb][blk][i]);
                    if (__builtin_amdgcn_ballot_w64(top > M[rb] + kRise) != 0ull) {
                        const float row_top = max_row(top);
                        const float level = row_top > M[rb] + kRise ? row_top - kBelow : M[rb];
                        const float r = __builtin_amdgcn_exp2f(M[rb] - level);
                        M[rb] = level;
                        l[rb] *= r;
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb) O[rb][cb] *= r;
                    }
#pragma unroll
                    for (int blk = 0; blk < 4; ++blk) {
                        float e[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(S[rb][blk][i] - M[rb]);
                        const h2 lo = pack_rn(e[0], e[1]), hi = pack_rn(e[2], e[3]);
                        P[rb][blk >> 1][4 * (blk & 1)] = lo[0];
                        P[rb][blk >> 1][4 * (blk & 1) + 1] = lo[1];
                        P[rb][blk >> 1][4 * (blk & 1) + 2] = hi[0];
                        P[rb][blk >> 1][4 * (blk & 1) + 3] = hi[1];
#pragma unroll
                        for (int i = 0; i < 4; ++i) l[rb] = __builtin_fmaf(e[i], inv[blk][i], l[rb]);
                    }
                }
                PASA_FENCE();
#pragma unroll
                for (int st = 0; st < 2; ++st)
#pragma unroll
                    for (int d = 0; d < VW; ++d) {
                        unsigned two[4][2];      // pairs of keys: channels 0 and 1, channels 2 and 3 of the word
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            two[e][0] = __builtin_amdgcn_perm(V[st][2 * e + 1][d], V[st][2 * e][d], 0x05010400u);
                            two[e][1] = __builtin_amdgcn_perm(V[st][2 * e + 1][d], V[st][2 * e][d], 0x07030602u);
                        }
#pragma unroll
                        for (int ch = 0; ch < 4; ++ch) {
                            h8 f;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const h2 y = ch & 1 ? widen2<E4M3, true>(two[e][ch >> 1]) : widen2<E4M3, false>(two[e][ch >> 1]);
                                f[2 * e] = y[0];
                                f[2 * e + 1] = y[1];
                            }
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb)
                                O[rb][4 * d + ch] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, P[rb][st], O[rb][4 * d + ch], 0, 0, 0);
                        }
                    }
                PASA_FENCE();
                page_now = page_next, pos_now = pos_next, at_now = at_next;
                load_v();
                PASA_FENCE();
            } while (++n < units);
        }

        // ---- the wavefronts' states brought to the highest of their levels and added ----
        int ln = lane;
        asm volatile("" : "+v"(ln));             // no address is to be worked out before the main loop and kept through it
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float sum = sum_row(l[rb]);
            if (ln < 16) {
                lds_m[wave][16 * rb + ln] = M[rb];
                lds_l[wave][16 * rb + ln] = sum;
            }
            // element i of block cb is channel CB * (4 g + i) + cb
            float* dst = lds_o + (wave * ROWS + 16 * rb + (ln & 15)) * LD + CB * 4 * (ln >> 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int cb = 0; cb < CB; cb += 4)
                    *reinterpret_cast<f4*>(dst + CB * i + cb) = f4{O[rb][cb][i], O[rb][cb + 1][i], O[rb][cb + 2][i], O[rb][cb + 3][i]};
        }
        if (__builtin_expect(group == 1, 0)) {
            __builtin_amdgcn_wave_barrier();     // a wavefront's LDS accesses are done in order
            asm volatile("" ::: "memory");
            constexpr int STEP = 64 / (D / 8);   // rows at a time, eight channels a lane
#pragma unroll
            for (int r0 = 0; r0 < ROWS; r0 += STEP) {
                const int r = r0 + ln / (D / 8), c8 = ln % (D / 8) * 8, p = p0 + r;
                const float* src = lds_o + (wave * ROWS + r) * LD + c8;
                const f4 acc[2] = {*reinterpret_cast<const f4*>(src), *reinterpret_cast<const f4*>(src + 4)};
                if (p < list) store_row(a, s.row0, hk, p, D, c8, acc, lds_l[wave][r]);
            }
            asm volatile("" ::: "memory");
            if (!take_short()) return;
            continue;
        }
        __syncthreads();
        const bool complete = us == 0 && ue == x.units;
        const unsigned my_slot = 2 * w + (first_piece ? 0u : 1u);
        float* slot = a.slots + (size_t)my_slot * cache_slot_floats(RB, D);
        auto bring_together = [&](auto size) {
            constexpr int GS = decltype(size)::value, STEP = 64 * GS / (D / 8);      // rows at a time, eight channels a lane
            const int w0 = wave - lead, th = 64 * lead + ln;
#pragma unroll
            for (int r0 = 0; r0 < ROWS; r0 += STEP) {
                const int r = r0 + th / (D / 8), c8 = th % (D / 8) * 8, p = p0 + r;
                if (r >= ROWS || p >= list) break;
                float level = lds_m[w0][r], sum = 0.f;
#pragma unroll
                for (int i = 1; i < GS; ++i) level = __builtin_fmaxf(level, lds_m[w0 + i][r]);
                f4 acc[2] = {(f4)0.f, (f4)0.f};
#pragma unroll
                for (int i = 0; i < GS; ++i) {
                    const float f = __builtin_amdgcn_exp2f(lds_m[w0 + i][r] - level);
                    sum += f * lds_l[w0 + i][r];
                    const float* src = lds_o + ((w0 + i) * ROWS + r) * LD + c8;
                    acc[0] += f * *reinterpret_cast<const f4*>(src);
                    acc[1] += f * *reinterpret_cast<const f4*>(src + 4);
                }
                if (complete) {
                    store_row(a, s.row0, hk, p, D, c8, acc, sum);
                } else {
                    if (c8 == 0) {
                        slot[2 * r] = sum;
                        slot[2 * r + 1] = level;
                    }
                    *reinterpret_cast<f4*>(slot + 2 * ROWS + (size_t)r * D + c8) = acc[0];
                    *reinterpret_cast<f4*>(slot + 2 * ROWS + (size_t)r * D + c8 + 4) = acc[1];
                }
            }
        };
        if (__builtin_expect(group == NW, 1)) bring_together(std::integral_constant<int, NW>{});
        else if (group == 4) bring_together(std::integral_constant<int, 4>{});
        else bring_together(std::integral_constant<int, 2>{});
        if (__builtin_expect(whole_blocks, 0)) {
            __syncthreads();                     // the LDS is free again
            if (!take_short()) return;
            continue;
        }
        left -= (unsigned)(end - pos);
        first_piece = first_piece && ue == us;
        bool more = left > 0;
        if (!more && tid == 0) {                 // begun here, and goes on in the ranges behind?
            MergeRecord m = {0, (int)my_slot, p0, list, s.row0, hk, {0, 0}};
            if (us == 0 && ue > 0 && ue < x.units) m.pieces = clamp_int(1 + (int)(((unsigned)(x.units - ue) + at.per - 1) / at.per), 0, (int)(grid - w));
            a.records[w] = m;
        }
        pos = 0;
        if (more && ++pair == (unsigned)x.row_blocks * (unsigned)a.c.Hkv) {
            pair = 0;
            do {                                 // the next sequence in the line
                if (++b >= a.c.S) {
                    if (tid == 0) a.records[w].pieces = 0;
                    more = false;
                    break;
                }
                s = sequence_at(a.c.length, a.row_start, b, a.R, most);
                x = extent_of<ROWS>(a, s);
            } while (s.rows == 0 || x.units <= (int)at.longest_short);
        }
        if (!more && at.shorts == 0) return;
        __syncthreads();                         // the LDS is free again
        if (!more) {
            whole_blocks = true;
            if (!take_short()) return;
        }
    }
}

// A row block that several workgroups have swept: pieces from the slot of the one that began it and the first slots of those behind it.
// Workgroup (w, part) adds rows of what workgroup w of the sweep has begun: all its wavefronts one row, or (EACH) each a row of its own, for blocks of
// few pieces.  D / 8 neighbouring lanes take a piece, eight channels each, and the groups of lanes are added at the end, always in the same order.
template <int D, int RB, bool EACH>
__global__ __launch_bounds__(kCacheThreads)
void pasa_cache_merge(RowsArgs a, FastDiv parts)
{
    constexpr int ROWS = 16 * RB, CHUNKS = D / 8, LANES = (EACH ? 64 : kCacheThreads) / CHUNKS, AT = 4;
    __shared__ float lds_acc[4][D];
    __shared__ float lds_state[4][2];
    const unsigned w = parts.quotient(blockIdx.x);
    const MergeRecord m = a.records[w];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, part = (int)parts.rest(blockIdx.x, w);
    const int r = EACH ? 4 * part + wave : part, p = m.p0 + r;
    if (m.pieces == 0 || r >= ROWS || p >= m.list) return;
    const int c8 = tid % CHUNKS * 8;
    float level = kNoLevel, sum = 0.f;
    f4 acc[2] = {(f4)0.f, (f4)0.f};
    for (int i0 = (EACH ? lane : tid) / CHUNKS; i0 < m.pieces; i0 += AT * LANES) {
        f2 state[AT];
        f4 part[AT][2];
#pragma unroll
        for (int j = 0; j < AT; ++j) {           // all loads at once; behind the last piece the first one of the lane again, for nothing
            const int i = i0 + j * LANES < m.pieces ? i0 + j * LANES : i0;
            const float* slot = a.slots + (size_t)(i == 0 ? (unsigned)m.slot : 2u * (w + (unsigned)i)) * cache_slot_floats(RB, D);
            state[j] = *reinterpret_cast<const f2*>(slot + 2 * r);
            part[j][0] = *reinterpret_cast<const f4*>(slot + 2 * ROWS + (size_t)r * D + c8);
            part[j][1] = *reinterpret_cast<const f4*>(slot + 2 * ROWS + (size_t)r * D + c8 + 4);
        }
        float top = level;
#pragma unroll
        for (int j = 0; j < AT; ++j) top = __builtin_fmaxf(top, state[j][1]);
        const float keep = __builtin_amdgcn_exp2f(level - top);
        sum *= keep;
        acc[0] *= keep;
        acc[1] *= keep;
#pragma unroll
        for (int j = 0; j < AT; ++j)
            if (i0 + j * LANES < m.pieces) {
                const float f = __builtin_amdgcn_exp2f(state[j][1] - top);
                sum += f * state[j][0];
                acc[0] += f * part[j][0];
                acc[1] += f * part[j][1];
            }
        level = top;
    }
    // the groups of lanes of a wavefront, then the wavefronts
    float top = level;
#pragma unroll
    for (int o = CHUNKS; o < 64; o <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, o));
    const float f = __builtin_amdgcn_exp2f(level - top);
    sum *= f;
    acc[0] *= f;
    acc[1] *= f;
#pragma unroll
    for (int o = CHUNKS; o < 64; o <<= 1) {
        sum += __shfl_xor(sum, o);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i >> 2][i & 3] += __shfl_xor(acc[i >> 2][i & 3], o);
    }
    if (EACH) {
        if (lane < CHUNKS) store_row(a, m.row0, m.hk, p, D, c8, acc, sum);
        return;
    }
    if (lane < CHUNKS) {
        *reinterpret_cast<f4*>(&lds_acc[wave][c8]) = acc[0];
        *reinterpret_cast<f4*>(&lds_acc[wave][c8 + 4]) = acc[1];
        if (lane == 0) lds_state[wave][0] = sum, lds_state[wave][1] = top;
    }
    __syncthreads();
    if (tid >= CHUNKS) return;
    top = lds_state[0][1];
#pragma unroll
    for (int i = 1; i < 4; ++i) top = __builtin_fmaxf(top, lds_state[i][1]);
    sum = 0.f;
    acc[0] = acc[1] = (f4)0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(lds_state[i][1] - top);
        sum += e * lds_state[i][0];
        acc[0] += e * *reinterpret_cast<const f4*>(&lds_acc[i][c8]);
        acc[1] += e * *reinterpret_cast<const f4*>(&lds_acc[i][c8 + 4]);
    }
    store_row(a, m.row0, m.hk, p, D, c8, acc, sum);
}

}  // namespace

hipError_t pasa_launch_attn_cache(const pasa_cache& c, const void* q, void* o, int R, long long row_stride, const int* row_start, int Hq,
                                  float scale, const unsigned long long* tree, const int* blocks, int count, int io_bf16,
                                  const CachePlan& plan, void* workspace, hipStream_t stream)
{
    constexpr int kSequences = 64 * kUnitsAtOnce;                    // of a launch: one a thread
    RowsArgs a;
    a.c = c;
    a.q = static_cast<const unsigned short*>(q);
    a.o = static_cast<unsigned short*>(o);
    a.row_start = row_start;
    a.tree = tree;
    a.blocks = blocks;
    a.records = static_cast<MergeRecord*>(workspace);
    a.slots = reinterpret_cast<float*>(a.records + plan.grid);
    a.row_stride = row_stride;
    a.scale2 = scale * LOG2E;
    a.R = R;
    a.Hq = Hq;
    a.count = count;
    a.io_bf16 = io_bf16;
    a.never_cut = plan.never_cut;
    a.page_log2 = log2_of(c.page);
    a.G = fast_div((unsigned)(Hq / c.Hkv));
    auto one = [&](auto rows, auto merge, auto merge_each) {
        rows<<<plan.grid, 64 * kUnitsAtOnce, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || plan.grid == 1 || plan.never_cut) return e;
        const long long most = (long long)R * (Hq / c.Hkv);          // rows of a block
        const unsigned each = (unsigned)(most < 16 * plan.row_blocks ? most : 16 * plan.row_blocks);
        // up to 16 pieces a block on average: a wavefront takes them in one step
        if ((long long)a.c.S * c.Hkv * 16 >= plan.grid) merge_each<<<(unsigned)plan.grid * ((each + 3) / 4), kCacheThreads, 0, stream>>>(a, fast_div((each + 3) / 4));
        else merge<<<(unsigned)plan.grid * each, kCacheThreads, 0, stream>>>(a, fast_div(each));
        return hipGetLastError();
    };
    auto go = [&](auto rows, auto merge, auto merge_each) {
        for (int b = 0; b < c.S; b += kSequences) {
            a.c.S = c.S - b < kSequences ? c.S - b : kSequences;
            a.c.table = c.table + (size_t)b * c.table_width;
            a.c.length = c.length + b;
            a.row_start = row_start + b;
            if (blocks != nullptr) a.blocks = blocks + (size_t)b * c.Hkv * count;
            const hipError_t e = one(rows, merge, merge_each);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    const bool e = c.format == PASA_CACHE_E4M3, l = blocks != nullptr;
    auto of_kind = [&](auto d, auto rb, auto far) {
        constexpr int D = decltype(d)::value, RB = decltype(rb)::value;
        constexpr bool F = decltype(far)::value;
        if (e) return l ? go(pasa_cache_rows<D, RB, true, true, F>, pasa_cache_merge<D, RB, false>, pasa_cache_merge<D, RB, true>) : go(pasa_cache_rows<D, RB, true, false, F>, pasa_cache_merge<D, RB, false>, pasa_cache_merge<D, RB, true>);
        return l ? go(pasa_cache_rows<D, RB, false, true, F>, pasa_cache_merge<D, RB, false>, pasa_cache_merge<D, RB, true>) : go(pasa_cache_rows<D, RB, false, false, F>, pasa_cache_merge<D, RB, false>, pasa_cache_merge<D, RB, true>);
    };
    // Keys and values that are read once and may be more than the last cache's 256 MB are read past the caches.  us, past / through them: 277 MB
    // (262144 keys, 4 heads) 54.3 / 58.9, 305 MB 63.2 / 65.5; 68 MB, which a program that does little else finds there again, 28.0 / 24.4
    const long long held = (blocks != nullptr && count < c.table_width ? count : c.table_width);
    const bool far = (double)held * c.page * c.S * c.Hkv * 2 * c.d > 256e6;
    auto of_format = [&](auto d, auto rb) {
        if constexpr (decltype(rb)::value == 1) {
            if (far) return of_kind(d, rb, std::true_type{});
        }
        return of_kind(d, rb, std::false_type{});
    };
    auto of_rows = [&](auto d) {
        return plan.row_blocks == 1 ? of_format(d, std::integral_constant<int, 1>{}) : of_format(d, std::integral_constant<int, 2>{});
    };
    return c.d == 128 ? of_rows(std::integral_constant<int, 128>{}) : of_rows(std::integral_constant<int, 64>{});
}
