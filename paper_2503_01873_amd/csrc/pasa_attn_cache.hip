// Attention of a few rows per sequence over the paged 8-bit cache: pasa_cache_rows, and the merge of what its workgroups leave.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "pasa_cache.h"

namespace {

// A row's output moves to a new level when a score exceeds the stored one by 2^8: P stays below 2^8 until then, far inside fp16.
constexpr float kRise = 8.f;
constexpr float kNoLevel = -1e30f;               // finite: a score of -inf against it gives 0 and no NaN

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
    int R, Hq, count, io_bf16, page_log2;
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

// What a workgroup sweeps first: units `us` on of block of rows `pair` (of all heads) of sequence b, and how many from there on; b < 0: nothing.
struct Start {
    int b, us;
    unsigned pair, left, per;
    Sequence s;
};

// Two ways to share out.  Few (sequence, head, row block)s, half as many as there are workgroups at most: each is cut into ranges of `per` units,
// one a workgroup, with `per` the least of eight sizes (one a wavefront tries) that gives no more ranges than workgroups: between an even share of the whole and
// that share for the workgroups that are left when every row block has one range that is not full, with which it always fits.  Many: the units of all are one line that is cut evenly, and a
// workgroup's range may end inside one block and begin inside the next.  That costs it what a range costs beside its keys, twice: 6 us (4 heads of 4999 keys 14.7 us,
// so 10.5).
template <int ROWS, int NT>
__device__ inline Start find_start(const RowsArgs& a, unsigned w, unsigned grid, int most)
{
    constexpr int NW = NT / 64;
    __shared__ unsigned lds_units[NT], lds_pairs[NT], lds_sum[3][NW], lds_try[NW];
    __shared__ Start found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // Place `rest` of a sequence's ranges (or units, where the line is cut)
    auto start_at = [&](int b, const Sequence& s, unsigned rest, unsigned total, unsigned per, bool ranges) {
        const Extent x = extent_of<ROWS>(a, s);
        const unsigned of_pair = ranges ? ((unsigned)x.units + per - 1) / per : (unsigned)x.units;
        Start st = {b, 0, rest / of_pair, 0, per, s};
        st.us = (int)((rest - st.pair * of_pair) * (ranges ? per : 1u));
        st.left = ranges ? (unsigned)(x.units - st.us) : total - w * per;
        if (st.left > per) st.left = per;
        return st;
    };
    if (a.c.S <= NT) {                           // a sequence a thread: what is read of it once is enough
        unsigned units = 1, pairs = 0;
        Sequence s = {0, 0, 0};
        if (tid < a.c.S) {
            s = sequence_at(a.c.length, a.row_start, tid, a.R, most);
            const Extent x = extent_of<ROWS>(a, s);
            units = (unsigned)x.units;
            pairs = (unsigned)x.row_blocks * (unsigned)a.c.Hkv;
        }
        lds_units[tid] = units;
        lds_pairs[tid] = pairs;
        const unsigned upto_u = scan64(units * pairs), upto_p = scan64(pairs);
        if (lane == 63) lds_sum[0][wave] = upto_u, lds_sum[1][wave] = upto_p;
        if (tid == 0) found.b = -1;
        __syncthreads();
        unsigned total = 0, all = 0, before = upto_u - units * pairs, mine = units * pairs;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            if (i < wave) before += lds_sum[0][i];
            total += lds_sum[0][i];
            all += lds_sum[1][i];
        }
        const bool ranges = 2 * all <= grid;
        unsigned per = whole_units((total + grid - 1) / grid), want = w * per;
        if (ranges) {
            const unsigned least = per, sure = whole_units((total + grid - all - 1) / (grid - all));
            auto size = [&](unsigned i) { return whole_units(least + (sure - least) * i / (NW - 1)); };
            const unsigned size_of_wave = size((unsigned)wave);
            unsigned sum = 0;
            for (int i = lane; i < a.c.S; i += 64) sum += size_of_wave > 0 ? lds_pairs[i] * ((lds_units[i] + size_of_wave - 1) / size_of_wave) : 0;
            sum = scan64(sum);
            if (lane == 63) lds_try[wave] = sum;
            __syncthreads();
            per = sure;
#pragma unroll
            for (int i = NW - 2; i >= 0; --i)
                if (lds_try[i] <= grid) per = size((unsigned)i);
            mine = per > 0 ? pairs * ((units + per - 1) / per) : 0;
            before = scan64(mine);
            if (lane == 63) lds_sum[2][wave] = before;
            __syncthreads();
            before -= mine;
#pragma unroll
            for (int i = 0; i < NW; ++i)
                if (i < wave) before += lds_sum[2][i];
            want = w;
        }
        if (want >= before && want < before + mine) found = start_at(tid, s, want - before, total, per, ranges);
        __syncthreads();
    } else {
        unsigned per = 0;
        const Place at = find_place<NT>(a.c.length, a.row_start, a.c.S, a.R, most, [&](const Sequence& s) {
            const Extent x = extent_of<ROWS>(a, s);
            return (unsigned)x.row_blocks * (unsigned)a.c.Hkv * (unsigned)x.units;
        }, [&](unsigned total) { return w * (per = whole_units((total + grid - 1) / grid)); });
        if (tid == 0) {
            if (at.b < 0) found.b = -1;
            else found = start_at(at.b, at.s, at.rest, at.total, per, false);
        }
        __syncthreads();
    }
    Start st;
    st.b = __builtin_amdgcn_readfirstlane(found.b);
    st.us = __builtin_amdgcn_readfirstlane(found.us);
    st.pair = (unsigned)__builtin_amdgcn_readfirstlane((int)found.pair);
    st.left = (unsigned)__builtin_amdgcn_readfirstlane((int)found.left);
    st.per = (unsigned)__builtin_amdgcn_readfirstlane((int)found.per);
    st.s.length = __builtin_amdgcn_readfirstlane(found.s.length);
    st.s.row0 = __builtin_amdgcn_readfirstlane(found.s.row0);
    st.s.rows = __builtin_amdgcn_readfirstlane(found.s.rows);
    return st;
}

// Workgroups are dealt round-robin to the 8 XCDs; each XCD gets a contiguous range of the work, so that blocks of rows that read the
// same keys share an L2.
__device__ inline unsigned logical_workgroup(unsigned idx, unsigned grid)
{
    const unsigned x = idx & 7, whole = grid >> 3, rest = grid & 7;
    return x * whole + (x < rest ? x : rest) + (idx >> 3);
}

// Eight channels of a row's output, divided by the sum of its softmax
__device__ inline void store_row(const RowsArgs& a, int row0, int hk, int p, int D, int c8, const f4 (&acc)[2], float sum)
{
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    const int t = (int)a.G.quotient((unsigned)p), h = (int)a.G.rest((unsigned)p, (unsigned)t);
    unsigned out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y0 = acc[i >> 1][2 * (i & 1)] * f, y1 = acc[i >> 1][2 * (i & 1) + 1] * f;
        out[i] = a.io_bf16 ? pack_bf16(y0, y1) : pack_f16(y0, y1);
    }
    *reinterpret_cast<uint4*>(a.o + ((size_t)(row0 + t) * a.Hq + hk * (int)a.G.d + h) * D + c8) = make_uint4(out[0], out[1], out[2], out[3]);
}

// One workgroup = 8 wavefronts sweeps a contiguous range of units; a range may end inside one (sequence, head, row block) and begin
// inside another, whose parts go to slots and are merged by a second kernel.  So the work is even whatever the lengths, and the host need not
// know them.  The rows are those of all query heads of a KV head: a decoding step reads its keys once.
//
// GEMMs on v_mfma_f32_16x16x32_f16, transposed: S^T = K Q^T, O^T += V^T P^T.  Lane l holds query row l % 16 and, with g = l / 16, keys
// 4g .. 4g+3 of a block of 16.  Which channels a k-step of the first GEMM consists of is free, so a lane takes 16 consecutive bytes of a
// key's row; which keys a k-step of the second consists of is free, so P needs no exchange; which channel a row of V^T is, is free too, so a lane takes D / 16
// consecutive bytes of a key's value, and the 8 keys x D / 16 channels that it holds are turned while they are widened.
//
// The value's scale is not applied to values (there are 128 of them per key, and one P per row): it goes into the exponent.  With
// t = score + log2(vscale), M the running maximum of t and P = 2^(t - M): O = sum P y, and the sum of the softmax is sum P / vscale.
// P is at most 1 (2^8 between moves of the level), so fp16 holds what matters of it whatever the scales.
template <int D, int RB, bool E4M3, bool LISTED>
__global__ __launch_bounds__(64 * kUnitsAtOnce, 2)
void pasa_cache_rows(RowsArgs a)
{
    constexpr int ROWS = 16 * RB, KS = D / 32, CB = D / 16, NW = kUnitsAtOnce, NT = 64 * NW;
    constexpr int LD = D + 4;                    // LDS row of the merge, in floats
    constexpr int VW = CB / 4;                   // words of a key's value that a lane takes
    __shared__ __attribute__((aligned(16))) float lds_o[NW * ROWS * LD];
    __shared__ __attribute__((aligned(16))) float lds_key[NW][3 * kUnit];       // per key: score factor, log2 of the value's scale, 1 / it
    __shared__ float lds_l[NW][ROWS], lds_m[NW][ROWS];
    constexpr bool QLDS = RB > 1;                // the query fragments wait in LDS: the registers are needed for RB blocks
    __shared__ __attribute__((aligned(16))) h8 lds_q[QLDS ? RB * KS * 64 : 1];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 15, g = lane >> 4;
    const int G = (int)a.G.d, most = a.c.table_width << a.page_log2, lg = a.page_log2;
    const unsigned w = logical_workgroup(blockIdx.x, gridDim.x);

    const Start at = find_start<ROWS, NT>(a, w, gridDim.x, most);
    if (at.b < 0) {
        if (tid == 0) a.records[w].pieces = 0;
        return;
    }
    unsigned left = at.left, pair = at.pair;     // units of this workgroup still to be swept
    int b = at.b, us = at.us;
    Sequence s = at.s;
    Extent x = extent_of<ROWS>(a, s);
    bool first_piece = true;
    float* const key_f = lds_key[wave];

    for (;;) {
        const int ue = (int)((unsigned)(x.units - us) < left ? x.units : us + (int)left);
        const int hk = (int)(pair / (unsigned)x.row_blocks), p0 = (int)(pair - (unsigned)hk * (unsigned)x.row_blocks) * ROWS;
        const int list = s.rows * G;             // rows of the KV head's query heads, by token, then head
        const int new0 = s.length - s.rows;      // position of the sequence's first row
        const int units = us + wave < ue ? (ue - us - wave + NW - 1) / NW : 0;      // of this wavefront

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
        if (QLDS) {
            for (int f = wave; f < RB * KS; f += NW) {
                const u16x8 raw = query(row_of(f / KS), f % KS);
                lds_q[f * 64 + lane] = a.io_bf16 ? bf16x8_to_h8(raw) : __builtin_bit_cast(h8, raw);
            }
            __syncthreads();
        }
        if (units > 0) {
            // Places of the blocks of 16 keys, lane group g that of block g, by way of the list where there is one.  Three steps, each an
            // iteration ahead of the next: the list's entry, the table's, the keys.  Entries are read at index 0 where there is no block, and not
            // used.  No load hangs on a branch: where ways with and without one meet, the compiler waits for all that is on its way.
            const int* const table = a.c.table + (size_t)b * a.c.table_width;
            const int* const chosen = LISTED ? a.blocks + ((size_t)b * a.c.Hkv + hk) * a.count : nullptr;
            int listed_a, place_b, entry_b;      // of the unit after the next two; of the one after the next
            int pos_next = 0, page_next = -1, pos_now = 0, page_now = -1;
            auto first_key = [&](int n) { return (us + wave + NW * n) * kUnit + 16 * g; };
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
            auto buffer_of = [&](void* base, int blk, int pages, int poss) {
                const int page = __builtin_amdgcn_readlane(pages, 16 * blk), pos = __builtin_amdgcn_readlane(poss, 16 * blk);
                const size_t slot = ((size_t)(unsigned)(page < 0 ? 0 : page) * (unsigned)a.c.Hkv + (unsigned)hk) * (unsigned)a.c.page + (unsigned)(pos & (a.c.page - 1));
                return __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(base) + slot * D, 0, page < 0 ? 0 : 16 * D, 0x00020000);
            };
            auto load_k = [&] {
#pragma unroll
                for (int blk = 0; blk < 4; ++blk) {
                    const __amdgpu_buffer_rsrc_t from = buffer_of(a.c.k, blk, page_next, pos_next);
#pragma unroll
                    for (int j = 0; j < D / 64; ++j) K[blk][j] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(from, koff + 64 * j, 0, 0));
                }
                // a lane a key
                const size_t slot = ((size_t)(unsigned)(page_next < 0 ? 0 : page_next) * (unsigned)a.c.Hkv + (unsigned)hk) * (unsigned)a.c.page +
                                    (unsigned)(pos_next & (a.c.page - 1)) + lq;
                ks_raw = a.c.kscale[slot];
                vs_raw = a.c.vscale[slot];
            };
            auto load_v = [&] {
#pragma unroll
                for (int blk = 0; blk < 4; ++blk) {
                    const __amdgpu_buffer_rsrc_t from = buffer_of(a.c.v, blk, page_now, pos_now);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (VW == 2) {
                            const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(from, voff + i * D, 0, 0));
                            V[blk >> 1][4 * (blk & 1) + i][0] = y.x;
                            V[blk >> 1][4 * (blk & 1) + i][VW - 1] = y.y;
                        } else {
                            V[blk >> 1][4 * (blk & 1) + i][0] = __builtin_amdgcn_raw_buffer_load_b32(from, voff + i * D, 0, 0);
                        }
                    }
                }
            };

            // query rows, and what each sees; rows behind the last one are the last one again, and not stored
            u16x8 raw[QLDS ? 1 : RB][KS];
            int last[RB];
            unsigned long long bits[RB];
            read_list(0);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int p = row_of(rb), t = (int)a.G.quotient((unsigned)p);
                last[rb] = a.tree != nullptr ? new0 - 1 : new0 + t;
                bits[rb] = a.tree != nullptr ? a.tree[s.row0 + t] : 0ull;
                if (!QLDS)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) raw[rb][ks] = query(p, ks);
            }
            read_entry(0);
            read_list(1);
            take_entry(0);
            read_entry(1);
            read_list(2);
            load_k();
            page_now = page_next, pos_now = pos_next;
            load_v();
            PASA_FENCE();
            h8 Qr[QLDS ? 1 : RB][KS];
            if (!QLDS) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) Qr[QLDS ? 0 : rb][ks] = __builtin_bit_cast(h8, raw[QLDS ? 0 : rb][ks]);
                if (a.io_bf16) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) Qr[QLDS ? 0 : rb][ks] = bf16x8_to_h8(raw[QLDS ? 0 : rb][ks]);
                }
            }
            auto Q = [&](int rb, int ks) { return QLDS ? lds_q[(rb * KS + ks) * 64 + lane] : Qr[QLDS ? 0 : rb][ks]; };

            int n = 0;
            do {
                const bool whole = __builtin_amdgcn_ballot_w64(page_now >= 0 && pos_now + 16 <= new0) == ~0ull;      // all rows see all keys of the unit
                // per key: what its score is multiplied by, and the value's scale; in the lanes' order of keys
                key_f[lane] = ks_raw * a.scale2;
                key_f[kUnit + lane] = __builtin_amdgcn_logf(vs_raw);
                key_f[2 * kUnit + lane] = __builtin_amdgcn_rcpf(vs_raw);
                __builtin_amdgcn_wave_barrier();                 // a wavefront's LDS accesses are done in order
                asm volatile("" ::: "memory");

                f4 S[RB][4];
#pragma unroll
                for (int blk = 0; blk < 4; ++blk) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) S[rb][blk] = (f4)0.f;
#pragma unroll
                    for (int j = 0; j < D / 64; ++j) {
                        const unsigned kw[4] = {K[blk][j].x, K[blk][j].y, K[blk][j].z, K[blk][j].w};
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            h8 f;
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const h2 lo = widen2<E4M3, false>(kw[2 * h + e]), hi = widen2<E4M3, true>(kw[2 * h + e]);
                                f[4 * e] = lo[0]; f[4 * e + 1] = lo[1]; f[4 * e + 2] = hi[0]; f[4 * e + 3] = hi[1];
                            }
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb)
                                S[rb][blk] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, Q(rb, 2 * j + h), S[rb][blk], 0, 0, 0);
                        }
                    }
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
                unsigned seen[RB];               // bit 4 blk + i, where not all keys are
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) seen[rb] = 0xffffu;
                if (__builtin_expect(!whole, 0)) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) seen[rb] = 0;
#pragma unroll
                    for (int blk = 0; blk < 4; ++blk) {
                        const int pos0 = __builtin_amdgcn_readlane(pos_now, 16 * blk), page = __builtin_amdgcn_readlane(page_now, 16 * blk);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int pos = pos0 + 4 * g + i, nth = pos - new0;
                            const bool there = page >= 0 && pos < s.length;
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb) {
                                const bool see = there && (pos <= last[rb] || (nth >= 0 && nth < 64 && (bits[rb] >> (nth & 63) & 1ull) != 0));
                                seen[rb] |= (unsigned)see << (4 * blk + i);
                                if (!see) S[rb][blk][i] = -__builtin_inff();
                            }
                            // what is no key may hold anything, NaN among it, and 0 times that is not 0
                            if (!there) {
#pragma unroll
                                for (int d = 0; d < VW; ++d) V[blk >> 1][4 * (blk & 1) + i][d] = 0;
                            }
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
                        const float level = row_top > M[rb] + kRise ? row_top : M[rb];
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
                        if (whole) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) l[rb] = __builtin_fmaf(e[i], inv[blk][i], l[rb]);
                        } else {                 // the scale of a key that is not seen may be NaN
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if ((seen[rb] >> (4 * blk + i) & 1u) != 0u) l[rb] = __builtin_fmaf(e[i], inv[blk][i], l[rb]);
                        }
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
                page_now = page_next, pos_now = pos_next;
                load_v();
                PASA_FENCE();
            } while (++n < units);
        }

        // ---- the wavefronts' states brought to the highest of their levels and added ----
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float sum = sum_row(l[rb]);
            if (g == 0) {
                lds_m[wave][16 * rb + lq] = M[rb];
                lds_l[wave][16 * rb + lq] = sum;
            }
            // element i of block cb is channel CB * (4 g + i) + cb
            float* dst = lds_o + (wave * ROWS + 16 * rb + lq) * LD + CB * 4 * g;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int cb = 0; cb < CB; cb += 4)
                    *reinterpret_cast<f4*>(dst + CB * i + cb) = f4{O[rb][cb][i], O[rb][cb + 1][i], O[rb][cb + 2][i], O[rb][cb + 3][i]};
        }
        __syncthreads();
        const bool complete = us == 0 && ue == x.units;
        const unsigned my_slot = 2 * w + (first_piece ? 0u : 1u);
        float* slot = a.slots + (size_t)my_slot * cache_slot_floats(RB, D);
        constexpr int STEP = NT / (D / 8);       // rows at a time, eight channels a lane
#pragma unroll
        for (int r0 = 0; r0 < ROWS; r0 += STEP) {
            const int r = r0 + tid / (D / 8), c8 = tid % (D / 8) * 8, p = p0 + r;
            if (r >= ROWS || p >= list) break;
            float level = lds_m[0][r], sum = 0.f;
#pragma unroll
            for (int i = 1; i < NW; ++i) level = __builtin_fmaxf(level, lds_m[i][r]);
            f4 acc[2] = {(f4)0.f, (f4)0.f};
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const float f = __builtin_amdgcn_exp2f(lds_m[i][r] - level);
                sum += f * lds_l[i][r];
                const float* src = lds_o + (i * ROWS + r) * LD + c8;
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
        left -= (unsigned)(ue - us);
        if (left == 0) {
            // begun here, and goes on in the ranges behind
            if (tid == 0) {
                MergeRecord m = {0, (int)my_slot, p0, list, s.row0, hk, {0, 0}};
                if (us == 0 && ue < x.units) m.pieces = clamp_int(1 + (int)(((unsigned)(x.units - ue) + at.per - 1) / at.per), 0, (int)(gridDim.x - w));
                a.records[w] = m;
            }
            return;
        }
        __syncthreads();                         // the LDS is free again
        first_piece = false;
        us = 0;
        if (++pair == (unsigned)x.row_blocks * (unsigned)a.c.Hkv) {
            pair = 0;
            do {
                if (++b >= a.c.S) {
                    if (tid == 0) a.records[w].pieces = 0;
                    return;
                }
                s = sequence_at(a.c.length, a.row_start, b, a.R, most);
            } while (s.rows == 0);
            x = extent_of<ROWS>(a, s);
        }
    }
}

// A row block that several workgroups have swept: pieces from the slot of the one that began it and the first slots of those behind it.
// Workgroup (w, r) adds row r of what workgroup w of the sweep has begun: D / 8 neighbouring lanes take a piece, eight channels each, and the
// groups of lanes are added at the end, always in the same order.
template <int D, int RB>
__global__ __launch_bounds__(kCacheThreads)
void pasa_cache_merge(RowsArgs a, FastDiv rows)
{
    constexpr int ROWS = 16 * RB, CHUNKS = D / 8, LANES = kCacheThreads / CHUNKS, AT = 4;
    __shared__ float lds_acc[4][D];
    __shared__ float lds_state[4][2];
    const unsigned w = rows.quotient(blockIdx.x);
    const MergeRecord m = a.records[w];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = (int)rows.rest(blockIdx.x, w), p = m.p0 + r;
    if (m.pieces == 0 || p >= m.list) return;
    const int c8 = tid % CHUNKS * 8;
    float level = kNoLevel, sum = 0.f;
    f4 acc[2] = {(f4)0.f, (f4)0.f};
    for (int i0 = tid / CHUNKS; i0 < m.pieces; i0 += AT * LANES) {
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
    a.page_log2 = log2_of(c.page);
    a.G = fast_div((unsigned)(Hq / c.Hkv));
    auto go = [&](auto rows, auto merge) {
        rows<<<plan.grid, 64 * kUnitsAtOnce, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || plan.grid == 1) return e;
        const long long most = (long long)R * (Hq / c.Hkv);          // rows of a block
        const unsigned each = (unsigned)(most < 16 * plan.row_blocks ? most : 16 * plan.row_blocks);
        merge<<<(unsigned)plan.grid * each, kCacheThreads, 0, stream>>>(a, fast_div(each));
        return hipGetLastError();
    };
    const bool e = c.format == PASA_CACHE_E4M3, l = blocks != nullptr;
    auto of_format = [&](auto d, auto rb) {
        constexpr int D = decltype(d)::value, RB = decltype(rb)::value;
        if (e) return l ? go(pasa_cache_rows<D, RB, true, true>, pasa_cache_merge<D, RB>) : go(pasa_cache_rows<D, RB, true, false>, pasa_cache_merge<D, RB>);
        return l ? go(pasa_cache_rows<D, RB, false, true>, pasa_cache_merge<D, RB>) : go(pasa_cache_rows<D, RB, false, false>, pasa_cache_merge<D, RB>);
    };
    auto of_rows = [&](auto d) {
        return plan.row_blocks == 1 ? of_format(d, std::integral_constant<int, 1>{}) : of_format(d, std::integral_constant<int, 2>{});
    };
    return c.d == 128 ? of_rows(std::integral_constant<int, 128>{}) : of_rows(std::integral_constant<int, 64>{});
}
