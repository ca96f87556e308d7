// Attention of a few rows per sequence over the paged 8-bit cache: pasa_cache_rows, and the merge of what its workgroups leave.
#include <hip/hip_runtime.h>
#include <stdint.h>

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

template <class T>
__device__ inline T at_bytes(const void* base, size_t uniform, unsigned lane)
{
    return *reinterpret_cast<const T*>(static_cast<const char*>(base) + uniform + lane);
}

struct RowsArgs {
    pasa_cache c;
    const unsigned short* q;
    unsigned short* o;
    const int* row_start;
    const unsigned long long* tree;
    const int* blocks;
    float* slots;
    long long row_stride;
    float scale2;                                // scale * log2(e)
    int R, Hq, count, io_bf16, page_log2;
    FastDiv G;
};

// What the workgroups share out: units of 64 keys, over sequences, KV heads and blocks of rows.
struct Shares {
    unsigned per;                                // units of a workgroup, a multiple of kUnitsAtOnce
    __device__ static inline unsigned of(unsigned total, unsigned grid)
    {
        return (total + kUnitsAtOnce * grid - 1) / (kUnitsAtOnce * grid) * kUnitsAtOnce;
    }
};

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

template <int ROWS>
__device__ inline unsigned units_of(const RowsArgs& a, int b)
{
    const Sequence s = sequence_at(a.c.length, a.row_start, b, a.R, a.c.table_width << a.page_log2);
    const Extent x = extent_of<ROWS>(a, s);
    return (unsigned)x.units * (unsigned)x.row_blocks * (unsigned)a.c.Hkv;
}

// Workgroups are dealt round-robin to the 8 XCDs; each XCD gets a contiguous range of the work, so that blocks of rows that read the
// same keys share an L2.
__device__ inline unsigned logical_workgroup(unsigned idx, unsigned grid)
{
    const unsigned x = idx & 7, whole = grid >> 3, rest = grid & 7;
    return x * whole + (x < rest ? x : rest) + (idx >> 3);
}

// One workgroup = 4 wavefronts sweeps a contiguous range of units; a range may end inside one (sequence, head, row block) and begin
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
template <int D, int RB, bool E4M3>
__global__ __launch_bounds__(kCacheThreads, 2)
void pasa_cache_rows(RowsArgs a)
{
    constexpr int ROWS = 16 * RB, KS = D / 32, CB = D / 16, NW = kUnitsAtOnce;
    constexpr int LD = D + 4;                    // LDS row of the merge, in floats
    constexpr int VW = CB / 4;                   // words of a key's value that a lane takes
    __shared__ __attribute__((aligned(16))) float lds_o[NW * ROWS * LD];
    __shared__ __attribute__((aligned(16))) float lds_key[NW][3][kUnit];        // per key: score factor, log2 of the value's scale, 1 / it
    __shared__ float lds_l[NW][ROWS], lds_m[NW][ROWS];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 15, g = lane >> 4;
    const int G = (int)a.G.d, most = a.c.table_width << a.page_log2;
    const unsigned w = logical_workgroup(blockIdx.x, gridDim.x);

    unsigned per = 0;
    const Place at = find_place(a.c.S, [&](int b) { return units_of<ROWS>(a, b); }, [&](unsigned total) {
        per = Shares::of(total, gridDim.x);
        return w * per;
    });
    if (at.b < 0) return;
    per = Shares::of(at.total, gridDim.x);
    unsigned left = at.total - w * per;          // units of this workgroup still to be swept
    if (left > per) left = per;

    int b = at.b;
    Sequence s = sequence_at(a.c.length, a.row_start, b, a.R, most);
    Extent x = extent_of<ROWS>(a, s);
    unsigned pair = at.rest / (unsigned)x.units;
    int us = (int)(at.rest - pair * (unsigned)x.units);
    bool first_piece = true;
    float* const key_f = lds_key[wave][0];

    for (;;) {
        const int ue = (int)((unsigned)(x.units - us) < left ? x.units : us + (int)left);
        const int hk = (int)(pair / (unsigned)x.row_blocks), p0 = (int)(pair - (unsigned)hk * (unsigned)x.row_blocks) * ROWS;
        const int list = s.rows * G;             // rows of the KV head's query heads, by token, then head
        const int new0 = s.length - s.rows;      // position of the sequence's first row

        // query rows, and what each sees
        h8 Q[RB][KS];
        int last[RB];
        unsigned long long bits[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int p = p0 + 16 * rb + lq;
            const bool real = p < list;
            const int t = real ? (int)a.G.quotient((unsigned)p) : 0, h = real ? (int)a.G.rest((unsigned)p, (unsigned)t) : 0;
            last[rb] = !real ? -1 : a.tree != nullptr ? new0 - 1 : new0 + t;
            bits[rb] = real && a.tree != nullptr ? a.tree[s.row0 + t] : 0ull;
            const unsigned short* row = a.q + (size_t)(s.row0 + t) * (size_t)a.row_stride + (size_t)(hk * G + h) * D + 16 * g;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                u16x8 raw = (u16x8)(unsigned short)0;
                if (real) raw = *reinterpret_cast<const u16x8*>(row + 64 * (ks / 2) + 8 * (ks & 1));
                Q[rb][ks] = a.io_bf16 ? bf16x8_to_h8(raw) : __builtin_bit_cast(h8, raw);
            }
        }

        f4 O[RB][CB];
        float M[RB], l[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            M[rb] = kNoLevel;
            l[rb] = 0.f;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) O[rb][cb] = (f4)0.f;
        }

        // Places of the wavefront's blocks of 16 keys, 64 at a time, one a lane: page in the pool (-1: no keys) and position
        int my_page = -1, my_pos = 0;
        auto look_up = [&](int n0) {             // from the wavefront's n0-th unit on
            const int u = us + wave + NW * (n0 + (lane >> 2)), vk = u * kUnit + 16 * (lane & 3);
            my_page = -1;
            my_pos = 0;
            if (u < ue && vk < x.keys) {
                int place = vk >> a.page_log2;
                if (a.blocks != nullptr) place = a.blocks[((size_t)b * a.c.Hkv + hk) * a.count + place];
                if (place >= 0 && place < a.c.table_width) {
                    my_pos = (place << a.page_log2) + (vk & (a.c.page - 1));
                    const int id = a.c.table[(size_t)b * a.c.table_width + place];
                    if (my_pos < s.length && id >= 0 && id < a.c.pages) my_page = id;
                }
            }
        };

        uint4 K[4][D / 64];
        unsigned V[2][8][VW];                    // k-step of 32 keys, key, word
        float ks_raw = 0.f, vs_raw = 0.f;
        int page_of[4], pos_of[4];               // of the unit whose keys are in K and V
        // n: the wavefront's n-th unit
        auto slot_of = [&](int n, int blk, int& page, int& pos) {
            page = __builtin_amdgcn_readlane(my_page, 4 * (n & 15) + blk);
            pos = __builtin_amdgcn_readlane(my_pos, 4 * (n & 15) + blk);
            const int id = page < 0 ? 0 : page;  // page 0 is there: what is read from it is not used
            return ((size_t)id * a.c.Hkv + hk) * a.c.page + (size_t)(pos & (a.c.page - 1));
        };
        int page_next[4], pos_next[4];
        auto load_k = [&](int n) {
            if ((n & 15) == 0) look_up(n);
#pragma unroll
            for (int blk = 0; blk < 4; ++blk) {
                const size_t slot = slot_of(n, blk, page_next[blk], pos_next[blk]);
#pragma unroll
                for (int j = 0; j < D / 64; ++j) K[blk][j] = at_bytes<uint4>(a.c.k, slot * D, lq * D + 16 * g + 64 * j);
            }
            const int mine = 4 * (n & 15) + (lane >> 4);
            const int pg = __shfl(my_page, mine), ps = __shfl(my_pos, mine);
            const size_t slot = ((size_t)(pg < 0 ? 0 : pg) * a.c.Hkv + hk) * a.c.page + (size_t)(ps & (a.c.page - 1)) + lq;
            ks_raw = a.c.kscale[slot];
            vs_raw = a.c.vscale[slot];
        };
        auto load_v = [&](int n) {
#pragma unroll
            for (int blk = 0; blk < 4; ++blk) {
                int page, pos;
                const size_t slot = slot_of(n, blk, page, pos);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned off = (4 * g + i) * D + lq * CB;
                    if constexpr (VW == 2) {
                        const uint2 y = at_bytes<uint2>(a.c.v, slot * D, off);
                        V[blk >> 1][4 * (blk & 1) + i][0] = y.x;
                        V[blk >> 1][4 * (blk & 1) + i][VW - 1] = y.y;
                    } else {
                        V[blk >> 1][4 * (blk & 1) + i][0] = at_bytes<unsigned>(a.c.v, slot * D, off);
                    }
                }
            }
        };

        const int units = us + wave < ue ? (ue - us - wave + NW - 1) / NW : 0;
        if (units > 0) {
            load_k(0);
            load_v(0);
        }
        for (int n = 0; n < units; ++n) {
            bool whole = true;                   // all rows see all keys of the unit
#pragma unroll
            for (int blk = 0; blk < 4; ++blk) {
                page_of[blk] = page_next[blk];
                pos_of[blk] = pos_next[blk];
                whole = whole && page_of[blk] >= 0 && pos_of[blk] + 16 <= new0;
            }
            // per key: what its score is multiplied by, and the value's scale; in the lanes' order of keys
            key_f[lane] = ks_raw * a.scale2;
            key_f[kUnit + lane] = __builtin_amdgcn_logf(vs_raw);
            key_f[2 * kUnit + lane] = __builtin_amdgcn_rcpf(vs_raw);
            __builtin_amdgcn_wave_barrier();     // a wavefront's LDS accesses are done in order
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
                            S[rb][blk] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, Q[rb][2 * j + h], S[rb][blk], 0, 0, 0);
                    }
                }
            }
            PASA_FENCE();
            if (n + 1 < units) load_k(n + 1);
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
            unsigned seen[RB];                   // bit 4 blk + i, where not all keys are
            if (!whole) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) seen[rb] = 0;
#pragma unroll
                for (int blk = 0; blk < 4; ++blk)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int pos = pos_of[blk] + 4 * g + i, nth = pos - new0;
                        const bool there = page_of[blk] >= 0 && pos < s.length;
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
                    for (int i = 0; i < 4; ++i) {
                        e[i] = __builtin_amdgcn_exp2f(S[rb][blk][i] - M[rb]);
                        float part = e[i] * inv[blk][i];
                        if (!whole && (seen[rb] >> (4 * blk + i) & 1u) == 0u) part = 0.f;
                        l[rb] += part;
                    }
                    const h2 lo = pack_rn(e[0], e[1]), hi = pack_rn(e[2], e[3]);
                    P[rb][blk >> 1][4 * (blk & 1)] = lo[0];
                    P[rb][blk >> 1][4 * (blk & 1) + 1] = lo[1];
                    P[rb][blk >> 1][4 * (blk & 1) + 2] = hi[0];
                    P[rb][blk >> 1][4 * (blk & 1) + 3] = hi[1];
                }
            }
            PASA_FENCE();
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int d = 0; d < VW; ++d) {
                    unsigned two[4][2];          // pairs of keys: channels 0 and 1, channels 2 and 3 of the word
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
            if (n + 1 < units) load_v(n + 1);
            PASA_FENCE();
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
        float* slot = a.slots + (size_t)(2 * w + (first_piece ? 0 : 1)) * cache_slot_floats(RB, D);
        constexpr int STEP = kCacheThreads / (D / 8);                // rows at a time, eight channels a lane
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
                const float f = sum == 0.f ? 0.f : 1.f / sum;
                const int t = (int)a.G.quotient((unsigned)p), h = (int)a.G.rest((unsigned)p, (unsigned)t);
                unsigned out[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float y0 = acc[i >> 1][2 * (i & 1)] * f, y1 = acc[i >> 1][2 * (i & 1) + 1] * f;
                    out[i] = a.io_bf16 ? pack_bf16(y0, y1) : pack_f16(y0, y1);
                }
                *reinterpret_cast<uint4*>(a.o + ((size_t)(s.row0 + t) * a.Hq + hk * G + h) * D + c8) = make_uint4(out[0], out[1], out[2], out[3]);
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
        if (left == 0) return;
        __syncthreads();                         // the LDS is free again
        first_piece = false;
        us = 0;
        if (++pair == (unsigned)x.row_blocks * (unsigned)a.c.Hkv) {
            pair = 0;
            do {
                if (++b >= a.c.S) return;
                s = sequence_at(a.c.length, a.row_start, b, a.R, most);
            } while (s.rows == 0);
            x = extent_of<ROWS>(a, s);
        }
    }
}

// The pieces of a block of rows that several workgroups have swept: workgroup w of the sweep that began it adds them up, here workgroup (w, part)
// for its share of the rows.  Pieces come in the order of the keys: the result does not depend on which was done first.
template <int D, int RB>
__global__ __launch_bounds__(kCacheThreads)
void pasa_cache_merge(RowsArgs a, unsigned grid)
{
    constexpr int ROWS = 16 * RB, STEP = kCacheThreads / (D / 8), PARTS = ROWS > STEP ? ROWS / STEP : 1;
    const int tid = threadIdx.x, G = (int)a.G.d;
    const unsigned w = blockIdx.x / PARTS, part = blockIdx.x % PARTS;
    unsigned per = 0;
    const Place at = find_place(a.c.S, [&](int b) { return units_of<ROWS>(a, b); }, [&](unsigned total) {
        per = Shares::of(total, grid);
        const unsigned end = (w + 1) * per;      // the last unit of the workgroup's range
        return (end < total ? end : total) - 1u;
    });
    if (at.b < 0) return;
    per = Shares::of(at.total, grid);
    const unsigned begin = w * per, end = begin + per;
    if (begin >= at.total || end >= at.total) return;        // nothing goes on behind the last range
    const int b = at.b;
    const Sequence s = sequence_at(a.c.length, a.row_start, b, a.R, a.c.table_width << a.page_log2);
    const Extent x = extent_of<ROWS>(a, s);
    const unsigned pair = at.rest / (unsigned)x.units, u = at.rest - pair * (unsigned)x.units;
    const unsigned first = end - 1u - u, after = first + (unsigned)x.units;      // units of the block of rows among all
    if (first < begin || after <= end) return;               // begun by another, or done
    const int hk = (int)(pair / (unsigned)x.row_blocks), p0 = (int)(pair - (unsigned)hk * (unsigned)x.row_blocks) * ROWS;
    const int r = (int)part * STEP + tid / (D / 8), c8 = tid % (D / 8) * 8, p = p0 + r;
    if (r >= ROWS || p >= s.rows * G) return;
    const unsigned w1 = (after - 1u) / per;
    auto slot_of = [&](unsigned i) { return a.slots + (size_t)(2 * i + (i == w && first != begin ? 1 : 0)) * cache_slot_floats(RB, D); };
    float level = kNoLevel;
    for (unsigned i = w; i <= w1; ++i) level = __builtin_fmaxf(level, slot_of(i)[2 * r + 1]);
    float sum = 0.f;
    f4 acc[2] = {(f4)0.f, (f4)0.f};
    for (unsigned i = w; i <= w1; ++i) {
        const float* slot = slot_of(i);
        const float f = __builtin_amdgcn_exp2f(slot[2 * r + 1] - level);
        sum += f * slot[2 * r];
        acc[0] += f * *reinterpret_cast<const f4*>(slot + 2 * ROWS + (size_t)r * D + c8);
        acc[1] += f * *reinterpret_cast<const f4*>(slot + 2 * ROWS + (size_t)r * D + c8 + 4);
    }
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    const int t = (int)a.G.quotient((unsigned)p), h = (int)a.G.rest((unsigned)p, (unsigned)t);
    unsigned out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y0 = acc[i >> 1][2 * (i & 1)] * f, y1 = acc[i >> 1][2 * (i & 1) + 1] * f;
        out[i] = a.io_bf16 ? pack_bf16(y0, y1) : pack_f16(y0, y1);
    }
    *reinterpret_cast<uint4*>(a.o + ((size_t)(s.row0 + t) * a.Hq + hk * G + h) * D + c8) = make_uint4(out[0], out[1], out[2], out[3]);
}

}  // namespace

hipError_t pasa_launch_attn_cache(const pasa_cache& c, const void* q, void* o, int R, long long row_stride, const int* row_start, int Hq,
                                  float scale, const unsigned long long* tree, const int* blocks, int count, int io_bf16,
                                  const CachePlan& plan, float* slots, hipStream_t stream)
{
    RowsArgs a;
    a.c = c;
    a.q = static_cast<const unsigned short*>(q);
    a.o = static_cast<unsigned short*>(o);
    a.row_start = row_start;
    a.tree = tree;
    a.blocks = blocks;
    a.slots = slots;
    a.row_stride = row_stride;
    a.scale2 = scale * LOG2E;
    a.R = R;
    a.Hq = Hq;
    a.count = count;
    a.io_bf16 = io_bf16;
    a.page_log2 = 0;
    while ((1 << a.page_log2) < c.page) ++a.page_log2;
    a.G = fast_div((unsigned)(Hq / c.Hkv));
    auto go = [&](auto rows, auto merge) {
        const int parts = 16 * plan.row_blocks * (c.d / 8) / kCacheThreads;
        rows<<<plan.grid, kCacheThreads, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || plan.grid == 1) return e;
        merge<<<plan.grid * (parts < 1 ? 1 : parts), kCacheThreads, 0, stream>>>(a, (unsigned)plan.grid);
        return hipGetLastError();
    };
    const bool e = c.format == PASA_CACHE_E4M3;
    if (c.d == 128) {
        if (plan.row_blocks == 1) return e ? go(pasa_cache_rows<128, 1, true>, pasa_cache_merge<128, 1>) : go(pasa_cache_rows<128, 1, false>, pasa_cache_merge<128, 1>);
        return e ? go(pasa_cache_rows<128, 2, true>, pasa_cache_merge<128, 2>) : go(pasa_cache_rows<128, 2, false>, pasa_cache_merge<128, 2>);
    }
    if (plan.row_blocks == 1) return e ? go(pasa_cache_rows<64, 1, true>, pasa_cache_merge<64, 1>) : go(pasa_cache_rows<64, 1, false>, pasa_cache_merge<64, 1>);
    return e ? go(pasa_cache_rows<64, 2, true>, pasa_cache_merge<64, 2>) : go(pasa_cache_rows<64, 2, false>, pasa_cache_merge<64, 2>);
}
