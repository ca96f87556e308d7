// The paged cache in 8 bits or 4: tokens enter (write), come back (read), and pages are chosen by their pseudo-averages (score, pick).
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "pasa_cache.h"

namespace {

// ---- tokens enter ----

constexpr float kRound = 12582912.f + 128.f;     // 1.5 2^23: a sum with it is rounded to whole numbers, and its low byte is number + 128

// Eight values of a token -> eight bytes, and the numbers that they hold.  `top`: the largest magnitude of the token, NaN where one is.
// Codes are the nearest of the exact quotients.  Products with 1 / scale are off by two steps of fp32 at most, which matters next to a tie only, and
// ties are common: fp16 and bf16 values over a multiple of one of them.  (Exact quotients as quotients: 28 instructions a value.)
//  Integers: one multiply-add rounds; where a value of the wavefront is next to a tie, x - number * scale, which fp32 holds exactly, says against scale / 2
//   whether the number is right, and a tie goes to the even one.  5 instructions a value, 13 then.
//  e4m3: the product and one correction by the exact remainder give the nearest fp32 value, and a tie of the quotient is one of that value; it
//   misleads where it is a tie and the quotient is not, as its own remainder shows, one in a million of what is no tie, and there moves by a step.  Ties are
//   where the 20 bits behind e4m3's three are a half; below 2^-6 steps are those from 2^-6 to 2^-5.  10 instructions a value.
template <bool E4M3>
__device__ inline uint2 encode8(const float (&x)[8], float top, float& scale, float (&held)[8])
{
    constexpr float most = E4M3 ? 448.f : 127.f;
    const bool finite = top < __builtin_inff();
    constexpr float part = 1.f / most;           // the quotient by way of it is the rounded one for every mantissa
    scale = top * part;
    scale = __builtin_fmaf(__builtin_fmaf(-scale, most, top), part, scale);
    if (top < 0x1p-100f) scale = 1.f;
    if (!finite) scale = __builtin_nanf("");
    const float inverse = __builtin_amdgcn_rcpf(scale);
    float q[8];
    if constexpr (E4M3) {
        float left[8];
        bool misled = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            q[i] = x[i] * inverse;
            q[i] = __builtin_fmaf(__builtin_fmaf(-q[i], scale, x[i]), inverse, q[i]);
            left[i] = __builtin_fmaf(-q[i], scale, x[i]);
            const float size = __builtin_fabsf(q[i]), as = size < 0x1p-6f ? size + 0x1p-6f : size;
            misled |= ((__float_as_uint(as) & 0xfffffu) == 0x80000u) & (left[i] != 0.f);
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(misled && finite) != 0ull, 0)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {        // the quotient where fp32 holds it, otherwise the value next to it whose last bit is set
                unsigned u = __float_as_uint(q[i]);
                if (left[i] != 0.f && q[i] != 0.f && (u & 1u) == 0u) u += (left[i] > 0.f) == (q[i] > 0.f) ? 1u : ~0u;
                q[i] = __uint_as_float(u);
            }
        }
    } else {
        float off = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            q[i] = __builtin_fmaf(x[i], inverse, kRound);
            held[i] = q[i] - kRound;
            off = __builtin_fmaxf(off, __builtin_fabsf(__builtin_fmaf(x[i], inverse, -held[i])));
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(off > 0.5f - 0x1p-15f && finite) != 0ull, 0)) {
            const unsigned half = __float_as_uint(0.5f * scale);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float r = __builtin_fmaf(-held[i], scale, x[i]);
                const float limit = __uint_as_float(half - (__float_as_uint(q[i]) & 1u));       // odd numbers move at a tie, even ones stay
                const float step = __builtin_fabsf(r) > limit ? __builtin_copysignf(1.f, r) : 0.f;
                held[i] += step;
                q[i] += step;
            }
        }
    }
    unsigned w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (E4M3) {
            const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h], q[4 * h + 1], 0, false);
            w[h] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h + 2], q[4 * h + 3], lo, true);
            if (!finite) w[h] = 0u;
            float z[4];
            widen4<true>(w[h], z);
#pragma unroll
            for (int i = 0; i < 4; ++i) held[4 * h + i] = z[i];
        } else {
            const unsigned lo = __builtin_amdgcn_perm(__float_as_uint(q[4 * h + 1]), __float_as_uint(q[4 * h]), 0x0c0c0400u);
            w[h] = lo | __builtin_amdgcn_perm(__float_as_uint(q[4 * h + 3]), __float_as_uint(q[4 * h + 2]), 0x04000c0cu);
            if (!finite) w[h] = 0x80808080u;
        }
    }
    return make_uint2(w[0], w[1]);
}

// The nearest whole number to x / unit, ties to even, where that is below 2^15 and unit has 16 significant bits: numbers times unit are exact in fp32, and so is what is left
// of x.  inverse: of unit, off by a step or two.
__device__ inline float nearest(float x, float unit, float inverse)
{
    float n = __builtin_rintf(x * inverse);
    const float left = __builtin_fabsf(__builtin_fmaf(-n, unit, x)), half = 0.5f * unit;
    const bool odd = ((int)n & 1) != 0;
    if (left > half || (left == half && odd)) n += __builtin_copysignf(1.f, __builtin_fmaf(-n, unit, x));
    return n;
}

// Eight values of a token -> eight codes of 4 bits, and the numbers factor * code that they hold.  top: the largest magnitude of the token, NaN where one is; of_group: that
// of the 32 channels that the factor is for.  All of it exact: scale has 8 significant bits, factor 8, code 3 and a half 4, so that limits are products
// that fp32 holds.  Codes from products with 1 / unit, off by 2^-18 at most, unless one of the wavefront is next to a tie.
__device__ inline unsigned encode4(const float (&x)[8], float top, float of_group, float& scale, unsigned& factor, float (&held)[8])
{
    const bool finite = top < __builtin_inff();
    constexpr float part = (float)((1.0 - 0x1p-20) / 1568.0);    // the product is below top / 1568, and by less than 8 bits show
    unsigned u = (__float_as_uint(top * part) & 0xffff0000u) + 0x10000u;
    if (__uint_as_float(u) * 1568.f < top) u += 0x10000u;
    scale = top < 0x1p-98f ? 1.f : __uint_as_float(u);
    const float group = 7.f * scale;
    float m = __builtin_fmaxf(nearest(of_group, group, __builtin_amdgcn_rcpf(group)), 1.f);
    if (!finite) scale = __builtin_nanf(""), m = 1.f;
    factor = (unsigned)m;
    const float unit = m * scale, inverse = __builtin_amdgcn_rcpf(unit);
    constexpr float shift = 12582912.f + 8.f;    // 1.5 2^23: a sum with it is rounded to whole numbers, and its low bits are number + 8
    float q[8], off = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = __builtin_amdgcn_fmed3f(x[i] * inverse, -7.f, 7.f);
        q[i] = y + shift;
        held[i] = q[i] - shift;
        off = __builtin_fmaxf(off, __builtin_fabsf(y - held[i]));
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(off > 0.5f - 0x1p-15f && finite) != 0ull, 0)) {     // next to a tie somewhere
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            held[i] = __builtin_amdgcn_fmed3f(nearest(x[i], unit, inverse), -7.f, 7.f);
            q[i] = held[i] + shift;
        }
    }
    // the low bytes, numbers + 8, of the even ones and of the odd ones side by side, and these between those
    unsigned half[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
        half[h] = __builtin_amdgcn_perm(__float_as_uint(q[2 + h]), __float_as_uint(q[h]), 0x0c0c0400u) |
                  __builtin_amdgcn_perm(__float_as_uint(q[6 + h]), __float_as_uint(q[4 + h]), 0x04000c0cu);
    unsigned word = half[0] | half[1] << 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) held[i] *= m;
    if (!finite) {
        word = 0x88888888u;
#pragma unroll
        for (int i = 0; i < 8; ++i) held[i] = 0.f;
    }
    return word;
}

// Eight codes of 4 bits and their factor -> fp32, exactly
__device__ inline void widen8(unsigned w, unsigned factor, float (&x)[8])
{
    const float m = (float)factor;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = ((float)((w >> (4 * i)) & 15u) - 8.f) * m;
}

__device__ inline void widen_io(u16x8 raw, int io_bf16, float (&x)[8])
{
    if (io_bf16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float((unsigned)raw[i] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)__builtin_bit_cast(_Float16, (unsigned short)raw[i]);
    }
}

// Largest of x over LANES neighbouring lanes (4, 8 or 16), NaN where one is
template <int LANES>
__device__ inline float largest(float x)
{
    auto with = [&](auto control) {
        const float y = __uint_as_float((unsigned)__builtin_amdgcn_update_dpp((int)__float_as_uint(x), (int)__float_as_uint(x), decltype(control)::value, 0xf, 0xf, false));
        x = __builtin_elementwise_maximum(x, y);
    };
    with(std::integral_constant<int, 0xb1>{});       // lane ^ 1, ^ 2 (quads), 7 - lane of 8, 15 - lane of 16
    with(std::integral_constant<int, 0x4e>{});
    if (LANES >= 8) with(std::integral_constant<int, 0x141>{});
    if (LANES == 16) with(std::integral_constant<int, 0x140>{});
    return x;
}

// Where piece `want` of work lies that is shared out over the sequences, of which one has count(sequence) pieces: in sequence `b`, the `rest`-th
// there; b < 0 where there is no such piece.  All NT threads call it.  Up to 64 sequences a wavefront has one a lane and needs no other; otherwise every thread
// counts its own share of them, one scan over the threads finds who has the piece, and that one walks its share (a single one up to NT
// sequences) and leaves what it has read: nothing is waited for twice.
struct Place {
    int b;
    unsigned rest;
    Sequence s;
};
template <int NT, class Count>
__device__ inline Place find_place(const int* __restrict__ length, const int* __restrict__ row_start, int S, int R, int most, unsigned want, Count count)
{
    __shared__ unsigned sums[NT / 64];
    __shared__ int found[5];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Place p;
    if (__builtin_expect(S <= 64, 1)) {
        Sequence s = {0, 0, 0};
        unsigned mine = 0;
        if (lane < S) {
            s = sequence_at(length, row_start, lane, R, most);
            mine = count(s);
        }
        const unsigned upto = scan64(mine);
        const unsigned before = upto - mine;
        const unsigned long long who = __builtin_amdgcn_ballot_w64(want >= before && want < upto);
        p.b = -1;
        if (who != 0ull) {
            p.b = __builtin_ctzll(who);
            p.rest = want - (unsigned)__builtin_amdgcn_readlane((int)before, p.b);
            p.s.length = __builtin_amdgcn_readlane(s.length, p.b);
            p.s.row0 = __builtin_amdgcn_readlane(s.row0, p.b);
            p.s.rows = __builtin_amdgcn_readlane(s.rows, p.b);
        }
        return p;
    }
    const int each = (S + NT - 1) / NT, b0 = tid * each;
    Sequence s = {0, 0, 0};
    unsigned mine = 0;
    for (int i = 0; i < each; ++i)
        if (b0 + i < S) {
            s = sequence_at(length, row_start, b0 + i, R, most);
            mine += count(s);
        }
    const unsigned upto = scan64(mine);
    if (tid == 0) found[0] = -1;
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    unsigned before = upto - mine;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w)
        if (w < wave) before += sums[w];
    if (want >= before && want < before + mine) {
        int b = b0;
        unsigned left = want - before;
        if (each > 1)
            for (;; ++b) {
                if (b >= S || b >= b0 + each) {      // not as it was counted: somebody writes to length or row_start meanwhile
                    b = -1;
                    break;
                }
                s = sequence_at(length, row_start, b, R, most);
                const unsigned c = count(s);
                if (left < c) break;
                left -= c;
            }
        found[0] = b;
        found[1] = (int)left;
        found[2] = s.length;
        found[3] = s.row0;
        found[4] = s.rows;
    }
    __syncthreads();
    p.b = __builtin_amdgcn_readfirstlane(found[0]);
    p.rest = (unsigned)__builtin_amdgcn_readfirstlane(found[1]);
    p.s.length = __builtin_amdgcn_readfirstlane(found[2]);
    p.s.row0 = __builtin_amdgcn_readfirstlane(found[3]);
    p.s.rows = __builtin_amdgcn_readfirstlane(found[4]);
    return p;
}

// One workgroup per page that is written to and KV head: D / 8 neighbouring lanes take a token.  Where means are kept, the page's
// older tokens are read too: a mean made from all tokens is the same whatever the steps that brought them, and writing a
// token again corrects it.  Partial sums of the lanes that share channels are added in a fixed order.
// What bounds it: a step, what is waited for in turn (lengths, the table's entry, tokens: 16 tokens 4.3 us); prompts, the vector unit (10 to 16 instructions a
// value) and memory: 32768 tokens on 8 heads, integers, 201 MB, 45 us, 4.5 TB/s; 13924 on 4, e4m3, 43.5 MB, 16.3 us, 2.7 TB/s, with few workgroups to a
// compute unit.  In 4 bits the same 13924 tokens on 4 heads take 14.2 us (tokens one or four at a time 0.3 and 1.3 more, stores past the L2s 3.4, keys and
// values by workgroups of their own 2.1).
template <int D, int FORMAT, int NT>
__global__ __launch_bounds__(NT)
void pasa_cache_write_k(pasa_cache c, const unsigned short* __restrict__ k, const unsigned short* __restrict__ v, int R, long long row_stride,
                        const int* __restrict__ row_start, int io_bf16, int page_log2, FastDiv heads)
{
    constexpr bool E4M3 = FORMAT == PASA_CACHE_E4M3, I4 = FORMAT == PASA_CACHE_I4;
    constexpr int LT = D / 8, AT = NT / LT, BATCH = 2;   // lanes of a token, tokens at a time, of which so many are on their way
    __shared__ __attribute__((aligned(16))) float sums[AT][D];
    const int tid = threadIdx.x, lt = tid % LT, t0 = tid / LT;
    const int most = c.table_width << page_log2;
    // workgroups of a page's heads follow one another
    const unsigned piece = heads.quotient(blockIdx.x);
    const int hk = (int)heads.rest(blockIdx.x, piece);
    f4 shift[2] = {(f4)0.f, (f4)0.f};
    if (c.kshift != nullptr) {
        shift[0] = *reinterpret_cast<const f4*>(c.kshift + hk * D + 8 * lt);
        shift[1] = *reinterpret_cast<const f4*>(c.kshift + hk * D + 8 * lt + 4);
    }
    auto first_page = [&](const Sequence& s) { return (s.length > s.rows ? s.length - s.rows : 0) >> page_log2; };
    const Place at = find_place<NT>(c.length, row_start, c.S, R, most, piece, [&](const Sequence& s) {
        return s.rows == 0 || s.length == 0 ? 0u : (unsigned)(((s.length - 1) >> page_log2) - first_page(s) + 1);
    });
    if (at.b < 0) return;
    const Sequence s = at.s;
    const int place = first_page(s) + (int)at.rest, pos0 = place << page_log2;
    const int id = c.table[(size_t)at.b * c.table_width + place];
    if (id < 0 || id >= c.pages) return;
    const int tokens = s.length - pos0 < c.page ? s.length - pos0 : c.page;      // of the page
    const int fresh = s.length - s.rows - pos0;                                  // the first new one, when not negative
    const size_t slot = ((size_t)id * c.Hkv + hk) * c.page;
    const size_t first_byte = slot * (I4 ? token_bytes4(D) : D);
    unsigned char* kc = static_cast<unsigned char*>(c.k) + first_byte;
    unsigned char* vc = static_cast<unsigned char*>(c.v) + first_byte;
    auto factor_at = [&](int t) { return c.page * (D / 2) + t * (D / kFactorChannels) + lt / (kFactorChannels / 8); };
    const bool means = c.kmean != nullptr;

    f4 sum[2] = {(f4)0.f, (f4)0.f};
    for (int begin = means || fresh < 0 ? 0 : fresh / AT * AT; begin < tokens; begin += BATCH * AT) {
        u16x8 kraw[BATCH], vraw[BATCH];
        uint2 older[BATCH];                      // in 4 bits codes and a factor
        float older_scale[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            const int t = begin + j * AT + t0;
            if (t < tokens && t >= fresh) {
                const size_t row = (size_t)(s.row0 + t - fresh) * (size_t)row_stride + (size_t)hk * D + 8 * lt;
                kraw[j] = *reinterpret_cast<const u16x8*>(k + row);
                vraw[j] = *reinterpret_cast<const u16x8*>(v + row);
            }
            if (t < tokens && t < fresh && means) {
                if constexpr (I4) {
                    older[j].x = *reinterpret_cast<const unsigned*>(kc + t * (D / 2) + 4 * lt);
                    older[j].y = kc[factor_at(t)];
                } else {
                    older[j] = *reinterpret_cast<const uint2*>(kc + (size_t)t * D + 8 * lt);
                }
                older_scale[j] = c.kscale[slot + t];
            }
        }
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            const int t = begin + j * AT + t0;
            if (t >= tokens) continue;                           // all lanes of a token go the same way
            float held[8], scale;
            if (t >= fresh) {
                float x[8], y[8], unused[8], vscale;
                widen_io(kraw[j], io_bf16, x);
                widen_io(vraw[j], io_bf16, y);
                float top_k = 0.f, top_v = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] -= shift[i >> 2][i & 3];
                    top_k = __builtin_elementwise_maximum(top_k, __builtin_fabsf(x[i]));
                    top_v = __builtin_elementwise_maximum(top_v, __builtin_fabsf(y[i]));
                }
                if constexpr (I4) {
                    unsigned kfactor, vfactor;
                    const unsigned vcode = encode4(y, largest<LT>(top_v), largest<4>(top_v), vscale, vfactor, unused);
                    const unsigned code = encode4(x, largest<LT>(top_k), largest<4>(top_k), scale, kfactor, held);
                    *reinterpret_cast<unsigned*>(kc + t * (D / 2) + 4 * lt) = code;
                    *reinterpret_cast<unsigned*>(vc + t * (D / 2) + 4 * lt) = vcode;
                    if (lt % 4 == 0) {
                        kc[factor_at(t)] = (unsigned char)kfactor;
                        vc[factor_at(t)] = (unsigned char)vfactor;
                    }
                } else {
                    const uint2 vcode = encode8<E4M3>(y, largest<LT>(top_v), vscale, unused);
                    const uint2 code = encode8<E4M3>(x, largest<LT>(top_k), scale, held);
                    *reinterpret_cast<uint2*>(kc + (size_t)t * D + 8 * lt) = code;
                    *reinterpret_cast<uint2*>(vc + (size_t)t * D + 8 * lt) = vcode;
                }
                if (lt == 0) {
                    c.kscale[slot + t] = scale;
                    c.vscale[slot + t] = vscale;
                }
            } else {
                if (!means) continue;
                scale = older_scale[j];
                if constexpr (I4) {
                    widen8(older[j].x, older[j].y, held);
                } else {
                    float lo[4], hi[4];
                    widen4<E4M3>(older[j].x, lo);
                    widen4<E4M3>(older[j].y, hi);
#pragma unroll
                    for (int i = 0; i < 4; ++i) held[i] = lo[i], held[4 + i] = hi[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i >> 2][i & 3] = __builtin_fmaf(held[i], scale, sum[i >> 2][i & 3]);
        }
    }
    if (!means) return;
    *reinterpret_cast<f4*>(&sums[t0][8 * lt]) = sum[0];
    *reinterpret_cast<f4*>(&sums[t0][8 * lt + 4]) = sum[1];
    __syncthreads();
    if (tid < D) {
        float total = 0.f;
#pragma unroll
        for (int i = 0; i < AT; ++i) total += sums[i][tid];
        c.kmean[((size_t)id * c.Hkv + hk) * D + tid] = total / (float)tokens;
    }
}

// ---- tokens come back ----

// D / 8 neighbouring lanes take a token, eight channels each, so that a wavefront's stores are 1 KiB of neighbouring bytes; a workgroup takes
// read_tokens(D) positions of one sequence and head.  The loads are asked for together: places, then codes and scales.
// STREAM: outputs of which the eight L2s would keep nothing are stored past them (two sequences of 32768 tokens on 4 heads, 134 MB of output:
// 31.9 us, 6.4 TB/s; through the L2s 42.4); smaller ones stay there for the one who reads them next (14 x 5 heads, d = 64, 2304 tokens, 21 MB each: 11.5 us, past
// them 11.9).  Out of 4 bits, four sequences of 8192 tokens on 4 heads, 75 MB: 14.5 us.
// Numbers of the type come back as such: one that rounding to its code, or the vector taken off it, leaves beyond the type's largest, by no more than a code
// may be off, is the largest.  A code is off by half a step (of 16 scales among the largest e4m3 codes), with 4 bits also where a factor's rounding, up to 3.5 scales, cuts the largest.
// Only wavefronts whose scales allow for such numbers look at values (four prompts' tokens in 4 bits, written and read, 28.3 us; if all look, 28.8; if none, 28.0).
constexpr int kReadBatch = 4;
constexpr int read_tokens(int d) { return kReadBatch * kCacheThreads / (d / 8); }
constexpr size_t kStreamBytes = (size_t)32 << 20;
typedef unsigned u4 __attribute__((ext_vector_type(4)));
template <int D, int FORMAT, bool STREAM>
__global__ __launch_bounds__(kCacheThreads)
void pasa_cache_read_k(pasa_cache c, unsigned short* __restrict__ k, unsigned short* __restrict__ v, const int* __restrict__ first, int N,
                       int io_bf16, int page_log2, FastDiv heads, FastDiv chunks)
{
    constexpr bool E4M3 = FORMAT == PASA_CACHE_E4M3, I4 = FORMAT == PASA_CACHE_I4;
    constexpr int LT = D / 8, AT = kCacheThreads / LT, BATCH = kReadBatch;
    const float most = io_bf16 ? kMostBf16 : kMostF16;
    const int tid = threadIdx.x, lt = tid % LT, t0 = tid / LT;
    const unsigned up = chunks.quotient(blockIdx.x);
    const int n1 = (int)chunks.rest(blockIdx.x, up) * read_tokens(D);
    const int b = (int)heads.quotient(up), hk = (int)heads.rest(up, (unsigned)b);
    const int length = clamp_int(c.length[b], 0, c.table_width << page_log2), begin = first != nullptr ? first[b] : 0;
    f4 shift[2] = {(f4)0.f, (f4)0.f};
    if (c.kshift != nullptr) {
        shift[0] = *reinterpret_cast<const f4*>(c.kshift + hk * D + 8 * lt);
        shift[1] = *reinterpret_cast<const f4*>(c.kshift + hk * D + 8 * lt + 4);
    }
    int id[BATCH], pos[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
        const long long p = (long long)begin + n1 + j * AT + t0;
        const bool in = n1 + j * AT + t0 < N && p >= 0 && p < length;
        pos[j] = in ? (int)p : -1;
        id[j] = c.table[(size_t)b * c.table_width + (in ? (int)p >> page_log2 : 0)];
    }
    uint2 code[BATCH][2];
    float scale[BATCH][2];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
        if (pos[j] < 0 || id[j] < 0 || id[j] >= c.pages) pos[j] = -1;
        const size_t slot = pos[j] < 0 ? 0 : (((size_t)id[j] * c.Hkv + hk) << page_log2) + (size_t)(pos[j] & (c.page - 1));
        if constexpr (I4) {                      // a word of codes, a factor
            const size_t at = pos[j] < 0 ? 0 : (size_t)(pos[j] & (c.page - 1)), first_byte = (slot - at) * token_bytes4(D);
            const size_t codes = first_byte + at * (D / 2) + 4 * lt;
            const size_t factor = first_byte + (size_t)c.page * (D / 2) + at * (D / kFactorChannels) + lt / (kFactorChannels / 8);
            code[j][0].x = *reinterpret_cast<const unsigned*>(static_cast<const unsigned char*>(c.k) + codes);
            code[j][1].x = *reinterpret_cast<const unsigned*>(static_cast<const unsigned char*>(c.v) + codes);
            code[j][0].y = static_cast<const unsigned char*>(c.k)[factor];
            code[j][1].y = static_cast<const unsigned char*>(c.v)[factor];
        } else {
            code[j][0] = *reinterpret_cast<const uint2*>(static_cast<const unsigned char*>(c.k) + slot * D + 8 * lt);
            code[j][1] = *reinterpret_cast<const uint2*>(static_cast<const unsigned char*>(c.v) + slot * D + 8 * lt);
        }
        scale[j][0] = c.kscale[slot];
        scale[j][1] = c.vscale[slot];
    }
    auto finish = [&](int j, auto near_most) {
        const int n = n1 + j * AT + t0;
        const size_t to = (((size_t)b * heads.d + hk) * N + n) * D + 8 * lt;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            unsigned out[4];
            float wide[8];
            if constexpr (I4) widen8(code[j][which].x, code[j][which].y, wide);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[4];
                if constexpr (I4) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = wide[4 * h + i];
                } else {
                    widen4<E4M3>(h == 0 ? code[j][which].x : code[j][which].y, x);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = pos[j] >= 0 ? __builtin_fmaf(x[i], scale[j][which], which == 0 ? shift[h][i] : 0.f) : 0.f;
                    if constexpr (decltype(near_most)::value) {
                        // 2^-20: the roundings of the difference from kshift and of the sum with it
                        const float off = (I4 ? 0.5f * (float)code[j][which].y + 3.5f : E4M3 ? 16.f : 0.5f) * scale[j][which];
                        if (__builtin_fabsf(x[i]) <= most + 0x1p-20f * most + off) x[i] = __builtin_amdgcn_fmed3f(x[i], -most, most);
                    }
                }
                out[2 * h] = io_bf16 ? pack_bf16(x[0], x[1]) : pack_f16(x[0], x[1]);
                out[2 * h + 1] = io_bf16 ? pack_bf16(x[2], x[3]) : pack_f16(x[2], x[3]);
            }
            u4* dst = reinterpret_cast<u4*>((which == 0 ? k : v) + to);
            const u4 x = {out[0], out[1], out[2], out[3]};
            if (STREAM) __builtin_nontemporal_store(x, dst);
            else *dst = x;
        }
    };
    float top_shift = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top_shift = __builtin_fmaxf(top_shift, __builtin_fabsf(shift[i >> 2][i & 3]));
    constexpr float most_code = I4 ? 8.f * 255.f : E4M3 ? 448.f : 128.f;
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
        if (n1 + j * AT + t0 >= N) break;
        // whether any value of the wavefront may be larger than the type's numbers
        const float top_scale = __builtin_fmaxf(__builtin_fabsf(scale[j][0]), __builtin_fabsf(scale[j][1]));
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(__builtin_fmaf(most_code, top_scale, top_shift) >= most) == 0ull, 1)) finish(j, std::false_type{});
        else finish(j, std::true_type{});
    }
}

// ---- pages are chosen ----

// Scores as words that order like them: larger scores, larger words.  0 stands for a page that is not there, the largest word for one that is always
// taken, the one before it for NaN.
constexpr unsigned long long kAlways = ~0ull;
__device__ inline unsigned long long order_of(double x)
{
    if (x != x) return kAlways - 1;
    const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);      // -0 becomes 0
    return (u >> 63) != 0 ? ~u : u | 0x8000000000000000ull;
}

// One wavefront takes 16 pages of a sequence and head, on v_mfma_f64_16x16x4f64: rows of queries times means, lane l with g = l / 16 holding
// a quarter of the channels (D / 4 from D / 4 * g on; which channels a k-step consists of is free) of query row and of page l % 16.
// The products of fp16 queries and fp32 means are exact in 64 bits, and so, nearly, are their sums: which pages are chosen does
// not depend on an order of additions unless two scores agree to 15 digits.  A wavefront's 32 steps (d = 128) take the matrix unit 0.9 us; what
// bounds it is what hangs on one another, lengths, table, means: 16 sequences of up to 512 pages on 4 heads, 8.6 MB, 7.5 us.
typedef double d4 __attribute__((ext_vector_type(4)));
template <int D>
__global__ __launch_bounds__(kCacheThreads)
void pasa_cache_score_k(pasa_cache c, const unsigned short* __restrict__ q, int R, long long row_stride, const int* __restrict__ row_start,
                        int head, int tail, int io_bf16, int page_log2, FastDiv G, FastDiv heads, FastDiv chunks, unsigned long long* __restrict__ scores)
{
    constexpr int CH = D / 4;                    // channels of a lane
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
    const unsigned up = chunks.quotient(blockIdx.x);
    const int b = (int)heads.quotient(up), hk = (int)heads.rest(up, (unsigned)b);
    const int p0 = (int)chunks.rest(blockIdx.x, up) * 64 + 16 * (int)(threadIdx.x >> 6), p = p0 + l16;
    const int wanted = p < c.table_width ? p : c.table_width - 1;
    const int id_read = c.table[(size_t)b * c.table_width + wanted];
    const Sequence s = sequence_at(c.length, row_start, b, R, c.table_width << page_log2);
    const int pages = (s.length + c.page - 1) >> page_log2;
    if (p0 >= pages || s.rows == 0) return;      // nobody reads these words
    const bool there = p < pages && id_read >= 0 && id_read < c.pages;
    const float* mean = c.kmean + ((size_t)(there ? id_read : 0) * c.Hkv + hk) * D + CH * g;
    f4 m[CH / 4];
#pragma unroll
    for (int i = 0; i < CH / 4; ++i) m[i] = *reinterpret_cast<const f4*>(mean + 4 * i);
    double best = -__builtin_inf();
    bool nan = false;
    const int all = s.rows * (int)G.d;
    for (int r0 = 0; r0 < all; r0 += 16) {
        const int r = r0 + l16 < all ? r0 + l16 : all - 1;       // the last one again: the maximum is the same
        const int t = (int)G.quotient((unsigned)r), h = (int)G.rest((unsigned)r, (unsigned)t);
        const unsigned short* row = q + (size_t)(s.row0 + t) * (size_t)row_stride + (size_t)(hk * (int)G.d + h) * D + CH * g;
        u16x8 raw[CH / 8];
#pragma unroll
        for (int i = 0; i < CH / 8; ++i) raw[i] = *reinterpret_cast<const u16x8*>(row + 8 * i);
        d4 x = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int i = 0; i < CH / 8; ++i) {
            float y[8];
            widen_io(raw[i], io_bf16, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x = __builtin_amdgcn_mfma_f64_16x16x4f64((double)y[e], (double)m[2 * i + (e >> 2)][e & 3], x, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {            // rows, of page l % 16
            nan |= x[i] != x[i];
            best = __builtin_fmax(best, x[i]);
        }
    }
    best = __builtin_fmax(best, __shfl_xor(best, 16));
    best = __builtin_fmax(best, __shfl_xor(best, 32));
    const unsigned long long nans = __builtin_amdgcn_ballot_w64(nan);
    nan = ((nans | nans >> 16 | nans >> 32 | nans >> 48) >> l16 & 1ull) != 0ull;
    if (g == 0 && p < pages) {
        const bool always = p < head || p >= pages - tail;
        scores[((size_t)b * c.Hkv + hk) * c.table_width + p] = always ? kAlways : !there ? 1ull : nan ? kAlways - 1 : order_of(best);
    }
}

// One workgroup per sequence and head.  The pages that are always taken leave first; of the others the want-th largest word is found
// digit by digit, 8 bits at a time, from the first bit on of the largest one's distance from the least (signs and exponents of scores are much alike), until
// the words that share the digits so far are all taken (one sequence of 4096 pages on 4 heads 6.4 us, with digits from the first bit on that words differ in 7.4).  Words above it are taken, and of its equals the first.  They leave in order.
// NT threads of EACH words: 256 of 4 for tables up to 1024 pages (16 x 4 of up to 512 pages 4.0 us, with 1024 threads and all 64 bits 6.7), which a barrier costs less.
template <int NT, int EACH>
__global__ __launch_bounds__(NT)
void pasa_cache_pick_k(pasa_cache c, const int* __restrict__ row_start, int R, int count, int page_log2, FastDiv heads,
                       const unsigned long long* __restrict__ scores, int* __restrict__ blocks)
{
    constexpr int NW = NT / 64;
    __shared__ unsigned bins[256];
    __shared__ unsigned sums[NW][2];
    __shared__ unsigned range[NW][3];
    __shared__ unsigned digit_found, above_found, done;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = (int)heads.quotient(blockIdx.x);
    const unsigned long long* in = scores + (size_t)blockIdx.x * c.table_width;
    // thread t has the words t * EACH .. : in order.  Read before the length is there; words behind the last page hold anything.
    unsigned long long word[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) word[i] = in[tid * EACH + i < c.table_width ? tid * EACH + i : 0];
    const Sequence s = sequence_at(c.length, row_start, b, R, c.table_width << page_log2);
    const int pages = s.rows == 0 ? 0 : (s.length + c.page - 1) >> page_log2;
    int* out = blocks + (size_t)blockIdx.x * count;
    const int taken = pages < count ? pages : count;
    for (int i = taken + tid; i < count; i += NT) out[i] = -1;
    if (pages <= count) {
        for (int i = tid; i < pages; i += NT) out[i] = i;
        return;
    }
    unsigned counts = 0;                         // always taken, and above << 16 of the others those that are not negative
    unsigned least = ~0u, least_up = ~0u, largest = 0;           // upper halves of those that are not always taken; of those that are not negative
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (tid * EACH + i >= pages) word[i] = 0ull;
        else if (word[i] == kAlways) ++counts;
        else {
            const unsigned x = (unsigned)(word[i] >> 32), up = x >> 31 != 0u ? x : ~0u;
            counts += x >> 31 << 16;
            least_up = min(least_up, up);
            least = min(least, x);
            largest = max(largest, x);
        }
    }
    unsigned n_all = scan64(counts);
    least = ~largest64(~least), least_up = ~largest64(~least_up), largest = largest64(largest);
    if (lane == 63) sums[wave][0] = n_all, range[wave][0] = least, range[wave][1] = least_up, range[wave][2] = largest;
    __syncthreads();
    n_all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        n_all += sums[w][0];
        least = min(least, range[w][0]);
        least_up = min(least_up, range[w][1]);
        largest = max(largest, range[w][2]);
    }
    const unsigned n_always = n_all & 0xffffu;
    // `limit`: words above it are taken, of its equals `want`; both seen from bit `shift` on
    unsigned long long limit = kAlways;
    unsigned want = (unsigned)count;
    int shift = 0;
    if (n_always < want) {
        want -= n_always;
        // What is counted from the least that may be the limit (its upper half) has exponents side by side in its digits; 0 is what lies below.
        if ((n_all >> 16) >= want) least = least_up;
        const unsigned long long base = (unsigned long long)least << 32, one = least != 0u ? 1ull : 0ull;
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (word[i] != kAlways) word[i] = word[i] >= base ? word[i] - base + one : 0ull;
        const int top = 63 - __builtin_clzll(((unsigned long long)(largest - least) << 32 | 0xffffffffull) + one);
        shift = top - 7;                         // top is 31 at least
        limit = 0ull;
        for (int from = top + 1;;) {             // the digit in hand: bits shift .. from - 1
            for (int i = tid; i < 256; i += NT) bins[i] = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (tid * EACH + i < pages && word[i] != kAlways && (from >= 64 || (word[i] >> from) == (limit >> from)))
                    atomicAdd(&bins[(word[i] >> shift) & ((1u << (from - shift)) - 1u)], 1u);
            __syncthreads();
            if (tid < 64) {                      // four bins a lane, from the top: lane 0 has 255 .. 252
                unsigned mine[4], total = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) total += mine[i] = bins[255 - 4 * lane - i];
                const unsigned upto = scan64(total);
                unsigned above = upto - total;
                if (above < want && want <= upto) {
                    int i = 0;
#pragma unroll
                    for (int j = 0; j < 3; ++j)
                        if (i == j && above + mine[j] < want) above += mine[j], ++i;
                    const unsigned here = i == 0 ? mine[0] : i == 1 ? mine[1] : i == 2 ? mine[2] : mine[3];
                    digit_found = 255u - 4u * lane - i;
                    above_found = above;
                    done = above + here == want;
                }
            }
            __syncthreads();
            limit |= (unsigned long long)digit_found << shift;
            want -= above_found;
            if (done || shift == 0) break;
            // the last digit has the bits that are left: with 8, words above the limit, which `want` no longer counts, would be counted again
            from = shift;
            shift = shift < 8 ? 0 : shift - 8;
        }
    }
    // pages that are always taken count as above, or, where there are more of them than wanted, as the equals
    const bool room = n_always < (unsigned)count;
    auto is_above = [&](unsigned long long x) { return x == kAlways ? room : (x >> shift) > (limit >> shift); };
    auto is_equal = [&](unsigned long long x) { return x == kAlways ? !room : (x >> shift) == (limit >> shift); };
    unsigned above = 0, equal = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        above += is_above(word[i]);
        equal += is_equal(word[i]);
    }
    unsigned at_a = scan64(above), at_e = scan64(equal);
    __syncthreads();
    if (lane == 63) sums[wave][0] = at_a, sums[wave][1] = at_e;
    __syncthreads();
    at_a -= above, at_e -= equal;
#pragma unroll
    for (int w = 0; w < NW; ++w)
        if (w < wave) at_a += sums[w][0], at_e += sums[w][1];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const bool a = is_above(word[i]), e = is_equal(word[i]);
        if (a || (e && at_e < want)) out[at_a + (at_e < want ? at_e : want)] = tid * EACH + i;
        at_a += a;
        at_e += e;
    }
}

}  // namespace

hipError_t pasa_launch_cache_write(const pasa_cache& c, const void* k, const void* v, int R, long long row_stride, const int* row_start,
                                   int io_bf16, hipStream_t stream)
{
    // a sequence of n rows writes to (n - 1) / page + 2 pages at most, and to n at most
    const long pages = (long)R / c.page + 2 * (long)c.S;
    const unsigned grid = (unsigned)((pages < R ? pages : R) * c.Hkv);
    // Threads that take a page in four steps of d / 8 lanes a token, 256 at least: two on their way at a time, and several workgroups to a compute unit.  us in
    // four steps / two / eight: 14000 tokens, 4 heads, d = 128, pages of 128 tokens, e4m3 18.7 / 21.2 / 21.2, of 64, integers 13.0 / 14.7 / 13.0;
    // 777 tokens in pages of 128 7.4 / 7.2 / 9.8
    const int lanes = c.page * (c.d / 8);
    auto go = [&](auto kernel, int threads) {
        kernel<<<grid, threads, 0, stream>>>(c, static_cast<const unsigned short*>(k), static_cast<const unsigned short*>(v), R, row_stride, row_start,
                                             io_bf16, log2_of(c.page), fast_div(c.Hkv));
    };
    auto of_threads = [&](auto d, auto nt) {
        constexpr int D = decltype(d)::value, NT = decltype(nt)::value;
        if (c.format == PASA_CACHE_I4) go(pasa_cache_write_k<D, PASA_CACHE_I4, NT>, NT);
        else if (c.format == PASA_CACHE_E4M3) go(pasa_cache_write_k<D, PASA_CACHE_E4M3, NT>, NT);
        else go(pasa_cache_write_k<D, PASA_CACHE_I8, NT>, NT);
    };
    auto of_size = [&](auto d) {
        if (lanes <= 1024) of_threads(d, std::integral_constant<int, 256>{});
        else of_threads(d, std::integral_constant<int, 512>{});
    };
    c.d == 128 ? of_size(std::integral_constant<int, 128>{}) : of_size(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

hipError_t pasa_launch_cache_read(const pasa_cache& c, void* k, void* v, const int* first, int N, int io_bf16, hipStream_t stream)
{
    const int each = read_tokens(c.d);
    const unsigned chunks = (unsigned)((N + each - 1) / each), grid = chunks * (unsigned)c.S * (unsigned)c.Hkv;
    auto go = [&](auto kernel) {
        kernel<<<grid, kCacheThreads, 0, stream>>>(c, static_cast<unsigned short*>(k), static_cast<unsigned short*>(v), first, N, io_bf16, log2_of(c.page),
                                                   fast_div(c.Hkv), fast_div(chunks));
    };
    const bool far = (size_t)4 * c.S * c.Hkv * N * c.d > kStreamBytes;
    auto of_size = [&](auto d) {
        constexpr int D = decltype(d)::value;
        auto held_as = [&](auto format) {
            constexpr int FORMAT = decltype(format)::value;
            far ? go(pasa_cache_read_k<D, FORMAT, true>) : go(pasa_cache_read_k<D, FORMAT, false>);
        };
        if (c.format == PASA_CACHE_I4) held_as(std::integral_constant<int, PASA_CACHE_I4>{});
        else if (c.format == PASA_CACHE_E4M3) held_as(std::integral_constant<int, PASA_CACHE_E4M3>{});
        else held_as(std::integral_constant<int, PASA_CACHE_I8>{});
    };
    c.d == 128 ? of_size(std::integral_constant<int, 128>{}) : of_size(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

hipError_t pasa_launch_cache_choose(const pasa_cache& c, const void* q, int R, long long row_stride, const int* row_start, int Hq,
                                    int count, int head, int tail, int* blocks, int io_bf16, unsigned long long* scores, hipStream_t stream)
{
    if (c.table_width > count) {                 // otherwise all pages are taken
        const unsigned chunks = (unsigned)((c.table_width + 63) / 64), grid = chunks * (unsigned)c.S * (unsigned)c.Hkv;
        auto score = [&](auto kernel) {
            kernel<<<grid, kCacheThreads, 0, stream>>>(c, static_cast<const unsigned short*>(q), R, row_stride, row_start, head, tail, io_bf16, log2_of(c.page),
                                                       fast_div((unsigned)(Hq / c.Hkv)), fast_div(c.Hkv), fast_div(chunks), scores);
        };
        c.d == 128 ? score(pasa_cache_score_k<128>) : score(pasa_cache_score_k<64>);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    auto pick = [&](auto kernel, int threads) {
        kernel<<<(unsigned)c.S * (unsigned)c.Hkv, threads, 0, stream>>>(c, row_start, R, count, log2_of(c.page), fast_div(c.Hkv), scores, blocks);
    };
    if (c.table_width <= 1024) pick(pasa_cache_pick_k<256, 4>, 256);
    else if (c.table_width <= 4096) pick(pasa_cache_pick_k<1024, 4>, 1024);
    else pick(pasa_cache_pick_k<1024, 16>, 1024);            // the largest table: 262144 tokens in pages of 16
    return hipGetLastError();
}
