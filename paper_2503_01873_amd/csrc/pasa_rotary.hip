// Rotary positions: pasa_rotary_set (host), pasa_rotate and pasa_cache_rotate with their kernel.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <type_traits>

#include "pasa.h"
#include "pasa_cache.h"

namespace {

constexpr int kMaxPairs = 64;
constexpr int kThreads = 256;
constexpr int kMaxHeads = 1 << 24;               // so that sums of them and of threads fit 31 bits
constexpr int kTokens = 32;                      // of a workgroup at most
// Of y: more is stored past the L2s, which would have to bring it to memory before the kernel ends (33 MB of keys 14.2 us, through them 17.2; 15 MB 7.6 / 8.6); the smallest
// outputs stay there for who reads them next.  With pasa_attn_fwd behind it (28 heads on 4), past / through, us: queries of 15 MB, one sequence, 63.4 / 64.0; 29 MB, 4096 rows
// 137.0 / 136.5, 8 x 512 rows 58.8 / 57.9, 64 x 64 rows 68.5 / 65.4, where attention is short and finds less in its L2; 59 MB 435 / 435.
constexpr long long kStreamBytes = 4 << 20;
constexpr int kAtOnce = 2;                       // heads of a thread that are on their way together

// Where a call's tokens are and what their positions are made of.  A token is a row of `heads` heads; b its batch entry, n its number there.
struct RotaryArgs {
    const unsigned short* x;
    unsigned short* y;
    long long xs[3], ys[3];                      // elements from one batch entry, head, row to the next
    const int* positions;                        // [B][N], or NULL: row0 + n
    // of a cache: rows lie where their sequences have come to
    const int* length;
    const int* row_start;
    const unsigned long long* tree;
    int S, most;
    int row0, tokens, heads, rot, io_bf16;
    int turned, in_place;                        // items of a head that are turned, the last one perhaps in part
    // A workgroup's threads: `items` of a head, times `lanes` heads at a time, times each_tokens tokens; and the heads of a workgroup
    int items, lanes, each_tokens, each_heads;
    float sign;
    double magnitude;
    FastDiv N, of_item, of_lane, of_pair, parts;
    double freq[kMaxPairs];
};

// cos and sin of 2 pi turns, in 64 bits: the nearest quarter is taken off, and the rest, up to pi / 4, goes through both Taylor series (the first term that is
// left out is 2e-14 there).  A position of 2^18 is off by 1e-10 turns of what `turns` carries at most, where fp32 would leave 2^-6.
__device__ inline void turn(double turns, double& c, double& s)
{
    const double whole = __builtin_rint(4.0 * turns);
    const double a = (turns - 0.25 * whole) * 6.283185307179586476925, z = a * a;
    double u = 1.0 / 6227020800.0;               // 13!
    u = __builtin_fma(u, z, -1.0 / 39916800.0);
    u = __builtin_fma(u, z, 1.0 / 362880.0);
    u = __builtin_fma(u, z, -1.0 / 5040.0);
    u = __builtin_fma(u, z, 1.0 / 120.0);
    u = __builtin_fma(u, z, -1.0 / 6.0);
    const double sine = __builtin_fma(u * z, a, a);
    double v = -1.0 / 87178291200.0;             // 14!
    v = __builtin_fma(v, z, 1.0 / 479001600.0);
    v = __builtin_fma(v, z, -1.0 / 3628800.0);
    v = __builtin_fma(v, z, 1.0 / 40320.0);
    v = __builtin_fma(v, z, -1.0 / 720.0);
    v = __builtin_fma(v, z, 1.0 / 24.0);
    v = __builtin_fma(v, z, -0.5);
    const double cosine = __builtin_fma(v, z, 1.0);
    const int quarter = (int)(whole - 4.0 * __builtin_floor(0.25 * whole));
    const bool odd = (quarter & 1) != 0;
    c = odd ? sine : cosine;
    s = odd ? cosine : sine;
    if (quarter == 1 || quarter == 2) c = -c;
    if (quarter >= 2) s = -s;
}

// Position of row r of a step, the same in all lanes of a wavefront; false where the row belongs to no sequence.  The sequence is found by 64 entries
// of row_start at a time; up to 63 sequences have all that is to be known of them on its way at once.
__device__ inline bool place_of_row(const RotaryArgs& a, int r, int& position)
{
    const int lane = threadIdx.x & 63;
    unsigned long long sees = a.tree != nullptr ? a.tree[r] : 0ull;
    // how many of the 64 entries, from the first on, are not above r
    auto leading = [&](bool not_above) {
        const unsigned long long above = ~__builtin_amdgcn_ballot_w64(not_above);
        return above == 0ull ? 64 : __builtin_ctzll(above);
    };
    Sequence s;
    if (__builtin_expect(a.S < 64, 1)) {
        const int start = clamp_int(a.row_start[lane <= a.S ? lane : a.S], 0, a.tokens);
        const int length = clamp_int(a.length[lane < a.S ? lane : a.S - 1], 0, a.most);
        const int n = leading(lane <= a.S && start <= r);
        if (n == 0 || n > a.S) return false;
        s.row0 = __builtin_amdgcn_readlane(start, n - 1);
        const int end = __builtin_amdgcn_readlane(start, n);
        s.rows = end > s.row0 ? end - s.row0 : 0;
        s.length = __builtin_amdgcn_readlane(length, n - 1);
    } else {
        int low = 0, size = a.S + 1;             // the last entry that is not above r is among `size` from `low` on
        while (size > 1) {
            const int step = (size + 63) / 64, at = low + lane * step;
            const int n = leading(lane * step < size && clamp_int(a.row_start[at <= a.S ? at : a.S], 0, a.tokens) <= r);
            if (n == 0) return false;
            low += (n - 1) * step;
            size = size - (n - 1) * step < step ? size - (n - 1) * step : step;
        }
        low = __builtin_amdgcn_readfirstlane(low);
        if (low >= a.S) return false;
        s = sequence_at(a.length, a.row_start, low, a.tokens, a.most);
    }
    const int t = r - s.row0;
    if (t < 0 || t >= s.rows) return false;
    position = s.length - s.rows + t;
    if (a.tree != nullptr) {                     // behind the older tokens, as many as it sees of the others
        if (s.rows < 64) sees &= (1ull << s.rows) - 1ull;
        if (t < 64) sees &= ~(1ull << t);
        position = s.length - s.rows + __builtin_popcountll(sees);
    }
    return true;
}

__device__ inline float widen(unsigned short raw, int io_bf16)
{
    return io_bf16 ? __uint_as_float((unsigned)raw << 16) : (float)__builtin_bit_cast(_Float16, raw);
}
__device__ inline unsigned pack(float lo, float hi, int io_bf16) { return io_bf16 ? pack_bf16(lo, hi) : pack_f16(lo, hi); }

typedef unsigned u4 __attribute__((ext_vector_type(4)));
enum { HALVES = 0, PAIRS = 1, ANY_HALVES = 2 };

// A thread has an item of a token, 16 bytes (HALVES: twice 16), and takes it of one head after the other: cos and sin, which a workgroup works out
// once a token and pair, in 64 bits, stay in its registers.  Two heads of a thread are on their way at a time, the first ones before the positions are known.
//  HALVES: halves that are whole items; an item is eight channels of each.
//  PAIRS: eight channels, four pairs, of which the last item may have fewer.
//  ANY_HALVES: eight channels, with the others of their pairs, which may lie anywhere in the row, by way of LDS: a row's items are neighbouring lanes.
// CACHE: rows of a step.  STREAM: y is stored past the L2s.
// What bounds it: memory; 2 x 16384 rows of 28 heads, bf16, out of a joint projection, 470 MB, 86.4 us, 5.4 TB/s (one head at a time 84.0, four 94.5; through the L2s 5 us more; four heads
// and small workgroups for all 103); 14 x 2305 rows of 5 heads of 64, a quarter of the channels, 41 MB, 9.5 us.  A step of 16 rows of 32 heads, 4.2 us: lengths,
// then angles, then stores.  (cos and sin with the smaller terms of their series in fp32: nothing gained.)
template <int MODE, bool CACHE, bool STREAM>
__global__ __launch_bounds__(kThreads)
void pasa_rotate_k(RotaryArgs a)
{
    constexpr int CS = MODE == PAIRS ? 4 : 8;            // pairs of an item
    __shared__ __attribute__((aligned(16))) float2 lds_cs[kTokens * kMaxPairs];
    __shared__ __attribute__((aligned(16))) unsigned short lds_row[MODE == ANY_HALVES ? kAtOnce * kThreads * 8 : 8];
    __shared__ int lds_position[kTokens], lds_there[kTokens];
    const int tid = threadIdx.x, half = a.rot / 2;
    const unsigned group = a.parts.quotient(blockIdx.x);
    const int h0 = (int)a.parts.rest(blockIdx.x, group) * a.each_heads;
    const int token0 = (int)group * a.each_tokens;
    const int tokens = a.tokens - token0 < a.each_tokens ? a.tokens - token0 : a.each_tokens;
    const int end = a.heads - h0 < a.each_heads ? a.heads : h0 + a.each_heads;

    const unsigned up = a.of_item.quotient((unsigned)tid);
    const int item = (int)a.of_item.rest((unsigned)tid, up);
    const int t = (int)a.of_lane.quotient(up), lane = (int)a.of_lane.rest(up, (unsigned)t);
    const bool there = t < tokens;
    const unsigned token = (unsigned)(token0 + (there ? t : 0)), b = a.N.quotient(token), n = a.N.rest(token, b);
    const bool turned = item < a.turned;
    // channels of the item, of its second part, and behind its last one that is turned
    const int c0 = MODE == HALVES && !turned ? a.rot + 8 * (item - a.turned) : 8 * item, c1 = turned ? c0 + half : c0;
    const bool whole = MODE == HALVES || c0 + 8 <= a.rot;
    const unsigned short* x = a.x + (long long)b * a.xs[0] + (long long)n * a.xs[2];
    unsigned short* y = a.y + (long long)b * a.ys[0] + (long long)n * a.ys[2];

    u16x8 lo[kAtOnce], hi[kAtOnce];
    auto load = [&](int h) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int at = h + j * a.lanes < end ? h + j * a.lanes : h0;         // a head again, for nothing
            const unsigned short* from = x + (long long)at * a.xs[1];
            lo[j] = *reinterpret_cast<const u16x8*>(from + c0);
            if (MODE == HALVES) hi[j] = *reinterpret_cast<const u16x8*>(from + c1);
        }
    };
    load(h0 + lane);
    if constexpr (CACHE) {
        for (int i = tid >> 6; i < tokens; i += kThreads / 64) {
            int position = 0;
            const bool found = place_of_row(a, token0 + i, position);
            if ((tid & 63) == 0) lds_position[i] = position, lds_there[i] = found;
        }
        __syncthreads();
    }
    for (int i = tid; i < tokens * half; i += kThreads) {
        const unsigned at = a.of_pair.quotient((unsigned)i), pair = a.of_pair.rest((unsigned)i, at);
        const unsigned of = (unsigned)token0 + at;
        int position;
        if constexpr (CACHE) position = lds_position[at];
        else position = a.positions != nullptr ? a.positions[of] : a.row0 + (int)a.N.rest(of, a.N.quotient(of));
        double c, s;
        turn((double)position * a.freq[pair] * 0.159154943091895335769, c, s);
        lds_cs[at * kMaxPairs + pair] = make_float2((float)(a.magnitude * c), a.sign * (float)(a.magnitude * s));
    }
    __syncthreads();
    if (!there || (CACHE && lds_there[t] == 0)) return;
    float2 cs[CS];
    int other[MODE == ANY_HALVES ? 8 : 1];               // where the other channel of the pair is, from the thread's first one on
#pragma unroll
    for (int i = 0; i < CS; ++i) {
        const int c = c0 + i;                            // ANY_HALVES
        const int pair = MODE == HALVES ? c0 + i : MODE == PAIRS ? c0 / 2 + i : c < half ? c : c - half;
        cs[i] = lds_cs[t * kMaxPairs + (turned && pair < half ? pair : 0)];
        if (MODE == ANY_HALVES) {
            other[i] = c >= a.rot ? i : c < half ? i + half : i - half;
            if (c < half) cs[i].y = -cs[i].y;            // y = x cos -+ other sin
        }
    }
    auto store = [&](unsigned short* at, u4 v) {
        if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u4*>(at));
        else *reinterpret_cast<u4*>(at) = v;
    };
    for (int h = h0 + lane; h < end; h += kAtOnce * a.lanes) {
        if (h != h0 + lane) load(h);
        if constexpr (MODE == ANY_HALVES) {
            __builtin_amdgcn_wave_barrier();             // a wavefront's LDS accesses are done in order
            asm volatile("" ::: "memory");
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) *reinterpret_cast<u16x8*>(lds_row + (j * kThreads + tid) * 8) = lo[j];
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (h + j * a.lanes >= end) break;
            unsigned short* to = y + (long long)(h + j * a.lanes) * a.ys[1];
            if (!turned) {
                if (!a.in_place) store(to + c0, __builtin_bit_cast(u4, lo[j]));
                continue;
            }
            u4 out[2];
            if constexpr (MODE == HALVES) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float p[2], q[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float u = widen(lo[j][2 * e + i], a.io_bf16), v = widen(hi[j][2 * e + i], a.io_bf16);
                        p[i] = __builtin_fmaf(u, cs[2 * e + i].x, -(v * cs[2 * e + i].y));
                        q[i] = __builtin_fmaf(v, cs[2 * e + i].x, u * cs[2 * e + i].y);
                    }
                    out[0][e] = pack(p[0], p[1], a.io_bf16);
                    out[1][e] = pack(q[0], q[1], a.io_bf16);
                }
                store(to + c1, out[1]);
            } else if constexpr (MODE == PAIRS) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = widen(lo[j][2 * e], a.io_bf16), q = widen(lo[j][2 * e + 1], a.io_bf16);
                    out[0][e] = pack(__builtin_fmaf(p, cs[e].x, -(q * cs[e].y)), __builtin_fmaf(q, cs[e].x, p * cs[e].y), a.io_bf16);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float p[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float u = widen(lo[j][2 * e + i], a.io_bf16), v = widen(lds_row[(j * kThreads + tid) * 8 + other[2 * e + i]], a.io_bf16);
                        p[i] = __builtin_fmaf(u, cs[2 * e + i].x, v * cs[2 * e + i].y);
                    }
                    out[0][e] = pack(p[0], p[1], a.io_bf16);
                }
            }
            // channels from rot on: as they were, or left alone
            u16x8 made = __builtin_bit_cast(u16x8, out[0]);
            if (MODE != HALVES && !whole) {
#pragma unroll
                for (int e = 0; e < 8; ++e) made[e] = c0 + e < a.rot ? made[e] : lo[j][e];
            }
            if (MODE == HALVES || whole || !a.in_place) {
                store(to + c0, __builtin_bit_cast(u4, made));
                continue;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c0 + e < a.rot) to[c0 + e] = made[e];
        }
    }
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool buffer(const void* p, uintptr_t a) { return p != nullptr && aligned(p, a); }

int check_rotary(const pasa_rotary* r, int d, int transposed, int io_dtype)
{
    if (r == nullptr || (r->layout != PASA_ROTARY_HALVES && r->layout != PASA_ROTARY_PAIRS)) return PASA_EINVAL;
    if (r->rot < 2 || r->rot % 2 != 0 || r->rot > d || r->rot > 2 * kMaxPairs || !isfinite(r->magnitude)) return PASA_EINVAL;
    if ((transposed != 0 && transposed != 1) || (io_dtype != PASA_IO_F16 && io_dtype != PASA_IO_BF16)) return PASA_EINVAL;
    for (int i = 0; i < r->rot / 2; ++i)
        if (!isfinite(r->freq[i])) return PASA_EINVAL;
    return PASA_OK;
}

// The rest of the arguments, and the launch
int launch(RotaryArgs& a, const pasa_rotary* r, int d, int transposed, int io_dtype, bool in_place, hipStream_t stream)
{
    a.rot = r->rot;
    a.io_bf16 = io_dtype == PASA_IO_BF16;
    a.sign = transposed ? -1.f : 1.f;
    a.magnitude = r->magnitude;
    for (int i = 0; i < a.rot / 2; ++i) a.freq[i] = r->freq[i];
    const bool pairs = r->layout == PASA_ROTARY_PAIRS, cache = a.row_start != nullptr;
    const int mode = pairs ? PAIRS : a.rot % 16 == 0 ? HALVES : ANY_HALVES;
    a.turned = mode == HALVES ? a.rot / 16 : (a.rot + 7) / 8;
    a.items = mode == ANY_HALVES ? d / 8 : a.turned + (in_place ? 0 : mode == HALVES ? (d - a.rot) / 8 : d / 8 - a.turned);
    a.in_place = in_place;
    // Heads at a time: so that a thread takes two or three of them, where there are workgroups enough for that, and few threads are left over; one each otherwise.
    const int groups = kThreads / a.items;
    const long long threads = (long long)a.tokens * a.heads * a.items;
    const int most_tokens = cache ? 4 : kTokens;
    if (threads >= 4LL * kAtOnce * kThreads * 256) {
        long best = -1;
        for (int lanes = 1; lanes <= groups && lanes <= a.heads; ++lanes) {
            const int turns = (a.heads + lanes - 1) / lanes;
            const int tokens = groups / lanes < most_tokens ? groups / lanes : most_tokens;
            const int used = turns < kAtOnce ? kAtOnce : turns;          // a thread of fewer waits as long
            const long worth = 4096L * tokens * a.heads / used;
            if (worth > best && (turns < 2 * kAtOnce || lanes == groups)) best = worth, a.lanes = lanes, a.each_tokens = tokens;
        }
        a.each_heads = (a.heads + a.lanes - 1) / a.lanes * a.lanes;
        if (a.each_heads > 2 * kAtOnce * a.lanes) a.each_heads = 2 * kAtOnce * a.lanes;
    } else {
        a.lanes = groups < a.heads ? groups : a.heads;
        a.each_tokens = groups / a.lanes < most_tokens ? groups / a.lanes : most_tokens;
        a.each_heads = a.lanes;
    }
    const long long parts = (a.heads + a.each_heads - 1) / a.each_heads, grid = ((long long)a.tokens + a.each_tokens - 1) / a.each_tokens * parts;
    if (grid * kThreads > 0xffffffffLL) return PASA_EUNSUPPORTED;
    a.of_item = fast_div((unsigned)a.items);
    a.of_lane = fast_div((unsigned)a.lanes);
    a.of_pair = fast_div((unsigned)a.rot / 2);
    a.parts = fast_div((unsigned)parts);
    auto go = [&](auto kernel) { kernel<<<(unsigned)grid, kThreads, 0, stream>>>(a); };
    const bool stream_out = threads * (mode == HALVES ? 32 : 16) > kStreamBytes;
    auto of_mode = [&](auto m) {
        constexpr int M = decltype(m)::value;
        if (cache) go(pasa_rotate_k<M, true, false>);
        else if (stream_out) go(pasa_rotate_k<M, false, true>);
        else go(pasa_rotate_k<M, false, false>);
    };
    if (mode == HALVES) of_mode(std::integral_constant<int, HALVES>{});
    else if (mode == PAIRS) of_mode(std::integral_constant<int, PAIRS>{});
    else of_mode(std::integral_constant<int, ANY_HALVES>{});
    return hipGetLastError() == hipSuccess ? PASA_OK : PASA_ELAUNCH;
}

}  // namespace

extern "C" {

int pasa_rotary_set(pasa_rotary* r, int layout, int rot, double base, int scaling, double factor, double original, double slow, double fast,
                    double magnitude)
{
    if (r == nullptr || (layout != PASA_ROTARY_HALVES && layout != PASA_ROTARY_PAIRS) || rot < 2 || rot % 2 != 0) return PASA_EINVAL;
    if (rot > 2 * kMaxPairs) return PASA_EUNSUPPORTED;
    if (!isfinite(base) || !(base > 1.0) || !isfinite(magnitude)) return PASA_EINVAL;
    if (scaling < PASA_ROTARY_PLAIN || scaling > PASA_ROTARY_WAVES) return PASA_EINVAL;
    if (scaling != PASA_ROTARY_PLAIN && (!isfinite(factor) || !(factor >= 1.0))) return PASA_EINVAL;
    const bool blended = scaling == PASA_ROTARY_RAMP || scaling == PASA_ROTARY_WAVES;
    if (blended && (!isfinite(original) || !(original > 0.0) || !(slow > 0.0) || !(fast > slow) || !isfinite(fast))) return PASA_EINVAL;
    const double two_pi = 6.283185307179586476925;
    if (scaling == PASA_ROTARY_BASE && rot > 2) base *= pow(factor, rot / (rot - 2.0));
    double first = 0.0, last = 0.0;
    if (scaling == PASA_ROTARY_RAMP) {           // pairs that turn `fast` times and `slow` times over the original length
        first = floor(0.5 * rot * log(original / (two_pi * fast)) / log(base));
        last = ceil(0.5 * rot * log(original / (two_pi * slow)) / log(base));
        if (first < 0.0) first = 0.0;
        if (last > rot - 1.0) last = rot - 1.0;
    }
    for (int i = 0; i < kMaxPairs; ++i) r->freq[i] = 0.0;
    for (int i = 0; i < rot / 2; ++i) {
        const double f = pow(base, -2.0 * i / rot);
        double keep = 1.0;                       // how much of the frequency stays
        if (scaling == PASA_ROTARY_LINEAR) keep = 0.0;
        else if (scaling == PASA_ROTARY_RAMP) keep = 1.0 - (i - first) / (last - first > 0.001 ? last - first : 0.001);
        else if (scaling == PASA_ROTARY_WAVES) keep = (original * f / two_pi - slow) / (fast - slow);
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        r->freq[i] = keep == 1.0 ? f : f / factor * (1.0 - keep) + f * keep;
    }
    r->magnitude = magnitude;
    r->rot = rot;
    r->layout = layout;
    return PASA_OK;
}

int pasa_rotate(const pasa_rotary* rotary, const void* x, void* y, int B, int H, int N, int d, const long long* x_strides, const long long* y_strides,
                const int* positions, int row0, int transposed, int io_dtype, void* stream)
{
    if (!buffer(x, 16) || !buffer(y, 16) || !aligned(positions, 4) || B <= 0 || H <= 0 || N <= 0 || d <= 0) return PASA_EINVAL;
    const int st = check_rotary(rotary, d, transposed, io_dtype);
    if (st != PASA_OK) return st;
    if (d != 64 && d != 128) return PASA_EUNSUPPORTED;
    RotaryArgs a = {};
    const long long plain[3] = {(long long)H * N * d, (long long)N * d, d};
    for (int i = 0; i < 3; ++i) {
        a.xs[i] = x_strides != nullptr ? x_strides[i] : plain[i];
        a.ys[i] = y_strides != nullptr ? y_strides[i] : plain[i];
        if (a.xs[i] < 0 || a.ys[i] < 0 || a.xs[i] % 8 != 0 || a.ys[i] % 8 != 0) return PASA_EINVAL;
    }
    // rows of y must not be one another's
    const int size[3] = {B, H, N};
    for (int i = 0; i < 3; ++i)
        if (size[i] > 1 && a.ys[i] < d) return PASA_EINVAL;
    if (x == y)
        for (int i = 0; i < 3; ++i)
            if (size[i] > 1 && a.xs[i] != a.ys[i]) return PASA_EINVAL;
    if (positions == nullptr && (long long)row0 + N - 1 > INT_MAX) return PASA_EINVAL;
    if ((long long)B * N > INT_MAX || H > kMaxHeads) return PASA_EUNSUPPORTED;
    a.x = static_cast<const unsigned short*>(x);
    a.y = static_cast<unsigned short*>(y);
    a.positions = positions;
    a.row0 = row0;
    a.tokens = B * N;
    a.heads = H;
    a.N = fast_div((unsigned)N);
    return launch(a, rotary, d, transposed, io_dtype, x == y, static_cast<hipStream_t>(stream));
}

int pasa_cache_rotate(const pasa_cache* cache, const pasa_rotary* rotary, const void* x, void* y, int heads, int R, long long x_stride, long long y_stride,
                      const int* row_start, const unsigned long long* tree, int transposed, int io_dtype, void* stream)
{
    int st = pasa_check_cache(cache);
    if (st != PASA_OK) return st;
    if (!buffer(x, 16) || !buffer(y, 16) || !buffer(row_start, 4) || !aligned(tree, 8) || heads <= 0 || R <= 0) return PASA_EINVAL;
    st = check_rotary(rotary, cache->d, transposed, io_dtype);
    if (st != PASA_OK) return st;
    const long long least = (long long)heads * cache->d;
    if (x_stride < least || y_stride < least || x_stride % 8 != 0 || y_stride % 8 != 0 || (x == y && x_stride != y_stride)) return PASA_EINVAL;
    if (R > INT_MAX - 1 || cache->S > 1 << 30 || heads > kMaxHeads) return PASA_EUNSUPPORTED;
    RotaryArgs a = {};
    a.x = static_cast<const unsigned short*>(x);
    a.y = static_cast<unsigned short*>(y);
    a.xs[1] = a.ys[1] = cache->d;
    a.xs[2] = x_stride;
    a.ys[2] = y_stride;
    a.length = cache->length;
    a.row_start = row_start;
    a.tree = tree;
    a.S = cache->S;
    a.most = cache->table_width * cache->page;
    a.tokens = R;
    a.heads = heads;
    a.N = fast_div((unsigned)R);
    return launch(a, rotary, cache->d, transposed, io_dtype, x == y, static_cast<hipStream_t>(stream));
}

}  // extern "C"
