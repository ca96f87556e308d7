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
constexpr int kTokens = 4;                       // of a workgroup at most
constexpr int kAtOnce = 4;                       // items of a thread whose loads are on their way together

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
    int row0, tokens, heads, d, rot, io_bf16, pairs_layout;
    int items, turned, each_heads;               // items of a head, those among them that are turned, heads of a workgroup
    int each_tokens;                             // tokens of a workgroup
    float sign;
    double magnitude;
    FastDiv N, of_item, of_head, parts;
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
// of row_start at a time.
__device__ inline bool place_of_row(const RotaryArgs& a, int r, int& position)
{
    const int lane = threadIdx.x & 63;
    int low = 0, size = a.S + 1;                 // the last entry that is not above r is among `size` from `low` on
    while (size > 1) {
        const int step = (size + 63) / 64, at = low + lane * step;
        const bool not_above = lane * step < size && clamp_int(a.row_start[at <= a.S ? at : a.S], 0, a.tokens) <= r;
        const int n = __builtin_ctzll(~__builtin_amdgcn_ballot_w64(not_above) | 1ull << 63);
        const int first = lane == 63 && n == 63 && not_above ? 64 : n;           // all 64 of them
        const int count = __builtin_amdgcn_readlane(first, 63);
        if (count == 0) return false;
        low += (count - 1) * step;
        size = size - (count - 1) * step < step ? size - (count - 1) * step : step;
    }
    low = __builtin_amdgcn_readfirstlane(low);
    if (low >= a.S) return false;
    const Sequence s = sequence_at(a.length, a.row_start, low, a.tokens, a.most);
    const int t = r - s.row0;
    if (t < 0 || t >= s.rows) return false;
    position = s.length - s.rows + t;
    if (a.tree != nullptr) {                     // behind the older tokens, as many as it sees of the others
        unsigned long long sees = a.tree[r];
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

// A workgroup takes up to four tokens and some of their heads: cos and sin once a token and pair, in 64 bits, into LDS; then the heads in items of 16 bytes a load,
// four items of a thread on their way at a time, the first of them before the positions are known.
// WIDE: items are eight channels (neighbouring pairs) or twice eight (halves); otherwise a pair of channels.
template <bool PAIRS, bool WIDE>
__global__ __launch_bounds__(kThreads)
void pasa_rotate_k(RotaryArgs a)
{
    __shared__ __attribute__((aligned(16))) float2 lds_cs[kTokens][kMaxPairs];
    __shared__ int lds_there[kTokens];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const unsigned group = a.parts.quotient(blockIdx.x);
    const int h0 = (int)a.parts.rest(blockIdx.x, group) * a.each_heads;
    const int token0 = (int)group * a.each_tokens;
    const int tokens = a.tokens - token0 < a.each_tokens ? a.tokens - token0 : a.each_tokens;
    const int heads = a.heads - h0 < a.each_heads ? a.heads - h0 : a.each_heads;
    const int all = tokens * a.each_heads * a.items, half = a.rot / 2;

    struct Item {
        size_t x, y;
        int token, item;
        bool there;
    };
    auto item_at = [&](int i) {
        Item m;
        const unsigned up = a.of_item.quotient((unsigned)i);
        m.item = (int)a.of_item.rest((unsigned)i, up);
        m.token = (int)a.of_head.quotient(up);
        const int h = (int)a.of_head.rest(up, (unsigned)m.token);
        m.there = i < all && h < heads;
        const int token = token0 + (m.there ? m.token : 0);
        const long long b = (long long)a.N.quotient((unsigned)token), n = (long long)a.N.rest((unsigned)token, (unsigned)b);
        const long long head = h0 + (m.there ? h : 0);
        if (!m.there) m.token = 0, m.item = 0;
        m.x = (size_t)(b * a.xs[0] + head * a.xs[1] + n * a.xs[2]);
        m.y = (size_t)(b * a.ys[0] + head * a.ys[1] + n * a.ys[2]);
        return m;
    };
    // channels of an item's first and second part
    auto first_of = [&](int item) { return WIDE ? 8 * item + (PAIRS || item < a.turned ? 0 : a.rot - 8 * a.turned) : item < a.turned ? (PAIRS ? 2 * item : item) : a.rot + 2 * (item - a.turned); };
    auto second_of = [&](int item) { return WIDE ? first_of(item) + half : item < a.turned && !PAIRS ? item + half : first_of(item) + 1; };

    Item m[kAtOnce];
    u16x8 lo[kAtOnce], hi[kAtOnce];
    auto load = [&](int base) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            m[j] = item_at(base + j * kThreads + tid);
            const unsigned short* x = a.x + m[j].x;
            if constexpr (WIDE) {
                lo[j] = *reinterpret_cast<const u16x8*>(x + first_of(m[j].item));
                if (!PAIRS) hi[j] = *reinterpret_cast<const u16x8*>(x + (m[j].item < a.turned ? second_of(m[j].item) : first_of(m[j].item)));
            } else {
                lo[j][0] = x[first_of(m[j].item)];
                hi[j][0] = x[second_of(m[j].item)];
            }
        }
    };
    load(0);
    for (int t = wave; t < tokens; t += kThreads / 64) {
        int position = 0;
        bool there = true;
        const int token = token0 + t;
        if (a.row_start != nullptr) there = place_of_row(a, token, position);
        else if (a.positions != nullptr) position = a.positions[token];
        else position = a.row0 + (int)a.N.rest((unsigned)token, a.N.quotient((unsigned)token));
        if (lane < half) {
            double c, s;
            turn((double)position * a.freq[lane] * 0.159154943091895335769, c, s);
            lds_cs[t][lane] = make_float2((float)(a.magnitude * c), a.sign * (float)(a.magnitude * s));
        }
        if (lane == 0) lds_there[t] = there;
    }
    __syncthreads();
    for (int base = 0; base < all; base += kAtOnce * kThreads) {
        if (base > 0) load(base);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (!m[j].there || lds_there[m[j].token] == 0) continue;
            unsigned short* y = a.y + m[j].y;
            const int c0 = first_of(m[j].item), c1 = second_of(m[j].item);
            const bool turned = m[j].item < a.turned;
            if constexpr (WIDE && PAIRS) {
                if (turned) {
                    unsigned out[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 cs = lds_cs[m[j].token][c0 / 2 + e];
                        const float p = widen(lo[j][2 * e], a.io_bf16), q = widen(lo[j][2 * e + 1], a.io_bf16);
                        out[e] = pack(__builtin_fmaf(p, cs.x, -(q * cs.y)), __builtin_fmaf(q, cs.x, p * cs.y), a.io_bf16);
                    }
                    *reinterpret_cast<uint4*>(y + c0) = make_uint4(out[0], out[1], out[2], out[3]);
                } else {
                    *reinterpret_cast<u16x8*>(y + c0) = lo[j];
                }
            } else if constexpr (WIDE) {
                if (turned) {
                    unsigned out[2][4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float p[2], q[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 cs = lds_cs[m[j].token][c0 + 2 * e + i];
                            const float u = widen(lo[j][2 * e + i], a.io_bf16), v = widen(hi[j][2 * e + i], a.io_bf16);
                            p[i] = __builtin_fmaf(u, cs.x, -(v * cs.y));
                            q[i] = __builtin_fmaf(v, cs.x, u * cs.y);
                        }
                        out[0][e] = pack(p[0], p[1], a.io_bf16);
                        out[1][e] = pack(q[0], q[1], a.io_bf16);
                    }
                    *reinterpret_cast<uint4*>(y + c0) = make_uint4(out[0][0], out[0][1], out[0][2], out[0][3]);
                    *reinterpret_cast<uint4*>(y + c1) = make_uint4(out[1][0], out[1][1], out[1][2], out[1][3]);
                } else {
                    *reinterpret_cast<u16x8*>(y + c0) = lo[j];
                }
            } else {
                if (turned) {
                    const float2 cs = lds_cs[m[j].token][m[j].item];
                    const float p = widen(lo[j][0], a.io_bf16), q = widen(hi[j][0], a.io_bf16);
                    const unsigned out = pack(__builtin_fmaf(p, cs.x, -(q * cs.y)), __builtin_fmaf(q, cs.x, p * cs.y), a.io_bf16);
                    y[c0] = (unsigned short)out;
                    y[c1] = (unsigned short)(out >> 16);
                } else {
                    y[c0] = lo[j][0];
                    y[c1] = hi[j][0];
                }
            }
        }
    }
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool buffer(const void* p, uintptr_t a) { return p != nullptr && aligned(p, a); }

int check_rotary(const pasa_rotary* r, int d, int transposed, int io_dtype)
{
    if (r == nullptr || (r->layout != PASA_ROTARY_HALVES && r->layout != PASA_ROTARY_PAIRS)) return PASA_EINVAL;
    if (r->rot < 2 || r->rot % 2 != 0 || r->rot > d || !isfinite(r->magnitude)) return PASA_EINVAL;
    if ((transposed != 0 && transposed != 1) || (io_dtype != PASA_IO_F16 && io_dtype != PASA_IO_BF16)) return PASA_EINVAL;
    for (int i = 0; i < r->rot / 2; ++i)
        if (!isfinite(r->freq[i])) return PASA_EINVAL;
    return PASA_OK;
}

// The rest of the arguments, and the launch
int launch(RotaryArgs& a, const pasa_rotary* r, int transposed, int io_dtype, bool in_place, hipStream_t stream)
{
    a.rot = r->rot;
    a.io_bf16 = io_dtype == PASA_IO_BF16;
    a.pairs_layout = r->layout == PASA_ROTARY_PAIRS;
    a.sign = transposed ? -1.f : 1.f;
    a.magnitude = r->magnitude;
    for (int i = 0; i < a.rot / 2; ++i) a.freq[i] = r->freq[i];
    // Items of eight channels where pairs keep to them.
    const bool wide = a.pairs_layout ? a.rot % 8 == 0 : a.rot % 16 == 0;
    a.turned = !wide ? a.rot / 2 : a.pairs_layout ? a.rot / 8 : a.rot / 16;
    a.items = a.turned + (in_place ? 0 : (a.d - a.rot) / (wide ? 8 : 2));
    // Four tokens a workgroup where that leaves every compute unit several workgroups, with heads for four to eight items a thread; otherwise one, with an item a thread.
    const long long total = (long long)a.tokens * a.heads * a.items;
    a.each_tokens = total >= 8LL * 256 * kThreads * kAtOnce ? kTokens : 1;
    const int target = (a.each_tokens == 1 ? 1 : 2 * kAtOnce) * kThreads / (a.each_tokens * a.items);
    a.each_heads = target < 1 ? 1 : target < a.heads ? target : a.heads;
    const long long parts = (a.heads + a.each_heads - 1) / a.each_heads, grid = ((long long)a.tokens + a.each_tokens - 1) / a.each_tokens * parts;
    if (grid * kThreads > 0xffffffffLL) return PASA_EUNSUPPORTED;
    a.of_item = fast_div((unsigned)a.items);
    a.of_head = fast_div((unsigned)a.each_heads);
    a.parts = fast_div((unsigned)parts);
    auto go = [&](auto kernel) { kernel<<<(unsigned)grid, kThreads, 0, stream>>>(a); };
    if (a.pairs_layout) wide ? go(pasa_rotate_k<true, true>) : go(pasa_rotate_k<true, false>);
    else wide ? go(pasa_rotate_k<false, true>) : go(pasa_rotate_k<false, false>);
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
    if ((long long)B * N > INT_MAX) return PASA_EUNSUPPORTED;
    a.x = static_cast<const unsigned short*>(x);
    a.y = static_cast<unsigned short*>(y);
    a.positions = positions;
    a.row0 = row0;
    a.tokens = B * N;
    a.heads = H;
    a.d = d;
    a.N = fast_div((unsigned)N);
    return launch(a, rotary, transposed, io_dtype, x == y, static_cast<hipStream_t>(stream));
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
    if (R > INT_MAX - 1 || cache->S > 1 << 30) return PASA_EUNSUPPORTED;
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
    a.d = cache->d;
    a.N = fast_div((unsigned)R);
    return launch(a, rotary, transposed, io_dtype, x == y, static_cast<hipStream_t>(stream));
}

}  // extern "C"
