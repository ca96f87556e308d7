// The paged 8-bit cache: tokens enter (write), come back (read), and pages are chosen by their pseudo-averages (score, pick).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pasa_cache.h"

namespace {

// ---- tokens enter ----

// x / scale for a conversion that rounds to 22 bits or fewer, nearest: the quotient where fp32 holds it, otherwise an fp32 value next
// to it whose last bit is set, so that no tie and no border of the coarser type is hit that the quotient itself does not hit.
// The first quotient is off by at most two steps of fp32, the second, from the exact remainder, is the nearest one or next to it,
// and the sign of its own remainder says on which side the quotient lies.
__device__ inline float sticky_quotient(float x, float scale, float inverse)
{
    float q = x * inverse;
    q = __builtin_fmaf(__builtin_fmaf(-q, scale, x), inverse, q);
    const float r = __builtin_fmaf(-q, scale, x);
    unsigned bits = __float_as_uint(q);
    if (r != 0.f && q != 0.f && (bits & 1u) == 0u) bits += (r > 0.f) == (q > 0.f) ? 1u : ~0u;
    return __uint_as_float(bits);
}

// Eight values of a token -> eight bytes.  `top`: the largest magnitude of the token as bits (a NaN is above all others).
template <bool E4M3>
__device__ inline uint2 encode8(const float (&x)[8], unsigned top, float& scale)
{
    constexpr float most = E4M3 ? 448.f : 127.f;
    const bool finite = top < 0x7f800000u;
    scale = __uint_as_float(top) / most;
    if (top < 0x0d800000u) scale = 1.f;          // below 2^-100
    if (!finite) scale = __builtin_nanf("");
    const float inverse = 1.f / scale;
    unsigned w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = finite ? __builtin_fminf(__builtin_fmaxf(sticky_quotient(x[4 * h + i], scale, inverse), -most), most) : 0.f;
        if (E4M3) {
            const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
            w[h] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
        } else {
            w[h] = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[h] |= (unsigned)((int)__builtin_rintf(q[i]) + 128) << (8 * i);
        }
    }
    return make_uint2(w[0], w[1]);
}

__device__ inline void widen_io(u16x8 raw, int io_bf16, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = io_bf16 ? __uint_as_float((unsigned)raw[i] << 16) : (float)__builtin_bit_cast(_Float16, (unsigned short)raw[i]);
}

// One workgroup per page that is written to and KV head: D / 8 neighbouring lanes take a token.  Where means are kept, the page's
// older tokens are read too: a mean made from all tokens is the same whatever the steps that brought them, and writing a
// token again corrects it.  Partial sums of the lanes that share channels are added in a fixed order.
template <int D, bool E4M3>
__global__ __launch_bounds__(kCacheThreads)
void pasa_cache_write_k(pasa_cache c, const unsigned short* __restrict__ k, const unsigned short* __restrict__ v, int R, long long row_stride,
                        const int* __restrict__ row_start, int io_bf16, FastDiv heads)
{
    constexpr int LT = D / 8, AT = kCacheThreads / LT;           // lanes of a token, tokens at a time
    __shared__ float sums[AT][D];
    const int tid = threadIdx.x, lt = tid % LT, t0 = tid / LT;
    const int most = c.table_width * c.page;
    // workgroups of a page's heads follow one another
    const unsigned piece = heads.quotient(blockIdx.x);
    const int hk = (int)heads.rest(blockIdx.x, piece);
    auto first_page = [&](const Sequence& s) { return (s.length > s.rows ? s.length - s.rows : 0) / c.page; };
    const Place at = find_place<kCacheThreads>(c.length, row_start, c.S, R, most, [&](const Sequence& s) {
        return s.rows == 0 || s.length == 0 ? 0u : (unsigned)((s.length - 1) / c.page - first_page(s) + 1);
    }, [&](unsigned) { return piece; });
    if (at.b < 0) return;
    const Sequence s = at.s;
    const int place = first_page(s) + (int)at.rest, pos0 = place * c.page;
    const int id = c.table[(size_t)at.b * c.table_width + place];
    if (id < 0 || id >= c.pages) return;
    const int tokens = s.length - pos0 < c.page ? s.length - pos0 : c.page;      // of the page
    const int fresh = s.length - s.rows - pos0;                                  // the first new one, when not negative
    const size_t slot = ((size_t)id * c.Hkv + hk) * c.page;
    unsigned char* kc = static_cast<unsigned char*>(c.k) + slot * D;
    unsigned char* vc = static_cast<unsigned char*>(c.v) + slot * D;
    float shift[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) shift[i] = c.kshift != nullptr ? c.kshift[hk * D + 8 * lt + i] : 0.f;

    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int start = c.kmean != nullptr || fresh < 0 ? 0 : fresh / AT * AT;
    for (int t = start + t0; t - t0 < tokens; t += AT) {                         // all lanes of a token go round together
        if (t >= tokens) continue;
        uint2 code;
        float scale;
        if (t >= fresh) {
            const size_t row = (size_t)(s.row0 + t - fresh) * (size_t)row_stride + (size_t)hk * D + 8 * lt;
            float x[8], y[8];
            widen_io(*reinterpret_cast<const u16x8*>(k + row), io_bf16, x);
            widen_io(*reinterpret_cast<const u16x8*>(v + row), io_bf16, y);
            unsigned top_k = 0, top_v = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] -= shift[i];
                const unsigned a = __float_as_uint(x[i]) & 0x7fffffffu, b = __float_as_uint(y[i]) & 0x7fffffffu;
                top_k = a > top_k ? a : top_k;
                top_v = b > top_v ? b : top_v;
            }
#pragma unroll
            for (int o = 1; o < LT; o <<= 1) {
                const unsigned a = __shfl_xor(top_k, o), b = __shfl_xor(top_v, o);
                top_k = a > top_k ? a : top_k;
                top_v = b > top_v ? b : top_v;
            }
            float vscale;
            const uint2 vcode = encode8<E4M3>(y, top_v, vscale);
            code = encode8<E4M3>(x, top_k, scale);
            *reinterpret_cast<uint2*>(kc + (size_t)t * D + 8 * lt) = code;
            *reinterpret_cast<uint2*>(vc + (size_t)t * D + 8 * lt) = vcode;
            if (lt == 0) {
                c.kscale[slot + t] = scale;
                c.vscale[slot + t] = vscale;
            }
        } else {
            if (c.kmean == nullptr) continue;
            code = *reinterpret_cast<const uint2*>(kc + (size_t)t * D + 8 * lt);
            scale = c.kscale[slot + t];
        }
        float z[4];
        widen4<E4M3>(code.x, z);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(z[i], scale, sum[i]);
        widen4<E4M3>(code.y, z);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[4 + i] = __builtin_fmaf(z[i], scale, sum[4 + i]);
    }
    if (c.kmean == nullptr) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[t0][8 * lt + i] = sum[i];
    __syncthreads();
    if (tid < D) {
        float total = 0.f;
#pragma unroll
        for (int i = 0; i < AT; ++i) total += sums[i][tid];
        c.kmean[((size_t)id * c.Hkv + hk) * D + tid] = total / (float)tokens;
    }
}

// ---- tokens come back ----

// D / 16 neighbouring lanes take a token, 16 channels each; a workgroup takes kReadTokens positions of one sequence and head.
constexpr int kReadTokens = 128;
template <int D, bool E4M3>
__global__ __launch_bounds__(kCacheThreads)
void pasa_cache_read_k(pasa_cache c, unsigned short* __restrict__ k, unsigned short* __restrict__ v, const int* __restrict__ first, int N,
                       int io_bf16, FastDiv heads, FastDiv chunks)
{
    constexpr int LT = D / 16, AT = kCacheThreads / LT, PASSES = kReadTokens / AT;
    const int tid = threadIdx.x, lt = tid % LT, t0 = tid / LT;
    const unsigned up = chunks.quotient(blockIdx.x);
    const int n0 = (int)chunks.rest(blockIdx.x, up) * kReadTokens;
    const int b = (int)heads.quotient(up), hk = (int)heads.rest(up, (unsigned)b);
    const int length = clamp_int(c.length[b], 0, c.table_width * c.page), begin = first != nullptr ? first[b] : 0;
    float shift[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) shift[i] = c.kshift != nullptr ? c.kshift[hk * D + 16 * lt + i] : 0.f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int n = n0 + p * AT + t0;
        if (n >= N) break;
        const long long pos = (long long)begin + n;
        uint4 code[2];
        float scale[2] = {0.f, 0.f};
        bool there = pos >= 0 && pos < length;
        if (there) {
            const int place = (int)pos / c.page, id = c.table[(size_t)b * c.table_width + place];
            there = id >= 0 && id < c.pages;
            if (there) {
                const size_t slot = ((size_t)id * c.Hkv + hk) * c.page + (size_t)((int)pos - place * c.page);
                code[0] = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(c.k) + slot * D + 16 * lt);
                code[1] = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(c.v) + slot * D + 16 * lt);
                scale[0] = c.kscale[slot];
                scale[1] = c.vscale[slot];
            }
        }
        const size_t to = (((size_t)b * heads.d + hk) * N + n) * D + 16 * lt;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            unsigned out[8];
            const unsigned w[4] = {code[which].x, code[which].y, code[which].z, code[which].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x[4];
                widen4<E4M3>(w[j], x);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = there ? __builtin_fmaf(x[i], scale[which], which == 0 ? shift[4 * j + i] : 0.f) : 0.f;
                out[2 * j] = io_bf16 ? pack_bf16(x[0], x[1]) : pack_f16(x[0], x[1]);
                out[2 * j + 1] = io_bf16 ? pack_bf16(x[2], x[3]) : pack_f16(x[2], x[3]);
            }
            uint4* dst = reinterpret_cast<uint4*>((which == 0 ? k : v) + to);
            dst[0] = make_uint4(out[0], out[1], out[2], out[3]);
            dst[1] = make_uint4(out[4], out[5], out[6], out[7]);
        }
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

// Four neighbouring lanes take a page, a quarter of the channels each; a workgroup takes 64 pages of one sequence and head.
// The products of fp16 queries and fp32 means are exact in 64 bits, and so, nearly, are their sums: which pages are chosen does
// not depend on an order of additions unless two scores agree to 15 digits.
template <int D>
__global__ __launch_bounds__(kCacheThreads)
void pasa_cache_score_k(pasa_cache c, const unsigned short* __restrict__ q, int R, long long row_stride, const int* __restrict__ row_start,
                        int G, int head, int tail, int io_bf16, FastDiv heads, FastDiv chunks, unsigned long long* __restrict__ scores)
{
    constexpr int CH = D / 4, ROWS = 8;          // channels of a lane, rows that wait in LDS at a time
    __shared__ double rows[ROWS][D + 2];
    const int tid = threadIdx.x, quarter = tid & 3;
    const unsigned up = chunks.quotient(blockIdx.x);
    const int b = (int)heads.quotient(up), hk = (int)heads.rest(up, (unsigned)b);
    const int p = (int)chunks.rest(blockIdx.x, up) * (kCacheThreads / 4) + tid / 4;
    const Sequence s = sequence_at(c.length, row_start, b, R, c.table_width * c.page);
    const int pages = (s.length + c.page - 1) / c.page;
    if ((int)chunks.rest(blockIdx.x, up) * (kCacheThreads / 4) >= pages || s.rows == 0) return;      // nobody reads these words
    const int id = p < pages ? c.table[(size_t)b * c.table_width + p] : -1;
    const bool there = id >= 0 && id < c.pages;
    double mean[CH];
#pragma unroll
    for (int i = 0; i < CH; i += 4) {
        f4 x = (f4)0.f;
        if (there) x = *reinterpret_cast<const f4*>(c.kmean + ((size_t)id * c.Hkv + hk) * D + CH * quarter + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) mean[i + e] = (double)x[e];
    }
    double best = -__builtin_inf();
    bool nan = false;
    const int all = s.rows * G;
    for (int r0 = 0; r0 < all; r0 += ROWS) {
        __syncthreads();
        for (int i = tid; i < ROWS * D; i += kCacheThreads) {
            const int r = r0 + i / D, ch = i % D;
            if (r < all) {
                const unsigned short raw = q[(size_t)(s.row0 + r / G) * (size_t)row_stride + (size_t)(hk * G + r % G) * D + ch];
                rows[i / D][ch] = io_bf16 ? (double)__uint_as_float((unsigned)raw << 16) : (double)__builtin_bit_cast(_Float16, raw);
            }
        }
        __syncthreads();
        const int here = all - r0 < ROWS ? all - r0 : ROWS;
        for (int r = 0; r < here; ++r) {
            double x = 0.0;
#pragma unroll
            for (int i = 0; i < CH; ++i) x = __builtin_fma(mean[i], rows[r][CH * quarter + i], x);
            x += __shfl_xor(x, 1);
            x += __shfl_xor(x, 2);
            nan |= x != x;
            best = __builtin_fmax(best, x);
        }
    }
    if (quarter == 0 && p < pages) {
        const bool always = p < head || p >= pages - tail;
        scores[((size_t)b * c.Hkv + hk) * c.table_width + p] = always ? kAlways : !there ? 1ull : nan ? kAlways - 1 : order_of(best);
    }
}

// One workgroup per sequence and head.  The count-th largest word is found digit by digit (8 bits at a time, from the top; done as soon
// as the words that share the digits so far are all taken); words above it are taken, and of its equals the first.  They leave in order.
template <int EACH>
__global__ __launch_bounds__(kPickThreads)
void pasa_cache_pick_k(pasa_cache c, const int* __restrict__ row_start, int R, int count, FastDiv heads,
                       const unsigned long long* __restrict__ scores, int* __restrict__ blocks)
{
    __shared__ unsigned bins[256];
    __shared__ unsigned sums[kPickThreads / 64][2];
    __shared__ unsigned digit_found, above_found, done;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = (int)heads.quotient(blockIdx.x);
    const Sequence s = sequence_at(c.length, row_start, b, R, c.table_width * c.page);
    const int pages = s.rows == 0 ? 0 : (s.length + c.page - 1) / c.page;
    int* out = blocks + (size_t)blockIdx.x * count;
    const unsigned long long* in = scores + (size_t)blockIdx.x * c.table_width;
    const int taken = pages < count ? pages : count;
    for (int i = taken + tid; i < count; i += kPickThreads) out[i] = -1;
    if (pages <= count) {
        for (int i = tid; i < pages; i += kPickThreads) out[i] = i;
        return;
    }
    // thread t has the words t * EACH .. : in order
    unsigned long long word[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) word[i] = tid * EACH + i < pages ? in[tid * EACH + i] : 0ull;
    unsigned long long prefix = 0;               // digits of the count-th largest so far
    unsigned want = (unsigned)count;             // of the words that share them, so many are taken
    int shift = 56;
    for (;; shift -= 8) {
        if (tid < 256) bins[tid] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (shift == 56 || (word[i] >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&bins[(word[i] >> shift) & 255u], 1u);
        __syncthreads();
        if (tid < 64) {                          // four bins a lane, from the top: lane 0 has 255 .. 252
            unsigned mine[4], total = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) total += mine[i] = bins[255 - 4 * lane - i];
            unsigned upto = total;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const unsigned x = __shfl_up(upto, o);
                if (lane >= o) upto += x;
            }
            unsigned above = upto - total;
            if (above < want && want <= upto) {
                int i = 0;
                while (above + mine[i] < want) above += mine[i++];
                digit_found = 255u - 4u * lane - i;
                above_found = above;
                done = above + mine[i] == want;
            }
        }
        __syncthreads();
        prefix |= (unsigned long long)digit_found << shift;
        want -= above_found;
        if (done || shift == 0) break;
    }
    // words whose digits are above the prefix, and `want` of those that share it
    unsigned above = 0, equal = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        above += (word[i] >> shift) > (prefix >> shift);
        equal += (word[i] >> shift) == (prefix >> shift);
    }
    unsigned up_a = above, up_e = equal;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned x = __shfl_up(up_a, o), y = __shfl_up(up_e, o);
        if (lane >= o) up_a += x, up_e += y;
    }
    if (lane == 63) sums[wave][0] = up_a, sums[wave][1] = up_e;
    __syncthreads();
    unsigned at_a = up_a - above, at_e = up_e - equal;
    for (int w = 0; w < wave; ++w) at_a += sums[w][0], at_e += sums[w][1];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const bool a = (word[i] >> shift) > (prefix >> shift), e = (word[i] >> shift) == (prefix >> shift);
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
    auto go = [&](auto kernel) {
        kernel<<<grid, kCacheThreads, 0, stream>>>(c, static_cast<const unsigned short*>(k), static_cast<const unsigned short*>(v), R, row_stride,
                                                   row_start, io_bf16, fast_div(c.Hkv));
    };
    const bool e = c.format == PASA_CACHE_E4M3;
    if (c.d == 128) e ? go(pasa_cache_write_k<128, true>) : go(pasa_cache_write_k<128, false>);
    else e ? go(pasa_cache_write_k<64, true>) : go(pasa_cache_write_k<64, false>);
    return hipGetLastError();
}

hipError_t pasa_launch_cache_read(const pasa_cache& c, void* k, void* v, const int* first, int N, int io_bf16, hipStream_t stream)
{
    const unsigned chunks = (unsigned)((N + kReadTokens - 1) / kReadTokens), grid = chunks * (unsigned)c.S * (unsigned)c.Hkv;
    auto go = [&](auto kernel) {
        kernel<<<grid, kCacheThreads, 0, stream>>>(c, static_cast<unsigned short*>(k), static_cast<unsigned short*>(v), first, N, io_bf16,
                                                   fast_div(c.Hkv), fast_div(chunks));
    };
    const bool e = c.format == PASA_CACHE_E4M3;
    if (c.d == 128) e ? go(pasa_cache_read_k<128, true>) : go(pasa_cache_read_k<128, false>);
    else e ? go(pasa_cache_read_k<64, true>) : go(pasa_cache_read_k<64, false>);
    return hipGetLastError();
}

hipError_t pasa_launch_cache_choose(const pasa_cache& c, const void* q, int R, long long row_stride, const int* row_start, int Hq,
                                    int count, int head, int tail, int* blocks, int io_bf16, unsigned long long* scores, hipStream_t stream)
{
    if (c.table_width > count) {                 // otherwise all pages are taken
        const unsigned chunks = (unsigned)((c.table_width + 63) / 64), grid = chunks * (unsigned)c.S * (unsigned)c.Hkv;
        auto score = [&](auto kernel) {
            kernel<<<grid, kCacheThreads, 0, stream>>>(c, static_cast<const unsigned short*>(q), R, row_stride, row_start, Hq / c.Hkv, head, tail,
                                                       io_bf16, fast_div(c.Hkv), fast_div(chunks), scores);
        };
        c.d == 128 ? score(pasa_cache_score_k<128>) : score(pasa_cache_score_k<64>);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    auto pick = [&](auto kernel) {
        kernel<<<(unsigned)c.S * (unsigned)c.Hkv, kPickThreads, 0, stream>>>(c, row_start, R, count, fast_div(c.Hkv), scores, blocks);
    };
    if (c.table_width <= kPickThreads) pick(pasa_cache_pick_k<1>);
    else if (c.table_width <= 4 * kPickThreads) pick(pasa_cache_pick_k<4>);
    else pick(pasa_cache_pick_k<16>);            // the largest table: 262144 tokens in pages of 16
    return hipGetLastError();
}
