// Internal interface of the paged 8-bit cache: what its host layer and its kernels share.  Not installed.
#ifndef PASA_CACHE_H
#define PASA_CACHE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pasa.h"
#include "pasa_device.h"

constexpr int kCacheThreads = 256;     // of a workgroup, in all the cache's kernels but the one that picks pages
constexpr int kPickThreads = 1024;

// The kernels of attention over the cache: rows per workgroup are 16 * row_blocks, `grid` workgroups share the units of work.
struct CachePlan {
    int row_blocks, grid;
};
constexpr int kUnit = 64;              // keys of a unit of work (of one wavefront)
constexpr int kUnitsAtOnce = 4;        // wavefronts of a workgroup: units that it sweeps at a time

// Per slot and row: sum of P and level, then the stored output; two slots per workgroup.
__host__ __device__ inline size_t cache_slot_floats(int row_blocks, int d) { return (size_t)16 * row_blocks * (d + 2); }

hipError_t pasa_launch_cache_write(const pasa_cache& c, const void* k, const void* v, int R, long long row_stride, const int* row_start,
                                   int io_bf16, hipStream_t stream);
hipError_t pasa_launch_cache_read(const pasa_cache& c, void* k, void* v, const int* first, int N, int io_bf16, hipStream_t stream);
// scores: [S][Hkv][table_width] 64-bit words
hipError_t pasa_launch_cache_choose(const pasa_cache& c, const void* q, int R, long long row_stride, const int* row_start, int Hq,
                                    int count, int head, int tail, int* blocks, int io_bf16, unsigned long long* scores, hipStream_t stream);
hipError_t pasa_launch_attn_cache(const pasa_cache& c, const void* q, void* o, int R, long long row_stride, const int* row_start, int Hq,
                                  float scale, const unsigned long long* tree, const int* blocks, int count, int io_bf16,
                                  const CachePlan& plan, float* slots, hipStream_t stream);

#ifdef __HIPCC__
namespace {

__device__ inline int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// What the device memory says of a sequence, kept to what the buffers hold.
struct Sequence {
    int length, row0, rows;            // tokens, first of its rows, how many
};
__device__ inline Sequence sequence_at(const int* __restrict__ length, const int* __restrict__ row_start, int b, int R, int most)
{
    Sequence s;
    s.length = clamp_int(length[b], 0, most);
    s.row0 = clamp_int(row_start[b], 0, R);
    const int end = clamp_int(row_start[b + 1], 0, R);
    s.rows = end > s.row0 ? end - s.row0 : 0;
    return s;
}

// A workgroup's place in work that is shared out over the sequences: sequence b has count(b) pieces, and piece `at(total)` of all
// lies in sequence `b`, the `rest`-th there.  b < 0 where there is no such piece.  All threads call it; every thread counts its own share of the sequences,
// one scan over the threads finds who has the piece, and that one walks its share.
struct Place {
    int b;
    unsigned rest, total;
};
template <class Count, class At>
__device__ inline Place find_place(int S, Count count, At at)
{
    __shared__ unsigned sums[kCacheThreads / 64];
    __shared__ int found_b;
    __shared__ unsigned found_rest;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (S + kCacheThreads - 1) / kCacheThreads, b0 = tid * each;
    unsigned mine = 0;
    for (int i = 0; i < each; ++i)
        if (b0 + i < S) mine += count(b0 + i);
    unsigned upto = mine;              // inclusive scan over the wavefront
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned x = __shfl_up(upto, o);
        if (lane >= o) upto += x;
    }
    if (tid == 0) found_b = -1;
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    Place p;
    p.total = 0;
    unsigned before = upto - mine;
#pragma unroll
    for (int w = 0; w < kCacheThreads / 64; ++w) {
        if (w < wave) before += sums[w];
        p.total += sums[w];
    }
    const unsigned want = at(p.total);
    if (want >= before && want < before + mine) {
        int b = b0;
        unsigned left = want - before;
        for (unsigned c = count(b); left >= c && b < b0 + each; c = count(b)) {
            left -= c;
            if (++b >= S) break;
        }
        found_b = b < S && b < b0 + each ? b : -1;
        found_rest = left;
    }
    __syncthreads();
    p.b = __builtin_amdgcn_readfirstlane(found_b);
    p.rest = __builtin_amdgcn_readfirstlane(found_rest);
    p.total = __builtin_amdgcn_readfirstlane(p.total);
    return p;
}

// Four e4m3 or excess-128 bytes -> fp32, exactly
template <bool E4M3>
__device__ inline void widen4(unsigned w, float (&x)[4])
{
    if (E4M3) {
        const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)((w >> (8 * i)) & 255u) - 128.f;
    }
}

}  // namespace
#endif
#endif
