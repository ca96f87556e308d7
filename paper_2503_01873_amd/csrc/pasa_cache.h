// Internal interface of the paged 8-bit cache: what its host layer and its kernels share.  Not installed.
#ifndef PASA_CACHE_H
#define PASA_CACHE_H

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "pasa.h"
#include "pasa_device.h"

constexpr int kCacheThreads = 256;     // of a workgroup
inline int log2_of(int page)
{
    int n = 0;
    while ((1 << n) < page) ++n;
    return n;
}

// The kernels of attention over the cache: rows per workgroup are 16 * row_blocks, `grid` workgroups share the units of work; no block of rows
// is shared by two of them (and nothing merged) where never_cut.
struct CachePlan {
    int row_blocks, grid, never_cut;
};
constexpr int kUnit = 64;              // keys of a unit of work (of one wavefront)
constexpr int kUnitsAtOnce = 8;        // wavefronts of a workgroup: units that it sweeps at a time

// Workspace: per workgroup a record of what is to be merged, then two slots; in a slot sum of P and level per row, then the rows' stored output.
struct MergeRecord {
    int pieces;                        // 0: none
    int slot, p0, list, row0, hk, unused[2];
};
__host__ __device__ inline size_t cache_slot_floats(int row_blocks, int d) { return (size_t)16 * row_blocks * (d + 2); }

hipError_t pasa_launch_cache_write(const pasa_cache& c, const void* k, const void* v, int R, long long row_stride, const int* row_start,
                                   int io_bf16, hipStream_t stream);
hipError_t pasa_launch_cache_read(const pasa_cache& c, void* k, void* v, const int* first, int N, int io_bf16, hipStream_t stream);
// scores: [S][Hkv][table_width] 64-bit words
hipError_t pasa_launch_cache_choose(const pasa_cache& c, const void* q, int R, long long row_stride, const int* row_start, int Hq,
                                    int count, int head, int tail, int* blocks, int io_bf16, unsigned long long* scores, hipStream_t stream);
hipError_t pasa_launch_attn_cache(const pasa_cache& c, const void* q, void* o, int R, long long row_stride, const int* row_start, int Hq,
                                  float scale, const unsigned long long* tree, const int* blocks, int count, int io_bf16,
                                  const CachePlan& plan, void* workspace, hipStream_t stream);

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

// Sum over the lanes of a wavefront up to and with one's own
__device__ inline unsigned scan64(unsigned x)
{
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);       // row_shr 1, 2, 4, 8: within 16 lanes
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);       // lane 15 to the second 16 lanes, 47 to the fourth
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);       // lane 31 to the upper half
    return x;
}

// Largest over the lanes of a wavefront, in all
__device__ inline unsigned largest64(unsigned x)
{
    auto with = [&](auto control, auto rows) {
        const unsigned y = (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, decltype(control)::value, decltype(rows)::value, 0xf, false);
        x = y > x ? y : x;
    };
    with(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
    with(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    with(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    with(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    with(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    with(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return (unsigned)__builtin_amdgcn_readlane((int)x, 63);
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
