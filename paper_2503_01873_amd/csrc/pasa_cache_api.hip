// Host layer of the paged 8-bit cache: the entry points of include/pasa.h that take a pasa_cache.  Argument validation and dispatch.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "pasa.h"
#include "pasa_cache.h"

namespace {

constexpr long long kMaxTokens = 262144;         // of a sequence, as in the other entry points
constexpr long long kMaxGrid = 0x7fffffff;       // of what the kernels count in 31 bits
constexpr long long kMaxThreads = 0xffffffff;    // of a launch: the hardware counts them in 32 bits
constexpr int kComputeUnits = 256;               // MI355X

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool fits(long long workgroups, int threads) { return workgroups <= kMaxThreads / threads; }
bool buffer(const void* p, uintptr_t a) { return p != nullptr && aligned(p, a); }

int check_cache(const pasa_cache* c)
{
    if (c == nullptr) return PASA_EINVAL;
    if (!buffer(c->k, 16) || !buffer(c->v, 16) || c->k == c->v || !buffer(c->kscale, 16) || !buffer(c->vscale, 16) ||
        c->kscale == c->vscale || !aligned(c->kmean, 16) || !aligned(c->kshift, 16) || !buffer(c->table, 4) || !buffer(c->length, 4))
        return PASA_EINVAL;
    if (c->S <= 0 || c->Hkv <= 0 || c->pages <= 0 || c->table_width <= 0 || c->d <= 0 || c->page <= 0) return PASA_EINVAL;
    if (c->format != PASA_CACHE_I8 && c->format != PASA_CACHE_E4M3) return PASA_EINVAL;
    if (c->d != 64 && c->d != 128) return PASA_EUNSUPPORTED;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return PASA_EUNSUPPORTED;
    if ((long long)c->table_width * c->page > kMaxTokens || (long long)c->S * c->Hkv > kMaxGrid) return PASA_EUNSUPPORTED;
    return PASA_OK;
}

// R rows of `heads` heads at p
int check_rows(const pasa_cache* c, const void* p, int R, long long row_stride, const int* row_start, int heads, int io_dtype)
{
    if (!buffer(p, 16) || !buffer(row_start, 4) || R <= 0 || heads <= 0) return PASA_EINVAL;
    if (row_stride < (long long)heads * c->d || row_stride % 8 != 0) return PASA_EINVAL;
    if (io_dtype != PASA_IO_F16 && io_dtype != PASA_IO_BF16) return PASA_EINVAL;
    if (R > kMaxGrid - 1) return PASA_EUNSUPPORTED;
    return PASA_OK;
}

int check_workspace(const void* ws, size_t bytes, size_t need) { return buffer(ws, 256) && bytes >= need ? PASA_OK : PASA_EWORKSPACE; }

// Rows per workgroup: 16 where the rows of a KV head fill no more on average, 32 otherwise (16 sequences of 8192 keys, 28 heads on 4, four rows each, that is 28 rows: 39.5 us, in
// blocks of 16, which read the keys twice, 45.2; 8 of 30000 keys, 8 KV heads, 20 rows: 103 / 153).  Workgroups: one to a compute unit (their eight
// wavefronts take its registers), and no more than there are blocks of rows or leave each wavefront a unit.  Never cut: up to 1024 keys, where a merge costs
// what it saves (us, never / cut: one sequence of 500 keys 10.6 / 12.4, of 1024 13.8 / 13.8, 64 of 1024 15.5 / 17.4; one of 2048 19.1 / 13.8).  All of it goes by what tables
// hold, as lengths are on the device: 16 ragged sequences of up to 500 keys in tables of 262144 tokens 13.9 us, in tables that fit 10.5; of up to 4096, 19.9 and 19.1.  False where
// the units, with what blocks cost beside them, do not fit 31 bits.
bool plan_of(const pasa_cache& c, int R, int Hq, int count, CachePlan* plan)
{
    const long long G = Hq / c.Hkv;
    plan->row_blocks = (long long)R * G <= 16LL * c.S ? 1 : 2;
    const long long pages = count > 0 && count < c.table_width ? count : c.table_width, units = (pages * c.page + kUnit - 1) / kUnit;
    const long long blocks = (long long)R * G / (16 * plan->row_blocks) + c.S;      // of rows, at most
    if (R * G > kMaxGrid || blocks > kMaxGrid / c.Hkv || blocks * c.Hkv > kMaxGrid / (units + 40)) return false;
    const long long pairs = blocks * c.Hkv, filled = (pairs * units + kUnitsAtOnce - 1) / kUnitsAtOnce, all = pairs > filled ? pairs : filled;
    plan->grid = (int)(all < kComputeUnits ? all : kComputeUnits);
    plan->never_cut = units <= 16;
    return true;
}

size_t attn_workspace_bytes(const pasa_cache& c, const CachePlan& plan)
{
    return (plan.grid * (sizeof(MergeRecord) + 2 * cache_slot_floats(plan.row_blocks, c.d) * sizeof(float)) + 255) / 256 * 256;
}

size_t choose_workspace_bytes(const pasa_cache& c) { return ((size_t)8 * c.S * c.Hkv * c.table_width + 255) / 256 * 256; }

int status(hipError_t e) { return e == hipSuccess ? PASA_OK : PASA_ELAUNCH; }

}  // namespace

extern "C" {

int pasa_cache_write(const pasa_cache* cache, const void* k, const void* v, int R, long long row_stride, const int* row_start, int io_dtype,
                     void* stream)
{
    int st = check_cache(cache);
    if (st != PASA_OK) return st;
    st = check_rows(cache, k, R, row_stride, row_start, cache->Hkv, io_dtype);
    if (st != PASA_OK) return st;
    if (!buffer(v, 16)) return PASA_EINVAL;
    const long long most = (long long)R / cache->page + 2LL * cache->S;  // pages that are written to
    if (!fits((most < R ? most : R) * cache->Hkv, 512)) return PASA_EUNSUPPORTED;
    return status(pasa_launch_cache_write(*cache, k, v, R, row_stride, row_start, io_dtype == PASA_IO_BF16, static_cast<hipStream_t>(stream)));
}

int pasa_cache_read(const pasa_cache* cache, void* k, void* v, const int* first, int N, int io_dtype, void* stream)
{
    const int st = check_cache(cache);
    if (st != PASA_OK) return st;
    if (!buffer(k, 16) || !buffer(v, 16) || k == v || !aligned(first, 4) || N <= 0) return PASA_EINVAL;
    if (io_dtype != PASA_IO_F16 && io_dtype != PASA_IO_BF16) return PASA_EINVAL;
    if (N > kMaxTokens || !fits((((long long)N + 63) / 64) * cache->S * cache->Hkv, kCacheThreads)) return PASA_EUNSUPPORTED;
    return status(pasa_launch_cache_read(*cache, k, v, first, N, io_dtype == PASA_IO_BF16, static_cast<hipStream_t>(stream)));
}

size_t pasa_cache_choose_workspace(const pasa_cache* cache) { return check_cache(cache) == PASA_OK ? choose_workspace_bytes(*cache) : 0; }

int pasa_cache_choose(const pasa_cache* cache, const void* q, int R, long long row_stride, const int* row_start, int Hq, int* blocks, int count,
                      int head, int tail, int io_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    int st = check_cache(cache);
    if (st != PASA_OK) return st;
    st = check_rows(cache, q, R, row_stride, row_start, Hq, io_dtype);
    if (st != PASA_OK) return st;
    if (Hq % cache->Hkv != 0 || cache->kmean == nullptr || !buffer(blocks, 4) || count < 1 || head < 0 || tail < 0) return PASA_EINVAL;
    const long long lists = (long long)cache->S * cache->Hkv;
    if (count > kMaxTokens || (long long)R * (Hq / cache->Hkv) > kMaxGrid || !fits(lists, 1024) ||
        (cache->table_width > count && !fits(((long long)cache->table_width + 63) / 64 * lists, kCacheThreads)))
        return PASA_EUNSUPPORTED;
    st = check_workspace(workspace, workspace_bytes, choose_workspace_bytes(*cache));
    if (st != PASA_OK) return st;
    return status(pasa_launch_cache_choose(*cache, q, R, row_stride, row_start, Hq, count, head, tail, blocks, io_dtype == PASA_IO_BF16,
                                           static_cast<unsigned long long*>(workspace), static_cast<hipStream_t>(stream)));
}

size_t pasa_attn_cache_workspace(const pasa_cache* cache, int R, int Hq)
{
    CachePlan plan;
    if (check_cache(cache) != PASA_OK || R <= 0 || Hq <= 0 || Hq % cache->Hkv != 0 || !plan_of(*cache, R, Hq, 0, &plan)) return 0;
    size_t bytes = attn_workspace_bytes(*cache, plan);
    if (plan.row_blocks == 2) {                  // as many rows as go in blocks of 16: half the slot, but more workgroups where there are few
        const int rows = (int)(16LL * cache->S / (Hq / cache->Hkv));
        if (rows > 0 && plan_of(*cache, rows, Hq, 0, &plan)) {
            const size_t fewer = attn_workspace_bytes(*cache, plan);
            if (fewer > bytes) bytes = fewer;
        }
    }
    return bytes;
}

int pasa_attn_cache(const pasa_cache* cache, const void* q, void* o, int R, long long row_stride, const int* row_start, int Hq, float scale,
                    const unsigned long long* tree, const int* blocks, int count, int io_dtype, void* workspace, size_t workspace_bytes,
                    void* stream)
{
    int st = check_cache(cache);
    if (st != PASA_OK) return st;
    st = check_rows(cache, q, R, row_stride, row_start, Hq, io_dtype);
    if (st != PASA_OK) return st;
    if (Hq % cache->Hkv != 0 || !buffer(o, 16) || o == q || !isfinite(scale) || !(scale > 0.f)) return PASA_EINVAL;
    if (!aligned(tree, 8) || !aligned(blocks, 4) || (blocks != nullptr && count < 1)) return PASA_EINVAL;
    if (blocks != nullptr && count > kMaxTokens) return PASA_EUNSUPPORTED;
    CachePlan plan;
    if (!plan_of(*cache, R, Hq, 0, &plan)) return PASA_EUNSUPPORTED;
    st = check_workspace(workspace, workspace_bytes, attn_workspace_bytes(*cache, plan));
    if (blocks != nullptr) plan_of(*cache, R, Hq, count, &plan);     // a smaller one
    if (st != PASA_OK) return st;
    return status(pasa_launch_attn_cache(*cache, q, o, R, row_stride, row_start, Hq, scale, tree, blocks, count, io_dtype == PASA_IO_BF16, plan,
                                         workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
