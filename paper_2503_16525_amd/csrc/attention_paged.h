// Internal declarations shared by the translation units of kvs_attention_paged (not part of the ABI).
#pragma once

#include "paged.h"

namespace kvs {

// Pieces of a cut launch leave, for each row and piece (slot = row * pieces + piece), unnormalised fp32 sums and (exponent reference, sum of the
// weights, sum of the weights as the second product saw them, unused); a piece without keys a sum of 0.
inline size_t paged_slot_bytes(int d) { return (size_t)d * sizeof(float) + sizeof(float4); }
constexpr int kPagedMaxPieces = 512;
struct PagedParts { float4 *ml; float *o; };
inline PagedParts paged_parts(void *workspace, int64_t slots)
{
    float4 *ml = reinterpret_cast<float4 *>(workspace);
    return {ml, reinterpret_cast<float *>(ml + slots)};
}
kvs_status launch_merge_paged(const kvs_shape *shape, const Paged &pg, int pieces, const PagedParts &parts, void *out, float *lse_out, hipStream_t hs);

// What the host knows of a call, and what it expects of its requests: all alike, and their contexts as long as they can be.
struct PagedCall {
    int64_t items;            // rows of all heads
    int32_t grp, row_blocks;  // blocks of 32 rows a request
    int32_t row_tiles;        // of 256
    double merge_us;          // of one piece: bytes written and read
};
inline PagedCall describe(const kvs_shape *shape, const Paged &pg)
{
    PagedCall c;
    c.grp = shape->n_q_heads / shape->n_kv_heads;
    c.items = (int64_t)pg.n_new * shape->n_q_heads;
    const int64_t rows = ((int64_t)pg.n_new * c.grp + pg.batch - 1) / pg.batch;
    c.row_blocks = (int32_t)((rows + 31) / 32);
    c.row_tiles = (int32_t)((rows + 255) / 256);
    c.merge_us = 2.0 * (double)c.items * (double)paged_slot_bytes(shape->head_dim) / 3.5e6;
    return c;
}
// The order of a launch's workgroups: (piece, KV head) pairs dealt to the eight XCDs where that comes out even, so that the blocks that read the
// same keys share an L2; else KV heads side by side.
struct PagedPlace { int piece, g, unit; };
__device__ __forceinline__ PagedPlace place_of(uint32_t wg, int units, int pieces, int n_kv_heads)
{
    if (pieces > 1 && pieces * n_kv_heads % 8 == 0) {
        const uint32_t slot = wg / 8, stream = slot / (uint32_t)units * 8 + wg % 8;
        return {(int)(stream / (uint32_t)n_kv_heads), (int)(stream % (uint32_t)n_kv_heads), (int)(slot % (uint32_t)units)};
    }
    const uint32_t rest = wg / (uint32_t)n_kv_heads;
    return {(int)(rest / (uint32_t)units), (int)(wg % (uint32_t)n_kv_heads), (int)(rest % (uint32_t)units)};
}

// 256 rows a workgroup (attention_paged_large.hip): whether a call can go there, how its keys are cut and about how long that takes.
struct PagedLargePlan { int32_t pieces, tiles; int64_t units; double us; bool dealt; };
bool attention_paged_takes_large(const kvs_shape *shape, const Paged &pg, const PagedCall &call, float scale, size_t workspace_bytes, PagedLargePlan *plan);
kvs_status launch_attention_paged_large(const kvs_shape *shape, const kvs_paged_cache *cache, const Paged &pg, const PagedLargePlan &plan, const void *q, float scale,
                                        void *out, float *lse_out, void *workspace, hipStream_t hs);
size_t attention_paged_large_workspace_bytes(const kvs_shape *shape, int32_t batch, int64_t n_new);
constexpr int kPagedLargeRows = 256;
// The test suite builds a second library, in which every call that the kernel of many rows can take goes there, its keys in so many pieces
// (0: as estimated).  The shipped one has no switch.
#ifdef KVS_PAGED_TEST
extern int32_t paged_forced_pieces;
#else
constexpr int32_t paged_forced_pieces = 0;
#endif
// The rows of those of its workgroups that say so once more, with the other kernel (attention_paged.hip); odd: one word a workgroup.
kvs_status launch_again_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const Paged &pg, const PagedLargePlan &plan, const int32_t *odd, const void *q, float scale,
                              void *out, float *lse_out, hipStream_t hs);

} // namespace kvs
