// What sa_cache4.hip and sa_pages.hip (caches in 4 bits and in pages) offer to the entry points.  Apart from sa_common.h: that one belongs to the
// sources that the traffic records of the other kernels were read with.
#pragma once

#include "sa_common.h"

namespace sa {

// K, V of the rows: written, or (write = false) read back into
hipError_t launch_cache4_rows(const sa_cache4_desc* c, bool write, void* K, void* V, int T, const int32_t* starts,
                              const int32_t* counts, const int32_t* table, void* pool, hipStream_t st);
int cache4_loaded_rows(int start, int count, int T, int half, int32_t* rows);
size_t cache4_decode_workspace_bytes(const sa_cache4_desc* c, int T);
hipError_t launch_cache4_decode(const sa_cache4_desc* c, const void* q, int T, const void* pool, const int32_t* table,
                                const int32_t* lens, int max_len, void* Y, float* LSE, void* ws, hipStream_t st);
int cache4_decode_plan(const sa_cache4_desc* c, int T, int max_len);  // blocks of query rows a wave takes (1, 2) | pieces << 2
int cache4_decode_dealt(const sa_cache4_desc* c, int T, int max_len);  // workgroups a sequence where the kernel may deal pieces by length, 0
size_t pages_extend_workspace_bytes(const sa_cache4_desc* c);
size_t pages_compact_workspace_bytes(const sa_cache4_desc* c);
hipError_t launch_pages_fork(const sa_cache4_desc* c, const int32_t* parents, const int32_t* table, const int32_t* lens, const int32_t* refs,
                             int32_t* table_out, int32_t* lens_out, int32_t* refs_out, hipStream_t st);
hipError_t launch_pages_free(const sa_cache4_desc* c, const int32_t* keep, int32_t* table, int32_t* refs, hipStream_t st);
hipError_t launch_pages_extend(const sa_cache4_desc* c, const int32_t* lens, const int32_t* add, int32_t* table, int32_t* refs, void* pool,
                               int32_t* info, void* ws, hipStream_t st);
hipError_t launch_pages_compact(const sa_cache4_desc* c, int max_moves, const int32_t* table, const int32_t* refs, int32_t* table_out,
                                int32_t* refs_out, void* pool, int32_t* info, void* ws, hipStream_t st);

}  // namespace sa

// For the tests, not part of include/sa.h.
extern "C" {
// how sa_cache4_decode_fwd is dealt: cache4_decode_plan, 0 for what it refuses
int sa_internal_cache4_plan(const sa_cache4_desc* desc, int T, int max_len);
int sa_internal_cache4_dealt(const sa_cache4_desc* desc, int T, int max_len);
// the 16 rows of K and V that sa_cache4_write loads for a half of a tile (counted from the one that holds the first position): 1, 0 if it
// loads none there, -1 past the last half that is looked at
int sa_internal_cache4_loaded_rows(int32_t start, int32_t count, int32_t T, int half, int32_t* rows);
}
