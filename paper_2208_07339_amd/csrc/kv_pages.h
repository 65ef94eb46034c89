// Launchers of kv_pages.hip.  Their arguments have been checked.
#pragma once
#include "kv.h"

namespace llmint8 {

constexpr int KV_MAX_PAGE = 1 << 20;  // positions to a page: counts of a page's pieces stay far below 2^31

hipError_t launch_kv_fork(const llmint8_kv_pool_t& p, const llmint8_kv_seqs_t& s, const int* parent, int grow,
                          const llmint8_kv_moves_t& m, hipStream_t st);
hipError_t launch_kv_reserve(const llmint8_kv_pool_t& p, const llmint8_kv_seqs_t& s, const int* row_start, int* ready, int more,
                             const llmint8_kv_moves_t& m, hipStream_t st);
hipError_t launch_kv_compact(const llmint8_kv_pool_t& p, const llmint8_kv_seqs_t& s, int* used, const llmint8_kv_moves_t& m, hipStream_t st);
hipError_t launch_kv_copy(const llmint8_kv_cache_t& c, const llmint8_kv_moves_t& m, int* status, hipStream_t st);

}  // namespace llmint8
