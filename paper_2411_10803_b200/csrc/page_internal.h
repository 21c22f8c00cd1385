// Declarations shared by the kernels of the paged 4-bit cache (page_cache.cu, page_attend.cu).
#pragma once

#include "mustdrop_internal.h"

namespace mustdrop {

constexpr int kPageGroup = 32;          // channels that share a scale and a centre
constexpr int kChunkTokens = 16;        // tokens of a chunk, the unit the attention kernel reads
constexpr int kTicketWord = 32;         // int32 word of the workspace that mustdrop_page_tables counts its CTAs in

// A chunk's parts, in bytes (the layout is described in mustdrop.h).
template <int D>
struct Chunk {
  static constexpr int kG = D / kPageGroup;
  static constexpr int kK = 0, kV = 8 * D, kKsz = 16 * D, kVs = 18 * D, kVz = 19 * D, kBytes = 20 * D;
};

// Row of a chunk's token: even tokens in rows 0..7, odd ones in rows 8..15.
__host__ __device__ inline int chunk_row(int token) { return ((token & 15) >> 1) | ((token & 1) << 3); }

inline int page_log2(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : -1; }

inline bool misaligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// The sizes every call of the family needs.
mustdrop_status_t check_page_sizes(const mustdrop_page_config_t* c);
mustdrop_status_t check_page_pool(const mustdrop_page_config_t* c);     // ... and the pool's
mustdrop_status_t check_page_queries(const mustdrop_page_config_t* c);  // ... and the query rows of mustdrop_page_attend
size_t page_attend_partial_bytes(const mustdrop_page_config_t* c);      // partial results in the workspace (of a checked configuration)

}  // namespace mustdrop
