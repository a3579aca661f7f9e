// Internal launch interface of the paged cache's management (not part of the ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "seq_launch.h"

struct WaPageLaunch {
  int32_t* refs;
  int32_t* tables;
  int32_t* lens;
  int32_t n_pages, sequences, width, shift;  // shift: log2 of the tokens of a page
  unsigned char* pool;
  int64_t page_bytes;
  int32_t planes;
  const int32_t* first;   // new lengths, parents, slots or sources
  const int32_t* second;  // children or destinations
  int32_t entries;
  int32_t* out_refs;
  int32_t* out_tables;
  int32_t* used;
  int32_t* status;
  int32_t* ws;            // wa_page_ws_ints int32
};

size_t wa_page_ws_ints(const WaPageLaunch& a);  // for the shape, entries included
hipError_t wa_launch_page_grow(const WaPageLaunch& a, hipStream_t stream);
hipError_t wa_launch_page_fork(const WaPageLaunch& a, hipStream_t stream);
hipError_t wa_launch_page_free(const WaPageLaunch& a, hipStream_t stream);
hipError_t wa_launch_page_compact(const WaPageLaunch& a, hipStream_t stream);
hipError_t wa_launch_page_copy(const WaPageLaunch& a, hipStream_t stream);
// a: k, v (rows), kp, vp, tables, starts, kv_lens, status, batch, tokens, kv_heads, head_dim
hipError_t wa_launch_page_store(const WaSeqLaunch& a, hipStream_t stream);
