// Attention of new tokens over a paged cache (seq_attn.h).

#include "seq_attn.h"

hipError_t wa_launch_paged_attn(const WaSeqLaunch& a, hipStream_t stream) { return wa::seq_launch_any<true>(a, stream); }
