// The paged cache and its operators as a translation unit of its own, compiled beside vitint_lib.cu.
#include "qk_norm_rotate.cu"
#include "cache_evict.cu"
#include "paged_attention.cu"
#include "cache_weigh.cu"

int vitint::take_cache_status_word() { return g_cache_called.load(std::memory_order_relaxed) ? take_status_word() : VITINT_OK; }
