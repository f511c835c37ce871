// Shared by the translation units of the paged cache.
#pragma once

#include "ea_internal.h"

ea_status ea_check_paged_shape(const ea_paged_shape* s);
// Workspace of ea_paged_attention (partial results of lists that several CTAs share).
size_t ea_paged_attn_ws_bytes(const ea_paged_shape& s, int max_q);
