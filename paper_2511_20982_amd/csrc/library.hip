// libdopd_attn.so is one translation unit: the attention hot path and its host
// helpers, then the entry points that build on them.
#include "dopd_attn.hip"

#include "dopd_variants.hpp"
