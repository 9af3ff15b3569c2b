// Between the entry points of the decode calls on caches of codes and their kernel's instances.
#pragma once

#include "decode_common.hpp"
#include "quant_common.hpp"

namespace kk {

struct QuantParams {
  DecodeParams d;
  float *k_scale, *v_scale;
};

// Launches the instance for a group size and plan; per dtype (T: uint16_t for bf16, float) and head dimension in a source of its own.
template <typename T, int D>
keepkv_status launch_quant(const QuantParams& p, int units, int G, bool step, hipStream_t st);

}  // namespace kk
