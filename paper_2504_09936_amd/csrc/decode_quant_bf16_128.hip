#include "decode_quant.hpp"

namespace kk {
template keepkv_status launch_quant<uint16_t, 128>(const QuantParams& p, int units, int G, bool step, hipStream_t st);
}
