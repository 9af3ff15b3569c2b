// keepkv_quantize, keepkv_dequantize, keepkv_append_quant: rows into e4m3 codes with a power-of-two scale per block of 32 slots,
// and back.  All three move bytes; the arithmetic is a maximum, a multiplication and a conversion per element.
#include <type_traits>

#include "quant_common.hpp"

namespace kk {
namespace {

// What the slots carry beside their rows.
struct SlotState {
  const int32_t *votes, *born;
  const float* log_s;
  const int32_t *t_obs, *len;
};
struct SlotStateOut {
  int32_t *votes, *born;
  float* log_s;
  int32_t *t_obs, *len;
};
SlotState state_of(const keepkv_cache& c) { return {c.votes, c.born, c.log_s, c.t_obs, c.len}; }
SlotStateOut state_out(const keepkv_cache& c) { return {c.votes, c.born, c.log_s, c.t_obs, c.len}; }

// One wavefront per (head, block, K or V): task = (head * blocks + block) * 2 + (0: K, 1: V).
constexpr int kTaskWaves = 4;
constexpr int64_t kMaxTasks = ((int64_t)1 << 26) - kTaskWaves;   // a launch has fewer than 2^32 threads (256 GiB of rows)

// The wavefront of a block's K also copies what its slots carry, that of block 0 the head's words.
__device__ __forceinline__ void copy_state(const SlotState& s, const SlotStateOut& d, size_t unit, int s_cap, int d_cap, int block, int n_live, int n,
                                           int lane) {
  if (lane < n_live) {
    const size_t a = unit * s_cap + block * kQBlock + lane, b = unit * d_cap + block * kQBlock + lane;
    d.votes[b] = s.votes[a];
    d.log_s[b] = s.log_s[a];
    d.born[b] = s.born[a];
  }
  if (block == 0 && lane == 0) {
    d.t_obs[unit] = s.t_obs[unit];
    d.len[unit] = n;
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kTaskWaves* kWave) void quantize_kernel(const void* k, const void* v, uint8_t* qk, uint8_t* qv, float* k_scale,
                                                                      float* v_scale, SlotState s, SlotStateOut d, int s_cap, int d_cap,
                                                                      int64_t tasks) {
  constexpr int EPV = 16 / (int)sizeof(T);        // elements of a 16-byte vector
  constexpr int VPL = 16 / EPV;                   // vectors that make 16 codes
  constexpr int STEPS = kQBlock * D / 16 / kWave; // 16 codes of every lane at a time
  const int64_t task = (int64_t)blockIdx.x * kTaskWaves + (threadIdx.x >> 6);
  if (task >= tasks) return;
  const int lane = threadIdx.x & 63;
  const int blocks = quant_blocks(s_cap);
  const bool is_v = task & 1;
  const size_t unit = (size_t)((task >> 1) / blocks);
  const int block = (int)((task >> 1) % blocks);
  const int n = s.len[unit], n_live = min(n - block * kQBlock, kQBlock);
  if (!is_v) copy_state(s, d, unit, s_cap, d_cap, block, n_live, n, lane);
  if (n_live <= 0) return;
  const uint4* src = reinterpret_cast<const uint4*>(is_v ? v : k) + (unit * s_cap + (size_t)block * kQBlock) * (D / EPV);
  float x[STEPS][VPL][EPV];
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int at = i * kWave + lane;              // the at-th 16 elements of the block
    const bool live = at * 16 / D < n_live;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      to_f32(live ? load_once(src + at * VPL + j) : make_uint4(0, 0, 0, 0), x[i][j]);
#pragma unroll
      for (int e = 0; e < EPV; ++e) amax = max(amax, finite_magnitude(x[i][j][e]));
    }
  }
  const uint32_t sb = scale_bits(wave_max(amax));
  const float inv = inverse_scale(sb);
  uint4* dst = reinterpret_cast<uint4*>((is_v ? qv : qk) + (unit * d_cap + (size_t)block * kQBlock) * D);
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int at = i * kWave + lane;
    uint32_t w[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      auto el = [&](int e) { return x[i][(4 * c + e) / EPV][(4 * c + e) % EPV] * inv; };
      w[c] = encode4(el(0), el(1), el(2), el(3));
    }
    if (at * 16 / D < n_live) dst[at] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  if (lane == 0) (is_v ? v_scale : k_scale)[unit * quant_blocks(d_cap) + block] = __builtin_bit_cast(float, sb);
}

template <typename T, int D>
__global__ __launch_bounds__(kTaskWaves* kWave) void dequantize_kernel(const uint8_t* qk, const uint8_t* qv, const float* k_scale,
                                                                        const float* v_scale, void* k, void* v, SlotState s, SlotStateOut d,
                                                                        int s_cap, int d_cap, int64_t tasks) {
  constexpr int EPV = 16 / (int)sizeof(T);
  constexpr int VPL = 16 / EPV;
  constexpr int STEPS = kQBlock * D / 16 / kWave;
  const int64_t task = (int64_t)blockIdx.x * kTaskWaves + (threadIdx.x >> 6);
  if (task >= tasks) return;
  const int lane = threadIdx.x & 63;
  const int blocks = quant_blocks(s_cap);
  const bool is_v = task & 1;
  const size_t unit = (size_t)((task >> 1) / blocks);
  const int block = (int)((task >> 1) % blocks);
  const int n = s.len[unit], n_live = min(n - block * kQBlock, kQBlock);
  if (!is_v) copy_state(s, d, unit, s_cap, d_cap, block, n_live, n, lane);
  if (n_live <= 0) return;
  const float scale = (is_v ? v_scale : k_scale)[unit * blocks + block];
  const uint4* src = reinterpret_cast<const uint4*>((is_v ? qv : qk) + (unit * s_cap + (size_t)block * kQBlock) * D);
  uint4* dst = reinterpret_cast<uint4*>(is_v ? v : k) + (unit * d_cap + (size_t)block * kQBlock) * (D / EPV);
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int at = i * kWave + lane;
    if (at * 16 / D >= n_live) break;
    const uint4 c = load_once(src + at);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    float x[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float y[4];
      decode4(w[j], y);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * j + e] = y[e] * scale;
    }
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      uint4 o;
      if constexpr (EPV == 4)
        o = make_uint4(__builtin_bit_cast(uint32_t, x[4 * j]), __builtin_bit_cast(uint32_t, x[4 * j + 1]),
                       __builtin_bit_cast(uint32_t, x[4 * j + 2]), __builtin_bit_cast(uint32_t, x[4 * j + 3]));
      else
        o = make_uint4(pack_bf16x2(x[8 * j], x[8 * j + 1]), pack_bf16x2(x[8 * j + 2], x[8 * j + 3]),
                       pack_bf16x2(x[8 * j + 4], x[8 * j + 5]), pack_bf16x2(x[8 * j + 6], x[8 * j + 7]));
      dst[at * VPL + j] = o;
    }
  }
}

// One workgroup per head; its wavefronts take the touched blocks' K and V in turn.  (The length is read by all of them and
// moved on behind a barrier.)
template <typename T, int D>
__global__ __launch_bounds__(256) void append_quant_kernel(uint8_t* qk, uint8_t* qv, float* k_scale, float* v_scale, SlotStateOut s, const T* k_t,
                                                           const T* v_t, const int32_t* counts, int32_t* overflow, int n_tokens, int capacity) {
  constexpr int EPV = 16 / (int)sizeof(T);
  constexpr int VPL = 16 / EPV;
  constexpr int LPR = D / 16;                     // lanes per row: 16 codes each
  constexpr int RPI = kWave / LPR;                // rows at a time
  const size_t unit = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int n = s.len[unit];
  const int want = counts ? min(max(counts[unit], 0), n_tokens) : n_tokens;
  const int take = min(want, capacity - n);
  const int born = s.t_obs[unit];
  const int first = n / kQBlock, last = (n + take - 1) / kQBlock;      // blocks (take > 0)
  const int sub = lane % LPR, row0 = lane / LPR;
  for (int task = wave; take > 0 && task < 2 * (last - first + 1); task += waves) {
    const bool is_v = task & 1;
    const int block = first + (task >> 1), base = block * kQBlock;
    const int from = max(n, base), to = min(n + take, base + kQBlock);
    const uint4* src = reinterpret_cast<const uint4*>(is_v ? v_t : k_t) + (unit * n_tokens - (ptrdiff_t)n) * (D / EPV) + sub * VPL;
    uint4* rows = reinterpret_cast<uint4*>((is_v ? qv : qk) + (unit * capacity + (size_t)base) * D) + sub;
    float* scale = (is_v ? v_scale : k_scale) + unit * quant_blocks(capacity) + block;
    uint32_t amax = 0;
    for (int r = from + row0; r < to; r += RPI)
#pragma unroll
      for (int j = 0; j < VPL; ++j) {
        float x[EPV];
        to_f32(src[(ptrdiff_t)r * (D / EPV) + j], x);
#pragma unroll
        for (int e = 0; e < EPV; ++e) amax = max(amax, finite_magnitude(x[e]));
      }
    uint32_t sb = scale_bits(wave_max(amax));
    if (from > base) {                            // the block held live slots
      const uint32_t old = __builtin_bit_cast(uint32_t, *scale);
      sb = max(sb, old);
      if (sb != old) {
        const float ratio = __builtin_bit_cast(float, old) * inverse_scale(sb);
        for (int r = row0; r < from - base; r += RPI) {
          uint4 c = rows[r * LPR];
          c = make_uint4(shift_codes(c.x, ratio), shift_codes(c.y, ratio), shift_codes(c.z, ratio), shift_codes(c.w, ratio));
          rows[r * LPR] = c;
        }
      }
    }
    const float inv = inverse_scale(sb);
    for (int r = from + row0; r < to; r += RPI) {
      float x[VPL][EPV];
#pragma unroll
      for (int j = 0; j < VPL; ++j) to_f32(src[(ptrdiff_t)r * (D / EPV) + j], x[j]);
      uint32_t w[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        auto el = [&](int e) { return x[(4 * c + e) / EPV][(4 * c + e) % EPV] * inv; };
        w[c] = encode4(el(0), el(1), el(2), el(3));
      }
      rows[(r - base) * LPR] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (lane == 0) *scale = __builtin_bit_cast(float, sb);
    if (!is_v && from + lane < to) {
      const size_t at = unit * capacity + from + lane;
      s.votes[at] = 1;
      s.log_s[at] = -INFINITY;
      s.born[at] = born;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    if (take > 0) s.len[unit] = n + take;
    if (take < want && overflow != nullptr) *overflow = 1;
  }
}

bool rows_aligned(const keepkv_cache& c) { return aligned16(c.k) && aligned16(c.v); }

// f(element type, head dim)
template <typename F>
void by_layout(const keepkv_layout* L, F f) {
  auto dim = [&](auto t) {
    if (L->head_dim == 128) f(t, std::integral_constant<int, 128>{});
    else f(t, std::integral_constant<int, 64>{});
  };
  if (L->dtype == KEEPKV_BF16) dim(uint16_t{});
  else dim(float{});
}

}  // namespace
}  // namespace kk

extern "C" keepkv_status keepkv_quantize(const keepkv_layout* layout, const keepkv_cache* src, keepkv_quant_cache* dst, void* stream) {
  using namespace kk;
  if (!layout_ok(layout) || !cache_ok(src) || !quant_cache_ok(dst) || !rows_aligned(*src) || !rows_aligned(dst->c)) return KEEPKV_ERR_INVALID_ARG;
  if (dst->c.capacity < src->capacity || src->k == dst->c.k || src->v == dst->c.v) return KEEPKV_ERR_INVALID_ARG;
  if (!layout_supported(layout) || !units_supported(layout)) return KEEPKV_ERR_UNSUPPORTED;
  const int64_t tasks = (int64_t)layout->batch * layout->n_kv_heads * quant_blocks(src->capacity) * 2;
  if (tasks > kMaxTasks) return KEEPKV_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)((tasks + kTaskWaves - 1) / kTaskWaves);
  by_layout(layout, [&](auto t, auto d) {
    quantize_kernel<decltype(t), decltype(d)::value><<<grid, kTaskWaves * kWave, 0, reinterpret_cast<hipStream_t>(stream)>>>(
        src->k, src->v, (uint8_t*)dst->c.k, (uint8_t*)dst->c.v, dst->k_scale, dst->v_scale, state_of(*src), state_out(dst->c), src->capacity,
        dst->c.capacity, tasks);
  });
  return launch_status();
}

extern "C" keepkv_status keepkv_dequantize(const keepkv_layout* layout, const keepkv_quant_cache* src, keepkv_cache* dst, void* stream) {
  using namespace kk;
  if (!layout_ok(layout) || !quant_cache_ok(src) || !cache_ok(dst) || !rows_aligned(src->c) || !rows_aligned(*dst)) return KEEPKV_ERR_INVALID_ARG;
  if (dst->capacity < src->c.capacity || src->c.k == dst->k || src->c.v == dst->v) return KEEPKV_ERR_INVALID_ARG;
  if (!layout_supported(layout) || !units_supported(layout)) return KEEPKV_ERR_UNSUPPORTED;
  const int64_t tasks = (int64_t)layout->batch * layout->n_kv_heads * quant_blocks(src->c.capacity) * 2;
  if (tasks > kMaxTasks) return KEEPKV_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)((tasks + kTaskWaves - 1) / kTaskWaves);
  by_layout(layout, [&](auto t, auto d) {
    dequantize_kernel<decltype(t), decltype(d)::value><<<grid, kTaskWaves * kWave, 0, reinterpret_cast<hipStream_t>(stream)>>>(
        (const uint8_t*)src->c.k, (const uint8_t*)src->c.v, src->k_scale, src->v_scale, dst->k, dst->v, state_of(src->c), state_out(*dst),
        src->c.capacity, dst->capacity, tasks);
  });
  return launch_status();
}

extern "C" keepkv_status keepkv_append_quant(const keepkv_layout* layout, keepkv_quant_cache* cache, const void* k_t, const void* v_t,
                                             int32_t n_tokens, const int32_t* counts, int32_t* overflow, void* stream) {
  using namespace kk;
  if (!layout_ok(layout) || !quant_cache_ok(cache) || !rows_aligned(cache->c) || !k_t || !v_t || !aligned16(k_t) || !aligned16(v_t) || n_tokens < 1)
    return KEEPKV_ERR_INVALID_ARG;
  if (!layout_supported(layout) || !units_supported(layout)) return KEEPKV_ERR_UNSUPPORTED;
  const int threads = n_tokens == 1 ? 128 : 256;
  by_layout(layout, [&](auto t, auto d) {
    using T = decltype(t);
    append_quant_kernel<T, decltype(d)::value>
        <<<layout->batch * layout->n_kv_heads, threads, 0, reinterpret_cast<hipStream_t>(stream)>>>(
            (uint8_t*)cache->c.k, (uint8_t*)cache->c.v, cache->k_scale, cache->v_scale, state_out(cache->c), (const T*)k_t, (const T*)v_t, counts,
            overflow, n_tokens, cache->c.capacity);
  });
  return launch_status();
}
