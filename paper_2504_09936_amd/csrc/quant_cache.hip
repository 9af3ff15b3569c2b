// keepkv_quantize, keepkv_dequantize, keepkv_append_quant: rows into e4m3 codes with a power-of-two scale per block of 32 slots,
// and back.  All three move bytes; the arithmetic is a maximum, a multiplication and a conversion per element.
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
struct Carried {
  int votes, born, t_obs;
  float log_s;
};
__device__ __forceinline__ Carried read_state(const SlotState& s, size_t unit, int s_cap, int block, int rows, int lane) {
  Carried c = {};
  if (lane < rows && lane < kQBlock) {
    const size_t at = unit * s_cap + block * kQBlock + lane;
    c.votes = s.votes[at];
    c.log_s = s.log_s[at];
    c.born = s.born[at];
  }
  if (block == 0) c.t_obs = s.t_obs[unit];
  return c;
}
__device__ __forceinline__ void write_state(const Carried& c, const SlotStateOut& d, size_t unit, int d_cap, int block, int n_live, int n, int lane) {
  if (lane < n_live) {
    const size_t at = unit * d_cap + block * kQBlock + lane;
    d.votes[at] = c.votes;
    d.log_s[at] = c.log_s;
    d.born[at] = c.born;
  }
  if (block == 0 && lane == 0) {
    d.t_obs[unit] = c.t_obs;
    d.len[unit] = n;
  }
}

// 16 codes from 16 f32 / scale
template <int VPL, int EPV>
__device__ __forceinline__ uint4 encode16(const float (&x)[VPL][EPV], float inv) {
  uint32_t w[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    auto el = [&](int e) { return x[(4 * c + e) / EPV][(4 * c + e) % EPV] * inv; };
    w[c] = encode4(el(0), el(1), el(2), el(3));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A 16-byte vector of row elements and the codes for it (8 bytes of bf16 rows, 4 of f32): a lane's piece of every step, so that loads and
// stores are both contiguous over the wavefront, and both streamed past the caches (nontemporal: each byte is used once).  Measured with
// two vectors to a lane and 16-byte stores of codes / so, cached / so: 64 heads x 8192 slots 81.5 / 76.4 / 71.6 us, 1024 x 884 149.8 / 149.3 / 124
// (5.8 TB/s), read back 158 / 148.7 / 134 (5.4 TB/s).
template <int EPV> struct CodeWords;
template <> struct CodeWords<8> { typedef __attribute__((ext_vector_type(2))) uint32_t type; };
template <> struct CodeWords<4> { typedef uint32_t type; };

// Up to kEarlyTasks tasks a launch is as long as its chain of memory round trips, and requests ahead of it what can be: quantize_kernel what
// the slots carry, beside the rows and not before them (8 heads x 884 slots 5.5 / 5.2 us; but 128 heads 18.3 / 19.0, 64 x 8192 67.3 / 68.9),
// dequantize_kernel everything that the capacity has, beside the length, for dead slots too: full and 30 % full 8 heads 5.38 / 4.11 and 4.90 / 3.87
// us, 32 heads 7.2 / 5.6 and 5.4 / 4.7, but 64 heads 9.9 / 11.2 and 7.5 / 7.3, 128 heads 17.5 / 17.8 and 8.6 / 11.4.  (Rows to quantise,
// twice the bytes or more, ahead of the length: 5.2 / 5.35.)
constexpr int64_t kEarlyTasks = 2048;
template <typename T, int D, bool kEarly>
__global__ __launch_bounds__(kTaskWaves* kWave) void quantize_kernel(const void* k, const void* v, uint8_t* qk, uint8_t* qv, float* k_scale,
                                                                      float* v_scale, SlotState s, SlotStateOut d, int s_cap, int d_cap,
                                                                      int64_t tasks) {
  constexpr int EPV = 16 / (int)sizeof(T), VPR = D / EPV;              // elements of a vector, vectors of a row
  constexpr int STEPS = kQBlock * VPR / kWave;
  typedef typename CodeWords<EPV>::type Codes;
  const int64_t task = (int64_t)blockIdx.x * kTaskWaves + (threadIdx.x >> 6);
  if (task >= tasks) return;
  const int lane = threadIdx.x & 63;
  const int blocks = quant_blocks(s_cap);
  const bool is_v = task & 1;
  const size_t unit = (size_t)((task >> 1) / blocks);
  const int block = (int)((task >> 1) % blocks);
  const int n = s.len[unit], n_live = min(n - block * kQBlock, kQBlock);
  Carried carried = {};
  if (!is_v) carried = read_state(s, unit, s_cap, block, n_live, lane);
  if (!kEarly && !is_v) write_state(carried, d, unit, d_cap, block, n_live, n, lane);
  if (!kEarly && n_live <= 0) return;
  const uint4* src = reinterpret_cast<const uint4*>(is_v ? v : k) + (unit * s_cap + (size_t)block * kQBlock) * VPR;
  uint4 raw[STEPS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int at = i * kWave + lane;              // the at-th vector of the block
    raw[i] = at / VPR < n_live ? load_once(src + at) : make_uint4(0, 0, 0, 0);
  }
  if (kEarly && !is_v) write_state(carried, d, unit, d_cap, block, n_live, n, lane);
  if (kEarly && n_live <= 0) return;
  float x[STEPS][EPV];
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    to_f32(raw[i], x[i]);
#pragma unroll
    for (int e = 0; e < EPV; ++e) amax = max(amax, finite_magnitude(x[i][e]));
  }
  const uint32_t sb = scale_bits(wave_max(amax));
  const float inv = inverse_scale(sb);
  Codes* dst = reinterpret_cast<Codes*>((is_v ? qv : qk) + (unit * d_cap + (size_t)block * kQBlock) * D);
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int at = i * kWave + lane;
    Codes w;
    if constexpr (EPV == 8)
      w = Codes{encode4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv),
                encode4(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv)};
    else
      w = encode4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv);
    if (at / VPR < n_live) __builtin_nontemporal_store(w, dst + at);
  }
  if (lane == 0) (is_v ? v_scale : k_scale)[unit * quant_blocks(d_cap) + block] = __builtin_bit_cast(float, sb);
}

template <typename T, int D, bool kEarly>
__global__ __launch_bounds__(kTaskWaves* kWave) void dequantize_kernel(const uint8_t* qk, const uint8_t* qv, const float* k_scale,
                                                                        const float* v_scale, void* k, void* v, SlotState s, SlotStateOut d,
                                                                        int s_cap, int d_cap, int64_t tasks) {
  constexpr int EPV = 16 / (int)sizeof(T), VPR = D / EPV;
  constexpr int STEPS = kQBlock * VPR / kWave;
  typedef typename CodeWords<EPV>::type Codes;
  const int64_t task = (int64_t)blockIdx.x * kTaskWaves + (threadIdx.x >> 6);
  if (task >= tasks) return;
  const int lane = threadIdx.x & 63;
  const int blocks = quant_blocks(s_cap);
  const bool is_v = task & 1;
  const size_t unit = (size_t)((task >> 1) / blocks);
  const int block = (int)((task >> 1) % blocks);
  const float scale = (is_v ? v_scale : k_scale)[unit * blocks + block];
  const Codes* src = reinterpret_cast<const Codes*>((is_v ? qv : qk) + (unit * s_cap + (size_t)block * kQBlock) * D);
  u32x4_t* dst = reinterpret_cast<u32x4_t*>(is_v ? v : k) + (unit * d_cap + (size_t)block * kQBlock) * VPR;
  Codes w[STEPS];
  const int n = s.len[unit], n_live = min(n - block * kQBlock, kQBlock);
  const int rows = kEarly ? s_cap - block * kQBlock : n_live;
  Carried carried = {};
  if (!is_v) carried = read_state(s, unit, s_cap, block, rows, lane);
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int at = i * kWave + lane;
    w[i] = at / VPR < rows ? __builtin_nontemporal_load(src + at) : Codes{};
  }
  if (!is_v) write_state(carried, d, unit, d_cap, block, n_live, n, lane);
  if (n_live <= 0) return;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int at = i * kWave + lane;
    u32x4_t o;
    float x[4];
    if constexpr (EPV == 4) {
      decode4(w[i], x);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_bit_cast(uint32_t, x[e] * scale);
    } else {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        decode4(w[i][c], x);
        o[2 * c] = pack_bf16x2(x[0] * scale, x[1] * scale);
        o[2 * c + 1] = pack_bf16x2(x[2] * scale, x[3] * scale);
      }
    }
    if (at / VPR < n_live) __builtin_nontemporal_store(o, dst + at);
  }
}

// The new rows [from, to) of one head, slots of one block, into its K or V codes: a wavefront's work.  Everything is requested before
// the first wait: the rows and the block's scale; its codes only if the scale grows.
template <typename T, int D>
__device__ __forceinline__ void append_rows(const T* tokens, uint8_t* codes, float* scale_at, int block, int from, int to, int lane) {
  constexpr int EPV = 16 / (int)sizeof(T), VPL = 16 / EPV;
  constexpr int LPR = D / 16;                     // lanes per row: 16 codes each
  constexpr int RPI = kWave / LPR;                // rows at a time
  constexpr int STEPS = kQBlock / RPI;
  const int base = block * kQBlock, sub = lane % LPR, row0 = lane / LPR;
  const uint4* src = reinterpret_cast<const uint4*>(tokens) + sub * VPL;         // of slot `from` on
  uint4* rows = reinterpret_cast<uint4*>(codes + (size_t)base * D) + sub;
  const uint32_t old = from > base ? __builtin_bit_cast(uint32_t, *scale_at) : 0u;
  float x[STEPS][VPL][EPV];
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {               // (row r of the new ones; 32 at most)
    const int r = i * RPI + row0;
    if (i * RPI >= to - from) break;              // uniform
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      to_f32(r < to - from ? src[(size_t)r * (D / EPV) + j] : make_uint4(0, 0, 0, 0), x[i][j]);
#pragma unroll
      for (int e = 0; e < EPV; ++e) amax = max(amax, finite_magnitude(x[i][j][e]));
    }
  }
  uint32_t sb = scale_bits(wave_max(amax));
  if (from > base) {                              // the block held live slots
    sb = max(sb, old);
    if (sb != old) {
      const float ratio = __builtin_bit_cast(float, old) * inverse_scale(sb);
      for (int r = row0; r < from - base; r += RPI) {
        const uint4 c = rows[r * LPR];
        rows[r * LPR] = make_uint4(shift_codes(c.x, ratio), shift_codes(c.y, ratio), shift_codes(c.z, ratio), shift_codes(c.w, ratio));
      }
    }
  }
  const float inv = inverse_scale(sb);
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int r = i * RPI + row0;
    if (r < to - from) rows[(r + from - base) * LPR] = encode16(x[i], inv);
  }
  if (lane == 0) *scale_at = __builtin_bit_cast(float, sb);
}

struct AppendParams {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  SlotStateOut s;
  const void *k_t, *v_t;
  const int32_t* counts;
  int32_t* overflow;
  int n_tokens, capacity;
};
// live slots of a head, its score updates, how many tokens are meant for it, how many fit
struct Range {
  int n, t_obs, want, take;
};
__device__ __forceinline__ Range append_range(const AppendParams& p, size_t unit) {
  Range r;
  r.n = p.s.len[unit];
  r.t_obs = p.s.t_obs[unit];
  r.want = p.counts ? min(max(p.counts[unit], 0), p.n_tokens) : p.n_tokens;
  r.take = min(r.want, p.capacity - r.n);
  return r;
}
__device__ __forceinline__ void append_move_on(const AppendParams& p, size_t unit, const Range& r) {
  if (r.take > 0) p.s.len[unit] = r.n + r.take;
  if (r.take < r.want && p.overflow != nullptr) *p.overflow = 1;
}
// task 2 b + (0: K, 1: V): the b-th block that the tokens touch
template <typename T, int D>
__device__ __forceinline__ void append_task(const AppendParams& p, size_t unit, int task, const Range& r, int lane) {
  const bool is_v = task & 1;
  const int block = r.n / kQBlock + (task >> 1), base = block * kQBlock;
  const int from = max(r.n, base), to = min(r.n + r.take, base + kQBlock);
  if (from >= to) return;
  const T* tokens = reinterpret_cast<const T*>(is_v ? p.v_t : p.k_t) + ((unit * p.n_tokens) + (from - r.n)) * D;
  append_rows<T, D>(tokens, (is_v ? p.v : p.k) + unit * p.capacity * D, (is_v ? p.v_scale : p.k_scale) + unit * quant_blocks(p.capacity) + block,
                    block, from, to, lane);
  if (!is_v && from + lane < to) {
    const size_t at = unit * p.capacity + from + lane;
    p.s.votes[at] = 1;
    p.s.log_s[at] = -INFINITY;
    p.s.born[at] = r.t_obs;
  }
}

// One workgroup per head, a wavefront per task in turn; the length is read by all of them and moved on behind a barrier.
template <typename T, int D>
__global__ __launch_bounds__(1024) void append_head_kernel(AppendParams p) {
  const size_t unit = blockIdx.x;
  const Range r = append_range(p, unit);
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int tasks = r.take > 0 ? 2 * ((r.n + r.take - 1) / kQBlock - r.n / kQBlock + 1) : 0;
  for (int task = threadIdx.x >> 6; task < tasks; task += waves) append_task<T, D>(p, unit, task, r, lane);
  __syncthreads();
  if (threadIdx.x == 0) append_move_on(p, unit, r);
}

// Chunks of more tasks than a workgroup has wavefronts: a wavefront per task of all heads, and the lengths in a launch behind it.  One
// workgroup per head / a wavefront per task: 500 tokens for 64 heads 17.6 / 14.4 us, 8000 for 8 heads 166 / 13.0, but 100 for 64 heads
// 15.5 / 18.9, 64 for 128 heads 9.2 / 10.4.
constexpr int kHeadTasks = 16;
template <typename T, int D>
__global__ __launch_bounds__(kTaskWaves* kWave) void append_blocks_kernel(AppendParams p, int tasks) {
  const size_t unit = blockIdx.y;
  const int task = blockIdx.x * kTaskWaves + (threadIdx.x >> 6);
  const Range r = append_range(p, unit);
  if (task < tasks && r.take > 0) append_task<T, D>(p, unit, task, r, threadIdx.x & 63);
}
__global__ __launch_bounds__(256) void append_lengths_kernel(AppendParams p, int units) {
  const int unit = blockIdx.x * 256 + threadIdx.x;
  if (unit >= units) return;
  append_move_on(p, unit, append_range(p, unit));
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
    auto* kernel = tasks <= kEarlyTasks ? quantize_kernel<decltype(t), decltype(d)::value, true>
                                        : quantize_kernel<decltype(t), decltype(d)::value, false>;
    kernel<<<grid, kTaskWaves * kWave, 0, reinterpret_cast<hipStream_t>(stream)>>>(
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
    auto* kernel = tasks <= kEarlyTasks ? dequantize_kernel<decltype(t), decltype(d)::value, true>
                                        : dequantize_kernel<decltype(t), decltype(d)::value, false>;
    kernel<<<grid, kTaskWaves * kWave, 0, reinterpret_cast<hipStream_t>(stream)>>>(
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
  const int units = layout->batch * layout->n_kv_heads;
  const AppendParams p = {(uint8_t*)cache->c.k, (uint8_t*)cache->c.v, cache->k_scale, cache->v_scale, state_out(cache->c), k_t, v_t, counts, overflow,
                          n_tokens, cache->c.capacity};
  const int fit = n_tokens < cache->c.capacity ? n_tokens : cache->c.capacity;
  const int tasks = 2 * ((fit + 2 * kQBlock - 2) / kQBlock);       // of a head, at most
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  by_layout(layout, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    if (tasks <= kHeadTasks) {
      append_head_kernel<T, D><<<units, (tasks < 16 ? tasks : 16) * kWave, 0, st>>>(p);
    } else {
      append_blocks_kernel<T, D><<<dim3((tasks + kTaskWaves - 1) / kTaskWaves, units), kTaskWaves * kWave, 0, st>>>(p, tasks);
      append_lengths_kernel<<<(units + 255) / 256, 256, 0, st>>>(p, units);
    }
  });
  return launch_status();
}
