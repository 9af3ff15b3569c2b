// keepkv_decode_attn_quant / keepkv_decode_step_quant: Eq. 6 over a cache of e4m3 codes.  One workgroup of four wavefronts per (batch, kv
// head, split); 16 lanes share a slot's row, D / 16 codes each.  The splits of a head are combined by the last of its workgroups.
#include "decode_common.hpp"
#include "quant_common.hpp"

namespace kk {
namespace {

constexpr int kQWaves = 4;
constexpr int kMaxQuantWorkgroups = 512;         // that share heads: bounds the workspace
constexpr int kMinQuantSplit = 64;

struct QuantParams {
  DecodeParams d;
  const float *k_scale, *v_scale;
};

// D / 16 consecutive codes as f32
__device__ __forceinline__ void load_codes(const uint8_t* p, float (&x)[8]) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  float a[4], b[4];
  decode4(w.x, a);
  decode4(w.y, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = a[i];
    x[4 + i] = b[i];
  }
}
__device__ __forceinline__ void load_codes(const uint8_t* p, float (&x)[4]) { decode4(*reinterpret_cast<const uint32_t*>(p), x); }

// SCORE: the EMA update of Eq. 8 with the logits just computed (the new token has joined the cache before).
template <typename T, int D, int G, bool SCORE>
__global__ __launch_bounds__(kQWaves* kWave) void decode_quant_kernel(QuantParams qp) {
  const DecodeParams& p = qp.d;
  constexpr int E = D / 16, kParts = kQWaves * 4;
  __shared__ int s_last;
  extern __shared__ __align__(16) float smem[];
  const int unit = blockIdx.y, split = blockIdx.x;
  const int sub = threadIdx.x & 15, row = threadIdx.x >> 4;
  const int len = p.len[unit], t_old = SCORE ? p.t_obs[unit] : 0;
  const int start = split * p.per, end = min(len, start + p.per);
  float q[G][E], m[G], l[G], acc[G][E];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    m[g] = kLowest;
    l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const size_t at = ((size_t)unit * G + g) * D + sub * E + e;
      q[g][e] = sizeof(T) == 2 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(p.q)[at]) : reinterpret_cast<const float*>(p.q)[at];
      acc[g][e] = 0.f;
    }
  }
  const size_t ubase = (size_t)unit * p.capacity;
  const int blocks = quant_blocks(p.capacity);
  for (int s = start + row; s < end; s += kParts) {      // (the same slot for all 16 lanes of a row)
    float k[E], v[E], z[G], sum = 0.f;
    load_codes(reinterpret_cast<const uint8_t*>(p.k) + (ubase + s) * D + sub * E, k);
    load_codes(reinterpret_cast<const uint8_t*>(p.v) + (ubase + s) * D + sub * E, v);
    const float ks = qp.k_scale[(size_t)unit * blocks + s / kQBlock], vs = qp.v_scale[(size_t)unit * blocks + s / kQBlock];
    const float lp = fast_log2((float)p.votes[ubase + s]);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float d = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) d = fmaf(q[g][e], k[e], d);
      d = group_sum<16>(d) * ks;
      sum += d;
      z[g] = fmaf(d, p.scale * kLog2e, lp);
    }
    const float x = sum * (p.scale * (1.0f / G));
    if (sub == 0) {
      if (p.logits_out != nullptr) p.logits_out[ubase + s] = x;
      if constexpr (SCORE) {
        const float a = p.ln_alpha + p.log_s[ubase + s], b = p.ln_1m_alpha + x;
        const float hi = fmaxf(a, b), lo = fminf(a, b);
        p.log_s[ubase + s] = lo == -INFINITY ? hi : hi + log1pf(expf(lo - hi));
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const float mn = fmaxf(m[g], z[g]);
      const float c = fast_exp2(m[g] - mn), pr = fast_exp2(z[g] - mn);
      m[g] = mn;
      l[g] = fmaf(l[g], c, pr);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[g][e] = fmaf(pr * vs, v[e], acc[g][e] * c);
    }
  }
  float* s_m = smem;                                     // [kParts][G]
  float* s_l = s_m + kParts * G;
  float* s_acc = s_l + kParts * G;                       // [kParts][G][D]
#pragma unroll
  for (int g = 0; g < G; ++g) {
    if (sub == 0) {
      s_m[row * G + g] = m[g];
      s_l[row * G + g] = l[g];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_acc[(row * G + g) * D + sub * E + e] = acc[g][e];
  }
  __syncthreads();
  combine_and_finish<T, D, G, kParts, SCORE, kQWaves, false, false, false>(p, s_m, s_l, s_acc, G, G * D, &s_last, unit, split, false, len, t_old,
                                                                            false);
}

DecodePlan plan_quant(const keepkv_layout* L, int capacity, int force_per, int force_waves) {
  DecodePlan pl = {};
  const long units = (long)L->batch * L->n_kv_heads;
  long ns = kMaxQuantWorkgroups / units;
  const long most = (capacity + kMinQuantSplit - 1) / kMinQuantSplit;
  ns = ns < 1 ? 1 : ns > most ? most : ns;
  long per = ((capacity + ns - 1) / ns + 63) / 64 * 64;
  if (force_per >= 64) per = force_per / kQBlock * kQBlock;
  ns = (capacity + per - 1) / per;
  if (ns > 1024) { ns = 1024; per = ((capacity + ns - 1) / ns + 63) / 64 * 64; ns = (capacity + per - 1) / per; }
  pl.nsplit = (int)ns;
  pl.per = (int)per;
  pl.waves = force_waves > 0 ? force_waves : kQWaves;
  pl.partial_off = kWorkspaceHead;
  pl.bytes = kWorkspaceHead + align_up((size_t)L->batch * L->n_q_heads * ns * (L->head_dim + 2) * sizeof(float), 256);
  return pl;
}

template <typename T, int D, int G>
keepkv_status launch_quant(const QuantParams& p, int units, bool score, hipStream_t st) {
  constexpr size_t smem = (size_t)kQWaves * 4 * G * (D + 2) * sizeof(float);
  if constexpr (smem > 60 * 1024) {
    static const bool allowed =
        hipFuncSetAttribute((const void*)decode_quant_kernel<T, D, G, true>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem) == hipSuccess &&
        hipFuncSetAttribute((const void*)decode_quant_kernel<T, D, G, false>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem) == hipSuccess;
    if (!allowed) return KEEPKV_ERR_DEVICE;
  }
  const dim3 grid(p.d.nsplit, units), block(kQWaves * kWave);
  if (score) decode_quant_kernel<T, D, G, true><<<grid, block, smem, st>>>(p);
  else decode_quant_kernel<T, D, G, false><<<grid, block, smem, st>>>(p);
  return launch_status();
}

template <typename T, int D>
keepkv_status by_group(const QuantParams& p, int units, int G, bool score, hipStream_t st) {
  switch (G) {
    case 1: return launch_quant<T, D, 1>(p, units, score, st);
    case 2: return launch_quant<T, D, 2>(p, units, score, st);
    case 4: return launch_quant<T, D, 4>(p, units, score, st);
    default: return launch_quant<T, D, 8>(p, units, score, st);
  }
}

keepkv_status run_quant(const keepkv_layout* layout, const keepkv_quant_cache* cache, const void* q, const void* k_t, const void* v_t, void* out,
                        float* logits_out, float* lse_out, float alpha, int32_t* overflow, bool step, void* workspace, size_t workspace_bytes,
                        void* stream) {
  if (!layout_ok(layout) || !quant_cache_ok(cache) || !q || !out) return KEEPKV_ERR_INVALID_ARG;
  const keepkv_cache& c = cache->c;
  if (!aligned16(q) || !aligned16(out) || !aligned16(c.k) || !aligned16(c.v)) return KEEPKV_ERR_INVALID_ARG;
  if (step && (!k_t || !v_t || !aligned16(k_t) || !aligned16(v_t) || !(alpha >= 0.f && alpha < 1.f))) return KEEPKV_ERR_INVALID_ARG;
  if (!layout_supported(layout) || !units_supported(layout)) return KEEPKV_ERR_UNSUPPORTED;
  const int fw = c.plan_wavefronts, fp = c.plan_slots_per_split;
  if (!(fw == 0 || fw == 4 || fw == 8) || fp < 0 || (fp > 0 && fp < 64)) return KEEPKV_ERR_INVALID_ARG;
  const DecodePlan pl = plan_quant(layout, c.capacity, fp, fw);
  if (pl.nsplit > 1 && (!workspace || workspace_bytes < pl.bytes || !aligned16(workspace))) return KEEPKV_ERR_WORKSPACE;
  if (step) {
    const keepkv_status rc = keepkv_append_quant(layout, const_cast<keepkv_quant_cache*>(cache), k_t, v_t, 1, nullptr, overflow, stream);
    if (rc != KEEPKV_OK) return rc;
  }
  QuantParams p = {};
  p.d.q = q; p.d.k = c.k; p.d.v = c.v; p.d.votes = c.votes; p.d.log_s = c.log_s; p.d.born = c.born; p.d.t_obs = c.t_obs; p.d.len = c.len;
  p.d.out = out; p.d.logits_out = logits_out; p.d.lse_out = lse_out;
  p.d.partial = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + pl.partial_off);
  p.d.ticket = reinterpret_cast<int32_t*>(workspace);
  p.d.split_stride = layout->n_q_heads / layout->n_kv_heads * (layout->head_dim + 2);
  p.d.n_kv_heads = layout->n_kv_heads; p.d.capacity = c.capacity; p.d.nsplit = pl.nsplit; p.d.per = pl.per; p.d.waves = pl.waves; p.d.scale = layout->scale;
  p.d.ln_alpha = (step && alpha > 0.f) ? logf(alpha) : -INFINITY;
  p.d.ln_1m_alpha = step ? log1pf(-alpha) : 0.f;
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  const int G = layout->n_q_heads / layout->n_kv_heads, units = layout->batch * layout->n_kv_heads;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (layout->dtype == KEEPKV_BF16)
    return layout->head_dim == 128 ? by_group<uint16_t, 128>(p, units, G, step, st) : by_group<uint16_t, 64>(p, units, G, step, st);
  return layout->head_dim == 128 ? by_group<float, 128>(p, units, G, step, st) : by_group<float, 64>(p, units, G, step, st);
}

}  // namespace

// For automatic plans of caches of up to `capacity` slots: a smaller one may be split finer.
size_t quant_workspace_bytes(const keepkv_layout* L, int capacity) {
  const long units = (long)L->batch * L->n_kv_heads;
  long ns = (capacity + kMinQuantSplit - 1) / kMinQuantSplit;
  if (ns > kMaxQuantWorkgroups / units) ns = kMaxQuantWorkgroups / units;
  if (ns <= 1) return kWorkspaceHead;
  return kWorkspaceHead + align_up((size_t)L->batch * L->n_q_heads * ns * (L->head_dim + 2) * sizeof(float), 256);
}

}  // namespace kk

extern "C" keepkv_status keepkv_decode_attn_quant(const keepkv_layout* layout, const keepkv_quant_cache* cache, const void* q, void* out,
                                                  float* logits_out, float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
  return kk::run_quant(layout, cache, q, nullptr, nullptr, out, logits_out, lse_out, 0.f, nullptr, false, workspace, workspace_bytes, stream);
}

extern "C" keepkv_status keepkv_decode_step_quant(const keepkv_layout* layout, keepkv_quant_cache* cache, const void* q, const void* k_t,
                                                  const void* v_t, void* out, float* logits_out, float alpha, int32_t* overflow, void* workspace,
                                                  size_t workspace_bytes, void* stream) {
  return kk::run_quant(layout, cache, q, k_t, v_t, out, logits_out, nullptr, alpha, overflow, true, workspace, workspace_bytes, stream);
}

extern "C" keepkv_status keepkv_decode_plan_quant(const keepkv_layout* layout, int32_t capacity, int32_t* n_split, int32_t* slots_per_split,
                                                  int32_t* wavefronts) {
  using namespace kk;
  if (!layout_ok(layout) || capacity < 1 || capacity > (1 << 20)) return KEEPKV_ERR_INVALID_ARG;
  if (!layout_supported(layout) || !units_supported(layout)) return KEEPKV_ERR_UNSUPPORTED;
  const DecodePlan pl = plan_quant(layout, capacity, 0, 0);
  if (n_split) *n_split = pl.nsplit;
  if (slots_per_split) *slots_per_split = pl.per;
  if (wavefronts) *wavefronts = pl.waves;
  return KEEPKV_OK;
}
