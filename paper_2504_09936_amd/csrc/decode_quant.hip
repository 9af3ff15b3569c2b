// keepkv_decode_attn_quant / keepkv_decode_step_quant: plans, arguments, entry points.  The kernel is in decode_quant.hpp.
#include <math.h>

#include "quant_launch.hpp"

namespace kk {
namespace {

constexpr int kMaxQuantWorkgroups = 512;         // that share heads: bounds the workspace
constexpr int kMinQuantSplit = 64;

// Workgroups that a compute unit holds: by LDS (K and V tiles and the query rows, once per wavefront or, the loop's, once) and registers.  (As the
// bf16 kernels are: two tiles of an f32 layout run as the loop, whose registers leave room for twelve wavefronts.)
int resident_quant(const keepkv_layout* L, long tiles_per_wave, int waves) {
  const bool f32 = L->dtype == KEEPKV_F32, loop = tiles_per_wave > 2;
  const int rows = (tiles_per_wave == 2 ? 4 : 2) * kQBlock * L->head_dim;
  const int query = (L->n_q_heads / L->n_kv_heads * L->head_dim * (f32 ? 4 : 2) + 1023) / 1024 * 1024;
  const int lds = waves * rows + (loop ? 1 : waves) * query + 1024;
  const int by_lds = 160 * 1024 / lds, by_regs = (tiles_per_wave == 1 ? 24 : f32 ? 8 : 16) / waves;
  const int n = by_lds < by_regs ? by_lds : by_regs;
  return n > 0 ? n : 1;
}

// Slots per split and workgroup size from the kind of cost model that the bf16 kernel has (choose_split in decode_attn.hip): a round of workgroups
// takes the longer of one workgroup's rows (a compute unit pulls 36 GB/s, shared by its workgroups; a wavefront 25 GB/s, 19 in the tile loop) and of
// all rows (6.2 TB/s); more rounds, smaller workgroups, a second tile, the loop and combining splits cost what stands below, in us.  The
// constants are a fit to 7042 measured (shape, plan) pairs of 375 shapes (1 to 1024 heads, 64 to 32768 slots, head dims 64 and 128, groups of 1 to
// 8), bf16, of which the plan chosen is 1.6 % slower than the best one (20 % at most); over 75 shapes of f32 it is 1.9 % (15 % at most).  Two
// things that it does not see: the next split's tiles, which a two-tile launch reads where its own has fewer (64 heads x 1180 slots: four splits of ten
// tiles on eight wavefronts), and whether splits may meet within an XCD.
void choose_split_quant(const keepkv_layout* L, int capacity, long& per, int& waves) {
  const double units = (double)L->batch * L->n_kv_heads;
  const int group = L->n_q_heads / L->n_kv_heads;
  const double slot_bytes = 2.0 * L->head_dim + 20.0;
  const long max_ns = (capacity + kMinQuantSplit - 1) / kMinQuantSplit;
  double best = 1e300;
  for (int wv = 4; wv <= 8; wv += 4) {
    for (long ns = 1; ns <= max_ns && (ns == 1 || units * (double)ns <= kMaxQuantWorkgroups); ++ns) {
      long cand = ((capacity + ns - 1) / ns + kQBlock - 1) / kQBlock * kQBlock;
      if (cand < kMinQuantSplit) cand = kMinQuantSplit;
      const double n_split = (double)((capacity + cand - 1) / cand);
      const double wgs = units * n_split;
      const long tiles = cand / kQBlock, per_wave = (tiles + wv - 1) / wv;
      const double res_max = 256.0 * resident_quant(L, per_wave, wv);
      const double streams = (per_wave <= 2 ? 25.0 : 19.0) * (double)(tiles < wv ? tiles : wv);   // GB/s
      auto round_of = [&](double n) {
        if (n <= 0.0) return 0.0;
        const double per_cu = (double)(long)((n + 255.0) / 256.0);
        const double rate = 36.0 / per_cu < streams ? 36.0 / per_cu : streams;
        const double alone = (double)cand * slot_bytes / (rate * 1e3);
        const double together = n * (units * capacity / wgs) * slot_bytes / (6.2e6 * pow(n / (256.0 * per_cu), 0.016));
        return alone > together ? alone : together;
      };
      const double full = (double)(long)(wgs / res_max), rest = wgs - full * res_max;
      const double rounds = full + (rest > 0.0 ? 1.0 : 0.0);
      const double elements = (double)((group * L->head_dim + wv * kWave - 1) / (wv * kWave));   // per thread
      // (a head of four tiles or less keeps no more wavefronts busy: 8 of them / 4 are 2 % slower on average over 117 measured shapes)
      const double small = wv == 4 && (n_split > 1.0 || tiles > 4) ? 2.0 : 0.0;
      double t = full * round_of(res_max) + round_of(rest) + 1.9 * (rounds - 1.0) + small + (per_wave > 2 ? 0.49 : per_wave == 2 ? 0.67 : 0.0);
      if (n_split > 1.0)
        t += (n_split <= 4.0 ? 2.26 : n_split <= 8.0 ? 2.95 : 3.9 + 3.0 * elements * (double)(long)((n_split - 1.0) / 16.0)) + 0.010 * n_split;
      if (t < best) {
        best = t;
        per = cand;
        waves = wv;
      }
    }
  }
}

DecodePlan make_quant_plan(const keepkv_layout* L, int capacity, int force_per, int force_waves, bool) {
  DecodePlan pl = {};
  long per = kMinQuantSplit;
  int waves = 4;
  choose_split_quant(L, capacity, per, waves);
  if (force_waves > 0) waves = force_waves;
  if (force_per >= 64) per = force_per / kQBlock * kQBlock;
  long ns = (capacity + per - 1) / per;
  if (ns > 1024) { ns = 1024; per = ((capacity + ns - 1) / ns + 63) / 64 * 64; ns = (capacity + per - 1) / per; }
  pl.nsplit = (int)ns;
  pl.per = (int)per;
  pl.waves = waves;
  pl.partial_off = kWorkspaceHead;
  pl.bytes = decode_bytes(L, ns);
  // Splits that can meet within an XCD do, with one tile or two to a wavefront: against meeting through memory, over 90 shapes of 8 to 256 heads
  // and 256 to 8192 slots, the step takes 3 % less on average and 2 % more at worst, attention alone 2 % less and 5 % more.
  const bool may_share = ns > 1 && ns <= kMaxLocalSplits && per <= (L->dtype == KEEPKV_BF16 ? 2L : 1L) * waves * kQBlock && heads_fit_xcds(L);
  pl.xcd_bytes = may_share ? decode_xcd_bytes(L, ns) : 0;
  return pl;
}
DecodePlan plan_quant(const keepkv_layout* L, int capacity, int force_per, int force_waves) {
  return kept_plan_of(L, capacity, force_per, force_waves, false, make_quant_plan);
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
  QuantParams p = {};
  p.d.q = q; p.d.k = c.k; p.d.v = c.v; p.d.votes = c.votes; p.d.log_s = c.log_s; p.d.born = c.born; p.d.t_obs = c.t_obs; p.d.len = c.len; p.d.k_t = k_t; p.d.v_t = v_t; p.d.overflow = overflow;
  p.d.out = out; p.d.logits_out = logits_out; p.d.lse_out = lse_out;
  char* const ws = reinterpret_cast<char*>(workspace);
  p.d.partial = reinterpret_cast<float*>(ws + pl.partial_off);
  p.d.ticket = reinterpret_cast<int32_t*>(ws);
  p.d.split_stride = layout->n_q_heads / layout->n_kv_heads * (layout->head_dim + 2);
  if (pl.xcd_bytes != 0 && workspace_bytes >= pl.xcd_bytes) {
    p.d.arrivals = reinterpret_cast<uint64_t*>(ws + kArrivalsOff);
    p.d.ticket_xcd = reinterpret_cast<int32_t*>(ws + kXcdTicketsOff);
    p.d.split_stride = xcd_split_stride(layout);
    p.d.partial = reinterpret_cast<float*>(align_up(reinterpret_cast<uintptr_t>(p.d.partial), kLine));
  }
  p.d.n_kv_heads = layout->n_kv_heads; p.d.capacity = c.capacity; p.d.nsplit = pl.nsplit; p.d.per = pl.per; p.d.waves = pl.waves;
  p.d.len_hint = c.len_hint > 0 ? c.len_hint : 0; p.d.scale = layout->scale;
  p.d.ln_alpha = (step && alpha > 0.f) ? logf(alpha) : -INFINITY;
  p.d.ln_1m_alpha = step ? log1pf(-alpha) : 0.f;
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  const int G = layout->n_q_heads / layout->n_kv_heads, units = layout->batch * layout->n_kv_heads;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (layout->dtype == KEEPKV_BF16)
    return layout->head_dim == 128 ? launch_quant<uint16_t, 128>(p, units, G, step, st) : launch_quant<uint16_t, 64>(p, units, G, step, st);
  return layout->head_dim == 128 ? launch_quant<float, 128>(p, units, G, step, st) : launch_quant<float, 64>(p, units, G, step, st);
}

}  // namespace

// For automatic plans of caches of up to `capacity` slots: a smaller one may be split finer.
size_t quant_workspace_bytes(const keepkv_layout* L, int capacity) {
  const long units = (long)L->batch * L->n_kv_heads;
  long ns = (capacity + kMinQuantSplit - 1) / kMinQuantSplit;
  if (ns > kMaxQuantWorkgroups / units) ns = kMaxQuantWorkgroups / units;
  if (ns <= 1) return kWorkspaceHead;
  size_t bytes = decode_bytes(L, ns);
  if (heads_fit_xcds(L) && decode_xcd_bytes(L, ns) > bytes) bytes = decode_xcd_bytes(L, ns);
  return bytes;
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
