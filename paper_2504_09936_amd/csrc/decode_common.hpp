// What the decode kernels share: their parameters, cross-lane moves, and the end of a workgroup's work -- its wavefronts' softmax
// states reduced, a head's splits combined by the last of its workgroups, through memory or within an XCD.
// Each source that includes this has its own instances.
#pragma once

#include <math.h>
#include <string.h>

#include <type_traits>
#include <utility>

#include "kk_common.hpp"

namespace kk {

// Phase timestamps for kernel tuning; compiled in only with -DKEEPKV_TRACE (never in the product build).
#ifdef KEEPKV_TRACE
static __device__ long long kk_trace[8 * 8192];
#define KK_TS(i) do { const int b_ = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x; if (threadIdx.x == 0 && b_ < 8192) \
  kk_trace[b_ * 8 + (i)] = wall_clock64(); } while (0)
#else
#define KK_TS(i) do { } while (0)
#endif

struct DecodeParams {
  const void* q;
  void* k;            // written only in step mode (the appended row)
  void* v;
  int32_t* votes;
  float* log_s;       // step mode / score fusion
  int32_t* born;      // step mode: the new slot's origin (a slot's observation count is t_obs - born)
  int32_t* t_obs;     // step mode: [B * Hkv] steps observed by the head, += 1 per step
  int32_t* len;
  const void* k_t;    // step mode: [B, Hkv, D] new token, else null
  const void* v_t;
  int32_t* overflow;
  void* out;
  float* logits_out;
  float* lse_out;
  float* partial;     // [B*Hkv, nsplit, split_stride]
  int32_t* ticket;    // [B*Hkv] zero between launches
  uint64_t* arrivals; // [B*Hkv] zero between launches: where the head's workgroups run (null: not recorded, any XCD)
  int32_t* ticket_xcd;   // [B*Hkv] zero between launches, like `ticket` but counted in the L2 of the head's XCD
  int split_stride;   // floats between the partial results of two splits
  int n_kv_heads;
  int capacity;
  int nsplit;
  int per;          // slots per split
  int len_hint;     // caller's upper bound on len (0: none)
  int waves;        // wavefronts per workgroup of the matrix-core kernel (4 or 8)
  float scale;
  float ln_alpha, ln_1m_alpha;
};

namespace {

// Control words of heads whose workgroups may share an XCD: at most kMaxXcdUnits heads, behind their tickets.
constexpr int kMaxXcdUnits = 2048;
constexpr size_t kXcdTicketsOff = 16 * 1024, kArrivalsOff = 32 * 1024;
static_assert(kMaxXcdUnits * sizeof(int32_t) <= kXcdTicketsOff && kXcdTicketsOff + kMaxXcdUnits * sizeof(int32_t) <= kArrivalsOff &&
              kArrivalsOff + kMaxXcdUnits * sizeof(uint64_t) <= kMatchCountersOff, "control words");
constexpr size_t kLine = 128;       // bytes of a cache line
inline int xcd_split_stride(const keepkv_layout* L) {           // floats of a split's partial result, whole lines
  return (int)align_up((size_t)L->n_q_heads / L->n_kv_heads * (L->head_dim + 2), kLine / sizeof(float));
}

// Asynchronous copy of 16 bytes per lane from base + lane_off + off (`bytes` long from base: beyond it reads give zero) to
// LDS, through a buffer descriptor: the compiler counts these in the order of issue, while behind a global_load_lds it
// waits for everything before it uses any register load.
template <int AUX>
__device__ __forceinline__ void copy_to_lds(const unsigned char* base, size_t bytes, unsigned char* lds, uint32_t lane_off,
                                            uint32_t off) {
#ifdef __HIP_DEVICE_COMPILE__                    // (the descriptor's type does not exist in the host pass)
  __builtin_amdgcn_raw_ptr_buffer_load_lds(
      __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, (int)bytes, 0x00027000),
      (__attribute__((address_space(3))) void*)lds, 16, lane_off, off, 0, AUX);
#endif
}

constexpr float kLowest = -3.402823466e38f;   // lower end of the running maxima: finite, so that maxima can be subtracted

__device__ __forceinline__ void st_agent(float* p, float v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float ld_agent(const float* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// loads of what another workgroup of this XCD wrote (see all_on_this_xcd): L1 holds none of these lines, so L2 serves them
__device__ __forceinline__ float ld_xcd(const float* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
__device__ __forceinline__ void ld_xcd2(const float* p, float& a, float& b) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  a = __builtin_bit_cast(float, (uint32_t)v);
  b = __builtin_bit_cast(float, (uint32_t)(v >> 32));
}

// Two floats that live side by side, as one device-scope access.
__device__ __forceinline__ void st_agent2(float* p, float a, float b) {
  const uint64_t v = (uint64_t)__builtin_bit_cast(uint32_t, a) | (uint64_t)__builtin_bit_cast(uint32_t, b) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void ld_agent2(const float* p, float& a, float& b) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  a = __builtin_bit_cast(float, (uint32_t)v);
  b = __builtin_bit_cast(float, (uint32_t)(v >> 32));
}

// a <- {a of the lower half, b of the lower half}, b <- {a of the upper half, b of the upper half} (lanes 0 .. 31 / 32 .. 63)
__device__ __forceinline__ void swap_halves(float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
  const uint32_t ra = r[0], rb = r[1];           // (a bit cast of a vector element itself reads element 0)
  a = __builtin_bit_cast(float, ra);
  b = __builtin_bit_cast(float, rb);
}
// the same for the rows of 16 lanes of each half: a <- {a row 0, b row 0, a row 2, b row 2}, b <- {a row 1, b row 1, a 3, b 3}
__device__ __forceinline__ void swap_rows(float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
  const uint32_t ra = r[0], rb = r[1];           // (a bit cast of a vector element itself reads element 0)
  a = __builtin_bit_cast(float, ra);
  b = __builtin_bit_cast(float, rb);
}
// maximum / sum over the lanes that hold the same head: equal l16 mod G in all four rows of 16 lanes
template <int G, typename F>
__device__ __forceinline__ float over_head_lanes(float x, F op) {
  if constexpr (G <= 1) x = op(x, dpp_f32<0x121>(x));   // row_ror:1
  if constexpr (G <= 2) x = op(x, dpp_f32<0x122>(x));   // row_ror:2
  if constexpr (G <= 4) x = op(x, dpp_f32<0x124>(x));   // row_ror:4
  x = op(x, dpp_f32<0x128>(x));                         // row_ror:8
  float y = x;
  swap_rows(x, y);
  x = y = op(x, y);
  swap_halves(x, y);
  return op(x, y);
}

// over the 16 lanes of a row
template <typename F>
__device__ __forceinline__ float row_reduce(float x, F op) {
  x = op(x, dpp_f32<0xB1>(x));                          // quad_perm [1,0,3,2]
  x = op(x, dpp_f32<0x4E>(x));                          // quad_perm [2,3,0,1]
  x = op(x, dpp_f32<0x141>(x));                         // row_half_mirror
  return op(x, dpp_f32<0x140>(x));                      // row_mirror
}

// ---- heads whose workgroups all run on one XCD ----------------------------------------------------------------
// Partial results and a ticket that travel at device scope go to memory and back three times (store, ticket, load), about
// 2.5 us of a 10 us step; through the L2 that the workgroups of one XCD share it is a third of that.  Workgroups are dealt to the
// eight XCDs in turn, so the grid puts the splits of a head eight workgroup ids apart; but that order is a habit of
// the hardware and nothing documented, so a workgroup only relies on what it can read: its own XCD's number.  It adds it to the head's
// `arrivals` when it starts (byte x: workgroups on XCD x; device scope, nothing waits for it) and looks at the word before it publishes its
// result, some microseconds later.  If by then all splits have arrived, all on its own XCD, it publishes within that XCD; every
// other workgroup of the head sees the same word and does the same, because a workgroup that finds the word incomplete
// marks it (kArriveMark, compare-and-swap on the incomplete word), and a marked word stays marked, so that those who look later
// use device scope too.
// What it gives stands at xcd_pays.  Arriving behind the copies of the query rows (whose address translation it then waits for) made short
// last splits look in vain: 8 heads x 1180 slots in six 8.0 us, 7.1 so, 7.4 through memory.
constexpr uint64_t kArriveMark = 1ull << 63;
constexpr int kMaxLocalSplits = 16;             // (at most 127: a byte of `arrivals`, less the mark)
__device__ __forceinline__ int xcd_id() { return __builtin_amdgcn_s_getreg(20 | (3 << 11)); }   // XCC_ID[3:0]
__device__ __forceinline__ uint64_t ld_arrivals(const DecodeParams& p, int unit) {
  return __hip_atomic_load(&p.arrivals[unit], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// v: the word as last read.  One thread per workgroup.  A workgroup with a short split may be done before the others of its head have
// arrived; it looks a few times more before it gives up.
constexpr int kLooks = 6;
__device__ __forceinline__ bool all_on_this_xcd(const DecodeParams& p, int unit, uint64_t v) {
  const uint64_t here = (uint64_t)p.nsplit << (8 * xcd_id());
  int looks = 0;
  while (v != here && !(v & kArriveMark)) {
    int sum = 0;
    for (int x = 0; x < 64; x += 8) sum += (int)(v >> x) & 255;
    if (sum >= p.nsplit) break;                  // complete, on several XCDs
    if (looks++ < kLooks) {
      v = ld_arrivals(p, unit);
      continue;
    }
    // still incomplete: mark it (at most nsplit attempts fail, one for each arrival)
    if (__hip_atomic_compare_exchange_strong(&p.arrivals[unit], &v, v | kArriveMark, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT))
      break;
  }
  return v == here;
}

template <int G>
__device__ __forceinline__ float head_sum(float x) {   // sum over the G heads held by G consecutive lanes
  if constexpr (G >= 2) x += dpp_f32<0xB1>(x);          // quad_perm [1,0,3,2]
  if constexpr (G >= 4) x += dpp_f32<0x4E>(x);          // quad_perm [2,3,0,1]
  if constexpr (G >= 8) x += dpp_f32<0x141>(x);         // row_half_mirror
  return x;
}

__device__ __forceinline__ uint32_t pack_hi16(float lo_elem, float hi_elem) {   // {bf16 trunc(lo_elem), bf16 trunc(hi_elem)}
  return (__builtin_bit_cast(uint32_t, lo_elem) >> 16) | (__builtin_bit_cast(uint32_t, hi_elem) & 0xFFFF0000u);
}

// ---- the two products of a 32-slot tile on 16x16x32 MFMA (bf16 operands, f32 sums) -----------------------------------------
// Scores come transposed, S^T = K Q^T: column c of lane (c, q) is head c mod G, and its 8 values are the slots
// 16 st + 4 q + i, i = 0 .. 3, in s[st][i].  The 16 / G lanes of a head share them: lane share r = c / G takes NV of the 8, from place
// pos0 on.  (NV = 1 for G <= 2: eight shares; of G = 1 the other eight have none.)
template <int G>
constexpr int kShare = G >= 2 ? G / 2 : 1;

template <int G>
__device__ __forceinline__ void take_shares(const f32x4_t (&s)[2], int r_l, int pos0, float (&sv)[kShare<G>]) {
  constexpr int NV = kShare<G>;
  if constexpr (NV == 4) {
#pragma unroll
    for (int v = 0; v < 4; ++v) sv[v] = (r_l & 1) ? s[1][v] : s[0][v];
  } else if constexpr (NV == 2) {
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const float t0 = (r_l & 1) ? s[0][2 + v] : s[0][v], t1 = (r_l & 1) ? s[1][2 + v] : s[1][v];
      sv[v] = (r_l & 2) ? t1 : t0;
    }
  } else {
    float t[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] = (pos0 & 1) ? s[j >> 1][2 * (j & 1) + 1] : s[j >> 1][2 * (j & 1)];
    const float u0 = (pos0 & 2) ? t[1] : t[0], u1 = (pos0 & 2) ? t[3] : t[2];
    sv[0] = (pos0 & 4) ? u1 : u0;
  }
}

// The weights of a lane share as the A operand of O = P V, hi + lo in bf16 (16 significant bits).  Each term is cut off (together within
// 2^-15 of the weight) or, kNearest, rounded (2^-18).  The places of the slots that other lanes took hold zero where V is made of codes
// (kNearest).  Where V is made of bf16 rows they hold the smallest normal number: an infinite value then stays infinite where the weight has both
// terms, and zero would always make it NaN; finite values add up to (16 / G - 1) 2^-125 sum |v| to an output (8 for G = 8 and
// one value near the largest f32).
template <int G, bool kNearest>
__device__ __forceinline__ void weights_operand(const float (&pr)[kShare<G>], int r_l, int pos0, uint32_t (&ah)[4], uint32_t (&al)[4]) {
  constexpr int NV = kShare<G>;
  constexpr uint32_t kNone = kNearest ? 0u : 0x00800080u;
  if constexpr (NV == 1) {
    const uint32_t hb = kNearest ? f32_to_bf16_bits(pr[0]) << 16 : __builtin_bit_cast(uint32_t, pr[0]) & 0xFFFF0000u;
    const float rest = pr[0] - __builtin_bit_cast(float, hb);
    const uint32_t lb = kNearest ? f32_to_bf16_bits(rest) << 16 : __builtin_bit_cast(uint32_t, rest) & 0xFFFF0000u;
    const uint32_t wh = (pos0 & 1) ? hb | (kNone & 0xFFFFu) : hb >> 16 | (kNone & 0xFFFF0000u);
    const uint32_t wl = (pos0 & 1) ? lb | (kNone & 0xFFFFu) : lb >> 16 | (kNone & 0xFFFF0000u);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      ah[d] = (pos0 >> 1) == d && (G > 1 || r_l < 8) ? wh : kNone;
      al[d] = (pos0 >> 1) == d && (G > 1 || r_l < 8) ? wl : kNone;
    }
  } else {
    constexpr int NW = NV / 2;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      const float p0 = pr[2 * j], p1 = pr[2 * j + 1];
      const uint32_t wh = kNearest ? pack_bf16x2(p0, p1) : pack_hi16(p0, p1);
      const float l0 = p0 - bf16_lo(wh), l1 = p1 - bf16_hi(wh);
      const uint32_t wl = kNearest ? pack_bf16x2(l0, l1) : pack_hi16(l0, l1);
#pragma unroll
      for (int d = j; d < 4; d += NW) {          // dword d holds the places 2 d, 2 d + 1
        ah[d] = r_l == d / NW ? wh : kNone;
        al[d] = r_l == d / NW ? wl : kNone;
      }
    }
  }
}

// The accumulators (row r of a channel tile = head r mod G) times c, which lane (l16, q) holds for head l16 mod G.
template <int G, int NTILE>
__device__ __forceinline__ void rescale_rows(f32x4_t (&O)[NTILE], float c, int l16, int q) {
  const float c_other = dpp_f32<0x124>(c);       // G = 8: of the head four further (every lane reads: not inside the choice)
  const float cq = G < 8 || ((l16 >> 2) & 1) == (q & 1) ? c : c_other;
  const float ci[4] = {dpp_f32<0x00>(cq), dpp_f32<G == 1 ? 0x00 : 0x55>(cq), dpp_f32<G <= 2 ? 0x00 : 0xAA>(cq),
                       dpp_f32<G == 1 ? 0x00 : G == 2 ? 0x55 : 0xFF>(cq)};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int nt = 0; nt < NTILE; ++nt) O[nt][i] *= ci[i];
}

// A wavefront's state into LDS: acc [D][G], ml ([G] maxima, [G] sums).  Rows of the second product: row 4 q + i is head (4 q + i) mod G,
// lane share (4 q + i) / G.  The shares are added in the lane (G <= 2), then over the lane halves and (G <= 4) the rows of 16 lanes; each
// exchange pairs two channel tiles, so the lanes end up with different channel tiles and the LDS stores are wide.
template <int D, int G>
__device__ __forceinline__ void deposit_state(const f32x4_t (&O)[D / 16], float m_run, float l_tot, float* acc_mine, float* ml_mine, int lane) {
  constexpr int NTILE = D / 16;
  const int l16 = lane & 15, q = lane >> 4;
  constexpr int NH = G < 4 ? G : 4;              // heads per lane
  float o[NTILE][NH];
#pragma unroll
  for (int nt = 0; nt < NTILE; ++nt)
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      if constexpr (G == 1) o[nt][h] = (O[nt][0] + O[nt][1]) + (O[nt][2] + O[nt][3]);
      else if constexpr (G == 2) o[nt][h] = O[nt][h] + O[nt][h + 2];
      else o[nt][h] = O[nt][h];
    }
#pragma unroll
  for (int nt = 0; nt < NTILE / 2; ++nt)
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      swap_halves(o[nt][h], o[nt + NTILE / 2][h]);
      o[nt][h] += o[nt + NTILE / 2][h];
    }
  constexpr int NO = G <= 4 ? NTILE / 4 : NTILE / 2;   // channel tiles per lane
  if constexpr (G <= 4) {
#pragma unroll
    for (int nt = 0; nt < NO; ++nt)
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        swap_rows(o[nt][h], o[nt + NO][h]);
        o[nt][h] += o[nt + NO][h];
      }
  }
  const int nt0 = (NTILE / 2) * (q >> 1) + (G <= 4 ? NO * (q & 1) : 0);
  const int h0 = G == 8 ? 4 * (q & 1) : 0;
#pragma unroll
  for (int nt = 0; nt < NO; ++nt) {
    float* at = acc_mine + (16 * (nt0 + nt) + l16) * G + h0;
    if constexpr (NH == 4) *reinterpret_cast<float4*>(at) = make_float4(o[nt][0], o[nt][1], o[nt][2], o[nt][3]);
    else if constexpr (NH == 2) *reinterpret_cast<float2*>(at) = make_float2(o[nt][0], o[nt][1]);
    else *at = o[nt][0];
  }
  if (q == 0 && l16 < G) {
    ml_mine[l16] = m_run;
    ml_mine[G + l16] = l_tot;
  }
}

// Everything after the workgroup's kParts partial softmax states (m, l, acc[D] per head) have been
// deposited in LDS and a barrier has passed: reduce them; a single split finishes the head, otherwise the
// partial result goes to the workspace and the last workgroup of the head to arrive combines the splits,
// resets the ticket and (step mode) publishes the new len.
// acc of a part: [D][G] (kInner) or [G][D]; parts are acc_stride / ml_stride floats apart.  A split's partial result in
// the workspace: acc in the same order, then (m, l) per head.
// one_xcd (uniform): every workgroup of the head runs on this XCD and knows it (see all_on_this_xcd).
// An empty part or split has l = 0 and any m; maxima are held at or above the lowest finite value, so that they can be
// subtracted without a test for -inf.
template <typename T, int D, int G, int kParts, bool STEP, int WAVES, bool kInner, bool kSolo, bool kMayShareXcd>
__device__ __forceinline__ void combine_and_finish(const DecodeParams& p, const float* s_m, const float* s_l,
                                                   const float* s_acc, int ml_stride, int acc_stride, int* s_last_p,
                                                   int unit, int split, bool grow, int len, int t_old, bool one_xcd_) {
  const bool one_xcd = kMayShareXcd && one_xcd_;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kThreads = WAVES * kWave;
  int& s_last = *s_last_p;
  auto head_of = [](int idx) { return kInner ? idx % G : idx / D; };
  auto finish = [&](int idx, float M, float L, float A) {
    const int g = head_of(idx), d = kInner ? idx / G : idx % D;
    const size_t row = (size_t)unit * G + g;   // == b * Hq + h * G + g
    const float o = L == 0.f ? 0.f : A / L;      // (no slot, or none of any weight: zero; a sum that is NaN shows as one)
    if constexpr (kBf16)
      reinterpret_cast<uint16_t*>(p.out)[row * D + d] = (uint16_t)f32_to_bf16_bits(o);
    else
      reinterpret_cast<float*>(p.out)[row * D + d] = o;
    if (d == 0 && p.lse_out != nullptr) p.lse_out[row] = L == 0.f ? -INFINITY : (M + fast_log2(L)) * kLn2;
  };

  float* const partials = p.partial + (size_t)unit * p.nsplit * p.split_stride;   // this head's splits
  // kInner: a lane's head is lane mod G for all of its elements, and what the splits weigh in that head is the same for
  // every channel, so lane i works out the weight of split i / G and the lanes of a head hand them around through a table of the wavefront's
  // own in LDS: one exponential per lane instead of one per split and element.  weigh(): n splits; m, l: those of split
  // lane / G (-inf and 0 beyond nsplit); leaves the head's M, its L (added up in the order of the splits) and the n weights.
  // (Not for the parts of a workgroup, whose maxima LDS holds at hand: the maximum over lanes, the exponential and the table
  // are one chain of latencies there, and an unsplit step of 100 to 300 slots took 0.1 us longer with them.)
  const int lane = threadIdx.x & 63;
  float* const s_c = const_cast<float*>(s_acc) + (threadIdx.x >> 6) * acc_stride + G * D + 16;   // 2 x [G][n], behind this wavefront's deposit
  auto weigh = [&](float m, float l, auto n_tag, float& M, float& L, float (&c)[decltype(n_tag)::value]) {
    constexpr int n = decltype(n_tag)::value;
    static_assert(n % 4 == 0 && n * G <= kWave, "one weight per lane");
    M = over_head_lanes<G>(m, [](float a, float b) { return fmaxf(a, b); });
    const float mine = lane < n * G ? fast_exp2(m - M) : 0.f;
    if (lane < n * G) {
      s_c[(lane % G) * n + lane / G] = mine;
      s_c[n * G + (lane % G) * n + lane / G] = l;
    }
    L = 0.f;
#pragma unroll
    for (int i = 0; i < n; i += 4) {
      const float4 t = *reinterpret_cast<const float4*>(s_c + (lane % G) * n + i);
      const float4 u = *reinterpret_cast<const float4*>(s_c + n * G + (lane % G) * n + i);
      c[i] = t.x; c[i + 1] = t.y; c[i + 2] = t.z; c[i + 3] = t.w;
      L = fmaf(u.w, t.w, fmaf(u.z, t.z, fmaf(u.y, t.y, fmaf(u.x, t.x, L))));
    }
  };
  for (int idx = threadIdx.x; idx < G * D; idx += kThreads) {
    const int g = head_of(idx);
    float M = kLowest, L = 0.f, A = 0.f;
    if constexpr (kInner) {
#pragma unroll
      for (int w = 0; w < kParts; ++w) M = fmaxf(M, s_m[w * ml_stride + g]);
#pragma unroll
      for (int w = 0; w < kParts; ++w) {
        const float c = fast_exp2(s_m[w * ml_stride + g] - M);
        L = fmaf(s_l[w * ml_stride + g], c, L);
        A = fmaf(s_acc[w * acc_stride + idx], c, A);
      }
    } else {                                     // a wavefront's elements are of one head: lane i of a row weighs part i
      // (sixteen exponentials per element before: 32 steps of 4 heads x 52 .. 84 slots and their event 145.4 us, now 143.3)
      static_assert(kInner || (kParts == 16 && D % kWave == 0), "one weight a lane");
      const int gw = __builtin_amdgcn_readfirstlane(g);
      const float m = s_m[(lane & 15) * ml_stride + gw];
      M = fmaxf(M, row_reduce(m, [](float a, float b) { return fmaxf(a, b); }));
      const float c = fast_exp2(m - M);
      L = row_reduce(s_l[(lane & 15) * ml_stride + gw] * c, [](float a, float b) { return a + b; });
#pragma unroll
      for (int w = 0; w < kParts; ++w)
        A = fmaf(s_acc[w * acc_stride + idx], __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, c), w)), A);
    }
    if (kSolo || p.nsplit == 1) {
      finish(idx, M, L, A);
    } else {
      float* dst = partials + (size_t)split * p.split_stride;
      const bool has_ml = (kInner ? idx / G : idx % D) == 0;
      if (one_xcd) {
        dst[idx] = A;
        if (has_ml) *reinterpret_cast<float2*>(dst + G * D + 2 * g) = make_float2(M, L);
      } else {                                   // device-coherent (write-through): the combining workgroup may run on another XCD
        st_agent(dst + idx, A);
        if (has_ml) st_agent2(dst + G * D + 2 * g, M, L);
      }
    }
  }

  if (kSolo || p.nsplit == 1) {
    if (STEP && threadIdx.x == 0) p.t_obs[unit] = t_old + 1;   // one more observation of every slot of the head
    if (STEP && threadIdx.x == 0 && grow) p.len[unit] = len;   // every wavefront read len before the barrier above
    if (STEP && threadIdx.x == 0 && !grow && p.overflow != nullptr) *p.overflow = 1;
    return;
  }

  KK_TS(3);
  // ---- the last workgroup of this head to arrive combines the splits ------------------------------
  // The partial results were stored write-through at device scope (or, one_xcd, into the L2 that all of the head's
  // workgroups share, where the ticket is counted too), so it is enough that every
  // wavefront's stores have completed before the ticket is taken: each wavefront waits on its own
  // memory counter (stores count there on this part), then the barrier orders all of them before
  // thread 0's ticket.  A workgroup-scope release fence emits no such wait here (the workgroup shares
  // one L2, so the compiler needs none for that scope), and a device-scope release fence would write
  // back the whole L2 per workgroup.  The combining workgroup reads the partials with device-scope loads; one_xcd: with loads
  // that find nothing in its L1, because a split's result has cache lines of its own (split_stride) that nobody reads but the
  // combining workgroup, once a launch.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const int before = one_xcd ? __hip_atomic_fetch_add(&p.ticket_xcd[unit], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)
                               : __hip_atomic_fetch_add(&p.ticket[unit], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = before == p.nsplit - 1;
  }
  __syncthreads();
  KK_TS(4);
  if (!s_last) return;
  // CH splits of EB output elements are fetched per round trip of device-scope loads: 4 or 8 splits of two
  // elements when that covers all splits (the common case; surplus loads would only cost), else 16 of one
  constexpr int kPerThread = (G * D + kThreads - 1) / kThreads;   // output elements per thread
  auto combine = [&](auto ch_tag, auto eb_tag, auto xcd_tag) {
    constexpr int CH = decltype(ch_tag)::value, EB = decltype(eb_tag)::value;
    constexpr bool kXcd = decltype(xcd_tag)::value;
    for (int e0 = 0; e0 < kPerThread; e0 += EB) {
      int idx[EB];
      float M[EB], L[EB], A[EB];
#pragma unroll
      for (int j = 0; j < EB; ++j) {
        idx[j] = min((int)threadIdx.x + (e0 + j) * kThreads, G * D - 1);   // surplus threads repeat the last element
        M[j] = kLowest;
        L[j] = 0.f;
        A[j] = 0.f;
      }
      for (int s0 = 0; s0 < p.nsplit; s0 += CH) {
        float ms[EB][CH], ls[EB][CH], as[EB][CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          const float* src = partials + (size_t)min(s0 + i, p.nsplit - 1) * p.split_stride;
#pragma unroll
          for (int j = 0; j < EB; ++j) {
            const float* ml = src + G * D + 2 * head_of(idx[j]);
            if constexpr (kXcd) {
              ld_xcd2(ml, ms[j][i], ls[j][i]);
              as[j][i] = ld_xcd(src + idx[j]);
            } else {
              ld_agent2(ml, ms[j][i], ls[j][i]);
              as[j][i] = ld_agent(src + idx[j]);
            }
          }
        }
#pragma unroll
        for (int j = 0; j < EB; ++j) {
          float mc = M[j];
#pragma unroll
          for (int i = 0; i < CH; ++i) mc = fmaxf(mc, ms[j][i]);
          const float c0 = fast_exp2(M[j] - mc);
          L[j] *= c0;
          A[j] *= c0;
#pragma unroll
          for (int i = 0; i < CH; ++i) {
            const float c = s0 + i < p.nsplit ? fast_exp2(ms[j][i] - mc) : 0.f;
            L[j] = fmaf(ls[j][i], c, L[j]);
            A[j] = fmaf(as[j][i], c, A[j]);
          }
          M[j] = mc;
        }
      }
#pragma unroll
      for (int j = 0; j < EB; ++j)
        if ((int)threadIdx.x + (e0 + j) * kThreads < G * D) finish(idx[j], M[j], L[j], A[j]);
    }
  };
  // kInner and no more than CH splits: the weights once per lane (see weigh), CH values of every element per round trip
  auto combine_few = [&](auto ch_tag, auto xcd_tag) {
    constexpr int CH = decltype(ch_tag)::value;
    constexpr bool kXcd = decltype(xcd_tag)::value;
    const int mine = lane / G;
    const float* ml = partials + (size_t)min(mine, p.nsplit - 1) * p.split_stride + G * D + 2 * (lane % G);
    float m, l, as[kPerThread][CH];
    if constexpr (kXcd) ld_xcd2(ml, m, l);
    else ld_agent2(ml, m, l);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const float* src = partials + (size_t)min(i, p.nsplit - 1) * p.split_stride;
#pragma unroll
      for (int j = 0; j < kPerThread; ++j) {
        const int idx = min((int)threadIdx.x + j * kThreads, G * D - 1);   // surplus threads repeat the last element
        as[j][i] = kXcd ? ld_xcd(src + idx) : ld_agent(src + idx);
      }
    }
    float M, L, c[CH];
    weigh(mine < p.nsplit ? m : -INFINITY, mine < p.nsplit ? l : 0.f, ch_tag, M, L, c);
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
      float A = 0.f;
#pragma unroll
      for (int i = 0; i < CH; ++i) A = fmaf(as[j][i], c[i], A);
      const int idx = (int)threadIdx.x + j * kThreads;
      if (idx < G * D) finish(idx, M, L, A);
    }
  };
  constexpr int kTwo = kPerThread >= 2 ? 2 : 1;
  auto combine_all = [&](auto xcd_tag) {
    if constexpr (kInner) {
      if (p.nsplit <= 4) return combine_few(std::integral_constant<int, 4>{}, xcd_tag);
      if (p.nsplit <= 8) return combine_few(std::integral_constant<int, 8>{}, xcd_tag);
      if constexpr (G <= 4)
        if (p.nsplit <= 16) return combine_few(std::integral_constant<int, 16>{}, xcd_tag);
    }
    if (p.nsplit <= 4) combine(std::integral_constant<int, 4>{}, std::integral_constant<int, kTwo>{}, xcd_tag);
    else if (p.nsplit <= 8) combine(std::integral_constant<int, 8>{}, std::integral_constant<int, kTwo>{}, xcd_tag);
    else combine(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}, xcd_tag);
  };
  bool combined = false;
  if constexpr (kMayShareXcd) {
    if (one_xcd) combine_all(std::true_type{});
    combined = one_xcd;
  }
  if (!combined) combine_all(std::false_type{});
  KK_TS(5);
  if (threadIdx.x == 0) {                        // the control words are ready for the next launch
    if (one_xcd) __hip_atomic_store(&p.ticket_xcd[unit], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    else __hip_atomic_store(&p.ticket[unit], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // (every workgroup of the head looked at this word before it took its ticket)
    if (kMayShareXcd) __hip_atomic_store(&p.arrivals[unit], 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (STEP) p.t_obs[unit] = t_old + 1;             // (every workgroup of the head read it before taking its ticket)
    if (STEP && grow) p.len[unit] = len;
    if (STEP && !grow && p.overflow != nullptr) *p.overflow = 1;
  }
}

// ---- plans (host) ----------------------------------------------------------------------------------------------
inline size_t decode_bytes(const keepkv_layout* L, long nsplit) {
  return kWorkspaceHead + (size_t)L->batch * L->n_q_heads * nsplit * (L->head_dim + 2) * sizeof(float);
}

// Partial results with cache lines of their own, for heads that are combined within an XCD.
inline size_t decode_xcd_bytes(const keepkv_layout* L, long nsplit) {
  return kWorkspaceHead + kLine + align_up((size_t)L->batch * L->n_kv_heads * nsplit * xcd_split_stride(L) * sizeof(float), 256);
}

// The heads have to divide evenly among the XCDs, or some would idle; with 4 heads, say, half of them.
inline bool heads_fit_xcds(const keepkv_layout* L) {
  const long units = (long)L->batch * L->n_kv_heads;
  return units % 8 == 0 && units <= kMaxXcdUnits;
}

// The cost model walks up to 1024 candidate plans, microseconds of host time, and a program asks for the same
// few plans again and again (one per layer shape and step): each thread keeps its last ones.  A plan is a pure function
// of the fields compared here.
template <typename Make>
inline DecodePlan kept_plan_of(const keepkv_layout* L, int capacity, int force_per, int force_waves, bool charge, Make make) {
  struct Entry {
    int32_t key[9];
    DecodePlan plan;
  };
  static thread_local Entry kept[8] = {};          // (a zero batch is no valid key)
  const int32_t key[9] = {L->batch, L->n_q_heads, L->n_kv_heads, L->head_dim, L->dtype, capacity, force_per, force_waves, charge};
  uint32_t h = 0;
  for (int32_t k : key) h = h * 31u + (uint32_t)k;
  Entry& e = kept[(h ^ (h >> 15)) & 7u];
  if (memcmp(e.key, key, sizeof key) != 0) {
    e.plan = make(L, capacity, force_per, force_waves, charge);
    memcpy(e.key, key, sizeof key);
  }
  return e.plan;
}

}  // namespace
}  // namespace kk
