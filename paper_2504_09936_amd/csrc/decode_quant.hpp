// The kernel of keepkv_decode_attn_quant / keepkv_decode_step_quant: Eq. 6 over a cache of e4m3 codes, optionally with the append of a
// token (quantised as keepkv_append_quant does it) and the EMA score update (Eq. 8).  Sources of their own instantiate launch_quant
// for a dtype and head dimension each, so that they compile side by side.
#pragma once

#include <type_traits>
#include <utility>

#include "decode_common.hpp"
#include "quant_launch.hpp"

namespace kk {
namespace {

// A wavefront owns tiles of 32 slots, which are the blocks that share a scale, and takes both products to the matrix cores (16x16x32,
// bf16 operands): a code times its scale has 4 significant bits, so it is exact in bf16, and the conversion instruction applies the scale.
// The query stays as it is (f32 queries as three bf16 terms, 24 bits) and products are summed in f32.  The weights of P V are two bf16
// terms rounded to nearest (2^-18, where the output is rounded to 2^-9), of f32 layouts three (2^-27; with two an output was 1.6e-6 off, so
// 1.3e-7, for 1 to 3 % of the time).
//
// K and V rows go to LDS by asynchronous copies of whole kilobytes.  (K rows loaded straight into the operand's registers, 64 bytes of a
// row at a time, streamed 13 % slower: 221 MB in 40.9 us, 35.9 so.)  A K operand is read in an order of the channels that suits 16-byte
// reads -- the sum over channels may run in any: lane (row l16, quarter q) takes the 16 bytes at 64 h + 16 q (h = 0, 1), and the queries
// are read alike.  Of V, ds_read_b64_tr_b8 returns a channel's 8 slots of a lane in the order in which the scores lie (checked on the
// device).  16-byte chunk c of row r sits at position c ^ swizzle(r), so that what is read at once lies in different banks: 8 rows in
// sequence of K, rows 4 q + i and 16 + 4 q + i of V.
//
// The appended token is a row of the block that its slot lies in, so the wavefront of that tile quantises it, moves the block's codes to a
// larger scale if the token needs one (in LDS, and back to memory), and puts the row in before the products.  No other wavefront
// reads that block.  What the row needs of the scale is worked out by every wavefront while its first tile travels: by the one
// alone, when the tile had landed, 8 heads x 852 slots took 6.54 us, 6.28 so.
template <int D>
__device__ __forceinline__ int swizzle(int row) {
  const int half = ((row >> 2) ^ (row >> 4)) & 1;
  if constexpr (D == 128) return (row & 3) | half << 2;
  else return ((row >> 1) & 1) | half << 1;                           // (two rows to 128 bytes)
}

// 8 codes (two words) times the scale, in bf16: exact
__device__ __forceinline__ bf16x8_t expand8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Two reads of 16 bytes from LDS that the compiler does not order behind outstanding copies into it.
template <typename V>
__device__ __forceinline__ void lds_read2(uint32_t at0, uint32_t at1, V& x0, V& x1) {
  asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)" : "=&v"(x0), "=&v"(x1) : "v"(at0), "v"(at1) : "memory");
}

// Four such reads.
template <typename V>
__device__ __forceinline__ void lds_read4(const uint32_t (&at)[4], V (&x)[4]) {
  asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
               : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3])
               : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }

// How many tiles a wavefront has at most: one, two (both requested before the first wait), more (a loop); and where splits
// meet: not at all, through memory, or within an XCD where their workgroups find that they may.
constexpr int kOne = 0, kTwo = 1, kLoop = 2;
constexpr int kSoloMeet = 0, kMemMeet = 1, kXcdMeet = 2;

// LDS: per wavefront K and V tiles and (not the loop) the query rows, whole kilobytes, later its deposit (and the weights of the splits behind
// it); the loop's wavefronts share one copy of the query rows.
template <typename T>
constexpr int quant_q_bytes(int D, int G) {
  return (G * D * (int)sizeof(T) + 1023) / 1024 * 1024;
}
template <typename T>
constexpr int quant_wave_bytes(int D, int G, int tiles) {
  const int rows = tiles == kLoop ? 2 * kQBlock * D : (tiles == kOne ? 1 : 2) * 2 * kQBlock * D + quant_q_bytes<T>(D, G);
  const int deposit = (G * D + 16 + 128) * 4;
  return (rows > deposit ? rows : deposit + 127) / 128 * 128;
}
template <typename T>
constexpr int quant_lds_bytes(int D, int G, int tiles, int waves) {
  return waves * quant_wave_bytes<T>(D, G, tiles) + (tiles == kLoop ? quant_q_bytes<T>(D, G) : 0);
}

// Registers: four wavefronts of the loop to a SIMD (f32 queries, three terms: two).
constexpr int quant_waves_per_simd(int element, int tiles) { return tiles == kLoop && element == 2 ? 4 : 2; }

template <typename T, int D, int G, bool STEP, int kTiles, int kMeet, int kWaves>
__global__ __launch_bounds__(kWaves* kWave, quant_waves_per_simd(sizeof(T), kTiles)) void decode_quant_kernel(QuantParams qp) {
  const DecodeParams& p = qp.d;
  constexpr bool kF32 = sizeof(T) == 4;
  constexpr int KH = D / 64, KS = D / 32, NTILE = D / 16, CHUNKS = D / 16;
  constexpr int TILE_BYTES = kQBlock * D, BUFFER = 2 * TILE_BYTES, VLOADS = TILE_BYTES / (kWave * 16);
  constexpr int NV = kShare<G>;
  constexpr int WAVE_BYTES = quant_wave_bytes<T>(D, G, kTiles);
  constexpr int QTERMS = kF32 ? 3 : 1, PTERMS = kF32 ? 3 : 2;           // bf16 terms of a query element, of a weight
  constexpr int SCALARS = 2 + (STEP ? 1 : 0), REQUESTS = SCALARS + 2 * VLOADS;        // requests of a tile
  constexpr int EPL = D / kWave;                 // channels of a lane in an appended row
  extern __shared__ __align__(256) unsigned char smem_tiles[];
  constexpr bool kMayShareXcd = kMeet == kXcdMeet;
  __shared__ int s_last, s_one_xcd;

  const int unit = kMayShareXcd ? (int)(blockIdx.z * 8 + blockIdx.x) : (int)blockIdx.y;
  const int split = kMayShareXcd ? blockIdx.y : blockIdx.x;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, q = lane >> 4;
  KK_TS(0);
  // The head's words, requested first of all and awaited when the first tile has landed.  (Vector loads, which complete in order: a scalar
  // load's wait would be for every scalar load, and a choice between len and the bound on it would wait before anything is requested.)
  const int len_word = __hip_atomic_load(&p.len[unit], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  const int t_word = STEP ? __hip_atomic_load(&p.t_obs[unit], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) : 0;
  const int start = split * p.per;
  const size_t ubase = (size_t)unit * p.capacity;
  const int blocks = quant_blocks(p.capacity);
  const uint8_t* kbytes = reinterpret_cast<const uint8_t*>(p.k) + ubase * D;
  const uint8_t* vbytes = reinterpret_cast<const uint8_t*>(p.v) + ubase * D;
  const float* scales = (lane & 1 ? qp.v_scale : qp.k_scale) + (size_t)unit * blocks;
  unsigned char* const Tb = smem_tiles + wave * WAVE_BYTES;

  // slots that may be read (len itself, or the caller's bound on it, so that nothing waits for len); tiles up to `lim`
  int bound;
  if (p.len_hint > 0) bound = min(p.len_hint, p.capacity);
  else bound = __builtin_amdgcn_readfirstlane(len_word);
  const int lim = min(min(bound + (STEP ? 1 : 0), p.capacity), start + p.per);
  const int last_row = max(bound - 1, 0);

  const int g_l = l16 % G, r_l = l16 / G;
  const int pos0 = (r_l * NV) & 7;
  const int row0 = 16 * (pos0 >> 2) + 4 * q + (pos0 & 3);
  const int row_mine = row0 + (g_l & (NV - 1));
  const bool writer = G == 1 ? r_l < 8 : g_l < NV;

  // This workgroup has arrived (the last wavefront, whose share is the shortest), ahead of its requests.
  if (kMayShareXcd && wave == kWaves - 1 && lane == 0)
    __hip_atomic_fetch_add(&p.arrivals[unit], 1ull << (8 * xcd_id()), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

  // ---- requests
  // STEP: this lane's channels EPL lane .. of the token, as they are in memory.
  typedef typename std::conditional<kF32, typename std::conditional<EPL == 2, float2, float>::type,
                                    typename std::conditional<EPL == 2, uint32_t, uint16_t>::type>::type RowPiece;
  RowPiece k_new{}, v_new{};
  if constexpr (STEP) {
    k_new = reinterpret_cast<const RowPiece*>(p.k_t)[(size_t)unit * kWave + lane];
    v_new = reinterpret_cast<const RowPiece*>(p.v_t)[(size_t)unit * kWave + lane];
  }
  auto piece_f32 = [](const RowPiece& r, float (&x)[EPL]) {
    if constexpr (kF32 && EPL == 2) {
      x[0] = r.x;
      x[EPL - 1] = r.y;
    } else if constexpr (kF32) {
      x[0] = r;
    } else {
      x[0] = bf16_to_f32((uint16_t)r);
      if constexpr (EPL == 2) x[EPL - 1] = bf16_hi((uint32_t)r);
    }
  };
  // The query rows go through LDS: gathered by the lanes that need them they would be 16 / G times their bytes.  Chunk c of head g sits at
  // position c ^ (g mod 8) of its row.
  unsigned char* const s_q = kTiles == kLoop ? smem_tiles + kWaves * WAVE_BYTES : Tb + (kTiles == kOne ? 1 : 2) * BUFFER;
  constexpr int QROW = D * (int)sizeof(T), QCHUNKS = QROW / 16, QPIECES = quant_q_bytes<T>(D, G) / 1024;
  static_assert(QPIECES <= 4, "at most one piece of the shared copy for a wavefront");
  auto request_q = [&](int j) {
    const int c = min(j * kWave + lane, G * QCHUNKS - 1), g = c / QCHUNKS;       // surplus lanes repeat the last chunk
    copy_to_lds<0>(reinterpret_cast<const unsigned char*>(p.q) + (size_t)unit * G * QROW, (size_t)G * QROW, s_q + j * 1024,
                   (uint32_t)((c ^ (g & 7)) * 16), 0);
  };
  if constexpr (kTiles == kLoop) {
    if (wave < QPIECES) request_q(wave);
  } else {
#pragma unroll
    for (int j = 0; j < QPIECES; ++j) request_q(j);
  }
  __builtin_amdgcn_sched_barrier(0);
  struct Tile {
    float scale;                                 // of K in even lanes, of V in odd ones
    int votes;
    float ls;                                    // ln S of slot row_mine
  };
  // A copy is 1024 bytes of the tile: this lane's place in it, with its chunk as the rows from 16 on have it in `at_upper`.  The descriptor
  // ends behind the last row that may be read; beyond it a copy brings zeros.
  constexpr int COPY_ROWS = 1024 / D;
  const uint32_t at_lower = (uint32_t)(lane / CHUNKS * D + ((lane % CHUNKS) ^ swizzle<D>(lane / CHUNKS)) * 16), at_upper = at_lower ^ (8 * CHUNKS);
  auto request_rows = [&](int tbase, const uint8_t* rows, unsigned char* to) {
#pragma unroll
    for (int i = 0; i < VLOADS; ++i)
      copy_to_lds<2>(rows, (size_t)(last_row + 1) * D, to + i * 1024, (i * COPY_ROWS < 16 ? at_lower : at_upper) + (uint32_t)(tbase * D + i * 1024), 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto request_k = [&](int tbase, Tile& t, unsigned char* buf) {       // and the scalars, ahead of it
    const uint32_t block = (uint32_t)min(tbase / kQBlock, blocks - 1), at = (uint32_t)min(tbase + row_mine, last_row);
    t.scale = scales[block];
    t.votes = *reinterpret_cast<const int32_t*>(reinterpret_cast<const char*>(p.votes + ubase) + at * 4u);
    if constexpr (STEP) t.ls = *reinterpret_cast<const float*>(reinterpret_cast<const char*>(p.log_s + ubase) + at * 4u);
    else t.ls = 0.f;
    request_rows(tbase, kbytes, buf);
  };
  auto request_v = [&](int tbase, unsigned char* buf) { request_rows(tbase, vbytes, buf + TILE_BYTES); };
  auto request = [&](int tbase, Tile& t, unsigned char* buf) {
    request_k(tbase, t, buf);
    request_v(tbase, buf);
  };

  // Column l16 of the B operand is head l16 mod G, of k-step 2 h + t this lane's channels 64 h + 16 q + 8 t + j; f32 queries in three terms.
  bf16x8_t qb[QTERMS][KS];
  auto await = [&](auto behind) { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(behind)::value) : "memory"); };   // that many requests may be under way
  auto read_q = [&]() {
    const uint32_t row = lds_address(s_q + g_l * QROW);
    auto chunk = [&](int c) { return row + (uint32_t)((c ^ (g_l & 7)) * 16); };
    if constexpr (!kF32) {
      lds_read2(chunk(2 * q), chunk(2 * q + 1), qb[0][0], qb[0][1]);
      if constexpr (KS == 4) lds_read2(chunk(8 + 2 * q), chunk(9 + 2 * q), qb[0][2], qb[0][3]);
    } else {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        f32x4_t a, b;
        const int c = 16 * (ks >> 1) + 4 * q + 2 * (ks & 1);
        lds_read2(chunk(c), chunk(c + 1), a, b);
        float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
        for (int t = 0; t < 3; ++t) {            // each term takes the 8 leading bits of what is left
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = pack_hi16(x[2 * i], x[2 * i + 1]);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x[i]) & 0xFFFF0000u);
          qb[t][ks] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
        }
      }
    }
  };

  bool grow;
  int len_old, t_old, len, live_end, new_row, own_base;                      // own_base: the tile that the appended token joins
  auto read_len = [&]() {
    len_old = __builtin_amdgcn_readfirstlane(len_word);
    t_old = __builtin_amdgcn_readfirstlane(t_word);
    grow = STEP && len_old < p.capacity;
    len = grow ? len_old + 1 : len_old;
    live_end = min(len, start + p.per);
    new_row = len_old % kQBlock;
    own_base = grow ? len_old - new_row : -1;
  };

  const float sl2 = p.scale * kLog2e;
  float m_run = kLowest, l_run = 0.f;
  f32x4_t O[NTILE];
#pragma unroll
  for (int nt = 0; nt < NTILE; ++nt) O[nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // The scales that the new rows need, worked out while the first tile travels.
  uint32_t need_k = 0, need_v = 0;
  auto read_new = [&]() {
    auto need = [&](const RowPiece& r) {
      float x[EPL], a = 0.f;
      piece_f32(r, x);
#pragma unroll
      for (int e = 0; e < EPL; ++e) a = fmaxf(a, __builtin_bit_cast(float, finite_magnitude(x[e])));
      a = over_head_lanes<1>(a, [](float u, float v) { return fmaxf(u, v); });
      return scale_bits((uint32_t)__builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, a)));
    };
    if constexpr (STEP) {
      need_k = need(k_new);
      need_v = need(v_new);
    }
  };
  bool wrote = false;                            // (uniform) this wavefront has the appended row
  uint32_t k_code = 0, v_code = 0;               // this lane's EPL codes of it
  float new_ks = 0.f, new_vs = 0.f;

  // The first wavefront requests the head's `arrivals` when its last tile's rows have landed, to have the word when the tile is done.
  uint64_t seen = 0;
  bool looked = !kMayShareXcd || wave != 0;      // uniform
  auto look = [&]() {
    if (!looked) seen = ld_arrivals(p, unit);
    looked = true;
  };

  // One tile; its K rows have landed when at most k_wait requests are outstanding, its V rows with v_wait.  Returns the group-mean logit of
  // slot row_mine and whether this lane stores it.
  // first: no tile of this wavefront has been computed.  last: it may be its last live one, which the appended token may join and which may
  // be partly live; all before it are full.
  // k_done(), v_done(): called when the rows have been read from LDS.
  auto compute = [&](int tbase, const Tile& t, unsigned char* Kb, bool first, auto last, auto k_wait, auto v_wait, auto k_done, auto v_done,
                     float& x_out, float& ls_old) -> bool {
    constexpr int kVWait = decltype(v_wait)::value;
    constexpr bool kLast = decltype(last)::value;
    const int n_live = kLast ? min(kQBlock, live_end - tbase) : kQBlock;
    x_out = ls_old = 0.f;
    if (n_live <= 0) return false;               // uniform: below the caller's bound but dead, its scales mean nothing
    float ks = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, t.scale), 0));
    float vs = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, t.scale), 1));
    const bool own = STEP && kLast && tbase == own_base;   // uniform
    unsigned char* const Vb = Kb + TILE_BYTES;
    if (own) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kVWait) : "memory");
      wrote = true;
      // into the tile and, rows moved to a larger scale, back to memory
      auto join = [&](const RowPiece& r, uint32_t need, float& scale, uint32_t& code, unsigned char* rows, uint8_t* memory) {
        const uint32_t old = __builtin_bit_cast(uint32_t, scale), bits = new_row > 0 ? max(need, old) : need;
        if (new_row > 0 && bits != old) {        // uniform
          const float ratio = scale * inverse_scale(bits);
          for (int i = lane; i < new_row * CHUNKS; i += kWave) {
            uint4 w = reinterpret_cast<const uint4*>(rows)[i];
            w = make_uint4(shift_codes(w.x, ratio), shift_codes(w.y, ratio), shift_codes(w.z, ratio), shift_codes(w.w, ratio));
            reinterpret_cast<uint4*>(rows)[i] = w;
            const int row = i / CHUNKS, chunk = (i % CHUNKS) ^ swizzle<D>(row);
            *reinterpret_cast<uint4*>(memory + (size_t)(tbase + row) * D + 16 * chunk) = w;
          }
        }
        scale = __builtin_bit_cast(float, bits);
        const float inv = inverse_scale(bits);
        float x[EPL];
        piece_f32(r, x);
        code = encode4(x[0] * inv, EPL == 2 ? x[EPL - 1] * inv : 0.f, 0.f, 0.f);
        unsigned char* at = rows + new_row * D + ((lane * EPL / 16) ^ swizzle<D>(new_row)) * 16 + lane * EPL % 16;
        if constexpr (EPL == 2) *reinterpret_cast<uint16_t*>(at) = (uint16_t)code;
        else *at = (unsigned char)code;
      };
      join(k_new, need_k, ks, k_code, Kb, const_cast<uint8_t*>(kbytes));
      join(v_new, need_v, vs, v_code, Vb, const_cast<uint8_t*>(vbytes));
      new_ks = ks;
      new_vs = vs;
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    // ---- S^T = K Q^T
    await(k_wait);
    u32x4_t kr[2 * KH];                          // [st][h]
    {
      uint32_t at = lds_address(Kb) + (uint32_t)(l16 * D + (q ^ swizzle<D>(l16)) * 16);
      if constexpr (kTiles == kLoop) asm volatile("" : "+v"(at));      // (addresses are worked out anew: registers are short)
      if constexpr (KH == 2) lds_read4({at, at ^ 64, (at ^ 64) + 16 * D, at + 16 * D}, kr);   // (bit 4 of a row turns bit 2 of its swizzle)
      else lds_read2(at, (at ^ 32) + 16 * D, kr[0], kr[1]);
    }
    k_done();
    bf16x8_t ka[2][KS];
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int k_step = 0; k_step < KS; ++k_step) {
        const u32x4_t w = kr[st * KH + (k_step >> 1)];
        ka[st][k_step] = expand8(w[2 * (k_step & 1)], w[2 * (k_step & 1) + 1], ks);
      }
    f32x4_t s[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int term = QTERMS - 1; term >= 0; --term)
#pragma unroll
      for (int k_step = 0; k_step < KS; ++k_step)
#pragma unroll
        for (int st = 0; st < 2; ++st) s[st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[st][k_step], qb[term][k_step], s[st], 0, 0, 0);
    float sv[NV];
    take_shares<G>(s, r_l, pos0, sv);
    // ---- logits (log2 domain, log2(votes) folded in), group-mean logit for the EMA
    const bool mine_new = own && row_mine == new_row;
    const float lp_lane = mine_new ? 0.f : fast_log2((float)t.votes);
    ls_old = mine_new ? -INFINITY : t.ls;
    float z[NV], xm[NV], lp[NV];
    if constexpr (NV == 1) lp[0] = lp_lane;
    else {                                       // slot row0 + v is loaded by lane v of the quad
      lp[0] = dpp_f32<0x00>(lp_lane);
      lp[1] = dpp_f32<0x55>(lp_lane);
      if constexpr (NV == 4) {
        lp[2] = dpp_f32<0xAA>(lp_lane);
        lp[3] = dpp_f32<0xFF>(lp_lane);
      }
    }
    float tm = -INFINITY;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const bool live = row0 + v < n_live && (G > 1 || r_l < 8);
      z[v] = live ? fmaf(sv[v], sl2, lp[v]) : -INFINITY;
      tm = fmaxf(tm, z[v]);
      xm[v] = head_sum<G>(sv[v]);
    }
    const float mn = fmaxf(m_run, over_head_lanes<G>(tm, [](float a, float b) { return fmaxf(a, b); }));
    const float c = fast_exp2(m_run - mn);
    float pr[NV], ps = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      pr[v] = fast_exp2(z[v] - mn);
      ps += pr[v];
    }
    l_run = fmaf(l_run, c, ps);
    m_run = mn;
    if (!first && __any(c != 1.f)) rescale_rows<G>(O, c, l16, q);
    // (tied to the softmax sum, so that the wait is not scheduled ahead of the arithmetic it is meant to hide)
    asm volatile("s_waitcnt vmcnt(%1)" : "+v"(l_run) : "n"(kVWait) : "memory");
    if (kVWait == 0) look();
    if (n_live < kQBlock) {                      // uniform: rows of masked slots are cleared (0 * NaN would be NaN)
      for (int i = n_live * CHUNKS + lane; i < kQBlock * CHUNKS; i += kWave) reinterpret_cast<uint4*>(Vb)[i] = make_uint4(0, 0, 0, 0);
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    // ---- O += P V
    uint32_t aw[PTERMS][4];
    weights_operand<G, true>(pr, r_l, pos0, aw[0], aw[1]);
    if constexpr (kF32) {                        // (and what two terms leave)
      float rest[NV];
      uint32_t none[4];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        auto nearest = [](float x) { return bf16_to_f32(f32_to_bf16_bits(x)); };
        rest[v] = pr[v] - nearest(pr[v]);
        rest[v] -= nearest(rest[v]);
      }
      weights_operand<G, true>(rest, r_l, pos0, aw[2], none);
    }
    const int vrow = 16 * (l16 >> 3) + 4 * q + ((l16 >> 1) & 3);      // the row whose half this lane's address names
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
    u32x2_t b[NTILE];
    uint32_t va[NTILE];
    uint32_t va0 = lds_address(Vb) + (uint32_t)(vrow * D + swizzle<D>(vrow) * 16 + (l16 & 1) * 8);
    if constexpr (kTiles == kLoop) asm volatile("" : "+v"(va0));
#pragma unroll
    for (int nt = 0; nt < NTILE; ++nt) va[nt] = va0 ^ (uint32_t)(nt * 16);
    if constexpr (NTILE == 8)
      asm volatile(
          "ds_read_b64_tr_b8 %0, %8\n\tds_read_b64_tr_b8 %1, %9\n\tds_read_b64_tr_b8 %2, %10\n\tds_read_b64_tr_b8 %3, %11\n\t"
          "ds_read_b64_tr_b8 %4, %12\n\tds_read_b64_tr_b8 %5, %13\n\tds_read_b64_tr_b8 %6, %14\n\tds_read_b64_tr_b8 %7, %15\n\t"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(b[0]), "=&v"(b[1]), "=&v"(b[2]), "=&v"(b[3]), "=&v"(b[4]), "=&v"(b[5]), "=&v"(b[6]), "=&v"(b[7])
          : "v"(va[0]), "v"(va[1]), "v"(va[2]), "v"(va[3]), "v"(va[4]), "v"(va[5]), "v"(va[6]), "v"(va[7])
          : "memory");
    else
      asm volatile(
          "ds_read_b64_tr_b8 %0, %4\n\tds_read_b64_tr_b8 %1, %5\n\tds_read_b64_tr_b8 %2, %6\n\tds_read_b64_tr_b8 %3, %7\n\t"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(b[0]), "=&v"(b[1]), "=&v"(b[2]), "=&v"(b[3])
          : "v"(va[0]), "v"(va[1]), "v"(va[2]), "v"(va[3])
          : "memory");
    v_done();
#pragma unroll
    for (int part = 0; part < PTERMS; ++part)
#pragma unroll
      for (int nt = 0; nt < NTILE; ++nt)
        O[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, make_uint4(aw[part][0], aw[part][1], aw[part][2], aw[part][3])),
                                                        expand8(b[nt][0], b[nt][1], vs), O[nt], 0, 0, 0);
    float x = xm[0];
#pragma unroll
    for (int v = 1; v < NV; ++v) x = (g_l & (NV - 1)) == v ? xm[v] : x;
    x_out = x * (p.scale * (1.0f / G));
    return writer && row_mine < n_live;
  };
  auto ema = [&](float ls_old, float x) {        // ln(alpha S + (1 - alpha) e^x)
    const float a = p.ln_alpha + ls_old, b = p.ln_1m_alpha + x;
    const float hi = fmaxf(a, b), lo = fminf(a, b);
    return (lo == -INFINITY) ? hi : hi + kLn2 * fast_log2(1.f + fast_exp2((lo - hi) * kLog2e));
  };

  constexpr int kTileStep = kWaves * kQBlock;
  constexpr std::true_type kIsLast{};
  constexpr std::false_type kNotLast{};
  constexpr std::integral_constant<int, 0> kAll{};
  constexpr std::integral_constant<int, VLOADS> kOwnV{};              // (the tile's own V rows)
  constexpr std::integral_constant<int, REQUESTS> kTile{};
  constexpr std::integral_constant<int, REQUESTS + VLOADS> kOwnVAndTile{};
  constexpr std::integral_constant<int, 2 * REQUESTS> kTwoTiles{};
  auto nothing = [] {};
  const int base = start + wave * kQBlock;
  bool own0 = false, own1 = false;               // results per slot that are stored at the very end
  float x0 = 0.f, x1 = 0.f, ls0 = 0.f, ls1 = 0.f;
  Tile t0, t1;
  if constexpr (kTiles == kOne) {
    if (base < lim) {
      request(base, t0, Tb);
      read_new();
      await(kTile);
      read_q();
      read_len();
      own0 = compute(base, t0, Tb, true, kIsLast, kOwnV, kAll, nothing, nothing, x0, ls0);
    }
  } else if constexpr (kTiles == kTwo) {
    if (base < lim) {
      request(base, t0, Tb);
      request(base + kTileStep, t1, Tb + BUFFER);                     // (beyond the head's last row zeros, beyond the split the next one's rows)
      read_new();
      await(kTwoTiles);
      read_q();
      read_len();
      own0 = compute(base, t0, Tb, true, kIsLast, kOwnVAndTile, kTile, nothing, nothing, x0, ls0);
      if (base + kTileStep < live_end)
        own1 = compute(base + kTileStep, t1, Tb + BUFFER, false, kIsLast, kOwnV, kAll, nothing, nothing, x1, ls1);
    }
  } else {
    auto publish = [&](int tbase, bool mine, float x, float ls_old) {
      if (p.logits_out != nullptr && mine) p.logits_out[ubase + tbase + row_mine] = x;
      if (STEP && mine) p.log_s[ubase + tbase + row_mine] = ema(ls_old, x);
    };
    // One buffer: the next tile's K rows are requested when this one's have been read from LDS, its V rows alike, and four wavefronts to a
    // SIMD cover what a wavefront waits.  Only tiles that exist are requested: a surplus request is a memory round trip before the
    // wavefront may deposit.  (Two tiles in flight and two wavefronts to a SIMD: 1024 heads x 852 slots 46.1 us and 45.4 so, 624 heads x 731
    // 34.0 and 28.7, attention over 64 heads x 8192 27.0 and 26.2.)  New scores are stored as they come: held back in LDS for the end they
    // gave nothing once a compute unit's workgroups all end together.
    if (base < lim) {
      request(base, t0, Tb);
      read_new();
      await(kTile);
    } else {
      await(kAll);
    }
    __builtin_amdgcn_s_barrier();                // every wavefront's piece of the query rows is there (tiles may be under way)
    if (base < lim) {
      read_q();
      read_len();
      int tb = base, left = live_end > base ? (live_end - base + kTileStep - 1) / kTileStep : 0;
      for (; left > 1; --left, tb += kTileStep) {
        float x, ls;
        const bool mine = compute(tb, t0, Tb, tb == base, kNotLast, kOwnV, std::integral_constant<int, SCALARS + VLOADS>{},
                                  [&] { request_k(tb + kTileStep, t1, Tb); }, [&] { request_v(tb + kTileStep, Tb); }, x, ls);
        publish(tb, mine, x, ls);
        t0 = t1;
      }
      if (left > 0) {
        float x, ls;
        const bool mine = compute(tb, t0, Tb, tb == base, kIsLast, kOwnV, kAll, nothing, nothing, x, ls);
        publish(tb, mine, x, ls);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                  // no copy may land in what follows
  }

  KK_TS(1);
  read_len();                                    // (a wavefront without a tile)
  // ---- this wavefront's state, then the workgroup's
  const float l_tot = over_head_lanes<G>(l_run, [](float a, float b) { return a + b; });
  constexpr int kPartStride = WAVE_BYTES / 4;
  float* s_acc = reinterpret_cast<float*>(smem_tiles);
  float* s_ml = s_acc + G * D;
  if constexpr (kTiles != kLoop) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the copies of a tile that was passed over)
  deposit_state<D, G>(O, m_run, l_tot, s_acc + wave * kPartStride, s_ml + wave * kPartStride, lane);
  if (threadIdx.x == 0) {
    look();                                      // (a wavefront without a tile)
    s_one_xcd = kMayShareXcd && all_on_this_xcd(p, unit, seen);
  }
  __syncthreads();
  KK_TS(2);
  if constexpr (kTiles != kLoop) {
    auto store = [&](int tbase, bool mine, float x, float ls_old) {
      const size_t at = ubase + tbase + row_mine;
      if (p.logits_out != nullptr && mine) p.logits_out[at] = x;
      if (STEP && mine) p.log_s[at] = ema(ls_old, x);
    };
    store(base, own0, x0, ls0);
    if constexpr (kTiles == kTwo) store(base + kTileStep, own1, x1, ls1);
  }
  if (STEP && wrote) {                           // the appended token joins the cache
    const size_t at = (size_t)len_old * D + lane * EPL;
    if constexpr (EPL == 2) {
      *reinterpret_cast<uint16_t*>(const_cast<uint8_t*>(kbytes) + at) = (uint16_t)k_code;
      *reinterpret_cast<uint16_t*>(const_cast<uint8_t*>(vbytes) + at) = (uint16_t)v_code;
    } else {
      const_cast<uint8_t*>(kbytes)[at] = (uint8_t)k_code;
      const_cast<uint8_t*>(vbytes)[at] = (uint8_t)v_code;
    }
    if (lane == 0) {
      p.votes[ubase + len_old] = 1;
      p.born[ubase + len_old] = t_old;
      qp.k_scale[(size_t)unit * blocks + len_old / kQBlock] = new_ks;
      qp.v_scale[(size_t)unit * blocks + len_old / kQBlock] = new_vs;
    }
  }
  combine_and_finish<T, D, G, kWaves, STEP, kWaves, true, kMeet == kSoloMeet, kMayShareXcd>(p, s_ml, s_ml + G, s_acc, kPartStride, kPartStride, &s_last,
                                                                                             unit, split, grow, len, t_old,
                                                                                             __builtin_amdgcn_readfirstlane(s_one_xcd) != 0);
}

template <typename T, int D, int G>
keepkv_status launch_quant_g(const QuantParams& p, int units, bool step, hipStream_t st) {
  auto go = [&](auto step_tag, auto tiles_tag, auto meet_tag, auto waves_tag) -> keepkv_status {
    constexpr int kTiles = decltype(tiles_tag)::value, kWaves = decltype(waves_tag)::value;
    constexpr size_t lds = quant_lds_bytes<T>(D, G, kTiles, kWaves);
    static_assert(lds + 1024 <= 160 * 1024, "LDS of a compute unit");
    auto* kernel = decode_quant_kernel<T, D, G, decltype(step_tag)::value, kTiles, decltype(meet_tag)::value, kWaves>;
    if constexpr (lds > 60 * 1024) {
      static const bool allowed = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) == hipSuccess;
      if (!allowed) return KEEPKV_ERR_DEVICE;
    }
    // (x, then y, is dealt first: with 8 heads along x the splits of a head come to one XCD, see all_on_this_xcd)
    const dim3 grid = decltype(meet_tag)::value == kXcdMeet ? dim3(8, p.d.nsplit, units / 8) : dim3(p.d.nsplit, units);
    kernel<<<grid, kWaves * kWave, lds, st>>>(p);
    return launch_status();
  };
  auto by_waves = [&](auto step_tag, auto tiles_tag, auto meet_tag) {
    if (p.d.waves == 8) return go(step_tag, tiles_tag, meet_tag, std::integral_constant<int, 8>{});
    return go(step_tag, tiles_tag, meet_tag, std::integral_constant<int, 4>{});
  };
  auto by_meet = [&](auto step_tag, auto tiles_tag) {
    if (p.d.nsplit == 1) return by_waves(step_tag, tiles_tag, std::integral_constant<int, kSoloMeet>{});
    if constexpr (decltype(tiles_tag)::value != kLoop)
      if (p.d.arrivals != nullptr) return by_waves(step_tag, tiles_tag, std::integral_constant<int, kXcdMeet>{});
    return by_waves(step_tag, tiles_tag, std::integral_constant<int, kMemMeet>{});
  };
  const int n_tiles = (p.d.per + p.d.waves * kQBlock - 1) / (p.d.waves * kQBlock);      // of a wavefront, at most
  auto by_tiles = [&](auto step_tag) {
    if (n_tiles == 1) return by_meet(step_tag, std::integral_constant<int, kOne>{});
    if constexpr (sizeof(T) == 2)                // (f32 layouts, which no large cache has, do with the loop)
      if (n_tiles == 2) return by_meet(step_tag, std::integral_constant<int, kTwo>{});
    return by_meet(step_tag, std::integral_constant<int, kLoop>{});
  };
  return step ? by_tiles(std::true_type{}) : by_tiles(std::false_type{});
}

}  // namespace

template <typename T, int D>
keepkv_status launch_quant(const QuantParams& p, int units, int G, bool step, hipStream_t st) {
  switch (G) {
    case 1: return launch_quant_g<T, D, 1>(p, units, step, st);
    case 2: return launch_quant_g<T, D, 2>(p, units, step, st);
    case 4: return launch_quant_g<T, D, 4>(p, units, step, st);
    default: return launch_quant_g<T, D, 8>(p, units, step, st);
  }
}

}  // namespace kk
