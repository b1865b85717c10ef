// HIP kernels for gfx950: decode attention over a cache whose rows are held in 4 bits (fp4.hpp).
//
// For every query head:  s_t = scale * <q, K_t>,  w = softmax(s),  out = sum_t w_t V_t, one pass over the cache with the running
// maximum and sum. A token of a kv head is 136 bytes (heads of 64: 68), a quarter of bf16's, so the arithmetic per byte is
// four times as much: at the rate of a streaming read, 48 cycles of a SIMD per token, whatever the number of heads.
//
// The cut of a launch, what becomes of requests that several waves share, and the combine pass are those of the other attention
// kernels (device.hpp); the work is dealt out in units of 16 rows of a chunk. A tile is U units. Both products are
// 16x16x32 matrix instructions with up to 16 q heads of a kv head as columns:
//   scores  S^T = K Q^T. Lane (g, c) of a wave (g = lane / 16, c = lane % 16) loads a quarter of row c: dims g D/4 .. of it, whose
//      codes the conversion instruction turns into bf16 values, exactly, eight dims (a word) to an operand. The contraction
//      index of lane group g is its own quarter of the dims; Q is laid out alike. Register i of a unit's result is the score
//      of token 4 g + i for head c.
//   softmax  a lane owns head c and four tokens of every unit; the weights are where the second product wants them.
//   PV      O^T = V^T P^T, two units at a time: contraction index of lane group g = its four tokens of either unit. Lane l loads a
//      quarter of row l / 4; as fp16 values with their scale on them the rows of two units go through LDS, which hands them
//      out transposed (a read that gives a lane 4 rows of one dim).
// Products in 4 and 8 bits with scales (16x16x128) would take the codes as they are, but do not add up in 32 bits: their results
// were 8e-5 of the sum of the products' magnitudes off.
// 16 requests of 32768 to 131072 tokens, 8 q heads each take 228 us (6.4 TB/s, the vector unit busy for half of the time): HBM. 64 of
// 512 to 24576, 16 q heads of 64, take 30.7 (3.5 TB/s): the vector unit, 60 % busy, between the ramp and the sums of shared requests.
// The K rows of the next tile are asked for when this one's scores are formed, its V rows when this one's have gone to LDS.
#include "fp4.hpp"
#include "fp4_walk.hpp"

namespace ellm {

// V rows of two units on their way through LDS, half of the dims at a time (heads of 64: all): two words, 16 dims, of every quarter.
// Rows are 32 bytes apart modulo the banks' 128, which keeps the transposing reads (32 bytes of 4 rows at a time) off each
// other's banks; the order of a quarter's two words in odd rows keeps the writes (16 bytes of all quarters of 2 rows) apart.
constexpr int STAGE_ROW = 4 * 32 + 32, STAGE_BYTES = 2 * UNIT_TOKENS * STAGE_ROW;
__device__ __forceinline__ int32_t stage_write(int32_t row, int32_t quarter, int32_t w) { return row * STAGE_ROW + quarter * 32 + ((w ^ (row & 1)) * 16); }
// 4 dims, the fourth `piece`, of the 16 of a quarter
__device__ __forceinline__ int32_t stage_read(int32_t row, int32_t piece, int32_t quarter) {
  return row * STAGE_ROW + quarter * 32 + ((piece * 8) ^ ((row & 1) * 16));
}

// The second product is one of fp16 values, of more bits than bf16 and a smaller range, which is used to its ends. A weight is held
// relative to the running maximum, at most 2^WEIGHT_BITS; what its rounding loses is 2^-12 of it, or, of the smallest ones, 2^-25 of
// 1 / 2^WEIGHT_BITS: 2^-37 of the largest weight (2^-25 over LARGE_SCORE, below). A scale of V is held relative to the largest one of the same block that the
// wave has met in the request, and the values are exact down to 2^-36 of it. (Weights as sums of two bf16 values, which need no such care, take twice as
// many products and 60 more of 310 instructions a tile: 16 requests of 32768 to 131072 tokens, 8 q heads each 249 us a call.)
constexpr int WEIGHT_BITS = 12, VALUE_BITS = 13;
// Scores over LARGE_SCORE are multiples of 2^-3 and more: the product with the scale is then rounded before the maximum is taken
// off, so that the largest comes out as 0 and no weight outside the range, and WEIGHT_BITS, which might be rounded up, stays away.
constexpr float LARGE_SCORE = 0x1p20f;
// what weights are relative to, for a largest score of `top`
__device__ __forceinline__ float reference(float top) { return __builtin_fabsf(top) > LARGE_SCORE ? top : top - WEIGHT_BITS; }

// a request's chunks
template <bool DIRECT>
struct Fp4Tensor {
  TensorWalk walk;
  const char* base;                  // start of the pool, or of the tensor's range
  Fp4Tensor() = default;
  __device__ __forceinline__ Fp4Tensor(const PoolView& pv, int32_t tensor) : walk(tensor_walk<DIRECT>(pv, tensor)), base(DIRECT ? walk.tbase : pv.base) {}
  __device__ __forceinline__ uint32_t chunk(int32_t slot) const { return DIRECT ? (uint32_t)slot : (uint32_t)walk.trow[slot]; }
};

typedef short __attribute__((ext_vector_type(4))) s16x4_t;
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;

// NW == 0: a wave walks its share, SW of them are a workgroup (SW == 1: single_waves()). NW > 0: NW waves share a step of up to NW * U units
// of one request, one tile each, and add up through LDS. HEADS: q heads that LDS has room for.
template <int D, int U, int HEADS, bool RUN, bool APPEND, bool DIRECT, int NW, int SW, class Args>
__device__ __forceinline__ void decode_fp4_body(const PoolView& pv, const uint16_t* __restrict__ q, const char* __restrict__ k_new,
                                                const char* __restrict__ v_new, float* __restrict__ ws, uint16_t* __restrict__ out,
                                                float scale_log2, int32_t g_first, int32_t n_heads, const Args& a, int32_t workgroup) {
  constexpr int W = D / 32, ROW = FP4_ROW<D>, SCALES = FP4_SCALES<D>;     // words of a lane's quarter of a row
  using Tile = Fp4Tile<U, RUN>;
  constexpr int NB = D / 16, F = D / 4;                                   // 16-dim blocks of the result; pieces of its rows
  static_assert(U % 2 == 0, "PV takes two units at a time");
  const int lane = threadIdx.x & 63, c = lane & 15, g16 = lane >> 4, vr = lane >> 2, vp = lane & 3;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Records<Args> records(a, lane);
  wanted(a.n_req, a.waves_per_head, a.units_each, a.units_extra, a.by_waves.mul, a.by_waves.shift, a.step_units, a.q_row0);
  wanted(pv.chunk_bytes, pv.tokens_per_chunk, pv.units_per_chunk, DIRECT ? 0 : pv.max_slots, pv.n_q_heads, pv.n_kv_heads, pv.group, g_first);
  wanted(DIRECT ? nullptr : pv.base, DIRECT ? nullptr : pv.table, pv.vbase, q, pv.by_chunk.mul, pv.by_chunk.shift, pv.by_units.mul, pv.by_units.shift);
  const int32_t Tc = pv.tokens_per_chunk;
  const uint32_t plane = (uint32_t)Tc * ROW, scale_plane = (uint32_t)Tc * SCALES;      // from K to V of the same head

  const int32_t index = NW ? workgroup : workgroup * SW + wave;
  const Share<Args> sh = locate_share(a, records, NW ? index : min(index, a.waves_per_head * pv.n_kv_heads - 1), lane);
  const int32_t g = sh.g;
  const int32_t hq0 = g * pv.group + g_first;        // first q head handled here
  const int32_t head = min(c, n_heads - 1);          // lanes beyond the last head repeat it and write nothing
  const uint64_t head_rows = (uint64_t)(2 * g) * plane, head_scales = fp4_scales_at<D>(pv) + (uint64_t)(2 * g) * scale_plane;

  // Scores are kept without the scale, of which only the sign goes into the query (the maximum has to be one): its size is part
  // of the exponential's argument, in log2 units, as are the reference m of the maximum and the other kernels' partial results.
  const float size = __builtin_fabsf(scale_log2);
  const uint32_t sign = scale_log2 < 0.f ? 0x80008000u : 0u;

  using Tensor = Fp4Tensor<DIRECT>;
  auto open = [&](int32_t tensor) __attribute__((always_inline)) { return Tensor(pv, tensor); };
  const typename Args::Req& first_rq = sh.first;
  Fp4Cursor<U, RUN, Tensor> cursor;
  cursor.template begin<NW>(pv, a, first_rq, sh.b, sh.w, sh.u_lo, sh.n_units, wave, open);
  auto advance = [&](Tile& t) __attribute__((always_inline)) { cursor.next(pv, a, open, t); };
  // a piece's K rows and scales (V's: plane, scale_plane further on)
  auto rows_base = [&](const Tile& t, int i) __attribute__((always_inline)) {
    return const_cast<char*>(t.base) + (uint64_t)t.at[i] * pv.chunk_bytes + head_rows + (uint32_t)t.r[i] * ROW;
  };
  auto scales_base = [&](const Tile& t, int i) __attribute__((always_inline)) {
    return const_cast<char*>(t.base) + (uint64_t)t.at[i] * pv.chunk_bytes + head_scales + (uint32_t)t.r[i] * SCALES;
  };
  auto there = [&](const Tile& t, int i) __attribute__((always_inline)) { return t.template there<APPEND>(i); };
  // rows of unit u
  auto rows_of = [&](const Tile& t, int u) __attribute__((always_inline)) {
    return RUN ? min(t.rows[0] - u * UNIT_TOKENS, UNIT_TOKENS) : t.rows[RUN ? 0 : u];
  };
  // the last piece of a tile (a unit that the tile does not have has the address of the one before it), and which row of it is
  // the tile's last
  constexpr int LAST = Tile::PIECES - 1;
  auto last_row = [&](const Tile& t) __attribute__((always_inline)) { return (RUN ? t.rows[0] : t.tail) - 1; };

  // ---- loads ----
  // Buffer loads with the unit's rows as their range: rows past its end, and units that the tile does not have, come back as
  // zeros (codes of 0, scales of 2^-127) without a memory access, and the number of loads does not depend on the tile.
  struct Quarter { uint32_t w[W]; };                 // of a row of codes
  Quarter k[U], v[U];
  uint32_t ks[U], vs[U];
  words4_t qr[W];
  uint32_t kn[D / 8], vn[D / 8];                     // the new row's quarter, in bf16
  const int scale_of_quarter = D == 128 ? 1 : 2;     // quarters that share a scale
  auto load_quarter = [&](__amdgpu_buffer_rsrc_t rows, int32_t at) __attribute__((always_inline)) {
    Quarter x;
    if constexpr (W == 4) {
      const words4_t w = __builtin_amdgcn_raw_buffer_load_b128(rows, at, 0, CPOL_NT);
      x.w[0] = w.x; x.w[1] = w.y; x.w[2] = w.z; x.w[3] = w.w;
    } else {
      const words2_t w = __builtin_amdgcn_raw_buffer_load_b64(rows, at, 0, CPOL_NT);
      x.w[0] = w.x; x.w[1] = w.y;
    }
    return x;
  };
  auto new_row = [&](const Tile& t) __attribute__((always_inline)) {
    return ((int64_t)(a.q_row0 + t.b) * pv.n_kv_heads + g) * (2 * D);
  };
  auto load_new = [&](const char* from, int32_t quarter, uint32_t (&x)[D / 8]) __attribute__((always_inline)) {
    const gptr_t p = (gptr_t)from + quarter * (D / 2);
#pragma unroll
    for (int i = 0; i < D / 32; i++) {
      const words4_t w = *(const __attribute__((address_space(1))) words4_t*)(p + 16 * i);
      x[4 * i] = w.x; x[4 * i + 1] = w.y; x[4 * i + 2] = w.z; x[4 * i + 3] = w.w;
    }
  };
  // ask(rows, scales, u, rows before unit u in them) for every unit of a tile, whose rows are so many bytes behind K's
  auto each_piece = [&](const Tile& t, uint32_t rows_off, uint32_t scales_off, auto ask) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < Tile::PIECES; i++) {
      const int32_t n = there(t, i);
      const auto rows = buffer_at(rows_base(t, i) + rows_off, n * ROW), scales = buffer_at(scales_base(t, i) + scales_off, n * SCALES);
#pragma unroll
      for (int u = RUN ? 0 : i; u < (RUN ? U : i + 1); u++) ask(rows, scales, u, RUN ? u * UNIT_TOKENS : 0);
    }
  };
  auto issue_k = [&](const Tile& t) __attribute__((always_inline)) {
    if (t.flags & T_FIRST) {
      const gptr_t qp = (gptr_t)(q + ((int64_t)(a.q_row0 + t.b) * pv.n_q_heads + hq0 + head) * D) + g16 * (D / 2);
#pragma unroll
      for (int w = 0; w < W; w++) qr[w] = *(const __attribute__((address_space(1))) words4_t*)(qp + w * 16) ^ sign;
    }
    if (APPEND && (t.flags & T_LAST)) load_new(k_new + new_row(t), g16, kn);
    auto ask = [&](const __amdgpu_buffer_rsrc_t rows, const __amdgpu_buffer_rsrc_t scales, int u, int at) __attribute__((always_inline)) {
      k[u] = load_quarter(rows, at * ROW + c * ROW + g16 * (4 * W));
      ks[u] = __builtin_amdgcn_raw_buffer_load_b8(scales, at * SCALES + c * SCALES + g16 / scale_of_quarter, 0, CPOL_NT);
    };
    each_piece(t, 0, 0, ask);
  };
  auto issue_v = [&](const Tile& t) __attribute__((always_inline)) {
    if (APPEND && (t.flags & T_LAST)) load_new(v_new + new_row(t), vp, vn);
    auto ask = [&](const __amdgpu_buffer_rsrc_t rows, const __amdgpu_buffer_rsrc_t scales, int u, int at) __attribute__((always_inline)) {
      v[u] = load_quarter(rows, at * ROW + lane * (4 * W));
      vs[u] = __builtin_amdgcn_raw_buffer_load_b8(scales, at * SCALES + vr * SCALES + vp / scale_of_quarter, 0, CPOL_NT);
    };
    each_piece(t, plane, scale_plane, ask);
  };
  // A quarter of a new row in 4 bits; `partner`: the larger magnitude of this lane's and that of the lane that has the other half of a
  // block (heads of 64)
  auto quantise = [&](const uint32_t (&x)[D / 8], Quarter& codes, uint32_t& scale, auto partner) __attribute__((always_inline)) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < D / 8; i++) top = max_magnitudes(top, x[i]);
    if constexpr (D == 64) top = partner(top);
    scale = fp4_scale(top);
#pragma unroll
    for (int w = 0; w < W; w++) {
      const uint32_t eight[4] = {x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]};
      codes.w[w] = fp4_codes(eight, scale);
    }
  };
  // stored where it belongs: row `row` of the unit whose rows and scales begin there, quarter `quarter`
  auto store_new = [&](char* rows, char* scales, int32_t row, int32_t quarter, const Quarter& codes, uint32_t scale) __attribute__((always_inline)) {
    const gwptr_t to = (gwptr_t)rows + row * ROW + quarter * (4 * W);
    if constexpr (W == 4) *(__attribute__((address_space(1))) words4_t*)to = words4_t{codes.w[0], codes.w[1], codes.w[2], codes.w[3]};
    else *(__attribute__((address_space(1))) words2_t*)to = words2_t{codes.w[0], codes.w[1]};
    if (quarter % scale_of_quarter == 0) *(__attribute__((address_space(1))) uint8_t*)((gwptr_t)scales + row * SCALES + quarter / scale_of_quarter) = (uint8_t)scale;
  };

  // ---- arithmetic ----
  float top = NEG_BIG, m = NEG_BIG, l = 0.f;         // the maximum so far, what weights are relative to, their sum
  float times = size;                                // what scores still have to be multiplied by: 1 if some head's maximum is large
  bool large = false;
  uint32_t largest = 0;                              // of V's scales in the request so far, of the block that lane & 3 is a quarter of
  f32x4_t acc[NB], s[U];
  auto scores = [&](const Tile& t) __attribute__((always_inline)) {
    if (APPEND && (t.flags & T_LAST)) {
      // the new token's K row takes the place of what the loads found there, and goes into the chunk (a unit that the tile
      // does not have has the address of the one before it)
      Quarter codes;
      uint32_t scale;
      quantise(kn, codes, scale, [](uint32_t x) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return max_magnitudes(r[0], r[1]);
      });
      const int32_t rl = t.tail - 1;
#pragma unroll
      for (int u = 0; u < U; u++) {
        const bool mine = u == t.n - 1 && c == rl;
#pragma unroll
        for (int w = 0; w < W; w++) k[u].w[w] = mine ? codes.w[w] : k[u].w[w];
        ks[u] = mine ? scale : ks[u];
      }
      if (c == rl) store_new(rows_base(t, LAST), scales_base(t, LAST), last_row(t), g16, codes, scale);
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      f32x4_t d = {0.f, 0.f, 0.f, 0.f};
      const float scale = fp4_scale_float(ks[u]);
#pragma unroll
      for (int w = 0; w < W; w++) d = mfma16(fp4_values(k[u].w[w], scale), qr[w], d);
      s[u] = d;
    }
  };
  auto weigh = [&](const Tile& t, char* stage) __attribute__((always_inline)) {
    if (t.flags & T_FIRST) {
      top = m = NEG_BIG;
      l = 0.f;
      large = false;
      times = size;
#pragma unroll
      for (int n = 0; n < NB; n++) acc[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    bool full = true;
#pragma unroll
    for (int i = 0; i < Tile::PIECES; i++) full &= t.rows[i] == (RUN ? U * UNIT_TOKENS : UNIT_TOKENS);
    if (!full) {
      // scores of rows that are not there
#pragma unroll
      for (int u = 0; u < U; u++)
#pragma unroll
        for (int i = 0; i < 4; i++) s[u][i] = 4 * g16 + i < rows_of(t, u) ? s[u][i] : -INFINITY;
    }
    if (APPEND && (t.flags & T_LAST)) {
      // the new token's V row
      Quarter codes;
      uint32_t scale;
      quantise(vn, codes, scale, [](uint32_t x) { return max_magnitudes_xor1(x); });
      const int32_t rl = t.tail - 1;
#pragma unroll
      for (int u = 0; u < U; u++) {
        const bool mine = u == t.n - 1 && vr == rl;
#pragma unroll
        for (int w = 0; w < W; w++) v[u].w[w] = mine ? codes.w[w] : v[u].w[w];
        vs[u] = mine ? scale : vs[u];
      }
      if (vr == rl) store_new(rows_base(t, LAST) + plane, scales_base(t, LAST) + scale_plane, last_row(t), vp, codes, scale);
    }
    float mx = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
#pragma unroll
    for (int u = 1; u < U; u++) mx = fmaxf(mx, fmaxf(fmaxf(s[u][0], s[u][1]), fmaxf(s[u][2], s[u][3])));
    const float tn = fmaxf(top, max_xor32(max_xor16(mx)) * size);
    if (__builtin_amdgcn_ballot_w64(tn > top) != 0 || large) {     // some head has a new maximum, or a large one
      const float mn = reference(tn), alpha = fast_exp2(m - mn);
      l *= alpha;
#pragma unroll
      for (int n = 0; n < NB; n++) acc[n] *= alpha;
      top = tn;
      m = mn;
      large = __builtin_amdgcn_ballot_w64(__builtin_fabsf(top) > LARGE_SCORE) != 0;
      times = large ? 1.f : size;
      if (large)
#pragma unroll
        for (int u = 0; u < U; u++) s[u] *= size;
    }
    // the largest of V's scales in this tile (a block that is NaN has none)
    uint32_t scale_top = 0;
#pragma unroll
    for (int u = 0; u < U; u++) scale_top = max(scale_top, vs[u] == FP4_SCALE_NAN ? 0u : vs[u]);
    if ((t.flags & T_FIRST) || __builtin_amdgcn_ballot_w64(scale_top > largest)) {
      const uint32_t now = max_of_quarter(scale_top), before = t.flags & T_FIRST ? now : largest;
      largest = max(now, before);
      const int by = (int)(before - largest);
#pragma unroll
      for (int n = 0; n < NB; n++)
#pragma unroll
        for (int i = 0; i < 4; i++) acc[n][i] = __builtin_amdgcn_ldexpf(acc[n][i], __builtin_amdgcn_readlane(by, n / (W / 2)));
    }
#pragma unroll
    for (int u = 0; u < U; u += 2) {
      words4_t weights;
#pragma unroll
      for (int h = 0; h < 4; h++) {
        const f32x4_t& x = s[u + h / 2];
        const float p0 = fast_exp2(x[2 * (h & 1)] * times - m), p1 = fast_exp2(x[2 * (h & 1) + 1] * times - m);
        l += p0 + p1;
        weights[h] = pack_f16(p0, p1);
      }
      float scale[2];
#pragma unroll
      for (int j = 0; j < 2; j++) {
        const uint32_t e = __builtin_elementwise_sub_sat(vs[u + j] + (127 + VALUE_BITS), largest);
        scale[j] = fp4_scale_float(vs[u + j] == FP4_SCALE_NAN ? FP4_SCALE_NAN : e);
      }
#pragma unroll
      for (int half = 0; half < W / 2; half++) {
        // rows of units u and u + 1 to LDS: row 16 j + vr, words of quarter vp
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
          for (int w = 0; w < 2; w++)
            *reinterpret_cast<words4_t*>(stage + stage_write(UNIT_TOKENS * j + vr, vp, w)) = fp4_values_f16(v[u + j].w[2 * half + w], scale[j]);
        // 16 dims of a quarter: lane (g, c) addresses 4 of them in row 4 g + c / 4 and gets the c-th of rows 4 g .. 4 g + 3
#pragma unroll
        for (int p = 0; p < 4; p++) {
          char* const from = stage + stage_read(4 * g16 + (c >> 2), c & 3, p);
          const words2_t lo = __builtin_bit_cast(words2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)from)),
                         hi = __builtin_bit_cast(words2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(from + UNIT_TOKENS * STAGE_ROW)));
          const int n = p * (W / 2) + half;
          acc[n] = mfma16_f16(words4_t{lo.x, lo.y, hi.x, hi.y}, weights, acc[n]);
        }
      }
    }
  };
  // When a request or the share ends: the sums become means, of weights that are `inv` of what was added up, and get V's scale back, in
  // this order: V may be as large as floats are, and the sums are up to 2^WEIGHT_BITS for every token of that.
  auto means = [&](float inv) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NB; n++)
#pragma unroll
      for (int i = 0; i < 4; i++)
        acc[n][i] = __builtin_amdgcn_ldexpf(acc[n][i] * inv, __builtin_amdgcn_readlane((int)largest - (127 + VALUE_BITS), n / (W / 2)));
  };
  // which piece of a row, in the order of partial_dim() for units, has dims 16 n + 4 g16 .. + 3
  auto piece = [&](int n) __attribute__((always_inline)) {
    if constexpr (D == 128) {
      const int e = 2 * n + (g16 >> 1);
      return (e & 3) * 8 + (g16 & 1) * 4 + (e >> 2);
    } else {
      return 4 * g16 + n;
    }
  };

  if constexpr (NW > 0) {
    constexpr int ROWF = D + 4;                        // a row of a head's accumulators, padded against bank conflicts
    // a wave's V rows on their way through LDS, and then its sums
    constexpr int MINE = std::max<int>(STAGE_BYTES, HEADS * ROWF * 4);
    __shared__ __attribute__((aligned(16))) char lds[NW][MINE];
    __shared__ float2 ml[NW][HEADS];
    float* const mine = reinterpret_cast<float*>(lds[wave]);
    if (cursor.rem_share > 0) {
      Tile t;
      advance(t);
      issue_k(t);
      issue_v(t);
      __builtin_amdgcn_sched_barrier(0);
      scores(t);
      weigh(t, lds[wave]);
      const float L = add_xor32(add_xor16(l));
      means(share_of(L));
      if (c < n_heads) {
#pragma unroll
        for (int n = 0; n < NB; n++)
          *reinterpret_cast<float4*>(mine + c * ROWF + piece(n) * 4) = make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
        if (g16 == 0) ml[wave][c] = make_float2(m, L);
      }
    } else {
      // nothing left for this wave: zeros, whose weight is 0
      if (lane < n_heads) ml[wave][lane] = make_float2(-INFINITY, 0.f);
      for (int i = lane; i < n_heads * F; i += 64) *reinterpret_cast<float4*>(mine + i / F * ROWF + i % F * 4) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
    // every wave takes 64 columns (pieces of the heads' rows in order), which need no other wave from here on
    const int32_t n_cols = n_heads * F;
    static_assert(HEADS * F <= NW * 64, "a thread for every column");
    const int32_t x = threadIdx.x, h = x / F, f = x % F;
    if (wave * 64 >= n_cols) return;
    Sum sum = {NEG_BIG, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    if (x < n_cols) {
      float2 p[NW];
      float4 v4[NW];
#pragma unroll
      for (int w = 0; w < NW; w++) {
        p[w] = ml[w][h];
        v4[w] = *reinterpret_cast<const float4*>(lds[w] + (h * ROWF + f * 4) * 4);
      }
#pragma unroll
      for (int w = 0; w < NW; w++) sum.M = fmaxf(sum.M, p[w].x);
      float L[NW], weight[NW];
#pragma unroll
      for (int w = 0; w < NW; w++) {
        L[w] = p[w].y;
        weight[w] = fast_exp2(p[w].x - sum.M);
      }
      add_means(sum, sum.M, L, v4, weight);
      if (cursor.part < 0) write_out<D, true>(pv, out, a, cursor.b, g, g_first, x, sum);
      else leave_partial<D>(pv, ws, a, cursor.part, g, g_first, n_heads, x, sum);
    }
    // one of several blocks of its request: the last of them to get here adds their results up
    const int32_t n_part = first_rq.n_part;
    if (n_part == 1 || n_part > a.merge_parts) return;
    stores_done();
    uint32_t before = 0;
    if (lane == 0) before = count_in(pv, g * a.waves_per_head + first_rq.wave_first + wave % n_part, wave, n_part);
    const Partials<D, true> all(ws, a.ws_slots, (int64_t)g * a.parts_per_head + first_rq.part0, n_part, held(pv.group), g_first, n_heads);
    if (__builtin_amdgcn_readfirstlane(before) != (uint32_t)n_part - 1u) return;
    Sum all_of[1];
    all.template sum<1, 8, 16>(all_of, x, 0, 0, n_part);
    if (x < n_cols) write_out<D, true>(pv, out, a, cursor.b, g, g_first, x, all_of[0]);
    return;
  }
  __shared__ __attribute__((aligned(16))) char stages[NW ? 1 : SW][NW ? 1 : STAGE_BYTES];
  __shared__ __attribute__((aligned(16))) Results<D, SW == 1 ? 1 : HEADS> results;     // (SW == 1: not used)
  char* const stage = stages[NW ? 0 : wave];
  auto finish = [&](const Tile& t) __attribute__((always_inline)) {
    const float L = add_xor32(add_xor16(l));
    means(t.part < 0 ? __builtin_amdgcn_rcpf(L) : share_of(L));
    if (c >= n_heads) return;
    if (t.part < 0) {
      // the whole request lay inside this wave's share: round and write the output rows
      uint16_t* o = out + ((int64_t)(a.q_row0 + t.b) * pv.n_q_heads + hq0 + c) * D + 4 * g16;
#pragma unroll
      for (int n = 0; n < NB; n++)
        *reinterpret_cast<uint2*>(o + 16 * n) = make_uint2(pack_bf16(acc[n][0], acc[n][1]), pack_bf16(acc[n][2], acc[n][3]));
    } else if constexpr (SW == 1) {
      // one of several waves of the request: a partial result
      const int64_t row = ((int64_t)g * a.parts_per_head + t.part) * pv.group + g_first + c;
#pragma unroll
      for (int n = 0; n < NB; n++)
        *reinterpret_cast<float4*>(ws + row * D + piece(n) * 4) = make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
      if (g16 == 0) *reinterpret_cast<float2*>(ws + (int64_t)a.ws_slots * pv.group * D + row * WS_ML) = make_float2(m, L);
    } else {
      // its results meet the others' in LDS
      const int32_t to = 2 * wave + (t.b == sh.b ? 0 : 1);
#pragma unroll
      for (int n = 0; n < NB; n++)
        results.rows[to][c][piece(n)] = make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
      if (g16 == 0) results.ml[to][c] = make_float2(m, L);
      if (lane == 0) results.whose[to] = g * MAX_LAUNCH_REQ + t.b;
    }
  };
  // No exit before the round's last load (the share's last round asks for rows it does not use): what is in flight when a
  // tile is waited for is the same on every path, so the compiler counts the loads exactly.
  if (index < a.waves_per_head * pv.n_kv_heads) {
    Tile t, next;
    advance(t);
    issue_k(t);
    issue_v(t);
    __builtin_amdgcn_sched_barrier(0);               // the loads stay where they are asked for
    if constexpr (SW > 1) results.clear(wave, lane);
    advance(next);
    uint32_t done;
    do {
      scores(t);
      issue_k(next);
      __builtin_amdgcn_sched_barrier(0);
      weigh(t, stage);
      if (t.flags & (T_LAST | T_FIN)) finish(t);     // the request ends here, or the share does
      done = t.flags & T_FIN;
      issue_v(next);
      __builtin_amdgcn_sched_barrier(0);
      t = next;
      advance(next);
    } while (!done);
  } else if constexpr (SW > 1) {
    results.clear(wave, lane);
  }
  if constexpr (SW > 1) end_shares<D, HEADS, 8, 4, true>(pv, ws, out, a, records, results, g_first, n_heads, workgroup, wave, lane);
}

template <int D, int U, int HEADS, int SW, bool RUN, bool APPEND, bool DIRECT, class Args>
__global__ __launch_bounds__(64 * SW) __attribute__((amdgpu_waves_per_eu(D * HEADS > FP4_TWO_WORKGROUPS ? 1 : 2, D * HEADS > FP4_TWO_WORKGROUPS ? 1 : 2))) void decode_fp4_kernel(
    PoolView pv, const uint16_t* __restrict__ q, const char* __restrict__ k_new, const char* __restrict__ v_new,
    float* __restrict__ ws, uint16_t* __restrict__ out, float scale_log2, int32_t g_first, int32_t n_heads, Args a) {
  in_launch(pv, ws, a, [&](const PoolView& pv, float* ws, const auto& a, int32_t workgroup) __attribute__((always_inline)) {
    decode_fp4_body<D, U, HEADS, RUN, APPEND, DIRECT, 0, SW>(pv, q, k_new, v_new, ws, out, scale_log2, g_first, n_heads, a, workgroup);
  });
}
template <int D, int U, int HEADS, int NW, bool APPEND, bool DIRECT, class Args>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void decode_fp4_block_kernel(
    PoolView pv, const uint16_t* __restrict__ q, const char* __restrict__ k_new, const char* __restrict__ v_new,
    float* __restrict__ ws, uint16_t* __restrict__ out, float scale_log2, int32_t g_first, int32_t n_heads, Args a) {
  in_launch(pv, ws, a, [&](const PoolView& pv, float* ws, const auto& a, int32_t workgroup) __attribute__((always_inline)) {
    decode_fp4_body<D, U, HEADS, false, APPEND, DIRECT, NW, 1>(pv, q, k_new, v_new, ws, out, scale_log2, g_first, n_heads, a, workgroup);
  });
}

// ---------------------------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------------------------
// Units per tile of heads of 128 in short shares, and of all others. Of shares of few tiles those count whose last tile, or the
// last of a request, is not full; of long ones the bytes on their way. 64 requests of 64 to 8192 tokens, 8 kv heads (15 units a
// wave) 19.9 us a call by 2 units, 20.8 by 4; 48, 6 q heads each 22.3, 24.6; chunks of 16 tokens 15.5, 17.0; 200 requests (28 units) 52.3,
// 52.4; 32 of 2048 to 16384, 40 heads 268, 251; 16 of 32768 to 131072 241, 228. Heads of 64, 16 q heads, 64 of 512 to 24576 34.8, 30.5.
constexpr int FP4_SHORT_TILE = 2, FP4_TILE = 4;

// calls go(heads that LDS has room for) for a pass over n of them
template <class Go>
static int for_heads(int n, Go go) {
  if (n <= 4) return go(std::integral_constant<int, 4>{});
  return n <= 8 ? go(std::integral_constant<int, 8>{}) : go(std::integral_constant<int, HEADS_PER_PASS>{});
}

// a: the plan, or one of the two in `args`, which run the same kernel; workgroups: of all of it
template <int D, bool APPEND, bool DIRECT, class Args>
static int launch_fp4_i(const PoolView& pv, const void* q, const void* k_new, const void* v_new, float* ws, void* out, float scale_log2,
                        const BatchArgs& a, const Args& args, unsigned workgroups, hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop) {
  constexpr bool PAIR = std::is_same_v<Args, PairArgs>;
  // a group of more than HEADS_PER_PASS q heads is covered by several launches over the same K/V: the first of them takes the
  // start time, the last one the end time
  for (int done = 0; done < pv.group; done += HEADS_PER_PASS) {
    const int n = std::min(HEADS_PER_PASS, pv.group - done);
    auto go = [&](auto kernel, unsigned waves, const auto& its) {
      return launch(kernel, dim3(workgroups), 64 * waves, stream, done == 0 ? ev_start : nullptr, done + n >= pv.group ? ev_stop : nullptr, pv,
                    (const uint16_t*)q, (const char*)k_new, (const char*)v_new, ws, (uint16_t*)out, scale_log2, (int32_t)done, (int32_t)n, its);
    };
    int e = -1;
    if (a.step_units > STEP_UNITS) {
      auto in_blocks = [&](const auto& its) {
        using Its = std::decay_t<decltype(its)>;
        if (a.step_units <= BLOCK_UNITS) return go(decode_fp4_block_kernel<D, 2, HEADS_PER_PASS, 8, APPEND, DIRECT, Its>, 8, its);
        return go(decode_fp4_block_kernel<D, WIDE_UNITS / WIDE_WAVES, HEADS_PER_PASS, WIDE_WAVES, APPEND, DIRECT, Its>, WIDE_WAVES, its);
      };
      e = in_blocks(args);
    } else {
      if constexpr (!PAIR)               // (single_waves() is for several passes)
        if (a.wg_waves == 1) e = go(decode_fp4_kernel<D, FP4_TILE, HEADS_PER_PASS, 1, false, APPEND, DIRECT, Args>, 1, args);
      if (e < 0)
        e = for_heads(std::min(HEADS_PER_PASS, pv.group), [&](auto heads) {
          auto in_tiles = [&](auto units) {
            if (pv.tokens_per_chunk >= FP4_RUN_TOKENS)
              return go(decode_fp4_kernel<D, units(), heads(), SHARE_WAVES, true, APPEND, DIRECT, Args>, SHARE_WAVES, args);
            return go(decode_fp4_kernel<D, units(), heads(), SHARE_WAVES, false, APPEND, DIRECT, Args>, SHARE_WAVES, args);
          };
          if constexpr (D == 128)
            if (fp4_short_shares(D, a)) return in_tiles(std::integral_constant<int, FP4_SHORT_TILE>{});
          return in_tiles(std::integral_constant<int, FP4_TILE>{});
        });
    }
    if (e) return e;
  }
  return 0;
}

int fp4_waves_per_cu(int head_dim, int group) {
  if (group > HEADS_PER_PASS) return fp4_most_waves_per_cu(head_dim, group);
  int n = 0;
  auto ask = [&](auto dim) {
    return for_heads(group, [&](auto h) {
      return (int)hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, (const void*)decode_fp4_kernel<dim(), FP4_TILE, h(), SHARE_WAVES, false, true, false, BatchArgs>,
                                                               64 * SHARE_WAVES, 0);
    });
  };
  const int e = head_dim == 128 ? ask(std::integral_constant<int, 128>{}) : ask(std::integral_constant<int, 64>{});
  if (e || n < 1) n = 1;
  return std::min(n * SHARE_WAVES, fp4_most_waves_per_cu(head_dim, group));
}

template <class Args>
static int launch_fp4(const PoolView& pv, const void* q, const void* k_new, const void* v_new, float* ws, void* out, float scale_log2,
                      const BatchArgs& a, const Args& args, unsigned workgroups, hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop) {
  auto go = [&](auto launch) { return launch(pv, q, k_new, v_new, ws, out, scale_log2, a, args, workgroups, stream, ev_start, ev_stop); };
  auto of_size = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    if (k_new) return pv.vbase ? go(launch_fp4_i<D, true, true, Args>) : go(launch_fp4_i<D, true, false, Args>);
    return pv.vbase ? go(launch_fp4_i<D, false, true, Args>) : go(launch_fp4_i<D, false, false, Args>);
  };
  return pv.head_dim == 128 ? of_size(std::integral_constant<int, 128>{}) : of_size(std::integral_constant<int, 64>{});
}

static unsigned workgroups_of(const PoolView& pv, const BatchArgs& a) {
  return ((unsigned)(a.waves_per_head * pv.n_kv_heads) + a.wg_waves - 1) / a.wg_waves;
}

int launch_fp4_decode(const PoolView& pv, const void* q, const void* k_new, const void* v_new, float* ws, void* out, float scale_log2,
                      const BatchArgs& a, hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop) {
  if (a.n_req <= 0 || a.waves_per_head <= 0) return 0;
  return launch_fp4(pv, q, k_new, v_new, ws, out, scale_log2, a, a, workgroups_of(pv, a), stream, ev_start, ev_stop);
}

int launch_fp4_decode_pair(const PoolView& pv, const void* q, const void* k_new, const void* v_new, float* ws, void* out, float scale_log2,
                           PairArgs& a, hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop) {
  a.workgroups = workgroups_of(pv, a.half[0]);
  return launch_fp4(pv, q, k_new, v_new, ws, out, scale_log2, a.half[0], a, a.workgroups + workgroups_of(pv, a.half[1]), stream, ev_start, ev_stop);
}

}  // namespace ellm
