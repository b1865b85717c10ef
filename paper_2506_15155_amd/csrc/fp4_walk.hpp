// Which rows a wave of the decode kernels over 4-bit rows asks for, tile by tile: integers only, for the device and, in tests, the host.
#pragma once
#include "kernels.hpp"

namespace ellm {

enum : uint32_t { T_FIRST = 1, T_LAST = 2, T_FIN = 4 };   // a tile starts a request here, ends it, ends the share
// What is known of a tile before its loads are issued (uniform). RUN: its units are neighbours in one chunk, a tile ends where its
// chunk does, and one address is enough for all of it; else every unit has an address of its own.
template <int U, bool RUN>
struct Fp4Tile {
  static constexpr int PIECES = RUN ? 1 : U;
  int32_t n, b, part;                // units, request, partial slot of the request in this wave (-1: finished here)
  uint32_t flags;                    // T_*
  int32_t tail;                      // rows of its last unit
  int32_t rows[PIECES];              // of the run, or of each unit (0: the tile has no such unit)
  int32_t r[PIECES];                 // first row in its chunk
  uint32_t at[PIECES];               // the chunk (table entry, or slot of the tensor's own range)
  const char* base;                  // start of the pool, or of the tensor's range

  // how many of a piece's rows are in the chunk: all but the one that a fused append is about to put there
  template <bool APPEND>
  ELLM_BOTH_INLINE int32_t there(int i) const {
    return rows[i] - (APPEND && (flags & T_LAST) && (RUN || i == n - 1) ? 1 : 0);
  }
};

// The next tile to be asked for. Tensor: a request's chunks, made from its handle by open(); chunk(slot), base.
template <int U, bool RUN, class Tensor>
struct Fp4Cursor {
  int32_t b, rem_share, len, slot, r, rem_req, part;
  uint32_t first;
  Tensor tensor;

  // Where a share begins. NW == 0: n_units steps of its head's sequence from u_lo on, the first of which belongs to request b (rq).
  // NW > 0: of such a step, which NW waves have, the units of wave `wave`.
  template <int NW, class Args, class Open>
  ELLM_BOTH_INLINE void begin(const PoolView& pv, const Args& a, const typename Args::Req& rq, int32_t b_, int32_t w, int32_t u_lo,
                              int32_t n_units, int32_t wave, Open open) {
    b = b_;
    first = T_FIRST;
    len = rq.len;
    tensor = open(rq.tensor);
    constexpr int32_t STEP_WAVES = NW ? NW : 1;
    const int32_t mine = NW ? wave * a.step_units / STEP_WAVES : 0;     // (at most U apart from one wave to the next)
    const int32_t u0 = (u_lo - rq.unit_prefix) * a.step_units + mine;
    rem_req = units_of(len, pv, pv.units_per_chunk) - u0;
    rem_share = n_units;
    if (NW) rem_share = least((wave + 1) * a.step_units / STEP_WAVES - mine, rem_req);
    else if (a.step_units > 1) rem_share = least(n_units * a.step_units, rem_req);
    slot = divide(u0, pv.by_units);
    r = (u0 - slot * pv.units_per_chunk) * UNIT_TOKENS;
    part = rq.n_part == 1 ? -1 : rq.part0 + (w - rq.wave_first);    // (which slot: only where a workgroup is a step)
  }

  template <class Args, class Open>
  ELLM_BOTH_INLINE void next(const PoolView& pv, const Args& a, Open open, Fp4Tile<U, RUN>& t) {
    const int32_t Tc = pv.tokens_per_chunk;
    t.n = least(U, least(rem_share, rem_req));
    t.b = b;
    t.part = part;
    t.flags = first;
    t.base = tensor.base;
    if constexpr (RUN) {
      t.n = least(t.n, (Tc - r + UNIT_TOKENS - 1) / UNIT_TOKENS);
      t.at[0] = tensor.chunk(slot);
      t.r[0] = r;
      t.rows[0] = least(t.n * UNIT_TOKENS, least(Tc - r, len - (slot * Tc + r)));      // (past the end of the share: 0)
      t.tail = t.rows[0] - (t.n - 1) * UNIT_TOKENS;
      if (rem_req > t.n) {                             // there is a next unit of this request
        r += t.n * UNIT_TOKENS;
        if (r >= Tc) { r = 0; slot += 1; }
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; u++) {
        if (u == 0 || u < t.n) {
          t.at[u] = tensor.chunk(slot);
          t.r[u] = r;
          t.rows[u] = least(UNIT_TOKENS, least(Tc - r, len - (slot * Tc + r)));
          t.tail = t.rows[u];
          if (u < t.n - 1 || (t.n > 0 && rem_req > t.n)) {   // there is a next unit of this request
            r += UNIT_TOKENS;
            if (r >= Tc) { r = 0; slot += 1; }
          }
        } else {
          t.at[u] = t.at[u - 1];
          t.r[u] = t.r[u - 1];
          t.rows[u] = 0;
        }
      }
      if (t.n == 0) t.rows[0] = 0;                     // past the end of the share
    }
    rem_req -= t.n;
    rem_share -= t.n;
    first = 0;
    if (rem_req == 0) {
      // (not a tile behind the share's last one, which has no row that a fused append could put anywhere: one less than no rows is, as
      // the range of a buffer, all of memory)
      if (t.n > 0) t.flags |= T_LAST;
      first = T_FIRST;
    }
    if (rem_share == 0) t.flags |= T_FIN;
    if (rem_req == 0 && rem_share > 0) {
      b += 1;
      const typename Args::Req rq = a.req[b];
      len = rq.len;
      rem_req = units_of(len, pv, pv.units_per_chunk);
      tensor = open(rq.tensor);
      slot = 0;
      r = 0;
      part = rq.n_part == 1 ? -1 : rq.part0;
    }
  }
};

}  // namespace ellm
