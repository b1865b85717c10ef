// What the kernels of this library share: bf16 and cross-lane helpers, addresses of chunks, the partition of a decode launch
// and what becomes of requests that several waves share, launches by address.
#pragma once
#include "kernels.hpp"

#include <hip/hip_runtime.h>
#include <hip/hip_ext.h>

#include <algorithm>
#include <type_traits>

namespace ellm {

// ---------------------------------------------------------------------------------------------
// small helpers
// ---------------------------------------------------------------------------------------------
// fp32 -> bf16 bits, round to nearest even; NaN stays NaN
__device__ __forceinline__ uint32_t f32_to_bf16_bits(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7fc0u;
  u += 0x7fffu + ((u >> 16) & 1u);
  return u >> 16;
}

// v + (v of lane ^ 16), v + (v of lane ^ 32): gfx950's row and half-wave swaps exchange the odd rows
// (upper half) of one register with the even rows (lower half) of another; fed the same value
// twice they return the two partners side by side, with no trip through the LDS crossbar
__device__ __forceinline__ float add_xor16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add_xor32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// DPP lane permutations inside a row of 16 lanes
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
constexpr int DPP_QUAD_XOR1 = 0xB1;        // quad_perm [1,0,3,2]
constexpr int DPP_QUAD_XOR2 = 0x4E;        // quad_perm [2,3,0,1]
constexpr int DPP_ROW_HALF_MIRROR = 0x141; // lane i <-> 7 - i within each 8 lanes
constexpr int DPP_ROW_MIRROR = 0x140;      // lane i <-> 15 - i within each 16 lanes

__device__ __forceinline__ float max_xor16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_xor32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// reductions over the 64 lanes, result in every lane: four steps inside the rows of 16 lanes (DPP),
// then the two swaps across rows
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp_f32<DPP_QUAD_XOR1>(v));
  v = fmaxf(v, dpp_f32<DPP_QUAD_XOR2>(v));
  v = fmaxf(v, dpp_f32<DPP_ROW_HALF_MIRROR>(v));
  v = fmaxf(v, dpp_f32<DPP_ROW_MIRROR>(v));
  return max_xor32(max_xor16(v));
}

__device__ __forceinline__ float wave_sum(float v) {
  v += dpp_f32<DPP_QUAD_XOR1>(v);
  v += dpp_f32<DPP_QUAD_XOR2>(v);
  v += dpp_f32<DPP_ROW_HALF_MIRROR>(v);
  v += dpp_f32<DPP_ROW_MIRROR>(v);
  return add_xor32(add_xor16(v));
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef short __attribute__((ext_vector_type(4))) bf16x4_bits_t;     // four bf16 values as the matrix instructions take them
typedef float __attribute__((ext_vector_type(4))) f32x4_t;

typedef __attribute__((ext_vector_type(2))) float f32x2_t;
// two floats rounded to nearest-even bf16, the first in the low half
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}

// c + a.lo * b.lo + a.hi * b.hi on packed bf16 pairs, fp32 accumulate
__device__ __forceinline__ float dot2_bf16(uint32_t a, uint32_t b, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a), __builtin_bit_cast(bf16x2_t, b), c, false);
}

// The same, with the first operand taken from lane N of this lane's row of 16 (a DPP broadcast
// folded into the instruction): lets 16 lanes share one register of query values.
template <int N>
__device__ __forceinline__ float dot2_bf16_rowlane(uint32_t row_shared, uint32_t b, float c) {
  asm("v_dot2c_f32_bf16_dpp %0, %1, %2 row_newbcast:%3 row_mask:0xf bank_mask:0xf"
      : "+v"(c) : "v"(row_shared), "v"(b), "n"(N));
  return c;
}

// The compiler cannot see that the inline-asm instruction above is a dot product, so it does not
// insert the wait states the hardware needs between a dot product's result and its first use by a
// different instruction (nor between a register write and its first use as a DPP source). Passing
// the value through this makes the gap explicit.
__device__ __forceinline__ void settle(float& v) { asm volatile("s_nop 3" : "+v"(v)); }
__device__ __forceinline__ void settle(uint32_t& v) { asm volatile("s_nop 1" : "+v"(v)); }

template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

// 16-byte load of data that is read once (the K/V stream): marked non-temporal, so that it does not
// displace what is reused (partials, queries, tables) from the caches on its way through
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_stream16(const void* p) {
  const u32x4_t t = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
  return make_uint4(t.x, t.y, t.z, t.w);
}
__device__ __forceinline__ void store_stream16(void* p, uint4 v) {
  const u32x4_t t = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(t, reinterpret_cast<u32x4_t*>(p));
}

// cache-policy operand of the buffer and load-to-LDS builtins: non-temporal; coherent across the GPU (past the L2
// of the wave's own XCD)
constexpr int CPOL_NT = 2, CPOL_DEVICE = 16;

typedef __attribute__((ext_vector_type(4))) uint32_t words4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t words2_t;

// memory from `base` on (the same for all lanes; said so, because the descriptor has to be in scalar registers) as a
// buffer: loads past its end return zeros, stores past it are dropped
constexpr int BUFFER_RAW = 0x00027000;    // last word of a buffer descriptor: raw dwords, range check on the byte offset
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* base, int32_t bytes) {
  const uint64_t b = (uint64_t)base;
  const uint64_t bs = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b) |
                      (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32)) << 32;
  return __builtin_amdgcn_make_buffer_rsrc((void*)bs, 0, __builtin_amdgcn_readfirstlane(bytes), BUFFER_RAW);
}

typedef const __attribute__((address_space(1))) void* global_cptr_t;
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef const int32_t __attribute__((address_space(4)))* const_i32_ptr;
typedef const uint64_t __attribute__((address_space(4)))* const_u64_ptr;

// How a kernel gets from (tensor, slot) to the chunk's bytes. With the software table the slot's
// entry names a chunk of the pool. DIRECT is the paper's own arrangement (Sec. 2.1.1, Sec. 3.2): the
// tensor is a contiguous virtual address range into which the driver has mapped the chunks, so a
// slot's bytes sit at base + slot * chunk_bytes and no table is read.
struct TensorWalk {
  const_i32_ptr trow;      // table row of the tensor (table addressing)
  const char* tbase;       // start of the tensor's virtual range (direct addressing)
};
template <bool DIRECT>
__device__ __forceinline__ TensorWalk tensor_walk(const PoolView& pv, int32_t tensor) {
  TensorWalk w;
  if (DIRECT) {
    w.trow = nullptr;
    w.tbase = reinterpret_cast<const char*>(((const_u64_ptr)pv.vbase)[tensor]);
  } else {
    w.trow = (const_i32_ptr)(pv.table + (int64_t)tensor * pv.max_slots);
    w.tbase = nullptr;
  }
  return w;
}
template <bool DIRECT>
__device__ __forceinline__ const char* chunk_addr(const PoolView& pv, const TensorWalk& w, int32_t slot) {
  if (DIRECT) return w.tbase + (uint64_t)slot * pv.chunk_bytes;
  return pv.base + (uint64_t)w.trow[slot] * pv.chunk_bytes;
}

// s_waitcnt immediates (gfx9 encoding): vmcnt in bits 3:0 and 15:14, expcnt 6:4, lgkmcnt 11:8
constexpr int waitcnt_vm(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0F70; }

constexpr float NEG_BIG = -3.402823466e38f;   // finite stand-in for "no score yet", below every score; exp2(NEG_BIG - x) == 0 but for x near it

// 16x16x32 matrix products; what becomes of a weight that is multiplied as two bf16 values
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef const __attribute__((address_space(1))) char* gptr_t;
typedef __attribute__((address_space(1))) char* gwptr_t;

__device__ __forceinline__ f32x4_t mfma16(words4_t a, words4_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// the largest bf16 value below a positive float, as a float's bits; 0 for 0, NaN for NaN
__device__ __forceinline__ uint32_t bf16_below(float p) {
  return __builtin_elementwise_sub_sat(__float_as_uint(p), 1u) & 0xffff0000u;
}

// ---------------------------------------------------------------------------------------------
// work partition shared by the partial pass, the combine pass and the calibration kernel
// ---------------------------------------------------------------------------------------------
// Kernel arguments that a wave needs early. Named in one place, they are asked for together when it starts; left to
// itself the compiler puts loads of them behind waits for other loads and behind branches, and no cache holds them yet.
// (eight to an asm statement: across such statements loads are not made into wider ones)
template <class A, class B, class C, class D, class E, class F, class G, class H>
__device__ __forceinline__ void wanted(A a, B b, C c, D d, E e, F f, G g, H h) {
  asm volatile("" :: "s"(a), "s"(b), "s"(c), "s"(d), "s"(e), "s"(f), "s"(g), "s"(h));
}

// A kernel argument as a value of its own, which is not loaded again later and from which nothing is derived earlier
template <class T>
__device__ __forceinline__ T held(T v) {
  asm volatile("" : "+s"(v));
  return v;
}

// The records of a launch's requests, spread over the lanes of a wave: lane l has those of requests l, l + 64, .. Where a
// wave begins used to be found in three dependent steps (header, a table of the waves' requests, the record), about a third
// of a microsecond each from the L2 and more from memory, which no cache holds the arguments of. Now all records are asked for
// at once, together with the header, when the wave starts. One request of 3300 tokens 8.25 -> 7.99 us a call, 8 requests, 4
// layers 52.3 -> 51.6, four short ones 7.38 -> 7.11; shares no different (8B-shaped step 1992, 1994).
template <class Args>
struct Records {
  using Req = typename Args::Req;
  static constexpr int N = (Args::MAX_REQ + 63) / 64;
  int32_t len[N], tensor[N], unit_prefix[N], wave_first[N], n_part[N], part0[N];
  __device__ __forceinline__ Records(const Args& a, int lane) {
    static_for<0, N>([&](auto kc) {
      constexpr int k = decltype(kc)::value;
      const Req& r = a.req[min(64 * k + lane, Args::MAX_REQ - 1)];
      len[k] = r.len; tensor[k] = r.tensor; unit_prefix[k] = r.unit_prefix;
      wave_first[k] = r.wave_first; n_part[k] = r.n_part; part0[k] = r.part0;
    });
  }
  // request whose units include unit number pos of a kv head's sequence: the last b with unit_prefix[b] <= pos
  __device__ __forceinline__ int32_t find(int32_t n_req, int32_t pos, int lane) const {
    int32_t cnt = 0;
    static_for<0, N>([&](auto kc) {
      constexpr int k = decltype(kc)::value;
      cnt += __popcll(__builtin_amdgcn_ballot_w64(64 * k + lane < n_req && unit_prefix[k] <= pos));
    });
    return cnt - 1;
  }
  __device__ __forceinline__ Req of(int32_t b) const {      // b: the same in all lanes
    return {get(len, b), get(tensor, b), get(unit_prefix, b), get(wave_first, b), get(n_part, b), get(part0, b)};
  }

 private:
  static __device__ __forceinline__ int32_t get(const int32_t (&field)[N], int32_t b) {
    int32_t v = field[0];
    // (values, not places, to choose from: a choice of places makes the compiler put the records into LDS and scratch memory)
    static_for<1, N>([&](auto kc) {
      const int32_t w = field[decltype(kc)::value];
      v = b >= 64 * decltype(kc)::value ? w : v;
    });
    return __builtin_amdgcn_readlane(v, b & 63);
  }
};

// what a wave (in blocks: a workgroup) handles: kv head g, wave w of that head, n_units steps of the head's
// sequence from step u_lo on, the first of which belongs to request b. A step is a unit (a tile in the
// kernel that walks tiles) or, where every wave gets one step, up to step_units units of one request
template <class Args>
struct Share { int32_t g, w, u_lo, n_units, b; typename Args::Req first; };

template <class Args>
__device__ __forceinline__ Share<Args> locate_share(const Args& a, const Records<Args>& records, int32_t index, int lane) {
  Share<Args> s;
  const int32_t W = a.waves_per_head, each = a.units_each, extra = a.units_extra;
  s.g = divide(index, a.by_waves);
  s.w = index - s.g * W;
  s.u_lo = s.w * each + min(s.w, extra);
  s.n_units = each + (s.w < extra ? 1 : 0);
  s.b = records.find(a.n_req, s.u_lo, lane);
  s.first = records.of(s.b);
  return s;
}

// Calls body(pool, workspace, plan, number of this workgroup in the plan): of a pair, with what belongs to this workgroup's half.
template <class Args, class Body>
__device__ __forceinline__ void in_launch(const PoolView& pv, float* ws, const Args& a, Body body) {
  if constexpr (std::is_same_v<Args, PairArgs>) {
    const bool second = blockIdx.x >= a.workgroups;
    PoolView mine = pv;
    mine.merged += second ? a.counters : 0u;
    body(mine, ws + (second ? a.floats : 0u), a.half[second ? 1 : 0], (int32_t)(blockIdx.x - (second ? a.workgroups : 0u)));
  } else {
    body(pv, ws, a, (int32_t)blockIdx.x);
  }
}

// which four dims of a head piece f of a partial result's row holds: rows keep the dims in the order in which the
// lanes of the kernel that wrote them store neighbouring pieces
template <int D>
__device__ __forceinline__ int32_t partial_dim(int32_t unit_tokens, int32_t f) {
  constexpr int LPR = D / 8, E = D / 16;
  return unit_tokens == TILE_TOKENS ? 8 * (f % LPR) + 4 * (f / LPR) : E * (4 * (f & 3) + f / E) + (f % E) / 4 * 4;
}

// ---------------------------------------------------------------------------------------------
// Requests that several waves share. The SHARE_WAVES waves of a workgroup (one per SIMD of a CU) walk neighbouring
// shares; a request that such a wave begins or ends in the middle of has its results of that wave put into LDS, and
// when all four are done the results of one request are added up there, the requests dealt out to the waves. What
// lies wholly inside the workgroup is finished by that. A request that reaches into other workgroups leaves one partial
// result in the workspace, written past the L2 of the XCD, and its workgroup counts itself in once it is there; the last
// to do so adds up all of them. Which one that is depends on who ends last, but the sum is taken in the order of the
// partials, so the result does not. Nobody waits for another workgroup, and the counter goes back to 0 by itself
// (an increment that wraps).
// This took the place of a combine launch behind every call, 4.6 us of which 3.4 are the launch: 8B-shaped step 2087 ->
// 2003 us, 8 requests of it, 4 layers 67.5 -> 63.7, 48 requests of 6 q heads each 52.2 -> 49.4, 64 of 16 heads of 64 68.2 ->
// 66.6, chunks of 16 tokens 36.9 -> 33.8. By single waves, without the sum in LDS, it was no faster than the pass: up to 29
// partials for one wave to add up, 6 us. A workgroup's chain behind its last wave is 2.2 to 3.3 us now (where the results go 0.6, LDS
// sum 0.3 and store 0.3, count 0.3, adding up 0.7 to 1.5).
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void store_partial(__amdgpu_buffer_rsrc_t rows, int32_t at, float4 v) {
  const words4_t w = {__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
  __builtin_amdgcn_raw_buffer_store_b128(w, rows, at, 0, CPOL_DEVICE);
}
__device__ __forceinline__ void store_partial(__amdgpu_buffer_rsrc_t pairs, int32_t at, float2 v) {
  __builtin_amdgcn_raw_buffer_store_b64(words2_t{__float_as_uint(v.x), __float_as_uint(v.y)}, pairs, at, 0, CPOL_DEVICE);
}
// this wave's stores have arrived where every XCD sees them
__device__ __forceinline__ void stores_done() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
  asm volatile("" ::: "memory");
}
// One more of n_part workgroups has its results in memory (asked by one lane): how many had before? `line`: of the counters,
// `k`: which in that line.
__device__ __forceinline__ uint32_t count_in(const PoolView& pv, int32_t line, int32_t k, int32_t n_part) {
  return atomicInc(pv.merged + (int64_t)line * MERGE_STRIDE + k, (uint32_t)n_part - 1u);
}

// sums of one 16-byte piece of a head's row over some partials: running maximum, normaliser, weighted sum
struct Sum { float M, L; float4 A; };
__device__ __forceinline__ void add(Sum& s, float L, const float4& v, float w) {
  s.L += L * w;
  s.A.x += v.x * w; s.A.y += v.y * w; s.A.z += v.z * w; s.A.w += v.w * w;
}
__device__ __forceinline__ void rescale(Sum& s, float M) {
  const float w = fast_exp2(s.M - M);
  s.M = M;
  s.L *= w;
  s.A.x *= w; s.A.y *= w; s.A.z *= w; s.A.w *= w;
}

// The same where the rows are means (sums divided by their L): the sum is one as well, so no weight of V's row is over 1 and nothing is
// out of range that V is not. A part of no weight at all (L of 0: every score -inf) has a row of zeros.
// (the reciprocal instruction, to 2^-23: weights are held to fewer bits, and L is never near the ends of a float's range)
__device__ __forceinline__ float share_of(float L) { return L == 0.f ? 0.f : __builtin_amdgcn_rcpf(L); }
template <int N>        // a power of two
__device__ __forceinline__ void add_means(Sum& s, float M, const float (&L)[N], const float4 (&v)[N], float (&w)[N]) {
  const float before = s.L * fast_exp2(s.M - M);
  float sums[N];                     // (pairs first: everything waits for it)
#pragma unroll
  for (int u = 0; u < N; u++) sums[u] = w[u] *= L[u];
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2)
#pragma unroll
    for (int u = 0; u < n; u++) sums[u] += sums[u + n];
  const float all = before + sums[0], share = share_of(all), keep = before * share;
  s.M = M;
  s.L = all;
  s.A.x *= keep; s.A.y *= keep; s.A.z *= keep; s.A.w *= keep;
#pragma unroll
  for (int u = 0; u < N; u++) {
    const float c = w[u] * share;
    s.A.x += v[u].x * c; s.A.y += v[u].y * c; s.A.z += v[u].z * c; s.A.w += v[u].w * c;
  }
}

// The partials of a request for n_heads q heads of kv head g from head g_first of the group on. Columns: the pieces of
// the heads' rows in order. MEANS: their rows are means.
template <int D, bool MEANS = false>
struct Partials {
  static constexpr int F = D / 4;
  __amdgpu_buffer_rsrc_t rows, pairs;
  int32_t group;
  // slot0: the first one's slot; ws_slots: all slots of the workspace
  __device__ __forceinline__ Partials(const float* ws, int32_t ws_slots, int64_t slot0, int32_t n_part, int32_t group, int32_t g_first,
                                      int32_t n_heads) : group(group) {
    const int64_t row0 = slot0 * group + g_first;
    const int32_t n_rows = (n_part - 1) * group + n_heads;
    rows = buffer_at(ws + row0 * D, n_rows * (D * 4));
    pairs = buffer_at(ws + (int64_t)ws_slots * group * D + row0 * WS_ML, n_rows * (WS_ML * 4));
  }
  // columns x, x + step, .. (KB of them) over partials j0 .. j1 - 1, FEW or MANY of them asked for at a time
  template <int KB, int FEW, int MANY>
  __device__ __forceinline__ void sum(Sum (&sums)[KB], int32_t x, int32_t step, int32_t j0, int32_t j1) const {
    asm volatile("" ::: "memory");     // nothing of this is read before the last one has counted itself in
#pragma unroll
    for (int k = 0; k < KB; k++) sums[k] = {NEG_BIG, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    auto some = [&](auto ahead) __attribute__((always_inline)) {
      constexpr int N = decltype(ahead)::value;
      words4_t v[KB][N];
      words2_t ml[KB][N];
#pragma unroll
      for (int u = 0; u < N; u++)
#pragma unroll
        for (int k = 0; k < KB; k++) {
          // (all of the offset lies in the lanes: it is what the buffer's range is compared with, while a part of it in a
          // scalar register is taken off the range first, of which rows past the last would leave less than nothing)
          const int32_t xk = x + k * step, row = (j0 + u) * group + xk / F;
          ml[k][u] = __builtin_amdgcn_raw_buffer_load_b64(pairs, row * (WS_ML * 4), 0, CPOL_DEVICE);
          v[k][u] = __builtin_amdgcn_raw_buffer_load_b128(rows, row * (D * 4) + xk % F * 16, 0, CPOL_DEVICE);
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < KB; k++) {
        float M = sums[k].M;
#pragma unroll
        for (int u = 0; u < N; u++) M = j0 + u < j1 ? fmaxf(M, __uint_as_float(ml[k][u].x)) : M;
        if constexpr (MEANS) {
          float L[N], w[N];
          float4 rows_of[N];
#pragma unroll
          for (int u = 0; u < N; u++) {
            const words4_t t = v[k][u];
            L[u] = __uint_as_float(ml[k][u].y);
            rows_of[u] = make_float4(__uint_as_float(t.x), __uint_as_float(t.y), __uint_as_float(t.z), __uint_as_float(t.w));
            w[u] = j0 + u < j1 ? fast_exp2(__uint_as_float(ml[k][u].x) - M) : 0.f;
          }
          add_means(sums[k], M, L, rows_of, w);
          continue;
        }
        rescale(sums[k], M);
#pragma unroll
        for (int u = 0; u < N; u++) {
          // (a row that is not there came back as zeros; a branch around each would make a chain of them)
          const words4_t t = v[k][u];
          add(sums[k], __uint_as_float(ml[k][u].y), make_float4(__uint_as_float(t.x), __uint_as_float(t.y), __uint_as_float(t.z), __uint_as_float(t.w)),
              j0 + u < j1 ? fast_exp2(__uint_as_float(ml[k][u].x) - M) : 0.f);
        }
      }
    };
    for (; j0 + FEW < j1; j0 += MANY) some(std::integral_constant<int, MANY>{});
    if (j0 < j1) some(std::integral_constant<int, FEW>{});
  }
};

// column x of request b's output: the four dims that piece x % (D / 4) of the rows holds, of head g_first + x / (D / 4)
template <int D, bool MEANS = false, class Args>
__device__ __forceinline__ void write_out(const PoolView& pv, uint16_t* __restrict__ out, const Args& a, int32_t b, int32_t g,
                                          int32_t g_first, int32_t x, const Sum& s) {
  constexpr int F = D / 4;
  // (no weight at all: 0 / 0, as the sums would have it)
  const float inv = MEANS ? s.L == 0.f ? __builtin_nanf("") : 1.f : 1.f / s.L;
  uint16_t* o = out + ((int64_t)(a.q_row0 + b) * pv.n_q_heads + g * pv.group + g_first + x / F) * D + partial_dim<D>(a.unit_tokens, x % F);
  *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(s.A.x * inv, s.A.y * inv), pack_bf16(s.A.z * inv, s.A.w * inv));
}

// Where a request's partial results are: the workgroups it reaches into, for kv head g, are numbered from 0 on
struct Parts { int32_t first, n; };    // workgroup of its first wave, how many
__device__ __forceinline__ Parts parts_of(int32_t wave_first, int32_t n_part, int32_t waves_per_head, int32_t g, int32_t wg_waves) {
  const int32_t w0 = g * waves_per_head + wave_first;
  if (wg_waves == 1) return {w0, n_part};     // a workgroup is one of the request's steps
  return {w0 / SHARE_WAVES, (w0 + n_part - 1) / SHARE_WAVES - w0 / SHARE_WAVES + 1};
}

// results of the workgroup's waves: slot 2 w of wave w's first request, 2 w + 1 of its last one, if it is another
template <int D, int HEADS>
struct Results {
  static constexpr int SLOTS = 2 * SHARE_WAVES, NONE = SLOTS;      // slot NONE: what takes part in a sum and adds nothing
  float4 rows[SLOTS + 1][HEADS][D / 4 + 1];    // (padded against bank conflicts)
  float2 ml[SLOTS + 1][HEADS];
  int32_t whose[SLOTS];      // request and kv head, -1: no result, or one that needs no other
  // by all waves, a slot in whose each, before their first results
  __device__ __forceinline__ void clear(int32_t wave, int32_t lane) {
    if (lane < 2) whose[2 * wave + lane] = -1;
    for (int32_t h = wave; h < HEADS; h += SHARE_WAVES) {
      if (lane < D / 4) rows[NONE][h][lane] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (lane == 0) ml[NONE][h] = make_float2(-INFINITY, 0.f);
    }
  }
};

// column x of a request's result of this workgroup becomes partial result `part` of the request
template <int D, class Args>
__device__ __forceinline__ void leave_partial(const PoolView& pv, float* ws, const Args& a, int32_t part, int32_t g, int32_t g_first,
                                              int32_t n_heads, int32_t x, const Sum& s) {
  constexpr int F = D / 4;
  const int64_t row0 = ((int64_t)g * a.parts_per_head + part) * pv.group + g_first;
  store_partial(buffer_at(ws + row0 * D, n_heads * (D * 4)), x * 16, s.A);
  if (x % F == 0)
    store_partial(buffer_at(ws + (int64_t)a.ws_slots * pv.group * D + row0 * WS_ML, n_heads * (WS_ML * 4)), x / F * (WS_ML * 4), make_float2(s.M, s.L));
}

// All waves of the workgroup have ended their shares. What follows is a chain of latencies with nothing beside it, so what
// it needs is in registers (`records`, the arguments) before the barrier, LDS is read without a branch, and the heads of a
// request are dealt out to the waves, in up to four pieces that are stored, counted in and added up each by itself: one
// request, four waves; two, two waves each; more, a wave each. (A piece is whole heads: their (m, l) pairs belong to it.) With one
// wave for a request and branches around the parts of each sum: 48 requests of 6 q heads each 49.95 -> 49.3 us, 64 of 16
// heads of 64 66.4 -> 65.7, chunks of 16 tokens 33.6 -> 33.3, the 8B-shaped step 1995 -> 1985.
// ONE, TWO: how many partial results a lane asks for at a time where it adds up one column, or two.
// MEANS: of what the rows are (Partials)
template <int D, int HEADS, int ONE = 16, int TWO = 8, bool MEANS = false, class Args>
__device__ __forceinline__ void end_shares(const PoolView& pv, float* ws_, uint16_t* __restrict__ out, const Args& a, const Records<Args>& records,
                                           const Results<D, HEADS>& res, int32_t g_first, int32_t n_heads, int32_t workgroup, int32_t wave, int32_t lane) {
  constexpr int F = D / 4, SLOTS = Results<D, HEADS>::SLOTS, NONE = Results<D, HEADS>::NONE;
  float* const ws = held(ws_);
  const int32_t waves_per_head = held(a.waves_per_head), parts_per_head = held(a.parts_per_head), ws_slots = held(a.ws_slots),
                merge_parts = held(a.merge_parts);
  __syncthreads();
  const int32_t whose = res.whose[lane % SLOTS];
  uint32_t left = (uint32_t)__builtin_amdgcn_ballot_w64(whose >= 0) & ((1u << SLOTS) - 1u);
  int32_t n_requests = 0;
  for (uint32_t l = left; l; n_requests++)
    l &= ~(uint32_t)__builtin_amdgcn_ballot_w64(whose == __builtin_amdgcn_readlane(whose, __builtin_ctz(l)));
  // pieces of 1, 2 or 4 heads; those that a wave has: piece p0 on, n_pieces of them
  const int32_t shift = n_heads <= 4 ? 0 : n_heads <= 8 ? 1 : 2, pieces = (n_heads + (1 << shift) - 1) >> shift;
  const int32_t each = n_requests == 1 ? 1 : n_requests == 2 ? 2 : 4, p0 = n_requests == 1 ? wave : n_requests == 2 ? wave & ~1 : 0;
  const int32_t n_pieces = min(each, pieces - p0), h0 = p0 << shift, h1 = min(n_heads, (p0 + each) << shift);
  if (n_pieces <= 0) return;
  for (int32_t nth = 0; left; nth++) {
    const int32_t id = __builtin_amdgcn_readlane(whose, __builtin_ctz(left));
    uint32_t mine = (uint32_t)__builtin_amdgcn_ballot_w64(whose == id) & ((1u << SLOTS) - 1u);      // the slots of one request
    left &= ~mine;
    if (n_requests == 2 ? nth != (wave & 1) : n_requests > 2 && nth % SHARE_WAVES != wave) continue;
    const int32_t b = id % MAX_LAUNCH_REQ, g = id / MAX_LAUNCH_REQ, group = held(pv.group);
    const typename Args::Req rq = records.of(b);
    const int32_t n = __builtin_popcount(mine);      // at most one slot of every wave
    int32_t slot[SHARE_WAVES];
#pragma unroll
    for (int i = 0; i < SHARE_WAVES; i++) {
      slot[i] = mine ? __builtin_ctz(mine) : NONE;
      mine &= mine - 1;
    }
    // (a request for the combine pass goes there also where no other workgroup has a part of it)
    const bool whole = n == rq.n_part && rq.n_part <= merge_parts;
    const Parts parts = parts_of(rq.wave_first, rq.n_part, waves_per_head, g, SHARE_WAVES);
    const int64_t slot0 = (int64_t)g * parts_per_head + rq.part0;
    const int64_t row0 = (slot0 + (workgroup - parts.first)) * group + g_first;
    // (stores past this wave's heads are dropped by the buffers' range)
    const auto rows = buffer_at(ws + row0 * D, h1 * (D * 4));
    const auto pairs = buffer_at(ws + (int64_t)ws_slots * group * D + row0 * WS_ML, h1 * (WS_ML * 4));
    for (int32_t x = h0 * F + lane; x - lane < h1 * F; x += 64) {
      const int32_t h = min(x / F, HEADS - 1), f = x % F;
      float2 ml[SHARE_WAVES];
      float4 v[SHARE_WAVES];
#pragma unroll
      for (int i = 0; i < SHARE_WAVES; i++) {
        ml[i] = res.ml[slot[i]][h];
        v[i] = res.rows[slot[i]][h][f];
      }
      Sum s = {ml[0].x, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
      for (int i = 1; i < SHARE_WAVES; i++) s.M = fmaxf(s.M, ml[i].x);
      if constexpr (MEANS) {
        float L[SHARE_WAVES], w[SHARE_WAVES];
#pragma unroll
        for (int i = 0; i < SHARE_WAVES; i++) {
          L[i] = ml[i].y;
          w[i] = fast_exp2(ml[i].x - s.M);
        }
        add_means(s, s.M, L, v, w);
      } else {
#pragma unroll
        for (int i = 0; i < SHARE_WAVES; i++) add(s, ml[i].y, v[i], fast_exp2(ml[i].x - s.M));
      }
      if (whole) {
        if (x < h1 * F) write_out<D, MEANS>(pv, out, a, b, g, g_first, x, s);
      } else {
        store_partial(rows, x * 16, s.A);
        if (f == 0) store_partial(pairs, x / F * (WS_ML * 4), make_float2(s.M, s.L));
      }
    }
    if (whole || rq.n_part > merge_parts) continue;
    stores_done();
    uint32_t before = 0;
    if (lane < n_pieces) before = count_in(pv, g * MAX_LAUNCH_REQ + b, p0 + lane, parts.n);
    const Partials<D, MEANS> all(ws, ws_slots, slot0, parts.n, held(pv.group), g_first, h1);
    // (all of a wave's pieces or none, as a rule)
    const uint32_t last = (uint32_t)__builtin_amdgcn_ballot_w64(lane < n_pieces && before == (uint32_t)parts.n - 1u);
    if (!last) continue;
    auto done = [&](int32_t x, const Sum& s) __attribute__((always_inline)) {
      if (x < h1 * F && (last >> ((x / F >> shift) - p0) & 1u)) write_out<D, MEANS>(pv, out, a, b, g, g_first, x, s);
    };
    const int32_t x = h0 * F + lane;
    if ((h1 - h0) * F <= 64) {
      Sum s[1];
      all.template sum<1, 4, ONE>(s, x, 0, 0, parts.n);
      done(x, s[0]);
    } else {
      for (int32_t at = x; at - lane < h1 * F; at += 128) {
        Sum s[2];
        all.template sum<2, 4, TWO>(s, at, 64, 0, parts.n);
        done(at, s[0]);
        done(at + 64, s[1]);
      }
    }
  }
}

// A launch by the kernel's address and the places of its arguments. The launch syntax copies every argument by value twice on
// the way to the same call and takes the launch's shape through thread-local storage: a decode call of one request 2.77 -> 2.52 us
// on the host, of four short ones 2.95 -> 2.70. ev0 / ev1 (either may be NULL): events that take the kernel's own start and end times (the runtime's extended
// launch attaches them to the kernel's dispatch, so no marker of its own goes into the stream and the time between them is the
// kernel's duration).
template <typename... P, typename... A>
static int launch(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t stream, hipEvent_t ev0, hipEvent_t ev1, const A&... a) {
  static_assert((std::is_same_v<std::remove_cv_t<P>, A> && ...), "the arguments are read as the kernel's own types");
  void* args[] = {const_cast<void*>(static_cast<const void*>(&a))...};
  const hipError_t e = ev0 || ev1 ? hipExtLaunchKernel((const void*)kernel, grid, dim3(threads), args, 0, stream, ev0, ev1, 0)
                                  : hipLaunchKernel((const void*)kernel, grid, dim3(threads), args, 0, stream);
  if (e != hipSuccess) (void)hipGetLastError();      // reported here, and not by the next one who asks
  return (int)e;
}
template <typename... P, typename... A>
static int launch(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t stream, const A&... a) {
  return launch(kernel, grid, threads, stream, (hipEvent_t) nullptr, (hipEvent_t) nullptr, a...);
}

}  // namespace ellm
