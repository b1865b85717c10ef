// HIP kernels for gfx950 that handle the tokens of a cache: quantised append, reading out, copying, compacting.
//
// All of them are bound by HBM (a few operations for every 16 bytes) and built alike: a workgroup has 16 KB of rows of one kv
// head (compacting: 64), asks for all of it at once, 16 bytes a lane and coalesced, and stores it where it belongs. Which rows those are is
// found in the launch's arguments, the chunks by one look at the table for each row.
#include "fp4.hpp"

namespace ellm {

// rows of a cache: bytes of a row and of its scales (0: bf16)
template <int D, bool FP4>
struct Rows {
  static constexpr int BYTES = FP4 ? FP4_ROW<D> : 2 * D, SCALES = FP4 ? FP4_SCALES<D> : 0, LPR = BYTES / 16;
  // (kv head h, plane p) in a chunk: its rows, its scales
  static __device__ __forceinline__ uint64_t rows_at(const PoolView& pv, int32_t h, int32_t p) {
    return (uint64_t)(h * 2 + p) * pv.tokens_per_chunk * BYTES;
  }
  static __device__ __forceinline__ uint64_t scales_at(const PoolView& pv, int32_t h, int32_t p) {
    return fp4_scales_at<D>(pv) + (uint64_t)(h * 2 + p) * pv.tokens_per_chunk * SCALES;
  }
};

// where a token's row is: chunk and row of the chunk, for a position of its own in every lane
struct RowAt { char* chunk; uint32_t row; };
template <bool DIRECT>
struct Tensor {
  char* base;                    // of the pool, or of the tensor's own range
  const int32_t* table;          // the tensor's row of it
  __device__ __forceinline__ Tensor(const PoolView& pv, int32_t tensor) {
    if (DIRECT) {
      base = reinterpret_cast<char*>(((const_u64_ptr)pv.vbase)[tensor]);
      table = nullptr;
    } else {
      base = pv.base;
      table = pv.table + (int64_t)tensor * pv.max_slots;
    }
  }
  __device__ __forceinline__ RowAt row(const PoolView& pv, int32_t pos) const {
    const int32_t slot = divide(pos, pv.by_chunk);
    const uint32_t chunk = DIRECT ? (uint32_t)slot : (uint32_t)table[slot];
    return {base + (uint64_t)chunk * pv.chunk_bytes, (uint32_t)(pos - slot * pv.tokens_per_chunk)};
  }
};

// the last i < n with first[i] <= x, in one round of loads: a search by halves, whose loads wait for each other, cost the appending of
// a token for 64 requests and its reading back 0.8 us each (3.9 -> 3.1)
__device__ __forceinline__ int32_t find_last(const int32_t* first, int32_t n, int32_t x) {
  const int lane = threadIdx.x & 63;
  static_assert(MAX_LAUNCH_REQ == 128, "two entries a lane");
  const int32_t f0 = first[lane], f1 = first[64 + lane];
  return __popcll(__builtin_amdgcn_ballot_w64(lane < n && f0 <= x)) + __popcll(__builtin_amdgcn_ballot_w64(64 + lane < n && f1 <= x)) - 1;
}

// A workgroup's tokens of the dense side: request b, positions p0 .. p1 - 1
struct TokenShare { int32_t b, p0, p1; };
__device__ __forceinline__ TokenShare token_share(const TokenArgs& a, int32_t block) {
  const int32_t b = find_last(a.block0, a.n_req, block);
  const TokenRange r = token_range(a.pos0[b], a.n[b], block - a.block0[b]);
  return {b, r.p0, r.p1};
}

// ---------------------------------------------------------------------------------------------
// Quantised append: rows of D bf16 become codes and scales (fp4.hpp). 16 (heads of 64: 8) lanes have a row, 8 dims each; a
// block's maximum is that of 4 lanes next to each other, each of which makes a word of codes, and one the scale.
// Prompts of 93600 tokens, 8 kv heads of 128: 89 us (5.4 TB/s read and written). With the heads of a token in neighbouring workgroups 95, with
// several heads for a workgroup one after the other, the next one's rows on their way, 84 to 98 by their number and no gain for reading.
// ---------------------------------------------------------------------------------------------
template <int D, bool DIRECT>
__global__ __launch_bounds__(256) void fp4_append_kernel(PoolView pv, const char* __restrict__ k_new, const char* __restrict__ v_new, TokenArgs a) {
  using R = Rows<D, true>;
  constexpr int LPR = D / 8, N = 2 * TOKEN_BLOCK * LPR / 256;     // lanes of a row; rows that a lane has a piece of
  const TokenShare s = token_share(a, blockIdx.x);
  const int32_t h = blockIdx.y, rows = s.p1 - s.p0, sub = threadIdx.x % LPR;
  const Tensor<DIRECT> t(pv, a.tensor[s.b]);
  const int64_t from = ((int64_t)(a.row0[s.b] + (s.p0 - a.pos0[s.b])) * pv.n_kv_heads + h) * (2 * D) + sub * 16;
  const int64_t token_bytes = (int64_t)pv.n_kv_heads * (2 * D);
  uint4 x[N];
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int32_t r = threadIdx.x / LPR + i * (256 / LPR), plane = r / TOKEN_BLOCK, k = r % TOKEN_BLOCK;
    x[i] = make_uint4(0, 0, 0, 0);
    if (k < rows) x[i] = load_stream16((plane ? v_new : k_new) + from + k * token_bytes);
  }
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int32_t r = threadIdx.x / LPR + i * (256 / LPR), plane = r / TOKEN_BLOCK, k = r % TOKEN_BLOCK;
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    const uint32_t top = max_magnitudes_xor2(max_magnitudes_xor1(max_magnitudes(max_magnitudes(w[0], w[1]), max_magnitudes(w[2], w[3]))));
    const uint32_t scale = fp4_scale(top), codes = fp4_codes(w, scale);
    if (k < rows) {
      const RowAt at = t.row(pv, s.p0 + k);
      *reinterpret_cast<uint32_t*>(at.chunk + R::rows_at(pv, h, plane) + at.row * R::BYTES + sub * 4) = codes;
      if (sub % 4 == 0) *reinterpret_cast<uint8_t*>(at.chunk + R::scales_at(pv, h, plane) + at.row * R::SCALES + sub / 4) = (uint8_t)scale;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Reading out: rows of a cache become dense rows [token][kv head][D] of bf16; 4-bit values are bf16 values exactly. The same
// prompts: 68 us (7.1 TB/s read and written).
// ---------------------------------------------------------------------------------------------
template <int D, bool FP4, bool DIRECT>
__global__ __launch_bounds__(256) void read_tokens_kernel(PoolView pv, char* __restrict__ k_out, char* __restrict__ v_out, TokenArgs a) {
  using R = Rows<D, FP4>;
  constexpr int LPR = D / 8, N = 2 * TOKEN_BLOCK * LPR / 256;
  const TokenShare s = token_share(a, blockIdx.x);
  const int32_t h = blockIdx.y, rows = s.p1 - s.p0, sub = threadIdx.x % LPR;
  const Tensor<DIRECT> t(pv, a.tensor[s.b]);
  const int64_t to = ((int64_t)(a.row0[s.b] + (s.p0 - a.pos0[s.b])) * pv.n_kv_heads + h) * (2 * D) + sub * 16;
  const int64_t token_bytes = (int64_t)pv.n_kv_heads * (2 * D);
  uint4 x[N];
  uint32_t codes[N], scale[N];
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int32_t r = threadIdx.x / LPR + i * (256 / LPR), plane = r / TOKEN_BLOCK, k = r % TOKEN_BLOCK;
    if (k >= rows) continue;
    const RowAt at = t.row(pv, s.p0 + k);
    const char* row = at.chunk + R::rows_at(pv, h, plane) + at.row * R::BYTES;
    if constexpr (FP4) {
      codes[i] = *reinterpret_cast<const uint32_t*>(row + sub * 4);
      scale[i] = *reinterpret_cast<const uint8_t*>(at.chunk + R::scales_at(pv, h, plane) + at.row * R::SCALES + sub / 4);
    } else {
      x[i] = load_stream16(row + sub * 16);
    }
  }
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int32_t r = threadIdx.x / LPR + i * (256 / LPR), plane = r / TOKEN_BLOCK, k = r % TOKEN_BLOCK;
    if (k >= rows) continue;
    if constexpr (FP4) {
      const words4_t v = fp4_values(codes[i], fp4_scale_float(scale[i]));
      x[i] = make_uint4(v.x, v.y, v.z, v.w);
    }
    store_stream16((plane ? v_out : k_out) + to + k * token_bytes, x[i]);
  }
}

// ---------------------------------------------------------------------------------------------
// Copying: a group's rows are read once and go to all of its destinations, one after the other. A few workgroups would take long
// over many destinations (each waits for the table): up to COPY_WORKGROUPS in all, the destinations are split among several, which
// read the same rows. us of the kernel: 247 tokens of 4-bit rows, 8 kv heads of 128, to 8 tensors (24 workgroups) 10.2, two parts 6.9, four
// 5.5, eight 4.8; four of 2000 to 8192 bf16 tokens to 4 tensors each (2500) 100, 110 in two parts.
// Rows are read without a streaming hint: they are the source's, which is read again. That call, sources in the last-level cache
// 99 us with the hint and 80 without, otherwise 100 and 95 (5.3 TB/s); stores without it 103, blocks of 32 KB 99.
// ---------------------------------------------------------------------------------------------
constexpr int COPY_WORKGROUPS = 1024;
template <int D, bool FP4> constexpr int COPY_TOKENS = COPY_BYTES / (2 * Rows<D, FP4>::BYTES);

template <int D, bool FP4, bool DIRECT>
__global__ __launch_bounds__(256) void copy_tokens_kernel(PoolView pv, CopyTokenArgs a) {
  using R = Rows<D, FP4>;
  constexpr int TOKENS = COPY_TOKENS<D, FP4>, N = COPY_BYTES / (16 * 256);
  const int32_t g = find_last(a.block0, a.n_groups, blockIdx.x), h = blockIdx.y, sub = threadIdx.x % R::LPR;
  const int32_t k0 = (blockIdx.x - a.block0[g]) * TOKENS, rows = min(TOKENS, a.n[g] - k0);
  const Tensor<DIRECT> from(pv, a.src[g]);
  auto plane_of = [&](int i) __attribute__((always_inline)) { return (int32_t)(threadIdx.x / R::LPR + i * (256 / R::LPR)) / TOKENS; };
  auto token_of = [&](int i) __attribute__((always_inline)) { return (int32_t)(threadIdx.x / R::LPR + i * (256 / R::LPR)) % TOKENS; };
  uint4 x[N];
#pragma unroll
  for (int i = 0; i < N; i++) {
    if (token_of(i) >= rows) continue;
    const RowAt at = from.row(pv, a.first[g] + k0 + token_of(i));
    x[i] = *reinterpret_cast<const uint4*>(at.chunk + R::rows_at(pv, h, plane_of(i)) + at.row * R::BYTES + sub * 16);
  }
  // the scales of a row by one lane: TOKENS rows of either plane are 256 lanes (heads of 64: two rounds)
  constexpr int NS = FP4 ? 2 * TOKENS / 256 : 1;
  using scales_t = std::conditional_t<R::SCALES == 4, uint32_t, uint16_t>;
  scales_t scales[NS];
  if constexpr (FP4) {
#pragma unroll
    for (int i = 0; i < NS; i++) {
      const int32_t r = threadIdx.x + i * 256, k = r % TOKENS;
      if (k >= rows) continue;
      const RowAt at = from.row(pv, a.first[g] + k0 + k);
      scales[i] = *reinterpret_cast<const scales_t*>(at.chunk + R::scales_at(pv, h, r / TOKENS) + at.row * R::SCALES);
    }
  }
  for (int32_t d = a.dst0[g] + (int32_t)blockIdx.z; d < a.dst0[g + 1]; d += (int32_t)gridDim.z) {
    const Tensor<DIRECT> to(pv, a.dst[d]);
    const int32_t pos = a.pos[d] + k0;
#pragma unroll
    for (int i = 0; i < N; i++) {
      if (token_of(i) >= rows) continue;
      const RowAt at = to.row(pv, pos + token_of(i));
      store_stream16(at.chunk + R::rows_at(pv, h, plane_of(i)) + at.row * R::BYTES + sub * 16, x[i]);
    }
    if constexpr (FP4) {
#pragma unroll
      for (int i = 0; i < NS; i++) {
        const int32_t r = threadIdx.x + i * 256, k = r % TOKENS;
        if (k >= rows) continue;
        const RowAt at = to.row(pv, pos + k);
        *reinterpret_cast<scales_t*>(at.chunk + R::scales_at(pv, h, r / TOKENS) + at.row * R::SCALES) = scales[i];
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Compacting, in place. The moved rows of a (request, kv head, plane), a chain, are cut into segments of STEP rows, which a
// workgroup holds in registers: it reads them where they are, and stores them where they go. Positions ascend, so what a
// segment stores may only be what itself and segments before it read: a segment's stores wait until those before it that
// read so far down have what they read in registers, which they say with a flag each, and wait for nothing else.
// The segments of a chain are numbered in the order in which their workgroups begin (a counter for each chain), so whoever is
// waited for is running already and does not wait itself: the launch comes to its end whatever order workgroups are started in.
// A position is held between its target and the tensor's last token: whatever the list holds, no row outside the tensor's tokens
// is touched.
//
// Chains of one segment need no flags and no counters. Where there is no room for flags (ONE_BY_ONE) a workgroup takes the segments
// of its chain one after the other. us a call that way / with flags: 8 requests of 4096 to 16384 bf16 tokens, four fifths of them kept, 8
// kv heads of 128 (240 MB read and as much written, 77 at a copy's rate) 446 / 106, one of 32768, half of them kept 587 / 37, in 4 bits 151 / 18.
// A segment of 16 KB and 256 threads 159, 54, 20, of 32 and 512 125, 42, 19, of 64 and 1024 (taken) 106, 37, 18, of 128 and 1024 103, 30, 23;
// 64 requests of 500 to 4000 4-bit tokens 72, 67, 69, 73. Without the streaming hints on loads and stores 152, 58, 28.
// ---------------------------------------------------------------------------------------------
template <int D, bool FP4> constexpr int COMPACT_ROWS = COMPACT_BYTES / Rows<D, FP4>::BYTES;
constexpr int COMPACT_THREADS = 1024;
// A wait takes microseconds. It ends all the same (after some seconds) where something else has written over the flags, which calls in order
// do not: the segment then stores nothing, since the rows that it would store over may not have been read yet, and says so to the host. So
// does a workgroup whose number is none of a segment.
template <int D, bool FP4, bool DIRECT, bool ONE_BY_ONE>
__global__ __launch_bounds__(COMPACT_THREADS) void compact_kernel(PoolView pv, const int32_t* __restrict__ keep, uint32_t* __restrict__ marks, CompactArgs a) {
  using R = Rows<D, FP4>;
  constexpr int STEP = COMPACT_ROWS<D, FP4>, N = COMPACT_BYTES / (16 * COMPACT_THREADS), RPT = COMPACT_THREADS / R::LPR;     // rows of all threads at a time
  constexpr int NS = FP4 ? (STEP + COMPACT_THREADS - 1) / COMPACT_THREADS : 1;
  using scales_t = std::conditional_t<R::SCALES == 4, uint32_t, uint16_t>;
  const int32_t b = ONE_BY_ONE ? blockIdx.x : find_last(a.segment0, a.n_req, blockIdx.x);
  const int32_t h = blockIdx.y >> 1, plane = blockIdx.y & 1, sub = threadIdx.x % R::LPR;
  const Tensor<DIRECT> t(pv, a.tensor[b]);
  const int32_t n = a.n[b], first = a.first[b], last = a.len[b] - 1, segments = (n + STEP - 1) / STEP;
  const int32_t* list = keep + a.key0[b];
  auto source = [&](int32_t i) __attribute__((always_inline)) { return max(first + i, min(list[i], last)); };

  auto gives_up = [&]() __attribute__((always_inline)) {
    if (threadIdx.x == 0) __hip_atomic_store(a.gave_up, (uint32_t)a.tensor[b] + 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  };
  __shared__ int32_t number;
  uint32_t* const flags = marks + gridDim.y * a.n_req * MERGE_STRIDE + (ONE_BY_ONE ? 0 : gridDim.y * a.segment0[b] + blockIdx.y * segments);
  int32_t seg = 0;
  if (!ONE_BY_ONE && segments > 1) {
    if (threadIdx.x == 0) number = (int32_t)atomicAdd(marks + (gridDim.y * b + blockIdx.y) * MERGE_STRIDE, 1u);
    __syncthreads();
    seg = number;
    if ((uint32_t)seg >= (uint32_t)segments) return gives_up();
  }
  do {
    const int32_t i0 = seg * STEP;
    uint4 x[N];
    scales_t scales[NS];
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int32_t i = i0 + threadIdx.x / R::LPR + j * RPT;
      if (i >= n) continue;
      const RowAt at = t.row(pv, source(i));
      x[j] = load_stream16(at.chunk + R::rows_at(pv, h, plane) + at.row * R::BYTES + sub * 16);
    }
    if constexpr (FP4) {
#pragma unroll
      for (int j = 0; j < NS; j++) {
        const int32_t i = i0 + threadIdx.x + j * COMPACT_THREADS;
        if (i >= n || threadIdx.x + j * COMPACT_THREADS >= STEP) continue;
        const RowAt at = t.row(pv, source(i));
        scales[j] = *reinterpret_cast<const scales_t*>(at.chunk + R::scales_at(pv, h, plane) + at.row * R::SCALES);
      }
    }
    stores_done();               // (and loads: all that this wave has asked for is here)
    __syncthreads();
    if (!ONE_BY_ONE && segments > 1) {
      if (threadIdx.x == 0) __hip_atomic_store(flags + seg, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // the segments before this one that read as far as this one stores
      for (int32_t j = threadIdx.x; j < seg; j += COMPACT_THREADS)
        if (source((j + 1) * STEP - 1) >= first + i0) {
          bool seen = false;
          for (int32_t look = 0; look < a.looks && !seen; look++) {
            seen = __hip_atomic_load(flags + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != 0;
            if (!seen) __builtin_amdgcn_s_sleep(1);
          }
          if (!seen) number = -1;            // (all have read it, two barriers ago)
        }
      __syncthreads();
      if (number < 0) return gives_up();
    }
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int32_t i = i0 + threadIdx.x / R::LPR + j * RPT;
      if (i >= n) continue;
      const RowAt at = t.row(pv, first + i);
      store_stream16(at.chunk + R::rows_at(pv, h, plane) + at.row * R::BYTES + sub * 16, x[j]);
    }
    if constexpr (FP4) {
#pragma unroll
      for (int j = 0; j < NS; j++) {
        const int32_t i = i0 + threadIdx.x + j * COMPACT_THREADS;
        if (i >= n || threadIdx.x + j * COMPACT_THREADS >= STEP) continue;
        const RowAt at = t.row(pv, first + i);
        *reinterpret_cast<scales_t*>(at.chunk + R::scales_at(pv, h, plane) + at.row * R::SCALES) = scales[j];
      }
    }
    seg++;
  } while (ONE_BY_ONE && seg < segments);
}

// ---------------------------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------------------------
// calls go(head size, rows in 4 bits, direct) with constants
template <class Go>
static int of_pool(const PoolView& pv, bool fp4, Go go) {
  auto addressed = [&](auto dim, auto four) {
    return pv.vbase ? go(dim, four, std::true_type{}) : go(dim, four, std::false_type{});
  };
  auto sized = [&](auto dim) { return fp4 ? addressed(dim, std::true_type{}) : addressed(dim, std::false_type{}); };
  return pv.head_dim == 128 ? sized(std::integral_constant<int, 128>{}) : sized(std::integral_constant<int, 64>{});
}

int launch_fp4_append(const PoolView& pv, const void* k_new, const void* v_new, const TokenArgs& a, hipStream_t stream) {
  if (a.blocks <= 0) return 0;
  return of_pool(pv, true, [&](auto dim, auto, auto direct) {
    return launch(fp4_append_kernel<dim(), direct()>, dim3((unsigned)a.blocks, pv.n_kv_heads), 256, stream, pv, (const char*)k_new, (const char*)v_new, a);
  });
}

int launch_read_tokens(const PoolView& pv, bool fp4, void* k_out, void* v_out, const TokenArgs& a, hipStream_t stream) {
  if (a.blocks <= 0) return 0;
  return of_pool(pv, fp4, [&](auto dim, auto four, auto direct) {
    return launch(read_tokens_kernel<dim(), four(), direct()>, dim3((unsigned)a.blocks, pv.n_kv_heads), 256, stream, pv, (char*)k_out, (char*)v_out, a);
  });
}

int copy_tokens_per_block(int head_dim, bool fp4) {
  return head_dim == 128 ? (fp4 ? COPY_TOKENS<128, true> : COPY_TOKENS<128, false>) : fp4 ? COPY_TOKENS<64, true> : COPY_TOKENS<64, false>;
}

int launch_copy_tokens(const PoolView& pv, bool fp4, const CopyTokenArgs& a, hipStream_t stream) {
  if (a.blocks <= 0) return 0;
  int32_t most = 1;
  for (int32_t g = 0; g < a.n_groups; g++) most = std::max(most, a.dst0[g + 1] - a.dst0[g]);
  const int32_t parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(most, COPY_WORKGROUPS / ((int64_t)a.blocks * pv.n_kv_heads)));
  return of_pool(pv, fp4, [&](auto dim, auto four, auto direct) {
    return launch(copy_tokens_kernel<dim(), four(), direct()>, dim3((unsigned)a.blocks, pv.n_kv_heads, parts), 256, stream, pv, a);
  });
}

int compact_rows_per_segment(int head_dim, bool fp4) {
  return head_dim == 128 ? (fp4 ? COMPACT_ROWS<128, true> : COMPACT_ROWS<128, false>) : fp4 ? COMPACT_ROWS<64, true> : COMPACT_ROWS<64, false>;
}

int launch_compact(const PoolView& pv, bool fp4, const int32_t* keep, uint32_t* marks, size_t n_marks, const CompactArgs& a, hipStream_t stream) {
  if (a.n_req <= 0) return 0;
  const unsigned chains = 2 * pv.n_kv_heads;
  const size_t need = compact_marks(a, chains);
  const bool flagged = a.segments > a.n_req;       // (some chain has several segments)
  const bool one_by_one = flagged && need > n_marks;
  if (flagged && !one_by_one) {
    const int e = launch_fill(marks, 0, need, stream);
    if (e) return e;
  }
  return of_pool(pv, fp4, [&](auto dim, auto four, auto direct) {
    auto go = [&](auto kernel, int blocks) { return launch(kernel, dim3((unsigned)blocks, chains), COMPACT_THREADS, stream, pv, keep, marks, a); };
    if (one_by_one) return go(compact_kernel<dim(), four(), direct(), true>, a.n_req);
    return go(compact_kernel<dim(), four(), direct(), false>, a.segments);
  });
}

}  // namespace ellm
