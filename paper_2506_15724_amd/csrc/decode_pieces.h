// What the decode kernels share: the arguments of a launch, where a head's rows live, how a head is cut into pieces and how
// the pieces of a head meet (decode.hip says what that costs).
#pragma once
#include "common.h"

#include <type_traits>

namespace madakv {

constexpr float DNEG_BIG = -1.0e30f;
constexpr int DEC_THREADS = 256;
typedef __attribute__((ext_vector_type(4))) unsigned int du32x4_t;
typedef __attribute__((ext_vector_type(2))) unsigned int du32x2_t;
typedef __attribute__((ext_vector_type(8))) __bf16 dbf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 dbf16x2_t;
typedef __attribute__((ext_vector_type(4))) float df32x4_t;
typedef __attribute__((ext_vector_type(2))) float df32x2_t;
typedef __attribute__((ext_vector_type(4))) short ds16x4_t;

struct DecodeArgs {
  const void* q; const void* k_new; const void* v_new; void* k_c; void* v_c;
  const int64_t* kv_off; int32_t* kv_len; void* out;
  int B, H, G, chunk_rows, out_fp32, has_new;
  int max_chunks;       // most pieces a head is cut into (head_chunk_rows)
  int max_new;          // rows a segment has room for behind those of the eviction
  float* part;          // [heads][slots][G][d] partial results of the pieces of the call's heads
  float* part_ml;       // [heads][slots][G][2] their (max, sum)
  int slots;            // most pieces of a head
  uint32_t by_heads;    // ceil(2^32 / heads), likewise, where heads * (heads + pieces) < 2^32
  uint32_t by_chunk;    // ceil(2^32 / chunk_rows): quotients of numbers below 2^21, 0 where a head may be longer (see pieces_of)
  Meet meet;            // how they meet
  long long capacity;   // rows in k_c / v_c
  // paged cache (page_rows > 0): see struct Paging
  int page_rows, page_shift, tbl_entries;
  int32_t* page_tbl; unsigned long long* pool_top;
  long long region_pages;      // pages in one batch item's region
  long long head0;             // index of the call's first head in the whole model (layer0 * B * H)
  float scale_log2;
  // kernels that leave the weights (WEIGHTS) only:
  const int32_t* slot;         // the row of every head that the new one replaces; null: it is appended, or there is none
  float* logits;               // [heads][G][logit_rows] scale * log2(e) * q . k of every row
  float* head_ml;              // [heads][G][2] their maximum and the sum of 2^(logit - maximum) over the head
  int32_t* fresh;              // [heads] the row that was new in this call, -1: none
  int logit_rows;
};

// The new row of a head: its place among the rows, and whether the head has one.  It is appended (its place is the first one
// past the rows so far), or takes the place a.slot names, where that is one of the head's rows.
struct Fresh { int row; bool there; };
template <bool WEIGHTS>
__device__ __forceinline__ Fresh fresh_row(const DecodeArgs& a, long long hidx, int len_old, bool can_append) {
  if (WEIGHTS && a.slot) {
    const int s = a.slot[hidx];
    return Fresh{s, s >= 0 && s < len_old};
  }
  return Fresh{len_old, can_append};
}

// 16 bytes that are read once per launch (cache rows): a non-temporal load, so that the stream
// does not push anything useful out of the caches.  Measured: 10-15% off the decode step.
typedef __attribute__((ext_vector_type(4))) unsigned int stream_u32x4_t;
__device__ __forceinline__ uint4 stream_load16(const void* p) {
  const stream_u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const stream_u32x4_t*>(p));
  return make_uint4(v[0], v[1], v[2], v[3]);
}

template <int LPR> __device__ __forceinline__ float row_sum(float x);
template <> __device__ __forceinline__ float row_sum<16>(float x) { return row16_sum(x); }
template <> __device__ __forceinline__ float row_sum<8>(float x) {
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, true));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, true));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x141, 0xF, 0xF, true));
  return x;
}
template <> __device__ __forceinline__ float row_sum<4>(float x) {
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, true));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, true));
  return x;
}
template <> __device__ __forceinline__ float row_sum<32>(float x) {
  x = row16_sum(x);
  return x + __shfl_xor(x, 16, 64);
}

template <typename T> struct Elems;
template <> struct Elems<uint16_t> {
  static constexpr int EPL = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float* f) {
    f[0] = bf16_lo(r.x); f[1] = bf16_hi(r.x); f[2] = bf16_lo(r.y); f[3] = bf16_hi(r.y);
    f[4] = bf16_lo(r.z); f[5] = bf16_hi(r.z); f[6] = bf16_lo(r.w); f[7] = bf16_hi(r.w);
  }
};
template <> struct Elems<uint8_t> {                  // E4M3 bytes of the 8-bit reduced cache
  static constexpr int EPL = 16;
  static __device__ __forceinline__ void unpack(const uint4& r, float* f) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {                     // the hardware conversion is exact (every code is a float)
      const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
      const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
      f[i * 4] = lo[0]; f[i * 4 + 1] = lo[1]; f[i * 4 + 2] = hi[0]; f[i * 4 + 3] = hi[1];
    }
  }
};
template <> struct Elems<float> {
  static constexpr int EPL = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float* f) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
  }
};

// EPL consecutive elements of the caller's type T (Q, k_new, v_new) as floats
template <typename T, int EPL>
__device__ __forceinline__ void load_floats(const T* p, float* f) {
  constexpr int PER = 16 / sizeof(T);                 // elements per 16-byte load
#pragma unroll
  for (int j = 0; j < EPL / PER; ++j) Elems<T>::unpack(*reinterpret_cast<const uint4*>(p + j * PER), f + j * PER);
}

// ---- where row r of a head lives ---------------------------------------------------------
// Contiguous segments: at off + r.  Paged cache: the first init_rows rows (the head's initial pages,
// which follow each other) likewise; later rows in pages listed in the head's table.  `fresh`
// is the page this workgroup has just taken for the row being appended, if it had to take one
// (the table entry it wrote is not yet visible to its other threads).
struct RowMap {
  long long off;
  int init_rows;               // INT_MAX without paging
  const int32_t* tbl;          // the head's table (entries 1.. = pages taken later)
  int shift, fresh_slot;
  long long fresh_page;
  __device__ __forceinline__ long long operator()(int r) const {
    if (r < init_rows) return off + r;
    const int q = r - init_rows, j = q >> shift;
    const long long pg = (j == fresh_slot) ? fresh_page : (long long)tbl[1 + j];
    return (pg << shift) + (q & ((1 << shift) - 1));
  }
};

template <bool PAGED>
__device__ __forceinline__ bool can_append_to(const DecodeArgs& a, long long off, int len_old) {
  // an empty segment (its budgets did not fit the cache) stays empty; contiguous segments also end at the cache's end
  return a.has_new && len_old > 0 && (PAGED || off + len_old < a.capacity);
}

// All threads of the workgroup.  rows [r_begin, r_end) are the workgroup's; when the appended row is
// among them and starts a new page, thread 0 takes the next page from the top of the batch item's region.
template <bool PAGED>
__device__ __forceinline__ RowMap make_row_map(const DecodeArgs& a, long long hidx, long long off, int len_old, bool can_append,
                                               int r_begin, int r_end) {
  RowMap m;
  m.off = off; m.init_rows = 0x7fffffff; m.tbl = nullptr; m.shift = 0; m.fresh_slot = -1; m.fresh_page = 0;
  if (!PAGED) return m;
  __shared__ long long s_fresh;
  int32_t* tbl = a.page_tbl + (a.head0 + hidx) * a.tbl_entries;
  m.tbl = tbl; m.shift = a.page_shift;
  m.init_rows = tbl[0] << a.page_shift;
  const int q = len_old - m.init_rows;
  const bool takes = can_append && len_old >= r_begin && len_old < r_end && q >= 0 && (q & (a.page_rows - 1)) == 0;   // uniform
  if (takes) {
    if (threadIdx.x == 0) {
      const long long b = ((a.head0 + hidx) / a.H) % a.B;
      const unsigned long long nth = atomicAdd(a.pool_top + b, 1ULL);
      const long long page = (b + 1) * a.region_pages - 1 - (long long)nth;
      tbl[1 + (q >> a.page_shift)] = (int32_t)page;
      s_fresh = page;
    }
    __syncthreads();
    m.fresh_slot = q >> a.page_shift;
    m.fresh_page = s_fresh;
  }
  return m;
}

// the 4-bit cache (decode4.hip)
hipError_t launch_decode4(const Dims& dm, const DecodeArgs& a, int grid_chunks, bool weights, hipStream_t st);

// Rows per piece of a head of `len` rows: a.chunk_rows, or for a head that would need more than max_chunks pieces a
// larger multiple of 32.  The grid then depends on the budget alone and not on the longest head a layer may have.  The
// host learns that length only once the eviction has run; sizing the grid for the whole context until then put 65
// instead of 17 workgroups per head in the grid (16K context, budget 2048), 5 of 36 us per layer call for
// workgroups that found nothing to do.
__device__ __forceinline__ int head_chunk_rows(const DecodeArgs& a, int len) {
  if (len <= a.chunk_rows * a.max_chunks) return a.chunk_rows;
  return ((len + a.max_chunks - 1) / a.max_chunks + 31) / 32 * 32;
}

// ceil(len / chunk_rows).  As a product: len + chunk_rows - 1 < 2^21 and chunk_rows <= 2^10, so what by_chunk is too large by
// (below chunk_rows / 2^32) stays below 1 in units of the next quotient.
__device__ __forceinline__ int pieces_of(const DecodeArgs& a, int len) {
  const uint32_t x = (uint32_t)(len + a.chunk_rows - 1);
  return a.by_chunk ? (int)__umulhi(x, a.by_chunk) : (int)(x / (uint32_t)a.chunk_rows);
}

// The head a workgroup works on.  Workgroups go to the 8 XCDs in turn; with the head as the fast grid dimension all
// pieces of a head would meet on one XCD (128 heads), and XCDs with long heads would finish last: the pieces of a head
// are rotated over the XCDs instead.
__device__ __forceinline__ int piece_head(const DecodeArgs& a) {
  const uint32_t x = blockIdx.x + blockIdx.y;
  if (x < gridDim.x) return (int)x;
  return (int)(x - (a.by_heads ? __umulhi(x, a.by_heads) : x / gridDim.x) * gridDim.x);
}

// The appended row of the 8-bit cache, encoded: written to the cache (Eq. 4) and left in LDS, K then V, for the tile it
// belongs to.  All threads; `row` is its place in the cache.  (Kept out of the load path of the tiles: the encoding,
// unrolled there, had made 48 KB of the grouped-query kernel, and by the wave of the tile, in its loop, it costs a single
// query head's calls 2%.)
template <int D>
__device__ __forceinline__ void stage_new_row(const DecodeArgs& a, long long hidx, long long row, uint8_t* s_new) {
  for (int e = threadIdx.x; e < 2 * D; e += (int)blockDim.x) {
    const bool is_k = e < D;
    const int c = is_k ? e : e - D;
    const uint8_t y = (uint8_t)f32_to_e4m3(bf16_bits_to_f32((reinterpret_cast<const uint16_t*>(is_k ? a.k_new : a.v_new))[hidx * D + c]));
    (reinterpret_cast<uint8_t*>(is_k ? a.k_c : a.v_c))[row * D + c] = y;
    s_new[e] = y;
  }
  __syncthreads();
}

// ---- the end of a piece ------------------------------------------------------------------------
// exp2 of something <= 0, a weight beside one of 1: the instruction itself (the library call spends seven more on keeping
// denormal results)
__device__ __forceinline__ float weight_of(float x) { return __builtin_amdgcn_exp2f(x); }

// The two values of lanes that are O apart (O = 4 ... 32: within a row by rotation, across rows by a swap of rows): the same
// pair in both lanes up to its order.  (Rotated by 4, lane i is paired with lane i - 4 and that one with i - 8: only the merge over 8
// that follows brings the four of a row together in every lane.)
template <int O>
__device__ __forceinline__ void lane_pair(float x, float& p, float& q) {
  const uint32_t u = __float_as_uint(x);
  if constexpr (O == 32) { const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false); p = __uint_as_float(r[0]); q = __uint_as_float(r[1]); }
  else if constexpr (O == 16) { const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false); p = __uint_as_float(r[0]); q = __uint_as_float(r[1]); }
  else { p = x; q = __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x120 + O, 0xF, 0xF, true)); }       // row_ror
}
// (max, sum, acc) of the lanes LPR, 2 LPR, ... apart merged, the result in all of them
template <int O, int N>
__device__ __forceinline__ void merge_lanes(float& m, float& l, float (&acc)[N]) {
  if constexpr (O < 64) {
    float m1, m2, l1, l2;
    lane_pair<O>(m, m1, m2);
    lane_pair<O>(l, l1, l2);
    m = fmaxf(m1, m2);
    const float c1 = weight_of(m1 - m), c2 = weight_of(m2 - m);
    l = l1 * c1 + l2 * c2;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float a1, a2;
      lane_pair<O>(acc[e], a1, a2);
      acc[e] = a1 * c1 + a2 * c2;
    }
    merge_lanes<O * 2, N>(m, l, acc);
  }
}

// Workgroups of the grid that arrive at a head's counters: those whose piece may exist before the next eviction.  It follows
// from what only an eviction changes (len1: 1 + the rows it left; 0: this handle has not seen one) and not from the head's length,
// which the last one to arrive has replaced by the time a workgroup further back in the grid starts.
__device__ __forceinline__ int arrivals(const DecodeArgs& a, int len1) {
  if (len1 == 0) return (int)gridDim.y;
  return max(1, min((int)gridDim.y, pieces_of(a, len1 - 1 + a.max_new)));
}
// four neighbouring elements of the output
template <typename T>
__device__ __forceinline__ void store_out4(const DecodeArgs& a, long long o, float4 x, float ls) {
  x = make_float4(x.x / ls, x.y / ls, x.z / ls, x.w / ls);
  if (a.out_fp32 || sizeof(T) == 4) {
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + o) = x;
  } else {
    const df32x2_t lo = {x.x, x.y}, hi = {x.z, x.w};                    // (to nearest even, in one instruction each)
    const uint2 y = make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, dbf16x2_t)), __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, dbf16x2_t)));
    *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + o) = y;
  }
}
// Partial results go past the caches that other XCDs do not see (the sc1 bit, which is what an agent-scope atomic access
// has; those move 8 bytes at most, and two per lane are twice the requests: 16 partial results of 7 query heads took 1.9 us
// to read instead of 1.3).
constexpr int AGENT = 16;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t agent_buffer(void* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(p, 0, bytes, 0x00020000); }
constexpr int NOWHERE = 0x7ffffff0;      // past the end of any of them: a read gives zeros and touches nothing

// The NW waves' (max, sum, acc) of a piece merged in wave order: the output if the head is this one piece.  Otherwise the
// piece's partial result goes to the head's record in the workspace, and the last workgroup to arrive at the head's counter merges them all,
// in piece order, and stores the head's new length (everybody has read the old one).  Behind the barrier every wave works
// for itself, with counters of its own: 64 / (D / 4) query heads per wave, four elements per lane (a single query head:
// the first wave alone, whose lanes share the pieces); a wave has its stores acknowledged, arrives, and leaves unless it is
// the last.
// s_ml: [NW][GT] (max, sum); s_acc: a wave's results WS floats behind those of the wave before it, AR floats per query head.
template <typename T, int D, int NW, int GT, int WS, int AR, bool WEIGHTS = false>
__device__ __forceinline__ void finish_piece(const DecodeArgs& a, long long hidx, int chunk, int len, int rows, bool can_append, int arrive,
                                             const float (*s_ml)[GT][2], const float* s_acc, Fresh fresh = Fresh{}) {
  constexpr int TL = D / 4, QW = 64 / TL;
  constexpr bool OWN = NW >= GT;                             // a query head per wave, whose lanes share the pieces
  constexpr int KP = OWN ? QW : 1, MB = OWN ? 8 : 16;        // MB: pieces in flight per lane
  constexpr int WK = OWN && (GT > 1 || NW == 8) ? KP : 1;    // and, of more than a few waves, their results
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave * (OWN ? 1 : QW) >= (GT == 1 ? 1 : a.G)) return;
  const int t = lane % TL, kp = OWN ? lane / TL : 0, g = OWN ? wave : wave * QW + lane / TL;
  const bool act = OWN ? kp == 0 : g < a.G;
  const int pieces = len <= rows ? 1 : rows == a.chunk_rows ? pieces_of(a, len) : (len + rows - 1) / rows;
  const long long o = (hidx * a.G + g) * D + 4 * t;
  // records of a head: [slots][G][D] accumulated elements, [slots][G] (max, sum)
  const int step = a.G * D * 4, step_ml = a.G * 8;
  const __amdgpu_buffer_rsrc_t rec = agent_buffer(a.part + hidx * a.slots * a.G * D, a.slots * step);
  const __amdgpu_buffer_rsrc_t rec_ml = agent_buffer(a.part_ml + hidx * a.slots * a.G * 2, a.slots * step_ml);
  if (chunk < pieces && (act || WK > 1)) {
    float mx = DNEG_BIG, ls = 0.f, av[4] = {0.f, 0.f, 0.f, 0.f};
    const int w0 = WK > 1 ? kp * (NW / WK) : 0;
#pragma unroll
    for (int w = 0; w < NW / WK; ++w) mx = fmaxf(mx, s_ml[w0 + w][g][0]);
#pragma unroll
    for (int w = 0; w < NW / WK; ++w) {
      const float c = weight_of(s_ml[w0 + w][g][0] - mx);
      const float4 x = *reinterpret_cast<const float4*>(s_acc + (w0 + w) * WS + g * AR + 4 * t);
      ls += s_ml[w0 + w][g][1] * c;
      av[0] += x.x * c; av[1] += x.y * c; av[2] += x.z * c; av[3] += x.w * c;
    }
    if (WK > 1) merge_lanes<TL, 4>(mx, ls, av);
    if (pieces == 1) {
      if (act) store_out4<T>(a, o, make_float4(av[0], av[1], av[2], av[3]), ls);
      if (WEIGHTS && act && t == 0) *reinterpret_cast<float2*>(a.head_ml + (hidx * a.G + g) * 2) = make_float2(mx, ls);
    } else if (act) {
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(du32x4_t, make_float4(av[0], av[1], av[2], av[3])), rec, (g * D + 4 * t) * 4, chunk * step, AGENT);
      if (t == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(du32x2_t, make_float2(mx, ls)), rec_ml, g * 8, chunk * step_ml, AGENT);
    }
  }
  if (arrive > 1) {
    const long long head = a.head0 + hidx;
    uint32_t* count = a.meet.count + (GT == 1 ? head : head * a.G + wave) * MEET_COUNT_STRIDE;
    uint32_t arrived = 0u;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // the wave's stores are where everybody sees them
    if (lane == 0) arrived = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    arrived = (uint32_t)__builtin_amdgcn_readfirstlane((int)arrived);
    if (arrived + 1u != (uint32_t)arrive) return;
    if (lane == 0) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (pieces > 1) {
      float m = DNEG_BIG, ls = 0.f, av[4] = {0.f, 0.f, 0.f, 0.f};
      const int gg = act || OWN ? g : 0;                       // (lanes without a query head read along)
      const int at = ((kp * a.G + gg) * D + 4 * t) * 4, at_ml = (kp * a.G + gg) * 8;
      const int left = min(pieces, a.slots);                   // (a head longer than the launch was sized for: what there is of it)
      const auto merge = [&](const float4 (&x)[MB], const float2 (&ml)[MB]) {
        float bm = m;
#pragma unroll
        for (int j = 0; j < MB; ++j) bm = fmaxf(bm, ml[j].x);
        const float sc = weight_of(m - bm);
        ls *= sc; av[0] *= sc; av[1] *= sc; av[2] *= sc; av[3] *= sc;
#pragma unroll
        for (int j = 0; j < MB; ++j) {
          const float f = weight_of(ml[j].x - bm);
          ls = fmaf(ml[j].y, f, ls);
          av[0] = fmaf(x[j].x, f, av[0]); av[1] = fmaf(x[j].y, f, av[1]); av[2] = fmaf(x[j].z, f, av[2]); av[3] = fmaf(x[j].w, f, av[3]);
        }
        m = bm;
      };
      // Whole trips of KP * MB pieces, without masks (2 heads of 8K rows, 64 to 128 pieces each, took 1 us more per call with them) and
      // out of the way of the last one, which is the only one of most heads (0.2 us per call of 4 heads of 700 rows).
      int c0 = 0;
      if (__builtin_expect(left > KP * MB, 0)) {
        for (; c0 + KP * MB < left; c0 += KP * MB) {
          float4 x[MB]; float2 ml[MB];
#pragma unroll
          for (int j = 0; j < MB; ++j) {
            ml[j] = __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(rec_ml, at_ml, (c0 + j * KP) * step_ml, AGENT));
            x[j] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(rec, at, (c0 + j * KP) * step, AGENT));
          }
          merge(x, ml);
        }
      }
      {
        float4 x[MB]; float2 ml[MB];
#pragma unroll
        for (int j = 0; j < MB; ++j) {
          const int c = c0 + j * KP;
          const bool mine = c + kp < left;
          ml[j] = __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(rec_ml, mine ? at_ml + c * step_ml : NOWHERE, 0, AGENT));
          x[j] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(rec, mine ? at + c * step : NOWHERE, 0, AGENT));
        }
#pragma unroll
        for (int j = 0; j < MB; ++j) ml[j].x = c0 + j * KP + kp < left ? ml[j].x : 2.f * DNEG_BIG;     // weight 0, of zeros
        merge(x, ml);
      }
      if (KP > 1) merge_lanes<TL, 4>(m, ls, av);
      if (act) store_out4<T>(a, o, make_float4(av[0], av[1], av[2], av[3]), ls);
      if (WEIGHTS && act && t == 0) *reinterpret_cast<float2*>(a.head_ml + (hidx * a.G + g) * 2) = make_float2(m, ls);
    }
  }
  if (can_append && threadIdx.x == 0) a.kv_len[hidx] = len;
  if (WEIGHTS && threadIdx.x == 0) a.fresh[hidx] = fresh.there ? fresh.row : -1;
}

}  // namespace madakv
