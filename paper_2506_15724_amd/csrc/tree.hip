// Several drafted tokens per step over the reduced, ragged cache (paper Sec. 3.1 Eq. 3-5 for a tree of tokens): the attention of all nodes of the
// tree, and the accepted nodes' rows into the cache.
//
// Attention: the G * T query rows of a KV head (T nodes) are the columns of attn_tile.h, its keys the rows of the head's segment and behind
// them the T nodes, of which a column sees those that its node's mask names:
//   out(c) = sum_r e^(s q_c . k_r) v_r / sum_r e^(s q_c . k_r),   r over the rows of the segment and the nodes i with bit i of tree[node of c]
// A head is cut into pieces; each leaves its partial (reference, sum, output) in the workspace, and a second launch joins them in their order, so results
// do not depend on who comes first.  (Joined by whoever comes last it took longer: results pass from one XCD's L2 to another's, a wait per piece.)
// Two kernels: tree_narrow_kernel, bound by how fast rows arrive (128 heads of 16384 bf16 rows, 32 nodes: 185 us, 5.8 TB/s), and tree_attn_kernel for more columns,
// bound by the arithmetic (60 nodes of 2 x 32/8 heads of 16384 4-bit rows: 51 us; by the profiler's clock 49 for the pieces, 660 TFLOP/s, some 8 of them for 32 MB of partial results, and 7 for
// the join).  Nodes' rows count with the
// values that the cache would give them.  Masked keys count for nothing whatever they hold, as in prompt_attn.hip.
#include "attn_tile.h"
#include "decode_pieces.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace madakv {

struct TreeArgs {
  const void* q; const void* k_new; const void* v_new; const unsigned char* k_c; const unsigned char* v_c;
  const unsigned long long* tree;      // [B][T]
  const int64_t* kv_off; const int32_t* kv_len; void* out;
  int B, H, G, T, R;                   // R = G * T columns
  int groups;                          // column groups of a head
  int chunk_rows, max_chunks, slots;
  float* part; float* part_ml;         // [heads][slots][R][D], [2]
  long long capacity;
  int page_rows, page_shift, tbl_entries;
  const int32_t* page_tbl;             // of the call's first head
  float scale_log2;
};

// Rows per piece of a head of so many, and how many pieces that makes; the nodes are with the last one.  An eighth of a piece more than whole pieces makes no
// piece of its own: heads that were cut to fill the chip once stay so while tokens are appended.
struct Cut { int rows, pieces; };
__device__ __forceinline__ Cut cut_of(int chunk_rows, int max_chunks, int len) {
  const int n = min(max(1, (len - chunk_rows / 8 + chunk_rows - 1) / chunk_rows), max_chunks);
  const int rows = max(1, ((len + n - 1) / n + ATT_TILE - 1) / ATT_TILE) * ATT_TILE;
  return Cut{rows, std::max(1, (len + rows - 1) / rows)};
}

// four neighbouring elements of the output
__device__ __forceinline__ void store4(float* to, const at_f32x4_t& o, float inv) { *reinterpret_cast<at_f32x4_t*>(to) = at_f32x4_t{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv}; }
__device__ __forceinline__ void store4(uint16_t* to, const at_f32x4_t& o, float inv) {
  *reinterpret_cast<uint2*>(to) = make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector((at_f32x2_t{o[0] * inv, o[1] * inv}), at_bf16x2_t)),
                                             __builtin_bit_cast(uint32_t, __builtin_convertvector((at_f32x2_t{o[2] * inv, o[3] * inv}), at_bf16x2_t)));
}

// 32 elements of a node's row as the 4-bit cache would have them: in place
__device__ __forceinline__ void as_mx4(uint4 (&x)[4]) {
  uint32_t top = 0;
  uint32_t y[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) { y[4 * i] = x[i].x; y[4 * i + 1] = x[i].y; y[4 * i + 2] = x[i].z; y[4 * i + 3] = x[i].w; }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t lo = min(y[i] & 0x7fffu, 0x7f7fu), hi = min(y[i] >> 16 & 0x7fffu, 0x7f7fu);
    top = max(top, max(lo, hi));
    y[i] = (y[i] & 0x80008000u) | lo | hi << 16;
  }
  const uint32_t byte = mx_scale_byte(top);
  const float s = mx_scale_value(byte);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t code = 0;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(mx_bf16x2_t, y[4 * i]), s, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(mx_bf16x2_t, y[4 * i + 1]), s, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(mx_bf16x2_t, y[4 * i + 2]), s, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(mx_bf16x2_t, y[4 * i + 3]), s, 3);
    x[i] = mx_decode8(code, byte);
  }
}
// four E4M3 bytes -> four bf16 (exact)
__device__ __forceinline__ uint2 from_e4m3(uint32_t w) {
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)));
}
// two bf16 pairs -> four E4M3 bytes, as f32_to_e4m3 (checked on every bf16): the instruction rounds to nearest even, magnitudes above 448 and NaN are made 448 first
__device__ __forceinline__ uint32_t e4m3_of(uint32_t a, uint32_t b) {
  const auto clamped = [](uint32_t x) {
    return __builtin_bit_cast(mx_bf16x2_t, __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(mx_u16x2_t, x & 0x7fff7fffu), mx_u16x2_t{0x43e0, 0x43e0})) | (x & 0x80008000u));
  };
  typedef __attribute__((ext_vector_type(2))) short i16x2_t;
  i16x2_t code = {0, 0};
  code = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(code, clamped(a), 1.f, false);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(code, clamped(b), 1.f, true);
  return __builtin_bit_cast(uint32_t, code);
}

// ---- more columns -----------------------------------------------------------------------------------------
// T: Q, nodes' rows; CACHE: 0 rows of T, CACHE_E4M3, CACHE_E2M1.  WC blocks of 32 columns, one per wave.  All waves share a tile of 64 keys; rows of the type of the model come straight into LDS, 8-bit and 4-bit rows
// through registers, which turn them into bf16 (exactly).  Up to 256 columns in a workgroup: rows are converted once for all of them (60 nodes of 2 x 32/8 heads
// of 16384 4-bit rows: 53 us, by workgroups of 128 columns 59).  Tiles further ahead of the products gain nothing for 8 and 4 bits (1, 2, 3: 53.8, 52.8, 53).
template <typename T, typename OT, int CACHE, int D, int WC>
__global__ __launch_bounds__(WC * 64) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2))) void tree_attn_kernel(TreeArgs a) {
  using Tile = AttnTile<T, D, CACHE != 0>;
  constexpr int PARTS = sizeof(T) == 2 && sizeof(OT) == 4 ? 3 : 1;
  constexpr int NT = WC * 64, COLS = WC * 32, ROWB = Tile::ROWB, PPR = Tile::PPR;
  constexpr int EPL = CACHE == CACHE_E2M1 ? 32 : CACHE == CACHE_E4M3 ? 16 : 16 / (int)sizeof(T);      // elements of a 16-byte load
  constexpr int LPR = D / EPL;                                                                          // loads of a row
  constexpr int LPT = (ATT_TILE * LPR + NT - 1) / NT;                                                   // of a thread, per tile and tensor
  constexpr int CROWB = CACHE ? LPR * 16 : ROWB;                                                        // bytes of a cache row
  constexpr int AHEAD = CACHE == 0 && sizeof(T) == 2 && WC == 8 ? 3 : 1;       // tiles on their way: as many as LDS has room for
  constexpr int SLOTS = CACHE ? 2 : AHEAD + 1;                 // tiles of K, of V in LDS
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * SLOTS * Tile::BYTES];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const uint32_t xy = blockIdx.x + blockIdx.y;                 // the pieces of a head on different XCDs
  const int x = (int)(xy % gridDim.x), chunk = blockIdx.y;
  const long long hidx = x / a.groups;
  const int group = x % a.groups;
  const int len = a.kv_len[hidx];
  const long long off = a.kv_off[hidx];
  const int total = len > 0 ? len + a.T : 0;                   // (an empty segment: its budgets did not fit the cache)
  const Cut cut_rows = cut_of(a.chunk_rows, a.max_chunks, len);
  const int rows = cut_rows.rows, pieces = cut_rows.pieces;
  if (chunk >= pieces) return;
  const int r_begin = chunk * rows, r_end = chunk == pieces - 1 ? total : r_begin + rows;
  const int ntiles = (r_end - r_begin + ATT_TILE - 1) / ATT_TILE;
  RowMap at;
  at.off = off; at.init_rows = 0x7fffffff; at.tbl = nullptr; at.shift = 0; at.fresh_slot = -1; at.fresh_page = 0;
  if (a.page_rows) { at.tbl = a.page_tbl + hidx * a.tbl_entries; at.shift = a.page_shift; at.init_rows = at.tbl[0] << a.page_shift; }

  const int c_own = group * COLS + wave * 32 + col, c = min(c_own, a.R - 1);       // (a column without a query: the last one's once more, not stored)
  typename Tile::Query q;
  Tile::load(q, reinterpret_cast<const T*>(a.q) + (hidx * a.R + c) * D, half);
  const unsigned long long mask = a.tree[(hidx / a.H % a.B) * a.T + c % a.T];

  Tile::await(q);

  const unsigned char* kn = reinterpret_cast<const unsigned char*>(a.k_new) + hidx * a.T * ROWB;
  const unsigned char* vn = reinterpret_cast<const unsigned char*>(a.v_new) + hidx * a.T * ROWB;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  // ---- rows of T: straight into LDS, tile t into slot t % SLOTS (rows past the end of the piece: its last one once more, masked where they are used)
  const auto load_direct = [&](int t) {
#pragma unroll
    for (int j = 0; j < LPT; ++j) {
      const int p = (wave * LPT + j) * 64 + lane, lr = p / PPR, s = p % PPR;
      const int r = min(r_begin + t * ATT_TILE + lr, r_end - 1);
      const bool node = r >= len;
      const long long row = node ? r - len : at(r);
      const unsigned char* kp = (node ? kn : a.k_c) + row * ROWB + Tile::k_slot(lr, s) * 16;
      const unsigned char* vp = (node ? vn : a.v_c) + row * ROWB + Tile::v_slot(lr, s) * 16;
      const uint32_t to = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds0 + (uint32_t)(t % SLOTS * Tile::BYTES + (wave * LPT + j) * 1024)));
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(kp) : "m0", "memory");
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to + SLOTS * Tile::BYTES), "v"(vp) : "m0", "memory");
    }
  };
  // ---- 8-bit and 4-bit rows: through registers
  struct Raw { uint4 k[CACHE ? LPT : 1], v[CACHE ? LPT : 1]; uint32_t ks[CACHE ? LPT : 1], vs[CACHE ? LPT : 1]; } raw;
  const auto fetch = [&](int t) {
#pragma unroll
    for (int j = 0; j < LPT; ++j) {
      const int p = j * NT + tid, lr = p / LPR, piece = p % LPR;
      if (ATT_TILE * LPR % NT && lr >= ATT_TILE) break;
      const long long row = at(min(r_begin + t * ATT_TILE + lr, min(r_end, len) - 1));        // (a node's row is read when it is wanted)
      raw.k[j] = *reinterpret_cast<const uint4*>(a.k_c + row * CROWB + piece * 16);
      raw.v[j] = *reinterpret_cast<const uint4*>(a.v_c + row * CROWB + piece * 16);
      if constexpr (CACHE == CACHE_E2M1) {
        raw.ks[j] = a.k_c[a.capacity * CROWB + row * (D / MX_BLOCK) + piece];
        raw.vs[j] = a.v_c[a.capacity * CROWB + row * (D / MX_BLOCK) + piece];
      }
    }
  };
  const auto park = [&](int t) {
#pragma unroll
    for (int j = 0; j < LPT; ++j) {
      const int p = j * NT + tid, lr = p / LPR, piece = p % LPR;
      if (ATT_TILE * LPR % NT && lr >= ATT_TILE) break;
      const int r = min(r_begin + t * ATT_TILE + lr, r_end - 1);
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        unsigned char* to = lds + (t % SLOTS + SLOTS * which) * Tile::BYTES + lr * ROWB;
        const unsigned char* nodes = which ? vn : kn;
        uint4 y[EPL / 8 ? EPL / 8 : 1];
        if (r >= len) {
          const uint4* from = reinterpret_cast<const uint4*>(nodes + (long long)(r - len) * ROWB + piece * EPL * 2);
#pragma unroll
          for (int i = 0; i < EPL / 8; ++i) y[i] = from[i];
          if constexpr (CACHE == CACHE_E2M1) {
            as_mx4(y);
          } else if constexpr (CACHE == CACHE_E4M3) {
#pragma unroll
            for (int i = 0; i < EPL / 8; ++i) {
              const uint2 lo = from_e4m3(e4m3_of(y[i].x, y[i].y)), hi = from_e4m3(e4m3_of(y[i].z, y[i].w));
              y[i] = make_uint4(lo.x, lo.y, hi.x, hi.y);
            }
          }
        } else {
          const uint4 z = which ? raw.v[j] : raw.k[j];
          if constexpr (CACHE == CACHE_E2M1) {
            const uint32_t scale = which ? raw.vs[j] : raw.ks[j];
            y[0] = mx_decode8(z.x, scale); y[1] = mx_decode8(z.y, scale); y[2] = mx_decode8(z.z, scale); y[3] = mx_decode8(z.w, scale);
          } else if constexpr (CACHE == CACHE_E4M3) {
            const uint2 e0 = from_e4m3(z.x), e1 = from_e4m3(z.y), e2 = from_e4m3(z.z), e3 = from_e4m3(z.w);
            y[0] = make_uint4(e0.x, e0.y, e1.x, e1.y); y[1] = make_uint4(e2.x, e2.y, e3.x, e3.y);
          }
        }
#pragma unroll
        for (int i = 0; i < EPL / 8; ++i) {
          const int s = which ? Tile::v_slot(lr, piece * (EPL / 8) + i) : Tile::k_slot(lr, piece * (EPL / 8) + i);
          *reinterpret_cast<uint4*>(to + s * 16) = y[i];
        }
      }
    }
  };

  AttnState<D> st;
  // the 32 keys from k32 on, rows row0 and on of the tile
  const auto finish = [&](auto careful, int k32, int row0, at_f32x16_t& s, const unsigned char* vt) {
    float p[16], more;
    typename Tile::template Weights<PARTS> w;
    const bool cut = k32 + 32 > min(len, r_end);
    const auto sees = [&](int key) { const int r = k32 + key; return r < r_end && (r < len || (mask >> (r - len) & 1)); };
    bool look = cut;
    if (!cut) {
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale_log2, -st.ref));
      more = sum16(p);
      look = __builtin_amdgcn_ballot_w64(!(st.sum + more < ATT_FAR)) != 0;
    }
    if (__builtin_expect(look, 0)) {
      if (cut) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = sees(key_of(i, half)) ? s[i] : -__builtin_inff();
      }
      attn_look<D>(st, s, p, more, a.scale_log2);
    }
    st.sum += more;
    Tile::template pack<PARTS>(p, w);
    if (decltype(careful)::value && (PARTS > 1 || cut)) {
#pragma unroll 1
      for (int key = 0; key < 32; ++key) {                     // its weight is with one of the column's lanes, element i of its 16
        const int i = 4 * (key >> 3) + (key & 3), owner = col + 32 * ((key >> 2) & 1);
        const float f = __shfl(Tile::template weight<PARTS>(w, i), owner, 64);
        if (!sees(key)) continue;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const at_f32x4_t y = Tile::value4(vt, row0 + key, 32 * db + 8 * g + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e) st.o[db][4 * g + e] = fmaf(f, y[e], st.o[db][4 * g + e]);
          }
      }
    } else {
      Tile::template add<PARTS>(vt, row0, lane, w, st.o);
    }
  };
  const auto compute = [&](auto careful, int t) {
    const unsigned char* kt = lds + t % SLOTS * Tile::BYTES;
    const unsigned char* vt = kt + SLOTS * Tile::BYTES;
    const int k0 = r_begin + t * ATT_TILE;
    at_f32x16_t s = Tile::scores(kt, 0, lane, q), s1 = Tile::scores(kt, 32, lane, q);       // (of the last row once more, past the end)
    finish(careful, k0, 0, s, vt);
    if (k0 + 32 < r_end) finish(careful, k0 + 32, 32, s1, vt);
  };
  const auto pass = [&](auto careful) {
    st.clear();
    if (ntiles <= 0) return;
    // (what is past the end: the last row, which nobody looks at; it keeps the count of loads on their way)
    if constexpr (CACHE) {
      fetch(0);
      park(0);
      fetch(1);
    } else {
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) load_direct(j);
    }
#pragma unroll 1
    for (int t = 0; t < ntiles; ++t) {
      // tile t is there for everybody, and nobody reads tile t - 1 any more
      if constexpr (CACHE) {
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        compute(careful, t);
        if (t + 1 < ntiles) park(t + 1);
        fetch(t + 2);
      } else {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * LPT * (AHEAD - 1)) : "memory");
        load_direct(t + AHEAD);
        compute(careful, t);
      }
    }
    if constexpr (CACHE == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  pass(std::false_type{});
  if (__builtin_expect(__syncthreads_or(not_finite(st)), 0)) {
    pass(std::true_type{});
  }

  const float sum = both_sum(st.sum);
  if (pieces == 1) {
    store_column<OT, D>(reinterpret_cast<OT*>(a.out) + (hidx * a.R + c) * D, c == c_own, half, st.o, 1.f / sum);
  } else if (c == c_own) {
    const long long record = (hidx * a.slots + chunk) * a.R + c;
    float* to = a.part + record * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<at_f32x4_t*>(to + 32 * db + 8 * g + 4 * half) = at_f32x4_t{st.o[db][4 * g], st.o[db][4 * g + 1], st.o[db][4 * g + 2], st.o[db][4 * g + 3]};
    if (half == 0) *reinterpret_cast<float2*>(a.part_ml + record * 2) = make_float2(st.ref, sum);
  }
}

// ---- up to 32 columns ------------------------------------------------------------------------------------
// Hardly more arithmetic per byte than decode: what counts is how much is on its way.  Every wave works for itself on tiles of 32 rows, without barriers:
// rows of the type of the model come straight into LDS tiles of the wave's own, those of 8 and 4 bits as operand A of K (a lane has one row's dims of 16 bytes at a time, and Q the
// same order of dims) and through registers into an LDS tile of V.  The next tile's are sent for as soon as there is room for them: eight waves on a
// compute unit have up to 128 KB of 16-bit rows on their way.  (32-bit rows of 128 dims: four waves; 32 heads of 8192 rows, 8 nodes, 82 us, bound by the fp32
// matrix instructions, of whose 32 columns 8 are used; by the kernel for many columns, two waves, 392.)
// Weights of two bf16 numbers for bf16 outputs, so that nodes are as near to their formula as decode's tokens (8 nodes of 128 heads of 2048 rows: bf16 27.3 -> 27.5 us,
// 8 bits 18.5 -> 19.1, 4 bits 18.4 -> 20.0; of uneven heads in 8 bits 19.8 -> 21.2).
template <typename T, typename OT, int CACHE, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2))) void tree_narrow_kernel(TreeArgs a) {
  using Tile = AttnTile<T, D, CACHE != 0>;
  constexpr int NW = 4, PARTS = sizeof(T) == 4 ? 1 : sizeof(OT) == 4 ? 3 : 2, ROWB = Tile::ROWB, RS = D + 4;
  constexpr int EPL = CACHE == CACHE_E2M1 ? 32 : CACHE == CACHE_E4M3 ? 16 : 16 / (int)sizeof(T);         // elements of a 16-byte load
  constexpr int NY = CACHE ? EPL / 8 : 1;                                               // 16-byte pieces in the type of the model
  constexpr int LPR = D / EPL, CROWB = LPR * 16;                                        // loads of a row, its bytes
  constexpr int KL = LPR / 2 ? LPR / 2 : 1, VL = LPR / 2 ? LPR / 2 : 1;                 // loads of a lane per tile: K, V
  static_assert(LPR >= 2, "both lanes of a row have something of it");
  constexpr int TILEB = 32 * ROWB, WAVEB = CACHE ? TILEB : 2 * TILEB, RESB = 32 * RS * 4;          // a wave's tiles (V, K), later its results
  constexpr int EACH = WAVEB > RESB ? WAVEB : RESB;
  __shared__ __attribute__((aligned(1024))) unsigned char s_tiles[NW * EACH];
  __shared__ float s_ml[NW][32][2];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  // (the pieces of a head on different XCDs, the column groups of a piece next to each other)
  const int chunk = (int)blockIdx.y / a.groups, group = (int)blockIdx.y - chunk * a.groups, xy = (int)blockIdx.x + chunk, x = xy < (int)gridDim.x ? xy : xy % (int)gridDim.x;
  const int c0 = group * 32, n_cols = min(32, a.R - c0);
  const int len = a.kv_len[x];
  const long long off = a.kv_off[x];
  const Cut cut_rows = cut_of(a.chunk_rows, a.max_chunks, len);
  const int rows = cut_rows.rows, pieces = cut_rows.pieces;
  if (chunk >= pieces) return;
  const int r_begin = chunk * rows, n_rows = max(0, min(len - r_begin, rows));          // (an empty segment sees nothing: its sums stay zero)
  const int row_tiles = (n_rows + 31) / 32, node_tiles = chunk == pieces - 1 && len > 0 ? (a.T + 31) / 32 : 0;
  RowMap at;
  at.off = off; at.init_rows = 0x7fffffff; at.tbl = nullptr; at.shift = 0; at.fresh_slot = -1; at.fresh_page = 0;
  if (a.page_rows) { at.tbl = a.page_tbl + (long long)x * a.tbl_entries; at.shift = a.page_shift; at.init_rows = at.tbl[0] << a.page_shift; }
  const int c = c0 + min(col, n_cols - 1);                     // (a column without a query: the last one's once more, not stored)
  // the query; of 8-bit and 4-bit rows for step i NY + e dims [(2 i + half) EPL + 8 e, + 8)
  typename Tile::Query q;
  const auto dim_of = [&](int ks) { return (2 * (ks / NY) + half) * EPL + 8 * (ks % NY); };
  {
    const T* qr = reinterpret_cast<const T*>(a.q) + ((long long)x * a.R + c) * D;
    if constexpr (CACHE == 0) {
      Tile::load(q, qr, half);
    } else {
#pragma unroll
      for (int ks = 0; ks < Tile::KS; ++ks) q.x[ks] = *reinterpret_cast<const at_bf16x8_t*>(qr + dim_of(ks));
    }
  }
  const unsigned long long mask = a.tree[(long long)(x / a.H % a.B) * a.T + c % a.T];

  unsigned char* vt = s_tiles + wave * EACH;
  unsigned char* kt = vt + TILEB;                              // (16-bit rows)
  // Where the rows of a tile are, r0 its first one in the piece: two stretches of 16, each within a page, that need not follow each other.
  struct Place { long long lo, hi; };
  const auto place = [&](int r0) {
    const int r = r_begin + r0;
    if (!a.page_rows) return Place{off + r, off + r + 16};
    return Place{at(r), r0 + 16 < n_rows ? at(r + 16) : 0};
  };
  // 8-bit and 4-bit rows: 16 bytes of row lr (past the end: the last one once more, masked where it is used) at byte `byte`
  struct Raw { uint4 k[KL], v[VL]; uint32_t ks[KL], vs[VL]; } raw;
  const auto row_of = [&](const Place& at, int r0, int lr) { lr = min(lr, n_rows - 1 - r0); return (lr < 16 ? at.lo : at.hi) + (lr & 15); };
  const auto load_k = [&](const Place& at, int r0) {
    const long long row = row_of(at, r0, col);
    const unsigned char* p = a.k_c + row * CROWB + half * 16;
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      raw.k[i] = *reinterpret_cast<const uint4*>(p + 32 * i);
      if constexpr (CACHE == CACHE_E2M1) raw.ks[i] = a.k_c[a.capacity * CROWB + row * (D / MX_BLOCK) + 2 * i + half];
    }
  };
  const auto load_v = [&](const Place& at, int r0) {
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const int p = j * 64 + lane;
      const long long row = row_of(at, r0, p / LPR);
      raw.v[j] = *reinterpret_cast<const uint4*>(a.v_c + row * CROWB + p % LPR * 16);
      if constexpr (CACHE == CACHE_E2M1) raw.vs[j] = a.v_c[a.capacity * CROWB + row * (D / MX_BLOCK) + p % LPR];
    }
  };
  // 16-bit rows: a load takes 1 KB, whole rows of one of the two stretches
  constexpr int GROUP = 1024 / ROWB, LOADS = 32 / GROUP;
  const uint32_t lds_v = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)vt;
  const auto send = [&](bool v, const Place& at, int r0) {
    const unsigned char* cache = v ? a.v_c : a.k_c;
    const unsigned char* from[2] = {cache + at.lo * ROWB, cache + at.hi * ROWB};
    const int valid = n_rows - r0;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      int lr = j * GROUP + lane / Tile::PPR;
      const int s = (v ? Tile::v_slot(lr, lane % Tile::PPR) : Tile::k_slot(lr, lane % Tile::PPR)) * 16;
      uint64_t p = reinterpret_cast<uint64_t>(from[2 * j / LOADS]);
      if (valid < 32) {                                        // (uniform)
        lr = min(lr, valid - 1);
        if (valid <= 16) p = reinterpret_cast<uint64_t>(from[0]);
        else if (2 * j >= LOADS) lr = max(lr, 16);
      }
      const uint64_t same = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane((int)(lds_v + (v ? 0u : (uint32_t)TILEB) + j * 1024u))), "v"((lr & 15) * ROWB + s), "s"(same) : "m0", "memory");
    }
  };
  // 16 bytes of an 8-bit or 4-bit row -> EPL bf16
  const auto unpack = [&](const uint4& z, uint32_t scale, uint4 (&y)[NY]) {
    if constexpr (CACHE == CACHE_E2M1) {
      y[0] = mx_decode8(z.x, scale); y[1] = mx_decode8(z.y, scale); y[2] = mx_decode8(z.z, scale); y[3] = mx_decode8(z.w, scale);
    } else if constexpr (CACHE == CACHE_E4M3) {
      const uint2 e0 = from_e4m3(z.x), e1 = from_e4m3(z.y), e2 = from_e4m3(z.z), e3 = from_e4m3(z.w);
      y[0] = make_uint4(e0.x, e0.y, e1.x, e1.y); y[1] = make_uint4(e2.x, e2.y, e3.x, e3.y);
    }
  };
  // EPL elements of a node's row, with the values that the cache would give them
  const auto node_part = [&](const void* nodes, int node, int piece, uint4 (&y)[NY]) {
    const uint4* from = reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned char*>(nodes) + ((long long)x * a.T + min(node, a.T - 1)) * ROWB) + piece * NY;
#pragma unroll
    for (int i = 0; i < NY; ++i) y[i] = from[i];
    if constexpr (CACHE == CACHE_E2M1) {
      as_mx4(y);
    } else if constexpr (CACHE == CACHE_E4M3) {
#pragma unroll
      for (int i = 0; i < NY; ++i) {
        const uint2 lo = from_e4m3(e4m3_of(y[i].x, y[i].y)), hi = from_e4m3(e4m3_of(y[i].z, y[i].w));
        y[i] = make_uint4(lo.x, lo.y, hi.x, hi.y);
      }
    }
  };
  const auto park = [&](int j, const uint4 (&y)[NY]) {         // piece j of the lane's V
    const int p = j * 64 + lane, lr = p / LPR;
#pragma unroll
    for (int i = 0; i < NY; ++i) *reinterpret_cast<uint4*>(vt + lr * ROWB + Tile::v_slot(lr, p % LPR * NY + i) * 16) = y[i];
  };
  AttnState<D> st;
  // (the tile that its lanes have written, read with another lane mapping: same wave, in order)
  const auto settle = [] {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  const auto weigh = [&](at_f32x16_t& s, bool cut, uint32_t keys, typename Tile::template Weights<PARTS>& w) {
    float p[16], more;
    bool look = cut;
    if (!cut) {
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale_log2, -st.ref));
      more = sum16(p);
      look = __builtin_amdgcn_ballot_w64(!(st.sum + more < ATT_FAR)) != 0;
    }
    if (__builtin_expect(look, 0)) {
      const uint32_t mine = keys >> (4 * half);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = mine >> key_of(i, 0) & 1 ? s[i] : -__builtin_inff();
      attn_look<D>(st, s, p, more, a.scale_log2);
    }
    st.sum += more;
    Tile::template pack<PARTS>(p, w);
  };
  const auto add = [&](auto careful, bool cut, uint32_t keys, const typename Tile::template Weights<PARTS>& w) {
    settle();
    if (decltype(careful)::value && (PARTS > 1 || cut)) {
#pragma unroll 1
      for (int key = 0; key < 32; ++key) {                     // its weight is with one of the column's lanes, element i of its 16
        const int i = 4 * (key >> 3) + (key & 3), owner = col + 32 * ((key >> 2) & 1);
        const float f = __shfl(Tile::template weight<PARTS>(w, i), owner, 64);
        if (!(keys >> key & 1)) continue;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const at_f32x4_t y = Tile::value4(vt, key, 32 * db + 8 * g + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e) st.o[db][4 * g + e] = fmaf(f, y[e], st.o[db][4 * g + e]);
          }
      }
    } else {
      Tile::template add<PARTS>(vt, 0, lane, w, st.o);
    }
    settle();
  };
  // once more, carefully, where outputs are no numbers: the formula's, or those of rows of V that nobody may see (see prompt_attn.hip)
  const auto pass = [&](auto careful) {
    st.clear();
    int r0 = wave * 32;
    const int last = (row_tiles - 1) * 32;                     // (past the end: the last tile, which nobody looks at; it keeps the count of loads in flight)
    if (r0 < n_rows) {
      const Place here = place(r0);
      if constexpr (CACHE == 0) { send(false, here, r0); send(true, here, r0); }
      else { load_k(here, r0); load_v(here, r0); }
    }
    Tile::await(q);
#pragma unroll 1
    for (; r0 < n_rows; r0 += NW * 32) {
      const int next = min(r0 + NW * 32, last);
      const Place there = place(next);
      const bool cut = r0 + 32 > n_rows;
      const uint32_t keys = cut ? (1u << (n_rows - r0)) - 1u : ~0u;
      typename Tile::template Weights<PARTS> w;
      at_f32x16_t s;
      if constexpr (CACHE == 0) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");       // K is there
        s = Tile::scores(kt, 0, lane, q);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        send(false, there, next);
        weigh(s, cut, keys, w);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");       // V is there
        add(careful, cut, keys, w);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        send(true, there, next);
      } else {
        s = zero16();
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          uint4 y[NY];
          unpack(raw.k[i], raw.ks[i], y);
#pragma unroll
          for (int e = 0; e < NY; ++e) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(at_bf16x8_t, y[e]), q.x[i * NY + e], s, 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        load_k(there, next);
#pragma unroll
        for (int j = 0; j < VL; ++j) {
          uint4 y[NY];
          unpack(raw.v[j], raw.vs[j], y);
          park(j, y);
        }
        __builtin_amdgcn_sched_barrier(0);
        load_v(there, next);
        weigh(s, cut, keys, w);
        __builtin_amdgcn_sched_barrier(0);
        add(careful, cut, keys, w);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (CACHE == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // (what was sent for past the end goes to LDS, too)
#pragma unroll 1
    for (int t = 0; t < node_tiles; ++t) {
      if ((row_tiles + t) % NW != wave) continue;
      at_f32x16_t s;
      if constexpr (CACHE == 0) {
#pragma unroll
        for (int j = 0; j < VL; ++j) {
          const int p = j * 64 + lane, lr = p / LPR;
          uint4 y[1];
          node_part(a.k_new, 32 * t + lr, p % LPR, y);
          *reinterpret_cast<uint4*>(kt + lr * ROWB + Tile::k_slot(lr, p % LPR) * 16) = y[0];
        }
        settle();
        s = Tile::scores(kt, 0, lane, q);
      } else {
        s = zero16();
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          uint4 y[NY];
          node_part(a.k_new, 32 * t + col, 2 * i + half, y);
#pragma unroll
          for (int e = 0; e < NY; ++e) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(at_bf16x8_t, y[e]), q.x[i * NY + e], s, 0, 0, 0);
        }
      }
#pragma unroll
      for (int j = 0; j < VL; ++j) {
        uint4 y[NY];
        node_part(a.v_new, 32 * t + (j * 64 + lane) / LPR, (j * 64 + lane) % LPR, y);
        park(j, y);
      }
      typename Tile::template Weights<PARTS> w;
      const int left = a.T - 32 * t;
      const uint32_t keys = (uint32_t)(mask >> (32 * t)) & (left >= 32 ? ~0u : (1u << left) - 1u);
      weigh(s, true, keys, w);
      add(careful, true, keys, w);
    }
  };
  pass(std::false_type{});
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(not_finite(st)) != 0, 0)) pass(std::true_type{});

  // ---- the waves' results, joined in wave order: four dims of a column per thread
  const float sum = both_sum(st.sum);
  const auto result = [&](int w, int c) { return reinterpret_cast<float*>(s_tiles + w * EACH) + c * RS; };
  if (half == 0) { s_ml[wave][col][0] = st.ref; s_ml[wave][col][1] = sum; }
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<at_f32x4_t*>(result(wave, col) + 32 * db + 8 * g + 4 * half) = at_f32x4_t{st.o[db][4 * g], st.o[db][4 * g + 1], st.o[db][4 * g + 2], st.o[db][4 * g + 3]};
  __syncthreads();
  constexpr int TL = D / 4;
  const int t4 = tid % TL;
#pragma unroll 1
  for (int cc = tid / TL; cc < n_cols; cc += 256 / TL) {
    float m = s_ml[0][cc][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) m = fmaxf(m, s_ml[w][cc][0]);
    float l = 0.f;
    at_f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      // (a wave that has seen nothing: reference -inf, sum 0)
      const float ref = s_ml[w][cc][0], f = ref == -__builtin_inff() && s_ml[w][cc][1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ref - m);
      const at_f32x4_t y = *reinterpret_cast<const at_f32x4_t*>(result(w, cc) + 4 * t4);
      l += s_ml[w][cc][1] * f;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += y[e] * f;
    }
    if (pieces > 1) {
      const long long record = ((long long)x * a.slots + chunk) * a.R + c0 + cc;
      *reinterpret_cast<at_f32x4_t*>(a.part + record * D + 4 * t4) = o;
      if (t4 == 0) *reinterpret_cast<float2*>(a.part_ml + record * 2) = make_float2(m, l);
    } else {
      store4(reinterpret_cast<OT*>(a.out) + ((long long)x * a.R + c0 + cc) * D + 4 * t4, o, 1.f / l);
    }
  }
}

// The pieces of a head joined, in their order: four dims of a column per thread, and the pieces of a column dealt to S threads, which load up to MB of them
// at once.  What it takes is launch and latency, not bytes.
template <typename OT, int D>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a, int n_columns, int shift) {      // S = 2^shift
  constexpr int TL = D / 4, MB = 8;
  __shared__ at_f32x4_t s_o[256];
  __shared__ float2 s_ml[256 / TL];
  const int tid = threadIdx.x, t4 = tid % TL, unit = tid / TL, S = 1 << shift, slice = unit & (S - 1);
  const int x_own = ((int)blockIdx.x * (256 / TL) + unit) >> shift, x = min(x_own, n_columns - 1);
  const int hidx = x / a.R, c = x - hidx * a.R;
  const int pieces = cut_of(a.chunk_rows, a.max_chunks, a.kv_len[hidx]).pieces;
  const long long record0 = (long long)hidx * a.slots * a.R + c;
  float m = -__builtin_inff(), l = 0.f;
  at_f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  // (what has seen nothing: reference -inf, sum 0)
  const auto factor = [](float ref, float sum, float m) { return ref == -__builtin_inff() && sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(ref - m); };
  if (pieces > 1) {
    for (int p0 = slice; p0 < pieces; p0 += S * MB) {
      at_f32x4_t y[MB]; float2 ml[MB];
#pragma unroll
      for (int j = 0; j < MB; ++j) {
        if (p0 + j * S < pieces) {
          const long long record = record0 + (long long)(p0 + j * S) * a.R;
          ml[j] = *reinterpret_cast<const float2*>(a.part_ml + record * 2);
          y[j] = *reinterpret_cast<const at_f32x4_t*>(a.part + record * D + 4 * t4);
        } else {
          ml[j] = make_float2(-__builtin_inff(), 0.f);
          y[j] = at_f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
      }
      float bm = m;
#pragma unroll
      for (int j = 0; j < MB; ++j) bm = fmaxf(bm, ml[j].x);
      const float f = factor(m, l, bm);
      l *= f;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] *= f;
#pragma unroll
      for (int j = 0; j < MB; ++j) {
        const float g = factor(ml[j].x, ml[j].y, bm);
        l = fmaf(ml[j].y, g, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(y[j][e], g, o[e]);
      }
      m = bm;
    }
  }
  s_o[tid] = o;
  if (t4 == 0) s_ml[unit] = make_float2(m, l);
  __syncthreads();
  if (slice || pieces == 1 || x != x_own) return;              // (one piece: the output is there)
  for (int i = 1; i < S; ++i) m = fmaxf(m, s_ml[unit + i].x);
  float sum = 0.f;
  o = at_f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < S; ++i) {
    const float2 ml = s_ml[unit + i];
    const at_f32x4_t y = s_o[tid + i * TL];
    const float f = factor(ml.x, ml.y, m);
    sum = fmaf(ml.y, f, sum);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(y[e], f, o[e]);
  }
  store4(reinterpret_cast<OT*>(a.out) + (long long)x * D + 4 * t4, o, 1.f / sum);
}

// Which kernel, and how heads are cut.  All times: us, bf16 rows and outputs, heads of 128 dims, unless they say otherwise.
//  - Narrow, where the columns of a head are at most two blocks of 32, or where there is little to do at all (columns * rows up to 2^23: 16 nodes of 28/4 heads
//    of 2048 rows 13.8, by the wide kernel 14.4; 64 nodes of 32/8 heads of 4096 rows 18.9 and 28.1; but 32 nodes of 4 x 32/8 heads of 16384 rows 88 and 72).
//  - As many pieces as there are workgroups at once: even heads one workgroup per compute unit, whose four waves have all the loads on their way that memory
//    needs (32 nodes of 128 heads of 16384 rows, fp32 outputs 184, with two 193, with one and a half 200; of 4 x 32/8 heads of 16384 72, with two 76); 4-bit rows, bound by
//    their conversion, two (5 nodes of 64 heads of 8192 rows 24.6, with one 28.3).  Uneven heads make half a piece more each, and XCDs do not get the same: 448 of 512
//    (8 nodes of 128 heads of 4096 rows of 16 / 8 / 4 bits 59 / 37 / 33, with 512 63 / 42 / 38; of 8192 rows 106 / 63 / 52 and 112 / 70 / 63; of 2048 34.5 / 22.4 / 21.2 and
//    34.1 / 21.9 / 20.7; with 384 the same, but 80 heads of 3000 rows of 64 dims 18.3 / 15.7 / 16.1 instead of 17.2 / 15.1 / 15.4; with 320 128 heads of 2048 39.9).
//    Heads are even where the cache keeps everything.  (Not where the host has heard that they are: nothing here but the grid depends on what it knows of lengths, so
//    that a call gives the same bits before and after they have reached it, and when it is replayed.)
//  - But a piece costs its partial results, too: with n pieces per head 0.06 ns * columns * rows / n of arithmetic, 0.17 ns * columns * heads * n of traffic, which is least
//    at rows per piece = sqrt(3 * rows * heads), and some tiles of latency whatever it has, which small calls cannot hide and which speaks for shorter ones.  Measured, with 1.4 /
//    2 / 3 in the place of 3: 4 nodes of 32 heads of 2048 rows 15.2 / 13.2 / 13.5, 16 nodes of 4 x 32/8 heads 22.4 / 18.4 / 19.0, 8 of 128 heads 34.0 / 34.0 / 35.7, 16 of 28/4 heads
//    13.7 / 13.8 / 13.2, 9 of 20 heads of 5000 rows of 64 dims 13.1 / 13.3 / 12.4, 3 of 64 heads of 6000 8-bit rows 30.0 / 30.1 / 26.7.
//  - Up to 512 rows one piece, whose results need no second launch (8 heads of 256 rows 7.3, in two pieces 10.1).
constexpr double TREE_LITTLE = 8388608.;
constexpr int TREE_ONE_PIECE = 512, TREE_LEAST_ROWS = 128, TREE_MOST_PIECES = 512;       // (more pieces of a head than the chip takes at once only cost room)
// wc: blocks of columns of a workgroup (0: tree_narrow_kernel); usual: pieces of the longer heads, for which the join is laid out; slots: pieces of the grid
struct TreePlan { int wc, groups, chunk_rows, max_chunks, usual, slots; };
static TreePlan tree_plan(const Dims& dm, const madakv_config& c, int T, int longest_rows) {
  TreePlan p;
  const int R = dm.G * T;
  const bool even = c.budget >= c.ctx_len;
  const long long typical = std::min(c.budget, c.ctx_len);
  p.wc = R <= 64 || (double)dm.heads * R * typical <= TREE_LITTLE ? 0 : R <= 128 || c.dtype != MADAKV_BF16 ? 4 : 8;
  p.groups = p.wc ? (R + 32 * p.wc - 1) / (32 * p.wc) : (R + 31) / 32;
  const bool large = c.dtype != MADAKV_BF16 && dm.d == 128;              // (rows of 512 bytes: LDS has room for one workgroup)
  const int resident = large || p.wc == 8 || (even && !(p.wc == 0 && c.cache_fp8 == CACHE_E2M1)) ? 256 : even || p.wc ? 512 : 448;
  double want = (double)resident / ((double)dm.heads * p.groups);         // pieces per head
  if (want >= 2) want = std::floor(want);
  const double each = want < 1 ? 2. * typical : typical / (want - 0.375); // (cut_of: an eighth more than `want` of these is still `want`)
  const double worth = typical <= TREE_ONE_PIECE ? TREE_ONE_PIECE : std::max<double>(TREE_LEAST_ROWS, std::sqrt(2. * typical * dm.heads));
  p.chunk_rows = (int)std::ceil(std::max(each, worth));
  p.max_chunks = (int)std::min<long long>(TREE_MOST_PIECES, (std::max(2, c.hcc_rho) * typical + p.chunk_rows - 1) / p.chunk_rows);
  const auto pieces = [&](long long rows) { return (int)std::min<long long>(p.max_chunks, std::max<long long>(1, (rows - p.chunk_rows / 8 + p.chunk_rows - 1) / p.chunk_rows)); };      // (see cut_of)
  p.usual = pieces(even ? typical + c.max_new_tokens : 2 * typical);
  p.slots = pieces(std::min(longest_rows, c.ctx_len + c.max_new_tokens));
  return p;
}
size_t tree_ws_bytes(const Dims& dm, const madakv_config& c, int T, int longest_rows) {
  const int slots = tree_plan(dm, c, T, longest_rows).slots;
  return slots == 1 ? 16 : (size_t)dm.heads * slots * dm.G * T * (dm.d + 2) * sizeof(float);
}

template <typename T, typename OT, int CACHE, int D>
static hipError_t launch_tree(const Dims& dm, const TreeArgs& a, const TreePlan& p, hipStream_t st) {
  const dim3 grid(dm.heads * p.groups, p.slots);
  if (p.wc == 0) hipLaunchKernelGGL((tree_narrow_kernel<T, OT, CACHE, D>), dim3(dm.heads, p.slots * p.groups), dim3(256), 0, st, a);
  else if (p.wc == 4) hipLaunchKernelGGL((tree_attn_kernel<T, OT, CACHE, D, 4>), grid, dim3(256), 0, st, a);
  else if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((tree_attn_kernel<T, OT, CACHE, D, 8>), grid, dim3(512), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.slots == 1) return e;
  constexpr int UNITS = 256 / (D / 4);
  int shift = 0;
  while (2 << shift <= UNITS && 8 << shift < p.usual) ++shift;
  const int n = dm.heads * a.R, per = UNITS >> shift;
  hipLaunchKernelGGL((tree_join_kernel<OT, D>), dim3((n + per - 1) / per), dim3(256), 0, st, a, n, shift);
  return hipGetLastError();
}
template <typename T, typename OT, int CACHE>
static hipError_t launch_tree_d(const Dims& dm, const TreeArgs& a, const TreePlan& p, hipStream_t st) {
  return dm.d == 128 ? launch_tree<T, OT, CACHE, 128>(dm, a, p, st) : launch_tree<T, OT, CACHE, 64>(dm, a, p, st);
}
template <int CACHE>
static hipError_t launch_tree_o(const Dims& dm, const madakv_config& c, const TreeArgs& a, const TreePlan& p, hipStream_t st) {
  return c.out_fp32 ? launch_tree_d<uint16_t, float, CACHE>(dm, a, p, st) : launch_tree_d<uint16_t, uint16_t, CACHE>(dm, a, p, st);
}
hipError_t launch_tree_attn(const Dims& dm, const madakv_config& c, int T, const void* q, const void* k_new, const void* v_new, const void* tree, const void* k_c,
                            const void* v_c, const int64_t* kv_off, const int32_t* kv_len, void* out, void* ws, long long capacity_tokens, int longest_rows,
                            const Paging& pg, int layer0, hipStream_t st) {
  const TreePlan p = tree_plan(dm, c, T, longest_rows);
  const long long head0 = (long long)layer0 * dm.B * dm.H;
  TreeArgs a;
  a.q = q; a.k_new = k_new; a.v_new = v_new; a.k_c = static_cast<const unsigned char*>(k_c); a.v_c = static_cast<const unsigned char*>(v_c);
  a.tree = static_cast<const unsigned long long*>(tree); a.kv_off = kv_off; a.kv_len = kv_len; a.out = out;
  a.B = dm.B; a.H = dm.H; a.G = dm.G; a.T = T; a.R = dm.G * T; a.groups = p.groups;
  a.chunk_rows = p.chunk_rows; a.max_chunks = std::min(p.max_chunks, p.slots); a.slots = p.slots;
  a.part = static_cast<float*>(ws); a.part_ml = a.part + (size_t)dm.heads * p.slots * a.R * dm.d;
  a.capacity = capacity_tokens;
  a.page_rows = pg.page_rows; a.tbl_entries = pg.entries; a.page_shift = 0;
  while (pg.page_rows && (1 << a.page_shift) < pg.page_rows) ++a.page_shift;
  a.page_tbl = pg.page_rows ? pg.table + head0 * pg.entries : nullptr;
  a.scale_log2 = (c.softmax_scale > 0.f ? c.softmax_scale : 1.0f / sqrtf((float)dm.d)) * 1.4426950408889634f;
  if (c.dtype != MADAKV_BF16) return launch_tree_d<float, float, 0>(dm, a, p, st);
  if (c.cache_fp8 == CACHE_E2M1) return launch_tree_o<CACHE_E2M1>(dm, c, a, p, st);
  if (c.cache_fp8 == CACHE_E4M3) return launch_tree_o<CACHE_E4M3>(dm, c, a, p, st);
  return launch_tree_o<0>(dm, c, a, p, st);
}

// ---- the accepted nodes' rows ---------------------------------------------------------------------------
// One workgroup per head.  The new rows' places follow from what the eviction left the head (Meet::len1) and `start`, not from its present
// length: the call can be repeated, and can take rows back.
struct CommitArgs {
  const unsigned char* k_new; const unsigned char* v_new; const int32_t* path; const int32_t* n_path; const int32_t* start;
  unsigned char* k_c; unsigned char* v_c; const int64_t* kv_off; int32_t* kv_len;
  const int32_t* len1;                 // of the call's first head
  int B, H, T, max_path, most;
  long long capacity;
  int page_rows, page_shift, tbl_entries;
  int32_t* page_tbl;                   // of the call's first head
  unsigned long long* pool_top;
  long long region_pages;
};

// What it takes is a chain of waits (lengths and places, the nodes, their rows) and the bytes: 6 of 16 nodes of 32 layers of 4 x 32 heads, 8-bit rows, 6.6 us by
// workgroups of 128 threads, all resident at once (256: 7.4; and 7.9 where every entry is asked for only when it is needed).  One layer of 4 heads: 2.8 us.
constexpr int COMMIT_THREADS = 128;
template <typename T, int CACHE, int D>
__global__ __launch_bounds__(COMMIT_THREADS) void tree_commit_kernel(CommitArgs a) {
  constexpr int EPL = 16 / (int)sizeof(T), LPR = D / EPL;      // elements per thread, threads per row
  __shared__ int s_path[64];
  const int tid = threadIdx.x;
  const long long hidx = blockIdx.x;
  const int b = (int)(hidx / a.H % a.B);
  // (everything that the rows' places depend on is sent for at once: the kernel is a chain of waits)
  const int kept = a.len1[hidx] - 1, len = a.kv_len[hidx], from = a.start[b], named = a.n_path[b], lane = tid & 63;
  const long long off = a.kv_off[hidx];
  const int step_node = a.path[b * a.max_path + min(lane, a.max_path - 1)];
  if (kept <= 0 || len <= 0) return;                           // never evicted, or an empty segment, which stays empty
  const int have = len - kept;
  if (from < 0 || from > have || (a.page_rows && from != have)) {
    // rows that are not there: the head is left as it is, but for what is more than `most`
    if (!a.page_rows && have > a.most && tid == 0) a.kv_len[hidx] = kept + a.most;
    return;
  }
  int n = max(0, min(min(named, a.max_path), a.most - from));
  {                                                            // (every wave for itself: an entry that is no node ends the path)
    const int node = lane < n ? step_node : 0;
    const unsigned long long bad = __builtin_amdgcn_ballot_w64(lane < n && (node < 0 || node >= a.T));
    if (bad) n = min(n, (int)__builtin_ctzll(bad));
    if (tid < 64) s_path[tid] = node;
  }
  RowMap at;
  at.off = off; at.init_rows = 0x7fffffff; at.tbl = nullptr; at.shift = 0; at.fresh_slot = -1; at.fresh_page = 0;
  if (a.page_rows) {
    int32_t* tbl = a.page_tbl + hidx * a.tbl_entries;
    at.tbl = tbl; at.shift = a.page_shift; at.init_rows = tbl[0] << a.page_shift;
    if (tid == 0) {
      const int q0 = len - at.init_rows, P = a.page_rows;
      const int j0 = q0 <= 0 ? 0 : (q0 + P - 1) >> a.page_shift, j1 = q0 + n <= 0 ? 0 : (q0 + n + P - 1) >> a.page_shift;     // pages the head has, will have
      if (j1 > j0) {
        const unsigned long long nth = atomicAdd(a.pool_top + b, (unsigned long long)(j1 - j0));
        for (int j = j0; j < j1; ++j) tbl[1 + j] = (int32_t)((b + 1) * a.region_pages - 1 - (long long)nth - (j - j0));
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < n * 2 * LPR; i += COMMIT_THREADS) {
    const int which = i / LPR & 1, piece = i % LPR, step = i / (2 * LPR);
    const unsigned char* src = (which ? a.v_new : a.k_new) + ((hidx * a.T + s_path[step]) * D + piece * EPL) * (long long)sizeof(T);
    const uint4 x = *reinterpret_cast<const uint4*>(src);
    const long long row = at(kept + from + step);
    unsigned char* cache = which ? a.v_c : a.k_c;
    if constexpr (CACHE == 0) {
      *reinterpret_cast<uint4*>(cache + (row * D + piece * EPL) * (long long)sizeof(T)) = x;
    } else if constexpr (CACHE == CACHE_E4M3) {
      *reinterpret_cast<uint2*>(cache + row * D + piece * EPL) = make_uint2(e4m3_of(x.x, x.y), e4m3_of(x.z, x.w));
    } else {                                                   // (rows are whole quads of threads)
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
      uint32_t scale;
      const uint32_t code = mx_encode8(w, scale);
      *reinterpret_cast<uint32_t*>(cache + row * (D / 2) + piece * 4) = code;
      if ((piece & 3) == 0) cache[a.capacity * (D / 2) + row * (D / MX_BLOCK) + piece / 4] = (uint8_t)scale;
    }
  }
  if (tid == 0) a.kv_len[hidx] = kept + (a.page_rows ? from + n : min(from + n, a.most));      // (a start past `most`: cut; pages are not given back)
}

template <typename T, int CACHE>
static hipError_t launch_commit(const Dims& dm, const CommitArgs& a, hipStream_t st) {
  if (dm.d == 128) hipLaunchKernelGGL((tree_commit_kernel<T, CACHE, 128>), dim3(dm.heads), dim3(COMMIT_THREADS), 0, st, a);
  else hipLaunchKernelGGL((tree_commit_kernel<T, CACHE, 64>), dim3(dm.heads), dim3(COMMIT_THREADS), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_tree_commit(const Dims& dm, const madakv_config& c, int T, const void* k_new, const void* v_new, const int32_t* path, const int32_t* n_path, int max_path,
                              const int32_t* start, int most, void* k_c, void* v_c, const int64_t* kv_off, int32_t* kv_len, const Meet& meet, long long capacity_tokens,
                              const Paging& pg, int layer0, hipStream_t st) {
  const long long head0 = (long long)layer0 * dm.B * dm.H;
  CommitArgs a;
  a.k_new = static_cast<const unsigned char*>(k_new); a.v_new = static_cast<const unsigned char*>(v_new); a.path = path; a.n_path = n_path; a.start = start;
  a.k_c = static_cast<unsigned char*>(k_c); a.v_c = static_cast<unsigned char*>(v_c); a.kv_off = kv_off; a.kv_len = kv_len; a.len1 = meet.len1 + head0;
  a.B = dm.B; a.H = dm.H; a.T = T; a.max_path = max_path; a.most = most; a.capacity = capacity_tokens;
  a.page_rows = pg.page_rows; a.tbl_entries = pg.entries; a.page_shift = 0;
  while (pg.page_rows && (1 << a.page_shift) < pg.page_rows) ++a.page_shift;
  a.page_tbl = pg.page_rows ? pg.table + head0 * pg.entries : nullptr; a.pool_top = pg.pool_top;
  a.region_pages = pg.page_rows ? pg.region_tokens / pg.page_rows : 0;
  if (c.dtype != MADAKV_BF16) return launch_commit<float, 0>(dm, a, st);
  if (c.cache_fp8 == CACHE_E2M1) return launch_commit<uint16_t, CACHE_E2M1>(dm, a, st);
  if (c.cache_fp8 == CACHE_E4M3) return launch_commit<uint16_t, CACHE_E4M3>(dm, a, st);
  return launch_commit<uint16_t, 0>(dm, a, st);
}

}  // namespace madakv
