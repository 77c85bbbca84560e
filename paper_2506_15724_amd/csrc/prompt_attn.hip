// Causal attention of a whole prompt (paper Sec. 3.1 Eq. 5 at every position) with grouped heads: per query head
//   out(r) = sum over i in the row's sequence, i <= r, of exp(scale * q_r . k_i - lse_r) v_i,   lse_r = log of the sum of exp(scale * q_r . k_i)
// The positions of a batch item are one sequence, or several that follow each other; positions of none are left alone.
//
// A workgroup has 32 query rows per wave of one query head and goes over the keys that they see, 64 at a time: K and V come straight into LDS (16 bytes per
// lane), one tile ahead of the arithmetic, which attn_tile.h describes.  A wave leaves out the tiles that none of its rows sees; the
// causal mask and the starts of sequences are looked at in the tiles that they cut, where keys that no row may see count for nothing
// whatever they hold: an infinite or undefined element of V, which zero weights would not keep out of a matrix product, is found by what it
// does to the output, and the workgroup goes over its keys a second time, adding the rows of V of such tiles one by one.
// Work: 4 D operations per query head, row and key it sees; bytes do not count (28/4 heads of 16384 rows: 1.9 TFLOP, 270 MB).  Bound by power there: 1.09-1.14 PFLOP/s
// (1.69-1.79 ms) with the matrix unit busy 62% of the time at 1.7 GHz, 1.35 of the same code on zeros.  Short prompts are bound by what every workgroup has at its beginning,
// on the diagonal and at its end: 4 x 32/8 heads of 2048 rows 150 us (0.91 PFLOP/s), 32/8 of 1024 20.
#include "attn_tile.h"

#include <algorithm>
#include <climits>
#include <type_traits>

namespace madakv {

// 16 bytes per lane from `at` + base of a buffer to LDS address dst + 16 lane, zeros past the buffer's end.  Written out, because the compiler
// would otherwise wait for all such loads in flight before every LDS access it sees; the loop's own waits are in `landed`.
__device__ __forceinline__ void tile_load(at_u32x4_t buffer, uint32_t dst, int at, int base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(dst), "v"(at), "s"(buffer), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ at_u32x4_t buffer_words(const void* p, int bytes) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  return at_u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32)), (uint32_t)bytes, 0x00020000u};
}

constexpr int PA_WAVES = 4;

struct PromptAttnArgs {
  const void* q; const void* k; const void* v;       // [n, B, Hq, L, d], [n, B, H, L, d]
  void* out; float* row_lse;                         // row_lse null: not wanted
  const int32_t* seq_off;                            // [B][n_seq + 1] or null
  int n_seq, B, Hq, G, L;
  int blocks, heads;                                 // workgroups of a query head, query heads
  float scale_log2;
};

// T: Q, K, V; OT: out (bf16 bits or float); WK waves share 32 rows and take halves of every tile; WAVES: of a SIMD
template <typename T, typename OT, int D, int WK, int WAVES>
__global__ __launch_bounds__(PA_WAVES * 64) __attribute__((amdgpu_waves_per_eu(WAVES, WAVES))) void prompt_attn_kernel(PromptAttnArgs a) {
  using Tile = AttnTile<T, D>;
  constexpr int PARTS = sizeof(T) == 2 && sizeof(OT) == 4 ? 3 : 1;
  constexpr int NW = PA_WAVES, BQ = NW / WK * 32, ROWB = Tile::ROWB, PPR = Tile::PPR;
  constexpr int LPT = ATT_TILE * PPR / (NW * 64);    // load instructions per wave, tile and tensor, 1 KB each
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * Tile::BYTES];       // two tiles of K, two of V; with WK = 2 the second halves' results
  __shared__ int s_start[BQ], s_base;
  __shared__ float s_ml[WK == 2 ? BQ : 1][2];

  // Workgroup -> query head and block of rows, the blocks that see the most keys first.  Workgroups go to the 8 XCDs in turn: each takes an eighth of the
  // heads, whose keys its L2 holds some of, and an eighth of the blocks of the heads that are left; where KV heads come in eights every XCD has
  // its part of every batch item, whose lengths may differ.  Eight blocks of all its heads, `rest` of the others: a period.
  // (Head after head instead: 28/4 heads of 6001 rows 275 us, now 252; four prompts of 1348 to 1873 rows, 32/8 heads, 150, now 113; of 16384 rows 1760, now 1687.)
  const int xcd = (int)(blockIdx.x & 7), nth = (int)(blockIdx.x >> 3), whole = a.heads / 8, rest = a.heads % 8;
  const int period = nth / a.heads, e = nth - period * a.heads;
  int qh, rb;
  if (e < rest) {
    const int id = (period * rest + e) * 8 + xcd;
    rb = id / rest;
    qh = whole * 8 + id - rb * rest;
  } else {
    const int id = period * 8 * whole + e - rest;
    rb = id / whole;
    const int i = id - rb * whole;
    qh = a.heads % (8 * a.G) == 0 ? (i / a.G * 8 + xcd) * a.G + i % a.G : xcd * whole + i;
  }
  if (rb >= a.blocks) return;
  const int r0 = (a.blocks - 1 - rb) * BQ;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;

  // the rows [first, end) that are in some sequence, the start of every row's own
  int first = 0, end = a.L, kmin = 0, start = 0;
  const int block = wave / WK, wk = wave % WK, w0 = r0 + block * 32;
  if (a.seq_off) {
    const int32_t* off = a.seq_off + (long long)(qh / a.Hq % a.B) * (a.n_seq + 1);
    first = max(off[0], 0);
    end = min(off[a.n_seq], a.L);
    if (r0 >= end || r0 + BQ <= first) return;
    kmin = start = first;
  }
  if (a.seq_off && a.n_seq > 1) {
    const int32_t* off = a.seq_off + (long long)(qh / a.Hq % a.B) * (a.n_seq + 1);
    if (tid < BQ) s_start[tid] = 0;
    if (tid == 0) s_base = 0;
    __syncthreads();
    for (int i = tid; i < a.n_seq; i += NW * 64) {
      const int o = max(off[i], 0);
      if (o <= r0) atomicMax(&s_base, o);
      else if (o < r0 + BQ) s_start[o - r0] = o;
    }
    __syncthreads();
    kmin = r0 >= first ? s_base : first;
    start = s_base;                                  // the latest start in front of every row: a running maximum, 32 rows at a time
    for (int c = 0; c <= block; ++c) {
      const int before = __builtin_amdgcn_readlane(start, 31);
      start = s_start[c * 32 + col];
      for (int s = 1; s < 32; s *= 2) { const int y = __shfl_up(start, s, 32); start = col >= s ? max(start, y) : start; }
      start = max(start, before);
    }
  }
  // the wave's rows [wfirst, wlast]; a column without one has a copy of another one's, which is not stored
  const int wfirst = max(w0, first), wlast = min(w0 + 31, end - 1);
  const bool any = wfirst <= wlast;                  // uniform
  const int row = any ? min(max(w0 + col, wfirst), wlast) : min(w0 + col, a.L - 1);
  const int min_start = __builtin_amdgcn_readlane(start, any ? wfirst - w0 : 0), max_start = __builtin_amdgcn_readlane(start, any ? wlast - w0 : 0);       // (starts ascend)
  start = w0 + col < wfirst ? min_start : w0 + col > wlast ? max_start : start;
  const int tile0 = kmin / ATT_TILE, ntiles = (min(r0 + BQ, end) + ATT_TILE - 1) / ATT_TILE - tile0;
  // The wave's subtiles of 32 keys: of tile t both (number j = 2 t, 2 t + 1), or with WK = 2 one (j = t).  Its rows see something of those from j0 to j1 - 1.
  const auto first_key = [&](int j) { return (tile0 * 2 + (WK == 2 ? 2 * j + wk : j)) * 32; };
  const auto row_in_tile = [&](int j) { return (WK == 2 ? wk : j & 1) * 32; };
  const auto number = [&](int x) { x -= tile0 * 2; return WK == 2 ? (x - wk + 1) >> 1 : x; };          // of the first of them from key 32 x on
  const int j0 = any ? number(min_start / 32) : 0, j1 = any ? number(wlast / 32 + 1) : 0;

  // Tiles -> LDS.  Load j of wave w fills pieces [(w LPT + j) 64, + 64) of the tile, lane i slot P mod PPR of row P / PPR, P = (w LPT +
  // j) 64 + i.  Through buffers that end with the prompt: rows past its end are zeros.
  const long long kvh = qh / a.G;
  const at_u32x4_t kb = buffer_words(reinterpret_cast<const T*>(a.k) + kvh * a.L * D, a.L * ROWB), vb = buffer_words(reinterpret_cast<const T*>(a.v) + kvh * a.L * D, a.L * ROWB);
  int koff[LPT], voff[LPT];
#pragma unroll
  for (int j = 0; j < LPT; ++j) {
    const int piece = (wave * LPT + j) * 64 + lane, r = piece / PPR, s = piece % PPR;
    koff[j] = r * ROWB + Tile::k_slot(r, s) * 16;    // (an exclusive or: the piece in slot s is the slot of piece s)
    voff[j] = r * ROWB + Tile::v_slot(r, s) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  const auto issue = [&](at_u32x4_t buffer, const int (&off)[LPT], int slot, int t) {
#pragma unroll
    for (int j = 0; j < LPT; ++j) tile_load(buffer, lds0 + (uint32_t)(slot * Tile::BYTES + (wave * LPT + j) * 1024), off[j], (tile0 + t) * (ATT_TILE * ROWB));
  };

  // Phase t of the loop below reads tile t of K and tile t - WK of V and sends for the ones after them.
  const auto send = [&](int t) {
    if (t + 1 < ntiles) issue(kb, koff, (t + 1) & 1, t + 1);
    const int v = t + 1 - WK;
    if (v >= 0 && v < ntiles) issue(vb, voff, 2 + (v & 1), v);
  };
  typename Tile::Query q;
  Tile::load(q, reinterpret_cast<const T*>(a.q) + ((long long)qh * a.L + row) * D, half);

  AttnState<D> st;
  using Weights = typename Tile::template Weights<PARTS>;
  Weights w, w_next;                                 // of the subtile before the one that s has the logits of
  at_f32x16_t s, s_next;
  const auto cut = [&](int j) {                      // some row does not see all of the subtile
    const int k32 = first_key(j);
    return k32 + 31 > wfirst || k32 < max_start;
  };
  // logits -> weights against the present references; whether these still serve
  const auto fast = [&](const at_f32x16_t& x, Weights& to) {
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(x[i], a.scale_log2, -st.ref));
    const float t = st.sum + sum16(p);
    Tile::template pack<PARTS>(p, to);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(t < ATT_FAR)) != 0, 0)) return false;
    st.sum = t;
    return true;
  };
  const auto pass = [&](auto careful) {
    st.clear();
    send(-1);
    if (!decltype(careful)::value) Tile::await(q);
    // Step j: the logits of subtile j + 1, the weights of subtile j, and what subtile j - 1 adds to the output.  None of them needs another
    // one's results: the matrix instructions of the first and the last run beside the vector instructions of the second.
    // Phase t has steps 2 t - 1 and 2 t, or with WK = 2 step t - 1.
    const auto begin = [&](int t) {
      // the phase's tiles are there for everybody, and nobody reads those before them any more
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      send(t);
    };
    const auto k_tile = [&](int t) { return lds + (t & 1) * Tile::BYTES; };
    const auto v_tile = [&](int t) { return lds + (2 + ((t - WK) & 1)) * Tile::BYTES; };
    // phases t0 .. t1 - 1: every row sees all keys of their steps
    const int ja = max(j0 + 1, number((max_start + 31) / 32)), jb = min(j1 - 1, number((wfirst + 1) / 32));          // steps [ja, jb)
    const int t0 = decltype(careful)::value ? INT_MAX : WK == 2 ? ja + 1 : (ja + 2) >> 1, t1 = WK == 2 ? jb + 1 : (jb + 1) >> 1;
    const int phases = ntiles + WK;
    int t = 0;
#pragma unroll 1
    while (t < phases) {
      begin(t);
      bool formed = false;                           // the step's logits and sums are there
      int j = WK == 2 ? t - 1 : 2 * t - 1;
      if (!decltype(careful)::value && t >= t0 && t < t1) {
#pragma unroll 1
        for (;;) {
          const unsigned char* kt = k_tile(t);
          const unsigned char* vt = v_tile(t);
          j = WK == 2 ? t - 1 : 2 * t - 1;
          s_next = Tile::scores(kt, row_in_tile(j + 1), lane, q);
          Tile::template add<PARTS>(vt, row_in_tile(j - 1), lane, w, st.o);
          formed = !fast(s, w_next);
          if (formed) break;
          if constexpr (WK == 1) {
            ++j;
            s = Tile::scores(kt, row_in_tile(j + 1), lane, q);
            Tile::template add<PARTS>(vt, row_in_tile(j - 1), lane, w_next, st.o);
            formed = !fast(s_next, w);
            if (formed) {
              const at_f32x16_t x = s;
              s = s_next; s_next = x;
              break;
            }
          } else {
            s = s_next; w = w_next;
          }
          ++t;
          if (t >= t1) break;
          begin(t);
        }
        if (!formed) continue;
      }
      const unsigned char* kt = k_tile(t);
      const unsigned char* vt = v_tile(t);
#pragma unroll 1
      for (const int last = WK == 2 ? t - 1 : 2 * t; j <= last; ++j) {
        if (!formed) {
          if (j + 1 >= j0 && j + 1 < j1) s_next = Tile::scores(kt, row_in_tile(j + 1), lane, q);
          if (j - 1 >= j0 && j - 1 < j1) {
            if (decltype(careful)::value && (PARTS > 1 || cut(j - 1))) {
#pragma unroll 1
              for (int key = 0; key < 32; ++key) {   // its weight is with one of the column's lanes, element i of its 16
                const int i = 4 * (key >> 3) + (key & 3), owner = col + 32 * ((key >> 2) & 1), k = first_key(j - 1) + key;
                const float x = __shfl(Tile::template weight<PARTS>(w, i), owner, 64);
                if (k > row || k < start) continue;
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                  for (int g = 0; g < 4; ++g) {
                    const at_f32x4_t y = Tile::value4(vt, row_in_tile(j - 1) + key, 32 * db + 8 * g + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.o[db][4 * g + e] = fmaf(x, y[e], st.o[db][4 * g + e]);
                  }
              }
            } else {
              Tile::template add<PARTS>(vt, row_in_tile(j - 1), lane, w, st.o);
            }
          }
        }
        formed = false;
        if (j >= j0 && j < j1) {
          float p[16], more;
          if (cut(j)) {
            const int behind = first_key(j) + 4 * half - start;          // (a key that the row sees: start <= key <= row)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = (unsigned)(behind + key_of(i, 0)) <= (unsigned)(row - start) ? s[i] : -__builtin_inff();
          }
          attn_look<D>(st, s, p, more, a.scale_log2);
          st.sum += more;
          Tile::template pack<PARTS>(p, w);
        }
        s = s_next;
      }
      ++t;
    }
  };
  pass(std::false_type{});
  // outputs that are no numbers: the formula's, or those of rows of V that nobody may see
  if (__builtin_expect(__syncthreads_or(any && not_finite(st)), 0)) {
    pass(std::true_type{});
    __syncthreads();
  }
  float sum = both_sum(st.sum);
  if constexpr (WK == 2) {                           // the second half's results go through LDS
    constexpr int RS = D + 4;
    static_assert(BQ * RS * 4 <= 4 * Tile::BYTES, "the results must fit the tiles' place");
    float* result = reinterpret_cast<float*>(lds) + (block * 32 + col) * RS;
    if (wk) {
      if (half == 0) { s_ml[block * 32 + col][0] = st.ref; s_ml[block * 32 + col][1] = sum; }
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<at_f32x4_t*>(result + 32 * db + 8 * g + 4 * half) = at_f32x4_t{st.o[db][4 * g], st.o[db][4 * g + 1], st.o[db][4 * g + 2], st.o[db][4 * g + 3]};
    }
    __syncthreads();
    if (wk) return;
    merge_halves<D>(st, sum, s_ml[block * 32 + col], result, half);
  }
  if (!any) return;

  const bool mine = w0 + col == row;
  const long long o = (long long)qh * a.L + row;
  if (a.row_lse && mine && half == 0) a.row_lse[o] = (st.ref + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
  store_column<OT, D>(reinterpret_cast<OT*>(a.out) + o * D, mine, half, st.o, 1.f / sum);
}

template <typename T, typename OT, int D, int WK, int WAVES>
static hipError_t launch_rows(PromptAttnArgs& a, int heads, hipStream_t st) {
  constexpr int BQ = PA_WAVES / WK * 32;
  a.blocks = (a.L + BQ - 1) / BQ;
  a.heads = heads;
  const long long periods = (a.blocks + 7) / 8;                // (see the kernel)
  hipLaunchKernelGGL((prompt_attn_kernel<T, OT, D, WK, WAVES>), dim3((unsigned)(periods * heads * 8)), dim3(PA_WAVES * 64), 0, st, a);
  return hipGetLastError();
}
template <typename T, typename OT, int D>
static hipError_t launch_pa(PromptAttnArgs& a, int heads, hipStream_t st) {
  const long long blocks = (long long)heads * ((a.L + 127) / 128);
  // Few blocks: two waves share 32 rows and take half of the keys each, so that the longest rows take half as long (us, 32 rows per wave / shared: 128 blocks of
  // 2048 positions 38.3 / 28.7, 256 of 1024 24.8 / 21.5; 448 of 2048 47.4 / 49.2, 512 of 2048 50.4 / 54.7, 1024 of 64 dims 325 / 376).
  if (blocks <= 384) return launch_rows<T, OT, D, 2, sizeof(T) == 2 ? 2 : 1>(a, heads, st);
  // Waves of 64 dims are bound by the exponentials: three per SIMD (two: 1024 blocks 325 instead of 307, 1504 173 and 166, 3584 1032 and 974).
  return launch_rows<T, OT, D, 1, sizeof(T) == 4 ? 1 : D == 64 ? 3 : 2>(a, heads, st);
}
hipError_t launch_prompt_attn(const Dims& dm, const madakv_config& c, const void* q, const void* k, const void* v, const int32_t* seq_off, int n_seq,
                              void* out, float* row_lse, hipStream_t st) {
  PromptAttnArgs a;
  a.q = q; a.k = k; a.v = v; a.out = out; a.row_lse = row_lse; a.seq_off = seq_off; a.n_seq = n_seq;
  a.B = dm.B; a.Hq = dm.Hq; a.G = dm.G; a.L = dm.L;
  a.scale_log2 = (c.softmax_scale > 0.f ? c.softmax_scale : 1.0f / sqrtf((float)dm.d)) * 1.4426950408889634f;
  const int heads = dm.n * dm.B * dm.Hq;
  if (c.dtype != MADAKV_BF16) return dm.d == 128 ? launch_pa<float, float, 128>(a, heads, st) : launch_pa<float, float, 64>(a, heads, st);
  if (c.out_fp32) return dm.d == 128 ? launch_pa<uint16_t, float, 128>(a, heads, st) : launch_pa<uint16_t, float, 64>(a, heads, st);
  return dm.d == 128 ? launch_pa<uint16_t, uint16_t, 128>(a, heads, st) : launch_pa<uint16_t, uint16_t, 64>(a, heads, st);
}

}  // namespace madakv
