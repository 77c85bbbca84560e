// Causal attention of a whole prompt (paper Sec. 3.1 Eq. 5 at every position) with grouped heads: per query head
//   out(r) = sum over i in the row's sequence, i <= r, of exp(scale * q_r . k_i - lse_r) v_i,   lse_r = log of the sum of exp(scale * q_r . k_i)
// The positions of a batch item are one sequence, or several that follow each other; positions of none are left alone.
//
// A workgroup has 32 query rows per wave of one query head and goes over the keys that they see, 64 at a time: K and V come straight into LDS (16 bytes per
// lane), one tile ahead of the arithmetic, which attn_tile.h describes.  A wave leaves out the tiles that none of its rows sees; the
// causal mask and the starts of sequences are looked at in the tiles that they cut, where keys that no row may see count for nothing
// whatever they hold: an infinite or undefined element of V, which zero weights would not keep out of a matrix product, is found by what it
// does to the output, and the workgroup goes over its keys a second time, adding the rows of V of such tiles one by one.
#include "attn_tile.h"

#include <algorithm>

namespace madakv {

// 16 bytes per lane from `at` + base of a buffer to LDS address dst + 16 lane, zeros past the buffer's end.  Written out, because the compiler
// would otherwise wait for all such loads in flight before every LDS access it sees; the loop's own waits are in `landed`.
__device__ __forceinline__ void tile_load(at_u32x4_t buffer, uint32_t dst, int at, int base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(dst), "v"(at), "s"(buffer), "s"(base));
}
__device__ __forceinline__ at_u32x4_t buffer_words(const void* p, int bytes) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  return at_u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32)), (uint32_t)bytes, 0x00020000u};
}

struct PromptAttnArgs {
  const void* q; const void* k; const void* v;       // [n, B, Hq, L, d], [n, B, H, L, d]
  void* out; float* row_lse;                         // row_lse null: not wanted
  const int32_t* seq_off;                            // [B][n_seq + 1] or null
  int n_seq, B, Hq, G, L;
  int blocks, total;                                 // workgroups of a query head, of all
  float scale_log2;
};

// T: Q, K, V; OT: out (bf16 bits or float); NW waves of 32 NQ rows
template <typename T, typename OT, int D, int NW, int NQ>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 && NQ == 1 ? 2 : 1, sizeof(T) == 2 && NQ == 1 ? 2 : 1))) void prompt_attn_kernel(PromptAttnArgs a) {
  using Tile = AttnTile<T, D>;
  constexpr int PARTS = sizeof(T) == 2 && sizeof(OT) == 4 ? 3 : 1;
  constexpr int WR = NQ * 32, BQ = NW * WR, ROWB = Tile::ROWB, PPR = Tile::PPR;
  constexpr int LPT = ATT_TILE * PPR / (NW * 64);    // load instructions per wave, tile and tensor, 1 KB each
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * Tile::BYTES];       // two tiles of K, two of V
  __shared__ int s_start[BQ], s_base;

  const int per_xcd = (a.total + 7) / 8;
  const int idx = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if (idx >= a.total || (int)(blockIdx.x >> 3) >= per_xcd) return;
  const int qh = idx / a.blocks, r0 = (a.blocks - 1 - (idx - qh * a.blocks)) * BQ;       // (rows that see the most first)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;

  // the rows [first, end) that are in some sequence, the start of every row's own
  int first = 0, end = a.L, kmin = 0, start[NQ];
  const int w0 = r0 + wave * WR;
#pragma unroll
  for (int b = 0; b < NQ; ++b) start[b] = 0;
  if (a.seq_off) {
    const int32_t* off = a.seq_off + (long long)(qh / a.Hq % a.B) * (a.n_seq + 1);
    first = max(off[0], 0);
    end = min(off[a.n_seq], a.L);
    if (r0 >= end || r0 + BQ <= first) return;
    for (int i = tid; i < BQ; i += NW * 64) s_start[i] = 0;
    if (tid == 0) s_base = 0;
    __syncthreads();
    for (int i = tid; i < a.n_seq; i += NW * 64) {
      const int o = max(off[i], 0);
      if (o <= r0) atomicMax(&s_base, o);
      else if (o < r0 + BQ) s_start[o - r0] = o;
    }
    __syncthreads();
    kmin = r0 >= first ? s_base : first;
    // the latest start in front of every row: a running maximum, 32 rows at a time
    int carry = s_base;
    for (int c = 0; c < (wave + 1) * NQ; ++c) {
      int x = s_start[c * 32 + col];
      for (int s = 1; s < 32; s *= 2) { const int y = __shfl_up(x, s, 32); x = col >= s ? max(x, y) : x; }
      x = max(x, carry);
      carry = __builtin_amdgcn_readlane(x, 31);
#pragma unroll
      for (int b = 0; b < NQ; ++b) start[b] = c == wave * NQ + b ? x : start[b];
    }
  }
  // the wave's rows [wfirst, wlast]; a column without one has a copy of another one's, which is not stored
  const int wfirst = max(w0, first), wlast = min(w0 + WR - 1, end - 1);
  const bool any = wfirst <= wlast;                  // uniform
  int row[NQ], min_start = 0, max_start = 0;
  {
    int own[NQ];
#pragma unroll
    for (int b = 0; b < NQ; ++b) own[b] = start[b];
    const auto start_of = [&](int r) {               // of row w0 + r, r the same in all lanes
      int x = __builtin_amdgcn_readlane(own[0], r & 31);
#pragma unroll
      for (int b = 1; b < NQ; ++b) { const int y = __builtin_amdgcn_readlane(own[b], r & 31); x = r >= 32 * b ? y : x; }
      return x;
    };
    if (any) { min_start = start_of(wfirst - w0); max_start = start_of(wlast - w0); }       // (starts ascend)
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      const int r = w0 + 32 * b + col;
      row[b] = any ? min(max(r, wfirst), wlast) : min(r, a.L - 1);
      start[b] = r < wfirst ? min_start : r > wlast ? max_start : start[b];
    }
  }
  const int tile0 = kmin / ATT_TILE, ntiles = (min(r0 + BQ, end) + ATT_TILE - 1) / ATT_TILE - tile0;
  // the subtiles of 32 keys that the wave's rows see something of, counted from tile0
  const int u0 = any ? min_start / 32 - tile0 * 2 : 0, u1 = any ? wlast / 32 + 1 - tile0 * 2 : 0;

  typename Tile::Query q[NQ];
#pragma unroll
  for (int b = 0; b < NQ; ++b) Tile::load(q[b], reinterpret_cast<const T*>(a.q) + ((long long)qh * a.L + row[b]) * D, half);

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

  AttnState<T, D, NQ> st;
  using Weights = typename Tile::template Weights<PARTS>;
  Weights w[NQ], w_next[NQ];                         // of the subtile before the one that s has the logits of
  at_f32x16_t s[NQ], s_next[NQ];
  bool careful = false;
  const auto cut = [&](int u) {                      // some row does not see all of the subtile
    const int k32 = (tile0 * 2 + u) * 32;
    return k32 + 31 > wfirst || k32 < max_start;
  };
  const auto row_in_tile = [](int u) { return (u & 1) * 32; };
  // logits -> weights against the present references; whether these still serve
  const auto fast = [&](const at_f32x16_t (&x)[NQ], Weights (&to)[NQ]) {
    float p[NQ][16], t[NQ];
    bool far = false;
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) p[b][i] = __builtin_amdgcn_exp2f(fmaf(x[b][i], a.scale_log2, -st.ref[b]));
      t[b] = st.sum[b] + sum16(p[b]);
      Tile::template pack<PARTS>(p[b], to[b]);
      far = far || !(t[b] < ATT_FAR);
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(far) != 0, 0)) return false;
#pragma unroll
    for (int b = 0; b < NQ; ++b) st.sum[b] = t[b];
    return true;
  };
  for (;;) {
    st.clear();
    issue(kb, koff, 0, 0);
    // Step u: the logits of subtile u + 1, the weights of subtile u, and what subtile u - 1 adds to the output.  None of them needs another
    // one's results: the matrix instructions of the first and the last run beside the vector instructions of the second.
    // Steps 2t - 1 and 2t read tile t of K and tile t - 1 of V.
#pragma unroll 1
    for (int t = 0; t <= ntiles; ++t) {
      // they are there for everybody, and nobody reads the tiles before them any more
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (t + 1 < ntiles) issue(kb, koff, (t + 1) & 1, t + 1);
      if (t < ntiles) issue(vb, voff, 2 + (t & 1), t);
      const unsigned char* kt = lds + (t & 1) * Tile::BYTES;
      const unsigned char* vt = lds + (2 + ((t + 1) & 1)) * Tile::BYTES;
      int u = 2 * t - 1;
      bool formed = false;                           // the step's logits and sums are there
      if (__builtin_expect(u - 1 >= u0 && u + 2 < u1 && !cut(u) && !cut(u + 1) && !careful, 1)) {
        Tile::template scores<NQ>(kt, 0, lane, q, s_next);
        Tile::template add<PARTS, NQ>(vt, 0, lane, w, st.o);
        formed = !fast(s, w_next);
        if (!formed) {
          ++u;
          Tile::template scores<NQ>(kt, 32, lane, q, s);
          Tile::template add<PARTS, NQ>(vt, 32, lane, w_next, st.o);
          formed = !fast(s_next, w);
          if (!formed) continue;
#pragma unroll
          for (int b = 0; b < NQ; ++b) { const at_f32x16_t x = s[b]; s[b] = s_next[b]; s_next[b] = x; }
        }
      }
#pragma unroll 1
      for (; u <= 2 * t; ++u) {
        if (!formed) {
          if (u + 1 >= u0 && u + 1 < u1) Tile::template scores<NQ>(kt, row_in_tile(u + 1), lane, q, s_next);
          if (u - 1 >= u0 && u - 1 < u1) {
            if (careful && (PARTS > 1 || cut(u - 1))) {
#pragma unroll 1
              for (int key = 0; key < 32; ++key) {   // its weight is with one of the column's lanes, element i of its 16
                const int i = 4 * (key >> 3) + (key & 3), owner = col + 32 * ((key >> 2) & 1), k = (tile0 * 2 + u - 1) * 32 + key;
#pragma unroll
                for (int b = 0; b < NQ; ++b) {
                  const float x = __shfl(Tile::template weight<PARTS>(w[b], i), owner, 64);
                  if (k > row[b] || k < start[b]) continue;
#pragma unroll
                  for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                      const at_f32x4_t y = Tile::value4(vt, row_in_tile(u - 1) + key, 32 * db + 8 * g + 4 * half);
#pragma unroll
                      for (int e = 0; e < 4; ++e) st.o[b][db][4 * g + e] = fmaf(x, y[e], st.o[b][db][4 * g + e]);
                    }
                }
              }
            } else {
              Tile::template add<PARTS, NQ>(vt, row_in_tile(u - 1), lane, w, st.o);
            }
          }
        }
        formed = false;
        if (u >= u0 && u < u1) {
          const int k32 = (tile0 * 2 + u) * 32;
#pragma unroll
          for (int b = 0; b < NQ; ++b) {
            float p[16], more;
            if (cut(u)) {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int key = k32 + key_of(i, half);
                s[b][i] = key <= row[b] && key >= start[b] ? s[b][i] : -__builtin_inff();
              }
            }
            attn_look<T, D, NQ>(st, b, s[b], p, more, a.scale_log2);
            st.sum[b] += more;
            Tile::template pack<PARTS>(p, w[b]);
          }
        }
#pragma unroll
        for (int b = 0; b < NQ; ++b) s[b] = s_next[b];
      }
    }
    // outputs that are no numbers: the formula's, or those of rows of V that nobody may see
    const int again = __syncthreads_or(!careful && any && not_finite(st));
    if (!again) break;
    careful = true;
  }
  if (!any) return;

#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    const float sum = both_sum(st.sum[b]);
    const bool mine = w0 + 32 * b + col == row[b];
    const long long o = (long long)qh * a.L + row[b];
    if (a.row_lse && mine && half == 0) a.row_lse[o] = (st.ref[b] + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
    store_column<OT, D>(reinterpret_cast<OT*>(a.out) + o * D, mine, half, st.o[b], 1.f / sum);
  }
}

template <typename T, typename OT, int D, int NW, int NQ>
static hipError_t launch_rows(PromptAttnArgs& a, int heads, hipStream_t st) {
  constexpr int BQ = NW * NQ * 32;
  a.blocks = (a.L + BQ - 1) / BQ;
  a.total = heads * a.blocks;
  hipLaunchKernelGGL((prompt_attn_kernel<T, OT, D, NW, NQ>), dim3((a.total + 7) / 8 * 8), dim3(NW * 64), 0, st, a);
  return hipGetLastError();
}
template <typename T, typename OT, int D>
static hipError_t launch_pa(PromptAttnArgs& a, int heads, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if ((long long)heads * a.L >= 256 * 256) return launch_rows<T, OT, D, 4, 2>(a, heads, st);
  }
  return launch_rows<T, OT, D, 4, 1>(a, heads, st);
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
