// Scores of every key against all queries of the prompt (paper Sec. 3.3 Eq. 7 with every position as a proxy token; the
// accumulated attention weight of heavy-hitter eviction): for KV head h with G query heads
//   psi(i) = sum over g, r >= i of exp(scale * q_gr . k_i - lse_gr),   lse_gr = log sum over j <= r of exp(scale * q_gr . k_j)
// L^2 / 2 logits per query head, which are never stored.  Prompts of up to PR_SHORT positions form them once (prompt_short_kernel).
// Longer ones take two sweeps: sweep 1 forms them for the normalisers (left out where the caller's
// prefill attention has them), sweep 2 once more for the column sums.
//
// Both sweeps are one kernel.  A workgroup holds a block of columns in registers as operand B (sweep 1: query rows, sweep 2: keys;
// a wave NCB blocks of 32) and streams the rows of the other side through LDS as operand A of the 32x32x16 bf16 MFMA: a lane
// then has 16 rows of one column of a 32 x 32 tile, and maximum, sum and column sum are in-lane work.
// What bounds it: a 32 x 32 tile of logits is 8 matrix instructions (256 cycles of a SIMD at 128 dims), 16 exp2, 16 multiply-adds into
// them and 16 additions (280 cycles, measured alone; 320 with the matrix instructions beside them).  That work at the chip's power
// limit: the loop without any loads takes 200 ns per tile and SIMD on random operands (the clock falls to 1.75 - 2.1 GHz), 169 on
// zeros (2.4 GHz), whether two, three or four waves share a SIMD and however the instructions are ordered.  So the layout saves
// instructions: sweep 1 looks for no maximum, but sums against the reference of the first tile and takes another
// one when a sum passes 2^60 (a tile is then formed again); rows that no column of a wave sees are left out and the causal mask is
// applied in diagonal tiles only; four blocks of columns share each operand read from LDS; a lane's offset in a tile is the same for all tiles.
// 16K tokens, 28 / 4 heads of 128 dims, both sweeps: 1.72-1.86 ms by the card, 235-255 ns per tile and SIMD, 1.03-1.12 PFLOP/s of logits (a library product of
// 16K x 16K x 16K bf16 runs at 1.36 on this card); 8K tokens, 32 heads, one sweep 0.27-0.29 ms.  Kept steps: address arithmetic per load -> a
// buffer with fixed offsets 1.85 -> 1.80; a block's contraction between the vector instructions of the one before it 1.89 -> 1.85.
// No gain at this size: blocks of two and three waves per SIMD (1.87; smaller calls take them, see prompt_plan), heads in plain order instead of one XCD's (1.84).  At 64 dims, half the
// matrix instructions, the vector unit alone bounds it, and the registers leave room for three waves: 16K, 28 / 4 heads 1.15-1.22 ms,
// 8K, 32 heads 0.376 (two waves 0.407, blocks of two and four waves 1.49 and 0.406, four waves with spills 1.38 and 0.437).
// The rows come straight into LDS (16 bytes per lane, pieces of a row permuted so that operand reads do not collide), in a
// ring of three tiles of 64 rows; LDS accesses and waits of the loop are written out, as in score.hip and for its reason.
//
// A head's triangle is cut into items of one column block by at most `chunk` rows, of nearly equal work but for the diagonal; the
// items of a head go to one XCD, whose L2 then holds the head's rows (4 MB at 16K x 128).  Partial results (sweep 1: maximum and
// sum, sweep 2: column sums) are joined in chunk order by small kernels.
#include "common.h"

#include <algorithm>

namespace madakv {

typedef __attribute__((ext_vector_type(8))) __bf16 pbf16x8_t;
typedef __attribute__((ext_vector_type(16))) float pf32x16_t;
typedef __attribute__((ext_vector_type(4))) float pf32x4_t;
typedef __attribute__((address_space(3))) void* plds_ptr_t;

constexpr int PR_WAVES = 4, PR_TILE = 64, PR_RING = 3;
constexpr float PR_FAR = 0x1p60f;               // sums beyond it have left their references behind

struct PromptArgs {
  const uint16_t* q; const uint16_t* k;         // [n, B, Hq, L, d], [n, B, H, L, d]
  float* lse2;                                  // [q heads][rows] log2 of the rows' normalisers; +inf past the prompt's end
  const float* row_lse;                         // the caller's, or null
  float2* stat;                                 // [q heads][chunks][rows] (maximum, sum) per chunk, log2 units
  float* part;                                  // [q heads][chunks][rows] column sums per chunk
  float* psi;
  int G, L, rows;                               // rows: L rounded up to whole tiles
  int per_chunk, chunks, blocks;                // column blocks per chunk, chunks, column blocks
  int items, total;                             // of a head and of all heads, in the sweep at hand
  float scale_log2;
};

// item -> (column block, chunk).  Sweep 1: block cb (queries) against chunks 0 .. cb / per_chunk of the keys; sweep 2: block cb
// (keys) against chunks cb / per_chunk .. of the queries.
template <int PASS>
__device__ __forceinline__ void item_of(const PromptArgs& a, int i, int& cb, int& chunk) {
  int g = 0;                                    // which stretch of per_chunk blocks, the one with the most chunks first
  for (; g < a.chunks; ++g) {
    const int first = (PASS == 1 ? a.chunks - 1 - g : g) * a.per_chunk;
    const int nb = min(a.per_chunk, a.blocks - first), each = a.chunks - g;
    if (i < nb * each) {
      cb = first + i / each;
      chunk = PASS == 1 ? i % each : g + i % each;
      return;
    }
    i -= nb * each;
  }
  cb = chunk = 0;                               // (there is no such item)
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000); }
// lane i: 16 (4) bytes from `at` + base of the buffer, zeros past its end, to LDS address dst + 16 i (4 i)
__device__ __forceinline__ void to_lds16(__amdgpu_buffer_rsrc_t b, uint32_t dst, int at, int base) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (plds_ptr_t)(uintptr_t)dst, 16, at, base, 0, 0);
}
__device__ __forceinline__ void to_lds4(__amdgpu_buffer_rsrc_t b, uint32_t dst, int at, int base) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (plds_ptr_t)(uintptr_t)dst, 4, at, base, 0, 0);
}

// log2 of the normaliser of row r: from the chunks' (maximum, sum), or from the caller's natural logarithm; +inf past the prompt's
// end, where rows count for nothing
__device__ __forceinline__ float normaliser_of(const PromptArgs& a, long long qh, int r, int cb_rows) {
  if (r >= a.L) return __builtin_inff();
  if (a.row_lse) return a.row_lse[qh * a.L + r] * 1.4426950408889634f;
  const int last = r / (a.per_chunk * cb_rows);              // the chunk with the row's own key
  float m = -__builtin_inff(), s = 0.f;
  for (int c0 = 0; c0 <= last; c0 += 4) {
    float2 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = c0 + u <= last ? a.stat[(qh * a.chunks + c0 + u) * a.rows + r] : make_float2(-__builtin_inff(), 0.f);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float t = fmaxf(m, x[u].x);
      s = (m == -__builtin_inff() ? 0.f : s * __builtin_amdgcn_exp2f(m - t)) + (x[u].x == -__builtin_inff() ? 0.f : x[u].y * __builtin_amdgcn_exp2f(x[u].x - t));
      m = t;
    }
  }
  return m + log2f(s);
}

template <int D, int NCB, int PASS, bool OWN_NORM = false>             // a wave's column blocks of 32; OWN_NORM: sweep 2 makes the normalisers of its rows itself
__global__ __launch_bounds__(PR_WAVES * 64) __attribute__((amdgpu_waves_per_eu(NCB == 4 && D == 64 ? 3 : 2, NCB == 4 ? (D == 64 ? 3 : 2) : 4))) void prompt_sweep_kernel(PromptArgs a) {
  constexpr int KS = D / 16;                    // MFMA steps over the head dimension
  constexpr int PPR = D / 8;                    // 16-byte pieces per row
  constexpr int ROWB = D * 2;
  constexpr int TILEB = PR_TILE * ROWB;
  constexpr int LPT = PR_TILE * PPR / (PR_WAVES * 64);     // load instructions per wave and tile, 1 KB each
  constexpr int CB = PR_WAVES * NCB * 32;
  constexpr int LOADS = LPT + (PASS == 2 && !OWN_NORM ? 1 : 0);            // of a wave, per tile
  // [ring][64 rows][D], sweep 2: [ring][waves][64] normalisers, or those of all rows of the item
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

  // workgroup -> item: XCD x (workgroups go to the XCDs in turn) takes the x-th eighth of all items, heads one after the other
  const int per_xcd = (a.total + 7) / 8;
  const int idx = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if (idx >= a.total || (int)(blockIdx.x >> 3) >= per_xcd) return;
  const int qh = idx / a.items;
  int cb, chunk;
  item_of<PASS>(a, idx - qh * a.items, cb, chunk);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const uint16_t* qrows = a.q + (long long)qh * a.L * D;
  const uint16_t* krows = a.k + (long long)(qh / a.G) * a.L * D;           // (query head j of a layer's batch item reads KV head j / G)
  const unsigned char* cols = reinterpret_cast<const unsigned char*>(PASS == 1 ? qrows : krows);
  const unsigned char* rows = reinterpret_cast<const unsigned char*>(PASS == 1 ? krows : qrows);
  const int c0 = cb * CB;
  const int my0 = c0 + wave * NCB * 32;         // the wave's first column
  const int chunk_rows = a.per_chunk * CB;
  const int row0 = PASS == 1 ? chunk * chunk_rows : max(chunk * chunk_rows, c0);
  const int row1 = min((chunk + 1) * chunk_rows, PASS == 1 ? min(a.rows, (c0 + CB + PR_TILE - 1) / PR_TILE * PR_TILE) : a.rows);
  const int ntiles = (row1 - row0) / PR_TILE;   // (all of them multiples of the tile; at least one)

  const uint32_t ring = (uint32_t)(uintptr_t)smem;
  const uint32_t ring_n = ring + PR_RING * TILEB;
  // tile T -> ring slot T mod 3: load j of wave w fills bytes [(w LPT + j) 1024, + 1024) of the slot, lane i slot P mod PPR of row P / PPR,
  // P = (w LPT + j) 64 + i, with that row's piece (P mod PPR) ^ (row mod PPR).  Through a buffer that ends with the prompt: keys
  // past its end are zeros, and a lane's offset in a tile is the same for all tiles but a last one that is not whole, whose queries past
  // the end are the last one again: their normalisers make nothing of a logit of any size, but zeros times an infinite key would be
  // no number.
  const __amdgpu_buffer_rsrc_t rows_buf = buffer_of(rows, a.L * ROWB), norm_buf = buffer_of(a.lse2 + (long long)qh * a.rows, a.rows * 4);
  int piece_off[LPT];
#pragma unroll
  for (int j = 0; j < LPT; ++j) {
    const int piece = (wave * LPT + j) * 64 + lane, row = piece / PPR;
    piece_off[j] = row * ROWB + ((piece % PPR) ^ (row % PPR)) * 16;
  }
  const auto issue = [&](int t) {
    const int r0 = row0 + t * PR_TILE;
    const uint32_t slot = (uint32_t)(t % PR_RING);
    const auto load = [&](int j, int at) { to_lds16(rows_buf, ring + slot * TILEB + (uint32_t)(wave * LPT + j) * 1024u, at, r0 * ROWB); };
    if (PASS == 2 && __builtin_expect(r0 + PR_TILE > a.L, 0)) {
#pragma unroll
      for (int j = 0; j < LPT; ++j) {
        int at = piece_off[j];
        asm volatile("" : "+v"(at));            // (made here: kept over the loop, its parts would take registers)
        load(j, min(at & -ROWB, (a.L - 1 - r0) * ROWB) + (at & (ROWB - 1)));
      }
    } else {
#pragma unroll
      for (int j = 0; j < LPT; ++j) load(j, piece_off[j]);
    }
    if (PASS == 2 && !OWN_NORM)                 // the rows' normalisers, every wave its own copy
      to_lds4(norm_buf, ring_n + (slot * PR_WAVES + wave) * (PR_TILE * 4u), lane * 4, r0 * 4);
  };
  issue(0);
  issue(min(1, ntiles - 1));
  if constexpr (OWN_NORM)
    for (int r = tid; r < row1 - row0; r += PR_WAVES * 64) reinterpret_cast<float*>(smem + PR_RING * TILEB)[r] = normaliser_of(a, qh, row0 + r, CB);

  // the wave's columns; a lane holds, for step ks, elements [half * D/2 + ks * 8, + 8) of column `col` of a block
  pbf16x8_t breg[NCB][KS];
#pragma unroll
  for (int b = 0; b < NCB; ++b) {
    const unsigned char* src = cols + (long long)min(my0 + b * 32 + col, a.L - 1) * ROWB + half * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) breg[b][ks] = *reinterpret_cast<const pbf16x8_t*>(src + ks * 16);
  }
  // (here and now: a wait for them in the loop would be one for the tiles behind them as well)
#pragma unroll
  for (int b = 0; b < NCB; ++b)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(breg[b][ks]));
  uint32_t frag[KS];                            // where the lane's pieces of row `col` of a subtile are
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) frag[ks] = (uint32_t)(col * ROWB + (((half * KS + ks) ^ (col % PPR)) * 16));

  float ref[NCB], sum[NCB];                     // sweep 1: reference (log2 units, -inf: none yet) and sum; sweep 2: column sums
#pragma unroll
  for (int b = 0; b < NCB; ++b) { ref[b] = -__builtin_inff(); sum[b] = 0.f; }

  pbf16x8_t areg[KS];
  float nreg[PASS == 2 ? 16 : 1];
  const auto logits = [&](int b) {
    pf32x16_t x = pf32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(areg[ks], breg[b][ks], x, 0, 0, 0);
    return x;
  };
  const auto masked = [&](pf32x16_t x) {        // the tile on the diagonal: a query sees the keys up to its own
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int row = 8 * (j >> 2) + 4 * half + (j & 3);
      x[j] = (PASS == 1 ? row <= col : row >= col) ? x[j] : -__builtin_inff();
    }
    return x;
  };
  // the sum of a column's 16 terms: against the rows' normalisers, or its own reference
  const auto sum16 = [](const float (&p)[16]) {
    return (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]))) + (((p[8] + p[9]) + (p[10] + p[11])) + ((p[12] + p[13]) + (p[14] + p[15])));
  };
  const auto term = [&](int b, const pf32x16_t& x, int j) { return __builtin_amdgcn_exp2f(fmaf(x[j], a.scale_log2, PASS == 2 ? -nreg[j % (PASS == 2 ? 16 : 1)] : -ref[b])); };
  const auto terms = [&](int b, const pf32x16_t& x) {
    float p[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) p[j] = term(b, x, j);
    return sum16(p);
  };
  // the same of sweep 2's diagonal tile where a normaliser is no number, or minus infinity: nothing from the rows that do not see the key
  const auto seen_terms = [&](int b, const pf32x16_t& x) {
    int first = col - 4 * half;
    asm volatile("" : "+v"(first));             // (made here: the comparisons, kept over the loop, would take registers)
    float p[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) p[j] = 8 * (j >> 2) + (j & 3) >= first ? term(b, x, j) : 0.f;
    return sum16(p);
  };
  // sweep 1, a tile for which some column has no reference yet or has left it far behind: there the largest logit becomes the
  // reference
  const auto look = [&](int b, const pf32x16_t& x) {
    float s = terms(b, x), top = x[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) top = fmaxf(top, x[j]);
    if (!(sum[b] + s < 0.25f * PR_FAR)) {       // (also: no number)
      if (top > -__builtin_inff()) {
        const float r = fmaxf(sum[b] < 0x1p50f ? ref[b] : ref[b] + 50.f, top * a.scale_log2);
        sum[b] = ref[b] == -__builtin_inff() ? 0.f : sum[b] * __builtin_amdgcn_exp2f(ref[b] - r);
        ref[b] = r;
        s = terms(b, x);
      } else if (top == top) {
        s = 0.f;                                // nothing but masked keys so far
      }
    }
    sum[b] += s;
  };

  for (int t = 0; t < ntiles; ++t) {
    // tile t has landed (the next one's loads may still be out); behind the barrier that holds for every wave, and nobody
    // reads tile t - 1 any more, whose slot the next loads take
    if (LOADS == 5) asm volatile("s_waitcnt vmcnt(5) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else if (LOADS == 4) asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else if (LOADS == 3) asm volatile("s_waitcnt vmcnt(3) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(2) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    static_assert(LOADS >= 2 && LOADS <= 5, "the waits above are written for these");
    issue(min(t + 2, ntiles - 1));              // (past the end: the last tile once more, which keeps the count of loads in flight)
    const uint32_t tile = ring + (uint32_t)(t % PR_RING) * TILEB;
    const uint32_t tile_n = ring_n + (uint32_t)(OWN_NORM ? t : (t % PR_RING) * PR_WAVES + wave) * (PR_TILE * 4u) + half * 16u;
#pragma unroll 1
    for (int sub = 0; sub < PR_TILE / 32; ++sub) {
      const int r = row0 + t * PR_TILE + sub * 32;
      // sweep 1: keys behind the wave's last query; sweep 2: queries in front of its first key
      if (PASS == 1 ? r > my0 + (NCB - 1) * 32 : r < my0) continue;
      const uint32_t at = tile + (uint32_t)sub * (32 * ROWB);
      if constexpr (KS == 8) {
        asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
                     "ds_read_b128 %4, %12\n\tds_read_b128 %5, %13\n\tds_read_b128 %6, %14\n\tds_read_b128 %7, %15\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(areg[0]), "=&v"(areg[1]), "=&v"(areg[2]), "=&v"(areg[3]), "=&v"(areg[4]), "=&v"(areg[5]), "=&v"(areg[6]), "=&v"(areg[7])
                     : "v"(at + frag[0]), "v"(at + frag[1]), "v"(at + frag[2]), "v"(at + frag[3]), "v"(at + frag[4]), "v"(at + frag[5]), "v"(at + frag[6]), "v"(at + frag[7])
                     : "memory");
      } else {
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(areg[0]), "=&v"(areg[1]), "=&v"(areg[2]), "=&v"(areg[3])
                     : "v"(at + frag[0]), "v"(at + frag[1]), "v"(at + frag[2]), "v"(at + frag[3]) : "memory");
      }
      if constexpr (PASS == 2) {
        pf32x4_t n0, n1, n2, n3;
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:32\n\tds_read_b128 %2, %4 offset:64\n\tds_read_b128 %3, %4 offset:96\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(n0), "=&v"(n1), "=&v"(n2), "=&v"(n3) : "v"(tile_n + (uint32_t)sub * 128u) : "memory");
#pragma unroll
        for (int j = 0; j < 4; ++j) { nreg[j] = n0[j]; nreg[4 + j] = n1[j]; nreg[8 + j] = n2[j]; nreg[12 + j] = n3[j]; }
      }
      if (PASS == 1 ? r < my0 : r > my0 + (NCB - 1) * 32) {        // off the diagonal for all blocks
        // a block's contraction is issued between the vector instructions of the block before it
        float s[NCB];
        pf32x16_t x = logits(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < NCB; ++b) {
          const pf32x16_t now = x;
          if (b + 1 < NCB) x = logits(b + 1);
          s[b] = sum[b] + terms(b, now);
          if (b + 1 < NCB) {
#pragma unroll
            for (int i = 0; i < KS; ++i) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);           // one matrix instruction,
              __builtin_amdgcn_sched_group_barrier(0x002, 32 / KS, 0);     // so many multiply-adds and additions,
              __builtin_amdgcn_sched_group_barrier(0x400, 16 / KS, 0);     // so many exp2
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (PASS == 1) {
          float all = s[0];
#pragma unroll
          for (int b = 1; b < NCB; ++b) all += s[b];
          if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(all < PR_FAR)) != 0, 0)) {
#pragma unroll
            for (int b = 0; b < NCB; ++b) look(b, logits(b));
            continue;
          }
        }
#pragma unroll
        for (int b = 0; b < NCB; ++b) sum[b] = s[b];
      } else {
#pragma unroll
        for (int b = 0; b < NCB; ++b) {
          const int mine = my0 + b * 32;
          if (PASS == 1 ? r > mine : r < mine) continue;
          const pf32x16_t x = r == mine ? masked(logits(b)) : logits(b);
          if (PASS == 1) { look(b, x); continue; }
          float s = terms(b, x);
          if (r == mine && __builtin_expect(__builtin_amdgcn_ballot_w64(s != s) != 0, 0)) s = seen_terms(b, x);
          sum[b] += s;
        }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // (the loads past the end write to LDS, too)

  // the two halves of a column
#pragma unroll
  for (int b = 0; b < NCB; ++b) {
    const int c = my0 + b * 32 + col;
    const float other = __shfl_xor(sum[b], 32, 64);
    if (PASS == 2) {
      if (half == 0 && c < a.L) {
        const float s = sum[b] + other;
        if (a.chunks == 1 && a.G == 1) a.psi[(long long)qh * a.L + c] = s;
        else a.part[((long long)qh * a.chunks + chunk) * a.rows + c] = s;
      }
    } else {
      const float other_ref = __shfl_xor(ref[b], 32, 64);
      // (a half that has seen no key: reference -inf, sum 0, whose weight is not asked for)
      const float r = fmaxf(ref[b], other_ref);
      const float w0 = ref[b] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(ref[b] - r), w1 = other_ref == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(other_ref - r);
      const float s = half == 0 ? sum[b] * w0 + other * w1 : other * w1 + sum[b] * w0;
      if (half == 0 && c < a.rows) {
        if (a.chunks == 1) a.lse2[(long long)qh * a.rows + c] = c < a.L ? r + log2f(s) : __builtin_inff();
        else a.stat[((long long)qh * a.chunks + chunk) * a.rows + c] = make_float2(r, s);
      }
    }
  }
}

// Prompts of up to PR_SHORT positions: one launch, a workgroup per query head, which has all keys in LDS and every wave a block of
// 32 queries.  A wave keeps its logits (keys x queries, up to 8 tiles of 32 x 32) in registers, so that each is formed once: maximum
// and sum of a query's column are the lane's own and the other half's, its weights follow, and a key's weights are added up over
// the 32 lanes that have its row, 16 keys at a time: exchanges in which a lane sends half of what it has left and keeps the other.
// Waves w and w + 4 share a SIMD and take blocks whose keys add up to the same.  What bounds it: a launch's latency on few heads, the vector
// unit on many.  us on the device, two sweeps / this: 8 heads of 40 x 64 6.9 / 3.6, of 203 x 64 11.8 / 7.2, 32 of 256 x 128 14.7 / 9.1 (normalisers
// given 9.5 / 8.0), 28 / 4 of 256 x 128 17.0 / 11.3, 256 of 130 x 128 15.1 / 7.8, 2048 of 256 x 128 139 / 77, of 200 x 64 86 / 53: it is taken
// wherever the logits of a block of queries fit a wave's registers.
constexpr int PR_SHORT = 256, PR_SHORT_WAVES = PR_SHORT / 32;

template <int CTRL>
__device__ __forceinline__ float from_lane(float x) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xF, 0xF, true)); }
// N values of a lane and N of its partner -> N / 2 sums: the upper ones where `high`
template <int CTRL, int N>
__device__ __forceinline__ void halve(float (&v)[16], bool high) {
#pragma unroll
  for (int j = 0; j < N / 2; ++j) {
    const float keep = high ? v[j + N / 2] : v[j], send = high ? v[j] : v[j + N / 2];
    v[j] = keep + from_lane<CTRL>(send);
  }
}

// What a wave's 32 queries (breg; a lane's is `col` of block `mine`) pay to each of the first 32 NT keys, to sums.  NT: mine + 1 or one
// more.  GIVEN: `norm` is the log2 of the query's normaliser.
template <int D, int NT, bool GIVEN>
__device__ __forceinline__ void short_block(const unsigned char* keys, const pbf16x8_t (&breg)[D / 16], int mine, bool there, float norm, float scale_log2, float* sums) {
  constexpr int KS = D / 16, PPR = D / 8, ROWB = D * 2;
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  pf32x16_t x[NT];
  float top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    pbf16x8_t areg[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) areg[ks] = *reinterpret_cast<const pbf16x8_t*>(keys + (i * 32 + col) * ROWB + ((half * KS + ks) ^ (col % PPR)) * 16);
    x[i] = pf32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) x[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(areg[ks], breg[ks], x[i], 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if (i >= NT - 2) x[i][j] = (i - mine) * 32 + 8 * (j >> 2) + 4 * half + (j & 3) <= col ? x[i][j] : -__builtin_inff();
      if (!GIVEN) top = fmaxf(top, x[i][j]);
    }
    __builtin_amdgcn_sched_barrier(0);          // (operands of one tile at a time: all of them do not fit)
  }
  // a lane whose normaliser is no number, or minus infinity: nothing to the keys that its query does not see, no number to the others
  const auto unseen = [&](bool lost, bool all) {
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const bool sees = (i - mine) * 32 + 8 * (j >> 2) + 4 * half + (j & 3) <= col;
        if (lost) x[i][j] = !sees ? 0.f : all ? __builtin_nanf("") : x[i][j];
      }
  };
  float share = 1.f;
  if (GIVEN) {
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) x[i][j] = __builtin_amdgcn_exp2f(fmaf(x[i][j], scale_log2, -norm));
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(norm > -__builtin_inff())) != 0, 0)) unseen(!(norm > -__builtin_inff()), false);
  } else {
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        x[i][j] = __builtin_amdgcn_exp2f((x[i][j] - top) * scale_log2);
        s[j & 3] += x[i][j];
      }
    const float sum = (s[0] + s[1]) + (s[2] + s[3]);
    share = there ? 1.f / (sum + __shfl_xor(sum, 32, 64)) : 0.f;
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(share != share) != 0, 0)) {
      unseen(share != share, true);
      share = share != share ? 1.f : share;
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    float v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = GIVEN ? x[i][j] : x[i][j] * share;
    halve<0x128, 16>(v, lane & 8);              // row_ror 8: lane ^ 8
    halve<0x141, 8>(v, lane & 4);               // row_half_mirror: lane ^ 7
    halve<0x4E, 4>(v, lane & 2);                // quad_perm [2,3,0,1]: lane ^ 2
    halve<0xB1, 2>(v, lane & 1);                // quad_perm [1,0,3,2]: lane ^ 1
    const float s = v[0] + __shfl_xor(v[0], 16, 64);              // lane j has row j of its half
    const int j = lane & 15;
    if ((lane & 16) == 0) sums[i * 32 + 8 * (j >> 2) + 4 * half + (j & 3)] = s;
  }
}

template <int D, bool GIVEN>
__global__ __launch_bounds__(PR_SHORT_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void prompt_short_kernel(PromptArgs a, const float* row_lse, float* scaled, float factor) {
  constexpr int KS = D / 16, PPR = D / 8, ROWB = D * 2;
  __shared__ __attribute__((aligned(16))) unsigned char s_keys[PR_SHORT * ROWB];
  __shared__ float s_sums[PR_SHORT_WAVES * PR_SHORT];        // what every block of queries pays to the keys
  const int qh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int nb = (a.L + 31) / 32, mine = wave < PR_SHORT_WAVES / 2 ? wave : PR_SHORT_WAVES * 3 / 2 - 1 - wave;
  const unsigned char* qrows = reinterpret_cast<const unsigned char*>(a.q) + (long long)qh * a.L * ROWB;
  const unsigned char* krows = reinterpret_cast<const unsigned char*>(a.k) + (long long)(qh / a.G) * a.L * ROWB;
  // keys as the sweeps have them in LDS; rows past the prompt's end are zeros
  const __amdgpu_buffer_rsrc_t keys_buf = buffer_of(krows, a.L * ROWB);
  for (int i = wave; i < nb * (32 * ROWB / 1024); i += PR_SHORT_WAVES) {
    const int piece = i * 64 + lane, row = piece / PPR;
    to_lds16(keys_buf, (uint32_t)(uintptr_t)(plds_ptr_t)s_keys + (uint32_t)i * 1024u, row * ROWB + ((piece % PPR) ^ (row % PPR)) * 16, 0);
  }
  const int query = mine * 32 + col;
  const bool there = query < a.L;
  pbf16x8_t breg[KS];
  const unsigned char* src = qrows + (long long)min(query, a.L - 1) * ROWB + half * D;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) breg[ks] = *reinterpret_cast<const pbf16x8_t*>(src + ks * 16);
  const float norm = GIVEN && there ? row_lse[(long long)qh * a.L + query] * 1.4426950408889634f : __builtin_inff();
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  float* sums = s_sums + mine * PR_SHORT;
  if (mine < nb) {                              // (a tile behind the wave's own is masked, whatever is there)
    if (mine >= 6) short_block<D, 8, GIVEN>(s_keys, breg, mine, there, norm, a.scale_log2, sums);
    else if (mine >= 4) short_block<D, 6, GIVEN>(s_keys, breg, mine, there, norm, a.scale_log2, sums);
    else if (mine >= 2) short_block<D, 4, GIVEN>(s_keys, breg, mine, there, norm, a.scale_log2, sums);
    else short_block<D, 2, GIVEN>(s_keys, breg, mine, there, norm, a.scale_log2, sums);
  }
  __syncthreads();
  if (tid >= a.L) return;
  float s = 0.f;
  for (int b = tid / 32; b < nb; ++b) s += s_sums[b * PR_SHORT + tid];
  if (a.G > 1) { a.part[(long long)qh * a.rows + tid] = s; return; }
  a.psi[(long long)qh * a.L + tid] = s;
  if (scaled) scaled[(long long)qh * a.L + tid] = s * factor;
}

// log2 of the rows' normalisers, where the items do not make them themselves
__global__ __launch_bounds__(256) void prompt_normaliser_kernel(PromptArgs a, int cb_rows, long long n) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const long long qh = i / a.rows;
  const int r = (int)(i - qh * a.rows);
  a.lse2[i] = normaliser_of(a, qh, r, cb_rows);
}

// psi = the column sums of the query heads and chunks, in that order; scaled: psi * factor beside it
__global__ __launch_bounds__(256) void prompt_sum_kernel(PromptArgs a, int cb_rows, float* scaled, float factor, long long n) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const long long kvh = i / a.L;
  const int c = (int)(i - kvh * a.L);
  float s = 0.f;
  if (a.chunks == 1 && a.G == 1) {
    s = a.psi[i];
  } else {
    // eight loads at a time: one behind the other, 28 terms per key took 16 us of a launch
    const int first = c / (a.per_chunk * cb_rows), terms = a.G * a.chunks;           // the chunk with the key's own query
    const float* p = a.part + kvh * terms * a.rows + c;
    for (int j0 = 0; j0 < terms; j0 += 8) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = j0 + u < terms && (j0 + u) % a.chunks >= first ? p[(long long)(j0 + u) * a.rows] : 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) s += x[u];
    }
    a.psi[i] = s;
  }
  if (scaled) scaled[i] = s * factor;
}

struct PromptPlan { int ncb, per_chunk, chunks, blocks, items[2]; };      // items of a head in sweep 1 and 2 (item_of)
// Column blocks of 512 (a wave has four blocks of 32) where those are enough items to fill the chip several times over, of 256 where
// it is those, of 128 otherwise, and none so large that more than 15% (20%) of the columns are past the prompt's end; chunks as long as
// leave 2300 (1300, 640) items, of which 512 (768, 1024) run at a time, so that the launch's last round of workgroups is a small
// part of it, but no shorter than 512 (256, 256) rows: every item starts with its columns and an empty ring.  The numbers are those
// with the least time over 122 calls of 8 to 128 heads and 300 to 9000 positions, 1.9% above the best choice for each (2.4% with
// 1800, 600, 600 items; 6.1% without blocks of 256).  us on the device, blocks of 512 / 256 / 128: 32 / 8 heads of 2K x 128 79 / 62 / 66, 80 of 1.7K x 64
// 87 / 69 / 76, 28 / 4 of 4K x 128 154 / 158 / 178, 20 of 6K x 128 236 / 227 / 251, 32 of 1K x 128 52 / 33 / 27.  28 / 4 heads of 16K x 128, at least 1200 / 2300 / 4100
// items: 2112 / 1788 / 1799, 32 heads of 8K with normalisers 293 / 274 / 279.
static PromptPlan prompt_plan(const Dims& dm) {
  struct Choice { int ncb, shortest, want, least, fill; };   // blocks, least blocks per chunk, items to aim for, least items, least % of columns in the prompt
  constexpr Choice choices[] = {{4, 1, 2300, 2000, 85}, {2, 1, 1300, 700, 80}, {1, 2, 640, 0, 0}};
  PromptPlan p;
  const long long qheads = (long long)dm.n * dm.B * dm.Hq;
  for (const Choice& c : choices) {
    const int cb = PR_WAVES * c.ncb * 32;
    p.ncb = c.ncb;
    p.blocks = (dm.L + cb - 1) / cb;
    for (p.per_chunk = p.blocks;; p.per_chunk = (p.per_chunk + 1) / 2) {
      p.chunks = (p.blocks + p.per_chunk - 1) / p.per_chunk;
      p.items[0] = p.items[1] = 0;
      for (int g = 0; g < p.chunks; ++g) {
        const int nb = std::min(p.per_chunk, p.blocks - g * p.per_chunk);
        p.items[0] += nb * (g + 1);
        p.items[1] += nb * (p.chunks - g);
      }
      if (qheads * p.items[0] >= c.want || p.per_chunk <= c.shortest) break;
    }
    if (qheads * p.items[0] >= c.least && 100ll * dm.L >= (long long)c.fill * p.blocks * cb) break;
  }
  return p;
}
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }
static size_t rows_of(const Dims& dm) { return (size_t)(dm.L + PR_TILE - 1) / PR_TILE * PR_TILE; }

// Items of few rows make the normalisers of their rows themselves, in sweep 2, which saves a launch.  us on the device, a launch of its own /
// this: 8 heads of 512 x 64 16.4 / 14.7, of 1K x 64 17.3 / 15.3, 28 / 4 of 1K x 128 30.6 / 27.8, 8 of 1K x 128 with normalisers
// given 12.0 / 10.2.  Up to 512, 1024 or 2048 rows: all the same; their normalisers take 4 KB of LDS at most.
constexpr int PR_OWN_ROWS = 1024;
static bool own_norm(const PromptPlan& p, bool given) { return p.ncb <= 2 && p.per_chunk * PR_WAVES * p.ncb * 32 <= PR_OWN_ROWS && (given || p.chunks > 1); }
// normalisers, then what the chunks leave (sweep 2's column sums take the place of sweep 1's statistics, but where sweep 2 still
// reads those), then the scaled scores
struct PromptWs { size_t stat, part, scaled, total; };
static PromptWs prompt_ws(const Dims& dm, const PromptPlan& p) {
  PromptWs w;
  const size_t qheads = (size_t)dm.n * dm.B * dm.Hq, entries = qheads * p.chunks * rows_of(dm);
  w.stat = up256(qheads * rows_of(dm) * 4);
  const bool apart = own_norm(p, false);
  w.part = apart ? w.stat + up256(entries * 8) : w.stat;
  w.scaled = w.part + up256(entries * (apart ? 4 : 8));
  w.total = w.scaled + up256((size_t)dm.heads * dm.L * 4);
  return w;
}
bool prompt_supported(const madakv_config& c) { return c.dtype == MADAKV_BF16; }
size_t prompt_ws_bytes(const Dims& dm) { return prompt_ws(dm, prompt_plan(dm)).total; }

template <int D>
static hipError_t launch_short(const Dims& dm, const PromptArgs& a, const float* row_lse, float* scaled, float factor, hipStream_t st) {
  const dim3 grid((unsigned)(dm.n * dm.B * dm.Hq)), block(PR_SHORT_WAVES * 64);
  if (row_lse) hipLaunchKernelGGL((prompt_short_kernel<D, true>), grid, block, 0, st, a, row_lse, scaled, factor);
  else hipLaunchKernelGGL((prompt_short_kernel<D, false>), grid, block, 0, st, a, row_lse, scaled, factor);
  if (a.G == 1) return hipGetLastError();
  if (hipError_t e = hipGetLastError()) return e;
  const long long npsi = (long long)dm.heads * dm.L;
  hipLaunchKernelGGL(prompt_sum_kernel, dim3((unsigned)((npsi + 255) / 256)), dim3(256), 0, st, a, PR_SHORT, scaled, factor, npsi);
  return hipGetLastError();
}

template <int D, int NCB>
static hipError_t launch_sweeps(const Dims& dm, const PromptPlan& p, PromptArgs& a, const float* row_lse, float* scaled, float factor, hipStream_t st) {
  constexpr int CB = PR_WAVES * NCB * 32;
  constexpr size_t lds1 = (size_t)PR_RING * PR_TILE * D * 2, lds2 = lds1 + (size_t)PR_RING * PR_WAVES * PR_TILE * 4;
  const dim3 block(PR_WAVES * 64);
  const auto grid_of = [&](int pass) {
    a.items = p.items[pass - 1];
    a.total = dm.n * dm.B * dm.Hq * a.items;
    return dim3((unsigned)((a.total + 7) / 8 * 8));
  };
  const long long nrows = (long long)dm.n * dm.B * dm.Hq * a.rows, npsi = (long long)dm.heads * dm.L;
  if (!row_lse) {
    const dim3 grid = grid_of(1);
    hipLaunchKernelGGL((prompt_sweep_kernel<D, NCB, 1>), grid, block, lds1, st, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  const bool own = own_norm(p, row_lse != nullptr);
  if (!own && (row_lse || a.chunks > 1)) {
    hipLaunchKernelGGL(prompt_normaliser_kernel, dim3((unsigned)((nrows + 255) / 256)), dim3(256), 0, st, a, CB, nrows);
    if (hipError_t e = hipGetLastError()) return e;
  }
  const dim3 grid = grid_of(2);
  if (own) {
    if constexpr (NCB <= 2) hipLaunchKernelGGL((prompt_sweep_kernel<D, NCB, 2, true>), grid, block, lds1 + (size_t)a.per_chunk * CB * 4, st, a);
  } else {
    hipLaunchKernelGGL((prompt_sweep_kernel<D, NCB, 2>), grid, block, lds2, st, a);
  }
  if (hipError_t e = hipGetLastError()) return e;
  if (a.chunks > 1 || a.G > 1 || scaled) hipLaunchKernelGGL(prompt_sum_kernel, dim3((unsigned)((npsi + 255) / 256)), dim3(256), 0, st, a, CB, scaled, factor, npsi);
  return hipGetLastError();
}

// scaled: psi * factor as well, at the workspace's end; its address is left in *scaled
hipError_t launch_prompt(const Dims& dm, const madakv_config& c, const void* q, const void* k, const float* row_lse, float* psi,
                         void* ws, float factor, float** scaled, hipStream_t st) {
  const PromptPlan p = prompt_plan(dm);
  PromptArgs a;
  a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k);
  a.psi = psi; a.row_lse = row_lse; a.G = dm.G; a.L = dm.L; a.rows = (int)rows_of(dm);
  char* w = static_cast<char*>(ws);
  const PromptWs at = prompt_ws(dm, p);
  a.lse2 = reinterpret_cast<float*>(w);
  a.stat = reinterpret_cast<float2*>(w + at.stat); a.part = reinterpret_cast<float*>(w + at.part);
  float* s = nullptr;
  if (scaled) *scaled = s = reinterpret_cast<float*>(w + at.scaled);
  a.per_chunk = p.per_chunk; a.chunks = p.chunks; a.blocks = p.blocks;
  a.scale_log2 = (c.softmax_scale > 0.f ? c.softmax_scale : 1.0f / sqrtf((float)dm.d)) * 1.4426950408889634f;
  if (dm.L <= PR_SHORT) {
    a.per_chunk = a.chunks = 1;
    return dm.d == 128 ? launch_short<128>(dm, a, row_lse, s, factor, st) : launch_short<64>(dm, a, row_lse, s, factor, st);
  }
  if (dm.d == 128) return p.ncb == 4 ? launch_sweeps<128, 4>(dm, p, a, row_lse, s, factor, st) : p.ncb == 2 ? launch_sweeps<128, 2>(dm, p, a, row_lse, s, factor, st) : launch_sweeps<128, 1>(dm, p, a, row_lse, s, factor, st);
  return p.ncb == 4 ? launch_sweeps<64, 4>(dm, p, a, row_lse, s, factor, st) : p.ncb == 2 ? launch_sweeps<64, 2>(dm, p, a, row_lse, s, factor, st) : launch_sweeps<64, 1>(dm, p, a, row_lse, s, factor, st);
}

}  // namespace madakv
