// Decode over a reduced cache of 4-bit floats (paper Sec. 3.1 Eq. 3-5, as in decode.hip): append the new row, encoded, then
// out = softmax(scale * q K_c^T) V_c over the rows as they are stored.
//
// A row of K is d / 2 bytes of codes and d / 32 scale bytes: 136 bytes of K and V per row of 128 dims, a quarter of bf16.  So the
// arithmetic per byte is four times that of decode.hip and a row must cost few instructions; one query head takes the same path as
// eight, on the matrix units:
//   S^T[key][q] = K . Q^T   on the 16x16x32 bf16 instruction: a lane holds one block of 32 dims of one row and its scale byte, which
//                           become the A operands of four contraction steps by one conversion per two elements (exact).
//                           (The block-scaled instruction takes K as it is stored, against the query as two E4M3 parts that
//                           add up to bf16.  But it aligns products of neighbouring elements to the largest of them with some
//                           14 bits: outputs were off by up to 2e-5 instead of 2e-7.)
//   O^T[d][q] += V^T . P^T  on the same instruction: V's codes become bf16 likewise, are parked in a wave-private LDS tile and
//                           come back through transposing reads, 32 keys at a time.  P goes in as three bf16 parts, which hold all 24
//                           bits of it (two parts left outputs 1-2e-6 off, three 2e-7): the first in columns 0-7 and the second
//                           in columns 8-15 of one instruction, the third in columns 0-7 of another.
// At most 8 query heads share a KV head and an instruction has 16 columns: S^T has the queries against the first 16 keys of a tile in
// columns 0-7 and against the other 16 in columns 8-15, so that a lane turns 4 logits of a tile into weights and not 8, half
// of them twice; for P it gives the other column of its query what that one needs, a rotation within 16 lanes.
// A load instruction of a wave takes 1 KB of consecutive codes (16 rows of 128 dims, 32 of 64) and one of 64 scale bytes.  Rows of
// 64 dims: lanes 0-31 have the blocks of rows 0-15, lanes 32-63 those of rows 16-31; columns 0-7 have the query in the half of the
// contraction that belongs to the former and zeros in the other, columns 8-15 the other way round.
// What bounds it: HBM for long caches, 128 heads of 16K rows of 128 dims (285 MB) 50-54 us by the card, 5.3-5.7 TB/s, with four waves per SIMD issuing
// most of the time; a launch's own latency for short ones, 8 heads of 256 rows of 64 dims 6.0-6.6 us, 28 / 4 heads of 2K rows of 128 dims 6.3-7.1.
// Measured against it at 285 MB: eight waves a workgroup 55.7, no loads ahead of a tile 53.7, loads of codes through the caches 58.6,
// 8 logits per lane with half of the columns idle 54.5 (now 52.9 on that card); scales
// as one load per 32 rows 0.4 us less at the most.
#include "decode_pieces.h"

namespace madakv {

typedef __attribute__((address_space(3))) ds16x4_t* lds4_s16x4_ptr_t;

// the two columns of a query
__device__ __forceinline__ uint32_t other_column(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, true); }      // row_ror 8
__device__ __forceinline__ float add_ror8(float x) { return x + __uint_as_float(other_column(__float_as_uint(x))); }

// The new row, encoded: written to the cache (Eq. 4) and left in LDS: codes of K, codes of V, scales of K, scales of V.  All
// threads; `row` is its place in the cache.
template <int D>
__device__ __forceinline__ void stage_new_row4(const DecodeArgs& a, long long hidx, long long row, uint8_t* s_new) {
  constexpr int LPR = D / 8;
  const int t = threadIdx.x;
  if (t < 2 * LPR) {
    const bool is_k = t < LPR;
    const int piece = is_k ? t : t - LPR;
    const uint4 x = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(is_k ? a.k_new : a.v_new) + hidx * D + piece * 8);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t scale;
    const uint32_t code = mx_encode8(w, scale);
    uint8_t* cache = reinterpret_cast<uint8_t*>(is_k ? a.k_c : a.v_c);
    *reinterpret_cast<uint32_t*>(cache + row * (D / 2) + piece * 4) = code;
    *reinterpret_cast<uint32_t*>(s_new + (is_k ? 0 : D / 2) + piece * 4) = code;
    if ((piece & 3) == 0) {
      cache[a.capacity * (D / 2) + row * (D / MX_BLOCK) + piece / 4] = (uint8_t)scale;
      s_new[D + (is_k ? 0 : D / MX_BLOCK) + piece / 4] = (uint8_t)scale;
    }
  }
  __syncthreads();
}

template <int D, bool PAGED, bool WEIGHTS, int NW>     // NW waves, which take turns on tiles of 32 rows
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(4, 4))) void decode_fp4_kernel(DecodeArgs a) {
  constexpr int GT = 8;                // query heads per KV head supported
  constexpr int TR = 32;               // rows of a wave's tile
  constexpr int UR = 2048 / D;         // rows a load instruction takes
  constexpr int NU = TR / UR;
  constexpr int DB = D / 16;           // 16-column blocks of the output
  constexpr int RS = D + 16;           // bf16 elements per LDS row of the V tile (rows 8 banks apart)
  constexpr int AR = D + 4;            // floats per query head of a wave's results
  constexpr int RB = D / 2, SB = D / MX_BLOCK;       // bytes of a row's codes, of its scales
  constexpr int WB = TR * RS * 2 > GT * AR * 4 ? TR * RS * 2 : GT * AR * 4;        // bytes of a wave's V tile, later of its results
  __shared__ float s_ml[NW][GT][2];
  __shared__ __attribute__((aligned(16))) unsigned char s_wave[NW][WB];
  __shared__ __attribute__((aligned(16))) uint8_t s_new[D + 2 * SB];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j16 = lane & 15, c = lane >> 4;
  const long long hidx = piece_head(a);
  const int chunk = blockIdx.y;
  const int len1 = a.meet.len1[a.head0 + hidx], len_old = a.kv_len[hidx];
  const long long off = a.kv_off[hidx];
  // Q as the B operand: lane (column j16, c) holds for step ks the dims that lane c of a row has there: [32 blk + 8 ks, + 8)
  const bool second = j16 >= 8;                        // this lane's column: against the second 16 keys of a tile
  const int urow = D == 128 ? j16 : j16 + 16 * (c >> 1), ublk = D == 128 ? c : c & 1;       // this lane's row of a load instruction's, and its block of that row
  dbf16x8_t qb[4];
  const uint16_t* qg = reinterpret_cast<const uint16_t*>(a.q) + (hidx * a.G + min(j16 & 7, a.G - 1)) * D + ublk * 32;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const du32x4_t x = *reinterpret_cast<const du32x4_t*>(qg + ks * 8), none = {0u, 0u, 0u, 0u};
    qb[ks] = __builtin_bit_cast(dbf16x8_t, D == 128 || (c >= 2) == second ? x : none);
  }
  asm volatile("" :: "s"(len1), "s"(len_old), "s"((int)off));             // (all three in one trip)
  const int arrive = arrivals(a, len1);
  if (chunk >= arrive) return;                       // the grid is the same for all heads (decode_plan)
  const bool can_append = can_append_to<PAGED>(a, off, len_old);
  const int len = len_old + (can_append ? 1 : 0);
  const int rows = head_chunk_rows(a, len);
  const int r_begin = chunk * rows;
  const int r_end = min(len, r_begin + rows);
  const RowMap at = make_row_map<PAGED>(a, hidx, off, len_old, can_append, r_begin, r_end);
  const Fresh fresh = fresh_row<WEIGHTS>(a, hidx, len_old, can_append);
  const bool has_fresh = fresh.there && fresh.row >= r_begin && fresh.row < r_end;   // uniform: the new row is in this piece

  // the piece's first row; the rows' offsets from it fit 32 bits
  const long long first_row = PAGED ? 0 : off + r_begin;
  const unsigned char* kc = reinterpret_cast<const unsigned char*>(a.k_c) + first_row * RB;
  const unsigned char* vc = reinterpret_cast<const unsigned char*>(a.v_c) + first_row * RB;
  const unsigned char* kcs = reinterpret_cast<const unsigned char*>(a.k_c) + a.capacity * RB + first_row * SB;
  const unsigned char* vcs = reinterpret_cast<const unsigned char*>(a.v_c) + a.capacity * RB + first_row * SB;

  struct Tile { du32x4_t k[NU], v[NU]; uint32_t ks[NU], vs[NU]; };
  // codes and scales of a tile; rows past the end of the piece: its last row once more, masked where they are used
  const auto load_tile = [&](Tile& x, int t) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int r = min(t + u * UR + urow, r_end - 1);
      if (PAGED) {
        const long long p = at(r);
        x.k[u] = __builtin_nontemporal_load(reinterpret_cast<const du32x4_t*>(kc + p * RB + ublk * 16));
        x.v[u] = __builtin_nontemporal_load(reinterpret_cast<const du32x4_t*>(vc + p * RB + ublk * 16));
        x.ks[u] = kcs[p * SB + ublk]; x.vs[u] = vcs[p * SB + ublk];
      } else {
        const uint32_t p = (uint32_t)(r - r_begin);
        x.k[u] = __builtin_nontemporal_load(reinterpret_cast<const du32x4_t*>(kc + p * RB + ublk * 16));
        x.v[u] = __builtin_nontemporal_load(reinterpret_cast<const du32x4_t*>(vc + p * RB + ublk * 16));
        x.ks[u] = kcs[p * SB + ublk]; x.vs[u] = vcs[p * SB + ublk];
      }
    }
  };
  const int first = r_begin + wave * TR;
  Tile next;
  if (first < r_end) load_tile(next, first);
  if (has_fresh) stage_new_row4<D>(a, hidx, at(fresh.row), s_new);       // (behind the loads)

  float m_run = DNEG_BIG, l_run = 0.f;       // of query j16 & 7 (all of its lanes hold a copy of m, a share of l)
  const uint32_t of_first = second ? 0u : ~0u;
  df32x4_t oacc[DB];                         // O^T[d = 16 db + 4c + r][column j16]
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = df32x4_t{0.f, 0.f, 0.f, 0.f};
  uint16_t* vt = reinterpret_cast<uint16_t*>(s_wave[wave]);
  const uint16_t* vf = vt + (4 * c + (j16 >> 2)) * RS + 4 * (j16 & 3);
#pragma unroll 1
  for (int t0 = first; t0 < r_end; t0 += NW * TR) {
    Tile x = next;
    load_tile(next, t0 + NW * TR);           // (past the end: the last row, which nobody looks at)
    if (has_fresh && t0 <= fresh.row && fresh.row < t0 + TR) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
        if (min(t0 + u * UR + urow, r_end - 1) == fresh.row) {
          x.k[u] = *reinterpret_cast<const du32x4_t*>(s_new + ublk * 16);
          x.v[u] = *reinterpret_cast<const du32x4_t*>(s_new + RB + ublk * 16);
          x.ks[u] = s_new[D + ublk]; x.vs[u] = s_new[D + SB + ublk];
        }
    }
    // ---- S^T: 4 keys of the column's 16
    df32x4_t s = {0.f, 0.f, 0.f, 0.f};
    if constexpr (D == 128) {
      df32x4_t s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(dbf16x8_t, mx_decode8(x.k[0][ks], x.ks[0])), qb[ks], s, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(dbf16x8_t, mx_decode8(x.k[NU - 1][ks], x.ks[NU - 1])), qb[ks], s1, 0, 0, 0);
      }
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) s[rr] = second ? s1[rr] : s[rr];
    } else {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(dbf16x8_t, mx_decode8(x.k[0][ks], x.ks[0])), qb[ks], s, 0, 0, 0);
    }
    const int key0 = t0 + (second ? 16 : 0) + 4 * c;
    float p[4], tmax = DNEG_BIG;
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) p[rr] = s[rr] * a.scale_log2;
    if (WEIGHTS && (j16 & 7) < a.G) *reinterpret_cast<df32x4_t*>(a.logits + (hidx * a.G + (j16 & 7)) * a.logit_rows + key0) = df32x4_t{p[0], p[1], p[2], p[3]};
    if (t0 + TR > r_end) {
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) p[rr] = key0 + rr < r_end ? p[rr] : 2.f * DNEG_BIG;
    }
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) tmax = fmaxf(tmax, p[rr]);
    float y0, y1;
    lane_pair<16>(tmax, y0, y1); tmax = fmaxf(y0, y1);
    lane_pair<32>(tmax, y0, y1); tmax = fmaxf(y0, y1);
    const float m_new = fmaxf(m_run, fmaxf(tmax, __uint_as_float(other_column(__float_as_uint(tmax)))));
    if (__builtin_amdgcn_ballot_w64(m_new > m_run)) {          // (of most tiles behind the first few nothing is rescaled)
      const float alpha = weight_of(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) oacc[db][rr] *= alpha;
      m_run = m_new;
    }
    // P of the lane's 4 keys in three parts.  The operands have all 32 keys in every column: first parts in columns 0-7 and second
    // ones in columns 8-15, then third ones in columns 0-7; the parts of the other 16 keys come from the query's other column.
    dbf16x8_t pb, pc;
    {
      uint32_t part[3][2], theirs[2], third[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        df32x2_t pv = {weight_of(p[2 * e] - m_run), weight_of(p[2 * e + 1] - m_run)};
        l_run += pv[0] + pv[1];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          part[i][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pv, dbf16x2_t));               // round to nearest even
          pv = df32x2_t{pv[0] - bf16_lo(part[i][e]), pv[1] - bf16_hi(part[i][e])};
        }
        theirs[e] = other_column(second ? part[0][e] : part[1][e]);
        third[e] = other_column(part[2][e]);
      }
      pb = __builtin_bit_cast(dbf16x8_t, second ? du32x4_t{theirs[0], theirs[1], part[1][0], part[1][1]} : du32x4_t{part[0][0], part[0][1], theirs[0], theirs[1]});
      pc = __builtin_bit_cast(dbf16x8_t, du32x4_t{part[2][0] & of_first, part[2][1] & of_first, third[0] & of_first, third[1] & of_first});
    }
    // ---- V through the wave's LDS tile
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      uint16_t* to = vt + (u * UR + urow) * RS + ublk * 32;
#pragma unroll
      for (int w = 0; w < 4; ++w) *reinterpret_cast<uint4*>(to + w * 8) = mx_decode8(x.v[u][w], x.vs[u]);
    }
    // the tile must be complete before it is read with another lane mapping (same wave: in order)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const ds16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_s16x4_ptr_t)(vf + db * 16));
      const ds16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_s16x4_ptr_t)(vf + 16 * RS + db * 16));
      const dbf16x8_t va = __builtin_bit_cast(dbf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
      oacc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pc, oacc[db], 0, 0, 0);
      oacc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb, oacc[db], 0, 0, 0);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  {
    float x, y;                                                // the sums of the lane groups
    lane_pair<16>(l_run, x, y); l_run = x + y;
    lane_pair<32>(l_run, x, y); l_run = x + y;
    l_run = add_ror8(l_run);                                   // and the two columns of a query
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) oacc[db][rr] = add_ror8(oacc[db][rr]);
  }
  // ---- per wave: everything to LDS in [q][d] form, where its V tile was
  if (j16 < GT) {
    if (c == 0) { s_ml[wave][j16][0] = m_run; s_ml[wave][j16][1] = l_run; }
    float* acc = reinterpret_cast<float*>(s_wave[wave]) + j16 * AR + 4 * c;
#pragma unroll
    for (int db = 0; db < DB; ++db) *reinterpret_cast<df32x4_t*>(acc + db * 16) = oacc[db];
  }
  __syncthreads();
  finish_piece<uint16_t, D, NW, GT, WB / 4, AR, WEIGHTS>(a, hidx, chunk, len, rows, can_append, arrive, s_ml, reinterpret_cast<const float*>(s_wave), fresh);
}

template <int D, bool WEIGHTS>
static void launch_fp4(const Dims& dm, const DecodeArgs& a, int grid_chunks, hipStream_t st) {
  const dim3 grid(dm.heads, grid_chunks);
  if (a.page_rows) hipLaunchKernelGGL((decode_fp4_kernel<D, true, WEIGHTS, 4>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((decode_fp4_kernel<D, false, WEIGHTS, 4>), grid, dim3(256), 0, st, a);
}
hipError_t launch_decode4(const Dims& dm, const DecodeArgs& a, int grid_chunks, bool weights, hipStream_t st) {
  if (dm.d == 128) weights ? launch_fp4<128, true>(dm, a, grid_chunks, st) : launch_fp4<128, false>(dm, a, grid_chunks, st);
  else if (dm.d == 64) weights ? launch_fp4<64, true>(dm, a, grid_chunks, st) : launch_fp4<64, false>(dm, a, grid_chunks, st);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace madakv
