// Attention of many query rows over tiles of 64 keys that lie in LDS: what the kernels of prompt attention and of attention of a
// drafted tree share.  A wave owns 32 query rows ("columns": they are operand B) and keeps their softmax and output in
// registers; K and V of a tile are operand A.
//   S^T[key][col] = K . Q^T      a lane then has 16 of 32 keys for ONE column, lane i and lane i + 32 the two halves: maximum, sum
//                                and weights of a column are in-lane work
//   O^T[dim][col] += V^T . P^T   the lane's weights are, as they come out of S^T, its elements of operand B under an order of the keys
//                                that transposing reads of V give operand A as well: no data moves between lanes
// The softmax goes over the keys once.  Weights are taken against a reference per column, the largest logit of the first tile that the column
// sees something of, and not against a running maximum: another reference, which rescales what has been summed, is only taken
// when a sum has passed ATT_FAR (relative precision does not depend on the reference, and bf16 has the range of fp32).  That saves the
// search for the maximum, a third of the vector instructions of a tile, and all rescaling for keys of ordinary logits.
// Logits, weights, sums and outputs are held in 32 bits.  bf16 inputs: the weights enter the second product as PARTS bf16 numbers, each of which leaves
// up to 2^-8 of what it stands for.  Three where the output is fp32: all 24 bits.  Where the output is bf16, too: two in trees of few columns, 16 bits as in
// decode; one, by choice, where the matrix unit is what a call waits for, in prompts and in trees of many columns.  There a rounding of up to 2^-8 of every weight,
// independent from key to key, leaves outputs off by 0.0021-0.0023 (2-norm, of random rows) where their own rounding makes 0.0016; a second part costs 14-37% more
// time (prompts of 8192 positions 524 -> 713 us, 28/4 heads of 16384 1770 -> 2430; 60 nodes of 2 x 32/8 heads of 16384 4-bit rows 51.8 -> 62.8, 32 nodes of
// 4 x 32/8 heads of bf16 ones 72 -> 83).  A caller who needs those bits has them with fp32 outputs.
#pragma once
#include "common.h"

// The loads straight into LDS say in their clobber lists that they set m0 and write memory: the compiler sees neither of them, and may set m0 once for several
// instructions of its own.  (It warns that m0 is a reserved register: it keeps nothing there that it would not set again.)
#pragma clang diagnostic ignored "-Winline-asm"

namespace madakv {

typedef __attribute__((ext_vector_type(8))) __bf16 at_bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 at_bf16x2_t;
typedef __attribute__((ext_vector_type(2))) float at_f32x2_t;
typedef __attribute__((ext_vector_type(4))) float at_f32x4_t;
typedef __attribute__((ext_vector_type(16))) float at_f32x16_t;
typedef __attribute__((ext_vector_type(4))) short at_s16x4_t;
typedef __attribute__((ext_vector_type(8))) unsigned short at_u16x8_t;
typedef __attribute__((ext_vector_type(4))) unsigned int at_u32x4_t;
typedef __attribute__((ext_vector_type(2))) unsigned int at_u32x2_t;
typedef __attribute__((address_space(3))) at_s16x4_t* at_lds_s16x4_ptr_t;
typedef __attribute__((address_space(3))) const at_u32x4_t* at_lds_u32x4_ptr_t;

constexpr int ATT_TILE = 64;                    // keys of a tile
constexpr float ATT_FAR = 0x1p24f;              // sums beyond it have left their reference behind

// the sum of a value over the two lanes of a column, in both of them; the larger one
__device__ __forceinline__ float both_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float both_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// the key of a subtile of 32 that element i of a lane's 16 logits belongs to
__device__ __forceinline__ int key_of(int i, int half) { return 8 * (i >> 2) + 4 * half + (i & 3); }
constexpr __device__ __forceinline__ at_f32x16_t zero16() {
  return at_f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}

// How rows of D elements of T lie in LDS and enter the matrix instructions.  Rows are as long as in memory; their 16-byte pieces are
// permuted (by an exclusive or with something of the row number), so that neither operand's reads collide in the banks.
// PARKED: V is written by threads that have two or four neighbouring pieces of a row each, whose stores would meet in the banks: rows permute the pieces of
// every four as well.  (Rows of 4 bits gain 3-5%, of 8 bits nothing; where rows come straight into LDS prompts of 64 dims lose 3%.)
template <typename T, int D, bool PARKED = false> struct AttnTile;

template <int D, bool PARKED> struct AttnTile<uint16_t, D, PARKED> {
  static constexpr int ROWB = D * 2, PPR = D / 8, BYTES = ATT_TILE * ROWB;
  static constexpr int KS = D / 16;             // contraction steps of S^T
  static constexpr int DB = D / 32;             // blocks of 32 dims of the output
  struct Query { at_bf16x8_t x[KS]; };
  template <int PARTS> struct Weights { at_bf16x8_t part[PARTS][2]; };          // of 32 keys, as operand B
  static __device__ __forceinline__ int k_slot(int row, int piece) { return piece ^ (D == 128 ? row & 15 : row >> 1 & 7); }
  static __device__ __forceinline__ int v_slot(int row, int piece) { return piece ^ (D == 128 ? 4 * (row & 3) : 4 * (row >> 1 & 1)) ^ (PARKED ? (D == 128 ? row & 3 : row >> 1 & 3) : 0); }
  // a column's query: for step ks elements [half D/2 + 8 ks, + 8)
  static __device__ __forceinline__ void load(Query& q, const uint16_t* row, int half) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q.x[ks] = *reinterpret_cast<const at_bf16x8_t*>(row + half * (D / 2) + ks * 8);
  }
  // (here and now: a wait for the query in a loop would be one for the tiles on their way as well)
  static __device__ __forceinline__ void await(Query& q) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q.x[ks]));
  }
  // logits of the 32 keys from row0 of the tile on
  static __device__ __forceinline__ at_f32x16_t scores(const unsigned char* kt, int row0, int lane, const Query& q) {
    const int half = lane >> 5, row = row0 + (lane & 31);
    at_f32x16_t s = zero16();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const at_bf16x8_t a = *reinterpret_cast<const at_bf16x8_t*>(kt + row * ROWB + k_slot(row, half * KS + ks) * 16);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q.x[ks], s, 0, 0, 0);
    }
    return s;
  }
  template <int PARTS>
  static __device__ __forceinline__ void pack(const float (&p)[16], Weights<PARTS>& w) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      at_u32x4_t x[PARTS];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        at_f32x2_t y = {p[8 * s + 2 * e], p[8 * s + 2 * e + 1]};
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          x[k][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, at_bf16x2_t));             // to nearest even
          if (k + 1 < PARTS) y = at_f32x2_t{y[0] - bf16_lo(x[k][e]), y[1] - bf16_hi(x[k][e])};
        }
      }
#pragma unroll
      for (int k = 0; k < PARTS; ++k) w.part[k][s] = __builtin_bit_cast(at_bf16x8_t, x[k]);
    }
  }
  template <int PARTS>
  static __device__ __forceinline__ float weight(const Weights<PARTS>& w, int i) {
    float x = 0.f;
#pragma unroll
    for (int k = PARTS - 1; k >= 0; --k)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float y = bf16_bits_to_f32(__builtin_bit_cast(at_u16x8_t, w.part[k][j >> 3])[j & 7]);
        x += i == j ? y : 0.f;
      }
    return x;
  }
  // output += V^T . P^T over the 32 keys from row0 on
  template <int PARTS>
  static __device__ __forceinline__ void add(const unsigned char* vt, int row0, int lane, const Weights<PARTS>& w, at_f32x16_t (&o)[DB]) {
    // A transposing read takes, per 16 lanes, four rows of 16 dims: lane j points at dims 4 (j & 3).. of row j >> 2 and gets dim j of
    // the four rows.  Lanes 0-15 take dims 0-15, 16-31 dims 16-31 of keys 0-3, lanes 32-63 the same of keys 4-7.
    const int half = lane >> 5, r = row0 + 4 * half + ((lane & 15) >> 2);
    const int d0 = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const auto read = [&](int row) {
          const int piece = (32 * db + d0) / 8;
          return __builtin_amdgcn_ds_read_tr16_b64_v4i16((at_lds_s16x4_ptr_t)(vt + row * ROWB + v_slot(row, piece) * 16 + (d0 & 7) * 2));
        };
        const at_s16x4_t v0 = read(r + 16 * s), v1 = read(r + 16 * s + 8);
        const at_bf16x8_t a = __builtin_bit_cast(at_bf16x8_t, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int k = PARTS - 1; k >= 0; --k) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, w.part[k][s], o[db], 0, 0, 0);
      }
  }
  // four neighbouring dims of a row of V
  static __device__ __forceinline__ at_f32x4_t value4(const unsigned char* vt, int row, int dim) {
    const at_u32x2_t x = *reinterpret_cast<const at_u32x2_t*>(vt + row * ROWB + v_slot(row, dim / 8) * 16 + (dim & 7) * 2);
    return at_f32x4_t{bf16_lo(x[0]), bf16_hi(x[0]), bf16_lo(x[1]), bf16_hi(x[1])};
  }
};

template <int D, bool PARKED> struct AttnTile<float, D, PARKED> {
  static constexpr int ROWB = D * 4, PPR = D / 4, BYTES = ATT_TILE * ROWB;
  static constexpr int DB = D / 32;
  struct Query { float x[D / 2]; };
  template <int PARTS> struct Weights { float x[16]; };
  template <int PARTS>
  static __device__ __forceinline__ void pack(const float (&p)[16], Weights<PARTS>& w) {
#pragma unroll
    for (int i = 0; i < 16; ++i) w.x[i] = p[i];
  }
  template <int PARTS>
  static __device__ __forceinline__ float weight(const Weights<PARTS>& w, int i) {
    float x = w.x[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) x = i == j ? w.x[j] : x;
    return x;
  }
  static __device__ __forceinline__ int k_slot(int row, int piece) { return piece ^ (row % 16); }
  static __device__ __forceinline__ int v_slot(int row, int piece) { return piece ^ (row % 16); }
  static __device__ __forceinline__ void load(Query& q, const float* row, int half) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const at_f32x4_t x = *reinterpret_cast<const at_f32x4_t*>(row + half * (D / 2) + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) q.x[4 * i + e] = x[e];
    }
  }
  static __device__ __forceinline__ void await(Query& q) {
#pragma unroll
    for (int i = 0; i < D / 2; ++i) asm volatile("" : "+v"(q.x[i]));
  }
  static __device__ __forceinline__ at_f32x16_t scores(const unsigned char* kt, int row0, int lane, const Query& q) {
    const int half = lane >> 5, row = row0 + (lane & 31);
    at_f32x16_t s = zero16();
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const at_f32x4_t a = *reinterpret_cast<const at_f32x4_t*>(kt + row * ROWB + k_slot(row, half * (D / 8) + i) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], q.x[4 * i + e], s, 0, 0, 0);
    }
    return s;
  }
  template <int PARTS>
  static __device__ __forceinline__ void add(const unsigned char* vt, int row0, int lane, const Weights<PARTS>& w, at_f32x16_t (&o)[DB]) {
    const int half = lane >> 5;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int row = row0 + key_of(i, half);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const int dim = 32 * db + (lane & 31);
        const float a = *reinterpret_cast<const float*>(vt + row * ROWB + v_slot(row, dim / 4) * 16 + (dim & 3) * 4);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w.x[i], o[db], 0, 0, 0);
      }
    }
  }
  static __device__ __forceinline__ at_f32x4_t value4(const unsigned char* vt, int row, int dim) {
    return *reinterpret_cast<const at_f32x4_t*>(vt + row * ROWB + v_slot(row, dim / 4) * 16);
  }
};

// What a wave holds of its columns: a lane has half of the keys of one column in sum (ref is the same in both lanes of a column), dims
// key_of(i, half) of each block of 32 in o.
template <int D> struct AttnState {
  float ref, sum;                               // ref: log2 units, -inf: nothing seen yet
  at_f32x16_t o[D / 32];
  __device__ __forceinline__ void clear() {
    ref = -__builtin_inff(); sum = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = zero16();
  }
};

// A column's output, divided by its sum: 8 (4-byte elements: 4) neighbouring dims per store, which the two lanes of a column bring together.
// to: the column's row; mine: it is to be stored.
template <typename OT, int D>
__device__ __forceinline__ void store_column(OT* to, bool mine, int half, const at_f32x16_t (&o)[D / 32], float inv) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    if constexpr (sizeof(OT) == 4) {
      if (mine) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<at_f32x4_t*>(to + 32 * db + 8 * g + 4 * half) = at_f32x4_t{o[db][4 * g] * inv, o[db][4 * g + 1] * inv, o[db][4 * g + 2] * inv, o[db][4 * g + 3] * inv};
      }
    } else {
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        uint32_t w[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int i = 4 * (g + h) + 2 * e;
            w[h][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((at_f32x2_t{o[db][i] * inv, o[db][i + 1] * inv}), at_bf16x2_t));
          }
        const auto x = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false), y = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
        if (mine) *reinterpret_cast<at_u32x4_t*>(to + 32 * db + 8 * (g + half)) = at_u32x4_t{x[0], y[0], x[1], y[1]};
      }
    }
  }
}
// what is not finite anywhere in a wave's output
template <int D>
__device__ __forceinline__ bool not_finite(const AttnState<D>& st) {
  float z = 0.f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) z = fmaf(st.o[db][i], 0.f, z);
  return z != z;
}

__device__ __forceinline__ float sum16(const float (&p)[16]) {
  return (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]))) + (((p[8] + p[9]) + (p[10] + p[11])) + ((p[12] + p[13]) + (p[14] + p[15])));
}

// What another wave has of the same columns from other keys, added: its reference and sum, its output [dims].  (One that has seen nothing: reference
// -inf, weight 0.)
template <int D>
__device__ __forceinline__ void merge_halves(AttnState<D>& st, float& sum, const float (&ml)[2], const float* o, int half) {
  const float m = fmaxf(st.ref, ml[0]);
  const float f1 = st.ref == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(st.ref - m), f2 = ml[0] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(ml[0] - m);
  // (what is no number stays none)
  sum = (st.ref == -__builtin_inff() && sum == 0.f ? 0.f : sum * f1) + (ml[0] == -__builtin_inff() && ml[1] == 0.f ? 0.f : ml[1] * f2);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const at_f32x4_t y = *reinterpret_cast<const at_f32x4_t*>(o + 32 * db + 8 * g + 4 * half);
#pragma unroll
      for (int e = 0; e < 4; ++e) st.o[db][4 * g + e] = st.o[db][4 * g + e] * f1 + y[e] * f2;
    }
  st.ref = m;
}

// The logits of a subtile -> weights and their sum t, against the column's reference, which moves where it has to:
// where a column has none yet, has left it far behind, or holds no number.  s: masked logits are -inf.
template <int D>
__device__ __forceinline__ void attn_look(AttnState<D>& st, const at_f32x16_t& s, float (&p)[16], float& t, float scale_log2) {
#pragma unroll
  for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale_log2, -st.ref));
  t = sum16(p);
  const bool near = both_sum(st.sum + t) < ATT_FAR;   // (the same in both lanes of a column; not: no number)
  if (__builtin_amdgcn_ballot_w64(!near) == 0) return;
  float top = s[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
  top = both_max(top) * scale_log2;
  if (near) return;
  if (top > -__builtin_inff()) {
    const float r = fmaxf(st.ref, top);
    const float f = st.ref == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(st.ref - r);
    st.sum *= f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[db][i] *= f;
    st.ref = r;
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale_log2, -r));
    t = sum16(p);
  } else if (st.ref == -__builtin_inff()) {           // nothing but masked keys, and nothing before
    bool number = true;
#pragma unroll
    for (int i = 0; i < 16; ++i) number = number && s[i] == s[i];
    if (number) {
      t = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = 0.f;
    }
  }
}

}  // namespace madakv
