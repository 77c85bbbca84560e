// Builds the reduced KV cache (paper Sec. 3.3: the evicted cache each head keeps):
//   k_c[kv_off + j, :] = k[head, kept_idx[kv_off + j], :]   and the same for v.
// Pure data movement, bound by HBM.  The reduced cache is one flat array of rows; a
// workgroup fills GATHER_ROWS consecutive rows of it, whichever heads they belong to, so
// every workgroup moves the same number of bytes whatever the per-head budgets are.
// A row is d * sizeof(T) bytes = LPR lanes x 16 bytes; a wave moves 64 / LPR rows per
// instruction and keeps UNROLL such loads of K and of V in flight before it stores.
#include "common.h"

#include <algorithm>

namespace madakv {

constexpr size_t GATHER_ROOM_LDS = 41 * 1024;   // three claims fit the 160 KB of a compute unit, four do not

// native vector type: arrays of it stay in registers (the HIP uint4 struct ends up in scratch)
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_t;

struct GatherArgs {
  const void* k; const void* v; const int32_t* kept_idx; const int64_t* kv_off; const int32_t* kv_len;
  void* k_c; void* v_c; const long long* call_range; const int32_t* blk2head;
  int n, B, H, L, blocks_per_batch;
  int li0, li1;          // layers [li0, li1) of the call are gathered by this launch
  long long capacity;    // rows of the reduced cache: the scales of a 4-bit cache sit behind the codes of so many
  long long region_tokens;
};

template <int LPR, int KIND>   // lanes per source row (row bytes / 16); KIND: 0 = rows are stored as they are, CACHE_E4M3 / CACHE_E2M1 = bf16 rows are encoded
__global__ __launch_bounds__(256) void gather_kernel(GatherArgs a) {
  constexpr int RPI = 64 / LPR;                 // rows per wave instruction
  constexpr int ROWS_PER_WAVE = GATHER_ROWS / 4;
  constexpr int ITERS = ROWS_PER_WAVE / RPI;
  const int b = blockIdx.y;
  const long long region = (long long)b * a.region_tokens;
  const long long call_start = a.call_range[b * 2], call_end = a.call_range[b * 2 + 1];
  // rows of the launch's layers: from the first head of layer li0 to the first head of layer li1
  const long long start = a.li0 == 0 ? call_start : a.kv_off[((long long)a.li0 * a.B + b) * a.H] - region;
  const long long end = a.li1 >= a.n ? call_end : a.kv_off[((long long)a.li1 * a.B + b) * a.H] - region;
  const long long blk = start / GATHER_ROWS + blockIdx.x;
  const long long tbl = blk - call_start / GATHER_ROWS;          // the block table is relative to the call's first block
  const long long row0 = blk * GATHER_ROWS;
  if (row0 >= end) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sub = lane / LPR, piece = lane % LPR;
  const int nh = a.n * a.H;
  int hh = a.blk2head[(long long)b * a.blocks_per_batch + tbl];
  const u32x4_t* kin = reinterpret_cast<const u32x4_t*>(a.k);
  const u32x4_t* vin = reinterpret_cast<const u32x4_t*>(a.v);
  u32x4_t* kout = reinterpret_cast<u32x4_t*>(a.k_c);
  u32x4_t* vout = reinterpret_cast<u32x4_t*>(a.v_c);

  // Phases, so that dependent index loads never sit between the row loads of another row
  // (load counters retire in order: a wait for an index would also wait for every row load
  // issued before it): kept positions + the segment table of the next few heads, then all
  // row loads, then all stores.
  long long dst[ITERS]; int kidx[ITERS]; bool inr[ITERS];
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    const long long r = row0 + wave * ROWS_PER_WAVE + it * RPI + sub;     // row relative to the region
    inr[it] = r >= start && r < end;
    dst[it] = region + r;
    kidx[it] = inr[it] ? a.kept_idx[dst[it]] : 0;                          // free slots hold garbage: unused below
  }
  // segments of the first head overlapping the block and its successors (they tile the range)
  constexpr int NC = 4;
  long long coff[NC + 1]; int clen[NC];
#pragma unroll
  for (int c = 0; c <= NC; ++c) {
    const int hc = min(hh + c, nh - 1);
    const long long hidx = ((long long)(hc / a.H) * a.B + b) * a.H + (hc % a.H);
    coff[c] = (hh + c < nh) ? a.kv_off[hidx] - region : end;               // past the last head: the end of the range
    if (c < NC) clen[c] = a.kv_len[hidx];
  }
  long long src[ITERS];
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    const long long r = dst[it] - region;
    src[it] = -1;
    if (inr[it]) {
      int hsel = hh; long long hoff = coff[0]; int hlen = clen[0];
#pragma unroll
      for (int c = 1; c < NC; ++c)
        if (hh + c < nh && coff[c] <= r) { hsel = hh + c; hoff = coff[c]; hlen = clen[c]; }
      if (hh + NC < nh && coff[NC] <= r) {
        // more than NC segments start inside this block (very short segments): walk on
        int h2 = hh + NC;
        while (h2 + 1 < nh) {
          const int li = (h2 + 1) / a.H, h = (h2 + 1) % a.H;
          if (a.kv_off[((long long)li * a.B + b) * a.H + h] - region > r) break;
          ++h2;
        }
        const long long hidx = ((long long)(h2 / a.H) * a.B + b) * a.H + (h2 % a.H);
        hsel = h2; hoff = a.kv_off[hidx] - region; hlen = a.kv_len[hidx];
      }
      const long long hidx = ((long long)(hsel / a.H) * a.B + b) * a.H + (hsel % a.H);
      if (r - hoff < hlen)                       // rows past kv_len are the free decode slots
        src[it] = hidx * a.L + kidx[it];
    }
  }
  u32x4_t kv[ITERS], vv[ITERS];
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    const long long s0 = src[it] >= 0 ? src[it] : 0;     // an in-bounds dummy keeps the load unconditional
    kv[it] = __builtin_nontemporal_load(kin + s0 * LPR + piece);     // rows are read once: keep them out of the caches
    vv[it] = __builtin_nontemporal_load(vin + s0 * LPR + piece);
  }
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    if (src[it] >= 0) {
      if (KIND == CACHE_E2M1) {
        // (a row's lanes are here together: mx_encode8 and mx_row_scales read across them)
        const uint32_t kx[4] = {kv[it][0], kv[it][1], kv[it][2], kv[it][3]}, vx[4] = {vv[it][0], vv[it][1], vv[it][2], vv[it][3]};
        uint32_t ks, vs;
        reinterpret_cast<uint32_t*>(a.k_c)[dst[it] * LPR + piece] = mx_encode8(kx, ks);
        reinterpret_cast<uint32_t*>(a.v_c)[dst[it] * LPR + piece] = mx_encode8(vx, vs);
        ks = mx_row_scales<LPR>(ks, piece); vs = mx_row_scales<LPR>(vs, piece);
        if (piece < 2) {                                             // lane 0 the scales of K, lane 1 those of V
          unsigned char* to = reinterpret_cast<unsigned char*>(piece ? a.v_c : a.k_c) + a.capacity * (LPR * 4);
          const uint32_t w = piece ? vs : ks;
          if (LPR == 16) reinterpret_cast<uint32_t*>(to)[dst[it]] = w;
          else reinterpret_cast<uint16_t*>(to)[dst[it]] = (uint16_t)w;
        }
      } else if (KIND == CACHE_E4M3) {
        // 8 bf16 -> 8 bytes per lane; a row of the reduced cache is LPR * 8 bytes
        typedef __attribute__((ext_vector_type(2))) unsigned int u32x2_t;
        u32x2_t ko, vo;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint32_t kb = 0, vb = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t kp = kv[it][w * 2 + e / 2], vp = vv[it][w * 2 + e / 2];
            const float kf = (e & 1) ? bf16_hi(kp) : bf16_lo(kp), vf = (e & 1) ? bf16_hi(vp) : bf16_lo(vp);
            kb |= f32_to_e4m3(kf) << (8 * e); vb |= f32_to_e4m3(vf) << (8 * e);
          }
          ko[w] = kb; vo[w] = vb;
        }
        reinterpret_cast<u32x2_t*>(a.k_c)[dst[it] * LPR + piece] = ko;
        reinterpret_cast<u32x2_t*>(a.v_c)[dst[it] * LPR + piece] = vo;
      } else {
        __builtin_nontemporal_store(kv[it], kout + dst[it] * LPR + piece);
        __builtin_nontemporal_store(vv[it], vout + dst[it] * LPR + piece);
      }
    }
  }
}

hipError_t launch_gather(const Dims& dm, const madakv_config& c, int li0, int nli, const void* k, const void* v,
                         const int32_t* kept_idx, const int64_t* kv_off, const int32_t* kv_len,
                         void* k_c, void* v_c, const void* ws, long long region_tokens,
                         int blocks_per_batch, int grid_blocks, hipStream_t st, bool leave_room) {
  GatherArgs a;
  a.k = k; a.v = v; a.kept_idx = kept_idx; a.kv_off = kv_off; a.kv_len = kv_len; a.k_c = k_c; a.v_c = v_c;
  a.call_range = reinterpret_cast<const long long*>(ws);
  a.blk2head = reinterpret_cast<const int32_t*>(reinterpret_cast<const char*>(ws) + ((size_t)dm.B * 2 * sizeof(long long) + 63) / 64 * 64);
  a.n = dm.n; a.B = dm.B; a.H = dm.H; a.L = dm.L; a.blocks_per_batch = blocks_per_batch;
  a.region_tokens = region_tokens;
  a.li0 = li0; a.li1 = li0 + nli;
  a.capacity = region_tokens * dm.B;
  const int row_bytes = dm.d * (c.dtype == MADAKV_BF16 ? 2 : 4);
  const int lpr = row_bytes / 16;
  dim3 grid(std::min(grid_blocks, blocks_per_batch), dm.B);
  // leave_room: statistics / selection kernels of another layer group run on a second stream meanwhile.
  // Eight of these workgroups fit a compute unit and would keep it full until the grid has drained; the
  // claim of GATHER_ROOM_LDS bytes of (unused) LDS holds them to three and leaves 37 KB: enough for a selection
  // workgroup over heads of up to 16K (34 KB; statistics, 50 KB, and longer heads once one of the three has left).  Eviction of 32 layers of 128 heads of 16K in one
  // call, median us: claims of 36 KB (four, 16 KB left) 4808, 41 KB 4795, 54 KB (two, 52 KB left) 4923; of 8 layers 1277,
  // 1274, 1292.  Beside such gathers a selection took 122 us and the statistics 125 on average (alone 58 and 60), when they
  // were 73 and 58 KB large and the claim 36 KB 245 and 166; the gather 444 instead of 425.
  const size_t lds = leave_room ? GATHER_ROOM_LDS : 0;
  if (c.cache_fp8 == CACHE_E2M1) {
    if (lpr == 8) hipLaunchKernelGGL((gather_kernel<8, CACHE_E2M1>), grid, dim3(256), lds, st, a);
    else if (lpr == 16) hipLaunchKernelGGL((gather_kernel<16, CACHE_E2M1>), grid, dim3(256), lds, st, a);
    else return hipErrorInvalidValue;
  } else if (c.cache_fp8) {
    if (lpr == 8) hipLaunchKernelGGL((gather_kernel<8, CACHE_E4M3>), grid, dim3(256), lds, st, a);
    else if (lpr == 16) hipLaunchKernelGGL((gather_kernel<16, CACHE_E4M3>), grid, dim3(256), lds, st, a);
    else return hipErrorInvalidValue;
  } else if (lpr == 8) hipLaunchKernelGGL((gather_kernel<8, 0>), grid, dim3(256), lds, st, a);
  else if (lpr == 16) hipLaunchKernelGGL((gather_kernel<16, 0>), grid, dim3(256), lds, st, a);
  else if (lpr == 32) hipLaunchKernelGGL((gather_kernel<32, 0>), grid, dim3(256), lds, st, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

// Rows of an encoded reduced cache back in the model's type, at the same places: k_rows[i, :] = k_c[i, :] for the rows the heads
// hold; the rest of k_rows and v_rows is left as it is.  A lane makes 16 bytes of a row.  Bound by HBM: a row is written with
// 4 d bytes and read with 2 d (8 bits) or 1.06 d (4 bits): 128 heads of 2K 4-bit rows of 128 dims 28 us, 6.1 TB/s.  (32 or 128 rows per
// workgroup, or stores through the caches: slower there, the same on few heads.)
struct RowsArgs {
  const void* k_c; const void* v_c; const int64_t* kv_off; const int32_t* kv_len; u32x4_t* k_rows; u32x4_t* v_rows;
  long long capacity;
  const int32_t* page_tbl; int entries, shift;      // of the call's first head; null without paging
  // null: rows go to the places they have in the cache.  Else: those of a batch item's heads (contiguous segments) to the front of its item_rows
  // rows, and where those of every head begin is left here
  int64_t* to_off;
  long long item_rows; int B, H, head0;             // head0: the launch's first head of the call
};
constexpr int ROWS_PER_BLOCK = 64;

template <int LPR, int KIND>   // lanes per row of the output
__global__ __launch_bounds__(256) void cache_rows_kernel(RowsArgs a) {
  constexpr int RPI = 256 / LPR, ITERS = ROWS_PER_BLOCK / RPI;
  const int head = blockIdx.y, len = a.kv_len[head];
  const int r0 = blockIdx.x * ROWS_PER_BLOCK;
  const long long off = a.kv_off[head];
  long long to = 0;
  if (a.to_off) {
    const int item = (a.head0 + head) / a.H % a.B;
    // (a batch item's segments follow each other: from the first of the call's on they fit its rows)
    to = min(max(off - a.kv_off[item * a.H - a.head0], 0ll), a.item_rows - max(len, 0)) + item * a.item_rows;
    if (r0 == 0 && threadIdx.x == 0) a.to_off[head] = to;
  }
  if (r0 >= len) return;
  const int32_t* tbl = a.page_tbl ? a.page_tbl + (long long)head * a.entries : nullptr;
  const int init_rows = tbl ? tbl[0] << a.shift : 0x7fffffff;
  const int sub = threadIdx.x / LPR, piece = threadIdx.x % LPR;
  long long at[ITERS];
  u32x4_t kv[ITERS], vv[ITERS];
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    const int r = min(r0 + it * RPI + sub, len - 1);       // (past the end: the last row once more)
    at[it] = off + r;
    if (r >= init_rows) { const int q = r - init_rows; at[it] = ((long long)tbl[1 + (q >> a.shift)] << a.shift) + (q & ((1 << a.shift) - 1)); }
  }
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    if (KIND == CACHE_E2M1) {
      const long long block = a.capacity * (LPR * 4) + at[it] * (LPR / 4) + piece / 4;          // of the scales
      const uint4 x = mx_decode8(reinterpret_cast<const uint32_t*>(a.k_c)[at[it] * LPR + piece], reinterpret_cast<const uint8_t*>(a.k_c)[block]);
      kv[it] = __builtin_bit_cast(u32x4_t, x);
      if (a.v_rows) vv[it] = __builtin_bit_cast(u32x4_t, mx_decode8(reinterpret_cast<const uint32_t*>(a.v_c)[at[it] * LPR + piece], reinterpret_cast<const uint8_t*>(a.v_c)[block]));
    } else {
      typedef __attribute__((ext_vector_type(2))) unsigned int u32x2_t;
      typedef __attribute__((ext_vector_type(2))) float f32x2_t;
      const u32x2_t k8 = reinterpret_cast<const u32x2_t*>(a.k_c)[at[it] * LPR + piece];
      const u32x2_t v8 = a.v_rows ? reinterpret_cast<const u32x2_t*>(a.v_c)[at[it] * LPR + piece] : u32x2_t{0u, 0u};
      // (every E4M3 value is a bf16: the upper half of the float is all there is of it)
      const auto pair = [](uint32_t w, bool high) {
        const f32x2_t f = high ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        return (__float_as_uint(f[0]) >> 16) | (__float_as_uint(f[1]) & 0xffff0000u);
      };
      kv[it] = u32x4_t{pair(k8[0], false), pair(k8[0], true), pair(k8[1], false), pair(k8[1], true)};
      vv[it] = u32x4_t{pair(v8[0], false), pair(v8[0], true), pair(v8[1], false), pair(v8[1], true)};
    }
  }
  if (a.to_off) {
#pragma unroll
    for (int it = 0; it < ITERS; ++it) at[it] = to + r0 + it * RPI + sub;
  }
#pragma unroll
  for (int it = 0; it < ITERS; ++it) {
    if (r0 + it * RPI + sub < len) {
      __builtin_nontemporal_store(kv[it], a.k_rows + at[it] * LPR + piece);
      if (a.v_rows) __builtin_nontemporal_store(vv[it], a.v_rows + at[it] * LPR + piece);
    }
  }
}

// most rows of a batch item that the call's heads hold, free ones included
static long long front_rows(const Dims& dm, const madakv_config& c) { return std::min(region_tokens_of(c), (long long)dm.n * dm.H * (c.ctx_len + c.max_new_tokens)); }
long long cache_rows_front(const Dims& dm, const madakv_config& c) { return dm.B * front_rows(dm, c); }
hipError_t launch_cache_rows(const Dims& dm, const madakv_config& c, const void* k_c, const void* v_c, const int64_t* kv_off, const int32_t* kv_len,
                             void* k_rows, void* v_rows, long long capacity_tokens, int longest_rows, const Paging& pg, int layer0, hipStream_t st,
                             int64_t* to_off) {
  RowsArgs a;
  a.to_off = to_off; a.B = dm.B; a.H = dm.H; a.item_rows = front_rows(dm, c);
  a.k_c = k_c; a.v_c = v_c; a.kv_off = kv_off; a.kv_len = kv_len; a.capacity = capacity_tokens;
  a.k_rows = static_cast<u32x4_t*>(k_rows); a.v_rows = static_cast<u32x4_t*>(v_rows);
  a.entries = pg.entries; a.shift = 0;
  while (pg.page_rows && (1 << a.shift) < pg.page_rows) ++a.shift;
  a.page_tbl = pg.page_rows ? pg.table + (long long)layer0 * dm.B * dm.H * pg.entries : nullptr;
  // heads in the second dimension of the grid, which holds 65535 of them
  for (int h0 = 0; h0 < dm.heads; h0 += 32768) {
    RowsArgs b = a;
    b.kv_off += h0; b.kv_len += h0;
    if (b.to_off) b.to_off += h0;
    b.head0 = h0;
    if (b.page_tbl) b.page_tbl += (long long)h0 * a.entries;
    const dim3 grid((unsigned)((std::max(longest_rows, 1) + ROWS_PER_BLOCK - 1) / ROWS_PER_BLOCK), std::min(32768, dm.heads - h0));
    const bool four = c.cache_fp8 == CACHE_E2M1;
    if (dm.d == 128 && four) hipLaunchKernelGGL((cache_rows_kernel<16, CACHE_E2M1>), grid, dim3(256), 0, st, b);
    else if (dm.d == 64 && four) hipLaunchKernelGGL((cache_rows_kernel<8, CACHE_E2M1>), grid, dim3(256), 0, st, b);
    else if (dm.d == 128) hipLaunchKernelGGL((cache_rows_kernel<16, CACHE_E4M3>), grid, dim3(256), 0, st, b);
    else if (dm.d == 64) hipLaunchKernelGGL((cache_rows_kernel<8, CACHE_E4M3>), grid, dim3(256), 0, st, b);
    else return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace madakv
