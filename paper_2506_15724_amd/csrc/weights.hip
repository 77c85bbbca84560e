// What a decode step paid to every row of the reduced cache, added up over the steps: acc[r] = decay * acc[r] + sum over the G
// query heads of softmax(scale * q K_c^T)[r], and the row of each head that has had the least of it.
//
// The attention kernels leave the logits of the step (4 bytes per row and query head beside the row's K and V of 68 to 1024)
// and, when a head's pieces have met, their maximum and the sum of 2^(logit - maximum); a second launch makes weights of them:
// a row's weight needs the whole head's sum, and a launch behind the first one knows it without anybody waiting for anybody.
// Per row: G logits, 4 bytes of acc read and written, 4 of its position.  What bounds it is a launch's latency: 4.5 us behind an
// attention of 17 (128 heads of 2K 8-bit rows) or 8 (4 heads of 2K rows, 7 queries each), 6.5 behind one of 91 (64 heads of
// 16K bf16 rows).  One launch instead of two would leave a head's rows to the one workgroup that finishes its attention (not measured).
// Workgroups of 1024 rows (256 to 4096: the same); the smallest sums of a
// head's workgroups meet like the pieces of its attention: as (sum, row) in one 64-bit word each, whose minimum does not depend
// on an order, counted at the head's counter, and the last one to arrive takes the least.
#include "decode_pieces.h"

#include <algorithm>

namespace madakv {

constexpr int RW_THREADS = 512, RW_UNROLL = 2, RW_ROWS = RW_THREADS * RW_UNROLL;

struct RowWeightArgs {
  WeightArgs w;
  const int64_t* kv_off; const int32_t* kv_len;
  uint32_t* count;                 // [heads of the model][G][MEET_COUNT_STRIDE], the counters of decode's pieces: zero between launches
  int G, B, H, page_shift, tbl_entries;
  const int32_t* page_tbl;         // null without paging
  long long head0;
};

template <int GT, bool PAGED>
__global__ __launch_bounds__(RW_THREADS) void row_weights_kernel(RowWeightArgs a) {
  const int hidx = blockIdx.x, chunk = blockIdx.y, tid = threadIdx.x;
  const WeightArgs& w = a.w;
  const long long off = a.kv_off[hidx], head = a.head0 + hidx;
  const int len = a.kv_len[hidx], fresh = w.fresh[hidx];
  const int pos = w.pos ? w.pos[(head / a.H) % a.B] : 0;
  const int32_t* tbl = PAGED ? a.page_tbl + head * a.tbl_entries : nullptr;
  const int init_rows = PAGED ? tbl[0] << a.page_shift : 0x7fffffff;
  asm volatile("" :: "s"(len), "s"((int)off), "s"(fresh), "s"(pos), "s"(init_rows));         // (all of them in one trip)
  const int chunks = max(1, min((int)gridDim.y, (len + RW_ROWS - 1) / RW_ROWS));
  if (chunk >= chunks) return;
  const long long newest = (long long)pos - w.recent;              // positions up to this one may go
  float mx[GT], inv[GT];
#pragma unroll
  for (int g = 0; g < GT; ++g) {
    const float2 ml = g < a.G ? *reinterpret_cast<const float2*>(w.head_ml + ((long long)hidx * a.G + g) * 2) : make_float2(0.f, 1.f);
    mx[g] = ml.x; inv[g] = __builtin_amdgcn_rcpf(ml.y);          // (1 unit of the last place: what exp2 is off by as well)
  }
  const float* lg = w.logits + (long long)hidx * a.G * w.logit_rows;
  // all of a thread's loads in front of what uses them
  float s[RW_UNROLL][GT], old[RW_UNROLL];
  long long at[RW_UNROLL];
  int kept[RW_UNROLL];
#pragma unroll
  for (int u = 0; u < RW_UNROLL; ++u) {
    const int r = min(chunk * RW_ROWS + u * RW_THREADS + tid, max(len, 1) - 1);      // (past the end: the last row once more)
    at[u] = off + r;
    if (PAGED && r >= init_rows) { const int q = r - init_rows; at[u] = ((long long)tbl[1 + (q >> a.page_shift)] << a.page_shift) + (q & ((1 << a.page_shift) - 1)); }
    if (len > 0) {
#pragma unroll
      for (int g = 0; g < GT; ++g) s[u][g] = g < a.G ? lg[(long long)g * w.logit_rows + r] : 0.f;
      old[u] = r == fresh ? 0.f : w.acc_in[at[u]];
      kept[u] = !w.kept_idx ? 0 : r == fresh ? pos : w.kept_idx[at[u]];
    }
  }
  unsigned long long best = ~0ull;
#pragma unroll
  for (int u = 0; u < RW_UNROLL; ++u) {
    const int r = chunk * RW_ROWS + u * RW_THREADS + tid;
    if (r >= len) continue;
    float paid = 0.f;
#pragma unroll
    for (int g = 0; g < GT; ++g) if (g < a.G) paid += weight_of(s[u][g] - mx[g]) * inv[g];
    const float sum = r == fresh ? paid : fmaf(w.decay, old[u], paid);
    w.acc_out[at[u]] = sum;
    if (w.kept_idx && r == fresh) w.kept_idx[at[u]] = pos;
    // (a sum that is no number: the last choice)
    const unsigned long long key = ((unsigned long long)(sum == sum ? float_key(sum) : 0xffffffffu) << 32) | (uint32_t)r;
    if (kept[u] <= newest) best = min(best, key);
  }
  if (!w.slot_out) return;
  __shared__ unsigned long long s_best[RW_THREADS / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) best = min(best, (unsigned long long)shfl_i64((long long)best, (tid & 63) ^ o));
  if ((tid & 63) == 0) s_best[tid >> 6] = best;
  __syncthreads();
  if (tid >= 64) return;
#pragma unroll
  for (int i = 0; i < RW_THREADS / 64; ++i) best = min(best, s_best[i]);
  if (chunks > 1) {
    unsigned long long* of_head = w.best + (long long)hidx * gridDim.y;
    uint32_t* count = a.count + head * a.G * MEET_COUNT_STRIDE;
    uint32_t arrived = 0u;
    if (tid == 0) __hip_atomic_store(of_head + chunk, best, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // the word is where everybody sees it
    if (tid == 0) arrived = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    arrived = (uint32_t)__builtin_amdgcn_readfirstlane((int)arrived);
    if (arrived + 1u != (uint32_t)chunks) return;
    if (tid == 0) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    best = ~0ull;
    for (int i = tid; i < chunks; i += 64) best = min(best, __hip_atomic_load(of_head + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = min(best, (unsigned long long)shfl_i64((long long)best, tid ^ o));
  }
  if (tid == 0) w.slot_out[hidx] = best == ~0ull ? -1 : (int32_t)(uint32_t)best;
}

static int row_chunks(int longest_rows) { return (std::max(longest_rows, 1) + RW_ROWS - 1) / RW_ROWS; }
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Behind what decode itself takes of the workspace: logits, the heads' (max, sum), their new rows, the smallest sums of
// their workgroups.  rows: the longest segment there can be.
size_t weights_ws_bytes(const Dims& dm, const madakv_config& c) {
  const size_t heads = dm.heads, rows = (size_t)c.ctx_len + c.max_new_tokens;
  return up256(decode_ws_bytes(dm, c)) + up256(heads * dm.G * ((rows + 31) / 32 * 32) * 4) + up256(heads * dm.G * 8) + up256(heads * 4) + up256(heads * row_chunks((int)rows) * 8);
}
void weights_ws_layout(const Dims& dm, const madakv_config& c, void* ws, WeightArgs& w) {
  const size_t heads = dm.heads, rows = (size_t)c.ctx_len + c.max_new_tokens;
  char* p = static_cast<char*>(ws) + up256(decode_ws_bytes(dm, c));
  w.logit_rows = (int)((rows + 31) / 32 * 32);
  w.logits = reinterpret_cast<float*>(p); p += up256(heads * dm.G * (size_t)w.logit_rows * 4);
  w.head_ml = reinterpret_cast<float*>(p); p += up256(heads * dm.G * 8);
  w.fresh = reinterpret_cast<int32_t*>(p); p += up256(heads * 4);
  w.best = reinterpret_cast<unsigned long long*>(p);
}

template <int GT>
static void launch_rw(const RowWeightArgs& a, const dim3& grid, hipStream_t st) {
  if (a.page_tbl) hipLaunchKernelGGL((row_weights_kernel<GT, true>), grid, dim3(RW_THREADS), 0, st, a);
  else hipLaunchKernelGGL((row_weights_kernel<GT, false>), grid, dim3(RW_THREADS), 0, st, a);
}
hipError_t launch_row_weights(const Dims& dm, const madakv_config& c, const WeightArgs& w, const int64_t* kv_off, const int32_t* kv_len,
                              const Meet& meet, int longest_rows, const Paging& pg, int layer0, hipStream_t st) {
  RowWeightArgs a;
  a.w = w; a.kv_off = kv_off; a.kv_len = kv_len; a.count = meet.count;
  a.G = dm.G; a.B = dm.B; a.H = dm.H; a.head0 = (long long)layer0 * dm.B * dm.H;
  a.page_shift = 0; a.tbl_entries = pg.entries; a.page_tbl = pg.page_rows ? pg.table : nullptr;
  while (pg.page_rows && (1 << a.page_shift) < pg.page_rows) ++a.page_shift;
  const dim3 grid(dm.heads, row_chunks(std::min(longest_rows, c.ctx_len + c.max_new_tokens)));
  if (dm.G == 1) launch_rw<1>(a, grid, st);
  else if (dm.G <= 4) launch_rw<4>(a, grid, st);
  else launch_rw<8>(a, grid, st);
  return hipGetLastError();
}

}  // namespace madakv
