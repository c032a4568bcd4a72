// The C ABI of quantised inference (include/awe.h): argument checks on the host, then the launches.
#include "awe_quant.h"

#include <algorithm>

namespace awe {
namespace {

awe_status refuse(awe_status st, const char* msg) {
  set_error(msg);
  return st;
}
awe_status invalid(const char* msg) { return refuse(AWE_ERR_INVALID_VALUE, msg); }

// No C++ exception crosses the interface (the messages allocate).
template <class F>
awe_status guarded(F f) {
  try {
    return f();
  } catch (...) {
    return AWE_ERR_HIP;
  }
}

int64_t elem_bytes(awe_dtype t) { return t == AWE_I8 ? 1 : (t == AWE_F32 ? 4 : 2); }
bool is_real(awe_dtype t) { return t == AWE_F32 || t == AWE_BF16 || t == AWE_F16; }
bool aligned(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

constexpr int64_t kMost = 0x7fffff00LL;          // sizes of a product, blocks of a cache
constexpr int64_t kMostTokens = int64_t(1) << 30;  // of a sequence (positions past its end stay within 32 bits)
constexpr int64_t kMostRows = int64_t(1) << 27;    // of a batch (they span the grid)
constexpr int64_t kMostStride = int64_t(1) << 40;
// Bytes from one row of a product's operand to the next: the kernels reach a tile's 256 rows by 32 bits.
constexpr int64_t kMostRow = int64_t(1) << 24;

awe_status w4_impl(const W4Launch& g, hipStream_t stream) {
  if (g.M < 0 || g.N < 0 || g.K < 0) return invalid("negative size");
  if (g.x_type != AWE_BF16 && g.x_type != AWE_F16 && g.x_type != AWE_I8) return invalid("bad x_type");
  if (!is_real(g.s_type)) return invalid("bad s_type");
  if (!is_real(g.y_type)) return invalid("bad y_type");
  if (g.x_scales != nullptr && g.x_type != AWE_I8) return invalid("x_scales belong to int8 X");
  if (g.group <= 0 || (g.group % 32 != 0 && g.group < g.K))
    return invalid("group must be a multiple of 32, or at least K");
  if (g.M > kMost || g.N > kMost || g.K > kMost) return refuse(AWE_ERR_UNSUPPORTED, "M, N or K too large");
  if (g.M == 0 || g.N == 0) return AWE_OK;
  if (g.y == nullptr || g.ldy < g.N) return invalid("bad Y or ldy");
  if (!aligned(g.y, elem_bytes(g.y_type))) return invalid("Y is not aligned to its element");
  if (g.K > 0) {
    const int64_t groups = (g.K + g.group - 1) / g.group;
    if (g.x == nullptr || g.w == nullptr || g.scales == nullptr) return invalid("X, W or w_scales is NULL");
    if (g.ldx < g.K || g.ldw < (g.K + 1) / 2 || g.lds < groups || (g.zeros != nullptr && g.ldz < groups))
      return invalid("leading dimension too small");
    if (g.ldx >= kMostRow / elem_bytes(g.x_type) || g.ldw >= kMostRow || g.lds >= kMostRow / elem_bytes(g.s_type) ||
        (g.zeros != nullptr && g.ldz >= kMostRow))
      return refuse(AWE_ERR_UNSUPPORTED, "rows of an operand too far apart");
    if (!aligned(g.x, elem_bytes(g.x_type)) || !aligned(g.scales, elem_bytes(g.s_type)) || !aligned(g.x_scales, 4))
      return invalid("an operand is not aligned to its element");
  }
  W4Launch h = g;
  if (h.K == 0) h.x_scales = nullptr;  // zeros, whatever the scales are
  return launch_w4(h, stream);
}

awe_status check_cache(const awe_cache* c) {
  if (c == nullptr) return invalid("cache is NULL");
  if (c->num_blocks < 0 || c->heads < 1) return invalid("bad number of blocks or heads");
  if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128)
    return refuse(AWE_ERR_UNSUPPORTED, "block must be 16, 32, 64 or 128 tokens");
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return refuse(AWE_ERR_UNSUPPORTED, "head_dim must be 64, 128 or 256");
  if (c->num_blocks > kMost || c->heads > 65535) return refuse(AWE_ERR_UNSUPPORTED, "too many blocks or heads");
  return AWE_OK;
}

awe_status check_batch(const awe_cache& c, const awe_batch* b) {
  if (b == nullptr) return invalid("batch is NULL");
  if (b->sequences < 0 || b->rows < 0 || b->max_rows < 0 || b->max_length < 0 || b->ld_blocks < 0)
    return invalid("negative size");
  if (b->rows > kMostRows || b->max_rows > kMostRows || b->max_length > kMostTokens || b->sequences > 0xffffff)
    return refuse(AWE_ERR_UNSUPPORTED, "too many rows, tokens or sequences");
  if (b->ld_blocks < (b->max_length + c.block - 1) / c.block) return invalid("ld_blocks * block < max_length");
  return AWE_OK;
}

// The device arrays of a call that has something to do.
awe_status check_arrays(const awe_cache& c, const awe_batch& b, const int32_t* flag) {
  if (b.starts == nullptr || b.lengths == nullptr || (b.blocks == nullptr && b.max_length > 0))
    return invalid("starts, lengths or blocks is NULL");
  if (!aligned(b.starts, 4) || !aligned(b.lengths, 4) || !aligned(b.blocks, 4) || !aligned(flag, 4))
    return invalid("an int32 array is not aligned");
  if (c.num_blocks > 0) {
    if (c.k == nullptr || c.v == nullptr || c.k_scales == nullptr || c.v_scales == nullptr)
      return invalid("a buffer of the cache is NULL");
    if (!aligned(c.k, 16) || !aligned(c.v, 16)) return invalid("k and v of the cache must be aligned to 16 bytes");
    if (!aligned(c.k_scales, 4) || !aligned(c.v_scales, 4)) return invalid("scales are not aligned");
  }
  return AWE_OK;
}

bool empty(const awe_batch& b) { return b.sequences == 0 || b.rows == 0 || b.max_rows == 0; }

awe_status check_rows(const Rows& r, awe_dtype type) {
  if (r.p == nullptr) return invalid("a row tensor is NULL");
  if (!aligned(r.p, elem_bytes(type))) return invalid("a row tensor is not aligned to its element");
  if (r.row < 0 || r.head < 0) return invalid("negative stride");
  if (r.row > kMostStride || r.head > kMostStride) return refuse(AWE_ERR_UNSUPPORTED, "stride too large");
  return AWE_OK;
}

// Whether the elements of a written row tensor are distinct: heads inside rows, or rows inside heads.
bool distinct(const Rows& r, int64_t rows, int64_t heads, int64_t dim) {
  using Wide = __int128;  // kMostRows rows at a stride of kMostStride pass 64 bits
  const bool by_row = (heads == 1 || r.head >= dim) && (rows == 1 || r.row >= Wide(heads - 1) * r.head + dim);
  const bool by_head = (rows == 1 || r.row >= dim) && (heads == 1 || r.head >= Wide(rows - 1) * r.row + dim);
  return by_row || by_head;
}

awe_status cache_impl(const awe_cache* cache, const awe_batch* batch, const Rows& k, const Rows& v, awe_dtype type,
                      int32_t* flag, bool load, hipStream_t stream) {
  awe_status st = check_cache(cache);
  if (st == AWE_OK) st = check_batch(*cache, batch);
  if (st != AWE_OK) return st;
  if (!is_real(type)) return invalid("bad type");
  if (empty(*batch)) return AWE_OK;
  st = check_arrays(*cache, *batch, flag);
  if (st == AWE_OK) st = check_rows(k, type);
  if (st == AWE_OK) st = check_rows(v, type);
  if (st != AWE_OK) return st;
  if (load)
    for (const Rows* r : {&k, &v})
      if (!distinct(*r, batch->rows, cache->heads, cache->head_dim)) return invalid("written elements share memory");
  const CacheLaunch g{*cache, *batch, type, k, v, flag};
  return load ? launch_cache_load(g, stream) : launch_cache_store(g, stream);
}

awe_status check_heads(const awe_cache& c, const awe_batch& b, int32_t q_heads) {
  if (q_heads < 1 || q_heads % c.heads != 0) return invalid("q_heads must be a multiple of the cache's heads");
  if (q_heads > 65535) return refuse(AWE_ERR_UNSUPPORTED, "too many heads");
  // (so that the plan's counts stay within 64 bits, and its columns within 32)
  if (std::min(b.rows, b.max_rows) * q_heads > (int64_t(1) << 30)) return refuse(AWE_ERR_UNSUPPORTED, "too many rows");
  return AWE_OK;
}

awe_status attend_impl(const awe_cache* cache, const awe_batch* batch, const Rows& q, int32_t q_heads, awe_dtype type,
                       float scale, bool causal, const Rows& o, void* ws, size_t ws_bytes, int32_t* flag,
                       hipStream_t stream) {
  awe_status st = check_cache(cache);
  if (st == AWE_OK) st = check_batch(*cache, batch);
  if (st == AWE_OK) st = check_heads(*cache, *batch, q_heads);
  if (st != AWE_OK) return st;
  if (type != AWE_BF16 && type != AWE_F16) return invalid("bad type");
  if (empty(*batch)) return AWE_OK;
  st = check_arrays(*cache, *batch, flag);
  if (st == AWE_OK) st = check_rows(q, type);
  if (st == AWE_OK) st = check_rows(o, type);
  if (st != AWE_OK) return st;
  if (!distinct(o, batch->rows, q_heads, cache->head_dim)) return invalid("written elements share memory");
  const size_t need = plan_attend(*cache, *batch, q_heads).workspace;
  if (need > 0 && (ws == nullptr || ws_bytes < need))
    return refuse(AWE_ERR_WORKSPACE, "workspace smaller than awe_cache_attend_workspace_bytes");
  if (need > 0 && !aligned(ws, 16)) return invalid("workspace must be aligned to 16 bytes");
  const AttendLaunch g{*cache, *batch, type, q, o, q_heads, scale, causal, ws, flag};
  return launch_cache_attend(g, stream);
}

}  // namespace

// Columns of their own read each token once for 128 columns, but a workgroup goes through all of a sequence; 16 columns
// whose tokens are split over waves and workgroups read it eight times as often.  So splitting wins while there are
// few tiles of 16 columns, or where columns leave most of a tile of 128 empty.  In us, split / own columns, 8 heads
// of 64, 128 and 256:
//   8 sequences of 2048, 64 columns each     22 /  80    33 /  96    59 / 115
//   8 of 2048, 256 (1024 tiles)              52 /  75    79 /  93   175 / 125
//   1 of 8192, 1024 (512 tiles)              82 / 264   140 / 322   327 / 416
//   1 of 8192, 2048 (1024 tiles)            138 / 264   231 / 321   523 / 418
//  64 of 2048, 8                             33 / 100    52 / 128   124 / 251
//  64 of 2048, 64 (2048 tiles)               97 / 100   178 / 132   406 / 256
// (Heads of 64 and 128 would gain from splitting a little beyond the 900 tiles, heads of 256 lose from there on.)
// The choice is the batch's, by max_rows: a prompt beside sequences of few rows makes all of them go the prompt's way
// (2048 rows and one row over 65,536 tokens, 8 heads of 128: 2805 us in one call, 110 and 35 in two).
AttendPlan plan_attend(const awe_cache& c, const awe_batch& b, int32_t q_heads) {
  constexpr int64_t kFewTiles = 900, kTilesPerWide = 3;
  constexpr int64_t kFill = 4096;   // workgroups that keep the chip busy to the end of ragged sequences
  constexpr int64_t kChunk = 1024;  // fewest tokens worth a workgroup of their own
  const int64_t rows = std::min(b.max_rows, b.rows);
  const int64_t cols = rows * (q_heads / c.heads);
  const int64_t base = (int64_t)b.sequences * c.heads;
  const int64_t narrow = (cols + 15) / 16, wide = (cols + kRowsColumns - 1) / kRowsColumns;
  AttendPlan p{};
  p.own_columns = base * narrow > std::max(kFewTiles, kTilesPerWide * base * wide);
  p.splits = 1;
  if (p.own_columns) {
    p.groups = (int32_t)wide;
    return p;
  }
  p.groups = (int32_t)narrow;
  const int64_t most = std::max<int64_t>(1, (b.max_length + kChunk - 1) / kChunk);
  const int64_t want = std::min(most, std::max<int64_t>(1, (kFill + base * narrow - 1) / std::max<int64_t>(base * narrow, 1)));
  const int64_t chunk = ((b.max_length + want - 1) / want + 255) / 256 * 256;
  p.chunk = (int32_t)std::max<int64_t>(chunk, 256);
  p.splits = (int32_t)std::max<int64_t>(1, (b.max_length + p.chunk - 1) / p.chunk);
  if (p.splits > 1) p.workspace = (size_t)b.sequences * c.heads * cols * p.splits * (c.head_dim + 4) * sizeof(float);
  return p;
}

}  // namespace awe

using namespace awe;

extern "C" {

awe_status awe_gemm_w4(int64_t M, int64_t N, int64_t K, const void* X, int64_t ldx, awe_dtype x_type,
                       const float* x_scales, const uint8_t* W, int64_t ldw, const void* w_scales, int64_t lds,
                       awe_dtype s_type, const uint8_t* zeros, int64_t ldz, int64_t group, void* Y, int64_t ldy,
                       awe_dtype y_type, hipStream_t stream) {
  const W4Launch g{M,      N,   K,      X,     ldx, x_type, x_scales, W,   ldw,
                   w_scales, lds, s_type, zeros, ldz, group,  Y,        ldy, y_type};
  return guarded([&] { return w4_impl(g, stream); });
}

awe_status awe_cache_store(const awe_cache* cache, const awe_batch* batch, const void* k, int64_t k_row,
                           int64_t k_head, const void* v, int64_t v_row, int64_t v_head, awe_dtype type,
                           int32_t* d_range_flag, hipStream_t stream) {
  const Rows rk{const_cast<void*>(k), k_row, k_head}, rv{const_cast<void*>(v), v_row, v_head};
  return guarded([&] { return cache_impl(cache, batch, rk, rv, type, d_range_flag, false, stream); });
}

awe_status awe_cache_load(const awe_cache* cache, const awe_batch* batch, void* k, int64_t k_row, int64_t k_head,
                          void* v, int64_t v_row, int64_t v_head, awe_dtype type, int32_t* d_range_flag,
                          hipStream_t stream) {
  const Rows rk{k, k_row, k_head}, rv{v, v_row, v_head};
  return guarded([&] { return cache_impl(cache, batch, rk, rv, type, d_range_flag, true, stream); });
}

awe_status awe_cache_attend_workspace_bytes(const awe_cache* cache, const awe_batch* batch, int32_t q_heads,
                                            size_t* bytes) {
  return guarded([&] {
    if (bytes == nullptr) return invalid("bytes is NULL");
    awe_status st = check_cache(cache);
    if (st == AWE_OK) st = check_batch(*cache, batch);
    if (st == AWE_OK) st = check_heads(*cache, *batch, q_heads);
    if (st == AWE_OK) *bytes = empty(*batch) ? 0 : plan_attend(*cache, *batch, q_heads).workspace;
    return st;
  });
}

awe_status awe_cache_attend(const awe_cache* cache, const awe_batch* batch, const void* q, int64_t q_row,
                            int64_t q_head, int32_t q_heads, awe_dtype type, float scale, int32_t causal, void* out,
                            int64_t out_row, int64_t out_head, void* workspace, size_t ws_bytes,
                            int32_t* d_range_flag, hipStream_t stream) {
  const Rows rq{const_cast<void*>(q), q_row, q_head}, ro{out, out_row, out_head};
  return guarded([&] {
    return attend_impl(cache, batch, rq, q_heads, type, scale, causal != 0, ro, workspace, ws_bytes, d_range_flag,
                       stream);
  });
}

}  // extern "C"
