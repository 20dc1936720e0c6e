// C ABI of the choice of blocks: mean keys, scores, the K best.  Argument checks,
// plans and launches; declared in include/mla_sparse.h.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/mla_sparse.h"
#include "mla_host.h"
#include "mla_select.h"

using namespace mla::host;

namespace {

mla_status_t bad(const std::string& m) { return fail(MLA_ERR_INVALID_ARGUMENT, m); }

mla_status_t launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return MLA_OK;
  return fail(MLA_ERR_HIP, std::string(what) + " kernel launch: " + hipGetErrorString(e));
}

mla_status_t means_call(const mla_tensor_t* ckv_pool, const mla_tensor_t* kpe_pool, const mla_tensor_t* slots,
                        const mla_tensor_t* means, void* stream) {
  mla_status_t st;
  if (!ckv_pool || !kpe_pool) return bad("ckv_pool/kpe_pool: null descriptor");
  if ((st = check_pool_types(ckv_pool, kpe_pool)) != MLA_OK) return st;
  if ((st = check_tensor(slots, "slots", MLA_DTYPE_INT32, 1)) != MLA_OK) return st;
  if ((st = check_tensor(means, "means", MLA_DTYPE_BF16, 2)) != MLA_OK) return st;
  const int64_t P = ckv_pool->shape[0], T = slots->shape[0];
  if ((st = check_pool_shapes(*ckv_pool, *kpe_pool)) != MLA_OK) return st;
  if ((st = check_pool_layout(*ckv_pool, *kpe_pool)) != MLA_OK) return st;
  if (!contiguous(*slots, {T})) return bad("slots: must be contiguous [T]");
  if (!contiguous(*means, {P, MLA_DLAT + MLA_DPE})) return bad("means: must be contiguous [P, 576] with the P of ckv_pool");
  if (!aligned16(means->data)) return bad("means must be 16-byte aligned");
  if (T > INT32_MAX || P > (INT32_MAX >> 6)) return fail(MLA_ERR_UNSUPPORTED, "sizes beyond the index range");
  const bool fp8 = ckv_pool->dtype == MLA_DTYPE_FP8_E4M3FN;
  auto scales = [&](const float* sc) -> Extent {
    if (!fp8 || P == 0) return {0, 0};
    return {(uintptr_t)sc, (uintptr_t)(sc + P)};
  };
  const Extent ins[5] = {extent(*ckv_pool), extent(*kpe_pool), extent(*slots), scales(ckv_pool->block_scale),
                         scales(kpe_pool->block_scale)};
  for (const Extent& i : ins)
    if (overlaps(extent(*means), i)) return bad("an output overlaps an input");
  if (T == 0 || P == 0) return MLA_OK;
  mla::MeansParams p{};
  p.ckv = (const uint8_t*)ckv_pool->data;
  p.kpe = (const uint8_t*)kpe_pool->data;
  p.ckv_scale = ckv_pool->block_scale;
  p.kpe_scale = kpe_pool->block_scale;
  p.slots = (const int32_t*)slots->data;
  p.means = (uint16_t*)means->data;
  p.T = T;
  p.n_slots = P * MLA_BLOCK;
  const int kv = fp8 ? mla::kKvFp8Shared : ckv_pool->dtype == MLA_DTYPE_MXFP4 ? mla::kKvMx4 : mla::kKvBf16;
  return launched(mla::launch_means(p, kv, reinterpret_cast<hipStream_t>(stream)), "means");
}

mla_status_t scores_call(const mla_tensor_t* q_lat, const mla_tensor_t* q_pe, const mla_tensor_t* means,
                         const mla_tensor_t* block_table, const mla_tensor_t* seq_lens, const mla_tensor_t* q_lens,
                         float scale, const mla_tensor_t* scores, const mla_scores_opts_t* opts, void* stream) {
  mla_status_t st;
  if ((st = check_tensor(q_lat, "q_lat", MLA_DTYPE_BF16, 4)) != MLA_OK) return st;
  if ((st = check_tensor(q_pe, "q_pe", MLA_DTYPE_BF16, 4)) != MLA_OK) return st;
  if ((st = check_tensor(means, "means", MLA_DTYPE_BF16, 2)) != MLA_OK) return st;
  if ((st = check_tensor(block_table, "block_table", MLA_DTYPE_INT32, 2)) != MLA_OK) return st;
  if ((st = check_tensor(seq_lens, "seq_lens", MLA_DTYPE_INT32, 1)) != MLA_OK) return st;
  if (q_lens && (st = check_tensor(q_lens, "q_lens", MLA_DTYPE_INT32, 1)) != MLA_OK) return st;
  if ((st = check_tensor(scores, "scores", MLA_DTYPE_FP32, 3)) != MLA_OK) return st;
  if (!opts) return bad("opts: null pointer");
  for (int i = 0; i < 5; ++i)
    if (opts->reserved[i]) return bad("opts.reserved must be zero");
  if (opts->window < 0) return bad("opts.window must be >= 0");
  if (opts->n_sink < 0) return bad("opts.n_sink must be >= 0");
  if (opts->n_splits < 0) return bad("opts.n_splits must be >= 0");
  const int64_t B = block_table->shape[0], NB = block_table->shape[1], P = means->shape[0];
  const int64_t Mq = q_lat->shape[1], H = q_lat->shape[2];
  if (!shape_is(q_lat, {B, Mq, H, MLA_DLAT})) return bad("q_lat: shape must be [B, Mq, H, 512] with the B of block_table");
  if (!shape_is(q_pe, {B, Mq, H, MLA_DPE})) return bad("q_pe: shape must be [B, Mq, H, 64]");
  if (!contiguous(*means, {P, MLA_DLAT + MLA_DPE})) return bad("means: must be contiguous [P, 576]");
  if (!aligned16(means->data)) return bad("means must be 16-byte aligned");
  if (!contiguous(*seq_lens, {B})) return bad("seq_lens: must be contiguous [B]");
  if (q_lens && !contiguous(*q_lens, {B})) return bad("q_lens: must be contiguous [B]");
  if (!shape_is(scores, {B, Mq, NB})) return bad("scores: shape must be [B, Mq, NB]");
  if (!rows_aligned(*q_lat, 2) || !rows_aligned(*q_pe, 2)) return bad("q_lat/q_pe rows must be 16-byte aligned");
  if (!rows_apart(*scores)) return bad("scores: rows overlap");
  if (!(std::fabs(scale) <= 18446744073709551616.0f)) return bad("scale must be finite with |scale| <= 2^64");
  if (B > INT32_MAX || Mq * H > (1 << 24) || NB > (INT32_MAX >> 6) || P > INT32_MAX)
    return fail(MLA_ERR_UNSUPPORTED, "sizes beyond the int32 index range");
  const Extent ins[6] = {extent(*q_lat), extent(*q_pe), extent(*means), extent(*block_table), extent(*seq_lens),
                         q_lens ? extent(*q_lens) : Extent{0, 0}};
  for (const Extent& i : ins)
    if (overlaps(extent(*scores), i)) return bad("an output overlaps an input");
  if (B == 0 || Mq == 0 || NB == 0) return MLA_OK;
  if (H == 0) return bad("q_lat: no heads");

  mla::ScoresParams p{};
  p.q_lat = (const uint16_t*)q_lat->data;
  p.q_pe = (const uint16_t*)q_pe->data;
  p.ql_s0 = q_lat->stride[0]; p.ql_s1 = q_lat->stride[1]; p.ql_s2 = q_lat->stride[2];
  p.qp_s0 = q_pe->stride[0]; p.qp_s1 = q_pe->stride[1]; p.qp_s2 = q_pe->stride[2];
  p.means = (const uint8_t*)means->data;
  p.table = (const int32_t*)block_table->data;
  p.table_s0 = block_table->stride[0];
  p.P = P;
  p.lens = (const int32_t*)seq_lens->data;
  p.q_lens = q_lens ? (const int32_t*)q_lens->data : nullptr;
  p.out = (float*)scores->data;
  p.out_s0 = scores->stride[0]; p.out_s1 = scores->stride[1];
  p.Mq = (int32_t)Mq;
  p.H = (int32_t)H;
  p.NB = (int32_t)NB;
  p.window = P > 0 ? opts->window : INT32_MAX;  // (no block to choose)
  p.first_block = (int32_t)(((int64_t)opts->n_sink + MLA_BLOCK - 1) / MLA_BLOCK);
  p.scale_log2 = (float)((double)scale * 1.4426950408889634074);
  // The shape by the chunks of a request's rows: the smallest that holds them reads its
  // keys for as few rows.  64 requests over 1024 blocks, in workgroups of 32, 64 and 128
  // rows: 2 chunks 31.7, 33.4 and 36.7 us, 4 chunks of one row 56.0, 33.9 and 37.2, of
  // four rows 36.3, 34.0 and 37.4, 8 chunks 101, 60.6 and 37.8; one row of 16 heads over
  // 64 blocks 6.8, 8.1 and 9.8.
  const int64_t C = (H + 15) / 16;
  const int shape = Mq * C > 4 ? mla::kScores128 : Mq * C > 2 ? mla::kScores64 : mla::kScores32;
  const int64_t slots = mla::kScoreChunksOf[shape];
  const int64_t group_rows = C >= slots ? 1 : std::min<int64_t>(Mq, slots / C);
  const int64_t n_groups = (Mq + group_rows - 1) / group_rows;
  // one workgroup a compute unit, which it fills (64 x 128 rows over 1024 blocks: 69 us in
  // one split, 46 in two, 36 in four, 51 in six)
  const int64_t tiles = (NB + mla::kScoreCols - 1) / mla::kScoreCols, items = B * n_groups;
  int64_t S = opts->n_splits ? opts->n_splits : (device_cus() + items - 1) / items;
  S = std::max<int64_t>(1, std::min<int64_t>(S, tiles));
  // (one launch holds less than 2^32 threads)
  if (items > (1 << 22)) return fail(MLA_ERR_UNSUPPORTED, "grid too large");
  S = std::min<int64_t>(S, (1 << 22) / items);
  p.shape = shape;
  p.row_chunks = (int32_t)C;
  p.group_rows = (int32_t)group_rows;
  p.group_chunks = (int32_t)(group_rows * C);
  p.n_groups = (int32_t)n_groups;
  p.by_groups = mla::make_div(n_groups);
  p.by_chunks = mla::make_div(C);
  const hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
  std::unique_lock<std::mutex> lock;  // held until the second pass is queued
  if (S > 1) {
    void* ws = nullptr;
    st = get_workspace(hs, (size_t)items * p.group_chunks * 16 * S * 8, &ws, lock);
    if (st != MLA_OK && opts->n_splits) return st;
    if (st != MLA_OK) {  // one workgroup does both passes
      S = 1;
      g_last_error.clear();
    }
    p.stats = (float*)ws;
  }
  p.n_splits = (int32_t)S;
  p.by_splits = mla::make_div(S);
  return launched(mla::launch_scores(p, (int)B, hs), "scores");
}

mla_status_t topk_call(const mla_tensor_t* scores, const mla_tensor_t* ids, void* stream) {
  mla_status_t st;
  const int nd = scores && scores->ndim == 2 ? 2 : 3;
  if ((st = check_tensor(scores, "scores", MLA_DTYPE_FP32, nd)) != MLA_OK) return st;
  if ((st = check_tensor(ids, "ids", MLA_DTYPE_INT32, nd)) != MLA_OK) return st;
  for (int d = 0; d + 1 < nd; ++d)
    if (scores->shape[d] != ids->shape[d]) return bad("ids: shape must be [.., K] with the rows of scores");
  if (!rows_apart(*ids)) return bad("ids: rows overlap");
  if (overlaps(extent(*ids), extent(*scores))) return bad("an output overlaps an input");
  const int64_t B = scores->shape[0], Mq = nd == 3 ? scores->shape[1] : 1;
  const int64_t N = scores->shape[nd - 1], K = ids->shape[nd - 1];
  if (B > INT32_MAX || Mq > INT32_MAX || N > INT32_MAX - 4096 || K > INT32_MAX - 4096 || B * Mq > INT32_MAX / 4)
    return fail(MLA_ERR_UNSUPPORTED, "sizes beyond the int32 index range");
  if (B * Mq == 0 || K == 0) return MLA_OK;
  mla::TopkParams p{};
  p.x = (const float*)scores->data;
  p.ids = (int32_t*)ids->data;
  p.x_s0 = scores->stride[0]; p.x_s1 = nd == 3 ? scores->stride[1] : 0;
  p.ids_s0 = ids->stride[0]; p.ids_s1 = nd == 3 ? ids->stride[1] : 0;
  p.rows = B * Mq;
  p.N = (int32_t)N;
  p.K = (int32_t)K;
  p.Mq = (int32_t)Mq;
  p.by_Mq = mla::make_div(Mq);
  const hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
  // Long rows in pieces, each the best of its piece, until one workgroup holds them
  // well: 32 rows of 65,536 are 32 workgroups' work in one go, 256 in pieces.  Two
  // halves of the workspace take turns.
  std::unique_lock<std::mutex> lock;  // held until the last step is queued
  char* half[2] = {};
  int turn = 0;
  while (p.N > 2 * mla::kTopPiece) {
    const int64_t pieces = (p.N + mla::kTopPiece - 1) / mla::kTopPiece, best = std::min<int64_t>(p.K, mla::kTopPiece);
    const int64_t n = pieces * best, bytes = p.rows * n * 8;
    if (2 * n > p.N || pieces > 65535 || bytes > (64ll << 20)) break;
    if (!half[0]) {
      // (the first step's are the most)
      void* ws = nullptr;
      if (get_workspace(hs, 2 * (size_t)bytes, &ws, lock) != MLA_OK) {
        g_last_error.clear();  // (it cannot grow here: a row is one workgroup's)
        break;
      }
      half[0] = (char*)ws;
      half[1] = half[0] + bytes;
    }
    mla::TopkParams q = p;
    q.K = (int32_t)best;
    q.best = (float*)half[turn];
    q.ids = (int32_t*)(half[turn] + p.rows * n * 4);
    q.ids_s0 = n * p.Mq;
    q.ids_s1 = n;
    if ((st = launched(mla::launch_topk(q, (int)pieces, hs), "topk")) != MLA_OK) return st;
    p.x = q.best;
    p.x_s0 = q.ids_s0;
    p.x_s1 = q.ids_s1;
    p.places = q.ids;
    p.N = (int32_t)n;
    turn ^= 1;
  }
  return launched(mla::launch_topk(p, 1, hs), "topk");
}

}  // namespace

extern "C" {

mla_status_t mla_block_means(const mla_tensor_t* ckv_pool, const mla_tensor_t* kpe_pool, const mla_tensor_t* slots,
                             const mla_tensor_t* means, void* stream) {
  try {
    g_last_error.clear();
    return means_call(ckv_pool, kpe_pool, slots, means, stream);
  } catch (...) {
    return fail(MLA_ERR_HIP, "internal error");
  }
}

mla_status_t mla_block_scores(const mla_tensor_t* q_lat, const mla_tensor_t* q_pe, const mla_tensor_t* means,
                              const mla_tensor_t* block_table, const mla_tensor_t* seq_lens,
                              const mla_tensor_t* q_lens, float scale, const mla_tensor_t* scores,
                              const mla_scores_opts_t* opts, void* stream) {
  try {
    g_last_error.clear();
    return scores_call(q_lat, q_pe, means, block_table, seq_lens, q_lens, scale, scores, opts, stream);
  } catch (...) {
    return fail(MLA_ERR_HIP, "internal error");
  }
}

mla_status_t mla_select_topk(const mla_tensor_t* scores, const mla_tensor_t* ids, void* stream) {
  try {
    g_last_error.clear();
    return topk_call(scores, ids, stream);
  } catch (...) {
    return fail(MLA_ERR_HIP, "internal error");
  }
}

}  // extern "C"
