// Internal interface between the C-ABI host code and the kernels of the choice of
// blocks (mla_select.hip).
#pragma once

#include "mla_kernels.h"

namespace mla {

// Mean keys of whole blocks.
struct MeansParams {
  const uint8_t* ckv;
  const uint8_t* kpe;
  const float* ckv_scale;  // [P] (fp8 only)
  const float* kpe_scale;
  const int32_t* slots;    // [T]; of those of n_slots that are a block's last row, that block's mean
  uint16_t* means;         // [P][576] bf16
  int64_t T, n_slots;
  int32_t sharers;         // workgroups to kMeanWindow slots (set by the launch)
  Div by_sharers;
};
constexpr int kMeanWindow = 1024;
hipError_t launch_means(const MeansParams& p, int kv, hipStream_t s);

// Scores of blocks by their mean keys: one workgroup a request, group of query rows
// and split of its blocks.  Its shape by the rows it holds (16-row chunks of heads): the
// smallest that a request's rows fill.
enum { kScores128, kScores64, kScores32 };
constexpr int kScoreChunksOf[] = {8, 4, 2};
constexpr int kScoreThreads = 512;
constexpr int kScoreCols = 64;
struct ScoresParams {
  const uint16_t* q_lat;
  const uint16_t* q_pe;
  int64_t ql_s0, ql_s1, ql_s2, qp_s0, qp_s1, qp_s2;  // element strides over (request, Mq, H)
  const uint8_t* means;    // [P][576] bf16
  const int32_t* table;
  int64_t table_s0, P;
  const int32_t* lens;
  const int32_t* q_lens;   // null: Mq
  float* out;              // [B][Mq][NB]
  int64_t out_s0, out_s1;
  float* stats;            // two floats of [B][groups][chunks of a group][16 rows][splits], the largest logit and sum
  int32_t Mq, H, NB;
  int32_t window, first_block;
  int32_t row_chunks;      // chunks of a query row
  int32_t group_rows, group_chunks, n_groups;  // query rows and chunks of a group
  int32_t n_splits, shape;  // shape: kScores*
  float scale_log2;        // softmax scale * log2(e)
  Div by_splits, by_groups, by_chunks;
};
hipError_t launch_scores(const ScoresParams& p, int B, hipStream_t s);

// The K best of each row of N scores.
struct TopkParams {
  const float* x;
  int32_t* ids;
  int64_t x_s0, x_s1, ids_s0, ids_s1;  // element strides over (request, Mq)
  int64_t rows;
  int64_t first_row;      // of a launch (set by it)
  int32_t N, K;
  Div by_Mq;
  int32_t Mq;
  const int32_t* places;  // [rows][N] of values that are the best of pieces; null: their own
  float* best;            // [rows][pieces][K] beside the ids; null: not asked for
};
constexpr int kTopPiece = 8192;   // of a row that goes in pieces
constexpr int kTopMost = 65536;   // values of a row that one workgroup holds
// (pieces > 1: ids and best of each piece of kTopPiece, rows apart by ids_s0 and ids_s1)
hipError_t launch_topk(const TopkParams& p, int pieces, hipStream_t s);

}  // namespace mla
