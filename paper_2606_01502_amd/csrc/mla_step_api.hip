// C ABI of a serving step's way into the paged cache: tables and slots, rotary
// positions, the write of new tokens.  Argument checks and launches; declared in
// include/mla_sparse.h.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/mla_sparse.h"
#include "mla_host.h"
#include "mla_kernels.h"

using namespace mla::host;

namespace {

mla_status_t launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return MLA_OK;
  return fail(MLA_ERR_HIP, std::string(what) + " kernel launch: " + hipGetErrorString(e));
}

// Outputs overlap neither each other nor an input.
template <size_t N, size_t M>
mla_status_t check_apart(const mla_tensor_t* const (&outs)[N], const mla_tensor_t* const (&ins)[M]) {
  for (size_t i = 0; i < N; ++i) {
    for (size_t j = i + 1; j < N; ++j)
      if (overlaps(extent(*outs[i]), extent(*outs[j])))
        return fail(MLA_ERR_INVALID_ARGUMENT, "two outputs overlap");
    for (size_t j = 0; j < M; ++j)
      if (overlaps(extent(*outs[i]), extent(*ins[j])))
        return fail(MLA_ERR_INVALID_ARGUMENT, "an output overlaps an input");
  }
  return MLA_OK;
}

// Turns a position of every pair (see mla_rope_opts_t).
void rope_turns(const mla_rope_opts_t& o, double* turns) {
  constexpr double kTwoPi = 6.283185307179586476925;
  const double d = o.rot_dim;
  double lo = 0.0, hi = 0.0;
  if (o.scaling == MLA_ROPE_YARN) {
    auto pair_of = [&](double b) { return 0.5 * d * std::log((double)o.orig_len / (kTwoPi * b)) / std::log(o.base); };
    lo = std::max(std::floor(pair_of(o.beta_fast)), 0.0);
    hi = std::min(std::ceil(pair_of(o.beta_slow)), d - 1.0);
  }
  for (int i = 0; i < o.rot_dim / 2; ++i) {
    double w = std::pow(o.base, -2.0 * i / d);
    if (o.scaling == MLA_ROPE_LINEAR) w /= o.factor;
    if (o.scaling == MLA_ROPE_YARN) {
      const double r = std::min(std::max((i - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
      w *= (1.0 - r) + r / o.factor;
    }
    turns[i] = w / kTwoPi;
  }
}

mla_status_t check_rope_opts(const mla_rope_opts_t* o, int64_t D) {
  auto bad = [](const char* m) { return fail(MLA_ERR_INVALID_ARGUMENT, m); };
  if (!o) return bad("opts: null pointer");
  if (o->reserved) return bad("opts.reserved must be zero");
  if (o->rot_dim < 2 || o->rot_dim % 2 || o->rot_dim > 2 * mla::kRopeMaxPairs)
    return bad("opts.rot_dim must be even, 2 .. 256");
  if (o->rot_offset < 0 || o->rot_offset > D - o->rot_dim)
    return bad("opts: the rotated dims must lie within the head");
  if (o->pairing != 0 && o->pairing != 1) return bad("opts.pairing must be 0 or 1");
  if (o->inverse != 0 && o->inverse != 1) return bad("opts.inverse must be 0 or 1");
  if (o->scaling != MLA_ROPE_PLAIN && o->scaling != MLA_ROPE_LINEAR && o->scaling != MLA_ROPE_YARN)
    return bad("opts.scaling must be MLA_ROPE_PLAIN, MLA_ROPE_LINEAR or MLA_ROPE_YARN");
  if (!(o->base > 0.0) || !std::isfinite(o->base)) return bad("opts.base must be finite and > 0");
  if (!std::isfinite((float)o->mscale)) return bad("opts.mscale must be finite in fp32");
  if (o->scaling != MLA_ROPE_PLAIN && (!(o->factor > 0.0) || !std::isfinite(o->factor)))
    return bad("opts.factor must be finite and > 0");
  if (o->scaling == MLA_ROPE_YARN &&
      (!(o->base > 1.0) || o->orig_len < 1 || !(o->beta_slow > 0.0) || !(o->beta_fast >= o->beta_slow) ||
       !std::isfinite(o->beta_fast)))
    return bad("opts: YARN takes base > 1, orig_len > 0 and beta_fast >= beta_slow > 0");
  return MLA_OK;
}

// The checks and parameters that mla_cache_append and mla_rope_append share.
mla_status_t append_params(const mla_tensor_t* ckv, const mla_tensor_t* kpe, const mla_tensor_t* slots,
                           const mla_tensor_t* ckv_pool, const mla_tensor_t* kpe_pool, mla::AppendParams& p) {
  mla_status_t st;
  if ((st = check_tensor(ckv, "ckv", MLA_DTYPE_BF16, 2)) != MLA_OK) return st;
  if ((st = check_tensor(kpe, "kpe", MLA_DTYPE_BF16, 2)) != MLA_OK) return st;
  if ((st = check_tensor(slots, "slots", MLA_DTYPE_INT32, 1)) != MLA_OK) return st;
  if (ckv_pool && ckv_pool->dtype == MLA_DTYPE_FP8_E4M3FN)
    return fail(MLA_ERR_UNSUPPORTED, "ckv_pool: an fp8 pool has one scale a block, which new tokens may exceed");
  const bool mx4 = ckv_pool && ckv_pool->dtype == MLA_DTYPE_MXFP4;
  if ((st = check_tensor(ckv_pool, "ckv_pool", mx4 ? MLA_DTYPE_MXFP4 : MLA_DTYPE_BF16, 3)) != MLA_OK) return st;
  if ((st = check_tensor(kpe_pool, "kpe_pool", MLA_DTYPE_BF16, 3)) != MLA_OK) return st;
  const int64_t T = ckv->shape[0], P = ckv_pool->shape[0];
  if (ckv->shape[1] != MLA_DLAT || kpe->shape[0] != T || kpe->shape[1] != MLA_DPE)
    return fail(MLA_ERR_INVALID_ARGUMENT, "ckv / kpe: shapes must be [T, 512] / [T, 64]");
  if (!contiguous(*slots, {T})) return fail(MLA_ERR_INVALID_ARGUMENT, "slots: must be contiguous [T]");
  if (!contiguous(*ckv_pool, {P, MLA_BLOCK, mx4 ? MLA_MX4_ROW : MLA_DLAT}) ||
      !contiguous(*kpe_pool, {P, MLA_BLOCK, MLA_DPE}))
    return fail(MLA_ERR_INVALID_ARGUMENT,
                "pools must be contiguous [P, 64, 512] (MXFP4: [P, 64, 272]) and [P, 64, 64]");
  if (!rows_aligned(*ckv, 2) || !rows_aligned(*kpe, 2))
    return fail(MLA_ERR_INVALID_ARGUMENT, "ckv / kpe rows must be 16-byte aligned");
  if (!aligned16(ckv_pool->data) || !aligned16(kpe_pool->data))
    return fail(MLA_ERR_INVALID_ARGUMENT, "pools must be 16-byte aligned");
  const mla_tensor_t* const outs[] = {ckv_pool, kpe_pool};
  const mla_tensor_t* const ins[] = {ckv, kpe, slots};
  if ((st = check_apart(outs, ins)) != MLA_OK) return st;
  if (T > INT32_MAX || P > (INT32_MAX >> 6)) return fail(MLA_ERR_UNSUPPORTED, "sizes beyond the index range");
  p.src_ckv = (const uint16_t*)ckv->data;
  p.src_kpe = (const uint16_t*)kpe->data;
  p.ckv_s0 = ckv->stride[0];
  p.kpe_s0 = kpe->stride[0];
  p.slots = (const int32_t*)slots->data;
  p.ckv = (uint8_t*)ckv_pool->data;
  p.kpe = (uint8_t*)kpe_pool->data;
  p.T = T;
  p.n_slots = P * MLA_BLOCK;
  p.mx4 = mx4;
  // one token a wave until that fills the chip, then four, whose loads overlap: 2048
  // tokens into a 4-bit cache 3.2 us with one, 3.4 with four, 8192 4.6 and 4.1, 30,001
  // 11.4 and 9.3 (bf16 3.3 and 3.3, 5.1 and 4.0, 13.2 and 11.1)
  p.wave_toks = T <= 4096 ? 1 : 4;
  return MLA_OK;
}

// What a position of 2^31 leaves of a turn: a double holds 2^31 turns to 2^-22 of one,
// more of them to less, 2^51 (a pair of 2^20 turns) to half a turn.
mla_status_t check_turns(const double* turns, int pairs) {
  for (int i = 0; i < pairs; ++i)
    if (!(turns[i] <= 1.0))
      return fail(MLA_ERR_INVALID_ARGUMENT,
                  "opts: a pair turns more than once a position, where far positions lose their angle (at 2^20 turns "
                  "a position of 2^31 all of it)");
  return MLA_OK;
}

}  // namespace

extern "C" {

mla_status_t mla_batch_slots(const mla_tensor_t* cached_lens, const mla_tensor_t* new_lens,
                             const mla_tensor_t* free_blocks, const mla_tensor_t* block_table,
                             const mla_tensor_t* slots, const mla_tensor_t* positions,
                             const mla_tensor_t* seq_lens, const mla_tensor_t* starts,
                             const mla_tensor_t* info, void* stream) {
  try {
    g_last_error.clear();
    const mla_tensor_t* const lists[] = {cached_lens, new_lens, free_blocks, slots, positions, seq_lens, starts, info};
    static const char* const names[] = {"cached_lens", "new_lens", "free_blocks", "slots",
                                        "positions",   "seq_lens", "starts",      "info"};
    mla_status_t st;
    for (int k = 0; k < 8; ++k) {
      if ((st = check_tensor(lists[k], names[k], MLA_DTYPE_INT32, 1)) != MLA_OK) return st;
      if (!contiguous(*lists[k], {lists[k]->shape[0]}))
        return fail(MLA_ERR_INVALID_ARGUMENT, std::string(names[k]) + ": must be contiguous");
    }
    if ((st = check_tensor(block_table, "block_table", MLA_DTYPE_INT32, 2)) != MLA_OK) return st;
    const int64_t B = cached_lens->shape[0], NB = block_table->shape[1], T = slots->shape[0];
    if (new_lens->shape[0] != B || block_table->shape[0] != B || seq_lens->shape[0] != B || starts->shape[0] != B + 1)
      return fail(MLA_ERR_INVALID_ARGUMENT,
                  "new_lens and seq_lens must be [B], block_table [B, NB], starts [B + 1], with the B of cached_lens");
    if (positions->shape[0] != T) return fail(MLA_ERR_INVALID_ARGUMENT, "positions: shape must be [T], as slots");
    if (info->shape[0] != 4) return fail(MLA_ERR_INVALID_ARGUMENT, "info: shape must be [4]");
    if (!rows_apart(*block_table)) return fail(MLA_ERR_INVALID_ARGUMENT, "block_table: rows overlap");
    if (B > mla::kMaxSlotRequests)
      return fail(MLA_ERR_UNSUPPORTED, "more than " + std::to_string(mla::kMaxSlotRequests) + " requests");
    if (NB > INT32_MAX || T > INT32_MAX || free_blocks->shape[0] > INT32_MAX)
      return fail(MLA_ERR_UNSUPPORTED, "sizes beyond the int32 index range");
    const mla_tensor_t* const outs[] = {block_table, slots, positions, seq_lens, starts, info};
    const mla_tensor_t* const ins[] = {cached_lens, new_lens, free_blocks};
    if ((st = check_apart(outs, ins)) != MLA_OK) return st;
    mla::SlotsParams p{};
    p.cached = (const int32_t*)cached_lens->data;
    p.fresh = (const int32_t*)new_lens->data;
    p.free_blocks = (const int32_t*)free_blocks->data;
    p.table = (int32_t*)block_table->data;
    p.table_s0 = block_table->stride[0];
    p.slots = (int32_t*)slots->data;
    p.positions = (int32_t*)positions->data;
    p.seq_lens = (int32_t*)seq_lens->data;
    p.starts = (int32_t*)starts->data;
    p.info = (int32_t*)info->data;
    p.F = free_blocks->shape[0];
    p.T = T;
    p.B = (int32_t)B;
    p.NB = (int32_t)NB;
    return launched(mla::launch_slots(p, reinterpret_cast<hipStream_t>(stream)), "slots");
  } catch (...) {
    return fail(MLA_ERR_HIP, "internal error");
  }
}

mla_status_t mla_rope(const mla_tensor_t* x, const mla_tensor_t* positions, const mla_tensor_t* out,
                      const mla_rope_opts_t* opts, void* stream) {
  try {
    g_last_error.clear();
    mla_status_t st;
    const bool fp32 = x && x->dtype == MLA_DTYPE_FP32;
    const int32_t dt = fp32 ? MLA_DTYPE_FP32 : MLA_DTYPE_BF16;
    if ((st = check_tensor(x, "x", dt, 3)) != MLA_OK) return st;
    if ((st = check_tensor(positions, "positions", MLA_DTYPE_INT32, 1)) != MLA_OK) return st;
    if ((st = check_tensor(out, "out", dt, 3)) != MLA_OK) return st;
    const int64_t T = x->shape[0], H = x->shape[1], D = x->shape[2];
    if (!contiguous(*positions, {T})) return fail(MLA_ERR_INVALID_ARGUMENT, "positions: must be contiguous [T]");
    if (out->shape[0] != T || out->shape[1] != H || out->shape[2] != D)
      return fail(MLA_ERR_INVALID_ARGUMENT, "out: shape must be that of x");
    if ((st = check_rope_opts(opts, D)) != MLA_OK) return st;
    if (!rows_apart(*out)) return fail(MLA_ERR_INVALID_ARGUMENT, "out: rows overlap");
    // the same view: turned in place, nothing to copy
    bool same = x->data == out->data;
    for (int d = 0; d < 2; ++d) same = same && (x->shape[d] == 1 || x->stride[d] == out->stride[d]);
    if (!same && overlaps(extent(*out), extent(*x))) return fail(MLA_ERR_INVALID_ARGUMENT, "out overlaps x");
    if (overlaps(extent(*out), extent(*positions)))
      return fail(MLA_ERR_INVALID_ARGUMENT, "out overlaps positions");
    if (H > (1 << 24) || D > (1 << 24) || T > INT32_MAX) return fail(MLA_ERR_UNSUPPORTED, "sizes beyond the index range");
    if (T * H == 0) return MLA_OK;

    mla::RopeParams p{};
    p.x = x->data;
    p.out = out->data;
    p.pos = (const int32_t*)positions->data;
    p.x_s0 = x->stride[0]; p.x_s1 = x->stride[1];
    p.out_s0 = out->stride[0]; p.out_s1 = out->stride[1];
    p.rows = T * H;
    p.H = (int32_t)H;
    p.at = opts->rot_offset;
    p.rot = opts->rot_dim;
    p.pairing = opts->pairing;
    p.fp32 = fp32;
    const int es = fp32 ? 4 : 2, E = 16 / es;
    const int half = p.rot / 2;
    p.vec = rows_aligned(*x, es) && rows_aligned(*out, es) && D % E == 0 && p.at % E == 0 &&
            (p.pairing == 0 ? p.rot : half) % E == 0;
    const int64_t n_rot = !p.vec ? half : p.pairing == 0 ? p.rot / E : half / E;
    const int64_t units = n_rot + (same ? 0 : (D - p.rot) / (p.vec ? E : 1));
    p.row_units = (int32_t)units;
    // about 2048 units a workgroup (eight a thread), down to 256 where that
    // leaves compute units without one: 4096 tokens of 128 x 192 dims take 65 us with
    // 2048 and 105 with 256 (inputs in the caches), 512 of 128 x 64 6.9 and 5.0, 64
    // of 8 x 64 6.9 and 3.6
    int64_t rows = std::max<int64_t>(2048 / units, 1);
    while (rows > 1 && rows * units > 256 && (p.rows + rows - 1) / rows < 512) rows = (rows + 1) / 2;
    // and no more tokens than 32 KiB of cosines and sines hold
    auto toks = [&](int64_t r) { return (H - 1 + r - 1) / H + 1; };
    while (rows > 1 && toks(rows) * p.rot * 4 > 32768) rows = (rows + 1) / 2;
    if ((p.rows + rows - 1) / rows > (1ll << 23)) return fail(MLA_ERR_UNSUPPORTED, "too many rows");
    p.wg_rows = (int32_t)rows;
    p.wg_toks = (int32_t)toks(rows);
    p.by_H = mla::make_div(H);
    p.by_units = mla::make_div(units);
    p.mscale = (float)opts->mscale;
    p.sin_scale = opts->inverse ? -p.mscale : p.mscale;
    rope_turns(*opts, p.turns);
    if ((st = check_turns(p.turns, half)) != MLA_OK) return st;
    return launched(mla::launch_rope(p, reinterpret_cast<hipStream_t>(stream)), "rope");
  } catch (...) {
    return fail(MLA_ERR_HIP, "internal error");
  }
}

mla_status_t mla_cache_append(const mla_tensor_t* ckv, const mla_tensor_t* kpe,
                              const mla_tensor_t* slots, const mla_tensor_t* ckv_pool,
                              const mla_tensor_t* kpe_pool, void* stream) {
  try {
    g_last_error.clear();
    mla::AppendParams p{};
    const mla_status_t st = append_params(ckv, kpe, slots, ckv_pool, kpe_pool, p);
    if (st != MLA_OK) return st;
    return launched(mla::launch_append(p, reinterpret_cast<hipStream_t>(stream)), "append");
  } catch (...) {
    return fail(MLA_ERR_HIP, "internal error");
  }
}

mla_status_t mla_rope_append(const mla_tensor_t* ckv, const mla_tensor_t* kpe, const mla_tensor_t* positions,
                             const mla_tensor_t* slots, const mla_tensor_t* ckv_pool, const mla_tensor_t* kpe_pool,
                             const mla_rope_opts_t* opts, void* stream) {
  try {
    g_last_error.clear();
    mla::RopeAppendParams p{};
    mla_status_t st = append_params(ckv, kpe, slots, ckv_pool, kpe_pool, p.a);
    if (st != MLA_OK) return st;
    if ((st = check_tensor(positions, "positions", MLA_DTYPE_INT32, 1)) != MLA_OK) return st;
    if (!contiguous(*positions, {p.a.T})) return fail(MLA_ERR_INVALID_ARGUMENT, "positions: must be contiguous [T]");
    if ((st = check_rope_opts(opts, MLA_DPE)) != MLA_OK) return st;
    const mla_tensor_t* const outs[] = {ckv_pool, kpe_pool};
    const mla_tensor_t* const ins[] = {positions};
    if ((st = check_apart(outs, ins)) != MLA_OK) return st;
    p.pos = (const int32_t*)positions->data;
    p.at = opts->rot_offset;
    p.rot = opts->rot_dim;
    p.pairing = opts->pairing;
    p.mscale = (float)opts->mscale;
    p.sin_scale = opts->inverse ? -p.mscale : p.mscale;
    rope_turns(*opts, p.turns);
    if ((st = check_turns(p.turns, p.rot / 2)) != MLA_OK) return st;
    return launched(mla::launch_rope_append(p, reinterpret_cast<hipStream_t>(stream)), "append");
  } catch (...) {
    return fail(MLA_ERR_HIP, "internal error");
  }
}

}  // extern "C"
