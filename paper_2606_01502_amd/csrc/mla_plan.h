// The plan of a partial call: row tile, splits and what they keep in the
// split-K workspace.  Host arithmetic only.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "mla_kernels.h"

namespace mla {

// What the plan is made from: jobs, query rows and heads of a job, logical
// blocks and slots of a selection, its kind, the caller's options (0: the
// library's choice) and the compute units of the device.
struct PlanArgs {
  int64_t R, Mq, H, NB, K;
  bool tokens, per_row, fp8;
  int32_t n_splits, row_tile;
  int64_t cus;
  bool mx4 = false;     // a 4-bit cache
  bool window = false;  // no selection: K is the blocks that a tile's rows may see
};

struct Plan {
  int row_groups;          // of 64 rows a tile: 1 or 2
  int64_t row_tiles;       // tiles of a job
  int64_t S, sps;          // splits of a tile's slots, slots of a split
  bool by_id;              // splits by logical block instead of slot range
  bool long_lists;         // 64-row tiles: lists too long for the eight-wave kernel
  double us;               // what the call should take
};

// Bytes of split rows that a plan stays within where any plan does: what the
// allocation-free entry's scratch array holds.
constexpr uint64_t kPlanScratch = 64ull << 20;

struct Planner {
  PlanArgs a;
  int64_t rows, Kb;        // of a job; slots in 64-token blocks
  int64_t tile_qrows = 1;  // per-row selections: query rows a tile spans (one mask bit each)
  int row_groups = 0;      // of every plan, or 0: either
  const char* refused = nullptr;
  Plan cover{};            // the fewest splits that give every compute unit a workgroup
  bool keep32 = false;     // split rows are held in fp32, whatever their number

  explicit Planner(const PlanArgs& args) : a(args), rows(a.Mq * a.H) {
    Kb = a.tokens ? (a.K + 63) / 64 : a.K;  // a token selection's slots fill K / 64 blocks
    // the row groups of the covering plan: the caller's; 1 where a job has no
    // more rows; 2 where splits are long (8 blocks and more).  Per-row selections
    // keep to them, for a tile of twice the rows shares more loads; elsewhere the
    // cheaper is taken
    int groups = 1;
    if (a.row_tile) {
      groups = a.row_tile / 64;
    } else if (rows > 64) {
      const int64_t units2 = a.R * row_tiles_of(2);
      const int64_t s2 = std::min<int64_t>((a.cus + units2 - 1) / units2, std::max<int64_t>(Kb / 2, 1));
      groups = Kb < 8 * s2 ? 1 : 2;
    }
    if (a.per_row) {
      if (groups == 2 && tile_query_rows(2) > kPerRowMaxRows) {
        if (a.row_tile == 128) {
          refused = "per-row selections: too many query rows per 128-row tile";
          return;
        }
        groups = 1;
      }
      tile_qrows = tile_query_rows(groups);
      if (tile_qrows > kPerRowMaxRows) refused = "per-row selections: too many query rows per tile";
      else if (a.NB * tile_qrows * 2 > kPerRowCounterBytes)
        refused = "per-row selections: NB x query rows per tile too large";
      if (refused) return;
    }
    row_groups = a.row_tile || rows <= 64 || a.per_row ? groups : 0;
    // at least two blocks a split: one block costs less than its split's fixed
    // part.  Two splits of at most two blocks save at most two blocks' time and
    // add the combine's launch: one split does better (4 blocks of one 16-row
    // job: 12.4 us in one split against 14.9 in two)
    const int64_t units = std::max<int64_t>(a.R * row_tiles_of(groups), 1);
    int64_t S = std::min<int64_t>((a.cus + units - 1) / units, std::max<int64_t>(most_blocks() / 2, 1));
    if (S == 2 && !by_id() && Kb <= 5) S = 1;
    cover = plan_of(groups, std::max<int64_t>(S, 1));
    // Sums that the covering plan holds in fp32 (in registers from the first
    // block to the last, or in a few split rows) are held so in any other.
    keep32 = a.n_splits == 0 && (cover.S == 1 || !ws_half(cover.S));
  }

  int64_t row_tiles_of(int rg) const { return (rows + 64 * rg - 1) / (64 * rg); }

  int64_t tile_query_rows(int rg) const {
    const int64_t rw = 64 * rg;
    int64_t most = 0;
    for (int64_t r0 = 0; r0 < rows; r0 += rw) {
      const int64_t last = std::min<int64_t>(r0 + rw, rows) - 1;
      most = std::max<int64_t>(most, last / a.H - r0 / a.H + 1);
    }
    return most;
  }

  // Split rows in the workspace, then their scales (fp16 rows only), then their
  // lse values and maxima.  fp16 rows halve the workspace round trip, which pays
  // from about a megabyte of split rows on; tiny workspaces keep fp32 rows,
  // whose epilogue is a little shorter, and so do plans of more splits than the
  // covering one where that holds fp32: 300 jobs of 16 rows x 64 blocks, one
  // split to cover the chip, take 256 us in that, 242 in three with fp32 rows
  // (240 with fp16 ones).
  uint64_t split_rows(int64_t S) const { return (uint64_t)a.R * S * rows; }
  bool ws_half(int64_t S) const { return !keep32 && split_rows(S) * kDLat * 4 >= kWsHalfMinBytes; }
  uint64_t ws_rows_bytes(int64_t S) const { return split_rows(S) * kDLat * (ws_half(S) ? 2 : 4); }
  // Windows whose requests may see unlike numbers of tokens: splits go by what each
  // sees, on the GPU (a window of less than half the table is mostly full).  16
  // requests of 128 bf16 rows with 1300 to 30,000 tokens 137 -> 95 us, 15 of 500
  // tokens and one of 32,768 140 -> 45.  Finding the shares takes 0.7 to 2 us, which
  // splits of few blocks do not gain: 4 requests of 16 rows with 1054 to 3916
  // tokens, two blocks a split, 16.2 -> 18.6.
  bool shares(int64_t S) const { return S > 1 && may_share() && a.K >= 8 * S; }
  bool may_share() const {
    return a.window && a.n_splits == 0 && a.R > 1 && a.R <= kShareRequests && a.NB <= (1 << 20) && 2 * a.K > a.NB;
  }
  uint64_t ws_size(int64_t S) const {
    return ws_rows_bytes(S) + 3 * split_rows(S) * 4 + (shares(S) ? 8 * kShareRequests : 0);
  }
  bool fits(const Plan& q) const { return q.S <= 1 || ws_size(q.S) <= kPlanScratch; }

  // entries one split's list holds (per-row selections with an fp8 cache: a
  // shorter one, see the kernel's LDS layout)
  int64_t list_cap() const { return a.window ? kWindowList / 2 : a.per_row && a.fp8 ? kPerRowListShort : kMaxSlotsPerSplit; }
  // per-row selections whose tile slots all fit one list split by logical
  // block: every split then scans all slots and the rows that chose a block
  // in different slots still share its load
  bool by_id() const { return a.per_row && tile_qrows > 1 && a.K * tile_qrows <= list_cap(); }
  // the most blocks a tile can visit
  int64_t most_blocks() const { return by_id() ? std::min<int64_t>(a.NB, a.K * tile_qrows) : Kb; }

  // the plan of about S splits with tiles of rg row groups, and its time
  Plan plan_of(int rg, int64_t S) const {
    Plan q{rg, row_tiles_of(rg), S, a.K, by_id(), false, 0.0};
    // a split's block list holds at most so many entries: its slots, or for
    // per-row selections its slots of every query row of the tile
    const int64_t cap = list_cap();
    if (a.tokens) {
      // whole virtual blocks per split, at most one list of tokens
      S = std::max<int64_t>(S, (a.K + kMaxSlotsPerSplit - 1) / kMaxSlotsPerSplit);
      q.sps = std::max<int64_t>(64, ((a.K + S - 1) / S + 63) / 64 * 64);
      q.sps = std::min<int64_t>(q.sps, kMaxSlotsPerSplit);
      q.S = std::max<int64_t>(1, (a.K + q.sps - 1) / q.sps);
    } else if (a.window) {
      // (split on the GPU, evenly: any number of splits goes)
      q.S = std::max<int64_t>(S, (a.K + cap - 1) / cap);
      q.sps = std::max<int64_t>(1, (a.K + q.S - 1) / q.S);
    } else if (!q.by_id) {
      S = std::max<int64_t>(S, (a.K * tile_qrows + cap - 1) / cap);
      q.sps = std::max<int64_t>(1, (a.K + S - 1) / S);
      if (a.per_row) q.sps = std::min<int64_t>(q.sps, std::max<int64_t>(1, cap / tile_qrows));
      q.S = std::max<int64_t>(1, (a.K + q.sps - 1) / q.sps);
    }
    q.long_lists = a.per_row && !a.fp8 && rg == 1 && q.sps * tile_qrows > kPerRowListShort;
    // What a call takes, microseconds.  A workgroup fills its CU, so that a
    // grid goes in waves of one a CU.  A wave takes as long as one of its work
    // items, a fixed part (its prologue, query rows and epilogue) and its blocks'
    // time, or as the bytes of all its blocks take from memory: a last wave of a
    // few workgroups is bound by the former, a full one often by the latter.
    // Splits add the combine, by the bytes of the rows it reads.  The rows' own
    // bytes are left out.  Fitted to 140000 timed plans of 28000 calls of 1..700
    // jobs of 8..256 rows x 1..1500 blocks or 16..6000 tokens (9 % rms in 128-row
    // tiles, 9 to 17 % in 64-row ones).
    const double blocks = a.window ? (double)((2 * a.K + q.S - 1) / q.S) / 2
                        : q.by_id ? (double)((most_blocks() + q.S - 1) / q.S)
                        : a.tokens ? (double)((q.sps + 63) / 64)
                        : a.per_row ? (double)std::min<int64_t>(std::max<int64_t>(a.NB, 1), q.sps * tile_qrows)
                        : (double)q.sps;
    struct Rate {
      double fixed, block, bytes;  // us, us, bytes a us
    };
    // by selection, cache and tile: half of a 64-row tile, one for all rows,
    // one of several, 128 rows
    static constexpr Rate kRate[2][2][4] = {
        {{{5.5, 1.62, 6.3e6}, {7.9, 1.83, 5.9e6}, {8.2, 1.85, 7.5e6}, {14.0, 3.27, 4.8e6}},
         {{6.6, 1.87, 5.5e6}, {9.4, 2.32, 5.5e6}, {9.4, 2.30, 5.5e6}, {14.1, 4.16, 5.5e6}}},
        {{{5.0, 1.99, 6.6e6}, {7.8, 2.19, 6.1e6}, {8.5, 2.17, 8.7e6}, {14.2, 3.78, 5.0e6}},
         {{5.7, 2.38, 5.5e6}, {8.4, 2.64, 5.5e6}, {9.2, 2.49, 5.5e6}, {14.5, 4.89, 5.5e6}}}};
    // 4-bit caches: 64-row tiles only, fitted to 256 work items of 2 .. 64 blocks, and
    // taken for token selections too, which were not fitted apart
    static constexpr Rate kRateMx4[3] = {{6.6, 2.1, 5.5e6}, {11.0, 2.45, 5.5e6}, {11.0, 2.3, 5.5e6}};
    const int kind = rg == 2 ? 3 : rows <= 32 ? 0 : rows <= 64 ? 1 : 2;
    const Rate& rate = a.mx4 && kind < 3 ? kRateMx4[kind] : kRate[a.tokens][a.fp8][kind];
    // (rows with selections of their own share blocks, nobody here knows which)
    const double token_bytes = a.mx4 ? kMx4Row + 2 * kDPe : (kDLat + kDPe) * (a.fp8 ? 1 : 2);
    // (a window's row tiles see much the same blocks, side by side on one XCD)
    const double item_bytes = a.per_row ? 0.0 : blocks * kBlock * token_bytes / (a.window && q.row_tiles > 1 ? 2 : 1);
    auto wave_us = [&](int64_t items) {
      return rate.fixed + std::max(blocks * rate.block, (double)items * item_bytes / rate.bytes);
    };
    const int64_t items = a.R * q.row_tiles * q.S, rest = items % a.cus;
    q.us = (double)(items / a.cus) * wave_us(a.cus) + (rest ? wave_us(rest) : 0.0);
    if (q.S > 1) q.us += 1.8 + 0.4e-6 * (double)ws_rows_bytes(q.S);
    // a row's splits are read one trip after another: 48 rows in 16, 32 and 64
    // splits 15.1, 20.0 and 26.5 us
    if (a.window && q.S > 8) q.us += 0.2 * (double)(q.S - 8);
    return q;
  }

  // Windows are short, and often few: the cheapest of a few split counts up to one
  // block a split, and of those that fill one, two or three waves.  One 16-row
  // request with a window of 512 tokens: 14.5 us in the covering three splits, 11.6
  // in nine; of 2000 tokens 15.1 in twelve, 20.9 in five.
  Plan choose_window() const {
    static constexpr int kCounts[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64};
    const int64_t most = std::max<int64_t>(a.K, 1);
    Plan plan = cover;
    // Long sequences of so many requests that the chip is full without splits: two at
    // least, so that there is something to share out.  128 requests of 128 4-bit rows:
    // 281 to 16,379 tokens 620 -> 457 us, 127 of 300 tokens and one of 16,384 614 -> 82,
    // all of 16,384 649 -> 687; from 128 blocks on, for all of 4096 take 169 -> 209.
    // The split rows' 64 MiB do not bind here: those of 512 tiles in two splits are up
    // to 256 MiB (held in fp32, as one split would have), and no window has to fit
    // the allocation-free entry's array.
    const bool two = may_share() && a.K >= 128 && a.R * row_tiles_of(2) <= 2 * a.cus;
    if (two && plan.S == 1) plan.us = INFINITY;
    for (int rg = 1; rg <= 2; ++rg) {
      if (row_groups && rg != row_groups) continue;
      const int64_t units = std::max<int64_t>(a.R * row_tiles_of(rg), 1);
      auto offer = [&](int64_t S) {
        if (two) S = std::max<int64_t>(S, 2);
        const Plan q = plan_of(rg, S);
        if (two) {
          if (q.us < plan.us) plan = q;
          return;
        }
        if (fits(plan) && !fits(q)) return;
        if ((fits(q) && !fits(plan)) || q.us < plan.us) plan = q;
      };
      for (int64_t S : kCounts)
        if (S <= most && S * units <= 3 * a.cus) offer(S);
      for (int waves = 1; waves <= 3; ++waves) offer(std::max<int64_t>(1, std::min<int64_t>(waves * a.cus / units, most)));
    }
    return plan;
  }

  Plan choose() const {
    Plan plan{};
    if (a.n_splits > 0) {
      for (int rg = 2; rg >= 1; --rg) {
        if (row_groups && rg != row_groups) continue;
        const Plan q = plan_of(rg, std::min<int64_t>(a.n_splits, std::max<int64_t>(by_id() ? a.NB : a.K, 1)));
        if (!plan.row_groups || q.us < plan.us) plan = q;
      }
      return plan;
    }
    // The covering plan, one split, or as many as one, two or three waves of
    // workgroups hold.  A grid just past a whole number of waves costs a wave
    // more: 20 jobs of 128 rows x 200 blocks take 122 us in 13 splits (260
    // workgroups) and 85 in 12, 40 x 600 blocks 622 and 420 (fp8 708 and 446), 24
    // of 2048 tokens 67 and 39.  Several waves of shorter splits where one wave
    // leaves CUs idle: 281 jobs of 8 rows x 86 fp8 blocks 327 us in one split,
    // 241 in three.  A plan has to promise 3 % over the covering one, about what
    // the prices are off between plans of one call: of the timed calls one in
    // 4000 then takes 2 % more than in the covering plan, and the mean is 9.3 %
    // less (9.5 with the best plan of each call; a fourth wave adds nothing).
    // A plan whose split rows fit the allocation-free entry's scratch (64 MiB)
    // goes before one whose rows do not, for every entry; where a list's limit
    // leaves none that fits, the cheapest is taken: 256 jobs of 128 rows x 2048
    // tokens, two splits at least, take 395 us in 64-row tiles and 211 in 128-row
    // ones, and their split rows are the same 65 MiB.
    // Per-row selections in ranges of slots keep the covering plan: a block that
    // rows chose in different slots is loaded once a range, so that other ranges
    // mean other loads, which only the ids tell (28 jobs of 10 x 16 rows with 144
    // blocks each: 268 us in four ranges, priced cheaper, 241 in the covering
    // five).
    plan = cover;
    if (a.window) return choose_window();
    if (a.per_row && tile_qrows > 1 && !by_id()) return plan;
    double best = 0.97 * cover.us;
    for (int rg = 1; rg <= 2; ++rg) {
      if (row_groups && rg != row_groups) continue;
      const int64_t units = std::max<int64_t>(a.R * row_tiles_of(rg), 1);
      const int64_t most = std::max<int64_t>(most_blocks() / 2, 1);
      int64_t last = 0;
      for (int waves = 0; waves <= 3; ++waves) {
        const int64_t S = std::max<int64_t>(1, std::min<int64_t>(waves * a.cus / units, most));
        if (S == last || (S == 2 && !by_id() && Kb <= 5)) continue;
        last = S;
        const Plan q = plan_of(rg, S);
        if (fits(plan) && !fits(q)) continue;
        if ((fits(q) && !fits(plan)) || q.us < best) {
          plan = q;
          best = q.us;
        }
      }
    }
    return plan;
  }
};

// The plan of attention behind shared prefixes: tiles of the groups' rows over the
// prefixes and of each request's rows over its own tokens, in one launch.
struct PrefixArgs {
  int64_t B, G, NBP, NB, rows;  // rows: of a request
  int64_t cus;
  int32_t n_splits, own_splits, row_tile;  // the caller's, or 0
  bool fp8, mx4;
};
struct PrefixPlan {
  int row_groups;                        // of 64 rows a tile: 1 or 2
  int64_t S, tiles, prefix_grid;         // splits of a prefix, tiles of all groups' rows, their workgroups
  int64_t own_S, own_tiles, own_items;   // splits and tiles of a request's own tokens
  int64_t tile_step, grid;
  bool ws_f16;
  uint64_t ws_bytes;
  double us;
};
inline PrefixPlan plan_prefix(const PrefixArgs& a) {
  PrefixPlan q{};
  auto up = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
  // Group g's rows begin with tile floor(first row / tile) + g, or where every request
  // fills whole tiles with that of its first row.
  auto shape = [&](int rg) {
    PrefixPlan c{};
    c.row_groups = rg;
    c.tile_step = a.rows % (64 * rg) ? 1 : 0;
    c.tiles = up(a.B * a.rows, 64 * rg) + c.tile_step * (a.G - 1);
    c.own_tiles = up(a.rows, 64 * rg);
    return c;
  };
  const int64_t cap = kWindowList / 2;
  const int64_t nbp = std::max<int64_t>(a.NBP, 1), nb = std::max<int64_t>(a.NB, 1);
  // Times of a work item's fixed part and of a block, as in Planner::plan_of, but the
  // 64-row tiles' with the chip full of long items: 64 requests of 128 rows behind 256
  // blocks take 319 us in two splits of them, 274 in four of 128-row ones.
  auto fixed = [&](int rg) { return rg == 2 ? 14.0 : a.mx4 ? 11.0 : a.fp8 ? 9.4 : 8.2; };
  auto block = [&](int rg) { return rg == 2 ? (a.fp8 ? 4.16 : 3.27) : a.fp8 || a.mx4 ? 2.4 : 2.15; };
  auto share = [&](int64_t n, int64_t S) { return 0.5 * (double)up(2 * n, S); };  // (splits are cut by half blocks)
  // What the launch takes: prefix items go out first, one to a compute unit at a time,
  // the requests' own where compute units come free.
  auto span = [&](int64_t n, double p, int64_t m, double o) {
    const int64_t rounds = n / a.cus, rest = n % a.cus, free = a.cus - rest;
    const double base = (double)rounds * p;
    if (rest == 0) return base + (double)up(m, a.cus) * o;
    const int64_t beside = free * (int64_t)(p / o);
    return m <= beside ? base + p : base + p + (double)up(m - beside, a.cus) * o;
  };
  auto offer = [&](int rg, int64_t S, int64_t T) {
    S = std::max<int64_t>({1, up(a.NBP, cap), a.n_splits ? std::min<int64_t>(a.n_splits, nbp) : std::min(S, nbp)});
    T = std::max<int64_t>({1, up(a.NB, cap), a.own_splits ? std::min<int64_t>(a.own_splits, nb) : std::min(T, nb)});
    const uint64_t rows = (uint64_t)(S + T) * a.B * a.rows;
    // (fp16 rows, scaled by the row's largest value, from a megabyte on: they halve the
    // round trip, and their half step, 2^-11, is an eighth of the bf16 weights'.  Against 64 bits the fp32 outputs of 4 x 16 rows behind 2000 tokens are 1.02e-3
    // off with fp16 rows, 1.10e-3 in one split of each kind with fp32 ones; of 64 x 128
    // behind 16,384 5.1e-4 with fp16 rows)
    const bool half = rows * kDLat * 4 >= kWsHalfMinBytes;
    PrefixPlan c = shape(rg);
    // (a row's splits come in one trip up to 16 of them: 4 requests of 16 rows behind 32
    // blocks take 17.1 us in 12 + 2 splits, 18.7 in 16 + 4)
    c.us = span(c.tiles * S, fixed(rg) + block(rg) * share(nbp, S), a.B * c.own_tiles * T,
                fixed(rg) + block(rg) * share(nb, T)) +
           0.4e-6 * (double)(rows * kDLat * (half ? 2 : 4)) + (S + T > 16 ? 1.5 + 0.2 * (double)(S + T - 16) : 0.0);
    if (q.S != 0 && c.us >= q.us) return;
    c.S = S;
    c.own_S = T;
    c.ws_f16 = half;
    c.ws_bytes = rows * (kDLat * (half ? 2 : 4) + 3 * 4);
    q = c;
  };
  static constexpr int kCounts[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 14, 16, 20, 24, 32, 48, 64};
  for (int rg = 1; rg <= (a.mx4 ? 1 : 2); ++rg) {
    // Tiles of 128 rows where a request has as many: its own tokens' tiles are of the same
    // size, half empty below that.  In 64-row tiles and in 128-row ones, behind 256 blocks:
    // 64 x 128 rows 323 and 284 us, 64 x 64 175 and 164, 200 x 16 147 and 158, 60 x 16 56
    // and 73 (fp8 355 and 324, 192 and 186, 163 and 180, 66 and 82); 40 x 96 fp8 rows in
    // five groups behind 200 blocks 160 and 162.
    if (a.row_tile ? a.row_tile != 64 * rg : rg == 2 && a.rows < 128) continue;
    const int64_t tiles = shape(rg).tiles, own = a.B * shape(rg).own_tiles;
    for (int64_t T = 1; T == 1 || (T <= a.NB && own * T <= 2 * a.cus); T *= 2) {
      for (int64_t S : kCounts)
        if (S == 1 || (S <= nbp && tiles * S <= 3 * a.cus)) offer(rg, S, T);
      for (int waves = 1; waves <= 4; ++waves) offer(rg, std::max<int64_t>(1, waves * a.cus / tiles), T);
    }
  }
  q.prefix_grid = up(q.tiles * q.S, 8) * 8;
  q.own_items = a.B * q.own_tiles * q.own_S;
  q.grid = q.prefix_grid + q.own_items;
  return q;
}

}  // namespace mla
