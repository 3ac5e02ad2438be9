// Which form of a kernel a call takes, by its sizes: of the int8 projection (linear_i8.cu), the norms (norm.cu) and the
// rotary positions (rope.cu).  Host code without CUDA, so that it can be asked without a device.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "ispa.h"

namespace ispa {

constexpr int TEAM_WARPS = 8;   // of a team of warps that takes a row or a token, at most

// ------------------------------------------------------------ int8 projection
constexpr int IM = 128;                 // rows (tokens) of a CTA's part of a tile
constexpr int IK = 64;                  // codes of a block: 64 bytes raw, 128 bytes (one swizzle row) as fp16

struct LinearForm {
  int tokens, channels;   // dp4a: of a warp; tokens 0: tensor cores
  int bn;                 // columns of a tile
  bool pair;              // of CTAs
  int split;              // CTAs that share a tile's contraction
};

// The tensor-core form with the shortest estimated run, and the estimate in ns.  Fitted to measured runs (weights in
// L2) of 9 to 9400 tokens, 64 to 5120 codes and 256 to 8960 channels: waves of tiles x (blocks x time of one + a tile's
// fixed part) + launch, fill and the last tile's way out.  A block of a pair of 192 columns costs little more than one
// of 128, so those win where tiles fill whole waves (4680 x 1536 -> 1536: 19.7 against 22.4 us with pairs of 128 and
// 23.6 with single CTAs); single CTAs win where there are few tiles (1000 x 1536 -> 1536: 10.0 against 10.9 and 10.3).
inline LinearForm gemm_form(int64_t T, int32_t D, int32_t Dout, int sms, int64_t* ns) {
  struct Shape {
    int bn, ctas, block_ns, tile_ns, start_ns;
  };
  constexpr Shape kShapes[3] = {{192, 2, 250, 500, 4600}, {128, 2, 230, 300, 3750}, {128, 1, 265, 300, 3100}};
  const int64_t n_kb = (D + IK - 1) / IK;
  LinearForm best{0, 0, 128, false, 1};
  *ns = INT64_MAX;
  for (const Shape& f : kShapes) {
    if (sms < f.ctas) continue;
    const int64_t rows = IM * f.ctas, units = sms / f.ctas;
    const int64_t tiles = (T + rows - 1) / rows * ((Dout + f.bn - 1) / f.bn);
    const int64_t cost = (tiles + units - 1) / units * (n_kb * f.block_ns + f.tile_ns) + f.start_ns;
    if (cost < *ns) {
      *ns = cost;
      best = {0, 0, f.bn, f.ctas == 2, 1};
    }
  }
  // Few tiles and a long contraction: clusters share a tile's blocks and add up through distributed shared memory.
  // 61 x 5120 -> 640: 24.2 us in pairs of 192, 18.2 / 11.9 / 9.2 with 2 / 4 / 8 CTAs a tile.  As many clusters as run
  // at once: of four or eight CTAs that is taken as four fifths of the chip.
  for (const int c : {2, 4, 8}) {
    const int64_t tiles = (T + IM - 1) / IM * ((Dout + 127) / 128);
    if (n_kb < c || tiles * c * (c > 2 ? 5 : 4) > 4 * static_cast<int64_t>(sms)) break;
    const int64_t cost = 5100 + (n_kb + c - 1) / c * 265 + 250 * c + 40 * std::min<int64_t>(T, IM) / c;
    if (cost < *ns) {
      *ns = cost;
      best = {0, 0, 128, false, c};
    }
  }
  return best;
}

inline LinearForm linear_i8_form(int64_t T, int32_t D, int32_t Dout, int sms) {
  int64_t gemm_ns = 0;
  LinearForm f = gemm_form(T, D, Dout, sms, &gemm_ns);
  // Few tokens: the warps' loads and dp4a against the tensor cores' long start.  16 x 1536 -> 1536: 4.5 against 7.7 us;
  // 16 x 5120 -> 5120: 20.8 against 16.4.
  if (T <= 32 && 2000 + 55 * (T * D * Dout / 1000000) + D / 2 < gemm_ns) {
    f.tokens = T == 1 ? 1 : T == 2 ? 2 : T <= 4 ? 4 : 8;
    // Two channels a warp share the tokens' loads, one makes twice the warps: 2 x 1536 -> 1536 2.1 us with one, 2.6
    // with two; 2 x 5120 -> 5120 7.7 with one, 5.4 with two; 16 x 1536 -> 1536, two groups of tokens, 5.5 and 4.5.
    f.channels = Dout <= 16 * sms && T <= 8 ? 1 : 2;
  }
  return f;
}

// ------------------------------------------------------------ norms
constexpr int S_DIM = 8192;             // four factors a column of such rows: 128 KB
static_assert(S_DIM <= 1024 * TEAM_WARPS, "four vectors of eight values a thread");
constexpr int S_SMEM = 224 * 1024;
// Threads a block: what the registers a thread needs leave room for (64, 80 or 96).
constexpr int s_threads(int v, bool res) { return !res ? 1024 : v == 4 ? 640 : 768; }

struct NormForm {
  bool stream;        // teams of warps over runs of rows; else a block a row
  int vectors;        // of eight values, of a thread
  int warps, teams;   // of a team, of a block (a block a row: its warps, 1)
  bool two;           // blocks an SM
  int64_t rows;       // of a block
  int smem;
};

inline NormForm norm_form(int64_t rows, int dim, bool x_fp32, bool residual, bool post_bias, bool modulated,
                          int64_t rows_per_group, int sms) {
  const int nv = dim / 8;
  // Many rows, by what a team keeps in shared memory: more than two an SM, of short rows one.  4680 x 1536 bf16 9.4 us
  // against 12.6 with a block a row, 620 x 5120 (both norms) 8.4 against 13.1, 310 x 4096 3.7 against 5.4, 310 x 1536
  // 2.9 each, 230 x 2560 3.3 against 3.0; 160 x 512 2.2 against 2.5.  With vectors of a few rows each (2: 14.5 us a
  // block a row) there is nothing for a team to keep.
  // Three vectors a thread in more warps where shared memory has room for their teams (5120 bf16, both norms 39.7 ->
  // 37.2 us, layer norms 48.9 -> 44.7; 5120 fp32, where it has not, 51.5 -> 55.7), else four.
  const int few = (nv + 127) / 128, team_warps = x_fp32 ? few : std::max(few, std::min(TEAM_WARPS, (nv + 95) / 96));
  const int v = (nv + 32 * team_warps - 1) / (32 * team_warps);
  const int fixed = 32 * (!residual ? 2 : post_bias ? 4 : 3) * nv;
  const int row_bytes = dim * ((x_fp32 ? 4 : 2) + (residual ? 2 : 0)), rest = 2 * 8 + 2 * TEAM_WARPS * 8;
  // registers, 15 named barriers, and what shared memory has room for
  int teams = std::min({s_threads(v, residual) / 32 / team_warps, team_warps > 1 ? 15 : 32,
                        (S_SMEM - fixed) / (2 * row_bytes + rest)});
  if (rows > (dim <= 512 ? 1 : 2) * sms && rows < INT32_MAX - 64 && dim <= S_DIM && teams >= 1 &&
      !(modulated && rows_per_group < 8)) {
    // Two blocks an SM where both fit and have rows enough: one starts, or waits for its factors, while the other works
    // (gate and norm of 1536 fp32: 4680 rows 17.4 us against 17.9 with one, 1560 8.5 against 7.7).
    const bool two = teams >= 8 && rows > 16 * sms &&
                     2 * (fixed + teams / 2 * (2 * row_bytes + rest) + 1024) <= S_SMEM;
    const int64_t per = two ? (rows + 2 * sms - 1) / (2 * sms) : (rows + sms - 1) / sms;
    teams = static_cast<int>(std::min<int64_t>(two ? teams / 2 : teams, per));
    return {true, v, team_warps, teams, two, per, fixed + teams * (2 * row_bytes + rest)};
  }
  const int warps = (nv + 31) / 32, w = warps <= 16 ? 1 : warps <= 32 ? 2 : warps <= 64 ? 4 : 8;
  return {false, w, (warps + w - 1) / w, 1, false, 1, 0};
}

// ------------------------------------------------------------ rotary positions
constexpr int R_SMEM = 224 * 1024;

struct RopeForm {
  bool stream;        // a team of warps a token; else a block for a token's queries or keys
  bool full;          // every feature turns and a head's lanes are a power of two
  int stages;         // tokens of a team in shared memory
  int warps, teams;   // of a team, of a block (a block a row: its warps, 1)
  int vectors;        // a block a row: 16-byte words that a thread holds at once
  int64_t tokens;     // of a block
  int smem;
};

// heads, norm: of the n_rows tensors; lph: lanes a head is dealt in.
inline RopeForm rope_form(int64_t n, int n_rows, const int32_t* heads_of, const int32_t* norm_of, int head_dim,
                          int pairs, int lph, bool half, int sms) {
  int heads = 0;
  int64_t values = 0;   // of a token's queries and keys
  for (int i = 0; i < n_rows; ++i) {
    heads = std::max(heads, heads_of[i]);
    values += static_cast<int64_t>(heads_of[i]) * head_dim;
  }
  // warps that take all heads of a token in one step
  const int64_t steps = (static_cast<int64_t>(heads) * lph + 31) / 32;
  const int norm = norm_of[0];
  const bool full = 2 * pairs == head_dim && 8 * lph == head_dim;
  // Estimates in ns, from measured runs of 150 to 4680 tokens: a block a row starts at once but takes blocks and values
  // slowly (norm over the token, 900 tokens of 2 x 1536 5.0 us against 6.9, of 2 x 5120 14.7 against 12.3; per head,
  // 450 of 24 and 8 heads 5.8 against 5.7, 1560 18.6 against 8.6; none, 310 of 2 x 5120 4.9 against 3.8).
  const int64_t lanes = 8 * values / head_dim * lph, work = n * lanes / 1000;   // idle ones too
  const bool token_norm = norm == ISPA_QK_NORM_TOKEN, head_norm = norm == ISPA_QK_NORM_HEAD;
  const int64_t block_ns =
      2000 + std::max(n * n_rows * 9 / 10, work * (token_norm ? 130 : !head_norm ? 114 : half ? 200 : 140) / 100);
  const int64_t stream_ns =
      token_norm ? std::max(5500 + std::min<int64_t>(1400, values * 45 / 100) + values * 9 / 100,
                            4500 + work * 80 / 100)
      : head_norm ? std::max(4800 + lanes / 4, 2000 + work * 85 / 100)
                  : std::max(3500 + values * 9 / 100, 2600 + work * 60 / 100);
  if (stream_ns < block_ns && values <= R_SMEM / 4 && (n_rows == 1 || norm_of[1] == norm)) {
    const int fixed = token_norm ? 4 * static_cast<int>(values) : 0;
    const auto token_bytes = [&](int stages) {
      return 2 * stages * static_cast<int>(values) + ((8 * pairs + 15) & ~15) + 16 + 2 * TEAM_WARPS * 8;
    };
    const auto teams_of = [&](int warps, int stages) {
      return std::min({32 / warps, warps > 1 ? 15 : 32, (R_SMEM - fixed) / token_bytes(stages)});
    };
    // Few warps a team where that makes more teams (4680 x 2 x 1536: one warp 15.0 us, two 17.1), more where shared
    // memory holds few tokens anyway (4680 x 2 x 5120: five warps 38.2 us, four 39.8, two 51.0).
    int warps = static_cast<int>(steps <= 6 ? 1 : std::min<int64_t>(TEAM_WARPS, (steps + 3) / 4));
    // A team's next token on its way while it works on one, unless that leaves half of the teams (1560 tokens of 160
    // and 40 heads of 96, per head: 36.9 us with one token each, 42.5 with two).
    int stages = teams_of(warps, 1) >= 2 * teams_of(warps, 2) ? 1 : 2;
    // A team for each of the SM's tokens where they all fit: none waits for another (per head, 1560 tokens of 24 and 8
    // heads 11.3 -> 8.6 us, 4680 of 2 x 1536 15.7 -> 13.5; over the token, 2600 of 2 x 1536 13.0 -> 10.6).
    const int64_t each = (n + sms - 1) / sms;
    const int all = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({TEAM_WARPS, 32 / each, (steps + 1) / 2})));
    const bool at_once = teams_of(all, 1) >= each;
    if (at_once) warps = all, stages = 1;
    const int teams = at_once ? static_cast<int>(each) : teams_of(warps, stages);
    if (teams >= 1)
      return {true, full, stages, warps, teams, 0, std::max<int64_t>(each, teams), fixed + teams * token_bytes(stages)};
  }
  const int w = steps <= 16 ? 1 : steps <= 32 ? 2 : 4;
  return {false, full, 1, static_cast<int>(std::min<int64_t>(16, (steps + w - 1) / w)), 1, w, 1, 0};
}

}  // namespace ispa
