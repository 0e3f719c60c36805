// Tile choice of the microscaled product: host code by itself, so that tests can ask which
// tile a shape takes.
#pragma once

#include <algorithm>
#include <cstdint>

namespace clq {
namespace mx {

constexpr int TN = 128;   // output channels a CTA
constexpr int KC = 256;   // codes of a K step: one 128-byte row (128 of 8 bits)

// A tile: `nt` rows of X by 128 cg channels.
struct TileShape {
  int nt, cg;
  int split = 1;  // CTAs that share its K steps
};

// The first column of Y of the channels from n0 on (a multiple of 32), two of which are one column if
// they are `gated`.
constexpr int first_column(int n0, bool gated) { return gated ? n0 / 2 : n0; }

// At most so many: a cluster's eight; more rows are better cut into more tiles.
constexpr int max_split(int nt) { return nt <= 32 ? 8 : nt <= 64 ? 4 : 1; }

// The tile of a product whose rows are `rows` for each of `matrices` matrices: the CTAs or
// pairs go ceil(tiles / units) rounds; a round takes its K steps and the part of an epilogue
// that the next round's MMAs do not cover, and the last epilogue and the launch come on top.
// The times are fitted to 112 products of 33 .. 8192 rows (step: us for 256 codes; epilogue:
// us a tile); the rule is within 10 % of the best of the five on all but six of them (18 % off at most).  Examples,
// us at 64 / 128 / 128 in pairs / 256 / 256 in pairs: 64 x 1152 -> 3456 3.8 / 4.1 / 4.1 / 5.1 /
// 4.8, 2048 x 4608 -> 1152 10.4 / 7.4 / 10.3 / 11.0 / 9.8, 4096 x 4608 -> 1152 18.4 / 11.7 /
// 13.9 / 11.2 / 15.3, 8192 x 4096 -> 8192 190 / 114 / 91 / 110 / 83.
inline TileShape pick_tile(int rows, int matrices, int N, int K, int sms, bool grouped) {
  if (rows <= 32) return {32, 1};
  struct Option {
    TileShape t;
    double step, epilogue;
    bool plan;  // a plan has such tiles
  };
  const Option options[] = {{{64, 1}, 0.22, 0.75, false},
                            {{128, 1}, 0.26, 1.03, true},
                            {{128, 2}, 0.21, 1.03, false},
                            {{256, 1}, 0.48, 1.8, false},
                            {{256, 2}, 0.36, 1.8, true}};
  TileShape best{128, 1};
  double least = 1e300;
  for (const Option& o : options) {
    if (grouped && !o.plan) continue;
    const int64_t tiles = static_cast<int64_t>(matrices) * ((rows + o.t.nt - 1) / o.t.nt) *
                          ((N + TN * o.t.cg - 1) / (TN * o.t.cg));
    const int64_t units = sms / o.t.cg;
    const double cost = ((tiles + units - 1) / units) *
                            ((K + KC - 1) / KC * o.step + 0.35 * o.epilogue) +
                        o.epilogue;
    if (cost < least) {
      least = cost;
      best = o.t;
    }
  }
  return best;
}

// The tile of a product of 8-bit codes, or of any with an activation or a residual behind it
// (`post`), whose tiles go 192 rows high as well.  As above, a round taking its K steps (of 128 bytes
// a row) and `round`, the launch, the first copies and the last epilogue `last`, us, fitted to 19
// shapes of 256 .. 32768 rows with each thing behind them: the rule is within 1 % of the best of the
// six in the mean and 11 % off at most (pick_tile's figures: 2 %, 19 %).  Examples, us at 64 / 128 /
// 128 in pairs / 192 in pairs / 256 / 256 in pairs: 8 bits 8192 x 4608 -> 1152 60 / 41 / 41 / 33 /
// 40 / 40, 8192 x 1152 -> 3456 50 / 36 / 32 / 28 / 34 / 28, 32768 x 4096 -> 8192 1375 / 906 / 781 /
// 716 / 860 / 677, 2048 x 1152 -> 1152 6.6 / 5.3 / 7.1 / 6.4 / 7.3 / 7.1; with GELU and a residual,
// blocks of 16, 8192 x 4608 -> 1152 40 / 31 / 29 / 25 / 28 / 31.
//
// Few rows with few channels leave most SMs without a tile, and a tile's K steps then take 0.19 us
// each, the time of their copies to one SM.  So 2, 4 or 8 CTAs share the K steps of a tile of 32 rows
// (2 or 4 of one of 64) where what they save is more than the `join`: us of its barriers, the sums on
// their way and the other epilogue.  Measured (with barriers at the CTA's scope; the cluster's, which they
// need, take 0.1 us more), us at 1 / 2 / 4 / 8, E4M3 stored as it is: 1 x
// 16384 -> 1024 25.7 / 15.7 / 10.3 / 9.0, 1 x 4608 -> 1152 9.0 / 7.2 / 6.0 / 6.8, 1 x 1152 -> 1152 4.0 /
// 4.8 / 4.7 / 6.2, 16 x 8192 -> 2048 14.3 / 9.8 / 7.5 / 14.8 (clusters that have to wait for one
// another), 64 x 4608 -> 1152 9.4 / 8.0 / 7.4, 256 x 4096 -> 1024 8.7 / 7.7 / 8.3; blocks of 16 with
// GELU and a residual 1 x 16384 -> 1024 16.5 / 11.0 / 8.2 / 8.3.  (Tiles of 128 rows, by two: 256 x
// 4608 -> 1152 9.7 where one of 64 takes 9.6 and two 8.2.)
inline TileShape pick_row_tile(int rows, int N, int row_bytes, int sms, bool codes8, bool post) {
  const int steps = (row_bytes + 127) / 128, channels = (N + TN - 1) / TN;
  // us that sharing a tile saves, against `least`; the split
  auto shared = [&](int nt, double step, double* least) {
    static const double join[2][3] = {{0.95, 1.4, 3.1}, {1.55, 2.45, 1e9}};
    const int64_t tiles = static_cast<int64_t>((rows + nt - 1) / nt) * channels;
    int best = 1;
    for (int i = 0, n = 2; n <= max_split(nt) && n <= steps; ++i, n *= 2) {
      if (tiles * n > (nt * n <= 128 ? sms : sms / 2)) break;
      const double cost = ((steps + n - 1) / n - steps) * step + join[nt > 32][i] + (post ? 0. : 0.5);
      if (cost < *least) {
        *least = cost;
        best = n;
      }
    }
    return best;
  };
  if (rows <= 32) {
    double least = 0.;
    return {32, 1, shared(32, codes8 ? 0.185 : 0.2, &least)};
  }
  struct Option {
    TileShape t;
    double step, round, last;
  };
  static const Option table[3][6] = {
      {{{64, 1}, 0.187, 0.39, 2.77},
       {{128, 1}, 0.226, 0.66, 2.99},
       {{128, 2}, 0.179, 0.63, 3.39},
       {{192, 2}, 0.232, 0.81, 3.70},
       {{256, 1}, 0.422, 1.10, 3.41},
       {{256, 2}, 0.303, 1.10, 3.84}},  // 8 bits, stored as they are
      {{{64, 1}, 0.174, 0.70, 3.53},
       {{128, 1}, 0.204, 1.03, 4.31},
       {{128, 2}, 0.173, 1.07, 4.31},
       {{192, 2}, 0.211, 1.77, 4.53},
       {{256, 1}, 0.375, 1.79, 5.05},
       {{256, 2}, 0.270, 2.20, 4.91}},  // 8 bits
      {{{64, 1}, 0.152, 1.02, 3.50},
       {{128, 1}, 0.179, 1.43, 4.38},
       {{128, 2}, 0.139, 1.52, 4.37},
       {{192, 2}, 0.170, 2.34, 4.39},
       {{256, 1}, 0.335, 2.53, 5.02},
       {{256, 2}, 0.234, 2.87, 4.90}}};  // 4 bits
  TileShape best{128, 1};
  double least = 1e300;
  for (const Option& o : table[codes8 ? (post ? 1 : 0) : 2]) {
    const int64_t tiles = static_cast<int64_t>((rows + o.t.nt - 1) / o.t.nt) *
                          ((N + TN * o.t.cg - 1) / (TN * o.t.cg));
    const int64_t units = sms / o.t.cg;
    const double cost = ((tiles + units - 1) / units) * (steps * o.step + o.round) + o.last;
    double less = 0.;
    const int split = o.t.nt == 64 ? shared(64, o.step, &less) : 1;
    if (cost + less < least) {
      least = cost + less;
      best = o.t;
      best.split = split;
    }
  }
  return best;
}

// The same for T tokens' rows to k of E matrices each.  They are taken as evenly spread over the
// matrices that have any; T rows at most meet one of them.
inline TileShape pick_grouped_tile(int T, int k, int E, int N, int K, int sms) {
  if (T <= 32) return {32, 1};
  const int64_t picks = static_cast<int64_t>(T) * k;
  const int64_t spread = std::max<int64_t>(1, std::min<int64_t>(E, picks));
  return pick_tile(std::max(33, static_cast<int>((picks + spread - 1) / spread)),
                   static_cast<int>(spread), N, K, sms, true);
}

}  // namespace mx
}  // namespace clq
