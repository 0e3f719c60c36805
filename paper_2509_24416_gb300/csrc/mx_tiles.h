// Tile choice of the microscaled product: host code by itself, so that tests can ask which
// tile a shape takes.
#pragma once

#include <algorithm>
#include <cstdint>

namespace clq {
namespace mx {

constexpr int TN = 128;   // output channels a CTA
constexpr int KC = 256;   // codes of a K step: one 128-byte row

// A tile: `nt` rows of X by 128 cg channels.
struct TileShape {
  int nt, cg;
};

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
