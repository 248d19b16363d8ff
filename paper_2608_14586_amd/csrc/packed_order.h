// The order in which workgroups of attention over packed prompts take tiles of queries.
#pragma once

namespace vla {

// The rank of workgroup wg among total tiles of queries times H heads (tiles longest first, a
// tile's heads side by side), below 0 where there is none for it: a launch has a workgroup for
// every tile that there may be, often more than there are.  div(n) = n / H.
//
// Where all workgroups run at once, workgroup i and i + 256 on one CU, a CU's two are a
// long and a short one, and the longest have a CU alone.  Against plain order: one prompt of 2048,
// 32 heads of 128, 48.0 us for 49.5; nine of 1 to 701, 14 heads of 64, 12.7 for 13.1; five of 700, 14
// heads of 128, 21.6 for 21.8.
template <class Div>
constexpr int packed_rank(int wg, int total, int H, Div div) {
  const int all = total * H;
  if (wg >= all) return -1;
  if (all <= 256 || all > 512) return wg;
  const int twice = all - 256;  // CUs with two
  if (wg < 256) return wg < twice ? 256 - twice + wg : wg - twice;
  // whole tiles from the shortest on, then what the first 256 left of theirs
  const int e = wg - 256, whole = (total - 1 - div(256)) * H, t = div(e);
  return e < whole ? (total - 1 - t) * H + e - t * H : 256 + e - whole;
}

}  // namespace vla
