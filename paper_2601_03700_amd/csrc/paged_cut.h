// How the keys of an entry or a tile are cut among workgroups: plain integer
// arithmetic, the same on the host and in a kernel.
#pragma once

namespace adept {

struct KeyRange {
  int begin, end;
};

// Part p of `parts` (at most 32) of the keys 0 .. n-1, in whole blocks of `block`;
// the parts behind the last key are empty.  The length is bounded before it is
// added: begin + per of the last part can pass the largest int.
constexpr KeyRange part_of_keys(int n, int parts, int p, int block) {
  const int per = ((n + block - 1) / block + parts - 1) / parts * block;
  const int begin = p * per < n ? p * per : n;
  return {begin, begin + (per < n - begin ? per : n - begin)};
}

// Units of a stretch of single entries' keys, so that `sum` units make about `want`
// stretches, and the stretches of an entry of `units` (an entry without keys is one).
// Longer than 2^24 units, the most that an entry has, means the same as 2^24.
constexpr int stretch_units(long long sum, int want, int least) {
  const long long most = 1 << 24, cut = (sum + want - 1) / want;
  return cut < least ? least : (int)(cut < most ? cut : most);
}
constexpr int stretches(int units, int cut) {
  const int n = (units + cut - 1) / cut;
  return n > 1 ? n : 1;
}

}  // namespace adept
