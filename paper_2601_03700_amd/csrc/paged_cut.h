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

}  // namespace adept
