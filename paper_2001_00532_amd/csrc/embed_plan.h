// What the gradient of the embedding lookup decides from sizes and tokens alone, in plain C++: kernels, host code and tests on a machine without a GPU share it.
#pragma once

namespace psk {

// A token's place among the `count` rows from `first` on, if it is less than count.  Unsigned: a token may be any 32-bit number, and those before `first` and
// below 0 have places from 2^31 - 2^28 on, behind any rows that there are.
constexpr unsigned place_from(int id, int first) { return (unsigned)id - (unsigned)first; }

}  // namespace psk
