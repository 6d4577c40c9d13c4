// The embedding lookup and its gradient: products by a matrix S (tokens x vocabulary) with one stored entry per row, `factor`, or none.
//
//   Y = S E:       Y[t][:] = factor E[ids[t]][:]
//   dE = S^T dY:   dE[v][:] = factor sum over { t : ids[t] = v }, in ascending t, of dY[t][:]
//
// Eight columns at a time.  Rows begin at any element, so these are loads and stores of 16 bytes at any address.
#pragma once
#include "row8.h"

namespace psk {

// Columns of a row go by eight; the last eight are the row's last, so some of them may be among those before too (`skip` of them).  Rows of less
// than eight columns are taken element by element.
struct Unit { int col, skip; };
__device__ __forceinline__ Unit unit_of(int unit, int dim)
{
    const int at = 8 * unit, col = min(at, dim - 8);
    return Unit{col, at - col};
}

}  // namespace psk
