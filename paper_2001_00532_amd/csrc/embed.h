// The embedding lookup and its gradient: products by a matrix S (tokens x vocabulary) with one stored entry per row, `factor`, or none.
//
//   Y = S E:       Y[t][:] = factor E[ids[t]][:]
//   dE = S^T dY:   dE[v][:] = factor sum over { t : ids[t] = v } of dY[t][:], in an order that depends on the sizes, the type of dY and the tokens alone
#pragma once
#include "row8.h"
