// The list of experts that a layer for a few tokens keeps in its workspace, and what is taken from it.  Integers only, so that a host
// program can try any content.
#pragma once

#include <cstdint>

#include "deal.h"

// The experts that a few tokens list, ascending: work items of a layer for a decoding step
struct fmoe_unit {
  int32_t expert, row0;         // row0: its first hidden row, the rows by expert and token
  uint32_t mask;                // tokens that list it
};

// The list is a workspace's content: whatever is read there (two calls that share a workspace without an order, say) is kept within the
// layer's experts and the call's rows.
struct ListBounds {
  int E, T, pairs;              // pairs: hidden rows
};
FMOE_HOST_DEVICE int units_within(int n, const ListBounds& b) {
  const int most = b.pairs < b.E ? b.pairs : b.E;
  return n < 0 ? 0 : n < most ? n : most;
}
FMOE_HOST_DEVICE fmoe_unit unit_within(fmoe_unit r, const ListBounds& b) {
  r.mask &= (1u << b.T) - 1u;
  const int last = b.pairs - (r.mask != 0u ? __builtin_popcount(r.mask) : 1);
  r.expert = r.expert < 0 ? 0 : r.expert < b.E ? r.expert : b.E - 1;
  r.row0 = r.row0 < last ? r.row0 : last;
  r.row0 = r.row0 < 0 ? 0 : r.row0;
  return r;
}
// Of the n units (as above, one at least), those that two tokens eight apart list: how many, and which
FMOE_HOST_DEVICE int full_units_within(int n_full, int n) { return n_full < 0 ? 0 : n_full < n ? n_full : n; }
FMOE_HOST_DEVICE int full_unit_within(int u, int n) { return u < 0 ? 0 : u < n ? u : n - 1; }
