// The walk of the states' chunks along their chain (dmc_chain.h) on the host: prod[i] is the product of
// chunk i's alphas, chunk 0 the first of the chain. For chunk c, walks[c] is the number of neighbours whose own
// sums it adds up, waits[c] the anchor whose `in` it waits for (-1: none); publishes[c] is 1 where
// chunk c publishes what comes into it.
#include "dmc_chain.h"

extern "C" void dmc_chain_rule(int chunks, const float* prod, int* walks, int* waits, int* publishes) {
  for (int c = 0; c < chunks; ++c) {
    walks[c] = 0;
    waits[c] = -1;
    publishes[c] = dmc::asked_for(c, prod[c]);
    if (c == 0) continue;
    const int reach = dmc::chain_reach(c);
    float upto = 1.f;
    bool end = false;
    while (walks[c] < reach && !end) {
      ++walks[c];
      upto *= prod[c - walks[c]];
      end = dmc::chain_ends(prod[c - walks[c]], upto);
    }
    if (!end && reach < c) waits[c] = c - reach;
  }
}
