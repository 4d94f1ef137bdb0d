// How far a chunk of the relaxed states looks back along its chain, and which chunks
// others may wait for. Used by the kernels and, compiled for the host, by a test: every chunk
// that is waited for publishes.
#pragma once

#ifdef __CUDACC__
#define DMC_CHAIN_FN __host__ __device__ __forceinline__
#else
#define DMC_CHAIN_FN inline
#endif

namespace dmc {

// Chunks between two whose `in` others may wait for; products of alphas below kTiny carry nothing.
constexpr int kAnchor = 16;
constexpr float kTiny = 1.17549435e-38f;  // 2^-126

// Whether others may ask for what comes into the chunk that has n neighbours on the side it comes
// from and whose own alphas have the product `prod`: the chunk then publishes it.
DMC_CHAIN_FN bool asked_for(int n, float prod) { return n > 0 && n % kAnchor == 0 && !(prod < kTiny); }

// The neighbour, counted from the nearest as 1, that a chunk with n > 0 of them need not look
// beyond: an anchor, waited for unless the walk ends before or at it, or the last one.
DMC_CHAIN_FN int chain_reach(int n) { return (n - 1) % kAnchor + 1; }

// Whether the walk ends at a neighbour whose own alphas have the product `prod`, those of all up to
// it `upto`. For numbers the second follows from the first; where an alpha between is not one,
// `upto` says nothing, and the first alone keeps the walk from an anchor that does not publish.
DMC_CHAIN_FN bool chain_ends(float prod, float upto) { return prod < kTiny || upto < kTiny; }

}  // namespace dmc
