// Stores past the caches, of what does not stay in them for its reader.
#pragma once
#include <hip/hip_runtime.h>

namespace cprune {

// Does an output of so many bytes go past the caches?  The last-level cache has 256 MB, for what is in use besides too.  The distillation step at bf16 and the output's next
// reader, us into the caches and past them: 33 MB 37.6 and 40.1, 67 MB 70.5 and 74.7, 134 MB 143.5 and 137.6; the step alone at 1 GB 477 and 439.
inline bool past_caches(double bytes) { return bytes > 100e6; }

// v to *p, of a type with an alignment of its own.  Without what stands around the one store the compiler makes a single one of both, into the caches.
#define CPRUNE_STORE(p, v, past)        \
  do {                                  \
    if (past) {                         \
      asm volatile("");                 \
      __builtin_nontemporal_store(v, p); \
      asm volatile("");                 \
    } else {                            \
      *(p) = v;                         \
    }                                   \
  } while (0)

}  // namespace cprune
