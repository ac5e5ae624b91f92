// A device buffer of a context that grows on demand, and what is known of its contents.  Host code only.
#pragma once
#include <stddef.h>

namespace csd {

struct HostIo {
  void* base = nullptr;
  size_t cap = 0;
  bool in_graph = false;   // a captured call used it: its graph holds the address
  bool cleared = false;    // its start has been set to zero since it was allocated
  void drop() { base = nullptr; cap = 0; in_graph = false; cleared = false; }
};

// Runs `clear` (0: done) unless the buffer's start has been cleared before.  One that failed is asked for again by the next call; one that was only
// captured runs with its graph, so a call outside cannot count on it.
template <typename Clear>
int clear_once(HostIo& b, bool captured, Clear clear) {
  if (b.cleared) return 0;
  const int rc = clear();
  b.cleared = rc == 0 && !captured;
  return rc;
}

}  // namespace csd
