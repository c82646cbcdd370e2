// Library-wide entry points: last-error text and version.
#include <atomic>

#include "common.hpp"

namespace fsr {
char* error_buffer() {
    static thread_local char buf[256] = {0};
    return buf;
}
// The upper 16 bits are none that flags, indexes, counts or ordinary numbers leave there: with a count alone, eight bytes of a mask in a workspace
// (1 0 1 0 0 0 0 0) were an arrival at a process's first call.  (As a float or a bf16 they are about -4e32.)
unsigned long long next_call_id() {
    static std::atomic<unsigned long long> counter{0};
    const unsigned long long n = counter.fetch_add(1, std::memory_order_relaxed) + 1;
    return (0xf5a300000000ull + n) & 0xffffffffffffull;
}
}  // namespace fsr

extern "C" const char* fsr_last_error(void) { return fsr::error_buffer(); }
extern "C" const char* fsr_version(void) { return "faser_verify 0.1 (gfx950)"; }
