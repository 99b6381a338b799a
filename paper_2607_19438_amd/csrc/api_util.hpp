// What the library's C entry points share, in whichever source they stand: the calling thread's last message,
// and the checks of a launch and of an address. Defined in qgemm_api.hip.
#pragma once

#include <stdint.h>

namespace qg {

// Keeps the message for qgemm_last_error and gives `code` back.
__attribute__((visibility("hidden"), format(printf, 2, 3))) int fail(int code, const char* fmt, ...);

// Clears the message; QGEMM_OK.
__attribute__((visibility("hidden"))) int ok();

// QGEMM_EHIP with a message if the launch before it failed.
__attribute__((visibility("hidden"))) int check_launch(const char* what);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace qg
