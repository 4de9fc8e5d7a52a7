// The text of a thread's last failure (ps_last_error) and the code that goes with it.
#pragma once
#include <stdint.h>

namespace psk {

// Sets the calling thread's error text and returns `code`.
int32_t fail(int32_t code, const char* fmt, ...);

}  // namespace psk
