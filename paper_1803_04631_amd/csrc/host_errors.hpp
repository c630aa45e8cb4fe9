// What the library's sources share on the host: the error message of a thread's most recent failure.
#pragma once

namespace mlda {

// Keeps "what: why" (why may be null) for mlda_last_error and returns the code; throws nothing.
int set_error(int code, const char* what, const char* why = nullptr) noexcept;

}  // namespace mlda
