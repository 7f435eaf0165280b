// errors.hpp -- the thread's error message (ql_last_error), for the C entries
// outside api.cpp.
#pragma once

namespace qlayer {

// Sets the message to "what: detail" (or "what") and returns the code. QL_OK
// with "" clears it.
int set_error(int code, const char* what, const char* detail = nullptr) noexcept;

}  // namespace qlayer
