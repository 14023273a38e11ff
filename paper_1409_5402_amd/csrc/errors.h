// The text of a failure in a call that has no handle: what same_lda_last_error(NULL) returns on the calling thread.
#pragma once

namespace same {

__attribute__((visibility("hidden"))) int fail_without_handle(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace same
