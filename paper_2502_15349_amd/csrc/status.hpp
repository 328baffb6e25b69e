// The library's error message, one per thread (defined in ae_attn.hip, read by ae_attn_last_error).
#pragma once
#include "../../include/ae_attn.h"

namespace ae {
ae_status_t fail(ae_status_t code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
}
