// The thread-local error text behind adst_last_error, for the other files
// that define calls of the C boundary. Neither throws.
#pragma once

#include "adst.h"

namespace adst {

// Keeps the text and returns the status.
adst_status report(adst_status st, const char* text);
// ADST_OK, with the text cleared.
adst_status report_ok();

}  // namespace adst
