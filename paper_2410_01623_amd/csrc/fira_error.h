// How a call without a context reports a failure: the message is kept for fira_last_error(NULL), per thread.
#pragma once
#include "../../include/fira.h"

__attribute__((visibility("hidden"))) fira_status fira_fail_without_context(fira_status st, const char* msg) noexcept;
