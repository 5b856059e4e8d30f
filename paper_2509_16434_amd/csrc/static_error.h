// The error text of the calls without a context (what ppo_last_error(NULL) gives), shared by the library's source files.
#pragma once

__attribute__((visibility("hidden"))) int ppo_static_fail(int code, const char* text);  // returns `code`
