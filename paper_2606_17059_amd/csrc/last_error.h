// last_error.h -- the message behind pr_last_error, for every file of the C ABI.
#ifndef PR_LAST_ERROR_H
#define PR_LAST_ERROR_H

#include "prefix_router.h"

namespace pr {

// Keeps msg as the calling thread's last error and returns s; PR_OK clears it.
pr_status set_last_error(pr_status s, const char *msg) noexcept;

}  // namespace pr

#endif
