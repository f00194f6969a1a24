// How much dynamic shared memory each kernel has been allowed on each device (host only).
#pragma once

#include <stddef.h>

#include <map>
#include <mutex>
#include <utility>

#include "cobalt.h"

namespace cobalt {

class KernelGrants {
public:
    // Calls set() unless the kernel has been granted `bytes` or more; COBALT_OK, or what set() or the host's memory failed with.  The lock is
    // held while it is set: of two first calls with different sizes the smaller one may not be set last while the larger one is remembered.
    template <typename Set>
    int ensure(const void* kernel, int device, size_t bytes, Set set)
    {
        try {                                                       // the map may run out of host memory
            std::lock_guard<std::mutex> guard(lock_);
            size_t& have = granted_[std::make_pair(kernel, device)];
            if (have > bytes) return COBALT_OK;
            const int rc = set();
            if (rc == COBALT_OK) have = bytes + 1;
            return rc;
        } catch (...) {
            return COBALT_ERR_HOST_ALLOC;
        }
    }

private:
    std::mutex lock_;
    std::map<std::pair<const void*, int>, size_t> granted_;         // bytes + 1 once set up
};

}  // namespace cobalt
