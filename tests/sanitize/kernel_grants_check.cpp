// First calls of one kernel with different sizes, from two threads.  The attribute is a plain number; the smaller call sets it only when
// the larger one has set its own, or after half a second.  Prints the attribute and what a later call at the larger size finds.
#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>

#include "kernel_grants.h"

int main()
{
    cobalt::KernelGrants grants;
    const int kernel = 0;
    std::atomic<size_t> attribute{0};
    std::atomic<bool> small_at_work{false};
    const size_t small = 60000, large = 100000;
    std::thread a([&] {
        grants.ensure(&kernel, 0, small, [&] {
            small_at_work = true;
            for (int i = 0; i < 500 && attribute < large; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
            attribute = small;
            return COBALT_OK;
        });
    });
    std::thread b([&] {
        while (!small_at_work) std::this_thread::yield();
        grants.ensure(&kernel, 0, large, [&] {
            attribute = large;
            return COBALT_OK;
        });
    });
    a.join();
    b.join();
    int calls = 0;
    auto count = [&] {
        ++calls;
        return COBALT_OK;
    };
    const int again = grants.ensure(&kernel, 0, large, count);           // granted
    const int lower = grants.ensure(&kernel, 0, 0, count);               // granted
    const int other = grants.ensure(&kernel, 1, small, count);           // another device's
    int failed = grants.ensure(&kernel, 2, small, [] { return COBALT_ERR_CUDA; });
    const int retried = grants.ensure(&kernel, 2, small, count);         // a failure is not remembered
    std::printf("%zu %d %d %d %d %d %d\n", attribute.load(), again, lower, other, failed, retried, calls);
    return 0;
}
