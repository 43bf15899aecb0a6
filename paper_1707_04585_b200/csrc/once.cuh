// Set-up that a kernel needs once per device.  (No CUDA in here: the host tests compile it by itself.)
#pragma once
#include <atomic>

// Function attributes (the dynamic shared-memory limit) belong to a device, not to the process: each kernel's launcher keeps one of these and sets its
// attributes the first time it runs on a device.  Setting them twice is harmless, so no lock; but a thread goes on only when they are set, by itself or
// by another that has finished: until then every caller sets them.
struct OncePerDevice {
    std::atomic<bool> done[64] = {};
    // set() -> whether it worked; if not, the next call tries again
    template <class F> bool ensure(int device, F set) {
        const bool known = device >= 0 && device < 64;
        if (known && done[device].load(std::memory_order_acquire)) return true;
        if (!set()) return false;
        if (known) done[device].store(true, std::memory_order_release);
        return true;
    }
};
