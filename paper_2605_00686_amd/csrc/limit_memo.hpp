// What kernels' LDS limits were raised to, so that the runtime is asked once: host code.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace moe {

struct LimitMemo {
    // The library has about 70 kernels that need it, a node 8 devices.
    static constexpr unsigned kPlaces = 4096;
    struct Entry {
        const void *kernel;
        int dev;
        size_t limit;
    };
    Entry at[kPlaces];  // (zeros to begin with)
    // The limit of a kernel on a device, 0 where it was not raised; NULL where there is no room to remember it.
    size_t *of(int dev, const void *kernel) {
        const uint64_t mixed = ((uint64_t)(uintptr_t)kernel + (uint64_t)(unsigned)dev * 0x632be59bd9b4e019ull) * 0x9e3779b97f4a7c15ull;
        unsigned i = (unsigned)(mixed >> 40);
        for (unsigned tries = 0; tries < kPlaces; ++tries, ++i) {
            Entry &e = at[i % kPlaces];
            if (!e.kernel) e.kernel = kernel, e.dev = dev;
            if (e.kernel == kernel && e.dev == dev) return &e.limit;
        }
        return nullptr;
    }
};

}  // namespace moe
