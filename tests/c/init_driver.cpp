// Runs nuna_init, then one all-reduce in XCD placement (made-up addresses: the
// launch stubs touch no buffer), and prints the three statuses and the flag.
#include <cstdint>
#include <cstdio>

#include "nuna.h"

int main() {
    const int init = nuna_init();
    nuna_device_info_t info = {};
    const int dev = nuna_get_device_info(&info);
    const uintptr_t base = uintptr_t(1) << 44;
    const void* in[2] = {reinterpret_cast<const void*>(base), reinterpret_cast<const void*>(base + (1 << 20))};
    void* out[2] = {reinterpret_cast<void*>(base + (2 << 20)), reinterpret_cast<void*>(base + (3 << 20))};
    const int call = nuna_allreduce(in, out, 2, 1024, NUNA_BF16, NUNA_ALGO_ONE_SHOT, NUNA_PLACE_XCD, nullptr);
    std::printf("init %d info %d verified %d allreduce %d\n", init, dev, info.map_verified, call);
    return 0;
}
