// rotated_probe_stub.cpp -- the host-only stand-in of hip_host_stub.cpp with a
// dispatch probe that records another map: STUB_MAP in the environment is
// "turned N" (workgroup b on XCD (b + N) mod 8), "mod4", "one_off", "one_xcd"
// or "far" (ids from 8 on).
#define launch_probe_xcc launch_probe_xcc_straight
#include "hip_host_stub.cpp"
#undef launch_probe_xcc

#include <string>

namespace nuna {

hipError_t launch_probe_xcc(int G, int32_t* xcc, int32_t* hw_id, hipStream_t stream) {
    launch_probe_xcc_straight(G, xcc, hw_id, stream);
    const char* const env = std::getenv("STUB_MAP");
    const std::string map = env ? env : "turned 0";
    for (int b = 0; b < G; ++b) {
        if (map.rfind("turned ", 0) == 0) xcc[b] = (b + std::atoi(map.c_str() + 7)) % 8;
        if (map == "mod4") xcc[b] = (b + 3) % 4;
        if (map == "one_off") xcc[b] = (b + 3 + (b == 1234)) % 8;
        if (map == "one_xcd") xcc[b] = 5;
        if (map == "far") xcc[b] = 8 + b % 8;
    }
    return hipSuccess;
}

}  // namespace nuna
