// The calling thread's last error, and the macros that set it: shared by
// every C entry of the library.
#pragma once
#include <hip/hip_runtime.h>

#include <string>
#include <tuple>
#include <type_traits>
#include <utility>

namespace nsg {

inline thread_local std::string g_err;

inline int set_err(int code, const std::string& msg) {
    g_err = msg;
    return code;
}

#define HIP_TRY(expr)                                                                  \
    do {                                                                               \
        hipError_t e_ = (expr);                                                        \
        if (e_ != hipSuccess)                                                          \
            return set_err(NSGCQT_EDEVICE, std::string(#expr) + ": " + hipGetErrorString(e_)); \
    } while (0)

// Launches kernel k with the arguments converted to its parameter types and
// returns the status of this launch alone. (hipGetLastError after a launch
// would also report an error that an earlier, unrelated HIP call of the
// caller left on the thread.)
template <typename... P, typename... A>
hipError_t launch_kernel(void (*k)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t s, A&&... a) {
    static_assert(sizeof...(P) == sizeof...(A), "kernel argument count");
    std::tuple<std::decay_t<P>...> vals(std::forward<A>(a)...);
    return std::apply(
        [&](auto&... v) {
            void* args[] = {static_cast<void*>(&v)...};
            return hipLaunchKernel(reinterpret_cast<const void*>(k), grid, block, args, lds, s);
        },
        vals);
}

#define LAUNCH_TRY(...)                                                                \
    do {                                                                               \
        hipError_t e_ = launch_kernel(__VA_ARGS__);                                    \
        if (e_ != hipSuccess)                                                          \
            return set_err(NSGCQT_EDEVICE, std::string("kernel launch: ") + hipGetErrorString(e_)); \
    } while (0)

}  // namespace nsg
