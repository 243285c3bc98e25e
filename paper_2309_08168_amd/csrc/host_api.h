// Host-side helpers that the library's C++ translation units share with
// model.hip: the per-thread error message behind sd_last_error(), the guard
// that keeps C++ exceptions inside the C ABI, and the model's layer count.
#pragma once

#include <new>
#include <string>

#include "sd.h"

namespace sdk {

// Records msg as the calling thread's last error and returns st.
sd_status report(sd_status st, const std::string &msg);

// Layers of the model (0 for NULL).
int32_t model_layers(const sd_model *m);

}  // namespace sdk

#define SD_GUARD(...)                                                                                  \
    try {                                                                                              \
        __VA_ARGS__                                                                                    \
    } catch (const std::bad_alloc &) {                                                                 \
        return sdk::report(SD_ERR_OOM, "host allocation failed");                                      \
    } catch (...) {                                                                                    \
        return sdk::report(SD_ERR_DEVICE, "unexpected internal error");                                \
    }
