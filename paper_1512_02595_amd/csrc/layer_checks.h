// What the host sides of the layers' calls share: their buffers are looked over before anything is enqueued.
#ifndef LAYER_CHECKS_H
#define LAYER_CHECKS_H

#include <cstddef>
#include <cstdint>
#include <initializer_list>

#include "ctc_layer.h"

namespace layer {

// The status of a launch; its error, if any, is what ctc_layer_last_hip_error tells the calling thread.
ctc_status_t launched(int err);

// A buffer of the call.  An output may not overlap any other buffer, unless it is `alias`-ed to it: the same
// address and, by the caller's word, the same shape.
struct Buffer {
    const void* at;
    size_t bytes;
    bool output;
    bool required = true;
    size_t align = 4;
    bool alias = false;              // this input may be the output that `may_alias` is set for
    bool may_alias = false;
};

inline bool buffers_in_order(std::initializer_list<Buffer> list)
{
    for (const Buffer& b : list) {
        if (!b.at && b.required) return false;
        if (reinterpret_cast<uintptr_t>(b.at) % b.align) return false;
    }
    for (const Buffer* a = list.begin(); a != list.end(); ++a)
        for (const Buffer* b = a + 1; b != list.end(); ++b) {
            if (!(a->output || b->output) || !a->at || !b->at) continue;
            if (a->at == b->at && ((a->alias && b->may_alias) || (b->alias && a->may_alias))) continue;
            const uintptr_t i = reinterpret_cast<uintptr_t>(a->at), j = reinterpret_cast<uintptr_t>(b->at);
            if (i < j + b->bytes && j < i + a->bytes) return false;
        }
    return true;
}

inline size_t element(ctc_dtype_t dtype) { return dtype == CTC_DTYPE_F32 ? 4 : 2; }
inline size_t matrix(int rows, int width, size_t elem) { return static_cast<size_t>(rows) * width * elem; }
inline size_t list_bytes(int rows) { return (static_cast<size_t>(rows) + 1) * 4; }
inline size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace layer

#endif  // LAYER_CHECKS_H
