// What the entry points' units share on the host: pieces of a workspace and its check.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/tfla_mlstm.h"

namespace tfla {

inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

struct Carver {
    char* base; size_t off = 0;
    explicit Carver(void* p) : base(reinterpret_cast<char*>(p)) {}
    char* take(size_t bytes) {
        char* r = base ? base + off : nullptr;
        off = align_up(off + bytes);
        return r;
    }
};

inline int check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return TFLA_OK;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || have < need) return TFLA_ERR_WORKSPACE;
    return TFLA_OK;
}

}  // namespace tfla
