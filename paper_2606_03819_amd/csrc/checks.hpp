// Argument checks that the C entry points share.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <initializer_list>

#include "treeflash.h"

namespace tf {

// Alignment.  An array not aligned to its element size is an invalid
// argument.  Operands read with 16-byte vector loads (h, h', the weights, the
// LM head) must also be 16-byte aligned; an element-aligned pointer that is
// not is a valid request this build does not implement (TF_ERR_UNSUPPORTED).
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool dtype_ok(tf_dtype_t dt) { return dt == TF_F32 || dt == TF_BF16; }
inline size_t elem_bytes(tf_dtype_t dt) { return dt == TF_BF16 ? 2 : 4; }
inline bool elem_aligned(const void* p, tf_dtype_t dt) { return (reinterpret_cast<uintptr_t>(p) % elem_bytes(dt)) == 0; }
// a vector-loaded operand of type dt (non-null)
inline tf_status_t vec_status(const void* p, tf_dtype_t dt) {
    if (!elem_aligned(p, dt)) return TF_ERR_INVALID_ARG;
    return aligned16(p) ? TF_OK : TF_ERR_UNSUPPORTED;
}
// the first non-OK status of a list of vector-loaded operands, invalid before unsupported
inline tf_status_t vec_status_all(std::initializer_list<const void*> ps, tf_dtype_t dt) {
    tf_status_t worst = TF_OK;
    for (const void* p : ps) {
        const tf_status_t st = vec_status(p, dt);
        if (st == TF_ERR_INVALID_ARG) return st;
        if (st != TF_OK) worst = st;
    }
    return worst;
}

}  // namespace tf
