// What the C ABI of the operators around the codec checks its arguments with.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mqgrad.h"
#include "mqg_internal.h"

namespace mqg {

inline bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline bool known(mqg_dtype t) { return t == MQG_F32 || t == MQG_BF16; }
inline uintptr_t bytes_of(mqg_dtype t) { return t == MQG_F32 ? 4 : 2; }
inline uintptr_t bytes_of(mqg_index t) { return t == MQG_I64 ? 8 : 4; }

inline mqg_status cuda_status(const char* what, cudaError_t err)
{
    return err == cudaSuccess ? MQG_OK : report_error(MQG_ERR_CUDA, "%s: %s", what, cudaGetErrorString(err));
}

// Memory that a call reads or writes; `bytes` = 0: none.
struct Region {
    const char* name;
    const void* p;
    uint64_t bytes;
    bool meets(const Region& r) const
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(r.p);
        return bytes != 0 && r.bytes != 0 && (a < b ? b - a < bytes : a - b < r.bytes);
    }
};

// Whether what is written shares memory with anything else: MQG_OK if not.
template <int N> mqg_status check_apart(const char* what, const Region& written, const Region (&others)[N])
{
    for (const Region& r : others)
        if (written.meets(r)) return report_error(MQG_ERR_INVALID, "%s: %s and %s share memory", what, written.name, r.name);
    return MQG_OK;
}

inline mqg_status check_buffer(const char* what, const char* name, const void* p, mqg_dtype t, bool empty)
{
    if (!known(t)) return report_error(MQG_ERR_INVALID, "%s: unknown dtype %d of %s", what, (int)t, name);
    if (empty) return MQG_OK;
    if (!p) return report_error(MQG_ERR_INVALID, "%s: %s is null", what, name);
    if (!aligned(p, bytes_of(t))) return report_error(MQG_ERR_ALIGN, "%s: %s is not aligned to its elements", what, name);
    return MQG_OK;
}

}  // namespace mqg
