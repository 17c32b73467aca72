// Address spaces of the pointers that kernels dereference.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lasgd {

// Every pointer the kernels dereference is device (global) memory.  Pointers
// that come out of the tables are generic as far as the compiler can tell and
// would be accessed with FLAT instructions; casting to the global address
// space makes every access a GLOBAL load or store.
#define LASGD_GLOBAL_AS __attribute__((address_space(1)))
template <class T> __device__ __forceinline__ const LASGD_GLOBAL_AS T *as_global(const void *p)
{
    return reinterpret_cast<const LASGD_GLOBAL_AS T *>(reinterpret_cast<uintptr_t>(p));
}
template <class T> __device__ __forceinline__ LASGD_GLOBAL_AS T *as_global(void *p)
{
    return reinterpret_cast<LASGD_GLOBAL_AS T *>(reinterpret_cast<uintptr_t>(p));
}

#define LASGD_CONST_AS __attribute__((address_space(4)))
template <class T> __device__ __forceinline__ const LASGD_CONST_AS T *as_const(const T *p)
{
    return reinterpret_cast<const LASGD_CONST_AS T *>(reinterpret_cast<uintptr_t>(p));
}

} // namespace lasgd
