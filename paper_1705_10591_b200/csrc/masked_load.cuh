// Loads that may be left out, without a branch.
#pragma once

#include "seq_common.cuh"

namespace conv2d_b200 {

// V adjacent elements, or zeros.  As `there ? load : zeros` this becomes a branch where lanes differ, with copies behind the load that wait for it: loads that
// should be under way together then follow one another (the walk of the delta rule's pieces stood 2000 cycles of 5500 at a load ahead).
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_masked(const T* p, bool there)
{
    constexpr int BYTES = sizeof(T) * V;
    Pack<T, V> v;
    if constexpr (BYTES >= 16) {
        uint32_t* r = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i)
            asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
                         "@q ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
                         : "=&r"(r[4 * i]), "=&r"(r[4 * i + 1]), "=&r"(r[4 * i + 2]), "=&r"(r[4 * i + 3]) : "l"(reinterpret_cast<const char*>(p) + 16 * i), "r"((int)there));
    } else if constexpr (BYTES == 8) {
        uint32_t* r = reinterpret_cast<uint32_t*>(&v);
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %3, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\t@q ld.global.v2.b32 {%0, %1}, [%2];\n\t}"
                     : "=&r"(r[0]), "=&r"(r[1]) : "l"(p), "r"((int)there));
    } else if constexpr (BYTES == 4) {
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\tmov.b32 %0, 0;\n\t@q ld.global.b32 %0, [%1];\n\t}"
                     : "=&r"(*reinterpret_cast<uint32_t*>(&v)) : "l"(p), "r"((int)there));
    } else {
        static_assert(BYTES == 2, "an element of 16 bits");
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\tmov.b16 %0, 0;\n\t@q ld.global.b16 %0, [%1];\n\t}"
                     : "=&h"(*reinterpret_cast<uint16_t*>(&v)) : "l"(p), "r"((int)there));
    }
    return v;
}

}  // namespace conv2d_b200
