// Reads groups of 32 floats and writes for each its scale byte, its 32 codes and the values that they stand for, as floats, by the
// kernels' own functions built for the host.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <hip/hip_runtime.h>

#undef __device__
#define __device__ __host__ __attribute__((device))
static inline __host__ unsigned host_float_as_uint(float f) { unsigned u; memcpy(&u, &f, 4); return u; }
static inline __host__ float host_uint_as_float(unsigned u) { float f; memcpy(&f, &u, 4); return f; }
#define __float_as_uint host_float_as_uint
#define __uint_as_float host_uint_as_float
typedef unsigned u32;
namespace lmk {
static inline __host__ float inverse_step(u32 scale) { return host_uint_as_float((scale == 0u || scale == 255u) ? 0u : (254u - scale) << 23); }
static inline __host__ float step_of(u32 scale) { return host_uint_as_float(scale << 23); }
}
#define LMK_GS_GROUPED_H
#include "block4.h"

int main()
{
    float v[32];
    while (fread(v, 4, 32, stdin) == 32) {
        u32 top = 0;
        for (float f : v) {
            const u32 b = host_float_as_uint(f) & 0x7fffffffu;
            top = top > b ? top : b;
        }
        float out[65];
        const u32 s = lmk::scale4_of_max(top);
        out[0] = (float)s;
        for (int i = 0; i < 32; ++i) {
            const u32 code = s == 255u ? 0u : lmk::code4_of(v[i], lmk::inverse_step(s));
            out[1 + i] = (float)code;
            out[33 + i] = lmk::value4_of(code, lmk::step_of(s));
        }
        fwrite(out, 4, 65, stdout);
    }
    return 0;
}
