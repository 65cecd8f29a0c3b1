// Element types of the training-side operators: loads, conversions, stores.
#pragma once
#include "icq_internal.h"

#include <atomic>

typedef float icq_f32x4 __attribute__((ext_vector_type(4)));
typedef int icq_i32x8 __attribute__((ext_vector_type(8)));

template <int TYPE> struct IcqElem;                    // TYPE: ICQ_F32, ICQ_F16, ICQ_BF16
template <> struct IcqElem<ICQ_F32> {
    typedef float raw;
    static constexpr int PER = 4;                      // elements in 16 bytes
    __device__ static float get(raw x) { return x; }
    __device__ static raw put(float x) { return x; }
    __device__ static void unpack(const uint4 &v, float *x) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    __device__ static uint4 pack(const float *x) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
template <> struct IcqElem<ICQ_F16> {
    typedef _Float16 raw;
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    static constexpr int PER = 8;
    __device__ static float get(raw x) { return (float)x; }
    __device__ static raw put(float x) { return (raw)x; }
    __device__ static void unpack2(uint32_t w, float *x) {
        const pair p = __builtin_bit_cast(pair, w);
        x[0] = (float)p.x; x[1] = (float)p.y;
    }
    __device__ static uint32_t pack2(float a, float b) { pair p = {(raw)a, (raw)b}; return __builtin_bit_cast(uint32_t, p); }
    __device__ static void unpack(const uint4 &v, float *x) {
        unpack2(v.x, x); unpack2(v.y, x + 2); unpack2(v.z, x + 4); unpack2(v.w, x + 6);
    }
    __device__ static uint4 pack(const float *x) {
        return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
    }
};
template <> struct IcqElem<ICQ_BF16> {
    typedef __bf16 raw;
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    static constexpr int PER = 8;
    __device__ static float get(raw x) { return __uint_as_float((uint32_t)__builtin_bit_cast(uint16_t, x) << 16); }
    __device__ static raw put(float x) { return (raw)x; }
    __device__ static void unpack2(uint32_t w, float *x) {
        x[0] = __uint_as_float(w << 16); x[1] = __uint_as_float(w & 0xffff0000u);
    }
    __device__ static uint32_t pack2(float a, float b) { pair p = {(raw)a, (raw)b}; return __builtin_bit_cast(uint32_t, p); }
    __device__ static void unpack(const uint4 &v, float *x) {
        unpack2(v.x, x); unpack2(v.y, x + 2); unpack2(v.z, x + 4); unpack2(v.w, x + 6);
    }
    __device__ static uint4 pack(const float *x) {
        return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
    }
};

static inline int icq_type_bytes(int type) { return type == ICQ_F32 ? 4 : type == ICQ_F16 || type == ICQ_BF16 ? 2 : 0; }

// Two values as 8-bit codes in the low (HI = false) or high half of `old`, rounded to nearest even.
template <int FORMAT, bool HI>
__device__ __forceinline__ uint32_t icq_codes2(float a, float b, uint32_t old) {
    if constexpr (FORMAT == ICQ_E4M3) return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, HI);
    else return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(a, b, (int)old, HI);
}

// Compute units of the current device; 0 when the runtime does not say.
static inline int icq_num_cu() {
    static std::atomic<int> seen[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 0;
    if ((n = seen[dev].load(std::memory_order_relaxed)) != 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
    seen[dev].store(n, std::memory_order_relaxed);
    return n;
}

// A call with enough of these types chosen at run time: TYPE in the body is a constant.
#define ICQ_FOR_TYPE(type, ...)                                             \
    switch (type) {                                                         \
        case ICQ_F32: { constexpr int TYPE = ICQ_F32; __VA_ARGS__; } break; \
        case ICQ_F16: { constexpr int TYPE = ICQ_F16; __VA_ARGS__; } break; \
        default: { constexpr int TYPE = ICQ_BF16; __VA_ARGS__; } break;     \
    }
