// Elements of the operators that have an element type (anr_dtype), and the activations: values are float32 from
// where they are loaded to where they are stored, with one rounding there.
#pragma once
#include <type_traits>

#include "anr.h"
#include "anr_device.h"

namespace anr {

typedef _Float16 half_t;
typedef __bf16 bf16_t;

template <typename T>
__device__ __forceinline__ float to_float(T v) { return (float)v; }
template <typename T>
__device__ __forceinline__ T from_float(float v) { return (T)v; }          // to nearest, ties to even

// V elements that are loaded and stored together; aligned as the pointer is known to be.
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
};

template <typename T, int V>
__device__ __forceinline__ void load_floats(const T* p, float (&out)[V])
{
    const Pack<T, V> a = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = to_float(a.v[i]);
}

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> pack_floats(const float (&in)[V])
{
    Pack<T, V> a;
#pragma unroll
    for (int i = 0; i < V; ++i) a.v[i] = from_float<T>(in[i]);
    return a;
}

// A store that goes past L2 (see stg4_nt) where STREAMING: neighbouring lanes write whole lines then.
template <bool STREAMING, typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& a)
{
    if constexpr (STREAMING && sizeof(T) * V == 16) __builtin_nontemporal_store(__builtin_bit_cast(f32x4, a), reinterpret_cast<f32x4*>(p));
    else *reinterpret_cast<Pack<T, V>*>(p) = a;
}
// f(std::true_type{}) or f(std::false_type{}): a loop of its own for each (in one loop the compiler makes the two stores one, an ordinary one).
template <typename F>
__device__ __forceinline__ void by_streaming(bool streaming, F f)
{
    if (streaming) f(std::true_type{});
    else f(std::false_type{});
}

template <typename T, int V>
__device__ __forceinline__ void store_floats(T* p, const float (&in)[V])
{
    *reinterpret_cast<Pack<T, V>*>(p) = pack_floats<T, V>(in);
}

// An element of a vector whose type is known at run time only (norm parameters: a few per thread).
__device__ __forceinline__ float load_any(const void* p, int64_t i, int dtype)
{
    return dtype == ANR_F32 ? static_cast<const float*>(p)[i] : dtype == ANR_F16 ? (float)static_cast<const half_t*>(p)[i] : (float)static_cast<const bf16_t*>(p)[i];
}
__device__ __forceinline__ void store_any(void* p, int64_t i, int dtype, float v)
{
    if (dtype == ANR_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == ANR_F16) static_cast<half_t*>(p)[i] = (half_t)v;
    else static_cast<bf16_t*>(p)[i] = (bf16_t)v;
}

// Sigmoid.  QUICK: by the hardware's exponential and reciprocal, whose relative error of about 2^-21 for |z| < 16 (it grows
// with |z|, the argument being rounded) is far below a rounding to 16 bits; else by the library's, for float32.
template <bool QUICK>
__device__ __forceinline__ float sigmoid(float z)
{
    if (QUICK) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z));
    return 1.f / (1.f + expf(-z));
}

// Phi(z), and exp(-z^2 / 2), from one exponential.  What lies beyond a = |z| is exp(-a^2 / 2) t P(t), t = 1 / (1 + 0.308 a), with the polynomial
// of six terms that is least off over [0, 14] relative to the result, 4e-6: QUICK, a 120th of a rounding to float16 wherever z is (formula 7.1.26 of Abramowitz
// and Stegun, whose 1.5e-7 is of 1, was off by 1.6e-3 of it at -4 and 3.6e-3 at -5, which reaches a product with a large up).  Else, for float32, it is
// to 10 u of itself (u = 2^-24) and z^2 / 4 more below -1 for the rounding of the exponential's argument: within a unit of zero as 0.5 + z P(z^2), otherwise
// by P(1 - 2 k t) with t = 1 / (a + k), k = 3.58, polynomials of least relative error over [1, 14] (1 u) and [0, 1].
// 0.5 (1 + erf), which has few bits left below -4 and none below -6, took longer: norm backward, 4 x 128^2 x 256, 69.9 us, so 68.2, with erfc 77.9;
// forward 39.4, 39.3, 42.1, but 8 x 56^2 x 320 24.1, 25.0, 26.8.
template <bool QUICK>
__device__ __forceinline__ float normal_below(float z, float& bell)
{
    const float a = fabsf(z);
    if (!QUICK) {
        const float w = z * z;
        bell = expf(-0.5f * w);
        const float middle = fmaf(z, fmaf(w, fmaf(w, fmaf(w, fmaf(w, fmaf(w, -7.65420373e-6f, 1.13486356e-4f), -1.18632987e-3f), 9.97332297e-3f), -0.0664903596f), 0.398942292f), 0.5f);
        const float t = __builtin_amdgcn_rcpf(a + 3.58f), q = fmaf(-7.16f, t, 1.f);
        const float tail = fmaf(q, fmaf(q, fmaf(q, fmaf(q, fmaf(q, fmaf(q, -0.00334144803f, 0.00508789485f), 0.0234102663f), -0.127396584f), 0.327804804f), -0.573150635f), 0.746405363f) * t * bell;
        return a < 1.f ? middle : z > 0.f ? 1.f - tail : tail;             // (a NaN's tail is one)
    }
    bell = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.308f, a, 1.f));
    const float tail = bell * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.0754302591f, 0.189618751f), 0.00727212941f), 0.136533991f), 0.118881121f), 0.123122714f);
    return z > 0.f ? 1.f - tail : tail;                                    // (a NaN's tail is one)
}

constexpr float kTwoRootTwoOverPi = 1.59576912160573071f;      // 2 sqrt(2 / pi)
constexpr float kOneOverRootTwoPi = 0.39894228040143268f;

// act(z).
template <int ACT, bool QUICK>
__device__ __forceinline__ float activation(float z)
{
    if (ACT == ANR_ACT_RELU) return z < 0.f ? 0.f : z;                     // (a NaN stays one)
    if (ACT == ANR_ACT_SILU) return z * sigmoid<QUICK>(z);
    if (ACT == ANR_ACT_GELU) {
        float bell;
        return z * normal_below<QUICK>(z, bell);
    }
    if (ACT == ANR_ACT_GELU_TANH) return z * sigmoid<QUICK>(kTwoRootTwoOverPi * fmaf(0.044715f * z * z, z, z));
    return z;
}

// act(z) and act'(z).  A factor of zero takes what it multiplies with it, also where that has overflowed.
template <int ACT, bool QUICK>
__device__ __forceinline__ float activation_and_slope(float z, float& slope)
{
    slope = 1.f;
    if (ACT == ANR_ACT_RELU) {
        slope = z > 0.f ? 1.f : z <= 0.f ? 0.f : z;                        // (a NaN stays one)
        return z < 0.f ? 0.f : z;
    }
    if (ACT == ANR_ACT_SILU) {
        const float s = sigmoid<QUICK>(z);
        slope = s * fmaf(__builtin_amdgcn_fmed3f(z, -128.f, 128.f), 1.f - s, 1.f);     // (s is 0 or 1 where z is cut)
        return z * s;
    }
    if (ACT == ANR_ACT_GELU) {
        float bell;
        const float phi = normal_below<QUICK>(z, bell), density = kOneOverRootTwoPi * bell;
        slope = density == 0.f ? phi : fmaf(z, density, phi);
        return z * phi;
    }
    if (ACT == ANR_ACT_GELU_TANH) {
        const float s = sigmoid<QUICK>(kTwoRootTwoOverPi * fmaf(0.044715f * z * z, z, z)), both = s * (1.f - s);
        slope = both == 0.f ? s : fmaf(both * z, kTwoRootTwoOverPi * fmaf(3.f * 0.044715f * z, z, 1.f), s);
        return z * s;
    }
    return z;
}

// f(std::integral_constant<int, ACT>) for the activation of a descriptor.
template <typename F>
inline auto with_activation(int act, F f)
{
    switch (act) {
        case ANR_ACT_RELU: return f(std::integral_constant<int, ANR_ACT_RELU>{});
        case ANR_ACT_SILU: return f(std::integral_constant<int, ANR_ACT_SILU>{});
        case ANR_ACT_GELU: return f(std::integral_constant<int, ANR_ACT_GELU>{});
        case ANR_ACT_GELU_TANH: return f(std::integral_constant<int, ANR_ACT_GELU_TANH>{});
        default: return f(std::integral_constant<int, ANR_ACT_NONE>{});
    }
}

// f(std::integral_constant<int, ACT>) on the device.
template <typename F>
__device__ __forceinline__ void device_activation(int act, F f)
{
    switch (act) {
        case ANR_ACT_RELU: f(std::integral_constant<int, ANR_ACT_RELU>{}); break;
        case ANR_ACT_SILU: f(std::integral_constant<int, ANR_ACT_SILU>{}); break;
        case ANR_ACT_GELU: f(std::integral_constant<int, ANR_ACT_GELU>{}); break;
        case ANR_ACT_GELU_TANH: f(std::integral_constant<int, ANR_ACT_GELU_TANH>{}); break;
        default: f(std::integral_constant<int, ANR_ACT_NONE>{}); break;
    }
}

// f(T{}) for the element type of a descriptor.
template <typename F>
inline auto with_type(int dtype, F f)
{
    switch (dtype) {
        case ANR_F16: return f(half_t{});
        case ANR_BF16: return f(bf16_t{});
        default: return f(float{});
    }
}

constexpr int element_bytes(int dtype) { return dtype == ANR_F32 ? 4 : 2; }

}  // namespace anr
