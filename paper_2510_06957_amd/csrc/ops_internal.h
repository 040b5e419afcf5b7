// Internal declarations shared by the operators around the ternary product (tst_ops.h).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "tst_ops.h"

namespace tst {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Geometry of packed 8-bit weights (tst_w8_pack): pieces of 16 columns x 64 rows.
constexpr int kW8Cols = 16, kW8Rows = 64, kW8Piece = kW8Cols * kW8Rows;
inline __host__ __device__ int blocks_of(int n, int size) { return n / size + (n % size != 0); }   // (n + size may pass 2^31)
inline size_t w8_bytes(int K, int N) { return (size_t)blocks_of(K, kW8Rows) * blocks_of(N, kW8Cols) * kW8Piece; }
constexpr int kW8MaxK = 131071;   // 131072 * (-128 * -128) = 2^31

inline bool type_ok(int type) { return type == TST_F32 || type == TST_BF16 || type == TST_F16; }
inline size_t type_bytes(int type) { return type == TST_F32 ? 4 : 2; }
inline bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// An entry of a type: bf16 and fp16 held as their 16 bits.
template <int TYPE> struct Entry;
template <> struct Entry<TST_F32> {
    typedef float bits;
    static __device__ __forceinline__ float get(bits b) { return b; }
    static __device__ __forceinline__ bits put(float v) { return v; }
};
template <> struct Entry<TST_BF16> {
    typedef uint16_t bits;
    static __device__ __forceinline__ float get(bits b) { return __uint_as_float((unsigned)b << 16); }
    static __device__ __forceinline__ bits put(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }   // to nearest, ties to even
};
template <> struct Entry<TST_F16> {
    typedef uint16_t bits;
    static __device__ __forceinline__ float get(bits b) { return (float)__builtin_bit_cast(_Float16, b); }
    static __device__ __forceinline__ bits put(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

// The largest of a wavefront's values, the same in all lanes: maxima of 2, 4, 8, 16 neighbours, of rows of 16 and of halves, in lane 63.
__device__ __forceinline__ unsigned wave_max(unsigned v)
{
    auto step = [&](auto control) { return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, decltype(control)::value, 0xf, 0xf, false)); };
    v = step(std::integral_constant<int, 0x111>{});   // row_shr 1
    v = step(std::integral_constant<int, 0x112>{});
    v = step(std::integral_constant<int, 0x114>{});
    v = step(std::integral_constant<int, 0x118>{});
    v = step(std::integral_constant<int, 0x142>{});   // row_bcast 15
    v = step(std::integral_constant<int, 0x143>{});   // row_bcast 31
    return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}

// Orders a wavefront's own stores and reads in the LDS, which its lanes exchange without a meeting of the workgroup: the LDS takes them as
// they come, the compiler would be free to move them.
__device__ __forceinline__ void order_wave()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// Bits that order as floats do: NaN above everything, -0 as +0.  No float has 0.
__device__ __forceinline__ unsigned order_bits(float v)
{
    const unsigned u = __float_as_uint(v + 0.f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// The float of bits that are not a NaN's.
__device__ __forceinline__ float from_order_bits(unsigned b) { return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b); }

int compute_units();   // (tstgemm_side.hip)

// A dimension of a grid has fewer than 2^32 threads, and a launch with more goes through with what is left of their number in 32 bits: kernels
// with a workgroup of 256 for a row are launched for so many rows at a time.
constexpr int kLaunchRows = 1 << 22;

inline int status(hipError_t e) { return e == hipSuccess ? TSTGEMM_OK : TSTGEMM_EHIP; }

// call(std::integral_constant<int, type>) for a run-time type
template <typename F> inline hipError_t for_type(int type, F call)
{
    switch (type) {
    case TST_F32: return call(std::integral_constant<int, TST_F32>{});
    case TST_BF16: return call(std::integral_constant<int, TST_BF16>{});
    default: return call(std::integral_constant<int, TST_F16>{});
    }
}

}  // namespace tst
