// Device helpers shared by the attention kernels: 16-byte pieces and matrix operands, weights as exponentials, rows staged in LDS,
// results that pass from one workgroup of a launch to another.
#pragma once

#include "mukv_internal.h"

namespace mukv {

typedef __attribute__((ext_vector_type(4))) unsigned int raw16; // 16 bytes as they come from memory
template <typename T>
__device__ __forceinline__ raw16 load16(const T *p) {
    return *reinterpret_cast<const raw16 *>(p);
}

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(8))) short i16x8;
// two floats as bf16, x below y: the conversion instruction rounds to nearest even and keeps NaN a NaN
__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
}
__device__ __forceinline__ void store_out(uint16_t *p, float x) { *p = (uint16_t)bf16_pair(x, 0.f); }
__device__ __forceinline__ void store_out(float *p, float x) { *p = x; }
// ds_read_b64_tr_b16, the LDS transpose read of 16-bit elements: every lane names 8 bytes; within each block
// of 16 lanes, result[t] of lane i is element i % 4 of the 8 bytes named by lane 4 * t + i / 4 of the block,
// t = 0..3 (lane layout checked by an in-bounds probe on the device).
__device__ __forceinline__ i16x4 lds_read_tr16(const unsigned char *p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((i16x4 __attribute__((address_space(3))) *)(p));
}

// Slot of 16-byte piece x of staged row `row`: x ^ row_swizzle.  The transpose reads of half a wave take two neighbouring
// pieces of eight neighbouring rows: 256 bytes over all banks.
template <int D>
__device__ __forceinline__ int row_swizzle(int row) {
    return ((row / (128 / D)) & (D / 16 - 1)) << 1;
}

// attend_kernel and prefill_colsum_kernel, fp32 rows and bf16 rows of 16: the queries are brought down before the product by a
// power of two, exactly, to where a score that is finite once scaled by log2(e) / sqrt(D) does not overflow before.
template <typename T, int D>
constexpr float query_factor() {
    return sizeof(T) == 2 && D > 16 ? 1.f : D <= 32 ? 0.25f : 0.125f; // (D = 16 .. 128: the scale is 0.361, 0.255, 0.180, 0.128)
}
template <typename T, int D>
__device__ __forceinline__ raw16 brought_down(raw16 x) {
    constexpr float f = query_factor<T, D>();
    if constexpr (f != 1.f)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4)
                x[e] = __float_as_uint(__uint_as_float(x[e]) * f);
            else
                x[e] = __float_as_uint(__uint_as_float(x[e] << 16) * f) >> 16 | (__float_as_uint(__uint_as_float(x[e] & 0xFFFF0000u) * f) & 0xFFFF0000u);
        }
    return x;
}

// x * s - y with the product rounded, as the maximum y was.
__device__ __forceinline__ float scaled_apart(float x, float s, float y) {
#pragma clang fp contract(off)
    const float p = x * s;
    return p - y;
}

// 2^(x s - ref), ref a whole number.  The difference itself would be rounded at its own size, so the whole number nearest to
// x s goes to the weight's exponent, exactly, and at most a half through the exponential.
__device__ __forceinline__ float weight_of(float x, float s, float ref) {
    const float n = fmaxf(rintf(x * s), ref - 256.f); // (a masked score is -inf, its weight 0)
    return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(fmaf(x, s, -n)), (int)(n - ref));
}

constexpr float kLargeRef = 16777216.f; // whole numbers up to here have no gaps
// The same for references of any size.
__device__ __forceinline__ float weight_of_any(float x, float s, float ref) {
    return fabsf(ref) > kLargeRef ? __builtin_amdgcn_exp2f(scaled_apart(x, s, ref)) : weight_of(x, s, ref);
}

// Two floats that another workgroup of the launch reads: written through to, and read from, the memory that all XCDs share.
__device__ __forceinline__ void store_far(float *p, float x, float y) {
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), __builtin_bit_cast(uint64_t, f32x2{x, y}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_far(const float *p) {
    return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
// The last of n workgroups to get here, all of whose store_far's are then there to be read, by every thread.  The arrival that makes
// n sets the count back to zero in the same step, so none is lost between the two.
__device__ __forceinline__ bool last_to_arrive(int *count, int n, int *s_last) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // this wave's stores are in the shared memory
    __syncthreads();                                 // every wave's are
    if (threadIdx.x == 0)
        *s_last = __builtin_amdgcn_atomic_inc32(reinterpret_cast<uint32_t *>(count), (uint32_t)(n - 1), __ATOMIC_RELAXED, "agent") == (uint32_t)(n - 1);
    __syncthreads();
    return *s_last != 0;
}

// The direct global -> LDS load: 16 bytes per lane from the lane's address to dst + 16 * lane (dst is the same in all
// lanes).  The instruction has no destination register, only addresses, which are read when it issues.  It is not the
// builtin because the compiler makes every later LDS read wait for that one, which would end the overlap of a step's
// loads with the step before: here rows_landed() and a barrier stand between a load and the first read of its rows.
__device__ __forceinline__ void load_to_lds(const unsigned char *src, unsigned char *dst) {
    const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)dst;
    unsigned saved; // m0, which carries the LDS address, is left as it was
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "s"(base), "v"(src)
                 : "memory");
}
__device__ __forceinline__ void load4_to_lds(const float *src, float *dst) { // 4 bytes per lane
    const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) float *)dst;
    unsigned saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "s"(base), "v"(src)
                 : "memory");
}
__device__ __forceinline__ void rows_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// over the two lanes lane % 32 and lane % 32 + 32, result in both
__device__ __forceinline__ float half_max(float v) {
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Slot of 16-byte piece `piece` of staged row `row` in a row of D * 2 bytes.
template <int D>
__device__ __forceinline__ int key_slot(int piece, int row) {
    // 16 lanes read one piece of 16 neighbouring rows: 256 B over all banks
    return D == 128 ? piece ^ (row & 15) : piece ^ ((row >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int val_slot(int piece, int row) {
    // half a wave reads 4 pieces of 4 neighbouring rows (4-aligned both)
    return D == 128 ? piece ^ (((row & 3) << 2) | ((row >> 2) & 3)) : piece ^ (((row >> 1) & 1) << 2);
}

// inclusive sum over the lanes up to this one
__device__ __forceinline__ int wave_prefix(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false); // within the 16 lanes of a row
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false); // the row before, in rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false); // the half before, in the upper half
    return v;
}

} // namespace mukv
