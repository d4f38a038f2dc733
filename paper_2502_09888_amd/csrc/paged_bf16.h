// Pieces that the bf16 kernels of the paged cache share (internal): operand types, rows in LDS and their fragments.
#pragma once
#include "lanes.h"
#include "paged.h"

namespace climber {
namespace paged {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef const __attribute__((address_space(1))) uint8_t glb_u8;

static __device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }
static __device__ __forceinline__ float half_max(float x)
{
    const unsigned u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Rows of D bf16 in LDS: 16-byte piece c of row r at slot c ^ f(r).  f takes 16 consecutive rows (key fragments: 16 lanes read one
// piece each) to 16 places of the 64 banks, and 4 consecutive ones (value fragments: 4 pieces of each) to 4 different quarters.
template <int D>
struct Rows {
    static constexpr int kPitch = 2 * D, kPieces = D / 8, kPerLoad = 64 / kPieces, kLoads = 16 / kPerLoad;  // (of 16 rows)
    static __device__ __forceinline__ int f(int r)
    {
        return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    }
    uint32_t k_at[D / 16], v_at[2][D / 32];
    __device__ __forceinline__ void init(int lane)
    {
        const int l32 = lane & 31, hf = lane >> 5, G = lane >> 4, i16 = lane & 15;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) k_at[s] = l32 * kPitch + ((2 * s + hf) ^ f(l32)) * 16;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
                const int r = 8 * hh + 4 * (G >> 1) + (i16 >> 2), c = 4 * db + 2 * (G & 1) + ((i16 >> 1) & 1);
                v_at[hh][db] = r * kPitch + (c ^ f(r)) * 16 + 8 * (i16 & 1);
            }
    }
};

// Fragments of 32 key rows, and of the 16 value rows from `base` on (A operands of the D / 32 blocks of dimensions).
template <int D>
struct KFrags { bf16x8 a[D / 16]; };
template <int D>
static __device__ __forceinline__ KFrags<D> read_k(const Rows<D> &w, const lds_u8 *base)
{
    KFrags<D> f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) f.a[s] = *(const __attribute__((address_space(3))) bf16x8 *)(base + w.k_at[s]);
    return f;
}
template <int D>
struct VFrags { u32x4 a[D / 32]; };
template <int D>
static __device__ __forceinline__ VFrags<D> read_v(const Rows<D> &w, lds_u8 *base)
{
    VFrags<D> f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(base + w.v_at[0][db])));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(base + w.v_at[1][db])));
        f.a[db] = u32x4{lo.x, lo.y, hi.x, hi.y};
    }
    return f;
}

static __device__ __forceinline__ bf16x8 frag(u32x4 x) { return __builtin_bit_cast(bf16x8, x); }

// 16 bytes a lane from anywhere to LDS, 1 KiB in a row
static __device__ __forceinline__ void copy16(glb_u8 *from, lds_u8 *to) { __builtin_amdgcn_global_load_lds(from, to, 16, 0, 0); }

}  // namespace paged
}  // namespace climber
