// Tiles of rows in LDS that are read both ways -- rows as they are, and transposed -- and what kernels that gather such
// rows share: the workgroups' order, direct-to-LDS copies with an address per lane, LDS reads by address.
#pragma once
#include "attn_tile.h"

namespace adaspark {

// Workgroup -> (KV head, slot among the head's workgroups).  Consecutive workgroups go to different XCDs, each with
// its own L2; the workgroups of one KV head stream the same tiles, so where the head count allows a head's
// workgroups stay on as few XCDs as possible.  head_grid is the matching launch size.
__host__ __device__ inline bool head_slot(int b, int Hkv, int per_head, int &kv, int &slot)
{
    if (Hkv <= 8 && 8 % Hkv == 0) {
        const int x = b & 7, idx = b >> 3, share = 8 / Hkv;
        kv = x % Hkv;
        slot = idx * share + x / Hkv;
    } else if (Hkv % 8 == 0) {
        const int x = b & 7, idx = b >> 3, m = Hkv / 8;
        kv = x + 8 * (idx % m);
        slot = idx / m;
    } else {
        kv = b % Hkv;
        slot = b / Hkv;
    }
    return slot < per_head;
}
inline unsigned head_grid(int Hkv, int per_head)
{
    if (Hkv <= 8 && 8 % Hkv == 0) return (unsigned)((per_head + 8 / Hkv - 1) / (8 / Hkv) * 8);
    return (unsigned)per_head * (unsigned)Hkv;
}

// Inclusive scan over a wavefront's lanes, without LDS: within rows of 16, then each row's sum carried on.
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

// Direct-to-LDS copies with an address per lane: lane l moves the 16 (4) bytes at src to lds_addr + 16 * l (4 * l).
__device__ __forceinline__ void dma_lane16(uint32_t lds_addr, const void *src)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_addr), "v"(src) : "memory", "m0");
}
__device__ __forceinline__ void dma_lane4(uint32_t lds_addr, const void *src)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds_addr), "v"(src) : "memory", "m0");
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Slot of 16-byte chunk c of tile row r.  An LDS line is 16 slots: one row of head-dim 128, two of 64.  A ds_read_b128 of 64 lanes is served
// 16 lanes at a time, lanes 0-3, 12-15, 20-27 first: with the chunk index equal in 0-15 and one higher in 16-31, the
// lines' swizzle values must be distinct and those of rows 4..11 closed under ^ 1.  A transposing read is served 32
// lanes at a time, 8 rows at two neighbouring chunks: their values must differ above bit 0 (measured: 241 bytes per
// clock for both kinds; a plain row number gives 227 and 122).
template <int D>
__device__ __forceinline__ int row_swizzle(int r)
{
    if (D == 128) return (((r & 7) ^ (((r >> 3) & 1) << 2)) << 1) | ((r >> 3) & 1);
    const int line = r >> 1;
    return (((line & 3) ^ (((line >> 2) & 1) << 1)) << 1) | ((line >> 2) & 1);
}
template <int D>
__device__ __forceinline__ int row_tile_off(int r, int c)
{
    if (D == 128) return r * 256 + ((c ^ row_swizzle<D>(r)) << 4);
    return (r >> 1) * 256 + (((((r & 1) << 3) | c) ^ row_swizzle<D>(r)) << 4);
}

// LDS reads by address.
template <typename T>
__device__ __forceinline__ T lds_read(uint32_t addr)
{
    return *reinterpret_cast<const __attribute__((address_space(3))) T *>(addr);
}
// Two transposing reads, `step` bytes apart.  In each, lane (n16, q4) gets the elements at column n16 of the four
// 16-element row pieces that lanes 16 q4 .. 16 q4 + 15 point to (lane 4 k + m of them: 8 bytes, elements 4 m .. 4 m + 3 of
// row k).
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ bf16x8 lds_read_tr2(uint32_t addr, int step)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>(addr));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>(addr + step));
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

}  // namespace adaspark
