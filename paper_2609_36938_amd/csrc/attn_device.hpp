// Device-side helpers shared by the attention kernels.
#pragma once

#include "janus_device.hpp"

namespace janus {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

JANUS_DEV v8bf as_v8bf(v4i x) { return __builtin_bit_cast(v8bf, x); }

constexpr float RESCALE_SLACK = 8.0f;           // log2 headroom before O is rescaled
// Running max before any valid logit: finite and below every logit, so that
// the rescale test needs no special case and exp2(x - m) of a padding key
// (x = -inf) is 0.
constexpr float M_INIT = -3.0e38f;

typedef short v4s16 __attribute__((ext_vector_type(4)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

// Four consecutive outputs at element `at` of out (fp32, or rounded to bf16),
// in one store whatever out's alignment.
typedef v4f v4f_any __attribute__((aligned(4)));
typedef v2i v2i_any __attribute__((aligned(2)));
JANUS_DEV void store_out4(void *out, int out_f32, int64_t at, v4f v)
{
    if (out_f32)
        *(v4f_any *)((float *)out + at) = v;
    else
        *(v2i_any *)((uint16_t *)out + at) = __builtin_bit_cast(v2i, __builtin_convertvector(v, v4bf));
}

// s_waitcnt immediate (gfx9 encoding) that waits for vmcnt <= n only.
constexpr int vmcnt_only(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }

// Workgroup barrier over LDS that leaves the tile gathers in flight: this
// wave's LDS operations are complete (lgkmcnt 0), the compiler may move no
// memory access across it, and no fence drains the outstanding loads.
JANUS_DEV void lds_barrier()
{
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) v4s16 lds_v4s16;

// The lane id made inside the code that uses it: the compiler can neither
// hoist it out of a rarely taken branch nor keep it live (and spill it)
// across the tile loop.
JANUS_DEV int lane_here()
{
    int ln;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(ln));
    return ln;
}

// Transposing LDS read (ds_read_b64_tr_b16): within each 16-lane group,
// lane i's element j is element i%4 of the 8 bytes addressed by lane 4j+i/4.
JANUS_DEV v4s16 lds_read_tr16(const uint8_t *lds_base, int byte_off)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_v4s16 *)((__attribute__((address_space(3))) uint8_t *)lds_base + byte_off));
}

// One 16-byte-per-lane gather into LDS (global_load_lds_dwordx4: lane l's
// 16 bytes from src land at dst + 16 l), written as assembly so that the
// compiler does not wait for every outstanding LDS read at the next use of
// any of them, as it does after the builtin.  M0 holds the LDS address (one
// wait state before the load reads it) and is restored afterwards.
JANUS_DEV void gather16(const uint8_t *src, uint8_t *dst)
{
    const uint32_t m = (uint32_t)(uintptr_t)(lds_void *)dst;
    int saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\t"
                 "s_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "s"(m), "v"(src)
                 : "memory");
}

// The same from a wave-uniform address and a byte offset per lane.
JANUS_DEV void gather16(const uint8_t *base, uint32_t off, uint8_t *dst)
{
    const uint32_t m = (uint32_t)(uintptr_t)(lds_void *)dst;
    int saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\t"
                 "s_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "s"(m), "v"(off), "s"(base)
                 : "memory");
}

} // namespace janus
