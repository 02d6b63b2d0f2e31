// What the operator kernels share: element types, eight elements of a row at a time, sums over a
// wavefront, the dropout mask, the launch.
#ifndef VMS_OPS_COMMON_HPP
#define VMS_OPS_COMMON_HPP
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/vms_ops.h"
#include "wave_hw.hpp"

typedef _Float16 f16;
typedef __bf16 bf16;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements.  Rows may start at any element, so the access asks for no more than an
// element's alignment: global memory takes 16-byte accesses at any address on this target, and one
// instruction for eight elements is what counts here, not where a line begins.
template <class T>
struct Eight {
    typedef T type __attribute__((ext_vector_type(8)));
    typedef type loose __attribute__((aligned(sizeof(T))));
};

// The elements at p, 0 beyond the first n.  ONCE: they are not read again before the caches have been filled with other
// data, and should not take the place of what is (passes_by below).
template <bool ONCE = false, class T>
DI typename Eight<T>::type load8_raw(const T *p, u32 n)
{
    const auto *const from = reinterpret_cast<const typename Eight<T>::loose *>(p);
    if (LIKELY(n >= 8)) return ONCE ? __builtin_nontemporal_load(from) : *from;
    typename Eight<T>::type x;
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = (u32)i < n ? p[i] : (T)0.f;
    return x;
}
template <bool ONCE = false, class T>
DI void load8(const T *p, u32 n, float v[8])
{
    const typename Eight<T>::type x = load8_raw<ONCE>(p, n);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (float)x[i];
}

// the first n of v[0..7], rounded to the type (to nearest, ties to even), to p
template <bool ONCE = false, class T>
DI void store8(T *p, u32 n, const float v[8])
{
    if (LIKELY(n >= 8)) {
        typename Eight<T>::type x;
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = (T)v[i];
        auto *const to = reinterpret_cast<typename Eight<T>::loose *>(p);
        if (ONCE)
            __builtin_nontemporal_store(x, to);
        else
            *to = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if ((u32)i < n) p[i] = (T)v[i];
    }
}

template <int CTRL, int ROWS>
DI float dpp_add(float v)
{
    return v + __uint_as_float((u32)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROWS, 0xF, false));
}

// sum over the 64 lanes, the same for all of them; always in the same order
DI float wave_sum(float v)
{
    v = dpp_add<DPP_QUAD_XOR1, 0xF>(v);
    v = dpp_add<DPP_QUAD_XOR2, 0xF>(v);
    v = dpp_add<DPP_ROW_HALF_MIRROR, 0xF>(v);
    v = dpp_add<DPP_ROW_MIRROR, 0xF>(v);
    v = dpp_add<DPP_ROW_BCAST15, 0xA>(v);
    v = dpp_add<DPP_ROW_BCAST31, 0xC>(v);
    return __uint_as_float(from_lane(__float_as_uint(v), 63));
}

// sum over the 16 lanes of a row, the same for all of them
DI float row16_sum(float v)
{
    v = dpp_add<DPP_QUAD_XOR1, 0xF>(v);
    v = dpp_add<DPP_QUAD_XOR2, 0xF>(v);
    v = dpp_add<DPP_ROW_HALF_MIRROR, 0xF>(v);
    return dpp_add<DPP_ROW_MIRROR, 0xF>(v);
}

// A dropout mask as the kernels take it; limit 0: nothing is dropped and no number drawn.
struct Mask {
    u64 seed;
    const u64 *d_seed;
    u64 call;
    u32 limit;          // dropped: numbers below it (65536: everything)
    float scale;        // of what is kept
};

inline int make_mask(const vms_dropout_mask &m, Mask *out)
{
    if (!(m.p >= 0.0 && m.p <= 1.0)) return VMS_EINVAL;
    if ((uintptr_t)m.d_seed % 8) return VMS_EINVAL;
    out->seed = m.seed;
    out->d_seed = m.d_seed;
    out->call = m.call;
    out->limit = (u32)floor(m.p * 65536.0 + 0.5);
    out->scale = out->limit < 65536 ? (float)(65536.0 / (65536.0 - out->limit)) : 0.f;
    return VMS_OK;
}

// Philox-4x32, ten rounds: four words for the counter (c0, c1, c2, c3) under the key (k0, k1).  Two
// 32 x 32 -> 64 bit products a round; at 16 bits for an element eight elements share the 20 products.
DI void philox(u32 c0, u32 c1, u32 c2, u32 c3, u32 k0, u32 k1, u32 w[4])
{
#pragma unroll
    for (int r = 0; r < 10; r++) {
        const u64 p0 = (u64)0xD2511F53u * c0, p1 = (u64)0xCD9E8D57u * c2;
        c0 = (u32)(p1 >> 32) ^ c1 ^ k0;
        c2 = (u32)(p0 >> 32) ^ c3 ^ k1;
        c1 = (u32)p1;
        c3 = (u32)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0;
    w[1] = c1;
    w[2] = c2;
    w[3] = c3;
}

DI u64 mask_seed(const Mask &m) { return m.d_seed ? *m.d_seed : m.seed; }

// v[0..7] = dropout of the eight elements of column group `group` (column / 8) of a row.  What is dropped becomes 0
// whatever it was, infinities and NaN included.
DI void drop8(const Mask &m, u64 seed, u32 row, u32 group, float v[8])
{
    u32 w[4];
    philox(group, row, (u32)m.call, (u32)(m.call >> 32), (u32)seed, (u32)(seed >> 32), w);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const u32 u = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu;
        v[i] = u >= m.limit ? v[i] * m.scale : 0.f;
    }
}

// Workgroups go to the eight dies in turn, and each die has a cache of its own.  Where neighbours of a grid share memory
// lines or walk through neighbouring ones, they are numbered so that a die gets a run of them: the b-th of n.
DI u32 die_order(u32 b, u32 n)
{
    const u32 die = b % 8, each = n / 8, more = n % 8;
    return die * each + min(die, more) + b / 8;
}

const u32 OPS_CUS = 256;        // compute units of the device that the grids are sized for

// Does a call that reads and writes so many bytes leave nothing of them in the last cache (256 MiB)?  Then its accesses are
// marked as not to be kept: dropout of 8192 x 16384 in 16 bits, 537 MB, takes 90 us, 97 without the marks.  What just fills the
// cache is better left in it (4096 x 16384: 42 us, 45 with them), and a smaller call's output may be found there by the next
// kernel.
inline bool passes_by(u64 bytes) { return bytes > 256u << 20; }

template <class P>
int ops_launch(void (*kernel)(P), dim3 grid, dim3 block, u32 lds, const P &p, void *stream)
{
    P copy = p;
    void *args[] = { &copy };
    if (hipLaunchKernel((const void *)kernel, grid, block, args, lds, (hipStream_t)stream) == hipSuccess) return VMS_OK;
    (void)hipGetLastError();            // reported here, and not again by whoever asks next
    return VMS_EHIP;
}

// calls f with a null pointer of the element type; VMS_EINVAL for a type that does not exist
template <class F>
int with_type(u32 dtype, F f)
{
    switch (dtype) {
    case VMS_F32: return f((float *)nullptr);
    case VMS_F16: return f((f16 *)nullptr);
    case VMS_BF16: return f((bf16 *)nullptr);
    }
    return VMS_EINVAL;
}

inline size_t type_bytes(u32 dtype) { return dtype == VMS_F32 ? 4 : 2; }

// may p be the first element of a matrix with this type and stride?
inline bool input_ok(const void *p, u32 dtype) { return p && (uintptr_t)p % type_bytes(dtype) == 0; }
inline bool output_ok(const void *p, u32 dtype, u64 ld, u64 cols) { return input_ok(p, dtype) && ld >= cols; }
// strides that keep row * ld inside 63 bits
inline bool stride_ok(u64 ld) { return ld < (1ull << 31); }

#endif
