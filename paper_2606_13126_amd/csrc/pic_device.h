// Device helpers shared by the kernels of libpic_attn (pic_kernels.hip, pic_tree.hip): bf16
// packing, K rotation, RoPE angles, work-group coordinates, LDS swizzles and copies.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pic_internal.h"

namespace pic {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

constexpr int kNeox = 0;
constexpr float kNegBig = -1.0e30f;  // finite "minus infinity" for running maxima

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Round two floats to bf16 (round to nearest even) and pack them, lo first.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    bf16x2_t v = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, v);
}

// (a.lo * b.lo + a.hi * b.hi) of two bf16 pairs, fp32 result.
__device__ __forceinline__ float dot2_bf16(uint32_t a, uint32_t b) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a), __builtin_bit_cast(bf16x2_t, b), 0.0f,
                                           false);
}

// ---------------------------------------------------------------------------------
// K rotation blocks.  A pair (x, y) turns into (x c - y s, y c + x s) as two
// 2-element dot products with the table entry e = (c, s): (x, y).(c, -s), the sign
// applied by the instruction's neg_hi modifier, and (y, x).(c, s).  The builtin
// dot product with a zero addend compiles to a v_mov of zero plus the accumulating
// VOP2 form (which has no modifiers); these blocks issue the VOP3P form with an
// inline-constant zero addend.  A DOT result read by another VALU instruction needs
// 3 wait states on gfx950, which the compiler cannot see inside inline assembly:
// each block orders its eight dot products before the four conversions that read
// them, so every result is read at least three instructions after it is written and
// no s_nop is needed.  Nothing outside a block reads a DOT result of the block.
// ---------------------------------------------------------------------------------
struct Words4 {
    uint32_t w[4];
};

// Rotate-half (NeoX) pairing, four pairs: A0/B0 hold elements (2m, 2m+1) of the two
// halves for one m, A1/B1 for the next; e0..e3 are the entries of those four pairs
// in order.  Returns the rotated A0, B0, A1, B1 (rounded to bf16, RNE).
__device__ __forceinline__ Words4 rot4_neox(uint32_t A0, uint32_t B0, uint32_t A1, uint32_t B1, uint32_t e0,
                                            uint32_t e1, uint32_t e2, uint32_t e3) {
    uint32_t p0, p1, p2, p3, q0, q1, q2, q3;
    float x0, y0, x1, y1, x2, y2, x3, y3;
    asm("v_perm_b32 %[p0], %[B0], %[A0], %[slo]\n\t"   // (x_2m, y_2m)
        "v_perm_b32 %[q0], %[A0], %[B0], %[slo]\n\t"   // (y_2m, x_2m)
        "v_perm_b32 %[p1], %[B0], %[A0], %[shi]\n\t"
        "v_perm_b32 %[q1], %[A0], %[B0], %[shi]\n\t"
        "v_perm_b32 %[p2], %[B1], %[A1], %[slo]\n\t"
        "v_perm_b32 %[q2], %[A1], %[B1], %[slo]\n\t"
        "v_perm_b32 %[p3], %[B1], %[A1], %[shi]\n\t"
        "v_perm_b32 %[q3], %[A1], %[B1], %[shi]\n\t"
        "v_dot2_f32_bf16 %[x0], %[p0], %[e0], 0 neg_hi:[0,1,0]\n\t"
        "v_dot2_f32_bf16 %[y0], %[q0], %[e0], 0\n\t"
        "v_dot2_f32_bf16 %[x1], %[p1], %[e1], 0 neg_hi:[0,1,0]\n\t"
        "v_dot2_f32_bf16 %[y1], %[q1], %[e1], 0\n\t"
        "v_dot2_f32_bf16 %[x2], %[p2], %[e2], 0 neg_hi:[0,1,0]\n\t"
        "v_dot2_f32_bf16 %[y2], %[q2], %[e2], 0\n\t"
        "v_dot2_f32_bf16 %[x3], %[p3], %[e3], 0 neg_hi:[0,1,0]\n\t"
        "v_dot2_f32_bf16 %[y3], %[q3], %[e3], 0\n\t"
        "v_cvt_pk_bf16_f32 %[A0], %[x0], %[x1]\n\t"
        "v_cvt_pk_bf16_f32 %[B0], %[y0], %[y1]\n\t"
        "v_cvt_pk_bf16_f32 %[A1], %[x2], %[x3]\n\t"
        "v_cvt_pk_bf16_f32 %[B1], %[y2], %[y3]"
        : [A0] "+v"(A0), [B0] "+v"(B0), [A1] "+v"(A1), [B1] "+v"(B1), [p0] "=&v"(p0), [p1] "=&v"(p1),
          [p2] "=&v"(p2), [p3] "=&v"(p3), [q0] "=&v"(q0), [q1] "=&v"(q1), [q2] "=&v"(q2), [q3] "=&v"(q3),
          [x0] "=&v"(x0), [y0] "=&v"(y0), [x1] "=&v"(x1), [y1] "=&v"(y1), [x2] "=&v"(x2), [y2] "=&v"(y2),
          [x3] "=&v"(x3), [y3] "=&v"(y3)
        : [e0] "v"(e0), [e1] "v"(e1), [e2] "v"(e2), [e3] "v"(e3), [slo] "s"(0x05040100u), [shi] "s"(0x07060302u));
    return Words4{{A0, B0, A1, B1}};
}

// Interleaved (GPT-J) pairing, four pairs: w_i holds the pair (x, y) itself.
__device__ __forceinline__ Words4 rot4_gptj(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, uint32_t e0,
                                            uint32_t e1, uint32_t e2, uint32_t e3) {
    uint32_t q0, q1, q2, q3;
    float x0, y0, x1, y1, x2, y2, x3, y3;
    asm("v_alignbit_b32 %[q0], %[w0], %[w0], 16\n\t"   // (y, x)
        "v_alignbit_b32 %[q1], %[w1], %[w1], 16\n\t"
        "v_alignbit_b32 %[q2], %[w2], %[w2], 16\n\t"
        "v_alignbit_b32 %[q3], %[w3], %[w3], 16\n\t"
        "v_dot2_f32_bf16 %[x0], %[w0], %[e0], 0 neg_hi:[0,1,0]\n\t"
        "v_dot2_f32_bf16 %[y0], %[q0], %[e0], 0\n\t"
        "v_dot2_f32_bf16 %[x1], %[w1], %[e1], 0 neg_hi:[0,1,0]\n\t"
        "v_dot2_f32_bf16 %[y1], %[q1], %[e1], 0\n\t"
        "v_dot2_f32_bf16 %[x2], %[w2], %[e2], 0 neg_hi:[0,1,0]\n\t"
        "v_dot2_f32_bf16 %[y2], %[q2], %[e2], 0\n\t"
        "v_dot2_f32_bf16 %[x3], %[w3], %[e3], 0 neg_hi:[0,1,0]\n\t"
        "v_dot2_f32_bf16 %[y3], %[q3], %[e3], 0\n\t"
        "v_cvt_pk_bf16_f32 %[w0], %[x0], %[y0]\n\t"
        "v_cvt_pk_bf16_f32 %[w1], %[x1], %[y1]\n\t"
        "v_cvt_pk_bf16_f32 %[w2], %[x2], %[y2]\n\t"
        "v_cvt_pk_bf16_f32 %[w3], %[x3], %[y3]"
        : [w0] "+v"(w0), [w1] "+v"(w1), [w2] "+v"(w2), [w3] "+v"(w3), [q0] "=&v"(q0), [q1] "=&v"(q1),
          [q2] "=&v"(q2), [q3] "=&v"(q3), [x0] "=&v"(x0), [y0] "=&v"(y0), [x1] "=&v"(x1), [y1] "=&v"(y1),
          [x2] "=&v"(x2), [y2] "=&v"(y2), [x3] "=&v"(x3), [y3] "=&v"(y3)
        : [e0] "v"(e0), [e1] "v"(e1), [e2] "v"(e2), [e3] "v"(e3));
    return Words4{{w0, w1, w2, w3}};
}

// Two rotate-half pairs (elements 2m and 2m+1 of both halves) in plain float32
// arithmetic, for a kernel that is bound by memory and leaves the schedule to the
// compiler.  (The attention kernels rotate by dot products: the FMA form has 8 vector
// instructions more per pair and cost prefill_bf16 2% on 16 tails over 4,096 keys.)
__device__ __forceinline__ void rot2_fma(uint32_t& A, uint32_t& B, uint32_t e0, uint32_t e1) {
    const float x0 = bf_lo(A), x1 = bf_hi(A), y0 = bf_lo(B), y1 = bf_hi(B);
    const float c0 = bf_lo(e0), s0 = bf_hi(e0), c1 = bf_lo(e1), s1 = bf_hi(e1);
    A = pack_bf16(__builtin_fmaf(x0, c0, -(y0 * s0)), __builtin_fmaf(x1, c1, -(y1 * s1)));
    B = pack_bf16(__builtin_fmaf(y0, c0, x0 * s0), __builtin_fmaf(y1, c1, x1 * s1));
}

// One key's share of 2 PW pairs: NeoX x and y runs, GPT-J the pairs in order.
template <int STYLE, int PW>
__device__ __forceinline__ void rotate_runs(uint32_t (&k)[2][PW], const uint32_t* cs) {
    if (STYLE == kNeox) {
#pragma unroll
        for (int i = 0; i < PW; ++i) rot2_fma(k[0][i], k[1][i], cs[2 * i], cs[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 2 * PW; ++i) {
            uint32_t& w = k[i / PW][i % PW];
            const float x = bf_lo(w), y = bf_hi(w), c = bf_lo(cs[i]), sn = bf_hi(cs[i]);
            w = pack_bf16(__builtin_fmaf(x, c, -(y * sn)), __builtin_fmaf(y, c, x * sn));
        }
    }
}

// (a.lo, b.lo) and (a.hi, b.hi) of two bf16 pairs: the rotate-half pairing brings
// element i of one 8-dim run together with element i of the run half a head
// further; one byte permute each (bytes 0-3 of the selector pick from a, 4-7 from b)
__device__ __forceinline__ uint32_t pair_lo(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t pair_hi(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// c + a.lo + a.hi for a pair of bf16 values (a dot product with (1, 1), one
// accumulate-in-place instruction)
__device__ __forceinline__ float sum2_bf16(uint32_t a, float c) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), c,
                                           false);
}

// ---------------------------------------------------------------------------------
// RoPE angles.  Pair i turns by p * omega_i.  The angle is kept as a 64-bit binary
// fraction of a revolution, F_i = frac(omega_i / 2pi) scaled by 2^64 (computed on
// the host from theta, or from explicit frequencies), so p * F_i (mod 2^64) is the
// exact phase of any int32 position (negative ones included) up to the rounding of
// F_i; sin/cos then only see a reduced argument in [-0.5, 0.5) revolutions.  A pair
// with F_i = 0 (past a partial rotary width) turns by nothing.
// ---------------------------------------------------------------------------------
__device__ __forceinline__ void rope_cs(int32_t pos, uint64_t step, float& c, float& s) {
    const uint64_t ph = (uint64_t)(int64_t)pos * step;
    const float r = (float)(int32_t)(ph >> 32) * 0x1p-32f;
    sincospif(2.0f * r, &s, &c);
}

__device__ __forceinline__ void rope_cs_f64(int32_t pos, uint64_t step, double& c, double& s) {
    const uint64_t ph = (uint64_t)(int64_t)pos * step;
    const double r = (double)(int64_t)ph * 0x1p-64;
    sincospi(2.0 * r, &s, &c);
}

// Model chunk (8 elements) read into kernel-layout chunk c of q or K.
__device__ __forceinline__ int model_chunk(uint64_t map, int c) { return (int)((map >> (4 * c)) & 15); }

// Table entries: float32 kernels read (cos, sin) as two floats; bf16 kernels read
// (cos, sin) as one bf16 pair, so that rotating a pair (x, y) is two 2-element dot
// products: x' = (x, y).(c, -s) with the sign folded into the instruction, and
// y' = (y, x).(c, s).
__device__ __forceinline__ uint32_t bf16_entry(float c, float s) { return pack_bf16(c, s); }

// cos/sin of N consecutive frequencies i0 .. i0+N-1 (i0 a multiple of 4) at
// position pos from a bf16 table when pos is inside it, else computed.
template <int N, bool TABLE>
__device__ __forceinline__ void rope_cs_n(const float* __restrict__ table, int rope_len, int half,
                                          const uint64_t* fstep, int32_t pos, int i0, float* c, float* s) {
    if (TABLE && (uint32_t)pos < (uint32_t)rope_len) {
        const u32x4_t* t = reinterpret_cast<const u32x4_t*>(reinterpret_cast<const uint32_t*>(table) + (size_t)pos * half + i0);
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            const u32x4_t v = t[k];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[4 * k + j] = bf_lo(v[j]);
                s[4 * k + j] = bf_hi(v[j]);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) rope_cs(pos, fstep[i0 + k], c[k], s[k]);
    }
}

// A wave-uniform element read through the scalar unit (the value lands in an
// SGPR and waits on the scalar counter, not on the vector-memory queue).
typedef __attribute__((address_space(4))) const int32_t const_i32_t;
__device__ __forceinline__ int32_t scalar_load(const int32_t* p, int i) { return ((const_i32_t*)p)[i]; }

// Group of attention block `bid` (MERGE: of merge block `bid`): binary search over
// the groups in the kernel arguments, or two scalar loads from the table the
// plan-upload launches wrote for a large batch.
template <bool MERGE, int N>
__device__ __forceinline__ Group group_of(const PlanOf<N>& plan, int bid) {
    if (plan.table != nullptr) {
        const int gi = scalar_load(MERGE ? plan.merge_map : plan.item_map, bid);
        const int32_t* src = reinterpret_cast<const int32_t*>(plan.table + gi);
        Group g;
        int32_t* dst = reinterpret_cast<int32_t*>(&g);
#pragma unroll
        for (int k = 0; k < (int)(sizeof(Group) / 4); ++k) dst[k] = scalar_load(src, k);
        return g;
    }
    return plan.g[MERGE ? plan_search<&Group::merge_base>(plan, bid) : plan_search<&Group::item_base>(plan, bid)];
}

// Item li of a group: its row tile and its cluster, the (KV head, key split) pair
// kvh * n_split + split.
struct ItemCoords {
    int cluster, rt, kvh, split;
};
__device__ __forceinline__ ItemCoords item_coords(const Group& g, int hkv, int n_rt, int li) {
    ItemCoords c;
    const int n_clusters = hkv * g.n_split;
    if ((hkv & 7) == 0) {
        // blocks bid, bid+8, ... run on one XCD: give them every (split, row tile) of
        // one KV head, so that the row tiles share K/V and the splits share Q in that
        // XCD's L2
        const int per_kvh = g.n_split * n_rt;
        const int x = li & 7, k = li >> 3;
        const int kv = x + 8 * (k / per_kvh), r = k % per_kvh;
        c.cluster = kv * g.n_split + r / n_rt;
        c.rt = r % n_rt;
    } else if ((n_clusters & 7) == 0) {
        // the same for the row tiles of one (KV head, split)
        const int x = li & 7, k = li >> 3;
        c.cluster = x + 8 * (k / n_rt);
        c.rt = k % n_rt;
    } else {
        c.cluster = li / n_rt;
        c.rt = li % n_rt;
    }
    c.kvh = c.cluster / g.n_split;
    c.split = c.cluster - c.kvh * g.n_split;
    return c;
}

template <int I>
struct Idx {
    static constexpr int value = I;
};

// max over lanes l and l^32 (one VALU permute, no LDS round trip)
__device__ __forceinline__ float max_xor32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_xor32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// XOR swizzle of the 16-byte chunks of LDS row `key`.  D = 128: 16 consecutive keys
// get 16 different patterns (conflict-free K operand reads) and 4 consecutive keys
// land in 4 different aligned groups of 4 chunks (conflict-free transposing V reads).
// D = 64 (two rows per bank line): 16 consecutive keys cover both halves x 8 chunks.
template <int D>
__device__ __forceinline__ int swz(int key) {
    if (D == 128) return ((key & 3) << 2) | ((key >> 2) & 3);
    return (key >> 1) & 7;
}

// The decode kernel's 16-key tiles: D = 128 puts key bits 0-1 on chunk bits 2-3,
// key bit 2 on chunk bit 1 and key bit 3 on chunk bit 0.  The 16 keys still get 16
// different patterns (conflict-free K operand reads), and the transposing V reads
// of 8 consecutive keys x 2 chunk halves (a 32-lane pass) cover all 16 chunks once.
template <int D>
__device__ __forceinline__ int dswz(int key) {
    if (D == 128) return ((key & 3) << 2) | (((key >> 2) & 1) << 1) | ((key >> 3) & 1);
    return swz<D>(key);
}

typedef __attribute__((address_space(3))) const uint16_t lds_u16_t;

// an LDS array element as an LDS-space pointer (constant offsets then fold into
// the instruction's offset field)
__device__ __forceinline__ lds_u16_t* as_lds(const uint16_t* p) { return (lds_u16_t*)p; }

typedef __attribute__((address_space(3))) const bf16x8_t lds_bf16x8_t;
// the LDS byte address of a shared array
__device__ __forceinline__ uint32_t lds_addr(const uint16_t* p) { return (uint32_t)(uintptr_t)(lds_u16_t*)p; }

// Transposing LDS read: within each 16-lane group, lane i receives element i%4 of
// the 8-byte rows that lanes i/4, i/4+4, i/4+8, i/4+12 point at.
__device__ __forceinline__ s16x4_t lds_read_tr(lds_u16_t* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)p);
}

__device__ __forceinline__ float max_xor16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_xor16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// cos/sin by the hardware's sine of a fraction of a revolution: within 2^-22.9 (measured against float64 at 2^24 phases of
// equal distance; rope_cs there: 2^-24.2), far below the 2^-12 to which the attention rounds what they turn
__device__ __forceinline__ void rope_cs_fast(int64_t pos, uint64_t step, float& c, float& s) {
    const uint64_t ph = (uint64_t)pos * step;
    const float r = (float)(int32_t)(ph >> 32) * 0x1p-32f;
    c = __builtin_amdgcn_cosf(r);
    s = __builtin_amdgcn_sinf(r);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, f16x2_t{(_Float16)lo, (_Float16)hi});
}

// max over the 8 lanes l & ~7 .. l | 7
__device__ __forceinline__ float max_of8(float x) {
    auto dpp = [&](auto ctrl) {
        return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(x), __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false)));
    };
    x = dpp(Idx<0xB1>{});    // lane ^ 1
    x = dpp(Idx<0x4E>{});    // lane ^ 2
    return dpp(Idx<0x141>{});   // lane ^ 7 (half rows mirrored)
}

// Bits of keys idx .. idx + 31 of a drafted token's mask row: keys before the span (idx < 0)
// are seen, keys past the row's words are not.
__device__ __forceinline__ uint32_t tree_bits(const uint32_t* __restrict__ row, int words, int idx) {
    const int w = idx >> 5;
    const uint32_t lo = w < 0 ? ~0u : w < words ? row[w] : 0u;
    const uint32_t hi = w + 1 < 0 ? ~0u : w + 1 < words ? row[w + 1] : 0u;
    return __builtin_amdgcn_alignbit(hi, lo, (uint32_t)idx & 31u);
}

// wait until this wave's global loads (including loads into LDS) have landed
__device__ __forceinline__ void wait_vmem() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// s_waitcnt on vector memory only: wait until at most N loads of this wave are
// outstanding (they complete in issue order)
template <int N>
__device__ __forceinline__ void wait_vmem_n() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

typedef __attribute__((address_space(3))) void lds_void_t;

// Global -> LDS copies written as inline assembly (global_load_lds_dword[x4], LDS
// base in M0): the compiler does not see their LDS writes, so it adds no
// vector-memory waits of its own before later LDS reads -- which it would do for
// every LDS read after the builtin form, draining the whole prefetch queue.  The
// kernel itself waits for them (wait_vmem_n, then a barrier) before reading what
// they wrote.  `lds_wave_base` is wave-uniform; lane i writes bytes
// [size*i, size*(i+1)) after it.
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const lds_void_t*)p);
}
__device__ __forceinline__ void dma_lds16(const void* src, const void* lds_wave_base) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "{m0}"(lds_offset(lds_wave_base)) : "memory");
}
// from a wave-uniform address plus a 32-bit byte offset per lane, and four bytes a lane, to a
// wave-uniform LDS byte address
__device__ __forceinline__ void copy_lds16(const void* base, uint32_t off, uint32_t to) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(to) : "memory");
}
__device__ __forceinline__ void copy_lds4(const void* src, uint32_t to) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "{m0}"(to) : "memory");
}
__device__ __forceinline__ void dma_lds16_s(const void* base, uint32_t off, const void* lds_wave_base) {
    copy_lds16(base, off, lds_offset(lds_wave_base));
}
__device__ __forceinline__ void dma_lds4(const void* src, const void* lds_wave_base) { copy_lds4(src, lds_offset(lds_wave_base)); }

// Workgroup barrier that leaves the vector-memory queue alone (__syncthreads
// would also drain every outstanding global->LDS load): this wave's LDS writes are
// waited for, and the compiler may move no memory access across it.
__device__ __forceinline__ void barrier_keep_vmem() {
    __builtin_amdgcn_s_waitcnt((15) | (3 << 14) | (7 << 4));   // lgkmcnt(0)
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

}  // namespace
}  // namespace pic
