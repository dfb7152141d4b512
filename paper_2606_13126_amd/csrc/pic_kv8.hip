// HIP kernels of the cache held in 8 bits, for MI355X (gfx950, CDNA4).
//
//  * qk_norm    norm of every query and key head of a projection, turned on the way where the
//               pool holds turned keys.
//  * kv8_write  key and value rows into the pool as codes and a scale per block and head.
//  * kv8_read   rows of the pool as numbers.
//  * kv8_few, kv8_many  attention over the codes in bf16; kv8_merge joins their key splits.  (float32: attn_f32
//               over Kv8Args, in pic_kernels.hip)
//  * kv8_keys   the call's turned copy of its keys, where many row tiles share them.
//
// Pools: codes [num_blocks][Hkv][16][D], one byte each, and scales [num_blocks][Hkv][2].  An
// element is code x scale.  The attention multiplies codes as they are (every code is exact in float16
// and bf16) and puts the keys' scale into the scores and the values' into the probabilities.
#include <type_traits>

#include "pic_device.h"

namespace pic {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef int32_t i32x4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// sum over the N lanes (4, 8 or 16, aligned) that hold a head
template <int N>
__device__ __forceinline__ float sum_of(float x) {
    auto dpp = [&](auto ctrl) {
        return x + __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(x), __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    x = dpp(Idx<0xB1>{});                       // lane ^ 1
    x = dpp(Idx<0x4E>{});                       // lane ^ 2
    if constexpr (N >= 8) x = dpp(Idx<0x141>{});    // lane ^ 7 (half rows mirrored)
    if constexpr (N >= 16) x = dpp(Idx<0x140>{});   // lane ^ 15 (rows mirrored)
    return x;
}

// ---------------------------------------------------------------------------------
// qk_norm: one workgroup per row; a unit is two 16-byte chunks of a head, NeoX the two runs whose
// elements pair up, GPT-J (and what does not turn) two neighbours.  The lanes of a head are
// neighbours, so its squares meet by lane permutes.  The row's threads put its cos/sin and the weights into
// LDS once, while its first units are on their way.
// Bound by memory: every element is read and written once.  16,384 rows of 64 + 8 heads of 128 (604 MB): 109 us, 5.5
// TB/s; 64 rows of 32 + 8 heads 3.0, two latencies.  Stores go through the caches, where what follows finds them: past
// them those calls took 100 to 105 where inputs repeat, but 164 against 136 with inputs and outputs out of the caches.
// ---------------------------------------------------------------------------------
constexpr int kNormThreads = 256;

// the elements of a 16-byte chunk as float32, and back (rounded to nearest even)
template <typename T>
__device__ __forceinline__ void unpack_chunk(const u32x4_t& w, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t u = w[i];
        if constexpr (sizeof(T) == 4) {
            f[i] = __uint_as_float(u);
        } else {
            f[2 * i] = bf_lo(u);
            f[2 * i + 1] = bf_hi(u);
        }
    }
}
template <typename T>
__device__ __forceinline__ u32x4_t pack_chunk(const float* f) {
    u32x4_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(f[i]) : pack_bf16(f[2 * i], f[2 * i + 1]);
    return w;
}

template <typename T, int D, int STYLE, bool ROT>
__global__ void __launch_bounds__(kNormThreads) qk_norm_kernel(const NormArgs a) {
    constexpr int PP = 16 / sizeof(T);     // elements per chunk, pairs per unit
    constexpr int CH = D / PP, UPH = CH / 2, U = 3;
    const int64_t row = blockIdx.x;
    const int unit = (int)threadIdx.x % UPH, step = (int)blockDim.x / UPH;
    const int rc = a.rot_half / PP;        // chunks of a half that turns (NeoX: rot_half is a multiple of 8)
    const bool turns = ROT && unit * PP < a.rot_half;
    // a turning unit's chunks, and any other's
    const int c0 = STYLE == kNeox ? (turns ? unit : 2 * rc + 2 * (unit - rc)) : 2 * unit;
    const int c1 = STYLE == kNeox && turns ? unit + rc : c0 + 1;
    const u32x4_t* qr = static_cast<const u32x4_t*>(a.q) + row * a.q_stride;
    const u32x4_t* kr = static_cast<const u32x4_t*>(a.k) + row * a.k_stride;
    u32x4_t* qo = static_cast<u32x4_t*>(a.q_out) + row * a.q_out_stride;
    u32x4_t* ko = static_cast<u32x4_t*>(a.k_out) + row * a.k_out_stride;
    const int heads = a.hq + a.hkv;
    __shared__ __attribute__((aligned(16))) float weight[2][D];
    __shared__ float2 cs[ROT ? D / 2 : 1];
    bool first = true;
    // (whole groups of UPH lanes take the same turns, so the lanes of a head are all there)
    for (int h0 = (int)threadIdx.x / UPH; first || h0 < heads; h0 += U * step) {
        u32x4_t x[U], y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = min(h0 + u * step, heads - 1);   // (past the last head: read, not stored)
            const u32x4_t* src = h < a.hq ? qr + h * CH : kr + (h - a.hq) * CH;
            x[u] = src[c0];
            y[u] = src[c1];
        }
        if (first) {
            for (int i = threadIdx.x; i < 2 * CH; i += blockDim.x) {
                const u32x4_t* from = static_cast<const u32x4_t*>(i < CH ? a.q_weight : a.k_weight);
                float f[PP];
#pragma unroll
                for (int k = 0; k < PP; ++k) f[k] = 1.f;
                if (from != nullptr) unpack_chunk<T>(from[i % CH], f);
#pragma unroll
                for (int k = 0; k < PP; ++k) weight[i / CH][i % CH * PP + k] = f[k];
            }
            if (ROT) {
                const int32_t pos = a.positions[row];
                for (int i = threadIdx.x; i < a.rot_half; i += blockDim.x) rope_cs(pos, a.fstep[i], cs[i].x, cs[i].y);
            }
            barrier_keep_vmem();
            first = false;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * step;
            if (h >= heads) break;
            float f[2 * PP], sum = 0.f;
            unpack_chunk<T>(x[u], f);
            unpack_chunk<T>(y[u], f + PP);
#pragma unroll
            for (int k = 0; k < 2 * PP; ++k) sum = __builtin_fmaf(f[k], f[k], sum);
            const float r = __builtin_amdgcn_rsqf(sum_of<UPH>(sum) * (1.f / D) + a.eps);   // (within an ulp; eps is normal, so is the argument)
            const float* w = weight[h < a.hq ? 0 : 1];
#pragma unroll
            for (int k = 0; k < 2 * PP; ++k) f[k] *= r * w[(k < PP ? c0 : c1) * PP + k % PP];
            if (turns)
#pragma unroll
                for (int k = 0; k < PP; ++k) {
                    if (STYLE != kNeox && unit * PP + k >= a.rot_half) break;
                    const float2 t = cs[unit * PP + k];
                    float& p = f[STYLE == kNeox ? k : 2 * k];
                    float& s = f[STYLE == kNeox ? PP + k : 2 * k + 1];
                    const float p0 = p, s0 = s;
                    p = __builtin_fmaf(p0, t.x, -(s0 * t.y));
                    s = __builtin_fmaf(p0, t.y, s0 * t.x);
                }
            u32x4_t* dst = h < a.hq ? qo + h * CH : ko + (h - a.hq) * CH;
            dst[c0] = pack_chunk<T>(f);
            dst[c1] = pack_chunk<T>(f + PP);
        }
    }
}

// ---------------------------------------------------------------------------------
// Codes
// ---------------------------------------------------------------------------------
template <int CODE>
struct Code {
    static constexpr float kMost = CODE == kCodeE4m3 ? 448.f : 127.f;
    static constexpr int kMaxExp = CODE == kCodeE4m3 ? 119 : 121;   // kMost times 2^kMaxExp is a finite bf16
    static constexpr int kMinExp = -126;
    // The smallest power of two s with x <= kMost s (x finite and >= 0), within the limits: kMost is
    // 1.75 x 2^8 or 1.984375 x 2^6, so the exponent of x decides, and its mantissa whether one more.
    static __device__ __forceinline__ float scale_of(float x) {
        const uint32_t b = __float_as_uint(x);
        const int up = (b & 0x7fffffu) > (CODE == kCodeE4m3 ? 0x600000u : 0x7e0000u) ? 1 : 0;
        const int e = (int)(b >> 23) - 127 - (CODE == kCodeE4m3 ? 8 : 6) + up;
        return __uint_as_float((uint32_t)(min(max(e, kMinExp), kMaxExp) + 127) << 23);
    }
    // Four numbers in units of the scale as codes: to nearest, ties to even, saturating; NaN 0
    static __device__ __forceinline__ uint32_t encode(float x0, float x1, float x2, float x3) {
        float x[4] = {x0, x1, x2, x3};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = x[i] == x[i] ? __builtin_amdgcn_fmed3f(x[i], -kMost, kMost) : 0.f;
        if constexpr (CODE == kCodeE4m3) {
            const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
            return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
        } else {
            // the low byte of 1.5 x 2^23 + x is x rounded, in two's complement
            uint32_t b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(x[i] + 0x1.8p23f);
            const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
            return lo | hi;
        }
    }
    // the four codes of a word as numbers
    static __device__ __forceinline__ f32x4_t decode(uint32_t w) {
        if constexpr (CODE == kCodeE4m3) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            return f32x4_t{lo[0], lo[1], hi[0], hi[1]};
        } else {
            return f32x4_t{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)};
        }
    }
    // ... as two words of float16 (exact)
    static __device__ __forceinline__ uint32_t halves_lo(uint32_t w) { return half2_of<false>(w); }
    static __device__ __forceinline__ uint32_t halves_hi(uint32_t w) { return half2_of<true>(w); }
    template <bool HI>
    static __device__ __forceinline__ uint32_t half2_of(uint32_t w) {
        if constexpr (CODE == kCodeE4m3) {
            const f16x2_t x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, HI);
            return __builtin_bit_cast(uint32_t, x);
        } else {
            // 0x64uu is 1024 + u: with u = code + 128, less 1152
            const f16x2_t off = {(_Float16)-1152.f, (_Float16)-1152.f};
            const uint32_t u = __builtin_amdgcn_perm(0x64646464u, w ^ 0x80808080u, HI ? 0x04030402u : 0x04010400u);
            const f16x2_t x = __builtin_bit_cast(f16x2_t, u) + off;
            return __builtin_bit_cast(uint32_t, x);
        }
    }
    // ... as two words of bf16 (exact: an upper half of a float32 holds 8 bits)
    static __device__ __forceinline__ u32x2_t bf16s(uint32_t w) {
        if constexpr (CODE == kCodeE4m3) {
            const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true);
            return u32x2_t{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
        }
        const f32x4_t x = decode(w);
        return u32x2_t{__builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u),
                       __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u)};
    }
};

// ---------------------------------------------------------------------------------
// kv8_write.  A unit is (block, head, keys or values), taken by a wave: the rows that the call
// stores in the block give the scale (a maximum over the wave), then lane l codes 16 elements of offset
// l / (D / 16) (and 64 / (D / 16) offsets on), so that a page leaves in whole lines.  A workgroup looks for runs (rows of one
// block that follow one another) that begin among `range` rows, and has to know whose a block of several runs is, and
// the others' rows:
//  - Calls of up to kWriteScan rows: every workgroup counts its blocks' rows in the call.  Where a run is all of them (a
//    request's tokens in order) that is all; else the block is the first run's, whose waves look for the others' rows.
//  - More rows: a launch ahead (kv8_notes) sets the sign of the scale of the block's head 0, which is not negative
//    otherwise, and leaves in every slot that the call writes the last of its rows.  A block is the run's that takes the sign
//    away, and its rows are what its slots hold.  (A slot's first bytes are a note where the row that they name stores there:
//    true of any bytes, so what was there before needs no clearing.)
// Counting costs nothing for 256 rows, 1 us of 8.0 for 1,024 of a prompt and 2.7 of 17.6 for 1,024 requests of a row; notes
// 4 us of 11.4 for 2,048 of a prompt, 6 of 28.0 for 16,876, and nothing for 2,048 requests of a row.  16 tokens of each of 64
// requests, token by token, take 101 us by counting, of 128 requests 31 by notes and of 1,024 58.
// Bound by memory for prompts (104 MB, 8 heads of 128: 20.4 us, 5.1 TB/s, beside the notes), by its chain of loads
// (slots, then rows) for a step's tokens (64 rows: 5.0 us).
// ---------------------------------------------------------------------------------
constexpr int kWriteWaves = 4, kNotedWaves = 16;
constexpr uint32_t kSign = 0x80000000u;

// Row i of a call stores in slot s
__device__ __forceinline__ bool stores_in(const Kv8WriteArgs& a, int32_t i, int32_t s) { return i >= 0 && i < a.n && a.slots[i] == s; }

// The first four bytes of a slot's keys of head 0, which the call writes anyway: the last row that stores there
template <int D>
__device__ __forceinline__ int32_t* note_of(const Kv8WriteArgs& a, int32_t slot) {
    return reinterpret_cast<int32_t*>(a.k_pool + ((int64_t)(slot >> 4) * a.hkv * kBlock + (slot & 15)) * D);
}

// Notes of a call for kv8_write_kernel
template <int D>
__global__ void __launch_bounds__(256) kv8_notes(const Kv8WriteArgs a) {
    const int64_t row = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (row >= a.n) return;
    const int32_t i = (int32_t)row, s = a.slots[i];
    if (s < 0 || s >= a.n_slots) return;
    const int32_t before = i > 0 ? a.slots[i - 1] : -1;
    if (before >> 4 != s >> 4) atomicOr(reinterpret_cast<uint32_t*>(a.scale) + (int64_t)(s >> 4) * a.hkv * 2, kSign);
    // (what no row of this slot left there is some code; a later row's note stays)
    int32_t* note = note_of<D>(a, s);
    for (int32_t have = *note; have < i || !stores_in(a, have, s);) {
        const int32_t now = atomicCAS(note, have, i);
        if (now == have) break;
        have = now;
    }
}

template <typename T, int D, int CODE, int WAVES, bool NOTED>
__global__ void __launch_bounds__(WAVES * 64) kv8_write_kernel(const Kv8WriteArgs a) {
    typedef Code<CODE> C;
    constexpr int LPO = D / 16;            // lanes of an offset
    constexpr int OPP = 64 / LPO, P = kBlock / OPP;   // offsets per pass, passes
    constexpr int V = 16 / sizeof(T), NV = 16 / V;    // elements of a load, loads of a lane per pass
    typedef T vec_t __attribute__((ext_vector_type(V)));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t r0 = (int64_t)blockIdx.x * a.range;
    const int n_here = (int)min((int64_t)a.range, a.n - r0);
    // the slots of 64 rows, and of the row before (a row that stores nothing: some number below 0, in no block)
    auto slot_of = [&](int64_t i) {
        const int32_t s = i >= 0 && i < a.n ? a.slots[i] : -1;
        return s < a.n_slots ? s : -1;
    };
    const int32_t mine = slot_of(r0 + lane), before = lane == 0 ? slot_of(r0 - 1) : 0;
    int32_t prev = __shfl_up(mine, 1);
    if (lane == 0) prev = before;
    const uint64_t leads = __builtin_amdgcn_ballot_w64(lane < n_here && mine >= 0 && mine >> 4 != prev >> 4);
    if (leads == 0) return;
    const int per = 2 * a.hkv, c16 = (lane % LPO) * 16;
    uint64_t taken = leads;                     // the runs whose blocks are this workgroup's
    __shared__ int rows_of[kWriteRange][kBlock];   // noted: of each block (by the lane of the run's first row), its rows or -1
    __shared__ int stored[kWriteRange];            // else how many rows of the call store there
    if constexpr (NOTED) {
        __shared__ unsigned mask;
        if (wave == 0) {
            bool first_here = false;
            if (leads >> lane & 1)
                first_here = (atomicAnd(reinterpret_cast<uint32_t*>(a.scale) + (int64_t)(mine >> 4) * a.hkv * 2, ~kSign) & kSign) != 0;
            const uint64_t m = __builtin_amdgcn_ballot_w64(first_here);
            if (lane == 0) mask = (unsigned)m;
        }
        __syncthreads();
        taken = mask;
        if (taken == 0) return;
        for (int i = wave; i < kWriteRange * kBlock / 64; i += WAVES) {
            const int at = i * 64 / kBlock + lane / kBlock, slot = (__shfl(mine, at) & ~15) + lane % kBlock;
            if (taken >> at & 1) {
                const int32_t row = *note_of<D>(a, slot);
                rows_of[at][lane % kBlock] = stores_in(a, row, slot) ? row : -1;
            }
        }
        __syncthreads();
    } else {
        if (threadIdx.x < kWriteRange) stored[threadIdx.x] = 0;
        __syncthreads();
        constexpr int U = 4, EACH = WAVES * 64 * 4;   // slots of a load of all threads
        for (uint32_t i0 = 0; i0 < (uint32_t)a.n; i0 += U * EACH) {
            i32x4_t s[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const uint32_t at = i0 + k * EACH + threadIdx.x * 4;
                if (i0 + (k + 1) * EACH <= (uint32_t)a.n) {
                    s[k] = *reinterpret_cast<const i32x4_t*>(a.slots + at);
                } else {
                    s[k] = i32x4_t{-1, -1, -1, -1};
                    if (i0 + k * EACH < (uint32_t)a.n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (at + e < (uint32_t)a.n) s[k][e] = a.slots[at + e];
                }
            }
            for (uint64_t rest = leads; rest; rest &= rest - 1) {
                const int first = __builtin_ctzll(rest), blk = __builtin_amdgcn_readlane(mine, first) >> 4;
                uint32_t least = ~0u;   // (below 16: a slot of the block; most lanes have none)
#pragma unroll
                for (int k = 0; k < U; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) least = min(least, (uint32_t)(s[k][e] ^ blk << 4));
                if (least >= kBlock) continue;
                int of = 0;
#pragma unroll
                for (int k = 0; k < U; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) of += s[k][e] >> 4 == blk;
                atomicAdd(&stored[first], of);
            }
        }
        __syncthreads();
    }
    const int units = __builtin_popcountll(taken) * per;
    for (int u = (int)blockIdx.y * WAVES + wave; u < units; u += (int)gridDim.y * WAVES) {
        uint64_t rest = taken;
        for (int i = u / per; i > 0; --i) rest &= rest - 1;
        const int first = __builtin_ctzll(rest);
        const int which = u & 1, h = (u % per) >> 1;
        // the rows of the block: of each offset the last
        const int blk = __builtin_amdgcn_readlane(mine, first) >> 4;
        int64_t row[P];
        bool fresh = false;
        if constexpr (NOTED) {
#pragma unroll
            for (int p = 0; p < P; ++p) row[p] = rows_of[first][p * OPP + lane / LPO];
            fresh = rows_of[first][0] >= 0;
        } else {
#pragma unroll
            for (int p = 0; p < P; ++p) row[p] = -1;
            auto take = [&](int64_t from, int32_t slot, uint64_t rows) {   // rows of 64 from `from` on
#pragma unroll
                for (int o = 0; o < kBlock; ++o) {
                    const uint64_t m = __builtin_amdgcn_ballot_w64((slot & 15) == o) & rows;
                    if (m == 0) continue;
                    if (o == 0) fresh = true;
                    if (o % OPP == lane / LPO) row[o / OPP] = from + 63 - __builtin_clzll(m);
                }
            };
            int32_t slot = mine;
            uint64_t live = ~0ull << first;   // lanes whose rows come into question
            int here = 0;                     // rows of the run
            for (int64_t from = r0;; from += 64) {
                const uint64_t others = __builtin_amdgcn_ballot_w64((slot >> 4) != blk) & live;
                const uint64_t run = others ? live & ((others & -others) - 1) : live;
                here += __builtin_popcountll(run);
                take(from, slot, run);
                if (others) break;
                live = ~0ull;   // (only rows of one slot over and over are more than a wave looks at)
                slot = slot_of(from + 64 + lane);
            }
            if (stored[first] != here) {   // the block has other runs
                constexpr int U = 4;   // times 64 rows on their way
                bool before_it = false;
                for (int64_t from = 0; from < r0 + first && !before_it; from += 64 * U) {
                    int32_t it[U];
#pragma unroll
                    for (int k = 0; k < U; ++k) it[k] = slot_of(from + 64 * k + lane);
#pragma unroll
                    for (int k = 0; k < U; ++k)
                        before_it |= __builtin_amdgcn_ballot_w64(from + 64 * k + lane < r0 + first && it[k] >> 4 == blk) != 0;
                }
                if (before_it) continue;
                for (int64_t from = r0 + first; from < a.n; from += 64 * U) {
                    int32_t it[U];
#pragma unroll
                    for (int k = 0; k < U; ++k) it[k] = slot_of(from + 64 * k + lane);
#pragma unroll
                    for (int k = 0; k < U; ++k) {
                        const uint64_t rows = __builtin_amdgcn_ballot_w64(it[k] >> 4 == blk);
                        if (rows) take(from + 64 * k, it[k], rows);
                    }
                }
            }
        }
        const T* src = static_cast<const T*>(which ? a.v : a.k);
        const int64_t stride = (which ? a.v_stride : a.k_stride) * V;
        vec_t x[P][NV];
        float big = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                x[p][i] = row[p] >= 0 ? *reinterpret_cast<const vec_t*>(src + row[p] * stride + h * D + c16 + i * V) : vec_t((T)0.f);
        float* sp = a.scale + ((int64_t)blk * a.hkv + h) * 2 + which;
        const float old = fresh ? 0.f : fabsf(*sp);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float y = fabsf((float)x[p][i][e]);
                    big = fmaxf(big, y < INFINITY ? y : 0.f);
                }
        big = max_xor32(max_xor16(max_of8(big)));
        big = fmaxf(big, __shfl_xor(big, 8));
        const float s = fmaxf(C::scale_of(big), old), inv = 1.f / s;
        const float ratio = old > 0.f ? old * inv : 0.f;
        uint8_t* page = (which ? a.v_pool : a.k_pool) + ((int64_t)blk * a.hkv + h) * kBlock * D;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int o = p * OPP + lane / LPO;
            u32x4_t* dst = reinterpret_cast<u32x4_t*>(page + o * D + c16);
            u32x4_t w;
            if (row[p] >= 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float f[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] = (float)x[p][(4 * i + e) / V][(4 * i + e) % V] * inv;
                    w[i] = C::encode(f[0], f[1], f[2], f[3]);
                }
            } else if (fresh) {
                w = u32x4_t{0, 0, 0, 0};
            } else if (s != old) {
                w = *dst;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4_t f = C::decode(w[i]) * ratio;
                    w[i] = C::encode(f[0], f[1], f[2], f[3]);
                }
            } else {
                continue;
            }
            *dst = w;
        }
        if (lane == 0 && s != old) *sp = s;
    }
}

// ---------------------------------------------------------------------------------
// kv8_read: a thread takes the codes of 16 bytes of output (4 or 8), U of them in flight.  Bound by memory: 33,280
// rows of 8 heads of 128 (204 MB) 41 us, 4.9 TB/s.  Stores go through the caches: past them the call took 31 us where the
// same blocks are read over and over, but 55.5 against 57 with its inputs out of the caches, and with a copy of its outputs
// behind it 121 against 103 (20,480 rows: 82 against 61).
// ---------------------------------------------------------------------------------
template <typename T, int D, int CODE>
__global__ void __launch_bounds__(256) kv8_read_kernel(const uint8_t* __restrict__ k_pool, const uint8_t* __restrict__ v_pool,
                                                       const float* __restrict__ scale, int64_t n_slots,
                                                       const int32_t* __restrict__ slots, int64_t n_units, int hkv,
                                                       T* __restrict__ k_out, T* __restrict__ v_out) {
    typedef Code<CODE> C;
    constexpr int V = 16 / sizeof(T), W = V / 4, CPR = D / V, U = 2;
    typedef T vec_t __attribute__((ext_vector_type(V)));
    typedef uint32_t word_t __attribute__((ext_vector_type(W)));
    const int64_t step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i0 < n_units; i0 += U * step) {
        word_t w[U][2];
        float2 sc[U];
        bool in[U];   // the unit exists and its slot lies in the pool
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * step;
            in[u] = false;
            if (i >= n_units) continue;
            const int64_t rh = i / CPR, row = rh <= UINT32_MAX ? (uint32_t)rh / (uint32_t)hkv : rh / hkv;
            const int32_t slot = slots[row];
            if (slot < 0 || slot >= n_slots) continue;
            in[u] = true;
            const int64_t page = (int64_t)(slot >> 4) * hkv + (rh - row * hkv);
            const int64_t at = (page * kBlock + (slot & 15)) * D + (i % CPR) * V;
            w[u][0] = *reinterpret_cast<const word_t*>(k_pool + at);
            w[u][1] = *reinterpret_cast<const word_t*>(v_pool + at);
            sc[u] = *reinterpret_cast<const float2*>(scale + 2 * page);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!in[u]) continue;
            const int64_t i = i0 + u * step;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                vec_t y;
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const f32x4_t f = C::decode(w[u][kv][j]) * (kv ? sc[u].y : sc[u].x);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[4 * j + e] = (T)f[e];
                }
                *reinterpret_cast<vec_t*>((kv ? v_out : k_out) + i * V) = y;
            }
        }
    }
}

// group_of for the kernels here: among groups in the arguments every lane looks at one, in one round trip
// (kernel arguments lie in host memory, and a binary search takes up to six, one after the other).
template <bool MERGE, int N>
__device__ __forceinline__ Group find_group(const PlanOf<N>& plan, int bid) {
    static_assert(N <= 64, "a lane per group");
    if (plan.table != nullptr) return group_of<MERGE>(plan, bid);
    if (plan.n_groups == 1) return plan.g[0];
    const int lane = (int)threadIdx.x & 63, i = lane < plan.n_groups ? lane : 0;
    const int base = MERGE ? plan.g[i].merge_base : plan.g[i].item_base;
    return plan.g[__builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < plan.n_groups && base <= bid)) - 1];
}

// ---------------------------------------------------------------------------------
// kv8_few: attention in bf16, up to 16 CB query rows (query token x query head of one KV head's
// group) per workgroup of eight waves, over one key range.  Every wave holds the rows and takes every
// eighth cache block of the range, which it copies to LDS some steps ahead, turns and multiplies
// without waiting for another wave; the eight results meet in LDS at the end.
//   S^T (16 keys x 16 rows) = K Q^T       v_mfma_f32_16x16x32_f16 (bf16 without rotation)
//   O^T (16 dims x 16 rows) += V^T P^T    v_mfma_f32_16x16x32_bf16
// After the scores lane l holds row l%16 of each block and keys 4 (l/16) + {0..3}, the B operand of
// the output product.  Its A operand: a transposing read of 16-bit elements gives a lane two
// neighbouring dimensions of four keys, two byte permutes part them.  The 32-deep product
// holds the 16 keys twice, for a probability as two bf16 numbers (16 bits in all).
//
// RoPE: with b the position of a block's first key and r that of the row tile's first query token, (R_p q).(R_(b+j) k) =
// (R_(r-b) R_(p-r) q).(R_j k).  Where a block's positions follow one another its keys turn by their place j in it, the same
// for every block, whose cos/sin a lane holds in registers (of its 4 KD pairs of key l%16), and the queries turn by r - b,
// whose cos/sin are 64 numbers of the whole wave, one of a lane.  Other blocks' keys turn by the positions that they have,
// less b.  Turning is done in packed float16, two pairs at a time: 16 operations of a lane for the queries of a block and 16
// for its keys (D 128: twice that), where angles of each key that advance from block to block cost 5 a pair beside the keys'
// own (64 requests x 8,192 keys of int8, 32 / 8 heads of 128: 204.6 us, 211.8 with those).  The first token's queries
// (all of a decode's) are rounded there alone: p = r.  Those of other tokens turn by p - r before, once, in float32, and are
// rounded to float16.
//
// Bound by memory and by the vector unit about alike where the card is full: the same call 196 us at its best, 5.5 TB/s, the
// vector unit busy 66% of the cycles and the matrix cores 10%; 192 without rotation.  Few keys: by the chain of
// plan, block ids, codes, products and the meeting of the waves (7.2 us over 1,537 keys).
// ---------------------------------------------------------------------------------

template <int D, int CB>
struct Kv8Few {
    static constexpr int NW = kKv8Waves, TK = kBlock;
    static constexpr int STEP = NW * TK;         // keys of all waves
    static constexpr int TILE = TK * D;          // bytes of a wave's keys or values of a step
    static constexpr int CPR = D / 16;           // 16-byte chunks per row
    static constexpr int KPC = 64 / CPR;         // keys of a copy (64 chunks)
    static constexpr int NC = TK / KPC;          // copies of a step, each of K and V
    // Steps in LDS, and waves per SIMD: at 16 rows of 128 dims four waves with two steps each hide more than two with four
    // (the call above 204 against 224 us, spans that 64 requests share 141 against 174)
    static constexpr int NST = D == 64 || CB > 1 ? 4 : 2;
    static constexpr int WAVES = CB > 1 ? 2 : 4;
    static constexpr int LPS = 2 * NC + 1;       // copies per lane per step
    static constexpr int META = 20;              // a step's positions (16) and its two scales
};

template <int D, int CB>
struct __attribute__((aligned(16))) Kv8FewLds {
    typedef Kv8Few<D, CB> S;
    uint8_t stages[S::NST][S::NW][2][S::TILE];
    uint16_t q[CB][D / 32][64][8];               // B operands: words of 4 pairs of the lanes, x then y
    float qs[16 * CB];
    uint64_t fstep[D / 2];
    uint16_t places[kBlock][D / 8][8];           // cos/sin of 0 .. 15 positions: of 4 pairs, cos then sin
    uint16_t base[S::NW][D / 8][8];              // ... of a wave's block, from the first token on
    int32_t meta[S::NW][S::NST][S::META];
};

// LDS rows of codes: 16-byte chunk c of key k lies at c ^ swizzle.  Keys are read by 8 bytes of 16 keys (two
// neighbouring 8-byte pieces of each in 32 lanes), values by 32 bytes of 8 keys; 256 bytes hold 256 / D keys.
template <int D>
__device__ __forceinline__ int kswz(int key) { return D == 128 ? (key >> 1) & 7 : (key >> 2) & 3; }
template <int D>
__device__ __forceinline__ int vswz(int key) { return D == 128 ? ((key >> 1) & 3) << 1 : ((key >> 2) & 1) << 1; }

// A query row whose largest element is big goes in times 2^-ex, within 1: its products with turned codes,
// of up to 634 each, stay in range
__device__ __forceinline__ int query_exponent(float big) { return big > 0.f && big < INFINITY ? __builtin_amdgcn_frexp_expf(big) : 0; }

// Four pairs (x 0-1, x 2-3, y 0-1, y 2-3) turned by the angles of cs (cos, then sin), or back by them
__device__ __forceinline__ u32x4_t turned(const u32x4_t& v, const u32x4_t& cs, bool back) {
    u32x4_t out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t xw = v[h], yw = v[2 + h], cw = cs[h], sw = cs[2 + h];   // (a bit cast of a vector's element would read its first)
        const f16x2_t x = __builtin_bit_cast(f16x2_t, xw), y = __builtin_bit_cast(f16x2_t, yw), c = __builtin_bit_cast(f16x2_t, cw);
        f16x2_t s = __builtin_bit_cast(f16x2_t, sw);
        if (back) s = -s;
        out[h] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(x, c, -(y * s)));
        out[2 + h] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(y, c, x * s));
    }
    return out;
}

template <int D, int STYLE, bool ROPE, int CODE, int CB, int NG>
__global__ void __launch_bounds__(kKv8Waves * 64, (Kv8Few<D, CB>::WAVES)) kv8_few(const PlanOf<NG> plan, const Kv8Args a) {
    typedef Kv8Few<D, CB> S;
    typedef Code<CODE> C;
    constexpr int KD = D / 32;             // 16x16x32 contraction steps of QK^T; words of 4 pairs of a lane
    constexpr int DB = D / 32;             // 32-dim blocks of O^T
    constexpr int TK = S::TK, NW = S::NW, NST = S::NST, HALF = D / 2;
    static_assert(S::TILE * 2 * NST >= CB * 2 * DB * 1024, "a wave's outputs fit its stages");

    __shared__ Kv8FewLds<D, CB> lds;
    __shared__ float2 mls[NW][16 * CB];

    const Group g = find_group<false>(plan, blockIdx.x);
    const int G = a.group, n_rt = g.n_rt;
    const int li = blockIdx.x - g.item_base;   // (a call's items are not padded: below the group's count)
    const ItemCoords ic = item_coords(g, a.hkv, n_rt, li);
    const int rt = n_rt - 1 - ic.rt;           // the longest first
    const int rows_total = g.n_tok * G, row_lo = rt * 16 * CB;
    const int t_last = g.tok0 + (min(row_lo + 16 * CB, rows_total) - 1) / G;
    const int kv_lo = g.win + ic.split * g.split_keys;
    if (kv_lo > t_last) return;                // (the row tile's splits end before this one)
    // (no sum below passes the last key: a request may have 2^31 - 1 of them)
    const int kv_hi = g.split_keys < t_last + 1 - kv_lo ? kv_lo + g.split_keys : t_last + 1;
    const int kt0 = kv_lo & ~(TK - 1);
    const int k_lo = kv_lo - kt0, k_hi = kv_hi - kt0;   // the range from the start of its first block
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c16 = lane & 15, q4 = lane >> 4;
    const int n_tiles = (k_hi - 1) / TK + 1;
    const int nt = n_tiles > wave ? (n_tiles - wave - 1) / NW + 1 : 0;
    const int32_t* btab = a.block_tables + (size_t)g.req * a.max_blocks + (kt0 >> 4);
    const int32_t* posv = a.positions + g.pos_off + kt0;
    const size_t page = (size_t)TK * D;
    const uint8_t* kpool = static_cast<const uint8_t*>(a.k_pool) + ic.kvh * page;
    const uint8_t* vpool = static_cast<const uint8_t*>(a.v_pool) + ic.kvh * page;
    const uint32_t stages_at = lds_offset(lds.stages), meta_at = lds_offset(&lds.meta[wave][0][0]);

    // the wave's copies of step u into stage st: a lane's 16 bytes are one chunk of one key, and a key outside
    // the range stands for the nearest one inside, so that nothing outside it is read (its score is masked)
    auto near_key = [&](int k) { return min(max(k, k_lo), k_hi - 1); };
    // the lane's bytes of a page in the first copy; the second one (D 128: 8 keys on) swizzles keys by another bit
    const int c_key = lane / S::CPR, k_from = c_key * D + (((lane % S::CPR) ^ kswz<D>(c_key)) << 4),
              v_from = c_key * D + (((lane % S::CPR) ^ vswz<D>(c_key)) << 4);
    static_assert(S::NC == 1 || D == 128, "one copy of a page, or two");
    auto issue = [&](int u, int st, int blk) {
        const int k0 = u * S::STEP + wave * TK;
        const uint32_t to = stages_at + (uint32_t)((st * NW + wave) * 2 * S::TILE);
        __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));   // the stage's last reads have returned
        const size_t at = (size_t)(uint32_t)blk * a.hkv * page;
        const bool whole = k0 >= k_lo && k0 + TK <= k_hi;   // the tile needs no nearest keys
#pragma unroll
        for (int i = 0; i < S::NC; ++i) {
            int moved = 0;
            if (!whole) {
                const int key = k0 + i * S::KPC + lane / S::CPR;
                moved = ((near_key(key) & (TK - 1)) - (key & (TK - 1))) * D;
            }
            copy_lds16(kpool + at, (uint32_t)((k_from ^ (i << 6)) + i * S::KPC * D + moved), to + i * 1024);
            copy_lds16(vpool + at, (uint32_t)(v_from + i * S::KPC * D + moved), to + S::TILE + i * 1024);
        }
        if (lane < 18) {
            const void* src = lane < 16 ? (const void*)(posv + (whole ? k0 + lane : near_key(k0 + lane)))
                                        : (const void*)(a.scale + ((size_t)(uint32_t)blk * a.hkv + ic.kvh) * 2 + (lane - 16));
            copy_lds4(src, meta_at + (uint32_t)(st * S::META * 4));
        }
    };
    auto block_at = [&](int u) { return scalar_load(btab, u * NW + wave); };   // (u < nt: the block holds a key of the range)

#pragma unroll
    for (int u = 0; u < NST - 1; ++u)
        if (u < nt) issue(u, u, block_at(u));
    // cos/sin of pair p to where the lanes of its word read them
    auto put_cs = [](uint16_t (*to)[8], int p, float c, float s) {
        to[p >> 2][p & 3] = __builtin_bit_cast(uint16_t, (_Float16)c);
        to[p >> 2][4 + (p & 3)] = __builtin_bit_cast(uint16_t, (_Float16)s);
    };
    const int my_pair = lane % HALF;
    const uint64_t my_step = ROPE ? a.fstep[my_pair] : 0;
    if (ROPE) {
        if (wave == 0) lds.fstep[my_pair] = my_step;
#pragma unroll
        for (int k = 0; k < TK; k += NW * 64 / HALF) {
            float c, s;
            const int place = k + (int)threadIdx.x / HALF;
            rope_cs_fast(place, my_step, c, s);
            put_cs(lds.places[place], my_pair, c, s);
        }
    }

    // the lane's words of 4 pairs: word i holds pairs 4 word_at(i) ..
    auto word_at = [&](int i) { return STYLE == kNeox ? i / 2 * 8 + 2 * q4 + i % 2 : 4 * i + q4; };

    // ---- queries: the waves turn 2 CB rows each, LPR lanes a row, and leave the B operands of all in LDS
    // (from where every tile reads them: in registers they would leave room for two waves per SIMD only)
    const int64_t first_pos = ROPE ? a.positions[g.pos_off + g.tok0 + row_lo / G] : 0;   // of the tile's first token
    int last[CB];     // last key that the lane's row sees, from kt0
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row_lo + 16 * cb + c16;
        last[cb] = min(k_hi - 1, g.tok0 + (row < rows_total ? row / G : 0) - kt0);
    }
    {
        constexpr int LPR = 32 / CB, PP = HALF / LPR;   // lanes of a row, pairs of a lane
        static_assert(NW * 64 == 16 * CB * LPR && PP <= 4, "every lane has a part of a row");
        typedef uint16_t part_t __attribute__((ext_vector_type(PP)));
        const int r = (wave * 64 + lane) / LPR, p0 = lane % LPR * PP, row = row_lo + r;
        const bool valid = row < rows_total;
        const int to = valid ? row / G : 0, hl = valid ? row - to * G : 0;
        // two runs of PP elements: NeoX the pairs' x and y, GPT-J one after the other
        const int e[2] = {STYLE == kNeox ? p0 : 2 * p0, STYLE == kNeox ? p0 + HALF : 2 * p0 + PP};
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((size_t)(g.q_row0 + to) * a.hq + (size_t)ic.kvh * G + hl) * D;
        uint16_t in[2 * PP];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const part_t w = *reinterpret_cast<const part_t*>(qp + model_chunk(a.chunk_map, e[h] >> 3) * 8 + (e[h] & 7));
#pragma unroll
            for (int k = 0; k < PP; ++k) {
                if constexpr (PP == 1) in[h] = w[0];
                else in[h * PP + k] = w[k];
            }
        }
        const int64_t from_first = ROPE ? (int64_t)a.positions[g.pos_off + g.tok0 + to] - first_pos : 0;
        __syncthreads();   // phase steps staged
        float x[PP], y[PP], big = 0.f;
#pragma unroll
        for (int k = 0; k < PP; ++k) {
            x[k] = valid ? __uint_as_float((uint32_t)in[STYLE == kNeox ? k : 2 * k] << 16) : 0.f;
            y[k] = valid ? __uint_as_float((uint32_t)in[STYLE == kNeox ? PP + k : 2 * k + 1] << 16) : 0.f;
        }
        float scale = a.scale_log2;
        int ex = 0;
        if (ROPE) {
#pragma unroll
            for (int k = 0; k < PP; ++k) {
                float c, s;
                rope_cs_fast(from_first, lds.fstep[p0 + k], c, s);
                const float x0 = x[k], y0 = y[k];
                x[k] = x0 * c - y0 * s;
                y[k] = y0 * c + x0 * s;
                big = fmaxf(big, fmaxf(fabsf(x[k]), fabsf(y[k])));
            }
            big = max_of8(big);
            big = fmaxf(big, __shfl_xor(big, 8));
            if (LPR == 32) big = max_xor16(big);
            ex = query_exponent(big);
            scale = ldexpf(scale, ex);
        }
        part_t xo, yo;
#pragma unroll
        for (int k = 0; k < PP; ++k) {
            const uint16_t xb = ROPE ? __builtin_bit_cast(uint16_t, (_Float16)ldexpf(x[k], -ex)) : (uint16_t)(__float_as_uint(x[k]) >> 16);
            const uint16_t yb = ROPE ? __builtin_bit_cast(uint16_t, (_Float16)ldexpf(y[k], -ex)) : (uint16_t)(__float_as_uint(y[k]) >> 16);
            xo[k] = xb;
            yo[k] = yb;
        }
        // pairs p0 .. p0 + PP - 1 belong to word i of the lanes 16 qq ..
        const int i = STYLE == kNeox ? (p0 >> 5) * 2 + ((p0 >> 2) & 1) : p0 >> 4, qq = STYLE == kNeox ? (p0 >> 3) & 3 : (p0 >> 2) & 3;
        uint16_t* to_lds = &lds.q[r >> 4][i][16 * qq + (r & 15)][p0 & 3];
        *reinterpret_cast<part_t*>(to_lds) = xo;
        *reinterpret_cast<part_t*>(to_lds + 4) = yo;
        if (lane % LPR == 0) lds.qs[r] = scale;
    }
    barrier_keep_vmem();
    float qs[CB];     // scores are the products times this and the block's scale (log2 units)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) qs[cb] = lds.qs[16 * cb + c16];

    // per-lane byte offsets within a tile: the K operand's 8 codes of each chunk, the V operand's pieces
    // (of block db of the dimensions: by xor)
    int k_off[KD], v_off;
#pragma unroll
    for (int kd = 0; kd < KD; ++kd) {
        const int c8 = model_chunk(a.chunk_map, kd * 4 + q4);
        k_off[kd] = c16 * D + (((c8 >> 1) ^ kswz<D>(c16)) << 4) + (c8 & 1) * 8;
    }
    {
        const int key = 4 * q4 + (c16 >> 2);
        v_off = S::TILE + key * D + ((((c16 >> 1) & 1) ^ vswz<D>(key)) << 4) + (c16 & 1) * 8;
    }

    f32x4_t acc[CB][2 * DB];   // even and odd dimensions of each block
    float m_run[CB], l_run[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        m_run[cb] = kNegBig;
        l_run[cb] = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) acc[cb][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    u32x4_t place[ROPE ? KD : 1];   // cos/sin of the lane's key's place in its block, words as in lds.places
    if constexpr (ROPE)
#pragma unroll
        for (int i = 0; i < KD; ++i) place[i] = *reinterpret_cast<const u32x4_t*>(lds.places[c16][word_at(i)]);

    int st = 0, blk = 0;
    if (NST - 1 < nt) blk = block_at(NST - 1);
    for (int t = 0; t < nt; ++t) {
        // step t's copies have landed once no more than those of the next ones are outstanding
        if (t + NST - 2 < nt) wait_vmem_n<(NST - 2) * S::LPS>();
        else wait_vmem();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        if (t + NST - 1 < nt) {
            issue(t + NST - 1, st == 0 ? NST - 1 : st - 1, blk);
            if (t + NST < nt) blk = block_at(t + NST);
        }
        const uint8_t* tile = lds.stages[st][wave][0];
        const int32_t* meta = lds.meta[wave][st];
        const int k0 = t * S::STEP + wave * TK;
        u32x2_t kw[KD];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) kw[kd] = *reinterpret_cast<const u32x2_t*>(tile + k_off[kd]);
        const float ks = __int_as_float(meta[16]), vs = __int_as_float(meta[17]);
        f32x4_t sc[CB];
        bool apart = false;   // the block's positions do not follow one another
        int64_t away = 0;     // the lane's key's position less the block's
        if constexpr (ROPE) {
            const int first = max(k_lo - k0, 0);   // (keys outside the range stand for others)
            const int32_t pos = meta[c16];
            const int64_t b = (int64_t)__builtin_amdgcn_readlane(pos, first) - first;
            away = pos - b;
            apart = __builtin_amdgcn_ballot_w64(away != c16 && c16 >= first && k0 + c16 < k_hi) != 0;
            float c, s;
            rope_cs_fast(b - first_pos, my_step, c, s);
            put_cs(lds.base[wave], my_pair, c, s);
            __atomic_signal_fence(__ATOMIC_SEQ_CST);
        }
#pragma unroll
        for (int i = 0; i < KD; ++i) {
            uint32_t xw, yw;   // codes of the x and y of 4 pairs
            u32x4_t kf;
            if (STYLE == kNeox) {
                xw = kw[i / 2][i % 2];
                yw = kw[KD / 2 + i / 2][i % 2];
            } else {
                xw = __builtin_amdgcn_perm(kw[i][1], kw[i][0], 0x06040200u);
                yw = __builtin_amdgcn_perm(kw[i][1], kw[i][0], 0x07050301u);
            }
            u32x4_t cs, bs;   // cos/sin of the keys' angles and of the queries'
            if constexpr (ROPE) {
                cs = place[i];
                if (apart) {
                    float c[4], s[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) rope_cs_fast(away, lds.fstep[4 * word_at(i) + e], c[e], s[e]);
                    cs = u32x4_t{pack_f16(c[0], c[1]), pack_f16(c[2], c[3]), pack_f16(s[0], s[1]), pack_f16(s[2], s[3])};
                }
                bs = *reinterpret_cast<const u32x4_t*>(lds.base[wave][word_at(i)]);
                const u32x4_t k = {C::halves_lo(xw), C::halves_hi(xw), C::halves_lo(yw), C::halves_hi(yw)};
                kf = turned(k, cs, false);
            } else {
                const u32x2_t xb = C::bf16s(xw), yb = C::bf16s(yw);
                kf = u32x4_t{xb[0], xb[1], yb[0], yb[1]};
            }
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const f32x4_t from = i == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[cb];
                const u32x4_t qb = *reinterpret_cast<const u32x4_t*>(lds.q[cb][i][lane]);
                if constexpr (ROPE)
                    sc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, kf), __builtin_bit_cast(f16x8_t, turned(qb, bs, true)), from, 0, 0, 0);
                else
                    sc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf), __builtin_bit_cast(bf16x8_t, qb), from, 0, 0, 0);
            }
            if (CB == 1) __builtin_amdgcn_sched_barrier(0);   // (side by side the words would take more registers than there are)
        }
        const bool masked = k0 < k_lo || k0 + TK > min(k_hi, g.tok0 + row_lo / G + 1 - kt0);   // some row may not see some key
        float mx[CB];
        bool moves = false;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            sc[cb] *= qs[cb] * ks;
            if (masked) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = k0 + 4 * q4 + r;
                    if (key < k_lo || key > last[cb]) sc[cb][r] = -INFINITY;
                }
            }
            mx[cb] = fmaxf(fmaxf(sc[cb][0], sc[cb][1]), fmaxf(sc[cb][2], sc[cb][3]));
            moves |= mx[cb] > m_run[cb] + 8.f;
        }
        // the reference maximum only moves when some row's maximum grows by more than 8
        // (probabilities stay below 2^8), so most tiles skip rescaling
        if (__builtin_amdgcn_ballot_w64(moves) != 0) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const float m_new = fmaxf(m_run[cb], max_xor32(max_xor16(mx[cb])));
                const float alpha = __builtin_amdgcn_exp2f(m_run[cb] - m_new);
                l_run[cb] *= alpha;
#pragma unroll
                for (int i = 0; i < 2 * DB; ++i) acc[cb][i] *= alpha;
                m_run[cb] = m_new;
            }
        }
        // upper and lower parts of the probabilities times the values' scale
        u32x4_t pw[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(sc[cb][r] - m_run[cb]);
            l_run[cb] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] *= vs;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pw[cb][h] = __builtin_amdgcn_perm(__float_as_uint(p[2 * h + 1]), __float_as_uint(p[2 * h]), 0x07060302u);
                pw[cb][2 + h] = pack_bf16(p[2 * h] - bf_lo(pw[cb][h]), p[2 * h + 1] - bf_hi(pw[cb][h]));
            }
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const u32x2_t both = __builtin_bit_cast(u32x2_t, lds_read_tr((lds_u16_t*)(tile + (v_off ^ (32 * db)))));
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                const u32x2_t v = C::bf16s(__builtin_amdgcn_perm(both[1], both[0], odd ? 0x07050301u : 0x06040200u));
                const u32x4_t twice = {v[0], v[1], v[0], v[1]};
#pragma unroll
                for (int cb = 0; cb < CB; ++cb)
                    acc[cb][2 * db + odd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8_t, twice), __builtin_bit_cast(bf16x8_t, pw[cb]), acc[cb][2 * db + odd], 0, 0, 0);
            }
        }
        st = st + 1 == NST ? 0 : st + 1;
    }

    // ---- the waves' results meet: a wave leaves its rows' maxima, sums and outputs (in its own part of
    // the stages, which no other wave reads before), then wave 2 db + half joins four of the eight dims that a
    // lane holds of block db
    constexpr int PPS = 2 * S::TILE / 1024;    // outputs of 16 x 16 in the place of a wave's stage
    const auto piece = [&](int w, int i) {
        return reinterpret_cast<f32x4_t*>(lds.stages[i / PPS][w][0]) + i % PPS * 64 + lane;
    };
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const float l = sum_xor32(sum_xor16(l_run[cb]));
        if (q4 == 0) mls[wave][16 * cb + c16] = make_float2(m_run[cb], l);
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) *piece(wave, cb * 2 * DB + i) = acc[cb][i];
    }
    __syncthreads();
    const int db = wave >> 1, half = wave & 1;
    if (db >= DB) return;
    const size_t prow0 = ((size_t)g.part_base + (size_t)ic.cluster * n_rt + rt) * (16 * CB);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row_lo + 16 * cb + c16;
        if (row >= rows_total) continue;
        float2 w[NW], even[NW], odd[NW];
        float M = kNegBig, den = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            w[i] = mls[i][16 * cb + c16];
            even[i] = reinterpret_cast<const float2*>(piece(i, (cb * DB + db) * 2))[half];
            odd[i] = reinterpret_cast<const float2*>(piece(i, (cb * DB + db) * 2 + 1))[half];
            M = fmaxf(M, w[i].x);
        }
        f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float f = __builtin_amdgcn_exp2f(w[i].x - M);
            den += w[i].y * f;
            x += f32x4_t{even[i].x, odd[i].x, even[i].y, odd[i].y} * f;
        }
        const int d = 32 * db + 8 * q4 + 4 * half;
        if (g.n_split > 1) {
            *reinterpret_cast<f32x4_t*>(a.part_o + (prow0 + 16 * cb + c16) * D + d) = x;
            if (wave == 0 && q4 == 0) *reinterpret_cast<float2*>(a.part_ml + (prow0 + 16 * cb + c16) * 2) = make_float2(M, den);
        } else {
            const float inv = 1.f / den;
            const int to = row / G, hl = row - to * G;
            uint16_t* op = static_cast<uint16_t*>(a.o) + ((size_t)(g.q_row0 + to) * a.hq + (size_t)ic.kvh * G + hl) * D;
            *reinterpret_cast<u32x2_t*>(op + d) = u32x2_t{pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
        }
    }
}

// ---------------------------------------------------------------------------------
// kv8_many: attention in bf16, 32 WR query rows (128 or 256) per workgroup of eight waves, in steps of 64
// keys that all waves share: WR row groups of KG = 8 / WR waves, which take 32 keys of a step at a time.
//   S^T (32 keys x 32 rows) = K Q^T       v_mfma_f32_32x32x16_f16 (bf16 without rotation)
//   O^T (32 dims x 32 rows) += V^T P^T    v_mfma_f32_32x32x16_bf16, V^T by ds_read_b64_tr_b16
// After the scores lane l holds row l%32 and keys 8 (j/4) + 4 (l/32) + j%4, the B operand of the
// output product.  A wave loads the codes of eight keys of a step into registers, a step and a half ahead, and
// turns them into float16 (keys) and bf16 (values) in LDS one step ahead, beside the products of the scores;
// two LDS buffers, one barrier per step.  LDS rows hold the x of all pairs, then the y, in either pairing.
// COPY: keys come turned from the call's copy (kv8_keys).
//
// The scales cost a few operations a step: the scores of a block's keys are multiplied in the addition that
// the exponential needs anyway, and the values' scale joins its exponent: p' = 2^(s - m + log2 v).
// The row sum adds the p' of a block, rounded to bf16 as they are multiplied, times 1 / v.  A second part of p' (kv8_few's)
// would bring outputs from 1.42 to 1.1 times the error of their own rounding and costs half as many products again: 2,048
// tokens of 64 heads over 18,432 keys 1,572 us, 1,210 without it.  float16 would bring as much for 1,250 us, but what
// of its range is left beside the row's largest p' is 2^31: a dimension in which the blocks of large values hold zeros
// would lose the others.
//
// Bound by products, vector work and LDS reads, which overlap in part: a step of 256 rows has 2,048 cycles of products and
// 2,300 of LDS, and takes about 5,100 cycles with turning (products 38%, vector unit 48% by the counters), 4,500 with
// the copy (45% and 37%).  2,048 tokens of 64 / 8 heads of 128 over 18,432 keys of int8: 1,142 to 1,225 us by the card with the copy, 954
// to 1,023 TFLOP/s; on one of them 1,204 with it, 1,350 without it, and 1,160 on a pool of turned keys.
// ---------------------------------------------------------------------------------
constexpr float kLeastValueScale = 0x1p-90f;   // (p' of 2^-36 and more stay above the type's least)

// Steps after which angles are computed again.  A pair's cos/sin start within 2^-22.4 (rope_cs_fast, as a vector), and an advance
// adds the stride's own error, 2^-23.7 at most, and two roundings of each, 2^-23.5: within 2^-17.5 after 32.
constexpr int kKv8Renew = 32;

template <int D>
struct __attribute__((aligned(2 * D))) Kv8ManyLds {
    uint16_t kv[2][2][64 * D];   // [buffer][keys, values], 16-byte chunks swizzled by key
    float2 stride_cs[D / 2];     // cos/sin of 64 positions
    uint64_t fstep[D / 2];
    float4 sc[2][4];             // per block of a step: its keys' scale, log2 and inverse of its values' scale
};

// The products of a wave's scores of a step: KD of each of its NT times 32 keys
template <int D, int WR>
struct Kv8Many {
    static constexpr int KG = kKv8Waves / WR, NT = 2 / KG;
    static constexpr int KD = D / 16;                  // 32x32x16 contraction steps of QK^T
    static constexpr int TAKEN = KD * NT;
    static constexpr int AHEAD = TAKEN < 5 ? TAKEN : 5;   // K reads in flight
};

template <int D, int STYLE, bool ROPE, bool COPY, int CODE, int WR, int NG>
__global__ void __launch_bounds__(kKv8Waves * 64, 2) kv8_many(const PlanOf<NG> plan, const Kv8Args a) {
    typedef Code<CODE> C;
    typedef Kv8Many<D, WR> S;
    constexpr int NW = kKv8Waves, KG = S::KG, KD = S::KD, STEP = 64, HALF = D / 2;
    constexpr int DB = D / 32;             // 32-dim blocks of O^T
    constexpr int PL = D / 16;             // pairs that a lane turns
    constexpr int KW = PL / (COPY ? 2 : 4), VW = D / 32;   // words of a lane: either run of its key (of the copy: in float16), its value
    static_assert(ROPE || !COPY, "a copy holds turned keys");
    static_assert(KG == 1 || KG == 2, "a step has two times 32 keys");

    __shared__ Kv8ManyLds<D> lds;
    __shared__ float2 mls[NW][32];
    static_assert(sizeof(lds.kv) >= NW * 16 * HALF * 8, "the queries' angles pass through the buffers");
    static_assert(sizeof(lds.kv) >= NW * DB * 2 * 64 * 16, "the outputs meet in the buffers");

    const Group g = find_group<false>(plan, blockIdx.x);
    const int G = a.group, n_rt = COPY ? row_tiles(g, G, 32 * WR) : g.n_rt;
    const int li = blockIdx.x - g.item_base;   // (a call's items are not padded: below the group's count)
    const ItemCoords ic = item_coords(g, a.hkv, n_rt, li);
    const int rt = n_rt - 1 - ic.rt;           // the longest first
    const int rows_total = g.n_tok * G, tile_lo = rt * 32 * WR;
    const int t_last = g.tok0 + (min(tile_lo + 32 * WR, rows_total) - 1) / G;
    const int kv_lo = g.win + ic.split * g.split_keys;
    if (kv_lo > t_last) return;                // (the row tile's splits end before this one)
    // (no sum below passes the last key: a request may have 2^31 - 1 of them)
    const int kv_hi = g.split_keys < t_last + 1 - kv_lo ? kv_lo + g.split_keys : t_last + 1;
    const int kt0 = kv_lo & ~(kBlock - 1);
    const int k_lo = kv_lo - kt0, k_hi = kv_hi - kt0;   // the range from the start of its first block
    const int nt = (k_hi - 1) / STEP + 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rg = wave / KG, kg = wave % KG, l32 = lane & 31, hi = lane >> 5;
    const int row_lo = tile_lo + rg * 32;
    const int32_t* btab = a.block_tables + (size_t)g.req * a.max_blocks + (kt0 >> 4);
    const int32_t* posv = a.positions + g.pos_off + kt0;
    const size_t page = (size_t)kBlock * D;
    const uint8_t* kpool = static_cast<const uint8_t*>(a.k_pool) + ic.kvh * page;
    const uint8_t* vpool = static_cast<const uint8_t*>(a.v_pool) + ic.kvh * page;

    // ---- the lane's part of a step's codes: of key own (of the step) pairs pair0 .. pair0 + PL - 1, and the values
    // of chunks sub and (D 128) sub + 8.  (The keys' order lets 16 neighbouring lanes write all LDS banks: at D 128
    // the rows of keys that differ in bit 1 lie in different halves of the swizzled chunks.)
    const int l8 = lane >> 3, sub = lane & 7, pair0 = sub * PL;
    const int own = wave * 8 + (D == 128 ? (l8 & 4) | ((l8 & 1) << 1) | ((l8 >> 1) & 1) : l8);
    int k_el[2];   // its two runs in a row: NeoX its x and its y, GPT-J one after the other, the copy x and y
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int e = COPY || STYLE == kNeox ? pair0 + h * HALF : 2 * pair0 + h * PL;
        k_el[h] = COPY ? e : model_chunk(a.chunk_map, e >> 3) * 8 + (e & 7);
    }
    const uint16_t* copy = COPY ? static_cast<const uint16_t*>(a.k_rot) + ((size_t)(g.krot0 + (kt0 >> 4)) * a.hkv + ic.kvh) * page : nullptr;
    typedef uint32_t run_t __attribute__((ext_vector_type(KW)));
    struct Raw {
        uint32_t k[2][KW], v[VW];
        int32_t pos;
        float ks, vs;
    };
    // Sets of codes on their way: one, a step and a half ahead, or with the copy, whose angles take no registers, two (the
    // call above 1,224 -> 1,204 us; without rotation 1,160 -> 1,152, but 42.3 -> 43.2 for 250 tokens over 5,376 keys: one)
    constexpr int SETS = COPY ? 2 : 1;
    Raw raw[SETS];
    auto block_at = [&](int u) { return scalar_load(btab, min(u * STEP + wave * 8, k_hi - 1) >> 4); };
    int blk = block_at(0);
    const int own_row = (wave * 8 & (kBlock - 1)) + own - wave * 8;   // of the key in its block
    const size_t blk_stride = (size_t)a.hkv * page;
    auto load = [&](int u, auto set) {
        if (u >= nt) return;
        Raw& r = raw[decltype(set)::value];
        // a key outside the range stands for the nearest one inside, so that nothing outside it is read
        int k = u * STEP + own, to_row = own_row * D;
        if (u * STEP < k_lo || (u + 1) * STEP > k_hi) {
            k = min(max(k, k_lo), k_hi - 1);
            to_row = (k & (kBlock - 1)) * D;
        }
        const size_t at = (size_t)(uint32_t)blk * blk_stride;
        const uint8_t* kp = kpool + at;
        const uint8_t* vp = vpool + at;
        const uint16_t* cp = COPY ? copy + (size_t)(uint32_t)(min(u * STEP + wave * 8, k_hi - 1) >> 4) * blk_stride : nullptr;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t from = (uint32_t)(to_row + k_el[h]);
            const run_t w = *(COPY ? reinterpret_cast<const run_t*>(cp + from) : reinterpret_cast<const run_t*>(kp + from));
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                if constexpr (KW == 1) r.k[h][i] = w[0];
                else r.k[h][i] = w[i];
            }
        }
#pragma unroll
        for (int h = 0; h < VW / 2; ++h) {
            const u32x2_t w = *reinterpret_cast<const u32x2_t*>(vp + (uint32_t)(to_row + (sub + 8 * h) * 8));
            r.v[2 * h] = w[0];
            r.v[2 * h + 1] = w[1];
        }
        if (ROPE && !COPY) r.pos = posv[(uint32_t)k];
        const int32_t* sp = reinterpret_cast<const int32_t*>(a.scale) + ((size_t)(uint32_t)blk * a.hkv + ic.kvh) * 2;
        r.ks = __int_as_float(scalar_load(sp, 0));
        r.vs = __int_as_float(scalar_load(sp, 1));
        if (u + 1 < nt) blk = block_at(u + 1);
    };
    load(0, Idx<0>{});
    if constexpr (SETS > 1) load(1, Idx<1>{});
    if (ROPE)
        for (int i = threadIdx.x; i < HALF; i += NW * 64) {
            lds.fstep[i] = a.fstep[i];
            if (!COPY) rope_cs(STEP, a.fstep[i], lds.stride_cs[i].x, lds.stride_cs[i].y);   // (its error comes again with every advance)
        }

    // ---- queries.  The cos/sin of their tokens (a token's heads share them) pass through the wave's
    // part of the buffers, which holds 16 tokens: more take two times 16 rows.
    const int row = row_lo + l32;
    const bool valid = row < rows_total;
    const int toff = valid ? row / G : 0, hl = valid ? row - toff * G : 0;
    const int last = min(k_hi - 1, g.tok0 + toff - kt0);   // last key that the row sees, from kt0
    u32x4_t qb[KD];
    float qs = a.scale_log2;   // the products times this and the block's scale are scores (log2 units)
    {
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((size_t)(g.q_row0 + toff) * a.hq + (size_t)ic.kvh * G + hl) * D;
        u32x4_t in[KD / 2][2];   // chunks 2 kd + hi of the pairs
#pragma unroll
        for (int kd = 0; kd < KD / 2; ++kd)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = 2 * kd + hi;
                in[kd][h] = *reinterpret_cast<const u32x4_t*>(qp + model_chunk(a.chunk_map, STYLE == kNeox ? c + h * (D / 16) : 2 * c + h) * 8);
                if (!valid) in[kd][h] = u32x4_t{0, 0, 0, 0};
            }
        __syncthreads();  // phase steps staged
        float x[HALF / 2], y[HALF / 2];   // of pairs 8 c .. 8 c + 7, c = 2 kd + hi for kd < KD / 2
#pragma unroll
        for (int kd = 0; kd < KD / 2; ++kd) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t wx = STYLE == kNeox ? in[kd][0][e / 2] : in[kd][e / 4][e % 4], wy = STYLE == kNeox ? in[kd][1][e / 2] : wx;
                x[8 * kd + e] = STYLE == kNeox && e % 2 ? bf_hi(wx) : bf_lo(wx);
                y[8 * kd + e] = STYLE == kNeox && e % 2 == 0 ? bf_lo(wy) : bf_hi(wy);
            }
        }
        if (ROPE) {
            float2* cs = reinterpret_cast<float2*>(&lds.kv[0][0][0]) + wave * 16 * HALF;
            float big = 0.f;
            const int each = min(row_lo + 31, rows_total - 1) / G - min(row_lo, rows_total - 1) / G < 16 ? 32 : 16;
#pragma unroll 1
            for (int h = 0; h < 32; h += each) {
                const int t0 = min(row_lo + h, rows_total - 1) / G, t1 = min(row_lo + h + each - 1, rows_total - 1) / G;
                const int32_t pos = a.positions[g.pos_off + g.tok0 + min(t0 + (lane & 15), t1)];   // of token t0 + lane
                const uint64_t step = lds.fstep[lane % HALF];
                for (int i = lane; i < (t1 - t0 + 1) * HALF; i += 64) {
                    float c, s;
                    rope_cs_fast(__shfl(pos, i / HALF), step, c, s);
                    cs[i] = make_float2(c, s);
                }
                __atomic_signal_fence(__ATOMIC_SEQ_CST);
                if (l32 >= h && l32 < h + each) {
                    const float2* tc = cs + (valid ? toff - t0 : 0) * HALF;
#pragma unroll
                    for (int i = 0; i < HALF / 2; ++i) {
                        const float2 t = tc[(2 * (i / 8) + hi) * 8 + i % 8];
                        const float x0 = x[i], y0 = y[i];
                        x[i] = x0 * t.x - y0 * t.y;
                        y[i] = y0 * t.x + x0 * t.y;
                        big = fmaxf(big, fmaxf(fabsf(x[i]), fabsf(y[i])));
                    }
                }
                __atomic_signal_fence(__ATOMIC_SEQ_CST);
            }
            const int ex = query_exponent(max_xor32(big));
            qs = ldexpf(qs, ex);
#pragma unroll
            for (int i = 0; i < HALF / 2; ++i) {
                x[i] = ldexpf(x[i], -ex);
                y[i] = ldexpf(y[i], -ex);
            }
        }
#pragma unroll
        for (int kd = 0; kd < KD / 2; ++kd)
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const int i = 8 * kd + 2 * m;
                qb[kd][m] = ROPE ? pack_f16(x[i], x[i + 1]) : pack_bf16(x[i], x[i + 1]);
                qb[kd + KD / 2][m] = ROPE ? pack_f16(y[i], y[i + 1]) : pack_bf16(y[i], y[i + 1]);
            }
    }
    barrier_keep_vmem();   // the angles have been read: the buffers may be filled

    // ---- codes into an LDS buffer, in parts that stand beside other work
    float rc[PL], rs[PL];      // cos/sin of the lane's pairs at position cs_pos
    int32_t cs_pos = 0;
    int renew = 0;             // steps until they are computed again
    const int t_chunk[2] = {(pair0 >> 3), (pair0 >> 3) + HALF / 8};   // of the turned runs, x and y
    auto at_lds = [&](int kv, int buf, int chunk) { return &lds.kv[buf][kv][own * D + ((chunk ^ dswz<D>(own & 15)) << 3)]; };
    constexpr int PARTS = PL / 2 + VW / 2;
    uint32_t turned[2][PL / 2];
    auto angles = [&]() {
        if (!ROPE || COPY) return;
        const int32_t pos = raw[0].pos;
        // (STEP on, and not past the type's end)
        if (renew == 0 || __builtin_amdgcn_ballot_w64((uint32_t)pos != (uint32_t)cs_pos + STEP || pos < cs_pos) != 0) {
#pragma unroll
            for (int i = 0; i < PL; ++i) rope_cs_fast((int64_t)pos - STEP, lds.fstep[pair0 + i], rc[i], rs[i]);
            renew = kKv8Renew;
        }
        --renew;
        cs_pos = pos;
    };
    auto part = [&](int buf, int i, auto set) {
        const Raw& r = raw[decltype(set)::value];
        if (i < PL / 2) {   // pairs 2 i and 2 i + 1
            const int w = i / 2, h = i % 2;
            uint32_t xw, yw;
            if constexpr (COPY) {
                xw = r.k[0][i];
                yw = r.k[1][i];
            } else if (STYLE == kNeox) {
                xw = r.k[0][w];
                yw = r.k[1][w];
            } else {   // neighbours: word 2 w and 2 w + 1 of the lane's words
                const uint32_t a0 = r.k[2 * w / KW][2 * w % KW], a1 = r.k[(2 * w + 1) / KW][(2 * w + 1) % KW];
                xw = __builtin_amdgcn_perm(a1, a0, 0x06040200u);
                yw = __builtin_amdgcn_perm(a1, a0, 0x07050301u);
            }
            if constexpr (COPY) {
                turned[0][i] = xw;
                turned[1][i] = yw;
            } else if constexpr (ROPE) {
#pragma unroll
                for (int p = 2 * i; p < 2 * i + 2; ++p) {
                    const float2 d = lds.stride_cs[pair0 + p];
                    const float c = rc[p], s = rs[p];
                    rc[p] = c * d.x - s * d.y;
                    rs[p] = s * d.x + c * d.y;
                }
                const uint32_t xb = h ? C::halves_hi(xw) : C::halves_lo(xw), yb = h ? C::halves_hi(yw) : C::halves_lo(yw);
                const f16x2_t x = __builtin_bit_cast(f16x2_t, xb), y = __builtin_bit_cast(f16x2_t, yb);
                const f16x2_t c = __builtin_bit_cast(f16x2_t, pack_f16(rc[2 * i], rc[2 * i + 1])), s = __builtin_bit_cast(f16x2_t, pack_f16(rs[2 * i], rs[2 * i + 1]));
                turned[0][i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(x, c, -(y * s)));
                turned[1][i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(y, c, x * s));
            } else {
                const u32x2_t xb = C::bf16s(xw), yb = C::bf16s(yw);
                turned[0][i] = xb[h];
                turned[1][i] = yb[h];
            }
            if (i == PL / 2 - 1) {
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    typedef uint32_t out_t __attribute__((ext_vector_type(PL / 2)));
                    out_t o;
#pragma unroll
                    for (int j = 0; j < PL / 2; ++j) o[j] = turned[z][j];
                    *reinterpret_cast<out_t*>(at_lds(0, buf, t_chunk[z]) + (pair0 & 7)) = o;
                }
                if (lane == 0 && (wave & 1) == 0) {
                    const float v = fmaxf(r.vs, kLeastValueScale);
                    lds.sc[buf][wave >> 1] = make_float4(r.ks, __builtin_amdgcn_logf(v), 1.f / v, 0.f);
                }
            }
        } else {   // a chunk of values
            const int h = i - PL / 2;
            const u32x2_t lo = C::bf16s(r.v[2 * h]), hi2 = C::bf16s(r.v[2 * h + 1]);
            *reinterpret_cast<u32x4_t*>(at_lds(1, buf, sub + 8 * h)) = u32x4_t{lo[0], lo[1], hi2[0], hi2[1]};
        }
    };

    f32x16_t acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = f32x16_t{};
    float m_run = kNegBig, l_run = 0.f;
    // per-lane byte offsets: the K operand's row among 32 keys, the V^T operand's among 8 (chunk c,
    // and the row 8 keys on, by xor)
    constexpr int kSw8 = D == 128 ? 1 : 4;
    uint32_t k_at = (uint32_t)(l32 * D + ((hi ^ dswz<D>(l32 & 15)) << 3)) * 2, v_at;
    {
        const int key = 4 * hi + ((lane & 15) >> 2), d = ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
        v_at = (uint32_t)(64 * D + key * D + (((d >> 3) ^ dswz<D>(key)) << 3) + (d & 7)) * 2;
    }
    const uint32_t lds_at = lds_addr(&lds.kv[0][0][0]);
    const int first_row_last = min(k_hi - 1, g.tok0 + min(row_lo, rows_total - 1) / G - kt0);   // last key that every row sees
    typedef __attribute__((address_space(3))) const u32x4_t lds_u32x4_t;

    constexpr int NT = S::NT, TAKEN = S::TAKEN, kAhead = S::AHEAD;
    static_assert(kAhead >= 1 && kAhead <= TAKEN, "no read past a step's operands");
    // ---- step s, in buffer P = s % 2, and the codes of the next step
    auto step = [&](int s, int P, auto set) {
        // (the offsets are not kept apart for every chunk: registers are short)
        asm volatile("" : "+v"(k_at), "+v"(v_at));
        const uint32_t at = lds_at + (uint32_t)(P * 128 * D + 32 * kg * D) * 2, kt = at + k_at, vt = at + v_at;
        u32x4_t kf[TAKEN];
        auto read_k = [&](int i) { kf[i] = *(lds_u32x4_t*)(uintptr_t)((kt ^ (32 * (i / NT))) + 64 * (i % NT) * D); };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read_k(i);
        float4 bs[2 * NT];
        if (s + 1 < nt) angles();
        f32x16_t sc[NT];
        __builtin_amdgcn_sched_barrier(0);
        // Every few vector instructions follow a product that they do not wait for, in the order written (past
        // the last step they turn what the registers hold, into a buffer that is not read again)
#pragma unroll
        for (int i = 0; i < TAKEN; ++i) {
            const int kd = i / NT, n = i % NT;
            const f32x16_t from = kd == 0 ? f32x16_t{} : sc[n];
            if (ROPE)
                sc[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, kf[i]), __builtin_bit_cast(f16x8_t, qb[kd]), from, 0, 0, 0);
            else
                sc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[i]), __builtin_bit_cast(bf16x8_t, qb[kd]), from, 0, 0, 0);
            if (i + kAhead < TAKEN) read_k(i + kAhead);
#pragma unroll
            for (int j = i * PARTS / TAKEN; j < (i + 1) * PARTS / TAKEN; ++j) part(1 - P, j, set);
            if (i == TAKEN - 2)
#pragma unroll
                for (int b = 0; b < 2 * NT; ++b) bs[b] = lds.sc[P][2 * kg + b];
            __builtin_amdgcn_sched_barrier(0);
        }
        load(s + 1 + SETS, set);
        float mul[2 * NT], add[2 * NT];   // of a block's scores and of their exponents
        float mx = kNegBig;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int k0 = s * STEP + 32 * (kg + n);
            if (k0 < k_lo || k0 + 31 > first_row_last) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int key = k0 + 8 * (j >> 2) + 4 * hi + (j & 3);
                    if (key < k_lo || key > last) sc[n][j] = -INFINITY;
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float bm = sc[n][8 * h];
#pragma unroll
                for (int j = 1; j < 8; ++j) bm = fmaxf(bm, sc[n][8 * h + j]);
                mul[2 * n + h] = fmaxf(qs * bs[2 * n + h].x, 0x1p-149f);   // (not 0, with which a masked -Inf would be NaN)
                mx = fmaxf(mx, bm * mul[2 * n + h]);
            }
        }
        // the reference maximum only moves when some row's maximum grows by more than 8
        // (probabilities stay below 2^8), so most steps skip rescaling
        if (__builtin_amdgcn_ballot_w64(mx > m_run + 8.f) != 0) {
            const float m_new = fmaxf(m_run, max_xor32(mx));
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] *= alpha;
            m_run = m_new;
        }
#pragma unroll
        for (int b = 0; b < 2 * NT; ++b) add[b] = bs[b].y - m_run;
        // ---- outputs, 16 keys (a block) at a time, with the next 16's probabilities and V reads beside
        constexpr int NH = 2 * NT;
        u32x4_t pw[2];               // probabilities times the values' scale, in bf16; the row sum adds exactly those
        u32x2_t af[2][2 * DB];
        float bsum = 0.f;
        // part i of DB of the probabilities of block h
        auto prob = [&](int h, int i) {
            constexpr int E = 8 / DB;
            if (i == 0) bsum = 0.f;
#pragma unroll
            for (int r = i * E; r < (i + 1) * E; r += 2) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[h / 2][8 * (h % 2) + r], mul[h], add[h]));
                const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[h / 2][8 * (h % 2) + r + 1], mul[h], add[h]));
                const uint32_t w = pack_bf16(x, y);
                pw[h % 2][r / 2] = w;
                bsum = sum2_bf16(w, bsum);
            }
            if (i == DB - 1) l_run = __builtin_fmaf(bsum, bs[h].z, l_run);
        };
        // V reads of block i of the dimensions
        auto read_v = [&](int h, int i) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {   // 8 keys each
                const uint32_t off = (vt ^ (uint32_t)(64 * i) ^ (e ? 16u * kSw8 : 0u)) + 32 * h * D + (e ? 16 * D : 0);
                af[h % 2][2 * i + e] = __builtin_bit_cast(u32x2_t, lds_read_tr((lds_u16_t*)(uintptr_t)off));
            }
        };
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            read_v(0, i);
            prob(0, i);
        }
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                const u32x4_t v = {af[h % 2][2 * i][0], af[h % 2][2 * i][1], af[h % 2][2 * i + 1][0], af[h % 2][2 * i + 1][1]};
                acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, pw[h % 2]), acc[i], 0, 0, 0);
                if (h + 1 < NH) {
                    read_v(h + 1, i);
                    prob(h + 1, i);
                }
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    // the codes of step u alone (also: of a wave without rows)
    auto only_codes = [&](int u, int buf, auto set) {
        if (u < nt) {
            angles();
#pragma unroll
            for (int i = 0; i < PARTS; ++i) part(buf, i, set);
        }
        load(u + SETS, set);
    };
    only_codes(0, 0, Idx<0>{});
    barrier_keep_vmem();
    const bool rows = row_lo < rows_total;
    // (the codes of step s + 1 are in set (s + 1) % SETS)
    auto one = [&](int s, int P, auto set) {
        if (rows) step(s, P, set);
        else only_codes(s + 1, 1 - P, set);
        barrier_keep_vmem();
    };
    if constexpr (SETS > 1) {
        for (int s = 0; s < nt; s += 2) {
            one(s, 0, Idx<1>{});
            if (s + 1 < nt) one(s + 1, 1, Idx<0>{});
        }
    } else {
        for (int s = 0; s < nt; ++s) one(s, s & 1, Idx<0>{});
    }

    // ---- the results of a row group's waves meet: rows by their common maximum, outputs through the buffers
    float den = sum_xor32(l_run), M = m_run, mine = 1.f;
    if constexpr (KG > 1) {
        if (hi == 0) mls[wave][l32] = make_float2(m_run, den);
        __syncthreads();
        const float2 other = mls[wave ^ 1][l32];
        M = fmaxf(m_run, other.x);
        mine = __builtin_amdgcn_exp2f(m_run - M);
        den = den * mine + other.y * __builtin_amdgcn_exp2f(other.x - M);
    }
    f32x4_t* meet = reinterpret_cast<f32x4_t*>(&lds.kv[0][0][0]);
    f32x4_t out[DB * 4];   // dims 8 c + 4 (l/32) + {0..3}
#pragma unroll
    for (int c = 0; c < DB * 4; ++c) {
        const f32x4_t x = {acc[c / 4][4 * (c % 4)], acc[c / 4][4 * (c % 4) + 1], acc[c / 4][4 * (c % 4) + 2], acc[c / 4][4 * (c % 4) + 3]};
        out[c] = x * mine;
    }
    if constexpr (KG > 1) {   // a wave leaves the half of its outputs that the other one joins
#pragma unroll
        for (int c = 0; c < DB * 4; ++c)
            if (c % 2 != kg) meet[(wave * DB * 2 + c / 2) * 64 + lane] = out[c];
        __syncthreads();
    }
    if (row >= rows_total) return;
    const size_t prow = ((size_t)g.part_base + (size_t)ic.cluster * n_rt + rt) * (32 * WR) + rg * 32 + l32;
    const float inv = 1.f / den;
    uint16_t* op = static_cast<uint16_t*>(a.o) + ((size_t)(g.q_row0 + toff) * a.hq + (size_t)ic.kvh * G + hl) * D;
#pragma unroll
    for (int c = 0; c < DB * 4; ++c) {
        if (KG > 1 && c % 2 != kg) continue;
        f32x4_t x = out[c];
        if (KG > 1) x += meet[((wave ^ 1) * DB * 2 + c / 2) * 64 + lane];
        const int d = 8 * c + 4 * hi;
        if (g.n_split > 1) *reinterpret_cast<f32x4_t*>(a.part_o + prow * D + d) = x;
        else *reinterpret_cast<u32x2_t*>(op + d) = u32x2_t{pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
    }
    if (g.n_split > 1 && kg == 0 && hi == 0) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(M, den);
}

// ---------------------------------------------------------------------------------
// kv8_keys: the call's copy of the keys that its queries see, turned, in float16: codes times cos/sin (the scales stay
// beside the pool's blocks), rounded once, the x of all pairs of a key and then the y.  Blocks in the order of the sequences.
// One workgroup per block: 8 lanes per key (D / 16 pairs each), every second KV head.  Bound by memory: each key read
// once and written twice as wide (18,432 keys of 8 heads of 128, 57 MB, in 13.0 us).
// ---------------------------------------------------------------------------------
template <int D, int STYLE, int CODE>
__global__ void __launch_bounds__(256) kv8_keys(const KeyPlan plan, const Kv8Args a) {
    typedef Code<CODE> C;
    constexpr int HALF = D / 2, PL = D / 16, KW = PL / 4, U = 4;
    typedef uint32_t run_t __attribute__((ext_vector_type(KW)));
    typedef uint32_t out_t __attribute__((ext_vector_type(PL / 2)));
    int lo = 0, up = plan.n - 1;
    while (lo < up) {
        const int mid = (lo + up + 1) >> 1;
        if (plan.seg[mid].blk0 <= (int)blockIdx.x) lo = mid;
        else up = mid - 1;
    }
    const KeySegment sg = plan.seg[lo];
    const int kb = (sg.lo >> 4) + (int)blockIdx.x - sg.blk0;   // block of the sequence
    const int key = ((int)threadIdx.x >> 3) & 15, pair0 = ((int)threadIdx.x & 7) * PL;
    const int64_t j = (int64_t)kb * kBlock + key;
    if (j < sg.lo || j >= sg.hi) return;                       // no query sees it
    const int32_t blk = a.block_tables[(size_t)sg.req * a.max_blocks + kb];
    const int32_t pos = a.positions[sg.pos_off + j];
    int el[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int e = STYLE == kNeox ? pair0 + h * HALF : 2 * pair0 + h * PL;
        el[h] = key * D + model_chunk(a.chunk_map, e >> 3) * 8 + (e & 7);
    }
    const uint8_t* kp = static_cast<const uint8_t*>(a.k_pool) + (size_t)(uint32_t)blk * a.hkv * kBlock * D;
    uint16_t* op = static_cast<uint16_t*>(const_cast<void*>(a.k_rot)) + (size_t)blockIdx.x * a.hkv * kBlock * D + key * D + pair0;
    float c[PL], s[PL];
#pragma unroll
    for (int i = 0; i < PL; ++i) rope_cs_fast(pos, a.fstep[pair0 + i], c[i], s[i]);
    // KV heads hp, hp + 2, ..: the loads of four go out together
    for (int h0 = (int)threadIdx.x >> 7; h0 < a.hkv; h0 += 2 * U) {
        uint32_t w[U][2 * KW];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const run_t in = *reinterpret_cast<const run_t*>(kp + (size_t)min(h0 + 2 * u, a.hkv - 1) * kBlock * D + el[h]);
#pragma unroll
                for (int i = 0; i < KW; ++i) {
                    if constexpr (KW == 1) w[u][h] = in[0];
                    else w[u][h * KW + i] = in[i];
                }
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (h0 + 2 * u >= a.hkv) continue;
            out_t ox, oy;
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                uint32_t xw, yw;
                if (STYLE == kNeox) {
                    xw = w[u][i];
                    yw = w[u][KW + i];
                } else {
                    xw = __builtin_amdgcn_perm(w[u][2 * i + 1], w[u][2 * i], 0x06040200u);
                    yw = __builtin_amdgcn_perm(w[u][2 * i + 1], w[u][2 * i], 0x07050301u);
                }
                const f32x4_t x = C::decode(xw), y = C::decode(yw);
                float tx[4], ty[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    tx[e] = x[e] * c[4 * i + e] - y[e] * s[4 * i + e];
                    ty[e] = y[e] * c[4 * i + e] + x[e] * s[4 * i + e];
                }
                ox[2 * i] = pack_f16(tx[0], tx[1]);
                ox[2 * i + 1] = pack_f16(tx[2], tx[3]);
                oy[2 * i] = pack_f16(ty[0], ty[1]);
                oy[2 * i + 1] = pack_f16(ty[2], ty[3]);
            }
            uint16_t* row = op + (size_t)(h0 + 2 * u) * kBlock * D;
            *reinterpret_cast<out_t*>(row) = ox;
            *reinterpret_cast<out_t*>(row + HALF) = oy;
        }
    }
}

template <int D>
void launch_keys_d(int style, const KeyPlan& plan, const Kv8Args& a, hipStream_t st) {
    const auto go = [&](auto s, auto c) {
        hipLaunchKernelGGL((kv8_keys<D, decltype(s)::value, decltype(c)::value>), dim3(plan.n_blocks), dim3(256), 0, st, plan, a);
    };
    if (a.code == kCodeE4m3) style == kNeox ? go(Idx<0>{}, Idx<kCodeE4m3>{}) : go(Idx<1>{}, Idx<kCodeE4m3>{});
    else style == kNeox ? go(Idx<0>{}, Idx<kCodeInt8>{}) : go(Idx<1>{}, Idx<kCodeInt8>{});
}

// Joins key splits: one block per kMergeRows rows of a (row tile, KV head), one float4 of a row per
// thread, U splits' loads in flight.  A row tile has splits up to its last token's.
struct Kv8MergeArgs {
    const float* part_o;
    const float* part_ml;
    void* o;
    int32_t tile_rows, hq, hkv, group;
    bool copied;   // the groups hold where their keys' copy begins
};

template <int D, int NG, int U>
__global__ void __launch_bounds__(kMergeRows * D / 4) kv8_merge(const PlanOf<NG> plan, const Kv8MergeArgs a) {
    constexpr int TPR = D / 4;
    const Group g = find_group<true>(plan, blockIdx.x);
    const int n_rt = a.copied ? row_tiles(g, a.group, a.tile_rows) : g.n_rt, chunks = a.tile_rows / kMergeRows;
    int li = blockIdx.x - g.merge_base;   // (only groups with splits have blocks here, and no more than they need)
    const int r = (li % chunks) * kMergeRows + (int)threadIdx.x / TPR, c4 = (int)threadIdx.x % TPR;
    li /= chunks;
    const int kvh = li / n_rt, rt = li - kvh * n_rt, G = a.group;
    const int row = rt * a.tile_rows + r, rows_total = g.n_tok * G;
    if (row >= rows_total) return;
    const int t_last = g.tok0 + (min((rt + 1) * a.tile_rows, rows_total) - 1) / G;
    const int n_live = min(g.n_split, (t_last - g.win) / g.split_keys + 1);
    const size_t slot0 = (size_t)g.part_base + (size_t)kvh * g.n_split * n_rt + rt;
    float M = kNegBig, den = 0.f;
    f32x4_t num = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n_live; s0 += U) {
        float2 ml[U];
        f32x4_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t prow = (slot0 + (size_t)min(s0 + u, n_live - 1) * n_rt) * a.tile_rows + r;
            ml[u] = *reinterpret_cast<const float2*>(a.part_ml + prow * 2);
            v[u] = *reinterpret_cast<const f32x4_t*>(a.part_o + prow * D + c4 * 4);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u >= n_live || ml[u].y == 0.f) continue;   // past the end, or no key of this row
            const float m_new = fmaxf(M, ml[u].x);
            const float c_old = __builtin_amdgcn_exp2f(M - m_new), c_new = __builtin_amdgcn_exp2f(ml[u].x - m_new);
            num = num * c_old + c_new * v[u];
            den = den * c_old + c_new * ml[u].y;
            M = m_new;
        }
    }
    const float inv = 1.f / den;
    const int to = row / G;
    uint16_t* op = static_cast<uint16_t*>(a.o) + ((size_t)(g.q_row0 + to) * a.hq + (size_t)kvh * G + (row - to * G)) * D + c4 * 4;
    *reinterpret_cast<u32x2_t*>(op) = u32x2_t{pack_bf16(num[0] * inv, num[1] * inv), pack_bf16(num[2] * inv, num[3] * inv)};
}

template <int D, int STYLE, bool ROPE, bool COPY, int CODE, int NG>
hipError_t launch_kv8_n(const PlanOf<NG>& plan, const Kv8Args& a, hipStream_t st) {
    const dim3 grid(plan.n_items), block(kKv8Waves * 64);
    if (a.tile_rows <= 32) {
        if constexpr (!COPY) {
            if (a.tile_rows == 16) hipLaunchKernelGGL((kv8_few<D, STYLE, ROPE, CODE, 1, NG>), grid, block, 0, st, plan, a);
            else hipLaunchKernelGGL((kv8_few<D, STYLE, ROPE, CODE, 2, NG>), grid, block, 0, st, plan, a);
        }
    } else if (a.tile_rows == 128) {
        hipLaunchKernelGGL((kv8_many<D, STYLE, ROPE, COPY, CODE, 4, NG>), grid, block, 0, st, plan, a);
    } else {
        hipLaunchKernelGGL((kv8_many<D, STYLE, ROPE, COPY, CODE, 8, NG>), grid, block, 0, st, plan, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.n_merge == 0) return e;
    const Kv8MergeArgs m = {a.part_o, a.part_ml, a.o, a.tile_rows, a.hq, a.hkv, a.group, COPY};
    const dim3 merges(plan.n_merge), threads(kMergeRows * D / 4);
    if (a.tile_rows <= 32) hipLaunchKernelGGL((kv8_merge<D, NG, 8>), merges, threads, 0, st, plan, m);
    else hipLaunchKernelGGL((kv8_merge<D, NG, 4>), merges, threads, 0, st, plan, m);
    return hipGetLastError();
}

template <int D, int STYLE, bool ROPE, bool COPY, int CODE>
hipError_t launch_kv8_t(const Plan& plan, const Kv8Args& a, hipStream_t st) {
    if (plan.n_groups > kFewGroups) return launch_kv8_n<D, STYLE, ROPE, COPY, CODE, kMaxGroups>(plan, a, st);
    PlanOf<kFewGroups> few = {plan.n_groups, plan.n_items, plan.n_merge, plan.merge_ways, plan.table, plan.item_map, plan.merge_map, {}};
    for (int i = 0; i < plan.n_groups; ++i) few.g[i] = plan.g[i];
    return launch_kv8_n<D, STYLE, ROPE, COPY, CODE, kFewGroups>(few, a, st);
}

template <int D, int CODE>
hipError_t launch_kv8_d(int style, bool rope, const Plan& plan, const Kv8Args& a, hipStream_t st) {
    if (!rope) return launch_kv8_t<D, 0, false, false, CODE>(plan, a, st);   // (without rotation the pairing makes no difference)
    if (a.k_rot != nullptr) return style == kNeox ? launch_kv8_t<D, 0, true, true, CODE>(plan, a, st) : launch_kv8_t<D, 1, true, true, CODE>(plan, a, st);
    return style == kNeox ? launch_kv8_t<D, 0, true, false, CODE>(plan, a, st) : launch_kv8_t<D, 1, true, false, CODE>(plan, a, st);
}

template <typename T, int D>
void launch_norm_d(int style, int n, int threads, const NormArgs& a, hipStream_t st) {
    if (a.rot_half == 0)
        hipLaunchKernelGGL((qk_norm_kernel<T, D, 1, false>), dim3(n), dim3(threads), 0, st, a);
    else if (style == kNeox)
        hipLaunchKernelGGL((qk_norm_kernel<T, D, 0, true>), dim3(n), dim3(threads), 0, st, a);
    else
        hipLaunchKernelGGL((qk_norm_kernel<T, D, 1, true>), dim3(n), dim3(threads), 0, st, a);
}

// f(type, head_dim, code) with the values as constants
template <typename F>
void by_types(int dtype, int d, int code, F f) {
    auto by_code = [&](auto t, auto dim) {
        if (code == kCodeE4m3) f(t, dim, Idx<kCodeE4m3>{});
        else f(t, dim, Idx<kCodeInt8>{});
    };
    auto by_dim = [&](auto t) {
        if (d == 64) by_code(t, Idx<64>{});
        else by_code(t, Idx<128>{});
    };
    if (dtype == 1) by_dim(float{});
    else by_dim(__bf16{});
}

}  // namespace

int launch_qk_norm(int dtype, int style, int d, int n, const NormArgs& a, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    const int64_t units = (int64_t)(a.hq + a.hkv) * (d * (dtype == 1 ? 4 : 2) / 32);
    const int threads = units >= kNormThreads ? kNormThreads : (int)((units + 63) / 64) * 64;
    const auto go = [&](auto t, auto dim) { launch_norm_d<decltype(t), decltype(dim)::value>(style, n, threads, a, st); };
    if (dtype == 1) d == 64 ? go(float{}, Idx<64>{}) : go(float{}, Idx<128>{});
    else d == 64 ? go(__bf16{}, Idx<64>{}) : go(__bf16{}, Idx<128>{});
    return hipGetLastError();
}

int launch_kv8_write(int dtype, int code, int d, const Kv8WriteArgs& a, void* stream) {
    const int per = 2 * a.hkv;   // units of a block
    const unsigned ranges = (unsigned)(((int64_t)a.n + a.range - 1) / a.range);
    by_types(dtype, d, code, [&](auto t, auto dim, auto c) {
        constexpr int D = decltype(dim)::value;
        const auto go = [&](auto waves, auto noted, unsigned y) {
            constexpr int W = decltype(waves)::value;
            hipLaunchKernelGGL((kv8_write_kernel<decltype(t), D, decltype(c)::value, W, decltype(noted)::value>), dim3(ranges, y), dim3(W * 64), 0,
                               (hipStream_t)stream, a);
        };
        if (a.n > kWriteScan) {
            hipLaunchKernelGGL((kv8_notes<D>), dim3((unsigned)(((int64_t)a.n + 255) / 256)), dim3(256), 0, (hipStream_t)stream, a);
            if (per > kWriteWaves) go(Idx<kNotedWaves>{}, std::true_type{}, 1);
            else go(Idx<kWriteWaves>{}, std::true_type{}, 1);
        } else {   // a block's units over workgroups in y, so that a few tokens fill the chip
            go(Idx<kWriteWaves>{}, std::false_type{}, per <= 3 * kWriteWaves ? (unsigned)((per + kWriteWaves - 1) / kWriteWaves) : 4);
        }
    });
    return hipGetLastError();
}

int launch_kv8_read(int dtype, int code, int d, int hkv, const uint8_t* k_pool, const uint8_t* v_pool, const float* scale,
                    int64_t n_slots, const int32_t* slots, int n, void* k_out, void* v_out, void* stream) {
    const int64_t units = (int64_t)n * hkv * (d * (dtype == 1 ? 4 : 2) / 16);
    const int64_t blocks = (units + 511) / 512;
    const dim3 grid((unsigned)(blocks < (1 << 22) ? blocks : 1 << 22));   // (lanes of a launch stay below 2^32)
    by_types(dtype, d, code, [&](auto t, auto dim, auto c) {
        typedef decltype(t) T;
        hipLaunchKernelGGL((kv8_read_kernel<T, decltype(dim)::value, decltype(c)::value>), grid, dim3(256), 0, (hipStream_t)stream, k_pool,
                           v_pool, scale, n_slots, slots, units, hkv, static_cast<T*>(k_out), static_cast<T*>(v_out));
    });
    return hipGetLastError();
}

int launch_kv8_keys(int style, int d, const KeyPlan& plan, const Kv8Args& args, void* stream) {
    if (d == 64) launch_keys_d<64>(style, plan, args, (hipStream_t)stream);
    else launch_keys_d<128>(style, plan, args, (hipStream_t)stream);
    return hipGetLastError();
}

int launch_kv8(int style, int d, bool rope, const Plan& plan, const Kv8Args& args, void* stream) {
    if (plan.n_items == 0) return hipSuccess;
    hipStream_t st = (hipStream_t)stream;
    if (d == 64) return args.code == kCodeE4m3 ? launch_kv8_d<64, kCodeE4m3>(style, rope, plan, args, st) : launch_kv8_d<64, kCodeInt8>(style, rope, plan, args, st);
    return args.code == kCodeE4m3 ? launch_kv8_d<128, kCodeE4m3>(style, rope, plan, args, st) : launch_kv8_d<128, kCodeInt8>(style, rope, plan, args, st);
}

}  // namespace pic
