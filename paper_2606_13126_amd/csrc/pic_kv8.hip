// HIP kernels of the cache held in 8 bits, for MI355X (gfx950, CDNA4).
//
//  * qk_norm    norm of every query and key head of a projection, turned on the way where the
//               pool holds turned keys.
//  * kv8_write  key and value rows into the pool as codes and a scale per block and head.
//  * kv8_read   rows of the pool as numbers.
//  * kv8_few    attention over the codes in bf16; kv8_merge joins its key splits.  (float32: attn_f32
//               over Kv8Args, in pic_kernels.hip)
//
// Pools: codes [num_blocks][Hkv][16][D], one byte each, and scales [num_blocks][Hkv][2].  An
// element is code x scale.  The attention multiplies codes as they are (every code is exact in float16
// and bf16) and puts the keys' scale into the scores and the values' into the probabilities.
#include <type_traits>

#include "pic_device.h"

namespace pic {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
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
// neighbours, so its squares meet by lane permutes; a thread's units lie on the same pairs of
// different heads, so it computes their cos/sin and reads their weights once.
// Bound by memory: every element is read and written once.
// ---------------------------------------------------------------------------------
constexpr int kNormThreads = 256;

template <typename T, int D, int STYLE, bool ROT>
__global__ void __launch_bounds__(kNormThreads) qk_norm_kernel(const NormArgs a) {
    constexpr int PP = 16 / sizeof(T);     // elements per chunk, pairs per unit
    constexpr int CH = D / PP, UPH = CH / 2, U = 4;
    typedef T vec_t __attribute__((ext_vector_type(PP)));
    const int64_t row = blockIdx.x;
    const int unit = (int)threadIdx.x % UPH, step = (int)blockDim.x / UPH;
    const int rc = a.rot_half / PP;        // chunks of a half that turns (NeoX: rot_half is a multiple of 8)
    const bool turns = ROT && unit * PP < a.rot_half;
    // a turning unit's chunks, and any other's
    const int c0 = STYLE == kNeox ? (turns ? unit : 2 * rc + 2 * (unit - rc)) : 2 * unit;
    const int c1 = STYLE == kNeox && turns ? unit + rc : c0 + 1;
    const vec_t* qr = static_cast<const vec_t*>(a.q) + row * a.q_stride;
    const vec_t* kr = static_cast<const vec_t*>(a.k) + row * a.k_stride;
    vec_t* qo = static_cast<vec_t*>(a.q_out) + row * a.q_out_stride;
    vec_t* ko = static_cast<vec_t*>(a.k_out) + row * a.k_out_stride;
    const int heads = a.hq + a.hkv;
    float c[PP], s[PP];
    vec_t w[2][2];                         // weights of q and k
    bool first = true;
    // (whole groups of UPH lanes take the same turns, so the lanes of a head are all there)
    for (int h0 = (int)threadIdx.x / UPH; h0 < heads; h0 += U * step) {
        vec_t x[U], y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * step;
            if (h >= heads) break;
            const vec_t* src = h < a.hq ? qr + h * CH : kr + (h - a.hq) * CH;
            x[u] = src[c0];
            y[u] = src[c1];
        }
        if (first) {
            const vec_t* from[2] = {static_cast<const vec_t*>(a.q_weight), static_cast<const vec_t*>(a.k_weight)};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                w[i][0] = from[i] ? from[i][c0] : vec_t((T)1.f);
                w[i][1] = from[i] ? from[i][c1] : vec_t((T)1.f);
            }
            if (turns) {
                const int32_t pos = a.positions[row];
#pragma unroll
                for (int k = 0; k < PP; ++k) rope_cs(pos, a.fstep[unit * PP + k], c[k], s[k]);
            }
            first = false;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * step;
            if (h >= heads) break;
            float f[2 * PP], sum = 0.f;
#pragma unroll
            for (int k = 0; k < 2 * PP; ++k) {
                f[k] = (float)(k < PP ? x[u][k] : y[u][k - PP]);
                sum = __builtin_fmaf(f[k], f[k], sum);
            }
            const float r = 1.f / sqrtf(sum_of<UPH>(sum) * (1.f / D) + a.eps);
            const int i = h < a.hq ? 0 : 1;
#pragma unroll
            for (int k = 0; k < 2 * PP; ++k) f[k] *= r * (float)(i ? w[1][k / PP][k % PP] : w[0][k / PP][k % PP]);
            if (turns)
#pragma unroll
                for (int k = 0; k < PP; ++k) {
                    if (STYLE != kNeox && unit * PP + k >= a.rot_half) break;
                    float& p = f[STYLE == kNeox ? k : 2 * k];
                    float& t = f[STYLE == kNeox ? PP + k : 2 * k + 1];
                    const float e = p, g = t;
                    p = __builtin_fmaf(e, c[k], -(g * s[k]));
                    t = __builtin_fmaf(e, s[k], g * c[k]);
                }
#pragma unroll
            for (int k = 0; k < PP; ++k) {
                x[u][k] = (T)f[k];
                y[u][k] = (T)f[PP + k];
            }
            vec_t* dst = h < a.hq ? qo + h * CH : ko + (h - a.hq) * CH;
            dst[c0] = x[u];
            dst[c1] = y[u];
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
    static __device__ __forceinline__ u32x2_t halves(uint32_t w) {
        if constexpr (CODE == kCodeE4m3) {
            const f16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true);
            return u32x2_t{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
        } else {
            // 0x64uu is 1024 + u: with u = code + 128, less 1152
            const uint32_t u = w ^ 0x80808080u;
            const f16x2_t off = {(_Float16)-1152.f, (_Float16)-1152.f};
            const f16x2_t lo = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off;
            const f16x2_t hi = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off;
            return u32x2_t{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
        }
    }
    // ... as two words of bf16 (exact: an upper half of a float32 holds 8 bits)
    static __device__ __forceinline__ u32x2_t bf16s(uint32_t w) {
        const f32x4_t x = decode(w);
        return u32x2_t{__builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u),
                       __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u)};
    }
};

// ---------------------------------------------------------------------------------
// kv8_write.  A unit is (block, head, keys or values), taken by a wave: the rows that the call
// stores in the block give the scale (a maximum over the wave), then lane l codes 16 elements of offset
// l / (D / 16) (and 64 / (D / 16) offsets on), so that a page leaves in whole lines.  A block belongs to the first of
// its rows, which follow one another: a workgroup looks for blocks that begin among `range` rows.
// Bound by memory for prompts, by its chain of loads (slots, then rows) for a step's tokens.
// ---------------------------------------------------------------------------------
constexpr int kWriteWaves = 4;

template <typename T, int D, int CODE>
__global__ void __launch_bounds__(kWriteWaves * 64) kv8_write_kernel(const Kv8WriteArgs a) {
    typedef Code<CODE> C;
    constexpr int LPO = D / 16;            // lanes of an offset
    constexpr int OPP = 64 / LPO, P = kBlock / OPP;   // offsets per pass, passes
    constexpr int V = 16 / sizeof(T), NV = 16 / V;    // elements of a load, loads of a lane per pass
    typedef T vec_t __attribute__((ext_vector_type(V)));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t r0 = (int64_t)blockIdx.x * a.range;
    const int n_here = (int)min((int64_t)a.range, a.n - r0);
    // block of row i (-1: it stores nothing)
    auto block_of = [&](int64_t i) {
        const int32_t s = a.slots[i];
        return s >= 0 && s < a.n_slots ? s >> 4 : -1;
    };
    bool lead = false;
    if (lane < n_here) {
        const int b = block_of(r0 + lane);
        lead = b >= 0 && (r0 + lane == 0 || block_of(r0 + lane - 1) != b);
    }
    const uint64_t leads = __builtin_amdgcn_ballot_w64(lead);
    const int per = 2 * a.hkv, units = __builtin_popcountll(leads) * per;
    const int c16 = (lane % LPO) * 16;
    for (int u = (int)blockIdx.y * kWriteWaves + wave; u < units; u += (int)gridDim.y * kWriteWaves) {
        uint64_t rest = leads;
        for (int i = u / per; i > 0; --i) rest &= rest - 1;
        const int64_t row0 = r0 + __builtin_ctzll(rest);
        const int which = u & 1, h = (u % per) >> 1;
        // the rows of the block: of each offset the last
        const int blk = a.slots[row0] >> 4;
        int64_t row[P];
        bool fresh = false;
#pragma unroll
        for (int p = 0; p < P; ++p) row[p] = -1;
        for (int64_t from = row0;; from += 64) {
            const int64_t i = from + lane;
            const int32_t s = i < a.n ? a.slots[i] : -1;
            const uint64_t others = __builtin_amdgcn_ballot_w64((s >> 4) != blk);
            const int run = others ? __builtin_ctzll(others) : 64;
#pragma unroll
            for (int o = 0; o < kBlock; ++o) {
                const uint64_t m = __builtin_amdgcn_ballot_w64(lane < run && (s & 15) == o);
                if (m == 0) continue;
                if (o == 0) fresh = true;
                if (o % OPP == lane / LPO) row[o / OPP] = from + 63 - __builtin_clzll(m);
            }
            if (run < 64) break;
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
        const float old = fresh ? 0.f : *sp;
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
// kv8_read: a thread takes the codes of 16 bytes of output (4 or 8), U of them in flight.  Bound by memory.
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
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * step;
            in[u] = false;
            if (i >= n_units) break;
            const int64_t rh = i / CPR;
            const int32_t slot = slots[rh / hkv];
            if (slot < 0 || slot >= n_slots) continue;
            in[u] = true;
            const int64_t page = (int64_t)(slot >> 4) * hkv + rh % hkv;
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
// RoPE: a lane holds 8 dimensions each of KD chunks of key l%16: PL pairs, whose cos/sin advance from one
// of the wave's blocks to its next by a constant rotation where the positions do (renewed every
// kKv8Renew steps), else are computed.  Codes turn in packed float16, two pairs at a time.
// ---------------------------------------------------------------------------------
constexpr int kKv8Renew = 32;

template <int D>
struct Kv8Few {
    static constexpr int NW = kKv8Waves, TK = kBlock;
    static constexpr int STEP = NW * TK;         // keys of all waves
    static constexpr int TILE = TK * D;          // bytes of a wave's keys or values of a step
    static constexpr int CPR = D / 16;           // 16-byte chunks per row
    static constexpr int KPC = 64 / CPR;         // keys of a copy (64 chunks)
    static constexpr int NC = TK / KPC;          // copies of a step, each of K and V
    static constexpr int NST = 4;                // steps in LDS
    static constexpr int LPS = 2 * NC + 1;       // copies per lane per step
    static constexpr int META = 20;              // a step's positions (16) and its two scales
};

template <int D>
struct __attribute__((aligned(16))) Kv8FewLds {
    typedef Kv8Few<D> S;
    uint8_t stages[S::NST][S::NW][2][S::TILE];
    float2 stride_cs[D / 2];                     // cos/sin of STEP positions
    uint64_t fstep[D / 2];
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

template <int D, int STYLE, bool ROPE, int CODE, int CB, int NG>
__global__ void __launch_bounds__(kKv8Waves * 64, 2) kv8_few(const PlanOf<NG> plan, const Kv8Args a) {
    typedef Kv8Few<D> S;
    typedef Code<CODE> C;
    constexpr int KD = D / 32;             // 16x16x32 contraction steps of QK^T; words of 4 pairs of a lane
    constexpr int DB = D / 32;             // 32-dim blocks of O^T
    constexpr int TK = S::TK, NW = S::NW, NST = S::NST, HALF = D / 2, PL = 4 * KD;
    static_assert(S::TILE * 2 * NST >= CB * 2 * DB * 1024, "a wave's outputs fit its stages");

    __shared__ Kv8FewLds<D> lds;
    __shared__ float2 mls[NW][16 * CB];

    const Group g = group_of<false>(plan, blockIdx.x);
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
    auto issue = [&](int u, int st, int blk) {
        const int k0 = u * S::STEP + wave * TK;
        const uint32_t to = stages_at + (uint32_t)((st * NW + wave) * 2 * S::TILE);
        __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));   // the stage's last reads have returned
        const size_t at = (size_t)(uint32_t)blk * a.hkv * page;
#pragma unroll
        for (int i = 0; i < S::NC; ++i) {
            const int key = i * S::KPC + lane / S::CPR, c = lane % S::CPR;
            const int row = (near_key(k0 + key)) & (TK - 1);
            copy_lds16(kpool + at, (uint32_t)(row * D + ((c ^ kswz<D>(key)) << 4)), to + i * 1024);
            copy_lds16(vpool + at, (uint32_t)(row * D + ((c ^ vswz<D>(key)) << 4)), to + S::TILE + i * 1024);
        }
        if (lane < 18) {
            const void* src = lane < 16 ? (const void*)(posv + near_key(k0 + lane))
                                        : (const void*)(a.scale + ((size_t)(uint32_t)blk * a.hkv + ic.kvh) * 2 + (lane - 16));
            copy_lds4(src, meta_at + (uint32_t)(st * S::META * 4));
        }
    };
    auto block_at = [&](int u) { return scalar_load(btab, u * NW + wave); };   // (u < nt: the block holds a key of the range)

#pragma unroll
    for (int u = 0; u < NST - 1; ++u)
        if (u < nt) issue(u, u, block_at(u));
    if (ROPE)
        for (int i = threadIdx.x; i < HALF; i += NW * 64) {
            lds.fstep[i] = a.fstep[i];
            rope_cs_fast(S::STEP, a.fstep[i], lds.stride_cs[i].x, lds.stride_cs[i].y);
        }
    __syncthreads();   // phase steps staged

    // pair e of word i of the lane's (4 pairs each); its elements as they come from the chunks of a row
    auto pair_of = [&](int i, int e) { return STYLE == kNeox ? 8 * ((i / 2) * 4 + q4) + 4 * (i % 2) + e : 4 * (i * 4 + q4) + e; };

    // ---- queries: B operand, turned at their tokens' positions
    u32x4_t qb[CB][KD];
    float qs[CB];     // scores are the products times this and the block's scale (log2 units)
    int last[CB];     // last key that the lane's row sees, from kt0
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row_lo + 16 * cb + c16;
        const bool valid = row < rows_total;
        const int to = valid ? row / G : 0, hl = valid ? row - to * G : 0;
        last[cb] = min(k_hi - 1, g.tok0 + to - kt0);
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((size_t)(g.q_row0 + to) * a.hq + (size_t)ic.kvh * G + hl) * D;
        u32x4_t raw[KD];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) {
            raw[kd] = *reinterpret_cast<const u32x4_t*>(qp + model_chunk(a.chunk_map, kd * 4 + q4) * 8);
            if (!valid) raw[kd] = u32x4_t{0, 0, 0, 0};
        }
        float x[PL], y[PL], big = 0.f;
#pragma unroll
        for (int i = 0; i < KD; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                auto el = [&](int kd, int k) { return k % 2 ? bf_hi(raw[kd][k / 2]) : bf_lo(raw[kd][k / 2]); };
                x[4 * i + e] = STYLE == kNeox ? el(i / 2, 4 * (i % 2) + e) : el(i, 2 * e);
                y[4 * i + e] = STYLE == kNeox ? el(KD / 2 + i / 2, 4 * (i % 2) + e) : el(i, 2 * e + 1);
            }
        qs[cb] = a.scale_log2;
        if (ROPE) {
            const int32_t pos = a.positions[g.pos_off + g.tok0 + to];
#pragma unroll
            for (int i = 0; i < KD; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float c, s;
                    rope_cs_fast(pos, lds.fstep[pair_of(i, e)], c, s);
                    float& u = x[4 * i + e];
                    float& v = y[4 * i + e];
                    const float u0 = u, v0 = v;
                    u = u0 * c - v0 * s;
                    v = v0 * c + u0 * s;
                    big = fmaxf(big, fmaxf(fabsf(u), fabsf(v)));
                }
            const int ex = query_exponent(max_xor32(max_xor16(big)));
            qs[cb] = ldexpf(qs[cb], ex);
#pragma unroll
            for (int i = 0; i < PL; ++i) {
                x[i] = ldexpf(x[i], -ex);
                y[i] = ldexpf(y[i], -ex);
            }
        }
#pragma unroll
        for (int i = 0; i < KD; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                qb[cb][i][h] = ROPE ? pack_f16(x[4 * i + 2 * h], x[4 * i + 2 * h + 1]) : pack_bf16(x[4 * i + 2 * h], x[4 * i + 2 * h + 1]);
                qb[cb][i][2 + h] = ROPE ? pack_f16(y[4 * i + 2 * h], y[4 * i + 2 * h + 1]) : pack_bf16(y[4 * i + 2 * h], y[4 * i + 2 * h + 1]);
            }
    }

    // per-lane byte offsets within a tile: the K operand's 8 codes of each chunk, the V operand's pieces
    int k_off[KD], v_off[DB];
#pragma unroll
    for (int kd = 0; kd < KD; ++kd) {
        const int c8 = model_chunk(a.chunk_map, kd * 4 + q4);
        k_off[kd] = c16 * D + (((c8 >> 1) ^ kswz<D>(c16)) << 4) + (c8 & 1) * 8;
    }
    {
        const int key = 4 * q4 + (c16 >> 2);
#pragma unroll
        for (int db = 0; db < DB; ++db)
            v_off[db] = S::TILE + key * D + (((2 * db + ((c16 >> 1) & 1)) ^ vswz<D>(key)) << 4) + (c16 & 1) * 8;
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
    float rc[PL], rs[PL];      // cos/sin of the lane's pairs at position cs_pos
    int32_t cs_pos = 0;
    int renew = 0;             // steps until they are computed again

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
        u32x4_t kf[KD];
        if constexpr (ROPE) {
            const int32_t pos = meta[c16];
            // (STEP on, and not past the type's end)
            if (renew == 0 || __builtin_amdgcn_ballot_w64((uint32_t)pos != (uint32_t)cs_pos + S::STEP || pos < cs_pos) != 0) {
#pragma unroll
                for (int i = 0; i < PL; ++i) rope_cs_fast(pos, lds.fstep[pair_of(i / 4, i % 4)], rc[i], rs[i]);
                renew = kKv8Renew;
            } else {
#pragma unroll
                for (int i = 0; i < PL; ++i) {
                    const float2 d = lds.stride_cs[pair_of(i / 4, i % 4)];
                    const float c = rc[i], s = rs[i];
                    rc[i] = c * d.x - s * d.y;
                    rs[i] = s * d.x + c * d.y;
                }
            }
            --renew;
            cs_pos = pos;
        }
#pragma unroll
        for (int i = 0; i < KD; ++i) {
            uint32_t xw, yw;   // codes of the x and y of 4 pairs
            if (STYLE == kNeox) {
                xw = kw[i / 2][i % 2];
                yw = kw[KD / 2 + i / 2][i % 2];
            } else {
                xw = __builtin_amdgcn_perm(kw[i][1], kw[i][0], 0x06040200u);
                yw = __builtin_amdgcn_perm(kw[i][1], kw[i][0], 0x07050301u);
            }
            if constexpr (ROPE) {
                const u32x2_t xh = C::halves(xw), yh = C::halves(yw);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t xb = xh[h], yb = yh[h];   // (a bit cast of a vector's element would read its first)
                    const f16x2_t x = __builtin_bit_cast(f16x2_t, xb), y = __builtin_bit_cast(f16x2_t, yb);
                    const int p = 4 * i + 2 * h;
                    const f16x2_t c = __builtin_bit_cast(f16x2_t, pack_f16(rc[p], rc[p + 1])), s = __builtin_bit_cast(f16x2_t, pack_f16(rs[p], rs[p + 1]));
                    kf[i][h] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(x, c, -(y * s)));
                    kf[i][2 + h] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(y, c, x * s));
                }
            } else {
                const u32x2_t xb = C::bf16s(xw), yb = C::bf16s(yw);
                kf[i] = u32x4_t{xb[0], xb[1], yb[0], yb[1]};
            }
        }
        f32x4_t sc[CB];
#pragma unroll
        for (int i = 0; i < KD; ++i)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const f32x4_t from = i == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[cb];
                if (ROPE)
                    sc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, kf[i]), __builtin_bit_cast(f16x8_t, qb[cb][i]), from, 0, 0, 0);
                else
                    sc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[i]), __builtin_bit_cast(bf16x8_t, qb[cb][i]), from, 0, 0, 0);
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
            mx[cb] = max_xor32(max_xor16(mx[cb]));
            moves |= mx[cb] > m_run[cb] + 8.f;
        }
        // the reference maximum only moves when some row's maximum grows by more than 8
        // (probabilities stay below 2^8), so most tiles skip rescaling
        if (__builtin_amdgcn_ballot_w64(moves) != 0) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const float m_new = fmaxf(m_run[cb], mx[cb]);
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
            const u32x2_t both = __builtin_bit_cast(u32x2_t, lds_read_tr((lds_u16_t*)(tile + v_off[db])));
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

// Joins key splits: one block per kMergeRows rows of a (row tile, KV head), one float4 of a row per
// thread, U splits' loads in flight.  A row tile has splits up to its last token's.
struct Kv8MergeArgs {
    const float* part_o;
    const float* part_ml;
    void* o;
    int32_t tile_rows, hq, hkv, group;
};

template <int D, int NG, int U>
__global__ void __launch_bounds__(kMergeRows * D / 4) kv8_merge(const PlanOf<NG> plan, const Kv8MergeArgs a) {
    constexpr int TPR = D / 4;
    const Group g = group_of<true>(plan, blockIdx.x);
    const int n_rt = g.n_rt, chunks = a.tile_rows / kMergeRows;
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

template <int D, int STYLE, bool ROPE, int CODE, int NG>
hipError_t launch_kv8_n(const PlanOf<NG>& plan, const Kv8Args& a, hipStream_t st) {
    const dim3 grid(plan.n_items), block(kKv8Waves * 64);
    if (a.tile_rows == 16) hipLaunchKernelGGL((kv8_few<D, STYLE, ROPE, CODE, 1, NG>), grid, block, 0, st, plan, a);
    else hipLaunchKernelGGL((kv8_few<D, STYLE, ROPE, CODE, 2, NG>), grid, block, 0, st, plan, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.n_merge == 0) return e;
    const Kv8MergeArgs m = {a.part_o, a.part_ml, a.o, a.tile_rows, a.hq, a.hkv, a.group};
    hipLaunchKernelGGL((kv8_merge<D, NG, 8>), dim3(plan.n_merge), dim3(kMergeRows * D / 4), 0, st, plan, m);
    return hipGetLastError();
}

template <int D, int STYLE, bool ROPE, int CODE>
hipError_t launch_kv8_t(const Plan& plan, const Kv8Args& a, hipStream_t st) {
    if (plan.n_groups > kFewGroups) return launch_kv8_n<D, STYLE, ROPE, CODE, kMaxGroups>(plan, a, st);
    PlanOf<kFewGroups> few = {plan.n_groups, plan.n_items, plan.n_merge, plan.merge_ways, plan.table, plan.item_map, plan.merge_map, {}};
    for (int i = 0; i < plan.n_groups; ++i) few.g[i] = plan.g[i];
    return launch_kv8_n<D, STYLE, ROPE, CODE, kFewGroups>(few, a, st);
}

template <int D, int CODE>
hipError_t launch_kv8_d(int style, bool rope, const Plan& plan, const Kv8Args& a, hipStream_t st) {
    if (!rope) return launch_kv8_t<D, 0, false, CODE>(plan, a, st);   // (without rotation the pairing makes no difference)
    return style == kNeox ? launch_kv8_t<D, 0, true, CODE>(plan, a, st) : launch_kv8_t<D, 1, true, CODE>(plan, a, st);
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
    if (dtype == 1) {
        if (d == 64) launch_norm_d<float, 64>(style, n, threads, a, st);
        else launch_norm_d<float, 128>(style, n, threads, a, st);
    } else {
        if (d == 64) launch_norm_d<__bf16, 64>(style, n, threads, a, st);
        else launch_norm_d<__bf16, 128>(style, n, threads, a, st);
    }
    return hipGetLastError();
}

int launch_kv8_write(int dtype, int code, int d, const Kv8WriteArgs& a, void* stream) {
    // a block's units over workgroups in y, so that a few tokens fill the chip
    const int64_t per = 2 * (int64_t)a.hkv;
    const dim3 grid((unsigned)((a.n + (int64_t)a.range - 1) / a.range), (unsigned)(per + kWriteWaves - 1 < 4 * kWriteWaves ? (per + kWriteWaves - 1) / kWriteWaves : 4));
    by_types(dtype, d, code, [&](auto t, auto dim, auto c) {
        hipLaunchKernelGGL((kv8_write_kernel<decltype(t), decltype(dim)::value, decltype(c)::value>), grid, dim3(kWriteWaves * 64), 0,
                           (hipStream_t)stream, a);
    });
    return hipGetLastError();
}

int launch_kv8_read(int dtype, int code, int d, int hkv, const uint8_t* k_pool, const uint8_t* v_pool, const float* scale,
                    int64_t n_slots, const int32_t* slots, int n, void* k_out, void* v_out, void* stream) {
    const int64_t units = (int64_t)n * hkv * (d * (dtype == 1 ? 4 : 2) / 16);
    const int64_t blocks = (units + 255) / 256;
    by_types(dtype, d, code, [&](auto t, auto dim, auto c) {
        typedef decltype(t) T;
        hipLaunchKernelGGL((kv8_read_kernel<T, decltype(dim)::value, decltype(c)::value>), dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256),
                           0, (hipStream_t)stream, k_pool, v_pool, scale, n_slots, slots, units, hkv, static_cast<T*>(k_out), static_cast<T*>(v_out));
    });
    return hipGetLastError();
}

int launch_kv8(int style, int d, bool rope, const Plan& plan, const Kv8Args& args, void* stream) {
    if (plan.n_items == 0) return hipSuccess;
    hipStream_t st = (hipStream_t)stream;
    if (d == 64) return args.code == kCodeE4m3 ? launch_kv8_d<64, kCodeE4m3>(style, rope, plan, args, st) : launch_kv8_d<64, kCodeInt8>(style, rope, plan, args, st);
    return args.code == kCodeE4m3 ? launch_kv8_d<128, kCodeE4m3>(style, rope, plan, args, st) : launch_kv8_d<128, kCodeInt8>(style, rope, plan, args, st);
}

}  // namespace pic
