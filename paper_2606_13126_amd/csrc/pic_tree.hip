// HIP kernels of speculative decoding over the paged cache, for MI355X (gfx950, CDNA4).
//
//  * kv_append  rows of a projection: k and v into the pool's slots, q packed; k and q
//               turned at their positions on the way where the pool holds turned keys.
//  * tree_mask  ancestor bits and depths of drafted trees.
//  * tree_bf16  attention of the drafted tokens, bf16 MFMA; tree_merge joins its key splits.
//               (float32: attn_f32 over TreeArgs, in pic_kernels.hip)
//  * kv_keep    the accepted rows of every tree move to the front of its slots.
#include <type_traits>

#include "pic_device.h"

namespace pic {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------------
// kv_append: one workgroup per row.  A unit is two 16-byte chunks of a head: NeoX the two
// runs whose elements pair up, GPT-J (and V, and what does not turn) two neighbours.  A
// thread's units lie on the same pairs of different heads, so it computes their cos/sin
// once.
// ---------------------------------------------------------------------------------
constexpr int kAppendThreads = 256;

template <typename T, int D, int STYLE, bool ROT>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(const AppendArgs a) {
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
    const int32_t slot = __builtin_amdgcn_readfirstlane(a.slots[row]);
    const bool stored = slot >= 0 && slot < a.n_slots;
    const vec_t* qr = static_cast<const vec_t*>(a.q) + row * a.q_stride;
    const vec_t* kr = static_cast<const vec_t*>(a.k) + row * a.k_stride;
    const vec_t* vr = static_cast<const vec_t*>(a.v) + row * a.v_stride;
    vec_t* qo = static_cast<vec_t*>(a.q_out) + row * a.hq * CH;
    const int64_t page = ((int64_t)(slot >> 4) * a.hkv * kBlock + (slot & 15)) * CH;
    vec_t* kp = static_cast<vec_t*>(a.k_pool) + page;
    vec_t* vp = static_cast<vec_t*>(a.v_pool) + page;
    const int heads = a.hq + 2 * a.hkv;
    float c[PP], s[PP];
    bool first = true;
    for (int h0 = (int)threadIdx.x / UPH; h0 < heads; h0 += U * step) {
        vec_t x[U], y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * step;
            if (h >= heads) break;
            const vec_t* src = h < a.hq ? qr + h * CH : h < a.hq + a.hkv ? kr + (h - a.hq) * CH : vr + (h - a.hq - a.hkv) * CH;
            const bool v = h >= a.hq + a.hkv;
            x[u] = src[v ? 2 * unit : c0];
            y[u] = src[v ? 2 * unit + 1 : c1];
        }
        if (turns && first) {
            const int32_t pos = a.positions[row];
#pragma unroll
            for (int k = 0; k < PP; ++k) rope_cs(pos, a.fstep[unit * PP + k], c[k], s[k]);
            first = false;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * step;
            if (h >= heads) break;
            const bool v = h >= a.hq + a.hkv;
            if (turns && !v) {
#pragma unroll
                for (int k = 0; k < PP; ++k) {
                    if (STYLE != kNeox && unit * PP + k >= a.rot_half) break;
                    auto& p = STYLE == kNeox || 2 * k < PP ? x[u] : y[u];
                    auto& r = STYLE != kNeox && 2 * k < PP ? x[u] : y[u];
                    const int ip = STYLE == kNeox ? k : 2 * k % PP, ir = STYLE == kNeox ? k : 2 * k % PP + 1;
                    const float e = (float)p[ip], f = (float)r[ir];
                    p[ip] = (T)__builtin_fmaf(e, c[k], -(f * s[k]));
                    r[ir] = (T)__builtin_fmaf(e, s[k], f * c[k]);
                }
            }
            vec_t* dst = h < a.hq ? qo + h * CH : v ? vp + (int64_t)(h - a.hq - a.hkv) * kBlock * CH : kp + (int64_t)(h - a.hq) * kBlock * CH;
            if (h < a.hq || stored) {
                dst[v ? 2 * unit : c0] = x[u];
                dst[v ? 2 * unit + 1 : c1] = y[u];
            }
        }
    }
}

// ---------------------------------------------------------------------------------
// tree_mask: bits(i) = {i} + bits(parent i), by pointer doubling: after round k a node has
// the bits of its 2^k nearest ancestors and points 2^k ancestors up.  One workgroup per
// (tree, 64-node word).  A parent that is not an earlier node of the tree makes a root.
// ---------------------------------------------------------------------------------
constexpr int kMaxMaskWords = 64;

__global__ void __launch_bounds__(1024) tree_mask_kernel(const int32_t* __restrict__ parents, const int32_t* __restrict__ cu_rows,
                                                         int total_rows, uint64_t* __restrict__ mask, int words,
                                                         int32_t* __restrict__ depth) {
    constexpr int R = kMaxMaskWords * 64 / 1024;   // nodes per thread at most
    extern __shared__ uint64_t smem[];
    const int word = blockIdx.x;
    const int64_t row0 = cu_rows[blockIdx.y];
    // (never outside the arrays, whatever cu_rows holds)
    const int64_t all = row0 < 0 ? 0 : min((int64_t)cu_rows[blockIdx.y + 1], (int64_t)total_rows) - row0;
    const int n = (int)max((int64_t)0, min(all, (int64_t)words * 64));
    uint64_t* bits = smem;
    int32_t* up = reinterpret_cast<int32_t*>(smem + words * 64);
    int32_t* dep = up + words * 64;
    bool more = false;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        int p = parents[row0 + i];
        if (p < 0 || p >= i) p = -1;
        bits[i] = (i >> 6) == word ? 1ull << (i & 63) : 0ull;
        up[i] = p;
        dep[i] = p >= 0;
        more |= p >= 0;
    }
    while (__syncthreads_or(more)) {
        uint64_t b[R];
        int32_t p[R], d[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int i = (int)threadIdx.x + k * (int)blockDim.x;
            if (i >= n) break;
            const int q = up[i];
            b[k] = bits[i];
            p[k] = -1;
            d[k] = dep[i];
            if (q >= 0) {
                b[k] |= bits[q];
                p[k] = up[q];
                d[k] += dep[q];
            }
        }
        __syncthreads();
        more = false;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int i = (int)threadIdx.x + k * (int)blockDim.x;
            if (i >= n) break;
            bits[i] = b[k];
            up[i] = p[k];
            dep[i] = d[k];
            more |= p[k] >= 0;
        }
    }
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        mask[(row0 + i) * words + word] = bits[i];
        if (word == 0 && depth != nullptr) depth[row0 + i] = dep[i];
    }
}

// ---------------------------------------------------------------------------------
// kv_keep: one workgroup per (tree, KV head).  Path entries ascend with path[i] >= i, so a
// pass over some of them, read before it writes, only overwrites rows that no later pass
// reads.
// ---------------------------------------------------------------------------------
template <int CPR>   // 16-byte chunks per row of one head
__global__ void __launch_bounds__(256) kv_keep_kernel(u32x4_t* __restrict__ k_pool, u32x4_t* __restrict__ v_pool, int64_t n_slots,
                                                      const int32_t* __restrict__ slots, const int32_t* __restrict__ cu_rows,
                                                      const int32_t* __restrict__ path, const int32_t* __restrict__ path_len,
                                                      int max_path, int hkv, int total_rows) {
    const int tree = blockIdx.x, h = blockIdx.y;
    const int64_t row0 = cu_rows[tree];
    const int64_t n = row0 < 0 ? 0 : min((int64_t)cu_rows[tree + 1], (int64_t)total_rows) - row0;
    const int m = (int)min((int64_t)min(path_len[tree], max_path), n);
    const int c = (int)threadIdx.x % CPR;
    for (int i0 = 0; i0 < m; i0 += 256 / CPR) {
        const int i = i0 + (int)threadIdx.x / CPR;
        u32x4_t k, v;
        int64_t dst = -1;
        if (i < m) {
            const int p = path[(int64_t)tree * max_path + i];
            if (p > i && p < n) {
                const int64_t from = slots[row0 + p], to = slots[row0 + i];
                if (from >= 0 && from < n_slots && to >= 0 && to < n_slots) {
                    const int64_t src = (((from >> 4) * hkv + h) * kBlock + (from & 15)) * CPR + c;
                    dst = (((to >> 4) * hkv + h) * kBlock + (to & 15)) * CPR + c;
                    k = k_pool[src];
                    v = v_pool[src];
                }
            }
        }
        __syncthreads();
        if (dst >= 0) {
            k_pool[dst] = k;
            v_pool[dst] = v;
        }
    }
}

// cos/sin by the hardware's sine of a fraction of a revolution (its error, about 2^-20, is far
// below the 2^-12 to which the attention rounds what they turn)
__device__ __forceinline__ void rope_cs_fast(int32_t pos, uint64_t step, float& c, float& s) {
    const uint64_t ph = (uint64_t)(int64_t)pos * step;
    const float r = (float)(int32_t)(ph >> 32) * 0x1p-32f;
    c = __builtin_amdgcn_cosf(r);
    s = __builtin_amdgcn_sinf(r);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, f16x2_t{(_Float16)lo, (_Float16)hi});
}

// ---------------------------------------------------------------------------------
// tree_bf16
//
// Workgroup: eight waves (two per SIMD, so that one's products run under the other's vector
// work) over up to 16 CB WR query rows (drafted token x query head of one KV head's group) and
// one key range.  The waves are WR row groups of KG = 8 / WR; a wave holds 16 CB rows.
//   Few rows (WR = 1): a wave takes every eighth 16-key tile (one cache block) of the range, which
//     it copies, turns and multiplies without waiting for another wave.
//   More rows: steps of 64 keys.  Each wave copies and turns eight keys of a step, in place, one
//     step before the row groups multiply them; one barrier per step.
// K, V and the keys' positions go straight to LDS.  The results of a row group's KG waves meet
// in LDS at the end.
//   S^T (16 keys x 16 rows) = K Q^T       v_mfma_f32_16x16x32_f16 (bf16 without rotation)
//   O^T (16 dims x 16 rows) += V^T P^T    v_mfma_f32_16x16x32_bf16, V^T by ds_read_b64_tr_b16
// After the scores lane l holds row l%16 of each block and keys 4 (l/16) + {0..3}, the B
// operand of the output product.
//
// Precision: a rotated key or query is rounded to 11 bits (float16), its size held by a power
// of two where it does not fit: as bf16, 8 bits, each of the two alone would put outputs as
// far from 64 bits as their own rounding does.  Without rotation q and k are exact.  A
// probability enters the product as two bf16 numbers, its upper 8 bits and the rest: the 32
// contraction steps of the instruction hold 16 keys twice, at the time of one.
//
// RoPE: a lane turns PL pairs of one key of a tile and holds their cos/sin.  Its next key is
// STEP keys further; where the positions are too, the angles advance by a constant rotation (4
// operations a pair, renewed every kRenew tiles), else they are computed.
// ---------------------------------------------------------------------------------
constexpr int kRenew = 32;

// max over the 8 lanes l & ~7 .. l | 7
__device__ __forceinline__ float max_of8(float x) {
    auto dpp = [&](auto ctrl) {
        return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(x), __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false)));
    };
    x = dpp(Idx<0xB1>{});    // lane ^ 1
    x = dpp(Idx<0x4E>{});    // lane ^ 2
    return dpp(Idx<0x141>{});   // lane ^ 7 (half rows mirrored)
}

// Global -> LDS copies (dma_lds4, dma_lds16_s) to a wave-uniform LDS byte address
__device__ __forceinline__ void copy_lds4(const void* src, uint32_t to) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "{m0}"(to) : "memory");
}
__device__ __forceinline__ void copy_lds16(const void* base, uint32_t off, uint32_t to) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(to) : "memory");
}

template <int D, int STYLE, bool ROPE, int CB, int WR>
__global__ void __launch_bounds__(kTreeWaves * 64, 2) tree_bf16(const Plan plan, const TreeArgs a) {
    constexpr bool SHARED = WR > 1;        // the waves share their keys
    constexpr int KD = D / 32;             // 16x16x32 contraction steps of QK^T
    constexpr int DB = D / 16;             // 16-dim blocks of O^T
    constexpr int CH = D / 8;              // 16-byte chunks per K/V row
    constexpr int HALF = D / 2;
    constexpr int TK = kBlock;
    constexpr int NW = kTreeWaves, KG = NW / WR;
    constexpr int STEP = SHARED ? 64 : NW * TK;    // keys of all waves
    constexpr int OWNK = SHARED ? STEP / NW : TK;  // keys that a wave copies and turns
    constexpr int PL = OWNK * HALF / 64;   // pairs that a lane turns
    constexpr int NST = SHARED || D == 64 ? 4 : 2;
    constexpr int DPL = OWNK * CH / 64;    // 16-byte copies per lane per step, each of K and V
    constexpr int LPS = 2 * DPL + (ROPE ? 1 : 0);
    constexpr int KV = STEP * D;           // elements of K or V in a stage
    constexpr int SE = 2 * KV;             // elements of a stage: K of every tile, then V
    constexpr int OWN = CB > KG ? CB / KG : 1;     // column blocks whose queries a wave turns
    constexpr int SPARE = SHARED ? 2 : 1;  // stages that the queries pass through
    constexpr int PER = SPARE * SE / NW;   // elements of them per wave
    static_assert((NST - 2) * LPS < 64, "vmcnt range");
    static_assert(NST * SE * 2 >= NW * CB * DB * 64 * 16, "the outputs meet in the stages");
    static_assert(PER * 2 >= 16 * HALF * 8 && PER * 2 >= OWN * KD * 64 * 16, "queries pass through the stages");

    __shared__ __attribute__((aligned(16))) uint16_t stages[NST * SE];
    __shared__ int32_t ps[NW][NST][OWNK];
    __shared__ float ksc[NST][STEP];       // powers of two held back from a step's keys
    __shared__ int32_t kbig[NST][NW];      // whether some key of a wave has one
    // Steps in which rows differ in what they see: infinities of V (bits 0-7: +, 8-15: -, of a
    // chunk's dimensions, a NaN both), and whether a wave's keys have some
    __shared__ uint16_t vinf[NST][STEP][CH];
    __shared__ int32_t vbad[NST][NW];
    __shared__ float2 mls[NW][16 * CB];
    __shared__ float qsl[NW][16 * CB];
    __shared__ __attribute__((aligned(4))) uint8_t infs[NW][CB][DB][64];   // infinities of V that a lane's rows see: +, 4 dims, and -, 4 dims
    __shared__ uint64_t fstep[HALF];
    __shared__ __attribute__((aligned(16))) float2 stride_cs[HALF];        // cos/sin of STEP positions

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rg = wave / KG, kg = wave % KG;
    const int c16 = lane & 15, q4 = lane >> 4;
    const Group g = group_of<false>(plan, blockIdx.x);
    const int G = a.group, n_rt = g.n_rt;
    const int li = blockIdx.x - g.item_base;
    if (li >= a.hkv * g.n_split * n_rt) return;
    const ItemCoords ic = item_coords(g, a.hkv, n_rt, li);
    const int rows_total = g.n_tok * G, row_lo = (ic.rt * WR + rg) * 16 * CB;
    const int kv_lo = g.win + ic.split * g.split_keys, end = g.tok0 + g.n_tok;
    // (no sum below passes the last key: a request may have 2^31 - 1 of them)
    const int kv_hi = g.split_keys < end - kv_lo ? kv_lo + g.split_keys : end;
    // keys relative to kt0, the start of the first tile's block
    const int kt0 = kv_lo & ~(TK - 1), k_lo = kv_lo - kt0, k_hi = kv_hi - kt0, k_tok = g.tok0 - kt0;
    const int n_tiles = (k_hi - 1) / TK + 1;
    // steps in which this wave copies keys
    const int nt = SHARED ? (k_hi - 1) / STEP + 1 : n_tiles > wave ? (n_tiles - wave - 1) / NW + 1 : 0;

    if (ROPE)
        for (int i = tid; i < HALF; i += NW * 64) {
            fstep[i] = a.fstep[i];
            rope_cs_fast(STEP, a.fstep[i], stride_cs[i].x, stride_cs[i].y);
        }
    for (int i = tid; i < NW * CB * DB * 16; i += NW * 64) reinterpret_cast<uint32_t*>(infs)[i] = 0;

    const int32_t* btab = a.block_tables + (size_t)g.req * a.max_blocks + (kt0 >> 4);
    const int32_t* posv = a.positions + g.pos_off + kt0;
    const size_t blk_stride = (size_t)a.hkv * kBlock * D;
    const uint16_t* kpool = static_cast<const uint16_t*>(a.k_pool) + (size_t)ic.kvh * kBlock * D;
    const uint16_t* vpool = static_cast<const uint16_t*>(a.v_pool) + (size_t)ic.kvh * kBlock * D;

    // The i-th copy of a step moves 64 chunks, 64 / CH keys from copy_key(i) on.  A key outside
    // [k_lo, k_hi) stands for the nearest one inside, so that nothing outside the range is
    // read (its score is masked).
    constexpr int KPC = 64 / CH;           // keys per copy
    auto copy_key = [&](int i) { return SHARED ? (i * NW + wave) * KPC : wave * TK + i * KPC; };
    auto near_key = [&](int k) { return min(max(k, k_lo), k_hi - 1); };
    // this lane's byte offset within one head's page of a block, but for the row
    uint32_t lane_off[DPL];
#pragma unroll
    for (int i = 0; i < DPL; ++i) {
        const int row = (copy_key(i) + lane / CH) & (TK - 1);
        lane_off[i] = (uint32_t)(row * D + (((lane % CH) ^ dswz<D>(row)) << 3)) * 2;
    }
    // own key j (0 .. OWNK - 1) of a step: its place in the step
    auto own_key = [&](int j) { return copy_key(j / KPC) + j % KPC; };
    struct Blocks {
        int b[SHARED ? DPL : 1];           // (without sharing a step's copies are of one block)
    };
    auto blocks_of = [&](int u) {
        Blocks r;
#pragma unroll
        for (int i = 0; i < (SHARED ? DPL : 1); ++i) r.b[i] = scalar_load(btab, min(u * STEP + copy_key(i), k_hi - 1) >> 4);
        return r;
    };
    const uint32_t stages_at = lds_offset(stages), ps_at = lds_offset(&ps[wave][0][0]);
    auto issue = [&](int u, int st, const Blocks& blk) {
        const uint32_t sg = stages_at + (uint32_t)st * SE * 2;
        __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));   // the stage's last reads have returned (lgkmcnt 0)
        if (ROPE && lane < OWNK) copy_lds4(posv + near_key(u * STEP + own_key(lane)), ps_at + (uint32_t)st * OWNK * 4);
#pragma unroll
        for (int i = 0; i < DPL; ++i) {
            const int k0 = u * STEP + copy_key(i);
            const size_t base = (size_t)(uint32_t)blk.b[SHARED ? i : 0] * blk_stride;
            uint32_t off = lane_off[i];
            if (k0 < k_lo || k_hi - k0 < KPC) {
                const int k = k0 + lane / CH, row = k & (TK - 1);
                off += ((near_key(k) & (TK - 1)) - row) * D * 2;
            }
            copy_lds16(kpool + base, off, sg + copy_key(i) * D * 2);
            copy_lds16(vpool + base, off, sg + KV * 2 + copy_key(i) * D * 2);
        }
    };
#pragma unroll
    for (int u = 0; u < NST - SPARE; ++u)
        if (u < nt) issue(u, u, blocks_of(u));

    // ---- queries: the KG waves of a row group turn its column blocks and pass them to each
    // other through stages that are filled later.  The cos/sin of a block's tokens (a token's
    // heads share them) go the same way before.
    int toff[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row_lo + 16 * cb + c16;
        toff[cb] = row < rows_total ? row / G : 0;
    }
    bf16x8_t qb[CB][KD];
    float qs[CB];     // scores are the products times this (log2 units)
    __syncthreads();  // phase steps staged
    {
        u32x4_t mine[OWN][KD];
        uint16_t* spare = stages + (NST - SPARE) * SE + wave * PER;
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            const int cb = kg + o * KG;
            if (cb >= CB) break;
            const int row0 = row_lo + 16 * cb, row = row0 + c16;
            const bool valid = row < rows_total;
            const int to = valid ? row / G : 0, hl = valid ? row - to * G : 0;
            const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((size_t)(g.q_row0 + to) * a.hq + (size_t)ic.kvh * G + hl) * D;
            u32x4_t raw[KD];
#pragma unroll
            for (int kd = 0; kd < KD; ++kd) {
                raw[kd] = *reinterpret_cast<const u32x4_t*>(qp + model_chunk(a.chunk_map, kd * 4 + q4) * 8);
                if (!valid) raw[kd] = u32x4_t{0, 0, 0, 0};
            }
            float scale = a.scale_log2;
            if (ROPE) {
                const int t0 = min(row0, rows_total - 1) / G, t1 = min(row0 + 15, rows_total - 1) / G;
                float2* cs = reinterpret_cast<float2*>(spare);
                for (int i = lane; i < (t1 - t0 + 1) * HALF; i += 64) {
                    float c, s;
                    rope_cs_fast(a.positions[g.pos_off + g.tok0 + t0 + i / HALF], fstep[i % HALF], c, s);
                    cs[i] = make_float2(c, s);
                }
                const float2* tc = cs + (valid ? to - t0 : 0) * HALF;
                float xf[KD][8], big = 0.f;
#pragma unroll
                for (int kd = 0; kd < KD; ++kd)
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        xf[kd][2 * m] = bf_lo(raw[kd][m]);
                        xf[kd][2 * m + 1] = bf_hi(raw[kd][m]);
                    }
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    // NeoX: pairs 32 kd + 8 q4 + e, elements e of chunks kd and kd + KD / 2; GPT-J:
                    // 16 kd + 4 q4 + m, elements 2 m and 2 m + 1 of chunk kd
                    const int kd = STYLE == kNeox ? i / 8 : i / 4, e = STYLE == kNeox ? i % 8 : i % 4;
                    const float2 t = tc[STYLE == kNeox ? kd * 32 + 8 * q4 + e : kd * 16 + 4 * q4 + e];
                    float& x = STYLE == kNeox ? xf[kd][e] : xf[kd][2 * e];
                    float& y = STYLE == kNeox ? xf[kd + KD / 2][e] : xf[kd][2 * e + 1];
                    const float x0 = x, y0 = y;
                    x = x0 * t.x - y0 * t.y;
                    y = y0 * t.x + x0 * t.y;
                    big = fmaxf(big, fmaxf(fabsf(x), fabsf(y)));
                }
                big = max_xor32(max_xor16(big));
                // the row times 2^-ex lies in [-1, 1]
                const int ex = big > 0.f && big < INFINITY ? __builtin_amdgcn_frexp_expf(big) : 0;
                scale = ldexpf(scale, ex);
#pragma unroll
                for (int kd = 0; kd < KD; ++kd)
#pragma unroll
                    for (int m = 0; m < 4; ++m) raw[kd][m] = pack_f16(ldexpf(xf[kd][2 * m], -ex), ldexpf(xf[kd][2 * m + 1], -ex));
            }
#pragma unroll
            for (int kd = 0; kd < KD; ++kd) mine[o][kd] = raw[kd];
            if (KG == 1) {
#pragma unroll
                for (int kd = 0; kd < KD; ++kd) qb[o][kd] = __builtin_bit_cast(bf16x8_t, raw[kd]);
                qs[o] = scale;
            } else if (q4 == 0) {
                qsl[rg * KG][16 * cb + c16] = scale;
            }
        }
        __atomic_signal_fence(__ATOMIC_SEQ_CST);   // the last block's cos/sin have been read
        if constexpr (KG > 1) {
#pragma unroll
            for (int o = 0; o < OWN; ++o)
                if (kg + o * KG < CB)
#pragma unroll
                    for (int kd = 0; kd < KD; ++kd) reinterpret_cast<u32x4_t*>(spare)[(o * KD + kd) * 64 + lane] = mine[o][kd];
            barrier_keep_vmem();
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const uint16_t* from = stages + (NST - SPARE) * SE + (rg * KG + cb % KG) * PER + (cb / KG) * KD * 64 * 8;
#pragma unroll
                for (int kd = 0; kd < KD; ++kd) qb[cb][kd] = *reinterpret_cast<const bf16x8_t*>(from + (kd * 64 + lane) * 8);
                qs[cb] = qsl[rg * KG][16 * cb + c16];
            }
        }
        barrier_keep_vmem();   // every wave has its rows: the stages may be filled
    }

    f32x4_t acc[CB][DB];
    float m_run[CB], l_run[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        m_run[cb] = kNegBig;
        l_run[cb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[cb][db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    // per-lane element offsets within a tile: K operand rows and V^T operand rows
    int k_off[KD], v_off[DB];
#pragma unroll
    for (int kd = 0; kd < KD; ++kd) k_off[kd] = c16 * D + ((model_chunk(a.chunk_map, kd * 4 + q4) ^ dswz<D>(c16)) << 3);
    {
        const int key = 4 * q4 + (c16 >> 2);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const int d = db * 16 + 4 * (lane & 3);
            v_off[db] = key * D + (((d >> 3) ^ dswz<D>(key)) << 3) + (d & 7);
        }
    }

    // ---- turning keys.  Without sharing a lane has the operand's elements of key c16: runs of 8
    // (NeoX pairs 32 kd + 8 q4 + e of chunks kd and kd + KD / 2; GPT-J pairs 16 kd + 4 q4 + m).
    // With sharing 8 lanes have one key, PL pairs (lane % 8) * PL + i each.
    constexpr int RUN = SHARED ? PL : STYLE == kNeox ? 8 : 4;   // pairs in a row
    const int own_j = SHARED ? lane >> 3 : c16;
    const int pair0 = SHARED ? (lane & 7) * PL : RUN * q4;
    auto pair_of = [&](int i) { return pair0 + (SHARED ? i : i / RUN * 4 * RUN + i % RUN); };
    const int sh_row = SHARED ? own_key(own_j) : 0;
    // SHARED: element offsets of the lane's two runs (NeoX) or of its 2 PL neighbours (GPT-J)
    int s_off[2];
    if (SHARED) {
        const int e0 = STYLE == kNeox ? pair0 : 2 * pair0, e1 = STYLE == kNeox ? pair0 + HALF : e0 + PL;
        const int row = sh_row & (TK - 1);
        s_off[0] = sh_row * D + ((model_chunk(a.chunk_map, e0 >> 3) ^ dswz<D>(row)) << 3) + (e0 & 7);
        s_off[1] = sh_row * D + ((model_chunk(a.chunk_map, e1 >> 3) ^ dswz<D>(row)) << 3) + (e1 & 7);
    }
    float rc[PL], rs[PL];   // cos/sin at position cs_pos
    uint32_t cs_pos = 0;
    int fresh = 0;          // steps until the angles are computed again
    // turns 2 PL elements, words w[0 .. PL): NeoX x in the first half and y in the second; returns
    // whether some key of the wave got a power of two
    auto turn = [&](int st, uint32_t (&w)[PL]) {
        const uint32_t pos = (uint32_t)ps[wave][st][own_j];
        if (fresh == 0 || __builtin_amdgcn_ballot_w64(pos != cs_pos + STEP) != 0) {
#pragma unroll
            for (int i = 0; i < PL; ++i) rope_cs_fast((int32_t)(pos - STEP), fstep[pair_of(i)], rc[i], rs[i]);
            fresh = kRenew;
        }
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            const float2 d = stride_cs[pair_of(i)];
            const float c = rc[i], s = rs[i];
            rc[i] = c * d.x - s * d.y;
            rs[i] = s * d.x + c * d.y;
        }
        --fresh;
        cs_pos = pos;
        float big = 0.f;
        uint32_t out[PL];
        auto rotate = [&](auto scaled, int ex) {
#pragma unroll
            for (int i = 0; i < PL; i += 2) {
                const uint32_t A = STYLE == kNeox ? w[i / 2] : w[i], B = STYLE == kNeox ? w[PL / 2 + i / 2] : w[i + 1];
                const float x0 = bf_lo(A), y0 = STYLE == kNeox ? bf_lo(B) : bf_hi(A);
                const float x1 = STYLE == kNeox ? bf_hi(A) : bf_lo(B), y1 = bf_hi(B);
                float p0 = x0 * rc[i] - y0 * rs[i], r0 = y0 * rc[i] + x0 * rs[i];
                float p1 = x1 * rc[i + 1] - y1 * rs[i + 1], r1 = y1 * rc[i + 1] + x1 * rs[i + 1];
                if (decltype(scaled)::value) {
                    p0 = ldexpf(p0, -ex); r0 = ldexpf(r0, -ex); p1 = ldexpf(p1, -ex); r1 = ldexpf(r1, -ex);
                } else {
                    big = fmaxf(fmaxf(big, fabsf(p0)), fabsf(r0));
                    big = fmaxf(fmaxf(big, fabsf(p1)), fabsf(r1));
                }
                out[STYLE == kNeox ? i / 2 : i] = STYLE == kNeox ? pack_f16(p0, p1) : pack_f16(p0, r0);
                out[STYLE == kNeox ? PL / 2 + i / 2 : i + 1] = STYLE == kNeox ? pack_f16(r0, r1) : pack_f16(p1, r1);
            }
        };
        rotate(std::false_type{}, 0);
        // a key whose largest element lies outside 2^-8 .. 2^15 goes in times a power of two
        big = SHARED ? max_of8(big) : max_xor32(max_xor16(big));
        const bool odd = big >= 0x1p15f || (big < 0x1p-8f && big > 0.f);
        const bool any = __builtin_amdgcn_ballot_w64(odd) != 0;
        int ex = 0;
        if (any) {
            ex = odd && big < INFINITY ? __builtin_amdgcn_frexp_expf(big) : 0;
            rotate(std::true_type{}, ex);
        }
        if (SHARED) {
            if ((lane & 7) == 0) ksc[st][sh_row] = ldexpf(1.f, ex);
            if (lane == 0) kbig[st][wave] = any;
        } else if (any && q4 == 0) {
            ksc[st][wave * TK + c16] = ldexpf(1.f, ex);
        }
#pragma unroll
        for (int i = 0; i < PL; ++i) w[i] = out[i];
        return any;
    };

    // ---- An infinity or NaN in V must not reach rows that do not see its key (0 x Inf in the product):
    // where a step has keys that not every row sees, the wave that copied them puts zeros in
    // their place and notes them; what rows see of them joins their outputs at the end.
    auto clean = [&](int u, int st) {
        if (u * STEP >= k_lo && (u + 1) * STEP <= min(k_hi, k_tok)) return;
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < DPL; ++i) {
            const int key = copy_key(i) + lane / CH;
            u32x4_t* at = reinterpret_cast<u32x4_t*>(stages + st * SE + KV + copy_key(i) * D + lane * 8);
            u32x4_t v = *at;
            uint32_t f = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t x = (v[e / 2] >> (16 * (e % 2))) & 0xffffu;
                if ((x & 0x7f80u) == 0x7f80u) {
                    f |= (x != 0xff80u ? 1u << e : 0u) | (x != 0x7f80u ? 0x100u << e : 0u);
                    v[e / 2] &= e % 2 ? 0xffffu : 0xffff0000u;
                }
            }
            vinf[st][key][(lane % CH) ^ dswz<D>(key & (TK - 1))] = (uint16_t)f;
            if (f != 0) *at = v;
            found |= f;
        }
        const bool any = __builtin_amdgcn_ballot_w64(found != 0) != 0;
        if (lane == 0) vbad[st][wave] = any;
    };

    // ---- NT tiles: their K operands, V tiles, first key, stage and place in it, and whether their
    // keys have powers of two to give back
    auto tiles = [&](auto ntc, const u32x4_t (*kf)[KD], const uint16_t* vt, int k0, int st, int tile0, bool powers) {
        constexpr int NT = decltype(ntc)::value;
        f32x4_t sc[NT][CB];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    const f32x4_t from = kd == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[n][cb];
                    if (ROPE)
                        sc[n][cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, kf[n][kd]), __builtin_bit_cast(f16x8_t, qb[cb][kd]), from, 0, 0, 0);
                    else
                        sc[n][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[n][kd]), qb[cb][kd], from, 0, 0, 0);
                }
        if (ROPE && powers) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[n][cb][r] *= ksc[st][tile0 + n * TK + 4 * q4 + r];
        }
        const bool masked = k0 < k_lo || k_hi - k0 < NT * TK || k_tok - k0 < NT * TK;
        uint32_t seen[CB];   // masked tiles: the row's bits of the tiles' keys
        if (masked) {
            // keys [k_lo, k_hi) of the tiles (k0 < k_hi)
            const int lo = max(k_lo - k0, 0), hi = min(k_hi - k0, NT * TK);
            const uint32_t inside = (hi < 32 ? (1u << hi) - 1u : ~0u) & ~((1u << lo) - 1u);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                seen[cb] = inside & tree_bits(a.mask + (size_t)(g.q_row0 + toff[cb]) * a.words, a.words, k0 - k_tok);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!((seen[cb] >> (16 * n + 4 * q4 + r)) & 1)) sc[n][cb][r] = -INFINITY;
            }
            if (__builtin_amdgcn_ballot_w64(vbad[st][lane % NW] != 0) != 0) {
                // which of this lane's outputs the seen infinities reach
#pragma unroll 1
                for (int k = 0; k < NT * TK; ++k)
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb)
                        if ((seen[cb] >> k) & 1)
#pragma unroll 1
                            for (int db = 0; db < DB; ++db) {
                                const uint32_t both = vinf[st][tile0 + k][2 * db + (q4 >> 1)] >> (4 * (q4 & 1));
                                infs[wave][cb][db][lane] |= (uint8_t)((both & 15u) | ((both >> 4) & 0xf0u));
                            }
            }
        }
        float mx[CB];
        bool moves = false;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            mx[cb] = fmaxf(fmaxf(sc[0][cb][0], sc[0][cb][1]), fmaxf(sc[0][cb][2], sc[0][cb][3]));
#pragma unroll
            for (int n = 1; n < NT; ++n) mx[cb] = fmaxf(fmaxf(fmaxf(mx[cb], sc[n][cb][0]), sc[n][cb][1]), fmaxf(sc[n][cb][2], sc[n][cb][3]));
            mx[cb] = max_xor32(max_xor16(mx[cb])) * qs[cb];
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
                for (int db = 0; db < DB; ++db) acc[cb][db] *= alpha;
                m_run[cb] = m_new;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            u32x2_t af[DB];
#pragma unroll
            for (int db = 0; db < DB; ++db) af[db] = __builtin_bit_cast(u32x2_t, lds_read_tr(as_lds(vt + n * TK * D) + v_off[db]));
            u32x4_t pw[CB];   // upper and lower parts of the probabilities
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                float p[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][cb][r], qs[cb], -m_run[cb]));
                l_run[cb] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    pw[cb][h] = pack_bf16(p[2 * h], p[2 * h + 1]);
                    pw[cb][2 + h] = pack_bf16(p[2 * h] - bf_lo(pw[cb][h]), p[2 * h + 1] - bf_hi(pw[cb][h]));
                }
            }
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const u32x4_t twice = {af[db][0], af[db][1], af[db][0], af[db][1]};
#pragma unroll
                for (int cb = 0; cb < CB; ++cb)
                    acc[cb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, twice), __builtin_bit_cast(bf16x8_t, pw[cb]), acc[cb][db], 0, 0, 0);
            }
        }
    };
    // a step's copies have landed once no more than those of the `later` next ones are outstanding
    auto wait_step = [&](int u, auto later) {
        constexpr int L = decltype(later)::value;
        if (L > 0 && u + L < nt) wait_vmem_n<L * LPS>();
        else wait_vmem();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
    };
    auto load_k = [&](u32x4_t (&kf)[KD], const uint16_t* kt) {
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) kf[kd] = *reinterpret_cast<const u32x4_t*>(kt + k_off[kd]);
    };

    int st = 0;
    auto next = [](int x) { return x + 1 == NST ? 0 : x + 1; };
    auto prev = [](int x) { return x == 0 ? NST - 1 : x - 1; };
    Blocks blk{};
    if constexpr (!SHARED) {
        if (NST - 1 < nt) blk = blocks_of(NST - 1);
        for (int t = 0; t < nt; ++t) {
            wait_step(t, Idx<NST - 2>{});
            if (t + NST - 1 < nt) {
                issue(t + NST - 1, prev(st), blk);
                if (t + NST < nt) blk = blocks_of(t + NST);
            }
            const uint16_t* kt = stages + st * SE + wave * TK * D;
            clean(t, st);
            u32x4_t kf[1][KD];
            load_k(kf[0], kt);
            bool powers = false;
            if constexpr (ROPE) {
                uint32_t w[PL];   // runs in pair order, NeoX: all x, then all y
#pragma unroll
                for (int i = 0; i < PL; ++i) w[i] = kf[0][i / 4][i % 4];
                powers = turn(st, w);
#pragma unroll
                for (int i = 0; i < PL; ++i) kf[0][i / 4][i % 4] = w[i];
            }
            tiles(Idx<1>{}, kf, kt + KV, t * STEP + wave * TK, st, wave * TK, powers);
            st = next(st);
        }
    } else {
        typedef uint32_t run_t __attribute__((ext_vector_type(PL / 2)));
        // step u has landed; its keys are turned in place
        auto prepare = [&](int u, int sl) {
            if (u >= nt) return;
            wait_step(u, Idx<NST - 2>{});
            clean(u, sl);
            if constexpr (ROPE) {
                uint16_t* kt = stages + sl * SE;
                uint32_t w[PL];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const run_t x = *reinterpret_cast<const run_t*>(kt + s_off[h]);
#pragma unroll
                    for (int i = 0; i < PL / 2; ++i) w[h * PL / 2 + i] = x[i];
                }
                turn(sl, w);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    run_t x;
#pragma unroll
                    for (int i = 0; i < PL / 2; ++i) x[i] = w[h * PL / 2 + i];
                    *reinterpret_cast<run_t*>(kt + s_off[h]) = x;
                }
            }
        };
#pragma unroll
        for (int u = NST - SPARE; u < NST - 1; ++u)
            if (u < nt) issue(u, u, blocks_of(u));
        if (NST - 1 < nt) blk = blocks_of(NST - 1);
        prepare(0, 0);
        barrier_keep_vmem();
        constexpr int NT = KG == 4 ? 1 : 2;    // tiles at a time
        const bool live = row_lo < rows_total;
        for (int s = 0; s < nt; ++s) {
            // step s + NST - 1 goes where step s - 1 was
            if (s + NST - 1 < nt) {
                issue(s + NST - 1, prev(st), blk);
                if (s + NST < nt) blk = blocks_of(s + NST);
            }
            prepare(s + 1, next(st));
            if (live) {
                uint32_t flags = 0;
                if (ROPE) flags = (uint32_t)kbig[st][lane % NW];
                const bool powers = ROPE && __builtin_amdgcn_ballot_w64(flags != 0) != 0;
#pragma unroll 1
                for (int n = 0; n < 4 / KG; n += NT) {
                    const int k0 = s * STEP + (kg * (4 / KG) + n) * TK;
                    if (k0 >= k_hi) break;
                    const uint16_t* kt = stages + st * SE + (kg * (4 / KG) + n) * TK * D;
                    u32x4_t kf[NT][KD];
#pragma unroll
                    for (int m = 0; m < NT; ++m) load_k(kf[m], kt + m * TK * D);
                    tiles(Idx<NT>{}, kf, kt + KV, k0, st, (kg * (4 / KG) + n) * TK, powers);
                }
            }
            barrier_keep_vmem();
            st = next(st);
        }
    }

    // ---- the results of a row group's waves meet: rows by their common maximum, outputs through
    // the stages
    float M[CB], den[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        den[cb] = sum_xor32(sum_xor16(l_run[cb]));
        M[cb] = m_run[cb];
        if (KG > 1 && q4 == 0) mls[wave][16 * cb + c16] = make_float2(m_run[cb], den[cb]);
    }
    if (KG > 1) __syncthreads();   // (every wave's copies have landed and been read)
    f32x4_t* meet = reinterpret_cast<f32x4_t*>(stages);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        float mine = 1.f;
        if (KG > 1) {
            float2 w[KG];
#pragma unroll
            for (int i = 0; i < KG; ++i) {
                w[i] = mls[rg * KG + i][16 * cb + c16];
                M[cb] = fmaxf(M[cb], w[i].x);
            }
            den[cb] = 0.f;
#pragma unroll
            for (int i = 0; i < KG; ++i) den[cb] += w[i].y * __builtin_amdgcn_exp2f(w[i].x - M[cb]);
            mine = __builtin_amdgcn_exp2f(m_run[cb] - M[cb]);
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            f32x4_t x = acc[cb][db] * mine;
            const uint32_t f = infs[wave][cb][db][lane];
            if (f != 0)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] += ((f >> i) & 1 ? INFINITY : 0.f) - ((f >> (4 + i)) & 1 ? INFINITY : 0.f);
            if (KG > 1) meet[((wave * CB + cb) * DB + db) * 64 + lane] = x;
            else acc[cb][db] = x;
        }
    }
    if (KG > 1) __syncthreads();
    const size_t prow0 = ((size_t)g.part_base + (size_t)ic.cluster * n_rt + ic.rt) * (16 * CB * WR) + rg * 16 * CB;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row_lo + 16 * cb + c16;
        if (row >= rows_total) continue;
        const float inv = den[cb] == 0.f ? 0.f : 1.f / den[cb];   // (a drafted token may see nothing: its output is 0)
#pragma unroll
        for (int i = 0; i < (DB + KG - 1) / KG; ++i) {
            const int db = i * KG + kg;
            if (db >= DB) break;
            f32x4_t x;
            if (KG > 1) {
                x = meet[((rg * KG * CB + cb) * DB + db) * 64 + lane];
#pragma unroll
                for (int w = 1; w < KG; ++w) x += meet[(((rg * KG + w) * CB + cb) * DB + db) * 64 + lane];
            } else {
                x = acc[cb][i];
            }
            if (g.n_split > 1) {
                *reinterpret_cast<f32x4_t*>(a.part_o + (prow0 + 16 * cb + c16) * D + db * 16 + 4 * q4) = x;
            } else {
                const int hl = row - toff[cb] * G;
                uint16_t* op = static_cast<uint16_t*>(a.o) + ((size_t)(g.q_row0 + toff[cb]) * a.hq + (size_t)ic.kvh * G + hl) * D;
                *reinterpret_cast<u32x2_t*>(op + db * 16 + 4 * q4) = u32x2_t{pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
            }
        }
        if (g.n_split > 1 && kg == 0 && q4 == 0)
            *reinterpret_cast<float2*>(a.part_ml + (prow0 + 16 * cb + c16) * 2) = make_float2(M[cb], den[cb]);
    }
}

// Joins the key splits of tree_bf16: one block per kMergeRows rows of a (row tile, KV head),
// one float4 of a row per thread, eight splits' loads in flight.
template <int D>
__global__ void __launch_bounds__(kMergeRows * D / 4) tree_merge(const Plan plan, const TreeArgs a) {
    constexpr int TPR = D / 4, U = 8;
    const Group g = group_of<true>(plan, blockIdx.x);
    if (g.n_split <= 1) return;
    const int n_rt = g.n_rt, chunks = a.tile_rows / kMergeRows;
    int li = blockIdx.x - g.merge_base;
    if (li >= a.hkv * n_rt * chunks) return;
    const int r = (li % chunks) * kMergeRows + (int)threadIdx.x / TPR, c4 = (int)threadIdx.x % TPR;
    li /= chunks;
    const int kvh = li / n_rt, rt = li - kvh * n_rt, G = a.group;
    const int row = rt * a.tile_rows + r;
    if (row >= g.n_tok * G) return;
    const size_t slot0 = (size_t)g.part_base + (size_t)kvh * g.n_split * n_rt + rt;
    float M = kNegBig, den = 0.f;
    f32x4_t num = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < g.n_split; s0 += U) {
        float2 ml[U];
        f32x4_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t prow = (slot0 + (size_t)min(s0 + u, g.n_split - 1) * n_rt) * a.tile_rows + r;
            ml[u] = *reinterpret_cast<const float2*>(a.part_ml + prow * 2);
            v[u] = *reinterpret_cast<const f32x4_t*>(a.part_o + prow * D + c4 * 4);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u >= g.n_split || ml[u].y == 0.f) continue;   // past the end, or no key of this row
            const float m_new = fmaxf(M, ml[u].x);
            const float c_old = __builtin_amdgcn_exp2f(M - m_new), c_new = __builtin_amdgcn_exp2f(ml[u].x - m_new);
            num = num * c_old + c_new * v[u];
            den = den * c_old + c_new * ml[u].y;
            M = m_new;
        }
    }
    const float inv = den == 0.f ? 0.f : 1.f / den;
    const int to = row / G;
    uint16_t* op = static_cast<uint16_t*>(a.o) + ((size_t)(g.q_row0 + to) * a.hq + (size_t)kvh * G + (row - to * G)) * D + c4 * 4;
    *reinterpret_cast<u32x2_t*>(op) = u32x2_t{pack_bf16(num[0] * inv, num[1] * inv), pack_bf16(num[2] * inv, num[3] * inv)};
}

template <int D, int STYLE, bool ROPE>
hipError_t launch_tree_t(const Plan& plan, const TreeArgs& a, hipStream_t st) {
    const dim3 grid(plan.n_items), block(kTreeWaves * 64);
    switch (a.tile_rows) {
    case 16: hipLaunchKernelGGL((tree_bf16<D, STYLE, ROPE, 1, 1>), grid, block, 0, st, plan, a); break;
    case 32: hipLaunchKernelGGL((tree_bf16<D, STYLE, ROPE, 2, 1>), grid, block, 0, st, plan, a); break;
    case 64: hipLaunchKernelGGL((tree_bf16<D, STYLE, ROPE, 2, 2>), grid, block, 0, st, plan, a); break;
    case 128: hipLaunchKernelGGL((tree_bf16<D, STYLE, ROPE, 2, 4>), grid, block, 0, st, plan, a); break;
    default: hipLaunchKernelGGL((tree_bf16<D, STYLE, ROPE, 2, 8>), grid, block, 0, st, plan, a); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.n_merge == 0) return e;
    hipLaunchKernelGGL((tree_merge<D>), dim3(plan.n_merge), dim3(kMergeRows * D / 4), 0, st, plan, a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_tree_d(int style, bool rope, const Plan& plan, const TreeArgs& a, hipStream_t st) {
    if (!rope) return launch_tree_t<D, 0, false>(plan, a, st);   // (without rotation the pairing makes no difference)
    return style == kNeox ? launch_tree_t<D, 0, true>(plan, a, st) : launch_tree_t<D, 1, true>(plan, a, st);
}

template <typename T, int D>
void launch_append_d(int style, int n, int threads, const AppendArgs& a, hipStream_t st) {
    if (a.rot_half == 0)
        hipLaunchKernelGGL((kv_append_kernel<T, D, 1, false>), dim3(n), dim3(threads), 0, st, a);
    else if (style == kNeox)
        hipLaunchKernelGGL((kv_append_kernel<T, D, 0, true>), dim3(n), dim3(threads), 0, st, a);
    else
        hipLaunchKernelGGL((kv_append_kernel<T, D, 1, true>), dim3(n), dim3(threads), 0, st, a);
}

}  // namespace

int launch_tree(int style, int d, bool rope, const Plan& plan, const TreeArgs& args, void* stream) {
    if (plan.n_items == 0) return hipSuccess;
    return d == 64 ? launch_tree_d<64>(style, rope, plan, args, (hipStream_t)stream)
                   : launch_tree_d<128>(style, rope, plan, args, (hipStream_t)stream);
}

int launch_tree_mask(const int32_t* parents, const int32_t* cu_rows, int n_trees, int total_rows, uint64_t* mask, int words,
                     int32_t* depth, void* stream) {
    const int threads = words * 64 < 1024 ? words * 64 : 1024;
    hipLaunchKernelGGL(tree_mask_kernel, dim3(words, n_trees), dim3(threads), (size_t)words * 64 * 16, (hipStream_t)stream, parents,
                       cu_rows, total_rows, mask, words, depth);
    return hipGetLastError();
}

int launch_kv_append(int dtype, int style, int d, int n, const AppendArgs& a, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    const int64_t units = (int64_t)(a.hq + 2 * a.hkv) * (d * (dtype == 1 ? 4 : 2) / 32);
    const int threads = units >= kAppendThreads ? kAppendThreads : (int)((units + 63) / 64) * 64;
    if (dtype == 1) {
        if (d == 64) launch_append_d<float, 64>(style, n, threads, a, st);
        else launch_append_d<float, 128>(style, n, threads, a, st);
    } else {
        if (d == 64) launch_append_d<__bf16, 64>(style, n, threads, a, st);
        else launch_append_d<__bf16, 128>(style, n, threads, a, st);
    }
    return hipGetLastError();
}

int launch_kv_keep(int dtype, int hkv, int d, void* k_pool, void* v_pool, int64_t n_slots, const int32_t* slots,
                   const int32_t* cu_rows, const int32_t* path, const int32_t* path_len, int n_trees, int max_path, int total_rows,
                   void* stream) {
    const dim3 grid(n_trees, hkv);
    u32x4_t *kp = static_cast<u32x4_t*>(k_pool), *vp = static_cast<u32x4_t*>(v_pool);
    hipStream_t st = (hipStream_t)stream;
    const int cpr = d * (dtype == 1 ? 4 : 2) / 16;
    auto go = [&](auto c) {
        hipLaunchKernelGGL((kv_keep_kernel<decltype(c)::value>), grid, dim3(256), 0, st, kp, vp, n_slots, slots, cu_rows, path,
                           path_len, max_path, hkv, total_rows);
    };
    if (cpr == 8) go(Idx<8>{});
    else if (cpr == 16) go(Idx<16>{});
    else go(Idx<32>{});
    return hipGetLastError();
}

}  // namespace pic
