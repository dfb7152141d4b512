// HIP kernels of speculative decoding over the paged cache, for MI355X (gfx950, CDNA4).
//
//  * kv_append  rows of a projection: k and v into the pool's slots, q packed; k and q
//               turned at their positions on the way where the pool holds turned keys.
//  * tree_mask  ancestor bits and depths of drafted trees.
//  * tree_few, tree_many  attention of the drafted tokens in bf16; tree_merge joins their key
//               splits.  (float32: attn_f32 over TreeArgs, in pic_kernels.hip)
//  * kv_keep    the accepted rows of every tree move to the front of its slots.
#include <type_traits>

#include "pic_device.h"

namespace pic {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) const u32x4_t lds_u32x4_t;

// ---------------------------------------------------------------------------------
// kv_append: one workgroup per row.  A unit is two 16-byte chunks of a head: NeoX the two
// runs whose elements pair up, GPT-J (and V, and what does not turn) two neighbours.  A
// thread's units lie on the same pairs of different heads, so it computes their cos/sin
// once, in float32 from the exact phase.  Bound by memory: every element is read once and
// written once, four units (128 bytes) of a thread in flight.  16,384 rows of 64 + 2 x 8 heads of
// 128 (671 MB) 121 us, 5.5 TB/s (a copy of 2 GiB 4.9); 8,192 such rows in float32 125 us, and 16,384
// that do not turn 124.  Few rows are bound by latency: the slot, which only the stores need, is waited
// for before a row is read, and the position asked for after it: 528 rows of 32 + 2 x 8 (13 MB) 5.4
// to 5.8 us, 2.6 at the copy's rate.
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
// Bound by latency: log2 of the depth rounds in LDS, where walking from parent to parent would take
// the depth.  64 trees of 15 to 61 tokens 3.8 us, 3 of 1,000 (16 words) 7.6.
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
// reads.  Bound by latency (lengths, path, slots, rows: four dependent reads); a pass moves 256
// chunks of 16 bytes.  64 trees keeping 8 rows of 8 heads of 128 2.9 us, 256 keeping 41 of 2
// heads of 64 in float32 (5.2 MB) 4.2.
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

// ---------------------------------------------------------------------------------
// Attention of drafted tokens in bf16: tree_few and tree_many
//
// Workgroup: eight waves (two per SIMD, so that one's products run under the other's vector
// work) over some query rows (drafted token x query head of one KV head's group) and one key
// range.  K, V and the keys' positions go straight to LDS, some steps ahead.
//   tree_few   up to 32 rows, held by every wave.  A wave takes every eighth 16-key tile (one
//              cache block) of the range, which it copies, turns and multiplies without waiting
//              for another wave; the eight results meet in LDS at the end.
//   tree_many  128 or 256 rows, 32 of a wave, in steps of 64 keys that all waves share.  A wave
//              copies and turns eight keys of a step, in place, one step before they are
//              multiplied; one barrier per step.
//
// Precision: a rotated key or query is rounded to 11 bits (float16), its size held by a power
// of two where it does not fit: as bf16, 8 bits, each of the two alone would put outputs as
// far from 64 bits as their own rounding does.  Without rotation q and k are exact.
// tree_few multiplies a probability as two bf16 numbers, its upper 8 bits and the rest, in the
// time of one.  In tree_many the second number would cost half as many products again (16 x 96
// tokens of 64 / 8 heads over 8,192 keys 766 us, without it 632): a probability is rounded to
// bf16, and the row sum adds the rounded ones, which brings outputs to 1.4 times the error of
// their own rounding.
//
// RoPE: a lane turns PL pairs of one key of a step and holds their cos/sin.  Its next key is
// STEP keys further; where the positions are too, the angles advance by a constant rotation (4
// operations a pair, renewed every kRenew steps), else they are computed.
// ---------------------------------------------------------------------------------
constexpr int kRenew = 32;

// Sizes of the two kernels' steps (SHARED: tree_many)
template <int D, bool SHARED>
struct TreeShape {
    static constexpr int CH = D / 8;             // 16-byte chunks per K/V row
    static constexpr int HALF = D / 2;
    static constexpr int NW = kTreeWaves;
    static constexpr int STEP = SHARED ? 64 : NW * kBlock;   // keys of all waves
    static constexpr int OWNK = STEP / NW;       // keys that a wave copies and turns
    static constexpr int PL = OWNK * HALF / 64;  // pairs that a lane turns
    static constexpr int NST = SHARED || D == 64 ? 4 : 2;    // steps in LDS
    static constexpr int KPC = 64 / CH;          // keys per copy (64 chunks)
    static constexpr int DPL = OWNK / KPC;       // copies per lane per step, each of K and V
    static constexpr int KV = STEP * D;          // elements of K or V in a stage
    static constexpr int SE = 2 * KV;            // elements of a stage: K of every tile, then V
};

// (SHARED: stages begin at a multiple of a row, within which chunks are found by an exclusive or on
// their addresses)
template <int D, bool SHARED>
struct __attribute__((aligned(SHARED ? 2 * D : 16))) TreeLds {
    typedef TreeShape<D, SHARED> S;
    uint16_t stages[S::NST * S::SE];
    float2 stride_cs[S::HALF];           // cos/sin of STEP positions
    uint64_t fstep[S::HALF];
    int32_t ps[S::NW][S::NST][S::OWNK];  // positions
    float ksc[S::NST][S::STEP];          // powers of two held back from a step's keys
    int32_t kbig[S::NST][S::NW];         // whether some key of a wave has one
    // Steps in which rows differ in what they see: infinities of V (bits 0-7: +, 8-15: -, of a
    // chunk's dimensions, a NaN both), and whether a wave's keys have some
    uint16_t vinf[S::NST][S::STEP][S::CH];
    int32_t vbad[S::NST][S::NW];
};

// A wave's share of the keys of a workgroup's range: copies into LDS, angles, turning.
template <int D, int STYLE, bool ROPE, bool SHARED>
struct TreeKeys : TreeShape<D, SHARED> {
    typedef TreeShape<D, SHARED> S;
    using S::CH; using S::HALF; using S::NW; using S::STEP; using S::OWNK; using S::PL; using S::NST; using S::KPC;
    using S::DPL; using S::KV; using S::SE;
    static constexpr int LPS = 2 * DPL + (ROPE ? 1 : 0);   // copies per lane per step
    static constexpr int RUN = SHARED ? PL : STYLE == kNeox ? 8 : 4;   // pairs in a row
    static_assert((NST - 2) * LPS < 64, "vmcnt range");

    TreeLds<D, SHARED>& s;
    int lane, wave;
    int k_lo, k_hi, k_tok;     // first and last key + 1 of the range, and the span's start, from kt0, the start of the first block
    int nt;                    // steps in which this wave copies keys
    const int32_t* btab;
    const int32_t* posv;
    const uint16_t* kpool;
    const uint16_t* vpool;
    size_t blk_stride;
    uint32_t stages_at, ps_at;
    uint32_t lane_off[DPL];    // byte offset within one head's page of a block
    int own_j, pair0, sh_row;  // the key that the lane turns (of the wave's, of the step), and its first pair
    // SHARED: element offsets of the lane's two runs (NeoX) or of its 2 PL neighbours (GPT-J), as
    // copied and (in the order of the kernel's chunks) as turned
    int s_off[2], t_off[2];
    float rc[PL], rs[PL];      // cos/sin at position cs_pos
    int32_t cs_pos = 0;
    int fresh = 0;             // steps until the angles are computed again

    struct Blocks {
        int b[SHARED ? DPL : 1];   // (without sharing a step's copies are of one block)
    };

    // The i-th copy of a step moves 64 chunks, KPC keys from copy_key(i) on.  A key outside
    // [k_lo, k_hi) stands for the nearest one inside, so that nothing outside the range is
    // read (its score is masked).
    __device__ __forceinline__ int copy_key(int i) const { return SHARED ? (i * NW + wave) * KPC : wave * kBlock + i * KPC; }
    __device__ __forceinline__ int near_key(int k) const { return min(max(k, k_lo), k_hi - 1); }
    // own key j (0 .. OWNK - 1) of a step: its place in the step
    __device__ __forceinline__ int own_key(int j) const { return copy_key(j / KPC) + j % KPC; }
    __device__ __forceinline__ int pair_of(int i) const { return pair0 + (SHARED ? i : i / RUN * 4 * RUN + i % RUN); }

    __device__ __forceinline__ TreeKeys(TreeLds<D, SHARED>& lds, const TreeArgs& a, const Group& g, const ItemCoords& ic)
        : s(lds), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) {
        const int kv_lo = g.win + ic.split * g.split_keys, end = g.tok0 + g.n_tok;
        // (no sum below passes the last key: a request may have 2^31 - 1 of them)
        const int kv_hi = g.split_keys < end - kv_lo ? kv_lo + g.split_keys : end;
        const int kt0 = kv_lo & ~(kBlock - 1);
        k_lo = kv_lo - kt0;
        k_hi = kv_hi - kt0;
        k_tok = g.tok0 - kt0;
        const int n_tiles = (k_hi - 1) / kBlock + 1;
        nt = SHARED ? (k_hi - 1) / STEP + 1 : n_tiles > wave ? (n_tiles - wave - 1) / NW + 1 : 0;
        btab = a.block_tables + (size_t)g.req * a.max_blocks + (kt0 >> 4);
        posv = a.positions + g.pos_off + kt0;
        blk_stride = (size_t)a.hkv * kBlock * D;
        kpool = static_cast<const uint16_t*>(a.k_pool) + (size_t)ic.kvh * kBlock * D;
        vpool = static_cast<const uint16_t*>(a.v_pool) + (size_t)ic.kvh * kBlock * D;
        stages_at = lds_offset(s.stages);
        ps_at = lds_offset(&s.ps[wave][0][0]);
#pragma unroll
        for (int i = 0; i < DPL; ++i) {
            const int row = (copy_key(i) + lane / CH) & (kBlock - 1);
            lane_off[i] = (uint32_t)(row * D + (((lane % CH) ^ dswz<D>(row)) << 3)) * 2;
        }
        // Without sharing a lane has the operand's elements of key lane % 16: runs of 8 (NeoX pairs
        // 32 kd + 8 (lane / 16) + e of chunks kd and kd + KD / 2; GPT-J pairs 16 kd + 4 (lane / 16)
        // + m).  With sharing 8 lanes have one key, PL pairs (lane % 8) * PL + i each.
        own_j = SHARED ? lane >> 3 : lane & 15;
        pair0 = SHARED ? (lane & 7) * PL : RUN * (lane >> 4);
        sh_row = own_key(own_j);
        if (SHARED) {
            const int e0 = STYLE == kNeox ? pair0 : 2 * pair0, e1 = STYLE == kNeox ? pair0 + HALF : e0 + PL;
            const int row = sh_row & (kBlock - 1);
            for (int h = 0; h < 2; ++h) {
                const int e = h == 0 ? e0 : e1;
                s_off[h] = sh_row * D + ((model_chunk(a.chunk_map, e >> 3) ^ dswz<D>(row)) << 3) + (e & 7);
                t_off[h] = sh_row * D + (((e >> 3) ^ dswz<D>(row)) << 3) + (e & 7);
            }
        }
    }

    // phase steps and the angles of STEP positions (all threads; a barrier follows)
    __device__ __forceinline__ void fill_steps(const TreeArgs& a) {
        if (ROPE)
            for (int i = threadIdx.x; i < HALF; i += NW * 64) {
                s.fstep[i] = a.fstep[i];
                rope_cs_fast(STEP, a.fstep[i], s.stride_cs[i].x, s.stride_cs[i].y);
            }
    }
    __device__ __forceinline__ Blocks blocks_of(int u) const {
        Blocks r;
#pragma unroll
        for (int i = 0; i < (SHARED ? DPL : 1); ++i) r.b[i] = scalar_load(btab, min(u * STEP + copy_key(i), k_hi - 1) >> 4);
        return r;
    }
    // the wave's copies of step u, into stage st
    __device__ __forceinline__ void issue(int u, int st, const Blocks& blk) const {
        const uint32_t sg = stages_at + (uint32_t)st * SE * 2;
        // the stage's last reads have returned (SHARED: before the last barrier)
        if (!SHARED) __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));
        const bool whole = u * STEP >= k_lo && (u + 1) * STEP <= k_hi;   // the step needs no nearest keys
        if (ROPE && lane < OWNK) {
            const int k = u * STEP + own_key(lane);
            copy_lds4(posv + (whole ? k : near_key(k)), ps_at + (uint32_t)st * OWNK * 4);
        }
#pragma unroll
        for (int i = 0; i < DPL; ++i) {
            const size_t base = (size_t)(uint32_t)blk.b[SHARED ? i : 0] * blk_stride;
            uint32_t off = lane_off[i];
            if (!whole) {
                const int k = u * STEP + copy_key(i) + lane / CH, row = k & (kBlock - 1);
                off += ((near_key(k) & (kBlock - 1)) - row) * D * 2;
            }
            copy_lds16(kpool + base, off, sg + copy_key(i) * D * 2);
            copy_lds16(vpool + base, off, sg + KV * 2 + copy_key(i) * D * 2);
        }
    }
    // step u's copies have landed once no more than those of the LATER next ones are outstanding
    template <int LATER>
    __device__ __forceinline__ void wait_step(int u) const {
        if (LATER > 0 && u + LATER < nt) wait_vmem_n<LATER * LPS>();
        else wait_vmem();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
    }
    // the first of ISSUED steps' positions have landed
    template <int ISSUED>
    __device__ __forceinline__ void wait_first() const {
        if (nt >= ISSUED) wait_vmem_n<ISSUED * LPS - 1>();
        else wait_vmem();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
    }
    // the angles of the lane's key of the step in stage st, computed where they cannot be advanced
    __device__ __forceinline__ void find_angles(int st) {
        const int32_t pos = s.ps[wave][st][own_j];
        // (STEP on, and not past the type's end)
        if (fresh == 0 || __builtin_amdgcn_ballot_w64((uint32_t)pos != (uint32_t)cs_pos + STEP || pos < cs_pos) != 0) {
#pragma unroll
            for (int i = 0; i < PL; ++i) rope_cs_fast((int64_t)pos - STEP, s.fstep[pair_of(i)], rc[i], rs[i]);
            fresh = kRenew;
        }
        --fresh;
        cs_pos = pos;
    }
    // pairs i and i + 1: their angles a step on, and 4 elements turned (times 2^-ex if SCALED; big
    // takes in their sizes)
    __device__ __forceinline__ void advance_pairs(int i0) {
#pragma unroll
        for (int i = i0; i < i0 + 2; ++i) {
            const float2 d = s.stride_cs[pair_of(i)];
            const float c = rc[i], sn = rs[i];
            rc[i] = c * d.x - sn * d.y;
            rs[i] = sn * d.x + c * d.y;
        }
    }
    template <bool SCALED>
    __device__ __forceinline__ void rotate_pairs(int i, const uint32_t (&w)[PL], uint32_t (&out)[PL], int ex, float& big) const {
        const uint32_t A = STYLE == kNeox ? w[i / 2] : w[i], B = STYLE == kNeox ? w[PL / 2 + i / 2] : w[i + 1];
        const float x0 = bf_lo(A), y0 = STYLE == kNeox ? bf_lo(B) : bf_hi(A);
        const float x1 = STYLE == kNeox ? bf_hi(A) : bf_lo(B), y1 = bf_hi(B);
        float p0 = x0 * rc[i] - y0 * rs[i], r0 = y0 * rc[i] + x0 * rs[i];
        float p1 = x1 * rc[i + 1] - y1 * rs[i + 1], r1 = y1 * rc[i + 1] + x1 * rs[i + 1];
        if (SCALED) {
            p0 = ldexpf(p0, -ex); r0 = ldexpf(r0, -ex); p1 = ldexpf(p1, -ex); r1 = ldexpf(r1, -ex);
        } else {
            big = fmaxf(fmaxf(big, fabsf(p0)), fabsf(r0));
            big = fmaxf(fmaxf(big, fabsf(p1)), fabsf(r1));
        }
        out[STYLE == kNeox ? i / 2 : i] = STYLE == kNeox ? pack_f16(p0, p1) : pack_f16(p0, r0);
        out[STYLE == kNeox ? PL / 2 + i / 2 : i + 1] = STYLE == kNeox ? pack_f16(r0, r1) : pack_f16(p1, r1);
    }
    // Turns 2 PL elements, words w[0 .. PL): NeoX x in the first half and y in the second.  Returns
    // the largest one's size (of the lane).
    __device__ __forceinline__ float turn(const uint32_t (&w)[PL], uint32_t (&out)[PL]) {
        float big = 0.f;
#pragma unroll
        for (int i = 0; i < PL; i += 2) {
            advance_pairs(i);
            rotate_pairs<false>(i, w, out, 0, big);
        }
        return big;
    }
    // A key whose largest element lies outside 2^-8 .. 2^15 goes in times a power of two that puts it
    // just below 2^15; returns whether some key of the wave does.
    __device__ __forceinline__ bool fit(int st, const uint32_t (&w)[PL], uint32_t (&out)[PL], float big) {
        big = SHARED ? max_of8(big) : max_xor32(max_xor16(big));
        const bool odd = big >= 0x1p15f || (big < 0x1p-8f && big > 0.f);
        const bool any = __builtin_amdgcn_ballot_w64(odd) != 0;
        int ex = 0;
        if (any) {
            ex = odd && big < INFINITY ? __builtin_amdgcn_frexp_expf(big) - 15 : 0;
            float none = 0.f;
#pragma unroll
            for (int i = 0; i < PL; i += 2) rotate_pairs<true>(i, w, out, ex, none);
        }
        if (SHARED) {
            if ((lane & 7) == 0) s.ksc[st][sh_row] = ldexpf(1.f, ex);
            if (lane == 0) s.kbig[st][wave] = any;
        } else if (any && lane < 16) {
            s.ksc[st][sh_row] = ldexpf(1.f, ex);
        }
        return any;
    }
    // SHARED: the lane's two runs of the step in stage st as copied, and as turned
    typedef uint32_t run_t __attribute__((ext_vector_type(PL / 2)));
    __device__ __forceinline__ void load_runs(int st, uint32_t (&w)[PL]) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const run_t x = *reinterpret_cast<const run_t*>(s.stages + st * SE + s_off[h]);
#pragma unroll
            for (int i = 0; i < PL / 2; ++i) w[h * PL / 2 + i] = x[i];
        }
    }
    __device__ __forceinline__ void store_runs(int st, const uint32_t (&w)[PL]) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            run_t x;
#pragma unroll
            for (int i = 0; i < PL / 2; ++i) x[i] = w[h * PL / 2 + i];
            *reinterpret_cast<run_t*>(s.stages + st * SE + t_off[h]) = x;
        }
    }
    // An infinity or NaN in V must not reach rows that do not see its key (0 x Inf in the
    // product): where keys that are scored together are not all seen by every row, the wave that
    // copied them puts zeros in their place and notes them; what rows see of them joins their
    // outputs at the end.
    static constexpr int TOGETHER = SHARED ? 32 : kBlock;
    __device__ __forceinline__ void clean(int u, int st) {
        if (!masked(u * STEP, STEP)) return;
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < DPL; ++i) {
            if (!masked(u * STEP + (copy_key(i) & ~(TOGETHER - 1)), TOGETHER)) continue;
            const int key = copy_key(i) + lane / CH;
            u32x4_t* at = reinterpret_cast<u32x4_t*>(s.stages + st * SE + KV + copy_key(i) * D + lane * 8);
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
            s.vinf[st][key][(lane % CH) ^ dswz<D>(key & (kBlock - 1))] = (uint16_t)f;
            if (f != 0) *at = v;
            found |= f;
        }
        const bool any = __builtin_amdgcn_ballot_w64(found != 0) != 0;
        if (lane == 0) s.vbad[st][wave] = any;
    }
    // the infinities of V that 4 dimensions (half h of chunk c) have in key k of a step: +, 4 bits, and -, 4 bits
    __device__ __forceinline__ uint32_t infs_of(int st, int k, int c, int h) const {
        const uint32_t both = (uint32_t)s.vinf[st][k][c] >> (4 * h);
        return (both & 15u) | ((both >> 4) & 0xf0u);
    }
    __device__ __forceinline__ bool wave_flag(const int32_t (&f)[NW]) const { return __builtin_amdgcn_ballot_w64(f[lane % NW] != 0) != 0; }
    // keys [k_lo, k_hi) among the 32 from k0 on
    __device__ __forceinline__ uint32_t inside(int k0, int n) const {
        const int lo = min(max(k_lo - k0, 0), 31), hi = max(min(k_hi - k0, n), 0);
        return (hi < 32 ? (1u << hi) - 1u : ~0u) & ~((1u << lo) - 1u);
    }
    // whether some row may not see one of n keys from k0 on
    __device__ __forceinline__ bool masked(int k0, int n) const { return k0 < k_lo || k_hi - k0 < n || k_tok - k0 < n; }
    static __device__ __forceinline__ int next(int st) { return st + 1 == NST ? 0 : st + 1; }
    static __device__ __forceinline__ int prev(int st) { return st == 0 ? NST - 1 : st - 1; }
};

// x with the infinities noted for its 4 dimensions
__device__ __forceinline__ f32x4_t with_infs(f32x4_t x, uint32_t f) {
    if (f != 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += ((f >> i) & 1 ? INFINITY : 0.f) - ((f >> (4 + i)) & 1 ? INFINITY : 0.f);
    return x;
}

// cos/sin of a wave's tokens t0 .. t1 of the span (at most 16; HALF pairs each) into cs
template <int HALF>
__device__ __forceinline__ void token_angles(const TreeArgs& a, const Group& g, const uint64_t* fstep, int lane, int t0, int t1, float2* cs) {
    const int32_t pos = a.positions[g.pos_off + g.tok0 + min(t0 + (lane & 15), t1)];   // of token t0 + lane
    const uint64_t step = fstep[lane % HALF];
    for (int i = lane; i < (t1 - t0 + 1) * HALF; i += 64) {
        float c, s;
        rope_cs_fast(__shfl(pos, i / HALF), step, c, s);
        cs[i] = make_float2(c, s);
    }
}

// A query row's N chunks of 8 elements in xf turned by the angles tc (HALF pairs); the lane has
// chunks c0 + i * dc (NeoX: the partners are N / 2 chunks on in xf).  Returns the largest size.
template <int STYLE, int N>
__device__ __forceinline__ float turn_row(float (&xf)[N][8], const float2* tc, int c0, int dc) {
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
        const int k = STYLE == kNeox ? i / 8 : i / 4, e = STYLE == kNeox ? i % 8 : i % 4;
        const float2 t = tc[STYLE == kNeox ? (c0 + k * dc) * 8 + e : (c0 + k * dc) * 4 + e];
        float& x = STYLE == kNeox ? xf[k][e] : xf[k][2 * e];
        float& y = STYLE == kNeox ? xf[k + N / 2][e] : xf[k][2 * e + 1];
        const float x0 = x, y0 = y;
        x = x0 * t.x - y0 * t.y;
        y = y0 * t.x + x0 * t.y;
        big = fmaxf(big, fmaxf(fabsf(x), fabsf(y)));
    }
    return big;
}

// A query row whose largest element is big goes in times 2^-ex, within 1.  A small row goes in
// within 2^-7: with a key of up to 2^15 its products stay below 2^15, and times the largest
// power of two of a key, 2^113, in range.  (Not a large one: its factor must stay in range too.)
__device__ __forceinline__ int query_exponent(float big) {
    return big > 0.f && big < INFINITY ? __builtin_amdgcn_frexp_expf(big) + (big < 1.f ? 7 : 0) : 0;
}
// The products' factor with it: not 0, with which a masked -Inf would be NaN.
__device__ __forceinline__ float back_scale(float scale, int ex) { return fmaxf(ldexpf(scale, ex), 0x1p-149f); }

// ---------------------------------------------------------------------------------
// tree_few: up to 16 CB rows.
//   S^T (16 keys x 16 rows) = K Q^T       v_mfma_f32_16x16x32_f16 (bf16 without rotation)
//   O^T (16 dims x 16 rows) += V^T P^T    v_mfma_f32_16x16x32_bf16, V^T by ds_read_b64_tr_b16
// After the scores lane l holds row l%16 of each block and keys 4 (l/16) + {0..3}, the B
// operand of the output product.
// With keys of their own bound by memory (32 requests of 8 tokens over 8,192 keys, 8 KV heads of
// 128: 191 to 196 us, 5.5 to 5.6 TB/s; the vector unit, which turns the keys, is busy 45%, the matrix
// cores 11%), with few keys by an item's start: about 6 us with 16 rows, 7 with 32, and 1.5 or 1.7 per step.
// ---------------------------------------------------------------------------------
template <int D, int STYLE, bool ROPE, int CB, int NG>
__global__ void __launch_bounds__(kTreeWaves * 64, 2) tree_few(const PlanOf<NG> plan, const TreeArgs a) {
    typedef TreeKeys<D, STYLE, ROPE, false> Keys;
    constexpr int KD = D / 32;             // 16x16x32 contraction steps of QK^T
    constexpr int DB = D / 16;             // 16-dim blocks of O^T
    constexpr int TK = kBlock, NW = kTreeWaves, NST = Keys::NST, PL = Keys::PL, HALF = D / 2;
    constexpr int PER = Keys::SE / NW;     // elements of a stage per wave
    constexpr int PPT = TK * D / 512;      // a wave's outputs of 16 x 16 in the place of a tile of K or V
    static_assert(NST * 2 * PPT >= CB * DB, "the outputs meet in the stages");
    static_assert(PER * 2 >= KD * 64 * 16, "queries pass through a stage");

    __shared__ TreeLds<D, false> lds;
    __shared__ float2 mls[NW][16 * CB];
    __shared__ float qsl[16 * CB];
    __shared__ uint8_t infs[NW][CB * DB][64];   // infinities of V that a lane's rows see (Keys::infs_of), if `noted`

    const Group g = group_of<false>(plan, blockIdx.x);
    const int G = a.group, n_rt = g.n_rt;
    const int li = blockIdx.x - g.item_base;   // (a call's items are not padded: below the group's count)
    const ItemCoords ic = item_coords(g, a.hkv, n_rt, li);
    const int rows_total = g.n_tok * G, row_lo = ic.rt * 16 * CB;
    Keys keys(lds, a, g, ic);
    const int lane = keys.lane, wave = keys.wave, nt = keys.nt;
    const int c16 = lane & 15, q4 = lane >> 4;
#pragma unroll
    for (int u = 0; u < NST - 1; ++u)
        if (u < nt) keys.issue(u, u, keys.blocks_of(u));
    keys.fill_steps(a);

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

    // ---- queries: a wave turns 2 CB rows, LPR lanes a row, and passes them to the others through the
    // stage that is filled last
    int toff[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row_lo + 16 * cb + c16;
        toff[cb] = row < rows_total ? row / G : 0;
    }
    {
        constexpr int LPR = 32 / CB, PP = HALF / LPR;   // lanes of a row, pairs of a lane
        static_assert(NW * 64 == 16 * CB * LPR, "every lane has a part of a row");
        typedef uint16_t part_t __attribute__((ext_vector_type(PP)));
        const int r = (wave * 64 + lane) / LPR, p0 = lane % LPR * PP, row = row_lo + r;
        const bool valid = row < rows_total;
        const int to = valid ? row / G : 0, hl = valid ? row - to * G : 0;
        // two runs of PP elements: NeoX the pairs' x and y, GPT-J one after the other
        const int e[2] = {STYLE == kNeox ? p0 : 2 * p0, STYLE == kNeox ? p0 + HALF : 2 * p0 + PP};
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((size_t)(g.q_row0 + to) * a.hq + (size_t)ic.kvh * G + hl) * D;
        part_t x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) x[h] = *reinterpret_cast<const part_t*>(qp + model_chunk(a.chunk_map, e[h] >> 3) * 8 + (e[h] & 7));
        const int32_t pos = ROPE ? a.positions[g.pos_off + g.tok0 + to] : 0;
        __syncthreads();  // phase steps staged
        float f[2 * PP];
#pragma unroll
        for (int i = 0; i < 2 * PP; ++i) f[i] = valid ? __uint_as_float((uint32_t)x[i / PP][i % PP] << 16) : 0.f;
        float scale = a.scale_log2;
        if (ROPE) {
            float big = 0.f;
#pragma unroll
            for (int i = 0; i < PP; ++i) {
                float c, s;
                rope_cs_fast(pos, lds.fstep[p0 + i], c, s);
                float& u = STYLE == kNeox ? f[i] : f[2 * i];
                float& v = STYLE == kNeox ? f[PP + i] : f[2 * i + 1];
                const float u0 = u, v0 = v;
                u = u0 * c - v0 * s;
                v = v0 * c + u0 * s;
                big = fmaxf(big, fmaxf(fabsf(u), fabsf(v)));
            }
            big = max_of8(big);
            big = fmaxf(big, __shfl_xor(big, 8));
            if (LPR == 32) big = max_xor16(big);
            const int ex = query_exponent(big);
            scale = back_scale(scale, ex);
#pragma unroll
            for (int i = 0; i < 2 * PP; ++i) x[i / PP][i % PP] = __builtin_bit_cast(uint16_t, (_Float16)ldexpf(f[i], -ex));
        } else if (!valid) {
            x[0] = x[1] = part_t(0);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = e[h] >> 3;   // chunk: of the lanes 16 (k % 4) + row of step k / 4
            *reinterpret_cast<part_t*>(lds.stages + (NST - 1) * Keys::SE + (r >> 4) * PER + ((k >> 2) * 64 + (k & 3) * 16 + (r & 15)) * 8 + (e[h] & 7)) = x[h];
        }
        if (lane % LPR == 0) qsl[r] = scale;
    }
    if (ROPE && nt > 0) {   // the first tile's angles, while its keys come
        keys.template wait_first<NST - 1>();
        keys.find_angles(0);
    }
    barrier_keep_vmem();
    bf16x8_t qb[CB][KD];
    float qs[CB];     // scores are the products times this (log2 units)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const uint16_t* from = lds.stages + (NST - 1) * Keys::SE + cb * PER;
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) qb[cb][kd] = *reinterpret_cast<const bf16x8_t*>(from + (kd * 64 + lane) * 8);
        qs[cb] = qsl[16 * cb + c16];
    }
    barrier_keep_vmem();   // every wave has its rows: the stage may be filled

    f32x4_t acc[CB][DB];
    float m_run[CB], l_run[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        m_run[cb] = kNegBig;
        l_run[cb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[cb][db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    int st = 0;
    bool noted = false;
    typename Keys::Blocks blk{};
    if (NST - 1 < nt) blk = keys.blocks_of(NST - 1);
    for (int t = 0; t < nt; ++t) {
        keys.template wait_step<NST - 2>(t);
        if (t + NST - 1 < nt) {
            keys.issue(t + NST - 1, keys.prev(st), blk);
            if (t + NST < nt) blk = keys.blocks_of(t + NST);
        }
        const uint16_t* kt = lds.stages + st * Keys::SE + wave * TK * D;
        const int k0 = t * Keys::STEP + wave * TK;
        keys.clean(t, st);
        u32x4_t kf[KD];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) kf[kd] = *reinterpret_cast<const u32x4_t*>(kt + k_off[kd]);
        bool powers = false;
        if constexpr (ROPE) {
            uint32_t w[PL];   // runs in pair order, NeoX: all x, then all y
#pragma unroll
            for (int i = 0; i < PL; ++i) w[i] = kf[i / 4][i % 4];
            uint32_t out[PL];
            if (t > 0) keys.find_angles(st);
            const float big = keys.turn(w, out);
            powers = keys.fit(st, w, out, big);
#pragma unroll
            for (int i = 0; i < PL; ++i) kf[i / 4][i % 4] = out[i];
        }
        f32x4_t sc[CB];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const f32x4_t from = kd == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[cb];
                if (ROPE)
                    sc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, kf[kd]), __builtin_bit_cast(f16x8_t, qb[cb][kd]), from, 0, 0, 0);
                else
                    sc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[kd]), qb[cb][kd], from, 0, 0, 0);
            }
        if (ROPE && powers) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int r = 0; r < 4; ++r) sc[cb][r] *= lds.ksc[st][wave * TK + 4 * q4 + r];
        }
        if (keys.masked(k0, Keys::TOGETHER)) {
            const uint32_t inside = keys.inside(k0, TK);
            uint32_t seen[CB];   // the row's bits of the tile's keys
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                seen[cb] = inside & tree_bits(a.mask + (size_t)(g.q_row0 + toff[cb]) * a.words, a.words, k0 - keys.k_tok);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (!((seen[cb] >> (4 * q4 + r)) & 1)) sc[cb][r] = -INFINITY;
            }
            if (__builtin_amdgcn_readfirstlane(lds.vbad[st][wave]) != 0) {
                // which of this lane's outputs the seen infinities reach
#pragma unroll 1
                for (int i = 0; i < CB * DB && !noted; ++i) infs[wave][i][lane] = 0;
                noted = true;
#pragma unroll 1
                for (int k = 0; k < TK; ++k)
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb)
                        if ((seen[cb] >> k) & 1)
#pragma unroll 1
                            for (int db = 0; db < DB; ++db)
                                infs[wave][cb * DB + db][lane] |= (uint8_t)keys.infs_of(st, wave * TK + k, 2 * db + (q4 >> 1), q4 & 1);
            }
        }
        float mx[CB];
        bool moves = false;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            mx[cb] = fmaxf(fmaxf(sc[cb][0], sc[cb][1]), fmaxf(sc[cb][2], sc[cb][3]));
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
        // Upper and lower parts of the probabilities: the upper cut off, so that no part is negative, the
        // lower of a probability above 0 never 0: an infinity that a row sees times them is that infinity.
        u32x4_t pw[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[cb][r], qs[cb], -m_run[cb]));
            l_run[cb] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pw[cb][h] = __builtin_amdgcn_perm(__float_as_uint(p[2 * h + 1]), __float_as_uint(p[2 * h]), 0x07060302u);
                pw[cb][2 + h] = pack_bf16(__builtin_amdgcn_fmed3f(p[2 * h] - bf_lo(pw[cb][h]), p[2 * h], 0x1p-126f),
                                          __builtin_amdgcn_fmed3f(p[2 * h + 1] - bf_hi(pw[cb][h]), p[2 * h + 1], 0x1p-126f));
            }
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const u32x2_t af = __builtin_bit_cast(u32x2_t, lds_read_tr(as_lds(kt + Keys::KV) + v_off[db]));
            const u32x4_t twice = {af[0], af[1], af[0], af[1]};
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                acc[cb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, twice), __builtin_bit_cast(bf16x8_t, pw[cb]), acc[cb][db], 0, 0, 0);
        }
        st = keys.next(st);
    }

    // ---- the waves' results meet: a wave leaves its rows' maxima, sums and outputs (in its own part of
    // the stages, which no other wave reads before), then wave db joins dims 16 db .. 16 db + 15
    const auto piece = [&](int w, int i) {
        const int r = i / PPT;   // K of stage 0, V of stage 0, K of stage 1 ..
        return reinterpret_cast<f32x4_t*>(lds.stages + r / 2 * Keys::SE + r % 2 * Keys::KV + w * TK * D) + i % PPT * 64 + lane;
    };
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const float l = sum_xor32(sum_xor16(l_run[cb]));
        if (q4 == 0) mls[wave][16 * cb + c16] = make_float2(m_run[cb], l);
#pragma unroll
        for (int db = 0; db < DB; ++db) *piece(wave, cb * DB + db) = acc[cb][db];
    }
    if (noted)
#pragma unroll 1
        for (int i = 0; i < CB * DB; ++i) *piece(wave, i) = with_infs(*piece(wave, i), infs[wave][i][lane]);
    __syncthreads();
    const size_t prow0 = ((size_t)g.part_base + (size_t)ic.cluster * n_rt + ic.rt) * (16 * CB);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row_lo + 16 * cb + c16, db = wave;
        if (row >= rows_total || db >= DB) continue;
        float2 w[NW];
        f32x4_t part[NW];
        float M = kNegBig, den = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            w[i] = mls[i][16 * cb + c16];
            part[i] = *piece(i, cb * DB + db);
            M = fmaxf(M, w[i].x);
        }
        f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float f = __builtin_amdgcn_exp2f(w[i].x - M);
            den += w[i].y * f;
            x += part[i] * f;
        }
        if (g.n_split > 1) {
            *reinterpret_cast<f32x4_t*>(a.part_o + (prow0 + 16 * cb + c16) * D + db * 16 + 4 * q4) = x;
            if (wave == 0 && q4 == 0) *reinterpret_cast<float2*>(a.part_ml + (prow0 + 16 * cb + c16) * 2) = make_float2(M, den);
        } else {
            const float inv = den == 0.f ? 0.f : 1.f / den;   // (a drafted token may see nothing: its output is 0)
            const int hl = row - toff[cb] * G;
            uint16_t* op = static_cast<uint16_t*>(a.o) + ((size_t)(g.q_row0 + toff[cb]) * a.hq + (size_t)ic.kvh * G + hl) * D;
            *reinterpret_cast<u32x2_t*>(op + db * 16 + 4 * q4) = u32x2_t{pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
        }
    }
}

// ---------------------------------------------------------------------------------
// tree_many: 32 WR rows, WR row groups of KG = 8 / WR waves, which take 32 keys of a step at a
// time (every KG-th).
//   S^T (32 keys x 32 rows) = K Q^T       v_mfma_f32_32x32x16_f16 (bf16 without rotation)
//   O^T (32 dims x 32 rows) += V^T P^T    v_mfma_f32_32x32x16_bf16, V^T by
//                                          ds_read_b64_tr_b16
// After the scores lane l holds row l%32 and keys 8 (j/4) + 4 (l/32) + j%4, the B operand of
// the output product.  A wave turns its
// keys of the next step beside the products of the scores.
// Bound by products and vector work that hardly overlap, although a SIMD has two waves: matrix cores
// busy 35% of the cycles and the vector unit 42% (keys turned already: 49% and 27%), 77% in all; a
// wave waits for data or the others a third of its time, and for its turn 22% (30%).  The clock is
// 1.75 to 2.0 GHz.  32 requests of 64 tokens of 32 heads over 8,192 keys 376 to 440 us by the card, 625
// to 730 TFLOP/s; keys turned already 302 to 358.  Half a step between the two waves of a SIMD, so
// that one's products run beside the other's softmax, changed nothing (387 against 388 us).
// ---------------------------------------------------------------------------------
template <int D, int STYLE, bool ROPE, int WR, int NG>
__global__ void __launch_bounds__(kTreeWaves * 64, 2) tree_many(const PlanOf<NG> plan, const TreeArgs a) {
    typedef TreeKeys<D, STYLE, ROPE, true> Keys;
    constexpr int KD = D / 16;             // 32x32x16 contraction steps of QK^T
    constexpr int DB = D / 32;             // 32-dim blocks of O^T
    constexpr int NW = kTreeWaves, KG = NW / WR, NST = Keys::NST, PL = Keys::PL, HALF = D / 2, SPARE = 2;
    constexpr int PER = SPARE * Keys::SE / NW;     // elements of the stages filled last, per wave
    static_assert(KG == 1 || KG == 2, "a step has two times 32 keys");
    static_assert(NST * Keys::SE * 2 >= NW * DB * 4 * 64 * 16, "the outputs meet in the stages");
    static_assert(PER * 2 >= 16 * HALF * 8, "the queries' angles pass through the stages");

    __shared__ TreeLds<D, true> lds;
    __shared__ float2 mls[NW][32];
    __shared__ uint8_t infs[NW][DB * 4][64];   // infinities of V that a lane's row sees (Keys::infs_of), if `noted`

    const Group g = group_of<false>(plan, blockIdx.x);
    const int G = a.group, n_rt = g.n_rt;
    const int li = blockIdx.x - g.item_base;   // (a call's items are not padded: below the group's count)
    const ItemCoords ic = item_coords(g, a.hkv, n_rt, li);
    Keys keys(lds, a, g, ic);
    const int lane = keys.lane, wave = keys.wave, nt = keys.nt;
    const int rg = wave / KG, kg = wave % KG, l32 = lane & 31, hi = lane >> 5;
    const int rows_total = g.n_tok * G, row_lo = (ic.rt * WR + rg) * 32;
#pragma unroll
    for (int u = 0; u < NST - SPARE; ++u)
        if (u < nt) keys.issue(u, u, keys.blocks_of(u));
    keys.fill_steps(a);

    // ---- queries.  The cos/sin of their tokens (a token's heads share them) go through the wave's
    // part of the stages filled last, which holds 16 tokens: more take two times 16 rows.
    const int row = row_lo + l32;
    const bool valid = row < rows_total;
    const int toff = valid ? row / G : 0, hl = valid ? row - toff * G : 0;
    bf16x8_t qb[KD];
    float qs = a.scale_log2;   // the products times this are scores (log2 units)
    __syncthreads();  // phase steps staged
    {
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((size_t)(g.q_row0 + toff) * a.hq + (size_t)ic.kvh * G + hl) * D;
        u32x4_t raw[KD];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) {
            raw[kd] = *reinterpret_cast<const u32x4_t*>(qp + model_chunk(a.chunk_map, 2 * kd + hi) * 8);
            if (!valid) raw[kd] = u32x4_t{0, 0, 0, 0};
        }
        if (ROPE) {
            float2* cs = reinterpret_cast<float2*>(lds.stages + (NST - SPARE) * Keys::SE + wave * PER);
            float xf[KD][8], big = 0.f;
#pragma unroll
            for (int kd = 0; kd < KD; ++kd)
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    xf[kd][2 * m] = bf_lo(raw[kd][m]);
                    xf[kd][2 * m + 1] = bf_hi(raw[kd][m]);
                }
            const int each = min(row_lo + 31, rows_total - 1) / G - min(row_lo, rows_total - 1) / G < 16 ? 32 : 16;
#pragma unroll 1
            for (int h = 0; h < 32; h += each) {
                const int row0 = row_lo + h;
                const int t0 = min(row0, rows_total - 1) / G, t1 = min(row0 + each - 1, rows_total - 1) / G;
                token_angles<HALF>(a, g, lds.fstep, lane, t0, t1, cs);
                if (l32 >= h && l32 < h + each) big = turn_row<STYLE, KD>(xf, cs + (valid ? toff - t0 : 0) * HALF, hi, 2);
                __atomic_signal_fence(__ATOMIC_SEQ_CST);
            }
            const int ex = query_exponent(max_xor32(big));
            qs = back_scale(qs, ex);
#pragma unroll
            for (int kd = 0; kd < KD; ++kd)
#pragma unroll
                for (int m = 0; m < 4; ++m) raw[kd][m] = pack_f16(ldexpf(xf[kd][2 * m], -ex), ldexpf(xf[kd][2 * m + 1], -ex));
        }
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) qb[kd] = __builtin_bit_cast(bf16x8_t, raw[kd]);
    }
    barrier_keep_vmem();   // the angles have been read: the stages may be filled

    f32x16_t acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = f32x16_t{};
    float m_run = kNegBig, l_run = 0.f;
    bool noted = false;
    // per-lane byte offsets: the K operand's row among 32 keys, the V^T operand's among 8 (chunk c,
    // and the row 8 keys on, by xor)
    constexpr int kSw8 = D == 128 ? 1 : 4;
    uint32_t k_at = (uint32_t)(l32 * D + ((hi ^ dswz<D>(l32 & 15)) << 3)) * 2, v_at;
    {
        const int key = 4 * hi + ((lane & 15) >> 2), d = ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
        v_at = (uint32_t)(Keys::KV + key * D + (((d >> 3) ^ dswz<D>(key)) << 3) + (d & 7)) * 2;
    }

    // step u has landed; this wave's keys of it are turned, but for the turning itself
    auto landed = [&](int u, int sl) {
        if (u >= nt) return;
        keys.template wait_step<NST - 2>(u);
        keys.clean(u, sl);
        if (ROPE) keys.find_angles(sl);
    };
    typename Keys::Blocks blk{};
    constexpr int NT = 2 / KG;   // times 32 keys of a step
    constexpr int TAKEN = KD * NT;
    // ---- step s in stage st, and the turning of the next
    auto step = [&](int s, int st) {
        const int sl = keys.next(st);
        // (the offsets are not kept apart for every chunk: registers are short)
        asm volatile("" : "+v"(k_at), "+v"(v_at));
        const uint32_t at = keys.stages_at + (uint32_t)(st * Keys::SE + 32 * kg * D) * 2, kt = at + k_at, vt = at + v_at;
        constexpr int kAhead = 4;                 // K reads in flight
        u32x4_t kf[TAKEN];
        auto read_k = [&](int i) { kf[i] = *(lds_u32x4_t*)(uintptr_t)((kt ^ (32 * (i / NT))) + 64 * (i % NT) * D); };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read_k(i);
        const int32_t flag = ROPE ? lds.kbig[st][lane % NW] : 0;
        // step s + NST - 1 goes where step s - 1 was
        if (s + NST - 1 < nt) {
            keys.issue(s + NST - 1, keys.prev(st), blk);
            if (s + NST < nt) blk = keys.blocks_of(s + NST);
        }
        landed(s + 1, sl);
        // ---- scores, with the next step's keys turned beside (past the last step: of nothing, into a
        // stage that is not read again)
        // Every few vector instructions follow a product that they do not wait for, in the order written:
        // left alone, the compiler puts the products side by side, and the vector unit idles.
        f32x16_t sc[NT];
        uint32_t w[PL], turned[PL];
        float big = 0.f;
        if constexpr (ROPE) keys.load_runs(sl, w);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TAKEN; ++i) {
            const int kd = i / NT, n = i % NT;
            const f32x16_t from = kd == 0 ? f32x16_t{} : sc[n];
            if (ROPE)
                sc[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, kf[i]), __builtin_bit_cast(f16x8_t, qb[kd]), from, 0, 0, 0);
            else
                sc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[i]), qb[kd], from, 0, 0, 0);
            if (i + kAhead < TAKEN) read_k(i + kAhead);
            if constexpr (ROPE) {
                // PL parts: the angles of two pairs, then their turning
#pragma unroll
                for (int part = i * PL / TAKEN; part < (i + 1) * PL / TAKEN; ++part) {
                    if (part % 2 == 0) keys.advance_pairs(part);
                    else keys.template rotate_pairs<false>(part - 1, w, turned, 0, big);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (ROPE) {
            keys.fit(sl, w, turned, big);
            keys.store_runs(sl, turned);
        }
        if (ROPE && __builtin_amdgcn_ballot_w64(flag != 0) != 0) {   // some key of the step came in times a power of two
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[n][j] *= lds.ksc[st][32 * (kg + n) + 8 * (j >> 2) + 4 * hi + (j & 3)];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int p0 = 32 * (kg + n), k0 = s * Keys::STEP + p0;
            if (keys.masked(k0, Keys::TOGETHER)) {
                // the row's bits of the keys (the step's second 32 may all lie past the range)
                const uint32_t seen = keys.inside(k0, 32) & tree_bits(a.mask + (size_t)(g.q_row0 + toff) * a.words, a.words, k0 - keys.k_tok);
                const uint32_t mine = seen >> (4 * hi);
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (!((mine >> (8 * (j >> 2) + (j & 3))) & 1)) sc[n][j] = -INFINITY;
                if (keys.wave_flag(lds.vbad[st])) {
                    // which of this lane's outputs the seen infinities reach
#pragma unroll 1
                    for (int c = 0; c < DB * 4 && !noted; ++c) infs[wave][c][lane] = 0;
                    noted = true;
#pragma unroll 1
                    for (int k = 0; k < 32; ++k)
                        if ((seen >> k) & 1)
#pragma unroll 1
                            for (int c = 0; c < DB * 4; ++c) infs[wave][c][lane] |= (uint8_t)keys.infs_of(st, p0 + k, c, hi);
                }
            }
        }
        float mx = kNegBig;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 16; ++j) mx = fmaxf(mx, sc[n][j]);
        mx = max_xor32(mx) * qs;
        // the reference maximum only moves when some row's maximum grows by more than 8
        // (probabilities stay below 2^8), so most steps skip rescaling
        if (__builtin_amdgcn_ballot_w64(mx > m_run + 8.f) != 0) {
            const float m_new = fmaxf(m_run, mx);
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] *= alpha;
            m_run = m_new;
        }
        // ---- outputs, 16 keys at a time, with the next 16's probabilities and V reads beside
        constexpr int NH = 2 * NT;   // groups of keys
        u32x4_t pw[2];               // probabilities rounded to bf16; the row sum adds exactly those
        u32x2_t af[2][2 * DB];
        // part i of DB of the probabilities of keys 16 h .. 16 h + 15
        auto prob = [&](int h, int i) {
            constexpr int E = 8 / DB;
#pragma unroll
            for (int r = i * E; r < (i + 1) * E; r += 2) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[h / 2][8 * (h % 2) + r], qs, -m_run));
                const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[h / 2][8 * (h % 2) + r + 1], qs, -m_run));
                pw[h % 2][r / 2] = pack_bf16(x, y);
                l_run = sum2_bf16(pw[h % 2][r / 2], l_run);
            }
        };
        // V reads of block i
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
    // a wave without rows copies and turns its keys only
    auto turn_only = [&](int u, int sl) {
        landed(u, sl);
        if constexpr (ROPE) {
            uint32_t w[PL], turned[PL];
            keys.load_runs(sl, w);
            const float big = keys.turn(w, turned);
            keys.fit(sl, w, turned, big);
            keys.store_runs(sl, turned);
        }
    };
#pragma unroll
    for (int u = NST - SPARE; u < NST - 1; ++u)
        if (u < nt) keys.issue(u, u, keys.blocks_of(u));
    if (NST - 1 < nt) blk = keys.blocks_of(NST - 1);
    turn_only(0, 0);
    barrier_keep_vmem();
    auto steps = [&](auto rows) {
        int st = 0;
        for (int s = 0; s < nt; ++s) {
            if (decltype(rows)::value) {
                step(s, st);
            } else {
                if (s + NST - 1 < nt) {
                    keys.issue(s + NST - 1, keys.prev(st), blk);
                    if (s + NST < nt) blk = keys.blocks_of(s + NST);
                }
                turn_only(s + 1, keys.next(st));
            }
            barrier_keep_vmem();
            st = keys.next(st);
        }
    };
    if (row_lo < rows_total) steps(std::true_type{});
    else steps(std::false_type{});

    // ---- the results of a row group's waves meet: rows by their common maximum, outputs through
    // the stages
    float den = sum_xor32(l_run), M = m_run, mine = 1.f;
    if constexpr (KG > 1) {
        if (hi == 0) mls[wave][l32] = make_float2(m_run, den);
        __syncthreads();   // (every wave's copies have landed and been read)
        const float2 other = mls[wave ^ 1][l32];
        M = fmaxf(m_run, other.x);
        mine = __builtin_amdgcn_exp2f(m_run - M);
        den = den * mine + other.y * __builtin_amdgcn_exp2f(other.x - M);
    }
    f32x4_t* meet = reinterpret_cast<f32x4_t*>(lds.stages);
    f32x4_t out[DB * 4];   // dims 8 c + 4 (l/32) + {0..3}
#pragma unroll
    for (int c = 0; c < DB * 4; ++c) {
        const f32x4_t x = {acc[c / 4][4 * (c % 4)], acc[c / 4][4 * (c % 4) + 1], acc[c / 4][4 * (c % 4) + 2], acc[c / 4][4 * (c % 4) + 3]};
        out[c] = x * mine;
    }
    if (noted)
#pragma unroll
        for (int c = 0; c < DB * 4; ++c) out[c] = with_infs(out[c], infs[wave][c][lane]);
    if (KG > 1)
#pragma unroll
        for (int c = 0; c < DB * 4; ++c) meet[(wave * DB * 4 + c) * 64 + lane] = out[c];
    if (KG > 1) __syncthreads();
    if (row >= rows_total) return;
    const size_t prow = ((size_t)g.part_base + (size_t)ic.cluster * n_rt + ic.rt) * (32 * WR) + rg * 32 + l32;
    const float inv = den == 0.f ? 0.f : 1.f / den;   // (a drafted token may see nothing: its output is 0)
    uint16_t* op = static_cast<uint16_t*>(a.o) + ((size_t)(g.q_row0 + toff) * a.hq + (size_t)ic.kvh * G + hl) * D;
#pragma unroll
    for (int c = 0; c < DB * 4; ++c) {
        if (KG > 1 && c % 2 != kg) continue;
        f32x4_t x = out[c];
        if (KG > 1) x += meet[((wave ^ 1) * DB * 4 + c) * 64 + lane];
        const int d = 8 * c + 4 * hi;
        if (g.n_split > 1) *reinterpret_cast<f32x4_t*>(a.part_o + prow * D + d) = x;
        else *reinterpret_cast<u32x2_t*>(op + d) = u32x2_t{pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
    }
    if (g.n_split > 1 && kg == 0 && hi == 0) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(M, den);
}

// Joins key splits: one block per kMergeRows rows of a (row tile, KV head),
// one float4 of a row per thread, U splits' loads in flight: 8 for row tiles of 16 or 32, of which
// small calls have many splits, 4 for larger ones, many of 2 splits, for which the repeats of the
// last count (U = 8 and 4: 8 tokens over 1,537 keys, 13 splits, 12.9 and 13.8 us, 1 over 20,000 20.2
// and 21.9; 16 trees of 96 tokens of 64 heads, 2 splits, 593 and 584, 16 ragged trees 61.6 and 60.3).
template <int D, int NG, int U>
__global__ void __launch_bounds__(kMergeRows * D / 4) tree_merge(const PlanOf<NG> plan, const TreeMergeArgs a) {
    constexpr int TPR = D / 4;
    const Group g = group_of<true>(plan, blockIdx.x);
    const int n_rt = g.n_rt, chunks = a.tile_rows / kMergeRows;
    int li = blockIdx.x - g.merge_base;   // (only groups with splits have blocks here, and no more than they need)
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

template <int D, int STYLE, bool ROPE, int NG>
hipError_t launch_tree_n(const PlanOf<NG>& plan, const TreeArgs& a, hipStream_t st) {
    const dim3 grid(plan.n_items), block(kTreeWaves * 64);
    switch (a.tile_rows) {
    case 16: hipLaunchKernelGGL((tree_few<D, STYLE, ROPE, 1, NG>), grid, block, 0, st, plan, a); break;
    case 32: hipLaunchKernelGGL((tree_few<D, STYLE, ROPE, 2, NG>), grid, block, 0, st, plan, a); break;
    case 128: hipLaunchKernelGGL((tree_many<D, STYLE, ROPE, 4, NG>), grid, block, 0, st, plan, a); break;
    default: hipLaunchKernelGGL((tree_many<D, STYLE, ROPE, 8, NG>), grid, block, 0, st, plan, a); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.n_merge == 0) return e;
    const TreeMergeArgs m = {a.part_o, a.part_ml, a.o, a.tile_rows, a.hq, a.hkv, a.group};
    const dim3 merges(plan.n_merge), threads(kMergeRows * D / 4);
    if (a.tile_rows <= 32) hipLaunchKernelGGL((tree_merge<D, NG, 8>), merges, threads, 0, st, plan, m);
    else hipLaunchKernelGGL((tree_merge<D, NG, 4>), merges, threads, 0, st, plan, m);
    return hipGetLastError();
}

template <int D, int STYLE, bool ROPE>
hipError_t launch_tree_t(const Plan& plan, const TreeArgs& a, hipStream_t st) {
    if (plan.n_groups > kFewGroups) return launch_tree_n<D, STYLE, ROPE, kMaxGroups>(plan, a, st);
    PlanOf<kFewGroups> few = {plan.n_groups, plan.n_items, plan.n_merge, plan.merge_ways, plan.table, plan.item_map, plan.merge_map, {}};
    for (int i = 0; i < plan.n_groups; ++i) few.g[i] = plan.g[i];
    return launch_tree_n<D, STYLE, ROPE, kFewGroups>(few, a, st);
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
