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

// cos/sin for bf16 entries: the hardware's sine of a fraction of a revolution (its error, about
// 2^-20, is far below the rounding to 8 bits)
__device__ __forceinline__ void rope_cs_fast(int32_t pos, uint64_t step, float& c, float& s) {
    const uint64_t ph = (uint64_t)(int64_t)pos * step;
    const float r = (float)(int32_t)(ph >> 32) * 0x1p-32f;
    c = __builtin_amdgcn_cosf(r);
    s = __builtin_amdgcn_sinf(r);
}

// ---------------------------------------------------------------------------------
// tree_bf16
//
// Workgroup: up to 16 CB query rows (drafted token x query head of one KV head's group) over
// one key range.  Its four waves hold the same rows and take every fourth 16-key tile (one
// cache block) of the range each, so that a wave reads, turns and multiplies its keys
// without waiting for another; their results meet in LDS at the end.
// Every read of the key loop goes straight to LDS, NST - 1 tiles ahead: K as stored, V, the
// cos/sin rows of the tile's keys, and the positions of a later tile.  The wave turns its K
// operand in registers and uses it for the CB column blocks:
//   S^T (16 keys x 16 rows) = K Q^T       v_mfma_f32_16x16x32_bf16
//   O^T (16 dims x 16 rows) += V^T P^T    v_mfma_f32_16x16x16_bf16, V^T by ds_read_b64_tr_b16
// After the scores lane l holds row l%16 of each block and keys 4 (l/16) + {0..3}, the B
// operand of the output product.
// ---------------------------------------------------------------------------------
template <int D, bool ROPE>
constexpr int tree_stages() { return ROPE ? 3 : 4; }

template <int D, int STYLE, bool ROPE, bool TABLE, int CB>
__global__ void __launch_bounds__(kTreeWaves * 64, D == 64 ? 2 : 1) tree_bf16(const Plan plan, const TreeArgs a) {
    constexpr int KD = D / 32;             // 16x16x32 contraction steps of QK^T
    constexpr int DB = D / 16;             // 16-dim blocks of O^T
    constexpr int CH = D / 8;              // 16-byte chunks per K/V row
    constexpr int HALF = D / 2;
    constexpr int TK = kBlock;
    constexpr int NW = kTreeWaves;
    constexpr int NST = tree_stages<D, ROPE>();
    constexpr int DPL = TK * CH / 64;      // 16-byte copies per lane per tile, each of K and V
    constexpr int TROW = HALF / 4;         // 16-byte chunks (4 entries) per cos/sin row
    constexpr int TPL = TK * TROW / 64;    // chunks of the tile's cos/sin rows per lane
    constexpr int LPS = 2 * DPL + (TABLE ? TPL : 0);   // copies per lane per tile
    constexpr int KV = TK * D;             // elements of a K or V tile
    constexpr int SE = 2 * KV + (ROPE ? TK * HALF * 2 : 0);   // 2-byte elements of a stage
    static_assert((NST - 2) * LPS < 64, "vmcnt range");
    static_assert(NW * NST * SE * 2 >= NW * CB * DB * 64 * 16, "the outputs meet in the stages");

    __shared__ __attribute__((aligned(16))) uint16_t stages[NW * NST * SE];
    __shared__ int32_t ps[NW][NST][TK];
    __shared__ float2 mls[NW][16 * CB];
    __shared__ __attribute__((aligned(4))) uint8_t infs[NW][CB][DB][64];   // infinities of V that a lane's rows see: +, 4 dims, and -, 4 dims
    __shared__ uint64_t fstep[HALF];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, q4 = lane >> 4;
    const Group g = group_of<false>(plan, blockIdx.x);
    const int G = a.group, n_rt = g.n_rt;
    const int li = blockIdx.x - g.item_base;
    if (li >= a.hkv * g.n_split * n_rt) return;
    const ItemCoords ic = item_coords(g, a.hkv, n_rt, li);
    const int rows_total = g.n_tok * G, row_lo = ic.rt * 16 * CB;
    const int kv_lo = g.win + ic.split * g.split_keys, end = g.tok0 + g.n_tok;
    // (no sum below passes the last key: a request may have 2^31 - 1 of them)
    const int kv_hi = g.split_keys < end - kv_lo ? kv_lo + g.split_keys : end;
    const int kt0 = kv_lo & ~(TK - 1);
    const int n_tiles = (kv_hi - 1 - kt0) / TK + 1;
    const int nt = n_tiles > wave ? (n_tiles - wave - 1) / NW + 1 : 0;   // this wave's
    auto tile_key = [&](int u) { return kt0 + (u * NW + wave) * TK; };

    if (ROPE)
        for (int i = tid; i < HALF; i += NW * 64) fstep[i] = a.fstep[i];
    for (int i = tid; i < NW * CB * DB * 16; i += NW * 64) reinterpret_cast<uint32_t*>(infs)[i] = 0;

    const int32_t* btab = a.block_tables + (size_t)g.req * a.max_blocks;
    const size_t blk_stride = (size_t)a.hkv * kBlock * D;
    const uint16_t* kpool = static_cast<const uint16_t*>(a.k_pool) + (size_t)ic.kvh * kBlock * D;
    const uint16_t* vpool = static_cast<const uint16_t*>(a.v_pool) + (size_t)ic.kvh * kBlock * D;
    uint16_t* my = stages + wave * NST * SE;

    // a key outside [kv_lo, kv_hi) stands for the tile's first key inside, so that nothing
    // outside the range is read (its score is masked)
    auto clamp_key = [&](int kt, int j) { return (j >= kv_lo && j < kv_hi) ? j : max(kt, kv_lo); };
    auto copy_positions = [&](int u, int slot) {
        if (!ROPE || u >= nt) return;
        const int kt = tile_key(u);
        if (lane < TK) dma_lds4(a.positions + g.pos_off + clamp_key(kt, kt + lane), &ps[wave][slot][0]);
    };
    // this lane's copies of a tile: byte offset within one head's page of a block
    uint32_t lane_off[DPL];
#pragma unroll
    for (int i = 0; i < DPL; ++i) {
        const int kk = (i * 64 + lane) / CH, pc = (i * 64 + lane) % CH;
        lane_off[i] = (uint32_t)(kk * D + ((pc ^ dswz<D>(kk)) << 3)) * 2;
    }
    int odd_tile = -1;   // last tile with fewer than LPS copies
    auto issue = [&](int u, int st, int blk) {
        uint16_t* sg = my + st * SE;
        const int kt = tile_key(u);
        __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));   // the stage's last reads have returned (lgkmcnt 0)
        copy_positions(u + NST - 1, st == 0 ? NST - 1 : st - 1);
        if (ROPE) {
            uint32_t* tab = reinterpret_cast<uint32_t*>(sg + 2 * KV);
#pragma unroll
            for (int i = 0; i < TPL; ++i) {
                const int c = i * 64 + lane;
                const int tkey = c / TROW, lc = (c % TROW) ^ (tkey & (TROW - 1));
                const int32_t pos = ps[wave][st][tkey];
                const bool in_table = TABLE && (uint32_t)pos < (uint32_t)a.rope_len;
                if (in_table)
                    dma_lds16(reinterpret_cast<const uint32_t*>(a.rope_table) + (size_t)pos * HALF + 4 * lc, tab + i * 64 * 4);
                if (!TABLE || __builtin_amdgcn_ballot_w64(!in_table) != 0) {
                    if (TABLE) odd_tile = u;
                    if (!in_table) {
                        u32x4_t w;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float ce, se;
                            rope_cs_fast(pos, fstep[4 * lc + e], ce, se);
                            w[e] = bf16_entry(ce, se);
                        }
                        *reinterpret_cast<u32x4_t*>(tab + c * 4) = w;
                    }
                }
            }
        }
        const uint16_t* kb = kpool + (size_t)(uint32_t)blk * blk_stride;
        const uint16_t* vb = vpool + (size_t)(uint32_t)blk * blk_stride;
        const bool whole = kt >= kv_lo && kv_hi - kt >= TK;
#pragma unroll
        for (int i = 0; i < DPL; ++i) {
            uint32_t off = lane_off[i];
            if (!whole) {
                const int kk = (i * 64 + lane) / CH;
                off += (clamp_key(kt, kt + kk) - kt - kk) * D * 2;
            }
            dma_lds16_s(kb, off, sg + i * 64 * 8);
            dma_lds16_s(vb, off, sg + KV + i * 64 * 8);
        }
    };

#pragma unroll
    for (int u = 0; u < NST - 1; ++u) copy_positions(u, u);

    // ---- queries: rows 16 cb .. 16 cb + 15 are turned and scaled by wave cb and passed to the
    // others through the stage that is filled last
    int toff[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row_lo + 16 * cb + c16;
        toff[cb] = row < rows_total ? row / G : 0;
    }
    bf16x8_t qb[CB][KD];
    __syncthreads();   // phase steps staged
    if (wave < CB) {
        const int row = row_lo + 16 * wave + c16;
        const bool valid = row < rows_total;
        const int to = valid ? row / G : 0, hl = valid ? row - to * G : 0;
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((size_t)(g.q_row0 + to) * a.hq + (size_t)ic.kvh * G + hl) * D;
        float xf[KD][8];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) {
            const u32x4_t raw = *reinterpret_cast<const u32x4_t*>(qp + model_chunk(a.chunk_map, kd * 4 + q4) * 8);
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                xf[kd][2 * m] = valid ? bf_lo(raw[m]) : 0.f;
                xf[kd][2 * m + 1] = valid ? bf_hi(raw[m]) : 0.f;
            }
        }
        if (ROPE) {
            const int32_t pos = a.positions[g.pos_off + g.tok0 + to];
#pragma unroll
            for (int kd = 0; kd < KD; ++kd) {
                if (STYLE == kNeox) {
                    if (kd >= KD / 2) break;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float c, s;
                        rope_cs_fast(pos, fstep[kd * 32 + 8 * q4 + e], c, s);
                        const float x = xf[kd][e], y = xf[kd + KD / 2][e];
                        xf[kd][e] = x * c - y * s;
                        xf[kd + KD / 2][e] = y * c + x * s;
                    }
                } else {
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        float c, s;
                        rope_cs_fast(pos, fstep[kd * 16 + 4 * q4 + m], c, s);
                        const float x = xf[kd][2 * m], y = xf[kd][2 * m + 1];
                        xf[kd][2 * m] = x * c - y * s;
                        xf[kd][2 * m + 1] = y * c + x * s;
                    }
                }
            }
        }
        u32x4_t* out = reinterpret_cast<u32x4_t*>(my + (NST - 1) * SE);
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) {
            u32x4_t w;
#pragma unroll
            for (int m = 0; m < 4; ++m) w[m] = pack_bf16(xf[kd][2 * m] * a.scale_log2, xf[kd][2 * m + 1] * a.scale_log2);
            out[kd * 64 + lane] = w;
        }
    }
    wait_vmem();       // the first positions have landed
    __syncthreads();
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int kd = 0; kd < KD; ++kd)
            qb[cb][kd] = *reinterpret_cast<const bf16x8_t*>(stages + (cb * NST + NST - 1) * SE + (kd * 64 + lane) * 8);
    __syncthreads();   // every wave has its rows: the stages may be filled

    f32x4_t acc[CB][DB];
    float m_run[CB], l_run[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        m_run[cb] = kNegBig;
        l_run[cb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[cb][db] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    // per-lane element offsets within a stage: K operand rows, cos/sin chunks, V^T operand rows
    int k_off[KD], t_off[KD], v_off[DB];
#pragma unroll
    for (int kd = 0; kd < KD; ++kd) {
        k_off[kd] = c16 * D + ((model_chunk(a.chunk_map, kd * 4 + q4) ^ dswz<D>(c16)) << 3);
        // NeoX: 2 chunks for each of the KD / 2 steps of a half; GPT-J: 1 for each step
        const int lc = STYLE == kNeox ? (kd / 2) * 8 + 2 * q4 + (kd % 2) : kd * 4 + q4;
        t_off[kd] = 2 * KV + (c16 * HALF + 4 * (lc ^ (c16 & (TROW - 1)))) * 2;
    }
    {
        const int key = 4 * q4 + (c16 >> 2);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const int d = db * 16 + 4 * (lane & 3);
            v_off[db] = KV + key * D + (((d >> 3) ^ dswz<D>(key)) << 3) + (d & 7);
        }
    }

    int blk_next = 0;
    auto block_of = [&](int u) { return scalar_load(btab, min(tile_key(u), kv_hi - 1) >> 4); };
#pragma unroll
    for (int u = 0; u < NST - 1; ++u)
        if (u < nt) issue(u, u, block_of(u));
    if (NST - 1 < nt) blk_next = block_of(NST - 1);
    int st = 0;
    for (int t = 0; t < nt; ++t) {
        // tile t has landed once no more than the later tiles' copies are outstanding
        if (t + NST - 2 < nt && odd_tile <= t) wait_vmem_n<(NST - 2) * LPS>();
        else wait_vmem();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        const uint16_t* sg = my + st * SE;
        const int kt = tile_key(t);
        if (t + NST - 1 < nt) {
            issue(t + NST - 1, st == 0 ? NST - 1 : st - 1, blk_next);
            if (t + NST < nt) blk_next = block_of(t + NST);
        }
        u32x4_t kf[KD];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) kf[kd] = *reinterpret_cast<const u32x4_t*>(sg + k_off[kd]);
        if (ROPE) {
            u32x4_t te[KD];
#pragma unroll
            for (int kd = 0; kd < KD; ++kd) te[kd] = *reinterpret_cast<const u32x4_t*>(sg + t_off[kd]);
            if (STYLE == kNeox) {
#pragma unroll
                for (int kd = 0; kd < KD / 2; ++kd)
#pragma unroll
                    for (int m = 0; m < 4; m += 2) {
                        const u32x4_t ee = te[2 * kd + m / 2];
                        const Words4 o = rot4_neox(kf[kd][m], kf[kd + KD / 2][m], kf[kd][m + 1], kf[kd + KD / 2][m + 1],
                                                   ee[0], ee[1], ee[2], ee[3]);
                        kf[kd][m] = o.w[0];
                        kf[kd + KD / 2][m] = o.w[1];
                        kf[kd][m + 1] = o.w[2];
                        kf[kd + KD / 2][m + 1] = o.w[3];
                    }
            } else {
#pragma unroll
                for (int kd = 0; kd < KD; ++kd) {
                    const u32x4_t ee = te[kd];
                    const Words4 o = rot4_gptj(kf[kd][0], kf[kd][1], kf[kd][2], kf[kd][3], ee[0], ee[1], ee[2], ee[3]);
#pragma unroll
                    for (int m = 0; m < 4; ++m) kf[kd][m] = o.w[m];
                }
            }
        }
        f32x4_t sc[CB];
#pragma unroll
        for (int kd = 0; kd < KD; ++kd)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                sc[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[kd]), qb[cb][kd],
                                                                 kd == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sc[cb], 0, 0, 0);
        const bool masked = kt < kv_lo || kv_hi - kt < TK || g.tok0 - kt < TK;
        uint32_t seen[CB];   // masked tiles: the row's bits of the tile's keys
        if (masked) {
            // keys [kv_lo, kv_hi) of the tile
            const int lo = max(kv_lo - kt, 0), hi = min(kv_hi - kt, TK);
            const uint32_t inside = ((1u << hi) - 1u) & ~((1u << lo) - 1u);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                seen[cb] = inside & tree_bits(a.mask + (size_t)(g.q_row0 + toff[cb]) * a.words, a.words, kt - g.tok0);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (!((seen[cb] >> (4 * q4 + r)) & 1)) sc[cb][r] = -INFINITY;
            }
        }
        float mx[CB];
        bool moves = false;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
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
                for (int db = 0; db < DB; ++db) acc[cb][db] *= alpha;
                m_run[cb] = m_new;
            }
        }
        // probabilities rounded to bf16 for P V; the row sum adds exactly those
        u32x2_t pw[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(sc[cb][r] - m_run[cb]);
            pw[cb] = u32x2_t{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3])};
            l_run[cb] = sum2_bf16(pw[cb][1], sum2_bf16(pw[cb][0], l_run[cb]));
        }
        lds_u16_t* vb = as_lds(sg);
        bf16x4_t af[DB];
        uint32_t huge = 0;   // masked tiles: whether V holds an infinity or NaN
#pragma unroll
        for (int db = 0; db < DB; ++db) af[db] = __builtin_bit_cast(bf16x4_t, lds_read_tr(vb + v_off[db]));
        if (masked) {
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const u32x2_t w = __builtin_bit_cast(u32x2_t, af[db]);
#pragma unroll
                for (int e = 0; e < 2; ++e) huge |= (uint32_t)((w[e] & 0x7f80u) == 0x7f80u) | (uint32_t)((w[e] & 0x7f800000u) == 0x7f800000u);
            }
        }
        if (masked && __builtin_amdgcn_ballot_w64(huge != 0) != 0) {
            // An infinity or NaN in V must not reach rows that do not see its key (0 x Inf in
            // the product below): the product takes the finite elements, and two more count
            // the seen infinities of either sign (a NaN as one of each) per row and dimension,
            // which join the outputs at the end.
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const u32x2_t w = __builtin_bit_cast(u32x2_t, af[db]);
                u32x2_t fin, up, down;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    fin[e] = up[e] = down[e] = 0;
#pragma unroll
                    for (int h = 0; h < 32; h += 16) {
                        const uint32_t x = (w[e] >> h) & 0xffffu, mag = x & 0x7fffu;
                        if (mag < 0x7f80u) fin[e] |= x << h;
                        else {
                            if (x != 0xff80u) up[e] |= 0x3f80u << h;
                            if (x != 0x7f80u) down[e] |= 0x3f80u << h;
                        }
                    }
                }
                af[db] = __builtin_bit_cast(bf16x4_t, fin);
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    const uint32_t k4 = seen[cb] >> (4 * q4);
                    const u32x2_t one = {(k4 & 1u) * 0x3f80u | ((k4 >> 1) & 1u) * 0x3f800000u,
                                         ((k4 >> 2) & 1u) * 0x3f80u | ((k4 >> 3) & 1u) * 0x3f800000u};
                    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
                    const f32x4_t u = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(bf16x4_t, up), __builtin_bit_cast(bf16x4_t, one), zero, 0, 0, 0);
                    const f32x4_t d = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(bf16x4_t, down), __builtin_bit_cast(bf16x4_t, one), zero, 0, 0, 0);
                    uint32_t f = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) f |= (u[i] > 0.f ? 1u << i : 0u) | (d[i] > 0.f ? 16u << i : 0u);
                    infs[wave][cb][db][lane] |= (uint8_t)f;
                }
            }
        }
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                acc[cb][db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(af[db], __builtin_bit_cast(bf16x4_t, pw[cb]), acc[cb][db], 0, 0, 0);
        st = st + 1 == NST ? 0 : st + 1;
    }

    // ---- the waves' results meet: rows by their common maximum, outputs through the stages
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const float l = sum_xor32(sum_xor16(l_run[cb]));
        if (q4 == 0) mls[wave][16 * cb + c16] = make_float2(m_run[cb], l);
    }
    __syncthreads();   // (every wave's copies have landed and been read)
    float M[CB], den[CB];
    f32x4_t* meet = reinterpret_cast<f32x4_t*>(stages);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        float2 w[NW];
        M[cb] = kNegBig;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            w[i] = mls[i][16 * cb + c16];
            M[cb] = fmaxf(M[cb], w[i].x);
        }
        den[cb] = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) den[cb] += w[i].y * __builtin_amdgcn_exp2f(w[i].x - M[cb]);
        const float mine = __builtin_amdgcn_exp2f(m_run[cb] - M[cb]);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            f32x4_t x = acc[cb][db] * mine;
            const uint32_t f = infs[wave][cb][db][lane];
            if (f != 0)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] += ((f >> i) & 1 ? INFINITY : 0.f) - ((f >> (4 + i)) & 1 ? INFINITY : 0.f);
            meet[((wave * CB + cb) * DB + db) * 64 + lane] = x;
        }
    }
    __syncthreads();
    const size_t prow0 = ((size_t)g.part_base + (size_t)ic.cluster * n_rt + ic.rt) * (16 * CB);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row_lo + 16 * cb + c16;
        if (row >= rows_total) continue;
        const float inv = den[cb] == 0.f ? 0.f : 1.f / den[cb];   // (a drafted token may see nothing: its output is 0)
#pragma unroll
        for (int i = 0; i < DB / NW; ++i) {
            const int db = i * NW + wave;
            f32x4_t x = meet[(cb * DB + db) * 64 + lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) x += meet[((w * CB + cb) * DB + db) * 64 + lane];
            if (g.n_split > 1) {
                *reinterpret_cast<f32x4_t*>(a.part_o + (prow0 + 16 * cb + c16) * D + db * 16 + 4 * q4) = x;
            } else {
                const int hl = row - toff[cb] * G;
                uint16_t* op = static_cast<uint16_t*>(a.o) + ((size_t)(g.q_row0 + toff[cb]) * a.hq + (size_t)ic.kvh * G + hl) * D;
                *reinterpret_cast<u32x2_t*>(op + db * 16 + 4 * q4) = u32x2_t{pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
            }
        }
        if (g.n_split > 1 && wave == 0 && q4 == 0)
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

template <int D, int STYLE, bool ROPE, bool TABLE>
hipError_t launch_tree_t(const Plan& plan, const TreeArgs& a, hipStream_t st) {
    const dim3 grid(plan.n_items), block(kTreeWaves * 64);
    if (a.tile_rows == 16) hipLaunchKernelGGL((tree_bf16<D, STYLE, ROPE, TABLE, 1>), grid, block, 0, st, plan, a);
    else if (a.tile_rows == 32) hipLaunchKernelGGL((tree_bf16<D, STYLE, ROPE, TABLE, 2>), grid, block, 0, st, plan, a);
    else hipLaunchKernelGGL((tree_bf16<D, STYLE, ROPE, TABLE, 4>), grid, block, 0, st, plan, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.n_merge == 0) return e;
    hipLaunchKernelGGL((tree_merge<D>), dim3(plan.n_merge), dim3(kMergeRows * D / 4), 0, st, plan, a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_tree_d(int style, bool rope, const Plan& plan, const TreeArgs& a, hipStream_t st) {
    const bool table = a.rope_table != nullptr && a.rope_len > 0;
    if (!rope) return launch_tree_t<D, 0, false, false>(plan, a, st);   // (without rotation the pairing makes no difference)
    if (style == kNeox) return table ? launch_tree_t<D, 0, true, true>(plan, a, st) : launch_tree_t<D, 0, true, false>(plan, a, st);
    return table ? launch_tree_t<D, 1, true, true>(plan, a, st) : launch_tree_t<D, 1, true, false>(plan, a, st);
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
