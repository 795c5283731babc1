// Attention on the tensor cores: bf16 heads of up to 128 (a multiple of 8), rows on the 16-byte grid.  This file: the parts that the
// three kernels share, and the forward pass.
//
// A tile is 128 tokens of one head in shared memory, as one or two blocks of 64 columns (TMA boxes with the 128-byte
// swizzle; columns from d on are filled with zeros).  The same tile is a K-major operand (rows against rows: scores) and an MN-major one
// (weights against rows: outputs and gradients), so nothing is ever transposed.
#pragma once
#include "attention.cuh"
#include "sm100_ptx.cuh"
#include "weight_grad_common.cuh"      // umma_desc_mn_sw128

namespace pamm {

constexpr int AU_ROWS = 128, AU_BLOCK_BYTES = AU_ROWS * 128;       // of a tile, and of 64 of its columns
constexpr int AU_TMA_WARP = 8, AU_MMA_WARP = 9;                    // behind eight warps that own rows
constexpr size_t AU_SMEM_LIMIT = 232448;

// The order of work.  Whole and padded batches: (batch, head) pairs in groups of about one per block, in a group the tiles of every pair
// from the last to the first -- the long ones first where causal -- so that a pair's keys are read again while they
// are in L2.  Packed sequences: by tile, all heads of a tile one after another.
struct AttentionOrder {
    int pairs, tiles, groups, per_group, owners;       // owners: heads of the rows that a tile owns
    bool packed, descending;
    __device__ __forceinline__ void at(int w, int& item, int& head) const {
        if (packed) {
            item = w / owners;
            head = w - item * owners;
            return;
        }
        const int full = per_group * tiles;
        int g = w / full;
        if (g > groups - 1) g = groups - 1;
        const int members = g == groups - 1 ? pairs - g * per_group : per_group;
        const int local = w - g * full, level = local / members, pair = g * per_group + (local - level * members);
        const int b = pair / owners;
        head = pair - b * owners;
        item = b * tiles + (descending ? tiles - 1 - level : level);
    }
};
inline AttentionOrder attention_order(const Sequences& s, int owners, int tile, int blocks, bool descending) {
    AttentionOrder o = {};
    o.owners = owners;
    o.packed = s.starts != nullptr;
    o.descending = descending;
    o.tiles = (int)((s.seq + tile - 1) / tile);
    o.pairs = s.batch * owners;
    o.groups = o.packed ? 1 : std::max(1, (int)(((int64_t)o.pairs + blocks / 2) / blocks));
    o.per_group = o.groups > 1 ? blocks : o.pairs;
    return o;
}

__device__ __forceinline__ float exp2_approx(float x) {       // 2 units, results below 2^-126 are 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// One tile into shared memory, counted on `bar` (AU_BLOCK_BYTES a block).
template <int DP>
__device__ __forceinline__ void au_load(uint8_t* dst, const CUtensorMap* tm, const Tile& t, int head, int at, uint64_t* bar) {
#pragma unroll
    for (int c = 0; c < DP / 64; ++c)
        ptx::tma_load_4d(dst + c * AU_BLOCK_BYTES, tm, c * 64, head, (int32_t)(t.first + at), (int32_t)t.b, bar);
}
// A wait of a whole warp: the same answer in every lane.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity, abort_flag));
}
// The producer's ring of tiles.  Called by the whole warp.
struct TileRing {
    uint8_t* tiles;
    uint64_t *full, *empty, *tail;       // tail: for a tile whose last rows are cleared before it is handed on
    volatile int* abort_flag;
    int slots, slot;
    uint32_t phase, tail_phase, used;
    bool tail_open;
    __device__ __forceinline__ void next() {
        if (++slot == slots) { slot = 0; phase ^= 1u; }
        ++used;
    }
};
// The next tile of the ring.  `clear`: rows from the sequence's end on are set to zero, because a product with a weight of 0 would keep
// their NaN or infinity; needed where the tensor goes on behind the end.
template <int DP>
__device__ __forceinline__ bool au_produce(TileRing& r, const CUtensorMap* tm, const Tile& t, int head, int at, bool clear) {
    if (!warp_wait(&r.empty[r.slot], r.phase ^ 1u, r.abort_flag)) return false;
    uint8_t* dst = r.tiles + (size_t)r.slot * (DP / 64) * AU_BLOCK_BYTES;
    const int valid = t.len - at;
    if (!clear || valid >= AU_ROWS) {
        if (ptx::elect_one()) {
            ptx::mbar_arrive_expect_tx(&r.full[r.slot], DP / 64 * AU_BLOCK_BYTES);
            au_load<DP>(dst, tm, t, head, at, &r.full[r.slot]);
        }
    } else {
        if (ptx::elect_one()) {
            ptx::mbar_arrive_expect_tx(r.tail, DP / 64 * AU_BLOCK_BYTES);
            au_load<DP>(dst, tm, t, head, at, r.tail);
        }
        r.tail_open = true;
        if (!warp_wait(r.tail, r.tail_phase, r.abort_flag)) return false;
        r.tail_open = false;
        r.tail_phase ^= 1u;
        for (int c = 0; c < DP / 64; ++c)
            for (int i = valid * 8 + (int)(threadIdx.x & 31); i < AU_ROWS * 8; i += 32)       // whole rows: the swizzle stays inside them
                *reinterpret_cast<uint4*>(dst + c * AU_BLOCK_BYTES + i * 16) = make_uint4(0, 0, 0, 0);
        ptx::fence_proxy_async();
        __syncwarp();
        if (ptx::elect_one()) ptx::mbar_arrive(&r.full[r.slot]);
    }
    __syncwarp();
    r.next();
    return true;
}
// After a wait ran out: the copies in flight land before the block's memory is given back.
__device__ __forceinline__ void au_drain(const TileRing& r) {
    int never = 0;
    if (r.tail_open) ptx::mbar_wait(r.tail, r.tail_phase, &never, 1u << 14);
    const uint32_t back = r.used < (uint32_t)r.slots ? r.used : (uint32_t)r.slots;
    for (uint32_t d = 1; d <= back; ++d) {
        const uint32_t it = r.used - d;
        ptx::mbar_wait(&r.full[it % r.slots], (it / r.slots) & 1u, &never, 1u << 14);
    }
}

// D (+)= A B^T over the heads' d columns, both tiles K-major: d = 16 steps.  One thread.
__device__ __forceinline__ void au_scores(uint32_t d_tmem, uint32_t a, uint32_t b, int steps, uint32_t idesc) {
    const uint64_t da = ptx::umma_desc_k_sw128(a), db = ptx::umma_desc_k_sw128(b);
    for (int k = 0; k < steps; ++k) {
        const uint64_t off = (uint64_t)((k >> 2) * (AU_BLOCK_BYTES >> 4) + (k & 3) * 2);
        ptx::umma_bf16(d_tmem, da + off, db + off, idesc, k > 0);
    }
}
// D (+)= W B over 128 rows of B: W bf16 in tensor memory, B MN-major.  One thread.
__device__ __forceinline__ void au_weighted(uint32_t d_tmem, uint32_t w_tmem, uint32_t b, uint32_t idesc, bool accumulate) {
#pragma unroll
    for (int k = 0; k < AU_ROWS / 16; ++k)
        ptx::umma_bf16_ts(d_tmem, w_tmem + 8 * k, umma_desc_mn_sw128(b + k * 2048, AU_BLOCK_BYTES, 1024), idesc, accumulate || k > 0);
}

struct AttentionMaps { CUtensorMap q, k, v, d_o; };
inline bool attention_map(CUtensorMap* tm, const HeadsView& t, const Sequences& s, int64_t heads, int d) {
    const auto ld = [](int64_t v) { return (uint64_t)(v > 0 ? v : 8); };      // of a dimension with one entry: any multiple of 16 bytes
    return make_tmap_heads_sw128(tm, t.p, (uint64_t)d, (uint64_t)heads, (uint64_t)s.seq, (uint64_t)s.batch, ld(t.head), ld(t.token), ld(t.batch), AU_ROWS);
}

// ---- forward ------------------------------------------------------------------------------------------------------------
// A block works on 256 rows of one query head at a time: two tiles, each with four warps whose threads own a row.  Per tile of 128
// keys: S = Q K^T into tensor memory; the row's thread takes its 128 scores, its maximum and exponentials and puts P back as bf16 over
// S; O += P V with P as the operand in tensor memory.  While one tile's warps are at their exponentials the tensor cores work for
// the other.  O stays in tensor memory; it is scaled down only where a row's maximum has risen by more than 2^8 since the
// reference that its exponentials are taken from (exact: l and O share the reference, and p <= 2^8 keeps its relative rounding).
// The rounding of P to bf16 is the operand's; its sum l is taken before it, in fp32.
constexpr int AF_THREADS = 384, AF_QUERIES = 2 * AU_ROWS;
// 168 registers a thread at the launch; a row's 128 scores and what goes with them take more, the other four warps (two of them idle)
// less: 256 x 208 + 128 x 88 = 384 x 168.
constexpr int AU_LAUNCH_REGS = 168, AU_ROW_REGS = 208, AU_OTHER_REGS = 88;
static_assert(256 * AU_ROW_REGS + 128 * AU_OTHER_REGS <= AF_THREADS * AU_LAUNCH_REGS, "what is taken has to have been given back");
constexpr float AF_RISE = 8.f;

template <int DP>
struct ForwardPlan {
    static constexpr int TILE_BYTES = DP / 64 * AU_BLOCK_BYTES;
    static constexpr int SLOTS = DP == 128 ? 5 : 8;
    static constexpr size_t SMEM = 1024 + (size_t)(2 + SLOTS) * TILE_BYTES;
};

// Tiles of keys that query tile x (0 or 1) of the item meets.
__device__ __forceinline__ int af_key_tiles(const Tile& t, bool causal, int x) {
    const int at = t.at + x * AU_ROWS;
    if (at >= t.len) return 0;
    const int end = causal ? min(t.len, at + AU_ROWS) : t.len;
    return (end + AU_ROWS - 1) / AU_ROWS;
}

template <int DP>
__global__ void __launch_bounds__(AF_THREADS, 1)
attention_forward_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionMaps m, const __grid_constant__ AttentionOrder order,
                         const int works) {
    using Plan = ForwardPlan<DP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t s_full[Plan::SLOTS], s_empty[Plan::SLOTS], s_qfull[2], s_qempty[2], s_scores[2], s_probs[2], s_done[2], s_tail;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* queries = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring_tiles = queries + 2 * Plan::TILE_BYTES;
    if (threadIdx.x == 0) {
        for (int i = 0; i < Plan::SLOTS; ++i) { ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&s_empty[i], 1); }
        for (int x = 0; x < 2; ++x) {
            ptx::mbar_init(&s_qfull[x], 1);
            ptx::mbar_init(&s_qempty[x], 1);
            ptx::mbar_init(&s_scores[x], 1);
            ptx::mbar_init(&s_probs[x], 4);
            ptx::mbar_init(&s_done[x], 1);
        }
        ptx::mbar_init(&s_tail, 1);
        s_abort = 0;
        ptx::fence_barrier_init();
        ptx::fence_proxy_async();
    }
    if (warp == AU_MMA_WARP) {
        ptx::tmem_alloc(&s_tmem, 512);
        ptx::tmem_relinquish();
    }
    grid_launch_dependents();
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = s_tmem;
    volatile int* abort_flag = &s_abort;
    grid_dependency_wait();
    bool ok = true;

    if (warp >= 8) {
      ptx::registers_down<AU_OTHER_REGS>();
      if (warp == AU_TMA_WARP) {
        TileRing ring = {ring_tiles, s_full, s_empty, &s_tail, abort_flag, Plan::SLOTS, 0, 0, 0, 0, false};
        uint32_t q_phase[2] = {0, 0};
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h;
            order.at(w, item, h);
            const Tile t = find_tile<AF_QUERIES>(a.s, item);
            if (!t.any) continue;
            const int n0 = af_key_tiles(t, a.causal, 0), n1 = af_key_tiles(t, a.causal, 1), n = max(n0, n1);
            const bool clear = t.first + t.len < a.s.seq;
            for (int x = 0; x < 2 && ok; ++x) {
                if ((x ? n1 : n0) == 0) continue;
                ok = warp_wait(&s_qempty[x], q_phase[x] ^ 1u, abort_flag);
                if (!ok) break;
                q_phase[x] ^= 1u;
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(&s_qfull[x], Plan::TILE_BYTES);
                    au_load<DP>(queries + x * Plan::TILE_BYTES, &m.q, t, h, t.at + x * AU_ROWS, &s_qfull[x]);
                }
                __syncwarp();
            }
            for (int j = 0; j < n && ok; ++j)
                ok = au_produce<DP>(ring, &m.k, t, h / a.group, j * AU_ROWS, false) && au_produce<DP>(ring, &m.v, t, h / a.group, j * AU_ROWS, clear);
        }
        if (!ok) {
            au_drain(ring);
            int never = 0;
            for (int x = 0; x < 2; ++x) ptx::mbar_wait(&s_qfull[x], q_phase[x] ^ 1u, &never, 1u << 14);
        }
      } else if (warp == AU_MMA_WARP) {
        const uint32_t idesc_s = ptx::umma_idesc_bf16(AU_ROWS, AU_ROWS);
        const uint32_t idesc_o = ptx::umma_idesc_bf16(AU_ROWS, (uint32_t)((a.d + 15) / 16 * 16)) | (1u << 16);      // B MN-major
        const int steps = (a.d + 15) / 16;
        const uint32_t q_addr = ptx::smem_u32(queries), ring_addr = ptx::smem_u32(ring_tiles);
        uint32_t q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
        uint32_t count = 0;                     // ring tiles of earlier items
        const auto slot_of = [&](uint32_t i) { return i % Plan::SLOTS; };
        const auto tile_ready = [&](uint32_t i) { return warp_wait(&s_full[slot_of(i)], (i / Plan::SLOTS) & 1u, abort_flag); };
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h;
            order.at(w, item, h);
            const Tile t = find_tile<AF_QUERIES>(a.s, item);
            if (!t.any) continue;
            const int n0 = af_key_tiles(t, a.causal, 0), n1 = af_key_tiles(t, a.causal, 1), n = max(n0, n1);
            // S of tile x and key tile j; the last use of key tile j frees its slot
            const auto scores = [&](int x, int j) {
                if (ptx::elect_one()) {
                    au_scores(tmem + x * 128, q_addr + x * Plan::TILE_BYTES, ring_addr + slot_of(count + 2 * j) * Plan::TILE_BYTES, steps, idesc_s);
                    ptx::umma_commit(&s_scores[x]);
                    if (j == (x ? n1 : n0) - 1) ptx::umma_commit(&s_qempty[x]);
                    if (x == 1 || j >= n1) ptx::umma_commit(&s_empty[slot_of(count + 2 * j)]);
                }
                __syncwarp();
            };
            for (int x = 0; x < 2 && ok; ++x) {
                if ((x ? n1 : n0) == 0) continue;
                ok = warp_wait(&s_qfull[x], q_phase[x], abort_flag) && tile_ready(count);
                q_phase[x] ^= 1u;
                ptx::tc_fence_after_sync();
                if (ok) scores(x, 0);
            }
            for (int j = 0; j < n && ok; ++j) {
                for (int x = 0; x < 2 && ok; ++x) {
                    const int mine = x ? n1 : n0;
                    if (j >= mine) continue;
                    ok = tile_ready(count + 2 * j + 1) && warp_wait(&s_probs[x], p_phase[x], abort_flag);
                    p_phase[x] ^= 1u;
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
                    if (ptx::elect_one()) {
                        au_weighted(tmem + 256 + x * 128, tmem + x * 128, ring_addr + slot_of(count + 2 * j + 1) * Plan::TILE_BYTES, idesc_o, j > 0);
                        if (j == mine - 1) ptx::umma_commit(&s_done[x]);
                        if (x == 1 || j >= n1) ptx::umma_commit(&s_empty[slot_of(count + 2 * j + 1)]);
                    }
                    __syncwarp();
                    if (j + 1 < mine) {
                        ok = tile_ready(count + 2 * j + 2);
                        ptx::tc_fence_after_sync();
                        if (ok) scores(x, j + 1);
                    }
                }
            }
            count += 2 * n;
        }
      }
    } else {
        ptx::registers_up<AU_ROW_REGS>();
        const int x = warp >> 2;
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = ((uint32_t)(warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + x * 128 + lanes, t_o = tmem + 256 + x * 128 + lanes;
        const float c = a.scale * LOG2E;
        uint32_t s_phase = 0, d_phase = 0;
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h;
            order.at(w, item, h);
            const Tile t = find_tile<AF_QUERIES>(a.s, item);
            if (!t.any) continue;
            const int n = af_key_tiles(t, a.causal, x), me = t.at + x * AU_ROWS + row;
            const int last = a.causal ? min(me, t.len - 1) : t.len - 1;       // the last key that the row sees
            float top = -INFINITY, sum = 0.f;
            for (int j = 0; j < n; ++j) {
                ok = warp_wait(&s_scores[x], s_phase, abort_flag);
                if (!ok) break;
                s_phase ^= 1u;
                ptx::tc_fence_after_sync();
                uint32_t s[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) ptx::tmem_ld_32x32(t_s + 32 * i, s[i]);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 4; ++i) ptx::tmem_ld_tie(s[i]);
                const int limit = last - j * AU_ROWS;
                if (__any_sync(0xffffffffu, limit < AU_ROWS - 1)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[i][e] = 32 * i + e <= limit ? s[i][e] : 0xFF800000u;
                }
                float best[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    best[i] = __uint_as_float(s[i][0]);
#pragma unroll
                    for (int e = 1; e < 32; ++e) best[i] = fmaxf(best[i], __uint_as_float(s[i][e]));
                }
                const float seen = fmaxf(top, fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3])));
                if (j == 0) {
                    top = seen;
                } else if (__any_sync(0xffffffffu, (seen - top) * c > AF_RISE)) {
                    // the scores' arrival means that the product before, the last to add to O, is done
                    const float keep = seen == top ? 1.f : exp2_approx((top - seen) * c);
                    top = seen;
                    sum *= keep;
#pragma unroll 1
                    for (int i = 0; i < DP; i += 32) {
                        uint32_t o[32];
                        ptx::tmem_ld_32x32(t_o + i, o);
                        ptx::tmem_ld_wait();
                        ptx::tmem_ld_tie(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                        ptx::tmem_st_32x32(t_o + i, o);
                    }
                }
                const float less = top == -INFINITY ? 0.f : -top * c;         // a row that has seen no finite score
                float2 part[2] = {twice(0.f), twice(0.f)};
                const float2 cc = twice(c), ll = twice(less);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t p[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const uint32_t *from = &s[2 * i + e / 16][2 * (e % 16)];
                        const float2 f = fma2(make_float2(__uint_as_float(from[0]), __uint_as_float(from[1])), cc, ll);
                        const float2 y = make_float2(exp2_approx(f.x), exp2_approx(f.y));
                        part[e & 1] = add2(part[e & 1], y);
                        p[e] = round_bf16x2(y.x, y.y);
                    }
                    ptx::tmem_st_32x32(t_s + 32 * i, p);
                }
                sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_probs[x]);
            }
            if (!ok) break;
            if (n > 0) {
                ok = warp_wait(&s_done[x], d_phase, abort_flag);
                if (!ok) break;
                d_phase ^= 1u;
                ptx::tc_fence_after_sync();
            }
            if (t.at + x * AU_ROWS >= t.rows) continue;
            const bool valid = me < t.len, written = me < t.rows;
            const float factor = 1.f / sum;
            __nv_bfloat16* out = a.o.at<__nv_bfloat16>(t.b, t.first + me, h);
#pragma unroll 1
            for (int i = 0; i < a.d; i += 32) {
                uint32_t o[32];
                if (n > 0) {
                    ptx::tmem_ld_32x32(t_o + i, o);
                    ptx::tmem_ld_wait();
                    ptx::tmem_ld_tie(o);
                }
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    uint32_t v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        v[u] = valid ? round_bf16x2(__uint_as_float(o[e + 2 * u]) * factor, __uint_as_float(o[e + 2 * u + 1]) * factor) : 0u;
                    if (written && i + e < a.d) st16(out + i + e, make_uint4(v[0], v[1], v[2], v[3]));
                }
            }
            if (written && a.lse) a.lse[a.row_number(t, h) + me] = valid ? fmaf(top, a.scale, logf(sum)) : -INFINITY;
            ptx::tc_fence_before_sync();       // O has been read before the next item's first probabilities are announced
        }
    }
    if (!ok && lane == 0) raise_status(DEV_TIMEOUT);
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == AU_MMA_WARP) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace pamm
