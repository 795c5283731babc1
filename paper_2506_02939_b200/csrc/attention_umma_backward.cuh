// The backward pass of attention on the tensor cores, in two kernels whose blocks own 128 rows each:
//   queries   S = Q K^T, dP = dO V^T;  dS = P (dP - delta);  dQ += dS K            over tiles of keys;  delta on the way
//   keys      S^T = K Q^T, dP^T = V dO^T;  dV += P^T dO;  dK += dS^T Q             over tiles of queries of every head of the group
// Two fixed tiles stay in shared memory, a ring brings the others in pairs.  Two threads own a row, each of them 64 of a tile's
// 128 scores.  They read scores from tensor memory and put P and dS back over them as bf16 operands, each thread inside its own
// half, so that neither waits for the other.  The products of the next item follow those of the last without a gap, its
// accumulators' first excepted, which waits until the last ones have been read.
// The roundings of P and dS to bf16 are the operands'; what leaves is accumulated in fp32 and rounded once.
#pragma once
#include "attention_umma.cuh"

namespace pamm {

// The products' steps, one tile of the ring's pair each, over all items of the block.
struct Step { bool any, first, last; };
// The tiles of queries that see a tile of keys: `per` of each of the group's heads, from tile `from` on.
__device__ __forceinline__ int ab_query_tiles(const Tile& t, bool causal, int group, int& from, int& per) {
    from = causal ? t.at / AU_ROWS : 0;
    per = (t.len + AU_ROWS - 1) / AU_ROWS - from;
    return per * group;
}
template <bool KEYS>
struct StepReader {
    ItemReader reader;
    int n = 0, j = 0;
    bool end = false;
    __device__ __forceinline__ Step next(bool causal, int group, bool& ok) {
        if (!end && j == n) {
            Item item;
            int from, per;
            end = !reader.next_alone(item, ok);
            if (!end) n = KEYS ? ab_query_tiles(item.t, causal, group, from, per) : au_key_tiles(item.t, causal, 0);
            j = 0;
        }
        const Step s = {!end, j == 0, j == n - 1};
        ++j;
        return s;
    }
};
// A fixed tile, as soon as its place is free.  The whole warp.
template <int DP>
__device__ __forceinline__ bool ab_load_fixed(uint8_t* dst, const CUtensorMap* tm, const Item& item, uint64_t* full, uint64_t* empty, uint32_t phase,
                                              volatile Watch* watch) {
    if (!warp_wait(empty, phase ^ 1u, watch)) return false;
    if (ptx::elect_one()) {
        ptx::mbar_arrive_expect_tx(full, DP / 64 * AU_BLOCK_BYTES);
        au_load<DP>(dst, tm, item.t, item.head, item.t.at, full);
    }
    __syncwarp();
    return true;
}
__device__ __forceinline__ void ab_drain(const TileRing& ring, uint64_t* full) {
    au_drain(ring);
    int never = 0;
    for (int x = 0; x < 4; ++x) ptx::mbar_wait(&full[x & 1], (uint32_t)x >> 1, &never, 1u << 14);
}

// Rows of queries: dQ and delta.  Tensor memory: two buffers of S (dS takes their place), dP, dQ.
template <int DP>
__global__ void __launch_bounds__(AU_THREADS, 1)
attention_queries_backward_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionMaps m, const __grid_constant__ AttentionOrder order) {
    using Plan = AttentionPlan<DP>;
    constexpr int K_SLOTS = (Plan::SLOTS + 1) / 2, V_SLOTS = Plan::SLOTS / 2;      // K stays for two products: rings of their own
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) ItemQueue s_queue;
    __shared__ uint64_t s_full[Plan::SLOTS], s_empty[Plan::SLOTS], s_ffull[2], s_fempty[2], s_scores[2], s_grads, s_read, s_ds[2], s_done, s_free, s_rows,
        s_rows_free, s_tail[2], s_last[2];
    __shared__ float s_less[AU_ROWS], s_delta[AU_ROWS];
    __shared__ uint32_t s_tmem;
    __shared__ Watch s_watch;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* fixed = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring_tiles = fixed + 2 * Plan::TILE_BYTES;
    if (threadIdx.x == 0) {
        s_queue.init(15);
        for (int i = 0; i < Plan::SLOTS; ++i) { ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&s_empty[i], 1); }
        for (int x = 0; x < 2; ++x) {
            ptx::mbar_init(&s_ffull[x], 1);
            ptx::mbar_init(&s_fempty[x], 1);
            ptx::mbar_init(&s_scores[x], 1);
            ptx::mbar_init(&s_ds[x], 8);
        }
        ptx::mbar_init(&s_grads, 1);
        ptx::mbar_init(&s_read, 8);
        ptx::mbar_init(&s_done, 1);
        ptx::mbar_init(&s_free, 4);
        ptx::mbar_init(&s_rows, 4);
        ptx::mbar_init(&s_rows_free, 8);
        ptx::mbar_init(&s_tail[0], 1);
        ptx::mbar_init(&s_tail[1], 1);
        ptx::mbar_init(&s_last[0], 1);
        ptx::mbar_init(&s_last[1], 1);
        s_watch = {};
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
    volatile Watch* watch = &s_watch;
    grid_dependency_wait();
    bool ok = true;
    ItemReader reader = {&s_queue, watch};
    Item item;

    if (warp >= AU_TMA_WARP) {
        ptx::registers_down<AU_OTHER_REGS>();
        if (warp == AU_ITEMS_WARP) {
            ok = au_find_items<AU_ROWS>(s_queue, a.s, order, watch, [&](const Tile& t) { return au_key_tiles(t, a.causal, 0); },
                                        [&](const Item& it) { au_clear(a.dq, it, AU_ROWS, a.d); });
        } else if (warp == AU_TMA_WARP) {
            TileRing keys = {ring_tiles, s_full, s_empty, &s_tail[0], watch, K_SLOTS, 0, 0, 0, 0, false};
            TileRing values = {ring_tiles + K_SLOTS * Plan::TILE_BYTES, s_full + K_SLOTS, s_empty + K_SLOTS, &s_tail[1], watch, V_SLOTS, 0, 0, 0, 0, false};
            uint32_t f_phase = 0;
            while (reader.next(item, ok)) {
                const Tile& t = item.t;
                const int n = au_key_tiles(t, a.causal, 0), hk = item.head / a.group;
                const bool clear = t.first + t.len < a.s.seq;
                for (int j = 0; j < n && ok; ++j) {
                    ok = (j > 0 || ab_load_fixed<DP>(fixed, &m.q, item, &s_ffull[0], &s_fempty[0], f_phase, watch)) &&
                         au_produce<DP>(keys, &m.k, t, hk, j * AU_ROWS, clear) &&
                         (j > 0 || ab_load_fixed<DP>(fixed + Plan::TILE_BYTES, &m.d_o, item, &s_ffull[1], &s_fempty[1], f_phase, watch)) &&
                         au_produce<DP>(values, &m.v, t, hk, j * AU_ROWS, clear);
                }
                if (!ok) break;
                f_phase ^= 1u;
            }
            if (!ok) {
                ab_drain(keys, s_ffull);
                au_drain(values);
            }
        } else if (warp == AU_MMA_WARP && ptx::elect_one()) {
            // S two steps ahead of dQ, whose dS takes the place of the scores it came from
            const uint32_t idesc_s = ptx::umma_idesc_bf16(AU_ROWS, AU_ROWS);
            const uint32_t idesc_g = ptx::umma_idesc_bf16(AU_ROWS, (uint32_t)((a.d + 15) / 16 * 16)) | (1u << 16);      // B MN-major
            const int steps = (a.d + 15) / 16;
            const uint32_t f_addr = ptx::smem_u32(fixed), ring_addr = ptx::smem_u32(ring_tiles);
            uint32_t q_phase = 0, free_phase = 1, scored = 0, taken = 0;        // the next tile of each kind of product
            const auto wait = [&](uint64_t& bar, uint32_t parity) { return au_wait(&bar, parity & 1u, watch); };
            StepReader<false> ahead = {reader};
            Step now = {}, one = {};
#pragma unroll 1
            for (int step = -2; ok; ++step) {
                const Step two = ahead.next(a.causal, a.group, ok);
                if (!ok || !(now.any || one.any || two.any)) break;
                const uint32_t buffer = tmem + (step & 1) * 128;
                if (now.any) {
                    if (!(ok = wait(s_ds[step & 1], (uint32_t)step >> 1))) break;
                    if (now.first) {
                        if (!(ok = wait(s_free, free_phase))) break;
                        free_phase ^= 1u;
                    }
                    const uint32_t slot = taken++ % K_SLOTS;
                    ptx::tc_fence_after_sync();
                    au_weighted(tmem + 384, buffer, ring_addr + slot * Plan::TILE_BYTES, idesc_g, !now.first);
                    ptx::umma_commit(&s_empty[slot]);
                    if (now.last) ptx::umma_commit(&s_done);
                }
                if (two.any) {
                    if (two.first) {
                        if (!(ok = wait(s_ffull[0], q_phase))) break;
                        q_phase ^= 1u;
                    }
                    const uint32_t slot = scored % K_SLOTS;
                    if (!(ok = wait(s_full[slot], scored / K_SLOTS))) break;
                    ++scored;
                    ptx::tc_fence_after_sync();
                    au_scores<DP>(buffer, f_addr, ring_addr + slot * Plan::TILE_BYTES, steps, idesc_s);
                    ptx::umma_commit(&s_scores[step & 1]);
                    if (two.last) ptx::umma_commit(&s_fempty[0]);
                }
                now = one;
                one = two;
            }
            if (!ok) au_settle(&s_last[0]);
        } else if (warp == AU_MMA_WARP + 1 && ptx::elect_one()) {
            // dP, as soon as the last one has been read
            const uint32_t idesc_s = ptx::umma_idesc_bf16(AU_ROWS, AU_ROWS);
            const int steps = (a.d + 15) / 16;
            const uint32_t f_addr = ptx::smem_u32(fixed) + Plan::TILE_BYTES, ring_addr = ptx::smem_u32(ring_tiles);
            uint32_t g_phase = 0;
            const auto wait = [&](uint64_t& bar, uint32_t parity) { return au_wait(&bar, parity & 1u, watch); };
            StepReader<false> ahead = {reader};
#pragma unroll 1
            for (uint32_t step = 0; ok; ++step) {
                const Step now = ahead.next(a.causal, a.group, ok);
                if (!ok || !now.any) break;
                if (now.first) {
                    if (!(ok = wait(s_ffull[1], g_phase))) break;
                    g_phase ^= 1u;
                }
                const uint32_t slot = K_SLOTS + step % V_SLOTS;
                if (!(ok = wait(s_full[slot], step / V_SLOTS) && wait(s_read, step + 1))) break;      // the first finds it free
                ptx::tc_fence_after_sync();
                au_scores<DP>(tmem + 256, f_addr, ring_addr + slot * Plan::TILE_BYTES, steps, idesc_s);
                ptx::umma_commit(&s_grads);
                ptx::umma_commit(&s_empty[slot]);
                if (now.last) ptx::umma_commit(&s_fempty[1]);
            }
            if (!ok) au_settle(&s_last[1]);
        }
    } else if (warp >= AU_FINISH_WARP) {
        // An item's deltas and log-sums before its first step, while the item before is computed; then the gradients of that one.
        ptx::registers_down<AU_OTHER_REGS>();
        const int quarter = (warp & 3) * 32, row = quarter + lane;
        const uint32_t lanes = (uint32_t)quarter << 16;
        uint32_t done_phase = 0, rows_phase = 1;
        Item before;
        bool any = false, more = true;
        while (more || any) {
            more = more && reader.next(item, ok);
            if (!ok) break;
            if (more) {
                const Tile& t = item.t;
                const int pieces = a.d / 8, piece = lane & 15, valid = t.len - t.at - quarter;      // of 16 bytes, 16 lanes a row
                const int64_t number = a.row_number(t, item.head) + t.at + quarter;
                const __nv_bfloat16 *o = a.o.at<__nv_bfloat16>(t.b, t.first + t.at + quarter, item.head) + piece * 8;
                const __nv_bfloat16 *g = a.d_o.at<__nv_bfloat16>(t.b, t.first + t.at + quarter, item.head) + piece * 8;
                if (lane < valid) {       // all rows are on their way to L2 before the first is waited for
                    const __nv_bfloat16 *o_row = o - piece * 8 + lane * a.o.token, *g_row = g - piece * 8 + lane * a.d_o.token;
                    for (int e = 0; e < a.d; e += 64) {
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(o_row + e));
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(g_row + e));
                    }
                }
                const float less = lane < valid ? -a.lse_in[number + lane] * LOG2E : 0.f;
                float delta = 0.f;
#pragma unroll 1
                for (int r = 0; r < 32; r += 8) {       // eight rows of loads in flight
                    uint4 x[4], y[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = r + 2 * i + (lane >> 4);
                        x[i] = y[i] = make_uint4(0, 0, 0, 0);
                        if (piece < pieces && at < valid) {
                            x[i] = *reinterpret_cast<const uint4*>(o + at * a.o.token);
                            y[i] = *reinterpret_cast<const uint4*>(g + at * a.d_o.token);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float p[8], q[8], part = 0.f;
                        unpack_vec<__nv_bfloat16>(x[i], p);
                        unpack_vec<__nv_bfloat16>(y[i], q);
#pragma unroll
                        for (int e = 0; e < 8; ++e) part = fmaf(p[e], q[e], part);
                        part = warp_sum<16>(part);
                        const float mine = __shfl_sync(0xffffffffu, part, (lane & 1) * 16);
                        if ((lane >> 1) == (r >> 1) + i) delta = mine;
                    }
                }
                if (lane < valid) a.delta[number + lane] = delta;
                ok = warp_wait(&s_rows_free, rows_phase, watch);
                if (!ok) break;
                rows_phase ^= 1u;
                s_less[row] = less;
                s_delta[row] = delta;
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_rows);
            }
            if (any) {
                const Tile& t = before.t;
                const int me = t.at + row;
                ok = warp_wait(&s_done, done_phase, watch);
                if (!ok) break;
                done_phase ^= 1u;
                ptx::tc_fence_after_sync();
                au_store(tmem + 384 + lanes, a.dq.at<__nv_bfloat16>(t.b, t.first + me, before.head), a.d, a.scale, true, me < t.len, me < t.rows, a.wide,
                         &s_free);
            }
            before = item;
            any = more;
        }
    } else {
        ptx::registers_up<AU_ROW_REGS>();
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = ((uint32_t)(warp & 3) * 32) << 16;
        const uint32_t t_g = tmem + 256 + half * 64 + lanes;
        const float c = a.scale * LOG2E;
        uint32_t step = 0, phase = 0;
        while (reader.next(item, ok)) {
            const Tile& t = item.t;
            const int n = au_key_tiles(t, a.causal, 0), me = t.at + row;
            const int last = a.causal ? min(me, t.len - 1) : t.len - 1;
            ok = warp_wait(&s_rows, phase, watch);
            if (!ok) break;
            phase ^= 1u;
            const float less = s_less[row], delta = s_delta[row];
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&s_rows_free);
            for (int j = 0; j < n; ++j, ++step) {
                const uint32_t t_s = tmem + (step & 1u) * 128 + half * 64 + lanes;
                ok = warp_wait(&s_scores[step & 1u], (step >> 1) & 1u, watch);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                uint32_t s[2][32];
                ptx::tmem_ld_32x32(t_s, s[0]);
                ptx::tmem_ld_32x32(t_s + 32, s[1]);
                ptx::tmem_ld_wait();
                ptx::tmem_ld_tie(s[0]);
                ptx::tmem_ld_tie(s[1]);
                const int limit = last - j * AU_ROWS - half * 64;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        s[i][e] = __float_as_uint(exp2_approx(fmaf(__uint_as_float(s[i][e]), c, less)));
                        s[i][e + 1] = __float_as_uint(exp2_approx(fmaf(__uint_as_float(s[i][e + 1]), c, less)));
                    }
                if (__any_sync(0xffffffffu, limit < 63)) {
                    mask_behind(s[0], limit, 0u);
                    mask_behind(s[1], limit - 32, 0u);
                }
                ok = warp_wait(&s_grads, step & 1u, watch);
                if (!ok) break;
                ptx::tc_fence_after_sync();
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t g[32], p[16];
                    ptx::tmem_ld_32x32(t_g + 32 * i, g);
                    ptx::tmem_ld_wait();
                    ptx::tmem_ld_tie(g);
                    if (i == 1) {
                        ptx::tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(&s_read);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        p[e] = round_bf16x2(__uint_as_float(s[i][2 * e]) * (__uint_as_float(g[2 * e]) - delta),
                                            __uint_as_float(s[i][2 * e + 1]) * (__uint_as_float(g[2 * e + 1]) - delta));
                    }
                    ptx::tmem_st_32x16(t_s + 16 * i, p);
                }
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_ds[step & 1u]);
            }
            if (!ok) break;
        }
    }
    if (!ok) raise_status(DEV_TIMEOUT);
    __syncwarp();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == AU_MMA_WARP) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 512);
    }
}

// Rows of keys: dK and dV.  Tensor memory: S^T (P^T takes its place), dP^T (dS^T), dV, dK.  The log-sums and deltas of a tile's
// queries, which are its columns, are brought to shared memory by a warp of their own, the next tile's as soon as the last use is over.
template <int DP>
__global__ void __launch_bounds__(AU_THREADS, 1)
attention_keys_backward_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionMaps m, const __grid_constant__ AttentionOrder order) {
    using Plan = AttentionPlan<DP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) ItemQueue s_queue;
    __shared__ uint64_t s_full[Plan::SLOTS], s_empty[Plan::SLOTS], s_ffull[2], s_fempty[2], s_scores[2], s_weights[2], s_done[2], s_free[2], s_stats[2],
        s_tail, s_last;      // [0]: S, P, dV, log-sums; [1]: dP, dS, dK, deltas
    __shared__ __align__(16) float s_less[AU_ROWS], s_delta[AU_ROWS];
    __shared__ uint32_t s_tmem;
    __shared__ Watch s_watch;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* fixed = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring_tiles = fixed + 2 * Plan::TILE_BYTES;
    if (threadIdx.x == 0) {
        s_queue.init(15);
        for (int i = 0; i < Plan::SLOTS; ++i) { ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&s_empty[i], 1); }
        for (int x = 0; x < 2; ++x) {
            ptx::mbar_init(&s_ffull[x], 1);
            ptx::mbar_init(&s_fempty[x], 1);
            ptx::mbar_init(&s_stats[x], 1);
            ptx::mbar_init(&s_scores[x], 1);
            ptx::mbar_init(&s_weights[x], 8);
            ptx::mbar_init(&s_done[x], 1);
            ptx::mbar_init(&s_free[x], 4);
        }
        ptx::mbar_init(&s_tail, 1);
        ptx::mbar_init(&s_last, 1);
        s_watch = {};
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
    volatile Watch* watch = &s_watch;
    grid_dependency_wait();
    bool ok = true;
    ItemReader reader = {&s_queue, watch};
    Item item;
    int from, per;

    if (warp >= AU_TMA_WARP) {
        ptx::registers_down<AU_OTHER_REGS>();
        if (warp == AU_ITEMS_WARP) {
            ok = au_find_items<AU_ROWS>(s_queue, a.s, order, watch, [&](const Tile& t) { return ab_query_tiles(t, a.causal, a.group, from, per); }, [&](const Item& it) {
                au_clear(a.dk, it, AU_ROWS, a.d);
                au_clear(a.dv, it, AU_ROWS, a.d);
            });
        } else if (warp == AU_TMA_WARP) {
            TileRing ring = {ring_tiles, s_full, s_empty, &s_tail, watch, Plan::SLOTS, 0, 0, 0, 0, false};
            uint32_t f_phase = 0;
            while (reader.next(item, ok)) {
                const Tile& t = item.t;
                const int n = ab_query_tiles(t, a.causal, a.group, from, per);
                const bool clear = t.first + t.len < a.s.seq;
                for (int j = 0; j < n && ok; ++j) {
                    const int g = j / per, at = (from + j - g * per) * AU_ROWS, h = item.head * a.group + g;
                    ok = (j > 0 || ab_load_fixed<DP>(fixed, &m.k, item, &s_ffull[0], &s_fempty[0], f_phase, watch)) &&
                         au_produce<DP>(ring, &m.q, t, h, at, clear) &&
                         (j > 0 || ab_load_fixed<DP>(fixed + Plan::TILE_BYTES, &m.v, item, &s_ffull[1], &s_fempty[1], f_phase, watch)) &&
                         au_produce<DP>(ring, &m.d_o, t, h, at, clear);
                }
                if (!ok) break;
                f_phase ^= 1u;
            }
            if (!ok) ab_drain(ring, s_ffull);
        } else if (warp == AU_MMA_WARP) {
          if (ptx::elect_one()) {
            // dV += P^T dO and the next S^T = K Q^T (what = 0), then dK += dS^T Q and the next dP^T = V dO^T (1): the scores that the rows'
            // warps wait for go first.  (Two threads, one a kind, had their products run between each other: 18% slower.)
            const uint32_t idesc_s = ptx::umma_idesc_bf16(AU_ROWS, AU_ROWS);
            const uint32_t idesc_g = ptx::umma_idesc_bf16(AU_ROWS, (uint32_t)((a.d + 15) / 16 * 16)) | (1u << 16);
            const int steps = (a.d + 15) / 16;
            const uint32_t f_addr = ptx::smem_u32(fixed), ring_addr = ptx::smem_u32(ring_tiles);
            uint32_t f_phase = 0, free_phase = 3, phase = 0;        // bit `what`
            uint32_t scored = 0, taken = 0;         // ring tiles before the pair that the scores, and the weighted operands, take next
            const auto wait = [&](uint64_t& bar, uint32_t parity) { return au_wait(&bar, parity & 1u, watch); };
            StepReader<true> ahead = {reader};
            Step now = {};
            for (bool begun = false; ok; begun = true) {
                const Step one = ahead.next(a.causal, a.group, ok);
                if (!ok || !(now.any || one.any)) break;
#pragma unroll 1
                for (int what = 0; what < 2; ++what) {
                    if (now.any) {
                        if (!(ok = wait(s_weights[what], phase))) break;
                        if (now.first) {
                            if (!(ok = wait(s_free[what], free_phase >> what))) break;
                            free_phase ^= 1u << what;
                        }
                        const uint32_t slot = (taken + 1 - what) % Plan::SLOTS;
                        ptx::tc_fence_after_sync();
                        au_weighted(tmem + 256 + what * 128, tmem + what * 128, ring_addr + slot * Plan::TILE_BYTES, idesc_g, !now.first);
                        ptx::umma_commit(&s_empty[slot]);
                        if (now.last) ptx::umma_commit(&s_done[what]);
                    }
                    if (one.any) {
                        if (one.first) {
                            if (!(ok = wait(s_ffull[what], f_phase >> what))) break;
                            f_phase ^= 1u << what;
                        }
                        const uint32_t tile = scored + what, slot = tile % Plan::SLOTS;
                        if (!(ok = wait(s_full[slot], tile / Plan::SLOTS))) break;
                        ptx::tc_fence_after_sync();
                        au_scores<DP>(tmem + what * 128, f_addr + what * Plan::TILE_BYTES, ring_addr + slot * Plan::TILE_BYTES, steps, idesc_s);
                        ptx::umma_commit(&s_scores[what]);
                        if (one.last) ptx::umma_commit(&s_fempty[what]);
                    }
                }
                scored += 2;
                if (begun) {
                    taken += 2;
                    phase ^= 1u;
                }
                now = one;
            }
            if (!ok) au_settle(&s_last);
          }
        } else {
            uint32_t phase = 1;      // the first tile waits for nothing
            while (reader.next(item, ok)) {
                const Tile& t = item.t;
                const int n = ab_query_tiles(t, a.causal, a.group, from, per);
                for (int j = 0; j < n && ok; ++j, phase ^= 1u) {
                    const int g = j / per, at = (from + j - g * per) * AU_ROWS;
                    const int64_t number = a.row_number(t, item.head * a.group + g);
                    float less[4], delta[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int q = at + lane + 32 * u;
                        const bool valid = q < t.len;      // others have scores of 0: their probabilities become 0
                        less[u] = valid ? -a.lse_in[number + q] * LOG2E : -INFINITY;
                        delta[u] = valid ? -a.delta[number + q] : 0.f;
                    }
                    ok = warp_wait(&s_weights[0], phase, watch);
                    if (!ok) break;
#pragma unroll
                    for (int u = 0; u < 4; ++u) s_less[lane + 32 * u] = less[u];
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&s_stats[0]);
                    ok = warp_wait(&s_weights[1], phase, watch);
                    if (!ok) break;
#pragma unroll
                    for (int u = 0; u < 4; ++u) s_delta[lane + 32 * u] = delta[u];
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&s_stats[1]);
                }
                if (!ok) break;
            }
        }
    } else if (warp >= AU_FINISH_WARP) {
        ptx::registers_down<AU_OTHER_REGS>();
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = ((uint32_t)(warp & 3) * 32) << 16;
        uint32_t phase = 0;
        while (reader.next(item, ok)) {
            const Tile& t = item.t;
            const int me = t.at + row;
            for (int what = 0; what < 2 && ok; ++what) {
                ok = warp_wait(&s_done[what], phase, watch);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                au_store(tmem + 256 + what * 128 + lanes, (what ? a.dk : a.dv).at<__nv_bfloat16>(t.b, t.first + me, item.head), a.d, what ? a.scale : 1.f, true,
                         me < t.len, me < t.rows, a.wide, &s_free[what]);
            }
            if (!ok) break;
            phase ^= 1u;
        }
    } else {
        ptx::registers_up<AU_ROW_REGS>();
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = ((uint32_t)(warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + half * 64 + lanes, t_g = t_s + 128;
        const float c = a.scale * LOG2E;
        uint32_t phase = 0;        // one phase a tile for all barriers of the tile
        while (reader.next(item, ok)) {
            const int n = ab_query_tiles(item.t, a.causal, a.group, from, per);
            for (int j = 0; j < n; ++j, phase ^= 1u) {
                ok = warp_wait(&s_stats[0], phase, watch) && warp_wait(&s_scores[0], phase, watch);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                uint32_t s[2][32];
                ptx::tmem_ld_32x32(t_s, s[0]);
                ptx::tmem_ld_32x32(t_s + 32, s[1]);
                ptx::tmem_ld_wait();
                ptx::tmem_ld_tie(s[0]);
                ptx::tmem_ld_tie(s[1]);
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const float4 less = *reinterpret_cast<const float4*>(s_less + half * 64 + 32 * u + e);
                        s[u][e] = __float_as_uint(exp2_approx(fmaf(__uint_as_float(s[u][e]), c, less.x)));
                        s[u][e + 1] = __float_as_uint(exp2_approx(fmaf(__uint_as_float(s[u][e + 1]), c, less.y)));
                        s[u][e + 2] = __float_as_uint(exp2_approx(fmaf(__uint_as_float(s[u][e + 2]), c, less.z)));
                        s[u][e + 3] = __float_as_uint(exp2_approx(fmaf(__uint_as_float(s[u][e + 3]), c, less.w)));
                    }
                if (a.causal && j % per == 0) {      // the tile on the diagonal: queries before the key do not see it
                    const int first = row - half * 64;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[u][e] = 32 * u + e >= first ? s[u][e] : 0u;
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) p[e] = round_bf16x2(__uint_as_float(s[u][2 * e]), __uint_as_float(s[u][2 * e + 1]));
                    ptx::tmem_st_32x16(t_s + 16 * u, p);
                }
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_weights[0]);
                ok = warp_wait(&s_stats[1], phase, watch) && warp_wait(&s_scores[1], phase, watch);
                if (!ok) break;
                ptx::tc_fence_after_sync();
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    uint32_t g[32], p[16];
                    ptx::tmem_ld_32x32(t_g + 32 * u, g);
                    ptx::tmem_ld_wait();
                    ptx::tmem_ld_tie(g);
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        const float4 d = *reinterpret_cast<const float4*>(s_delta + half * 64 + 32 * u + 2 * e);
                        p[e] = round_bf16x2(__uint_as_float(s[u][2 * e]) * (__uint_as_float(g[2 * e]) + d.x),
                                            __uint_as_float(s[u][2 * e + 1]) * (__uint_as_float(g[2 * e + 1]) + d.y));
                        p[e + 1] = round_bf16x2(__uint_as_float(s[u][2 * e + 2]) * (__uint_as_float(g[2 * e + 2]) + d.z),
                                                __uint_as_float(s[u][2 * e + 3]) * (__uint_as_float(g[2 * e + 3]) + d.w));
                    }
                    // the second half's gradients are still to be read: dS stays inside what the first half left
                    ptx::tmem_st_32x16(t_g + 16 * u, p);
                }
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_weights[1]);
            }
            if (!ok) break;
        }
    }
    if (!ok) raise_status(DEV_TIMEOUT);
    __syncwarp();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == AU_MMA_WARP) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace pamm
