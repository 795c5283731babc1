// The backward pass of attention on the tensor cores, in two kernels whose blocks own 128 rows each:
//   queries   S = Q K^T, dP = dO V^T;  dS = P (dP - delta);  dQ += dS K            over tiles of keys;  delta on the way
//   keys      S^T = K Q^T, dP^T = V dO^T;  dV += P^T dO;  dK += dS^T Q             over tiles of queries of every head of the group
// Two fixed tiles stay in shared memory, a ring brings the others in pairs.  Eight warps: two threads own a row, each of
// them 64 of a tile's 128 scores.  They read scores from tensor memory and put P and dS back over them as bf16 operands, each thread
// inside its own half, so that neither waits for the other.
// The roundings of P and dS to bf16 are the operands'; what leaves is accumulated in fp32 and rounded once.
#pragma once
#include "attention_umma.cuh"

namespace pamm {

constexpr int AB_THREADS = 384, AB_STATS_WARP = 10;

template <int DP>
struct BackwardPlan {
    static constexpr int TILE_BYTES = DP / 64 * AU_BLOCK_BYTES;
    static constexpr int SLOTS = DP == 128 ? 5 : 8;
    static constexpr size_t SMEM = 1024 + (size_t)(2 + SLOTS) * TILE_BYTES;
};

// D (+)= W B with W's two halves of 64 columns 64 tensor-memory columns apart.  One thread.
__device__ __forceinline__ void ab_weighted(uint32_t d_tmem, uint32_t w_tmem, uint32_t b, uint32_t idesc, bool accumulate) {
#pragma unroll
    for (int k = 0; k < AU_ROWS / 16; ++k)
        ptx::umma_bf16_ts(d_tmem, w_tmem + (k >> 2) * 64 + (k & 3) * 8, umma_desc_mn_sw128(b + k * 2048, AU_BLOCK_BYTES, 1024), idesc, accumulate || k > 0);
}
// Columns from .. from + 32 n of a row's accumulator to memory, zero where the token is not valid.  A whole warp.
__device__ __forceinline__ void ab_store(uint32_t t_acc, __nv_bfloat16* out, int from, int to, int d, float factor, bool loaded, bool valid, bool written) {
#pragma unroll 1
    for (int i = from; i < to && i < d; i += 32) {
        uint32_t o[32];
        if (loaded) {
            ptx::tmem_ld_32x32(t_acc + i, o);
            ptx::tmem_ld_wait();
            ptx::tmem_ld_tie(o);
        }
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
            uint32_t v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                v[u] = valid ? round_bf16x2(__uint_as_float(o[e + 2 * u]) * factor, __uint_as_float(o[e + 2 * u + 1]) * factor) : 0u;
            if (written && i + e < d) st16(out + i + e, make_uint4(v[0], v[1], v[2], v[3]));
        }
    }
}
// The fixed tiles of an item, each as soon as its place is free.  The whole warp.
template <int DP>
__device__ __forceinline__ bool ab_load_fixed(uint8_t* tiles, const CUtensorMap* m0, const CUtensorMap* m1, const Tile& t, int head, uint64_t* full,
                                              uint64_t* empty, uint32_t& phase, volatile int* abort_flag) {
    constexpr int BYTES = DP / 64 * AU_BLOCK_BYTES;
    for (int x = 0; x < 2; ++x) {
        if (!warp_wait(&empty[x], phase ^ 1u, abort_flag)) return false;
        if (ptx::elect_one()) {
            ptx::mbar_arrive_expect_tx(&full[x], BYTES);
            au_load<DP>(tiles + x * BYTES, x ? m1 : m0, t, head, t.at, &full[x]);
        }
        __syncwarp();
    }
    phase ^= 1u;
    return true;
}

// Rows of queries: dQ and delta.  Tensor memory: two buffers of S (dS takes their place), dP, dQ.
template <int DP>
__global__ void __launch_bounds__(AB_THREADS, 1)
attention_queries_backward_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionMaps m, const __grid_constant__ AttentionOrder order,
                                  const int works) {
    using Plan = BackwardPlan<DP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t s_full[Plan::SLOTS], s_empty[Plan::SLOTS], s_ffull[2], s_fempty[2], s_scores[2], s_grads, s_read, s_ds[2], s_done, s_tail, s_halves;
    __shared__ float s_delta[2][AU_ROWS];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* fixed = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring_tiles = fixed + 2 * Plan::TILE_BYTES;
    if (threadIdx.x == 0) {
        for (int i = 0; i < Plan::SLOTS; ++i) { ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&s_empty[i], 1); }
        for (int x = 0; x < 2; ++x) {
            ptx::mbar_init(&s_ffull[x], 1);
            ptx::mbar_init(&s_fempty[x], 1);
            ptx::mbar_init(&s_scores[x], 1);
            ptx::mbar_init(&s_ds[x], 8);
        }
        ptx::mbar_init(&s_grads, 1);
        ptx::mbar_init(&s_read, 8);
        ptx::mbar_init(&s_halves, 8);
        ptx::mbar_init(&s_done, 1);
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

    if (warp == AU_TMA_WARP) {
        TileRing ring = {ring_tiles, s_full, s_empty, &s_tail, abort_flag, Plan::SLOTS, 0, 0, 0, 0, false};
        uint32_t f_phase = 0;
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h;
            order.at(w, item, h);
            const Tile t = find_tile<AU_ROWS>(a.s, item);
            const int n = t.any ? af_key_tiles(t, a.causal, 0) : 0;
            if (n == 0) continue;
            const bool clear = t.first + t.len < a.s.seq;
            ok = ab_load_fixed<DP>(fixed, &m.q, &m.d_o, t, h, s_ffull, s_fempty, f_phase, abort_flag);
            for (int j = 0; j < n && ok; ++j)
                ok = au_produce<DP>(ring, &m.k, t, h / a.group, j * AU_ROWS, clear) && au_produce<DP>(ring, &m.v, t, h / a.group, j * AU_ROWS, clear);
        }
        if (!ok) {
            au_drain(ring);
            int never = 0;
            for (int x = 0; x < 4; ++x) ptx::mbar_wait(&s_ffull[x & 1], f_phase ^ (x >> 1), &never, 1u << 14);
        }
    } else if (warp == AU_MMA_WARP) {
        const uint32_t idesc_s = ptx::umma_idesc_bf16(AU_ROWS, AU_ROWS);
        const uint32_t idesc_g = ptx::umma_idesc_bf16(AU_ROWS, (uint32_t)((a.d + 15) / 16 * 16)) | (1u << 16);      // B MN-major
        const int steps = (a.d + 15) / 16;
        const uint32_t f_addr = ptx::smem_u32(fixed), ring_addr = ptx::smem_u32(ring_tiles);
        uint32_t f_phase = 0, r_phase = 0, d_phase[2] = {0, 0};
        uint32_t count = 0;
        const auto slot_of = [&](uint32_t i) { return i % Plan::SLOTS; };
        const auto address = [&](uint32_t i) { return ring_addr + slot_of(i) * Plan::TILE_BYTES; };
        const auto tile_ready = [&](uint32_t i) { return warp_wait(&s_full[slot_of(i)], (i / Plan::SLOTS) & 1u, abort_flag); };
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h;
            order.at(w, item, h);
            const Tile t = find_tile<AU_ROWS>(a.s, item);
            const int n = t.any ? af_key_tiles(t, a.causal, 0) : 0;
            if (n == 0) continue;
            const auto scores = [&](int j) {
                if (!tile_ready(count + 2 * j)) return false;
                ptx::tc_fence_after_sync();
                if (ptx::elect_one()) {
                    au_scores(tmem + (j & 1) * 128, f_addr, address(count + 2 * j), steps, idesc_s);
                    ptx::umma_commit(&s_scores[j & 1]);
                    if (j == n - 1) ptx::umma_commit(&s_fempty[0]);
                }
                __syncwarp();
                return true;
            };
            const auto grads = [&](int j) {
                if (!tile_ready(count + 2 * j + 1)) return false;
                ptx::tc_fence_after_sync();
                if (ptx::elect_one()) {
                    au_scores(tmem + 256, f_addr + Plan::TILE_BYTES, address(count + 2 * j + 1), steps, idesc_s);
                    ptx::umma_commit(&s_grads);
                    ptx::umma_commit(&s_empty[slot_of(count + 2 * j + 1)]);
                    if (j == n - 1) ptx::umma_commit(&s_fempty[1]);
                }
                __syncwarp();
                return true;
            };
            ok = warp_wait(&s_ffull[0], f_phase, abort_flag) && scores(0) && warp_wait(&s_ffull[1], f_phase, abort_flag) && grads(0);
            f_phase ^= 1u;
            if (ok && n > 1) ok = scores(1);
            for (int j = 0; j < n && ok; ++j) {
                ok = warp_wait(&s_read, r_phase, abort_flag);
                r_phase ^= 1u;
                if (ok && j + 1 < n) ok = grads(j + 1);
                ok = ok && warp_wait(&s_ds[j & 1], d_phase[j & 1], abort_flag);
                d_phase[j & 1] ^= 1u;
                if (!ok) break;
                ptx::tc_fence_after_sync();
                if (ptx::elect_one()) {
                    ab_weighted(tmem + 384, tmem + (j & 1) * 128, address(count + 2 * j), idesc_g, j > 0);
                    ptx::umma_commit(&s_empty[slot_of(count + 2 * j)]);
                    if (j == n - 1) ptx::umma_commit(&s_done);
                }
                __syncwarp();
                if (j + 2 < n) ok = scores(j + 2);
            }
            count += 2 * n;
        }
    } else if (warp < 8) {
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = ((uint32_t)(warp & 3) * 32) << 16;
        const float c = a.scale * LOG2E;
        uint32_t s_phase[2] = {0, 0}, g_phase = 0, d_phase = 0, h_phase = 0;
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h;
            order.at(w, item, h);
            const Tile t = find_tile<AU_ROWS>(a.s, item);
            if (!t.any) continue;
            const int n = af_key_tiles(t, a.causal, 0), me = t.at + row;
            const bool valid = me < t.len, written = me < t.rows;
            const int last = a.causal ? min(me, t.len - 1) : t.len - 1;
            float less = 0.f, delta = 0.f;
            if (n > 0) {
                float part = 0.f;
                if (valid) {
                    less = -a.lse_in[a.row_number(t, h) + me] * LOG2E;
                    const __nv_bfloat16 *o = a.o.at<__nv_bfloat16>(t.b, t.first + me, h), *g = a.d_o.at<__nv_bfloat16>(t.b, t.first + me, h);
                    const int vectors = a.d / 8, end = half ? vectors : vectors / 2;
#pragma unroll 4
                    for (int v = half ? vectors / 2 : 0; v < end; ++v) {
                        using P = Piece<__nv_bfloat16, 8>;
                        float x[8], y[8];
                        P::unpack(P::load(o + 8 * v), x);
                        P::unpack(P::load(g + 8 * v), y);
#pragma unroll
                        for (int e = 0; e < 8; ++e) part = fmaf(x[e], y[e], part);
                    }
                }
                s_delta[half][row] = part;
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_halves);
                ok = warp_wait(&s_halves, h_phase, abort_flag);
                h_phase ^= 1u;
                if (!ok) break;
                delta = s_delta[0][row] + s_delta[1][row];
                if (half == 0 && valid) a.delta[a.row_number(t, h) + me] = delta;
            }
            for (int j = 0; j < n; ++j) {
                const uint32_t t_s = tmem + (j & 1) * 128 + half * 64 + lanes;
                ok = warp_wait(&s_scores[j & 1], s_phase[j & 1], abort_flag);
                s_phase[j & 1] ^= 1u;
                if (!ok) break;
                ptx::tc_fence_after_sync();
                uint32_t s[2][32];
                ptx::tmem_ld_32x32(t_s, s[0]);
                ptx::tmem_ld_32x32(t_s + 32, s[1]);
                ptx::tmem_ld_wait();
                ptx::tmem_ld_tie(s[0]);
                ptx::tmem_ld_tie(s[1]);
                const int limit = last - j * AU_ROWS - half * 64;
                const float2 cc = twice(c), ll = twice(less);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float2 f = fma2(make_float2(__uint_as_float(s[i][e]), __uint_as_float(s[i][e + 1])), cc, ll);
                        s[i][e] = __float_as_uint(exp2_approx(f.x));
                        s[i][e + 1] = __float_as_uint(exp2_approx(f.y));
                    }
                if (__any_sync(0xffffffffu, limit < 63)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[i][e] = 32 * i + e <= limit ? s[i][e] : 0u;
                }
                ok = warp_wait(&s_grads, g_phase, abort_flag);
                g_phase ^= 1u;
                if (!ok) break;
                ptx::tc_fence_after_sync();
                uint32_t g[2][32];
                ptx::tmem_ld_32x32(tmem + 256 + half * 64 + lanes, g[0]);
                ptx::tmem_ld_32x32(tmem + 256 + half * 64 + 32 + lanes, g[1]);
                ptx::tmem_ld_wait();
                ptx::tmem_ld_tie(g[0]);
                ptx::tmem_ld_tie(g[1]);
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_read);
                uint32_t p[32];
                const float2 dd = twice(-delta);
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const uint32_t *u = &s[e / 16][2 * (e % 16)], *v = &g[e / 16][2 * (e % 16)];
                    const float2 x = mul2(make_float2(__uint_as_float(u[0]), __uint_as_float(u[1])),
                                          add2(make_float2(__uint_as_float(v[0]), __uint_as_float(v[1])), dd));
                    p[e] = round_bf16x2(x.x, x.y);
                }
                ptx::tmem_st_32x32(t_s, p);
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_ds[j & 1]);
            }
            if (!ok) break;
            if (n > 0) {
                ok = warp_wait(&s_done, d_phase, abort_flag);
                d_phase ^= 1u;
                if (!ok) break;
                ptx::tc_fence_after_sync();
            }
            ab_store(tmem + 384 + lanes, a.dq.at<__nv_bfloat16>(t.b, t.first + me, h), half * (DP / 2), (half + 1) * (DP / 2), a.d, a.scale, n > 0, valid, written);
            ptx::tc_fence_before_sync();
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

// Rows of keys: dK and dV.  Tensor memory: S^T (P^T takes its place), dP^T (dS^T), dV, dK.  The log-sums and deltas of a tile's
// queries, which are its columns, are brought to shared memory by a warp of their own, the next tile's as soon as the last use is over.
template <int DP>
__global__ void __launch_bounds__(AB_THREADS, 1)
attention_keys_backward_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionMaps m, const __grid_constant__ AttentionOrder order,
                               const int works) {
    using Plan = BackwardPlan<DP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t s_full[Plan::SLOTS], s_empty[Plan::SLOTS], s_ffull[2], s_fempty[2], s_scores, s_probs, s_grads, s_ds, s_done, s_tail, s_stats[2];
    __shared__ __align__(16) float s_less[AU_ROWS], s_delta[AU_ROWS];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* fixed = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring_tiles = fixed + 2 * Plan::TILE_BYTES;
    if (threadIdx.x == 0) {
        for (int i = 0; i < Plan::SLOTS; ++i) { ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&s_empty[i], 1); }
        for (int x = 0; x < 2; ++x) {
            ptx::mbar_init(&s_ffull[x], 1);
            ptx::mbar_init(&s_fempty[x], 1);
            ptx::mbar_init(&s_stats[x], 1);
        }
        ptx::mbar_init(&s_scores, 1);
        ptx::mbar_init(&s_probs, 8);
        ptx::mbar_init(&s_grads, 1);
        ptx::mbar_init(&s_ds, 8);
        ptx::mbar_init(&s_done, 1);
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

    // The tiles of queries that see the item's keys: `per` of each of the group's heads, from tile `from` on.
    const auto steps_of = [&](const Tile& t, int& from, int& per) {
        from = a.causal ? t.at / AU_ROWS : 0;
        per = t.at < t.len ? (t.len + AU_ROWS - 1) / AU_ROWS - from : 0;
        return per * a.group;
    };
    if (warp >= 8) {
      ptx::registers_down<AU_OTHER_REGS>();
      if (warp == AU_TMA_WARP) {
        TileRing ring = {ring_tiles, s_full, s_empty, &s_tail, abort_flag, Plan::SLOTS, 0, 0, 0, 0, false};
        uint32_t f_phase = 0;
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h, from, per;
            order.at(w, item, h);
            const Tile t = find_tile<AU_ROWS>(a.s, item);
            if (!t.any || steps_of(t, from, per) == 0) continue;
            const bool clear = t.first + t.len < a.s.seq;
            ok = ab_load_fixed<DP>(fixed, &m.k, &m.v, t, h, s_ffull, s_fempty, f_phase, abort_flag);
            for (int g = 0; g < a.group && ok; ++g)
                for (int i = from; i < from + per && ok; ++i)
                    ok = au_produce<DP>(ring, &m.q, t, h * a.group + g, i * AU_ROWS, clear) && au_produce<DP>(ring, &m.d_o, t, h * a.group + g, i * AU_ROWS, clear);
        }
        if (!ok) {
            au_drain(ring);
            int never = 0;
            for (int x = 0; x < 4; ++x) ptx::mbar_wait(&s_ffull[x & 1], f_phase ^ (x >> 1), &never, 1u << 14);
        }
      } else if (warp == AU_MMA_WARP) {
        const uint32_t idesc_s = ptx::umma_idesc_bf16(AU_ROWS, AU_ROWS);
        const uint32_t idesc_g = ptx::umma_idesc_bf16(AU_ROWS, (uint32_t)((a.d + 15) / 16 * 16)) | (1u << 16);
        const int steps = (a.d + 15) / 16;
        const uint32_t f_addr = ptx::smem_u32(fixed), ring_addr = ptx::smem_u32(ring_tiles);
        uint32_t f_phase = 0, p_phase = 0, d_phase = 0;
        uint32_t count = 0;
        const auto slot_of = [&](uint32_t i) { return i % Plan::SLOTS; };
        const auto address = [&](uint32_t i) { return ring_addr + slot_of(i) * Plan::TILE_BYTES; };
        const auto tile_ready = [&](uint32_t i) { return warp_wait(&s_full[slot_of(i)], (i / Plan::SLOTS) & 1u, abort_flag); };
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h, from, per;
            order.at(w, item, h);
            const Tile t = find_tile<AU_ROWS>(a.s, item);
            const int n = t.any ? steps_of(t, from, per) : 0;
            if (n == 0) continue;
            // what = 0: S^T from K and Q; 1: dP^T from V and dO
            const auto scores = [&](int what, int i) {
                if (!tile_ready(count + 2 * i + what)) return false;
                ptx::tc_fence_after_sync();
                if (ptx::elect_one()) {
                    au_scores(tmem + what * 128, f_addr + what * Plan::TILE_BYTES, address(count + 2 * i + what), steps, idesc_s);
                    ptx::umma_commit(what ? &s_grads : &s_scores);
                    if (i == n - 1) ptx::umma_commit(&s_fempty[what]);
                }
                __syncwarp();
                return true;
            };
            ok = warp_wait(&s_ffull[0], f_phase, abort_flag) && scores(0, 0) && warp_wait(&s_ffull[1], f_phase, abort_flag) && scores(1, 0);
            f_phase ^= 1u;
            for (int i = 0; i < n && ok; ++i) {
                ok = warp_wait(&s_probs, p_phase, abort_flag);
                p_phase ^= 1u;
                if (!ok) break;
                ptx::tc_fence_after_sync();
                if (ptx::elect_one()) {
                    ab_weighted(tmem + 256, tmem, address(count + 2 * i + 1), idesc_g, i > 0);
                    ptx::umma_commit(&s_empty[slot_of(count + 2 * i + 1)]);
                }
                __syncwarp();
                if (i + 1 < n) ok = scores(0, i + 1);
                ok = ok && warp_wait(&s_ds, d_phase, abort_flag);
                d_phase ^= 1u;
                if (!ok) break;
                ptx::tc_fence_after_sync();
                if (ptx::elect_one()) {
                    ab_weighted(tmem + 384, tmem + 128, address(count + 2 * i), idesc_g, i > 0);
                    ptx::umma_commit(&s_empty[slot_of(count + 2 * i)]);
                    if (i == n - 1) ptx::umma_commit(&s_done);
                }
                __syncwarp();
                if (i + 1 < n) ok = scores(1, i + 1);
            }
            count += 2 * n;
        }
      } else if (warp == AB_STATS_WARP) {
        uint32_t p_phase = 1, d_phase = 1;      // the first tile waits for nothing
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h, from, per;
            order.at(w, item, h);
            const Tile t = find_tile<AU_ROWS>(a.s, item);
            if (!t.any || steps_of(t, from, per) == 0) continue;
            for (int g = 0; g < a.group && ok; ++g) {
                const int64_t number = a.row_number(t, h * a.group + g);
                for (int i = from; i < from + per && ok; ++i) {
                    float less[4], delta[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int q = i * AU_ROWS + lane + 32 * u;
                        const bool valid = q < t.len;      // others have scores of 0: their probabilities become 0
                        less[u] = valid ? -a.lse_in[number + q] * LOG2E : -INFINITY;
                        delta[u] = valid ? -a.delta[number + q] : 0.f;
                    }
                    ok = warp_wait(&s_probs, p_phase, abort_flag);
                    p_phase ^= 1u;
                    if (!ok) break;
#pragma unroll
                    for (int u = 0; u < 4; ++u) s_less[lane + 32 * u] = less[u];
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&s_stats[0]);
                    ok = warp_wait(&s_ds, d_phase, abort_flag);
                    d_phase ^= 1u;
                    if (!ok) break;
#pragma unroll
                    for (int u = 0; u < 4; ++u) s_delta[lane + 32 * u] = delta[u];
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(&s_stats[1]);
                }
            }
        }
      }
    } else {
        ptx::registers_up<AU_ROW_REGS>();
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = ((uint32_t)(warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + half * 64 + lanes, t_g = t_s + 128;
        const float c = a.scale * LOG2E;
        uint32_t phase = 0, d_phase = 0;        // one phase a tile for all barriers of the tile
        for (int w = blockIdx.x; w < works && ok; w += gridDim.x) {
            int item, h, from, per;
            order.at(w, item, h);
            const Tile t = find_tile<AU_ROWS>(a.s, item);
            if (!t.any) continue;
            const int n = steps_of(t, from, per), me = t.at + row;
            const bool valid = me < t.len, written = me < t.rows;
            for (int i = 0; i < n; ++i, phase ^= 1u) {
                ok = warp_wait(&s_stats[0], phase, abort_flag) && warp_wait(&s_scores, phase, abort_flag);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                uint32_t s[2][32];
                ptx::tmem_ld_32x32(t_s, s[0]);
                ptx::tmem_ld_32x32(t_s + 32, s[1]);
                ptx::tmem_ld_wait();
                ptx::tmem_ld_tie(s[0]);
                ptx::tmem_ld_tie(s[1]);
                const float2 cc = twice(c);
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const float4 less = *reinterpret_cast<const float4*>(s_less + half * 64 + 32 * u + e);
                        const float2 f = fma2(make_float2(__uint_as_float(s[u][e]), __uint_as_float(s[u][e + 1])), cc, make_float2(less.x, less.y));
                        const float2 g = fma2(make_float2(__uint_as_float(s[u][e + 2]), __uint_as_float(s[u][e + 3])), cc, make_float2(less.z, less.w));
                        s[u][e] = __float_as_uint(exp2_approx(f.x));
                        s[u][e + 1] = __float_as_uint(exp2_approx(f.y));
                        s[u][e + 2] = __float_as_uint(exp2_approx(g.x));
                        s[u][e + 3] = __float_as_uint(exp2_approx(g.y));
                    }
                if (a.causal && i % per == 0) {      // the tile on the diagonal: queries before the key do not see it
                    const int first = row - half * 64;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[u][e] = 32 * u + e >= first ? s[u][e] : 0u;
                }
                {
                    uint32_t p[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        p[e] = round_bf16x2(__uint_as_float(s[e / 16][2 * (e % 16)]), __uint_as_float(s[e / 16][2 * (e % 16) + 1]));
                    ptx::tmem_st_32x32(t_s, p);
                }
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_probs);
                ok = warp_wait(&s_stats[1], phase, abort_flag) && warp_wait(&s_grads, phase, abort_flag);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                uint32_t g[2][32];
                ptx::tmem_ld_32x32(t_g, g[0]);
                ptx::tmem_ld_32x32(t_g + 32, g[1]);
                ptx::tmem_ld_wait();
                ptx::tmem_ld_tie(g[0]);
                ptx::tmem_ld_tie(g[1]);
                uint32_t p[32];
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const float4 d = *reinterpret_cast<const float4*>(s_delta + half * 64 + 2 * e);
                    const uint32_t *u = &s[e / 16][2 * (e % 16)], *v = &g[e / 16][2 * (e % 16)];
                    const float2 x = mul2(make_float2(__uint_as_float(u[0]), __uint_as_float(u[1])),
                                          add2(make_float2(__uint_as_float(v[0]), __uint_as_float(v[1])), make_float2(d.x, d.y)));
                    const float2 y = mul2(make_float2(__uint_as_float(u[2]), __uint_as_float(u[3])),
                                          add2(make_float2(__uint_as_float(v[2]), __uint_as_float(v[3])), make_float2(d.z, d.w)));
                    p[e] = round_bf16x2(x.x, x.y);
                    p[e + 1] = round_bf16x2(y.x, y.y);
                }
                ptx::tmem_st_32x32(t_g, p);
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_ds);
            }
            if (!ok) break;
            if (n > 0) {
                ok = warp_wait(&s_done, d_phase, abort_flag);
                d_phase ^= 1u;
                if (!ok) break;
                ptx::tc_fence_after_sync();
            }
            if (half == 0) ab_store(tmem + 256 + lanes, a.dv.at<__nv_bfloat16>(t.b, t.first + me, h), 0, DP, a.d, 1.f, n > 0, valid, written);
            else ab_store(tmem + 384 + lanes, a.dk.at<__nv_bfloat16>(t.b, t.first + me, h), 0, DP, a.d, a.scale, n > 0, valid, written);
            ptx::tc_fence_before_sync();
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
