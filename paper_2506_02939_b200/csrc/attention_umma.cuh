// Attention on the tensor cores: bf16 heads of up to 128 (a multiple of 8), rows on the 16-byte grid.  This file: the parts that the
// three kernels share, and the forward pass.
//
// A tile is 128 tokens of one head in shared memory, as one or two blocks of 64 columns (TMA boxes with the 128-byte
// swizzle; columns from d on are filled with zeros).  The same tile is a K-major operand (rows against rows: scores) and an MN-major one
// (weights against rows: outputs and gradients), so nothing is ever transposed.
#pragma once
#include "attention.cuh"
#include "sm100_ptx.cuh"

namespace pamm {

constexpr int AU_ROWS = 128, AU_BLOCK_BYTES = AU_ROWS * 128;       // of a tile, and of 64 of its columns

// The 16 warps of a block: eight own rows of scores, four take accumulators out of tensor memory (a warp reaches the 32
// lanes of its number modulo 4 only), one copies tiles in, one or two issue products, one brings
// numbers of rows (backward, keys) and one finds the next items.  A thread's wait gets its answer only when the thread's own
// products before it have been taken by the tensor cores (165 clocks a wait that is long over, where products follow
// each other without a gap otherwise); where products wait for different warps, a second thread's fill that time.
// Registers: 128 a thread at the launch; the rows' warps take what the others give back.
constexpr int AU_THREADS = 512, AU_FINISH_WARP = 8, AU_TMA_WARP = 12, AU_MMA_WARP = 13, AU_ITEMS_WARP = 15;
constexpr int AU_ROW_REGS = 168, AU_OTHER_REGS = 88;
static_assert(256 * AU_ROW_REGS + 256 * AU_OTHER_REGS <= 65536, "what is taken has to have been given back");

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
// A wait for another warp's whole item lasts as long as the item, which grows with the context: a tile of keys meets (tokens / 128) x
// (query heads that share it) steps of 1.4 us.  So polls are counted from the block's last sign of progress on: a tile that is on its way,
// or an item that has been looked at.  Both come to an end with the work, so every wait does.  (2^22 polls of 4 us: 17 seconds without one.)
struct Watch {
    int abort;                      // set by a wait that ran out
    uint32_t tiles, items;          // written by the warp that copies, and by the one that finds the items
};
__device__ __forceinline__ bool au_wait(uint64_t* bar, uint32_t parity, volatile Watch* watch, uint32_t polls = ptx::WAIT_POLLS) {
    uint32_t seen = 0;
    for (uint32_t it = 0; it < polls; ++it) {
        if (ptx::mbar_try_wait(bar, parity)) return true;
        if ((it & 63u) == 63u) {
            if (watch->abort) return false;
            const uint32_t now = watch->tiles + watch->items;
            if (now != seen) { seen = now; it = 0; }
            __nanosleep(64);
        }
    }
    watch->abort = 1;
    return false;
}
// A wait of a whole warp: the same answer in every lane.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile Watch* watch, uint32_t polls = ptx::WAIT_POLLS) {
    return __all_sync(0xffffffffu, au_wait(bar, parity, watch, polls));
}
// The block's items, found ahead by one warp and read by all others (`readers` warps: each gives an entry back as soon as it has it in
// registers).  An entry with rows < 0 is the end.  Every item has a block in the grid; a block that is through with its own takes over
// the next one that has not started, so that no block is left with more than the others whatever the sequences' lengths are.
constexpr int AU_ITEMS = 2;
struct Item { Tile t; int head; };
struct ItemQueue {
    uint4 response;
    Item items[AU_ITEMS];
    uint64_t full[AU_ITEMS], empty[AU_ITEMS], answered;
    __device__ __forceinline__ void init(int readers) {
        for (int i = 0; i < AU_ITEMS; ++i) { ptx::mbar_init(&full[i], 1); ptx::mbar_init(&empty[i], readers); }
        ptx::mbar_init(&answered, 1);
    }
};
struct ItemReader {
    ItemQueue* q;
    volatile Watch* watch;
    uint32_t count = 0;
    // False at the end and where a wait ran out (`ok`).
    __device__ __forceinline__ bool next(Item& item, bool& ok) {
        const uint32_t slot = count % AU_ITEMS;
        if (!warp_wait(&q->full[slot], (count / AU_ITEMS) & 1u, watch)) { ok = false; return false; }
        item = q->items[slot];
        __syncwarp();
        if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(&q->empty[slot]);
        ++count;
        return item.t.rows >= 0;
    }
    // The same for a thread that reads for its warp.
    __device__ __forceinline__ bool next_alone(Item& item, bool& ok) {
        const uint32_t slot = count % AU_ITEMS;
        if (!au_wait(&q->full[slot], (count / AU_ITEMS) & 1u, watch)) { ok = false; return false; }
        item = q->items[slot];
        ptx::mbar_arrive(&q->empty[slot]);
        ++count;
        return item.t.rows >= 0;
    }
};
// The warp that finds them.  `steps` says how long an item takes: behind one of a few steps the next is taken at once, so that its tiles
// come in time; behind a longer one when that has begun, so that no block holds work that another could start on.
// Items without a valid row are not handed on: this warp writes their zeros itself (`clear`).  So every item that is has at least a
// step, and a reader that looks two steps ahead never needs more than two items ahead -- no more than the queue holds while another
// reader waits for what the first one does with its present item.
template <int SIZE, typename F, typename G>
__device__ __forceinline__ bool au_find_items(ItemQueue& q, const Sequences& s, const AttentionOrder& order, volatile Watch* watch, F steps, G clear) {
    uint32_t count = 0, phase = 0, looked = 0;
    int w = (int)blockIdx.x;
    while (true) {
        ++looked;
        if ((threadIdx.x & 31) == 0) watch->items = looked;
        Item item;
        item.t.rows = -1;
        if (w >= 0) {
            int number;
            order.at(w, number, item.head);
            item.t = find_tile<SIZE>(s, number);
        }
        if (w >= 0 && item.t.any && item.t.at >= item.t.len) {
            clear(item);
            __syncwarp();
        } else if (w < 0 || item.t.any) {
            const uint32_t slot = count % AU_ITEMS;
            if (!warp_wait(&q.empty[slot], ((count / AU_ITEMS) & 1u) ^ 1u, watch)) return false;
            if ((threadIdx.x & 31) == 0) {
                q.items[slot] = item;
                ptx::mbar_arrive(&q.full[slot]);
            }
            __syncwarp();
            if (w < 0) return true;
            if (steps(item.t) >= 4 && !warp_wait(&q.empty[slot], (count / AU_ITEMS) & 1u, watch)) return false;
            ++count;
        }
        if ((threadIdx.x & 31) == 0) {
            ptx::fence_proxy_async();          // the last answer has been read
            ptx::mbar_arrive_expect_tx(&q.answered, 16);
            ptx::take_next_block(&q.response, &q.answered);
        }
        __syncwarp();
        if (!warp_wait(&q.answered, phase, watch)) {       // the answer lands before the block's memory is given back
            int never = 0;
            ptx::mbar_wait(&q.answered, phase, &never, 1u << 14);
            return false;
        }
        phase ^= 1u;
        w = ptx::taken_block(&q.response);
        __syncwarp();
    }
}
// Zeros in the rows of an item from `at` on, at most `size` of them.  A whole warp, whose stores follow each other in memory.
__device__ __forceinline__ void au_clear(const HeadsView& y, const Item& item, int size, int d) {
    const int pieces = d / 8, end = min(size, item.t.rows - item.t.at) * pieces;
    __nv_bfloat16* p = y.at<__nv_bfloat16>(item.t.b, item.t.first + item.t.at, item.head);
    for (int i = threadIdx.x & 31; i < end; i += 32) {
        const int r = i / pieces;
        st16(p + r * y.token + (i - r * pieces) * 8, make_uint4(0, 0, 0, 0));
    }
}
// The producer's ring of tiles.  Called by the whole warp.
struct TileRing {
    uint8_t* tiles;
    uint64_t *full, *empty, *tail;       // tail: for a tile whose last rows are cleared before it is handed on
    volatile Watch* watch;
    int slots, slot;
    uint32_t phase, tail_phase, used;
    bool tail_open;
    __device__ __forceinline__ void next() {
        if (++slot == slots) { slot = 0; phase ^= 1u; }
        ++used;
        if ((threadIdx.x & 31) == 0) watch->tiles = used;
    }
};
// The next tile of the ring.  `clear`: rows from the sequence's end on are set to zero, because a product with a weight of 0 would keep
// their NaN or infinity; needed where the tensor goes on behind the end.
template <int DP>
__device__ __forceinline__ bool au_produce(TileRing& r, const CUtensorMap* tm, const Tile& t, int head, int at, bool clear) {
    if (!warp_wait(&r.empty[r.slot], r.phase ^ 1u, r.watch)) return false;
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
        if (!warp_wait(r.tail, r.tail_phase, r.watch)) return false;
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
// The same for the products of the thread that issued them: they end before the memory of their operands and sums is given back.
__device__ __forceinline__ void au_settle(uint64_t* last) {
    int never = 0;
    ptx::umma_commit(last);
    ptx::mbar_wait(last, 0, &never, 1u << 14);
}

// The products.  One thread.  A product is issued only shortly before it runs, so what this thread computes between two of them counts.
// D = A B^T over the heads' columns, both tiles K-major: steps of 16 columns.  (N, and from which row of B on, is the caller's.)
template <int DP>
__device__ __forceinline__ void au_scores(uint32_t d_tmem, uint32_t a, uint32_t b, int steps, uint32_t idesc) {
    const uint32_t la = ptx::umma_desc_lower_k(a), lb = ptx::umma_desc_lower_k(b);
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const uint32_t off = (uint32_t)((k >> 2) * (AU_BLOCK_BYTES >> 4) + (k & 3) * 2);
        if (k < steps) ptx::umma_bf16_lower(d_tmem, la + off, lb + off, idesc, k > 0);
    }
}
// D (+)= W B over half of B's 128 rows: W bf16 in tensor memory, its two halves 64 columns apart (each over the scores it came
// from), B MN-major.
__device__ __forceinline__ void au_weighted_half(uint32_t d_tmem, uint32_t w_tmem, uint32_t b, int half, uint32_t idesc, bool accumulate) {
    const uint32_t lb = ptx::umma_desc_lower_mn(b, AU_BLOCK_BYTES) + half * (4 * 2048 >> 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) ptx::umma_bf16_ts(d_tmem, w_tmem + half * 64 + k * 8, lb + k * (2048 >> 4), idesc, accumulate || k > 0);
}
__device__ __forceinline__ void au_weighted(uint32_t d_tmem, uint32_t w_tmem, uint32_t b, uint32_t idesc, bool accumulate) {
    au_weighted_half(d_tmem, w_tmem, b, 0, idesc, accumulate);
    au_weighted_half(d_tmem, w_tmem, b, 1, idesc, true);
}
// A row's accumulator times `factor` to memory (zero where the token is not valid).  `loaded`: there is one.  A whole warp, one row a
// thread: a store of 32 bytes a row costs the memory pipe as much as one of 16.  `free`: arrived on once the accumulator is read.
__device__ __forceinline__ void st32(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]),
                 "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void au_store(uint32_t t_acc, __nv_bfloat16* out, int d, float factor, bool loaded, bool valid, bool written, bool wide, uint64_t* free) {
#pragma unroll 1
    for (int i = 0; i < d; i += 32) {
        uint32_t o[32];
        if (loaded) {
            ptx::tmem_ld_32x32(t_acc + i, o);
            ptx::tmem_ld_wait();
            ptx::tmem_ld_tie(o);
            if (i + 32 >= d) {
                ptx::tc_fence_before_sync();
                __syncwarp();
                if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(free);
            }
        }
#pragma unroll
        for (int e = 0; e < 32; e += 16) {
            uint32_t v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                v[u] = valid ? round_bf16x2(__uint_as_float(o[e + 2 * u]) * factor, __uint_as_float(o[e + 2 * u + 1]) * factor) : 0u;
            if (written && i + e < d) {
                if (wide) {
                    st32(out + i + e, v);
                } else {
                    st16(out + i + e, make_uint4(v[0], v[1], v[2], v[3]));
                    if (i + e + 8 < d) st16(out + i + e + 8, make_uint4(v[4], v[5], v[6], v[7]));
                }
            }
        }
    }
}

struct AttentionMaps { CUtensorMap q, k, v, d_o; };
inline bool attention_map(CUtensorMap* tm, const HeadsView& t, const Sequences& s, int64_t heads, int d) {
    const auto ld = [](int64_t v) { return (uint64_t)(v > 0 ? v : 8); };      // of a dimension with one entry: any multiple of 16 bytes
    return make_tmap_heads_sw128(tm, t.p, (uint64_t)d, (uint64_t)heads, (uint64_t)s.seq, (uint64_t)s.batch, ld(t.head), ld(t.token), ld(t.batch), AU_ROWS);
}

// ---- forward ------------------------------------------------------------------------------------------------------------
// A block works on 256 rows of one query head at a time: two tiles, each with four warps whose threads own a row and one thread that
// issues its products.  Per 64 keys: S = Q K^T into tensor memory; the row's thread takes its 64 scores and their exponentials
// and puts P back as bf16 over S; O += P V with P as the operand in tensor memory.  Two such halves of a tile of keys are under way
// at a time, so that the scores of the one come while the exponentials of the other are taken.  (Whole tiles, S of 128 columns: the
// chain from P to the next scores, 1500 clocks, was exposed, 4000 clocks for both query tiles against 2900 that
// products of 64 columns take, whose other operand is read from shared memory more often.)
// The exponentials are taken from a reference that the row's maximum had before, without waiting for the new one; where that has risen
// by more than 2^8, O and the sum l are scaled down and the half is taken again (exact: O and l share the reference, and p <= 2^8
// keeps its relative rounding).  The rounding of P to bf16 is the operand's; l is taken before it.
// An item's first scores follow the last product of the item before, and O leaves through warps of its own.
// (Exponentials on the multiply-add units, one pair of four, of eight: 2 to 5% slower; the special-function unit is half busy.)
constexpr int AF_QUERIES = 2 * AU_ROWS;
constexpr float AF_RISE = 8.f;

template <int DP>
struct AttentionPlan {
    static constexpr int TILE_BYTES = DP / 64 * AU_BLOCK_BYTES;
    static constexpr int SLOTS = DP == 128 ? 5 : 8;
    static constexpr size_t SMEM = 1024 + (size_t)(2 + SLOTS) * TILE_BYTES;        // two fixed tiles and the ring
};

// Groups of `size` keys that query tile x of the item meets, and tiles of them.
__device__ __forceinline__ int au_key_groups(const Tile& t, bool causal, int x, int size) {
    const int at = t.at + x * AU_ROWS;
    if (at >= t.len) return 0;
    const int end = causal ? min(t.len, at + AU_ROWS) : t.len;
    return (end + size - 1) / size;
}
__device__ __forceinline__ int au_key_tiles(const Tile& t, bool causal, int x) { return au_key_groups(t, causal, x, AU_ROWS); }
__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
// The maximum of 32 scores and x; NaN are passed over.
__device__ __forceinline__ float max_of(const uint32_t (&s)[32], float x) {
    float a = __uint_as_float(s[0]), b = x;
#pragma unroll
    for (int e = 1; e + 3 < 32; e += 4) {
        a = max3(a, __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
        b = max3(b, __uint_as_float(s[e + 2]), __uint_as_float(s[e + 3]));
    }
    return fmaxf(max3(a, __uint_as_float(s[29]), __uint_as_float(s[30])), fmaxf(b, __uint_as_float(s[31])));
}
__device__ __forceinline__ void mask_behind(uint32_t (&s)[32], int limit, uint32_t value) {      // entries behind `limit`
#pragma unroll
    for (int e = 0; e < 32; ++e) s[e] = e <= limit ? s[e] : value;
}

template <int DP>
__global__ void __launch_bounds__(AU_THREADS, 1)
attention_forward_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionMaps m, const __grid_constant__ AttentionOrder order) {
    using Plan = AttentionPlan<DP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) ItemQueue s_queue;
    __shared__ uint64_t s_full[Plan::SLOTS], s_empty[Plan::SLOTS], s_qfull[2], s_qempty[2], s_scores[2][2], s_probs[2][2], s_added[2], s_done[2], s_sums[2], s_free[2], s_tail, s_last[2];
    __shared__ float s_sum[2][AU_ROWS];
    __shared__ uint32_t s_tmem;
    __shared__ Watch s_watch;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* queries = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring_tiles = queries + 2 * Plan::TILE_BYTES;
    if (threadIdx.x == 0) {
        s_queue.init(15);
        for (int i = 0; i < Plan::SLOTS; ++i) { ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&s_empty[i], 2); }
        for (int x = 0; x < 2; ++x) {
            ptx::mbar_init(&s_qfull[x], 1);
            ptx::mbar_init(&s_qempty[x], 1);
            for (int half = 0; half < 2; ++half) {
                ptx::mbar_init(&s_scores[x][half], 1);
                ptx::mbar_init(&s_probs[x][half], 4);
            }
            ptx::mbar_init(&s_added[x], 1);
            ptx::mbar_init(&s_done[x], 1);
            ptx::mbar_init(&s_sums[x], 4);
            ptx::mbar_init(&s_free[x], 4);
            ptx::mbar_init(&s_last[x], 1);
        }
        ptx::mbar_init(&s_tail, 1);
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
            ok = au_find_items<AF_QUERIES>(s_queue, a.s, order, watch, [&](const Tile& t) { return au_key_tiles(t, a.causal, 0); }, [&](const Item& it) {
                au_clear(a.o, it, AF_QUERIES, a.d);
                for (int r = it.t.at + lane; a.lse && r < min(it.t.at + AF_QUERIES, it.t.rows); r += 32) a.lse[a.row_number(it.t, it.head) + r] = -INFINITY;
            });
        } else if (warp == AU_TMA_WARP) {
            TileRing ring = {ring_tiles, s_full, s_empty, &s_tail, watch, Plan::SLOTS, 0, 0, 0, 0, false};
            uint32_t q_phase[2] = {0, 0};
            while (reader.next(item, ok)) {
                const Tile& t = item.t;
                const int n0 = au_key_tiles(t, a.causal, 0), n1 = au_key_tiles(t, a.causal, 1), n = max(n0, n1), hk = item.head / a.group;
                const bool clear = t.first + t.len < a.s.seq;
                // the second tile's queries come behind the first keys: their place is free later
                for (int j = 0; j < n && ok; ++j) {
                    for (int x = 0; x < 2 && ok; ++x) {
                        if (j == 0 && (x ? n1 : n0) > 0) {
                            ok = warp_wait(&s_qempty[x], q_phase[x] ^ 1u, watch);
                            if (!ok) break;
                            q_phase[x] ^= 1u;
                            if (ptx::elect_one()) {
                                ptx::mbar_arrive_expect_tx(&s_qfull[x], Plan::TILE_BYTES);
                                au_load<DP>(queries + x * Plan::TILE_BYTES, &m.q, t, item.head, t.at + x * AU_ROWS, &s_qfull[x]);
                            }
                            __syncwarp();
                        }
                        ok = x == 0 ? au_produce<DP>(ring, &m.k, t, hk, j * AU_ROWS, false) : au_produce<DP>(ring, &m.v, t, hk, j * AU_ROWS, clear);
                    }
                }
                if (!ok) break;
            }
            if (!ok) {
                au_drain(ring);
                int never = 0;
                for (int x = 0; x < 2; ++x) ptx::mbar_wait(&s_qfull[x], q_phase[x] ^ 1u, &never, 1u << 14);
            }
        } else if (ptx::elect_one()) {
            // The products of tile x.  Both threads go through all ring tiles, so that each tile is given back twice.
            const int x = warp - AU_MMA_WARP;
            const uint32_t idesc_s = ptx::umma_idesc_bf16(AU_ROWS, 64);
            const uint32_t idesc_o = ptx::umma_idesc_bf16(AU_ROWS, (uint32_t)((a.d + 15) / 16 * 16)) | (1u << 16);      // B MN-major
            const int steps = (a.d + 15) / 16;
            const uint32_t q_addr = ptx::smem_u32(queries) + x * Plan::TILE_BYTES, ring_addr = ptx::smem_u32(ring_tiles);
            const uint32_t t_s = tmem + x * 128, t_o = tmem + 256 + x * 128;
            uint32_t q_phase = 0, p_phase = 0, f_phase = 1, base = 0;        // p_phase: bit `half`; base: ring tiles before the item
            const auto wait = [&](uint64_t& bar, uint32_t parity) { return au_wait(&bar, parity & 1u, watch); };
            while (reader.next_alone(item, ok)) {
                const int n = max(au_key_tiles(item.t, a.causal, 0), au_key_tiles(item.t, a.causal, 1)), mine = au_key_groups(item.t, a.causal, x, 64);
                if (mine > 0) {
                    if (!(ok = wait(s_qfull[x], q_phase))) break;
                    q_phase ^= 1u;
                }
                // step i: O += P V of group i, then the scores of group i + 2, which take its place
#pragma unroll 1
                for (int i = -2; i < mine; ++i) {
                    const int half = i & 1, next = i + 2;
                    // what is there long before is waited for first, so that nothing stands between P's arrival and the products
                    const uint32_t v_tile = base + (i | 1), v_slot = v_tile % Plan::SLOTS, k_tile = base + (next & ~1), k_slot = k_tile % Plan::SLOTS;
                    if (next < mine && !half && !(ok = wait(s_full[k_slot], k_tile / Plan::SLOTS))) break;
                    if (i >= 0) {
                        if (!half && !(ok = wait(s_full[v_slot], v_tile / Plan::SLOTS))) break;
                        if (i == 0) {
                            if (!(ok = wait(s_free[x], f_phase))) break;
                            f_phase ^= 1u;
                        }
                        if (!(ok = wait(s_probs[x][half], p_phase >> half))) break;
                        p_phase ^= 1u << half;
                        ptx::tc_fence_after_sync();
                        au_weighted_half(t_o, t_s, ring_addr + v_slot * Plan::TILE_BYTES, half, idesc_o, i > 0);
                        ptx::umma_commit(&s_added[x]);
                        if (half || i == mine - 1) ptx::umma_commit(&s_empty[v_slot]);
                        if (i == mine - 1) ptx::umma_commit(&s_done[x]);
                    }
                    if (next < mine) {
                        ptx::tc_fence_after_sync();
                        au_scores<DP>(t_s + 64 * half, q_addr, ring_addr + k_slot * Plan::TILE_BYTES + half * 64 * 128, steps, idesc_s);
                        ptx::umma_commit(&s_scores[x][half]);
                        if (half || next == mine - 1) ptx::umma_commit(&s_empty[k_slot]);
                        if (next == mine - 1) ptx::umma_commit(&s_qempty[x]);
                    }
                }
                if (!ok) break;
                for (uint32_t tile = base + (uint32_t)((mine + 1) & ~1); tile < base + 2 * n; ++tile) {      // tiles of the other's only
                    const uint32_t slot = tile % Plan::SLOTS;
                    if (!(ok = wait(s_full[slot], tile / Plan::SLOTS))) break;
                    ptx::mbar_arrive(&s_empty[slot]);
                }
                if (!ok) break;
                base += 2 * n;
            }
            if (!ok) au_settle(&s_last[x]);
        }
    } else if (warp >= AU_FINISH_WARP) {
        ptx::registers_down<AU_OTHER_REGS>();
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = ((uint32_t)(warp & 3) * 32) << 16;
        uint32_t phase[2] = {0, 0};
        while (reader.next(item, ok)) {
            const Tile& t = item.t;
            for (int x = 0; x < 2 && ok; ++x) {
                const int me = t.at + x * AU_ROWS + row, n = au_key_tiles(t, a.causal, x);
                if (t.at + x * AU_ROWS >= t.rows) continue;
                float sum = 1.f;
                if (n > 0) {
                    ok = warp_wait(&s_sums[x], phase[x], watch) && warp_wait(&s_done[x], phase[x], watch);
                    phase[x] ^= 1u;
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
                    sum = s_sum[x][row];
                }
                const bool valid = me < t.len, written = me < t.rows;
                au_store(tmem + 256 + x * 128 + lanes, a.o.at<__nv_bfloat16>(t.b, t.first + me, item.head), a.d, 1.f / sum, n > 0, valid, written, a.wide, &s_free[x]);
            }
            if (!ok) break;
        }
    } else {
        ptx::registers_up<AU_ROW_REGS>();
        const int x = warp >> 2;
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = ((uint32_t)(warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + x * 128 + lanes, t_o = tmem + 256 + x * 128 + lanes;
        const float c = a.scale * LOG2E;
        uint32_t s_phase = 0, f_phase = 1, total = 0;      // s_phase: bit `half`; total: groups so far
        while (reader.next(item, ok)) {
            const Tile& t = item.t;
            const int n = au_key_groups(t, a.causal, x, 64), me = t.at + x * AU_ROWS + row;
            const int last = a.causal ? min(me, t.len - 1) : t.len - 1;       // the last key that the row sees
            float top = -INFINITY, sum = 0.f;
#pragma unroll 1
            for (int g = 0; g < n; ++g, ++total) {
                const int half = g & 1;
                const uint32_t t_g = t_s + 64 * half;
                ok = warp_wait(&s_scores[x][half], s_phase >> half & 1u, watch);
                if (!ok) break;
                s_phase ^= 1u << half;
                ptx::tc_fence_after_sync();
                uint32_t s[2][32];
                ptx::tmem_ld_32x32(t_g, s[0]);
                ptx::tmem_ld_32x32(t_g + 32, s[1]);
                ptx::tmem_ld_wait();
                ptx::tmem_ld_tie(s[0]);
                ptx::tmem_ld_tie(s[1]);
                const int limit = last - g * 64;
                if (__any_sync(0xffffffffu, limit < 63)) {
                    mask_behind(s[0], limit, 0xFF800000u);
                    mask_behind(s[1], limit - 32, 0xFF800000u);
                }
                if (g == 0) top = fmaxf(max_of(s[0], top), max_of(s[1], top));
                float2 part[2];
                uint32_t p[32];
#pragma unroll 1
                for (int pass = 0;; ++pass) {
                    const float less = top == -INFINITY ? 0.f : -top * c;         // or the row has seen no finite score
                    part[0] = part[1] = twice(0.f);
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const uint32_t* from = &s[e / 16][2 * (e % 16)];
                        const float2 y = make_float2(exp2_approx(fmaf(__uint_as_float(from[0]), c, less)), exp2_approx(fmaf(__uint_as_float(from[1]), c, less)));
                        part[e & 1] = add2(part[e & 1], y);
                        p[e] = round_bf16x2(y.x, y.y);
                    }
                    if (g == 0 || pass > 0) break;
                    const float seen = fmaxf(max_of(s[0], top), max_of(s[1], top));
                    const bool rises = (seen - top) * c > AF_RISE;       // each row for itself: its result does not depend on its neighbours
                    if (!__any_sync(0xffffffffu, rises)) break;
                    // O is at rest once the last product handed over has been added to it
                    ok = warp_wait(&s_added[x], total - 1 & 1u, watch);
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
                    const float keep = rises ? exp2_approx((top - seen) * c) : 1.f;
                    if (rises) top = seen;
                    sum *= keep;
#pragma unroll 1
                    for (int i = 0; i < DP; i += 8) {
                        uint32_t o[8];
                        ptx::tmem_ld_32x8(t_o + i, o);
                        ptx::tmem_ld_wait(o);
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                        ptx::tmem_st_32x8(t_o + i, o);
                    }
                }
                if (!ok) break;
                ptx::tmem_st_32x32(t_g, p);
                sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
                ptx::tmem_st_wait();
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_probs[x][half]);
            }
            if (!ok) break;
            if (a.lse && me < t.rows) a.lse[a.row_number(t, item.head) + me] = me < t.len ? fmaf(top, a.scale, logf(sum)) : -INFINITY;
            if (n > 0) {
                ok = warp_wait(&s_free[x], f_phase, watch);       // the item before has left, and its sums have been read
                if (!ok) break;
                f_phase ^= 1u;
                s_sum[x][row] = sum;
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&s_sums[x]);
            }
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
