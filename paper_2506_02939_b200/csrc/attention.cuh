// Attention over the heads of the fused row [Q|K|V]: what its kernels share, and the kernels that take every type, size
// and order of memory.  With J(i) the valid tokens that token i sees (of its sequence; up to itself where causal):
//   s_ij = scale q_i k_j;  lse_i = log sum_{j in J(i)} exp(s_ij);  p_ij = exp(s_ij - lse_i);  o_i = sum_j p_ij v_j
//   delta_i = do_i o_i;  ds_ij = p_ij (do_i v_j - delta_i)
//   dq_i = scale sum_j ds_ij k_j;  dk_j = scale sum_i ds_ij q_i;  dv_j = sum_i p_ij do_i
// (dk and dv over all query heads that share the key head).  The backward pass makes p anew from lse.  It is two kernels,
// one that owns rows of queries (and writes delta) and one that owns rows of keys, so that every sum has one owner
// and a fixed order: 7 products of tiles where one kernel would do with 5, but would add to dq in the order of its blocks.
#pragma once
#include "pamm_common.cuh"
#include "row_io.cuh"

#include <algorithm>

namespace pamm {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int ATT_MAX_DIM = 256;

// Element (b, s, h, d) of a tensor lies at p + b batch + s token + h head + d.
struct HeadsView {
    void* p;
    int64_t batch, token, head;
    template <typename T>
    __device__ __forceinline__ T* at(int64_t b, int64_t s, int64_t h) const { return static_cast<T*>(p) + (b * batch + s * token + h * head); }
};

// The sequences: `batch` of `seq` tokens of which the first lengths[b] are valid (null: all), or, packed along one axis of `seq`
// tokens, `count` sequences between starts[i] and starts[i + 1].
struct Sequences {
    const void *lengths, *starts;
    int64_t seq;
    int batch, count;
    bool i64;
};
// A tile of one sequence: tokens first .. first + rows - 1 of batch entry b are written, the first `len` of them are valid.
struct Tile {
    int64_t b, first;
    int rows, len, at;              // `at`: the tile's first row within the sequence
    bool any;
};

__device__ __forceinline__ int64_t sequence_entry(const void* p, bool i64, int64_t i) {
    return i64 ? static_cast<const int64_t*>(p)[i] : (int64_t)static_cast<const int32_t*>(p)[i];
}
__device__ __forceinline__ int64_t clamped(int64_t v, int64_t lo, int64_t hi, bool& bad) {
    if (v < lo || v > hi) bad = true;
    return v < lo ? lo : v > hi ? hi : v;
}

// Tile number `item` of `size` rows; called by whole warps with the same item.  Packed: the axis falls into `count` + 2 pieces, what
// lies before the first and behind the last sequence among them (no token of those is valid: their outputs are zero).  Piece i starts
// with item bound(i) / size + i: between two neighbours there is room for every tile that the piece can have, and the piece of an
// item is found by a search with 32 probes a step, without a list of the pieces' tiles.
template <int SIZE>
__device__ __forceinline__ Tile find_tile(const Sequences& s, int item) {
    Tile t;
    bool bad = false;
    if (!s.starts) {
        const int per = (int)((s.seq + SIZE - 1) / SIZE);
        t.b = item / per;
        t.at = (int)(item - t.b * per) * SIZE;
        t.first = 0;
        t.rows = (int)s.seq;
        t.len = s.lengths ? (int)clamped(sequence_entry(s.lengths, s.i64, t.b), 0, s.seq, bad) : t.rows;
        t.any = true;
    } else {
        const int lane = threadIdx.x & 31;
        const auto bound = [&](int i) {
            return i == 0 ? 0 : i == s.count + 2 ? s.seq : clamped(sequence_entry(s.starts, s.i64, i - 1), 0, s.seq, bad);
        };
        int lo = 0, n = s.count + 2;
        while (n > 1) {
            const int step = (n + 31) / 32, probe = lo + lane * step;
            const bool before = lane * step < n && bound(probe) / SIZE + probe <= item;
            const uint32_t hits = __ballot_sync(0xffffffffu, before);
            const int last = hits ? 31 - __clz(hits) : 0;
            lo += last * step;
            n = min(step, n - last * step);
        }
        const int64_t begin = bound(lo), end = bound(lo + 1);
        // there are more items than pieces: each looks at one pair of entries, whether or not the search meets it
        if (item < s.count + 2 && bound(item + 1) < bound(item)) bad = true;
        t.b = 0;
        t.first = begin;
        t.rows = end > begin ? (int)(end - begin) : 0;
        t.len = lo >= 1 && lo <= s.count ? t.rows : 0;
        t.at = (item - (int)(begin / SIZE + lo)) * SIZE;
        t.any = t.at >= 0 && t.at < t.rows;
        bad = __any_sync(0xffffffffu, bad);
    }
    if (bad && (threadIdx.x & 31) == 0) raise_status(DEV_BAD_INDEX);
    return t;
}

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

struct AttentionArgs {
    HeadsView q, k, v, o, d_o, dq, dk, dv;
    const float* lse_in;
    float *lse, *delta;             // (batch, heads, seq) fp32, as the log-sums
    Sequences s;
    int heads, group, d;            // query heads; how many of them share a key head
    float scale;
    bool causal, vectors, wide;     // vectors: every row is on the 16-byte grid with whole vectors; wide: outputs on the 32-byte grid
    __device__ __forceinline__ int64_t row_number(const Tile& t, int h) const { return (t.b * heads + h) * s.seq + t.first; }
};

// ---- kernels for every type, size and order ---------------------------------------------------------------------
// Products in fp32 by fused multiply-adds: tiles of 32 x 64 scores, 16 a thread in 4 rows, whose operands come out of shared
// memory as vectors along the head (rows 4 words past a multiple of 32 apart: no bank conflicts).  They serve fp32, heads
// that are not multiples of 8 or wider than 128, and rows off the 16-byte grid.  Bound by multiply-adds and reads of shared memory, and
// by their latency where an SM's last blocks are alone.  8 x 256 tokens of 8 heads of 64, causal, in a CUDA graph: 29 us forward, 80 backward
// (through the Python entry 35 and 92); 31 and 87 with one multiply-add an instruction; 33 and 113 in blocks of 64 rows and 256 threads,
// 2 an SM and unevenly loaded.  The sizes of blocks and tiles were measured on that batch alone.
constexpr int AG_ROWS = 32, AG_TILE = 64, AG_THREADS = 4 * AG_ROWS, AG_P_LD = AG_TILE + 4;       // owned rows, streamed rows

// Whether the two streamed tiles have a place each, so that the one is on its way while the other is worked on.
template <int DP>
constexpr bool ag_split = DP <= 128;
// Owned tiles (Q, or two), streamed ones, P, and two numbers a streamed row.
template <int DP, bool BACK>
constexpr size_t ag_smem = (size_t)(((BACK ? 2 : 1) * AG_ROWS + (ag_split<DP> ? 2 : 1) * AG_TILE) * (DP + 4) + AG_ROWS * AG_P_LD + 2 * AG_TILE) * 4;

// 16 bytes to shared memory without passing through registers, or zeros.
__device__ __forceinline__ void ag_copy16(float* dst, const void* src, bool any) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(any ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ag_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void ag_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Rows `at` .. of the sequence into a tile, as one group of copies: rows from `valid` on and columns from d on are zero.  fp32 in vectors
// goes asynchronously; other forms are there when the call returns.
template <typename T, int DP, int ROWS>
__device__ __forceinline__ void ag_load(float* tile, const HeadsView& x, const Tile& t, int64_t head, int at, int valid, int d, bool vectors) {
    constexpr int V = 16 / (int)sizeof(T), LD = DP + 4, PER = DP / V, EACH = ROWS * PER / AG_THREADS;
    const T* base = x.at<T>(t.b, t.first + at, head);
    if (vectors) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int at_i = threadIdx.x + i * AG_THREADS, row = at_i / PER, col = (at_i % PER) * V;
                const bool any = at + row < valid && col < d;
                ag_copy16(tile + row * LD + col, any ? base + row * x.token + col : base, any);
            }
        } else {
            typename Piece<T, V>::Raw raw[EACH];       // all of a thread's loads are in flight before the first is waited for
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int at_i = threadIdx.x + i * AG_THREADS, row = at_i / PER, col = (at_i % PER) * V;
                raw[i] = Piece<T, V>::zero();
                if (at + row < valid && col < d) raw[i] = Piece<T, V>::load(base + row * x.token + col);
            }
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int at_i = threadIdx.x + i * AG_THREADS, row = at_i / PER, col = (at_i % PER) * V;
                float f[V];
                Piece<T, V>::unpack(raw[i], f);
#pragma unroll
                for (int e = 0; e < V; e += 4) *reinterpret_cast<float4*>(tile + row * LD + col + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
            }
        }
    } else {
#pragma unroll 4
        for (int i = threadIdx.x; i < ROWS * DP; i += AG_THREADS) {
            const int row = i / DP, col = i % DP;
            tile[row * LD + col] = at + row < valid && col < d ? to_float(base[row * x.token + col]) : 0.f;
        }
    }
    ag_commit();
}

// c[r][j] = row (4 ty + r) of A times row (tx + 16 j) of B
template <int DP>
__device__ __forceinline__ void ag_scores(const float* A, const float* B, int d, float (&c)[4][4]) {
    constexpr int LD = DP + 4;
    const float* a = A + (threadIdx.x / 16) * 4 * LD;
    const float* b = B + (threadIdx.x % 16) * LD;
    float2 sums[4][4];        // over even and odd columns: two multiply-adds an instruction
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[r][j] = twice(0.f);
#pragma unroll 2
    for (int e = 0; e < d; e += 4) {
        float4 x[4], y[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = *reinterpret_cast<const float4*>(a + r * LD + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(b + 16 * j * LD + e);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sums[r][j] = fma2(make_float2(x[r].z, x[r].w), make_float2(y[j].z, y[j].w), fma2(make_float2(x[r].x, x[r].y), make_float2(y[j].x, y[j].y), sums[r][j]));
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[r][j] = sums[r][j].x + sums[r][j].y;
}
// acc[r][.] += sum over the first `keys` entries of row (4 ty + r) of P times B's rows; a thread has columns 4 tx .. of every 64
template <int DP>
__device__ __forceinline__ void ag_accumulate(const float* P, const float* B, int keys, float (&acc)[4][DP / 16]) {
    constexpr int LD = DP + 4;
    const float* p = P + (threadIdx.x / 16) * 4 * AG_P_LD;
    const float* b = B + (threadIdx.x % 16) * 4;
#pragma unroll 2
    for (int j = 0; j < keys; j += 4) {
        float4 x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = *reinterpret_cast<const float4*>(p + r * AG_P_LD + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int c = 0; c < DP / 64; ++c) {
                const float4 y = *reinterpret_cast<const float4*>(b + (j + e) * LD + 64 * c);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float w = e == 0 ? x[r].x : e == 1 ? x[r].y : e == 2 ? x[r].z : x[r].w;
                    const float2 lo = fma2(twice(w), make_float2(y.x, y.y), make_float2(acc[r][4 * c], acc[r][4 * c + 1]));
                    const float2 hi = fma2(twice(w), make_float2(y.z, y.w), make_float2(acc[r][4 * c + 2], acc[r][4 * c + 3]));
                    acc[r][4 * c] = lo.x;
                    acc[r][4 * c + 1] = lo.y;
                    acc[r][4 * c + 2] = hi.x;
                    acc[r][4 * c + 3] = hi.y;
                }
            }
        }
    }
}
__device__ __forceinline__ void ag_store_scores(float* P, const float (&c)[4][4]) {
    float* p = P + (threadIdx.x / 16) * 4 * AG_P_LD + threadIdx.x % 16;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) p[r * AG_P_LD + 16 * j] = c[r][j];
}
// Rows of the tile times `factor` (per row), zero from the sequence's end on
template <typename T, int DP>
__device__ __forceinline__ void ag_store(const HeadsView& y, const Tile& t, int64_t head, int d, const float (&acc)[4][DP / 16], const float (&factor)[4]) {
    const int tx = threadIdx.x % 16, row0 = t.at + (threadIdx.x / 16) * 4;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (row0 + r >= t.rows) continue;
        T* p = y.at<T>(t.b, t.first + row0 + r, head);
        const bool valid = row0 + r < t.len;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            const int col = (c / 4) * 64 + tx * 4 + c % 4;
            if (col < d) p[col] = from_float<T>(valid ? acc[r][c] * factor[r] : 0.f);
        }
    }
}

// One block: AG_ROWS rows of one query head, over all tiles of keys with the running maximum and sum of the softmax.  Rows of P are written
// and read by the same half of a warp.
template <typename T, int DP>
__global__ void __launch_bounds__(AG_THREADS, DP <= 64 ? 4 : 2)
attention_forward_generic_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionOrder order) {
    constexpr bool SPLIT = ag_split<DP>;
    constexpr int OWNED = AG_ROWS * (DP + 4), TILE = AG_TILE * (DP + 4);
    extern __shared__ __align__(16) float ag_shared[];
    float *Q = ag_shared, *K = Q + OWNED, *V = SPLIT ? K + TILE : K, *P = V + TILE;
    grid_dependency_wait();
    grid_launch_dependents();
    int h, item;
    order.at((int)blockIdx.x, item, h);
    const Tile t = find_tile<AG_ROWS>(a.s, item);
    if (!t.any) return;
    const int tx = threadIdx.x % 16, row0 = t.at + (threadIdx.x / 16) * 4;
    const float c = a.scale * LOG2E;
    float acc[4][DP / 16], top[4], sum[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        top[r] = -INFINITY;
        sum[r] = 0.f;
#pragma unroll
        for (int e = 0; e < DP / 16; ++e) acc[r][e] = 0.f;
    }
    const int end = t.at < t.len ? (a.causal ? min(t.len, t.at + AG_ROWS) : t.len) : 0;
    const auto load = [&](float* to, const HeadsView& x, int k0) { ag_load<T, DP, AG_TILE>(to, x, t, h / a.group, k0, t.len, a.d, a.vectors); };
    if (end > 0) {
        ag_load<T, DP, AG_ROWS>(Q, a.q, t, h, t.at, t.len, a.d, a.vectors);
        load(K, a.k, 0);
        if (SPLIT) load(V, a.v, 0);
    }
    for (int k0 = 0; k0 < end; k0 += AG_TILE) {
        const bool more = k0 + AG_TILE < end;
        if (SPLIT) ag_wait<1>();
        else ag_wait<0>();
        __syncthreads();
        float s[4][4];
        ag_scores<DP>(Q, K, a.d, s);
        __syncthreads();
        if (!SPLIT) load(V, a.v, k0);
        else if (more) load(K, a.k, k0 + AG_TILE);
        else ag_commit();                                       // as many groups, so that V's is the last but one
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int last = a.causal ? min(row0 + r, t.len - 1) : t.len - 1;
            float m = top[r];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[r][j] = k0 + tx + 16 * j <= last ? s[r][j] : -INFINITY;
                m = fmaxf(m, s[r][j]);
            }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
            const float mc = m == -INFINITY ? 0.f : m * c;                   // a row that sees no finite score so far
            const float keep = exp2f(fmaf(top[r], c, -mc));
            sum[r] *= keep;
#pragma unroll
            for (int e = 0; e < DP / 16; ++e) acc[r][e] *= keep;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[r][j] = exp2f(fmaf(s[r][j], c, -mc));
                sum[r] += s[r][j];
            }
            top[r] = m;
        }
        ag_store_scores(P, s);
        if (SPLIT) ag_wait<1>();
        else ag_wait<0>();
        __syncthreads();
        ag_accumulate<DP>(P, V, min(AG_TILE, (end - k0 + 3) & ~3), acc);
        if (more) {
            __syncthreads();
            if (SPLIT) load(V, a.v, k0 + AG_TILE);
            else load(K, a.k, k0 + AG_TILE);
        }
    }
    float factor[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float l = sum[r];
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
        factor[r] = 1.f / l;
        if (tx == 0 && row0 + r < t.rows && a.lse)
            a.lse[a.row_number(t, h) + row0 + r] = row0 + r < t.len ? fmaf(top[r], a.scale, logf(l)) : -INFINITY;
    }
    ag_store<T, DP>(a.o, t, h, a.d, acc, factor);
}

// One block: AG_ROWS rows of the queries (KEYS false: A0 = Q, A1 = dO against X0 = K, X1 = V; dq, and delta on the way) or of the
// keys (A0 = K, A1 = V against X0 = Q, X1 = dO of every head of the group; dk and dv).
template <typename T, int DP, bool KEYS>
__global__ void __launch_bounds__(AG_THREADS, DP <= 64 ? 3 : DP <= 128 ? 2 : 1)
attention_backward_generic_kernel(const __grid_constant__ AttentionArgs a, const __grid_constant__ AttentionOrder order) {
    constexpr bool SPLIT = ag_split<DP>;
    constexpr int OWNED = AG_ROWS * (DP + 4), TILE = AG_TILE * (DP + 4);
    extern __shared__ __align__(16) float ag_shared[];
    float *A0 = ag_shared, *A1 = A0 + OWNED, *X0 = A1 + OWNED, *X1 = SPLIT ? X0 + TILE : X0, *P = X1 + TILE, *lse = P + AG_ROWS * AG_P_LD, *delta = lse + AG_TILE;
    grid_dependency_wait();
    grid_launch_dependents();
    int owner, item;                                          // query head or key head
    order.at((int)blockIdx.x, item, owner);
    const Tile t = find_tile<AG_ROWS>(a.s, item);
    if (!t.any) return;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16, row0 = t.at + ty * 4;
    const float c = a.scale * LOG2E;
    float acc0[4][DP / 16], acc1[4][KEYS ? DP / 16 : 1], row_lse[4], row_delta[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int e = 0; e < DP / 16; ++e) {
            acc0[r][e] = 0.f;
            if (KEYS) acc1[r][KEYS ? e : 0] = 0.f;
        }
    }
    // step i of n: tile i % per of the streamed rows, of head i / per of those that share the keys
    const int begin = KEYS && a.causal ? t.at : 0;
    const int end = t.at >= t.len ? begin : !KEYS && a.causal ? min(t.len, t.at + AG_ROWS) : t.len;
    const int per = (end - begin + AG_TILE - 1) / AG_TILE, n = per * (KEYS ? a.group : 1);
    const auto head_of = [&](int i) { return KEYS ? owner * a.group + i / per : owner / a.group; };
    const auto at_of = [&](int i) { return begin + i % per * AG_TILE; };
    const auto load0 = [&](int i) { ag_load<T, DP, AG_TILE>(X0, KEYS ? a.q : a.k, t, head_of(i), at_of(i), t.len, a.d, a.vectors); };
    const auto load1 = [&](int i) { ag_load<T, DP, AG_TILE>(X1, KEYS ? a.d_o : a.v, t, head_of(i), at_of(i), t.len, a.d, a.vectors); };
    float next_lse = 0.f, next_delta = 0.f;                   // of the next step's columns, on their way
    const auto numbers = [&](int i) {
        const int row = at_of(i) + (int)threadIdx.x;
        if (!KEYS || threadIdx.x >= AG_TILE) return;
        const int64_t number = a.row_number(t, head_of(i)) + row;
        next_lse = row < t.len ? a.lse_in[number] * LOG2E : 0.f;
        next_delta = row < t.len ? a.delta[number] : 0.f;
    };
    if (n > 0) {
        ag_load<T, DP, AG_ROWS>(A0, KEYS ? a.k : a.q, t, owner, t.at, t.len, a.d, a.vectors);
        ag_load<T, DP, AG_ROWS>(A1, KEYS ? a.v : a.d_o, t, owner, t.at, t.len, a.d, a.vectors);
        numbers(0);
        load0(0);
        if (SPLIT) load1(0);
    }
    if (!KEYS) {
        const int64_t number = a.row_number(t, owner);
        if (SPLIT) ag_wait<2>();
        else ag_wait<1>();
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float sum = 0.f;
            if (row0 + r < t.len) {
                const T* o = a.o.at<T>(t.b, t.first + row0 + r, owner);
                for (int e = tx; e < a.d; e += 16) sum = fmaf(to_float(o[e]), A1[(ty * 4 + r) * (DP + 4) + e], sum);
            }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            row_delta[r] = sum;
            row_lse[r] = row0 + r < t.len ? a.lse_in[number + row0 + r] * LOG2E : 0.f;
            if (tx == 0 && row0 + r < t.rows) a.delta[number + row0 + r] = sum;
        }
    }
    for (int i = 0; i < n; ++i) {
        const bool more = i + 1 < n;
        const int x0 = at_of(i);
        if (KEYS && threadIdx.x < AG_TILE) {
            lse[threadIdx.x] = next_lse;
            delta[threadIdx.x] = next_delta;
        }
        if (SPLIT) ag_wait<1>();
        else ag_wait<0>();
        __syncthreads();
        if (more) numbers(i + 1);
        float p[4][4], dp[4][4];
        ag_scores<DP>(A0, X0, a.d, p);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = row0 + r, col = x0 + tx + 16 * j;
                const bool sees = col < t.len && (!a.causal || (KEYS ? col >= row : col <= row));
                p[r][j] = sees ? exp2f(fmaf(p[r][j], c, -(KEYS ? lse[tx + 16 * j] : row_lse[r]))) : 0.f;
            }
        if (!SPLIT) {
            __syncthreads();
            load1(i);
        }
        ag_wait<0>();
        __syncthreads();
        ag_scores<DP>(A1, X1, a.d, dp);
        const int used = min(AG_TILE, (end - x0 + 3) & ~3);
        if constexpr (KEYS) {
            ag_store_scores(P, p);
            __syncwarp();
            ag_accumulate<DP>(P, X1, used, acc1);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j)      // a masked place stays 0 whatever dp is there
                p[r][j] = p[r][j] == 0.f ? 0.f : p[r][j] * (dp[r][j] - (KEYS ? delta[tx + 16 * j] : row_delta[r]));
        if (!SPLIT) {
            __syncthreads();
            load0(i);
            ag_wait<0>();
            __syncthreads();
        }
        __syncwarp();
        ag_store_scores(P, p);
        __syncwarp();
        ag_accumulate<DP>(P, X0, used, acc0);
        if (more) {
            __syncthreads();
            load0(i + 1);
            if (SPLIT) load1(i + 1);
        }
    }
    const float factor[4] = {a.scale, a.scale, a.scale, a.scale}, one[4] = {1.f, 1.f, 1.f, 1.f};
    ag_store<T, DP>(KEYS ? a.dk : a.dq, t, owner, a.d, acc0, factor);
    if constexpr (KEYS) ag_store<T, DP>(a.dv, t, owner, a.d, acc1, one);
}

}  // namespace pamm
