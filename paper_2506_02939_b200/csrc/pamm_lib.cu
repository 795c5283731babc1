// C ABI of the PAMM sm_100a library: argument checks, kernel selection, launches.
// Every step of the path runs in the kernels included below; nothing here
// computes on the host apart from pamm_draw_indices_host.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <map>
#include <tuple>
#include <mutex>
#include <utility>
#include <vector>

#include "pamm_common.cuh"
#include "select.cuh"
#include "compress_simt.cuh"
#include "compress_umma.cuh"
#include "contract.cuh"
#include "contract_stream.cuh"
#include "weight_grad_simt.cuh"
#include "weight_grad_persist.cuh"
#include "weight_grad_chunked.cuh"
#include "weight_grad_planes.cuh"
#include "compress_pair.cuh"
#include "linear_forward.cuh"
#include "linear_forward_pair.cuh"
#include "small_k.cuh"
#include "read_probe.cuh"
#include "norm.cuh"
#include "rotary.cuh"
#include "grad_clip.cuh"
#include "attention.cuh"
#include "attention_umma.cuh"
#include "attention_umma_backward.cuh"
#include "dropout.cuh"

using namespace pamm;

namespace pamm {
static thread_local char g_cuda_detail[256] = "";
void note_cuda_failure(const char* what, cudaError_t err) {
    snprintf(g_cuda_detail, sizeof g_cuda_detail, "%s: %s (%s)", what, cudaGetErrorName(err), cudaGetErrorString(err));
}

pamm_status tensor_map_failed() {
    const TmapFailure& f = last_tmap_failure();
    snprintf(g_cuda_detail, sizeof g_cuda_detail,
             "cuTensorMapEncodeTiled failed (CUresult %d; no driver entry point if 0) for a %llu x %llu matrix of %u-byte elements "
             "at %p, leading dimension %llu, boxes of %u rows",
             f.result, (unsigned long long)f.rows, (unsigned long long)f.cols, f.elem_bytes, f.base, (unsigned long long)f.ld,
             f.box_rows);
    return PAMM_ERR_CUDA;
}

bool ensure_dynamic_smem(const void* kernel, size_t bytes) {
    if (bytes <= 48 * 1024) return true;
    static std::mutex mu;
    static std::map<std::pair<int, const void*>, size_t> granted;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    std::lock_guard<std::mutex> lock(mu);
    size_t& have = granted[{dev, kernel}];
    if (have >= bytes) return true;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) {
        note_cuda_failure("cudaFuncSetAttribute(MaxDynamicSharedMemorySize)", e);
        cudaGetLastError();
        return false;
    }
    have = bytes;
    return true;
}

bool cta_pairs_can_launch(const void* kernel, int threads, size_t dynamic_smem) {
    if (!ensure_dynamic_smem(kernel, dynamic_smem)) return false;
    static std::mutex mu;
    static std::map<std::tuple<int, const void*, size_t>, bool> known;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    std::lock_guard<std::mutex> lock(mu);
    const auto key = std::make_tuple(dev, kernel, dynamic_smem);
    const auto it = known.find(key);
    if (it != known.end()) return it->second;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = dynamic_smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
    if (e != cudaSuccess) cudaGetLastError();
    return known[key] = (e == cudaSuccess && clusters >= 1);
}
}  // namespace pamm

namespace {

inline size_t esize(pamm_dtype dt) { return dt == PAMM_BF16 ? 2 : 4; }
inline bool dtype_ok(pamm_dtype dt) { return dt == PAMM_F32 || dt == PAMM_BF16; }
inline bool layout_ok(pamm_layout l) { return l == PAMM_DW_NM || l == PAMM_DW_MN; }
inline bool index_type_ok(pamm_index_type t) { return t == PAMM_IDX_I32 || t == PAMM_IDX_U16 || t == PAMM_IDX_U8; }
inline size_t index_size(pamm_index_type t) { return t == PAMM_IDX_I32 ? 4 : t == PAMM_IDX_U16 ? 2 : 1; }
inline int64_t index_limit(pamm_index_type t) { return t == PAMM_IDX_I32 ? (1ll << 31) - 1 : t == PAMM_IDX_U16 ? 65536 : 256; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool ld_ok(int64_t ld, int64_t cols, size_t es) { return ld >= cols && (ld * (int64_t)es) % 16 == 0; }
inline pamm_status launch_status() { return launch_result("kernel launch"); }
constexpr int64_t MAX_ROWS = (1ll << 31) - 1024;   // row ids, counts and offsets are int32

// Kernel launches issued so far (all streams), and optional event pairs that
// bracket the dominant kernel of a step so a benchmark can time it in place.
std::atomic<unsigned long long> g_launches{0};
cudaEvent_t g_prof[3][2] = {{nullptr, nullptr}, {nullptr, nullptr}, {nullptr, nullptr}};
inline void prof_begin(int kind, cudaStream_t st) { if (g_prof[kind][0]) cudaEventRecord(g_prof[kind][0], st); }
inline void prof_end(int kind, cudaStream_t st) { if (g_prof[kind][1]) cudaEventRecord(g_prof[kind][1], st); }

// Launch with or without the programmatic-serialization attribute.  With it, the
// kernel may begin while the previous kernel of the stream is still running and
// must call grid_dependency_wait() before it depends on that kernel.
template <typename... P, typename... A>
inline void launch(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool overlap_prev, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = overlap_prev ? 1 : 0;
    cudaLaunchKernelEx(&cfg, kern, P(args)...);
    g_launches += 1;
}

int sm_count() {
    static int sms = 0;
    if (!sms) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
            sms = 148;
    }
    return sms;
}

// The row partition shared by the compress pass and the counting sort of the backward pass.
inline int64_t sort_rows_per_block(int64_t b) { return compress_rows_per_cta(b, sm_count()); }
inline ContractWs contract_ws(void* base, int64_t b, int64_t m, int64_t k) {
    return contract_ws_layout(base, b, m, k, sort_rows_per_block(b));
}
// Bytes of the per-block histograms of f for one generator set (the "sort products").
inline size_t sort_products_bytes(int64_t b, int64_t k) {
    const int64_t rpb = sort_rows_per_block(b);
    return (size_t)round_up(((b + rpb - 1) / rpb) * k * 4, 256);
}

struct StepArena {
    char *X, *dY, *C, *dW, *Bt, *ws, *products;
    float *invnorm, *alpha;
    int32_t *idx, *f;
    int64_t ldx, ldy, ldc, ldw, ldb;
    size_t ws_bytes, bytes;
};

StepArena step_arena_layout(void* base, int64_t b, int64_t n, int64_t m, int64_t k, pamm_dtype dt) {
    StepArena a;
    const size_t es = esize(dt);
    const int64_t v = 16 / (int64_t)es;
    a.ldx = round_up(n, v); a.ldy = round_up(m, v); a.ldc = a.ldx;
    a.ldw = round_up(m, 4); a.ldb = a.ldw;
    char* p = (char*)base;
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = (size_t)round_up((int64_t)(off + bytes), 256); return p ? p + o : (char*)0; };
    a.X = take((size_t)b * a.ldx * es);
    a.dY = take((size_t)b * a.ldy * es);
    a.C = take((size_t)k * a.ldc * es);
    a.invnorm = (float*)take((size_t)2 * k * 4);
    a.idx = (int32_t*)take((size_t)k * 4);
    a.f = (int32_t*)take((size_t)b * 4);
    a.alpha = (float*)take((size_t)b * 4);
    a.Bt = take((size_t)k * a.ldb * 4);
    a.dW = take((size_t)n * a.ldw * 4);
    a.ws_bytes = contract_ws(nullptr, b, m, k).bytes_with_planes;
    a.ws = take(a.ws_bytes);
    a.products = take(sort_products_bytes(b, k));
    a.bytes = off;
    return a;
}

template <typename T>
pamm_status launch_select(const void* X, int64_t ldx, int64_t b, int64_t n, int64_t k, uint64_t seed,
                          const int32_t* idx_in, int32_t* idx_out, void* C, int64_t ldc, float* c_invnorm,
                          cudaStream_t st, int32_t* zero_words = nullptr, int64_t zero_count = 0) {
    const size_t smem = (size_t)k * 4;
    if (!ensure_dynamic_smem((const void*)select_kernel<T>, smem)) return PAMM_ERR_CUDA;
    const PermKey pk = make_perm_key(seed, (uint32_t)b);
    const int grid = (int)k;
    launch(select_kernel<T>, dim3(grid), dim3(SEL_THREADS), smem, st, true, (const T*)X, ldx, b, n, (int)k, pk, idx_in,
           idx_out, (T*)C, ldc, c_invnorm, zero_words, zero_count);
    return launch_status();
}

// The neighbourhood condition (Eq. 2) applied or not: eps as given by the caller, the
// device counter of dropped rows (zeroed on the stream before the kernel).
struct Neighbourhood {
    bool on;
    float eps;
    int32_t* dropped;
};
constexpr Neighbourhood NO_NEIGHBOURHOOD = {false, 0.f, nullptr};

template <typename T>
pamm_status launch_compress_simt(const void* X, int64_t ldx, int64_t b, int64_t n, const void* C, int64_t ldc,
                                 int64_t k, const float* c_invnorm, void* f, int f_type, float* alpha,
                                 const Neighbourhood& nb, cudaStream_t st) {
    const int64_t want = (b + CS_WARPS - 1) / CS_WARPS;
    const int grid = (int)std::min<int64_t>(want, 148 * 8);
    const float eps2 = nb.eps * nb.eps, slack = neighbourhood_slack(n);
    auto kern = nb.on ? (k <= 4 ? compress_simt_kernel<T, 4, true> : compress_simt_kernel<T, 8, true>)
                      : (k <= 4 ? compress_simt_kernel<T, 4, false> : compress_simt_kernel<T, 8, false>);
    prof_begin(PAMM_PROF_COMPRESS, st);
    launch(kern, dim3(grid), dim3(CS_THREADS), 0, st, true, (const T*)X, ldx, b, n, (const T*)C, ldc, (int)k, c_invnorm, f,
           f_type, alpha, eps2, slack, nb.dropped);
    prof_end(PAMM_PROF_COMPRESS, st);
    return launch_status();
}

// Largest nb * nb * k (histogram words read by all scatter blocks together) for
// which every block rebuilds the scan on its own instead of a separate launch.
constexpr int64_t FUSED_SCAN_LIMIT = 1ll << 24;

// The counting sort of the rows by f.  `products` (the per-block histograms the compress
// pass left behind) saves the histogram launch.
pamm_status launch_sort(const void* f, int f_type, const float* alpha, int64_t b, int64_t k, const int32_t* products,
                        const ContractWs& w, cudaStream_t st) {
    if (k <= SK_MAX_K) products = nullptr;     // the forward pass for so few generators leaves no counts
    const size_t hsmem = (size_t)k * 4;
    const int rpb = (int)w.rows_per_block;
    const int tbl_warps = scatter_table_warps(rpb, k);
    const size_t ssmem = (size_t)(1 + tbl_warps) * k * 4;
    if (!ensure_dynamic_smem((const void*)contract_hist_kernel, hsmem) ||
        !ensure_dynamic_smem((const void*)contract_scatter_kernel, ssmem) ||
        !ensure_dynamic_smem((const void*)contract_scan_scatter_kernel, ssmem))
        return PAMM_ERR_CUDA;
    const bool fused_scan = w.nb * w.nb * k <= FUSED_SCAN_LIMIT;
    const int32_t* hist = w.hist;
    if (products && fused_scan) {
        hist = products;            // read in place
    } else if (products) {          // the scan below rewrites the table: work on a copy
        if (cudaMemcpyAsync(w.hist, products, (size_t)w.nb * k * 4, cudaMemcpyDeviceToDevice, st) != cudaSuccess)
            return PAMM_ERR_CUDA;
    } else {
        launch(contract_hist_kernel, dim3((unsigned)w.nb), dim3(SORT_BLK), hsmem, st, true, f, f_type, alpha, b, (int)k, rpb, w.hist);
    }
    if (fused_scan) {
        launch(contract_scan_scatter_kernel, dim3((unsigned)w.nb), dim3(SORT_BLK), ssmem, st, true, f, f_type, alpha, b, (int)k,
               rpb, tbl_warps, hist, (int)w.nb, w.seg_start, w.perm);
    } else {
        launch(contract_scan_kernel, dim3(1), dim3(SCAN_THREADS), 0, st, true, w.hist, (int)w.nb, (int)k, w.seg_start);
        launch(contract_scatter_kernel, dim3((unsigned)w.nb), dim3(SORT_BLK), ssmem, st, true, f, f_type, alpha, b, (int)k, rpb,
               tbl_warps, (const int32_t*)w.hist, (const int32_t*)w.seg_start, w.perm);
    }
    return launch_status();
}

template <typename T>
pamm_status launch_contract(const void* f, int f_type, const float* alpha, const void* dY, int64_t ldy, int64_t b,
                            int64_t m, int64_t k, float* Bt, int64_t ldb, const int32_t* products, const ContractWs& w,
                            cudaStream_t st, bool with_planes = false) {
    constexpr int V = Vec16<T>::N;
    uint16_t* planes = with_planes ? w.planes : nullptr;     // B~ also as bf16 hi / lo, for the product that follows
    pamm_status s = launch_sort(f, f_type, alpha, b, k, products, w, st);
    if (s != PAMM_OK) return s;
    if (contract_stream_supported(m, sizeof(T))) {
        // one balanced wave, two CTAs per SM: rows of dY stream through a shared-memory ring
        const ContractStreamPlan p = contract_stream_plan(m, sizeof(T));
        int64_t ranges = std::min<int64_t>(CT_MAX_CTAS, (int64_t)sm_count() * CS_CTAS_PER_SM);
        const int64_t rows_per_cta = std::max<int64_t>(32, (b + ranges - 1) / ranges);
        ranges = (b + rows_per_cta - 1) / rows_per_cta;
        auto kern = p.vpt == 4   ? contract_stream_kernel<T, 4, 1>
                    : p.vpt == 2 ? contract_stream_kernel<T, 2, 1>
                    : p.rps == 4 ? contract_stream_kernel<T, 1, 4>
                    : p.rps == 2 ? contract_stream_kernel<T, 1, 2>
                                 : contract_stream_kernel<T, 1, 1>;
        if (!ensure_dynamic_smem((const void*)kern, p.smem_bytes)) return PAMM_ERR_CUDA;
        prof_begin(PAMM_PROF_CONTRACT, st);
        launch(kern, dim3((unsigned)ranges), dim3(p.consumers + 32), p.smem_bytes, st, true, f, f_type, alpha, (const T*)dY,
               ldy, b, m, (int)k, (const int32_t*)w.seg_start, (const int32_t*)w.perm, (int)ranges, p.slots,
               p.row_pitch, p.bulk_bytes, w.partials, w.m_pad, Bt, ldb);
        prof_end(PAMM_PROF_CONTRACT, st);
        launch(contract_reduce_kernel, dim3((unsigned)((w.m_pad / 4 + RED_THREADS - 1) / RED_THREADS), (unsigned)std::min<int64_t>(k, 65535)), dim3(RED_THREADS), 0, st,
               true, (const float*)w.partials, w.m_pad, m, (int)k, b, (const int32_t*)w.seg_start, (int)ranges, Bt, ldb, planes, w.plane_ld);
        return launch_status();
    }
    // very wide rows: column slabs, register staging
    const int64_t vecs = (m + V - 1) / V;
    const int64_t slabs = (vecs + CT_MAX_THREADS - 1) / CT_MAX_THREADS;
    const int threads = (int)round_up((vecs + slabs - 1) / slabs, 32);
    int occ = 1;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, contract_main_kernel<T>, threads, 0) != cudaSuccess || occ < 1)
        occ = 1;
    int64_t ranges = std::max<int64_t>(1, std::min<int64_t>(CT_MAX_CTAS, (int64_t)sm_count() * occ / slabs));
    const int64_t rows_per_cta = std::max<int64_t>(32, (b + ranges - 1) / ranges);
    ranges = (b + rows_per_cta - 1) / rows_per_cta;
    dim3 grid((unsigned)ranges, (unsigned)slabs);
    prof_begin(PAMM_PROF_CONTRACT, st);
    launch(contract_main_kernel<T>, grid, dim3(threads), 0, st, true, alpha, (const T*)dY, ldy, b, m, (int)k,
           (const int32_t*)w.seg_start, (const int32_t*)w.perm, (int)ranges, w.partials, w.m_pad, Bt, ldb);
    prof_end(PAMM_PROF_CONTRACT, st);
    launch(contract_reduce_kernel, dim3((unsigned)((w.m_pad / 4 + RED_THREADS - 1) / RED_THREADS), (unsigned)std::min<int64_t>(k, 65535)), dim3(RED_THREADS), 0, st, true,
           (const float*)w.partials, w.m_pad, m, (int)k, b, (const int32_t*)w.seg_start, (int)ranges, Bt, ldb, planes, w.plane_ld);
    return launch_status();
}

// How the weight gradient is stored.
struct DwSpec {
    void* ptr;
    int64_t ld;
    pamm_dtype dt;
    pamm_layout layout;
};

template <typename T>
pamm_status launch_weight_grad_simt(const void* C, int64_t ldc, int64_t k, int64_t n, const float* Bt, int64_t ldb,
                                    int64_t m, const DwSpec& dw, cudaStream_t st, int64_t b_rows,
                                    const int32_t* dropped, bool accumulate) {
    const bool swap = dw.layout == PAMM_DW_MN;
    const int64_t rows = swap ? m : n, cols = swap ? n : m;
    const int64_t items = rows * ((cols + 3) / 4);
    const dim3 grid((unsigned)((items + WG_THREADS - 1) / WG_THREADS)), block(WG_THREADS);
    prof_begin(PAMM_PROF_WEIGHT_GRAD, st);
    if (dw.dt == PAMM_F32) {
        auto kern = swap ? weight_grad_simt_kernel<T, float, true> : weight_grad_simt_kernel<T, float, false>;
        launch(kern, grid, block, 0, st, true, (const T*)C, ldc, (int)k, n, Bt, ldb, m, (float*)dw.ptr, dw.ld, b_rows, dropped,
               accumulate ? 1 : 0);
    } else {
        auto kern = swap ? weight_grad_simt_kernel<T, __nv_bfloat16, true> : weight_grad_simt_kernel<T, __nv_bfloat16, false>;
        launch(kern, grid, block, 0, st, true, (const T*)C, ldc, (int)k, n, Bt, ldb, m, (__nv_bfloat16*)dw.ptr, dw.ld, b_rows,
               dropped, accumulate ? 1 : 0);
    }
    prof_end(PAMM_PROF_WEIGHT_GRAD, st);
    return launch_status();
}

// ---- a handful of generators (k <= 8): three launches for the whole path ----
template <typename T>
pamm_status launch_small_forward(const void* X, int64_t ldx, int64_t b, int64_t n, int64_t k, uint64_t seed,
                                 const int32_t* idx_in, int32_t* idx_out, void* C, int64_t ldc, float* c_invnorm,
                                 void* f, int f_type, float* alpha, cudaStream_t st) {
    constexpr int V = Vec16<T>::N;
    const size_t smem = (size_t)k * round_up(n, V) * sizeof(T);
    if (!ensure_dynamic_smem((const void*)compress_small_kernel<T>, smem)) return PAMM_ERR_CUDA;
    // a row per warp while there are few rows; enough rows per CTA to pay for its copy of the generators otherwise
    const int64_t rows_per_cta = std::max<int64_t>(SK_WARPS, (b + 4 * sm_count() - 1) / (4 * sm_count()));
    const PermKey pk = make_perm_key(seed, (uint32_t)b);
    prof_begin(PAMM_PROF_COMPRESS, st);
    launch(compress_small_kernel<T>, dim3((unsigned)((b + rows_per_cta - 1) / rows_per_cta)), dim3(SK_THREADS), smem, st, true,
           (const T*)X, ldx, b, n, (int)k, pk, idx_in, idx_out, (T*)C, ldc, c_invnorm, f, f_type, alpha, (int)rows_per_cta);
    prof_end(PAMM_PROF_COMPRESS, st);
    return launch_status();
}

template <typename T, typename OutT>
void launch_wgrad_small(const void* C, int64_t ldc, int64_t k, int64_t n, const float* partials, int ranges, int64_t m_pad,
                        int64_t m, float* Bt, int64_t ldb, const DwSpec& dw, bool accumulate, cudaStream_t st) {
    const dim3 grid((unsigned)((m + SK_WG_COLS - 1) / SK_WG_COLS), (unsigned)((n + SK_WG_ROWS - 1) / SK_WG_ROWS));
    if (dw.layout == PAMM_DW_MN)
        launch(wgrad_small_kernel<T, OutT, true>, grid, dim3(SK_THREADS), 0, st, true, (const T*)C, ldc, (int)k, n, partials, ranges,
               m_pad, m, Bt, ldb, (OutT*)dw.ptr, dw.ld, accumulate ? 1 : 0);
    else
        launch(wgrad_small_kernel<T, OutT, false>, grid, dim3(SK_THREADS), 0, st, true, (const T*)C, ldc, (int)k, n, partials, ranges,
               m_pad, m, Bt, ldb, (OutT*)dw.ptr, dw.ld, accumulate ? 1 : 0);
}

template <typename T>
pamm_status launch_small_backward(const void* C, int64_t ldc, int64_t n, const void* f, int f_type, const float* alpha,
                                  const void* dY, int64_t ldy, int64_t b, int64_t m, int64_t k, float* Bt, int64_t ldb,
                                  const DwSpec& dw, const ContractWs& w, cudaStream_t st) {
    constexpr int V = Vec16<T>::N;
    // one partial B~ (k rows) per row range, in the workspace's partial rows
    int64_t ranges = std::max<int64_t>(1, std::min<int64_t>((b + 31) / 32, std::min<int64_t>(CT_MAX_CTAS / k, 2 * sm_count())));
    const int64_t rows_per_range = (b + ranges - 1) / ranges;
    ranges = (b + rows_per_range - 1) / rows_per_range;
    const int64_t vecs = (m + V - 1) / V;
    const int threads = (int)std::min<int64_t>(SK_CT_THREADS, round_up(vecs, 32));
    const int64_t slabs = (vecs + threads - 1) / threads;
    prof_begin(PAMM_PROF_CONTRACT, st);
    launch(contract_small_kernel<T>, dim3((unsigned)ranges, (unsigned)slabs), dim3(threads), 0, st, true, f, f_type, alpha,
           (const T*)dY, ldy, b, m, (int)k, (int)rows_per_range, w.partials, w.m_pad);
    prof_end(PAMM_PROF_CONTRACT, st);
    prof_begin(PAMM_PROF_WEIGHT_GRAD, st);
    if (dw.dt == PAMM_F32)
        launch_wgrad_small<T, float>(C, ldc, k, n, w.partials, (int)ranges, w.m_pad, m, Bt, ldb, dw, false, st);
    else
        launch_wgrad_small<T, __nv_bfloat16>(C, ldc, k, n, w.partials, (int)ranges, w.m_pad, m, Bt, ldb, dw, false, st);
    prof_end(PAMM_PROF_WEIGHT_GRAD, st);
    return launch_status();
}

pamm_status check_select(const void* X, int64_t ldx, int64_t b, int64_t n, pamm_dtype dt, int64_t k,
                         int32_t* idx_out, void* C, int64_t ldc, float* c_invnorm) {
    if (!dtype_ok(dt)) return PAMM_ERR_UNSUPPORTED;
    if (!X || !idx_out || !C || !c_invnorm) return PAMM_ERR_INVALID_ARG;
    if (b < 1 || n < 1 || k < 1 || k > b || b > MAX_ROWS) return PAMM_ERR_INVALID_ARG;
    if (!ld_ok(ldx, n, esize(dt)) || !ld_ok(ldc, n, esize(dt))) return PAMM_ERR_INVALID_ARG;
    if (!aligned(X, 16) || !aligned(C, 16) || !aligned(idx_out, 4) || !aligned(c_invnorm, 4)) return PAMM_ERR_INVALID_ARG;
    if (k > SEL_MAX_K) return PAMM_ERR_UNSUPPORTED;
    return PAMM_OK;
}

// The sort products are optional: no buffer, none written.
pamm_status check_products_out(const void* ws, size_t ws_bytes, int64_t b, int64_t k, int groups) {
    if (!ws) return PAMM_OK;
    if (!aligned(ws, 256) || ws_bytes < (size_t)groups * sort_products_bytes(b, k)) return PAMM_ERR_WORKSPACE;
    return PAMM_OK;
}

pamm_status check_compress(const void* X, int64_t ldx, int64_t b, int64_t n, pamm_dtype dt, const void* C,
                           int64_t ldc, int64_t k, const float* c_invnorm, void* f, pamm_index_type f_type, float* alpha) {
    if (!dtype_ok(dt) || !index_type_ok(f_type)) return PAMM_ERR_UNSUPPORTED;
    if (!X || !C || !c_invnorm || !f || !alpha) return PAMM_ERR_INVALID_ARG;
    if (b < 1 || n < 1 || k < 1 || k > b || b > MAX_ROWS) return PAMM_ERR_INVALID_ARG;
    if (k > index_limit(f_type)) return PAMM_ERR_INVALID_ARG;     // f_i would not fit its storage type
    if (!ld_ok(ldx, n, esize(dt)) || !ld_ok(ldc, n, esize(dt))) return PAMM_ERR_INVALID_ARG;
    if (!aligned(X, 16) || !aligned(C, 16) || !aligned(f, index_size(f_type)) || !aligned(alpha, 4) || !aligned(c_invnorm, 4))
        return PAMM_ERR_INVALID_ARG;
    return PAMM_OK;
}

pamm_status check_contract(const void* f, pamm_index_type f_type, const float* alpha, const void* dY, int64_t ldy,
                           int64_t b, int64_t m, pamm_dtype dt, int64_t k, const float* Bt, int64_t ldb, bool bt_required,
                           const void* products, const void* ws, size_t ws_bytes) {
    if (!dtype_ok(dt) || !index_type_ok(f_type)) return PAMM_ERR_UNSUPPORTED;
    if (!f || !alpha || !dY || (bt_required && !Bt)) return PAMM_ERR_INVALID_ARG;
    if (b < 1 || m < 1 || k < 1 || k > b || b > MAX_ROWS) return PAMM_ERR_INVALID_ARG;
    if (k > index_limit(f_type)) return PAMM_ERR_INVALID_ARG;
    if (!ld_ok(ldy, m, esize(dt)) || (Bt && !ld_ok(ldb, m, 4))) return PAMM_ERR_INVALID_ARG;
    if (!aligned(dY, 16) || (Bt && !aligned(Bt, 16)) || !aligned(f, index_size(f_type)) || !aligned(alpha, 4))
        return PAMM_ERR_INVALID_ARG;
    if (products && !aligned(products, 256)) return PAMM_ERR_INVALID_ARG;
    if (k > CT_MAX_K) return PAMM_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256)) return PAMM_ERR_WORKSPACE;
    if (ws_bytes < contract_ws(nullptr, b, m, k).bytes) return PAMM_ERR_WORKSPACE;
    return PAMM_OK;
}

pamm_status check_weight_grad(const void* C, int64_t ldc, int64_t k, int64_t n, pamm_dtype dt, const float* Bt,
                              int64_t ldb, int64_t m, const DwSpec& dw) {
    if (!dtype_ok(dt) || !dtype_ok(dw.dt) || !layout_ok(dw.layout)) return PAMM_ERR_UNSUPPORTED;
    if (!C || !Bt || !dw.ptr) return PAMM_ERR_INVALID_ARG;
    if (k < 1 || n < 1 || m < 1) return PAMM_ERR_INVALID_ARG;
    const int64_t out_cols = dw.layout == PAMM_DW_MN ? n : m;
    if (!ld_ok(ldc, n, esize(dt)) || !ld_ok(ldb, m, 4) || !ld_ok(dw.ld, out_cols, esize(dw.dt))) return PAMM_ERR_INVALID_ARG;
    if (!aligned(C, 16) || !aligned(Bt, 16) || !aligned(dw.ptr, 16)) return PAMM_ERR_INVALID_ARG;
    return PAMM_OK;
}

// x_is_ready: X was complete before the previous kernel of the stream started (true
// after our own select kernel), so the compress kernel may read it before that
// kernel has finished.  `groups` generator sets are served by one pass over X where the
// tensor-core kernel applies, else by one CUDA-core pass per set.  `products` (optional)
// receives the per-block histograms of f.
pamm_status do_compress(const void* X, int64_t ldx, int64_t b, int64_t n, pamm_dtype dt, const void* C, int64_t ldc,
                        int64_t k, int groups, const float* c_invnorm, void* f, pamm_index_type f_type, float* alpha,
                        int64_t out_stride, int32_t* products, bool x_is_ready, cudaStream_t st,
                        const Neighbourhood& nb = NO_NEIGHBOURHOOD) {
    if (dt == PAMM_BF16 && compress_umma_usable(b, n, k, groups, sm_count(), nb.on)) {
        const CompressOut out = {f, alpha, out_stride, products, (int64_t)(sort_products_bytes(b, k) / 4), (int)f_type};
        // many generators per chunk (tensor-bound): pairs of CTAs on one MMA tile; the same rows, results and counts
        const bool pairs = !nb.on && compress_pair_usable(b, n, k, groups, sm_count());
        prof_begin(PAMM_PROF_COMPRESS, st);
        const pamm_status s = pairs
            ? launch_compress_pair(X, ldx, b, n, C, ldc, k, groups, c_invnorm, out, sm_count(), x_is_ready, st)
            : launch_compress_umma(X, ldx, b, n, C, ldc, k, groups, c_invnorm, out, sm_count(), x_is_ready, st, nb.on, nb.eps,
                                   nb.dropped);
        prof_end(PAMM_PROF_COMPRESS, st);
        g_launches += 1;
        return s;
    }
    const size_t es = esize(dt), fs = index_size(f_type);
    const int64_t rpb = sort_rows_per_block(b), nblk = (b + rpb - 1) / rpb;
    if (products && !ensure_dynamic_smem((const void*)contract_hist_kernel, (size_t)k * 4)) return PAMM_ERR_CUDA;
    for (int g = 0; g < groups; ++g) {
        const char* Cg = (const char*)C + (size_t)g * k * ldc * es;
        void* fg = (char*)f + (size_t)g * out_stride * fs;
        float* ag = alpha + (size_t)g * out_stride;
        const pamm_status s = dt == PAMM_F32
            ? launch_compress_simt<float>(X, ldx, b, n, Cg, ldc, k, c_invnorm + (size_t)g * 2 * k, fg, (int)f_type, ag, nb, st)
            : launch_compress_simt<__nv_bfloat16>(X, ldx, b, n, Cg, ldc, k, c_invnorm + (size_t)g * 2 * k, fg, (int)f_type, ag, nb, st);
        if (s != PAMM_OK) return s;
        if (products)
            launch(contract_hist_kernel, dim3((unsigned)nblk), dim3(SORT_BLK), (size_t)k * 4, st, true, (const void*)fg,
                   (int)f_type, (const float*)ag, b, (int)k, (int)rpb, products + (size_t)g * (sort_products_bytes(b, k) / 4));
    }
    return launch_status();
}

pamm_status do_weight_grad(const void* C, int64_t ldc, int64_t k, int64_t n, pamm_dtype dt, const float* Bt,
                           int64_t ldb, int64_t m, const DwSpec& dw, cudaStream_t st, int64_t b_rows = 0,
                           const int32_t* dropped = nullptr, bool accumulate = false) {
    if (dt == PAMM_F32)
        return launch_weight_grad_simt<float>(C, ldc, k, n, Bt, ldb, m, dw, st, b_rows, dropped, accumulate);
    const bool bf16_out = dw.dt == PAMM_BF16, swap = dw.layout == PAMM_DW_MN;
    // the TMA stores need at least one whole 16-byte unit per output row
    const bool tma_ok = (swap ? n : m) * (int64_t)esize(dw.dt) >= 16;
    if (tma_ok && weight_grad_persist_supported(k, n, m)) {
        prof_begin(PAMM_PROF_WEIGHT_GRAD, st);
        const pamm_status s = launch_weight_grad_persist(C, ldc, k, n, Bt, ldb, m, dw.ptr, dw.ld, bf16_out, swap, sm_count(), st,
                                                          b_rows, dropped, accumulate);
        prof_end(PAMM_PROF_WEIGHT_GRAD, st);
        g_launches += 1;
        return s;
    }
    if (tma_ok && weight_grad_chunked_supported(k, n, m)) {
        prof_begin(PAMM_PROF_WEIGHT_GRAD, st);
        const pamm_status s = launch_weight_grad_chunked(C, ldc, k, n, Bt, ldb, m, dw.ptr, dw.ld, bf16_out, swap, sm_count(), st,
                                                         b_rows, dropped, accumulate);
        prof_end(PAMM_PROF_WEIGHT_GRAD, st);
        g_launches += 1;
        return s;
    }
    return launch_weight_grad_simt<__nv_bfloat16>(C, ldc, k, n, Bt, ldb, m, dw, st, b_rows, dropped, accumulate);
}

}  // namespace

// One CTA waits, with the library's bounded wait and a short limit, on a barrier that
// nothing will ever complete; the wait must give up, raise the status word and let the
// kernel end normally.
__global__ void selftest_bounded_wait_kernel(uint32_t polls) {
    __shared__ uint64_t s_bar;
    __shared__ int s_abort;
    if (threadIdx.x == 0) {
        ptx::mbar_init(&s_bar, 1);
        s_abort = 0;
        ptx::fence_barrier_init();
    }
    __syncthreads();
    volatile int* abort_flag = &s_abort;
    const bool done = ptx::mbar_wait(&s_bar, 0, abort_flag, polls);
    if (!done && (threadIdx.x & 31) == 0) raise_status(DEV_TIMEOUT);
}
// One warp waits with a limit of 256 polls (about a millisecond) for another that shows progress every quarter of one, 32 times, and
// only then arrives: eight times the limit.
__global__ void selftest_progress_wait_kernel(uint32_t polls) {
    __shared__ uint64_t s_bar;
    __shared__ Watch s_watch;
    if (threadIdx.x == 0) {
        ptx::mbar_init(&s_bar, 1);
        s_watch = {};
        ptx::fence_barrier_init();
    }
    __syncthreads();
    volatile Watch* watch = &s_watch;
    if (threadIdx.x >= 32) {
        const bool done = warp_wait(&s_bar, 0, watch, polls);
        if (!done && threadIdx.x == 32) raise_status(DEV_TIMEOUT);
    } else if (threadIdx.x == 0) {
        for (uint32_t i = 1; i <= 32; ++i) {
            for (int n = 0; n < 256; ++n) __nanosleep(1000);
            watch->items = i;
        }
        ptx::mbar_arrive(&s_bar);
    }
}

// ---- the operators around the projection ---------------------------------------------------
namespace {

// Row partition of the norm's column sums where they are a launch of their own, and the scratch that holds the partial sums.
inline int64_t norm_splits(int64_t b) { return std::max<int64_t>(1, std::min<int64_t>((b + 31) / 32, 2 * sm_count())); }
// Blocks per SM of the fused backward pass, at most: the registers allow no more where rows are wide.
inline int norm_backward_blocks(int64_t n) { return n <= 2048 ? 4 : 3; }
inline size_t norm_backward_ws_bytes(int64_t b, int64_t n) {
    return (size_t)round_up(std::min<int64_t>(b + 8, norm_backward_blocks(n) * sm_count()) * 2 * round_up(n, 8) * 4, 256);
}
inline size_t attention_backward_ws_bytes(int64_t tokens, int64_t heads) { return (size_t)round_up(tokens * heads * 4, 256); }
inline int grad_norm_blocks() { return sm_count() * GC_BLOCKS_PER_SM; }
inline size_t grad_norm_ws_bytes() { return (size_t)round_up((int64_t)grad_norm_blocks() * 8, 256) + 256; }      // and the factor

// An element-aligned row-major matrix of at least one row; leading dimension in elements.
inline bool matrix_ok(const void* p, int64_t ld, int64_t cols, size_t es) { return p && aligned(p, es) && ld >= cols; }

cudaLaunchConfig_t cluster_config(unsigned clusters, int cluster, int threads, size_t smem, cudaStream_t st, cudaLaunchAttribute (&attr)[2]) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(clusters * cluster);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cfg;
}
template <typename... P, typename... A>
void launch_clusters(void (*kern)(P...), unsigned clusters, int cluster, int threads, size_t smem, cudaStream_t st, A... args) {
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = cluster_config(clusters, cluster, threads, smem, st, attr);
    cudaLaunchKernelEx(&cfg, kern, P(args)...);
    g_launches += 1;
}

// How many blocks of a kernel an SM of the current device holds, and how many clusters the device (asked once for each device,
// kernel and size).
int resident(const void* kernel, int threads, size_t smem, int cluster) {
    static std::mutex mu;
    static std::map<std::tuple<int, const void*, int, size_t, int>, int> known;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 1;
    std::lock_guard<std::mutex> lock(mu);
    const auto key = std::make_tuple(dev, kernel, threads, smem, cluster);
    const auto it = known.find(key);
    if (it != known.end()) return it->second;
    int count = 0;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = cluster_config(1, cluster, threads, smem, nullptr, attr);
    cfg.numAttrs = 1;
    const cudaError_t e = cluster == 1 ? cudaOccupancyMaxActiveBlocksPerMultiprocessor(&count, kernel, threads, smem)
                                       : cudaOccupancyMaxActiveClusters(&count, kernel, &cfg);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return 1;
    }
    return known[key] = std::max(1, count);
}

// How the matrices of a call can be accessed (the three ways are described in norm.cuh).
enum class RowAccess { whole, ragged, elements };
struct RowMatrix { const void* p; int64_t ld; };
template <int N>
RowAccess row_access(const RowMatrix (&m)[N], int64_t n, size_t es, bool weights_aligned) {
    const auto phase = [&](int i) { return reinterpret_cast<uintptr_t>(m[i].p) % 16; };
    const auto turn = [&](int i) { return (m[i].ld * (int64_t)es) % 16; };
    bool same = true, zero = phase(0) == 0 && turn(0) == 0;
    for (int i = 1; i < N; ++i) same = same && (!m[i].p || (phase(i) == phase(0) && turn(i) == turn(0)));
    if (same && zero && (n * es) % 16 == 0 && weights_aligned) return RowAccess::whole;
    return same ? RowAccess::ragged : RowAccess::elements;
}

template <typename T, typename W, int V, int EPT, int LANES, int ROWS, bool RAGGED>
pamm_status launch_norm_forward(NormForwardArgs a, cudaStream_t st) {
    a.warps = (a.n + LANES * EPT - 1) / (LANES * EPT);
    const int64_t jobs = (a.b + ROWS - 1) / ROWS;
    const int threads = a.warps > 1 ? 32 * a.warps : jobs * LANES >= 256 ? 256 : (int)round_up(jobs * LANES, 32);
    const int64_t jobs_per_block = a.warps > 1 ? 1 : threads / LANES;
    launch(norm_forward_kernel<T, W, V, EPT, LANES, ROWS, RAGGED>, dim3((unsigned)((jobs + jobs_per_block - 1) / jobs_per_block)), dim3(threads),
           0, st, true, a);
    return launch_status();
}
// Elements and rows a thread: 8 of one row while the rows do not fill the device (8 warps an SM at least are wanted, of narrow rows 32), then as many as
// registers hold, narrow rows in parts of a warp.  A ragged row needs 16 lanes for its ends.
template <typename T, typename W, int V, bool RAGGED>
pamm_status launch_norm_forward(const NormForwardArgs& a, cudaStream_t st) {
    const int64_t thin_warps = (a.n + 255) / 256;
    const bool many = a.b >= 32 * sm_count();
    if (a.n <= 64 && !RAGGED) return launch_norm_forward<T, W, V, 8, RAGGED ? 16 : 8, 1, RAGGED>(a, st);
    // 8 elements a thread, and 16 or 32 where there are rows enough: 10^6 x 128 bf16 101 and 92 us, 500000 x 256 107 and 91, 262144 x 512 with bias
    // (16 elements of a row or of two, and 32) 111, 95 and 91
    if (a.n <= 128 && !RAGGED && many) return launch_norm_forward<T, W, V, 16, RAGGED ? 16 : 8, 1, RAGGED>(a, st);
    if (a.n <= 128 && !many) return launch_norm_forward<T, W, V, 8, 16, 1, RAGGED>(a, st);
    if (a.n <= 256 && many) return launch_norm_forward<T, W, V, 16, 16, 1, RAGGED>(a, st);
    if (thin_warps <= 32 && (thin_warps == 1 || a.b * thin_warps <= 8 * sm_count())) return launch_norm_forward<T, W, V, 8, 32, 1, RAGGED>(a, st);
    if (a.n <= 512 && many && V > 1) return launch_norm_forward<T, W, V, (V > 1 ? 32 : 16), 16, 1, RAGGED>(a, st);
    // Two rows a thread where the weights weigh: fp32 weights, beside bf16 rows with a bias too.  Both sides measured, one row and two: 65536 x 2048
    // bf16 with fp32 weights and bias 124 and 98, with bf16 ones 93 and 98, with bf16 weights alone 85 and 89; 32768 x 2048 fp32 85
    // and 81.
    if constexpr (V > 1 && !RAGGED)
        if (a.n <= 4096 && sizeof(W) == 4 && (sizeof(T) == 4 || a.c) && a.b * ((a.n + 511) / 512) >= 64 * sm_count())
            return launch_norm_forward<T, W, V, 16, 32, 2, RAGGED>(a, st);
    if (a.n <= 512 || (V == 1 && a.n <= 16384)) return launch_norm_forward<T, W, V, 16, 32, 1, RAGGED>(a, st);
    return launch_norm_forward<T, W, V, 32, 32, 1, RAGGED>(a, st);
}
template <typename T, typename W>
pamm_status launch_norm_forward(const NormForwardArgs& a, RowAccess access, cudaStream_t st) {
    if (access == RowAccess::whole) return launch_norm_forward<T, W, Vec16<T>::N, false>(a, st);
    if (access == RowAccess::ragged) return launch_norm_forward<T, W, Vec16<T>::N, true>(a, st);
    return launch_norm_forward<T, W, 1, false>(a, st);
}

template <typename T, int V, int EPT, int LANES, bool RAGGED>
pamm_status launch_norm_backward_fused(NormBackwardArgs& a, cudaStream_t st) {
    a.cluster = 1;
    a.slice = a.n;
    a.warps = (a.n + LANES * EPT - 1) / (LANES * EPT);
    const int threads = a.warps > NB_WARPS / 2 ? 32 * a.warps : 32 * a.warps * (NB_WARPS / a.warps);
    a.groups = threads / (a.warps * LANES);
    const size_t ring = V > 1 ? (size_t)norm_stages<T, EPT>() * (a.dh ? 3 : 2) * (EPT / V) * threads * 16 : 0;
    const size_t smem = std::max(ring, (size_t)2 * norm_sums_pitch(a.n) * 4);
    const auto kernel = !a.rms || a.dc ? norm_backward_kernel<T, V, EPT, LANES, true, RAGGED, false>
                                       : norm_backward_kernel<T, V, EPT, LANES, false, RAGGED, false>;
    // the 48 KB that need no asking for hold the kernel's own arrays as well
    if (!ensure_dynamic_smem((const void*)kernel, smem > 44 * 1024 ? std::max<size_t>(smem, 49 * 1024) : smem)) return PAMM_ERR_CUDA;
    const int64_t want = ((a.b + a.period - 1) / a.period + a.groups - 1) / a.groups;      // blocks of each phase
    const int64_t most = (int64_t)sm_count() * std::min(norm_backward_blocks(a.n), resident((const void*)kernel, threads, smem, 1));
    a.splits = (int)(a.period * std::min<int64_t>(want, std::max<int64_t>(1, most / a.period)));
    launch(kernel, dim3((unsigned)a.splits), dim3(threads), smem, st, true, a);
    return launch_status();
}
template <typename T, int V, bool RAGGED>
pamm_status launch_norm_backward_clusters(NormBackwardArgs& a, cudaStream_t st) {
    constexpr int EPT = 16;                           // 8192 elements a block
    a.cluster = a.n <= 2 * 512 * EPT ? 2 : 4;
    a.slice = (int)round_up((a.n + a.cluster - 1) / a.cluster, V);
    a.warps = (a.slice + 32 * EPT - 1) / (32 * EPT);
    a.groups = 1;
    const int threads = 32 * a.warps;
    const size_t ring = (size_t)norm_stages<T, EPT>() * (a.dh ? 3 : 2) * (EPT / V) * threads * 16;
    const size_t smem = std::max(ring, (size_t)2 * norm_sums_pitch(a.slice + 16) * 4);
    const auto kernel = !a.rms || a.dc ? norm_backward_kernel<T, V, EPT, 32, true, RAGGED, true> : norm_backward_kernel<T, V, EPT, 32, false, RAGGED, true>;
    if (!ensure_dynamic_smem((const void*)kernel, std::max<size_t>(smem, 49 * 1024))) return PAMM_ERR_CUDA;
    const int64_t want = (a.b + a.period - 1) / a.period, most = resident((const void*)kernel, threads, smem, a.cluster);
    a.splits = (int)(a.period * std::min<int64_t>(want, std::max<int64_t>(1, most / a.period)));
    launch_clusters(kernel, a.splits, a.cluster, threads, smem, st, a);
    return launch_status();
}
// Elements a thread: 8 of a row of up to 256 in as many lanes as it needs, then 32 bytes of each matrix, or 64 of fp32; rows wider than the
// 8192 elements that 16 such warps hold go over clusters.
template <typename T, int V, bool RAGGED>
pamm_status launch_norm_backward_fused(NormBackwardArgs& a, cudaStream_t st) {
    constexpr int E = 2 * (int)Vec16<T>::N;
    const int64_t turn = (a.ldx * (int64_t)sizeof(T)) % 16;
    a.period = 1;
    while (RAGGED && (a.period * turn) % 16 != 0) a.period *= 2;
    if constexpr (V > 1) {
        if (a.n <= 64 && !RAGGED) return launch_norm_backward_fused<T, V, 8, RAGGED ? 16 : 8, RAGGED>(a, st);
        if (a.n <= 128) return launch_norm_backward_fused<T, V, 8, 16, RAGGED>(a, st);        // a ragged row needs 16 lanes for its ends
        if (a.n <= 256) return launch_norm_backward_fused<T, V, 8, 32, RAGGED>(a, st);
        if (a.n > 8192) return launch_norm_backward_clusters<T, V, RAGGED>(a, st);
        // fp32 with a mean or a bias, measured at 32 and at 64 bytes: 65536 x 1024 149 and 127 us, 16384 x 4096 151 and 123, but 2048 x 512 7.3
        // and 8.9; without them 120 and 129 us at 65536 x 1024
        const bool wide32 = (!a.rms || a.dc) && (a.n > 1024 || a.b * a.n > (8 << 20));
        if (sizeof(T) == 4 && (a.n > 512 * E || wide32)) return launch_norm_backward_fused<T, V, 16, 32, RAGGED>(a, st);
    }
    return launch_norm_backward_fused<T, V, E, 32, RAGGED>(a, st);
}

template <typename T>
pamm_status launch_norm_backward(NormBackwardArgs a, RowAccess access, cudaStream_t st) {
    constexpr int V = Vec16<T>::N;
    const bool sums = a.dw || a.dc;
    const bool fused = access != RowAccess::elements || a.n <= 1024 * V;
    a.splits = 0;
    if (fused && a.b) {
        const pamm_status s = access == RowAccess::whole    ? launch_norm_backward_fused<T, V, false>(a, st)
                              : access == RowAccess::ragged ? launch_norm_backward_fused<T, V, true>(a, st)
                                                            : launch_norm_backward_fused<T, 1, false>(a, st);
        if (s != PAMM_OK) return s;
    } else if (a.b && sums) {
        // too wide for a block, element by element: the column sums by themselves, before dX may take the place of dY or X
        a.rows_per_split = (a.b + norm_splits(a.b) - 1) / norm_splits(a.b);
        a.splits = (int)((a.b + a.rows_per_split - 1) / a.rows_per_split);
        launch(norm_backward_columns_kernel<T>, dim3((unsigned)((a.n + NB_COL_THREADS - 1) / NB_COL_THREADS), (unsigned)a.splits),
               dim3(NB_COL_THREADS), 0, st, true, a);
    }
    if (sums) {
        // at most about 512 blocks.  With 8, 16 and 32 columns a block: 256 x 4096 bf16 6.0, 6.6 and 7.8 us; 256 x 8192 11.1, 9.4 and 10.7; 64 x
        // 16384 10.5, 9.2 and 7.7
        const auto finish = [&](auto kernel, int cols) {
            launch(kernel, dim3((unsigned)((a.n + cols - 1) / cols)), dim3(NB_FINISH_THREADS), 0, st, true, a);
        };
        if (a.n <= 4096) finish(norm_backward_finish_kernel<8>, 8);
        else if (a.n <= 8192) finish(norm_backward_finish_kernel<16>, 16);
        else finish(norm_backward_finish_kernel<32>, 32);
    }
    if (a.b && !fused) launch(norm_backward_row_kernel<T>, dim3((unsigned)a.b), dim3(NB_WIDE_THREADS), 0, st, true, a);
    return launch_status();
}

struct RotaryShape { int64_t batch, seq, heads, rotated, head_dim; bool adjacent, in_place; };

template <typename T, int V, bool ADJACENT, int HEADS>
pamm_status launch_rotary(RotaryArgs a, const RotaryShape& g, cudaStream_t st) {
    const int per_turn = ADJACENT ? (V == 1 ? 2 : V) : 2 * V;             // elements of a turned unit
    a.turns = a.rot / per_turn;
    const int64_t rest = g.in_place ? 0 : (g.head_dim - a.rot) / V, whole = g.in_place ? 0 : g.head_dim / V;
    a.turned_step = (int)((g.rotated + HEADS - 1) / HEADS);
    a.whole_step = (int)((g.heads - g.rotated + HEADS - 1) / HEADS);
    a.turned_units = (int)(a.turned_step * (a.turns + rest));
    const int64_t units = a.turned_units + a.whole_step * whole;
    if (units == 0) return PAMM_OK;
    a.tokens = g.batch * g.seq;
    a.heads = (int)g.heads; a.rotated = (int)g.rotated;
    a.seq = make_divisor((uint32_t)g.seq);
    a.units = make_divisor((uint32_t)units);
    a.per_turned = make_divisor((uint32_t)(a.turns + rest));
    a.per_whole = make_divisor((uint32_t)std::max<int64_t>(1, whole));
    // 128 threads a block or a little less where several tokens of few units share one, at most 256 of a token of many
    a.tokens_per_block = (int)std::max<int64_t>(1, std::min<int64_t>(128 / units, a.tokens));
    const int64_t work = a.tokens_per_block * units, parts = (work + 255) / 256;
    const int threads = (int)round_up((work + parts - 1) / parts, 32);
    // a token of 2^24 units has 65536 parts, one more than a grid's y holds: the largest go along z as well
    const unsigned deep = (unsigned)((parts + 65534) / 65535);
    const dim3 grid((unsigned)((a.tokens + a.tokens_per_block - 1) / a.tokens_per_block), (unsigned)((parts + deep - 1) / deep), deep);
    launch(rotary_kernel<T, V, ADJACENT, HEADS>, grid, dim3(threads), 0, st, true, a);
    return launch_status();
}
template <typename T, int V>
pamm_status launch_rotary(const RotaryArgs& a, const RotaryShape& g, cudaStream_t st) {
    return g.adjacent ? launch_rotary<T, V, true, 8>(a, g, st) : launch_rotary<T, V, false, 4>(a, g, st);
}
// `width`: the elements, a power of two, that everything the call touches is a multiple of and aligned to
template <typename T>
pamm_status launch_rotary(const RotaryArgs& a, const RotaryShape& g, int width, cudaStream_t st) {
    if constexpr (sizeof(T) == 2)
        if (width >= 8) return launch_rotary<T, 8>(a, g, st);
    if (width >= 4) return launch_rotary<T, 4>(a, g, st);
    return width >= 2 ? launch_rotary<T, 2>(a, g, st) : launch_rotary<T, 1>(a, g, st);
}

// A launch whose parameters are too large to be copied from call to call.
template <typename... A>
void launch_in_place(const void* kern, unsigned grid, int block, cudaStream_t st, A*... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void* pointers[] = {(void*)args...};
    cudaLaunchKernelExC(&cfg, kern, pointers);
    g_launches += 1;
}

pamm_status check_tensors(const pamm_tensor* t, int64_t count) {
    if (count < 0 || (count > 0 && !t)) return PAMM_ERR_INVALID_ARG;
    for (int64_t i = 0; i < count; ++i) {
        if (t[i].dt != PAMM_F32 && t[i].dt != PAMM_BF16) return PAMM_ERR_UNSUPPORTED;
        if (t[i].rows < 0 || t[i].cols < 0 || t[i].rows > (1ll << 40) || t[i].cols > (1ll << 40)) return PAMM_ERR_INVALID_ARG;
        if (t[i].rows == 0 || t[i].cols == 0) continue;
        if (!t[i].data || !aligned(t[i].data, esize((pamm_dtype)t[i].dt)) || (t[i].rows > 1 && t[i].ld < t[i].cols))
            return PAMM_ERR_INVALID_ARG;
        if (t[i].rows > (1ll << 40) / t[i].cols) return PAMM_ERR_INVALID_ARG;
    }
    return PAMM_OK;
}

// Fills the list with the tensors from `at` on that one launch holds; returns the first one left.
template <int CAP>
int64_t fill_grad_list(GradList<CAP>& list, const pamm_tensor* in, const pamm_tensor* out, int64_t at, int64_t count, int chunk) {
    list.count = 0;
    list.chunks = 0;
    list.in_place = 1;
    list.chunk = chunk;
    for (; at < count && list.count < CAP; ++at) {
        const pamm_tensor& t = in[at];
        const pamm_tensor& o = out ? out[at] : t;
        if (t.rows == 0 || t.cols == 0) continue;
        GradEntry& e = list.e[list.count++];
        e.in = t.data;
        e.out = o.data;
        e.in_bf16 = t.dt == PAMM_BF16;
        e.out_bf16 = o.dt == PAMM_BF16;
        if (t.data != o.data || t.dt != o.dt || (t.rows > 1 && t.ld != o.ld)) list.in_place = 0;
        const bool dense = t.rows == 1 || (t.ld == t.cols && o.ld == o.cols);       // one long row
        e.rows = dense ? 1 : t.rows;
        e.cols = dense ? t.rows * t.cols : t.cols;
        e.ld_in = t.ld;
        e.ld_out = o.ld;
        e.first_chunk = list.chunks;
        e.pieces = (e.cols + chunk - 1) / chunk;
        e.off = dense ? (int)(reinterpret_cast<uintptr_t>(t.data) % 16 / esize((pamm_dtype)t.dt)) : 0;
        list.chunks += grad_chunks(e.rows, e.cols + e.off, chunk);
    }
    return at;
}

template <int CAP>
pamm_status run_grad_clip(const pamm_tensor* in, const pamm_tensor* out, int64_t count, bool scale, double max_norm, float* norm,
                          double* partial, cudaStream_t st) {
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) total += in[i].rows * in[i].cols;
    // chunks: some for every block of the sum, few enough that finding its place costs a block little
    int chunk = GC_MIN_CHUNK;
    while (chunk < GC_MAX_CHUNK && (int64_t)chunk * 4 * grad_norm_blocks() < total) chunk *= 2;
    GradList<CAP> list;
    int64_t at = fill_grad_list(list, in, nullptr, 0, count, chunk);
    // one list: as many blocks as there are chunks; several: the same blocks for each, whose sums go on
    int parts = at < count ? grad_norm_blocks() : (int)std::max<int64_t>(1, std::min<int64_t>(list.chunks, grad_norm_blocks()));
    list.add = 0;
    for (;;) {
        launch_in_place((const void*)grad_squares_kernel<CAP>, (unsigned)parts, GC_THREADS, st, &list, &partial);
        if (at >= count) break;
        at = fill_grad_list(list, in, nullptr, at, count, chunk);
        list.add = 1;
    }
    const double* sums = partial;
    GradFactor* factor = (GradFactor*)(partial + round_up(grad_norm_blocks(), 32));
    // Few sums are joined by each of the scaling's blocks, which saves a launch.  24 fp32 tensors, joined there and apart: in place, below the
    // limit, 6 M elements 7.8 and 8.1 us, 14 M 13.4 and 13.4 (13.7 and 14.0 a call among others), 18 M 17.1 and 16.3; into others, where all blocks
    // go on, 1 M 7.0 and 8.0, 2 M 7.9 and 8.6 (10.0 and 9.3 a call), 3 M 9.7 and 10.4 (12.2 and 11.5), 4 M 16.1 and 11.8
    int self = scale && total <= (out ? 2 << 20 : 14 << 20) ? parts : 0;
    if (!self) launch_in_place((const void*)grad_norm_finish_kernel, 1, GC_THREADS, st, &sums, &parts, &max_norm, &norm, &factor);
    if (!scale) return launch_status();
    at = 0;
    do {
        at = fill_grad_list(list, in, out, at, count, GC_SCALE_CHUNK);
        // several waves of blocks stream faster than one (403 MB of bf16 into fp32, the whole call: 342 us with 1, 318 with 4,
        // 309 with a block a chunk); fewer in place, where every block returns at once below the limit (400 MB: 70 us with
        // one wave, 72 with 4, 75 with 8).  One block at least, which writes the norm.
        const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(list.chunks, (int64_t)grad_norm_blocks() * (list.in_place ? 4 : 8)));
        const GradFactor* f = factor;
        launch_in_place((const void*)grad_scale_kernel<CAP>, (unsigned)blocks, GC_THREADS, st, &list, &f, &sums, &self, &max_norm, &norm);
    } while (at < count);
    return launch_status();
}

pamm_status grad_clip(const pamm_tensor* in, const pamm_tensor* out, int64_t count, bool scale, double max_norm, float* norm,
                      void* workspace, size_t ws_bytes, void* stream) {
    pamm_status s = check_tensors(in, count);
    if (s != PAMM_OK) return s;
    if (out) {
        s = check_tensors(out, count);
        if (s != PAMM_OK) return s;
        for (int64_t i = 0; i < count; ++i)
            if (out[i].rows != in[i].rows || out[i].cols != in[i].cols) return PAMM_ERR_INVALID_ARG;
    }
    if (!norm || !aligned(norm, 4) || !(max_norm >= 0.0)) return PAMM_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || ws_bytes < grad_norm_ws_bytes()) return PAMM_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    double* partial = (double*)workspace;
    if (count <= GC_SMALL) return run_grad_clip<GC_SMALL>(in, out, count, scale, max_norm, norm, partial, st);
    if (count <= GC_MEDIUM) return run_grad_clip<GC_MEDIUM>(in, out, count, scale, max_norm, norm, partial, st);
    return run_grad_clip<GC_LARGE>(in, out, count, scale, max_norm, norm, partial, st);
}

// ---- attention ------------------------------------------------------------------------------------
struct AttentionShape { int64_t batch, seq, heads, kv_heads, d, sequences; };

// A tensor of the call: its address and distances, where a distance between the only one of something and its next does not count.
bool heads_view(const pamm_heads* t, const AttentionShape& g, int64_t heads, size_t es, bool output, HeadsView& out) {
    if (!t || !t->data || !aligned(t->data, es)) return false;
    out = {t->data, g.batch > 1 ? t->batch : 0, g.seq > 1 ? t->token : 0, heads > 1 ? t->head : 0};
    return !output || ((g.batch == 1 || out.batch != 0) && (g.seq == 1 || out.token != 0) && (heads == 1 || out.head != 0));
}
// No output begins where an input or another output does: that much of an overlap is seen here.
bool begin_apart(std::initializer_list<const void*> inputs, std::initializer_list<const void*> outputs) {
    for (auto y = outputs.begin(); y != outputs.end(); ++y)
        if (std::find(inputs.begin(), inputs.end(), *y) != inputs.end() || std::find(outputs.begin(), y, *y) != y) return false;
    return true;
}
// Whole 16-byte vectors on memory's grid in every row.
bool heads_aligned(const HeadsView& t, size_t es, int64_t to = 16) {
    const auto on = [&](int64_t stride) { return stride * (int64_t)es % to == 0; };
    return aligned(t.p, (size_t)to) && on(t.batch) && on(t.token) && on(t.head);
}

pamm_status check_attention(const AttentionShape& g, pamm_dtype dt, float scale, const void* lengths, const void* starts,
                            pamm_position_type index_type) {
    if (!dtype_ok(dt) || ((lengths || starts) && index_type != PAMM_POS_I32 && index_type != PAMM_POS_I64)) return PAMM_ERR_UNSUPPORTED;
    if (g.batch < 0 || g.seq < 0 || g.heads < 0 || g.kv_heads < 0 || g.d < 1 || !(scale > 0.f) || !std::isfinite(scale)) return PAMM_ERR_INVALID_ARG;
    if (lengths && starts) return PAMM_ERR_INVALID_ARG;
    if (starts && (g.batch != 1 || g.sequences < 0)) return PAMM_ERR_INVALID_ARG;
    if (g.heads > 0 ? g.kv_heads == 0 || g.heads % g.kv_heads : g.kv_heads > 0) return PAMM_ERR_INVALID_ARG;
    const size_t entry = index_type == PAMM_POS_I64 ? 8 : 4;
    if ((lengths && !aligned(lengths, entry)) || (starts && !aligned(starts, entry))) return PAMM_ERR_INVALID_ARG;
    if (g.d > ATT_MAX_DIM || g.batch > MAX_ROWS || g.seq > MAX_ROWS || g.heads > MAX_ROWS || (starts && g.sequences > MAX_ROWS - 2))
        return PAMM_ERR_UNSUPPORTED;
    if (g.batch == 0 || g.seq == 0 || g.heads == 0) return PAMM_OK;
    const int64_t most = 1ll << 40;
    if (g.batch > most / g.seq || g.batch * g.seq > most / g.heads) return PAMM_ERR_UNSUPPORTED;
    const int64_t tiles = starts ? g.seq / AG_ROWS + g.sequences + 2 : g.batch * ((g.seq + AG_ROWS - 1) / AG_ROWS);
    return tiles > MAX_ROWS / g.heads ? PAMM_ERR_UNSUPPORTED : PAMM_OK;
}
// Tiles of all sequences, one head's; an upper bound where packed.
inline int tiles_of(const Sequences& s, int64_t size) {
    return (int)(s.starts ? s.seq / size + s.count + 2 : s.batch * ((s.seq + size - 1) / size));
}
Sequences sequences_of(const AttentionShape& g, const void* lengths, const void* starts, pamm_position_type index_type) {
    return {lengths, starts, g.seq, (int)g.batch, starts ? (int)g.sequences : 0, index_type == PAMM_POS_I64};
}

template <typename T, int DP>
pamm_status launch_attention_forward_generic(const AttentionArgs& a, cudaStream_t st) {
    const size_t smem = ag_smem<DP, false>;
    if (!ensure_dynamic_smem((const void*)attention_forward_generic_kernel<T, DP>, smem)) return PAMM_ERR_CUDA;
    const int items = tiles_of(a.s, AG_ROWS);
    launch(attention_forward_generic_kernel<T, DP>, dim3((unsigned)items * a.heads), dim3(AG_THREADS), smem, st, true, a,
           attention_order(a.s, a.heads, AG_ROWS, sm_count(), a.causal));
    return launch_result("attention_forward_generic_kernel launch");
}
template <typename T, int DP>
pamm_status launch_attention_backward_generic(const AttentionArgs& a, cudaStream_t st) {
    const size_t smem = ag_smem<DP, true>;
    if (!ensure_dynamic_smem((const void*)attention_backward_generic_kernel<T, DP, false>, smem) ||
        !ensure_dynamic_smem((const void*)attention_backward_generic_kernel<T, DP, true>, smem))
        return PAMM_ERR_CUDA;
    const int items = tiles_of(a.s, AG_ROWS);
    const int kv = a.heads / a.group, sms = sm_count();
    launch(attention_backward_generic_kernel<T, DP, false>, dim3((unsigned)items * a.heads), dim3(AG_THREADS), smem, st, true, a,
           attention_order(a.s, a.heads, AG_ROWS, sms, a.causal));
    launch(attention_backward_generic_kernel<T, DP, true>, dim3((unsigned)items * kv), dim3(AG_THREADS), smem, st, true, a,
           attention_order(a.s, kv, AG_ROWS, sms, false));
    return launch_result("attention_backward_generic_kernel launch");
}
template <typename T>
pamm_status run_attention_generic(const AttentionArgs& a, bool back, cudaStream_t st) {
    if (a.d <= 64) return back ? launch_attention_backward_generic<T, 64>(a, st) : launch_attention_forward_generic<T, 64>(a, st);
    if (a.d <= 128) return back ? launch_attention_backward_generic<T, 128>(a, st) : launch_attention_forward_generic<T, 128>(a, st);
    return back ? launch_attention_backward_generic<T, 256>(a, st) : launch_attention_forward_generic<T, 256>(a, st);
}

template <int DP>
pamm_status launch_attention_forward(const AttentionArgs& a, const AttentionMaps& m, cudaStream_t st) {
    using Plan = AttentionPlan<DP>;
    if (!ensure_dynamic_smem((const void*)attention_forward_kernel<DP>, Plan::SMEM)) return PAMM_ERR_CUDA;
    const int items = tiles_of(a.s, AF_QUERIES);
    launch(attention_forward_kernel<DP>, dim3((unsigned)(items * a.heads)), dim3(AU_THREADS), Plan::SMEM, st, true, a, m,
           attention_order(a.s, a.heads, AF_QUERIES, sm_count(), a.causal));
    return launch_result("attention_forward_kernel launch");
}

template <int DP>
pamm_status launch_attention_backward(const AttentionArgs& a, const AttentionMaps& m, cudaStream_t st) {
    using Plan = AttentionPlan<DP>;
    if (!ensure_dynamic_smem((const void*)attention_queries_backward_kernel<DP>, Plan::SMEM) ||
        !ensure_dynamic_smem((const void*)attention_keys_backward_kernel<DP>, Plan::SMEM))
        return PAMM_ERR_CUDA;
    const int items = tiles_of(a.s, AU_ROWS);
    const int kv = a.heads / a.group;
    launch(attention_queries_backward_kernel<DP>, dim3((unsigned)(items * a.heads)), dim3(AU_THREADS), Plan::SMEM, st, true, a, m,
           attention_order(a.s, a.heads, AU_ROWS, sm_count(), a.causal));
    launch(attention_keys_backward_kernel<DP>, dim3((unsigned)(items * kv)), dim3(AU_THREADS), Plan::SMEM, st, true, a, m,
           attention_order(a.s, kv, AU_ROWS, sm_count(), false));
    return launch_result("attention_keys_backward_kernel launch");
}

// Tensor maps need distances that go up, of whole 16-byte vectors (checked: a.vectors).
bool attention_on_tensor_cores(const AttentionArgs& a, pamm_dtype dt, bool back) {
    if (dt != PAMM_BF16 || a.d > 128 || !a.vectors) return false;
    const auto fits = [&](const HeadsView& t, int heads) {
        const auto up = [](int64_t n, int64_t ld) { return n == 1 || (ld > 0 && ld < (1ll << 38)); };
        return up(a.s.batch, t.batch) && up(a.s.seq, t.token) && up(heads, t.head);
    };
    const int kv = a.heads / a.group;
    return fits(a.q, a.heads) && fits(a.k, kv) && fits(a.v, kv) && (!back || fits(a.d_o, a.heads));
}
pamm_status run_attention(const AttentionArgs& a, pamm_dtype dt, bool back, cudaStream_t st) {
    if (attention_on_tensor_cores(a, dt, back)) {
        AttentionMaps m;
        const int kv = a.heads / a.group;
        if (!attention_map(&m.q, a.q, a.s, a.heads, a.d) || !attention_map(&m.k, a.k, a.s, kv, a.d) || !attention_map(&m.v, a.v, a.s, kv, a.d))
            return tensor_map_failed();
        m.d_o = m.q;       // not looked at in the forward pass
        if (back) {
            if (!attention_map(&m.d_o, a.d_o, a.s, a.heads, a.d)) return tensor_map_failed();
            return a.d <= 64 ? launch_attention_backward<64>(a, m, st) : launch_attention_backward<128>(a, m, st);
        }
        return a.d <= 64 ? launch_attention_forward<64>(a, m, st) : launch_attention_forward<128>(a, m, st);
    }
    return dt == PAMM_F32 ? run_attention_generic<float>(a, back, st) : run_attention_generic<__nv_bfloat16>(a, back, st);
}

template <typename T>
pamm_status run_dropout(DropoutArgs a, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    const auto grid = [](const void* p, int64_t ld, int64_t rows) { return !p || (aligned(p, 16) && (rows == 1 || ld % V == 0)); };
    const bool whole = (a.rows == 1 || a.n % V == 0) && grid(a.x, a.ldx, a.rows) && grid(a.r, a.ldr, a.rows) && grid(a.y, a.ldy, a.rows);
    const int64_t per = 256 * (whole ? V : 4);
    const dim3 blocks((unsigned)((a.total + per - 1) / per));
    if (whole) {
        if (a.r) launch(dropout_kernel<T, V, true>, blocks, dim3(256), 0, st, true, a);
        else launch(dropout_kernel<T, V, false>, blocks, dim3(256), 0, st, true, a);
    } else {
        if (a.r) launch(dropout_kernel<T, 1, true>, blocks, dim3(256), 0, st, true, a);
        else launch(dropout_kernel<T, 1, false>, blocks, dim3(256), 0, st, true, a);
    }
    return launch_result("dropout_kernel launch");
}

}  // namespace

extern "C" {

pamm_status pamm_attention_forward(const pamm_heads* Q, const pamm_heads* K, const pamm_heads* V, const pamm_heads* O, float* lse,
                                   int64_t batch, int64_t seq, int64_t heads, int64_t kv_heads, int64_t head_dim, pamm_dtype dt,
                                   float scale, int causal, const void* lengths, const void* starts, int64_t sequences,
                                   pamm_position_type index_type, void* stream) {
    const AttentionShape g = {batch, seq, heads, kv_heads, head_dim, sequences};
    const pamm_status s = check_attention(g, dt, scale, lengths, starts, index_type);
    if (s != PAMM_OK || batch == 0 || seq == 0 || heads == 0) return s;
    const size_t es = esize(dt);
    AttentionArgs a = {};
    if (!heads_view(Q, g, heads, es, false, a.q) || !heads_view(K, g, kv_heads, es, false, a.k) || !heads_view(V, g, kv_heads, es, false, a.v) ||
        !heads_view(O, g, heads, es, true, a.o) || !aligned(lse, 4) || !begin_apart({Q->data, K->data, V->data}, {O->data, lse}))
        return PAMM_ERR_INVALID_ARG;
    a.lse = lse;
    a.s = sequences_of(g, lengths, starts, index_type);
    a.heads = (int)heads; a.group = (int)(heads / kv_heads); a.d = (int)head_dim;
    a.scale = scale; a.causal = causal != 0;
    a.vectors = head_dim * (int64_t)es % 16 == 0 && heads_aligned(a.q, es) && heads_aligned(a.k, es) && heads_aligned(a.v, es) && heads_aligned(a.o, es);
    a.wide = head_dim * (int64_t)es % 32 == 0 && heads_aligned(a.o, es, 32);
    return run_attention(a, dt, false, (cudaStream_t)stream);
}

pamm_status pamm_attention_backward(const pamm_heads* dO, const pamm_heads* Q, const pamm_heads* K, const pamm_heads* V,
                                    const pamm_heads* O, const float* lse, const pamm_heads* dQ, const pamm_heads* dK,
                                    const pamm_heads* dV, int64_t batch, int64_t seq, int64_t heads, int64_t kv_heads,
                                    int64_t head_dim, pamm_dtype dt, float scale, int causal, const void* lengths, const void* starts,
                                    int64_t sequences, pamm_position_type index_type, void* workspace, size_t ws_bytes, void* stream) {
    const AttentionShape g = {batch, seq, heads, kv_heads, head_dim, sequences};
    const pamm_status s = check_attention(g, dt, scale, lengths, starts, index_type);
    if (s != PAMM_OK || batch == 0 || seq == 0 || heads == 0) return s;
    const size_t es = esize(dt);
    AttentionArgs a = {};
    if (!heads_view(dO, g, heads, es, false, a.d_o) || !heads_view(Q, g, heads, es, false, a.q) || !heads_view(K, g, kv_heads, es, false, a.k) ||
        !heads_view(V, g, kv_heads, es, false, a.v) || !heads_view(O, g, heads, es, false, a.o) || !heads_view(dQ, g, heads, es, true, a.dq) ||
        !heads_view(dK, g, kv_heads, es, true, a.dk) || !heads_view(dV, g, kv_heads, es, true, a.dv) || !lse || !aligned(lse, 4))
        return PAMM_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 16) || ws_bytes < attention_backward_ws_bytes(batch * seq, heads)) return PAMM_ERR_WORKSPACE;
    if (!begin_apart({dO->data, Q->data, K->data, V->data, O->data, lse}, {dQ->data, dK->data, dV->data, workspace})) return PAMM_ERR_INVALID_ARG;
    a.lse_in = lse;
    a.delta = static_cast<float*>(workspace);
    a.s = sequences_of(g, lengths, starts, index_type);
    a.heads = (int)heads; a.group = (int)(heads / kv_heads); a.d = (int)head_dim;
    a.scale = scale; a.causal = causal != 0;
    a.vectors = head_dim * (int64_t)es % 16 == 0;
    for (const HeadsView* t : {&a.q, &a.k, &a.v, &a.o, &a.d_o, &a.dq, &a.dk, &a.dv}) a.vectors = a.vectors && heads_aligned(*t, es);
    a.wide = head_dim * (int64_t)es % 32 == 0 && heads_aligned(a.dq, es, 32) && heads_aligned(a.dk, es, 32) && heads_aligned(a.dv, es, 32);
    return run_attention(a, dt, true, (cudaStream_t)stream);
}

pamm_status pamm_dropout(const void* X, int64_t ldx, const void* R, int64_t ldr, int64_t b, int64_t n, pamm_dtype dt, double p,
                         uint64_t seed, uint64_t offset, const int64_t* counter, void* Y, int64_t ldy, void* stream) {
    if (!dtype_ok(dt)) return PAMM_ERR_UNSUPPORTED;
    if (b < 0 || n < 0 || !(p >= 0.0 && p <= 1.0) || !aligned(counter, 8)) return PAMM_ERR_INVALID_ARG;
    if (b > (1ll << 40) || n > (1ll << 40) || (n > 0 && b > (1ll << 38) / n)) return PAMM_ERR_UNSUPPORTED;
    if (b == 0 || n == 0) return PAMM_OK;
    const size_t es = esize(dt);
    if (b == 1) ldx = ldr = ldy = n;
    if (!matrix_ok(X, ldx, n, es) || !matrix_ok(Y, ldy, n, es) || (R && !matrix_ok(R, ldr, n, es))) return PAMM_ERR_INVALID_ARG;
    if ((Y == X && ldy != ldx) || (Y == R && ldy != ldr)) return PAMM_ERR_INVALID_ARG;
    if (ldx == n && ldy == n && (!R || ldr == n)) {       // without gaps the rows are one
        n *= b;
        ldx = ldr = ldy = n;
        b = 1;
    }
    DropoutArgs a = {};
    a.x = X; a.r = R; a.y = Y; a.rows = b; a.n = n; a.ldx = ldx; a.ldr = ldr; a.ldy = ldy; a.total = b * n;
    a.counter = counter; a.offset = offset;
    dropout_keys(seed, a.keys);
    a.none = p == 1.0;
    a.threshold = a.none ? 0 : (uint32_t)(p * 4294967296.0);       // floor; below 2^32, p being the nearest double to 1 at most
    a.factor = p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.f;
    return dt == PAMM_F32 ? run_dropout<float>(a, (cudaStream_t)stream) : run_dropout<__nv_bfloat16>(a, (cudaStream_t)stream);
}

pamm_status pamm_norm_forward(pamm_norm_kind kind, const void* X, int64_t ldx, const void* R, int64_t ldr, int64_t b, int64_t n,
                              pamm_dtype dt, const void* w, const void* c, pamm_dtype w_dt, float eps, void* Y, int64_t ldy,
                              void* H, int64_t ldh, float* mean, float* rstd, void* stream) {
    if (!dtype_ok(dt) || !dtype_ok(w_dt) || (kind != PAMM_NORM_LAYER && kind != PAMM_NORM_RMS)) return PAMM_ERR_UNSUPPORTED;
    if (b < 0 || n < 1 || b > MAX_ROWS || !(eps >= 0.f)) return PAMM_ERR_INVALID_ARG;
    if (n > NORM_MAX_N) return PAMM_ERR_UNSUPPORTED;
    if (b == 0) return PAMM_OK;
    const size_t es = esize(dt), ws = esize(w_dt);
    if (!matrix_ok(X, ldx, n, es) || !matrix_ok(Y, ldy, n, es) || (R && !matrix_ok(R, ldr, n, es)) || (H && !matrix_ok(H, ldh, n, es)))
        return PAMM_ERR_INVALID_ARG;
    if (!aligned(w, ws) || !aligned(c, ws) || !aligned(mean, 4) || !aligned(rstd, 4) || H == Y) return PAMM_ERR_INVALID_ARG;
    NormForwardArgs a;
    a.x = X; a.r = R; a.w = w; a.c = c; a.y = Y; a.h = H; a.mean = mean; a.rstd = rstd;
    a.ldx = ldx; a.ldr = ldr; a.ldy = ldy; a.ldh = ldh; a.b = b;
    a.n = (int)n; a.warps = 0; a.eps = eps;
    a.rms = kind == PAMM_NORM_RMS;
    a.h_over_input = H && R && (H == X || H == R);
    const RowMatrix all[] = {{X, ldx}, {R, ldr}, {Y, ldy}, {H, ldh}};
    const RowAccess access = row_access(all, n, es, aligned(w, 16) && aligned(c, 16));
    cudaStream_t st = (cudaStream_t)stream;
    using bf16 = __nv_bfloat16;
    if (dt == PAMM_F32) return w_dt == PAMM_F32 ? launch_norm_forward<float, float>(a, access, st) : launch_norm_forward<float, bf16>(a, access, st);
    return w_dt == PAMM_F32 ? launch_norm_forward<bf16, float>(a, access, st) : launch_norm_forward<bf16, bf16>(a, access, st);
}

pamm_status pamm_norm_backward(pamm_norm_kind kind, const void* dY, int64_t lddy, const void* X, int64_t ldx, const float* mean,
                               const float* rstd, int64_t b, int64_t n, pamm_dtype dt, const void* w, pamm_dtype w_dt,
                               const void* dH, int64_t lddh, void* dX, int64_t lddx, void* dw, void* dc, pamm_dtype dw_dt,
                               void* workspace, size_t ws_bytes, void* stream) {
    if (!dtype_ok(dt) || !dtype_ok(w_dt) || !dtype_ok(dw_dt) || (kind != PAMM_NORM_LAYER && kind != PAMM_NORM_RMS))
        return PAMM_ERR_UNSUPPORTED;
    if (b < 0 || n < 1 || b > MAX_ROWS) return PAMM_ERR_INVALID_ARG;
    if (n > NORM_MAX_N) return PAMM_ERR_UNSUPPORTED;
    const size_t es = esize(dt);
    const bool rms = kind == PAMM_NORM_RMS;
    if (!aligned(w, esize(w_dt)) || !aligned(dw, esize(dw_dt)) || !aligned(dc, esize(dw_dt)) || (dw && dw == dc))
        return PAMM_ERR_INVALID_ARG;
    if (b > 0) {
        if (!matrix_ok(dY, lddy, n, es) || !matrix_ok(X, ldx, n, es) || !matrix_ok(dX, lddx, n, es) || (dH && !matrix_ok(dH, lddh, n, es)))
            return PAMM_ERR_INVALID_ARG;
        if (!rstd || !aligned(rstd, 4) || (!rms && !mean) || !aligned(mean, 4)) return PAMM_ERR_INVALID_ARG;
    }
    if ((dw || dc) && (!workspace || !aligned(workspace, 256) || ws_bytes < norm_backward_ws_bytes(b, n))) return PAMM_ERR_WORKSPACE;
    if (b == 0 && !dw && !dc) return PAMM_OK;
    NormBackwardArgs a;
    a.dy = dY; a.x = X; a.w = w; a.dh = dH; a.mean = mean; a.rstd = rstd; a.dx = dX; a.dw = dw; a.dc = dc;
    a.part = dw || dc ? (float*)workspace : nullptr;
    a.lddy = lddy; a.ldx = ldx; a.lddh = lddh; a.lddx = lddx; a.b = b; a.rows_per_split = 0;
    a.n = (int)n; a.pitch = (int)round_up(n, 8); a.splits = a.warps = a.groups = a.period = 0;
    a.rms = rms; a.w_bf16 = w_dt == PAMM_BF16; a.dw_bf16 = dw_dt == PAMM_BF16;
    const RowMatrix all[] = {{X, ldx}, {dY, lddy}, {dH, lddh}, {dX, lddx}};
    const RowAccess access = row_access(all, n, es, aligned(w, 16));
    cudaStream_t st = (cudaStream_t)stream;
    return dt == PAMM_F32 ? launch_norm_backward<float>(a, access, st) : launch_norm_backward<__nv_bfloat16>(a, access, st);
}

pamm_status pamm_rotary_frequencies_host(int64_t rot_dim, double base, pamm_rotary_scaling scaling, double factor,
                                         int64_t trained_length, double slow, double fast, double* freq, double* amplitude) {
    if (!freq || !amplitude || rot_dim < 2 || rot_dim % 2 || !(base > 0.0) || std::isinf(base)) return PAMM_ERR_INVALID_ARG;
    if (rot_dim > ROTARY_MAX_ROT) return PAMM_ERR_UNSUPPORTED;
    if (scaling < PAMM_ROTARY_PLAIN || scaling > PAMM_ROTARY_PARTS) return PAMM_ERR_UNSUPPORTED;
    if (scaling != PAMM_ROTARY_PLAIN && (!(factor >= 1.0) || std::isinf(factor))) return PAMM_ERR_INVALID_ARG;
    if (scaling == PAMM_ROTARY_PARTS && (trained_length < 1 || !(slow >= 0.0) || !(fast > slow))) return PAMM_ERR_INVALID_ARG;
    if (scaling == PAMM_ROTARY_BASE && rot_dim > 2) base *= pow(factor, (double)rot_dim / (double)(rot_dim - 2));
    *amplitude = scaling == PAMM_ROTARY_PARTS ? 0.1 * log(factor) + 1.0 : 1.0;
    for (int64_t i = 0; i < rot_dim / 2; ++i) {
        const double f = pow(base, -2.0 * (double)i / (double)rot_dim);
        double keep = 1.0;                        // share of the unscaled frequency
        if (scaling == PAMM_ROTARY_LINEAR) keep = 0.0;
        if (scaling == PAMM_ROTARY_PARTS) {
            const double turns = (double)trained_length * f / 6.283185307179586476925;
            keep = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
        }
        freq[i] = keep == 1.0 ? f : f / factor + keep * (f - f / factor);
    }
    return PAMM_OK;
}

pamm_status pamm_rotary_table(const double* freq, int64_t rot_dim, double amplitude, int64_t first, int64_t length, float* table,
                              void* stream) {
    if (!freq || rot_dim < 2 || rot_dim % 2 || length < 0 || first < 0 || first > (1ll << 50) || length > (1ll << 40))
        return PAMM_ERR_INVALID_ARG;
    if (rot_dim > ROTARY_MAX_ROT) return PAMM_ERR_UNSUPPORTED;
    if (length == 0) return PAMM_OK;
    if (!table || !aligned(table, 4)) return PAMM_ERR_INVALID_ARG;
    RotaryFrequencies f = {};
    std::copy(freq, freq + rot_dim / 2, f.f);
    const int64_t want = (length * (rot_dim / 2) + ROTARY_THREADS - 1) / ROTARY_THREADS;
    launch(rotary_table_kernel, dim3((unsigned)std::min<int64_t>(want, 8 * sm_count())), dim3(ROTARY_THREADS), 0, (cudaStream_t)stream,
           true, f, (int)(rot_dim / 2), amplitude, first, length, table);
    return launch_status();
}

pamm_status pamm_rotary(const void* X, int64_t x_batch, int64_t x_token, int64_t x_head, void* Y, int64_t y_batch, int64_t y_token,
                        int64_t y_head, int64_t batch, int64_t seq, int64_t heads, int64_t rotated, int64_t head_dim,
                        int64_t rot_dim, pamm_dtype dt, pamm_rotary_pairs pairs, int transposed, const float* table,
                        int64_t table_rows, const void* positions, pamm_position_type pos_type, int64_t pos_batch,
                        int64_t pos_token, int64_t first, void* stream) {
    if (!dtype_ok(dt) || (pairs != PAMM_PAIRS_HALF && pairs != PAMM_PAIRS_ADJACENT)) return PAMM_ERR_UNSUPPORTED;
    if (positions && pos_type != PAMM_POS_I32 && pos_type != PAMM_POS_I64) return PAMM_ERR_UNSUPPORTED;
    if (batch < 0 || seq < 0 || heads < 0 || rotated < 0 || rotated > heads || head_dim < 1 || rot_dim < 2 || rot_dim % 2 ||
        rot_dim > head_dim)
        return PAMM_ERR_INVALID_ARG;
    if (rot_dim > ROTARY_MAX_ROT || seq > MAX_ROWS || heads > ROTARY_MAX_ROW || head_dim > ROTARY_MAX_ROW || heads * head_dim > ROTARY_MAX_ROW ||
        (seq > 0 && batch > MAX_ROWS / seq))
        return PAMM_ERR_UNSUPPORTED;
    if (batch == 0 || seq == 0 || heads == 0) return PAMM_OK;
    const size_t es = esize(dt);
    if (!X || !Y || !table || !aligned(X, es) || !aligned(Y, es) || !aligned(table, 4) || table_rows < 1) return PAMM_ERR_INVALID_ARG;
    if (positions ? !aligned(positions, pos_type == PAMM_POS_I64 ? 8 : 4)
                  : first < 0 || first > table_rows || seq > table_rows - first)
        return PAMM_ERR_INVALID_ARG;
    // a distance between the only one of something and its next does not count
    if (batch == 1) x_batch = y_batch = 0;
    if (seq == 1) x_token = y_token = 0;
    if (heads == 1) x_head = y_head = 0;
    // the same matrix in and out is turned in place; other overlaps are the caller's error
    const bool in_place = X == (const void*)Y;
    if (in_place && (x_batch != y_batch || x_token != y_token || x_head != y_head)) return PAMM_ERR_INVALID_ARG;
    RotaryArgs a = {};
    a.x = X; a.y = Y; a.table = table; a.positions = positions;
    a.xb = x_batch; a.xs = x_token; a.xh = x_head; a.yb = y_batch; a.ys = y_token; a.yh = y_head;
    a.pb = pos_batch; a.ps = pos_token; a.table_rows = table_rows; a.first = first;
    a.rot = (int)rot_dim; a.transposed = transposed != 0; a.pos64 = pos_type == PAMM_POS_I64;
    const RotaryShape g = {batch, seq, heads, rotated, head_dim, pairs == PAMM_PAIRS_ADJACENT, in_place};
    // the lowest bit of all sizes, distances and addresses (in elements): the widest access that fits everything
    uint64_t bits = (uint64_t)(16 / es) | (uint64_t)head_dim | (uint64_t)(g.adjacent ? rot_dim : rot_dim / 2) |
                    reinterpret_cast<uintptr_t>(X) / es | reinterpret_cast<uintptr_t>(Y) / es | (uint64_t)x_batch | (uint64_t)x_token |
                    (uint64_t)x_head | (uint64_t)y_batch | (uint64_t)y_token | (uint64_t)y_head;
    const int width = aligned(table, 16) ? (int)(bits & (~bits + 1)) : 1;
    cudaStream_t st = (cudaStream_t)stream;
    return dt == PAMM_F32 ? launch_rotary<float>(a, g, width, st) : launch_rotary<__nv_bfloat16>(a, g, width, st);
}

pamm_status pamm_grad_norm(const pamm_tensor* grads, int64_t count, float* norm, void* workspace, size_t ws_bytes, void* stream) {
    return grad_clip(grads, nullptr, count, false, 0.0, norm, workspace, ws_bytes, stream);
}

pamm_status pamm_clip_grad_norm(const pamm_tensor* grads, const pamm_tensor* out, int64_t count, double max_norm, float* norm,
                                void* workspace, size_t ws_bytes, void* stream) {
    return grad_clip(grads, out, count, true, max_norm, norm, workspace, ws_bytes, stream);
}


pamm_status pamm_selftest_bounded_wait(void* stream) {
    launch(selftest_bounded_wait_kernel, dim3(1), dim3(64), 0, (cudaStream_t)stream, false, (uint32_t)2048);
    return launch_status();
}

pamm_status pamm_selftest_progress_wait(void* stream) {
    launch(selftest_progress_wait_kernel, dim3(1), dim3(64), 0, (cudaStream_t)stream, false, (uint32_t)256);
    return launch_status();
}

pamm_status pamm_probe_read(pamm_probe_kind kind, const void* base, int64_t rows, int64_t row_bytes, int64_t ld_bytes,
                            const int32_t* order, uint32_t* sum32, void* stream) {
    if (!base || !sum32 || rows < 1 || row_bytes < 16 || row_bytes % 16 || ld_bytes < row_bytes || ld_bytes % 16 ||
        !aligned(base, 16) || !aligned(sum32, 4) || rows > MAX_ROWS)
        return PAMM_ERR_INVALID_ARG;
    if (kind != PAMM_PROBE_SUM && kind != PAMM_PROBE_ROWS) return PAMM_ERR_INVALID_ARG;
    if (kind == PAMM_PROBE_SUM && order) return PAMM_ERR_INVALID_ARG;
    if (kind == PAMM_PROBE_ROWS && (row_bytes > 24576 || (order && !aligned(order, 4)))) return PAMM_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemsetAsync(sum32, 0, 4, st) != cudaSuccess) return PAMM_ERR_CUDA;
    if (kind == PAMM_PROBE_SUM) {
        const int64_t vecs = rows * (row_bytes / 16);
        const int64_t want = (vecs + RP_SUM_THREADS - 1) / RP_SUM_THREADS;
        const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>(want, (int64_t)sm_count() * 4));
        launch(read_probe_sum_kernel, dim3(grid), dim3(RP_SUM_THREADS), 0, st, false, (const uint8_t*)base, rows, row_bytes,
               ld_bytes, sum32);
        return launch_status();
    }
    const int pitch = (int)round_up(row_bytes, 128);
    const int slots = std::max(2, std::min(RP_MAX_SLOTS, RP_RING_BYTES / pitch));
    const size_t smem = 128 + (size_t)slots * pitch;
    if (!ensure_dynamic_smem((const void*)read_probe_rows_kernel, smem)) return PAMM_ERR_CUDA;
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>(rows, (int64_t)sm_count() * 2));
    launch(read_probe_rows_kernel, dim3(grid), dim3(RP_ROW_THREADS), smem, st, false, (const uint8_t*)base, rows,
           (uint32_t)row_bytes, ld_bytes, order, slots, pitch, sum32);
    return launch_status();
}

const char* pamm_status_string(pamm_status s) {
    switch (s) {
        case PAMM_OK: return "ok";
        case PAMM_ERR_INVALID_ARG: return "invalid argument";
        case PAMM_ERR_UNSUPPORTED: return "unsupported dtype or shape";
        case PAMM_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case PAMM_ERR_CUDA: return "CUDA error";
        case PAMM_ERR_TIMEOUT: return "a bounded device-side wait ran out";
        case PAMM_ERR_BAD_INDEX: return "index out of range or duplicated on the device";
    }
    return "unknown status";
}

int pamm_version(void) { return 200; }

const char* pamm_last_error_detail(void) { return g_cuda_detail; }

unsigned long long pamm_launch_count(void) { return g_launches; }

pamm_status pamm_set_profile_events(pamm_prof_kind kind, void* start_event, void* stop_event) {
    if ((int)kind < 0 || (int)kind > 2) return PAMM_ERR_INVALID_ARG;
    g_prof[kind][0] = (cudaEvent_t)start_event;
    g_prof[kind][1] = (cudaEvent_t)stop_event;
    return PAMM_OK;
}

size_t pamm_workspace_bytes(pamm_ws_kind kind, int64_t b, int64_t n, int64_t m, int64_t k, pamm_dtype dt) {
    if (kind == PAMM_WS_NORM_BACKWARD) {
        if (!dtype_ok(dt) || b < 0 || b > MAX_ROWS || n < 1 || n > NORM_MAX_N) return (size_t)-1;
        return norm_backward_ws_bytes(b, n);
    }
    if (kind == PAMM_WS_GRAD_NORM) return grad_norm_ws_bytes();
    if (kind == PAMM_WS_ATTENTION_BACKWARD) {
        if (b < 0 || n < 0 || (n > 0 && b > (1ll << 40) / n)) return (size_t)-1;
        return std::max<size_t>(256, attention_backward_ws_bytes(b, n));
    }
    if (!dtype_ok(dt) || b < 1 || k < 1 || k > b || b > MAX_ROWS) return (size_t)-1;
    switch (kind) {
        case PAMM_WS_COMPRESS:
            if (n < 1) return (size_t)-1;
            return sort_products_bytes(b, k);
        case PAMM_WS_CONTRACT:
            if (m < 1) return (size_t)-1;
            return contract_ws(nullptr, b, m, k).bytes_with_planes;     // pamm_contract itself needs less
        case PAMM_WS_STEP_HOST:
            if (n < 1 || m < 1) return (size_t)-1;
            return step_arena_layout(nullptr, b, n, m, k, dt).bytes;
        default: break;
    }
    return (size_t)-1;
}

pamm_status pamm_saved_bytes(int64_t b, int64_t n, int64_t k, pamm_dtype dt, pamm_index_type f_type, int64_t out[4]) {
    if (!dtype_ok(dt) || !index_type_ok(f_type)) return PAMM_ERR_UNSUPPORTED;
    if (!out || b < 1 || n < 1 || k < 1 || k > b || k > index_limit(f_type)) return PAMM_ERR_INVALID_ARG;
    const int64_t e = (int64_t)esize(dt);
    out[0] = b * n * e;                                             // X itself
    out[1] = k * n * e + b * (int64_t)index_size(f_type) + b * 4;   // C, f, alpha
    out[2] = b * n;                                                 // scalars, as the paper counts them
    out[3] = k * n + 2 * b;
    return PAMM_OK;
}

pamm_status pamm_draw_indices_host(int64_t b, int64_t k, uint64_t seed, int32_t* idx_out) {
    if (!idx_out || b < 1 || k < 1 || k > b || b > MAX_ROWS) return PAMM_ERR_INVALID_ARG;
    const PermKey pk = make_perm_key(seed, (uint32_t)b);
    for (int64_t j = 0; j < k; ++j) idx_out[j] = (int32_t)perm_apply(pk, (uint32_t)j);
    std::sort(idx_out, idx_out + k);
    return PAMM_OK;
}

pamm_status pamm_select_generators(const void* X, int64_t ldx, int64_t b, int64_t n, pamm_dtype dt, int64_t k,
                                   uint64_t seed, const int32_t* idx_in, int32_t* idx_out, void* C, int64_t ldc,
                                   float* c_invnorm, void* stream) {
    pamm_status s = check_select(X, ldx, b, n, dt, k, idx_out, C, ldc, c_invnorm);
    if (s != PAMM_OK) return s;
    cudaStream_t st = (cudaStream_t)stream;
    return dt == PAMM_F32 ? launch_select<float>(X, ldx, b, n, k, seed, idx_in, idx_out, C, ldc, c_invnorm, st)
                          : launch_select<__nv_bfloat16>(X, ldx, b, n, k, seed, idx_in, idx_out, C, ldc, c_invnorm, st);
}

pamm_status pamm_compress(const void* X, int64_t ldx, int64_t b, int64_t n, pamm_dtype dt, const void* C, int64_t ldc,
                          int64_t k, const float* c_invnorm, void* f, pamm_index_type f_type, float* alpha,
                          void* workspace, size_t ws_bytes, void* stream) {
    pamm_status s = check_compress(X, ldx, b, n, dt, C, ldc, k, c_invnorm, f, f_type, alpha);
    if (s != PAMM_OK) return s;
    s = check_products_out(workspace, ws_bytes, b, k, 1);
    if (s != PAMM_OK) return s;
    return do_compress(X, ldx, b, n, dt, C, ldc, k, 1, c_invnorm, f, f_type, alpha, b, (int32_t*)workspace, false,
                       (cudaStream_t)stream);
}

pamm_status pamm_compress_projections(const void* X, int64_t ldx, int64_t b, int64_t n, pamm_dtype dt, const void* C,
                                      int64_t ldc, int64_t k, int64_t sets, const float* c_invnorm, void* f,
                                      pamm_index_type f_type, float* alpha, int64_t out_stride, void* workspace,
                                      size_t ws_bytes, void* stream) {
    pamm_status s = check_compress(X, ldx, b, n, dt, C, ldc, k, c_invnorm, f, f_type, alpha);
    if (s != PAMM_OK) return s;
    if (sets < 1 || sets > 64 || out_stride < b || (out_stride * (int64_t)index_size(f_type)) % 4) return PAMM_ERR_INVALID_ARG;
    s = check_products_out(workspace, ws_bytes, b, k, (int)sets);
    if (s != PAMM_OK) return s;
    return do_compress(X, ldx, b, n, dt, C, ldc, k, (int)sets, c_invnorm, f, f_type, alpha, out_stride, (int32_t*)workspace,
                       false, (cudaStream_t)stream);
}

pamm_status pamm_compress_fused(const void* X, int64_t ldx, int64_t b, int64_t n, pamm_dtype dt, int64_t k,
                                uint64_t seed, const int32_t* idx_in, int32_t* idx_out, void* C, int64_t ldc,
                                float* c_invnorm, void* f, pamm_index_type f_type, float* alpha, void* workspace,
                                size_t ws_bytes, void* stream) {
    pamm_status s = check_select(X, ldx, b, n, dt, k, idx_out, C, ldc, c_invnorm);
    if (s != PAMM_OK) return s;
    s = check_compress(X, ldx, b, n, dt, C, ldc, k, c_invnorm, f, f_type, alpha);
    if (s != PAMM_OK) return s;
    s = check_products_out(workspace, ws_bytes, b, k, 1);
    if (s != PAMM_OK) return s;
    cudaStream_t st = (cudaStream_t)stream;
    // a handful of generators: selection and compression in one launch, generator rows kept in shared memory
    if (dt == PAMM_F32 && small_k_compress_supported<float>(n, k))
        return launch_small_forward<float>(X, ldx, b, n, k, seed, idx_in, idx_out, C, ldc, c_invnorm, f, (int)f_type, alpha, st);
    if (dt == PAMM_BF16 && small_k_compress_supported<__nv_bfloat16>(n, k))
        return launch_small_forward<__nv_bfloat16>(X, ldx, b, n, k, seed, idx_in, idx_out, C, ldc, c_invnorm, f, (int)f_type,
                                                   alpha, st);
    s = dt == PAMM_F32 ? launch_select<float>(X, ldx, b, n, k, seed, idx_in, idx_out, C, ldc, c_invnorm, st)
                       : launch_select<__nv_bfloat16>(X, ldx, b, n, k, seed, idx_in, idx_out, C, ldc, c_invnorm, st);
    if (s != PAMM_OK) return s;
    return do_compress(X, ldx, b, n, dt, C, ldc, k, 1, c_invnorm, f, f_type, alpha, b, (int32_t*)workspace, true, st);
}

pamm_status pamm_linear_forward(const void* X, int64_t ldx, int64_t b, int64_t n, const void* W, int64_t ldw, int64_t m,
                                pamm_dtype dt, int64_t k, uint64_t seed, const int32_t* idx_in, int32_t* idx_out,
                                void* C, int64_t ldc, float* c_invnorm, void* Z, int64_t ldz, void* f,
                                pamm_index_type f_type, float* alpha, void* workspace, size_t ws_bytes, void* stream) {
    if (!dtype_ok(dt)) return PAMM_ERR_UNSUPPORTED;
    if (!X || !W || !Z || b < 1 || n < 1 || m < 1 || k < 0 || b > MAX_ROWS) return PAMM_ERR_INVALID_ARG;
    if (!ld_ok(ldx, n, esize(dt)) || !ld_ok(ldw, m, esize(dt)) || !ld_ok(ldz, m, esize(dt))) return PAMM_ERR_INVALID_ARG;
    if (!aligned(X, 16) || !aligned(W, 16) || !aligned(Z, 16)) return PAMM_ERR_INVALID_ARG;
    pamm_status s = PAMM_OK;
    if (k > 0) {
        s = check_select(X, ldx, b, n, dt, k, idx_out, C, ldc, c_invnorm);
        if (s != PAMM_OK) return s;
        s = check_compress(X, ldx, b, n, dt, C, ldc, k, c_invnorm, f, f_type, alpha);
        if (s != PAMM_OK) return s;
        s = check_products_out(workspace, ws_bytes, b, k, 1);
        if (s != PAMM_OK) return s;
    }
    // the tensor-core kernel is the only implementation: no CUDA-core or library GEMM stands in for it
    if (dt != PAMM_BF16 || !linear_forward_supported(b, n, m, k) ||
        linear_forward_plan_for(b, m, k, sm_count()).stages < 2)
        return PAMM_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    const int64_t rpb = sort_rows_per_block(b);
    int32_t* hist = k > 0 ? (int32_t*)workspace : nullptr;
    if (k > 0) {
        s = launch_select<__nv_bfloat16>(X, ldx, b, n, k, seed, idx_in, idx_out, C, ldc, c_invnorm, st, hist,
                                         hist ? ((b + rpb - 1) / rpb) * k : 0);
        if (s != PAMM_OK) return s;
    }
    const LinearForwardOut out = {f, alpha, hist, (int)rpb, (int)f_type};
    // pairs of CTAs on one 256-row tile wherever there are at least 256 rows; else one CTA per 128-row tile
    const LinearForwardPlan pp = linear_forward_pair_plan_for(b, m, k, sm_count());
    const bool pairs = b >= LP_PAIR_M && sm_count() >= 2 && pp.stages >= 2 &&
                       cta_pairs_can_launch((const void*)linear_forward_pair_kernel, LF_THREADS, pp.smem_bytes);
    prof_begin(PAMM_PROF_COMPRESS, st);
    s = pairs ? launch_linear_forward_pair(X, ldx, b, n, W, ldw, m, C, ldc, k, c_invnorm, Z, ldz, out, sm_count(), st)
              : launch_linear_forward(X, ldx, b, n, W, ldw, m, C, ldc, k, c_invnorm, Z, ldz, out, sm_count(), st);
    prof_end(PAMM_PROF_COMPRESS, st);
    g_launches += 1;
    return s;
}

pamm_status pamm_linear_backward_input(const void* dZ, int64_t lddz, int64_t b, int64_t m, const void* W, int64_t ldw,
                                       int64_t n, pamm_dtype dt, void* dX, int64_t lddx, void* stream) {
    if (!dtype_ok(dt)) return PAMM_ERR_UNSUPPORTED;
    if (!dZ || !W || !dX || b < 1 || n < 1 || m < 1 || b > MAX_ROWS) return PAMM_ERR_INVALID_ARG;
    if (!ld_ok(lddz, m, esize(dt)) || !ld_ok(ldw, m, esize(dt)) || !ld_ok(lddx, n, esize(dt))) return PAMM_ERR_INVALID_ARG;
    if (!aligned(dZ, 16) || !aligned(W, 16) || !aligned(dX, 16)) return PAMM_ERR_INVALID_ARG;
    // the forward kernel with the roles renamed: rows of dZ, contraction over m, n output columns, W as columns x hidden
    if (dt != PAMM_BF16 || !linear_forward_supported(b, m, n, 0) || linear_forward_plan_for(b, n, 0, sm_count()).stages < 2)
        return PAMM_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    const LinearForwardOut out = {nullptr, nullptr, nullptr, 1, (int)PAMM_IDX_I32};
    const LinearForwardPlan pp = linear_forward_pair_plan_for(b, n, 0, sm_count());
    const bool pairs = b >= LP_PAIR_M && sm_count() >= 2 && pp.stages >= 2 &&
                       cta_pairs_can_launch((const void*)linear_forward_pair_kernel, LF_THREADS, pp.smem_bytes);
    const pamm_status s = pairs
        ? launch_linear_forward_pair(dZ, lddz, b, m, W, ldw, n, nullptr, 0, 0, nullptr, dX, lddx, out, sm_count(), st, true)
        : launch_linear_forward(dZ, lddz, b, m, W, ldw, n, nullptr, 0, 0, nullptr, dX, lddx, out, sm_count(), st, true);
    g_launches += 1;
    return s;
}

pamm_status pamm_contract(const void* f, pamm_index_type f_type, const float* alpha, const void* dY, int64_t ldy,
                          int64_t b, int64_t m, pamm_dtype dt, int64_t k, float* Btilde, int64_t ldb,
                          const void* sort_products, void* workspace, size_t ws_bytes, void* stream) {
    pamm_status s = check_contract(f, f_type, alpha, dY, ldy, b, m, dt, k, Btilde, ldb, true, sort_products, workspace, ws_bytes);
    if (s != PAMM_OK) return s;
    const ContractWs w = contract_ws(workspace, b, m, k);
    cudaStream_t st = (cudaStream_t)stream;
    const int32_t* pr = (const int32_t*)sort_products;
    return dt == PAMM_F32 ? launch_contract<float>(f, (int)f_type, alpha, dY, ldy, b, m, k, Btilde, ldb, pr, w, st)
                          : launch_contract<__nv_bfloat16>(f, (int)f_type, alpha, dY, ldy, b, m, k, Btilde, ldb, pr, w, st);
}

pamm_status pamm_weight_grad(const void* C, int64_t ldc, int64_t k, int64_t n, pamm_dtype dt, const float* Btilde,
                             int64_t ldb, int64_t m, void* dW, int64_t ldw, pamm_dtype dw_dt, pamm_layout layout,
                             void* stream) {
    const DwSpec dw = {dW, ldw, dw_dt, layout};
    pamm_status s = check_weight_grad(C, ldc, k, n, dt, Btilde, ldb, m, dw);
    if (s != PAMM_OK) return s;
    return do_weight_grad(C, ldc, k, n, dt, Btilde, ldb, m, dw, (cudaStream_t)stream);
}

pamm_status pamm_compress_eps(const void* X, int64_t ldx, int64_t b, int64_t n, pamm_dtype dt, const void* C,
                              int64_t ldc, int64_t k, const float* c_invnorm, float eps, void* f,
                              pamm_index_type f_type, float* alpha, int32_t* dropped, void* workspace, size_t ws_bytes,
                              void* stream) {
    pamm_status s = check_compress(X, ldx, b, n, dt, C, ldc, k, c_invnorm, f, f_type, alpha);
    if (s != PAMM_OK) return s;
    if (!dropped || !aligned(dropped, 4) || !(eps >= 0.f)) return PAMM_ERR_INVALID_ARG;     // also rejects NaN
    s = check_products_out(workspace, ws_bytes, b, k, 1);
    if (s != PAMM_OK) return s;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemsetAsync(dropped, 0, sizeof(int32_t), st) != cudaSuccess) return PAMM_ERR_CUDA;
    // ||X_i - alpha C_f|| <= ||X_i|| always, so eps >= 1 keeps every row: the plain kernel does
    const bool on = eps < 1.f;
    return do_compress(X, ldx, b, n, dt, C, ldc, k, 1, c_invnorm, f, f_type, alpha, b, (int32_t*)workspace, false, st,
                       Neighbourhood{on, eps, dropped});
}

pamm_status pamm_weight_grad_beta(const void* C, int64_t ldc, int64_t k, int64_t n, pamm_dtype dt, const float* Btilde,
                                  int64_t ldb, int64_t m, int64_t b, const int32_t* dropped, void* dW, int64_t ldw,
                                  pamm_dtype dw_dt, pamm_layout layout, void* stream) {
    const DwSpec dw = {dW, ldw, dw_dt, layout};
    pamm_status s = check_weight_grad(C, ldc, k, n, dt, Btilde, ldb, m, dw);
    if (s != PAMM_OK) return s;
    if (b < 1 || (dropped && !aligned(dropped, 4))) return PAMM_ERR_INVALID_ARG;
    return do_weight_grad(C, ldc, k, n, dt, Btilde, ldb, m, dw, (cudaStream_t)stream, b, dropped);
}

pamm_status pamm_weight_grad_accumulate(const void* C, int64_t ldc, int64_t k, int64_t n, pamm_dtype dt,
                                        const float* Btilde, int64_t ldb, int64_t m, float* dW, int64_t ldw,
                                        pamm_layout layout, void* stream) {
    const DwSpec dw = {dW, ldw, PAMM_F32, layout};
    pamm_status s = check_weight_grad(C, ldc, k, n, dt, Btilde, ldb, m, dw);
    if (s != PAMM_OK) return s;
    return do_weight_grad(C, ldc, k, n, dt, Btilde, ldb, m, dw, (cudaStream_t)stream, 0, nullptr, true);
}

pamm_status pamm_contract_weight_grad(const void* C, int64_t ldc, int64_t n, const void* f, pamm_index_type f_type,
                                      const float* alpha, const void* dY, int64_t ldy, int64_t b, int64_t m,
                                      pamm_dtype dt, int64_t k, float* Btilde, int64_t ldb, void* dW, int64_t ldw,
                                      pamm_dtype dw_dt, pamm_layout layout, const void* sort_products, void* workspace,
                                      size_t ws_bytes, void* stream) {
    pamm_status s = check_contract(f, f_type, alpha, dY, ldy, b, m, dt, k, Btilde, ldb, false, sort_products, workspace, ws_bytes);
    if (s != PAMM_OK) return s;
    const ContractWs w = contract_ws(workspace, b, m, k);
    float* Bt = Btilde ? Btilde : w.btilde;
    const int64_t ldbt = Btilde ? ldb : w.m_pad;
    const DwSpec dw = {dW, ldw, dw_dt, layout};
    s = check_weight_grad(C, ldc, k, n, dt, Bt, ldbt, m, dw);
    if (s != PAMM_OK) return s;
    cudaStream_t st = (cudaStream_t)stream;
    if (k <= SK_MAX_K)      // a handful of generators: no sort, two launches (the caller's B~, if any, is still filled)
        return dt == PAMM_F32
            ? launch_small_backward<float>(C, ldc, n, f, (int)f_type, alpha, dY, ldy, b, m, k, Btilde, ldb, dw, w, st)
            : launch_small_backward<__nv_bfloat16>(C, ldc, n, f, (int)f_type, alpha, dY, ldy, b, m, k, Btilde, ldb, dw, w, st);
    const int32_t* pr = (const int32_t*)sort_products;
    // Many generators: the reduction also leaves B~ split into bf16 hi / lo planes and the product takes all its
    // operands by TMA (a workspace of the size pamm_workspace_bytes gives has room for the planes).
    const bool swap = layout == PAMM_DW_MN;
    const bool planes = dt == PAMM_BF16 && ws_bytes >= w.bytes_with_planes && !weight_grad_persist_supported(k, n, m) &&
                        weight_grad_chunked_supported(k, n, m) && (swap ? n : m) * (int64_t)esize(dw_dt) >= 16;
    s = dt == PAMM_F32 ? launch_contract<float>(f, (int)f_type, alpha, dY, ldy, b, m, k, Bt, ldbt, pr, w, st)
                       : launch_contract<__nv_bfloat16>(f, (int)f_type, alpha, dY, ldy, b, m, k, Bt, ldbt, pr, w, st, planes);
    if (s != PAMM_OK) return s;
    if (planes) {
        prof_begin(PAMM_PROF_WEIGHT_GRAD, st);
        s = launch_weight_grad_planes(C, ldc, k, n, w.planes, w.plane_ld, m, dW, ldw, dw_dt == PAMM_BF16, swap, sm_count(), st);
        prof_end(PAMM_PROF_WEIGHT_GRAD, st);
        g_launches += 1;
        return s;
    }
    return do_weight_grad(C, ldc, k, n, dt, Bt, ldbt, m, dw, st);
}

pamm_status pamm_qkv_step_host(const void* X_host, const void* dY_host, int64_t b, int64_t n, int64_t m,
                               pamm_dtype dt, int64_t k, uint64_t seed, float* dW_host, int32_t* f_host,
                               float* alpha_host, void* arena, size_t arena_bytes, void* stream) {
    if (!dtype_ok(dt)) return PAMM_ERR_UNSUPPORTED;
    if (!X_host || !dY_host || !dW_host) return PAMM_ERR_INVALID_ARG;
    if (b < 1 || n < 1 || m < 1 || k < 1 || k > b || b > MAX_ROWS) return PAMM_ERR_INVALID_ARG;
    if (k > SEL_MAX_K) return PAMM_ERR_UNSUPPORTED;
    if (!arena || !aligned(arena, 256)) return PAMM_ERR_WORKSPACE;
    const StepArena a = step_arena_layout(arena, b, n, m, k, dt);
    if (arena_bytes < a.bytes) return PAMM_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    const size_t es = esize(dt);
    if (cudaMemcpy2DAsync(a.X, a.ldx * es, X_host, n * es, n * es, b, cudaMemcpyHostToDevice, st) != cudaSuccess ||
        cudaMemcpy2DAsync(a.dY, a.ldy * es, dY_host, m * es, m * es, b, cudaMemcpyHostToDevice, st) != cudaSuccess)
        return PAMM_ERR_CUDA;
    pamm_status s = pamm_compress_fused(a.X, a.ldx, b, n, dt, k, seed, nullptr, a.idx, a.C, a.ldc, a.invnorm, a.f,
                                        PAMM_IDX_I32, a.alpha, a.products, sort_products_bytes(b, k), stream);
    if (s != PAMM_OK) return s;
    s = pamm_contract_weight_grad(a.C, a.ldc, n, a.f, PAMM_IDX_I32, a.alpha, a.dY, a.ldy, b, m, dt, k, (float*)a.Bt, a.ldb,
                                  a.dW, a.ldw, PAMM_F32, PAMM_DW_NM, a.products, a.ws, a.ws_bytes, stream);
    if (s != PAMM_OK) return s;
    if (cudaMemcpy2DAsync(dW_host, m * 4, a.dW, a.ldw * 4, m * 4, n, cudaMemcpyDeviceToHost, st) != cudaSuccess)
        return PAMM_ERR_CUDA;
    if (f_host && cudaMemcpyAsync(f_host, a.f, (size_t)b * 4, cudaMemcpyDeviceToHost, st) != cudaSuccess)
        return PAMM_ERR_CUDA;
    if (alpha_host && cudaMemcpyAsync(alpha_host, a.alpha, (size_t)b * 4, cudaMemcpyDeviceToHost, st) != cudaSuccess)
        return PAMM_ERR_CUDA;
    return PAMM_OK;
}

// One small pinned host word and one private stream per device carry the status word
// to the host without touching the caller's streams.
namespace {
struct StatusReader {
    cudaStream_t stream = nullptr;
    int* host_word = nullptr;
    int* dev_word = nullptr;
};
StatusReader g_status_reader[64];
std::mutex g_status_mutex;
}  // namespace

pamm_status pamm_last_device_status(void* stream) {
    (void)stream;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return PAMM_ERR_CUDA;
    std::lock_guard<std::mutex> lock(g_status_mutex);
    StatusReader& r = g_status_reader[dev];
    if (!r.stream) {
        void* sym = nullptr;
        if (cudaGetSymbolAddress(&sym, g_status_word) != cudaSuccess || !sym) return PAMM_ERR_CUDA;
        if (cudaHostAlloc((void**)&r.host_word, sizeof(int), cudaHostAllocDefault) != cudaSuccess) return PAMM_ERR_CUDA;
        if (cudaStreamCreateWithFlags(&r.stream, cudaStreamNonBlocking) != cudaSuccess) {
            cudaFreeHost(r.host_word);
            r.host_word = nullptr;
            r.stream = nullptr;
            return PAMM_ERR_CUDA;
        }
        r.dev_word = (int*)sym;
    }
    // a copy on the private stream: it waits for no kernel and blocks no stream of the caller
    if (cudaMemcpyAsync(r.host_word, r.dev_word, sizeof(int), cudaMemcpyDeviceToHost, r.stream) != cudaSuccess ||
        cudaStreamSynchronize(r.stream) != cudaSuccess)
        return PAMM_ERR_CUDA;
    const int word = *r.host_word;
    if (word) {
        if (cudaMemsetAsync(r.dev_word, 0, sizeof(int), r.stream) != cudaSuccess ||
            cudaStreamSynchronize(r.stream) != cudaSuccess)
            return PAMM_ERR_CUDA;
    }
    if (word & DEV_TIMEOUT) return PAMM_ERR_TIMEOUT;
    if (word & DEV_BAD_INDEX) return PAMM_ERR_BAD_INDEX;
    return PAMM_OK;
}

}  // extern "C"

// ---- scratch of pamm_contract_no_alloc -----------------------------------------
// Lives in the library image, one copy per device that loads it.  In host code
// the name below is only a stand-in for the symbol: the device address has to be
// asked for with cudaGetSymbolAddress, once per device, with that device current.
static __device__ __align__(256) unsigned char g_no_alloc_scratch[PAMM_NO_ALLOC_SCRATCH_BYTES];

namespace {
constexpr int NO_ALLOC_MAX_DEVICES = 64;
void* g_no_alloc_ptr[NO_ALLOC_MAX_DEVICES] = {};
std::mutex g_no_alloc_mutex;

// Device address of the fixed scratch on the current device (nullptr on failure).
void* no_alloc_scratch_ptr() {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= NO_ALLOC_MAX_DEVICES) return nullptr;
    std::lock_guard<std::mutex> lock(g_no_alloc_mutex);
    if (!g_no_alloc_ptr[dev]) {
        void* p = nullptr;
        if (cudaGetSymbolAddress(&p, g_no_alloc_scratch) != cudaSuccess || !p) return nullptr;
        g_no_alloc_ptr[dev] = p;
    }
    return g_no_alloc_ptr[dev];
}
}  // namespace

extern "C" pamm_status pamm_contract_no_alloc(const int32_t* f, const float* alpha, const void* dY, int64_t ldy,
                                              int64_t b, int64_t m, pamm_dtype dt, int64_t k, float* Btilde,
                                              int64_t ldb, void* stream) {
    // sizes first: the fixed array is the only scratch there is
    if (!dtype_ok(dt)) return PAMM_ERR_UNSUPPORTED;
    if (b < 1 || m < 1 || k < 1 || k > b || b > MAX_ROWS) return PAMM_ERR_INVALID_ARG;
    if (contract_ws(nullptr, b, m, k).bytes > (size_t)PAMM_NO_ALLOC_SCRATCH_BYTES) return PAMM_ERR_WORKSPACE;
    void* scratch = no_alloc_scratch_ptr();
    if (!scratch) return PAMM_ERR_CUDA;
    pamm_status s = check_contract(f, PAMM_IDX_I32, alpha, dY, ldy, b, m, dt, k, Btilde, ldb, true, nullptr, scratch,
                                   (size_t)PAMM_NO_ALLOC_SCRATCH_BYTES);
    if (s != PAMM_OK) return s;
    const ContractWs w = contract_ws(scratch, b, m, k);
    cudaStream_t st = (cudaStream_t)stream;
    return dt == PAMM_F32
        ? launch_contract<float>(f, PAMM_IDX_I32, alpha, dY, ldy, b, m, k, Btilde, ldb, nullptr, w, st)
        : launch_contract<__nv_bfloat16>(f, PAMM_IDX_I32, alpha, dY, ldy, b, m, k, Btilde, ldb, nullptr, w, st);
}
