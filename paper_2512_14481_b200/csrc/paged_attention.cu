// sasq_paged_attention: host side, and the kernels' instantiations.
#include <atomic>

#include "paged_rows.cuh"
#include "paged_tiles.cuh"

namespace sasq {

long long debug_wait_limit();       // sasq_debug_set_wait_limit's setting

SASQ_DEFINE_STATUS_WORD(g_paged_status)

int paged_status_read_and_clear(cudaStream_t st) { return g_paged_status_read_and_clear(st); }

int* paged_status_ptr() {
    static std::atomic<int*> cache[64];      // any host thread may make the first call on a device
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    int* p = cache[dev].load(std::memory_order_acquire);
    if (p == nullptr) {
        if (cudaGetSymbolAddress(reinterpret_cast<void**>(&p), g_paged_status) != cudaSuccess) return nullptr;
        cache[dev].store(p, std::memory_order_release);
    }
    return p;
}

namespace {

constexpr int kMaxSms = 256;
constexpr int kClusterKeysPerWarp = 1536;

struct Layout {
    size_t ml, o, total;        // byte offsets behind the part items
};
Layout layout_of(int blocks, int R, int D) {
    Layout l;
    l.ml = (size_t)blocks * sizeof(PartItem);
    l.o = l.ml + (size_t)2 * blocks * R * sizeof(float2);
    l.total = l.o + (size_t)2 * blocks * R * D * sizeof(float);
    return l;
}

struct Plan {
    bool tiles;                 // the tensor-core kernel for many rows; else the few-row kernel
    int cluster;                // few-row kernel: warps of the blocks of an item's cluster, or 0
    int tile_bound;
    int nb;                     // few-row kernel: blocks of 8 rows
    int blocks;
    int rows;                   // of an item
    int slot_rows;              // room for an item's rows in a part slot
    int unit;
    long long items;            // by the host's bounds
    int fill;                   // blocks that are resident at once
    int max_rows;               // (token, head) rows of a sequence and KV head at most, by the host's bound
};

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// The equal-stretch plan of the few-row kernel, and of the tensor-core kernel.
Plan rows_plan(const sasq_kv_cache_t* c, const sasq_kv_batch_t* b, int heads, int sms) {
    Plan pl{};
    const long long rows = (long long)b->max_q_len * (heads / c->num_kv_heads);
    const bool d128 = c->head_dim == 128;
    pl.nb = rows <= 8 ? 1 : 2;
    pl.rows = pl.slot_rows = 8 * pl.nb;
    const int units[2][3] = {{kRowsUnit<1, 0>, kRowsUnit<1, 1>, kRowsUnit<1, 2>}, {kRowsUnit<2, 0>, kRowsUnit<2, 1>, kRowsUnit<2, 2>}};
    pl.unit = units[pl.nb - 1][c->kind];
    pl.tile_bound = rows < 1 ? 1 : ceil_div(rows, pl.rows);
    const int blocks[2][3] = {{kRowsBlocksPerSm<64, 1, 0>, kRowsBlocksPerSm<64, 1, 1>, kRowsBlocksPerSm<64, 1, 2>},
                              {kRowsBlocksPerSm<128, 1, 0>, kRowsBlocksPerSm<128, 1, 1>, kRowsBlocksPerSm<128, 1, 2>}};
    const int per_sm = pl.nb == 1 ? blocks[d128][c->kind] : kRowsBlocksPerSm<128, 2, 0>;
    pl.items = (long long)b->batch * c->num_kv_heads * pl.tile_bound;
    pl.fill = sms * per_sm;
    return pl;
}
Plan tiles_plan(const sasq_kv_cache_t* c, const sasq_kv_batch_t* b, int heads, int sms) {
    Plan pl{};
    const int group = heads / c->num_kv_heads;
    pl.tiles = true;
    pl.rows = 2 * (128 / group * group);
    pl.slot_rows = 256;
    pl.unit = kTileKeys;
    pl.items = (long long)b->batch * c->num_kv_heads * ceil_div((long long)b->max_q_len * group, pl.rows);
    pl.fill = sms;
    return pl;
}
void set_blocks(Plan* pl, const sasq_kv_batch_t* b) {
    const long long most = pl->items * (b->max_seq_len < 1 ? 1 : ceil_div(b->max_seq_len, pl->unit));
    pl->blocks = (int)(most < pl->fill ? (most < 1 ? 1 : most) : pl->fill);
}
bool tiles_possible(const sasq_kv_cache_t* c, const sasq_kv_batch_t* b, int heads) {
    const int group = heads / c->num_kv_heads;
    return (long long)b->max_q_len * group > 16 && group <= 128 && c->num_pages > 0;
}

// The batch with its bounds cut to what q and the page table can hold (the device cuts lengths to the same), so that a
// caller who leaves a bound wide open gets the plan, and the workspace, of one who gives it.
sasq_kv_batch_t with_cut_bounds(const sasq_kv_batch_t* b, const PagedParams& p) {
    sasq_kv_batch_t cut = *b;
    const long long room = (long long)p.max_pages << p.page_shift;
    if (cut.max_seq_len > room) cut.max_seq_len = (int32_t)room;
    if (cut.max_q_len > cut.total_q) cut.max_q_len = cut.total_q;
    return cut;
}

Plan make_plan(const sasq_kv_cache_t* c, const sasq_kv_batch_t* b, int heads, int sms) {
    Plan pl = rows_plan(c, b, heads, sms);
    const long long rows = (long long)b->max_q_len * (heads / c->num_kv_heads);
    // Few items: a cluster each, if all clusters are resident at once and a block's eighth of the keys is not long.  One
    // token, 32 heads over 1000 keys: 8.2 us in clusters, 15.0 us in equal stretches with a joining launch; over 4000 keys
    // 19.1 and 22.8 us; over 16000 keys 58.5 and 51.7 us.  Where there is no more than a block for each SM its warps are
    // eight (8 heads over 4000 keys: 10.3 us; with four 13.4 us), and the keys may be twice as many.
    const int warps = pl.items * kClusterBlocks <= sms && pl.nb * c->head_dim <= 128 ? 8 : 4;
    if (pl.items > 0 && pl.items * kClusterBlocks <= pl.fill && b->max_seq_len <= kClusterKeysPerWarp * warps) pl.cluster = warps;
    // More rows than one item of the few-row kernel holds: the tensor-core kernel, except for up to 64 rows in clusters
    // (8 KV heads with 20, 32 and 64 rows over 1000 keys: 9.0, 9.6 and 9.8 us, on the tensor cores 14.4, 14.4 and 15.0 us;
    // 128 rows: 22.5 and 17.8 us; 16 sequences with 20 rows, not in clusters: 35.0 and 28.3 us).
    if (tiles_possible(c, b, heads) && (pl.cluster == 0 || rows > 64)) pl = tiles_plan(c, b, heads, sms);
    if (pl.cluster != 0) pl.blocks = (int)pl.items * kClusterBlocks;
    else set_blocks(&pl, b);
    pl.max_rows = (int)(rows < (1 << 30) ? rows : 1 << 30);
    return pl;
}

// What any plan can need, whatever the device's number of SMs.
size_t most_workspace(const sasq_kv_cache_t* c, const sasq_kv_batch_t* b, int heads) {
    Plan few = rows_plan(c, b, heads, kMaxSms);
    set_blocks(&few, b);
    size_t bytes = layout_of(few.blocks, few.slot_rows, c->head_dim).total;
    if (tiles_possible(c, b, heads)) {
        Plan many = tiles_plan(c, b, heads, kMaxSms);
        set_blocks(&many, b);
        const size_t m = layout_of(many.blocks, many.slot_rows, c->head_dim).total;
        bytes = m > bytes ? m : bytes;
    }
    return bytes;
}

int attend_check(const sasq_kv_cache_t* cache, const sasq_kv_batch_t* batch, int num_q_heads, int dt, PagedParams* p) {
    const int rc = paged_check(cache, batch, dt, p);
    if (rc != SASQ_OK) return rc;
    if (num_q_heads <= 0 || num_q_heads % cache->num_kv_heads != 0) return SASQ_ERR_INVALID_ARG;
    if (cache->head_dim != 64 && cache->head_dim != 128) return SASQ_ERR_UNSUPPORTED;
    if ((long long)batch->total_q * (num_q_heads / cache->num_kv_heads) > (1 << 30)) return SASQ_ERR_UNSUPPORTED;
    return SASQ_OK;
}

template <typename Kernel>
cudaError_t launch(Kernel kernel, dim3 grid, int threads, size_t smem, cudaStream_t st, const AttendParams& p, int cluster = 1) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0] = pdl_attribute();
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <int D, int NB, bool BF, int KIND>
cudaError_t launch_rows(const Plan& pl, const AttendParams& p, cudaStream_t st) {
    const dim3 grid((unsigned)p.max_blocks);
    if constexpr (NB * D <= 128) {             // eight warps' sums fit 48 KB of shared memory
        if (pl.cluster == 8) return launch(paged_rows_kernel<D, NB, BF, KIND, true, 8>, grid, 256, 0, st, p, kClusterBlocks);
    }
    if (pl.cluster != 0) return launch(paged_rows_kernel<D, NB, BF, KIND, true, 4>, grid, 128, 0, st, p, kClusterBlocks);
    const cudaError_t e = launch(paged_rows_kernel<D, NB, BF, KIND, false, 4>, grid, 128, 0, st, p);
    if (e != cudaSuccess || !p.split) return e;
    return launch(paged_join_kernel<8 * NB, 8 * NB, D, BF, true, KIND == SASQ_KV_INT4>, dim3(p.max_blocks, 8 * NB), 256, 0, st, p);
}
template <int D, bool BF, int KIND>
cudaError_t launch_few(const Plan& pl, const AttendParams& p, cudaStream_t st) {
    return pl.nb == 1 ? launch_rows<D, 1, BF, KIND>(pl, p, st) : launch_rows<D, 2, BF, KIND>(pl, p, st);
}

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static std::atomic<EncodeTiledFn> fn{nullptr};
    if (fn.load() == nullptr) {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn.store(reinterpret_cast<EncodeTiledFn>(f));
    }
    return fn.load();
}

template <bool BF>
bool encode_map(CUtensorMap* m, void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    const EncodeTiledFn fn = encode_fn();
    const cuuint32_t one[4] = {1, 1, 1, 1};
    return fn != nullptr &&
           fn(m, BF ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, base, dims, strides, box, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// 16-bit pages as [page][head][row][dim]: boxes of 64 dims x up to 128 rows of one page and head, 128-byte swizzle; a
// page index outside the cache reads zeros.
template <int D, bool BF>
bool encode_pages(CUtensorMap* m, const sasq_kv_cache_t* c, void* base) {
    const cuuint64_t dims[4] = {D, (cuuint64_t)c->page_size, (cuuint64_t)c->num_kv_heads, (cuuint64_t)c->num_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)c->token_stride * 2, (cuuint64_t)c->head_stride * 2, (cuuint64_t)c->page_stride * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)(c->page_size < kTileKeys ? c->page_size : kTileKeys), 1, 1};
    return encode_map<BF>(m, base, 4, dims, strides, box);
}

// queries as [token][head][dim]: boxes of 64 dims x the heads of a group x the tokens of a row tile
template <int D, bool BF>
bool encode_queries(CUtensorMap* m, const AttendParams& p) {
    const cuuint64_t dims[3] = {D, (cuuint64_t)p.heads, (cuuint64_t)p.c.total_q};
    const cuuint64_t strides[2] = {D * 2, (cuuint64_t)p.q_stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)p.group, (cuuint32_t)(128 / p.group)};
    return encode_map<BF>(m, const_cast<uint16_t*>(p.q), 3, dims, strides, box);
}

// groups of eight rows of the joining launch: all that an item can have (by the host's bound; the kernel walks on over
// rows beyond it)
unsigned join_rows(const AttendParams& p, int max_rows) {
    return max_rows > p.item_rows / 2 ? 256 / 8 : (unsigned)ceil_div(max_rows < 1 ? 1 : max_rows, 8);
}

template <int D, bool BF, int KIND>
cudaError_t launch_tiles(const AttendParams& p, const sasq_kv_cache_t* c, int max_rows, cudaStream_t st) {
    static std::atomic<unsigned long long> ready{0};          // devices whose shared-memory limit has been raised
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!(ready.load() >> (dev & 63) & 1)) {
        e = cudaFuncSetAttribute(paged_tiles_kernel<D, BF, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kTileSmem<D>);
        if (e != cudaSuccess) return e;
        ready.fetch_or(1ull << (dev & 63));
    }
    CUtensorMap map_q{}, map_k{}, map_v{};
    if (!encode_queries<D, BF>(&map_q, p)) return cudaErrorInvalidValue;
    if (KIND == SASQ_KV_16BIT && (!encode_pages<D, BF>(&map_k, c, c->k) || !encode_pages<D, BF>(&map_v, c, c->v))) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)p.max_blocks);
    cfg.blockDim = dim3(kTileThreads<KIND>);
    cfg.dynamicSmemBytes = kTileSmem<D>;
    cfg.stream = st;
    cudaLaunchAttribute attr = pdl_attribute();
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, paged_tiles_kernel<D, BF, KIND>, map_q, map_k, map_v, p);
    if (e != cudaSuccess || !p.split) return e;
    return launch(paged_join_kernel<256, 128, D, BF, false, KIND == SASQ_KV_INT4>, dim3(p.max_blocks, join_rows(p, max_rows)), 256, 0, st, p);
}

template <int D, bool BF>
cudaError_t launch_all(const Plan& pl, const AttendParams& p, const sasq_kv_cache_t* c, cudaStream_t st) {
    if (pl.tiles)
        return c->kind == SASQ_KV_INT4   ? launch_tiles<D, BF, SASQ_KV_INT4>(p, c, pl.max_rows, st)
               : c->kind == SASQ_KV_INT8 ? launch_tiles<D, BF, SASQ_KV_INT8>(p, c, pl.max_rows, st)
                                         : launch_tiles<D, BF, SASQ_KV_16BIT>(p, c, pl.max_rows, st);
    return c->kind == SASQ_KV_INT4   ? launch_few<D, BF, SASQ_KV_INT4>(pl, p, st)
           : c->kind == SASQ_KV_INT8 ? launch_few<D, BF, SASQ_KV_INT8>(pl, p, st)
                                     : launch_few<D, BF, SASQ_KV_16BIT>(pl, p, st);
}

}  // namespace
}  // namespace sasq

extern "C" {

size_t sasq_paged_attention_workspace(const sasq_kv_cache_t* cache, const sasq_kv_batch_t* batch, int num_q_heads) {
    using namespace sasq;
    PagedParams p{};
    if (attend_check(cache, batch, num_q_heads, SASQ_BF16, &p) != SASQ_OK) return 0;
    const sasq_kv_batch_t cut = with_cut_bounds(batch, p);
    return most_workspace(cache, &cut, num_q_heads);
}

int sasq_paged_attention(const sasq_kv_cache_t* cache, const sasq_kv_batch_t* batch, const void* q, void* out, float* lse,
                         int64_t q_stride, int64_t out_stride, int num_q_heads, float softmax_scale, int causal, int dt,
                         void* workspace, size_t ws_bytes, void* stream) {
    using namespace sasq;
    AttendParams p{};
    const int rc = attend_check(cache, batch, num_q_heads, dt, &p.c);
    if (rc != SASQ_OK) return rc;
    const int64_t row = (int64_t)num_q_heads * cache->head_dim;
    if (!(softmax_scale == softmax_scale) || softmax_scale - softmax_scale != 0.0f) return SASQ_ERR_INVALID_ARG;
    if (batch->total_q > 0) {
        if (q == nullptr || out == nullptr || !aligned16(q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3u) || q == out)
            return SASQ_ERR_INVALID_ARG;
        if (q_stride < row || out_stride < row || q_stride % 8 != 0 || out_stride % 8 != 0) return SASQ_ERR_INVALID_ARG;
    }
    if (batch->total_q == 0 || batch->batch == 0) return SASQ_OK;
    if (workspace == nullptr || !aligned16(workspace) || ws_bytes < sasq_paged_attention_workspace(cache, batch, num_q_heads))
        return SASQ_ERR_WORKSPACE;
    const int sms = device_sm_count_if_sm100();
    if (sms <= 0 || sms > kMaxSms) return SASQ_ERR_UNSUPPORTED;
    p.c.status = paged_status_ptr();
    if (p.c.status == nullptr) return SASQ_ERR_CUDA;
    const sasq_kv_batch_t cut = with_cut_bounds(batch, p.c);
    const Plan pl = make_plan(cache, &cut, num_q_heads, sms);
    const Layout l = layout_of(pl.blocks, pl.slot_rows, cache->head_dim);
    if (pl.cluster == 0 && l.total > ws_bytes) return SASQ_ERR_WORKSPACE;      // most_workspace covers every plan
    p.q = static_cast<const uint16_t*>(q);
    p.out = static_cast<uint16_t*>(out);
    p.lse = lse;
    p.q_stride = q_stride;
    p.out_stride = out_stride;
    p.heads = num_q_heads;
    p.group = num_q_heads / cache->num_kv_heads;
    p.scale = softmax_scale * 1.4426950408889634f;
    p.causal = causal != 0;
    // no item has more than one unit when the host's bound says so: nothing to cut, no joining launch
    p.split = cut.max_seq_len > pl.unit;
    p.max_blocks = pl.blocks;
    p.item_rows = pl.rows;
    p.tile_bound = pl.tile_bound;
    p.wait_limit = debug_wait_limit();
    p.flips = kFlips;
    p.half_flips = kHalfFlips;
    p.part_items = static_cast<PartItem*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + l.ml);
    p.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + l.o);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (cache->head_dim == 128)
        e = dt == SASQ_BF16 ? launch_all<128, true>(pl, p, cache, st) : launch_all<128, false>(pl, p, cache, st);
    else
        e = dt == SASQ_BF16 ? launch_all<64, true>(pl, p, cache, st) : launch_all<64, false>(pl, p, cache, st);
    return e == cudaSuccess ? SASQ_OK : SASQ_ERR_CUDA;
}

}  // extern "C"
