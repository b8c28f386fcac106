// C entry points of the operators on a cache kept in pages (see include/sdv.h): checks of the arguments and launches.
#include "../../include/sdv.h"

#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include <initializer_list>

#include "device_once.h"
#include "overlap.h"
#include "paged.cuh"
#include "tensor_map.h"
#include "tree_attention.cuh"
#include "verify_sampled.cuh"

using namespace sdv;

namespace {

constexpr unsigned long long kWaitNs = 2000000000ull;
constexpr int kMaxRows = 1 << 30;    // row numbers plus a grid's stride stay within 32 bits, and the elements of a row of heads
constexpr int kMaxVocab = 1 << 21;   // tile sums of a block of sdv_verify_sampled stay within 32 KB

// Device memory of the current device (where the runtime can tell), on a boundary of `align` bytes.
bool on_device(const void* p, int dev, size_t align) {
    if (!p || ((uintptr_t)p & (align - 1))) return false;
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    return at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == dev);
}
bool on_device(std::initializer_list<const void*> ps, int dev, size_t align) {
    for (const void* p : ps)
        if (!on_device(p, dev, align)) return false;
    return true;
}

int sm_count(int dev) {   // 1 where it cannot be told
    static std::atomic<int> known[64];
    const bool keep = dev >= 0 && dev < 64;
    int n = keep ? known[dev].load(std::memory_order_relaxed) : 0;
    if (!n && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && keep) known[dev].store(n, std::memory_order_relaxed);
    return max(n, 1);
}

// A launch, in clusters of `cluster` blocks, that may overlap the tail of the kernel before it: each kernel waits for that one's end before it reads what it may have written.
template <typename... KArgs, typename... Args>
int launch(void (*kernel)(KArgs...), int grid, int block, size_t smem, void* stream, int cluster, const Args&... args) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess) return SDV_OK;
    cudaGetLastError();   // not to be reported by another call's check
    return SDV_ECUDA;
}

// No output starts where an input or another output does (those left out are null).  Needs no device; how far they reach is looked at once their addresses are known to be real.
bool apart(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
    for (const void* const* o = outs.begin(); o != outs.end(); ++o) {
        if (!*o) continue;
        for (const void* p : ins)
            if (p == *o) return false;
        for (const void* const* other = outs.begin(); other != o; ++other)
            if (*other == *o) return false;
    }
    return true;
}

// No output shares memory with an input or another output.
bool distinct(std::initializer_list<Area> outs, std::initializer_list<Area> ins) {
    Overlap meet;
    for (const Area* o = outs.begin(); o != outs.end(); ++o) {
        for (const Area& a : ins)
            if (meet(*o, a)) return false;
        for (const Area* other = outs.begin(); other != o; ++other)
            if (meet(*o, *other)) return false;
    }
    return true;
}
Area ints(const void* p, long long n) { return area(p, 4 * n); }
// [rows][heads][head dim] of 16-bit elements.
Area heads_area(const void* p, int rows, long long row_stride, int heads, long long head_stride, int dim) { return area(p, 2ll * dim, rows, 2 * row_stride, heads, 2 * head_stride); }
Area pool_area(const void* p, const sdv_pages& s) {
    return area(p, 2ll * s.head_dim, s.n_pages, 2 * s.page_stride, s.n_kv_heads, 2 * s.head_stride, s.page_size, 2 * s.token_stride);
}

// An output's rows (or heads) do not lie on top of each other.
bool spread(int n, long long stride) { return n <= 1 || stride > 0; }

bool pages_ok(const sdv_pages* p, int dev) {
    if (!p || (p->dtype != SDV_BF16 && p->dtype != SDV_FP16)) return false;
    if (p->n_pages < 1 || p->page_size < 1 || p->n_kv_heads < 1 || p->head_dim < 1 || (long long)p->n_pages * p->page_size > INT_MAX) return false;
    if (!spread(p->n_pages, p->page_stride) || !spread(p->n_kv_heads, p->head_stride) || !spread(p->page_size, p->token_stride)) return false;
    if (p->page_stride < 0 || p->head_stride < 0 || p->token_stride < 0 || ((p->page_stride | p->head_stride | p->token_stride) & 7)) return false;
    return on_device(p->k, dev, 16) && on_device(p->v, dev, 16);
}

typedef void (*RopeKernel)(const sdv_rope_args, const sdv_pages, int);
template <typename T>
RopeKernel rope_kernel(bool interleaved, bool wide) {
    return interleaved ? wide ? rope_append_kernel<T, true, 8> : rope_append_kernel<T, true, 1> : wide ? rope_append_kernel<T, false, 8> : rope_append_kernel<T, false, 1>;
}
RopeKernel rope_kernel(int dtype, bool interleaved, bool wide) { return dtype == SDV_BF16 ? rope_kernel<__nv_bfloat16>(interleaved, wide) : rope_kernel<__half>(interleaved, wide); }
typedef void (*RopeStaged)(const sdv_rope_args, const sdv_pages, int, int);
RopeStaged rope_staged(int dtype) { return dtype == SDV_BF16 ? rope_staged_kernel<__nv_bfloat16> : rope_staged_kernel<__half>; }

typedef void (*TreeKernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const TreeParams);
typedef void (*MergeKernel)(const TreeParams, int, int);
TreeKernel tree_kernel(int dtype, int hd) {
    if (dtype == SDV_BF16) return hd == 128 ? tree_attention_kernel<__nv_bfloat16, 128> : tree_attention_kernel<__nv_bfloat16, 64>;
    return hd == 128 ? tree_attention_kernel<__half, 128> : tree_attention_kernel<__half, 64>;
}
MergeKernel merge_kernel(int dtype, int hd) {
    if (dtype == SDV_BF16) return hd == 128 ? tree_merge_kernel<__nv_bfloat16, 128> : tree_merge_kernel<__nv_bfloat16, 64>;
    return hd == 128 ? tree_merge_kernel<__half, 128> : tree_merge_kernel<__half, 64>;
}
size_t tree_smem(int hd) { return hd == 128 ? TreeShape<128>::kSmemBytes : TreeShape<64>::kSmemBytes; }

// Code of every kernel is loaded, and the attention's shared memory allowed, by the first call on a device.
int prepare_device(int dev) {
    static DeviceOnce once;
    const cudaError_t e = once.run(dev, []() {
        cudaError_t r = cudaSuccess;
        cudaFuncAttributes fa;
        const auto load = [&](const void* f) { if (r == cudaSuccess) r = cudaFuncGetAttributes(&fa, f); };
        load((const void*)paged_slots_kernel);
        load((const void*)verify_sampled_kernel);
        for (int t = SDV_BF16; t <= SDV_FP16; ++t) {
            for (int i = 0; i < 4; ++i) load((const void*)rope_kernel(t, (i & 1) != 0, (i & 2) != 0));
            load((const void*)rope_staged(t));
            for (int hd = 64; hd <= 128; hd += 64) {
                load((const void*)merge_kernel(t, hd));
                if (r == cudaSuccess) r = cudaFuncSetAttribute((const void*)tree_kernel(t, hd), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tree_smem(hd));
            }
        }
        return r;
    });
    if (e == cudaSuccess) return SDV_OK;
    cudaGetLastError();
    return SDV_ECUDA;
}

// Tensor map of 16-bit elements (strides in elements, of every dimension but the first), 128-byte swizzle, zeros outside.
bool make_map(CUtensorMap* m, const void* base, int dtype, int rank, const long long* dims, const long long* strides, const int* box) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t d[4], s[3];
    cuuint32_t b[4], one[4];
    for (int i = 0; i < rank; ++i) {
        d[i] = (cuuint64_t)dims[i];
        b[i] = (cuuint32_t)box[i];
        one[i] = 1;
        if (i && dims[i] > 1 && strides[i - 1] <= 0) return false;   // (rows on top of each other are not known to the copies)
        if (i) s[i - 1] = (cuuint64_t)(dims[i] > 1 ? strides[i - 1] * 2 : 16);   // of a dimension of one: anything valid
    }
    return fn(m, dtype == SDV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank, const_cast<void*>(base), d, s, b, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Keys (or values): head_dim x tokens of a page x KV heads x pages; boxes of 64 elements of box_keys tokens.
bool make_page_map(CUtensorMap* m, const void* base, const sdv_pages* p, int box_keys) {
    const long long dims[4] = {p->head_dim, p->page_size, p->n_kv_heads, p->n_pages}, strides[3] = {p->token_stride, p->head_stride, p->page_stride};
    const int box[4] = {64, box_keys, 1, 1};
    return make_map(m, base, p->dtype, 4, dims, strides, box);
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
int tree_blocks(int dev) { return min(kTreeBlocksPerSm * sm_count(dev), kTreeMaxBlocks); }
// Workspace: maxima and sums | outputs, of up to two partial items a block.
size_t tree_bytes(int head_dim, int blocks, int rows) {
    const size_t parts = (size_t)blocks * 2 * rows;
    return align256(parts * sizeof(float2)) + parts * head_dim * sizeof(float);
}

}  // namespace

extern "C" {

int sdv_paged_slots(const sdv_slots_args* a, void* cuda_stream) {
    if (!a || a->n_seqs < 0 || a->n_seqs > SDV_MAX_SEQUENCES || a->n_rows < 0 || a->n_rows > kMaxRows || a->page_size < 1 || a->table_width < 0 || a->n_free < 0) return SDV_EINVAL;
    if (a->table_stride < a->table_width && a->n_seqs > 1) return SDV_EINVAL;
    if (a->parent && a->n_rows > SDV_MAX_SEQUENCES * SDV_TREE_ROWS) return SDV_EINVAL;
    if ((long long)a->n_seqs * a->table_width > INT_MAX) return SDV_EINVAL;
    // blocks read the inputs while others write
    if (!apart({a->block_table, a->slots, a->positions, a->n_held_out, a->free_state_out}, {a->kv_len, a->cu_rows, a->parent, a->n_held, a->free_pages, a->free_state})) return SDV_EINVAL;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SDV_ECUDA;
    if (!on_device({a->cu_rows, a->free_state, a->free_state_out}, dev, 4)) return SDV_EINVAL;
    if (a->n_seqs && !on_device({a->kv_len, a->n_held, a->n_held_out}, dev, 4)) return SDV_EINVAL;
    if (a->n_seqs && a->table_width && !on_device(a->block_table, dev, 4)) return SDV_EINVAL;
    if (a->n_free && !on_device(a->free_pages, dev, 4)) return SDV_EINVAL;
    if (a->n_rows && (!on_device({a->slots, a->positions}, dev, 4) || (a->parent && !on_device(a->parent, dev, 4)))) return SDV_EINVAL;
    if (!distinct({area(a->block_table, 4ll * a->table_width, a->n_seqs, 4 * a->table_stride), ints(a->slots, a->n_rows), ints(a->positions, a->n_rows), ints(a->n_held_out, a->n_seqs),
                   ints(a->free_state_out, 2)},
                  {ints(a->kv_len, a->n_seqs), ints(a->cu_rows, a->n_seqs + 1ll), ints(a->parent, a->n_rows), ints(a->n_held, a->n_seqs), ints(a->free_pages, a->n_free), ints(a->free_state, 1)}))
        return SDV_EINVAL;
    const int rc = prepare_device(dev);
    if (rc != SDV_OK) return rc;
    const long long items = (long long)a->n_rows + min((long long)a->n_free, (long long)a->n_seqs * a->table_width);
    const int grid = (int)max(1ll, min((items + kSlotThreads - 1) / kSlotThreads, (long long)sm_count(dev)));
    return launch(paged_slots_kernel, grid, kSlotThreads, 0, cuda_stream, 1, *a);
}

int sdv_rope_append(const sdv_rope_args* a, const sdv_pages* pages, void* cuda_stream) {
    if (!a || a->n_rows < 0 || a->n_rows > kMaxRows || (a->dtype != SDV_BF16 && a->dtype != SDV_FP16)) return SDV_EINVAL;
    if (a->head_dim < 2 || a->head_dim > 256 || a->head_dim % 2 || a->rot_dim < 2 || a->rot_dim > a->head_dim || a->rot_dim % 2) return SDV_EINVAL;
    if ((!a->k) != (!a->v) || (!a->q && !a->k) || (a->q && a->n_q_heads < 1) || (a->k && a->n_kv_heads < 1)) return SDV_EINVAL;
    if (((a->q ? (long long)a->n_q_heads : 0) + (a->k ? 2ll * a->n_kv_heads : 0)) * a->head_dim > kMaxRows) return SDV_EINVAL;
    if (a->q && (!spread(a->n_rows, a->out_row_stride) || !spread(a->n_q_heads, a->out_head_stride))) return SDV_EINVAL;
    if (a->q && !apart({a->q_out}, {a->k, a->v, a->positions, a->slots, a->frequencies})) return SDV_EINVAL;
    if (a->q && a->q_out == a->q && ((a->n_rows > 1 && a->out_row_stride != a->q_row_stride) || (a->n_q_heads > 1 && a->out_head_stride != a->q_head_stride))) return SDV_EINVAL;
    if (a->k && pages && !apart({pages->k, pages->v}, {a->q, a->q ? a->q_out : nullptr, a->k, a->v, a->positions, a->slots, a->frequencies})) return SDV_EINVAL;
    if (a->n_rows == 0) return SDV_OK;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SDV_ECUDA;
    if (!on_device(a->positions, dev, 4) || !on_device(a->frequencies, dev, 8)) return SDV_EINVAL;
    uintptr_t bits = 0;   // what the addresses of a row have in common, in elements
    if (a->q) {
        if (!on_device({a->q, a->q_out}, dev, 2)) return SDV_EINVAL;
        bits |= (uintptr_t)a->q >> 1 | (uintptr_t)a->q_out >> 1 | (uintptr_t)(a->q_row_stride | a->q_head_stride | a->out_row_stride | a->out_head_stride);
    }
    sdv_pages none;
    memset(&none, 0, sizeof(none));
    none.page_size = 1;
    if (a->k) {
        if (!on_device({a->k, a->v}, dev, 2) || !on_device(a->slots, dev, 4) || !pages_ok(pages, dev)) return SDV_EINVAL;
        if (pages->dtype != a->dtype || pages->n_kv_heads != a->n_kv_heads || pages->head_dim != a->head_dim) return SDV_EINVAL;
        bits |= (uintptr_t)a->k >> 1 | (uintptr_t)a->v >> 1 | (uintptr_t)(a->k_row_stride | a->k_head_stride | a->v_row_stride | a->v_head_stride);
    }
    {
        const Area none_there = area(nullptr, 0), positions = ints(a->positions, a->n_rows), frequencies = area(a->frequencies, 4ll * a->rot_dim);
        const Area q = a->q ? heads_area(a->q, a->n_rows, a->q_row_stride, a->n_q_heads, a->q_head_stride, a->head_dim) : none_there;
        const Area out = a->q ? heads_area(a->q_out, a->n_rows, a->out_row_stride, a->n_q_heads, a->out_head_stride, a->head_dim) : none_there;
        const Area k = a->k ? heads_area(a->k, a->n_rows, a->k_row_stride, a->n_kv_heads, a->k_head_stride, a->head_dim) : none_there;
        const Area v = a->k ? heads_area(a->v, a->n_rows, a->v_row_stride, a->n_kv_heads, a->v_head_stride, a->head_dim) : none_there;
        const Area slots = a->k ? ints(a->slots, a->n_rows) : none_there, kp = a->k ? pool_area(pages->k, *pages) : none_there, vp = a->k ? pool_area(pages->v, *pages) : none_there;
        if (!distinct({out, kp, vp}, {k, v, positions, slots, frequencies}) || !distinct({kp, vp}, {q}) || (a->q_out != a->q && !distinct({out}, {q}))) return SDV_EINVAL;
    }
    const int rc = prepare_device(dev);
    if (rc != SDV_OK) return rc;
    // Eight elements at once where rows begin on 16-byte boundaries, one otherwise.  The two halves of a rotated head that are no multiple of eight go through shared memory.
    const int half = a->rot_dim / 2;
    const bool aligned = (bits & 7) == 0 && a->head_dim % 8 == 0, wide = aligned && a->head_dim % 16 == 0 && (a->interleaved || half % 8 == 0);
    // rows of a block: about four units of 16 elements a thread, fewer while there are blocks to spare (8191 rows of 24 + 8 heads: 29.7 us with two to four rows a block, 33.6
    // with six)
    const int heads = (a->q ? a->n_q_heads : 0) + (a->k ? 2 * a->n_kv_heads : 0), units = max(1, heads * a->head_dim / 16);
    const int tokens = max(1, min(min(8, 4 * kRopeThreads / units), a->n_rows / (sm_count(dev) * 8)));
    const int grid = (a->n_rows + tokens - 1) / tokens;
    if (aligned && !wide && !a->interleaved) {
        const int staged = min(heads - (a->k ? a->n_kv_heads : 0), 16384 / a->head_dim);   // 32 KB of heads at most
        return launch(rope_staged(a->dtype), grid, kRopeThreads, (size_t)staged * a->head_dim * 2 + (size_t)tokens * half * sizeof(float2), cuda_stream, 1, *a, a->k ? *pages : none,
                      tokens, staged);
    }
    return launch(rope_kernel(a->dtype, a->interleaved != 0, wide), grid, kRopeThreads, (size_t)tokens * half * sizeof(float2), cuda_stream, 1, *a, a->k ? *pages : none, tokens);
}

size_t sdv_tree_attention_workspace_bytes(int n_seqs, int head_dim) {
    int dev = 0;
    if (n_seqs < 0 || n_seqs > SDV_MAX_SEQUENCES || (head_dim != 64 && head_dim != 128) || cudaGetDevice(&dev) != cudaSuccess) return 0;
    return tree_bytes(head_dim, tree_blocks(dev), kTreeTileRows);
}

// clear: see sdv_tree_attention_fresh; wait_ns: of the waits that may be given up; tiles: see sdv_debug_tree_attention.
static int tree_attention(const sdv_attention_args* a, const sdv_pages* pages, bool clear, unsigned long long wait_ns, int tiles, void* cuda_stream) {
    if (!a || !pages || a->n_seqs < 0 || a->n_seqs > SDV_MAX_SEQUENCES || a->n_rows < 0 || a->table_width < 0) return SDV_EINVAL;
    if (pages->head_dim != 64 && pages->head_dim != 128) return SDV_EINVAL;
    if (pages->page_size < 8 || (pages->page_size & (pages->page_size - 1)) || pages->n_kv_heads < 1) return SDV_EINVAL;
    if (a->n_q_heads < 1 || a->n_q_heads % pages->n_kv_heads || a->n_q_heads / pages->n_kv_heads > kTreeTileRows || !(a->scale > 0.f) || !isfinite(a->scale)) return SDV_EINVAL;
    if (a->table_stride < a->table_width && a->n_seqs > 1) return SDV_EINVAL;
    if ((a->q_row_stride | a->q_head_stride | a->out_row_stride | a->out_head_stride) & 7) return SDV_EINVAL;
    if (!spread(a->n_rows, a->out_row_stride) || !spread(a->n_q_heads, a->out_head_stride)) return SDV_EINVAL;
    if (!apart({a->out, a->workspace, a->status}, {a->q, pages->k, pages->v, a->block_table, a->kv_len, a->cu_rows, a->parent})) return SDV_EINVAL;
    if (a->n_seqs == 0 || a->n_rows == 0 || a->table_width == 0) return SDV_OK;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SDV_ECUDA;
    if (!pages_ok(pages, dev) || !on_device({a->q, a->out}, dev, 16) || !on_device({a->block_table, a->kv_len, a->cu_rows}, dev, 4)) return SDV_EINVAL;
    if ((a->parent && !on_device(a->parent, dev, 4)) || (a->status && !on_device(a->status, dev, 4)) || !on_device(a->workspace, dev, 256)) return SDV_EINVAL;
    const int rc = prepare_device(dev);
    if (rc != SDV_OK) return rc;

    TreeParams P;
    memset(&P, 0, sizeof(P));
    const int hd = pages->head_dim, g = a->n_q_heads / pages->n_kv_heads;
    const int chunk = kTreeTileRows / g, rows = min(a->n_rows, SDV_TREE_ROWS), chunks = (rows + chunk - 1) / chunk;
    const long long units = (((long long)a->n_rows * g + 3) / 4 + a->n_rows / chunk + a->n_seqs) * pages->n_kv_heads;   // of the merge
    if ((long long)a->n_rows * a->n_q_heads > INT_MAX / 2 || units * (hd / 16) > INT_MAX) return SDV_EINVAL;
    const long long keys = min((long long)a->table_width * pages->page_size, (long long)INT_MAX);
    const long long each = ((keys + kTreeKeys - 1) / kTreeKeys) * chunks * pages->n_kv_heads, most = each * min(a->n_seqs, a->n_rows);   // no more tiles than this
    if (each * a->n_seqs > INT_MAX / 2) return SDV_EINVAL;   // (whatever cu_rows holds)
    // Short tables: a block goes through whole items and nothing is merged, which saves a launch (2 us on the host) and the merge (2 to 5 us).  Tile by tile against whole,
    // device time in us, by sequences x rows:
    //   4 + 4 heads of 64     1 x 1: 2 tiles of 64 keys 8.2:6.5, 4 8.3:8.0, 6 8.3:9.5     64 x 20: 4 13.8:9.3, 8 16.7:12.9, 10 18.2:14.7, 16 23.0:20.2     300 x 1: 6 37.4:36.6, 8 43.7:44.7
    //   12 + 2 heads of 128   1 x 1: 2 9.0:7.5, 4 9.0:9.3, 6 9.1:11.3                     64 x 1: 8 16.7:15.4, 10 17.3:17.7     64 x 20: 8 25.6:17.5, 10 26.9:20.0, 16 32.2:27.4
    //   24 + 8 heads of 128   1 x 17: 4 10.6:9.5, 6 11.8:11.6, 8 12.9:13.4                64 x 20: 8 45.7:32.3, 10 51.9:37.6, 16 66.6:52.9     300 x 1: 8 111.9:110.2, 12 158.5:159.5
    // The rule knows the table's width, not the rows, heads and lengths: it takes shares where many sequences have many rows behind tables of more than eight tiles, up to 38 percent slower,
    // and whole items for hundreds of single rows, up to 3 percent slower.
    const long long key_tiles = (keys + kTreeKeys - 1) / kTreeKeys;
    P.whole = key_tiles <= 4 || (key_tiles <= 8 && a->n_seqs >= 8);
    P.blocks = (int)min((long long)tree_blocks(dev), P.whole ? (long long)chunks * pages->n_kv_heads * min(a->n_seqs, a->n_rows) : most);
    P.part_rows = (min(rows, chunk) * g + 3) / 4 * 4;
    if (a->workspace_bytes < tree_bytes(hd, P.blocks, P.part_rows)) return SDV_ENOMEM;
    if (!distinct({heads_area(a->out, a->n_rows, a->out_row_stride, a->n_q_heads, a->out_head_stride, hd), area(a->workspace, (long long)tree_bytes(hd, P.blocks, P.part_rows)), ints(a->status, 1)},
                  {heads_area(a->q, a->n_rows, a->q_row_stride, a->n_q_heads, a->q_head_stride, hd), pool_area(pages->k, *pages), pool_area(pages->v, *pages),
                   area(a->block_table, 4ll * a->table_width, a->n_seqs, 4 * a->table_stride), ints(a->kv_len, a->n_seqs), ints(a->cu_rows, a->n_seqs + 1ll), ints(a->parent, a->n_rows)}))
        return SDV_EINVAL;
    const size_t parts = (size_t)P.blocks * 2 * P.part_rows;
    uint8_t* ws = (uint8_t*)a->workspace;
    P.part_ml = (float2*)ws;
    P.part_o = (float*)(ws + align256(parts * sizeof(float2)));
    P.out = a->out;
    P.v = pages->v;
    P.block_table = a->block_table;
    P.kv_len = a->kv_len;
    P.cu_rows = a->cu_rows;
    P.parent = a->parent;
    P.status = a->status;
    P.clear = clear;
    P.out_row_stride = a->out_row_stride;
    P.out_head_stride = a->out_head_stride;
    P.table_stride = a->table_stride;
    P.page_stride = pages->page_stride;
    P.head_stride = pages->head_stride;
    P.token_stride = pages->token_stride;
    P.n_seqs = a->n_seqs;
    P.n_rows = a->n_rows;
    P.n_kv = pages->n_kv_heads;
    P.g = g;
    P.chunk = chunk;
    P.q_step = min(8, chunk);
    P.table_width = a->table_width;
    P.page_size = pages->page_size;
    while ((1 << P.page_shift) < pages->page_size) ++P.page_shift;
    P.n_pages = pages->n_pages;
    P.scale_log2e = a->scale * 1.4426950408889634f;
    P.copies = 2 * tiles;
    P.wait_limit_ns = wait_ns;
    P.drain_limit_ns = kWaitNs;
    CUtensorMap map_q, map_q1, map_k, map_v;
    const int box_keys = min(pages->page_size, kTreeKeys);
    if (!make_page_map(&map_k, pages->k, pages, box_keys) || !make_page_map(&map_v, pages->v, pages, box_keys)) return SDV_EINVAL;
    // queries: head_dim x heads x rows; boxes of 64 elements of all heads of a group, of q_step rows and of one
    const long long q_dims[3] = {hd, a->n_q_heads, a->n_rows}, q_strides[2] = {a->q_head_stride, a->q_row_stride};
    const int q_box[3] = {64, g, P.q_step}, q_box1[3] = {64, g, 1};
    if (!make_map(&map_q, a->q, pages->dtype, 3, q_dims, q_strides, q_box) || !make_map(&map_q1, a->q, pages->dtype, 3, q_dims, q_strides, q_box1)) return SDV_EINVAL;
    const int first = launch(tree_kernel(pages->dtype, hd), P.blocks, kTreeThreads, tree_smem(hd), cuda_stream, 1, map_q, map_q1, map_k, map_v, P);
    if (first != SDV_OK || P.whole || P.blocks == 1) return first;   // nothing is in parts
    // Merge: units of four (row, head) pairs, of 16 columns where that leaves no more than three blocks an SM (see tree_merge_kernel); as many at a time for a block
    // as three blocks an SM need.
    const long long room = (long long)sm_count(dev) * 3;
    const int split = units * (hd / 16) <= room ? hd / 16 : 1;
    const int group = (int)min((long long)kMergeWarps, (units * split + room - 1) / room);
    return launch(merge_kernel(pages->dtype, hd), (int)min((units * split + group - 1) / group, room), kMergeThreads, 0, cuda_stream, 1, P, group, split);
}

int sdv_tree_attention(const sdv_attention_args* a, const sdv_pages* pages, void* cuda_stream) { return tree_attention(a, pages, false, kWaitNs, INT_MAX / 2, cuda_stream); }

int sdv_tree_attention_fresh(const sdv_attention_args* a, const sdv_pages* pages, void* cuda_stream) { return tree_attention(a, pages, true, kWaitNs, INT_MAX / 2, cuda_stream); }

int sdv_debug_tree_attention(const sdv_attention_args* a, const sdv_pages* pages, unsigned long long wait_ns, int tiles, void* cuda_stream) {
    return tiles < 0 || tiles > INT_MAX / 2 ? SDV_EINVAL : tree_attention(a, pages, false, wait_ns, tiles, cuda_stream);
}

int sdv_verify_sampled(const sdv_verify_args* a, void* cuda_stream) {
    if (!a || a->n_seqs < 0 || a->n_seqs > SDV_MAX_SEQUENCES || a->n_rows < 0 || a->n_rows > kMaxRows || a->vocab < 1 || a->vocab > kMaxVocab) return SDV_EINVAL;
    if ((a->draft && a->parent) || (!a->slots) != (!a->out_slots)) return SDV_EINVAL;
    if (a->target_stride < a->vocab || (a->draft && a->draft_stride < a->vocab)) return SDV_EINVAL;
    // a sequence's blocks read what these hold while the first of them writes
    if (!apart({a->accept_len, a->out_tokens, a->out_rows, a->out_slots}, {a->target, a->draft, a->tokens, a->cu_rows, a->parent, a->slots, a->uniforms})) return SDV_EINVAL;
    if (a->n_seqs == 0 || a->n_rows == 0) return SDV_OK;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SDV_ECUDA;
    if (!on_device({a->target, a->tokens, a->cu_rows, a->uniforms, a->accept_len, a->out_tokens, a->out_rows}, dev, 4)) return SDV_EINVAL;
    if ((a->draft && !on_device(a->draft, dev, 4)) || (a->parent && !on_device(a->parent, dev, 4)) || (a->slots && !on_device({a->slots, a->out_slots}, dev, 4))) return SDV_EINVAL;
    if (!distinct({ints(a->accept_len, a->n_seqs), ints(a->out_tokens, a->n_rows), ints(a->out_rows, a->n_rows), ints(a->out_slots, a->n_rows)},
                  {area(a->target, 4ll * a->vocab, a->n_rows, 4 * a->target_stride), area(a->draft, 4ll * a->vocab, a->n_rows, 4 * a->draft_stride), ints(a->tokens, a->n_rows),
                   ints(a->cu_rows, a->n_seqs + 1ll), ints(a->parent, a->n_rows), ints(a->slots, a->n_rows), ints(a->uniforms, a->n_rows)}))
        return SDV_EINVAL;
    const int rc = prepare_device(dev);
    if (rc != SDV_OK) return rc;
    // blocks that share a sequence's vocabulary: doubled while every warp keeps a tile and all blocks are resident at once (two an SM)
    const int tiles = (a->vocab + kVerifyTile - 1) / kVerifyTile;
    int cs = 1;
    while (cs < kVerifyMaxCluster && tiles >= 2 * cs * kVerifyWarps && (long long)a->n_seqs * cs * 2 <= 2ll * sm_count(dev)) cs *= 2;
    const int per = (tiles + cs - 1) / cs;
    return launch(verify_sampled_kernel, a->n_seqs * cs, kVerifyThreads, (size_t)per * sizeof(double), cuda_stream, cs, *a, per);
}

}  // extern "C"
