// Pieces that the tensor-core kernels of the packed-row attentions share: bounded waits, arithmetic in
// pairs, and tiles of K and V out of the pages.
//
// A tile of 128 slots and D channels lies in shared memory as 16 groups of 8 slots, and in each group 64
// channels a block of 1 KB with the 128-byte swizzle: one copy then moves all channels of as many slots as a
// page allows.  (Copies of 64 channels each cost 156 cycles whatever their size: with pages of 16 slots a
// step of the attention took 5000 cycles instead of 4000.)
#pragma once
#include <cudaTypedefs.h>

#include "rows_redo.cuh"
#include "tc.cuh"

namespace ikv {
namespace {

constexpr int kAtom = 128 * 128;            // bytes of 64 channels of 128 query rows
constexpr int kBlock = 1024;                // bytes of 64 channels of 8 slots
constexpr uint64_t kLimitNs = 1000000000ull;
constexpr uint64_t kStallNs = 10000ull;     // of the wait that a test makes run out

__device__ unsigned int g_tc_timeout = 0;   // (each file's own)

struct TcMap {
    int32_t rows_per_box, box_shift;        // a power of two
    int32_t pool_rows;                      // rows of the layer: a row behind the end
    int32_t stall;                          // nonzero: the products wait for what never comes (a test's launch)
};

// Bounded: false where the phase does not complete in time (which also raises the CTA's abort flag and the
// error word), or once another warp has given up.
__device__ __forceinline__ bool bar_wait_long(uint32_t bar, uint32_t parity, volatile int *abort,
                                              uint64_t limit = kLimitNs) {
    const uint64_t start = global_ns();
    for (;;) {
        if (mbar_try(bar, parity, 2000)) return true;
        if (*abort) return false;
        if (global_ns() - start > limit) break;
    }
    *abort = 1;
    atomicOr(&g_tc_timeout, 1u);
    return false;
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *abort) {
    return mbar_try(bar, parity, 2000) || bar_wait_long(bar, parity, abort);
}
// by a converged warp, with one answer for all of it
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abort) {
    if (__all_sync(0xffffffffu, mbar_try(bar, parity, 2000))) return true;
    return __all_sync(0xffffffffu, bar_wait_long(bar, parity, abort));
}
// of one's own copies or products, whatever the abort flag says
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity) {
    if (mbar_test(bar, parity)) return;
    const uint64_t start = global_ns();
    while (!mbar_try(bar, parity, 2000))
        if (global_ns() - start > kLimitNs) {
            atomicOr(&g_tc_timeout, 1u);
            return;
        }
}
// The row of a layer's pool that holds slot s of sequence b, KV head g
__device__ __forceinline__ int pool_row(const RowsArgs &a, int b, int g, int s) {
    const int lp = a.pv.page_shift >= 0 ? s >> a.pv.page_shift : s / a.pv.page_size;
    const int page = __ldg(a.pv.block_table + (int64_t)b * a.pv.max_pages + lp);
    return (page * a.pv.kv_heads + g) * a.pv.page_size + (s - lp * a.pv.page_size);
}
// rows_per_box rows from `row` (a multiple of 8) on, all channels
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap *map, int row, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %2, %3}], "
        "[%4];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row >> 3), "r"(bar)
        : "memory");
}

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        cudaDriverEntryPointQueryResult q;
        void *p = nullptr;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q);
        return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p)
                                                                    : nullptr;
    }();
    return fn;
}

// A layer's rows as [groups of 8][64-channel blocks][8 rows][64 channels]
bool layer_map(CUtensorMap *m, const void *pool, const RowsArgs &a, int head_dim, TcMap *t, int most = 64) {
    const auto fn = encode_fn();
    if (!fn) return false;
    const uint64_t rows = (uint64_t)a.pv.num_pages * a.pv.kv_heads * a.pv.page_size, row = (uint64_t)head_dim * 2;
    t->pool_rows = (int32_t)rows;
    // boxes as high as the page allows, at most `most` rows: they are also the grain in which what a unit sees is read
    t->rows_per_box = 8;
    while (t->rows_per_box < most && a.pv.page_size % (2 * t->rows_per_box) == 0) t->rows_per_box *= 2;
    t->box_shift = __builtin_ctz((unsigned)t->rows_per_box);
    const cuuint64_t dims[4] = {64, 8, (cuuint64_t)head_dim / 64, rows / 8}, strides[3] = {row, 128, 8 * row};
    const cuuint32_t box[4] = {64, 8, (cuuint32_t)head_dim / 64, (cuuint32_t)t->rows_per_box / 8}, es[4] = {1, 1, 1, 1};
    const void *rows0 = static_cast<const char *>(pool) + (size_t)a.layer * rows * row;
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(rows0), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t read_clear_timeout(unsigned int *v) {
    unsigned int z = 0;
    cudaError_t e = cudaMemcpyFromSymbol(v, g_tc_timeout, sizeof(*v));
    if (e == cudaSuccess && *v) e = cudaMemcpyToSymbol(g_tc_timeout, &z, sizeof(z));
    return e;
}

}  // namespace
}  // namespace ikv
