// The matrix-product engine of the head kernels: D[m, n] = sum_k A[m, k] B[n, k] on the tensor cores (tcgen05), one
// persistent CTA (or pair of CTAs) per SM, with an epilogue that takes the accumulators out of tensor memory.
//
// Shape.  A cluster of kCtas (1 or 2) computes a tile of 128 * kCtas rows by `nt` <= 256 columns.  With a pair, each
// CTA keeps 128 rows of A and half of B's rows, and one instruction (issued by the leader) drives both SMs: each SM
// then reads half of B from L2 that a single CTA would.  A stage is 128 bytes of k: 16 KB of A and up to 16 (pair) or
// 32 KB of B, moved by TMA with the 128-byte swizzle; as many stages as fit run ahead of the tensor cores.  The
// accumulator is double-buffered in tensor memory (2 x 256 columns of fp32 / int32), so that the epilogue of a tile
// overlaps the next tile's products.
//
// Roles.  Warp 0: TMA producer (one lane).  Warp 1: allocates tensor memory, issues the products (one lane of the
// leader CTA).  The other warps: epilogue, warp w reading tensor-memory lanes 32 (w mod 4) ... + 31.
//
// Operands are K-major (k contiguous) or MN-major (m or n contiguous), each from a plain row-major matrix or from panels:
// [columns / 64][rows][64], a matrix that this library laid out itself so that a 64-column box is contiguous memory (whole
// DRAM pages and full lines, whichever way it is read).  Out-of-range rows and columns of a copy read as zero, so that
// ragged sizes need no special case before the epilogue.
//
// Two products.  A kernel can carry a second product of the same tile width: its tiles follow the first's on every cluster,
// so that neither's last round leaves the machine idle and a product bound by memory runs beside one bound by arithmetic.
//
// Waits.  Every wait on a barrier is bounded (kWaitLimit polls).  One that runs out sets an abort flag in shared memory
// and TSLT_STATUS_WAIT_TIMEOUT in the status word; every role then leaves its loop, copies in flight are waited for
// (bounded as well), tensor memory is freed and the kernel returns.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "tslt_common.cuh"

namespace tslt {
namespace gemm {

constexpr int kBarrierBytes = 1024;      // barriers and flags at the start of shared memory
constexpr int kStageA = 128 * 128;       // bytes of A per CTA and stage
constexpr int kMaxStages = 12;
constexpr int kSmemLimit = 227 * 1024;
constexpr int kStageOut = 4096;          // bytes of an epilogue warp's output box: 32 rows of 128 bytes
constexpr int kScratch = 256;            // bytes of an epilogue warp's scratch (where the epilogue has output boxes)
constexpr int kTmemCols = 512;
constexpr int kAccCols = 256;            // columns of one accumulator buffer
constexpr int kWaitLimit = 1 << 22;

// One product.  m_limit / k_limit (device, may be null): the number of rows / of k actually present, at most the
// host's figures; tiles beyond them are skipped.
struct Product {
    int m_tiles, n_tiles, splits;  // tiles of 128 * kCtas rows, of nt columns; cuts of k
    int k_blocks;                  // stages of k in all (128 bytes of k each when K-major, 64 elements when MN-major)
    int nt, stages, group_m;
    int a_layout, b_layout;        // Layout
    int pitch;                     // rows of a panel (kPanelsK)
    int k_elems;                   // elements of k in a stage
    int m_total;                   // rows of A
    const int* m_limit;
    const int* k_limit;
    uint32_t idesc;
    int clear_status;  // CTA 0 clears the status word first (another sets it only after a wait of kWaitLimit polls)
    int* status;
};

struct WarpSmem {  // an epilogue warp's own shared memory: two output boxes used in turn, and a scratch
    uint32_t box, scratch;
    int turn;
};

struct Tile {
    int m, n, split;   // tile coordinates
    int row0;          // global row of this CTA's lane 0
    int rows;          // rows of A there are (the limit, not the tile's)
    int col0, nt;
    int k_begin, k_end;  // in stages
};

// ---- PTX ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <int kCtas>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if (kCtas == 2)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
}
template <int kCtas>
__device__ __forceinline__ void tma_load3(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    if (kCtas == 2)
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
}
// How an operand lies in memory, and so how a stage of it is copied.  Few large boxes: the copy engine's rate falls with the
// number of instructions (stages of four 8 KB boxes instead of two of 16 KB: 570 instead of 390 us for the copies alone of
// a 6144 x 16128 x 4096 product).
enum Layout {
    kRowsK = 0,    // row-major, k contiguous: box of 128 bytes of k by n rows
    kPanelsK = 1,  // panels, k along the columns: the same box, contiguous memory
    kBlocksMN = 2, // m (n) contiguous, seen as [64-column blocks][k][64]: one box for the whole stage.  Panels, or a row-major
                   // matrix whose width is a multiple of 64
    kRowsMN = 3,   // m (n) contiguous, row-major of any width: a box for each 64 columns
};
// A stage: `n` rows of the operand from mn0 on, 128 bytes of k (64 elements of it when m is contiguous) from k0 on.
template <int kCtas>
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* map, int layout, int pitch, int mn0, int n, int k0, uint32_t bar) {
    if (layout == kRowsK) tma_load<kCtas>(dst, map, k0, mn0, bar);
    else if (layout == kPanelsK) tma_load<kCtas>(dst, map, 0, (k0 >> 6) * pitch + mn0, bar);
    else if (layout == kBlocksMN) tma_load3<kCtas>(dst, map, 0, k0, mn0 >> 6, bar);
    else
        for (int j = 0; j < n; j += 64) tma_load<kCtas>(dst + j * 128, map, mn0 + j, k0, bar);
}
template <int kCtas> __device__ __forceinline__ void tmem_alloc(uint32_t dst_smem) {
    if (kCtas == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <int kCtas> __device__ __forceinline__ void tmem_free(uint32_t tmem) {
    if (kCtas == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols));
}
template <int kCtas, bool kInt8>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
#define TSLT_MMA(GROUP, KIND)                                                                   \
    asm volatile(                                                                               \
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"                                       \
        "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, p;\n\t}" ::"r"(d),   \
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)                                             \
        : "memory")
    if (kCtas == 2) {
        if (kInt8) TSLT_MMA("2", "i8");
        else TSLT_MMA("2", "f16");
    } else {
        if (kInt8) TSLT_MMA("1", "i8");
        else TSLT_MMA("1", "f16");
    }
#undef TSLT_MMA
}
// Arrives on the barrier (of both CTAs of a pair) when every product issued so far has completed.
template <int kCtas> __device__ __forceinline__ void mma_commit(uint32_t bar) {
    if (kCtas == 2)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of this warp's 32 lanes (all of them take part: they meet first); the values may be used after tmem_wait32().
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t* r) {
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
// The registers are operands of the wait, so that no use of them moves above it.
__device__ __forceinline__ void tmem_wait32(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
          "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
          "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
          "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
        :
        : "memory");
}
__device__ __forceinline__ uint32_t tmem_ld1(uint32_t addr) {  // one column, waited for
    uint32_t v;
    __syncwarp();
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

template <int kPending> __device__ __forceinline__ void store_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kPending) : "memory");
}
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// An epilogue warp's output box: 32 rows of 128 bytes (lane l's row in b), written with the 128-byte swizzle (16-byte chunk i of row r
// at chunk i ^ (r mod 8)) and sent off by one lane as one copy, which clips it at the matrix's edges.  The boxes change at a copy and at
// nothing else, so that "all copies but the newest have read their box" always speaks of this box: what is not copied out takes no box.
__device__ __forceinline__ void send_box(WarpSmem& own, const uint32_t* b, int lane, const CUtensorMap* map, int x, int y) {
    if (lane == 0) store_wait_read<1>();
    __syncwarp();
    const uint32_t box = own.box + own.turn * kStageOut, line = box + lane * 128;
    own.turn ^= 1;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(line + ((i ^ (lane & 7)) << 4)), "r"(b[4 * i]), "r"(b[4 * i + 1]),
                     "r"(b[4 * i + 2]), "r"(b[4 * i + 3])
                     : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(box) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}

// Shared-memory matrix descriptor, 128-byte swizzle.  K-major: rows of 128 bytes, 8-row groups 1024 bytes apart (sbo).
// MN-major: 64 contiguous elements of m per 128-byte row, one row per k; 8-k groups 1024 bytes apart (sbo), the next
// 64 elements of m `lbo` bytes on.
__device__ __forceinline__ uint64_t make_desc(uint32_t addr, uint32_t lbo) {
    return (uint64_t)((addr >> 4) & 0x3fff) | ((uint64_t)((lbo >> 4) & 0x3fff) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}

struct Waiter {
    volatile int* abort;
    int* status;
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const {
        if (mbar_try(bar, parity)) return true;
        for (int i = 0; i < kWaitLimit; ++i) {
            if (mbar_try(bar, parity)) return true;
            if (*abort) return false;
        }
        *abort = 1;
        atomicOr(status, TSLT_STATUS_WAIT_TIMEOUT);
        return false;
    }
};

// The tiles of a product: every role of both CTAs decodes the same list.  Order: groups of group_m row tiles, all column tiles
// of a group before the next group, row tiles fastest (the rows of a group stay in L2 while B streams).
struct Walk {
    int m_tiles, per_split, total, rows, k_blocks;
    __device__ __forceinline__ Walk(const Product& p, int tile_rows) {
        rows = p.m_limit ? min(*p.m_limit, p.m_total) : p.m_total;
        m_tiles = p.m_limit ? min((rows + tile_rows - 1) / tile_rows, p.m_tiles) : p.m_tiles;
        k_blocks = p.k_limit ? min((*p.k_limit + p.k_elems - 1) / p.k_elems, p.k_blocks) : p.k_blocks;
        per_split = m_tiles * p.n_tiles;
        total = per_split * p.splits;
    }
    __device__ __forceinline__ Tile at(const Product& p, int idx, int tile_rows, int rank) const {
        Tile t;
        t.split = idx / per_split;
        idx -= t.split * per_split;
        const int per_group = p.group_m * p.n_tiles;
        const int g = idx / per_group;
        idx -= g * per_group;
        const int first = g * p.group_m, width = min(p.group_m, m_tiles - first);
        t.n = idx / width;
        t.m = first + (idx - t.n * width);
        t.row0 = t.m * tile_rows + rank * 128;
        t.rows = rows;
        t.col0 = t.n * p.nt;
        t.nt = p.nt;
        t.k_begin = (int)((long long)k_blocks * t.split / p.splits);
        t.k_end = (int)((long long)k_blocks * (t.split + 1) / p.splits);
        return t;
    }
};

// Which tiles a cluster takes.  The first product's in turn: q or q + 1 of them, the first r clusters one more.  Then the second's:
// the clusters that had one less take `ahead` of its tiles before the others join, as many as that one tile was worth.
struct Plan {
    int clusters, cluster, total1, total2, mine1, fewer, ahead;
    __device__ __forceinline__ Plan(int cluster_, int clusters_, int total1_, int total2_, int cost1, int cost2)
        : clusters(clusters_), cluster(cluster_), total1(total1_), total2(total2_) {
        const int r = total1 % clusters;
        mine1 = total1 / clusters + (cluster < r);
        fewer = clusters - r;  // clusters with one tile less (all of them when r = 0)
        ahead = r ? (cost1 + cost2 / 2) / cost2 : 0;
    }
    // the i-th tile of this cluster: its number in its product, or -1 behind the last
    __device__ __forceinline__ int at(int i, bool* second) const {
        *second = i >= mine1;
        if (i < mine1) return cluster + i * clusters;
        i -= mine1;
        const int first = clusters - fewer;
        int n;
        if (cluster >= first && i < ahead) n = i * fewer + cluster - first;
        else n = ahead * fewer + (cluster >= first ? i - ahead : i) * clusters + cluster;
        return n < total2 ? n : -1;
    }
};

struct Maps {
    CUtensorMap a, b;
};
struct NoEpilogue {
    static constexpr bool kOutBox = false;
    struct Params {};
};
// A tile whose sum is short costs its epilogue: about ten stages.
__device__ __forceinline__ int tile_cost(int k_blocks) { return k_blocks > 10 ? k_blocks : 10; }

template <bool kInt8, int kCtas, int kEpiWarps, class Epi, class Epi2>
__global__ void __launch_bounds__(64 + 32 * kEpiWarps, 1)
    gemm_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Product p, const __grid_constant__ typename Epi::Params ep,
                const __grid_constant__ Maps maps2, const __grid_constant__ Product p2, const __grid_constant__ typename Epi2::Params ep2) {
    constexpr bool kDual = !std::is_same<Epi2, NoEpilogue>::value;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u;
    uint8_t* const basep = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t full = base, empty = base + 8 * kMaxStages, tfull = base + 16 * kMaxStages, tempty = tfull + 16,
                   drain = tfull + 32, tmem_slot = tfull + 40;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(basep + 16 * kMaxStages + 48);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = kCtas == 2 ? cluster_rank() : 0;
    constexpr int kTileRows = 128 * kCtas;
    const int bytes_b = p.nt / kCtas * 128, stage_bytes = kStageA + bytes_b;
    const uint32_t data = base + kBarrierBytes;
    const int cluster = blockIdx.x / kCtas, clusters = gridDim.x / kCtas;

    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(tfull + 8 * i, 1);
            mbar_init(tempty + 8 * i, kEpiWarps * kCtas);
        }
        mbar_init(drain, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.b) : "memory");
    }
    if (warp == 1) tmem_alloc<kCtas>(tmem_slot);
    tc_fence_before();
    if (kCtas == 2) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(basep + 16 * kMaxStages + 40);
    wait_for_primary_kernel();  // the set-up above overlaps the end of the kernel before this one in the call
    allow_dependent_launch();
    if (p.clear_status && blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0;
    const Waiter wait = {abort_flag, p.status};
    const Walk walk(p, kTileRows), walk2(kDual ? p2 : p, kTileRows);
    const Plan plan(cluster, clusters, walk.total, kDual ? walk2.total : 0, tile_cost(walk.k_blocks / p.splits), tile_cost(walk2.k_blocks));
    bool second;

    if (warp == 0) {
        if (lane == 0) {
            const uint32_t tx = (uint32_t)stage_bytes * kCtas;
            int stage = 0, phase = 0;
            bool ok = true;
            for (int i = 0, idx; ok && (idx = plan.at(i, &second)) >= 0; ++i) {
                const bool two = kDual && second;
                const Tile t = two ? walk2.at(p2, idx, kTileRows, rank) : walk.at(p, idx, kTileRows, rank);
                const int brow = t.col0 + rank * (p.nt / kCtas);
                const int a_layout = two ? p2.a_layout : p.a_layout, b_layout = two ? p2.b_layout : p.b_layout;
                const int pitch = two ? p2.pitch : p.pitch, k_elems = two ? p2.k_elems : p.k_elems;
                const CUtensorMap *ta = two ? &maps2.a : &maps.a, *tb = two ? &maps2.b : &maps.b;
                for (int kb = t.k_begin; kb < t.k_end; ++kb) {
                    if (!wait(empty + 8 * stage, phase ^ 1)) {
                        ok = false;
                        break;
                    }
                    const uint32_t sa = data + stage * stage_bytes, sb = sa + kStageA;
                    uint32_t bar = full + 8 * stage;
                    if (rank == 0) mbar_expect(bar, tx);
                    if (kCtas == 2) bar = map_to_rank(bar, 0);
                    const int k0 = kb * k_elems;
                    load_operand<kCtas>(sa, ta, a_layout, pitch, t.row0, 128, k0, bar);
                    load_operand<kCtas>(sb, tb, b_layout, pitch, brow, p.nt / kCtas, k0, bar);
                    if (++stage == p.stages) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
            }
            for (int i = 0; i < p.stages && ok; ++i) {  // the last products have read shared memory, and told so
                ok = wait(empty + 8 * stage, phase ^ 1);
                if (++stage == p.stages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
            if (!ok && rank == 0) {  // leave no copy in flight behind: wait for the stages already asked for
                for (int i = 0; i < p.stages; ++i) {
                    const int par = i < stage ? phase : phase ^ 1;
                    for (int n = 0; n < kWaitLimit / 16 && !mbar_try(full + 8 * i, par); ++n) {}
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            int stage = 0, phase = 0, acc = 0, acc_phase = 0;
            bool ok = true;
            for (int i = 0, idx; ok && (idx = plan.at(i, &second)) >= 0; ++i) {
                const bool two = kDual && second;
                const Tile t = two ? walk2.at(p2, idx, kTileRows, rank) : walk.at(p, idx, kTileRows, rank);
                const bool a_mn = (two ? p2.a_layout : p.a_layout) >= kBlocksMN, b_mn = (two ? p2.b_layout : p.b_layout) >= kBlocksMN;
                const uint32_t a_step = a_mn ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;
                const uint32_t idesc = two ? p2.idesc : p.idesc;
                if (t.k_begin >= t.k_end) continue;  // nothing to add up: the epilogue takes zeros
                if (!wait(tempty + 8 * acc, acc_phase ^ 1)) break;
                tc_fence_after();
                const uint32_t d = tmem + acc * kAccCols;
                for (int kb = t.k_begin; kb < t.k_end; ++kb) {
                    if (!wait(full + 8 * stage, phase)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t sa = data + stage * stage_bytes;
                    const uint64_t da = make_desc(sa, a_mn ? 8192 : 16), db = make_desc(sa + kStageA, b_mn ? 8192 : 16);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mma<kCtas, kInt8>(d, da + j * a_step, db + j * b_step, idesc, kb > t.k_begin || j > 0);
                    mma_commit<kCtas>(empty + 8 * stage);
                    if (++stage == p.stages) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
                if (!ok) break;
                mma_commit<kCtas>(tfull + 8 * acc);
                acc ^= 1;
                if (acc == 0) acc_phase ^= 1;
            }
            if (*abort_flag) {  // the products already issued end before tensor memory is given back
                mma_commit<kCtas>(drain);
                for (int n = 0; n < kWaitLimit / 16 && !mbar_try(drain, 0); ++n) {}
            }
        }
    } else {
        const int quad = warp & 3, part = (warp - 2) >> 2;
        const uint32_t out = data + p.stages * stage_bytes;
        WarpSmem own = {out + (warp - 2) * 2 * kStageOut, out + kEpiWarps * 2 * kStageOut + (warp - 2) * kScratch, 0};
        int acc = 0, acc_phase = 0;
        for (int i = 0, idx; (idx = plan.at(i, &second)) >= 0; ++i) {
            const bool two = kDual && second;
            const Tile t = two ? walk2.at(p2, idx, kTileRows, rank) : walk.at(p, idx, kTileRows, rank);
            const bool empty_sum = t.k_begin >= t.k_end;
            if (!empty_sum) {
                const bool got = wait(tfull + 8 * acc, acc_phase);
                if (!__all_sync(0xffffffffu, got)) break;
                tc_fence_after();
            }
            const uint32_t sums = tmem + ((uint32_t)(quad * 32) << 16) + acc * kAccCols;
            const int row = t.row0 + quad * 32 + lane;
            if constexpr (kDual) {
                if (two) Epi2::template run<kEpiWarps / 4>(ep2, sums, empty_sum, t, row, lane, part, own);
                else Epi::template run<kEpiWarps / 4>(ep, sums, empty_sum, t, row, lane, part, own);
            } else {
                Epi::template run<kEpiWarps / 4>(ep, sums, empty_sum, t, row, lane, part, own);
            }
            if (!empty_sum) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(kCtas == 2 ? map_to_rank(tempty + 8 * acc, 0) : map_to_rank(tempty + 8 * acc, rank));
                acc ^= 1;
                if (acc == 0) acc_phase ^= 1;
            }
        }
    }
    if ((Epi::kOutBox || Epi2::kOutBox) && warp >= 2 && lane == 0) store_wait_all();
    __syncwarp();
    tc_fence_before();
    if (kCtas == 2) cluster_sync();
    else __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_free<kCtas>(tmem);
    }
}

// ---- host --------------------------------------------------------------------------------------------------
// A 2-d tensor map of `outer` rows of `inner` elements (row stride in bytes, a multiple of 16), boxes of box_inner x
// box_outer with box_inner elements = 128 bytes.
// encode_blocks: bf16 as [blocks][rows][64] (kBlocksMN), boxes of box_blocks x 64 x 64; strides in bytes.
enum Element { kElemInt8, kElemBf16, kElemFp32 };
bool encode_blocks(CUtensorMap* map, const void* base, long long rows, long long row_bytes, long long blocks, long long block_bytes, int box_blocks);
bool encode_map(CUtensorMap* map, Element e, const void* base, long long inner, long long outer, long long row_bytes, int box_outer);

inline int sm_count() {  // of the current device; 0 if it cannot be found out
    static int cached[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
    if (dev < 64 && cached[dev]) return cached[dev];
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev < 64) cached[dev] = n;
    return n;
}

inline uint32_t instruction_desc(bool int8, int m, int n, bool a_mn, bool b_mn) {
    const uint32_t d = int8 ? 2u : 1u, ab = 1u;  // accumulator s32 / f32; operands s8 / bf16
    return d << 4 | ab << 7 | ab << 10 | (a_mn ? 1u << 15 : 0) | (b_mn ? 1u << 16 : 0) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

// A kernel that waits for the one before it on the stream itself (wait_for_primary_kernel() before it touches global memory), so
// that its launch and set-up overlap that kernel's end, whatever kernel that is: one that never allows dependents early
// simply ends first.  Whatever such a kernel reads may have been written during its own life, by the kernel before it: its loads are
// plain ones, none through the path for data that nobody writes meanwhile.
template <typename... Params, typename... Args>
cudaError_t launch_early(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

// Fills idesc and stages from nt, launches on min(tiles, SMs) clusters.
template <bool kInt8, int kCtas, int kEpiWarps, class Epi, class Epi2>
int launch_two(const Maps& maps, Product p, const typename Epi::Params& ep, const Maps& maps2, Product p2, const typename Epi2::Params& ep2,
               cudaStream_t st) {
    constexpr bool kDual = !std::is_same<Epi2, NoEpilogue>::value;
    const int sms = sm_count();
    if (sms <= 0) return TSLT_ERR_CUDA;
    const int stage = kStageA + p.nt / kCtas * 128, boxes = Epi::kOutBox || Epi2::kOutBox ? kEpiWarps * (2 * kStageOut + kScratch) : 0;
    p.stages = (kSmemLimit - 1024 - kBarrierBytes - boxes) / stage;
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    p.idesc = instruction_desc(kInt8, 128 * kCtas, p.nt, p.a_layout >= kBlocksMN, p.b_layout >= kBlocksMN);
    p2.idesc = instruction_desc(kInt8, 128 * kCtas, p.nt, p2.a_layout >= kBlocksMN, p2.b_layout >= kBlocksMN);
    auto kern = gemm_kernel<kInt8, kCtas, kEpiWarps, Epi, Epi2>;
    const int smem = 1024 + kBarrierBytes + p.stages * stage + boxes;
    static bool done[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return TSLT_ERR_CUDA;
    if (dev < 0 || dev >= 64 || !done[dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) != cudaSuccess) return TSLT_ERR_CUDA;
        if (dev >= 0 && dev < 64) done[dev] = true;
    }
    const long long tiles = (long long)p.m_tiles * p.n_tiles * p.splits, tiles2 = kDual ? (long long)p2.m_tiles * p2.n_tiles * p2.splits : 0;
    if (tiles + tiles2 <= 0) return TSLT_OK;
    if (tiles > 0x3fffffffLL || tiles2 > 0x3fffffffLL) return TSLT_ERR_UNSUPPORTED;
    const long long clusters = tiles + tiles2 < sms / kCtas ? tiles + tiles2 : sms / kCtas;
    return launch_early(kern, dim3((unsigned)(clusters * kCtas)), 64 + 32 * kEpiWarps, smem, kCtas, st, maps, p, ep, maps2, p2, ep2) == cudaSuccess
               ? TSLT_OK
               : TSLT_ERR_CUDA;
}
template <bool kInt8, int kCtas, int kEpiWarps, class Epi>
int launch(const Maps& maps, const Product& p, const typename Epi::Params& ep, cudaStream_t st) {
    return launch_two<kInt8, kCtas, kEpiWarps, Epi, NoEpilogue>(maps, p, ep, maps, p, NoEpilogue::Params{}, st);
}

// The column width of a tile, a multiple of `unit`, at most 256: the one whose rounds of tiles over the machine's clusters cost
// least, the widest of equals.  A stage costs nt + 256 (pair; nt + 128 for a single CTA) in units of its time in shared
// memory, which its copies in and the tensor cores' reads share: 128 rows of A and the CTA's part of B, once each.
inline int choose_nt(long long m_tiles, long long cols, bool pair, int unit) {
    const long long slots = pair ? 74 : 148;
    int best = 256;
    long long least = -1;
    for (int nt = 256; nt >= 64; nt -= unit) {
        const long long tiles = m_tiles * ((cols + nt - 1) / nt), cost = (tiles + slots - 1) / slots * (nt + (pair ? 256 : 128));
        if (least < 0 || cost < least) {
            least = cost;
            best = nt;
        }
    }
    return best;
}

// Row tiles of a group: as many as keep the group's rows of A in half of L2, so that B streams past them from HBM once (6144 rows,
// sustained: groups of 24 / 16 / 8 tiles 597 / 607 / 621 us for a piece of z).
inline int rows_in_l2(long long tile_rows, long long row_bytes) {
    const long long n = (64ll << 20) / (tile_rows * row_bytes);
    return n < 1 ? 1 : n > 1024 ? 1024 : (int)n;
}

}  // namespace gemm
}  // namespace tslt
