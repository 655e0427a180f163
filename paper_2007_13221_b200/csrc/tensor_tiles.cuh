// tensor_tiles.cuh - the tile pipeline under the operators of cser_train.h (sm_100a): products on the
// fifth-generation tensor cores with operands brought by asynchronous copies, accumulators in tensor memory, and
// an epilogue of the operator's own.  Device code; included by orth.cu and xent.cu inside their unnamed namespaces.
//
// Roles.  A CTA is 20 warps: warp 0 issues the copies, warp 1 issues the matrix instructions, warp 2 works out what the next
// tiles are, waits for what they read and leaves them in shared memory, warp 3 may copy for the epilogue, warps 4-19 are the
// epilogue (warp w reads
// the tensor-memory lanes 32*(w%4)..+31, the quarter (w-4)/4 of the columns; with 8 epilogue warps, two to a scheduler, the
// latencies of their arithmetic showed: 3000 cycles for 128 x 64 values).  Two
// accumulators of 256 columns take turns, so the epilogue of one tile runs under the products of the next.  With
// CG = 2 the CTAs of a cluster of two work on one 256 x 256 tile: each brings half of both operands (half the
// traffic per product of a single CTA's 128 x 256 tile), and the first one issues the instructions for both.
//
// Operands are 16-bit "panels": 64 columns (128 bytes) wide, rows one after the other, the eight 16-byte chunks
// of row r stored in the order c ^ (r & 7).  That is the 128-byte-swizzled layout the tensor cores read, so a run
// of rows of a panel is one plain bulk copy, and the same bytes serve as an operand whose columns are the
// product's inner dimension ("K-major") or whose rows are ("MN-major"): no operand is ever transposed in memory.
//
// Waits.  Every wait is bounded by the SM's clock.  One that runs out sets a word of the handle that the host
// looks at on every later call, the CTA's other roles see it and leave, copies and products in flight are
// waited for (bounded too), tensor memory is given back, and the kernel ends.
#pragma once

#include "bulk_copy.cuh"

constexpr int kStageK = 64;                        // inner dimension of one stage: one panel's width
constexpr int kEpiWarp0 = 4, kEpiWarps = 16;
constexpr int kThreads = (kEpiWarp0 + kEpiWarps) * 32;

// ------------------------------------------------------------------ small PTX
// Kernels of one call are launched to overlap: the next one's CTAs may set up (barriers, tensor memory) while this one's
// last ones run.  let_next_start() allows it, earlier_done() waits until all earlier kernels are complete and their writes
// visible; nothing that they write, or read and we write, is touched before it.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void earlier_done() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Arrival on the barrier at the same shared-memory offset in CTA `rank` of the cluster.
__device__ __forceinline__ void mbar_arrive_remote(uint64_t *bar, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(bar)), "r"(rank));
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(a) : "memory");
}
// Whether the phase is over, without waiting.
__device__ __forceinline__ bool mbar_test(uint64_t *bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_addr(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
// Bulk copy without an L2 hint.
__device__ __forceinline__ void bulk_copy_in(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(smem_addr(bar))
                 : "memory");
}
// `bytes` from shared memory to global; the thread's copies are counted in groups.
__device__ __forceinline__ void bulk_copy_out(void *dst, uint32_t src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_out_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// Until all but the last LEFT groups have read their source / are done.
template <int LEFT> __device__ __forceinline__ void bulk_out_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void bulk_out_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ uint4 shared_load16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void shared_store16(uint32_t at, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// A box of a three-dimensional tensor (column, row, worker); the column is a multiple of 64 everywhere here.
__device__ __forceinline__ void tensor_copy_in(uint32_t dst, const CUtensorMap *map, int col, int row, int worker,
                                               uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::
            "r"(dst),
        "l"(map), "r"(smem_addr(bar)), "r"(col), "r"(row), "r"(worker)
        : "memory");
}
// The same from shared memory, what lies outside the tensor left out; counted in the thread's groups of copies.
__device__ __forceinline__ void tensor_copy_out(const CUtensorMap *map, uint32_t src, int col, int row, int worker) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(col),
                 "r"(row), "r"(worker)
                 : "memory");
}
__device__ __forceinline__ void prefetch_tensor_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// Between ordinary accesses to shared memory and the copy engine's, and to global memory.  (The fence over both takes about 1100
// cycles: in the epilogue of every panel that was a third of its time.)
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t *dst, uint32_t cols) {
    if constexpr (CG == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(dst)), "r"(cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(dst)), "r"(cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
template <int CG>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
}
// One arrival on `bar` (with CG = 2: on the barrier of both CTAs of the pair) when all products issued so far by
// this thread are done.
template <int CG>
__device__ __forceinline__ void mma_commit(uint64_t *bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar))
                     : "memory");
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                smem_addr(bar)),
            "h"((uint16_t)3)
            : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 16 or 32 columns of this warp's 32 lanes: thread = lane (row), register = column.
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// Shared-memory operand descriptor, 128-byte swizzle, without the address (its bits 4..17 go into the lowest 14).  K-major:
// 8-row groups are 1024 bytes apart.  MN-major: panels of 64 along M or N are 64 rows (8192 bytes) apart, 8-row groups
// along K 1024 bytes.
__device__ __forceinline__ constexpr uint64_t operand_desc(bool mn) {
    return ((uint64_t)(mn ? 8192 / 16 : 1) << 16) | ((uint64_t)(1024 / 16) << 32) | (1ull << 46) | (2ull << 61);
}
// Descriptor units (16 bytes) from one 16 of the inner dimension to the next inside a stage.
__device__ __forceinline__ constexpr uint32_t operand_step(bool mn) { return mn ? 2048 / 16 : 32 / 16; }
// Instruction descriptor: fp32 accumulators, A and B both fp16 (0) or bf16 (1), M = 128 * CG; bits 15 and 16 say that A and
// B are MN-major.
__device__ __forceinline__ uint32_t instr_desc(int bf16, int n, int cg) {
    return (1u << 4) | ((uint32_t)bf16 << 7) | ((uint32_t)bf16 << 10) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(128 * cg >> 4) << 24);
}

// Byte offset of the 16-byte chunk `c` (0..7) of row r inside a panel.
__device__ __forceinline__ uint32_t panel_chunk(uint32_t row, uint32_t c) { return row * 128 + ((c ^ (row & 7)) << 4); }

// ------------------------------------------------------------------ rows of results
__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t pack_bf162(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// min(n, N) values to 16-bit elements at, at + 1, ... ; 16 bytes at a time where they are aligned.
template <int N>
__device__ __forceinline__ void store_row(void *base, long long at, int n, bool bf16, const float (&v)[N]) {
    uint32_t w[N / 2];
#pragma unroll
    for (int k = 0; k < N / 2; ++k) w[k] = bf16 ? pack_bf162(v[2 * k], v[2 * k + 1]) : pack_half2(v[2 * k], v[2 * k + 1]);
    uint16_t *o = static_cast<uint16_t *>(base) + at;
    if (n >= N && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
#pragma unroll
        for (int k = 0; k < N / 8; ++k)
            reinterpret_cast<uint4 *>(o)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < n) o[k] = (uint16_t)(k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffff);
    }
}

// ------------------------------------------------------------------ the pipeline
// TN: columns of a tile (at most 256).  EXTRA: bytes of shared memory for the epilogue, a multiple of 1024.  PAIR: operands are
// pairs hi + lo of 16-bit values: a stage holds all four and makes hi hi in one accumulator and hi lo + lo hi, 2^-11 of it, in
// another (three products as three passes over the inner dimension brought half as many bytes again, and the copies were the
// bound); TN is at most 128 then.
template <int CG, int TN = 256, int EXTRA = 0, bool PAIR = false>
struct Pipe {
    static constexpr int kABytes = 128 * 128;                       // this CTA's 128 rows of the first operand
    static constexpr int kBBytes = TN / CG * 128;                   // this CTA's share of the second
    static constexpr int kLoOffset = kABytes + kBBytes;             // of the lo halves in a stage
    static constexpr int kStageBytes = (kABytes + kBBytes) * (PAIR ? 2 : 1);
    static constexpr int kAccCols = PAIR ? 128 : 256;               // of an accumulator; two, and two more for the small products
    static_assert(TN <= kAccCols, "an accumulator's columns");
    static constexpr int kStages = (225 * 1024 - EXTRA) / kStageBytes;

    static constexpr int kTiles = 4, kTileBytes = 256;               // tiles known ahead

    struct Shared {
        uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], small_full[2], small_empty[2], drain;
        uint64_t extra_full[3], extra_done[3], extra_free[3];         // the epilogue's buffers, see orth.cu
        uint64_t tile_full[kTiles], tile_empty[kTiles];
        uint32_t tmem;
        volatile int dead;
        alignas(16) unsigned char tile[kTiles][kTileBytes];
    };
    static constexpr size_t kSharedBytes = 1024 + (size_t)kStages * kStageBytes + EXTRA + sizeof(Shared);
    static_assert(kSharedBytes <= 227 * 1024, "shared memory of a CTA");

    uint32_t stage0, extra;                                         // 1024-byte aligned shared addresses
    Shared *sh;
    unsigned *err;                                                  // the handle's word, mapped host memory
    uint32_t rank;
    long long limit;                                                // of a wait, in cycles

    __device__ __forceinline__ void fail() {
        sh->dead = 1;
        if (err) {
            *reinterpret_cast<volatile unsigned *>(err) = 1u;
            __threadfence_system();
        }
    }
    __device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity) {
        if (mbar_try_wait(bar, parity)) return true;
        const long long t0 = clock64();
        for (;;) {
#pragma unroll 1
            for (int k = 0; k < 64; ++k)
                if (mbar_try_wait(bar, parity)) return true;
            if (sh->dead) return false;
            if (clock64() - t0 > limit) {
                fail();
                return false;
            }
        }
    }
    // Until *counter >= target (written by other CTAs of this launch, which are all resident).
    __device__ __forceinline__ bool wait_counter(const unsigned *counter, unsigned target) {
        unsigned v;
        const long long t0 = clock64();
        for (int k = 0;; ++k) {
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
            if (v >= target) return true;
            if (sh->dead) return false;
            if ((k & 63) == 63 && clock64() - t0 > limit) {
                fail();
                return false;
            }
        }
    }

    template <class Job>
    __device__ __forceinline__ void setup(unsigned char *raw, unsigned *err_word, long long wait_cycles = kWaitCycles) {
        static_assert(sizeof(typename Job::Tile) <= kTileBytes && alignof(typename Job::Tile) <= 16, "a tile in shared memory");
        stage0 = (smem_addr(raw) + 1023u) & ~1023u;
        extra = stage0 + kStages * kStageBytes;
        sh = reinterpret_cast<Shared *>(raw + (extra - smem_addr(raw)) + EXTRA);
        err = err_word, limit = wait_cycles;
        rank = CG == 1 ? 0 : cluster_rank();
        if (threadIdx.x == 0) {
            for (int s = 0; s < kStages; ++s) {
                mbar_init(&sh->full[s], CG == 2 && rank == 0 ? 2 : 1);   // the peer's copies are passed on by an arrival
                mbar_init(&sh->empty[s], 1);
            }
            for (int k = 0; k < 2; ++k) {
                mbar_init(&sh->acc_full[k], 1), mbar_init(&sh->acc_empty[k], kEpiWarps * CG);
                mbar_init(&sh->small_full[k], 1), mbar_init(&sh->small_empty[k], kEpiWarps * CG);
            }
            for (int k = 0; k < 3; ++k)
                mbar_init(&sh->extra_full[k], 1), mbar_init(&sh->extra_done[k], kEpiWarps), mbar_init(&sh->extra_free[k], kEpiWarps);
            for (int k = 0; k < kTiles; ++k)
                mbar_init(&sh->tile_full[k], 1), mbar_init(&sh->tile_empty[k], 2 + kEpiWarps + Job::kCopier);
            mbar_init(&sh->drain, 1);
            sh->dead = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            mbar_init_fence();
        }
        if (threadIdx.x / 32 == 2) tmem_alloc<CG>(&sh->tmem, 512);
        tmem_fence_before();
        __syncthreads();
        if (CG == 2) cluster_sync_all();
        tmem_fence_after();
    }

    // Which accumulator an epilogue warp takes next.
    struct Turn {
        int acc = 0;
        uint32_t ph = 0;
        int small = 0;                                              // of the small products', one a tile
        uint32_t small_ph = 0;
    };
    // One role's way through the tiles.
    struct Walk {
        int slot = 0;
        uint32_t ph = 0;
        __device__ __forceinline__ void step() {
            if (++slot == kTiles) slot = 0, ph ^= 1;
        }
    };
    template <class T>
    __device__ __forceinline__ const T *tile_at(const Walk &w) const { return reinterpret_cast<const T *>(sh->tile[w.slot]); }
    __device__ __forceinline__ void tile_done(Walk &w) {
        mbar_arrive(&sh->tile_empty[w.slot]);
        w.step();
    }

    // Runs the tiles that `job` lists.  What a role does per stage is kept to a few instructions: one thread issues
    // a stage's copies and one its products, about 500 cycles' worth, and address arithmetic there is what it waits for
    // (a kernel that worked out descriptors and majorness anew in every stage ran at 1.08 instead of 1.5 PFLOP/s).  Nor does
    // a role look up what the next tile is: a chain of loads from the lists in memory at each tile's start left
    // the tensor cores idle for about 2 us a tile.  Job:
    //   Tile                       all that the roles need of a tile; n: columns, a multiple of 64 * CG, 0: no more tiles; stages: its inner
    //                              dimension; a_lim, b_lim: from which stage on that operand is MN-major
    //   void tile(Tile &, int i, int rank)   the i-th tile of this CTA (pair); each lane asks for growing i only
    //   bool chunk_ends(tile, k)   after this stage the epilogue takes the accumulator (always after the last)
    //   kWaits; bool ready(pipe, tile)   whether tiles read what this launch writes; then waits until that is in memory (before any role
    //                              hears of the tile).  If not, the launch may overlap the end of the kernel before it: tiles are worked
    //                              out from the kernel's arguments alone, and every role calls earlier_done() before its first wait for
    //                              another role's work: however long the kernel before it takes, that is no wait of this one
    //   Loader                     made from a tile; uint32_t bytes(); settle(job, tile), unless kWaits: what it reads that earlier kernels
    //                              wrote; void load(k, a, b, bar): copies of bytes() bytes into a and b (shared addresses; the lo halves
    //                              of pairs kLoOffset behind)
    //   int bf16()
    //   bool epilogue(pipe, tile, turn, warp, lane)   warp 0..15: for each chunk take(), read its columns, release();
    //                              false once a wait was.  Its warps do not wait for one another but on bounded barriers
    //   kRemainders; bool remainders()   whether rows 32..63 of the first operand are what rounding left of its rows 0..31, which are all
    //              there are: they meet the second operand's same 16 bits, with no copy and no stage of their own
    //   kCopier; bool copier(pipe)  a thread of its own for what the epilogue brings and takes away through shared memory; walks the
    //                              tiles itself
    template <class Job>
    __device__ __forceinline__ void run(Job &job) {
        typedef typename Job::Tile Tile;
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        Walk walk;
        bool ok = true;
        if (warp == 0 && lane == 0) {
            int s = 0, issued = 0;
            uint32_t ph = 0;
            bool first = !Job::kWaits;
            while (ok) {
                ok = wait(&sh->tile_full[walk.slot], walk.ph);
                const Tile &t = *tile_at<Tile>(walk);
                if (!ok || t.n == 0) break;
                if (Job::kWaits) fence_async_global();  // what ready() saw written, for the copy engine
                typename Job::Loader from(job, t);
                const uint32_t bytes = from.bytes();
                const int stages = t.stages;
                if (first) earlier_done(), fence_async_global(), first = false;
                if constexpr (!Job::kWaits) from.settle(job, t);
                tile_done(walk);
                for (int k = 0; k < stages; ++k) {
                    ok = wait(&sh->empty[s], ph ^ 1);
                    if (!ok) break;
                    mbar_arrive_expect(&sh->full[s], bytes);
                    const uint32_t at = stage0 + (uint32_t)s * kStageBytes;
                    from.load(k, at, at + kABytes, &sh->full[s]);
                    ++issued;
                    if (++s == kStages) s = 0, ph ^= 1;
                }
            }
            if (!ok) {                                  // copies in flight land before the CTA's memory is given up
                const long long t0 = clock64();
                const int pending = issued < kStages ? issued : kStages;
                for (int k = 0; k < pending; ++k) {
                    s = s == 0 ? kStages - 1 : s - 1;
                    if (s == kStages - 1) ph ^= 1;
                    while (!(CG == 2 && rank == 0) && !mbar_try_wait(&sh->full[s], ph) && clock64() - t0 < limit) {}
                }
                if (CG == 2 && rank == 0)               // its barriers also count the peer's arrivals: allow time instead
                    while (clock64() - t0 < 2000000ll) {}
            }
        } else if (warp == 1 && lane == 0 && rank == 0) {
            int s = 0;
            uint32_t ph = 0;
            Turn turn;
            const uint32_t tmem = sh->tmem;
            if (!Job::kWaits) earlier_done();
            while (ok) {
                ok = wait(&sh->tile_full[walk.slot], walk.ph);
                if (!ok || tile_at<Tile>(walk)->n == 0) break;
                const Tile t = *tile_at<Tile>(walk);
                tile_done(walk);
                const uint32_t id = instr_desc(job.bf16(), t.n, CG);
                bool fresh = true;
                uint32_t d = 0;
                const uint32_t d_small = tmem + 2 * kAccCols + (uint32_t)turn.small * kAccCols;
                if (PAIR) ok = wait(&sh->small_empty[turn.small], turn.small_ph ^ 1);
                for (int k = 0; ok && k < t.stages; ++k) {
                    if (fresh) {
                        ok = wait(&sh->acc_empty[turn.acc], turn.ph ^ 1);
                        if (!ok) break;
                        d = tmem + (uint32_t)turn.acc * kAccCols;
                    }
                    ok = wait(&sh->full[s], ph);
                    if (!ok) break;
                    tmem_fence_after();
                    const bool a_mn = k >= t.a_lim, b_mn = k >= t.b_lim;
                    const uint32_t at = (stage0 + (uint32_t)s * kStageBytes) >> 4;
                    const uint64_t da = (a_mn ? operand_desc(true) : operand_desc(false)) + at;
                    const uint64_t db = (b_mn ? operand_desc(true) : operand_desc(false)) + at + (kABytes >> 4);
                    const uint32_t sa = operand_step(a_mn), sb = operand_step(b_mn);
                    const uint32_t di = id | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16);
                    bool lows = false;
                    if constexpr (Job::kRemainders) lows = job.remainders();
                    if (lows) {
                        const uint32_t lo = a_mn ? 2 * sa : 32 * 128 / 16;   // MN-major: 32 on in the inner dimension; K-major: 32 rows on
#pragma unroll
                        for (int e = 0; e < kStageK / 16; ++e) {
                            if (a_mn && e >= 2) break;
                            mma_f16<CG>(d, da + e * sa, db + e * sb, di, e == 0 ? !fresh : 1);
                            mma_f16<CG>(d, da + lo + e * sa, db + e * sb, di, 1);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < kStageK / 16; ++e)
                            mma_f16<CG>(d, da + e * sa, db + e * sb, di, e == 0 ? !fresh : 1);
                    }
                    if (PAIR) {
                        constexpr uint32_t lo = kLoOffset >> 4;
#pragma unroll
                        for (int e = 0; e < kStageK / 16; ++e) {
                            mma_f16<CG>(d_small, da + e * sa, db + lo + e * sb, di, e == 0 ? k != 0 : 1);
                            mma_f16<CG>(d_small, da + lo + e * sa, db + e * sb, di, 1);
                        }
                    }
                    mma_commit<CG>(&sh->empty[s]);
                    if (++s == kStages) s = 0, ph ^= 1;
                    fresh = job.chunk_ends(t, k);
                    if (fresh) {
                        mma_commit<CG>(&sh->acc_full[turn.acc]);
                        if (++turn.acc == 2) turn.acc = 0, turn.ph ^= 1;
                    }
                }
                if (PAIR && ok) {
                    mma_commit<CG>(&sh->small_full[turn.small]);
                    if (++turn.small == 2) turn.small = 0, turn.small_ph ^= 1;
                }
            }
            if (!ok) {                                  // products in flight end before tensor memory is given back
                mma_commit<CG>(&sh->drain);
                const long long t0 = clock64();
                while (!mbar_try_wait(&sh->drain, 0) && clock64() - t0 < limit) {}
            }
        } else if (CG == 2 && warp == 1 && lane == 0) {
            // The pair's second CTA passes "this stage has landed" on to the first one's barrier.
            int s = 0;
            uint32_t ph = 0;
            if (!Job::kWaits) earlier_done();
            while (ok) {
                ok = wait(&sh->tile_full[walk.slot], walk.ph);
                const Tile &t = *tile_at<Tile>(walk);
                if (!ok || t.n == 0) break;
                int k = t.stages;
                tile_done(walk);
                for (; ok && k > 0; --k) {
                    ok = wait(&sh->full[s], ph);
                    if (ok) mbar_arrive_remote(&sh->full[s], 0);
                    if (++s == kStages) s = 0, ph ^= 1;
                }
            }
        } else if (warp == 2 && lane < kTiles) {
            // Lane l works out every kTiles-th tile, before its place is free.
            Tile t;
            for (int i = lane; ok; i += kTiles) {
                job.tile(t, i, (int)rank);
                if (!Job::kWaits && i == lane + kTiles) earlier_done();
                ok = wait(&sh->tile_empty[lane], (uint32_t)(i / kTiles & 1) ^ 1);
                // One at a time looks at memory: the lane of the tile before has done with it.
                if (ok && i) ok = wait(&sh->tile_full[(i - 1) % kTiles], (uint32_t)((i - 1) / kTiles & 1));
                if (ok && t.n) ok = job.ready(*this, t);
                if (!ok) break;
                *reinterpret_cast<Tile *>(sh->tile[lane]) = t;
                mbar_arrive(&sh->tile_full[lane]);
                if (t.n == 0) break;
            }
        } else if (Job::kCopier && warp == 3 && lane == 0) {
            if constexpr (Job::kCopier) {
                if (!job.copier(*this)) {
                    bulk_out_done();                    // its copies, and time for those into shared memory
                    const long long t0 = clock64();
                    while (clock64() - t0 < 2000000ll) {}
                }
            }
        } else if (warp >= kEpiWarp0) {
            Turn turn;
            if (!Job::kWaits) earlier_done();
            while (ok) {
                ok = warp_wait(&sh->tile_full[walk.slot], walk.ph);
                const Tile &t = *tile_at<Tile>(walk);
                if (!ok || t.n == 0) break;
                ok = job.epilogue(*this, t, turn, warp - kEpiWarp0, lane);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->tile_empty[walk.slot]);
                walk.step();
            }
        }
        __syncwarp();
    }
    // wait() by all lanes of a warp, which go on or leave together.
    __device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity) { return __all_sync(~0u, wait(bar, parity)); }
    // Waits for the next accumulator; `at` is its address for this warp's lanes.
    __device__ __forceinline__ bool take(Turn &t, uint32_t &at) {
        if (!warp_wait(&sh->acc_full[t.acc], t.ph)) return false;
        tmem_fence_after();
        at = acc_at(t);
        return true;
    }
    // Where the accumulator taken last is.
    __device__ __forceinline__ uint32_t acc_at(const Turn &t) const {
        return sh->tmem + (uint32_t)t.acc * kAccCols + ((uint32_t)(threadIdx.x / 32 % 4) << 21);
    }
    // The same for the tile's small products, after its last chunk.
    __device__ __forceinline__ bool take_small(Turn &t, uint32_t &at) {
        if (!warp_wait(&sh->small_full[t.small], t.small_ph)) return false;
        tmem_fence_after();
        at = sh->tmem + (uint32_t)(2 + t.small) * kAccCols + ((uint32_t)(threadIdx.x / 32 % 4) << 21);
        return true;
    }
    __device__ __forceinline__ void release_small(Turn &t, int lane) {
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) {
            if (CG == 1) mbar_arrive(&sh->small_empty[t.small]);
            else mbar_arrive_remote(&sh->small_empty[t.small], 0);
        }
        if (++t.small == 2) t.small = 0, t.small_ph ^= 1;
    }
    // Called by every epilogue warp once it has read its part of the accumulator for the last time.
    __device__ __forceinline__ void release(Turn &t, int lane) {
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) {
            if (CG == 1) mbar_arrive(&sh->acc_empty[t.acc]);
            else mbar_arrive_remote(&sh->acc_empty[t.acc], 0);
        }
        if (++t.acc == 2) t.acc = 0, t.ph ^= 1;
    }
    __device__ __forceinline__ void teardown() {
        tmem_fence_before();
        __syncthreads();
        if (CG == 2) cluster_sync_all();
        tmem_fence_after();
        if (threadIdx.x / 32 == 2) tmem_free<CG>(sh->tmem, 512);
    }
};

// ------------------------------------------------------------------ launches
// `after`: this kernel may be set up while the one before it in the stream, whichever that is, ends (it calls earlier_done()).
template <typename... P, typename... A>
cudaError_t launch_kernel(void (*kernel)(P...), unsigned grid, unsigned block, size_t shared, unsigned cluster, bool after, cudaStream_t st,
                          A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid), cfg.blockDim = dim3(block), cfg.dynamicSmemBytes = shared, cfg.stream = st;
    cudaLaunchAttribute at[2];
    unsigned n = 0;
    if (cluster > 1) {
        at[n].id = cudaLaunchAttributeClusterDimension;
        at[n].val.clusterDim.x = cluster, at[n].val.clusterDim.y = 1, at[n].val.clusterDim.z = 1;
        ++n;
    }
    if (after) {
        at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = at, cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
