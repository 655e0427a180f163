// tensor_tiles.cuh - the tile pipeline under the operators of cser_train.h (sm_100a): products on the
// fifth-generation tensor cores with operands brought by asynchronous copies, accumulators in tensor memory, and
// an epilogue of the operator's own.  Device code; included by orth.cu and xent.cu inside their unnamed namespaces.
//
// Roles.  A CTA is 12 warps: warp 0 issues the copies, warp 1 issues the matrix instructions, warps 4-11 are the
// epilogue (warp w reads the tensor-memory lanes 32*(w%4)..+31, the half (w-4)/4 of a tile's columns).  Two
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
constexpr int kThreads = 384;
constexpr int kEpiWarp0 = 4;
constexpr int kEpiThreads = 256;

// ------------------------------------------------------------------ small PTX
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
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(a) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait_cluster(uint64_t *bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
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
// A box of a three-dimensional tensor (column, row, worker); the column is a multiple of 64 everywhere here.
__device__ __forceinline__ void tensor_copy_in(uint32_t dst, const CUtensorMap *map, int col, int row, int worker,
                                               uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::
            "r"(dst),
        "l"(map), "r"(smem_addr(bar)), "r"(col), "r"(row), "r"(worker)
        : "memory");
}
__device__ __forceinline__ void prefetch_tensor_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async;" ::: "memory"); }

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

// 32 columns of this warp's 32 lanes: thread = lane (row), register = column.
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
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

// Shared-memory operand descriptor, 128-byte swizzle.  K-major: 8-row groups are 1024 bytes apart.  MN-major: panels
// of 64 along M or N are 64 rows (8192 bytes) apart, 8-row groups along K 1024 bytes.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn) {
    const uint64_t lead = mn ? 8192 / 16 : 1, stride = 1024 / 16;
    return (uint64_t)((addr & 0x3ffff) >> 4) | (lead << 16) | (stride << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: fp32 accumulators, A and B both fp16 (0) or bf16 (1), M = 128 * CG.
__device__ __forceinline__ uint32_t instr_desc(int bf16, bool a_mn, bool b_mn, int n, int cg) {
    return (1u << 4) | ((uint32_t)bf16 << 7) | ((uint32_t)bf16 << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 * cg >> 4) << 24);
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
// min(n, 32) values to elements at, at + 1, ... of an array of CSER_TYPE_* `type`; 16 bytes at a time where they are aligned.
__device__ __forceinline__ void store_row32(void *base, long long at, int n, int type, const float (&v)[32]) {
    if (type == CSER_TYPE_F32) {
        float *o = static_cast<float *>(base) + at;
        if (n >= 32 && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                reinterpret_cast<float4 *>(o)[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
        } else {
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (k < n) o[k] = v[k];
        }
    } else {
        uint32_t w[16];
#pragma unroll
        for (int k = 0; k < 16; ++k)
            w[k] = type == CSER_TYPE_BF16 ? pack_bf162(v[2 * k], v[2 * k + 1]) : pack_half2(v[2 * k], v[2 * k + 1]);
        uint16_t *o = static_cast<uint16_t *>(base) + at;
        if (n >= 32 && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                reinterpret_cast<uint4 *>(o)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        } else {
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (k < n) o[k] = (uint16_t)(k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffff);
        }
    }
}

// ------------------------------------------------------------------ the pipeline
template <int CG>
struct Pipe {
    static constexpr int kABytes = 128 * 128;                       // this CTA's 128 rows of the first operand
    static constexpr int kBBytes = (CG == 1 ? 256 : 128) * 128;     // this CTA's share of the second
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = CG == 1 ? 4 : 6;
    static constexpr int kTileM = 128 * CG;

    struct Shared {
        uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drain;
        uint32_t tmem;
        volatile int dead;
    };
    static constexpr size_t kSharedBytes = 1024 + (size_t)kStages * kStageBytes + sizeof(Shared);

    uint32_t stage0;                                                // 1024-byte aligned shared address
    Shared *sh;
    unsigned *err;                                                  // the handle's word, mapped host memory
    uint32_t rank;

    __device__ __forceinline__ void fail() {
        sh->dead = 1;
        if (err) {
            *reinterpret_cast<volatile unsigned *>(err) = 1u;
            __threadfence_system();
        }
    }
    __device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity) {
        if (CG == 1 ? mbar_try_wait(bar, parity) : mbar_try_wait_cluster(bar, parity)) return true;
        const long long t0 = clock64();
        for (;;) {
#pragma unroll 1
            for (int k = 0; k < 64; ++k)
                if (CG == 1 ? mbar_try_wait(bar, parity) : mbar_try_wait_cluster(bar, parity)) return true;
            if (sh->dead) return false;
            if (clock64() - t0 > kWaitCycles) {
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
            if ((k & 63) == 63 && clock64() - t0 > kWaitCycles) {
                fail();
                return false;
            }
        }
    }

    __device__ __forceinline__ void setup(unsigned char *raw, unsigned *err_word) {
        stage0 = (smem_addr(raw) + 1023u) & ~1023u;
        sh = reinterpret_cast<Shared *>(raw + (stage0 - smem_addr(raw)) + (size_t)kStages * kStageBytes);
        err = err_word;
        rank = CG == 1 ? 0 : cluster_rank();
        if (threadIdx.x == 0) {
            for (int s = 0; s < kStages; ++s) {
                mbar_init(&sh->full[s], CG == 2 && rank == 0 ? 2 : 1);   // the peer's copies are passed on by an arrival
                mbar_init(&sh->empty[s], 1);
            }
            for (int k = 0; k < 2; ++k) mbar_init(&sh->acc_full[k], 1), mbar_init(&sh->acc_empty[k], 8 * CG);
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
    };
    // Runs the tiles that `job` lists.  Job:
    //   Tile                       what one tile is; fields k_blocks (stages) and n (columns, a multiple of 64 * CG)
    //   bool chunk_ends(tile, kb)  after this stage the epilogue takes the accumulator (always after the last)
    //   bool next(Tile &, int i)   the i-th tile of this CTA (pair); false after the last
    //   bool ready(pipe, tile)     producer: what the tile reads is there
    //   void load(tile, kb, a, b, bar)       copies into a and b (shared addresses); must bring bytes(tile) bytes
    //   uint32_t bytes(tile)
    //   bool a_mn(tile, kb), b_mn(tile, kb)  majorness of the stage's operands
    //   int bf16()
    //   bool epilogue(pipe, tile, turn, warp, lane)   warp 0..7: for each chunk take(), read its columns, release();
    //                              false once take() is
    template <class Job>
    __device__ __forceinline__ void run(Job &job) {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        if (warp == 0 && lane == 0) {
            int s = 0, issued = 0;
            uint32_t ph = 0;
            typename Job::Tile t;
            bool ok = true;
            for (int i = 0; ok && job.next(t, i); ++i) {
                ok = job.ready(*this, t);
                for (int kb = 0; ok && kb < t.k_blocks; ++kb) {
                    ok = wait(&sh->empty[s], ph ^ 1);
                    if (!ok) break;
                    mbar_arrive_expect(&sh->full[s], job.bytes(t));
                    const uint32_t at = stage0 + (uint32_t)s * kStageBytes;
                    job.load(t, kb, at, at + kABytes, &sh->full[s]);
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
                    while (!(CG == 2 && rank == 0) && !mbar_try_wait(&sh->full[s], ph) && clock64() - t0 < kWaitCycles) {}
                }
                if (CG == 2 && rank == 0)               // its barriers also count the peer's arrivals: allow time instead
                    while (clock64() - t0 < 2000000ll) {}
            }
        } else if (warp == 1 && lane == 0 && rank == 0) {
            int s = 0, acc = 0;
            uint32_t ph = 0, acc_ph = 0;
            typename Job::Tile t;
            bool ok = true;
            for (int i = 0; ok && job.next(t, i); ++i) {
                bool fresh = true;
                for (int kb = 0; kb < t.k_blocks; ++kb) {
                    if (fresh) {
                        ok = wait(&sh->acc_empty[acc], acc_ph ^ 1);
                        if (!ok) break;
                    }
                    const uint32_t d = sh->tmem + (uint32_t)acc * 256;
                    ok = wait(&sh->full[s], ph);
                    if (!ok) break;
                    tmem_fence_after();
                    const bool a_mn = job.a_mn(t, kb), b_mn = job.b_mn(t, kb);
                    const uint32_t at = stage0 + (uint32_t)s * kStageBytes;
                    const uint64_t da = operand_desc(at, a_mn), db = operand_desc(at + kABytes, b_mn);
                    const uint32_t id = instr_desc(job.bf16(), a_mn, b_mn, t.n, CG);
                    const uint32_t sa = a_mn ? 2048 / 16 : 32 / 16, sb = b_mn ? 2048 / 16 : 32 / 16;
#pragma unroll
                    for (int k = 0; k < kStageK / 16; ++k)
                        mma_f16<CG>(d, da + (uint64_t)k * sa, db + (uint64_t)k * sb, id, !(fresh && k == 0));
                    mma_commit<CG>(&sh->empty[s]);
                    if (++s == kStages) s = 0, ph ^= 1;
                    fresh = job.chunk_ends(t, kb);
                    if (fresh) {
                        mma_commit<CG>(&sh->acc_full[acc]);
                        if (++acc == 2) acc = 0, acc_ph ^= 1;
                    }
                }
            }
            if (!ok) {                                  // products in flight end before tensor memory is given back
                mma_commit<CG>(&sh->drain);
                const long long t0 = clock64();
                while (!mbar_try_wait(&sh->drain, 0) && clock64() - t0 < kWaitCycles) {}
            }
        } else if (CG == 2 && warp == 1 && lane == 0) {
            // The pair's second CTA passes "this stage has landed" on to the first one's barrier.
            int s = 0;
            uint32_t ph = 0;
            typename Job::Tile t;
            bool ok = true;
            for (int i = 0; ok && job.next(t, i); ++i)
                for (int kb = 0; ok && kb < t.k_blocks; ++kb) {
                    ok = wait(&sh->full[s], ph);
                    if (ok) mbar_arrive_remote(&sh->full[s], 0);
                    if (++s == kStages) s = 0, ph ^= 1;
                }
        } else if (warp >= kEpiWarp0) {
            Turn turn;
            typename Job::Tile t;
            for (int i = 0; job.next(t, i); ++i)
                if (!job.epilogue(*this, t, turn, warp - kEpiWarp0, lane)) break;
        }
        __syncwarp();
    }
    // Vote of the 256 epilogue threads.
    __device__ __forceinline__ bool epi_all(bool ok) {
        int all;
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\t"
            "barrier.red.and.pred q, 1, 256, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
            : "=r"(all)
            : "r"((int)ok)
            : "memory");
        return all != 0;
    }
    __device__ __forceinline__ void epi_sync() { asm volatile("barrier.sync 1, 256;" ::: "memory"); }
    // Waits for the next accumulator; `at` is its address for this warp's lanes.  All epilogue threads get the same
    // answer, so that none waits at a barrier for one that left.
    __device__ __forceinline__ bool take(Turn &t, uint32_t &at) {
        if (!epi_all(wait(&sh->acc_full[t.acc], t.ph))) return false;
        tmem_fence_after();
        at = sh->tmem + (uint32_t)t.acc * 256 + ((uint32_t)(threadIdx.x / 32 % 4) << 21);
        return true;
    }
    // Called by every epilogue warp once it has read its part of the accumulator.
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
