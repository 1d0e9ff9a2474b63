// 8-bit floating point beside the packed ternary formats: the quantiser to e4m3 with one scale per row and group of 128,
// and the product of e4m3 activations with e4m3 weights that carry one scale per block of 128 x 128,
//
//     y[t][m] = sum over groups g of  xs[t][g] * ws[m / 128][g] * (sum over k in g of W[m][k] * x[t][k]),
//
// dense and over the routed pairs of a mixture-of-experts layer.
//
// The scales change with every group of 128, so the tensor cores may add up one group only: each group is four
// tcgen05.mma (K = 32) into a fresh accumulator in tensor memory, and warps of their own ("promoters") read it back, multiply with
// the two scales and add in fp32 registers while the next groups are being multiplied into other accumulators.
//
// Two operand orders, chosen by the host from the sizes:
//   tokens first   (more than 64 rows, longer groups) A = 256 tokens, B = 256 weight rows, two blocks of a cluster as one
//                  (cta_group::2): each loads its 128 tokens and half of the weight rows, 32 KB a group of 128, where a block by itself would
//                  load 48.  A promoter thread holds 128 columns of one token; the scales of a group are one number per thread.
//                  Persistent.  A group takes about 770 clocks for the 512 of its products, whether one pair of blocks is at work or
//                  all (764, 771, 747, 718 and 837 clocks with 1, 8, 32, 64 and 74 tiles; L2 then gives 29 % of its sectors at most): what bounds
//                  it is the round products -> promoters -> products over two accumulators, all that tensor memory holds of 256 columns, and not
//                  L2.  At the power limit the clock comes on top: 4095 x 8192 x 5120 is 280 groups one after another, recorded 146 to 152 us
//                  on a cool board (2.3 PFLOP/s, 1.4 GHz), 168 to 176 on a warm one.
//   weights first  A = 128 weight rows, B = 16, 32 or 64 tokens (16 of routed pairs).  Two or three blocks per multiprocessor keep enough of the weights
//                  under way, and K is cut over the blocks of a cluster where there are few row blocks: each leaves its sums in shared
//                  memory, and the cluster adds them in order of rank (no workspace, no atomics, the same bits every time).  Bound by
//                  memory: 25600 x 5120 at one token 22.6 us (5.8 TB/s).
//
// Operands come by TMA (128-byte swizzle, 128 bytes of K per stage); rows of routed pairs by cp.async from two warps of their own.
#include "bitcos.h"
#include "common.cuh"

#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <climits>

using namespace bitcos_kernels;

namespace {

constexpr int kGroup = BITCOS_GROUP;
constexpr uint32_t kFull = 0xFFFFFFFFu;
constexpr float kE4m3Max = 448.0f;

// ------------------------------------------------------------------ quantiser
//     a = max(max |x| over the group, 2^-100),  scale = a / 448,  code = e4m3(x * (448 / a))
// IEEE quotients and product, one rounding to nearest even.  Sixteen lanes per group of 128, eight values a lane.
// Bound by memory: 8191 x 5120 bf16 21.6 us (5.9 TB/s, 90 % of a copy); four groups a half warp, so that as many loads are under way.
template <typename T>
struct Eight;
template <>
struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = __ldg(reinterpret_cast<const float4 *>(p));
        b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
};
template <>
struct Eight<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { a = __ldg(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = bf16_lo(a.x), v[1] = bf16_hi(a.x), v[2] = bf16_lo(a.y), v[3] = bf16_hi(a.y);
        v[4] = bf16_lo(a.z), v[5] = bf16_hi(a.z), v[6] = bf16_lo(a.w), v[7] = bf16_hi(a.w);
    }
};

__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

constexpr int kQuantGroups = 4;           // groups per half warp, so that as many loads are under way
template <typename T>
__global__ void __launch_bounds__(256) fp8_quantize_kernel(const T *__restrict__ x, uint8_t *__restrict__ q, float *__restrict__ scale,
                                                           int64_t n_groups) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int part = threadIdx.x & 15, half = threadIdx.x >> 4;
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * kQuantGroups * 16) + half;
    Eight<T> in[kQuantGroups];
#pragma unroll
    for (int i = 0; i < kQuantGroups; ++i)
        if (first + i * 16 < n_groups) in[i].load(x + (first + i * 16) * kGroup + part * 8);
#pragma unroll
    for (int i = 0; i < kQuantGroups; ++i) {
        const int64_t grp = first + i * 16;
        if (grp >= n_groups) break;                 // (the same for all sixteen lanes; the shuffles name only those)
        float v[8];
        in[i].get(v);
        float a = fabsf(v[0]);
#pragma unroll
        for (int j = 1; j < 8; ++j) a = fmaxf(a, fabsf(v[j]));
        const uint32_t lanes = 0xFFFFu << (threadIdx.x & 16);
#pragma unroll
        for (int d = 8; d; d >>= 1) a = fmaxf(a, __shfl_xor_sync(lanes, a, d));
        a = fmaxf(a, kAmaxFloor);
        const float factor = __fdiv_rn(kE4m3Max, a);
        uint2 code;
        code.x = e4m3_pair(__fmul_rn(v[0], factor), __fmul_rn(v[1], factor)) | (e4m3_pair(__fmul_rn(v[2], factor), __fmul_rn(v[3], factor)) << 16);
        code.y = e4m3_pair(__fmul_rn(v[4], factor), __fmul_rn(v[5], factor)) | (e4m3_pair(__fmul_rn(v[6], factor), __fmul_rn(v[7], factor)) << 16);
        *reinterpret_cast<uint2 *>(q + grp * kGroup + part * 8) = code;
        if (part == 0) scale[grp] = __fdiv_rn(a, kE4m3Max);
    }
}

// ------------------------------------------------------------------ product: device side
constexpr int kARows = 128;               // rows of the A operand
constexpr uint32_t kABytes = kARows * kGroup;
constexpr int kMaxGroups = BITCOS_GROUP_EXPERTS_MAX;
constexpr int kMaxSplits = 8;             // portable cluster size
// Registers per thread, tokens first: what the block is launched with (checked before the first launch), and what the warps in
// front and the promoters split it into.
constexpr int kLaunchRegisters = 168, kFrontRegisters = 72, kPromoterRegisters = 216;

// How long a wait goes on, and for how long at a time it sleeps.
struct Patience {
    uint64_t limit_ns;
    uint32_t sleep_ns;
};
constexpr uint32_t kSleepNs = 1000000;
constexpr uint64_t kLooks = 1000;         // a limit below this is a number of looks

struct Fp8Args {
    const float *w_scale;       // [experts][w_blocks][G]
    const float *x_scale;       // [x rows][G]
    const uint8_t *x;           // grouped: rows to gather
    void *y;
    unsigned int *status;       // NULL, or the workspace's status word
    Patience patience;          // of the waits that the roles have for one another
    int64_t M;
    int64_t rows;               // dense: tokens; grouped: pairs
    int G;                      // groups of 128 along K
    int w_blocks;               // ceil(M / 128)
    int out_bf16;
    int vector;                 // rows of y may be written 16 bytes at a time
    int splits;                 // blocks of a cluster, each with its share of K (weights first)
    int row_tiles, w_tiles;     // dense: tiles along the tokens, along the weights (grouped: w_tiles only)
    // grouped
    const int32_t *group_expert, *group_begin, *n_groups, *pair_xrow;
    int max_groups, n_experts, n_xrows;
};

// The status word: a bit for each kind of trouble, so that none hides another (calls that run at the same time may share the word).
constexpr unsigned int kGaveUp = 1, kBadList = 2;
__device__ __forceinline__ void mark(const Fp8Args &a, unsigned int what) {
    if (a.status) atomicOr(a.status, what);
}

struct Tile {
    int64_t row0;               // first token / pair
    int rows;                   // tokens / pairs of the tile
    int w0;                     // first weight row
    int expert;
};
// The producer hands the tiles on in a ring.  It is ahead by the stages, the accumulators and the tile that is being written out at
// most, less than the ring holds: nobody has to say that an entry has been read.
constexpr int kTileRing = 16;

// A place in the ring of stages and the parity of its round.  (Counted along: a remainder and a quotient at every step are 50 clocks of
// a warp that has about 500 for one.)
template <int STAGES>
struct Stage {
    uint32_t s = 0, phase = 0;
    __device__ __forceinline__ void next() {
        if (++s == STAGES) {
            s = 0;
            phase ^= 1;
        }
    }
};

// The routing lists as every role of a block looks tiles up in them.
struct GroupLists {
    int32_t tiles[kMaxGroups + 1];         // in front of every group, and of all
    int32_t begin[kMaxGroups + 1];
    int32_t expert[kMaxGroups];
};

// N columns of an accumulator; PAIR: tokens first; GROUPED: over routed pairs.
template <int N, bool PAIR, bool GROUPED>
struct Layout {
    static constexpr int kBRows = PAIR ? N / 2 : N;     // of the B operand in this block's shared memory
    static constexpr uint32_t kBBytes = kBRows * kGroup;
    static constexpr uint32_t kStageBytes = kABytes + kBBytes;
    static constexpr int kBlocks = PAIR ? 1 : GROUPED ? 3 : 2;       // per multiprocessor
    // (PAIR: four stages leave room for the outputs; a fifth changed no time by more than 0.5 %)
    static constexpr int kStages = kBlocks == 3 ? 3 : N <= 32 ? 5 : 4;
    static constexpr int kParts = PAIR ? 2 : 1;          // of an accumulator's columns, one for every four promoter warps
    static constexpr int kAcc = PAIR ? 2 : 4;            // accumulators in turn
    static constexpr int kColumns = N / kParts;         // per promoter thread
    static constexpr int kPromoters = 4 * kParts;       // warps
    static constexpr int kFirst = GROUPED || PAIR ? 4 : 2;      // the first of them (in front: TMA, tensor cores, two for gathered rows)
    static constexpr int kThreads = (kFirst + kPromoters) * 32;
    static constexpr int kRowsPerTile = PAIR ? kARows : N;              // tokens of a tile in this block
    static constexpr int kTileRows = PAIR ? 2 * kRowsPerTile : kRowsPerTile;
    static constexpr int kWRowsPerTile = PAIR ? N : kARows;
    static constexpr uint32_t kTmemColumns = kAcc * N;
    // byte offsets behind the stages
    // PAIR: two boxes of 32 rows of 128 bytes per promoter warp, swizzled as TMA wants them, from which the outputs go to memory
    static constexpr uint32_t kOutBox = 32 * 128, kOutBoxes = 2;
    static constexpr uint32_t kOut = kStages * kStageBytes;
    static constexpr uint32_t kBars = kOut + (PAIR ? kPromoters * kOutBoxes * kOutBox : 0);
    static constexpr uint32_t kTiles = kBars + (3 * kStages + 2 * kAcc + 1 + kTileRing) * 8;
    static constexpr uint32_t kRows = kTiles + kTileRing * sizeof(Tile);
    static constexpr uint32_t kTmem = kRows + (GROUPED ? 2 * kRowsPerTile * 4 : 0);
    static constexpr uint32_t kEnds = (kTmem + 4 + 15) / 16 * 16;       // PAIR: how far both blocks got
    static constexpr uint32_t kScales = kEnds + (PAIR ? 32 : 0);
    static constexpr uint32_t kPrefix = kScales + (PAIR ? 0 : kPromoters * 2 * N * 4);
    static constexpr uint32_t kTotal = kPrefix + (GROUPED ? sizeof(GroupLists) : 0);
    static constexpr uint32_t kDynamic = kTotal + 1024;  // (the stages start on a 1024-byte boundary)
};

__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
                 "r"(c0), "r"(c1), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
                 : "memory");
}
// The same for a block of a pair, whose copies are counted by a barrier of the first block (an address in the cluster).
__device__ __forceinline__ void tma_2d_pair(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(map), "r"(c0), "r"(c1), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tma_3d_pair(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, int c0, int c1, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(c0), "r"(c1), "r"(src) : "memory");
}

// 16 bytes from anywhere in global memory, asynchronously; with there = 0 nothing is read and zeros are written.  (The rows of routed
// pairs: tile::gather4 costs the TMA unit about 25 clocks a row of 128 bytes, 3300 a stage of 128 rows.)
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there));
}

// Shared-memory matrix descriptor: K-major rows of 128 bytes, 128-byte swizzle, eight rows (1024 bytes) apart per step.
__device__ __forceinline__ uint64_t matrix_desc(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: e4m3 x e4m3 -> fp32, M rows of A and N of B.
__host__ __device__ constexpr uint32_t instruction_desc(int m, int n) {
    return (1u << 4) | (static_cast<uint32_t>(n / 8) << 17) | (static_cast<uint32_t>(m / 16) << 24);
}
template <bool PAIR>
__device__ __forceinline__ void mma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    if constexpr (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add)
            : "memory");
}
// An arrival when all products so far are done (PAIR: at this barrier of both blocks, or with ALONE of this one).
template <bool PAIR, bool ALONE = false>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (PAIR && ALONE) asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(static_cast<uint16_t>(3))
                     : "memory");
    else asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}
// (the registers pass through, so that nothing that reads them is moved in front of the wait)
__device__ __forceinline__ void tmem_wait16(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait32(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}
// One lane of a converged warp, the same one every time.  (Known to the compiler as one: the operands of tcgen05 and TMA instructions are
// uniform registers, and behind a plain `lane == 0` every such instruction is wrapped in a loop over the lanes that may differ.)
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
// Asks whether a phase is complete, asleep for up to a millisecond until it is.  (Without the time a question returns at once, and ten
// warps that keep asking leave every other access to shared memory 600 clocks in the queue.)
__device__ __forceinline__ uint32_t ask(uint32_t bar, uint32_t parity, uint32_t sleep_ns) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity), "r"(sleep_ns)
        : "memory");
    return done;
}
// Asks without waiting.
__device__ __forceinline__ uint32_t test(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done;
}
// A bounded wait.  (No call in it: with one, ptxas keeps every role to the registers that the block is launched with.)
__device__ __forceinline__ bool wait_here(uint32_t bar, uint32_t parity, const Patience &p) {
    uint64_t t0 = 0;
    while (!ask(bar, parity, p.sleep_ns)) {
        const uint64_t now = global_timer_ns();
        if (t0 == 0) t0 = now;
        if (now - t0 >= p.limit_ns) return false;
    }
    return true;
}
// The same with so little patience that a number of looks decides: a question sleeps for a while whatever time it is given.
__device__ __forceinline__ bool look_here(uint32_t bar, uint32_t parity, const Patience &p) {
    for (uint32_t i = 0; i <= p.sleep_ns; ++i)
        if (test(bar, parity)) return true;
    return false;
}
// A bounded wait by a whole warp, which goes on or gives up as one (what follows are instructions of whole warps).  PATIENT is one of the
// kernel's parameters because the choice at run time, in every wait, cost 1.5 %.
template <bool PATIENT>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const Patience &p) {
    return __all_sync(kFull, PATIENT ? wait_here(bar, parity, p) : look_here(bar, parity, p));
}
// The same for what is under way already and arrives by itself, whatever the roles have given up.
__device__ __forceinline__ bool drain_wait(uint32_t bar, uint32_t parity) {
    constexpr Patience p{kWaitLimitNs, kSleepNs};
    return warp_wait<true>(bar, parity, p);
}
// a += d * s, two at a time
__device__ __forceinline__ void fma_pair(float &a0, float &a1, uint32_t d0, uint32_t d1, float s0, float s1) {
    asm("{\n\t.reg .b64 a, d, s;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 d, {%2, %3};\n\tmov.b64 s, {%4, %5};\n\t"
        "fma.rn.f32x2 a, d, s, a;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "+f"(a0), "+f"(a1)
        : "r"(d0), "r"(d1), "f"(s0), "f"(s1));
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ float4 cluster_load(uint32_t addr, uint32_t rank) {
    float4 v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr), "r"(rank)
                 : "memory");
    return v;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
// The address in the cluster of another block's shared memory.
__device__ __forceinline__ uint32_t cluster_address(uint32_t addr, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
// (Without .release.cluster: that waits for all of the thread's memory traffic, 1000 clocks a time, and what the arrival stands for
// is done before it goes out and is nobody else's: reads of tensor memory that tcgen05.wait::ld has seen done, or copies that a
// barrier has seen land in this block's shared memory, where this multiprocessor's own tensor cores read them.)
__device__ __forceinline__ void cluster_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_store(uint32_t addr, uint32_t rank, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_address(addr, rank)), "r"(v) : "memory");
}
// Takes bytes that will not come off a phase.
__device__ __forceinline__ void mbar_complete_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}

// Where tile t lies.  Dense: bands of 16 tiles along the tokens, inside a band the tokens vary fastest, so that the tiles
// that run at the same time share rows and weights in L2.  Grouped: the group by bisection in the running tile counts; inside a group
// the tokens vary fastest (the tiles of one stretch of weights run side by side).
template <int N, bool PAIR, bool GROUPED>
__device__ __forceinline__ Tile find_tile(const Fp8Args &a, const GroupLists *lists, int n_groups, int64_t t, int rank) {
    using L = Layout<N, PAIR, GROUPED>;
    Tile r;
    if constexpr (!GROUPED) {
        constexpr int kBand = 16;
        const int64_t per_band = static_cast<int64_t>(kBand) * a.w_tiles;
        const int band = static_cast<int>(t / per_band);
        const int wide = min(kBand, a.row_tiles - band * kBand);
        const int in = static_cast<int>(t - band * per_band);
        const int w = in / wide, row_tile = band * kBand + in - w * wide;
        r.row0 = static_cast<int64_t>(row_tile) * L::kTileRows + (PAIR ? rank * L::kRowsPerTile : 0);
        r.rows = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(L::kRowsPerTile), a.rows - r.row0)));
        r.w0 = w * L::kWRowsPerTile;
        r.expert = 0;
    } else {
        int lo = 0, hi = n_groups;                 // tiles[lo] <= t < tiles[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (lists->tiles[mid] <= t) lo = mid;
            else hi = mid;
        }
        const int begin = lists->begin[lo], end = lists->begin[lo + 1];
        const int row_tiles = (end - begin + L::kTileRows - 1) / L::kTileRows;
        const int in = static_cast<int>(t) - lists->tiles[lo];
        const int w = in / row_tiles, row_tile = in - w * row_tiles;
        r.row0 = begin + static_cast<int64_t>(row_tile) * L::kTileRows + (PAIR ? rank * L::kRowsPerTile : 0);
        r.rows = max(0, min(L::kRowsPerTile, static_cast<int>(end - r.row0)));
        r.w0 = w * L::kWRowsPerTile;
        r.expert = lists->expert[lo];
    }
    return r;
}

template <int N, bool PAIR, bool GROUPED, bool PATIENT>
__global__ void __launch_bounds__(Layout<N, PAIR, GROUPED>::kThreads, Layout<N, PAIR, GROUPED>::kBlocks)
fp8_matmul_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap ymap,
                  const __grid_constant__ Fp8Args a) {
    using L = Layout<N, PAIR, GROUPED>;
    constexpr int kStages = L::kStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_addr(smem_raw);
    uint8_t *smem = smem_raw + (1024u - (raw & 1023u)) % 1024u;
    const uint32_t base = smem_addr(smem);
    const uint32_t full = base + L::kBars, empty = full + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 8 * L::kAcc;
    const uint32_t drained = acc_empty + 8 * L::kAcc, gathered = drained + 8;
    const uint32_t told = gathered + 8 * kStages;            // [kTileRing] the entry has been written
    Tile *ring = reinterpret_cast<Tile *>(smem + L::kTiles);
    GroupLists *lists = reinterpret_cast<GroupLists *>(smem + L::kPrefix);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int splits = PAIR ? 1 : a.splits;
    const bool gather = GROUPED && a.pair_xrow != nullptr;
    const int rank = PAIR || splits > 1 ? static_cast<int>(cluster_rank()) : 0;
    const int k_rank = PAIR ? 0 : rank;
    const int k0 = static_cast<int>(static_cast<int64_t>(a.G) * k_rank / splits), k1 = static_cast<int>(static_cast<int64_t>(a.G) * (k_rank + 1) / splits);
    const int64_t per_tile = PAIR ? 2 : splits;              // blocks that work on one tile
    const int64_t t_first = blockIdx.x / per_tile, t_step = gridDim.x / per_tile;
    // PAIR: the barriers that the tensor cores wait on are the first block's
    const uint32_t lead_full = PAIR ? cluster_address(full, 0) : full, lead_acc_empty = PAIR ? cluster_address(acc_empty, 0) : acc_empty;
    const auto send_weights = [&](uint32_t stage, const Tile &t, int kb, uint32_t bar) {
        const uint32_t dst = base + stage * L::kStageBytes + (PAIR ? kABytes : 0);
        if constexpr (PAIR) tma_3d_pair(dst, &wmap, kb * kGroup, t.w0 + rank * L::kBRows, t.expert, bar);
        else tma_3d(dst, &wmap, kb * kGroup, t.w0, t.expert, bar);
    };
    // PAIR: how far the two blocks got, words that both have: stages sent by each, stages of routed rows that the second has
    // announced, stages multiplied, whether any wait has run out
    constexpr int kIssued = 0, kAnnounced = 2, kMultiplied = 3, kStopped = 4;
    const auto tell = [&](int word, uint32_t v) {
        for (uint32_t r = 0; r < 2; ++r) cluster_store(base + L::kEnds + 4 * word, r, v);
    };
    // the first weights are on their way before the kernel in front of this one has finished: they are nobody's output
    const auto send_first = [&]() {
        if (t_first < static_cast<int64_t>(a.row_tiles) * a.w_tiles) {
            const Tile t = find_tile<N, PAIR, GROUPED>(a, lists, 0, t_first, rank);
            for (int i = 0; i < kStages && k0 + i < k1; ++i) {
                if (!PAIR || rank == 0) mbar_expect_tx(full + 8 * i, (PAIR ? 2 : 1) * L::kStageBytes);
                send_weights(i, t, k0 + i, lead_full + 8 * i);
            }
        }
    };

    if (warp == 0 && elect_one()) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full + 8 * s, gather && PAIR ? 2 : 1);
            mbar_init(empty + 8 * s, 1);
            mbar_init(gathered + 8 * s, 32);
        }
        for (int b = 0; b < L::kAcc; ++b) {
            mbar_init(acc_full + 8 * b, 1);
            mbar_init(acc_empty + 8 * b, (PAIR ? 2 : 1) * L::kPromoters);
        }
        mbar_init(drained, 1);
        for (int i = 0; i < kTileRing; ++i) mbar_init(told + 8 * i, 1);
        if (PAIR) *reinterpret_cast<volatile uint32_t *>(smem + L::kEnds + 4 * kStopped) = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (!GROUPED && !PAIR) send_first();
    }
    if (warp == 1) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + L::kTmem), "n"(L::kTmemColumns) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + L::kTmem), "n"(L::kTmemColumns) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        tmem_fence_before();
    }
    if constexpr (PAIR) cluster_sync();                      // (the other block's barriers are there, and its tensor memory)
    else __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(smem + L::kTmem);
    // The next kernel's blocks may start only once every block of this one holds its tensor memory: a block of the next kernel that
    // got it first would keep it until this kernel is done.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (PAIR && !GROUPED && warp == 0 && elect_one()) send_first();
    __syncwarp();
    asm volatile("griddepcontrol.wait;" ::: "memory");

    int n_groups = 0;
    int64_t n_tiles = static_cast<int64_t>(a.row_tiles) * a.w_tiles;
    if constexpr (GROUPED) {
        // (the first 32 groups are asked for together with their number: one trip to memory less; each further 32 are one trip
        // more, three for 128)
        int e0 = 0, begin0 = 0, end0 = 0;
        if (warp == 0 && lane < a.max_groups) {
            e0 = __ldg(a.group_expert + lane);
            begin0 = __ldg(a.group_begin + lane);
            end0 = __ldg(a.group_begin + lane + 1);
        }
        n_groups = min(max(__ldg(a.n_groups), 0), a.max_groups);
        if (warp == 0) {
            int64_t sum = 0;
            for (int g0 = 0; g0 < n_groups; g0 += 32) {
                const int g = g0 + lane;
                int64_t tiles = 0;
                if (g < n_groups) {
                    const int e = g0 ? __ldg(a.group_expert + g) : e0, begin = g0 ? __ldg(a.group_begin + g) : begin0;
                    const int end = g0 ? __ldg(a.group_begin + g + 1) : end0;
                    lists->expert[g] = e;
                    lists->begin[g] = begin;
                    lists->begin[g + 1] = end;               // (twice the same where the next group is another lane's)
                    if (end > begin) {
                        // a malformed group is skipped whole and marked (an empty one without a mark)
                        if (e >= 0 && e < a.n_experts && begin >= 0 && end <= a.rows)
                            tiles = static_cast<int64_t>((end - begin + L::kTileRows - 1) / L::kTileRows) * a.w_tiles;
                        else if (blockIdx.x == 0) mark(a, kBadList);
                    }
                }
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int64_t up = __shfl_up_sync(kFull, tiles, d);
                    if (lane >= d) tiles += up;
                }
                // (groups that do not overlap have fewer tiles than 2^31, the host has seen to it; of overlapping ones the rest is left out)
                if (g < n_groups) lists->tiles[g + 1] = static_cast<int32_t>(min(sum + tiles, static_cast<int64_t>(INT_MAX)));
                sum += __shfl_sync(kFull, tiles, 31);
            }
            if (lane == 0) lists->tiles[0] = 0;
        }
        __syncthreads();
        n_tiles = lists->tiles[n_groups];
        if (splits > 1 && n_tiles > t_step) {                // (a cluster adds up one tile; groups that do not overlap have no more)
            n_tiles = t_step;
            if (blockIdx.x == 0 && threadIdx.x == 0) mark(a, kBadList);
        }
    }
    constexpr uint32_t kXBytes = PAIR ? kABytes : L::kBBytes;
    bool ok = true;
    uint32_t it = 0;                       // groups of 128 so far, over all tiles
    uint32_t tiles = 0;                    // tiles so far
    const auto next_tile = [&](Tile &t) {  // the block's next tile, from the ring
        if (!warp_wait<PATIENT>(told + 8 * (tiles % kTileRing), (tiles / kTileRing) & 1, a.patience)) return false;
        t = ring[tiles++ % kTileRing];
        return true;
    };

    // Tokens first: a promoter holds 128 sums and 64 columns on their way; what it takes over 168 registers the four warps in
    // front give.  (In the two branches themselves: where they meet, the smaller number holds.)
    static_assert(!PAIR || 128 * kFrontRegisters + L::kPromoters * 32 * kPromoterRegisters == L::kThreads * kLaunchRegisters, "the block's registers");
    if (warp < L::kFirst) {
        if (PAIR) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFrontRegisters));
        if (warp == 0) {
            // ---- producer
            Stage<kStages> at;
            for (int64_t t = t_first; ok && t < n_tiles; t += t_step) {
                const Tile tile = find_tile<N, PAIR, GROUPED>(a, lists, n_groups, t, rank);
                if (elect_one()) {
                    ring[tiles % kTileRing] = tile;
                    mbar_arrive(told + 8 * (tiles % kTileRing));
                }
                ++tiles;
                __syncwarp();
                for (int kb = k0; ok && kb < k1; ++kb, ++it) {
                    const uint32_t s = at.s;
                    const uint32_t x_dst = base + s * L::kStageBytes + (PAIR ? 0 : kABytes);
                    if (it >= kStages && !warp_wait<PATIENT>(empty + 8 * s, at.phase ^ 1, a.patience)) {
                        ok = false;
                        break;
                    }
                    const bool sent = !GROUPED && it < kStages && t == t_first;       // (announced and the weights sent above)
                    if (elect_one()) {
                        if (!sent) {
                            if (!PAIR || rank == 0) mbar_expect_tx(full + 8 * s, (PAIR ? 2 : 1) * (gather ? L::kStageBytes - kXBytes : L::kStageBytes));
                            send_weights(s, tile, kb, lead_full + 8 * s);
                        }
                        if (!gather) {
                            if constexpr (PAIR) tma_2d_pair(x_dst, &xmap, kb * kGroup, static_cast<int>(tile.row0), lead_full + 8 * s);
                            else tma_2d(x_dst, &xmap, kb * kGroup, static_cast<int>(tile.row0), full + 8 * s);
                        }
                    }
                    __syncwarp();
                    at.next();
                }
            }
            // no copy may outlive the block, also where a wait has run out; PAIR: nor an arrival from the other block's products,
            // so every stage has been read (if not, both blocks settle what is left, below)
            for (uint32_t i = it > kStages ? it - kStages : 0; (ok || !PAIR) && i < it; ++i) {
                if (PAIR) ok = warp_wait<PATIENT>(empty + 8 * (i % kStages), (i / kStages) & 1, a.patience);
                else ok &= drain_wait(full + 8 * (i % kStages), (i / kStages) & 1);
            }
            if (PAIR && elect_one()) tell(kIssued + rank, it);
            __syncwarp();
        } else if (warp == 1) {
            // ---- tensor cores: the warp waits, one lane issues
            constexpr uint32_t idesc = instruction_desc(PAIR ? 2 * kARows : kARows, N);
            Stage<kStages> at;
            const uint64_t desc_a = matrix_desc(base), desc_b = matrix_desc(base + kABytes);
            const bool issues = !PAIR || rank == 0;
            for (int64_t t = t_first; issues && ok && t < n_tiles; t += t_step) {
                for (int kb = k0; kb < k1; ++kb, ++it) {
                    const uint32_t s = at.s, b = it % L::kAcc, again = (it / L::kAcc & 1) ^ 1;
                    // (the barriers are asked before any answer is looked at: an answer takes about 200 clocks here, and
                    // this warp's turn has to stay below the 512 clocks of its products)
                    const auto there = [&](uint32_t bar, uint32_t parity) { return PATIENT ? ask(bar, parity, a.patience.sleep_ns) : test(bar, parity); };
                    const uint32_t have = there(full + 8 * s, at.phase);
                    const uint32_t rows = !gather || there(gathered + 8 * s, at.phase);
                    const uint32_t room = it < L::kAcc || there(acc_empty + 8 * b, again);
                    if (!__all_sync(kFull, have & room & rows)) {
                        if ((it >= L::kAcc && !warp_wait<PATIENT>(acc_empty + 8 * b, again, a.patience)) || !warp_wait<PATIENT>(full + 8 * s, at.phase, a.patience) ||
                            (gather && !warp_wait<PATIENT>(gathered + 8 * s, at.phase, a.patience))) {
                            ok = false;
                            break;
                        }
                    }
                    // (rows that other threads copied, for the tensor cores to read.  Here, and not by the copying warps: there it would
                    // wait for all their copies under way, and no two stages would be)
                    if (gather) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    tmem_fence_after();
                    if (elect_one()) {
                        const uint64_t da = desc_a + s * (L::kStageBytes >> 4), db = desc_b + s * (L::kStageBytes >> 4);
#pragma unroll
                        for (int k = 0; k < 4; ++k) mma_e4m3<PAIR>(tmem + b * N, da + 2 * k, db + 2 * k, idesc, k > 0);
                        mma_commit<PAIR>(acc_full + 8 * b);
                        mma_commit<PAIR>(empty + 8 * s);
                    }
                    __syncwarp();
                    at.next();
                }
            }
            // the second block's rows are announced to the first one's tensor cores
            for (int64_t t = t_first; gather && !issues && ok && t < n_tiles; t += t_step) {
                for (int kb = k0; kb < k1; ++kb, ++it) {
                    const uint32_t s = it % kStages;
                    if (!warp_wait<PATIENT>(gathered + 8 * s, (it / kStages) & 1, a.patience)) {
                        ok = false;
                        break;
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) cluster_arrive(lead_full + 8 * s);
                }
            }
            // nothing may be in flight when the tensor memory goes
            if (issues) {
                if (elect_one()) mma_commit<PAIR, true>(drained);
                __syncwarp();
                ok &= drain_wait(drained, 0);
            }
            if (PAIR && elect_one()) tell(issues ? kMultiplied : kAnnounced, it);
            __syncwarp();
        } else if (L::kFirst == 4 && warp < L::kFirst) {
            // ---- rows of routed pairs: two warps take the stages in turn; eight lanes per row of 128 bytes, 16 bytes each, put where the
            // 128-byte swizzle has them.  Bound by the copies: 512 bytes take an instruction of these about 18 clocks.
            if (gather) {
                constexpr int kOwn = L::kRowsPerTile / 4, kBatch = kOwn < 16 ? kOwn : 16;
                const uint32_t turn = warp - 2;
                const int r0 = lane >> 3, chunk = lane & 7;
                const uint32_t x_off = (PAIR ? 0 : kABytes) + r0 * kGroup;
                const uint32_t swizzled[2] = {static_cast<uint32_t>((chunk ^ r0) << 4), static_cast<uint32_t>((chunk ^ (r0 + 4)) << 4)};
                const uint8_t *x = a.x + chunk * 16;
                const uint32_t K = static_cast<uint32_t>(a.G) * kGroup;
                Stage<kStages> at;
                // the tile's rows (-1: no row of the tile, or no row of x: zeros, and dropped later), a list per warp
                int32_t *rows = reinterpret_cast<int32_t *>(smem + L::kRows) + turn * L::kRowsPerTile;
                for (int64_t t = t_first; ok && t < n_tiles; t += t_step) {
                    Tile tile;
                    if (!next_tile(tile)) {
                        ok = false;
                        break;
                    }
                    __syncwarp();                        // (the list is read no more)
                    for (int i = lane; i < L::kRowsPerTile; i += 32) {
                        const int r = i < tile.rows ? __ldg(a.pair_xrow + tile.row0 + i) : -1;
                        rows[i] = r < a.n_xrows ? r : -1;
                    }
                    __syncwarp();
                    for (int kb = k0; kb < k1; ++kb, ++it, at.next()) {
                        if ((it & 1) != turn) continue;
                        if (it >= kStages && !warp_wait<PATIENT>(empty + 8 * at.s, at.phase ^ 1, a.patience)) {
                            ok = false;
                            break;
                        }
                        const uint32_t dst = base + at.s * L::kStageBytes + x_off;
                        const uint8_t *from = x + kb * kGroup;
                        // (no branches: a copy is a multiplication and the instruction itself)
#pragma unroll
                        for (int j0 = 0; j0 < kOwn; j0 += kBatch) {
                            int src[kBatch];
#pragma unroll
                            for (int j = 0; j < kBatch; ++j) src[j] = rows[r0 + 4 * (j0 + j)];
#pragma unroll
                            for (int j = 0; j < kBatch; ++j)
                                copy16(dst + (j0 + j) * 4 * kGroup + swizzled[j & 1],
                                       from + static_cast<uint64_t>(static_cast<uint32_t>(max(src[j], 0))) * K, src[j] >= 0 ? 16u : 0u);
                        }
                        // (arrives by itself when this thread's copies have landed)
                        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(gathered + 8 * at.s) : "memory");
                    }
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                // (their arrivals too: the last rounds of this warp)
                for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i)
                    if ((i & 1) == turn) ok &= drain_wait(gathered + 8 * (i % kStages), (i / kStages) & 1);
            }
        }
    } else {
        // ---- promoters: warp w of four reads lanes 32 (w % 4) .. + 31 of the accumulators
        if (PAIR) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPromoterRegisters));
        constexpr int kCols = L::kColumns;
        const int quarter = warp & 3, part = PAIR ? (warp - L::kFirst) >> 2 : 0;
        const int row = quarter * 32 + lane;       // of A
        const uint32_t tmem_row = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + part * kCols;
        // (PAIR) what a tile needs of the lists and the scales, asked for during the last groups of the tile before
        Tile tile, coming;
        int64_t xr = -1;                   // this thread's row of x (-1: none)
        float sx0 = 0.f, sx1 = 0.f, sw0 = 0.f, sw1 = 0.f;      // the scales of the first two groups
        const auto look_up = [&]() {
            ok = next_tile(coming);
            xr = ok && row < coming.rows ? coming.row0 + row : -1;
            if (GROUPED && a.pair_xrow && xr >= 0) xr = __ldg(a.pair_xrow + xr);
        };
        const auto row_scales = [&]() { return a.x_scale + (xr >= 0 && (!GROUPED || xr < a.n_xrows) ? xr : 0) * a.G; };
        const auto column_scales = [&](const Tile &t) {
            const int block = (t.w0 + part * kCols) / kGroup;
            return a.w_scale + (static_cast<int64_t>(t.expert) * a.w_blocks + (block < a.w_blocks ? block : 0)) * a.G;
        };
        const auto first_scales = [&]() {
            const float *xs = row_scales(), *ws = column_scales(coming);
            sx0 = __ldg(xs);
            sw0 = __ldg(ws);
            sx1 = a.G > 1 ? __ldg(xs + 1) : 0.f;
            sw1 = a.G > 1 ? __ldg(ws + 1) : 0.f;
        };
        if (PAIR && t_first < n_tiles) {
            look_up();
            if (ok) first_scales();
        }
        for (int64_t t = t_first; ok && t < n_tiles; t += t_step) {
            if (PAIR) tile = coming;
            else tile = find_tile<N, PAIR, GROUPED>(a, lists, n_groups, t, rank);
            float acc[kCols];
#pragma unroll
            for (int i = 0; i < kCols; ++i) acc[i] = 0.f;
            const float *ws = a.w_scale + (static_cast<int64_t>(tile.expert) * a.w_blocks) * a.G;
            if constexpr (PAIR) {
                bool mine = row < tile.rows;
                if (GROUPED && mine && (xr < 0 || xr >= a.n_xrows)) {
                    mine = false;
                    mark(a, kBadList);
                }
                const float *xs = row_scales();
                ws = column_scales(tile);
                // The columns pass 32 at a time through two buffers: while one is added, the other is on its way, across the groups
                // too; the scales are asked for two groups ahead.
                float scale = sx0 * sw0, sx = sx1, sw = sw1;
                const bool more = t + t_step < n_tiles;
                uint32_t d[2][32];
                ok = warp_wait<PATIENT>(acc_full + 8 * (it % L::kAcc), (it / L::kAcc) & 1, a.patience);
                if (ok) {
                    tmem_fence_after();
                    tmem_load32(tmem_row + (it % L::kAcc) * N, d[0]);
                }
                // (in three runs, so that looking ahead to the next tile costs the loop itself nothing)
                int kb = k0;
#pragma unroll 1
                for (int run = 0; run < 3; ++run) {
                    const int stop = run == 0 ? max(k0, k1 - 3) : run == 1 ? max(k0, k1 - 1) : k1;
#pragma unroll 1
                    for (; ok && kb < stop; ++kb) {
                        const uint32_t b = it % L::kAcc;
                        const float s = scale;
                        scale = sx * sw;
                        if (kb + 2 < k1) {
                            sx = __ldg(xs + kb + 2);
                            sw = __ldg(ws + kb + 2);
                        }
                        ++it;
                        uint32_t next = 1;
#pragma unroll
                        for (int c = 0; c < kCols / 32; ++c) {
                            tmem_wait32(d[c & 1]);
                            if (c + 1 < kCols / 32) {
                                tmem_load32(tmem_row + b * N + (c + 1) * 32, d[(c + 1) & 1]);
                            } else {
                                tmem_fence_before();
                                __syncwarp();
                                if (lane == 0) {
                                    cluster_arrive(lead_acc_empty + 8 * b);
                                }
                                if (kb + 1 < k1) next = test(acc_full + 8 * (it % L::kAcc), (it / L::kAcc) & 1);
                            }
#pragma unroll
                            for (int i = 0; i < 32; i += 2) fma_pair(acc[c * 32 + i], acc[c * 32 + i + 1], d[c & 1][i], d[c & 1][i + 1], s, s);
                        }
                        if (kb + 1 < k1) {
                            ok = __all_sync(kFull, next) || warp_wait<PATIENT>(acc_full + 8 * (it % L::kAcc), (it / L::kAcc) & 1, a.patience);
                            if (ok) {
                                tmem_fence_after();
                                tmem_load32(tmem_row + (it % L::kAcc) * N, d[0]);
                            }
                        }
                    }
                    if (more && ok && run == 0) look_up();
                    if (more && ok && run == 1) first_scales();
                }
                if (!ok) {
                    tmem_wait32(d[0]);                   // (may be on its way: the look ahead may have given up)
                    break;
                }
                const int64_t c0 = tile.w0 + part * kCols;
                // A thread has a row, memory wants lines: each warp puts its 32 rows into shared memory, two boxes of 128 bytes of a row at
                // a time, and TMA writes them while the next tile's groups are added.  (Stored by the warp itself, line by line, a tile
                // waited 1.2 us for its 64 KB; straight from the registers, 32 rows an instruction and half a sector each, 5 us.)  Where not all 32 rows
                // are the tile's (dense: behind the last one TMA writes nothing), or rows are not whole 16 bytes, the warp does it.
                const uint32_t rows_mask = __ballot_sync(kFull, mine);
                const int64_t first = tile.row0 + quarter * 32;
                uint8_t *out = smem + L::kOut + (warp - L::kFirst) * L::kOutBoxes * L::kOutBox;
                const bool bulk = a.vector && (rows_mask == kFull || (!GROUPED && rows_mask));
                const int size = a.out_bf16 ? 2 : 4, width = 128 / size;         // bytes of an output, columns of a box
                const auto boxes_free = [&]() {                        // TMA has read the last ones
                    if (elect_one()) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
                };
                const auto put = [&](int box, int i, uint4 v) {        // 16 bytes i of this thread's row
                    *reinterpret_cast<uint4 *>(out + box * L::kOutBox + lane * 128 + ((i ^ (lane & 7)) << 4)) = v;
                };
                const auto send = [&](int from) {                      // columns from .. + 2 * width
                    if (bulk) {
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (elect_one()) {
                            for (int box = 0; box < static_cast<int>(L::kOutBoxes); ++box)
                                if (c0 + from + box * width < a.M)
                                    tma_store_2d(&ymap, static_cast<int>(c0) + from + box * width, static_cast<int>(first), smem_addr(out + box * L::kOutBox));
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                        __syncwarp();
                        return;
                    }
                    __syncwarp();
#pragma unroll
                    for (int box = 0; box < static_cast<int>(L::kOutBoxes); ++box) {
                        const uint8_t *o = out + box * L::kOutBox;
                        const int64_t column = c0 + from + box * width;
                        const int left = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(width), a.M - column)));
                        if (a.vector) {
                            const int at = (lane & 7) * (width / 8);
                            uint8_t *to = static_cast<uint8_t *>(a.y) + ((first + (lane >> 3)) * a.M + column + at) * size;
                            const int64_t step = 4 * a.M * size;
                            const uint8_t *from_even = o + (lane >> 3) * 128 + (((lane & 7) ^ (lane >> 3)) << 4);
                            const uint8_t *from_odd = o + ((lane >> 3) + 4) * 128 + (((lane & 7) ^ ((lane >> 3) + 4)) << 4);
                            const uint32_t mask = at < left ? rows_mask >> (lane >> 3) : 0u;
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const uint4 v = *reinterpret_cast<const uint4 *>((j & 1 ? from_odd : from_even) + (j / 2) * 1024);
                                if ((mask >> (4 * j)) & 1u) *reinterpret_cast<uint4 *>(to) = v;
                                to += step;
                            }
                        } else {
                            for (int r = 0; r < 32; ++r)
                                if ((rows_mask >> r) & 1u)
                                    for (int i = lane; i < left; i += 32) {
                                        const int64_t to = (first + r) * a.M + column + i;
                                        const uint8_t *v = o + r * 128 + ((i * size) ^ ((r & 7) << 4));
                                        if (size == 2) static_cast<uint16_t *>(a.y)[to] = *reinterpret_cast<const uint16_t *>(v);
                                        else static_cast<uint32_t *>(a.y)[to] = *reinterpret_cast<const uint32_t *>(v);
                                    }
                        }
                    }
                    __syncwarp();
                };
                if (rows_mask) {
                    if (a.out_bf16) {
                        boxes_free();
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float *v = acc + i * 8;
                            put(i / 8, i % 8, make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])));
                        }
                        send(0);
                    } else {
#pragma unroll
                        for (int c = 0; c < kCols; c += 64) {
                            boxes_free();
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float *v = acc + c + i * 4;
                                put(i / 8, i % 8, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
                            }
                            send(c);
                        }
                    }
                }
            } else {
                ws += static_cast<int64_t>(tile.w0 / kGroup) * a.G;
                // the scales of the tile's tokens: lane l looks after columns l, l + 32, ...; a group's products with the weights'
                // scale pass through shared memory, a copy per warp
                constexpr int kOwn = (N + 31) / 32;
                float *scales = reinterpret_cast<float *>(smem + L::kScales) + (warp - L::kFirst) * 2 * N;
                const float *xs[kOwn];
                uint32_t bad[kOwn];                // columns whose row of x does not exist: not written
                float sx[kOwn], sx_next[kOwn];     // the scales of this group and the next, the one after is asked for
                float sw = __ldg(ws + k0), sw_next = k0 + 1 < k1 ? __ldg(ws + k0 + 1) : 0.f;
#pragma unroll
                for (int j = 0; j < kOwn; ++j) {
                    const int n = lane + 32 * j;
                    bool there = n < tile.rows;
                    int64_t xr = tile.row0 + n;
                    if (GROUPED && a.pair_xrow && there) xr = __ldg(a.pair_xrow + xr);
                    const bool wrong = GROUPED && there && (xr < 0 || xr >= a.n_xrows);
                    bad[j] = __ballot_sync(kFull, wrong);
                    if (wrong) {
                        there = false;
                        mark(a, kBadList);
                    }
                    xs[j] = there ? a.x_scale + xr * a.G : nullptr;
                    sx[j] = there ? __ldg(xs[j] + k0) : 0.f;
                    sx_next[j] = there && k0 + 1 < k1 ? __ldg(xs[j] + k0 + 1) : 0.f;
                }
#pragma unroll 1
                for (int kb = k0; kb < k1; ++kb, ++it) {
                    const uint32_t b = it % L::kAcc;
                    float *scale = scales + (it & 1) * N;
#pragma unroll
                    for (int j = 0; j < kOwn; ++j) {
                        if (N % 32 == 0 || lane < N) scale[lane + 32 * j] = sx[j] * sw;
                        sx[j] = sx_next[j];
                        if (kb + 2 < k1 && xs[j]) sx_next[j] = __ldg(xs[j] + kb + 2);
                    }
                    sw = sw_next;
                    if (kb + 2 < k1) sw_next = __ldg(ws + kb + 2);
                    __syncwarp();
                    if (!warp_wait<PATIENT>(acc_full + 8 * b, (it / L::kAcc) & 1, a.patience)) {
                        ok = false;
                        break;
                    }
                    tmem_fence_after();
                    // all columns at once, so that the accumulator goes back before they are added
                    constexpr int kWide = kCols < 32 ? 16 : 32, kLoads = kCols / kWide;
                    uint32_t d[kLoads][kWide];
#pragma unroll
                    for (int c = 0; c < kLoads; ++c) {
                        if constexpr (kWide == 16) tmem_load16(tmem_row + b * N + c * kWide, d[c]);
                        else tmem_load32(tmem_row + b * N + c * kWide, d[c]);
                    }
#pragma unroll
                    for (int c = 0; c < kLoads; ++c) {
                        if constexpr (kWide == 16) tmem_wait16(d[c]);
                        else tmem_wait32(d[c]);
                    }
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acc_empty + 8 * b);
#pragma unroll
                    for (int i = 0; i < kCols; i += 4) {
                        const float4 sc = *reinterpret_cast<const float4 *>(scale + i);
                        fma_pair(acc[i], acc[i + 1], d[i / kWide][i % kWide], d[i / kWide][i % kWide + 1], sc.x, sc.y);
                        fma_pair(acc[i + 2], acc[i + 3], d[i / kWide][i % kWide + 2], d[i / kWide][i % kWide + 3], sc.z, sc.w);
                    }
                }
                if (!ok) break;
                const int64_t m = tile.w0 + row;
                if (splits == 1) {
                    if (m < a.M) {
#pragma unroll
                        for (int n = 0; n < N; ++n) {
                            if (n < tile.rows && !((bad[n / 32] >> (n % 32)) & 1u)) {
                                const int64_t at = (tile.row0 + n) * a.M + m;
                                if (a.out_bf16) static_cast<__nv_bfloat16 *>(a.y)[at] = __float2bfloat16_rn(acc[n]);
                                else static_cast<float *>(a.y)[at] = acc[n];
                            }
                        }
                    }
                } else {
                    // (every stage has been read: the last group's accumulator is complete)
                    float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        if (n < tile.rows) sums[n * kARows + row] = acc[n];
                }
            }
        }
    }
    if (!ok) {
        mark(a, kGaveUp);
        if (PAIR) tell(kStopped, 1);
    }
    if constexpr (PAIR) {                  // (the outputs are in memory before the block goes)
        if (warp >= L::kFirst && elect_one()) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }

    if constexpr (!PAIR) {
        if (splits > 1) {
            cluster_sync();
            if (warp >= L::kFirst && t_first < n_tiles) {
                // a warp adds a token's 128 rows, four a lane; the blocks of the cluster share out the tokens
                const Tile tile = find_tile<N, PAIR, GROUPED>(a, lists, n_groups, t_first, rank);
                const int64_t m = tile.w0 + lane * 4;
                for (int n = rank + splits * (warp - L::kFirst); n < tile.rows; n += splits * L::kPromoters) {
                    if (GROUPED) {                           // (a row of x that does not exist: not written)
                        const int64_t r = a.pair_xrow ? __ldg(a.pair_xrow + tile.row0 + n) : tile.row0 + n;
                        if (r < 0 || r >= a.n_xrows) continue;
                    }
                    float4 part[kMaxSplits];
#pragma unroll
                    for (int r = 0; r < kMaxSplits; ++r)
                        if (r < splits) part[r] = cluster_load(base + static_cast<uint32_t>(n * kARows + lane * 4) * 4u, r);
                    float4 sum = part[0];
#pragma unroll
                    for (int r = 1; r < kMaxSplits; ++r)
                        if (r < splits) sum = make_float4(sum.x + part[r].x, sum.y + part[r].y, sum.z + part[r].z, sum.w + part[r].w);
                    const int64_t at = (tile.row0 + n) * a.M + m;
                    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
                    if (a.vector && m < a.M) {               // (M is a multiple of four, or of eight)
                        if (a.out_bf16) *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.y) + at) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
                        else *reinterpret_cast<float4 *>(static_cast<float *>(a.y) + at) = sum;
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (m + i < a.M) {
                                if (a.out_bf16) static_cast<__nv_bfloat16 *>(a.y)[at + i] = __float2bfloat16_rn(v[i]);
                                else static_cast<float *>(a.y)[at + i] = v[i];
                            }
                    }
                }
            }
            cluster_sync();                // (nobody's sums go while they may be read)
        }
    }
    tmem_fence_before();
    if constexpr (PAIR) {
        cluster_sync();                    // (neither block goes while the other's copies or products may reach it)
        const volatile uint32_t *ends = reinterpret_cast<const volatile uint32_t *>(smem + L::kEnds);
        if (ends[kStopped]) {
            // A wait has run out somewhere, and the blocks stopped at different stages (no two more than the ring apart: a stage
            // is filled again only when its products are done).  The first block makes up for the arrivals and bytes that will not come, so
            // that the phases complete when the copies of both blocks that are under way have landed; both blocks wait for the
            // arrivals that stand for products.
            if (warp == 0) {
                const uint32_t sent0 = ends[kIssued], sent1 = ends[kIssued + 1], rows1 = ends[kAnnounced], products = ends[kMultiplied];
                const uint32_t bytes = gather ? L::kStageBytes - kXBytes : L::kStageBytes;
                const uint32_t top = max(max(sent0, sent1), gather ? rows1 : 0u);
                for (uint32_t i = top > kStages ? top - kStages : 0; rank == 0 && i < top; ++i) {
                    const uint32_t bar = full + 8 * (i % kStages);
                    if (elect_one()) {
                        if (i >= sent0 && i < sent1) mbar_expect_tx(bar, bytes);
                        else if (i >= sent0) mbar_arrive(bar);
                        else if (i >= sent1) mbar_complete_tx(bar, bytes);
                        if (gather && i >= rows1) mbar_arrive(bar);
                    }
                    __syncwarp();
                    drain_wait(bar, (i / kStages) & 1);
                }
                for (uint32_t i = products > kStages ? products - kStages : 0; i < products; ++i) drain_wait(empty + 8 * (i % kStages), (i / kStages) & 1);
                for (uint32_t i = products > L::kAcc ? products - L::kAcc : 0; i < products; ++i) drain_wait(acc_full + 8 * (i % L::kAcc), (i / L::kAcc) & 1);
            }
            __syncwarp();
            cluster_sync();
        }
    } else __syncthreads();
    if (warp == 1) {
        tmem_fence_after();
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(L::kTmemColumns) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(L::kTmemColumns) : "memory");
    }
}

// ------------------------------------------------------------------ product: host side
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}

// Rows of K bytes, box_rows of them and 128 bytes of each per copy; experts > 0: a third dimension of that many matrices.
int encode(CUtensorMap *map, const void *data, int64_t K, int64_t rows, int experts, int box_rows) {
    const EncodeTiled f = encode_tiled();
    if (!f) {
        g_last_cuda_error = cudaErrorNotSupported;
        return BITCOS_ERR_CUDA;
    }
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(K), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(experts > 0 ? experts : 1)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(K), static_cast<cuuint64_t>(K) * static_cast<cuuint64_t>(rows)};
    const cuuint32_t box[3] = {kGroup, static_cast<cuuint32_t>(box_rows), 1}, ones[3] = {1, 1, 1};
    const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, experts > 0 ? 3 : 2, const_cast<void *>(data), dims, strides, box, ones,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        g_last_cuda_error = cudaErrorInvalidValue;
        return BITCOS_ERR_CUDA;
    }
    return BITCOS_OK;
}

// The outputs: boxes of 32 rows of 128 bytes.
int encode_outputs(CUtensorMap *map, const Fp8Args &a) {
    const EncodeTiled f = encode_tiled();
    const cuuint64_t size = a.out_bf16 ? 2 : 4;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(a.M), static_cast<cuuint64_t>(a.rows)}, strides[1] = {static_cast<cuuint64_t>(a.M) * size};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(128 / size), 32}, ones[2] = {1, 1};
    const CUresult r = f(map, a.out_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, a.y, dims, strides, box, ones,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        g_last_cuda_error = cudaErrorInvalidValue;
        return BITCOS_ERR_CUDA;
    }
    return BITCOS_OK;
}

// Once per kernel and device, as in prepare_kernel, and all of the cache as shared memory.
template <int N, bool PAIR, bool GROUPED, bool PATIENT>
int prepare_fp8(int dev) {
    using L = Layout<N, PAIR, GROUPED>;
    auto *kernel = fp8_matmul_kernel<N, PAIR, GROUPED, PATIENT>;
    static bool prepared[32];
    if (dev < 32 && prepared[dev]) return BITCOS_OK;
    int rc = BITCOS_OK;
    if (PAIR) {
        cudaFuncAttributes attributes{};
        rc = check_cuda(cudaFuncGetAttributes(&attributes, kernel));
        if (rc) return rc;
        if (attributes.numRegs != kLaunchRegisters) {          // (the split would wait for registers that are not there)
            g_last_cuda_error = cudaErrorInvalidDeviceFunction;
            return BITCOS_ERR_CUDA;
        }
    }
    rc = check_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(L::kDynamic)));
    if (rc == BITCOS_OK)
        rc = check_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    if (rc == BITCOS_OK && dev < 32) prepared[dev] = true;
    return rc;
}

template <int N, bool PAIR, bool GROUPED, bool PATIENT = true>
int launch_fp8(const void *W, const void *x, int64_t K, int experts, int64_t x_rows, const Fp8Args &args, int64_t blocks, cudaStream_t stream) {
    if (PATIENT && args.patience.limit_ns < kLooks) return launch_fp8<N, PAIR, GROUPED, false>(W, x, K, experts, x_rows, args, blocks, stream);
    using L = Layout<N, PAIR, GROUPED>;
    static_assert(L::kStages + L::kAcc + 1 < kTileRing, "the producer's lead");
    static_assert(L::kBlocks * (L::kDynamic + 1024) <= 228 * 1024 && L::kBlocks * L::kTmemColumns <= 512, "the blocks of a multiprocessor");
    static_assert(L::kDynamic <= 227 * 1024, "shared memory of a block");
    CUtensorMap wmap, xmap, ymap{};
    int rc = encode(&wmap, W, K, args.M, experts, PAIR ? L::kBRows : kARows);
    if (rc) return rc;
    rc = encode(&xmap, x, K, x_rows, 0, L::kRowsPerTile);
    if (rc) return rc;
    if (PAIR && args.vector) rc = encode_outputs(&ymap, args);
    if (rc) return rc;
    auto *kernel = fp8_matmul_kernel<N, PAIR, GROUPED, PATIENT>;
    int dev = 0;
    rc = check_cuda(cudaGetDevice(&dev));
    if (rc == BITCOS_OK) rc = prepare_fp8<N, PAIR, GROUPED, PATIENT>(dev);
    if (rc) return rc;
    static const char *env = std::getenv("BITCOS_PDL");
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(L::kThreads);
    cfg.dynamicSmemBytes = L::kDynamic;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    const int cluster = PAIR ? 2 : args.splits;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = cluster > 1 ? attr : attr + 1;
    cfg.numAttrs = (cluster > 1 ? 1 : 0) + ((env && env[0] == '0') ? 0 : 1);
    void *pointers[] = {&wmap, &xmap, &ymap, const_cast<Fp8Args *>(&args)};
    return check_cuda(cudaLaunchKernelExC(&cfg, reinterpret_cast<const void *>(kernel), pointers));
}

int multiprocessors(int *sms) {
    static int cache[32];
    int dev = 0;
    int rc = check_cuda(cudaGetDevice(&dev));
    if (rc) return rc;
    if (dev < 32 && cache[dev] > 0) {
        *sms = cache[dev];
        return BITCOS_OK;
    }
    rc = check_cuda(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
    if (rc == BITCOS_OK && dev < 32) cache[dev] = *sms;
    return rc;
}

// Dense, weights first: into how many shares K is cut, and the nanoseconds expected of it.  A block takes 270, 310 or 490 ns for a group
// of 128 at 16, 32 and 64 tokens (640 rows, K = 6400 and 25600), or, with all multiprocessors at it, what memory needs for its
// 16 KB; start, first copies and the cluster's sum cost 2 us more per round.  The clusters that the device holds at once are asked for
// once per kernel and device (of seven blocks there are 30: 40 row blocks of 5120 x 25600 took two rounds and 36 us).  Tokens first 410 ns a
// group, its 770 clocks at 1.9 GHz: calls this short are not at the power limit.
constexpr int64_t kGroupNs16 = 270, kGroupNs32 = 310, kGroupNs64 = 490, kRoundNs = 2000, kPairGroupNs = 410, kPairNs = 3500;
template <int N, bool GROUPED>
int plan_weights_first(const Fp8Args &a, int64_t tiles, int sms, int *splits_out, int64_t *ns_out) {
    *splits_out = 1;
    if (tiles > INT_MAX / kMaxSplits) return GROUPED ? BITCOS_OK : BITCOS_ERR_SHAPE;
    static int held[32][kMaxSplits + 1];
    int dev = 0;
    int rc = check_cuda(cudaGetDevice(&dev));
    if (rc) return rc;
    rc = prepare_fp8<N, false, GROUPED, true>(dev);
    if (rc) return rc;
    constexpr int64_t group_ns = N == 16 ? kGroupNs16 : N == 32 ? kGroupNs32 : kGroupNs64;
    *ns_out = INT64_MAX;
    for (int splits = 1; splits <= kMaxSplits && (splits == 1 || a.G / splits >= 2); ++splits) {
        int clusters = dev < 32 ? held[dev][splits] : 0;
        if (clusters == 0) {
            cudaLaunchConfig_t cfg{};
            cudaLaunchAttribute attr{};
            cfg.gridDim = dim3(static_cast<unsigned>(splits));
            cfg.blockDim = dim3(Layout<N, false, GROUPED>::kThreads);
            cfg.dynamicSmemBytes = Layout<N, false, GROUPED>::kDynamic;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = static_cast<unsigned>(splits);
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            rc = check_cuda(cudaOccupancyMaxActiveClusters(&clusters, fp8_matmul_kernel<N, false, GROUPED, true>, &cfg));
            if (rc) return rc;
            clusters = Layout<N, false, GROUPED>::kBlocks * std::max(clusters, 1);      // (it counts one block per multiprocessor, whatever its size)
            if (dev < 32) held[dev][splits] = clusters;
        }
        const int64_t rounds = (tiles + clusters - 1) / clusters;
        if (GROUPED && splits > 1 && rounds > 1) continue;                    // (the blocks of a cluster take one tile)
        const int64_t active = std::min<int64_t>(tiles, clusters) * splits;
        const int64_t memory_ns = active * 365 / sms;                         // 16 KB each at 6.5 TB/s
        const int64_t ns = rounds * (kRoundNs + (a.G + splits - 1) / splits * std::max(group_ns, memory_ns));
        if (ns < *ns_out) {
            *ns_out = ns;
            *splits_out = splits;
        }
    }
    return BITCOS_OK;
}
template <int N>
int launch_weights_first(const void *W, const void *x, int64_t K, Fp8Args &a, int sms, cudaStream_t stream) {
    int64_t ns = 0;
    const int64_t row_tiles = (a.rows + N - 1) / N;
    const int rc = plan_weights_first<N, false>(a, row_tiles * a.w_blocks, sms, &a.splits, &ns);
    if (rc) return rc;
    a.row_tiles = static_cast<int>(row_tiles);
    a.w_tiles = a.w_blocks;
    return launch_fp8<N, false, false>(W, x, K, 1, a.rows, a, row_tiles * a.w_blocks * a.splits, stream);
}

Patience patience_of(uint64_t limit_ns) { return Patience{limit_ns, static_cast<uint32_t>(std::min<uint64_t>(limit_ns, kSleepNs))}; }

int status_word(void *workspace, size_t workspace_bytes, unsigned int **status) {
    *status = static_cast<unsigned int *>(workspace);
    if (!workspace) return BITCOS_OK;
    if (!aligned16(workspace)) return BITCOS_ERR_ALIGN;
    return workspace_bytes < BITCOS_FP8_WORKSPACE_BYTES ? BITCOS_ERR_CAPACITY : BITCOS_OK;
}

}  // namespace

extern "C" {

int bitcos_fp8_quantize(const void *x, int x_type, int64_t rows, int64_t K, uint8_t *q, float *scale, void *cuda_stream) {
    if (!x || !q || !scale) return BITCOS_ERR_NULL;
    if (rows < 0 || K < kGroup || K % kGroup != 0 || (x_type != BITCOS_FP32 && x_type != BITCOS_BF16)) return BITCOS_ERR_SHAPE;
    const int64_t per_block = 16 * kQuantGroups;
    if (rows > INT_MAX || K / kGroup > INT_MAX || rows * (K / kGroup) > per_block * INT_MAX) return BITCOS_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(q) || reinterpret_cast<uintptr_t>(scale) % 4) return BITCOS_ERR_ALIGN;
    if (rows == 0) return BITCOS_OK;
    const int64_t n_groups = rows * (K / kGroup);
    const dim3 grid(static_cast<unsigned>((n_groups + per_block - 1) / per_block));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (x_type == BITCOS_FP32) return launch_pdl(fp8_quantize_kernel<float>, grid, 256, 0, stream, static_cast<const float *>(x), q, scale, n_groups);
    return launch_pdl(fp8_quantize_kernel<__nv_bfloat16>, grid, 256, 0, stream, static_cast<const __nv_bfloat16 *>(x), q, scale, n_groups);
}

int bitcos_fp8_matmul(const uint8_t *W, const float *w_scale, int64_t M, int64_t K, const uint8_t *x, const float *x_scale, int64_t rows,
                      void *y, int y_type, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    return bitcos_fp8_matmul_limited(W, w_scale, M, K, x, x_scale, rows, y, y_type, workspace, workspace_bytes, kWaitLimitNs, cuda_stream);
}

int bitcos_fp8_matmul_limited(const uint8_t *W, const float *w_scale, int64_t M, int64_t K, const uint8_t *x, const float *x_scale, int64_t rows,
                              void *y, int y_type, void *workspace, size_t workspace_bytes, uint64_t wait_limit_ns, void *cuda_stream) {
    if (!W || !w_scale || !x || !x_scale || !y) return BITCOS_ERR_NULL;
    if (M < 1 || M > BITCOS_FP8_ROWS_MAX || K < kGroup || K % kGroup != 0 || K > BITCOS_FP8_ROWS_MAX || rows < 0 || rows > BITCOS_FP8_ROWS_MAX ||
        (y_type != BITCOS_FP32 && y_type != BITCOS_BF16))
        return BITCOS_ERR_SHAPE;
    if (!aligned16(W) || !aligned16(x) || !aligned16(y) || reinterpret_cast<uintptr_t>(w_scale) % 4 || reinterpret_cast<uintptr_t>(x_scale) % 4)
        return BITCOS_ERR_ALIGN;
    Fp8Args a{};
    int rc = status_word(workspace, workspace_bytes, &a.status);
    if (rc) return rc;
    if (rows == 0) return BITCOS_OK;
    a.patience = patience_of(wait_limit_ns);
    a.w_scale = w_scale;
    a.x_scale = x_scale;
    a.y = y;
    a.M = M;
    a.rows = rows;
    a.G = static_cast<int>(K / kGroup);
    a.w_blocks = static_cast<int>((M + kGroup - 1) / kGroup);
    a.out_bf16 = y_type == BITCOS_BF16;
    a.vector = M % (a.out_bf16 ? 8 : 4) == 0;
    a.splits = 1;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int sms = 0;
    rc = multiprocessors(&sms);
    if (rc) return rc;
    const int64_t row_tiles = (rows + 255) / 256, w_tiles = (M + 255) / 256;
    // Above 512 rows tokens first: 600 x 6912 x 2560 23.3 us against 35.6 weights first, 1024 x 8192 x 5120 42.4 against 122, 2048 x 2560 x 2560
    // 23.4 against 54.9.  (The other way round where M leaves most pairs without a tile and K is long: 513 x 128 x 25600 83 us against 18,
    // 1024 x 256 x 25600 86 against 25, 4095 x 64 x 25600 89 against 35.  The rule does not look at that.)
    bool pairs = rows > 512;
    if (rows > 64 && !pairs) {
        // few rows: whichever ends sooner (200 x 8192 x 5120 tokens first 22.7 us against 29.9, 300 x 6912 x 2560 14.3 against 18.0, 128 x 2560 x 6912
        // weights first 11.7 against 26.8)
        int splits = 0;
        int64_t ns = 0;
        rc = plan_weights_first<64, false>(a, (rows + 63) / 64 * a.w_blocks, sms, &splits, &ns);
        if (rc) return rc;
        pairs = kPairNs + (row_tiles * w_tiles + sms / 2 - 1) / (sms / 2) * a.G * kPairGroupNs <= ns;
    }
    if (pairs) {
        if (row_tiles * w_tiles > INT_MAX) return BITCOS_ERR_SHAPE;
        a.row_tiles = static_cast<int>(row_tiles);
        a.w_tiles = static_cast<int>(w_tiles);
        return launch_fp8<256, true, false>(W, x, K, 1, rows, a, 2 * std::min<int64_t>(row_tiles * w_tiles, sms / 2), stream);
    }
    // (the narrowest tile that takes all rows: 25600 x 5120 at 32 rows 25.0 us, with two tiles of 16 35.2; at 64 rows 29.6, with tiles of 32
    // 38.6, of 16 46.5; 6912 x 2560 at 16 rows 6.55, with a tile of 32 6.74)
    if (rows <= 16) return launch_weights_first<16>(W, x, K, a, sms, stream);
    if (rows <= 32) return launch_weights_first<32>(W, x, K, a, sms, stream);
    return launch_weights_first<64>(W, x, K, a, sms, stream);
}

int bitcos_fp8_matmul_grouped(const uint8_t *W, const float *w_scale, int n_experts, int64_t M, int64_t K, const int32_t *group_expert,
                              const int32_t *group_begin, const int32_t *n_groups_device, int max_groups, const int32_t *pair_xrow,
                              int64_t n_pairs, const uint8_t *x, const float *x_scale, int64_t n_xrows, void *y, int y_type, void *workspace,
                              size_t workspace_bytes, void *cuda_stream) {
    return bitcos_fp8_matmul_grouped_limited(W, w_scale, n_experts, M, K, group_expert, group_begin, n_groups_device, max_groups, pair_xrow, n_pairs,
                                             x, x_scale, n_xrows, y, y_type, workspace, workspace_bytes, kWaitLimitNs, cuda_stream);
}

int bitcos_fp8_matmul_grouped_limited(const uint8_t *W, const float *w_scale, int n_experts, int64_t M, int64_t K, const int32_t *group_expert,
                                      const int32_t *group_begin, const int32_t *n_groups_device, int max_groups, const int32_t *pair_xrow,
                                      int64_t n_pairs, const uint8_t *x, const float *x_scale, int64_t n_xrows, void *y, int y_type, void *workspace,
                                      size_t workspace_bytes, uint64_t wait_limit_ns, void *cuda_stream) {
    if (!W || !w_scale || !group_expert || !group_begin || !n_groups_device || !x || !x_scale || !y) return BITCOS_ERR_NULL;
    if (M < 1 || M > BITCOS_FP8_ROWS_MAX || K < kGroup || K % kGroup != 0 || K > BITCOS_FP8_ROWS_MAX || n_experts < 1 || max_groups < 1 ||
        max_groups > kMaxGroups || n_pairs < 0 || n_pairs > BITCOS_FP8_ROWS_MAX || n_xrows < 1 || n_xrows > BITCOS_FP8_ROWS_MAX ||
        (y_type != BITCOS_FP32 && y_type != BITCOS_BF16))
        return BITCOS_ERR_SHAPE;
    if (!aligned16(W) || !aligned16(x) || !aligned16(y) || reinterpret_cast<uintptr_t>(w_scale) % 4 || reinterpret_cast<uintptr_t>(x_scale) % 4 ||
        reinterpret_cast<uintptr_t>(group_expert) % 4 || reinterpret_cast<uintptr_t>(group_begin) % 4 ||
        reinterpret_cast<uintptr_t>(n_groups_device) % 4 || reinterpret_cast<uintptr_t>(pair_xrow) % 4)
        return BITCOS_ERR_ALIGN;
    Fp8Args a{};
    int rc = status_word(workspace, workspace_bytes, &a.status);
    if (rc) return rc;
    if (n_pairs == 0) return BITCOS_OK;
    a.patience = patience_of(wait_limit_ns);
    a.w_scale = w_scale;
    a.x_scale = x_scale;
    a.y = y;
    a.M = M;
    a.rows = n_pairs;
    a.G = static_cast<int>(K / kGroup);
    a.w_blocks = static_cast<int>((M + kGroup - 1) / kGroup);
    a.out_bf16 = y_type == BITCOS_BF16;
    a.vector = M % (a.out_bf16 ? 8 : 4) == 0;
    a.splits = 1;
    a.x = x;
    a.group_expert = group_expert;
    a.group_begin = group_begin;
    a.n_groups = n_groups_device;
    a.pair_xrow = pair_xrow;
    a.max_groups = max_groups;
    a.n_experts = n_experts;
    a.n_xrows = static_cast<int>(n_xrows);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int sms = 0;
    rc = multiprocessors(&sms);
    if (rc) return rc;
    // what the host knows of the groups' lengths is their mean, if all of them are there
    const int64_t mean = (n_pairs + max_groups - 1) / max_groups;
    a.w_tiles = a.w_blocks;
    if ((n_pairs / 16 + max_groups) * a.w_tiles > INT_MAX) return BITCOS_ERR_SHAPE;
    // 16 tokens a tile, weights first, against 256, tokens first: 128 experts of 1536 x 2048 (2048 x 768), mean 16 75 us against 123 (39 against
    // 77), 38 109 against 132 (62 against 75), 48 129 against 131 (76 against 75), 64 165 against 132 (93 against 74).  With groups as routing makes
    // them, of all lengths, the line is where it is: mean 48 118 against 120 (74 against 76; 64 experts of 1000 x 2048 43 against 48, 32 of 1024 x 512
    // 11.5 against 12.8), mean 64 156 against 128 (94 against 78; 56 against 48, 14.3 against 13.0).  Tiles of 32 and 64 tokens
    // lay between: 32 gained 5 to 7 % at means of 20 to 32 on the first shape and lost as much on the second, 64 won 5 % at 48 and nowhere else;
    // and tiles of 16 cost what the groups' lengths are, whatever their mean.
    if (mean <= 48) {
        // (no more blocks than there can be tiles; a tile per pair at most: with few pairs K is cut as in the dense product)
        int64_t ns = 0;
        rc = plan_weights_first<16, true>(a, n_pairs * a.w_blocks, sms, &a.splits, &ns);
        if (rc) return rc;
        const int64_t most = (n_pairs / 16 + std::min<int64_t>(max_groups, n_pairs)) * a.w_tiles;
        return launch_fp8<16, false, true>(W, x, K, n_experts, n_xrows, a,
                                           a.splits > 1 ? n_pairs * a.w_blocks * a.splits : std::min<int64_t>(3 * sms, most), stream);
    }
    a.w_tiles = static_cast<int>((M + 255) / 256);
    return launch_fp8<256, true, true>(W, x, K, n_experts, n_xrows, a, sms / 2 * 2, stream);
}

}  // extern "C"
