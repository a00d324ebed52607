// Batched products of 8-bit layers on the 5th-generation tensor cores, one problem per node:
//
//   kForward   y[b][o]  = act(sum_k x[b][k] W[o][k] + bias[o])     both operands E4M3, contiguous along k
//   kInput     dx[b][k] = sum_o d[b][o] W[o][k]                    both E4M3; W contiguous along the output index
//   kWeight    gW[o][k] = sum_b d[b][o] x[b][k]                    both bf16 (the exact values of E4M3 numbers with
//                                                                  their scales), contiguous along the output indices
//
// kForward and kInput multiply with tcgen05.mma kind::mxf8f6f4.block_scale, which applies one power-of-two scale per
// operand row and 32 elements of the contraction.  A block of 128 is four of those with the same scale, so the four
// exponents of 512 consecutive k form one 32-bit word of a row's scale operand and k-block t uses byte t % 4: a scale
// costs nothing in the inner loop and no partial sum leaves the tensor core for it.  In kWeight the scales of both
// operands change from one step of the contraction (a sample) to the next, which the block-scaled form cannot express;
// E4M3 times 2^(e - 127) is exact in bf16 for e >= 3 (blocks whose largest magnitude is above 2^-116; below, what falls under
// 2^-133 is lost), so that product runs on kind::f16 at half the 8-bit rate, without rounding.
//
// A tile belongs to one CTA (128 rows) or to a pair of CTAs in a cluster (PAIR: 256 rows x 256 columns, tcgen05 with
// cta_group::2): each CTA of a pair keeps 128 rows of A and half the columns of B in shared memory and 128 rows of the
// accumulator in tensor memory, the first one (the leader) issues the MMAs for both, and a k-block brings 32 KB into an SM
// instead of 48.  An SM takes about 64 bytes per cycle from L2, so 128x256 tiles of one CTA run at 835 cycles per k-block
// (4096 x 4096 x 4096, tensor pipe 72 % active on the fullest SM) where the tensor core needs 512.
//
// Roles of a CTA (persistent, one per SM, tile t = team + i * teams, samples fastest so that CTAs side by side share a
// node's weights in L2):
//   TMA warp      one thread fills a ring of stages (128-byte swizzle; out-of-range rows, columns and k read as zero)
//   MMA warp      one thread issues the MMAs; tcgen05.commit frees stages and hands over accumulators
//   scale warps   (4, not in kWeight) read the exponent words of the next 512 k and put them in tensor memory: row r of an
//                 operand on lane r % 32, column r / 32, the same in all four lane quadrants
//   epilogue      (8) tcgen05.ld, bias, ReLU, rounding; a warp turns its 32 rows round in 4 KB of shared memory and writes
//                 whole 128-byte lines
// The tensor core truncates when it adds to an fp32 accumulator.  Where that can be seen in the result (fp32, or 8 bits,
// where a value next to a tie rounds the other way) the accumulator is handed over every 16 MMAs (kSegment) or, for 8 bits,
// every 8 (kFineHand), and added up by the epilogue warps in registers, rounding to nearest.  bf16 results are handed over
// every 128 MMAs (kCoarseHand, 4096 of the contraction): what that loses stays below 2^-16 of the sum of magnitudes, and
// products of up to 4096 keep one accumulator per tile (every 64 MMAs cost 307 -> 318 us on 4 nodes 4096x4096x4096).
// 8 MMAs instead of 16 bring the sums behind a checkpoint from 1.06-1.25 times the error of plain fp32 sums to 0.96-1.20 (32
// nodes 32x784x1024 over six seeds) and cost 39.0 -> 40.5 us there, 473.6 -> 480.8 us on 112 nodes 64x2048x2048, three
// accumulators in turn (40.9 and 484 us with two).  256 columns leave room for one accumulator beside the scales, which waits
// at each hand-over (weights and product of 4 nodes 4096x4096x4096: 411 us every 16 MMAs, 521 every 8), so they are for bf16.
// The epilogue takes an accumulator into registers and frees it before it does anything else, so that even a single
// 256-column one (two leave no room for the scales) keeps the tensor core waiting for a few hundred cycles only.  The
// registers come from the other warps (setmaxnreg).
// Measured: forward with a checkpoint out, 112 nodes 64 x 2048 x 2048: 95 us, 4.9 TB/s of 8-bit weights (the last round of
// tiles is a tenth full; 92 us with 16 MMAs per accumulator); backward of the same layer without dx: 434 us from single CTAs,
// 370 from pairs, 5.1 TB/s of stores, held back by its operand loads; forward, 4 nodes 4096 x 4096 x 4096: 201 us, 2.7 PFLOP/s.
// Every mbarrier wait is bounded; one that runs out raises the status word, the TMA thread waits (bounded) for its loads
// in flight and the CTA frees its tensor memory before it returns.
#pragma once
#include <cuda.h>

#include "fp8_num.cuh"
#include "launch.h"
#include "tc_stream.cuh"

namespace dpsgd {
namespace f8g {

using tc::mbar_arrive;
using tc::mbar_init;
using tc::mbar_wait;
using tc::smem_u32;
using tcs::mbar_expect_tx;
using tcs::tma_load_3d;

enum { kForward = 0, kInput = 1, kWeight = 2 };

constexpr int kTileM = 128;
constexpr int kEpiWarps = 8;
constexpr uint32_t kStageOut = 4096;                 // shared memory per epilogue warp
constexpr uint32_t kSmemLimit = 232448;              // 227 KB per CTA
constexpr int kSegment = 4;                          // k-blocks per scale word, and per accumulator handed over
constexpr int kFineHand = 2, kCoarseHand = 32;       // the same where the result is rounded to 8 bits, to bf16
constexpr int kPairSamples = 128;                    // samples of a weight gradient that pairs of CTAs take at most
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kScaleCol = 256, kScaleSet = 16;  // scale columns of a segment: 4 for A, up to 8 for B
constexpr int kScaleSets = 4;
constexpr int kMaxStages = 32;

struct Args {
    int M, N, K;                                     // rows, columns and contraction of a node's problem
    int m_tiles, n_tiles, total;                     // total = nodes * m_tiles * n_tiles; m_tiles of Shape::TM rows
    const uint8_t* ae; int64_t ae_pitch;             // exponents of A: row node * M + m, one byte per k-block
    const uint8_t* we; int64_t we_node, we_pitch;    // exponents of W: [node][128 outputs][128 inputs]
    uint8_t* out; int64_t out_node, out_pitch;       // result in bytes strides; NULL: not wanted
    int out_size, out_vec;                           // 4 (fp32) or 2 (bf16) bytes; rows aligned to 16 bytes
    uint8_t* q; int64_t q_pitch;                     // kForward: the result as a checkpoint, rows node * M + m
    uint8_t* qe; int64_t qe_pitch;
    const float* bias; int64_t bias_node;            // kForward; NULL: none
    int relu;
    int hand;                                        // k-blocks after which an accumulator is handed over
    uint32_t a_rows;                                 // rows of A a stage loads (8 .. 128);  kWeight: samples it loads (16 .. 64)
    uint32_t a_bytes, block_bytes;                   // of a k-block: A, and A with B; a stage is Shape::KPS of them
    int stages;
    int* status;
};

template <int MODE, int BN, bool PAIR> struct Shape {
    static_assert(!PAIR || BN == 256, "a pair shares 256 columns");
    static constexpr int CTAS = PAIR ? 2 : 1;                      // CTAs that share a tile: 128 rows of A each, the columns of B halved
    static constexpr int TM = kTileM * CTAS;                       // rows of a tile
    static constexpr int BH = BN / CTAS;                           // columns of B in one CTA's shared memory
    static constexpr bool SCALED = MODE != kWeight;
    static constexpr int KB = SCALED ? 128 : 64;                   // contraction per stage: one scale block / 64 samples
    static constexpr int KI = SCALED ? 32 : 16;                    // contraction per MMA
    static constexpr uint32_t B_BYTES = BH * 128;                  // of a k-block, per CTA
    static constexpr int KPS = BN >= 256 ? 1 : BN == 128 ? 2 : 4;  // k-blocks per stage
    static constexpr int HALVES = BN >= 64 ? 2 : 1;                // column halves, four warps each
    static constexpr int COLS = BN / HALVES;                       // columns of a row one epilogue thread holds
    // accumulators in tensor memory: one after the other from column 0, the third of 128 columns behind the scales
    static constexpr int ACCS = SCALED && BN == 256 ? 1 : SCALED && BN == 128 ? 3 : 2;
    static __device__ __forceinline__ uint32_t acc_col(uint32_t i) {
        return i * (uint32_t)BN + (ACCS == 3 && i == 2 ? kScaleCol + kScaleSets * kScaleSet - 2 * (uint32_t)BN : 0u);
    }
    static constexpr uint32_t MAXIMA = MODE == kForward && BN == 128 ? 2048 : 0;   // [tile parity][half][128 rows]
    // alignment, output staging, barriers
    static constexpr uint32_t OUT = MODE == kWeight ? 0 : kStageOut;                // output staging of a warp
    static constexpr uint32_t FIXED = 1024 + kEpiWarps * OUT + MAXIMA + 1024;
    static constexpr int FIRST_EPI = SCALED ? 8 : 4;               // warps 4-7 write scales where there are any
    static constexpr int THREADS = 32 * (FIRST_EPI + kEpiWarps);
    // registers per thread: launched with 65536 / THREADS rounded down to a multiple of 8 (128 or 168); the first
    // FIRST_EPI warps give theirs to the epilogue: 256 * 88 + 256 * 168 = 256 * 72 + 256 * 184 = 512 * 128,
    // 128 * 80 + 256 * 208 < 384 * 168.  With 72 / 184 the scale warps spill, but for kInput of 128 columns (302 us for the
    // forward of 4 nodes 4096x4096x4096, 297 with 88 / 168); with 96 / 160 the epilogue of 256 columns does.  kInput of 128
    // columns is level or better with 72 / 184 (backward of 32 nodes 32x784x1024: 36.1 against 36.6 us).
    static constexpr int REGS_FEW = !SCALED ? 80 : MODE == kInput && BN == 128 ? 72 : 88, REGS_EPI = SCALED ? 256 - REGS_FEW : 208;
};

// Shared-memory descriptor of an operand stored with the 128-byte swizzle.  k contiguous: rows of 128 bytes, 8-row
// groups 1024 bytes apart (lbo unused).  Row index contiguous: 128 bytes of it per k, groups of 8 k 1024 bytes apart,
// the next 128 bytes of the row index lbo bytes further.
__device__ __forceinline__ uint64_t desc_sw128(uint32_t addr, uint32_t lbo) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) | ((uint64_t)(1024u >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}

template <bool PAIR>
__device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                       uint32_t accumulate) {
    if (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
    else asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// ---- a pair of CTAs on one tile: barriers of the first CTA (the leader) collect what both have done ----
// Address of the leader's copy of a shared-memory object
__device__ __forceinline__ uint32_t leader_addr(const void* p) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(p)));
    return r;
}
template <bool PAIR>
__device__ __forceinline__ void arrive_leader(uint64_t* bar) {
    if (PAIR) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_addr(bar)) : "memory");
    else mbar_arrive(bar);
}
// MMAs issued so far: arrive on this barrier (of both CTAs) once they are done
template <bool PAIR>
__device__ __forceinline__ void commit(uint64_t* bar) {
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
    else tc::mma_commit(bar);
}
// A tile of this CTA's own memory and shared memory, reported to the leader's barrier
template <bool PAIR>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    if (PAIR)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
            ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(leader_addr(bar)) : "memory");
    else tma_load_3d(dst, map, x, y, z, bar);
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// Whether the phase is complete now (no wait)
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(r) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return r != 0;
}
// True in one thread of a converged warp, always the same one.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// 32 consecutive columns of this thread's TMEM lane.  The values may be used after tmem_wait on the same registers.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_wait(float* v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])::"memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t addr, const uint32_t (&r)[4]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 lds128u(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint32_t lds32u(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}

// A warp's 32 rows x W words (lane = row) to memory through its 4 KB of shared memory.  Row r goes to dst + r * pitch;
// rows at or beyond `rows` and bytes at or beyond `bytes` lie outside the result.  vec: rows are 16-byte aligned and
// `bytes` is a multiple of 16 (or beyond the W words); otherwise elements of `size` bytes are written one by one.
// 16-byte chunks are stored at chunk ^ f(row), which makes both directions free of bank conflicts.
template <int W>
__device__ __forceinline__ void store_rows(const uint32_t (&w)[W], uint32_t st, uint8_t* dst, int64_t pitch, int rows,
                                           int bytes, bool vec, int size, int lane) {
    constexpr int CH = W / 4;                                       // chunks per row: 8 or 4
    const auto at = [&](int row, int ch) {
        return st + (uint32_t)row * (W * 4) + (uint32_t)((ch ^ (CH == 8 ? row : row >> 1)) & (CH - 1)) * 16;
    };
    __syncwarp();
#pragma unroll
    for (int c = 0; c < CH; ++c) sts128(at(lane, c), w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
    __syncwarp();
    if (vec) {
        constexpr int RPI = 32 / CH;                                // rows per instruction
        const int ch = lane % CH;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int row = i * RPI + lane / CH;
            const uint4 v = lds128u(at(row, ch));
            if (row < rows && ch * 16 < bytes) *reinterpret_cast<uint4*>(dst + (int64_t)row * pitch + ch * 16) = v;
        }
    } else {
        const int n = min(rows, 32);
        for (int row = 0; row < n; ++row) {
            if (lane >= W) break;
            const uint32_t v = lds32u(at(row, lane / 4) + (uint32_t)(lane & 3) * 4);
            uint8_t* p = dst + (int64_t)row * pitch + lane * 4;
            if (size == 4) {
                if (lane * 4 < bytes) *reinterpret_cast<uint32_t*>(p) = v;
            } else {
                if (lane * 4 < bytes) *reinterpret_cast<uint16_t*>(p) = (uint16_t)v;
                if (lane * 4 + 2 < bytes) *reinterpret_cast<uint16_t*>(p + 2) = (uint16_t)(v >> 16);
            }
        }
    }
}

// kWeight: lanes run along the input index, which is contiguous in the parameter row, so a warp stores 128 bytes of a row per
// instruction straight from its registers and the four lane quadrants 512, at any alignment of the row.
__device__ __forceinline__ float* weight_row(const Args& g, int node, int o, int k) {
    return reinterpret_cast<float*>(g.out + (int64_t)node * g.out_node) + (int64_t)o * g.M + k;
}
template <int COLS>
__device__ __forceinline__ void store_weights(const float* v, float* dst, int pitch, int cols) {
    if (cols >= COLS) {
#pragma unroll
        for (int j = 0; j < COLS; ++j) __stcs(dst + (int64_t)j * pitch, v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < COLS; ++j) if (j < cols) __stcs(dst + (int64_t)j * pitch, v[j]);
    }
}

template <int MODE, int BN, bool PAIR>
__global__ void __launch_bounds__(Shape<MODE, BN, PAIR>::THREADS, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, Args g) {
    using S = Shape<MODE, BN, PAIR>;
    constexpr int COLS = S::COLS, ACCS = S::ACCS, KPS = S::KPS;
    static_assert(kSegment % KPS == 0, "a stage lies in one segment");
    const uint32_t stage_bytes = g.block_bytes * KPS;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* fixed_ptr = smem_raw + (base - smem_u32(smem_raw)) + (uint32_t)g.stages * stage_bytes;
    const uint32_t out_stage = base + (uint32_t)g.stages * stage_bytes;
    uint32_t* maxima = reinterpret_cast<uint32_t*>(fixed_ptr + kEpiWarps * S::OUT);   // [tile parity][half][128]
    uint64_t* full = reinterpret_cast<uint64_t*>(fixed_ptr + kEpiWarps * S::OUT + S::MAXIMA);
    uint64_t* empty = full + kMaxStages;
    uint64_t* acc_full = empty + kMaxStages;  // [2]
    uint64_t* acc_empty = acc_full + 3;       // [3]
    uint64_t* sf_full = acc_empty + 3;        // [kScaleSets]
    uint64_t* sf_empty = sf_full + kScaleSets;
    uint64_t* max_full = sf_empty + kScaleSets;   // [4] both column halves of a lane quadrant have left their maxima
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(max_full + 4);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = PAIR ? (int)(blockIdx.x & 1u) : 0;             // clusters are pairs of neighbours: rank 0 leads
    const int KBS = (g.K + S::KB - 1) / S::KB;                      // k-blocks
    const int SEGS = (KBS + kSegment - 1) / kSegment;

    if (tid == 32) {           // the maps are kernel parameters: their fetch need not wait for the predecessor
        asm volatile("prefetch.tensormap [%0];" ::"l"(&mapA) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&mapB) : "memory");
    }
    if (tid == 0) {
        for (int s = 0; s < g.stages; ++s) { mbar_init(full + s, 1); mbar_init(empty + s, 1); }
        for (int b = 0; b < 3; ++b) { mbar_init(acc_full + b, 1); mbar_init(acc_empty + b, 32 * 4 * S::HALVES * S::CTAS); }
        for (int b = 0; b < kScaleSets; ++b) { mbar_init(sf_full + b, 128 * S::CTAS); mbar_init(sf_empty + b, 1); }
        for (int b = 0; b < 4; ++b) mbar_init(max_full + b, 64);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc::tc_fence_before();
    if (PAIR) cluster_sync();       // the peer's barriers are ready before anything reaches them
    else __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    chain_next();
    chain_wait();
    const int per_node = g.m_tiles * g.n_tiles;
    bool ok = true;

    if (warp < S::FIRST_EPI) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::REGS_FEW));
        if (warp == 0) {
            // ------------------------------ TMA ------------------------------
            if (lane == 0) {
                uint32_t s = 0, ph = 0, issued = 0;
                const uint32_t rows = g.a_rows, tx = MODE == kWeight ? g.block_bytes : rows * 128u + S::B_BYTES;
                for (int t = (int)blockIdx.x / S::CTAS; ok && t < g.total; t += (int)gridDim.x / S::CTAS) {
                    const int node = t / per_node, rem = t - node * per_node;
                    const int nt = rem / g.m_tiles, m0 = (rem - nt * g.m_tiles) * S::TM + rank * kTileM, n0 = nt * BN;
                    for (int kb0 = 0; kb0 < KBS; kb0 += KPS) {
                        if (!mbar_wait(empty + s, ph ^ 1u)) { ok = false; break; }
                        if (rank == 0) mbar_expect_tx(full + s, tx * (uint32_t)(S::CTAS * min(KPS, KBS - kb0)));   // of both CTAs
                        uint32_t a = base + s * stage_bytes;
#pragma unroll
                        for (int i = 0; i < KPS; ++i, a += g.block_bytes) {
                            if (kb0 + i >= KBS) break;
                            const uint32_t b = a + g.a_bytes;
                            const int k = (kb0 + i) * S::KB, nb = n0 + rank * S::BH;
                            if (MODE == kWeight) {
#pragma unroll
                                for (int j = 0; j < 2; ++j) load_tile<PAIR>(a + j * rows * 128u, &mapA, m0 + j * 64, k, node, full + s);
#pragma unroll
                                for (int j = 0; j < S::BH / 64; ++j) load_tile<PAIR>(b + j * rows * 128u, &mapB, nb + j * 64, k, node, full + s);
                            } else {
                                load_tile<PAIR>(a, &mapA, k, m0, node, full + s);
                                if (MODE == kForward) load_tile<PAIR>(b, &mapB, k, nb, node, full + s);
                                else
#pragma unroll
                                    for (int j = 0; j < S::BH / 128; ++j) load_tile<PAIR>(b + j * 16384, &mapB, nb + j * 128, k, node, full + s);
                            }
                        }
                        ++issued;
                        if (++s == (uint32_t)g.stages) { s = 0; ph ^= 1u; }
                    }
                }
                if (!ok) atomicExch(g.status, (int)DPSGD_ERR_TIMEOUT);
                // copies in flight land before the CTA ends (the leader's barriers count the peer's too)
                for (uint32_t i = rank == 0 ? min(issued, (uint32_t)g.stages) : 0u; i > 0; --i) {
                    if (s == 0) { s = (uint32_t)g.stages; ph ^= 1u; }
                    --s;
                    if (!mbar_wait(full + s, ph)) break;
                }
            }
        } else if (warp == 1) {
            // ------------------------------ MMA ------------------------------
            // One thread issues everything.  Its own instructions are what a short k-block costs (a satisfied wait takes
            // about 100 cycles, an issue 40 to 60), so the next stage is looked at before the current one is issued,
            // narrow tiles take several k-blocks per stage and descriptors are stepped, not rebuilt.
            if (rank == 0 && elect_one()) {
                // kind::mxf8f6f4: E4M3 x E4M3, UE8M0 scales;  kind::f16: bf16 x bf16 into fp32.  Bit 15 / 16: A / B
                // contiguous along its row index.
                const uint32_t idesc =
                    S::SCALED ? ((MODE == kInput ? 1u << 16 : 0u) | ((uint32_t)(BN >> 3) << 17) | (1u << 23) | ((uint32_t)(S::TM >> 7) << 27))
                              : ((1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(BN >> 3) << 17) |
                                 ((uint32_t)(S::TM >> 4) << 24));
                // bytes between operand pieces: of 64 row indices (kWeight), of 128 (kInput's B); bytes per MMA step of k
                constexpr uint32_t A_STEP = MODE == kWeight ? 2048 : 32, B_STEP = MODE == kForward ? 32 : MODE == kInput ? 4096 : 2048;
                const uint32_t chunk = g.a_rows * 128u;
                const uint64_t a_base = desc_sw128(base, MODE == kWeight ? chunk : 16);
                const uint64_t b_base = desc_sw128(base + g.a_bytes, MODE == kWeight ? chunk : MODE == kInput ? 16384 : 16);
                const uint32_t block_step = g.block_bytes >> 4, stage_step = stage_bytes >> 4;
                const int last_mmas = (g.K - (KBS - 1) * S::KB + S::KI - 1) / S::KI;      // of the last k-block
                uint32_t s = 0, ph = 0, seg_i = 0, acc_i = 0;
                bool ready = false;                                 // the stage about to be used has been seen full
                for (int t = (int)blockIdx.x / S::CTAS; ok && t < g.total; t += (int)gridDim.x / S::CTAS) {
                    int hand = 0;                                   // k-blocks in the accumulator so far
                    for (int kb0 = 0; kb0 < KBS; kb0 += KPS) {
                        const uint32_t ab0 = acc_i % ACCS;
                        if (S::SCALED && kb0 % kSegment == 0 && !mbar_wait(sf_full + seg_i % kScaleSets, (seg_i / kScaleSets) & 1u)) { ok = false; break; }
                        if (hand == 0 && !mbar_wait(acc_empty + ab0, ((acc_i / ACCS) & 1u) ^ 1u)) { ok = false; break; }
                        if (!ready && !mbar_wait(full + s, ph)) { ok = false; break; }
                        const uint32_t ns = s + 1 == (uint32_t)g.stages ? 0u : s + 1, nph = ns == 0 ? ph ^ 1u : ph;
                        ready = mbar_test(full + ns, nph);
                        tc::tc_fence_after();
                        uint64_t ad = a_base + s * stage_step, bd = b_base + s * stage_step;
                        const uint32_t sfa = tmem + kScaleCol + (seg_i % kScaleSets) * kScaleSet;
                        const uint32_t d = tmem + S::acc_col(ab0);
#pragma unroll
                        for (int i = 0; i < KPS; ++i, ad += block_step, bd += block_step) {
                            const int kb = kb0 + i;
                            if (kb >= KBS) break;
                            const uint32_t sub = (uint32_t)(kb % kSegment);
                            const uint32_t id = S::SCALED ? idesc | (sub << 29) | (sub << 4) : idesc;
                            const int mmas = kb + 1 == KBS ? last_mmas : S::KB / S::KI;
#pragma unroll
                            for (int j = 0; j < S::KB / S::KI; ++j) {
                                if (j >= mmas) break;
                                const uint32_t acc = (uint32_t)(hand > 0 || j > 0);       // 0: overwrites the accumulator
                                if (S::SCALED) mma_mx<PAIR>(d, ad + j * (A_STEP >> 4), bd + j * (B_STEP >> 4), id, sfa, sfa + 4, acc);
                                else mma_bf16<PAIR>(d, ad + j * (A_STEP >> 4), bd + j * (B_STEP >> 4), id, acc);
                            }
                            ++hand;
                        }
                        commit<PAIR>(empty + s);
                        const bool last = kb0 + KPS >= KBS;
                        if (last || (kb0 + KPS) % kSegment == 0) {
                            if (S::SCALED) commit<PAIR>(sf_empty + seg_i % kScaleSets);
                            ++seg_i;
                        }
                        if (last || hand == g.hand) { commit<PAIR>(acc_full + ab0); ++acc_i; hand = 0; }
                        s = ns; ph = nph;
                    }
                }
                if (!ok) atomicExch(g.status, (int)DPSGD_ERR_TIMEOUT);
            }
        } else if (S::SCALED && warp >= 4) {
            // ------------------------------ scales ------------------------------
            // The words of up to kScaleSets segments are loaded before the first is waited for, so that their latency is
            // paid once per 2048 k while the tensor core works through the sets written before.
            const uint32_t quad = tmem + ((uint32_t)((warp - 4) * 32) << 16) + kScaleCol;
            uint32_t seg_i = 0;
            for (int t = (int)blockIdx.x / S::CTAS; ok && t < g.total; t += (int)gridDim.x / S::CTAS) {
                const int node = t / per_node, rem = t - node * per_node;
                const int nt = rem / g.m_tiles, m0 = (rem - nt * g.m_tiles) * S::TM + rank * kTileM, n0 = nt * BN;
                const uint8_t* ae = g.ae + ((int64_t)node * g.M + m0 + lane) * g.ae_pitch;
                const uint8_t* we = g.we + (int64_t)node * g.we_node;
                for (int seg0 = 0; ok && seg0 < SEGS; seg0 += kScaleSets) {
                    uint32_t sa[kScaleSets][4], w[kScaleSets][2];
#pragma unroll
                    for (int u = 0; u < kScaleSets; ++u) {
                        const int seg = seg0 + u;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            sa[u][j] = seg < SEGS && m0 + lane + 32 * j < g.M
                                           ? __ldg(reinterpret_cast<const uint32_t*>(ae + (int64_t)(32 * j) * g.ae_pitch + seg * 4))
                                           : 0x7F7F7F7Fu;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            w[u][h] = 0x7F7F7F7Fu;
                            const int nb = n0 / f8::kBlock + h;      // block of 128 output columns
                            if (h >= (BN == 256 ? 2 : 1) || seg >= SEGS || nb * f8::kBlock >= g.N) continue;
                            if (MODE == kForward) {
                                w[u][h] = __ldg(reinterpret_cast<const uint32_t*>(we + (int64_t)nb * g.we_pitch + seg * 4));
                            } else {
                                uint32_t v = 0;
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const int kb = seg * 4 + j;
                                    v |= (kb < KBS ? (uint32_t)__ldg(we + (int64_t)kb * g.we_pitch + nb) : 127u) << (8 * j);
                                }
                                w[u][h] = v;
                            }
                        }
                    }
#pragma unroll
                    for (int u = 0; u < kScaleSets; ++u) {
                        if (seg0 + u >= SEGS || !ok) break;
                        const uint32_t b = seg_i % kScaleSets;
                        const bool go = mbar_wait(sf_empty + b, ((seg_i / kScaleSets) & 1u) ^ 1u);
                        if (!__all_sync(0xffffffffu, go)) { ok = false; break; }      // tcgen05.st needs the whole warp
                        tc::tc_fence_after();
                        const uint32_t col = quad + b * kScaleSet;
                        tmem_st4(col, sa[u]);
                        const uint32_t w0[4] = {w[u][0], w[u][0], w[u][0], w[u][0]};
                        tmem_st4(col + 4, w0);
                        if (BN == 256) {
                            const uint32_t w1[4] = {w[u][1], w[u][1], w[u][1], w[u][1]};
                            tmem_st4(col + 8, w1);
                        }
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                        tc::tc_fence_before();
                        arrive_leader<PAIR>(sf_full + b);
                        ++seg_i;
                    }
                }
            }
            if (!ok && lane == 0) atomicExch(g.status, (int)DPSGD_ERR_TIMEOUT);
        }
    } else {
        // ------------------------------ epilogue ------------------------------
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::REGS_EPI));
        const int ew = warp - S::FIRST_EPI, quad = warp & 3, half = ew >> 2;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * COLS);
        const uint32_t st = out_stage + (uint32_t)ew * S::OUT;
        uint32_t acc_i = 0, tile_i = 0;
        for (int t = (int)blockIdx.x / S::CTAS; ok && half < S::HALVES && t < g.total; t += (int)gridDim.x / S::CTAS, ++tile_i) {
            const int node = t / per_node, rem = t - node * per_node;
            const int nt = rem / g.m_tiles, m0 = (rem - nt * g.m_tiles) * S::TM + rank * kTileM + quad * 32;
            const int n0 = nt * BN + half * COLS;
            const int rows = g.M - m0;                              // valid rows of this warp (may be <= 0)
            if constexpr (MODE == kWeight) {
                // Few samples (all that a pair of CTAs is given): the tile is one accumulator and the time is that of its
                // stores.  32 columns at a time, so that the stores of one piece drain while the next is read from tensor
                // memory.
                static_assert(kPairSamples <= kSegment * S::KB, "one accumulator");
                if (PAIR || SEGS == 1) {
                    const uint32_t ab = acc_i % ACCS;
                    const bool go = mbar_wait(acc_full + ab, (acc_i / ACCS) & 1u);
                    if (!__all_sync(0xffffffffu, go)) { ok = false; break; }
                    tc::tc_fence_after();
                    float* dst = weight_row(g, node, n0, m0 + lane);
#pragma unroll 1
                    for (int c = 0; c < COLS; c += 32) {
                        float v[32];
                        tmem_ld32(lanes + ab * (uint32_t)BN + c, v);
                        tmem_wait(v);
                        if (lane < rows) store_weights<32>(v, dst + (int64_t)c * g.M, g.M, g.N - n0 - c);
                    }
                    tc::tc_fence_before();
                    arrive_leader<PAIR>(acc_empty + ab);
                    ++acc_i;
                    continue;
                }
            }
            float sum[COLS];
#pragma unroll
            for (int j = 0; j < COLS; ++j) sum[j] = 0.f;
            for (int kb = 0; kb < KBS; kb += g.hand, ++acc_i) {
                const uint32_t ab = acc_i % ACCS;
                const bool go = mbar_wait(acc_full + ab, (acc_i / ACCS) & 1u);
                if (!__all_sync(0xffffffffu, go)) { ok = false; break; }  // tcgen05.ld needs the whole warp
                tc::tc_fence_after();
                const uint32_t acc = lanes + S::acc_col(ab);
#pragma unroll
                for (int c = 0; c < COLS / 32; ++c) {
                    float v[32];
                    tmem_ld32(acc + c * 32, v);
                    tmem_wait(v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[c * 32 + j] += v[j];
                }
                tc::tc_fence_before();
                arrive_leader<PAIR>(acc_empty + ab);
            }
            if (!ok) break;
            if (MODE == kForward) {
                const float* bias = g.bias ? g.bias + (int64_t)node * g.bias_node : nullptr;
#pragma unroll
                for (int c = 0; c < COLS / 32; ++c) {
                    const int col = n0 + c * 32 + lane;
                    const float bv = bias && col < g.N ? __ldg(bias + col) : 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const float x = sum[c * 32 + j] + __shfl_sync(0xffffffffu, bv, j);
                        sum[c * 32 + j] = g.relu && x < 0.f ? 0.f : x;
                    }
                }
            }
            if constexpr (MODE == kWeight) {
                if (lane < rows) store_weights<COLS>(sum, weight_row(g, node, n0, m0 + lane), g.M, g.N - n0);
            } else if (g.out) {
                uint8_t* dst = g.out + (int64_t)node * g.out_node + (int64_t)m0 * g.out_pitch + (int64_t)n0 * g.out_size;
                const int bytes = (g.N - n0) * g.out_size;
                if (BN < 256 && g.out_size == 4) {
#pragma unroll
                    for (int c = 0; c < COLS / 32; ++c) {
                        uint32_t w[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) w[j] = __float_as_uint(sum[c * 32 + j]);
                        store_rows<32>(w, st, dst + c * 128, g.out_pitch, rows, bytes - c * 128, g.out_vec, 4, lane);
                    }
                } else {
                    constexpr int W = COLS >= 64 ? 32 : 16;
#pragma unroll
                    for (int c = 0; c < COLS / (2 * W); ++c) {
                        uint32_t w[W];
#pragma unroll
                        for (int j = 0; j < W; ++j) w[j] = f8::pack_bf16(sum[2 * (c * W + j)], sum[2 * (c * W + j) + 1]);
                        store_rows<W>(w, st, dst + c * 128, g.out_pitch, rows, bytes - c * 128, g.out_vec, 2, lane);
                    }
                }
            }
            if constexpr (MODE == kForward && BN == 128) {
                if (g.q) {
                    // columns beyond the result are 0 in the padding, also in rows that hold a NaN
                    if (n0 + COLS > g.N) {
#pragma unroll
                        for (int j = 0; j < COLS; ++j) sum[j] = n0 + j < g.N ? sum[j] : 0.f;
                    }
                    // the row's block of 128 columns, shared with the warp of the other half.  Two buffers: a warp writes one
                    // again only after its partner has arrived for the tile between, hence has read it
                    uint32_t top = 0;
#pragma unroll
                    for (int j = 0; j < COLS; ++j) top = max(top, f8::magnitude(sum[j]));
                    uint32_t* mx = maxima + (tile_i & 1u) * 256 + quad * 32 + lane;
                    mx[half * 128] = top;
                    mbar_arrive(max_full + quad);
                    const bool go = mbar_wait(max_full + quad, tile_i & 1u);
                    if (!__all_sync(0xffffffffu, go)) { ok = false; break; }
                    top = max(top, mx[(half ^ 1) * 128]);
                    const uint32_t ex = f8::scale_byte(top);
                    constexpr int W = COLS / 4;
                    uint32_t w[W];
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        w[j] = f8::encode_block4(sum[4 * j], sum[4 * j + 1], sum[4 * j + 2], sum[4 * j + 3], ex);
                    const int64_t row0 = (int64_t)node * g.M + m0;
                    store_rows<W>(w, st, g.q + row0 * g.q_pitch + n0, g.q_pitch, rows, (int)g.q_pitch - n0, true, 1, lane);
                    if (lane < rows && half == 0 && n0 < g.N) {
                        uint8_t* pe = g.qe + (row0 + lane) * g.qe_pitch;
                        const int blk = n0 / f8::kBlock;
                        pe[blk] = (uint8_t)ex;
                        if ((blk + 1) * f8::kBlock >= g.N)              // last block: the row's padding
                            for (int i = blk + 1; i < (int)g.qe_pitch; ++i) pe[i] = 127u;
                    }
                }
            }
        }
        if (!ok && lane == 0) atomicExch(g.status, (int)DPSGD_ERR_TIMEOUT);
    }
    tc::tc_fence_before();
    if (PAIR) cluster_sync();       // neither CTA leaves while the other may still reach its shared memory
    else __syncthreads();
    if (warp == 1) {
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

}  // namespace f8g
}  // namespace dpsgd
