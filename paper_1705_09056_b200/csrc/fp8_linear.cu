// Host side of the 8-bit layers: tile shapes, tensor maps and the launches of one forward or backward pass over all
// nodes.  The kernels are in fp8_gemm.cuh (products) and ckpt8.cu (everything that only moves data).
#include <algorithm>
#include <new>

#include "ctx.h"
#include "fp8_gemm.cuh"
#include "launch.h"
#include "tma_host.h"

namespace dpsgd {
namespace {

using namespace f8g;

int sm_count(const dpsgd_ctx* c) {
    int v = 0;
    return cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, c->device) == cudaSuccess && v > 0 ? v : 1;
}

// A problem's operands: A [node][M][K] (kForward, kInput) or [node][K][M] (kWeight), B [node][N][K] (kForward) or
// [node][K][N]; element size 1 (E4M3) or 2 (bf16); pitches in bytes.
struct Operands {
    const void *a, *b;
    int64_t a_pitch, b_pitch;
};

// What the result is rounded to, which decides how often sums are handed over (see fp8_gemm.cuh).
enum Rounding { kTo8, kToBf16, kToF32 };

template <int MODE, int BN, bool PAIR>
cudaError_t launch(dpsgd_ctx* c, const Operands& o, Args g, Rounding to) {
    using S = Shape<MODE, BN, PAIR>;
    auto kernel = fp8_gemm_kernel<MODE, BN, PAIR>;
    const cudaError_t attr = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemLimit);
    if (attr != cudaSuccess) return attr;
    const uint64_t nodes = (uint64_t)c->n, M = (uint64_t)g.M, N = (uint64_t)g.N, K = (uint64_t)g.K;
    const uint64_t ap = (uint64_t)o.a_pitch, bp = (uint64_t)o.b_pitch;
    CUtensorMap mapA, mapB;
    bool ok;
    if (MODE == kWeight) {
        g.a_rows = (uint32_t)std::min(64, (g.K + 15) / 16 * 16);
        g.a_bytes = 2 * 128 * g.a_rows;
        g.block_bytes = (2 + S::BH / 64) * 128 * g.a_rows;
        ok = make_map_3d_sw128(&mapA, o.a, 2, M, K, nodes, ap, K * ap, 64, g.a_rows) &&
             make_map_3d_sw128(&mapB, o.b, 2, N, K, nodes, bp, K * bp, 64, g.a_rows);
    } else {
        g.a_rows = (uint32_t)std::min(kTileM, (g.M + 7) / 8 * 8);
        g.a_bytes = 128 * g.a_rows;
        g.block_bytes = g.a_bytes + S::B_BYTES;
        ok = make_map_3d_sw128(&mapA, o.a, 1, K, M, nodes, ap, M * ap, 128, g.a_rows) &&
             (MODE == kForward ? make_map_3d_sw128(&mapB, o.b, 1, K, N, nodes, bp, N * bp, 128, (uint32_t)S::BH)
                               : make_map_3d_sw128(&mapB, o.b, 1, N, K, nodes, bp, K * bp, 128, 128));
    }
    if (!ok) return cudaErrorInvalidValue;
    const uint32_t stage_bytes = g.block_bytes * S::KPS;
    g.stages = std::min<int>(kMaxStages, (int)((kSmemLimit - S::FIXED) / stage_bytes));
    if (BN == 256 && S::SCALED && to != kToBf16) return cudaErrorInvalidValue;      // their epilogue rounds to bf16 only
    g.hand = to == kToBf16 ? kCoarseHand : to == kTo8 ? kFineHand : kSegment;
    g.m_tiles = (g.M + S::TM - 1) / S::TM;
    g.n_tiles = (g.N + BN - 1) / BN;
    const int64_t total = (int64_t)c->n * g.m_tiles * g.n_tiles;
    if (total > INT32_MAX) return cudaErrorInvalidValue;
    g.total = (int)total;
    g.status = &c->d_result->status;
    // the tensor core reads A to its 128th row: rows beyond a_rows come from whatever follows in shared memory (B, the next
    // stage or the output staging) and only reach rows that are not stored
    c->launches++;
    const int64_t teams = std::max(1, sm_count(c) / S::CTAS);       // persistent CTAs or pairs of them
    return launch_chained_clusters(kernel, S::CTAS, (unsigned)(std::min(total, teams) * S::CTAS), S::THREADS,
                                   S::FIXED + g.stages * stage_bytes, c->stream, mapA, mapB, g);
}

int64_t rounds(int64_t tiles, int64_t places) { return (tiles + places - 1) / places; }

// Tiles of the forward product by the time they are expected to take, in us: rounds over the SMs (over pairs of them for the
// pair), times what a tile costs by itself (more where rows of the result are not aligned to 16 bytes and leave element by
// element) and per k-block.  The costs are a fit to 1634 random shapes (1 to 112 nodes, 1 to 4096 rows, widths of 128 to
// 4096) and choose a tile within 0.4 % of the best one on average, 26 % at worst.  Narrow tiles give every SM one when there are
// few rows; a pair (bf16 results only: its one accumulator waits at each hand-over, which others need every 8 or 16 MMAs)
// reads 32 KB per k-block and SM where single CTAs of 256 columns read 48 (an SM takes about 64 bytes per cycle from L2):
// training forward of 4 nodes 4096x4096x4096 293 us, 312 from single CTAs of 256 columns, 393 of 128.  With fp32 results and
// checkpoints 128 columns are level with the pair at best and up to 1.5 times as fast (32 nodes 400x2048x1003 fp32: 55 against
// 84 us; 16 nodes 512x2048x2048 with a checkpoint 55 against 61).
struct TileCost { int rows, cols; double once, tile, odd_tile, block; };
constexpr TileCost kTiles[] = {{128, 32, 0.0, 0.60, 1.2, 0.155}, {128, 64, 0.0, 0.82, 1.6, 0.18}, {128, 128, 0.0, 1.4, 3.4, 0.28},
                               {256, 256, 1.4, 2.9, 4.4, 0.34}};

cudaError_t launch_forward(dpsgd_ctx* c, const Operands& o, const Args& g, Rounding to) {
    const int sms = sm_count(c);
    int best = 2;                                                   // a checkpoint needs whole blocks of 128 columns in a tile
    double least = 0.0;
    for (int i = 0; i < 4 && to != kTo8; ++i) {
        const TileCost& t = kTiles[i];
        if (t.rows > kTileM && (g.M <= kTileM || to != kToBf16)) continue;
        const int64_t tiles = (int64_t)c->n * ((g.M + t.rows - 1) / t.rows) * ((g.N + t.cols - 1) / t.cols);
        const double each = (g.out_vec ? t.tile : t.odd_tile) + t.block * ((g.K + 127) / 128);
        const double us = t.once + (double)rounds(tiles, std::max(1, sms / (t.rows / kTileM))) * each;
        if (i == 0 || us <= least) { least = us; best = i; }
    }
    switch (best) {
        case 0: return launch<kForward, 32, false>(c, o, g, to);
        case 1: return launch<kForward, 64, false>(c, o, g, to);
        case 2: return launch<kForward, 128, false>(c, o, g, to);
        default: return launch<kForward, 256, true>(c, o, g, to);
    }
}

// dx: 256 columns for bf16 results with more than 128 rows, unless such tiles leave far more SMs idle in the last round.  1.2 to
// 1.3 as a limit is within 0.1 % of the better one of the two over 135 random shapes (always 128: 1.8 %).  With fp32 results
// 128 columns stay within 0.3 % (143 shapes; one accumulator, as above).
cudaError_t launch_input(dpsgd_ctx* c, const Operands& o, const Args& g, Rounding to) {
    const auto cost = [&](int cols) {
        return rounds((int64_t)c->n * ((g.M + kTileM - 1) / kTileM) * ((g.N + cols - 1) / cols), sm_count(c)) * cols;
    };
    if (to == kToBf16 && g.M > kTileM && cost(256) <= cost(128) * 1.3) return launch<kInput, 256, false>(c, o, g, to);
    return launch<kInput, 128, false>(c, o, g, to);
}

Rounding rounding(int dtype) { return dtype == DPSGD_F32 ? kToF32 : kToBf16; }

void set_out(Args& g, void* out, int dtype, int rows, int cols) {
    const int size = dtype == DPSGD_F32 ? 4 : 2;
    g.out = static_cast<uint8_t*>(out);
    g.out_size = size;
    g.out_pitch = (int64_t)cols * size;
    g.out_node = (int64_t)rows * g.out_pitch;
    g.out_vec = reinterpret_cast<uintptr_t>(out) % 16 == 0 && g.out_pitch % 16 == 0;
}

// Workspace of a backward pass: d in 8 bits | its exponents | d in bf16 | x in bf16 | bias partial sums
struct Workspace {
    int64_t ldv, ldx;                      // elements between rows of the bf16 copies
    size_t e, v, x, parts, total;          // byte offsets
};
Workspace make_workspace(const dpsgd_ctx* c, int B, int K, int O) {
    const auto round_up = [](size_t v) { return (v + 255) / 256 * 256; };
    const size_t rows = (size_t)c->n * B;
    const int chunks = delta_chunks(B);
    Workspace w{};
    w.ldv = (O + 7) / 8 * 8; w.ldx = (K + 7) / 8 * 8;
    w.e = round_up(rows * f8::q_pitch(O));
    w.v = w.e + round_up(rows * f8::e_pitch(O));
    w.x = w.v + round_up(rows * w.ldv * 2);
    w.parts = w.x + round_up(rows * w.ldx * 2);
    w.total = w.parts + (chunks > 1 ? round_up((size_t)c->n * chunks * O * 4) : 0);
    return w;
}

}  // namespace

// The workspace holds nothing between calls, but a graph that a caller captures holds its address: what such a graph was
// recorded on is kept until the context goes, and a capture that would need a larger one is refused before it records.
cudaError_t reserve_fp8_workspace(dpsgd_ctx* c, int B, int K, int O) {
    const size_t need = make_workspace(c, B, K, O).total;
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    bool capturing = true;                                          // also where the legacy stream cannot be asked during one
    if (cudaStreamIsCapturing(c->stream, &status) == cudaSuccess) capturing = status != cudaStreamCaptureStatusNone;
    else cudaGetLastError();
    if (need > c->fp8_ws_bytes) {
        if (capturing) return cudaErrorStreamCaptureUnsupported;
        if (c->fp8_ws_captured) {
            try { c->fp8_ws_kept.push_back(c->d_fp8_ws); } catch (const std::bad_alloc&) { return cudaErrorMemoryAllocation; }
        } else {
            cudaFree(c->d_fp8_ws);
        }
        c->d_fp8_ws = nullptr;
        c->fp8_ws_bytes = 0;
        c->fp8_ws_captured = false;
        const cudaError_t e = cudaMalloc(&c->d_fp8_ws, need);
        if (e != cudaSuccess) { c->d_fp8_ws = nullptr; return e; }
        c->fp8_ws_bytes = need;
    }
    c->fp8_ws_captured |= capturing;
    return cudaSuccess;
}

cudaError_t launch_fp8_forward(dpsgd_ctx* c, const uint8_t* xq, const uint8_t* xe, const uint8_t* wq, const uint8_t* we,
                               int B, int K, int O, const float* bias, int relu, void* y, int dtype, uint8_t* yq,
                               uint8_t* ye) {
    Args g{};
    g.M = B; g.N = O; g.K = K;
    g.ae = xe; g.ae_pitch = f8::e_pitch(K);
    g.we = we; g.we_pitch = f8::e_pitch(K); g.we_node = g.we_pitch * ((O + f8::kBlock - 1) / f8::kBlock);
    if (y) set_out(g, y, dtype, B, O);
    g.q = yq; g.q_pitch = f8::q_pitch(O); g.qe = ye; g.qe_pitch = f8::e_pitch(O);
    g.bias = bias; g.bias_node = c->ld; g.relu = relu;
    const Operands o{xq, wq, f8::q_pitch(K), f8::q_pitch(K)};
    return launch_forward(c, o, g, yq ? kTo8 : rounding(dtype));
}

cudaError_t launch_fp8_backward(dpsgd_ctx* c, const uint8_t* xq, const uint8_t* xe, const uint8_t* wq, const uint8_t* we,
                                const uint8_t* gate, const void* dy, int dy_dtype, int B, int K, int O, float* gw,
                                float* gb, void* dx, int dx_dtype) {
    cudaError_t e = reserve_fp8_workspace(c, B, K, O);
    if (e != cudaSuccess) return e;
    const Workspace ws = make_workspace(c, B, K, O);
    const int64_t ldv = ws.ldv, ldx = ws.ldx;
    uint8_t* dq = c->d_fp8_ws;
    uint8_t* de = dq + ws.e;
    uint8_t* dv = dq + ws.v;
    uint8_t* xv = dq + ws.x;
    float* parts = reinterpret_cast<float*>(dq + ws.parts);

    e = launch_delta(c, dy, dy_dtype, B, O, gate, dx ? dq : nullptr, de, dv, ldv, parts, gb, xq, xe, K, xv, ldx);
    if (e != cudaSuccess) return e;
    Args g{};
    g.M = K; g.N = O; g.K = B;
    g.out = reinterpret_cast<uint8_t*>(gw);
    g.out_node = c->ld * 4;
    const Operands w{xv, dv, ldx * 2, ldv * 2};
    // A gradient well beyond L2 from at most two k-blocks of samples: pairs of CTAs, which read the operands a third less.
    // Otherwise single CTAs, whose stores start sooner.  Without dx, single CTAs against pairs, us: 64 samples of 1024x1024 on
    // 64 nodes (256 MiB) 56.3 / 61.0, 96 88.0 / 87.9, 128 (512 MiB) 121.8 / 116.5, 256 260 / 235; of 2048x2048 on 32 nodes
    // (512 MiB) 107 / 109, 40 137 / 133, 112 434 / 372; 128 samples on these 471 / 429, 192 486 / 501, 256 448 / 525; 1024
    // samples on 64 nodes 674 / 691; 4096 samples of 4096x4096 on 4 nodes 478 / 500.
    const bool stream = K > kTileM && B <= kPairSamples && (double)c->n * K * O * 4.0 >= 512.0 * 1024 * 1024;
    e = stream ? launch<kWeight, 256, true>(c, w, g, kToF32) : launch<kWeight, 256, false>(c, w, g, kToF32);
    if (e != cudaSuccess || !dx) return e;
    // dx waits for the weight gradient, although it needs the launch before it only: a kernel may read what it has not itself
    // waited for only at its own risk (33.0 us without the wait against 36.0 on 32 nodes 32x784x1024, 23.9 against 25.3 on 7
    // nodes 77x1001x1003).
    Args h{};
    h.M = B; h.N = K; h.K = O;
    h.ae = de; h.ae_pitch = f8::e_pitch(O);
    h.we = we; h.we_pitch = f8::e_pitch(K); h.we_node = h.we_pitch * ((O + f8::kBlock - 1) / f8::kBlock);
    set_out(h, dx, dx_dtype, B, K);
    return launch_input(c, Operands{dq, wq, f8::q_pitch(O), f8::q_pitch(K)}, h, rounding(dx_dtype));
}

}  // namespace dpsgd
