// Expert products on the tensor cores (bf16 I/O): persistent pairs of CTAs on 256 x 256 tiles.
//
// A pair (cluster of two, tcgen05 cta_group::2) owns 256 rows x 256 columns: each CTA stages its own 128 rows of A and 128
// columns of B, the pair's MMA reads both halves, and each CTA's tensor memory ends up with its 128 rows of all 256 columns.
// That takes a third off the operand traffic per flop of a single CTA's 128 x 256 tile (64 bytes per clock and SM at full rate
// instead of 96; TMA loads that hit the L2 reach 67).  Two accumulators alternate, so the epilogue of a tile runs under the MMAs of the next.
//   warp 0: TMA loads, four to six stages of 128-byte slices (three or four of the 256 x 512 tiles; a slice is 64 deep in bf16, 128 in bytes);  warp 1: TMEM, and in the leading CTA the MMAs;
//   the other eight (sixteen): epilogue, a TMEM lane quarter and a part of the columns each, out through staging boxes.
// Both operand majors are read in place through the descriptors: no weight is ever transposed.
//
// Ragged loads.  Rows: a tile is whole or partial, rows behind the load come out as zeros (the epilogue warps write the whole
// tiles of zeros before they look at the first accumulator; the MMAs run two tiles ahead meanwhile).  Contraction over rows (dW): the
// last slice goes up to the load only; the up to 15 rows between the load and the next multiple of the MMA depth are zeroed in
// shared memory by the producer warp before the pair's MMA may read the slice.
//
// Form kInt8: the same slices of 128 bytes hold twice the depth and the pipe is twice as fast, so operands need 64 bytes a clock and SM where
// loads from the L2 reach 67.  E 32, C 4096: h at K 4096 3 000 TOPS (tensor pipe 90 % active), y at K 1024 2 400 (69 %, the results' stores on
// top of the loads); long runs at E 128 2 700 to 2 800 and 2 050 to 2 150.  What a sum stands for is worked out in the epilogue.
// Form kKeep8: h as ever, then g and u block by block from the accumulator into 8 bits (E 128, C 4096, 4096 -> 1024: 7.0 to 7.9 ms, as when they are
// kept in bf16; 6.3 without).  The backward pass takes them into registers, a sector a lane, one step ahead of its use, and forms h again: E 64, C 2560,
// 2048 -> 1000 640 to 680 us, 810 TFLOP/s, where the bf16 form without h takes 580 to 630.  A tile takes 27 000 clocks there, its MMAs 16 400 of them at the
// full rate: for the rest they wait for operands (the tensor pipe is active in 58 % of the clocks), though the epilogue, 18 000 clocks, is hidden.  The ring is
// a stage shorter than in bf16, and kept values pass the L2 as 32 sectors in 32 lines a load.
#pragma once
#include "expert.cuh"
#include "int8.cuh"

namespace msr {

// ---- cta_group::2 wrappers -----------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t map_to_rank(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
// Arrival that orders nothing: a release at cluster scope waits for every global store of the warp (4 500 clocks an epilogue).
// Enough where what the other side waits for has already been consumed into registers.
__device__ __forceinline__ void mbar_arrive_cluster_relaxed(uint32_t addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* bar, uint32_t phase, uint32_t limit = 1u << 22) {
  for (uint32_t it = 0; it < limit; ++it) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(phase) : "memory");
    if (ok) return true;
    if (it > 64) __nanosleep(32);
  }
  return false;
}
__device__ __forceinline__ void prefetch_tmap(const CUtensorMap* tm) { asm volatile("prefetch.tensormap [%0];" ::"l"(tm) : "memory"); }
// loads into this CTA's shared memory that complete on a barrier of either CTA of the pair
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
               ::"r"(dst), "l"(tm), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
               ::"r"(dst), "l"(tm), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z) : "memory");
}
// the same for [E][rows][columns] seen as [E][column chunks of 64][rows][64]: several chunks come in with one copy
__device__ __forceinline__ void tma_load_4d_pair(uint32_t dst, const CUtensorMap* tm, int row, int chunk, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(tm), "r"(bar), "r"(0), "r"(row), "r"(chunk), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* tm, int row, int chunk, int z, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(tm), "r"(smem_u32(bar)), "r"(0), "r"(row), "r"(chunk), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* tm, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(tm), "r"(src), "r"(x), "r"(y),
               "r"(z) : "memory");
}
__device__ __forceinline__ void umma_bf16_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_i8_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// What differs between the operands' types in an instruction descriptor: bf16 x bf16 -> fp32, or signed bytes -> 32-bit integers.
__host__ __device__ constexpr uint32_t idesc_types(int form) { return (form == kInt8 ? 2u << 4 : 1u << 4) | (1u << 7) | (1u << 10); }
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar) {     // arrives on the same barrier of both CTAs
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"((uint16_t)3) : "memory");
}

// ---- the kernel ----------------------------------------------------------------------------------------------------
constexpr int kXTile = 256, kXBK = 64;
// The tensor pipe cuts what an MMA adds off at 24 bits of the accumulator (products two bits further down) instead of rounding it, so a
// long sum of one sign shrinks, by 1.4e-5 over 4096 rows and 6e-9 of itself a row in the end: too much for dW, whose result is fp32.  There an accumulator
// takes kXPartKb slices at a time, and the epilogue adds these parts up in registers, with rounding, while the next part runs in the
// other accumulator.  Error of dW on positive rows, whatever their number: 3.8e-7 (8 slices 9.0e-7, plain fp32 sums 2.6e-7 over 512
// rows, 9.7e-7 over 4096).  What it costs: E 64, C 2560, 2048 x 2048 1 290 us, 8 slices 1 265; undivided sums in 256 x 512 tiles, for
// which the registers do not reach, 1 165.
constexpr int kXPartKb = 4, kXPartRows = kXPartKb * kXBK;
// W: column tiles of a pair at a time (1: 256 x 256, two accumulators in turn; 2: 256 x 512)
__host__ __device__ constexpr int x_stage_bytes(int w) { return 16384 * (1 + w); }
// Epilogue warps: two for each of the four TMEM lane quarters; four in the backward of the activation, whose epilogue (two
// operands in, two results out, an exponential and a quotient each) is what bounds it up to K of a few thousand.
__host__ __device__ constexpr int x_epi_warps(int epi) { return epi == kEpiDact ? 16 : 8; }
__host__ __device__ constexpr int x_threads(int epi) { return 64 + 32 * x_epi_warps(epi); }
// Staging of an epilogue warp: boxes of 32 rows of 128 bytes (64 bytes in the backward), one for dW, a pair for the others, three for the
// backward of kept activations (its third result, held in registers until a box was free, made it spill: 35 000 clocks a tile instead of 18 000).
__host__ __device__ constexpr int x_box_bytes(int epi, int form) { return epi == kEpiDact && form == kKeep8 ? 6144 : epi == kEpiDw || epi == kEpiDact ? 4096 : 8192; }
__host__ __device__ constexpr int x_stages(int epi, int w, int form) { return (w == 2 ? 3 : 5) + (epi == kEpiDw ? 1 : 0) - (epi == kEpiDact && form == kKeep8 ? 1 : 0); }
__host__ __device__ constexpr int x_smem(int epi, int w, int form) {
  return x_stages(epi, w, form) * x_stage_bytes(w) + x_epi_warps(epi) * x_box_bytes(epi, form) + 1024;
}

struct XSmem {
  uint64_t full[6], empty[6], acc_full[2], acc_empty[2], tail, tail_peer[6];
  uint32_t tmem;
  int failed;
  int rows[kMaxE], first[kMaxE + 1];     // rows in use; tiles before each expert
  int start;                             // expert of the pair's first tile
};

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&u)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]) : "r"(taddr));
  tmem_ld_wait();
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&h);
}

__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}

struct XTile { int e, m, n, subs, rows; };     // expert, tile row, first column tile and their number, rows of the expert in use

// Walks the tiles t, t + step, ... (t only grows, so the expert is found by stepping on from the last one).
template <int W>
struct XWalk {
  const XSmem& sm; const ExpertArgs& a; int ntn, ntw; int t, step, e;
  __device__ XWalk(const XSmem& s, const ExpertArgs& args, int ntn_, int t0, int step_)
      : sm(s), a(args), ntn(ntn_), ntw((ntn_ + W - 1) / W), t(t0), step(step_), e(s.start) {}
  __device__ bool next(XTile& x) {
    if (t >= sm.first[a.E]) return false;
    while (t >= sm.first[e + 1]) ++e;
    const int l = t - sm.first[e];
    x.e = e; x.m = l / ntw; x.n = (l - x.m * ntw) * W; x.subs = min(W, ntn - x.n); x.rows = sm.rows[e];
    t += step;
    return true;
  }
};

// Rows in use and tile counts of every expert, by one warp; `per` = tiles of an expert with rows r.  start: the expert of tile t0 (stepping there from
// the first expert costs a microsecond where few of many experts have rows).
template <typename F>
__device__ __forceinline__ void expert_prefix(const ExpertArgs& a, int* rows, int* first, int t0, int* start, F per) {
  const int lane = threadIdx.x & 31;
  int mine[kMaxE / 32], sum = 0;
#pragma unroll
  for (int i = 0; i < kMaxE / 32; ++i) {
    const int e = lane * (kMaxE / 32) + i;
    const int r = e < a.E ? expert_rows(a, e) : 0;
    if (e < a.E) rows[e] = r;
    mine[i] = e < a.E ? per(r) : 0;
    sum += mine[i];
  }
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  int run = incl - sum, before = 0;
#pragma unroll
  for (int i = 0; i < kMaxE / 32; ++i) {
    const int e = lane * (kMaxE / 32) + i;
    if (e <= a.E) first[e] = run;
    run += mine[i];
    before += e < a.E && run <= t0;
  }
  before = __reduce_add_sync(0xffffffffu, before);
  if (lane == 0) *start = before;
  if (lane == 31 && a.E == kMaxE) first[kMaxE] = run;
}

// EPI as in expert.cuh.  B_MN: B is stored with its columns contiguous.  dW: both operands run along the rows.
// Maps: tA; tB0 / tB1 = B of the leading / the other CTA (gate and up columns in the gated form, else the same).
// Add: dW is added to what is there.  W = 2 with dW: one sum whatever its length, for capacities up to kXPartRows.
// tO0: y or h; tO1 / tO2: g / u kept (gated).  out: y, h, dpre or dW; pre_out: [g | u] kept or null, h or null in the backward of kKeep8;
// pre_in: [g | u] (backward of kBf16).
template <int EPI, bool B_MN, int W, bool Add = false, int Form = kBf16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(x_threads(EPI))
expert_tc_kernel(const __grid_constant__ CUtensorMap tA, const __grid_constant__ CUtensorMap tB0, const __grid_constant__ CUtensorMap tB1,
                 const __grid_constant__ CUtensorMap tO0, const __grid_constant__ CUtensorMap tO1, const __grid_constant__ CUtensorMap tO2,
                 char* __restrict__ out, char* __restrict__ pre_out, const char* __restrict__ pre_in, ExpertArgs a, unsigned* error_flag) {
  constexpr bool kDw = EPI == kEpiDw, kA_MN = kDw, kParts = kDw && W == 1;
  constexpr int kEpiWarps = x_epi_warps(EPI), kBK = Form == kInt8 ? 2 * kXBK : kXBK;      // depth of a slice: 128 bytes
  constexpr int kStages = x_stages(EPI, W, Form), kStageBytes = x_stage_bytes(W);
  constexpr int kTileN = EPI == kEpiGlu ? 128 : kXTile;               // output columns of a tile
  extern __shared__ unsigned char xsm_raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(xsm_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ XSmem sm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_rank();
  const int ntn = (a.N + kTileN - 1) / kTileN, ntm_dw = (a.M + kXTile - 1) / kXTile;

  if (threadIdx.x == 0) {
    prefetch_tmap(&tA); prefetch_tmap(rank ? &tB1 : &tB0);
    for (int s = 0; s < kStages; ++s) { mbar_init(&sm.full[s], 1); mbar_init(&sm.empty[s], 1); mbar_init(&sm.tail_peer[s], 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(&sm.acc_full[b], 1); mbar_init(&sm.acc_empty[b], 2 * kEpiWarps); }
    mbar_init(&sm.tail, 1);
    sm.failed = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (warp == 2)
    expert_prefix(a, sm.rows, sm.first, blockIdx.x >> 1, &sm.start, [&](int r) { return (kDw ? ntm_dw : (r + kXTile - 1) / kXTile) * ((ntn + W - 1) / W); });
  tc_fence_before();
  __syncwarp();
  cluster_sync();                                       // barriers of both CTAs are ready, shared memory written above is seen
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (warp == 0) {
    // ---- producer ----------------------------------------------------------------------------------------------
    XWalk<W> walk(sm, a, ntn, pair, pairs);
    XTile x;
    int it = 0; uint32_t tail_phase = 0, peer_phase = 0; bool ok = true;      // peer_phase: bit s, parity to wait for at tail_peer[s]
    const uint32_t full0 = map_to_rank(smem_u32(&sm.full[0]), 0), tail_peer0 = map_to_rank(smem_u32(&sm.tail_peer[0]), 0);
    const CUtensorMap* tB = rank ? &tB1 : &tB0;
    while (ok && walk.next(x)) {
      const int K = kDw ? x.rows : a.K;
      const int nkb = (K + kBK - 1) / kBK;
      const int ax = x.m * kXTile + 128 * rank;
      const int bx = EPI == kEpiGlu ? x.n * 128 : x.n * kXTile + 128 * rank;
      const uint32_t bytes = 16384u * (uint32_t)(1 + x.subs);
      for (int kb = 0; kb < nkb && ok; ++kb, ++it) {
        const int s = it % kStages;
        const uint32_t ph = (uint32_t)((it / kStages) & 1);
        const uint32_t sa = smem_u32(base) + (uint32_t)(s * kStageBytes), sb = sa + 16384;
        const uint32_t full = full0 + 8u * (uint32_t)s;
        const int k0 = kb * kBK;
        const bool masked = kDw && kb == nkb - 1 && (K & 15);          // the load ends inside an MMA's depth
        int good = 1;
        if (lane == 0) {
          if (it >= kStages) good = mbar_wait_bounded(&sm.empty[s], ph ^ 1);
          if (good) {
            // the leading CTA's barrier counts both CTAs' copies.  A remote arrival per slice instead (each CTA announcing its own
            // half) held the whole pipeline at 0.74 us a slice: 743 TFLOP/s where this form gave 1 372.
            if (masked) mbar_expect_tx(&sm.tail, bytes);
            else if (rank == 0) mbar_expect_tx(&sm.full[s], 2 * bytes);
            auto put = [&](uint32_t dst, const CUtensorMap* tm, int xx, int yy) {
              if (masked) tma_load_3d(dst, tm, xx, yy, x.e, &sm.tail);
              else tma_load_3d_pair(dst, tm, xx, yy, x.e, full);
            };
            // columns contiguous: two 64-column chunks, with one copy where the width allows such a map (one 16 KB copy
            // instead of two of 8 KB: dW at E 16, C 4096, 2048 x 2048 went from 1 110 to 1 248 TFLOP/s)
            auto put_mn = [&](uint32_t dst, const CUtensorMap* tm, int xx, int chunks) {
              if (!chunks) { put(dst, tm, xx, k0); put(dst + 8192, tm, xx + 64, k0); }
              else if (masked) tma_load_4d(dst, tm, k0, xx >> 6, x.e, &sm.tail);
              else tma_load_4d_pair(dst, tm, k0, xx >> 6, x.e, full);
            };
            if (kA_MN) put_mn(sa, &tA, ax, a.a_chunks); else put(sa, &tA, k0, ax);
#pragma unroll
            for (int h = 0; h < W; ++h)
              if (h < x.subs) {
                const int bh = bx + h * (EPI == kEpiGlu ? 128 : kXTile);
                if (B_MN) put_mn(sb + h * 16384, tB, bh, a.b_chunks); else put(sb + h * 16384, tB, k0, bh);
              }
          }
        }
        if (kDw && masked) {
          // this CTA's copies land on its own barrier; rows from the load to the next multiple of 16 become zero
          good = __shfl_sync(0xffffffffu, good, 0);
          if (good) good = mbar_wait_warp(&sm.tail, tail_phase);
          tail_phase ^= 1;
          if (good) {
            const int r0 = K - k0, r1 = (r0 + 15) & ~15;               // a row is 128 bytes of a box, whatever the swizzle
            unsigned char* st = base + (size_t)s * kStageBytes;
            const int per_box = (r1 - r0) * 8;
            for (int i = lane; i < 2 * (1 + x.subs) * per_box; i += 32)
              *reinterpret_cast<uint4*>(st + (i / per_box) * 8192 + r0 * 128 + (i % per_box) * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async();
            __syncwarp();
            // The other CTA reports to the leading one, which then releases the slice to the MMA.  One barrier a stage: the other CTA
            // may be several masked slices ahead, and reuses a stage only after the MMA has read it.
            if (rank == 1) { if (lane == 0) mbar_arrive_cluster(tail_peer0 + 8u * (uint32_t)s); }
            else {
              good = __all_sync(0xffffffffu, mbar_wait_cluster(&sm.tail_peer[s], (peer_phase >> s) & 1));
              peer_phase ^= 1u << s;
              if (good && lane == 0) mbar_arrive(&sm.full[s]);
            }
          }
        }
        ok = __shfl_sync(0xffffffffu, good, 0) != 0;
      }
    }
    if (!ok && lane == 0) sm.failed = 1;
  } else if (warp == 1 && rank == 0) {
    // ---- MMA issuer of the pair --------------------------------------------------------------------------------------
    // The tensor pipe holds little beyond the MMA it runs, so every clock between a slice's last MMA and the next one's
    // first shows.  The whole warp walks and waits (its values stay in uniform registers, where the MMA wants them), one
    // elected lane issues a slice's four MMAs and its commit in a row.
    const uint32_t idesc = idesc_types(Form) | (kA_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) |
                           ((uint32_t)(kXTile >> 3) << 17) | ((uint32_t)(kXTile >> 4) << 24);
    constexpr uint32_t kAStep = kA_MN ? 128 : 2, kBStep = B_MN ? 128 : 2;      // an MMA's depth (32 bytes) in descriptor units of 16 bytes
    constexpr int kDepth = kBK / 4;
    auto mma = [](uint32_t d, uint64_t ad, uint64_t bd, uint32_t id, uint32_t add) {
      if constexpr (Form == kInt8) umma_i8_pair(d, ad, bd, id, add); else umma_bf16_pair(d, ad, bd, id, add);
    };
    const uint64_t adesc0 = kA_MN ? smem_desc_mn128(smem_u32(base), 8192u) : smem_desc_k128(smem_u32(base));
    const uint64_t bdesc0 = B_MN ? smem_desc_mn128(smem_u32(base) + 16384, 8192u) : smem_desc_k128(smem_u32(base) + 16384);
    XWalk<W> walk(sm, a, ntn, pair, pairs);
    XTile x;
    uint32_t acc_ph = 3, full_ph = 0;                   // bit b: parity to wait for at accumulator b; parity of the ring
    int s0 = 0, turn = 0; bool ok = true;               // s0: ring position of slice kb
    while (ok && walk.next(x)) {
      const int K = kDw ? x.rows : a.K;
      const int nkb = (K + kBK - 1) / kBK;
      if (nkb == 0) continue;
      // With two column tiles the first and the last slices are multiplied group-wise, the first column tile ahead of the
      // second: its accumulator is complete (and free again) that much earlier, which is what hides the epilogues.
      const int group = x.subs == 2 ? kStages : 1;
      int begin = 0, end = kParts ? min(nkb, kXPartKb) : nkb;          // slices of the present sum
      for (int kb = 0; kb < nkb && ok;) {
        if (kParts && kb == end) { begin = end; end = min(nkb, end + kXPartKb); ++turn; }
        const int n = (kb == begin || end - kb <= group) ? min(group, end - kb) : 1;
        int s = s0;
#pragma unroll
        for (int h = 0; h < W; ++h) {
          if (h >= x.subs) break;
          const uint32_t buf = W == 2 ? h : turn & 1;
          const uint32_t acc = tmem + buf * 256;
          if (kb == begin) { ok = ok && mbar_wait_warp(&sm.acc_empty[buf], (acc_ph >> buf) & 1); acc_ph ^= 1u << buf; }
          s = s0;
          uint32_t ph = full_ph;
          for (int j = 0; j < n; ++j) {
            if (h == 0) ok = ok && mbar_wait_warp(&sm.full[s], ph);
            if (!ok) break;
            tc_fence_after();
            const uint64_t ad = adesc0 + (uint64_t)(s * (kStageBytes / 16)), bd = bdesc0 + (uint64_t)(s * (kStageBytes / 16) + h * 1024);
            const int left = K - (kb + j) * kBK;
            if (elect_one()) {
              mma(acc, ad, bd, idesc, kb + j > begin ? 1u : 0u);
              if (left > kDepth) mma(acc, ad + kAStep, bd + kBStep, idesc, 1u);
              if (left > 2 * kDepth) mma(acc, ad + 2 * kAStep, bd + 2 * kBStep, idesc, 1u);
              if (left > 3 * kDepth) mma(acc, ad + 3 * kAStep, bd + 3 * kBStep, idesc, 1u);
              if (h == x.subs - 1) umma_commit_pair(&sm.empty[s]);
              if (kb + j == end - 1) umma_commit_pair(&sm.acc_full[buf]);
            }
            __syncwarp();
            if (++s == kStages) { s = 0; ph ^= 1; }
          }
          if (h == x.subs - 1) full_ph = ph;
        }
        s0 = s; kb += n;
      }
      ++turn;
    }
    if (!ok && lane == 0) sm.failed = 1;
  } else if (warp >= 2) {
    // ---- epilogue ------------------------------------------------------------------------------------------------------
    const int q = warp & 3, part = (warp - 2) >> 2;     // TMEM lanes this warp may read; its part of a tile's columns
    if constexpr (!kDw) {
      const int worker = (blockIdx.x * kEpiWarps + warp - 2) * 32 + lane, workers = gridDim.x * kEpiWarps * 32;
      expert_zero_behind(a, sm.rows, out, 2 * (size_t)(EPI == kEpiDact ? 2 * a.N : a.N), kXTile, worker, workers);
      if (EPI == kEpiGlu && pre_out) expert_zero_behind(a, sm.rows, pre_out, 4 * (size_t)a.N, kXTile, worker, workers);
      if (EPI == kEpiDact && Form == kKeep8 && pre_out) expert_zero_behind(a, sm.rows, pre_out, 2 * (size_t)a.N, kXTile, worker, workers);
    }
    unsigned char* stage = base + kStages * kStageBytes + (size_t)(warp - 2) * x_box_bytes(EPI, Form);
    const uint32_t acc_empty0 = map_to_rank(smem_u32(&sm.acc_empty[0]), 0);
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    // A lane computes 128 bytes of its own row; a box of 32 such rows turns them into whole lines for memory.  16-byte chunk c
    // of row r sits at c ^ (r & 7) (the copy engine's 128-byte swizzle), which spreads both sides over the banks.
    // y and h leave through tile stores, two boxes in turn: 1 331 TFLOP/s in a long run at E 128, C 4096, 4096 -> 2048 against
    // 1 260 with stores by the warp (less energy, so a higher clock under the power cap).  dW and the backward of the activation
    // leave through the warp's own stores: their boxes come faster than the copy engine, busy with operands, takes them.
    constexpr int kRow = EPI == kEpiDact ? 64 : 128, kPer = kRow / 16, kRows = 32 / kPer;      // bytes of a box row; chunks; rows a warp moves at once
    auto swz = [](int r) { return kRow == 128 ? r & 7 : (r >> 1) & 3; };
    auto to_box = [&](unsigned char* box, int i, uint4 v) { *reinterpret_cast<uint4*>(box + lane * kRow + ((i ^ swz(lane)) << 4)) = v; };
    auto put16 = [&](unsigned char* box, int i, const uint32_t (&u)[16], bool keep) {      // the i-th 16 values of the row, as bf16
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = keep ? pack_bf16(__uint_as_float(u[2 * j]), __uint_as_float(u[2 * j + 1])) : 0u;
      to_box(box, 2 * i, make_uint4(w[0], w[1], w[2], w[3]));
      to_box(box, 2 * i + 1, make_uint4(w[4], w[5], w[6], w[7]));
    };
    // Box -> memory: rows and bytes beyond the tensor are left out.  Add: reductions at the L2, one per entry and call, so nothing
    // depends on an order; rounded to nearest, subnormal results may come out as zeros.  (E 64, C 2560, 2048 x 2048: 1 400 us;
    // loads, sums and stores by the warp 1 610.)
    auto box_out = [&](const unsigned char* box, char* dst, size_t stride, int rows, int bytes) {
      const int c = (int)((unsigned)lane % kPer), r0 = (int)((unsigned)lane / kPer);
      if (c * 16 >= bytes) rows = 0;
      dst += r0 * stride + c * 16;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int r = i * kRows + r0;
        const uint4 v = *reinterpret_cast<const uint4*>(box + r * kRow + ((c ^ swz(r)) << 4));
        if (r < rows) {
          if constexpr (Add)
            asm volatile("red.relaxed.gpu.global.v4.f32.add [%0], {%1, %2, %3, %4};" ::"l"(dst), "f"(__uint_as_float(v.x)), "f"(__uint_as_float(v.y)),
                         "f"(__uint_as_float(v.z)), "f"(__uint_as_float(v.w)) : "memory");
          else *reinterpret_cast<uint4*>(dst) = v;
        }
        dst += kRows * stride;
      }
      __syncwarp();
    };
    int box = 0;
    auto next_box = [&]() -> unsigned char* {                          // for tile stores: the box the store before last has left
      if (lane == 0 && box >= 2) bulk_wait_read<1>();
      __syncwarp();
      return stage + (box & 1) * 4096;
    };
    auto box_store = [&](const CUtensorMap* tm, int xx, int yy, int zz, bool in) {
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        if (in) tma_store_3d(tm, xx, yy, zz, smem_u32(stage + (box & 1) * 4096));
        bulk_commit();
      }
      ++box;
    };
    // backward: 32 columns of g and of u into the pair of boxes, 16-byte copies that do not pass the copy engine either
    auto fetch = [&](size_t row0, int rows, int col) {
      const int c = lane % kPer;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int r = i * kRows + lane / kPer;
        const bool in = r < rows && col + c * 8 < a.N;
        const char* g = in ? pre_in + ((row0 + r) * 2 * a.N + col + c * 8) * 2 : pre_in;     // out of the tensor: zeros, nothing is read
        const uint32_t d = smem_u32(stage + r * kRow + ((c ^ swz(r)) << 4));
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(g), "r"(in ? 16 : 0) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d + 32 * kRow), "l"(g + (size_t)a.N * 2), "r"(in ? 16 : 0) : "memory");
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    XWalk<W> walk(sm, a, ntn, pair, pairs);
    XTile x;
    uint32_t acc_ph = 0;                                // bit b: parity to wait for at accumulator b
    int turn = 0; bool ok = true;
    while (ok && walk.next(x)) {
      const int nkb = ((kDw ? x.rows : a.K) + kBK - 1) / kBK;
      const int y0 = x.m * kXTile + 128 * rank + 32 * q;              // first row of this warp
      const int rows = min(32, (kDw ? a.M : a.C) - y0);               // rows of the tensor; may be none
      const size_t row0 = (size_t)x.e * (kDw ? a.M : a.C) + y0;
      constexpr int kTileCols = EPI == kEpiGlu ? 128 : kXTile, kCols = kTileCols / (kEpiWarps / 4);     // columns of this warp
      if constexpr (kParts) {
        const int col0 = x.n * kTileCols + part * kCols;
        char* dst = out + (row0 * a.N + col0) * 4;
        float2 sum[kCols / 2];
#pragma unroll
        for (int i = 0; i < kCols / 2; ++i) sum[i] = both(0.f);
        for (int kb = 0; kb < nkb; kb += kXPartKb, ++turn) {
          const int buf = turn & 1;
          const uint32_t acc = tmem + lanes + (uint32_t)(buf * 256 + part * kCols);
          ok = mbar_wait_warp(&sm.acc_full[buf], (acc_ph >> buf) & 1);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int c0 = 0; c0 < kCols; c0 += 32) {
            uint32_t u[2][16];
            tmem_ld16_issue(acc + c0, u[0]); tmem_ld16_issue(acc + c0 + 16, u[1]);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              uint32_t &lo = u[i >> 3][(i & 7) * 2], &hi = u[i >> 3][(i & 7) * 2 + 1];
              asm volatile("" : "+r"(lo), "+r"(hi));                   // the sum stays behind the wait
              sum[c0 / 2 + i] = add2(sum[c0 / 2 + i], make_float2(__uint_as_float(lo), __uint_as_float(hi)));
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster_relaxed(acc_empty0 + 8u * (uint32_t)buf);
          acc_ph ^= 1u << buf;
        }
        if (!ok || (Add && nkb == 0)) continue;                        // an expert without rows adds nothing
#pragma unroll
        for (int c0 = 0; c0 < kCols; c0 += 32) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 p0 = sum[c0 / 2 + 2 * i], p1 = sum[c0 / 2 + 2 * i + 1];
            to_box(stage, i, make_uint4(__float_as_uint(p0.x), __float_as_uint(p0.y), __float_as_uint(p1.x), __float_as_uint(p1.y)));
          }
          box_out(stage, dst + c0 * 4, (size_t)a.N * 4, rows, (a.N - col0 - c0) * 4);
        }
      } else   // one sum per column tile
      for (int sub = 0; sub < x.subs && ok; ++sub) {
        const int buf = W == 2 ? sub : turn & 1;
        const int col0 = (x.n + sub) * kTileCols + part * kCols;
        const uint32_t acc = tmem + lanes + (uint32_t)(buf * 256 + part * kCols);
        const bool keep_row = kDw || y0 + lane < x.rows;              // rows behind the load come out as zeros
        float row_scale = 0.f;
        if (Form == kInt8 && keep_row) row_scale = __ldg(a.x_scale + row0 + lane);
        // whether any scale of the warp's rows and columns lies far from 1; asked for ahead of the accumulator
        bool far = false;
        if constexpr (Form == kInt8) {
          constexpr int kHalf = EPI == kEpiGlu ? 16 : 32;             // lanes for the columns, four each; gated: g's, then u's
          static_assert(kCols == 4 * kHalf, "a lane looks at four columns");
          const int col = col0 + (lane % kHalf) * 4;
          const float* of = a.w_scale + (size_t)x.e * (EPI == kEpiGlu ? 2 * a.N : a.N) + (lane / kHalf) * (size_t)a.N;
          const bool mine = far8(row_scale) || (col < a.N && far8(__ldg(reinterpret_cast<const float4*>(of + col))));
          far = __any_sync(0xffffffffu, mine);
        }
        // 16 columns from `col` on (of N; the weights' column `of` has column 0) as products of fp32 values: an integer is exact up to 2^24 and
        // else rounded once
        auto unscale = [&](uint32_t (&u)[16], int col, const float* of, auto product) {
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const float4 c = col + i < a.N ? __ldg(reinterpret_cast<const float4*>(of + col + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
            u[i] = product(u[i], c.x); u[i + 1] = product(u[i + 1], c.y); u[i + 2] = product(u[i + 2], c.z); u[i + 3] = product(u[i + 3], c.w);
          }
        };
        auto near_1 = [&](uint32_t u, float c) { return __float_as_uint((float)(int)u * (row_scale * c)); };
        auto anywhere = [&](uint32_t u, float c) { return __float_as_uint(value8((int)u, row_scale, c)); };
        uint32_t kg[8] = {}, ku[8] = {};                               // kKeep8: 32 columns of the row's g and u, and their steps
        float sg = 0.f, su = 0.f;
        auto fetch8 = [&](int col) {
          if (keep_row && col < a.N) {
            const int fp = keep_width(a.N), blocks = fp / kKeepBlock;
            const int8_t* g = a.keep + (row0 + lane) * 2 * fp + col;
            auto load = [](uint32_t (&w)[8], const int8_t* p) {
              asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]),
                           "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
            };
            load(kg, g); load(ku, g + fp);
            const float* st8 = a.keep_scale + ((size_t)x.e * 2 * blocks + col / kKeepBlock) * a.C + y0 + lane;
            sg = __ldg(st8); su = __ldg(st8 + (size_t)blocks * a.C);
          } else {                                                     // rows behind the load, columns behind d_ff: g = u = 0
            sg = su = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) kg[j] = ku[j] = 0;
          }
          __syncwarp();
        };
        if constexpr (EPI == kEpiDact) { if constexpr (Form == kKeep8) fetch8(col0); else fetch(row0, rows, col0); }
        if (nkb > 0) {
          ok = mbar_wait_warp(&sm.acc_full[buf], (acc_ph >> buf) & 1);
          if (!ok) break;
          tc_fence_after();
        }
        if constexpr (kDw) {
#pragma unroll 1
          for (int c0 = 0; c0 < kCols; c0 += 32) {
            uint32_t u[2][16];
            if (nkb > 0) {
              tmem_ld16_issue(acc + c0, u[0]); tmem_ld16_issue(acc + c0 + 16, u[1]);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) u[0][i] = u[1][i] = 0;
            }
            if (Add && nkb == 0) continue;                             // an expert without rows adds nothing
#pragma unroll
            for (int i = 0; i < 8; ++i)
              to_box(stage, i, make_uint4(u[i >> 2][(i & 3) * 4], u[i >> 2][(i & 3) * 4 + 1], u[i >> 2][(i & 3) * 4 + 2], u[i >> 2][(i & 3) * 4 + 3]));
            box_out(stage, out + (row0 * a.N + col0 + c0) * 4, (size_t)a.N * 4, rows, (a.N - col0 - c0) * 4);
          }
        } else if constexpr (EPI == kEpiPlain) {
#pragma unroll 1
          for (int c0 = 0; c0 < kCols; c0 += 64) {
            if (far) {
              unsigned char* to = next_box();
#pragma unroll 1
              for (int i = 0; i < 4; ++i) {
                uint32_t u[16];
                tmem_ld16_issue(acc + c0 + 16 * i, u);
                tmem_ld_wait();
                unscale(u, col0 + c0 + 16 * i, a.w_scale + (size_t)x.e * a.N, anywhere);
                put16(to, i, u, keep_row);
              }
            } else {
              uint32_t u[4][16];
#pragma unroll
              for (int i = 0; i < 4; ++i) tmem_ld16_issue(acc + c0 + 16 * i, u[i]);
              tmem_ld_wait();
              unsigned char* to = next_box();
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                if constexpr (Form == kInt8) unscale(u[i], col0 + c0 + 16 * i, a.w_scale + (size_t)x.e * a.N, near_1);
                put16(to, i, u[i], keep_row);
              }
            }
            box_store(&tO0, col0 + c0, y0, x.e, rows > 0 && col0 + c0 < a.N);
          }
        } else if constexpr (EPI == kEpiGlu) {
          // h, then g and u if they are kept: the accumulator is read again for each rather than held in registers
#pragma unroll 1
          for (int what = 0; what < (Form == kBf16 && pre_out ? 3 : 1); ++what) {
            unsigned char* to = next_box();
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
              uint32_t g[16], u[16];
              tmem_ld16_issue(acc + 16 * i + (what == 2 ? 128 : 0), g);
              if (what == 0) tmem_ld16_issue(acc + 128 + 16 * i, u);
              tmem_ld_wait();
              if constexpr (Form == kInt8) {
                const float* of = a.w_scale + (size_t)x.e * 2 * a.N;
                if (far) { unscale(g, col0 + 16 * i, of, anywhere); unscale(u, col0 + 16 * i, of + a.N, anywhere); }
                else { unscale(g, col0 + 16 * i, of, near_1); unscale(u, col0 + 16 * i, of + a.N, near_1); }
              }
              if (what == 0) {
#pragma unroll
                for (int j = 0; j < 16; ++j) g[j] = __float_as_uint(silu_mul<true>(__uint_as_float(g[j]), __uint_as_float(u[j])));
              }
              put16(to, i, g, keep_row);
            }
            box_store(what == 0 ? &tO0 : what == 1 ? &tO1 : &tO2, col0, y0, x.e, rows > 0 && col0 < a.N);
          }
          if constexpr (Form == kKeep8) {
            // A lane's 32 columns of its row are a block: 32 bytes, a sector of memory, and the lanes' scales a line.  Columns behind d_ff are
            // zero in the accumulator (the copies filled the weights up), rows behind the load are left out.
            const int fp = keep_width(a.N), blocks = fp / kKeepBlock;
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
              const int half = i >> 1, col = col0 + (i & 1) * kKeepBlock;
              uint32_t u[2][16];
              float m = 0.f;
              tmem_ld16_issue(acc + half * 128 + (i & 1) * kKeepBlock, u[0]);
              tmem_ld16_issue(acc + half * 128 + (i & 1) * kKeepBlock + 16, u[1]);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j) m = max_abs(m, __uint_as_float(u[0][j]), __uint_as_float(u[1][j]));
              if (keep_row && col < a.N) {
                const Step8 st8 = step8(__float_as_uint(m));
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  const uint32_t(&v)[16] = u[j >> 2];
                  const int k = (j & 3) * 4;
                  w[j] = pack8(round8(__uint_as_float(v[k]), st8.inv), round8(__uint_as_float(v[k + 1]), st8.inv),
                               round8(__uint_as_float(v[k + 2]), st8.inv), round8(__uint_as_float(v[k + 3]), st8.inv));
                  if (!(st8.inv > 0.f)) w[j] = 0;
                }
                int8_t* to = a.keep + ((row0 + lane) * 2 + half) * fp + col;
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                             "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
                a.keep_scale[((size_t)x.e * 2 * blocks + half * blocks + col / kKeepBlock) * a.C + y0 + lane] = st8.scale;
              }
              __syncwarp();
            }
          }
        } else {
          if constexpr (Form == kKeep8) {
            // As below, with g and u from their integers: a lane lays them into its row of the third box, eight of g and of u to 16 bytes, which h =
            // silu(g) u, formed again on the way, then takes over.
#pragma unroll 1
            for (int c0 = 0; c0 < kCols; c0 += 32) {
              unsigned char* row = stage + lane * kRow;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                *reinterpret_cast<uint4*>(row + 64 * kRow + ((i ^ swz(lane)) << 4)) = make_uint4(kg[2 * i], kg[2 * i + 1], ku[2 * i], ku[2 * i + 1]);
              const float2 step_g = both(sg), step_u = both(su);
              if (c0 + 32 < kCols) fetch8(col0 + c0 + 32);             // on its way from here on
#pragma unroll 1
              for (int i = 0; i < 4; ++i) {
                uint32_t u[8], dg[4], du[4], h[4];
                uint4* at = reinterpret_cast<uint4*>(row + ((i ^ swz(lane)) << 4));
                const uint4 kept = at[64 * kRow / 16];
                tmem_ld8(acc + c0 + 8 * i, u);
#pragma unroll
                for (int p = 0; p < 4; ++p) {                          // columns 2 p and 2 p + 1 of the eight, packed
                  const uint32_t gw = (p < 2 ? kept.x : kept.y) ^ 0x80808080u, uw = (p < 2 ? kept.z : kept.w) ^ 0x80808080u;
                  const int b = (p & 1) * 2;
                  const float2 g = mul2(add2(make_float2(byte8_raw(gw, b), byte8_raw(gw, b + 1)), both(-kByte8Zero)), step_g);
                  const float2 up = mul2(add2(make_float2(byte8_raw(uw, b), byte8_raw(uw, b + 1)), both(-kByte8Zero)), step_u);
                  const float2 dh = make_float2(keep_row ? __uint_as_float(u[2 * p]) : 0.f, keep_row ? __uint_as_float(u[2 * p + 1]) : 0.f);
                  float2 t = mul2(g, both(-1.44269504f)), s;           // s = 1 / (1 + 2^t), as sigmoid_f<true>
                  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t.x) : "f"(t.x));
                  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t.y) : "f"(t.y));
                  t = add2(t, both(1.f));
                  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.x) : "f"(t.x));
                  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.y) : "f"(t.y));
                  const float2 gs = mul2(g, s), slope = fma2(g, fma2(s, both(-1.f), both(1.f)), both(1.f));
                  const float2 a = mul2(mul2(mul2(dh, up), s), slope), c = mul2(dh, gs), hv = mul2(gs, up);
                  dg[p] = pack_bf16(a.x, a.y); du[p] = pack_bf16(c.x, c.y);
                  h[p] = pack_bf16(hv.x, hv.y);
                }
                at[0] = make_uint4(dg[0], dg[1], dg[2], dg[3]);
                at[32 * kRow / 16] = make_uint4(du[0], du[1], du[2], du[3]);
                at[64 * kRow / 16] = make_uint4(h[0], h[1], h[2], h[3]);
              }
              char* dst = out + (row0 * 2 * a.N + col0 + c0) * 2;
              const int left = (a.N - col0 - c0) * 2;
              box_out(stage, dst, (size_t)a.N * 4, rows, left);
              box_out(stage + 32 * kRow, dst + (size_t)a.N * 2, (size_t)a.N * 4, rows, left);
              if (pre_out) box_out(stage + 64 * kRow, pre_out + (row0 * a.N + col0 + c0) * 2, (size_t)a.N * 2, rows, left);
            }
          } else {
          // dh in the accumulator; g and u sit in a pair of boxes, which dg and du then leave from
#pragma unroll 1
          for (int c0 = 0; c0 < kCols; c0 += 32) {
            if (c0) fetch(row0, rows, col0 + c0);                      // the first one was asked for ahead of the accumulator
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
            unsigned char* row = stage + lane * kRow;
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
              uint32_t u[8];
              tmem_ld8(acc + c0 + 8 * i, u);
              uint4* pg = reinterpret_cast<uint4*>(row + ((i ^ swz(lane)) << 4));
              uint4* pu = reinterpret_cast<uint4*>(row + 32 * kRow + ((i ^ swz(lane)) << 4));
              float g[8], up[8];
              Vec16<__nv_bfloat16>::unpack(*pg, g); Vec16<__nv_bfloat16>::unpack(*pu, up);
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                float dg, du;
                dact<true>(__uint_as_float(u[j]), g[j], up[j], dg, du);
                g[j] = keep_row ? dg : 0.f; up[j] = keep_row ? du : 0.f;
              }
              Vec16<__nv_bfloat16>::store(reinterpret_cast<__nv_bfloat16*>(pg), g);
              Vec16<__nv_bfloat16>::store(reinterpret_cast<__nv_bfloat16*>(pu), up);
            }
            char* dst = out + (row0 * 2 * a.N + col0 + c0) * 2;
            box_out(stage, dst, (size_t)a.N * 4, rows, (a.N - col0 - c0) * 2);
            box_out(stage + 32 * kRow, dst + (size_t)a.N * 2, (size_t)a.N * 4, rows, (a.N - col0 - c0) * 2);
          }
          }
        }
        if (nkb > 0) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster_relaxed(acc_empty0 + 8u * (uint32_t)buf);
          acc_ph ^= 1u << buf;
        }
      }
      if (!kParts && nkb > 0) ++turn;
    }
    if (EPI == kEpiDact && Form != kKeep8) asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (lane == 0) bulk_wait_all<0>();
    if (!ok && lane == 0) sm.failed = 1;
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && sm.failed) {
    atomicOr(error_flag, 4u);
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // a wait gave up: let the copies that were in flight land
  }
  __syncwarp();
  cluster_sync();                                       // neither CTA leaves while the other may still reach its barriers
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

}  // namespace msr
