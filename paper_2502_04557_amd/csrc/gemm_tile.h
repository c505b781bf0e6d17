// The matrix product of 17 and more rows, one output tile per workgroup: what k_gemm_tile.hip and the grouped products of
// k_experts_tile.hip are made of.
#pragma once
#include "gemm.h"

namespace sprinter {

// bf16-mode GEMM (float16 operands) over a TM x TN output tile, both operands staged in LDS.  Weights and activations are
// stored as operand tiles of 16 rows x 32 k (1 KiB, in the lane order of the matrix instruction), so a tile goes from
// memory to LDS with one global_load_lds of 16 bytes a lane - no registers, no address swizzle - and from LDS into the
// instruction with one conflict-free ds_read_b128.  A ring of S stages of one k tile: at the top of k tile kt the wave waits
// until its own loads of stage kt + 1 have landed (its later ones stay in flight), the barrier makes that true for every
// wave and says that nobody reads stage kt - 1 any more, whose slot takes the loads of stage kt + S - 1.  The fragments of
// kt + 1 are read into a second register set between the matrix instructions of kt.
// The weight fragment is the first operand, so that the accumulator holds four consecutive COLUMNS of one row per lane:
// the epilogue stores 16 bytes of float32 or 8 bytes of an activation operand tile at a time.
// The 256 x 256 tile is four waves of 128 x 128, one per SIMD, whose accumulators are all 256 accumulation registers: a k tile
// costs the LDS 64 KiB of fragment reads and 32 KiB of arriving loads, 768 of the 1024 cycles that its matrix instructions take at
// 128 B a cycle (eight waves of 64 x 128: 96 KiB, as many cycles as the products).  What bounds it (4096 rows): 1150 - 1180 cycles
// per k tile (eight waves: 1310 - 1410) at a clock that the power holds to 1.7 GHz in a loop of this launch and 1.9 - 2.0 in a whole
// prefill; then the epilogue, whose stores (float32) or activations no other wave hides.  In a loop of one launch, eight waves -> four, us:
// FFN-up 2 x 14336 x 4096 746 -> 722, 2 x 11008 x 4096 603 -> 563, 2 x 8192 x 2048 227 -> 229, QKV 12288 x 4096 337 -> 311,
// O-proj 4096 x 4096 113 -> 111, FFN-down 4096 x 14336 373 -> 347 (1.39 PFLOP/s).
// GELU stays on eight waves: one wave per SIMD does not hide its arithmetic (6400 x 1600 at 1811 / 2500 / 4096 rows 55.6 / 60.6 / 106.0 us;
// four waves, the epilogue through LDS as for gate + up, 60.0 / 64.7 / 114.7).
// Also measured: 32 x 32 x 16 instructions (8 - 20 % slower), a fifth stage (no faster), two fragment reads per row tile instead of
// three and a later first one (equal), 256 x 128 tiles of four waves (10 - 20 % slower but where the last round is half empty).
template <int WM, int WN, int MT, int NT, int S>
struct GemmTile {                                       // WM x WN waves, MT x NT operand tiles per wave, S stages
  static constexpr int wm = WM, wn = WN, mt = MT, nt = NT, stages = S, waves = WM * WN;
  static constexpr bool pinned = MT == 8;               // accumulators pinned to accumulation registers (256 x 256: all 256 of a wave)
};
using TileL = GemmTile<2, 2, 8, 8, 4>;                  // 256 x 256, 128 KiB: one workgroup per compute unit
using TileH = GemmTile<2, 2, 8, 4, 4>;                  // 256 x 128, for the last round of the one above
using TileT = GemmTile<2, 2, 4, 8, 4>;                  // 128 x 256, for row blocks of at most 128 rows among those of the first one
using TileQ = GemmTile<2, 2, 2, 8, 4>;                  // 64 x 256, of at most 64
using TileG = GemmTile<4, 2, 4, 8, 4>;                  // 256 x 256 of eight waves, for GELU
using TileM = GemmTile<2, 2, 4, 4, 5>;                  // 128 x 128, 80 KiB: two
using TileS = GemmTile<2, 2, 2, 4, 6>;                  // 64 x 128, 72 KiB: two
using TileX = GemmTile<2, 2, 2, 2, 8>;                  // 64 x 64, 64 KiB: two
using TileN = GemmTile<1, 2, 2, 2, 8>;                  // 32 x 64, 48 KiB: three

// Workgroups go round-robin over the 8 XCDs: each XCD takes a contiguous run of the n_blk workgroups' work.
__device__ __forceinline__ int xcd_run(int id, int n_blk) {
  const int xcd = id & 7, q = n_blk >> 3, rem = n_blk & 7;
  return xcd * q + min(xcd, rem) + (id >> 3);
}

// Row blocks of grouped products: the operand tiles from row tile tile0 on, rows up to `end`; or, with RowsGathered, row i is row
// row_of[i] of a row-major float16 matrix (rows row_bytes apart, whole k tiles).  Four lanes next to each other fetch the 64 bytes of a
// row's k tile (in the lane order of the operand they would be 16 lanes apart: 2002 for 1876 us at 8192 rows of 2 x 14336 x 4096); in LDS
// a row's octets are exchanged by row / 2 % 4, so that the fragment reads stay free of bank conflicts.
struct RowsOfTiles { int tile0, end; };
struct RowsGathered { int tile0, end; const int* row_of; long long row_bytes; };

// Output tile (bm, bn) of share sk of SK; a grouped product's rows are `rows`.
template <typename T, int EPI, typename Rows = Nothing>
__device__ __forceinline__ void gemm_tile(const GemmArgs& a, int x_tiles, int bm, int bn, int sk, int SK, void* lds, const Rows& rows = Rows{}) {
  constexpr bool GROUPED = !std::is_same_v<Rows, Nothing>, GATHER = std::is_same_v<Rows, RowsGathered>;
  constexpr bool DUAL = (EPI == EPI_SWIGLU);
  constexpr int WN = T::wn, MT = T::mt, NT = T::nt, S = T::stages;
  constexpr int TMT = T::wm * MT, TNT = WN * NT, LT = TMT + TNT, PER = LT / T::waves;   // operand tiles per stage, per wave
  constexpr int COLS = DUAL ? NT / 2 : NT;              // output column tiles of a wave (SwiGLU: gate tiles, then up tiles)
  static_assert(LT % T::waves == 0 && NT % 2 == 0 && S >= 4, "");
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  auto& ring = *reinterpret_cast<u32x4(*)[S][LT][64]>(lds);
  const int lane = threadIdx.x & 63, w = wave_index(), wm = w / WN, wn = w % WN;
  const int Kt = a.Kt;
  const void *const w_lo = a.W, *const w_up = a.W2;
  // EPI_PART: the partial product goes to part[share] (summed by the norm that follows)
  const int k0 = (int)((long long)Kt * sk / SK), k1 = (int)((long long)Kt * (sk + 1) / SK);
  // this wave's PER operand tiles of a stage; tiles beyond the buffers are clamped, their products dropped by the epilogue
  const char* src[PER];
  int row0 = bm * TMT;                                  // first row tile
  if constexpr (GROUPED) row0 = rows.tile0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int l = w * PER + i;
    const void* base;
    int tile;
    if (l < TMT) {
      if constexpr (GATHER) {
        src[i] = (const char*)a.X + (long long)rows.row_of[min((row0 + l) * 16 + (lane >> 2), rows.end - 1)] * rows.row_bytes + ((lane & 3) ^ ((lane >> 3) & 3)) * 16;
        continue;
      }
      base = a.X;
      tile = min(row0 + l, x_tiles - 1);
    } else {
      const int j = l - TMT, jw = j / NT, jj = j % NT;
      const bool up = DUAL && jj >= COLS;
      base = up ? w_up : w_lo;
      tile = min((bn * WN + jw) * COLS + (up ? jj - COLS : jj), a.n_tiles - 1);
    }
    src[i] = (const char*)base + (size_t)tile * Kt * 1024 + lane * 16;
  }
  // bytes from a k tile to the next one: 64 of a row, or a whole operand tile
  auto stride = [&](int i) { return (unsigned)(GATHER && w * PER + i < TMT ? 64 : 1024); };
  auto issue = [&](int kt) {                            // (k tiles beyond the share: its last one again, never read)
    const size_t at = (size_t)min(kt, k1 - 1);
    const int slot = (kt - k0) % S;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src[i] + at * stride(i)),
                                       (__attribute__((address_space(3))) void*)&ring[slot][w * PER + i][0], 16, 0, 0);
  };
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = (f32x4){0.f, 0.f, 0.f, 0.f};
  // this lane's 16 bytes of an activation tile in LDS, relative to its own of a weight tile
  const int x_at = GATHER ? (lane & 15) * 4 + ((lane >> 4) ^ ((lane >> 1) & 3)) - lane : 0;
  struct Frag { u32x4 x[MT], w[NT]; };
  auto read = [&](Frag& f, int kt) {
    const u32x4* s = &ring[(kt - k0) % S][0][lane];
#pragma unroll
    for (int j = 0; j < NT; ++j) f.w[j] = s[(TMT + wn * NT + j) * 64];
#pragma unroll
    for (int i = 0; i < MT; ++i) f.x[i] = s[(wm * MT + i) * 64 + x_at];
  };
  auto mul = [&](const Frag& f) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
        acc[i][j] = mfma_f16(__builtin_bit_cast(uint4, f.w[j]), __builtin_bit_cast(uint4, f.x[i]), acc[i][j]);
  };
  auto top = [&](int kt) {
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((S - 3) * PER) : "memory");
    issue(kt + S - 1);
    __builtin_amdgcn_sched_barrier(0);
  };
  // fragment reads of the next k tile between the matrix instructions of this one (left alone, the scheduler sinks the
  // reads to the end of the block)
  auto weave = [&]() {
    constexpr int PACE = MT * NT >= 2 * (MT + NT) ? 2 : 1;
#pragma unroll
    for (int i = 0; i < MT + NT; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, PACE, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, MT * NT, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  int kv_b[EPI == EPI_QKV ? MT : 1], kv_slot[EPI == EPI_QKV ? MT : 1];   // the cache slots of this lane's rows
  if constexpr (EPI == EPI_QKV) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int mc = min((row0 + wm * MT + i) * 16 + (lane & 15), a.rows_live - 1);
      kv_b[i] = a.kv.b[mc]; kv_slot[i] = a.kv.slot[mc];
    }
  }
#pragma unroll
  for (int i = 0; i < S - 1; ++i) issue(k0 + i);
  int n_rows;                                           // only the epilogue needs it
  if constexpr (GROUPED) n_rows = rows.end; else n_rows = *a.n_rows;
  Frag A, B;
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((S - 2) * PER) : "memory");
  __builtin_amdgcn_sched_barrier(0);
  read(A, k0);
  // Pinned accumulators: one wave per SIMD has nobody to hide behind, so the order of a k tile is written out - a fragment read of
  // the next k tile after every second product, a load to LDS after every NT - and the products are in asm, which keeps the
  // accumulators where they are (given the builtins in pieces, the compiler moves them between the register files: 600 moves per two
  // k tiles).  The first s_nop lies between the accumulators' initialisation and their first use.
  auto product = [&](f32x4& c, const u32x4& wf, const u32x4& xf) {
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(wf), "v"(xf));
  };
  auto step = [&](const Frag& f, Frag& nx, int kt) {
    constexpr int RPR = NT == 8 ? 3 : 2, GAP = (NT + RPR - 1) / (RPR + 1);   // fragment reads per row tile, products between them
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier\n\ts_nop 3" ::"n"((S - 3) * PER) : "memory");
    const u32x4* sn = &ring[(kt + 1 - k0) % S][0][lane];
    const size_t at = (size_t)min(kt + S - 1, k1 - 1);
    const int slot = (kt + S - 1 - k0) % S;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        product(acc[i][j], f.w[j], f.x[i]);
        const int r = i * RPR + j / GAP;
        if (j % GAP == GAP - 1 && j / GAP < RPR && r < MT + NT) {
          if (r < NT) nx.w[r] = sn[(TMT + wn * NT + r) * 64];
          else nx.x[r - NT] = sn[(wm * MT + r - NT) * 64 + x_at];
          __builtin_amdgcn_sched_barrier(0);
        }
        if (j == NT - 1) {
#pragma unroll
          for (int q = i * PER / MT; q < (i + 1) * PER / MT; ++q)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src[q] + at * stride(q)),
                                             (__attribute__((address_space(3))) void*)&ring[slot][w * PER + q][0], 16, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
  };
  // The last products are on their way for some cycles more, which the compiler does not know: before anything that may read an
  // accumulator (the end of the loop is such a place).
  auto settle = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  int kt = k0;
  if constexpr (T::pinned) {
    for (; kt + 2 <= k1; kt += 2) {
      step(A, B, kt);
      step(B, A, kt + 1);
      settle();
    }
    if (kt < k1) {
      asm volatile("s_nop 3");
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) product(acc[i][j], A.w[j], A.x[i]);
      settle();
    }
  } else {
    for (; kt + 2 <= k1; kt += 2) {
      top(kt);
      read(B, kt + 1);
      mul(A);
      weave();
      top(kt + 1);
      read(A, kt + 2);
      mul(B);
      weave();
    }
    if (kt < k1) mul(A);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the clamped loads of the last stages still write to LDS
  // lane (lq, l16): row l16 of a row tile, columns 4 lq .. + 3 of a column tile (N is a multiple of 8)
  const int l16 = lane & 15, lq = lane >> 4;
  float* part = (EPI == EPI_PART) ? a.part + (size_t)sk * a.part_stride : nullptr;
  if constexpr (T::pinned && (EPI == EPI_F32 || EPI == EPI_PART || EPI == EPI_RESID)) {
    // float32 rows: 16 rows at a time through a wave's own piece of the ring, so that a store covers 512 bytes of a row (64 bytes of
    // 16 rows each took 10.5 us per workgroup, now 7.5)
    __syncthreads();
    constexpr int LD = NT * 16 + 4, LPR = NT * 4;       // floats per row in LDS, lanes per row
    float* buf = reinterpret_cast<float*>(&ring[0][0][0]) + w * 16 * LD;
    const int c4 = (lane % LPR) * 4, n = (bn * WN + wn) * NT * 16 + c4;
    const bool n_ok = n < a.N;
    f32x4 bias = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (EPI != EPI_PART && a.bias && n_ok) bias = *reinterpret_cast<const f32x4*>(a.bias + n);
    float* __restrict__ dst = (EPI == EPI_PART ? part : a.out_f32) + (n_ok ? n : 0);
    constexpr int RPI = 64 / LPR, NR = 16 / RPI;        // rows per instruction, instructions per row tile
    // EPI_RESID: the rows' own values, requested a row tile ahead (rows beyond the count: the last one again, dropped)
    f32x4 own[2][EPI == EPI_RESID ? NR : 1];
    auto fetch = [&](int i) {
      const int m0 = (row0 + wm * MT + i) * 16;
#pragma unroll
      for (int q = 0; q < NR; ++q) own[i & 1][q] = *reinterpret_cast<const f32x4*>(dst + (size_t)max(min(m0 + q * RPI + lane / LPR, n_rows - 1), 0) * a.ldo);
    };
    if constexpr (EPI == EPI_RESID) fetch(0);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m0 = (row0 + wm * MT + i) * 16;
      if constexpr (EPI == EPI_RESID) if (i + 1 < MT) fetch(i + 1);
#pragma unroll
      for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4*>(buf + l16 * LD + j * 16 + lq * 4) = acc[i][j];
      __builtin_amdgcn_wave_barrier();                  // (LDS operations of one wave complete in order)
#pragma unroll
      for (int q = 0; q < NR; ++q) {
        const int row = q * RPI + lane / LPR, m = m0 + row;
        f32x4 v = *reinterpret_cast<const f32x4*>(buf + row * LD + c4);
        if (EPI == EPI_F32) v += bias;
        if constexpr (EPI == EPI_RESID) v = (own[i & 1][q] + bias) + v;   // the norm's order: row, bias, product
        if (m < n_rows && n_ok) *reinterpret_cast<f32x4*>(dst + (size_t)m * a.ldo) = v;
      }
      __builtin_amdgcn_wave_barrier();
    }
    return;
  }
  if constexpr (T::pinned && EPI == EPI_SWIGLU) {
    // Gate + up: two row tiles at a time into LDS, then one operand tile of the output (16 rows x 32 columns, 8 columns a lane) per
    // round of a loop that stays a loop: written out over the accumulators it is thousands of instructions, run once per workgroup and
    // fetched from L2 (the loop unrolled by 2 or 8: equal).
    __syncthreads();
    constexpr int LD = NT * 16 + 4, RT = 2, OT = COLS / 2;
    float* buf = reinterpret_cast<float*>(&ring[0][0][0]) + w * RT * 16 * LD;
#pragma unroll
    for (int i0 = 0; i0 < MT; i0 += RT) {
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4*>(buf + (i * 16 + l16) * LD + j * 16 + lq * 4) = acc[i0 + i][j];
      __builtin_amdgcn_wave_barrier();                  // (LDS operations of one wave complete in order)
#pragma unroll 1
      for (int q = 0; q < RT * OT; ++q) {
        const int i = q / OT, ct = q % OT, m = (row0 + wm * MT + i0 + i) * 16 + l16, n = (bn * WN + wn) * COLS * 16 + ct * 32 + lq * 8;
        const float* p = buf + (i * 16 + l16) * LD + ct * 32 + lq * 8;
        float c[8], o[8];
        *reinterpret_cast<f32x4*>(&c[0]) = *reinterpret_cast<const f32x4*>(p);
        *reinterpret_cast<f32x4*>(&c[4]) = *reinterpret_cast<const f32x4*>(p + 4);
        // (the columns behind N of a grouped product's last k tile are its own to clear: rows change their expert from call to call)
        const bool ok = m < n_rows && n < (GROUPED ? round_up(a.N, 32) : a.N);
        float u[8];
        *reinterpret_cast<f32x4*>(&u[0]) = *reinterpret_cast<const f32x4*>(p + COLS * 16);
        *reinterpret_cast<f32x4*>(&u[4]) = *reinterpret_cast<const f32x4*>(p + COLS * 16 + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = GROUPED && n >= a.N ? 0.f : silu(c[e]) * u[e];
        if (ok)
          *reinterpret_cast<uint4*>((bf16_t*)a.out_act + act_idx<bf16_t>(m, n, a.out_K)) =
              make_uint4(pk_f16(o[0], o[1]), pk_f16(o[2], o[3]), pk_f16(o[4], o[5]), pk_f16(o[6], o[7]));
      }
      __builtin_amdgcn_wave_barrier();
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < COLS; ++j) {
    const int n = ((bn * WN + wn) * COLS + j) * 16 + lq * 4;
    if (n >= (GROUPED && DUAL ? round_up(a.N, 32) : a.N)) continue;
    float4 bias = make_float4(0.f, 0.f, 0.f, 0.f);
    if (EPI != EPI_PART && a.bias) bias = *reinterpret_cast<const float4*>(a.bias + n);
    float4 own[EPI == EPI_RESID ? MT : 1];              // (requested together; rows beyond the count: the last one again, dropped)
    if constexpr (EPI == EPI_RESID) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
        own[i] = *reinterpret_cast<const float4*>(a.out_f32 + (size_t)max(min((row0 + wm * MT + i) * 16 + l16, n_rows - 1), 0) * a.ldo + n);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = (row0 + wm * MT + i) * 16 + l16;
      if (m >= n_rows) continue;
      const f32x4 c = acc[i][j];
      if constexpr (EPI == EPI_PART) {
        *reinterpret_cast<float4*>(part + (size_t)m * a.ldo + n) = make_float4(c[0], c[1], c[2], c[3]);
      } else if constexpr (EPI == EPI_RESID) {          // the norm's order: row, bias, product
        *reinterpret_cast<float4*>(a.out_f32 + (size_t)m * a.ldo + n) = make_float4((own[i].x + bias.x) + c[0], (own[i].y + bias.y) + c[1],
                                                                                     (own[i].z + bias.z) + c[2], (own[i].w + bias.w) + c[3]);
      } else if constexpr (EPI == EPI_QKV) {
        const float o[4] = {c[0] + bias.x, c[1] + bias.y, c[2] + bias.z, c[3] + bias.w};
        if (n < a.kv.q_cols) {                          // (the three parts and a head are multiples of 4 columns)
          *reinterpret_cast<float4*>(a.out_f32 + (size_t)m * a.ldo + n) = make_float4(o[0], o[1], o[2], o[3]);
        } else {
          bf16_t* p = kv_element(a.kv, kv_b[i], kv_slot[i], n);
          if (n < a.kv.q_cols + a.kv.kv_cols) *reinterpret_cast<uint2*>(p) = make_uint2(pk_bf16(o[0], o[1]), pk_bf16(o[2], o[3]));
          else {                                        // (columns of a value tile are 8 elements apart)
#pragma unroll
            for (int e = 0; e < 4; ++e) p[8 * e] = f2bf(o[e]);
          }
        }
      } else if constexpr (EPI == EPI_F32) {
        *reinterpret_cast<float4*>(a.out_f32 + (size_t)m * a.ldo + n) =
            make_float4(c[0] + bias.x, c[1] + bias.y, c[2] + bias.z, c[3] + bias.w);
      } else {
        float o[4];
        if constexpr (EPI == EPI_GELU) {
          o[0] = gelu_tanh(c[0] + bias.x); o[1] = gelu_tanh(c[1] + bias.y);
          o[2] = gelu_tanh(c[2] + bias.z); o[3] = gelu_tanh(c[3] + bias.w);
        } else {
          const f32x4 u = acc[i][COLS + j];
#pragma unroll
          for (int v = 0; v < 4; ++v) o[v] = GROUPED && n >= a.N ? 0.f : silu(c[v]) * u[v];
        }
        *reinterpret_cast<uint2*>((bf16_t*)a.out_act + act_idx<bf16_t>(m, n, a.out_K)) = make_uint2(pk_f16(o[0], o[1]), pk_f16(o[2], o[3]));
      }
    }
  }
}

// blockIdx.y = K share (partial products).  Tiles in bands of GM row groups, so that what an XCD has in flight at a time (32 compute
// units) shares rows and columns in its own L2.
template <typename T>
__device__ __forceinline__ void tile_place(int t, int gm, int gn, int& bm, int& bn) {
  constexpr int GM = T::wm * T::mt >= 16 ? 4 : 8;
  const int band = t / (GM * gn), in_band = t - band * GM * gn, bh = min(GM, gm - band * GM);
  bm = band * GM + in_band % bh; bn = in_band / bh;
}

// One workgroup of the 256 x 256 tile runs per compute unit: a last round with work for at most half of them is dealt out in halves of
// 256 x 128, 0.6 of a round.  us: 384 tiles (6144 x 4096 at 4096 rows) 196 -> 168, 336 (3528 rows) 182 -> 152, 602 (2 x 11008 x 4096 at
// 1792 rows) 288 -> 259, 1376 (4096 rows) 596 -> 567, 1568 (2 x 14336 x 4096 at 3528 rows) 698 -> 678.
static __host__ __device__ inline int tiles_in_halves(int tiles) { return tiles > 256 && tiles % 256 <= 128 ? tiles % 256 : 0; }

}  // namespace sprinter
