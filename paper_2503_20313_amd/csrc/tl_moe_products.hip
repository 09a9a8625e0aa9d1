// The experts' products on rows sorted by expert, and their gradients: Y_e = X_e W_e, dX_e = dY_e W_e^T, dW_e = X_e^T dY_e, with X_e the
// rows [expert_offsets[e], expert_offsets[e + 1]).  gfx950 only.
//
// One tile kernel in three layouts (tl_gemm_tile.h): W as it is, W read along its rows, and both operands read along the rows of the
// expert, which is then the axis that is summed over.
#include "tl_gemm_tile.h"
#include "tl_moe_choice.h"

namespace tl {

struct ProductParams {
  const bf16_t *x, *w, *dy;
  const int* offsets;
  bf16_t* out;
  const float* add;
  float* out32;
  int max_rows, K, N, E;
  int nbm, nbn;            // column blocks; for dW also row blocks of an expert's K x N
  int k_units;             // Y and dX: units of kPartUnit values of a sum that may be cut
  float* partial;
  int group_m;
};

// Where dW goes: stored as streaming (the layer's weights are larger than the caches, and nobody reads their gradient soon: 32 of
// 4096 x 1792 288 -> 270 us).
struct GradRows16 {
  static constexpr bool SCALED = false, GATED = false;
  bf16_t* c;
  long ldc;
  __device__ __forceinline__ bf16_t* row(int r, float& scale) const { return c + (long)r * ldc; }
  __device__ __forceinline__ void group(int /*r0*/) const {}
  __device__ __forceinline__ void store(int r, int col, u32x4 v) const { __builtin_nontemporal_store(v, (u32x4*)(c + (long)r * ldc + col)); }
};
struct GradRows32 {
  static constexpr bool SCALED = false, GATED = false, F32 = true;
  const float* add;        // or null
  float* c;
  long ldc;
  __device__ __forceinline__ bf16_t* row(int, float&) const { return nullptr; }
  __device__ __forceinline__ void group(int) const {}
  __device__ __forceinline__ void store(int, int, u32x4) const {}
  __device__ __forceinline__ floatx4 load4(int r, int col) const {
    return add ? __builtin_nontemporal_load((const floatx4*)(add + (long)r * ldc + col)) : floatx4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void store4(int r, int col, floatx4 v) const { __builtin_nontemporal_store(v, (floatx4*)(c + (long)r * ldc + col)); }
};

// A part of a cut sum, as it is.
struct PartRows {
  static constexpr bool SCALED = false, GATED = false, F32 = true;
  float* c;
  long ldc;
  __device__ __forceinline__ bf16_t* row(int, float&) const { return nullptr; }
  __device__ __forceinline__ void group(int) const {}
  __device__ __forceinline__ void store(int, int, u32x4) const {}
  __device__ __forceinline__ floatx4 load4(int, int) const { return floatx4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void store4(int r, int col, floatx4 v) const { *(floatx4*)(c + (long)r * ldc + col) = v; }
};

// Rows of expert e, whatever expert_offsets holds: inside [0, max_rows), or none.
__device__ __forceinline__ void rows_of(const ProductParams& p, int e, int* lo, int* n) {
  *lo = min(max(p.offsets[e], 0), p.max_rows);
  *n = max(min(max(p.offsets[e + 1], 0), p.max_rows) - *lo, 0);
}

// Where part number `part` of n things in `parts` begins.
__device__ __forceinline__ int part_start(int n, int parts, int part) { return n / parts * part + min(part, n % parts); }

// The number, among ascending starts, of the last start at or before x, for a wave whose lane i holds starts 4i .. 4i + 3.
__device__ __forceinline__ int last_start(const int (&start)[4], int x) {
  int c = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) c += __builtin_popcountll(__builtin_amdgcn_ballot_w64(start[i] <= x));
  return c - 1;
}
// Exclusive scan over 256 numbers, lane i has 4i .. 4i + 3; returns their sum.
__device__ __forceinline__ int scan_starts(const int (&count)[4], int (&start)[4]) {
  const int lane = threadIdx.x & 63;
  int v = count[0] + count[1] + count[2] + count[3];
  const int mine = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  int at = v - mine;
#pragma unroll
  for (int i = 0; i < 4; i++) { start[i] = at; at += count[i]; }
  return __builtin_amdgcn_readlane(v, 63);
}

// Y and dX.  An expert's rows make tiles of BM rows, and a half one where the rest fits into that (an expert's last tile is half empty in the
// mean; with whole ones alone 16384 rows of 32 experts cost a fifth more); whole tiles first, in patches that share rows and columns in
// a die's L2, then the half ones.
struct ProductJob { bool big; int e, rows, col, cols; long at; };

template <int BM, int BN>
struct ProductTiles {
  int big_at[4], half_at[4];      // first whole and first half tile of experts 4 lane .. 4 lane + 3
  Sched sc;
  int n_all;
  const int *s_lo, *s_n, *s_at;   // in LDS: an expert's rows, its first whole tile
  // By all threads of the workgroup.
  __device__ __forceinline__ void init(const ProductParams& p, int grid, int (&lds)[3][kMaxProductExperts]) {
    const int tid = threadIdx.x, lane = tid & 63;
    for (int e = tid; e < kMaxProductExperts; e += blockDim.x) {
      int lo = 0, n = 0;
      if (e < p.E) rows_of(p, e, &lo, &n);
      lds[0][e] = lo;
      lds[1][e] = n;
    }
    __syncthreads();
    int big[4], half[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int n = lds[1][lane * 4 + i], rest = n % BM;
      half[i] = rest > 0 && rest <= BM / 2 ? 1 : 0;
      big[i] = n / BM + (rest > BM / 2 ? 1 : 0);
    }
    sc.nbm = scan_starts(big, big_at);
    const int n_half = scan_starts(half, half_at);
    if (tid < 64) {
#pragma unroll
      for (int i = 0; i < 4; i++) lds[2][lane * 4 + i] = big_at[i];
    }
    __syncthreads();
    s_lo = lds[0]; s_n = lds[1]; s_at = lds[2];
    sc.nbn = p.nbn;
    sc.n_tiles = sc.nbm * sc.nbn;
    sc.G = grid;
    sc.first_block = 0;
    sc.swizzle = 1;
    sc.group_m = p.group_m < sc.nbm ? p.group_m : (sc.nbm > 0 ? sc.nbm : 1);
    n_all = sc.n_tiles + n_half * sc.nbn;
  }
  // Tile number pos < n_all; by whole waves.
  __device__ __forceinline__ ProductJob at(int pos, int ndim) const {
    ProductJob j;
    j.big = pos < sc.n_tiles;
    int bm, bn, r0;
    if (j.big) {
      const int tile = sched_tile(sc, pos);
      bm = tile / sc.nbn;
      bn = tile - bm * sc.nbn;
      j.e = last_start(big_at, bm);
      r0 = (bm - __builtin_amdgcn_readfirstlane(s_at[j.e])) * BM;
    } else {
      bm = (pos - sc.n_tiles) / sc.nbn;
      bn = pos - sc.n_tiles - bm * sc.nbn;
      j.e = last_start(half_at, bm);
      r0 = __builtin_amdgcn_readfirstlane(s_n[j.e]) / BM * BM;
    }
    j.rows = min(__builtin_amdgcn_readfirstlane(s_n[j.e]) - r0, BM);
    j.at = __builtin_amdgcn_readfirstlane(s_lo[j.e]) + r0;
    j.col = bn * BN;
    j.cols = min(BN, ndim - j.col);
    return j;
  }
};

// The tiles of the last round, where they would leave half the workgroups or more without one: their sums are cut, into as many
// parts as there are workgroups for each.  Parts go to the workspace (place (tile - first) * parts + part), the join kernel adds them up in their order.
struct ProductRest {
  int first, n, parts;      // tiles; parts of a sum, 1: uncut
  __device__ __forceinline__ ProductRest(const ProductParams& p, int n_all, int grid) {
    n = n_all % grid;
    first = n_all - n;
    parts = n > 0 ? min(min(grid / n, kMaxParts), p.k_units) : 1;
  }
};

template <class Big, class Half, bool GRAD_X, bool CUT>
__global__ void __launch_bounds__(Big::NTHREADS) moe_product_kernel(const ProductParams p) {
  static_assert(Big::NTHREADS == Half::NTHREADS && Big::BN == Half::BN && Big::BM == 2 * Half::BM, "the two shapes share workgroup and columns");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  __shared__ int s_experts[3][kMaxProductExperts];
  ProductTiles<Big::BM, Big::BN> tiles;
  tiles.init(p, gridDim.x, s_experts);
  const int kdim = GRAD_X ? p.N : p.K, ndim = GRAD_X ? p.K : p.N;
  const ProductRest rest(p, tiles.n_all, gridDim.x);
  const int n_items = CUT ? rest.first + rest.n * rest.parts : tiles.n_all;
  for (int pos = blockIdx.x; pos < n_items; pos += gridDim.x) {
    int tile = pos, part = 0, k0 = 0, k = kdim;
    if (CUT && pos >= rest.first) {
      part = (pos - rest.first) / rest.n;
      tile = pos - part * rest.n;
      k0 = part_start(p.k_units, rest.parts, part) * kPartUnit;
      k = min(part_start(p.k_units, rest.parts, part + 1) * kPartUnit, kdim) - k0;
    }
    const ProductJob j = tiles.at(tile, ndim);
    const bf16_t* a = (GRAD_X ? p.dy : p.x) + j.at * kdim + k0;
    const bf16_t* b = p.w + (long)j.e * p.K * p.N + (GRAD_X ? (long)j.col * p.N + k0 : (long)k0 * p.N + j.col);
    if (CUT && pos >= rest.first && rest.parts > 1) {
      const PartRows out{p.partial + ((long)(tile - rest.first) * rest.parts + part) * (Big::BM * Big::BN), Big::BN};
      if (j.big) gemm_tile<Big>(a, kdim, nullptr, 1, b, p.N, out, j.rows, j.cols, k, smem);
      else gemm_tile<Half>(a, kdim, nullptr, 1, b, p.N, out, j.rows, j.cols, k, smem);
    } else {
      const DenseRows out{p.out + j.at * ndim + j.col, ndim};
      if (j.big) gemm_tile<Big>(a, kdim, nullptr, 1, b, p.N, out, j.rows, j.cols, k, smem);
      else gemm_tile<Half>(a, kdim, nullptr, 1, b, p.N, out, j.rows, j.cols, k, smem);
    }
  }
}

// Sum of up to kMaxParts partial results of eight neighbouring columns, `step` apart, in their order: all loads in flight together.
__device__ __forceinline__ void join_parts(const float* src, long step, int parts, float (&o)[8]) {
  floatx4 v[kMaxParts][2];
#pragma unroll
  for (int q = 0; q < kMaxParts; q++) {
    v[q][0] = v[q][1] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (q < parts) {
      v[q][0] = __builtin_nontemporal_load((const floatx4*)(src + q * step));
      v[q][1] = __builtin_nontemporal_load((const floatx4*)(src + q * step + 4));
    }
  }
#pragma unroll
  for (int c = 0; c < 8; c++) o[c] = v[0][c / 4][c % 4];
#pragma unroll
  for (int q = 1; q < kMaxParts; q++)
#pragma unroll
    for (int c = 0; c < 8; c++) o[c] += v[q][c / 4][c % 4];
}

template <int BM, int BN, bool GRAD_X>
__global__ void __launch_bounds__(256) moe_product_join_kernel(const ProductParams p, int grid) {
  __shared__ int s_experts[3][kMaxProductExperts];
  ProductTiles<BM, BN> tiles;
  tiles.init(p, grid, s_experts);
  const ProductRest rest(p, tiles.n_all, grid);
  if (rest.parts == 1) return;
  const int ndim = GRAD_X ? p.K : p.N;
  constexpr int kSlices = BM * BN / 8 / 256;
  for (int i = blockIdx.x; i < rest.n * kSlices; i += gridDim.x) {
    const int tile = rest.first + i / kSlices, chunk = i % kSlices * 256 + threadIdx.x, y = chunk / (BN / 8), x = chunk % (BN / 8) * 8;
    const ProductJob j = tiles.at(tile, ndim);
    if (y >= j.rows || x >= j.cols) continue;
    float o[8];
    join_parts(p.partial + (long)(tile - rest.first) * rest.parts * (BM * BN) + y * BN + x, BM * BN, rest.parts, o);
    *(u32x4*)(p.out + (j.at + y) * ndim + j.col + x) = pack_bf16x8(o);
  }
}

// ======================================================================================
// Few rows for an expert (single tokens being decoded, a small batch over many experts): bound by reading the weights once.  A unit is up
// to 64 rows of an expert times a block of output columns; it is a wave's alone, or NW waves take its steps along the summed axis in turn,
// each through a ring of its own in LDS, so that no wave waits for another; their sums are joined at the end, in the order of the waves.
// Per step
//   Y^T[columns, rows] += W^T . X^T   (16x16x32 matrix instructions; a lane owns one row and four columns)
// W as it lies (forward: 32 k-rows, transposing LDS reads) or along its rows (dX: pieces of 64 values, plain reads), 4 KiB or, WIDE, 8 KiB of
// it a step.  Measured for 320 rows of 32 experts of 2048 x 1536 (195 MB): 64 columns a wave 44.7 us, 128 columns 42.9, two waves side by side
// on 256 columns -- half a KiB of every row -- 40.8, four 57.5 (a compute unit takes no more than about 60 GB/s by direct-to-LDS
// loads); marked as streaming 42.9 against 45.7.  The kernel alone reaches 5.5 to 6.3 TB/s.
// ======================================================================================
struct FewUnit {
  const bf16_t *x, *w;      // first row; W at the unit's first column
  bf16_t* out;              // first row, first column
  int ldx, ldw, ldo;
  int rows, cols, kdim;
  bool once;                // the weights are this unit's alone: streaming loads
};

constexpr int kFewRing = 40 * 1024;       // LDS of a wave: four waves a compute unit, up to 40 KiB of each in flight
constexpr int kFewRows = 64;

template <bool NK, int RT, bool WIDE>     // RT: row tiles of 16
struct FewShape {
  static constexpr int CW = few_columns(NK, WIDE), BK = NK ? 64 : 32, CT = CW / 16, KH = BK / 32;
  static constexpr int PITCH = NK ? BK * 2 : CW * 2, RPL = 1024 / PITCH;     // bytes of a row of memory, rows of a load
  static constexpr int W_LOADS = WIDE ? 8 : 4, X_LOADS = RT * BK / 32, LPS = W_LOADS + X_LOADS, STAGE = LPS * 1024;
  static constexpr int NS = kFewRing / STAGE;
  static_assert(NS >= 2 && NS * LPS <= 63, "ring depth, vmcnt range");
};

template <bool NK, int RT, bool WIDE, int NW>
__device__ __forceinline__ void few_unit(const FewUnit& f, char* smem) {
  typedef FewShape<NK, RT, WIDE> S;
  const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, gr = lane >> 4;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  const int steps = (f.kdim + S::BK - 1) / S::BK;
  const int mine = steps > wave ? (steps - wave + NW - 1) / NW : 0;
  char* ring = smem + wave * kFewRing;
  const unsigned ring_u = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)ring);
  // ---- W: load j covers RPL rows of memory; LDS place (row, c) holds piece c ^ w_twist(row), which keeps the fragment reads apart
  auto w_twist = [](int row) { return NK ? (row >> 1) & 7 : WIDE ? (row & 3) << 1 | ((row >> 3) & 1) << 3 : ((row >> 1) & 1) << 1 | ((row >> 3) & 1) << 2; };
  constexpr int WC = S::PITCH / 16;                 // pieces of a row
  auto w_variant = [](int j) { return S::RPL == 8 ? j & 1 : (j >> 1) & 1; };      // bit 3 of the load's rows
  unsigned w_off[2], x_off[S::X_LOADS];
#pragma unroll
  for (int j = 0; j < 2; j++) {
    const int row = lane / WC + 8 * j;
    w_off[j] = (unsigned)(lane / WC) * (unsigned)(f.ldw * 2) + (unsigned)(((lane % WC) ^ w_twist(row)) << 4);
  }
  // ---- X: rows of BK values, 16-byte pieces twisted by their row; rows that are not there repeat the last one
  constexpr int XC = S::BK / 8;                     // pieces of a row
  auto x_twist = [](int row) { return NK ? (row >> 1) & 7 : (row >> 2) & 3; };
  auto x_row = [&](int q) { return q * (64 / XC) + lane / XC; };
  auto x_piece = [&](int q) { return (lane % XC) ^ x_twist(x_row(q)); };
#pragma unroll
  for (int q = 0; q < S::X_LOADS; q++) x_off[q] = (unsigned)min(x_row(q), f.rows - 1) * (unsigned)(f.ldx * 2) + (unsigned)(x_piece(q) << 4);
  const bool whole_cols = f.cols == S::CW;
  auto issue = [&](int i, int slot) __attribute__((always_inline)) {
    const int k0 = (wave + i * NW) * S::BK;
    const unsigned dst = ring_u + slot * S::STAGE;
    if (whole_cols && k0 + S::BK <= f.kdim) {
      const char* wb = (const char*)uniform64((unsigned long long)(f.w + (NK ? (long)k0 : (long)k0 * f.ldw)));
      const char* xb = (const char*)uniform64((unsigned long long)(f.x + k0));
      const long w8 = (long)f.ldw * (2 * S::RPL);
      if (f.once) {
#pragma unroll
        for (int j = 0; j < S::W_LOADS; j++) lds_load16_sbase_nt(wb + j * w8, w_off[w_variant(j)], dst + j * 1024);
      } else {
#pragma unroll
        for (int j = 0; j < S::W_LOADS; j++) lds_load16_sbase(wb + j * w8, w_off[w_variant(j)], dst + j * 1024);
      }
#pragma unroll
      for (int q = 0; q < S::X_LOADS; q++) lds_load16_sbase(xb, x_off[q], dst + (S::W_LOADS + q) * 1024);
      return;
    }
    // an edge: columns beyond the last repeat the last ones, values beyond the summed axis are zeros
#pragma unroll
    for (int j = 0; j < S::W_LOADS; j++) {
      const int row = j * S::RPL + lane / WC, piece = (lane % WC) ^ w_twist(row);
      const int k = k0 + (NK ? piece * 8 : row), c = NK ? min(row, f.cols - 1) : min(piece * 8, f.cols - 8);
      const bf16_t* src = NK ? f.w + (long)c * f.ldw + k : f.w + (long)k * f.ldw + c;
      lds_load16_at(k < f.kdim ? (const char*)src : (const char*)g_zero_chunk, dst + j * 1024);
    }
#pragma unroll
    for (int q = 0; q < S::X_LOADS; q++) {
      const char* src = (const char*)(f.x + k0) + x_off[q];
      lds_load16_at(k0 + x_piece(q) * 8 < f.kdim ? src : (const char*)g_zero_chunk, dst + (S::W_LOADS + q) * 1024);
    }
  };
  floatx4 acc[RT][S::CT];
#pragma unroll
  for (int u = 0; u < RT; u++)
#pragma unroll
    for (int c = 0; c < S::CT; c++) acc[u][c] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < S::NS; i++)
    if (i < mine) issue(i, i);
  // ---- where the lane's fragments lie in a stage
  const int r = l15 >> 2;
  const int w_rd = NK ? l15 * 128 : (8 * gr + r) * S::PITCH + (lane & 1) * 8;
  const int w_x = NK ? w_twist(l15) : w_twist(8 * gr + r);
  int slot = 0;
  for (int i = 0; i < mine; i++) {
    if (i + S::NS <= mine) wait_vmcnt<(S::NS - 1) * S::LPS>(); else wait_vmcnt<0>();
    const char* st = ring + slot * S::STAGE;
    bf16x8 wf[S::KH][S::CT], xf[S::KH][RT];
#pragma unroll
    for (int h = 0; h < S::KH; h++) {
#pragma unroll
      for (int c = 0; c < S::CT; c++) {
        if constexpr (NK) {
          wf[h][c] = *(const bf16x8*)(st + w_rd + c * 2048 + (((4 * h + gr) ^ w_x) << 4));
        } else {
          typedef short short8_t __attribute__((ext_vector_type(8)));
          const char* p = st + w_rd + (((2 * c + ((lane & 2) >> 1)) ^ w_x) << 4);
          const short4_t lo = lds_read_tr(p), hi = lds_read_tr(p + 4 * S::PITCH);
          wf[h][c] = __builtin_bit_cast(bf16x8, (short8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
      }
#pragma unroll
      for (int u = 0; u < RT; u++) {
        const int row = u * 16 + l15;
        xf[h][u] = *(const bf16x8*)(st + S::W_LOADS * 1024 + row * (XC * 16) + (((4 * h + gr) ^ x_twist(row)) << 4));
      }
    }
    if (i + S::NS < mine) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the fragments are in registers: their place may be filled again
      issue(i + S::NS, slot);
    }
#pragma unroll
    for (int h = 0; h < S::KH; h++)
#pragma unroll
      for (int c = 0; c < S::CT; c++)
#pragma unroll
        for (int u = 0; u < RT; u++) acc[u][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[h][c], xf[h][u], acc[u][c], 0, 0, 0);
    slot = slot + 1 == S::NS ? 0 : slot + 1;
  }
  // ---- join and store.  Lane (l15, gr): row l15 of a row tile, columns 4 gr .. + 3 of a column tile
  if constexpr (NW > 1) {
    constexpr int PITCH = S::CW + 4;
    static_assert(RT * 16 * PITCH * 4 <= kFewRing, "a wave's sums fit its ring");
    __syncthreads();
    float* own = (float*)ring;
#pragma unroll
    for (int u = 0; u < RT; u++)
#pragma unroll
      for (int c = 0; c < S::CT; c++) *(floatx4*)(own + (u * 16 + l15) * PITCH + c * 16 + gr * 4) = acc[u][c];
    __syncthreads();
    for (int i = tid; i < f.rows * (S::CW / 4); i += NW * 64) {
      const int row = i / (S::CW / 4), col = (i - row * (S::CW / 4)) * 4;
      if (col >= f.cols) continue;
      floatx4 v = *(const floatx4*)((const float*)smem + row * PITCH + col);
#pragma unroll
      for (int w = 1; w < NW; w++) {
        const floatx4 o = *(const floatx4*)((const float*)(smem + w * kFewRing) + row * PITCH + col);
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] += o[e];
      }
      bf16x4 b;
#pragma unroll
      for (int e = 0; e < 4; e++) b[e] = (bf16_t)v[e];
      *(bf16x4*)(f.out + (long)row * f.ldo + col) = b;
    }
  } else {
#pragma unroll
    for (int u = 0; u < RT; u++)
#pragma unroll
      for (int c = 0; c < S::CT; c++) {
        const int row = u * 16 + l15, col = c * 16 + gr * 4;
        bf16x4 b;
#pragma unroll
        for (int e = 0; e < 4; e++) b[e] = (bf16_t)acc[u][c][e];
        if (row < f.rows && col < f.cols) *(bf16x4*)(f.out + (long)row * f.ldo + col) = b;
      }
  }
}

// NW waves share a unit, or NC = 2 take one each, side by side.
template <bool GRAD_X, bool WIDE, int NW, int NC>
__global__ void __launch_bounds__(NW * NC * 64) moe_few_rows_kernel(const ProductParams p) {
  static_assert(NW == 1 || NC == 1, "waves share a unit or have one each");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int beside = NC == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  constexpr int CW = FewShape<GRAD_X, 1, WIDE>::CW;
  const int ndim = GRAD_X ? p.K : p.N, kdim = GRAD_X ? p.N : p.K;
  // ---- the row tiles of all experts, in every wave: lane i the experts 4i .. 4i + 3
  int tiles = 0, t4[4], n4[4], lo4[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    lo4[i] = n4[i] = 0;
    if (lane * 4 + i < p.E) rows_of(p, lane * 4 + i, &lo4[i], &n4[i]);
    t4[i] = (n4[i] + kFewRows - 1) / kFewRows;
    tiles += t4[i];
  }
  int scan = tiles;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(scan, d);
    if (lane >= d) scan += o;
  }
  // ---- a die takes a run of units, whose rows of X it then reads once (1024 rows of 32 experts 51.6 -> 47.4 us; no difference with fewer)
  const int units = __builtin_amdgcn_readlane(scan, 63) * p.nbn;
  const int per = (units + kXcds * NC - 1) / (kXcds * NC) * NC, i = blockIdx.x / kXcds * NC + beside, unit = (blockIdx.x % kXcds) * per + i;
  if (i >= per || unit >= units) return;                // (there are fewer than the grid has room for)
  const int bm = unit / p.nbn, bn = unit - bm * p.nbn;
  int at = scan - tiles, e4 = 0, first = 0, n = 0, lo = 0;     // in the lane that has it: which of its four
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (at <= bm && bm < at + t4[i]) { e4 = i; first = at; n = n4[i]; lo = lo4[i]; }
    at += t4[i];
  }
  const int owner = __builtin_ctzll(__builtin_amdgcn_ballot_w64(scan > bm));
  const int e = owner * 4 + __builtin_amdgcn_readlane(e4, owner);
  first = __builtin_amdgcn_readlane(first, owner);
  n = __builtin_amdgcn_readlane(n, owner);
  lo = __builtin_amdgcn_readlane(lo, owner);
  const int r0 = (bm - first) * kFewRows, col = bn * CW;
  FewUnit f;
  f.rows = min(n - r0, kFewRows);
  f.cols = min(CW, ndim - col);
  f.kdim = kdim;
  f.once = n <= kFewRows;
  const bf16_t* w = p.w + (long)e * p.K * p.N;
  f.w = GRAD_X ? w + (long)col * p.N : w + col;
  f.ldw = p.N;
  f.x = (GRAD_X ? p.dy : p.x) + (long)(lo + r0) * kdim;
  f.ldx = kdim;
  f.out = p.out + (long)(lo + r0) * ndim + col;
  f.ldo = ndim;
  if (f.rows <= 16) few_unit<GRAD_X, 1, WIDE, NW>(f, smem + beside * kFewRing);
  else if (f.rows <= 32) few_unit<GRAD_X, 2, WIDE, NW>(f, smem + beside * kFewRing);
  else few_unit<GRAD_X, 4, WIDE, NW>(f, smem + beside * kFewRing);
}

// ======================================================================================
// dW.  An expert's tiles sum over its rows, many or few, so the work is laid out by length, by a launch of its own (one workgroup): an even
// share of all rows x tiles for every compute unit is the longest an item should be, a longer sum is cut into parts, and the items stand
// in the order of their length, the longest first, for the hardware to hand out (8 gradients of 2048 x 1536 over 114 .. 4701 rows, added in fp32:
// 184 us uncut in the experts' order, 152 so; 2 of 1024 x 1024 over 32768 rows 504 and 147).  The parts of a cut sum go to the workspace in fp32,
// and a third launch adds them up in their order.
// A workgroup takes one item: it may end while its stores are on their way.  (A persistent one that requests the next item's first stages
// before it stores this one's result has to wait, a few steps later, for those stores to be complete, as loads and stores are counted
// together: 32 gradients of 4096 x 1792 over 512 rows each 284 us against 272.  Two smaller workgroups a compute unit, of 128 x 256, are held up by
// their direct-to-LDS loads: 289.)
// ======================================================================================
struct GradWParams {
  ProductParams p;
  GradWPlan* plan;
  float* partial;          // [places][BM * BN]
  int places, share_of;    // places of partial sums; compute units that share the work
  int run;
};

__global__ void __launch_bounds__(kPlanThreads) moe_grad_w_plan_kernel(const GradWParams g) {
  static_assert(kPlanThreads == kMaxProductExperts, "an expert to a thread");
  __shared__ int s_n[kMaxProductExperts], s_rank[kMaxProductExperts], s_by_rank[kMaxProductExperts];
  const ProductParams& p = g.p;
  const int tid = threadIdx.x, lane = tid & 63;
  const int per = p.nbm * p.nbn;
  int lo = 0, n = -1;
  if (tid < p.E) rows_of(p, tid, &lo, &n);
  s_n[tid] = n;
  __syncthreads();
  int rank = 0;
  long all = 0;
#pragma unroll 8
  for (int o = 0; o < p.E; o++) {
    const int m = s_n[o];
    rank += m > n || (m == n && o < tid);
    all += m;
  }
  // the longest part there is to be
  const long share = (all * per + g.share_of - 1) / g.share_of;
  const unsigned chunk = g.places ? (unsigned)max(min(share, 0x7fffffffL), (long)kMinPart) : 0x7fffffffu;
  auto parts_of = [&](int m) { return max(min((int)(((unsigned)max(m, 0) + (chunk - 1)) / chunk), kMaxParts), 1); };     // (both below 2^31)
  s_by_rank[tid] = -1;
  // Many rounds of items: those of more than 1.5 times the mean first, the others as they come, so that some workgroups store while others
  // multiply (64 gradients of 2048 x 1536 over 256 rows each in the mean 190 us longest first, 179 so, before the dies took turns); what the last round is then left
  // with weighs little.
  const bool cut_any = __syncthreads_or(parts_of(n) > 1);
  if (!cut_any && (long)p.E * per >= 4L * g.share_of) {
    const int some = (int)min(all * 3 / (2 * p.E), 0x7fffffffL);
    if (n <= some) {
      rank = 0;
#pragma unroll 8
      for (int o = 0; o < p.E; o++) rank += s_n[o] > some || o < tid;
    }
  }
  if (tid < p.E) {
    s_by_rank[rank] = n;
    s_rank[tid] = rank;
  }
  __syncthreads();
  if (tid < 64) {
    int items[4], places[4], at[4], pl[4], cut = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = lane * 4 + i, parts = r < p.E ? parts_of(s_by_rank[r]) : 0;
      items[i] = parts * per;
      places[i] = parts > 1 ? items[i] : 0;
      cut += parts > 1 ? per : 0;
    }
    const int n_items = scan_starts(items, at);
    scan_starts(places, pl);       // (at most g.places: see grad_w_shape)
#pragma unroll
    for (int d = 1; d < 64; d *= 2) cut += __shfl_xor(cut, d);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      g.plan->first[lane * 4 + i] = at[i];
      s_n[lane * 4 + i] = pl[i];
    }
    if (lane == 0) {
      g.plan->n_items = n_items;
      g.plan->n_cut = cut;
    }
  }
  __syncthreads();
  if (tid < p.E) g.plan->expert[s_rank[tid]] = GradWExpert{lo, n, (unsigned)tid | (unsigned)parts_of(n) << 8, s_n[s_rank[tid]]};
}

template <class Cfg, class Out>
__global__ void __launch_bounds__(Cfg::NTHREADS, Cfg::LDS_BYTES <= 80 * 1024 ? 2 : 1) moe_grad_w_kernel(const GradWParams g) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const ProductParams& p = g.p;
  // Runs of g.run items, a quarter of an expert's, go to one die, which then reads its part of the rows once (32 gradients of 4096 x 1792: 322 us
  // without, 288 with eighths; quarters 2 to 10 % less where sums are of one length, halves leave dies without work); every other turn in
  // reverse, or the first die would get the longest item of each (64 gradients of 2048 x 1536: 190 -> 172 us).
  const int i = blockIdx.x / kXcds, turn = i / g.run, die = blockIdx.x % kXcds;
  const int l = (turn * kXcds + (turn % 2 ? kXcds - 1 - die : die)) * g.run + i % g.run;
  const u32x4 starts = ((const u32x4*)g.plan->first)[threadIdx.x & 63];
  if (l >= g.plan->n_items) return;
  int start[4];
#pragma unroll
  for (int c = 0; c < 4; c++) start[c] = (int)starts[c];
  const int r = last_start(start, l);
  const u32x4 rec = ((const u32x4*)g.plan->expert)[r];
  const int lo = __builtin_amdgcn_readfirstlane(rec[0]), all = __builtin_amdgcn_readfirstlane(rec[1]), place0 = __builtin_amdgcn_readfirstlane(rec[3]);
  const unsigned what = __builtin_amdgcn_readfirstlane(rec[2]);
  const int e = what & 255, parts = what >> 8;
  const int per = p.nbm * p.nbn, item = l - __builtin_amdgcn_readfirstlane(g.plan->first[r]), part = item / per, tile = item - part * per;
  const int k0 = part_start(all, parts, part), n = part_start(all, parts, part + 1) - k0, row0 = lo + k0, place = place0 + tile * parts + part;
  const int bm = tile / p.nbn, bn = tile - bm * p.nbn;
  const int row = bm * Cfg::BM, rows = min(Cfg::BM, p.K - row), col = bn * Cfg::BN, cols = min(Cfg::BN, p.N - col);
  const long at = ((long)e * p.K + row) * p.N + col;
  Out out;
  if constexpr (StoresF32<Out>::value) out = Out{p.add ? p.add + at : nullptr, p.out32 + at, p.N};
  else out = Out{p.out + at, p.N};
  if (n == 0) {     // an expert without rows: zeros, or what there was (whole lines, four
                    // of them in flight: 32 experts of 2048 x 1536, 24 of them without, 308 -> 154 us)
    if constexpr (StoresF32<Out>::value) {
      if (p.add == p.out32) return;
      const int width = cols / 4, pieces = rows * width;
      for (int c0 = threadIdx.x; c0 < pieces; c0 += 4 * Cfg::NTHREADS) {
        floatx4 v[4];
#pragma unroll
        for (int u = 0; u < 4; u++) {
          const int c = c0 + u * Cfg::NTHREADS;
          if (c < pieces) v[u] = out.load4(c / width, c % width * 4);
        }
#pragma unroll
        for (int u = 0; u < 4; u++) {
          const int c = c0 + u * Cfg::NTHREADS;
          if (c < pieces) out.store4(c / width, c % width * 4, v[u]);
        }
      }
    } else {
      for (int c = threadIdx.x; c < rows * (cols / 8); c += Cfg::NTHREADS) {
        const int y = c / (cols / 8), x = (c - y * (cols / 8)) * 8;
        out.store(y, x, u32x4{0, 0, 0, 0});
      }
    }
    return;
  }
  const bf16_t *a = p.x + (long)row0 * p.K + row, *b = p.dy + (long)row0 * p.N + col;
  if (parts == 1) gemm_tile<Cfg, Out>(a, p.K, nullptr, 1, b, p.N, out, rows, cols, n, smem);
  else gemm_tile<Cfg, PartRows>(a, p.K, nullptr, 1, b, p.N, PartRows{g.partial + (long)place * (Cfg::BM * Cfg::BN), Cfg::BN}, rows, cols, n, smem);
}

// The cut sums: eight neighbouring columns to a thread.
template <class Cfg, class Out>
__global__ void __launch_bounds__(256) moe_grad_w_join_kernel(const GradWParams g) {
  const ProductParams& p = g.p;
  constexpr int BM = Cfg::BM, BN = Cfg::BN, kSlices = BM * BN / 8 / 256;
  const int n = g.plan->n_cut * kSlices, per = p.nbm * p.nbn;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const GradWExpert x4 = g.plan->expert[i / kSlices / per];           // (the experts with cut sums come first)
    const int e = x4.what & 255, parts = x4.what >> 8, tile = i / kSlices % per;
    const int chunk = i % kSlices * 256 + threadIdx.x, y = chunk / (BN / 8), x = chunk % (BN / 8) * 8;
    const int bm = tile / p.nbn, bn = tile - bm * p.nbn;
    if (bm * BM + y >= p.K || bn * BN + x >= p.N) continue;
    const float* src = g.partial + ((long)x4.place + (long)tile * parts) * (BM * BN) + y * BN + x;
    float o[8];
    join_parts(src, BM * BN, parts, o);
    const long at = ((long)e * p.K + bm * BM) * p.N + bn * BN;
    if constexpr (StoresF32<Out>::value) {
      const Out out{p.add ? p.add + at : nullptr, p.out32 + at, p.N};
#pragma unroll
      for (int h = 0; h < 2; h++) {
        floatx4 w = out.load4(y, x + 4 * h);
#pragma unroll
        for (int c = 0; c < 4; c++) w[c] += o[4 * h + c];
        out.store4(y, x + 4 * h, w);
      }
    } else {
      Out{p.out + at, p.N}.store(y, x, pack_bf16x8(o));
    }
  }
}

// ======================================================================================
// Host side
// ======================================================================================
template <bool NK> using ProductBig = TileCfg<256, 256, 2, 4, 32, 4, false, NK>;
template <bool NK> using ProductBigHalf = TileCfg<128, 256, 2, 4, 32, 4, false, NK>;
template <bool NK> using ProductSmall = TileCfg<128, 128, 2, 2, 64, 4, false, NK>;
template <bool NK> using ProductSmallHalf = TileCfg<64, 128, 2, 2, 64, 4, false, NK>;
typedef TileCfg<256, 256, 2, 4, 32, 4, true, false> CfgW256;
typedef TileCfg<128, 256, 2, 2, 32, 3, true, false> CfgW128x256;      // two workgroups a compute unit
typedef TileCfg<128, 128, 2, 2, 64, 4, true, false> CfgW128;

static int check_product(const char* what, int max_rows, int K, int N, int E) {
  if (max_rows <= 0 || K <= 0 || N <= 0 || E <= 0) return fail(TL_ERR_INVALID_ARG, "%s: max_rows, K, N and E must be positive", what);
  if (E > kMaxProductExperts) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: at most %d experts (got %d)", what, kMaxProductExperts, E);
  if (K % 8 || N % 8) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: K=%d and N=%d must be multiples of 8", what, K, N);
  if (K > (1 << 20) || N > (1 << 20)) return fail(TL_ERR_UNSUPPORTED_SHAPE, "%s: K and N must not exceed 2^20", what);
  return TL_OK;
}

static int check_product_call(tl_ctx* ctx, const char* what, int way, const void* a, const void* b, const void* out, const int* offsets, int max_rows, int K, int N,
                              int E, const void* workspace, size_t ws_bytes) {
  if (int e = check_ctx(ctx)) return e;
  size_t need;
  if (int e = check_product(what, max_rows, K, N, E)) return e;
  if (!a || !b || !out || !offsets || !workspace) return fail(TL_ERR_INVALID_ARG, "%s: null pointer argument", what);
  if (!aligned16(a) || !aligned16(b) || !aligned16(out) || ((uintptr_t)offsets & 3) || !aligned128(workspace))
    return fail(TL_ERR_INVALID_ARG, "%s: matrices must be 16-byte aligned, the workspace 128-byte, expert_offsets 4-byte", what);
  if (int e = tl_moe_gemm_query(ctx, way, max_rows, K, N, E, &need)) return e;
  if (ws_bytes < need) return fail(TL_ERR_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need);
  return check_op_ctx(ctx);
}

template <bool GRAD_X, bool WIDE, int NW, int NC>
static int launch_few(ProductParams& p, int ndim, hipStream_t s) {
  p.nbn = ceil_div(ndim, FewShape<GRAD_X, 1, WIDE>::CW);
  const long row_tiles = (p.max_rows < p.E ? p.max_rows : p.E) + p.max_rows / kFewRows;       // at most
  const long grid = (row_tiles * p.nbn + kXcds * NC - 1) / (kXcds * NC) * kXcds;
  constexpr int kWaves = NW * NC;
  TL_HIP(hipFuncSetAttribute((const void*)moe_few_rows_kernel<GRAD_X, WIDE, NW, NC>, hipFuncAttributeMaxDynamicSharedMemorySize, kWaves * kFewRing));
  hipLaunchKernelGGL((moe_few_rows_kernel<GRAD_X, WIDE, NW, NC>), dim3((unsigned)grid), dim3(kWaves * 64), kWaves * kFewRing, s, p);
  TL_HIP(hipGetLastError());
  return TL_OK;
}

template <class Big, class Half, bool GRAD_X>
static int launch_tiles(tl_ctx* ctx, ProductParams& p, bool cut, int ndim, hipStream_t s) {
  p.nbn = ceil_div(ndim, Big::BN);
  if (!cut) return launch_fused<Big>(moe_product_kernel<Big, Half, GRAD_X, false>, p, ctx->num_cus, s);
  if (int e = launch_fused<Big>(moe_product_kernel<Big, Half, GRAD_X, true>, p, ctx->num_cus, s)) return e;
  hipLaunchKernelGGL((moe_product_join_kernel<Big::BM, Big::BN, GRAD_X>), dim3(ctx->num_cus), dim3(256), 0, s, p, ctx->num_cus);
  TL_HIP(hipGetLastError());
  return TL_OK;
}

template <bool GRAD_X>
static int launch_product(tl_ctx* ctx, ProductParams& p, void* workspace, hipStream_t s) {
  const int ndim = GRAD_X ? p.K : p.N;
  const ProductShape shape = product_shape(ctx, GRAD_X, p.max_rows, p.K, p.N, p.E);
  if (!shape.tile) {
    const FewChoice c = few_choice(ctx, GRAD_X, p.max_rows, p.E, ndim);
    if (c.beside == 2) return launch_few<GRAD_X, true, 1, 2>(p, ndim, s);
    if (c.wide) return launch_few<GRAD_X, true, 2, 1>(p, ndim, s);
    if (c.waves == 2) return launch_few<GRAD_X, false, 2, 1>(p, ndim, s);
    return launch_few<GRAD_X, false, 4, 1>(p, ndim, s);
  }
  p.group_m = 4;
  p.k_units = ceil_div(GRAD_X ? p.N : p.K, kPartUnit);
  p.partial = (float*)workspace;
  if (shape.tile == 128) return launch_tiles<ProductSmall<GRAD_X>, ProductSmallHalf<GRAD_X>, GRAD_X>(ctx, p, shape.cut, ndim, s);
  return launch_tiles<ProductBig<GRAD_X>, ProductBigHalf<GRAD_X>, GRAD_X>(ctx, p, shape.cut, ndim, s);
}

template <class Cfg, class Out>
static int launch_grad_w(const GradWParams& g, long grid, hipStream_t s) {
  hipLaunchKernelGGL(moe_grad_w_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, g);
  TL_HIP(hipGetLastError());
  if (int e = launch_fused<Cfg>(moe_grad_w_kernel<Cfg, Out>, g, (int)grid, s)) return e;
  if (g.places) {
    hipLaunchKernelGGL((moe_grad_w_join_kernel<Cfg, Out>), dim3(512), dim3(256), 0, s, g);
    TL_HIP(hipGetLastError());
  }
  return TL_OK;
}

}  // namespace tl

using namespace tl;

extern "C" {

int tl_moe_gemm_query(const tl_ctx* ctx, int way, int max_rows, int K, int N, int E, size_t* ws_bytes) {
  if (int e = check_ctx(ctx)) return e;
  if (!ws_bytes) return fail(TL_ERR_INVALID_ARG, "tl_moe_gemm_query: ws_bytes must not be null");
  if (way != TL_MOE_FORWARD && way != TL_MOE_GRAD_X && way != TL_MOE_GRAD_W) return fail(TL_ERR_INVALID_ARG, "tl_moe_gemm_query: %d is not one of the three products", way);
  if (int e = check_product("tl_moe_gemm_query", max_rows, K, N, E)) return e;
  if (way == TL_MOE_GRAD_W && (long)E * ceil_div(K, 128) * ceil_div(N, 128) >= (1L << 22)) return fail(TL_ERR_UNSUPPORTED_SHAPE, "tl_moe_gemm_query: E*K*N has 2^22 tiles or more");
  if (way == TL_MOE_GRAD_W) *ws_bytes = grad_w_shape(ctx, max_rows, K, N, E).ws_bytes;
  else *ws_bytes = product_shape(ctx, way == TL_MOE_GRAD_X, max_rows, K, N, E).ws_bytes;
  return TL_OK;
}

int tl_moe_gemm(tl_ctx* ctx, const void* x, const void* w, const int* expert_offsets, int max_rows, int K, int N, int E, void* y, void* workspace, size_t ws_bytes,
                void* stream) {
  if (int e = check_product_call(ctx, "tl_moe_gemm", TL_MOE_FORWARD, x, w, y, expert_offsets, max_rows, K, N, E, workspace, ws_bytes)) return e;
  ProductParams p;
  memset(&p, 0, sizeof p);
  p.x = (const bf16_t*)x; p.w = (const bf16_t*)w; p.out = (bf16_t*)y; p.offsets = expert_offsets;
  p.max_rows = max_rows; p.K = K; p.N = N; p.E = E;
  return launch_product<false>(ctx, p, workspace, (hipStream_t)stream);
}

int tl_moe_gemm_grad_x(tl_ctx* ctx, const void* dy, const void* w, const int* expert_offsets, int max_rows, int K, int N, int E, void* dx, void* workspace,
                       size_t ws_bytes, void* stream) {
  if (int e = check_product_call(ctx, "tl_moe_gemm_grad_x", TL_MOE_GRAD_X, dy, w, dx, expert_offsets, max_rows, K, N, E, workspace, ws_bytes)) return e;
  ProductParams p;
  memset(&p, 0, sizeof p);
  p.dy = (const bf16_t*)dy; p.w = (const bf16_t*)w; p.out = (bf16_t*)dx; p.offsets = expert_offsets;
  p.max_rows = max_rows; p.K = K; p.N = N; p.E = E;
  return launch_product<true>(ctx, p, workspace, (hipStream_t)stream);
}

int tl_moe_gemm_grad_w(tl_ctx* ctx, const void* x, const void* dy, const int* expert_offsets, int max_rows, int K, int N, int E, const float* dw_add, void* dw,
                       int dw_f32, void* workspace, size_t ws_bytes, void* stream) {
  if (int e = check_ctx(ctx)) return e;
  if (dw_add && !dw_f32) return fail(TL_ERR_INVALID_ARG, "tl_moe_gemm_grad_w: dw_add needs dw in fp32");
  if (!aligned16(dw_add)) return fail(TL_ERR_INVALID_ARG, "tl_moe_gemm_grad_w: dw_add must be 16-byte aligned");
  if (int e = check_product_call(ctx, "tl_moe_gemm_grad_w", TL_MOE_GRAD_W, x, dy, dw, expert_offsets, max_rows, K, N, E, workspace, ws_bytes)) return e;
  const GradWShape shape = grad_w_shape(ctx, max_rows, K, N, E);
  GradWParams g;
  memset(&g, 0, sizeof g);
  ProductParams& p = g.p;
  p.x = (const bf16_t*)x; p.dy = (const bf16_t*)dy; p.offsets = expert_offsets;
  p.out = (bf16_t*)dw; p.out32 = (float*)dw; p.add = dw_add;
  p.max_rows = max_rows; p.K = K; p.N = N; p.E = E;
  p.nbm = shape.nbm; p.nbn = shape.nbn;
  char* ws = (char*)workspace;
  g.plan = (GradWPlan*)ws;
  g.partial = (float*)(ws + shape.partial_at);
  g.places = shape.places;
  g.share_of = ctx->num_cus;
  g.run = shape.run;
  hipStream_t s = (hipStream_t)stream;
  if (shape.bm != shape.bn) return dw_f32 ? launch_grad_w<CfgW128x256, GradRows32>(g, shape.grid, s) : launch_grad_w<CfgW128x256, GradRows16>(g, shape.grid, s);
  if (shape.bm == 128) return dw_f32 ? launch_grad_w<CfgW128, GradRows32>(g, shape.grid, s) : launch_grad_w<CfgW128, GradRows16>(g, shape.grid, s);
  return dw_f32 ? launch_grad_w<CfgW256, GradRows32>(g, shape.grid, s) : launch_grad_w<CfgW256, GradRows16>(g, shape.grid, s);
}

}  // extern "C"
