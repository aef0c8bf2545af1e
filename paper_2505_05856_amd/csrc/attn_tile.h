// What the matrix-core attention kernels share: tiles of 64 rows brought into LDS by the load unit, their layouts and the
// addresses of their fragments, the order in which workgroups take row tiles, results turned into whole rows.
#pragma once
#include "common.h"
#include "kernels.h"

namespace dp {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int BKV = 64;    // keys (forward, dQ) or queries (dK/dV) per LDS stage
constexpr int BROWS = 128; // rows a block owns (4 waves x 32)

__device__ __forceinline__ uint4 ld16(const bf16 *p) { return *reinterpret_cast<const uint4 *>(p); }
__device__ __forceinline__ bf16x8 as_frag(uint4 v) {
  union { uint4 u; bf16x8 f; } c;
  c.u = v;
  return c.f;
}
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// elements e0..e0+7 of an MFMA result as a bf16 operand fragment
__device__ __forceinline__ bf16x8 pack8(const f32x16 &v, int e0) {
  bf16x8 r;
#pragma unroll
  for (int t = 0; t < 8; ++t) r[t] = (bf16)v[e0 + t];
  return r;
}

// Workgroups are dealt to the 8 XCDs round-robin by launch index.  This maps the launch
// index to a work index so that each XCD gets one contiguous run of work items: the
// row tiles of one (batch, head) then share K/V (or Q/dO) in a single XCD's L2
// instead of being fetched from HBM once per XCD.
__device__ __forceinline__ int xcd_contiguous(int pid, int n) {
  const int xcd = pid & 7, idx = pid >> 3, base = n >> 3, rem = n & 7;
  return xcd * base + (xcd < rem ? xcd : rem) + idx;
}

// Which row tile (rank 0: the heaviest under a causal mask) of which (batch, head) a workgroup is.
// Without an order of its own (own == 0) head after head.  A causal grid of more blocks than CUs goes by weight: the blocks of
// one head in their order gave every CU of an XCD blocks of one weight, since head lengths of 4, 8 and 16 tiles divide the 32
// CUs, and the CUs with the heavy ones ended last (batch 4, sequence 1024, 25 heads of 64: 48 tiles on some CUs where the mean
// is 27).  An XCD now takes `own` whole heads in groups of `group`, the heaviest tiles of all heads of a group first, and ahead
// of them its part of the `shared` heads that 8 XCDs cannot share out whole.  Groups hold the heads that fill the XCD's CUs, or
// whose streamed tensors fill its L2 if that is more.  Forward / backward, us, head after head and by weight:
//   batch 4, sequence 1024, 25 heads of 64: 31.7 / 83.7, 25.3 / 73.7    8, 1024, 16 of 64: 37.0 / 101.9, 28.6 / 81.1
//   batch 3, sequence 512, 25 heads of 128: 18.9 / 61.8, 15.4 / 44.2    8, 2048, 16 of 128: 162 / 559, 152 / 536
// With a block a CU at most there is nothing to share out (4, 512, 16 of 64: 9.8 / 23.8 head after head, 10.2 / 25.3 by weight).
struct RowOrder { int own, shared, group; };
template <int PER_CU> RowOrder row_order(int causal, int blocks, int tiles, int streamed, int dh) {
  constexpr int kCus = 256, kL2 = 4 << 20;
  if (!causal || blocks <= kCus || blocks / tiles < 8) return RowOrder{0, 0, 0};
  const int heads = blocks / tiles, own = heads / 8;
  int want = kL2 / 4 / (streamed * dh) > 0 ? kL2 / 4 / (streamed * dh) : 1;   // (two tensors of 2 bytes an element)
  if (want < kCus / 8 * PER_CU / tiles) want = kCus / 8 * PER_CU / tiles;
  const int groups = (own + want - 1) / want;
  return RowOrder{own, heads % 8, (own + groups - 1) / groups};
}
template <bool ORDERED> __device__ __forceinline__ void row_tile(const RowOrder &o, int pid, int n, int tiles, int *rank, int *head) {
  if (!ORDERED) {
    const int wid = xcd_contiguous(pid, n);
    *rank = wid % tiles;
    *head = wid / tiles;
    return;
  }
  const int xcd = pid & 7, mine = (n >> 3) + (xcd < (n & 7) ? 1 : 0), first = mine - o.own * tiles;
  int idx = pid >> 3;
  if (idx < first) {   // shared heads: tile by tile to the XCDs in turn
    const int j = xcd + 8 * idx;
    *rank = j / o.shared;
    *head = 8 * o.own + j % o.shared;
    return;
  }
  idx -= first;
  const int g = idx / (o.group * tiles), r = idx - g * o.group * tiles, heads = min(o.group, o.own - g * o.group);
  *rank = r / heads;
  *head = xcd * o.own + g * o.group + r % heads;
}

// Row index, inside its 32-row block, of element e of a 32x32 MFMA result held by `lane`.
__device__ __forceinline__ int acc_row(int e, int lane) { return 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3); }

// ---- K/V (or Q/dO) tiles brought into LDS by the load unit itself ------------------------
// One request: lane l fetches 16 bytes from uniform_base + byte_off and the unit stores them at
// LDS byte lds_base + 16*l (global_load_lds_dwordx4): no staging registers, no LDS store
// instructions, nothing to wait for until the tile is needed.  Invisible to the compiler's
// wait-count pass: the kernels wait with s_waitcnt vmcnt(0) themselves before the barrier that
// publishes a tile.  M0 is reserved by the compiler and nothing else in the files with these loads uses it.
__device__ __forceinline__ void dma16(unsigned lds_base, unsigned byte_off, const void *uniform_base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(lds_base), "v"(byte_off), "s"(uniform_base) : "m0", "memory");
}
__device__ __forceinline__ void wait_dma() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ const char *uniform_ptr(const char *p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const char *)(((uint64_t)hi << 32) | lo);
}

// A [64 rows][DH] tile in LDS, laid out for fragments whose contraction runs ALONG a row
// (frag_rows_sw): DH/64 half-tiles of [64][64] with unpadded 128-byte rows; 16-byte chunk c of
// row r sits at chunk position c ^ ((r >> 1) & 7), which spreads the 16 rows one fragment read
// phase touches over all banks.  The load unit writes 1 KB of consecutive LDS a request, so a
// lane fetches the global chunk that belongs at its LDS position: request q of the tile is rows
// 8q..8q+7 of half-tile q / 8; lane l is row 8q + l/8, position l%8.  Rows past `nrows` repeat
// the last row (their logits are masked; as values they meet probabilities that are zero).
// `ldb`: row stride of the source in bytes.  Every wave issues its DH/32 requests of the tile.
template <int DH>
__device__ __forceinline__ void dma_tile_rows(unsigned lds_byte, const char *src_col0, unsigned ldb, int row0, int nrows,
                                              int wave, int lane) {
  constexpr int NREQ = DH / 32;   // per wave: 64 * DH * 2 bytes / 1 KB / 4 waves
#pragma unroll
  for (int i = 0; i < NREQ; ++i) {
    const int q = wave * NREQ + i, half = q >> 3, r = 8 * (q & 7) + (lane >> 3);
    const int rg = min(row0 + r, nrows - 1);
    const unsigned chunk = (unsigned)((lane & 7) ^ ((r >> 1) & 7));
    dma16(lds_byte + (unsigned)q * 1024u, (unsigned)rg * ldb + (unsigned)half * 128u + chunk * 16u, src_col0);
  }
}
// fragment (32 rows from row0, contraction elements k0..k0+15) of such a tile
__device__ __forceinline__ bf16x8 frag_rows_sw(const unsigned char *tile, int row0, int k0, int lane) {
  const unsigned r = (unsigned)(row0 + (lane & 31));
  const unsigned c = (unsigned)(((k0 & 63) >> 3) + (lane >> 5));
  return *reinterpret_cast<const bf16x8 *>(tile + (unsigned)(k0 >> 6) * 8192u + r * 128u + ((c ^ ((r >> 1) & 7u)) << 4));
}

// The same tile laid out as loaded, [64 rows][DH * 2 bytes], for fragments whose contraction
// runs DOWN the rows (through the transpose read, which touches four consecutive
// rows x 64 bytes per 16 lanes): chunk c of row r sits at c ^ swz(r), swz = (r & 3) << 2 for
// 256-byte rows (the four rows land in the four 64-byte quarters of the bank period) and
// ((r >> 1) & 1) << 2 for 128-byte rows (rows r and r+2 swap 64-byte halves).
template <int DH> __device__ __forceinline__ constexpr unsigned swz_cols(unsigned r) {
  return DH == 128 ? (r & 3u) << 2 : ((r >> 1) & 1u) << 2;
}
template <int DH>
__device__ __forceinline__ void dma_tile_cols(unsigned lds_byte, const char *src_col0, unsigned ldb, int row0, int nrows,
                                              int wave, int lane) {
  constexpr int NREQ = DH / 32, RPR = 1024 / (DH * 2), CPR = DH / 8;   // rows per request, chunks per row
#pragma unroll
  for (int i = 0; i < NREQ; ++i) {
    const int q = wave * NREQ + i, r = RPR * q + lane / CPR;
    const int rg = min(row0 + r, nrows - 1);
    const unsigned chunk = (unsigned)(lane % CPR) ^ swz_cols<DH>((unsigned)r);
    dma16(lds_byte + (unsigned)q * 1024u, (unsigned)rg * ldb + chunk * 16u, src_col0);
  }
}
// fragment: lane l gets column col0 + l%32 for the rows r0 + 4*(l/32) + {0,1,2,3} and those 8 further
// (the order in which a 32x32 MFMA result holds 16 consecutive rows of one column)
template <int DH>
__device__ __forceinline__ bf16x8 frag_cols_sw(const unsigned char *tile, int r0, int col0, int lane) {
  constexpr unsigned ROWB = DH * 2;
  const unsigned i = (unsigned)(lane & 15), tt = i >> 2;
  const unsigned row = (unsigned)r0 + 4u * (unsigned)(lane >> 5) + tt;
  const unsigned cw = (unsigned)(col0 >> 3) + 2u * (unsigned)((lane >> 4) & 1) + ((i & 3u) >> 1);
  const unsigned char *p = tile + row * ROWB + ((cw ^ swz_cols<DH>(tt)) << 4) + (i & 1u) * 8u;
  union { s16x4 h[2]; bf16x8 v; } u;
  u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p));
  u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 8u * ROWB));
  return u.v;
}

// A [64 rows][DH] tile laid out for BOTH kinds of fragment (the backward kernels read Q, dO and
// K along the rows and down the rows): rows as loaded, chunk c of row r at position c ^ both(r),
//   256-byte rows: both(r) = ((r & 3) << 2) | ((r >> 2) & 3)    128-byte rows: (((r >> 1) & 1) << 2) | ((r >> 2) & 3)
// The high part is the column-fragment swizzle above (the four rows of a transpose read land in
// four 64-byte quarters); the low part makes the map a bijection over 16 consecutive rows, so the
// 16 rows of one row-fragment read phase cover every bank once.
template <int DH> __device__ __forceinline__ constexpr unsigned swz_both(unsigned r) {
  return swz_cols<DH>(r) | ((r >> 2) & 3u);
}
// (request i of the DH/32 a wave issues for a tile: rows past the end read the last row, so a tile
// index past the end is harmless too)
template <int DH>
__device__ __forceinline__ void dma_req_both(int i, unsigned lds_byte, const char *src_col0, unsigned ldb, int row0,
                                             int nrows, int wave, int lane) {
  constexpr int NREQ = DH / 32, RPR = 1024 / (DH * 2), CPR = DH / 8;
  const int q = wave * NREQ + i, r = RPR * q + lane / CPR;
  const int rg = min(row0 + r, nrows - 1);
  const unsigned chunk = (unsigned)(lane % CPR) ^ swz_both<DH>((unsigned)r);
  dma16(lds_byte + (unsigned)q * 1024u, (unsigned)rg * ldb + chunk * 16u, src_col0);
}
template <int DH>
__device__ __forceinline__ void dma_tile_both(unsigned lds_byte, const char *src_col0, unsigned ldb, int row0, int nrows,
                                              int wave, int lane) {
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) dma_req_both<DH>(i, lds_byte, src_col0, ldb, row0, nrows, wave, lane);
}
// A wave's 32 x DH result (lane l holds row l % 32; accumulator element e of block d is column
// 32 d + 8 (e / 4) + 4 (l / 32) + e % 4) goes out as whole rows: a store from the accumulators would
// touch 32 rows with 16 bytes each, so the tile is turned through `ew`, 64 DH bytes of LDS that only
// this wave uses (16-byte chunk c of row r at position c ^ (r % chunks a row)), and leaves as
// 16 bytes a lane, DH / 8 lanes a row.  `mul` is the lane's (its row's) factor; rows >= nrows stay unwritten.
template <int DH>
__device__ __forceinline__ void store_rows_via_lds(unsigned char *ew, const f32x16 (&acc)[DH / 32], float mul, bf16 *dst,
                                                   long ld, int nrows, int lane) {
  constexpr int ND = DH / 32, CPR = DH / 8, RPI = 64 / CPR;
  const int row = lane & 31, hh = lane >> 5;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      bf16x4 v;
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = (bf16)(acc[d][e4 * 4 + t] * mul);
      const int pos = (d * 4 + e4) ^ (row & (CPR - 1));
      *reinterpret_cast<bf16x4 *>(ew + row * (DH * 2) + pos * 16 + hh * 8) = v;
    }
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i) {
    const int r = i * RPI + lane / CPR, c = lane % CPR;
    const uint4 q = *reinterpret_cast<const uint4 *>(ew + r * (DH * 2) + ((c ^ (r & (CPR - 1))) * 16));
    if (r < nrows) *reinterpret_cast<uint4 *>(dst + (long)r * ld + c * 8) = q;
  }
}
// maximum of a value over the two halves of the wave (lanes l and l ^ 32), in every lane: the swap
// leaves lanes 0..31 of x beside lanes 32..63 of x in both registers, in the one or the other order
__device__ __forceinline__ float halves_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// The fragment addresses of such a tile, as LDS byte addresses a lane keeps in registers: the
// swizzle of a row depends on its low four bits only, so every fragment of the tile is one of
// these DH/16 (along the rows) + 2 * DH/32 (down the rows) addresses plus a compile-time offset
// (a multiple of 16 rows, another tile of the stage), which the read instruction carries.  The
// two stages lie a power of two apart: flip() moves every address to the other stage.
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) unsigned char lds_u8;
template <int DH>
struct BothAddr {
  static constexpr unsigned ROWB = DH * 2;
  unsigned row[DH / 16], col[2][DH / 32];
  __device__ __forceinline__ void init(int lane) {
    const unsigned r = (unsigned)(lane & 31), hh = (unsigned)(lane >> 5);
#pragma unroll
    for (int kd = 0; kd < DH / 16; ++kd) row[kd] = r * ROWB + (((2u * kd + hh) ^ swz_both<DH>(r)) << 4);
    const unsigned i = (unsigned)(lane & 15), tt = i >> 2, rc = 4u * hh + tt;
    const unsigned cl = 2u * (unsigned)((lane >> 4) & 1) + ((i & 3u) >> 1);
#pragma unroll
    for (int d = 0; d < DH / 32; ++d) {
      col[0][d] = rc * ROWB + (((4u * d + cl) ^ swz_both<DH>(rc)) << 4) + (i & 1u) * 8u;
      col[1][d] = (rc + 8u) * ROWB + (((4u * d + cl) ^ swz_both<DH>(rc + 8u)) << 4) + (i & 1u) * 8u;
    }
  }
  __device__ __forceinline__ void flip_cols(unsigned stage_bytes) {
#pragma unroll
    for (int d = 0; d < DH / 32; ++d) { col[0][d] ^= stage_bytes; col[1][d] ^= stage_bytes; }
  }
  __device__ __forceinline__ void flip(unsigned stage_bytes) {
#pragma unroll
    for (int kd = 0; kd < DH / 16; ++kd) row[kd] ^= stage_bytes;
    flip_cols(stage_bytes);
  }
  // 32 rows from row0 (a multiple of 16) of the tile at byte `tile_off` of the stage, contraction elements 16 kd ..
  // (tile_off, row0, r0, kd, d: constants once the callers' loops are unrolled)
  __device__ __forceinline__ bf16x8 rows(unsigned tile_off, int row0, int kd) const {
    return *(const lds_bf16x8 *)(uintptr_t)(row[kd] + tile_off + (unsigned)row0 * ROWB);
  }
  // column 32 d + lane % 32 for the rows r0 + 4 * (lane / 32) + {0,1,2,3} and those 8 further; r0 a multiple of 16
  __device__ __forceinline__ bf16x8 cols(unsigned tile_off, int r0, int d) const {
    union { s16x4 h[2]; bf16x8 v; } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(col[0][d] + tile_off + (unsigned)r0 * ROWB));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(col[1][d] + tile_off + (unsigned)r0 * ROWB));
    return u.v;
  }
};

}  // namespace
}  // namespace dp
