// What the bf16 kernels of sliding-window attention share.
#pragma once
#include "window_tile.h"

namespace dp {

namespace {

// ---- tiles whose heads may be narrower than the kernel ---------------------------------------------------
// A tile of ROWS rows from row0 on: its first row and how many more there are (a tile past the end: the last row).  Offsets count from
// the tile's own start, so a sample may span more than 4 GiB.
struct TileRows { const char *at; int more; };
__device__ __forceinline__ TileRows tile_rows(const char *src, unsigned ldb, int row0, int nrows) {
  const int first = min(row0, nrows - 1);
  return TileRows{src + (long)first * ldb, nrows - 1 - first};
}
// request i of those a wave issues for it (as dma_req_both): chunks past the head's `nch` read its first
template <int DH, int ROWS, int WAVES> constexpr int tile_reqs() { return ROWS * DH * 2 / 1024 / WAVES; }
template <int DH, int ROWS = BKV, int WAVES = 4>
__device__ __forceinline__ void dma_req(int i, unsigned lds_byte, const TileRows &rows, unsigned ldb, int nch, int wave, int lane) {
  constexpr int NREQ = tile_reqs<DH, ROWS, WAVES>(), RPR = 1024 / (DH * 2), CPR = DH / 8;
  const int q = wave * NREQ + i, r = RPR * q + lane / CPR;
  const int chunk = (int)((unsigned)(lane % CPR) ^ swz_both<DH>((unsigned)r));
  dma16(lds_byte + (unsigned)q * 1024u, (unsigned)min(r, rows.more) * ldb + (unsigned)(chunk < nch ? chunk : 0) * 16u, rows.at);
}
template <int DH, int ROWS = BKV, int WAVES = 4>
__device__ __forceinline__ void dma_tile(unsigned lds_byte, const char *src, unsigned ldb, int row0, int nrows, int nch, int wave, int lane) {
  const TileRows rows = tile_rows(src, ldb, row0, nrows);
#pragma unroll
  for (int i = 0; i < tile_reqs<DH, ROWS, WAVES>(); ++i) dma_req<DH, ROWS, WAVES>(i, lds_byte, rows, ldb, nch, wave, lane);
}
// elements 16 kd + 8 (lane / 32) .. of a row as an operand fragment, zeros past the head
__device__ __forceinline__ bf16x8 row_frag(const bf16 *row, int kd, int hh, int dh) {
  const int at = kd * 16 + 8 * hh;
  const uint4 v = ld16(row + (at < dh ? at : 0));   // (unguarded: the compiler would wait for each load on its own)
  return as_frag(at < dh ? v : make_uint4(0u, 0u, 0u, 0u));
}
// as store_rows_via_lds, for heads of `nch` 16-byte chunks; rows from `valid` on become zeros
template <int DH>
__device__ __forceinline__ void store_rows(unsigned char *ew, const f32x16 (&acc)[DH / 32], float mul, bf16 *dst, long ld, int nrows,
                                           int valid, int nch, int lane) {
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
    uint4 q = *reinterpret_cast<const uint4 *>(ew + r * (DH * 2) + ((c ^ (r & (CPR - 1))) * 16));
    if (r >= valid) q = make_uint4(0u, 0u, 0u, 0u);
    if (r < nrows && c < nch) *reinterpret_cast<uint4 *>(dst + (long)r * ld + c * 8) = q;
  }
}
// rows r0 .. r1-1 of a head become zeros (by the whole block)
__device__ __forceinline__ void zero_rows(bf16 *dst, long ld, int r0, int r1, int nch) {
  for (int i = threadIdx.x; i < (r1 - r0) * nch; i += blockDim.x) {
    const int r = r0 + i / nch, c = i % nch;
    *reinterpret_cast<uint4 *>(dst + (long)r * ld + c * 8) = make_uint4(0u, 0u, 0u, 0u);
  }
}

inline int columns(const WindowArgs &a) { return a.dh <= 64 ? 64 : 128; }
// Keys of a workgroup of dK, dV: 128, eight waves that have a CU to themselves and bring every tile once, or, where walks are short,
// 64 and four waves, two workgroups a CU, of which one works while the other starts or ends.  Backward, us, 128 and 64 keys:
//   heads of 128: 200 tokens, 8 + 2 heads, window 64: 34.1, 30.1    2 x 700, 8 + 2, 128: 44.0, 37.7    4096, 8 + 8, 512: 71.9, 60.8
//                 4 x 2048, 32 + 8, 256: 221, 211    8 x 2048, 32 + 8, 512: 587, 575    4096, 8 + 2, 1024: 88, 92    16384, 4 + 1, 4096: 418, 449
//   heads of 64:  2 x 700, 8 + 2, 128: 33.0, 27.8    4096, 8 + 8, 512: 50.7, 41.2    4 x 2048, 32 + 8, 256: 133, 121    16384, 4 + 1, 4096: 257, 268
inline int key_rows(const WindowArgs &a) {
  const int tiles = (a.S + BKV - 1) / BKV, in_window = (BROWS + a.window - 2) / BKV + 1;
  return (long)(a.nq / a.nk) * (tiles < in_window ? tiles : in_window) <= 40 ? 64 : 128;   // (items: tiles of 64 queries of a head)
}
// (An item is about 2 us, of 64 keys 1; a slot, two [ROWS][columns] arrays, about a 40th of an item of the whole chip's time.  Costs
// half or twice as high make the backwards of 24 shapes up to 2 % slower, on average.)
template <int ROWS> KeyWork work_of(const WindowArgs &a) {
  return key_work<ROWS>(a, ROWS == 64 ? 2 * kCus : kCus, Costs{3, 0.025, 2}, (int)sizeof(bf16));
}

}  // namespace

hipError_t launch_window_dkv(const WindowArgs &a, const float *drow, float *sums, hipStream_t s);   // dK and dV, after dQ

}  // namespace dp
