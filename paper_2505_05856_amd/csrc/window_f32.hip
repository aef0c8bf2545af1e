// Sliding-window attention in fp32 on the matrix cores (v_mfma_f32_32x32x2_f32: 4096 operations in 64 clocks, a 16th of the bf16
// rate, so the instructions beside it and the LDS hardly count and the kernels are plain ones).  A wave owns 32 rows, queries
// forward and for dQ, keys for dK and dV, which lie along the lanes of every result: softmax sums are in-lane plus one exchange
// of the half waves, and an element of P or dS is the operand of the next product as it stands.  32 rows of the other side at a
// time come through registers into LDS, the next ones on their way while these are worked on.
//
// Operands: a fragment of a product along a row takes elements 8 j + 4 (lane / 32) + t of a row, t = 0..3 for four instructions
// (both sides the same, so the order of the sum is all it decides), one 16-byte LDS read for the four; products down the rows
// take the rows in the order a result holds them (acc_row), 4 bytes a lane, lanes along a row.
#include "window_tile.h"

namespace dp {

namespace {

constexpr int FR = 32, WAVES = 2, ROWS = 32 * WAVES, THREADS = 64 * WAVES;   // rows of a tile; waves, rows and threads of a block

// A tile of FR rows in LDS, rows of ND * 32 columns and 4 more (16 rows' 16-byte reads then start in 16 different places)
template <int ND> struct Tile {
  static constexpr int LD = 32 * ND + 4, PER = FR * 8 * ND / THREADS;   // PER: 16-byte pieces a thread brings
  // rows r0 .. r0+31 of a head on their way: rows past the end are the last one, columns past the head zeros
  static __device__ __forceinline__ void ask(f32x4 (&v)[PER], const float *src, long ld, int r0, int nrows, int dh) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int p = threadIdx.x + THREADS * i, r = min(r0 + p / (8 * ND), nrows - 1), c = (p % (8 * ND)) * 4;
      v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (c < dh) v[i] = *reinterpret_cast<const f32x4 *>(src + (long)r * ld + c);
    }
  }
  static __device__ __forceinline__ void put(const f32x4 (&v)[PER], float *lds) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int p = threadIdx.x + THREADS * i;
      *reinterpret_cast<f32x4 *>(lds + (p / (8 * ND)) * LD + (p % (8 * ND)) * 4) = v[i];
    }
  }
};

// a wave's row as operand fragments (columns past the head zeros)
template <int ND> __device__ __forceinline__ void row_frags(f32x4 (&f)[4 * ND], const float *row, int hh, int dh) {
#pragma unroll
  for (int j = 0; j < 4 * ND; ++j) {
    const int c = 8 * j + 4 * hh;
    f[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (c < dh) f[j] = *reinterpret_cast<const f32x4 *>(row + c);
  }
}
// += <rows of the tile, the lane's row>
template <int ND> __device__ __forceinline__ void along(f32x16 &s, const float *tile, const f32x4 (&f)[4 * ND], int lane) {
  const float *p = tile + (lane & 31) * Tile<ND>::LD + 4 * (lane >> 5);
#pragma unroll
  for (int j = 0; j < 4 * ND; ++j) {
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p + 8 * j);
#pragma unroll
    for (int t = 0; t < 4; ++t) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[t], f[j][t], s, 0, 0, 0);
  }
}
// acc[d] += sum over the tile's rows of (row's columns 32 d ..) x (the lane's weight for the row)
template <int ND> __device__ __forceinline__ void down(f32x16 (&acc)[ND], const float *tile, const f32x16 &w, int lane) {
  const float *p = tile + 4 * (lane >> 5) * Tile<ND>::LD + (lane & 31);
#pragma unroll
  for (int e = 0; e < 16; ++e)
#pragma unroll
    for (int d = 0; d < ND; ++d)
      acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(p[(8 * (e >> 2) + (e & 3)) * Tile<ND>::LD + 32 * d], w[e], acc[d], 0, 0, 0);
}
__device__ __forceinline__ void zero16(f32x16 &v) {
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = 0.f;
}
// the lane's row of a result, times `mul`, or zeros
template <int ND>
__device__ __forceinline__ void put_row(float *row, const f32x16 (&acc)[ND], float mul, bool valid, int hh, int dh) {
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const int c = 32 * d + 8 * e4 + 4 * hh;
      f32x4 v;
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = valid ? acc[d][4 * e4 + u] * mul : 0.f;
      if (c < dh) *reinterpret_cast<f32x4 *>(row + c) = v;
    }
}

// ------------------------------------------------------------------ forward
template <int ND>
__global__ __launch_bounds__(THREADS, ND <= 2 ? 2 : 1) void window_fwd_f32_kernel(WindowArgs a) {
  __shared__ __attribute__((aligned(16))) float ks[FR * Tile<ND>::LD], vs[FR * Tile<ND>::LD];
  const int S = a.S, nqt = (S + ROWS - 1) / ROWS, wid = xcd_contiguous(blockIdx.x, gridDim.x);
  const int q0 = (nqt - 1 - wid % nqt) * ROWS, head = wid / nqt;
  const int h = head % a.nq, b = head / a.nq, kh = h / (a.nq / a.nk), len = sample_len(a, b);
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int qi = q0 + (int)(threadIdx.x >> 6) * 32 + (lane & 31);
  float *orow = (float *)a.o + ((long)b * S + qi) * a.ldo + (long)h * a.dh;
  float *lse = a.lse + ((long)b * a.nq + h) * S + qi;
  f32x16 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) zero16(acc[d]);
  float m = -1e30f, l = 0.f;   // m: running maximum of the scaled logits (log2 domain)
  if (q0 < len) {
    const float *k = (const float *)a.k + (long)b * S * a.ldk + (long)kh * a.dh, *v = (const float *)a.v + (long)b * S * a.ldv + (long)kh * a.dh;
    const float c = a.scale * kLog2e;
    const KeyTiles<FR, ROWS> kt(q0, len, a.window, a.sinks);
    f32x4 kr[Tile<ND>::PER], vr[Tile<ND>::PER], qf[4 * ND];
    Tile<ND>::ask(kr, k, a.ldk, kt.first_key(0), len, a.dh);
    Tile<ND>::ask(vr, v, a.ldv, kt.first_key(0), len, a.dh);
    row_frags<ND>(qf, (const float *)a.q + ((long)b * S + min(qi, len - 1)) * a.ldq + (long)h * a.dh, hh, a.dh);
    for (int t = 0; t < kt.n; ++t) {
      __syncthreads();   // everyone is done with the tile before
      Tile<ND>::put(kr, ks);
      Tile<ND>::put(vr, vs);
      __syncthreads();
      if (t + 1 < kt.n) {
        Tile<ND>::ask(kr, k, a.ldk, kt.first_key(t + 1), len, a.dh);
        Tile<ND>::ask(vr, v, a.ldv, kt.first_key(t + 1), len, a.dh);
      }
      const uint32_t hidden = hidden_keys(qi, kt.first_key(t), a.window, a.sinks);
      if (__builtin_amdgcn_ballot_w64(hidden != ~0u) == 0) continue;   // (no query of the wave sees a key of the tile)
      f32x16 s;
      zero16(s);
      along<ND>(s, ks, qf, lane);
      hide(s, hidden, hh);
      float mx = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
      const float m_new = fmaxf(m, halves_max(mx) * c);
      if (__builtin_amdgcn_ballot_w64(m_new > m) != 0) {
        const float alpha = fast_exp2(m - m_new);
        l *= alpha;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
        m = m_new;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) { s[e] = fast_exp2(__builtin_fmaf(s[e], c, -m)); l += s[e]; }
      down<ND>(acc, vs, s, lane);
    }
  }
  l += __shfl_xor(l, 32, 64);
  if (qi >= S) return;
  const bool valid = qi < len;
  if (a.lse != nullptr && hh == 0) *lse = valid ? (m + __log2f(l)) * kLn2 : -INFINITY;
  if (a.o != nullptr) put_row<ND>(orow, acc, 1.0f / l, valid, hh, a.dh);
}

// ------------------------------------------------------------------ backward: dQ, and the row dots <dO_i, O_i>
template <int ND>
__global__ __launch_bounds__(THREADS, ND <= 2 ? 2 : 1) void window_dq_f32_kernel(WindowArgs a) {
  __shared__ __attribute__((aligned(16))) float ks[FR * Tile<ND>::LD], vs[FR * Tile<ND>::LD];
  const int S = a.S, nqt = (S + ROWS - 1) / ROWS, wid = xcd_contiguous(blockIdx.x, gridDim.x);
  const int q0 = (nqt - 1 - wid % nqt) * ROWS, head = wid / nqt;
  const int h = head % a.nq, b = head / a.nq, kh = h / (a.nq / a.nk), len = sample_len(a, b);
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int qi = q0 + (int)(threadIdx.x >> 6) * 32 + (lane & 31);
  f32x16 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) zero16(acc[d]);
  if (q0 < len) {
    const float *k = (const float *)a.k + (long)b * S * a.ldk + (long)kh * a.dh, *v = (const float *)a.v + (long)b * S * a.ldv + (long)kh * a.dh;
    const float c = a.scale * kLog2e;
    const KeyTiles<FR, ROWS> kt(q0, len, a.window, a.sinks);
    f32x4 kr[Tile<ND>::PER], vr[Tile<ND>::PER], qf[4 * ND], gf[4 * ND];
    Tile<ND>::ask(kr, k, a.ldk, kt.first_key(0), len, a.dh);
    Tile<ND>::ask(vr, v, a.ldv, kt.first_key(0), len, a.dh);
    const long row = (long)b * S + min(qi, len - 1), at_o = row * a.ldo + (long)h * a.dh;
    row_frags<ND>(qf, (const float *)a.q + row * a.ldq + (long)h * a.dh, hh, a.dh);
    row_frags<ND>(gf, (const float *)a.d_o + at_o, hh, a.dh);
    float dsum = 0.f;
#pragma unroll
    for (int j = 0; j < 4 * ND; ++j) {
      const int col = 8 * j + 4 * hh;
      if (col < a.dh) {
        const f32x4 o = *reinterpret_cast<const f32x4 *>((const float *)a.o_in + at_o + col);
#pragma unroll
        for (int t = 0; t < 4; ++t) dsum += o[t] * gf[j][t];
      }
    }
    dsum += __shfl_xor(dsum, 32, 64);
    const long row_at = ((long)b * a.nq + h) * S + qi;
    if (qi < len && hh == 0) a.ws[row_at] = dsum;
    const float lq = qi < len ? a.lse[row_at] * kLog2e : INFINITY;
    for (int t = 0; t < kt.n; ++t) {
      __syncthreads();
      Tile<ND>::put(kr, ks);
      Tile<ND>::put(vr, vs);
      __syncthreads();
      if (t + 1 < kt.n) {
        Tile<ND>::ask(kr, k, a.ldk, kt.first_key(t + 1), len, a.dh);
        Tile<ND>::ask(vr, v, a.ldv, kt.first_key(t + 1), len, a.dh);
      }
      const uint32_t hidden = hidden_keys(qi, kt.first_key(t), a.window, a.sinks);
      if (__builtin_amdgcn_ballot_w64(hidden != ~0u) == 0) continue;
      f32x16 s, dp;
      zero16(s);
#pragma unroll
      for (int e = 0; e < 16; ++e) dp[e] = -dsum;
      along<ND>(s, ks, qf, lane);
      along<ND>(dp, vs, gf, lane);
      hide(s, hidden, hh);
#pragma unroll
      for (int e = 0; e < 16; ++e) dp[e] *= fast_exp2(__builtin_fmaf(s[e], c, -lq));
      down<ND>(acc, ks, dp, lane);
    }
  }
  if (qi < S) put_row<ND>((float *)a.dq + ((long)b * S + qi) * a.ldq + (long)h * a.dh, acc, a.scale, qi < len, hh, a.dh);
}

// ------------------------------------------------------------------ backward: dK and dV
// Pieces of walks as in bf16; an item (64 queries of one head) goes in two tiles.
template <int ND>
__global__ __launch_bounds__(THREADS, ND <= 2 ? 2 : 1) void window_dkv_f32_kernel(WindowArgs a, KeyWork w, const float *__restrict__ drow,
                                                                            float *__restrict__ sums) {
  __shared__ __attribute__((aligned(16))) float qs[FR * Tile<ND>::LD], gs[FR * Tile<ND>::LD];
  __shared__ __attribute__((aligned(16))) float rows[2][FR];   // log-sum-exps (log2 domain) and row dots, negated
  const int S = a.S, group = a.nq / a.nk;
  const Piece at = piece_at(w, blockIdx.x, a.B * a.nk);
  const int head = at.head, kb = at.kb, piece = at.piece;
  const int kh = head % a.nk, b = head / a.nk, len = sample_len(a, b);
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  const int in_block = (int)(threadIdx.x >> 6) * 32 + (lane & 31), kj = kb * ROWS + in_block;
  const long slot = slot_of(w, head, kb, piece);
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) { zero16(dk[d]); zero16(dv[d]); }
  if (kb * ROWS < len) {
    const Walk walk = walk_of<ROWS>(w, kb, piece, len, a.window, group);
    if (slot >= 0 && walk.begin == walk.end) return;   // (the kernel that adds the pieces up knows)
    const long row = (long)b * S + min(kj, len - 1);
    const float c = a.scale * kLog2e;
    f32x4 qr[Tile<ND>::PER], gr[Tile<ND>::PER], kf[4 * ND], vf[4 * ND];
    row_frags<ND>(kf, (const float *)a.k + row * a.ldk + (long)kh * a.dh, hh, a.dh);
    row_frags<ND>(vf, (const float *)a.v + row * a.ldv + (long)kh * a.dh, hh, a.dh);
    float rl = 0.f;   // threads 0..31 carry a tile's log-sum-exps, 32..63 its row dots
    int i0 = 0;       // first query of the tile asked for last
    auto ask = [&](int half) {   // tile half % 2 of item half / 2
      const int it = half >> 1, g = it / walk.nt, h = kh * group + g;
      i0 = (walk.t0 + it - g * walk.nt) * BKV + (half & 1) * FR;
      Tile<ND>::ask(qr, (const float *)a.q + (long)b * S * a.ldq + (long)h * a.dh, a.ldq, i0, len, a.dh);
      Tile<ND>::ask(gr, (const float *)a.d_o + (long)b * S * a.ldo + (long)h * a.dh, a.ldo, i0, len, a.dh);
      if (threadIdx.x < 2 * FR) {
        const int i = i0 + (threadIdx.x & 31);
        const float *src = (threadIdx.x < FR ? a.lse : drow) + ((long)b * a.nq + h) * S;
        const float x = src[min(i, len - 1)];
        rl = threadIdx.x < FR ? (i < len ? x * kLog2e : INFINITY) : (i < len ? -x : 0.f);   // (rows past the end: P = 0)
      }
    };
    const int n0 = 2 * walk.begin, n1 = 2 * walk.end;
    if (n0 < n1) ask(n0);
    for (int half = n0; half < n1; ++half) {
      __syncthreads();
      Tile<ND>::put(qr, qs);
      Tile<ND>::put(gr, gs);
      if (threadIdx.x < 2 * FR) rows[threadIdx.x >> 5][threadIdx.x & 31] = rl;
      const int ib = i0;
      __syncthreads();
      if (half + 1 < n1) ask(half + 1);
      const uint32_t hidden = hidden_queries(kj, ib, a.window, a.sinks);
      if (ib >= len || __builtin_amdgcn_ballot_w64(hidden != ~0u) == 0) continue;
      f32x16 s, dp, ls;
      zero16(s);
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(&rows[0][8 * e4 + 4 * hh]), y = *reinterpret_cast<const f32x4 *>(&rows[1][8 * e4 + 4 * hh]);
#pragma unroll
        for (int u = 0; u < 4; ++u) { ls[4 * e4 + u] = x[u]; dp[4 * e4 + u] = y[u]; }
      }
      along<ND>(s, qs, kf, lane);
      along<ND>(dp, gs, vf, lane);
      hide(s, hidden, hh);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = fast_exp2(__builtin_fmaf(s[e], c, -ls[e]));
        dp[e] *= s[e];
      }
      down<ND>(dv, gs, s, lane);
      down<ND>(dk, qs, dp, lane);
    }
  }
  if (slot >= 0) {
    if (kb * ROWS >= len) return;
    float *out = sums + slot * (2 * ROWS * 32 * ND) + in_block * (32 * ND);
    put_row<ND>(out, dk, 1.f, true, hh, 32 * ND);
    put_row<ND>(out + ROWS * 32 * ND, dv, 1.f, true, hh, 32 * ND);
  } else if (kj < S) {
    put_row<ND>((float *)a.dk + ((long)b * S + kj) * a.ldk + (long)kh * a.dh, dk, a.scale, kj < len, hh, a.dh);
    put_row<ND>((float *)a.dv + ((long)b * S + kj) * a.ldv + (long)kh * a.dh, dv, 1.f, kj < len, hh, a.dh);
  }
}

// (Waves at once: two a SIMD at up to 64 columns, else one.  An item is about 8 us at 64 columns, a slot two [64][64] arrays.)
KeyWork work_of(const WindowArgs &a) { return key_work<ROWS>(a, kCus * 4 / WAVES * (a.dh <= 64 ? 2 : 1), Costs{0.4, 0.002, 0.4}); }

template <int ND> hipError_t fwd(const WindowArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((window_fwd_f32_kernel<ND>), dim3((a.S + ROWS - 1) / ROWS * a.nq * a.B), dim3(THREADS), 0, s, a);
  return hipGetLastError();
}
template <int ND> hipError_t bwd(const WindowArgs &a, hipStream_t s) {
  const KeyWork w = work_of(a);
  hipLaunchKernelGGL((window_dq_f32_kernel<ND>), dim3((a.S + ROWS - 1) / ROWS * a.nq * a.B), dim3(THREADS), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  float *sums = (float *)((char *)a.ws + dots_bytes(a));
  const int heads = a.B * a.nk;
  hipLaunchKernelGGL((window_dkv_f32_kernel<ND>), dim3((unsigned)(heads * pieces_of(w))), dim3(THREADS), 0, s, a, w, a.ws, sums);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int cut = key_blocks_cut(w);
  if (cut == 0) return hipSuccess;
  hipLaunchKernelGGL((window_dkv_sum_kernel<float, ROWS, 32 * ND>), dim3(heads * cut * 2 * (ROWS / 32)), dim3(256), 0, s, a, w, sums, cut);
  return hipGetLastError();
}
int blocks_of_32(const WindowArgs &a) { return (a.dh + 31) / 32; }
bool aligned(const void *p, long ld) { return ((uintptr_t)p & 15) == 0 && ld % 4 == 0; }

}  // namespace

bool window_f32_supported(const WindowArgs &a) {
  return a.dh <= 128 && aligned(a.q, a.ldq) && aligned(a.k, a.ldk) && aligned(a.v, a.ldv) && aligned(a.o, a.ldo) && aligned(a.o_in, a.ldo) &&
         aligned(a.d_o, a.ldo) && aligned(a.dq, a.ldq) && aligned(a.dk, a.ldk) && aligned(a.dv, a.ldv) && ((uintptr_t)a.ws & 15) == 0;
}
size_t window_f32_ws_bytes(const WindowArgs &a) {
  return a.dh > 128 ? 0 : dots_bytes(a) + slots_of(a, work_of(a)) * 2 * ROWS * 32 * (size_t)blocks_of_32(a) * sizeof(float);
}
hipError_t launch_window_fwd_f32(const WindowArgs &a, hipStream_t s) {
  switch (blocks_of_32(a)) { case 1: return fwd<1>(a, s); case 2: return fwd<2>(a, s); case 3: return fwd<3>(a, s); default: return fwd<4>(a, s); }
}
hipError_t launch_window_bwd_f32(const WindowArgs &a, hipStream_t s) {
  switch (blocks_of_32(a)) { case 1: return bwd<1>(a, s); case 2: return bwd<2>(a, s); case 3: return bwd<3>(a, s); default: return bwd<4>(a, s); }
}

}  // namespace dp
