// Sliding-window attention in fp32 on the matrix cores (v_mfma_f32_16x16x4_f32: 2048 operations in 32 clocks, a 16th of the bf16
// rate, so the instructions beside it and the LDS hardly count and the kernels are plain ones).  A wave owns 16 rows, queries
// forward and for dQ, keys for dK and dV, which lie along the lanes of every result (lanes l, l + 16, l + 32, l + 48 share one):
// softmax sums are in-lane plus exchanges of the four, and an element of P or dS is the operand of the next product as it stands.
// 32 rows of the other side at a time come through registers into LDS, the next ones on their way while these are worked on, and
// those 16 of them that nobody in the wave sees are passed over.
//
// Operands: a fragment of a product along a row takes elements 16 j + 4 (lane / 16) + t of a row, t = 0..3 for four instructions
// (both sides the same, so the order of the sum is all it decides), one 16-byte LDS read for the four; products down the rows
// take the rows in the order a result holds them (4 (lane / 16) + e), 4 bytes a lane, lanes along a row.
//
// 2 x 512 tokens of 16 heads of 64, window 128: 15 us forward, 40 backward (30 TFLOP/s of the formula's; the floor at the rate of a
// large fp32 product, 154 TFLOP/s, is 11 for both: 2048 waves, two a SIMD, of 9 or 10 blocks of 16 x 16, half of them masked,
// backward 7 products for 5); 8 x 2048 tokens, 16 heads of 64, window 512, backward 1030 us.  Waves of 32 rows (32x32x2): 20, 58, 1116.
#include "window_tile.h"

namespace dp {

namespace {

constexpr int FR = 32, WAVES = 4, ROWS = 16 * WAVES, THREADS = 64 * WAVES;   // rows of a tile; waves, rows and threads of a block

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

// a lane's row as operand fragments (columns past the head zeros)
template <int ND> __device__ __forceinline__ void row_frags(f32x4 (&f)[2 * ND], const float *row, int quarter, int dh) {
#pragma unroll
  for (int j = 0; j < 2 * ND; ++j) {
    const int c = 16 * j + 4 * quarter;
    f[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (c < dh) f[j] = *reinterpret_cast<const f32x4 *>(row + c);
  }
}
// += <16 rows, the lane's row>
template <int ND> __device__ __forceinline__ void along(f32x4 &s, const float *rows, const f32x4 (&f)[2 * ND], int lane) {
  const float *p = rows + (lane & 15) * Tile<ND>::LD + 4 * (lane >> 4);
#pragma unroll
  for (int j = 0; j < 2 * ND; ++j) {
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p + 16 * j);
#pragma unroll
    for (int t = 0; t < 4; ++t) s = __builtin_amdgcn_mfma_f32_16x16x4f32(x[t], f[j][t], s, 0, 0, 0);
  }
}
// acc[d] += sum over 16 rows of (row's columns 16 d ..) x (the lane's weight for the row)
template <int ND> __device__ __forceinline__ void down(f32x4 (&acc)[2 * ND], const float *rows, const f32x4 &w, int lane) {
  const float *p = rows + 4 * (lane >> 4) * Tile<ND>::LD + (lane & 15);
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int d = 0; d < 2 * ND; ++d) acc[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[e * Tile<ND>::LD + 16 * d], w[e], acc[d], 0, 0, 0);
}
// -inf where the lane's four of 16 bits say hidden
__device__ __forceinline__ void hide4(f32x4 &s, uint32_t hidden, int quarter) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (hidden >> (4 * quarter + e) & 1) s[e] = -INFINITY;
}
// over the four lanes that share a row
__device__ __forceinline__ float quarters_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarters_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}
template <int N> __device__ __forceinline__ void zeros(f32x4 (&v)[N]) {
#pragma unroll
  for (int d = 0; d < N; ++d) v[d] = f32x4{0.f, 0.f, 0.f, 0.f};
}
// the lane's row of a result, times `mul`, or zeros
template <int ND>
__device__ __forceinline__ void put_row(float *row, const f32x4 (&acc)[2 * ND], float mul, bool valid, int quarter, int dh) {
#pragma unroll
  for (int d = 0; d < 2 * ND; ++d) {
    const int c = 16 * d + 4 * quarter;
    f32x4 v;
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = valid ? acc[d][u] * mul : 0.f;
    if (c < dh) *reinterpret_cast<f32x4 *>(row + c) = v;
  }
}
// whether anything of sixteen is seen by anyone in the wave
__device__ __forceinline__ bool any_seen(uint32_t hidden) { return __builtin_amdgcn_ballot_w64((hidden & 0xffffu) != 0xffffu) != 0; }

// ------------------------------------------------------------------ forward
template <int ND>
__global__ __launch_bounds__(THREADS, ND <= 2 ? 3 : 2) void window_fwd_f32_kernel(WindowArgs a) {
  __shared__ __attribute__((aligned(16))) float ks[FR * Tile<ND>::LD], vs[FR * Tile<ND>::LD];
  const int S = a.S, nqt = (S + ROWS - 1) / ROWS, wid = xcd_contiguous(blockIdx.x, gridDim.x);
  const int q0 = (nqt - 1 - wid % nqt) * ROWS, head = wid / nqt;
  const int h = head % a.nq, b = head / a.nq, kh = h / (a.nq / a.nk), len = sample_len(a, b);
  const int lane = threadIdx.x & 63, quarter = lane >> 4;
  const int qi = q0 + (int)(threadIdx.x >> 6) * 16 + (lane & 15);
  float *orow = (float *)a.o + ((long)b * S + qi) * a.ldo + (long)h * a.dh;
  float *lse = a.lse + ((long)b * a.nq + h) * S + qi;
  f32x4 acc[2 * ND];
  zeros(acc);
  float m = -1e30f, l = 0.f;   // m: running maximum of the scaled logits (log2 domain)
  if (q0 < len) {
    const float *k = (const float *)a.k + (long)b * S * a.ldk + (long)kh * a.dh, *v = (const float *)a.v + (long)b * S * a.ldv + (long)kh * a.dh;
    const float c = a.scale * kLog2e;
    const KeyTiles<FR, ROWS> kt(q0, len, a.window, a.sinks);
    f32x4 kr[Tile<ND>::PER], vr[Tile<ND>::PER], qf[2 * ND];
    Tile<ND>::ask(kr, k, a.ldk, kt.first_key(0), len, a.dh);
    Tile<ND>::ask(vr, v, a.ldv, kt.first_key(0), len, a.dh);
    row_frags<ND>(qf, (const float *)a.q + ((long)b * S + min(qi, len - 1)) * a.ldq + (long)h * a.dh, quarter, a.dh);
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
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t h16 = hidden >> (16 * u);
        if (!any_seen(h16)) continue;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        along<ND>(s, ks + 16 * u * Tile<ND>::LD, qf, lane);
        hide4(s, h16, quarter);
        const float m_new = fmaxf(m, quarters_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))) * c);
        if (__builtin_amdgcn_ballot_w64(m_new > m) != 0) {
          const float alpha = fast_exp2(m - m_new);
          l *= alpha;
#pragma unroll
          for (int d = 0; d < 2 * ND; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[d][e] *= alpha;
          m = m_new;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) { s[e] = fast_exp2(__builtin_fmaf(s[e], c, -m)); l += s[e]; }
        down<ND>(acc, vs + 16 * u * Tile<ND>::LD, s, lane);
      }
    }
  }
  l = quarters_sum(l);
  if (qi >= S) return;
  const bool valid = qi < len;
  if (a.lse != nullptr && quarter == 0) *lse = valid ? (m + __log2f(l)) * kLn2 : -INFINITY;
  if (a.o != nullptr) put_row<ND>(orow, acc, 1.0f / l, valid, quarter, a.dh);
}

// ------------------------------------------------------------------ backward: dQ, and the row dots <dO_i, O_i>
template <int ND>
__global__ __launch_bounds__(THREADS, ND <= 2 ? 3 : 2) void window_dq_f32_kernel(WindowArgs a) {
  __shared__ __attribute__((aligned(16))) float ks[FR * Tile<ND>::LD], vs[FR * Tile<ND>::LD];
  const int S = a.S, nqt = (S + ROWS - 1) / ROWS, wid = xcd_contiguous(blockIdx.x, gridDim.x);
  const int q0 = (nqt - 1 - wid % nqt) * ROWS, head = wid / nqt;
  const int h = head % a.nq, b = head / a.nq, kh = h / (a.nq / a.nk), len = sample_len(a, b);
  const int lane = threadIdx.x & 63, quarter = lane >> 4;
  const int qi = q0 + (int)(threadIdx.x >> 6) * 16 + (lane & 15);
  f32x4 acc[2 * ND];
  zeros(acc);
  if (q0 < len) {
    const float *k = (const float *)a.k + (long)b * S * a.ldk + (long)kh * a.dh, *v = (const float *)a.v + (long)b * S * a.ldv + (long)kh * a.dh;
    const float c = a.scale * kLog2e;
    const KeyTiles<FR, ROWS> kt(q0, len, a.window, a.sinks);
    f32x4 kr[Tile<ND>::PER], vr[Tile<ND>::PER], qf[2 * ND], gf[2 * ND];
    Tile<ND>::ask(kr, k, a.ldk, kt.first_key(0), len, a.dh);
    Tile<ND>::ask(vr, v, a.ldv, kt.first_key(0), len, a.dh);
    const long row = (long)b * S + min(qi, len - 1), at_o = row * a.ldo + (long)h * a.dh;
    row_frags<ND>(qf, (const float *)a.q + row * a.ldq + (long)h * a.dh, quarter, a.dh);
    row_frags<ND>(gf, (const float *)a.d_o + at_o, quarter, a.dh);
    float dsum = 0.f;
#pragma unroll
    for (int j = 0; j < 2 * ND; ++j) {
      const int col = 16 * j + 4 * quarter;
      if (col < a.dh) {
        const f32x4 o = *reinterpret_cast<const f32x4 *>((const float *)a.o_in + at_o + col);
#pragma unroll
        for (int t = 0; t < 4; ++t) dsum += o[t] * gf[j][t];
      }
    }
    dsum = quarters_sum(dsum);
    const long row_at = ((long)b * a.nq + h) * S + qi;
    if (qi < len && quarter == 0) a.ws[row_at] = dsum;
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
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t h16 = hidden >> (16 * u);
        if (!any_seen(h16)) continue;
        f32x4 s = {0.f, 0.f, 0.f, 0.f}, dp = {-dsum, -dsum, -dsum, -dsum};
        along<ND>(s, ks + 16 * u * Tile<ND>::LD, qf, lane);
        along<ND>(dp, vs + 16 * u * Tile<ND>::LD, gf, lane);
        hide4(s, h16, quarter);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[e] *= fast_exp2(__builtin_fmaf(s[e], c, -lq));
        down<ND>(acc, ks + 16 * u * Tile<ND>::LD, dp, lane);
      }
    }
  }
  if (qi < S) put_row<ND>((float *)a.dq + ((long)b * S + qi) * a.ldq + (long)h * a.dh, acc, a.scale, qi < len, quarter, a.dh);
}

// ------------------------------------------------------------------ backward: dK and dV
// Pieces of walks as in bf16; an item (64 queries of one head) goes in two tiles.
template <int ND>
__global__ __launch_bounds__(THREADS, ND <= 2 ? 3 : 2) void window_dkv_f32_kernel(WindowArgs a, KeyWork w, const float *__restrict__ drow,
                                                                            float *__restrict__ sums) {
  __shared__ __attribute__((aligned(16))) float qs[FR * Tile<ND>::LD], gs[FR * Tile<ND>::LD];
  __shared__ __attribute__((aligned(16))) float rows[2][FR];   // log-sum-exps (log2 domain) and row dots, negated
  constexpr int HALVES = ND == 4 ? 1 : 2;   // of a tile at once (128 columns: two spill)
  const int S = a.S, group = a.nq / a.nk;
  const Piece at = piece_at(w, blockIdx.x, a.B * a.nk);
  const int head = at.head, kb = at.kb, piece = at.piece;
  const int kh = head % a.nk, b = head / a.nk, len = sample_len(a, b);
  const int lane = threadIdx.x & 63, quarter = lane >> 4;
  const int in_block = (int)(threadIdx.x >> 6) * 16 + (lane & 15), kj = kb * ROWS + in_block;
  const long slot = slot_of(w, head, kb, piece);
  f32x4 dk[2 * ND], dv[2 * ND];
  zeros(dk);
  zeros(dv);
  if (kb * ROWS < len) {
    const Walk walk = walk_of<ROWS>(w, kb, piece, len, a.window, group);
    if (slot >= 0 && walk.begin == walk.end) return;   // (the kernel that adds the pieces up knows)
    const long row = (long)b * S + min(kj, len - 1);
    const float c = a.scale * kLog2e;
    f32x4 qr[Tile<ND>::PER], gr[Tile<ND>::PER], kf[2 * ND], vf[2 * ND];
    row_frags<ND>(kf, (const float *)a.k + row * a.ldk + (long)kh * a.dh, quarter, a.dh);
    row_frags<ND>(vf, (const float *)a.v + row * a.ldv + (long)kh * a.dh, quarter, a.dh);
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
#pragma unroll HALVES
      for (int u = 0; u < 2; ++u) {
        const uint32_t h16 = hidden >> (16 * u);
        if (ib + 16 * u >= len || !any_seen(h16)) continue;
        const f32x4 ls = *reinterpret_cast<const f32x4 *>(&rows[0][16 * u + 4 * quarter]);
        f32x4 s = {0.f, 0.f, 0.f, 0.f}, dp = *reinterpret_cast<const f32x4 *>(&rows[1][16 * u + 4 * quarter]);
        along<ND>(s, qs + 16 * u * Tile<ND>::LD, kf, lane);
        along<ND>(dp, gs + 16 * u * Tile<ND>::LD, vf, lane);
        hide4(s, h16, quarter);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[e] = fast_exp2(__builtin_fmaf(s[e], c, -ls[e]));
          dp[e] *= s[e];
        }
        down<ND>(dv, gs + 16 * u * Tile<ND>::LD, s, lane);
        down<ND>(dk, qs + 16 * u * Tile<ND>::LD, dp, lane);
      }
    }
  }
  if (slot >= 0) {
    if (kb * ROWS >= len) return;
    float *out = sums + slot * (2 * ROWS * 32 * ND) + in_block * (32 * ND);
    put_row<ND>(out, dk, 1.f, true, quarter, 32 * ND);
    put_row<ND>(out + ROWS * 32 * ND, dv, 1.f, true, quarter, 32 * ND);
  } else if (kj < S) {
    put_row<ND>((float *)a.dk + ((long)b * S + kj) * a.ldk + (long)kh * a.dh, dk, a.scale, kj < len, quarter, a.dh);
    put_row<ND>((float *)a.dv + ((long)b * S + kj) * a.ldv + (long)kh * a.dh, dv, 1.f, kj < len, quarter, a.dh);
  }
}

// (Workgroups at once: two a CU at up to 64 columns, else one.  An item is about 8 us at 64 columns, a slot two [64][64] arrays.)
KeyWork work_of(const WindowArgs &a) { return key_work<ROWS>(a, kCus * (a.dh <= 64 ? 2 : 1), Costs{0.4, 0.002, 0.4}, (int)sizeof(float)); }

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
  hipLaunchKernelGGL((window_dkv_sum_kernel<float, ROWS, 32 * ND>), dim3(heads * cut * 2 * (ROWS / kSumRows)), dim3(kSumRows * 8 * ND), 0, s, a, w, sums, cut);
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
