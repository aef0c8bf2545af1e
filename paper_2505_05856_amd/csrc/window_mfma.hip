// Sliding-window attention on the matrix cores (bf16 in, fp32 accumulate): query i of a sample sees key j when j <= i < len and
// (i - j < window or j < sinks).  The tiles and layouts are those of the full attention; what is different:
//
// - A block of 128 queries walks two runs of key tiles, those that hold the first keys and those of its window, as one list: the
//   loads of the second run's start are in flight while the first run ends.
// - Which keys of 32 a lane's query sees is a 32-bit word (three shifts), from which each logit takes a bit: two instructions a
//   logit, as a causal mask alone would take, and only where 32 keys hold one that is hidden from one of a wave's queries.  32
//   keys that are hidden from all of them are passed over (dQ, dK and dV, and the forward of short windows).
// - Query heads that share a key head are separate blocks forward and for dQ (next to each other, so one L2 serves their keys);
//   dK and dV walk the queries of all of them, tile after tile, so no gradient is added up outside a block ...
// - ... unless that leaves CUs idle, or keys are seen by every later query (the first ones): such a walk is cut into parts of
//   about the length of the others; each leaves fp32 sums in the workspace, and a last kernel adds them in a fixed order.
// - Rows past a sample's length are never read (tiles end with copies of the last row, whose products are masked) and become 0.
// - Head dimensions of 8..128: kernels for 64 and 128 columns; columns past the head are zeros on the side that waits in
//   registers and copies of the first ones in LDS, and are not stored.
//
// Measured at 8 x 2048 tokens of 32 + 8 heads of 128, window 512, 16 first keys: 175 us forward (124 GFLOP for the pairs that are
// seen, 705 TFLOP/s, where a large matrix product reaches 1606) and 575 backward (537 TFLOP/s of the formula's; S and dP are taken
// twice); 16384 tokens of 4 + 1 heads, window 4096: 131 (920 TFLOP/s) and 422.  Of a SIMD's time forward, dQ, dK/dV there the
// matrix pipe works 35, 34 and 42 % (45, 48 and 47 % at the long window), the vector ALU 44, 33 and 35 %, LDS 20, 19 and 33 %:
// none of them bounds the kernels alone.  The rest are a wave's own dependences, products to softmax to products, which two or
// three waves a SIMD do not fill, blocks' starts and ends, and tiles of which the mask leaves a part.
// What lost: 64 rows a wave (half the LDS reads, one wave a SIMD: forward 224 us for 197, dQ 338 for 294, dK/dV 587 for 450);
// loads two tiles ahead (forward 175, dK/dV 6 % slower, spills); lane offsets of the loads worked out once (no change); dQ by
// tiles of 32 keys (backward 591 for 575).
#include "window_bf16.h"

#include <type_traits>

namespace dp {

namespace {

// ------------------------------------------------------------------ forward, many blocks and short windows
// Tiles of 32 keys, one after the other, and none that the window or the order of the tokens hides from all of a wave's queries: of
// a window of 512 the pipeline below takes 704 keys a query, this 560.  What hides the softmax are two (64 columns: three) more
// waves on the SIMD, which half as much LDS leaves room for; where a CU has fewer blocks than that, or the window is long, the
// pipeline is ahead.  The pipeline and this, us (heads of 128 with a quarter as many key heads):
//   blocks of 128 queries       window 64       256           1024          4096
//   256 (4096 tokens, 8 heads)  11.1, 11.1      14.5, 15.5    27.0, 30.8    72.9, 86.9
//   1024 (2 x 4096, 16)         27.0, 24.6      36.9, 38.0    76.7, 81.9    143, 163
//   2048 (4 x 2048, 32)         48.6, 42.5      67.4, 59.1    127, 122      151, 160
//   4096 (8 x 2048, 32)         105, 94.6       144, 125      255, 242      304, 303
// Heads of 64:  1024 blocks     15.8, 14.9      24.4, 20.8    50.9, 47.3    85.3, 89.4
//   4096                        52.3, 41.3      74.5, 64.3    141, 139      173, 174
constexpr int KEYS = 32;
bool by_blocks(const WindowArgs &a, int blocks) { return blocks > 2 * kCus && a.window <= 512; }
template <int DH>
__global__ __launch_bounds__(256, DH == 64 ? 4 : 3) void window_fwd_blocks_kernel(WindowArgs a, RowOrder ro) {
  constexpr int ND = DH / 32, NK = DH / 16;
  // LDS, in bytes: [stage 0: K, V][stage 1: K, V]
  constexpr unsigned TILE = KEYS * DH * 2, STAGE = 2 * TILE;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_b[];

  const int S = a.S, nqt = (S + BROWS - 1) / BROWS, nch = a.dh / 8;
  int rank, head;
  if (ro.own > 0) row_tile<true>(ro, blockIdx.x, gridDim.x, nqt, &rank, &head);
  else row_tile<false>(ro, blockIdx.x, gridDim.x, nqt, &rank, &head);
  const int q0 = (nqt - 1 - rank) * BROWS;   // (late tiles are the heavy ones)
  const int h = head % a.nq, b = head / a.nq, kh = h / (a.nq / a.nk);
  const int len = sample_len(a, b);
  const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int iw0 = q0 + wave * 32, qi = iw0 + (lane & 31);
  bf16 *ob = (bf16 *)a.o + (long)b * S * a.ldo + (long)h * a.dh;
  float *lb = a.lse + ((long)b * a.nq + h) * S;
  if (q0 >= len) {
    const int r1 = min(q0 + BROWS, S);
    if (a.o != nullptr) zero_rows(ob, a.ldo, q0, r1, nch);
    if (a.lse != nullptr && q0 + tid < r1) lb[q0 + tid] = -INFINITY;
    return;
  }
  const bf16 *qb = (const bf16 *)a.q + (long)b * S * a.ldq + (long)h * a.dh;
  const char *kb = uniform_ptr((const char *)((const bf16 *)a.k + (long)b * S * a.ldk + (long)kh * a.dh));
  const char *vb = uniform_ptr((const char *)((const bf16 *)a.v + (long)b * S * a.ldv + (long)kh * a.dh));
  const unsigned ldkb = (unsigned)a.ldk * 2u, ldvb = (unsigned)a.ldv * 2u;
  const float c = a.scale * kLog2e;
  const int window = a.window, sinks = a.sinks;
  const KeyTiles<KEYS, BROWS> kt(q0, len, window, sinks);
  auto fetch = [&](int t, unsigned buf) {
    const int j0 = kt.first_key(t);
    dma_tile<DH, KEYS, 4>(buf, kb, ldkb, j0, len, nch, wave, lane);
    dma_tile<DH, KEYS, 4>(buf + TILE, vb, ldvb, j0, len, nch, wave, lane);
  };
  fetch(0, 0u);

  bf16x8 qf[NK];
  const bf16 *qrow = qb + (long)min(qi, len - 1) * a.ldq;   // (a query past the end reads the last row, and nothing of it is stored)
#pragma unroll
  for (int kd = 0; kd < NK; ++kd) qf[kd] = row_frag(qrow, kd, hh, a.dh);

  f32x16 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
  float m = -1e30f, l = 0.f;   // m: reference point of the exponents (log2 domain)

  BothAddr<DH> at;
  at.init(lane);
  wait_dma();
#pragma unroll
  for (int kd = 0; kd < NK; ++kd) asm volatile("" ::"v"(qf[kd]));   // (the fragments are waited for here, not in the tile loop)
  __syncthreads();

  constexpr int AHEAD = 3, RING = 4;
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  // keys jb .. jb+31, a tile
  auto block = [&](auto stage_tag, int jb) {
    constexpr unsigned base = decltype(stage_tag)::value * STAGE;
    bf16x8 fx[RING];
    auto ld_rows = [&](int i) { if (i < NK) fx[i % RING] = at.rows(base, 0, i); };
    auto ld_cols = [&](int i) { if (i < NK) fx[i % RING] = at.cols(base + TILE, (i / ND) * 16, i % ND); };
    f32x16 s;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ld_rows(i);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      ld_rows(i + AHEAD);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], qf[i], s, 0, 0, 0);
      fence();
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ld_cols(i);
    if (jb + 31 > iw0 || (iw0 + 31 - jb >= window && jb + 32 > sinks)) hide(s, hidden_keys(qi, jb, window, sinks), hh);
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
    const float m_new = fmaxf(m, halves_max(mx) * c);
    constexpr float kLag = 8.f;   // (the reference point follows the maximum only when it is left behind by a factor of 2^8)
    if (__builtin_amdgcn_ballot_w64(m_new > m + kLag) != 0) {
      const float alpha = fast_exp2(m - m_new);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
      m = m_new;
    }
    bf16x8 pf[2];
    float ps = 0.f;
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2) {
#pragma unroll
      for (int e = 8 * h2; e < 8 * h2 + 8; ++e) {
        s[e] = fast_exp2(__builtin_fmaf(s[e], c, -m));
        ps += s[e];
      }
      pf[h2] = pack8(s, 8 * h2);
    }
    l += ps;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      ld_cols(i + AHEAD);
      acc[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], pf[i / ND], acc[i % ND], 0, 0, 0);
      fence();
    }
  };
  // (nothing to do where every key comes after the queries or before their windows, past the first keys)
  auto seen = [&](int jb) { return jb <= iw0 + 31 && (iw0 - (jb + 31) < window || jb < sinks); };
  auto tile = [&](int t, auto stage_tag) {
    constexpr int stage = decltype(stage_tag)::value;
    const int j0 = kt.first_key(t);
    if (t + 1 < kt.n) fetch(t + 1, (unsigned)(stage ^ 1) * STAGE);   // (every wave left that stage at the barrier below)
    if (seen(j0)) block(stage_tag, j0);
    wait_dma();
    __syncthreads();
  };
  for (int t = 0; t < kt.n; t += 2) {
    tile(t, std::integral_constant<int, 0>{});
    if (t + 1 < kt.n) tile(t + 1, std::integral_constant<int, 1>{});
  }

  l += __shfl_xor(l, 32, 64);
  if (a.lse != nullptr && hh == 0 && qi < S) lb[qi] = qi < len ? (m + __log2f(l)) * kLn2 : -INFINITY;
  if (a.o == nullptr) return;
  store_rows<DH>(smem_b + wave * (64 * DH), acc, 1.0f / l, ob + (long)iw0 * a.ldo, a.ldo, S - iw0, len - iw0, nch, lane);
}

// ------------------------------------------------------------------ forward, otherwise
// The pipeline of a tile is the full attention's (attn_mfma.hip): the logits of tile t+1 are taken beside the softmax of tile t.
template <int DH, bool ORDERED>
__global__ __launch_bounds__(256, DH == 64 ? 3 : 2) void window_fwd_kernel(WindowArgs a, RowOrder ro) {
  constexpr int ND = DH / 32, NK = DH / 16;
  // LDS, in bytes: [K even][K odd][V even][V odd]; tile t of the walk lives in the buffers of t's parity
  constexpr unsigned TILE = BKV * DH * 2, VOFF = 2 * TILE;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_b[];

  const int S = a.S, nqt = (S + BROWS - 1) / BROWS, nch = a.dh / 8;
  int rank, head;
  row_tile<ORDERED>(ro, blockIdx.x, gridDim.x, nqt, &rank, &head);
  const int q0 = (nqt - 1 - rank) * BROWS;   // (late tiles are the heavy ones)
  const int h = head % a.nq, b = head / a.nq, kh = h / (a.nq / a.nk);
  const int len = sample_len(a, b);
  const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int iw0 = q0 + wave * 32, qi = iw0 + (lane & 31);
  bf16 *ob = (bf16 *)a.o + (long)b * S * a.ldo + (long)h * a.dh;
  float *lb = a.lse + ((long)b * a.nq + h) * S;
  if (q0 >= len) {
    const int r1 = min(q0 + BROWS, S);
    if (a.o != nullptr) zero_rows(ob, a.ldo, q0, r1, nch);
    if (a.lse != nullptr && q0 + tid < r1) lb[q0 + tid] = -INFINITY;
    return;
  }
  const bf16 *qb = (const bf16 *)a.q + (long)b * S * a.ldq + (long)h * a.dh;
  const char *kb = uniform_ptr((const char *)((const bf16 *)a.k + (long)b * S * a.ldk + (long)kh * a.dh));
  const char *vb = uniform_ptr((const char *)((const bf16 *)a.v + (long)b * S * a.ldv + (long)kh * a.dh));
  const unsigned ldkb = (unsigned)a.ldk * 2u, ldvb = (unsigned)a.ldv * 2u;
  const float c = a.scale * kLog2e;
  const int window = a.window, sinks = a.sinks;
  const KeyTiles<BKV, BROWS> kt(q0, len, window, sinks);
  // whether tile t of the walk hides a key from a query of the block
  auto hides = [&](int t) {
    const int j0 = kt.first_key(t);
    return j0 + BKV - 1 > q0 || (q0 + BROWS - 1 - j0 >= window && j0 + BKV > sinks);
  };

  auto fetch_k = [&](int t) { dma_tile<DH>((unsigned)(t & 1) * TILE, kb, ldkb, kt.first_key(t), len, nch, wave, lane); };
  fetch_k(0);
  dma_tile<DH>(VOFF, vb, ldvb, kt.first_key(0), len, nch, wave, lane);
  if (kt.n > 1) fetch_k(1);

  bf16x8 qf[NK];
  const bf16 *qrow = qb + (long)min(qi, len - 1) * a.ldq;   // (a query past the end reads the last row, and nothing of it is stored)
#pragma unroll
  for (int kd = 0; kd < NK; ++kd) qf[kd] = row_frag(qrow, kd, hh, a.dh);

  f32x16 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
  float m = -1e30f, l = 0.f;   // m: reference point of the exponents (log2 domain)

  BothAddr<DH> at;
  at.init(lane);
  wait_dma();
#pragma unroll
  for (int kd = 0; kd < NK; ++kd) asm volatile("" ::"v"(qf[kd]));   // (the fragments are waited for here, not in the tile loop)
  __syncthreads();

  bf16x8 fx[2];                  // fragment double buffer
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  auto ld_k = [&](unsigned buf, int slot, int sub, int kd) { fx[slot] = at.rows(buf, sub * 32, kd); };
  auto ld_v = [&](unsigned buf, int slot, int sub, int j) { fx[slot] = at.cols(buf, sub * 32 + (j / ND) * 16, j % ND); };
  auto zero = [](f32x16 &v) {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = 0.f;
  };
  auto mask = [&](f32x16 (&sv)[2], int j0) {
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) hide(sv[sub], hidden_keys(qi, j0 + 32 * sub, window, sinks), hh);
  };
  f32x16 lg[2][2];         // raw logits: those of tile t in lg[t & 1]
  float mx = -INFINITY;    // maximum over the raw logits of the tile about to be worked on (this lane's keys)

  auto tile = [&](int t, auto par_tag, auto more_tag) {
    constexpr int PAR = decltype(par_tag)::value;
    constexpr bool MORE = decltype(more_tag)::value;
    constexpr unsigned KN = (PAR ^ 1) * TILE, V = VOFF + PAR * TILE;   // K of tile t+1, V of tile t
    f32x16 (&cur)[2] = lg[PAR], (&nxt)[2] = lg[PAR ^ 1];
    mx = halves_max(mx);
    const float m_new = fmaxf(m, mx * c);
    constexpr float kLag = 8.f;   // (the reference point follows the maximum only when it is left behind by a factor of 2^8)
    if (__builtin_amdgcn_ballot_w64(m_new > m + kLag) != 0) {
      const float alpha = fast_exp2(m - m_new);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
      m = m_new;
    }
    mx = -INFINITY;
    float ps = 0.f;
    auto soft = [&](f32x16 &sv, int e0, int n) {
#pragma unroll
      for (int u = 0; u < n; ++u) {
        sv[e0 + u] = fast_exp2(__builtin_fmaf(sv[e0 + u], c, -m));
        ps += sv[e0 + u];
      }
    };
    auto vmax = [&](const f32x16 &sv, int e0, int n) {
#pragma unroll
      for (int u = 0; u < n; ++u) mx = fmaxf(mx, sv[e0 + u]);
    };
    const int jn = kt.first_key(t + 1);
    const TileRows kn = tile_rows(kb, ldkb, kt.first_key(t + 2), len), vn = tile_rows(vb, ldvb, jn, len);   // (past the walk's end: rows it has, which nobody reads)
    if (MORE) { zero(nxt[0]); zero(nxt[1]); ld_k(KN, 0, 0, 0); ld_k(KN, 1, 1, 0); }
#pragma unroll
    for (int kd = 0; kd < NK; ++kd) {
      if (MORE) {
        if (kd < NK / 2) dma_req<DH>(kd, PAR * TILE, kn, ldkb, nch, wave, lane);
        else dma_req<DH>(kd - NK / 2, VOFF + (PAR ^ 1) * TILE, vn, ldvb, nch, wave, lane);
        const bf16x8 ka = fx[0], kb2 = fx[1];
        if (kd + 1 < NK) { ld_k(KN, 0, 0, kd + 1); ld_k(KN, 1, 1, kd + 1); }
        nxt[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qf[kd], nxt[0], 0, 0, 0);
        nxt[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb2, qf[kd], nxt[1], 0, 0, 0);
      }
      if (kd + 1 == NK) ld_v(V, 0, 0, 0);
      soft(cur[0], kd * (16 / NK), 16 / NK);
      fence();
    }
    if (MORE && hides(t + 1)) mask(nxt, jn);
    bf16x8 pf[2];
    pf[0] = pack8(cur[0], 0); pf[1] = pack8(cur[0], 8);
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      if (j + 1 < NK) ld_v(V, (j + 1) & 1, 0, j + 1); else ld_v(V, (j + 1) & 1, 1, 0);
      acc[j % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[j & 1], pf[j / ND], acc[j % ND], 0, 0, 0);
      if ((j * 8) % NK == 0) soft(cur[1], j * 8 / NK, 8 / NK >= 1 ? 8 / NK : 1);
      if (MORE) vmax(nxt[0], j * (16 / NK), 16 / NK);
      fence();
    }
    pf[0] = pack8(cur[1], 0);
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      if (j + 1 < NK) ld_v(V, (j + 1) & 1, 1, j + 1);
      if (j == ND) pf[1] = pack8(cur[1], 8);
      acc[j % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[j & 1], pf[j / ND], acc[j % ND], 0, 0, 0);
      if (j < ND) soft(cur[1], 8 + j * (8 / ND), 8 / ND);
      else if (MORE) vmax(nxt[1], (j - ND) * (16 / ND), 16 / ND);
      fence();
    }
    l += ps;
    wait_dma();        // this wave's parts of the tiles on their way are in
    __syncthreads();   // everyone's are, and everyone is done with this tile's
  };

  using P0 = std::integral_constant<int, 0>;
  using P1 = std::integral_constant<int, 1>;
  using Yes = std::true_type;
  using No = std::false_type;
  zero(lg[0][0]); zero(lg[0][1]);
#pragma unroll
  for (int kd = 0; kd < NK; ++kd) {
    lg[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.rows(0u, 0, kd), qf[kd], lg[0][0], 0, 0, 0);
    lg[0][1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.rows(0u, 32, kd), qf[kd], lg[0][1], 0, 0, 0);
  }
  if (hides(0)) mask(lg[0], kt.first_key(0));
#pragma unroll
  for (int e = 0; e < 16; ++e) mx = fmaxf(mx, fmaxf(lg[0][0][e], lg[0][1][e]));
  __syncthreads();   // everyone has read K tile 0: the first tile below refills its buffer with K tile 2
  int t = 0;
  for (; t + 2 < kt.n; t += 2) {
    tile(t, P0{}, Yes{});
    tile(t + 1, P1{}, Yes{});
  }
  if (t + 1 < kt.n) {   // (the last tile has one form, that of even t: an odd one is made to look even)
    tile(t, P0{}, Yes{});
    lg[0][0] = lg[1][0]; lg[0][1] = lg[1][1];
    at.flip_cols(TILE);
    ++t;
  }
  tile(t, P0{}, No{});

  l += __shfl_xor(l, 32, 64);
  if (a.lse != nullptr && hh == 0 && qi < S) lb[qi] = qi < len ? (m + __log2f(l)) * kLn2 : -INFINITY;
  if (a.o == nullptr) return;
  store_rows<DH>(smem_b + wave * (64 * DH), acc, 1.0f / l, ob + (long)iw0 * a.ldo, a.ldo, S - iw0, len - iw0, nch, lane);
}

// ------------------------------------------------------------------ backward: dQ, and the row dots D_i
// 32 keys at a time, operands three steps ahead; the two waves of a SIMD hide each other's softmax.  (Two blocks of 32 in flight
// within a wave, operands one step ahead: 8 x 2048 tokens of 32 + 8 heads of 128, window 512, 290 us where 256 were.  The first sweep and D's sums cost 1 %.)
constexpr int kShort = 4;   // tiles
template <int DH, bool ORDERED>
__global__ __launch_bounds__(256, 2) void window_dq_kernel(WindowArgs a, RowOrder ro) {
  constexpr int ND = DH / 32, NK = DH / 16;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_b[];
  constexpr unsigned TILE = BKV * DH * 2, STAGE = 2 * TILE;   // [stage 0: K, V][stage 1: K, V]

  const int S = a.S, nqt = (S + BROWS - 1) / BROWS, nch = a.dh / 8;
  int rank, head;
  row_tile<ORDERED>(ro, blockIdx.x, gridDim.x, nqt, &rank, &head);
  const int q0 = (nqt - 1 - rank) * BROWS;
  const int h = head % a.nq, b = head / a.nq, kh = h / (a.nq / a.nk);
  const int len = sample_len(a, b);
  const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  bf16 *dqb = (bf16 *)a.dq + (long)b * S * a.ldq + (long)h * a.dh;
  if (q0 >= len) {
    zero_rows(dqb, a.ldq, q0, min(q0 + BROWS, S), nch);
    return;
  }
  const bf16 *qb = (const bf16 *)a.q + (long)b * S * a.ldq + (long)h * a.dh;
  const char *ksrc = uniform_ptr((const char *)((const bf16 *)a.k + (long)b * S * a.ldk + (long)kh * a.dh));
  const char *vsrc = uniform_ptr((const char *)((const bf16 *)a.v + (long)b * S * a.ldv + (long)kh * a.dh));
  const unsigned ldkb = (unsigned)a.ldk * 2u, ldvb = (unsigned)a.ldv * 2u;
  const int iw0 = q0 + wave * 32, qi = iw0 + (lane & 31);
  const float c = a.scale * kLog2e;
  const int window = a.window, sinks = a.sinks;
  const KeyTiles<BKV, BROWS> kt(q0, len, window, sinks);
  auto fetch = [&](int t, unsigned buf) {
    const int j0 = kt.first_key(t);
    dma_tile<DH>(buf, ksrc, ldkb, j0, len, nch, wave, lane);
    dma_tile<DH>(buf + TILE, vsrc, ldvb, j0, len, nch, wave, lane);
  };
  fetch(0, 0u);

  const long qc = min(qi, len - 1);
  const bf16 *qrow = qb + qc * a.ldq;
  const bf16 *grow = (const bf16 *)a.d_o + (long)b * S * a.ldo + (long)h * a.dh + qc * a.ldo;
  const bf16 *orow = (const bf16 *)a.o_in + (long)b * S * a.ldo + (long)h * a.dh + qc * a.ldo;
  bf16x8 qf[NK], gf[NK], of[NK];
#pragma unroll
  for (int kd = 0; kd < NK; ++kd) {
    qf[kd] = row_frag(qrow, kd, hh, a.dh);
    gf[kd] = row_frag(grow, kd, hh, a.dh);
    of[kd] = row_frag(orow, kd, hh, a.dh);
  }
  float dsum = 0.f;
#pragma unroll
  for (int kd = 0; kd < NK; ++kd)
#pragma unroll
    for (int i = 0; i < 8; ++i) dsum += (float)of[kd][i] * (float)gf[kd][i];
  float dot = dsum + __shfl_xor(dsum, 32, 64);   // the two halves of the row
  const long row_at = ((long)b * a.nq + h) * S + qi;
  const float lq = qi < len ? a.lse[row_at] * kLog2e : INFINITY;   // (queries past the end: P = 0)

  f32x16 dq[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) dq[d][e] = 0.f;

  BothAddr<DH> at;
  at.init(lane);
  wait_dma();
  __syncthreads();

  constexpr int AHEAD = 3, RING = 4;
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  // dS of the 32 keys from jb on (sub-tile `sub` of the tile at hand), and what they add to dQ
  float rest = 0.f;   // the sum of dS over this lane's keys
  auto block = [&](auto sub_tag, int jb, bool add) {
    constexpr int sub = decltype(sub_tag)::value;
    bf16x8 fx[RING], fy[RING];
    auto ld_rows = [&](int i) {   // K and V along the rows: operands of S and dP
      if (i >= NK) return;
      fx[i % RING] = at.rows(0u, sub * 32, i);
      fy[i % RING] = at.rows(TILE, sub * 32, i);
    };
    auto ld_cols = [&](int i) {   // K down the rows: operand of dQ
      if (i < NK) fx[i % RING] = at.cols(0u, sub * 32 + (i / ND) * 16, i % ND);
    };
    f32x16 s, dp;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ld_rows(i);
#pragma unroll
    for (int e = 0; e < 16; ++e) { s[e] = 0.f; dp[e] = -dot; }   // (dP starts at -D)
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      ld_rows(i + AHEAD);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], qf[i], s, 0, 0, 0);
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[i % RING], gf[i], dp, 0, 0, 0);
      fence();
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ld_cols(i);
    if (jb + 31 > iw0 || (iw0 + 31 - jb >= window && jb + 32 > sinks)) hide(s, hidden_keys(qi, jb, window, sinks), hh);
    bf16x8 dsf[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int e = 8 * h; e < 8 * h + 8; ++e) {
        dp[e] *= fast_exp2(s[e] * c - lq);
        rest += dp[e];
      }
      dsf[h] = pack8(dp, 8 * h);
    }
    if (!add) return;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      ld_cols(i + AHEAD);
      dq[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], dsf[i / ND], dq[i % ND], 0, 0, 0);
      fence();
    }
  };
  // (nothing to do where every key comes after the queries or before their windows, past the first keys)
  auto seen = [&](int jb) { return jb <= iw0 + 31 && (iw0 - (jb + 31) < window || jb < sinks); };
  // The dS of a query add up to 0 if D is the sum of its P dP, and to what <dO, O> is off by as O was rounded.  dK gets the D put
  // right by that; so does dQ where walks are short, by a first sweep over the tiles: with few keys to a query the rounding of O
  // counts as much as that of dS (a window of 64: dQ off by 1.6 times what rounding the result costs, else 1.4 times).
  unsigned at_hand = 0;   // the stage of the tile at hand
  for (int sweep = kt.n <= kShort ? 0 : 1; sweep < 2; ++sweep) {
    for (int t = 0; t < kt.n; ++t) {
      const int j0 = kt.first_key(t);
      at_hand ^= STAGE;
      // (every wave left that stage at the barrier below; the first sweep ends with the first tile again)
      if (t + 1 < kt.n || sweep == 0) fetch(t + 1 < kt.n ? t + 1 : 0, at_hand);
      if (seen(j0)) block(std::integral_constant<int, 0>{}, j0, sweep == 1);
      if (seen(j0 + 32)) block(std::integral_constant<int, 1>{}, j0 + 32, sweep == 1);
      at.flip(STAGE);
      wait_dma();
      __syncthreads();
    }
    dot += rest + __shfl_xor(rest, 32, 64);
    rest = 0.f;
  }
  if (qi < len && hh == 0) a.ws[row_at] = dot;

  store_rows<DH>(smem_b + wave * (64 * DH), dq, a.scale, dqb + (long)iw0 * a.ldq, a.ldq, S - iw0, len - iw0, nch, lane);
}


// Blocks of the same weight go head after head; those of a window that most of the sequence fits in are as uneven as a causal
// mask's and go by weight.
template <int PER_CU> RowOrder order_of(const WindowArgs &a, int blocks, int tiles, int dh) {
  return row_order<PER_CU>(2 * (long)a.window >= a.S, blocks, tiles, a.S, dh);
}

template <int DH> hipError_t fwd_launch(const WindowArgs &a, hipStream_t s) {
  const int tiles = (a.S + BROWS - 1) / BROWS, blocks = tiles * a.nq * a.B;
  if (by_blocks(a, blocks)) {
    constexpr size_t smem = 2 * 2 * (size_t)KEYS * DH * sizeof(bf16);
    const RowOrder ro = order_of<DH == 64 ? 4 : 3>(a, blocks, tiles, DH);
    hipLaunchKernelGGL((window_fwd_blocks_kernel<DH>), dim3(blocks), dim3(256), smem, s, a, ro);
    return hipGetLastError();
  }
  constexpr size_t smem = 2 * 2 * (size_t)BKV * DH * sizeof(bf16);
  const RowOrder ro = order_of<DH == 64 ? 3 : 2>(a, blocks, tiles, DH);
  if (ro.own > 0) hipLaunchKernelGGL((window_fwd_kernel<DH, true>), dim3(blocks), dim3(256), smem, s, a, ro);
  else hipLaunchKernelGGL((window_fwd_kernel<DH, false>), dim3(blocks), dim3(256), smem, s, a, ro);
  return hipGetLastError();
}

template <int DH> hipError_t bwd_launch(const WindowArgs &a, hipStream_t s) {
  const int tiles = (a.S + BROWS - 1) / BROWS, blocks = tiles * a.nq * a.B;
  constexpr size_t smem = 2 * 2 * (size_t)BKV * DH * sizeof(bf16);
  // dQ first: it leaves the row dots <dO_i, O_i> in the workspace
  const RowOrder ro = order_of<2>(a, blocks, tiles, DH);
  if (ro.own > 0) hipLaunchKernelGGL((window_dq_kernel<DH, true>), dim3(blocks), dim3(256), smem, s, a, ro);
  else hipLaunchKernelGGL((window_dq_kernel<DH, false>), dim3(blocks), dim3(256), smem, s, a, ro);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_window_dkv(a, a.ws, (float *)((char *)a.ws + dots_bytes(a)), s);
}

bool fits(const void *p, long ld) {
  return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld < (1 << 25);   // (a tile's 64 rows in 32-bit offsets)
}

}  // namespace

bool window_mfma_supported(const WindowArgs &a) {
  return a.dh <= 128 && fits(a.q, a.ldq) && fits(a.k, a.ldk) && fits(a.v, a.ldv) && fits(a.o, a.ldo) &&
         fits(a.o_in, a.ldo) && fits(a.d_o, a.ldo) && fits(a.dq, a.ldq) && fits(a.dk, a.ldk) && fits(a.dv, a.ldv) &&
         ((uintptr_t)a.ws & 15) == 0;
}
size_t window_mfma_ws_bytes(const WindowArgs &a) {
  if (a.dh > 128) return 0;
  const int rows = key_rows(a);
  const size_t slots = rows == 64 ? slots_of(a, work_of<64>(a)) : slots_of(a, work_of<128>(a));
  return dots_bytes(a) + slots * 2 * rows * (size_t)columns(a) * sizeof(float);
}
hipError_t launch_window_fwd_mfma(const WindowArgs &a, hipStream_t s) { return columns(a) == 64 ? fwd_launch<64>(a, s) : fwd_launch<128>(a, s); }
hipError_t launch_window_bwd_mfma(const WindowArgs &a, hipStream_t s) { return columns(a) == 64 ? bwd_launch<64>(a, s) : bwd_launch<128>(a, s); }

}  // namespace dp
