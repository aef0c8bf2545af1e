// Sliding-window attention in bf16: dK and dV.
#include "window_bf16.h"

namespace dp {

namespace {

// Block: ROWS keys of a key head, two waves for every 32 of them, each with one half (32 queries) of every tile: the two waves of a
// SIMD have blocks of 32 x 32 of their own to issue beside each other's, and leave out those that the mask hides whole.  dK and dV
// of the two halves are added at the end.  256 registers a wave at 128 columns: 128 of sums, 32 of K; V's fragments stand in LDS.
// 8 x 2048 tokens of 32 + 8 heads of 128, window 512: 307 us where four waves a block with K and V in registers took 427.  Per tile
// of 64 queries and 128 keys the products take 2048 clocks of a SIMD and the LDS reads 1700, of about 3600: a barrier a tile, and
// blocks of a tile that are not alike.
// fragments of 16 columns of V that stand in LDS: all, but where two blocks of 128 columns share 160 KB
template <int DH, int ROWS> constexpr int v_in_lds() { return DH == 128 && ROWS == 64 ? 7 : DH / 16; }
template <int DH, int ROWS>
__global__ __launch_bounds__(4 * ROWS, 2) void window_dkv_kernel(WindowArgs a, KeyWork w, const float *__restrict__ drow,
                                                            float *__restrict__ sums) {
  constexpr int ND = DH / 32, NK = DH / 16, GROUPS = ROWS / 32, WAVES = 2 * GROUPS, VKD = v_in_lds<DH, ROWS>();
  // LDS, in bytes: [stage 0: Q, dO][stage 1: Q, dO][V of the block's keys][stage 0: lse, row dots][stage 1: lse, row dots]
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_b[];
  constexpr unsigned TILE = BKV * DH * 2, STAGE = 2 * TILE, VBASE = 2 * STAGE, FBASE = VBASE + GROUPS * VKD * 1024, FSTAGE = 8 * BKV, ROWB = DH * 2;

  const int S = a.S, nch = a.dh / 8, group = a.nq / a.nk;
  const Piece at = piece_at(w, blockIdx.x, a.B * a.nk);
  const int head = at.head, kb = at.kb, piece = at.piece;
  const int kh = head % a.nk, b = head / a.nk;
  const int len = sample_len(a, b);
  const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = wave / GROUPS, kg = half ? WAVES - 1 - wave : wave;   // (the halves of a SIMD's pair differ in keys: edges are as uneven)
  const int j0 = kb * ROWS, jw0 = j0 + kg * 32, kj = jw0 + (lane & 31);
  const long slot = slot_of(w, head, kb, piece);
  bf16 *dkb = (bf16 *)a.dk + (long)b * S * a.ldk + (long)kh * a.dh, *dvb = (bf16 *)a.dv + (long)b * S * a.ldv + (long)kh * a.dh;
  if (j0 >= len) {
    if (slot < 0) {
      zero_rows(dkb, a.ldk, j0, min(j0 + ROWS, S), nch);
      zero_rows(dvb, a.ldv, j0, min(j0 + ROWS, S), nch);
    }
    return;
  }
  const Walk walk = walk_of<ROWS>(w, kb, piece, len, a.window, group);
  if (walk.begin == walk.end) return;   // (a piece of several: the kernel that adds them up knows)
  const bf16 *krow = (const bf16 *)a.k + ((long)b * S + min(kj, len - 1)) * a.ldk + (long)kh * a.dh;
  const bf16 *vrow = (const bf16 *)a.v + ((long)b * S + min(kj, len - 1)) * a.ldv + (long)kh * a.dh;
  const float c = a.scale * kLog2e;
  const int window = a.window, sinks = a.sinks;

  // item `it` of the walk: tile walk.t0 + it % nt of head it / nt; (g, t) is the next one to be fetched
  int g = walk.begin / walk.nt, t = walk.begin - g * walk.nt;
  const char *qsrc = uniform_ptr((const char *)((const bf16 *)a.q + (long)b * S * a.ldq + (long)(kh * group + g) * a.dh));
  const char *osrc = uniform_ptr((const char *)((const bf16 *)a.d_o + (long)b * S * a.ldo + (long)(kh * group + g) * a.dh));
  const long row0 = ((long)b * a.nq + kh * group + g) * S;
  const unsigned ldqb = (unsigned)a.ldq * 2u, ldob = (unsigned)a.ldo * 2u;
  // the two scalars per query go through a register: even waves carry the 64 log-sum-exps, odd waves the 64 row dots
  const float *fsrc = ((wave & 1) ? drow : (const float *)a.lse) + row0;
  const float fmul = (wave & 1) ? -1.f : kLog2e;   // (dP starts at -D)
  const float fpad = (wave & 1) ? 0.f : INFINITY;  // (rows past the end: P = 0)
  float sl = 0.f;
  int i_next = 0;   // first query of the tile fetched last
  auto fetch = [&](unsigned buf) {
    int lane = tid & 63;
    if constexpr (VKD < NK) asm volatile("" : "+v"(lane));   // (what follows from it is worked out again for every tile: no registers left)
    i_next = (walk.t0 + t) * BKV;
    dma_tile<DH, BKV, WAVES>(buf, qsrc, ldqb, i_next, len, nch, wave, lane);
    dma_tile<DH, BKV, WAVES>(buf + TILE, osrc, ldob, i_next, len, nch, wave, lane);
    if (wave < 2) sl = fsrc[min(i_next + lane, len - 1)];
    if (++t == walk.nt) { t = 0; qsrc += 2 * a.dh; osrc += 2 * a.dh; fsrc += S; }
  };
  auto stash = [&](unsigned stage) {   // [0,64): lse, [64,128): row dots
    if (wave < 2) reinterpret_cast<float *>(smem_b + FBASE + stage * FSTAGE)[tid] = i_next + lane < len ? sl * fmul : fpad;
  };
  fetch(0u);

  // fragments of the block's keys: K's in registers, V's in LDS, one after the other
  const unsigned r = (unsigned)(lane & 31), rowb = r * ROWB + (((unsigned)hh ^ swz_both<DH>(r)) << 4);   // (element 0; 16 kd: ^ kd << 5)
  const unsigned vat = VBASE + (unsigned)(kg * VKD) * 1024u + (unsigned)lane * 16u;
  bf16x8 kf[NK];
#pragma unroll
  for (int kd = 0; kd < NK; ++kd) kf[kd] = row_frag(krow, kd, hh, a.dh);
#pragma unroll
  for (int kd = 0; kd < NK / 2; ++kd) {
    const int k2 = kd + half * (NK / 2);
    if (k2 < VKD) *(lds_bf16x8 *)(uintptr_t)(vat + (unsigned)k2 * 1024u) = row_frag(vrow, k2, hh, a.dh);
  }
  bf16x8 vlast;   // (what LDS has no room for)
  if constexpr (VKD < NK) vlast = row_frag(vrow, NK - 1, hh, a.dh);
  stash(0u);
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) { dk[d][e] = 0.f; dv[d][e] = 0.f; }

  // LDS addresses of the wave's half of the tile at hand; the swizzle leaves the bits of kd and d to an exclusive or
  unsigned row = (unsigned)half * (32 * ROWB) + rowb, col[2];
  {
    const unsigned i = (unsigned)(lane & 15), tt = i >> 2, rc = 4u * (unsigned)hh + tt, cl = 2u * (unsigned)((lane >> 4) & 1) + ((i & 3u) >> 1);
    col[0] = (unsigned)half * (32 * ROWB) + rc * ROWB + ((cl ^ swz_both<DH>(rc)) << 4) + (i & 1u) * 8u;
    col[1] = (unsigned)half * (32 * ROWB) + (rc + 8u) * ROWB + ((cl ^ swz_both<DH>(rc + 8u)) << 4) + (i & 1u) * 8u;
  }
  auto rows_of = [&](unsigned at, unsigned tile_off, int kd) { return *(const lds_bf16x8 *)(uintptr_t)((at ^ ((unsigned)kd << 5)) + tile_off); };
  auto cols_of = [&](unsigned tile_off, int r0, int d) {
    union { s16x4 h[2]; bf16x8 v; } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)((col[0] ^ ((unsigned)d << 6)) + tile_off + (unsigned)r0 * ROWB));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)((col[1] ^ ((unsigned)d << 6)) + tile_off + (unsigned)r0 * ROWB));
    return u.v;
  };
  wait_dma();
  __syncthreads();

  constexpr int AHEAD = 2, RING = 3;
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  const float *lds_f = reinterpret_cast<const float *>(smem_b + FBASE) + 32 * half + 4 * hh;   // the current tile's scalars
  unsigned cur = 0;   // the stage at hand
  // P, dP, and what they add to dK and dV, of queries ib .. ib+31
  auto block = [&](int ib) {
    bf16x8 fx[RING], fy[RING], fv[RING];
    auto ld_rows = [&](int i) {
      if (i >= NK) return;
      fx[i % RING] = rows_of(row, 0u, i);
      fy[i % RING] = rows_of(row, TILE, i);
      if (i < VKD) fv[i % RING] = *(const lds_bf16x8 *)(uintptr_t)(vat + (unsigned)i * 1024u);
    };
    auto ld_cols = [&](int i) {   // dO, Q down the rows
      if (i >= NK) return;
      fx[i % RING] = cols_of(TILE, (i / ND) * 16, i % ND);
      fy[i % RING] = cols_of(0u, (i / ND) * 16, i % ND);
    };
    f32x16 s, dp;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ld_rows(i);
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const f32x4 d = *reinterpret_cast<const f32x4 *>(lds_f + BKV + 8 * e4);
#pragma unroll
      for (int u = 0; u < 4; ++u) { dp[4 * e4 + u] = d[u]; s[4 * e4 + u] = 0.f; }
    }
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      ld_rows(i + AHEAD);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], kf[i], s, 0, 0, 0);
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[i % RING], i < VKD ? fv[i % RING] : vlast, dp, 0, 0, 0);
      fence();
    }
    f32x4 l[4];
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) l[e4] = *reinterpret_cast<const f32x4 *>(lds_f + 8 * e4);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ld_cols(i);
    if (ib < jw0 + 31 || (ib + 31 - jw0 >= window && jw0 + 32 > sinks)) hide(s, hidden_queries(kj, ib, window, sinks), hh);
    bf16x8 pf[2], dsf[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int e = 8 * h; e < 8 * h + 8; ++e) {
        const float p = fast_exp2(s[e] * c - l[e >> 2][e & 3]);
        s[e] = p;
        dp[e] *= p;
      }
      pf[h] = pack8(s, 8 * h);
      dsf[h] = pack8(dp, 8 * h);
    }
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      ld_cols(i + AHEAD);
      dv[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], pf[i / ND], dv[i % ND], 0, 0, 0);
      dk[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[i % RING], dsf[i / ND], dk[i % ND], 0, 0, 0);
      fence();
    }
  };
  int i0 = i_next;
  for (int it = walk.begin; it < walk.end; ++it) {
    const unsigned nxt = cur ^ 1u;
    const bool more = it + 1 < walk.end;
    if (more) fetch(nxt * STAGE);   // (every wave left that stage at the barrier below)
    const int ib = i0 + 32 * half;
    // (nothing to do where every query comes before the keys, past their window or past the end)
    if (ib + 31 >= jw0 && ib < len && (ib - (jw0 + 31) < window || jw0 < sinks)) block(ib);
    if (more) stash(nxt);
    row ^= STAGE; col[0] ^= STAGE; col[1] ^= STAGE;
    lds_f = reinterpret_cast<const float *>(smem_b + FBASE + nxt * FSTAGE) + 32 * half + 4 * hh;
    wait_dma();
    __syncthreads();
    cur = nxt;
    i0 = i_next;
  }

  // a wave's dK, dV and those of the other half for the same keys are added through LDS, half of the columns at a time: the first
  // half of the waves ends with dK, the second with dV
  float *mine = reinterpret_cast<float *>(smem_b) + (half * GROUPS + kg) * (ND / 2 * 1024) + lane * 4;
  const float *other = reinterpret_cast<const float *>(smem_b) + ((half ^ 1) * GROUPS + kg) * (ND / 2 * 1024) + lane * 4;
  auto give = [&](const f32x16 &v, int d) {
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const f32x4 x = {v[4 * e4], v[4 * e4 + 1], v[4 * e4 + 2], v[4 * e4 + 3]};
      *reinterpret_cast<f32x4 *>(mine + d * 1024 + e4 * 256) = x;
    }
  };
  auto take = [&](f32x16 &v, int d) {
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(other + d * 1024 + e4 * 256);
#pragma unroll
      for (int u = 0; u < 4; ++u) v[4 * e4 + u] += x[u];
    }
  };
#pragma unroll
  for (int d0 = 0; d0 < ND; d0 += ND / 2) {
#pragma unroll
    for (int d = 0; d < ND / 2; ++d) {
      if (half == 0) give(dv[d0 + d], d);
      else give(dk[d0 + d], d);
    }
    __syncthreads();
#pragma unroll
    for (int d = 0; d < ND / 2; ++d) {
      if (half == 0) take(dk[d0 + d], d);
      else take(dv[d0 + d], d);
    }
    __syncthreads();
  }
  auto out = [&](const f32x16 (&v)[ND], float mul, bf16 *dst, long ld) {
    if (slot < 0) {
      store_rows<DH>(smem_b + wave * (64 * DH), v, mul, dst + (long)jw0 * ld, ld, S - jw0, len - jw0, nch, lane);
      return;
    }
    // sums of this piece: a lane's key is a row, its four consecutive columns one store
    float *to = sums + slot * (2 * ROWS * DH) + half * (ROWS * DH) + (kg * 32 + (lane & 31)) * DH + 4 * hh;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const f32x4 x = {v[d][4 * e4], v[d][4 * e4 + 1], v[d][4 * e4 + 2], v[d][4 * e4 + 3]};
        *reinterpret_cast<f32x4 *>(to + 32 * d + 8 * e4) = x;
      }
  };
  if (half == 0) out(dk, a.scale, dkb, a.ldk);
  else out(dv, 1.f, dvb, a.ldv);
}

template <int DH, int ROWS> hipError_t go(const WindowArgs &a, const float *drow, float *sums, hipStream_t s) {
  constexpr size_t smem = 4 * (size_t)BKV * DH * sizeof(bf16) + ROWS / 32 * v_in_lds<DH, ROWS>() * 1024 + 4 * BKV * sizeof(float);
  const auto kern = window_dkv_kernel<DH, ROWS>;
  if (smem > 64 * 1024) {   // (beyond that it has to be asked for, on every device)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != hipSuccess) return e;
  }
  const KeyWork w = work_of<ROWS>(a);
  const int heads = a.B * a.nk, cut = key_blocks_cut(w);
  hipLaunchKernelGGL(kern, dim3((unsigned)(heads * pieces_of(w))), dim3(4 * ROWS), smem, s, a, w, drow, sums);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || cut == 0) return e;
  hipLaunchKernelGGL((window_dkv_sum_kernel<bf16, ROWS, DH>), dim3(heads * cut * 2 * (ROWS / kSumRows)), dim3(kSumRows * DH / 4), 0, s, a, w, sums, cut);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_window_dkv(const WindowArgs &a, const float *drow, float *sums, hipStream_t s) {
  if (key_rows(a) == 64) return columns(a) == 64 ? go<64, 64>(a, drow, sums, s) : go<128, 64>(a, drow, sums, s);
  return columns(a) == 64 ? go<64, 128>(a, drow, sums, s) : go<128, 128>(a, drow, sums, s);
}

}  // namespace dp
