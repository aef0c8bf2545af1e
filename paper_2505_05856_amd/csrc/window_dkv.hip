// Sliding-window attention in bf16: dK and dV.
#include "window_bf16.h"

#include <type_traits>
#include <utility>

namespace dp {

namespace {

// f(integral_constant<int, 0>) .. f(integral_constant<int, N-1>)
template <typename F, int... I> __device__ __forceinline__ void static_for(F &&f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F> __device__ __forceinline__ void static_for(F &&f) { static_for(f, std::make_integer_sequence<int, N>{}); }

template <int DH>
__global__ __launch_bounds__(256, DH == 128 ? 1 : 2) void window_dkv_kernel(WindowArgs a, KeyWork w, const float *__restrict__ drow,
                                                                          float *__restrict__ sums) {
  constexpr int ND = DH / 32, NK = DH / 16;
  // LDS, in bytes: [stage 0: Q, dO][stage 1: Q, dO][stage 0: lse, row dots][stage 1: lse, row dots]
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_b[];
  constexpr unsigned TILE = BKV * DH * 2, STAGE = 2 * TILE, FBASE = 2 * STAGE, FSTAGE = 8 * BKV;

  const int S = a.S, nch = a.dh / 8, group = a.nq / a.nk;
  // a head's pieces: the far ones first, then the windows' from the first key block on
  const int per_head = w.key_blocks * w.parts + w.first * w.far;
  const int wid = xcd_contiguous(blockIdx.x, gridDim.x);
  const int head = wid / per_head, id = wid - head * per_head, nfar = w.first * w.far;
  const int kb = id < nfar ? id / w.far : (id - nfar) / w.parts;
  const int piece = id < nfar ? w.parts + id % w.far : (id - nfar) % w.parts;
  const int kh = head % a.nk, b = head / a.nk;
  const int len = sample_len(a, b);
  const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j0 = kb * BROWS, jw0 = j0 + wave * 32, kj = jw0 + (lane & 31);
  const long slot = slot_of(w, head, kb, piece);
  bf16 *dkb = (bf16 *)a.dk + (long)b * S * a.ldk + (long)kh * a.dh, *dvb = (bf16 *)a.dv + (long)b * S * a.ldv + (long)kh * a.dh;
  if (j0 >= len) {
    if (slot < 0) {
      zero_rows(dkb, a.ldk, j0, min(j0 + BROWS, S), nch);
      zero_rows(dvb, a.ldv, j0, min(j0 + BROWS, S), nch);
    }
    return;
  }
  const Walk walk = walk_of<BROWS>(w, kb, piece, len, a.window, group);
  if (walk.begin == walk.end) return;   // (a piece of several: the kernel that adds them up knows)
  const bf16 *krow = (const bf16 *)a.k + ((long)b * S + min(kj, len - 1)) * a.ldk + (long)kh * a.dh;
  const bf16 *vrow = (const bf16 *)a.v + ((long)b * S + min(kj, len - 1)) * a.ldv + (long)kh * a.dh;
  const float c = a.scale * kLog2e;
  const int window = a.window, sinks = a.sinks;

  bf16x8 kf[NK], vf[NK];
#pragma unroll
  for (int kd = 0; kd < NK; ++kd) {
    kf[kd] = row_frag(krow, kd, hh, a.dh);
    vf[kd] = row_frag(vrow, kd, hh, a.dh);
  }
  // (At 128 columns the keys' fragments stand in accumulation registers, where the matrix instructions take them from; left alone
  // the compiler moves them to and fro, 139 moves a tile beside 64 matrix instructions.)
  if (DH == 128) {
#pragma unroll
    for (int kd = 0; kd < NK; ++kd) asm volatile("" : "+a"(kf[kd]), "+a"(vf[kd]));
  }
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) { dk[d][e] = 0.f; dv[d][e] = 0.f; }

  // item `it` of the walk: tile walk.t0 + it % nt of head it / nt; (g, t) is the next one to be fetched
  int g = walk.nt > 0 ? walk.begin / walk.nt : 0, t = walk.nt > 0 ? walk.begin - g * walk.nt : 0;
  const char *qsrc = uniform_ptr((const char *)((const bf16 *)a.q + (long)b * S * a.ldq + (long)(kh * group + g) * a.dh));
  const char *osrc = uniform_ptr((const char *)((const bf16 *)a.d_o + (long)b * S * a.ldo + (long)(kh * group + g) * a.dh));
  const float *lrow = a.lse + ((long)b * a.nq + kh * group + g) * S, *drw = drow + ((long)b * a.nq + kh * group + g) * S;
  const unsigned ldqb = (unsigned)a.ldq * 2u, ldob = (unsigned)a.ldo * 2u;
  // the two scalars per query go through a register: even waves carry the 64 log-sum-exps, odd waves the 64 row dots
  const float *fsrc = (wave & 1) ? drw : lrow;
  const float fmul = (wave & 1) ? -1.f : kLog2e;   // (dP starts at -D)
  const float fpad = (wave & 1) ? 0.f : INFINITY;  // (rows past the end: P = 0)
  float sl = 0.f;
  int i_next = 0;   // first query of the tile fetched last
  auto fetch = [&](unsigned buf) {
    i_next = (walk.t0 + t) * BKV;
    dma_tile<DH>(buf, qsrc, ldqb, i_next, len, nch, wave, lane);
    dma_tile<DH>(buf + TILE, osrc, ldob, i_next, len, nch, wave, lane);
    sl = fsrc[min(i_next + lane, len - 1)];
    if (++t == walk.nt) { t = 0; qsrc += 2 * a.dh; osrc += 2 * a.dh; fsrc += S; }
  };
  auto stash = [&](unsigned stage) {   // [0,64): lse, [64,128): row dots
    reinterpret_cast<float *>(smem_b + FBASE + stage * FSTAGE)[tid & 127] = i_next + lane < len ? sl * fmul : fpad;
  };
  if (walk.begin < walk.end) { fetch(0u); stash(0u); }
  BothAddr<DH> at;
  at.init(lane);
  wait_dma();
  __syncthreads();

  // the pipeline over the two 32-query sub-tiles A and B of a tile, as in the full attention's dK/dV kernel
  constexpr int EPS = 16 / NK;
  // The operands of the 4 NK steps of a tile, in the order they are asked for, AHEAD steps before they are used: Q and dO along
  // the rows for S and dP of A (steps 0 ..), of B (NK ..), dO and Q down the rows for dV and dK of A (2 NK ..), of B (3 NK ..).
  constexpr int AHEAD = 3, RING = 4;
  bf16x8 fx[RING], fy[RING];
  auto ld = [&](auto step_tag) {
    constexpr int i = decltype(step_tag)::value;
    if constexpr (i < 2 * NK) {
      fx[i % RING] = at.rows(0u, (i / NK) * 32, i % NK);
      fy[i % RING] = at.rows(TILE, (i / NK) * 32, i % NK);
    } else if constexpr (i < 4 * NK) {
      constexpr int sub = i / NK - 2, j = i % NK;
      fx[i % RING] = at.cols(TILE, sub * 32 + (j / ND) * 16, j % ND);
      fy[i % RING] = at.cols(0u, sub * 32 + (j / ND) * 16, j % ND);
    }
  };
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  const float *lds_f = reinterpret_cast<const float *>(smem_b + FBASE);   // the current tile's scalars
  float lsc[2][EPS];
  auto ld_soft = [&](int q) {
    const int e0 = (q % NK) * EPS, r0 = (q / NK) * 32 + 8 * (e0 >> 2) + 4 * hh + (e0 & 3);
    typedef float vec __attribute__((ext_vector_type(EPS)));
    const vec l = *reinterpret_cast<const vec *>(lds_f + r0);
#pragma unroll
    for (int u = 0; u < EPS; ++u) lsc[q & 1][u] = l[u];
  };
  auto dp_start = [&](f32x16 &v, int sub) {   // dP starts at -D
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const f32x4 d = *reinterpret_cast<const f32x4 *>(lds_f + BKV + sub * 32 + 8 * e4 + 4 * hh);
#pragma unroll
      for (int u = 0; u < 4; ++u) v[4 * e4 + u] = d[u];
    }
  };
  unsigned cur = 0;   // the stage at hand
  auto tile = [&](int i0, auto more_tag, auto mask_tag) {
    constexpr bool MORE = decltype(more_tag)::value, MASK = decltype(mask_tag)::value;
    const unsigned nxt = cur ^ 1u;
    f32x16 sA, dpA, sB, dpB;
    dp_start(dpA, 0);
    dp_start(dpB, 1);
    static_for<AHEAD>(ld);
    if (MORE) fetch(nxt * STAGE);   // (every wave left that stage at the barrier below)
    auto soft = [&](f32x16 &sv, f32x16 &dpv, int q) {   // logits -> P, dP -> dS
      const int e0 = (q % NK) * EPS;
#pragma unroll
      for (int u = 0; u < EPS; ++u) {
        const float pr = fast_exp2(sv[e0 + u] * c - lsc[q & 1][u]);
        sv[e0 + u] = pr;
        dpv[e0 + u] *= pr;
      }
    };
    auto mask = [&](f32x16 &sv, int sub) {
      const int ib = i0 + 32 * sub;
      if (MASK) hide(sv, hidden_queries(kj, ib, window, sinks), hh);
    };
#pragma unroll
    for (int e = 0; e < 16; ++e) { sA[e] = 0.f; sB[e] = 0.f; }
    static_for<NK>([&](auto kd_tag) {   // S, dP of A
      constexpr int i = decltype(kd_tag)::value;
      ld(std::integral_constant<int, i + AHEAD>{});
      if (i == NK - 1) ld_soft(0);
      sA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], kf[i], sA, 0, 0, 0);
      dpA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[i % RING], vf[i], dpA, 0, 0, 0);
      fence();
    });
    mask(sA, 0);
    static_for<NK>([&](auto kd_tag) {   // S, dP of B beside P, dS of A
      constexpr int kd = decltype(kd_tag)::value, i = NK + kd;
      ld(std::integral_constant<int, i + AHEAD>{});
      ld_soft(kd + 1);
      sB = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], kf[kd], sB, 0, 0, 0);
      dpB = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[i % RING], vf[kd], dpB, 0, 0, 0);
      soft(sA, dpA, kd);
      fence();
    });
    bf16x8 pf[2], dsf[2];
    pf[0] = pack8(sA, 0); pf[1] = pack8(sA, 8); dsf[0] = pack8(dpA, 0); dsf[1] = pack8(dpA, 8);
    mask(sB, 1);
    static_for<NK>([&](auto j_tag) {    // dV, dK += A's, beside P, dS of B
      constexpr int j = decltype(j_tag)::value, i = 2 * NK + j;
      ld(std::integral_constant<int, i + AHEAD>{});
      if (j + 1 < NK) ld_soft(NK + j + 1);
      dv[j % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], pf[j / ND], dv[j % ND], 0, 0, 0);
      dk[j % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[i % RING], dsf[j / ND], dk[j % ND], 0, 0, 0);
      soft(sB, dpB, NK + j);
      fence();
    });
    pf[0] = pack8(sB, 0); pf[1] = pack8(sB, 8); dsf[0] = pack8(dpB, 0); dsf[1] = pack8(dpB, 8);
    static_for<NK>([&](auto j_tag) {    // dV, dK += B's
      constexpr int j = decltype(j_tag)::value, i = 3 * NK + j;
      ld(std::integral_constant<int, i + AHEAD>{});
      dv[j % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i % RING], pf[j / ND], dv[j % ND], 0, 0, 0);
      dk[j % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[i % RING], dsf[j / ND], dk[j % ND], 0, 0, 0);
      fence();
    });
    if (MORE) stash(nxt);
    at.flip(STAGE);
    lds_f = reinterpret_cast<const float *>(smem_b + FBASE + nxt * FSTAGE);
    wait_dma();
    __syncthreads();
    cur = nxt;
  };
  if (walk.begin < walk.end) {
    int i0 = i_next, it = walk.begin;
    auto hides = [&](int i) { return i < j0 + BROWS - 1 || (i + BKV - 1 - j0 >= window && j0 + BROWS > sinks); };
    while (it + 1 < walk.end) {
      for (; it + 1 < walk.end && hides(i0); ++it) { tile(i0, std::true_type{}, std::true_type{}); i0 = i_next; }
      for (; it + 1 < walk.end && !hides(i0); ++it) { tile(i0, std::true_type{}, std::false_type{}); i0 = i_next; }
    }
    tile(i0, std::false_type{}, std::true_type{});
  }

  if (slot < 0) {
    unsigned char *ew = smem_b + wave * (128 * DH);
    store_rows<DH>(ew, dk, a.scale, dkb + (long)jw0 * a.ldk, a.ldk, S - jw0, len - jw0, nch, lane);
    store_rows<DH>(ew + 64 * DH, dv, 1.f, dvb + (long)jw0 * a.ldv, a.ldv, S - jw0, len - jw0, nch, lane);
    return;
  }
  // sums of this piece: a lane's key is a row, its four consecutive columns one store
  float *out = sums + slot * (2 * BROWS * DH) + (wave * 32 + (lane & 31)) * DH + 4 * hh;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      f32x4 x, y;
#pragma unroll
      for (int u = 0; u < 4; ++u) { x[u] = dk[d][4 * e4 + u]; y[u] = dv[d][4 * e4 + u]; }
      *reinterpret_cast<f32x4 *>(out + 32 * d + 8 * e4) = x;
      *reinterpret_cast<f32x4 *>(out + BROWS * DH + 32 * d + 8 * e4) = y;
    }
}

template <int DH> hipError_t go(const WindowArgs &a, const float *drow, float *sums, hipStream_t s) {
  constexpr size_t smem = 2 * (2 * (size_t)BKV * DH * sizeof(bf16) + 2 * BKV * sizeof(float));
  if (smem > 64 * 1024) {   // (beyond that it has to be asked for, on every device)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(window_dkv_kernel<DH>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != hipSuccess) return e;
  }
  const KeyWork w = work_of(a);
  const int heads = a.B * a.nk, cut = key_blocks_cut(w);
  hipLaunchKernelGGL((window_dkv_kernel<DH>), dim3((unsigned)(heads * pieces_of(w))), dim3(256), smem, s, a, w, drow, sums);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || cut == 0) return e;
  hipLaunchKernelGGL((window_dkv_sum_kernel<bf16, BROWS, DH>), dim3(heads * cut * 2 * (BROWS / 32)), dim3(256), 0, s, a, w, sums, cut);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_window_dkv(const WindowArgs &a, const float *drow, float *sums, hipStream_t s) {
  return columns(a) == 64 ? go<64>(a, drow, sums, s) : go<128>(a, drow, sums, s);
}

}  // namespace dp
