// Queries and keys between their projection and the attention: every head's vector x (dh elements) is divided by its root
// mean square and multiplied by a gain, then its first 2 * half elements are turned by the token's position,
//   n = g x r, r = 1 / sqrt(mean(x^2) + eps)          (without a gain n = x)
//   (a, b) -> (a c - b s, b c + a s),  c, s = scale * cos, sin of position * freq[i]
// for the pairs (a, b) = (n[i], n[i + half]) or, interleaved, (n[2 i], n[2 i + 1]).  Backward, with u = x r:
//   dn = the transposed turn of dy;  dg = sum over tokens and heads of dn u;  dx = r (g dn - u mean(g dn u)).
// r is taken again from x, which the backward reads anyway: nothing is saved.
//
// Memory bounds it (2 elements moved an element forward, 3 backward, about 20 operations): 16384 tokens of 32 + 8 heads of 128
// in bf16 take 66 us forward and 111 us backward, 839 MB in all at 4.7 TB/s, where a copy of 2 GB reaches 4.9; 4096 tokens of 25
// + 25 heads of 64 without a norm 11 and 18 us.  So one pass each way and 16-byte accesses: a lane holds 16 elements of a head,
// eight pairs, both halves of a pair in the same lane, so the turn needs no exchange and the row sums cross 4 (dh 64) or 8
// (dh 128) lanes.  The angles of a token are worked out once for all its heads, into LDS: in 64 bits up to the fraction of a turn
// (at a position of 10^6 and a frequency near 1, 32 bits are 0.06 radians apart), then sin and cos of that fraction in 32.
#include "common.h"
#include "kernels.h"

#include <cmath>

namespace dp {

namespace {

constexpr int kThreads = 256;
// How a lane's pairs lie in memory: in halves 8 or 4 elements on end, in turn 8 elements (4 pairs) on end; kScalar: either way,
// element by element.
enum { kScalar = 0, kHalves = 1, kHalves4 = 2, kInterleaved = 3 };

template <typename T, int N> struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Run { T v[N]; };

// What one lane holds of a head: eight pairs (a, b), in runs of W consecutive ones.  `u`: the lane's place in its group of G
// lanes.  Pairs beyond the turned ones are neighbours in memory.
template <typename T, int FORM> struct Pairs {
  static constexpr int W = FORM == kHalves ? 8 : 4;
  int u, G, half, dh;
  bool inter;
  // pair i of the lane: its number, and whether the head has it
  __device__ __forceinline__ int number(int i) const { return FORM == kScalar ? u + G * i : 8 * u + i; }
  __device__ __forceinline__ bool has(int i) const { return FORM == kScalar ? number(i) < dh / 2 : 2 * number(i / W * W) < dh; }
  __device__ __forceinline__ bool turned(int i) const { return FORM == kScalar ? number(i) < half : number(i / W * W) < half; }
  // the elements a and b of pair i
  __device__ __forceinline__ int at(int i, int which) const {
    const int p = number(i);
    if (FORM == kInterleaved) return 2 * p + which;
    if (FORM == kScalar) return turned(i) && !inter ? p + which * half : 2 * p + which;
    return turned(i) ? p + which * half : 2 * number(i / W * W) + which * W + i % W;
  }
  // the lane's elements as they lie in memory, for loads that wait in registers
  struct Raw { Run<T, W> a[8 / W], b[8 / W]; };
  __device__ __forceinline__ void ask(const T *x, Raw &r) const {
#pragma unroll
    for (int i = 0; i < 8; i += W) {
      if (FORM == kScalar) {
#pragma unroll
        for (int j = 0; j < W; ++j)
          if (has(i + j)) { r.a[i / W].v[j] = x[at(i + j, 0)]; r.b[i / W].v[j] = x[at(i + j, 1)]; }
      } else if (has(i)) {   // (in turn: the four pairs' eight elements, in two parts)
        r.a[i / W] = *reinterpret_cast<const Run<T, W> *>(x + at(i, 0));
        r.b[i / W] = *reinterpret_cast<const Run<T, W> *>(x + (FORM == kInterleaved ? at(i, 0) + W : at(i, 1)));
      }
    }
  }
  __device__ __forceinline__ void take(const Raw &r, float (&a)[8], float (&b)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      T x = r.a[i / W].v[i % W], y = r.b[i / W].v[i % W];
      if (FORM == kInterleaved) {
        const int j = i % W;
        x = j < 2 ? r.a[i / W].v[2 * j] : r.b[i / W].v[2 * j - W];
        y = j < 2 ? r.a[i / W].v[2 * j + 1] : r.b[i / W].v[2 * j + 1 - W];
      }
      a[i] = has(i) ? (float)x : 0.f;   // (a head that does not fill its lanes: the rest adds nothing to the sums)
      b[i] = has(i) ? (float)y : 0.f;
    }
  }
  __device__ __forceinline__ void store(T *y, const float (&a)[8], const float (&b)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; i += W) {
      if (FORM == kScalar) {
#pragma unroll
        for (int j = i; j < i + W; ++j)
          if (has(j)) { stf(y + at(j, 0), a[j]); stf(y + at(j, 1), b[j]); }
      } else if (has(i)) {
        Run<T, W> lo, hi;
#pragma unroll
        for (int j = 0; j < W; ++j) {
          if (FORM == kInterleaved) {
            (j < 2 ? lo.v[2 * j] : hi.v[2 * j - W]) = (T)a[i + j];
            (j < 2 ? lo.v[2 * j + 1] : hi.v[2 * j + 1 - W]) = (T)b[i + j];
          } else {
            lo.v[j] = (T)a[i + j];
            hi.v[j] = (T)b[i + j];
          }
        }
        *reinterpret_cast<Run<T, W> *>(y + at(i, 0)) = lo;
        *reinterpret_cast<Run<T, W> *>(y + (FORM == kInterleaved ? at(i, 0) + W : at(i, 1))) = hi;
      }
    }
  }
  // turned by the token's angles (cs: cos and sin of its pairs), the other way round if BACK
  template <bool BACK> __device__ __forceinline__ void turn(const float2 *cs, float (&a)[8], float (&b)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (!turned(i)) continue;
      const float2 w = cs[number(i)];
      const float s = BACK ? -w.y : w.y, x = a[i], y = b[i];
      a[i] = x * w.x - y * s;
      b[i] = y * w.x + x * s;
    }
  }
};

// Sum over the G lanes of a group (a power of two, lanes side by side), in every one of them: up to 16 by exchanges inside the
// vector unit (neighbours, pairs, then mirrored quads and halves, whose lanes agree by then), beyond through LDS.
template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float group_sum(float v, int G) {
  if (G > 1) v = dpp_add<0xb1>(v);    // quad_perm 1 0 3 2
  if (G > 2) v = dpp_add<0x4e>(v);    // quad_perm 2 3 0 1
  if (G > 4) v = dpp_add<0x141>(v);   // row_half_mirror
  if (G > 8) v = dpp_add<0x140>(v);   // row_mirror
  if (G > 16) v += __shfl_xor(v, 16, 64);
  if (G > 32) v += __shfl_xor(v, 32, 64);
  return v;
}

// A vector of a block's tile: token t of the tile, head h (the queries' heads, then the keys').  Groups take them in turn: the
// step to a group's next one is kept as whole tokens and heads (a division a step cost a tenth of the instructions).
struct Place {
  int t, h;
  __device__ __forceinline__ void first(int it, int heads) { t = it / heads; h = it - t * heads; }
  __device__ __forceinline__ void advance(int dt, int dh, int heads) {
    t += dt; h += dh;
    if (h >= heads) { h -= heads; ++t; }
  }
};

// cos and sin of `tokens` tokens' pairs, from row r0 on
__device__ __forceinline__ void angles(const RotaryArgs &p, int r0, int tokens, float2 *cs) {
  for (int i = threadIdx.x; i < tokens * p.half; i += kThreads) {
    const int t = i / p.half, k = i - t * p.half, r = r0 + t;
    const int pos = p.positions != nullptr ? p.positions[r] : r % p.seq;
    const double turns = (double)pos * (double)p.freq[k] * 0.15915494309189533577;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    cs[i] = make_float2(p.scale * c, p.scale * s);
  }
}

// The vectors of a block's tokens, queries' and keys' heads of one token after the other, are dealt out to its groups of lanes;
// a group asks for its next vector before it works on the one it has.
template <typename T, int FORM, bool GAIN>
__global__ __launch_bounds__(kThreads) void qk_rotary_fwd_kernel(RotaryArgs p) {
  extern __shared__ float2 cs[];
  using P = Pairs<T, FORM>;
  const P me{(int)threadIdx.x & (p.group - 1), p.group, p.half, p.dh, p.interleaved != 0};
  const int heads = p.nq + p.nk, step_t = kThreads / p.group / heads, step_h = kThreads / p.group - step_t * heads;
  const int r0 = blockIdx.x * p.tokens, tokens = min(p.tokens, p.rows - r0);
  typename P::Raw next, gq, gk;
  auto ask = [&](const Place &at) {
    if (at.t >= tokens) return;
    const long r = r0 + at.t;
    me.ask(at.h < p.nq ? (const T *)p.q + r * p.ldq_in + (long)at.h * p.dh : (const T *)p.k + r * p.ldk_in + (long)(at.h - p.nq) * p.dh, next);
  };
  Place at;
  at.first(threadIdx.x / p.group, heads);
  ask(at);
  if (GAIN && p.q_gain != nullptr) me.ask((const T *)p.q_gain, gq);
  if (GAIN && p.k_gain != nullptr) me.ask((const T *)p.k_gain, gk);
  angles(p, r0, tokens, cs);
  __syncthreads();
  while (at.t < tokens) {
    float a[8], b[8];
    me.take(next, a, b);
    const int t = at.t, h = at.h;
    at.advance(step_t, step_h, heads);
    ask(at);
    const long r = r0 + t;
    const bool is_q = h < p.nq;
    if (GAIN && (is_q ? p.q_gain : p.k_gain) != nullptr) {
      float s = 0.f, ga[8], gb[8];
      if (is_q) me.take(gq, ga, gb); else me.take(gk, ga, gb);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += a[i] * a[i] + b[i] * b[i];
      const float rr = rsqrtf(group_sum(s, p.group) / (float)p.dh + p.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) { a[i] = a[i] * rr * ga[i]; b[i] = b[i] * rr * gb[i]; }
    }
    me.template turn<false>(cs + t * p.half, a, b);
    me.store(is_q ? (T *)p.q_out + r * p.ldq_out + (long)h * p.dh : (T *)p.k_out + r * p.ldk_out + (long)(h - p.nq) * p.dh, a, b);
  }
}

// A block leaves its sums of the gains' gradients in part[blockIdx.x] (dh for each gain there is, the queries' first); they are
// added over the blocks, in order, by launch_reduce_jobs.  A block alone writes them out itself (dq_gain, dk_gain).
template <typename T, int FORM, bool GAIN>
__global__ __launch_bounds__(kThreads) void qk_rotary_bwd_kernel(RotaryArgs p, T *dq_gain, T *dk_gain) {
  extern __shared__ float2 cs[];
  using P = Pairs<T, FORM>;
  const P me{(int)threadIdx.x & (p.group - 1), p.group, p.half, p.dh, p.interleaved != 0};
  const int heads = max(p.nq + p.nk, 1), step_t = kThreads / p.group / heads, step_h = kThreads / p.group - step_t * heads;
  float dq_a[8], dq_b[8], dk_a[8], dk_b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dq_a[i] = dq_b[i] = dk_a[i] = dk_b[i] = 0.f;
  // (dy: the gradient of what the forward wrote, at the rows of q_out, k_out; x and its gradient at those of q, k)
  typename P::Raw dy, x, gq, gk;
  int r0 = 0, tokens = 0;   // the tile at hand
  auto ask = [&](const Place &at) {
    if (at.t >= tokens) return;
    const long r = r0 + at.t;
    if (at.h < p.nq) {
      me.ask((const T *)p.dq_out + r * p.ldq_out + (long)at.h * p.dh, dy);
      if (GAIN && p.q_gain != nullptr) me.ask((const T *)p.q + r * p.ldq_in + (long)at.h * p.dh, x);
    } else {
      me.ask((const T *)p.dk_out + r * p.ldk_out + (long)(at.h - p.nq) * p.dh, dy);
      if (GAIN && p.k_gain != nullptr) me.ask((const T *)p.k + r * p.ldk_in + (long)(at.h - p.nq) * p.dh, x);
    }
  };
  if (GAIN && p.q_gain != nullptr) me.ask((const T *)p.q_gain, gq);
  if (GAIN && p.k_gain != nullptr) me.ask((const T *)p.k_gain, gk);
  for (long first = (long)blockIdx.x * p.tokens; first < p.rows; first += (long)gridDim.x * p.tokens) {
    r0 = (int)first;
    tokens = min(p.tokens, p.rows - r0);
    Place at;
    at.first(threadIdx.x / p.group, heads);
    ask(at);
    angles(p, r0, tokens, cs);
    __syncthreads();
    while (at.t < tokens) {
      const int t = at.t, h = at.h;
      const long r = r0 + t;
      const bool is_q = h < p.nq, gained = GAIN && (is_q ? p.q_gain : p.k_gain) != nullptr;
      float a[8], b[8], xa[8], xb[8], ga[8], gb[8];
      me.take(dy, a, b);
      if (gained) {
        me.take(x, xa, xb);
        if (is_q) me.take(gq, ga, gb); else me.take(gk, ga, gb);
      }
      at.advance(step_t, step_h, heads);
      ask(at);
      me.template turn<true>(cs + t * p.half, a, b);
      if (gained) {
        float s = 0.f, d = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s += xa[i] * xa[i] + xb[i] * xb[i];
          d += a[i] * ga[i] * xa[i] + b[i] * gb[i] * xb[i];
        }
        s = group_sum(s, p.group);
        d = group_sum(d, p.group);
        const float w = 1.f / (float)p.dh, rr = rsqrtf(s * w + p.eps), m = d * rr * w;   // m: mean(g dn u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float ua = xa[i] * rr, ub = xb[i] * rr, va = a[i] * ua, vb = b[i] * ub;
          dq_a[i] += is_q ? va : 0.f;
          dq_b[i] += is_q ? vb : 0.f;
          dk_a[i] += is_q ? 0.f : va;
          dk_b[i] += is_q ? 0.f : vb;
          a[i] = rr * (a[i] * ga[i] - ua * m);
          b[i] = rr * (b[i] * gb[i] - ub * m);
        }
      }
      me.store(is_q ? (T *)p.dq + r * p.ldq_in + (long)h * p.dh : (T *)p.dk + r * p.ldk_in + (long)(h - p.nq) * p.dh, a, b);
    }
    __syncthreads();   // (the next tile's angles, or the sums, go where this one's angles are)
  }
  if (!GAIN) return;
  // the block's sums: over the lanes of a wave that hold the same pairs, then over the waves, in order
  float *sums = reinterpret_cast<float *>(cs);   // [4 waves][dh]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto add = [&](float (&da)[8], float (&db)[8], float *to, T *out) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      for (int m = p.group; m < 64; m <<= 1) { da[i] += __shfl_xor(da[i], m, 64); db[i] += __shfl_xor(db[i], m, 64); }
    if (lane < p.group) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (me.has(i)) { sums[wave * p.dh + me.at(i, 0)] = da[i]; sums[wave * p.dh + me.at(i, 1)] = db[i]; }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.dh; e += kThreads) {
      const float v = ((sums[e] + sums[p.dh + e]) + sums[2 * p.dh + e]) + sums[3 * p.dh + e];
      if (gridDim.x == 1) stf(out + e, v); else to[e] = v;
    }
    __syncthreads();
  };
  float *part = p.part + (size_t)blockIdx.x * p.dh * ((p.q_gain != nullptr) + (p.k_gain != nullptr));
  if (p.q_gain != nullptr) { add(dq_a, dq_b, part, dq_gain); part += p.dh; }
  if (p.k_gain != nullptr) add(dk_a, dk_b, part, dk_gain);
}

constexpr int kSums = 1024;   // most blocks of a backward with gains (four a CU), each with its own sums

int lanes(int dh) {   // of a head: 16 elements each, a power of two of them
  int g = 1;
  while (16 * g < dh) g <<= 1;
  return g;
}
// Tokens a block takes at a time: about four vectors a group of lanes, so that a block's angles and its start are spread over
// them, as long as there are eight blocks a CU; at most 16 KB of angles.  (Forward and backward of 16384 tokens of 32 + 8 heads
// of 128, bf16, at 2 / 4 / 8 tokens: 191 / 178 / 188 us.)  Gradients of gains that fit one block's four vectors a group need
// no second launch to add them up (5 tokens of 2 + 1 heads: 11.3 us, 13.8 with it).
int tile_tokens(int rows, int heads, int group, int half, bool sums) {
  const int few = 4 * (kThreads / group), want = heads > 0 ? (few + heads - 1) / heads : 1, spread = (rows + 2047) / 2048;
  int t = sums && (long)rows * heads <= few ? rows : want < spread ? want : spread;
  if (half > 0 && t > 2048 / half) t = 2048 / half;
  return t < 1 ? 1 : t;
}

bool aligned(const void *a, const void *b, const void *c, long ld1, long ld2) {
  return ((((uintptr_t)a | (uintptr_t)b | (uintptr_t)c) & 15) | ((ld1 | ld2) & 7)) == 0;
}
int form(const RotaryArgs &p, bool bwd) {
  bool vec = p.dh % 8 == 0 && p.half % 4 == 0 && ((((uintptr_t)p.q_gain | (uintptr_t)p.k_gain) & 15) == 0);
  if (bwd) vec = vec && aligned(p.dq_out, p.dq, p.q_gain != nullptr ? p.q : nullptr, p.ldq_in, p.ldq_out) &&
                 aligned(p.dk_out, p.dk, p.k_gain != nullptr ? p.k : nullptr, p.ldk_in, p.ldk_out);
  else vec = vec && aligned(p.q, p.q_out, nullptr, p.ldq_in, p.ldq_out) && aligned(p.k, p.k_out, nullptr, p.ldk_in, p.ldk_out);
  return !vec ? kScalar : p.interleaved ? kInterleaved : p.dh % 16 == 0 && p.half % 8 == 0 ? kHalves : kHalves4;
}

template <typename T, int FORM, bool GAIN> hipError_t go(const RotaryArgs &p, bool bwd, int blocks, void *dq_gain, void *dk_gain, hipStream_t s) {
  size_t smem = (size_t)p.tokens * p.half * sizeof(float2);
  if (!bwd) {
    hipLaunchKernelGGL((qk_rotary_fwd_kernel<T, FORM, GAIN>), dim3(blocks), dim3(kThreads), smem, s, p);
  } else {
    if (smem < 16 * (size_t)p.dh) smem = 16 * (size_t)p.dh;
    hipLaunchKernelGGL((qk_rotary_bwd_kernel<T, FORM, GAIN>), dim3(blocks), dim3(kThreads), smem, s, p, (T *)dq_gain, (T *)dk_gain);
  }
  return hipGetLastError();
}
template <typename T, int FORM> hipError_t go(const RotaryArgs &p, bool bwd, int blocks, void *dq_gain, void *dk_gain, hipStream_t s) {
  return p.q_gain != nullptr || p.k_gain != nullptr ? go<T, FORM, true>(p, bwd, blocks, dq_gain, dk_gain, s)
                                                    : go<T, FORM, false>(p, bwd, blocks, dq_gain, dk_gain, s);
}
template <typename T> hipError_t go_form(const RotaryArgs &p, bool bwd, int blocks, void *dq_gain, void *dk_gain, hipStream_t s) {
  switch (form(p, bwd)) {
    case kHalves: return go<T, kHalves>(p, bwd, blocks, dq_gain, dk_gain, s);
    case kHalves4: return go<T, kHalves4>(p, bwd, blocks, dq_gain, dk_gain, s);
    case kInterleaved: return go<T, kInterleaved>(p, bwd, blocks, dq_gain, dk_gain, s);
    default: return go<T, kScalar>(p, bwd, blocks, dq_gain, dk_gain, s);
  }
}

}  // namespace

bool qk_rotary_supported(int dh) { return dh >= 2 && dh <= 1024 && dh % 2 == 0; }

size_t qk_rotary_ws_bytes(int rows, int dh) {
  return (size_t)(rows < 1 ? 1 : rows < kSums ? rows : kSums) * 2 * (size_t)dh * sizeof(float);
}

hipError_t launch_qk_rotary_fwd(int dtype, RotaryArgs p, hipStream_t s) {
  if (p.rows == 0 || p.nq + p.nk == 0) return hipSuccess;
  p.group = lanes(p.dh);
  p.tokens = tile_tokens(p.rows, p.nq + p.nk, p.group, p.half, false);
  const int blocks = (int)(((long)p.rows + p.tokens - 1) / p.tokens);
  return dtype == kBF16 ? go_form<bf16>(p, false, blocks, nullptr, nullptr, s) : go_form<float>(p, false, blocks, nullptr, nullptr, s);
}

hipError_t launch_qk_rotary_bwd(int dtype, RotaryArgs p, void *dq_gain, void *dk_gain, hipStream_t s) {
  const int sums = (p.q_gain != nullptr) + (p.k_gain != nullptr);
  if (p.nq + p.nk == 0) p.rows = 0;
  if (p.rows == 0 && sums == 0) return hipSuccess;
  p.group = lanes(p.dh);
  p.tokens = tile_tokens(p.rows, p.nq + p.nk, p.group, p.half, sums > 0);
  const int tiles = (int)(((long)p.rows + p.tokens - 1) / p.tokens);
  const int blocks = tiles < 1 ? 1 : sums && tiles > kSums ? kSums : tiles;   // (no rows: one block, which writes zeros)
  const hipError_t e = dtype == kBF16 ? go_form<bf16>(p, true, blocks, dq_gain, dk_gain, s) : go_form<float>(p, true, blocks, dq_gain, dk_gain, s);
  if (e != hipSuccess || sums == 0 || blocks == 1) return e;
  const ReduceJob j{p.part, blocks, sums * p.dh, p.dh, p.q_gain != nullptr ? dq_gain : dk_gain, dk_gain, nullptr};
  return launch_reduce_jobs(dtype, &j, 1, s);
}

}  // namespace dp
