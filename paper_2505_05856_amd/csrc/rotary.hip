// Queries and keys between their projection and the attention: every head's vector x (dh elements) is divided by its root
// mean square and multiplied by a gain, then its first 2 * half elements are turned by the token's position,
//   n = g x r, r = 1 / sqrt(mean(x^2) + eps)          (without a gain n = x)
//   (a, b) -> (a c - b s, b c + a s),  c, s = scale * cos, sin of position * freq[i]
// for the pairs (a, b) = (n[i], n[i + half]) or, interleaved, (n[2 i], n[2 i + 1]).  Backward, with u = x r:
//   dn = the transposed turn of dy;  dg = sum over tokens and heads of dn u;  dx = r (g dn - u mean(g dn u)).
// r is taken again from x, which the backward reads anyway: nothing is saved.
//
// Memory bounds it (2 elements moved an element forward, 3 backward, about 20 operations), so one pass each way and 16-byte
// accesses: a lane holds 16 elements of a head, eight pairs, both halves of a pair in the same lane, so the turn needs no
// exchange and the row sums cross 4 (dh 64) or 8 (dh 128) lanes.  The angles of a token are worked out once for all its heads,
// into LDS: in 64 bits up to the fraction of a turn (a position of 10^6 times a frequency near 1 has lost 0.06 of a turn's
// 32-bit digits), then sin and cos of that fraction in 32.
#include "common.h"
#include "kernels.h"

#include <cmath>

namespace dp {

namespace {

enum { kScalar = 0, kHalves = 1, kInterleaved = 2 };   // how a lane's pairs lie in memory; kScalar: either, element by element

// What one lane holds of a head: eight pairs (a, b).  `u`: the lane's place in its group of G lanes.
template <typename T, int FORM> struct Pairs {
  int u, G, half, dh;
  bool inter;
  // pair i of the lane: its number, and whether the head has it
  __device__ __forceinline__ int number(int i) const { return FORM == kScalar ? u + G * i : 8 * u + i; }
  __device__ __forceinline__ bool has(int i) const { return FORM == kScalar ? number(i) < dh / 2 : 16 * u < dh; }
  __device__ __forceinline__ bool turned(int i) const { return FORM == kScalar ? number(i) < half : 8 * u < half; }
  // the elements a and b of pair i; pairs that are not turned are neighbours (16 elements a lane in the vector forms)
  __device__ __forceinline__ int at(int i, int which) const {
    const int p = number(i);
    if (FORM == kScalar) return turned(i) ? (inter ? 2 * p + which : p + which * half) : 2 * p + which;
    if (FORM == kInterleaved) return 16 * u + 2 * i + which;
    return turned(i) ? p + which * half : 16 * u + 8 * which + i;
  }
  __device__ __forceinline__ void load(const T *x, float (&a)[8], float (&b)[8]) const {
    if constexpr (FORM == kScalar) {
#pragma unroll
      for (int i = 0; i < 8; ++i) { a[i] = has(i) ? ldf(x + at(i, 0)) : 0.f; b[i] = has(i) ? ldf(x + at(i, 1)) : 0.f; }
    } else if (!has(0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = b[i] = 0.f;
    } else if constexpr (FORM == kHalves) {
      load8(x + at(0, 0), a);
      load8(x + at(0, 1), b);
    } else {
      float lo[8], hi[8];
      load8(x + 16 * u, lo);
      load8(x + 16 * u + 8, hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) { a[i] = lo[2 * i]; b[i] = lo[2 * i + 1]; a[i + 4] = hi[2 * i]; b[i + 4] = hi[2 * i + 1]; }
    }
  }
  __device__ __forceinline__ void store(T *y, const float (&a)[8], const float (&b)[8]) const {
    if constexpr (FORM == kScalar) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (has(i)) { stf(y + at(i, 0), a[i]); stf(y + at(i, 1), b[i]); }
    } else if (has(0)) {
      if constexpr (FORM == kHalves) {
        store8(y + at(0, 0), a);
        store8(y + at(0, 1), b);
      } else {
        float lo[8], hi[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) { lo[2 * i] = a[i]; lo[2 * i + 1] = b[i]; hi[2 * i] = a[i + 4]; hi[2 * i + 1] = b[i + 4]; }
        store8(y + 16 * u, lo);
        store8(y + 16 * u + 8, hi);
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

__device__ __forceinline__ float group_sum(float v, int G) {
  for (int m = 1; m < G; m <<= 1) v += __shfl_xor(v, m, 64);
  return v;
}

// cos and sin of `tokens` tokens' pairs, from row r0 on
__device__ __forceinline__ void angles(const RotaryArgs &p, int r0, int tokens, float2 *cs) {
  for (int i = threadIdx.x; i < tokens * p.half; i += 256) {
    const int t = i / p.half, k = i - t * p.half, r = r0 + t;
    const int pos = p.positions != nullptr ? p.positions[r] : r % p.seq;
    const double turns = (double)pos * (double)p.freq[k] * 0.15915494309189533577;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    cs[i] = make_float2(p.scale * c, p.scale * s);
  }
}

template <typename T, int FORM>
__global__ __launch_bounds__(256) void qk_rotary_fwd_kernel(RotaryArgs p) {
  extern __shared__ float2 cs[];
  Pairs<T, FORM> me{(int)threadIdx.x & (p.group - 1), p.group, p.half, p.dh, p.interleaved != 0};
  const int first = threadIdx.x / p.group, step = 256 / p.group;
  const int r0 = blockIdx.x * p.tokens, tokens = min(p.tokens, p.rows - r0);
  angles(p, r0, tokens, cs);
  __syncthreads();
  auto side = [&](const void *in, void *out, const void *gain, int heads, long ld_in, long ld_out) {
    float ga[8], gb[8];
    if (gain != nullptr) me.load((const T *)gain, ga, gb);
    for (int it = first; it < tokens * heads; it += step) {
      const int t = it / heads, h = it - t * heads;
      float a[8], b[8];
      me.load((const T *)in + (long)(r0 + t) * ld_in + (long)h * p.dh, a, b);
      if (gain != nullptr) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += a[i] * a[i] + b[i] * b[i];
        const float r = rsqrtf(group_sum(s, p.group) / (float)p.dh + p.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) { a[i] = a[i] * r * ga[i]; b[i] = b[i] * r * gb[i]; }
      }
      me.template turn<false>(cs + t * p.half, a, b);
      me.store((T *)out + (long)(r0 + t) * ld_out + (long)h * p.dh, a, b);
    }
  };
  side(p.q, p.q_out, p.q_gain, p.nq, p.ldq_in, p.ldq_out);
  side(p.k, p.k_out, p.k_gain, p.nk, p.ldk_in, p.ldk_out);
}

// A block takes token tiles blockIdx.x, blockIdx.x + gridDim.x, ... and leaves its sums of the gains' gradients in
// part[blockIdx.x] (dh for each gain there is, the queries' first); they are added over the blocks, in order, by
// launch_reduce_jobs.
template <typename T, int FORM>
__global__ __launch_bounds__(256) void qk_rotary_bwd_kernel(RotaryArgs p) {
  extern __shared__ float2 cs[];
  Pairs<T, FORM> me{(int)threadIdx.x & (p.group - 1), p.group, p.half, p.dh, p.interleaved != 0};
  const int first = threadIdx.x / p.group, step = 256 / p.group;
  float dq_a[8], dq_b[8], dk_a[8], dk_b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dq_a[i] = dq_b[i] = dk_a[i] = dk_b[i] = 0.f;
  for (long r = (long)blockIdx.x * p.tokens; r < p.rows; r += (long)gridDim.x * p.tokens) {
    const int r0 = (int)r, tokens = min(p.tokens, p.rows - r0);
    angles(p, r0, tokens, cs);
    __syncthreads();
    // (dy: the gradient of what the forward wrote, at the rows of q_out, k_out; x and its gradient at those of q, k)
    auto side = [&](const void *dy, const void *in, void *dx, const void *gain, int heads, long ld_in, long ld_out, float (&da)[8],
                    float (&db)[8]) {
      float ga[8], gb[8];
      if (gain != nullptr) me.load((const T *)gain, ga, gb);
      for (int it = first; it < tokens * heads; it += step) {
        const int t = it / heads, h = it - t * heads;
        const long at_in = (long)(r0 + t) * ld_in + (long)h * p.dh;
        float a[8], b[8];
        me.load((const T *)dy + (long)(r0 + t) * ld_out + (long)h * p.dh, a, b);
        if (gain == nullptr) {
          me.template turn<true>(cs + t * p.half, a, b);
        } else {
          float xa[8], xb[8];
          me.load((const T *)in + at_in, xa, xb);
          me.template turn<true>(cs + t * p.half, a, b);
          float s = 0.f, d = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            s += xa[i] * xa[i] + xb[i] * xb[i];
            d += a[i] * ga[i] * xa[i] + b[i] * gb[i] * xb[i];
          }
          s = group_sum(s, p.group);
          d = group_sum(d, p.group);
          const float n = 1.f / (float)p.dh, rr = rsqrtf(s * n + p.eps), m = d * rr * n;   // m: mean(g dn u)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float ua = xa[i] * rr, ub = xb[i] * rr;
            da[i] += a[i] * ua;
            db[i] += b[i] * ub;
            a[i] = rr * (a[i] * ga[i] - ua * m);
            b[i] = rr * (b[i] * gb[i] - ub * m);
          }
        }
        me.store((T *)dx + at_in, a, b);
      }
    };
    side(p.dq_out, p.q, p.dq, p.q_gain, p.nq, p.ldq_in, p.ldq_out, dq_a, dq_b);
    side(p.dk_out, p.k, p.dk, p.k_gain, p.nk, p.ldk_in, p.ldk_out, dk_a, dk_b);
    __syncthreads();   // (the next tile's angles go where this one's are)
  }
  // the block's sums: over the lanes of a wave that hold the same pairs, then over the waves, in order
  float *sums = reinterpret_cast<float *>(cs);   // [4 waves][dh]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto add = [&](float (&da)[8], float (&db)[8], float *to) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      for (int m = p.group; m < 64; m <<= 1) { da[i] += __shfl_xor(da[i], m, 64); db[i] += __shfl_xor(db[i], m, 64); }
    if (lane < p.group) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (me.has(i)) { sums[wave * p.dh + me.at(i, 0)] = da[i]; sums[wave * p.dh + me.at(i, 1)] = db[i]; }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.dh; e += 256)
      to[e] = ((sums[e] + sums[p.dh + e]) + sums[2 * p.dh + e]) + sums[3 * p.dh + e];
    __syncthreads();
  };
  float *part = p.part + (size_t)blockIdx.x * p.dh * ((p.q_gain != nullptr) + (p.k_gain != nullptr));
  if (p.q_gain != nullptr) { add(dq_a, dq_b, part); part += p.dh; }
  if (p.k_gain != nullptr) add(dk_a, dk_b, part);
}

constexpr int kBlocks = 1024;   // most blocks of the backward (four a CU), each with its own sums

// Tokens a block takes at a time: about four vectors a group of lanes, so that a block's angles and its start are spread over
// them, as long as there are eight blocks a CU; at most 32 KB of angles.
int tile_tokens(int rows, int heads, int group, int half) {
  const int want = (4 * (256 / group) + heads - 1) / heads, spread = (rows + 2047) / 2048;
  int t = want < spread ? want : spread;
  if (half > 0 && t > 4096 / half) t = 4096 / half;
  return t < 1 ? 1 : t;
}
int lanes(int dh) {   // of a head: 16 elements each, a power of two of them
  int g = 1;
  while (16 * g < dh) g <<= 1;
  return g;
}
int bwd_blocks(int rows, int tokens) {
  const int tiles = (rows + tokens - 1) / tokens;
  return tiles < 1 ? 1 : tiles < kBlocks ? tiles : kBlocks;
}

bool aligned(const void *a, const void *b, const void *c, long ld1, long ld2) {
  return ((((uintptr_t)a | (uintptr_t)b | (uintptr_t)c) & 15) | ((ld1 | ld2) & 7)) == 0;
}
int form(const RotaryArgs &p, bool bwd) {
  bool vec = p.dh % 16 == 0 && p.half % 8 == 0 && ((((uintptr_t)p.q_gain | (uintptr_t)p.k_gain) & 15) == 0);
  if (bwd) vec = vec && aligned(p.dq_out, p.dq, p.q_gain != nullptr ? p.q : nullptr, p.ldq_in, p.ldq_out) &&
                 aligned(p.dk_out, p.dk, p.k_gain != nullptr ? p.k : nullptr, p.ldk_in, p.ldk_out);
  else vec = vec && aligned(p.q, p.q_out, nullptr, p.ldq_in, p.ldq_out) && aligned(p.k, p.k_out, nullptr, p.ldk_in, p.ldk_out);
  return !vec ? kScalar : p.interleaved ? kInterleaved : kHalves;
}

template <typename T, int FORM> hipError_t go(const RotaryArgs &p, bool bwd, int blocks, hipStream_t s) {
  size_t smem = (size_t)p.tokens * p.half * sizeof(float2);
  if (!bwd) {
    hipLaunchKernelGGL((qk_rotary_fwd_kernel<T, FORM>), dim3(blocks), dim3(256), smem, s, p);
  } else {
    if (smem < 16 * (size_t)p.dh) smem = 16 * (size_t)p.dh;
    hipLaunchKernelGGL((qk_rotary_bwd_kernel<T, FORM>), dim3(blocks), dim3(256), smem, s, p);
  }
  return hipGetLastError();
}
template <typename T> hipError_t go_form(const RotaryArgs &p, bool bwd, int blocks, hipStream_t s) {
  switch (form(p, bwd)) {
    case kHalves: return go<T, kHalves>(p, bwd, blocks, s);
    case kInterleaved: return go<T, kInterleaved>(p, bwd, blocks, s);
    default: return go<T, kScalar>(p, bwd, blocks, s);
  }
}

}  // namespace

bool qk_rotary_supported(int dh) { return dh >= 2 && dh <= 1024 && dh % 2 == 0; }

size_t qk_rotary_ws_bytes(int rows, int dh) {
  return (size_t)(rows < kBlocks ? (rows < 1 ? 1 : rows) : kBlocks) * 2 * (size_t)dh * sizeof(float);
}

hipError_t launch_qk_rotary_fwd(int dtype, RotaryArgs p, hipStream_t s) {
  if (p.rows == 0 || p.nq + p.nk == 0) return hipSuccess;
  p.group = lanes(p.dh);
  p.tokens = tile_tokens(p.rows, p.nq + p.nk, p.group, p.half);
  const int blocks = (p.rows + p.tokens - 1) / p.tokens;
  return dtype == kBF16 ? go_form<bf16>(p, false, blocks, s) : go_form<float>(p, false, blocks, s);
}

hipError_t launch_qk_rotary_bwd(int dtype, RotaryArgs p, void *dq_gain, void *dk_gain, hipStream_t s) {
  if (p.nq + p.nk == 0 || (p.rows == 0 && p.q_gain == nullptr && p.k_gain == nullptr)) return hipSuccess;
  p.group = lanes(p.dh);
  p.tokens = tile_tokens(p.rows, p.nq + p.nk, p.group, p.half);
  const int sums = (p.q_gain != nullptr) + (p.k_gain != nullptr);
  const int blocks = sums ? bwd_blocks(p.rows, p.tokens) : (p.rows + p.tokens - 1) / p.tokens;
  const hipError_t e = dtype == kBF16 ? go_form<bf16>(p, true, blocks, s) : go_form<float>(p, true, blocks, s);
  if (e != hipSuccess || sums == 0) return e;
  const ReduceJob j{p.part, blocks, sums * p.dh, p.dh, p.q_gain != nullptr ? dq_gain : dk_gain, dk_gain, nullptr};
  return launch_reduce_jobs(dtype, &j, 1, s);
}

}  // namespace dp
