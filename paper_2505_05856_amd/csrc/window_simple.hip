// Sliding-window attention on the vector ALUs, one wavefront per query row (forward, dQ) or per key row (dK, dV): any alignment and
// head dimensions up to 256, for the operands the matrix-core kernels do not take.  A row's keys are two runs, the first `sinks`
// keys and the window, and only those are read, 64 at a time: a lane takes one key's logit (a dot product along its row), then
// the wave adds the 64 weighted rows with its lanes along the head's columns.  The softmax is taken in one pass, with a running
// maximum and sum.  (fp32, 64 samples of 16 tokens, 32 + 8 heads of 64: 127 us forward, 418 backward, where the matrix cores take 19
// and 50; 40 tokens: 300 and 956 for 31 and 102; alone with one token a sample it is level.)
#include "common.h"
#include "kernels.h"

namespace dp {

namespace {

constexpr int kMaxDim = 256, kCols = kMaxDim / 64;

template <typename T> __device__ __forceinline__ float dot(const float *a, const T *p, int dh) {
  float s = 0.f;
  for (int d = 0; d < dh; ++d) s += a[d] * ldf(p + d);
  return s;
}

// What lanes of this wave wrote to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The runs of keys that query i sees: [0, n0) and [k1, i].
struct Runs { int n0, k1; };
__device__ __forceinline__ Runs runs_of(const WindowArgs &a, int i) {
  const int first = i >= a.window ? i - a.window + 1 : 0;
  return Runs{min(a.sinks, first), first};
}

// one wave a (sample, head, query); rows past the sample's length become zeros
template <typename T> __global__ __launch_bounds__(256) void window_fwd_simple_kernel(WindowArgs a) {
  __shared__ float rows[4][kMaxDim];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float *qs = rows[wave];
  const long n = (long)a.B * a.nq * a.S;
  for (long id = (long)blockIdx.x * 4 + wave; id < n; id += (long)gridDim.x * 4) {
    const int i = (int)(id % a.S), h = (int)(id / a.S % a.nq), b = (int)(id / ((long)a.S * a.nq));
    const int len = window_len(a, a.lens != nullptr ? a.lens[b] : 0);
    const long row = (long)b * a.S;
    const T *q = (const T *)a.q + (row + i) * a.ldq + (long)h * a.dh;
    const int kh = h / (a.nq / a.nk);
    const T *k = (const T *)a.k + row * a.ldk + (long)kh * a.dh, *v = (const T *)a.v + row * a.ldv + (long)kh * a.dh;
    float m = -INFINITY, l = 0.f, acc[kCols] = {};
    if (i < len) {
      for (int d = lane; d < a.dh; d += 64) qs[d] = ldf(q + d);
      wave_sync();
      auto run = [&](int j0, int j1) {
        for (int jb = j0; jb < j1; jb += 64) {
          const int j = jb + lane, cnt = min(64, j1 - jb);
          const float x = j < j1 ? a.scale * dot(qs, k + (long)j * a.ldk, a.dh) : -INFINITY;
          const float m_new = fmaxf(m, wave_max(x)), old = m == -INFINITY ? 0.f : expf(m - m_new);
          const float p = m_new == -INFINITY || j >= j1 ? 0.f : expf(x - m_new);
          l = l * old + wave_sum(p);
#pragma unroll
          for (int c = 0; c < kCols; ++c) acc[c] *= old;
          for (int t = 0; t < cnt; ++t) {
            const float w = __shfl(p, t, 64);
#pragma unroll
            for (int c = 0; c < kCols; ++c)
              if (lane + 64 * c < a.dh) acc[c] += w * ldf(v + (long)(jb + t) * a.ldv + lane + 64 * c);
          }
          m = m_new;
        }
      };
      const Runs r = runs_of(a, i);
      run(0, r.n0);
      run(r.k1, i + 1);
      wave_sync();
    }
    if (a.lse != nullptr && lane == 0) a.lse[id] = i < len ? m + logf(l) : -INFINITY;
    if (a.o != nullptr) {
      T *o = (T *)a.o + (row + i) * a.ldo + (long)h * a.dh;
#pragma unroll
      for (int c = 0; c < kCols; ++c)
        if (lane + 64 * c < a.dh) stf(o + lane + 64 * c, i < len ? acc[c] / l : 0.f);
    }
  }
}

// D_i = <dO_i, O_i>, left in ws[b, h, i];  dS_ij = P_ij (dP_ij - D_i);  dQ_i = scale * sum_j dS_ij K_j
template <typename T> __global__ __launch_bounds__(256) void window_dq_simple_kernel(WindowArgs a) {
  __shared__ float rows[4][2 * kMaxDim];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float *qs = rows[wave], *gs = qs + kMaxDim;
  const long n = (long)a.B * a.nq * a.S;
  for (long id = (long)blockIdx.x * 4 + wave; id < n; id += (long)gridDim.x * 4) {
    const int i = (int)(id % a.S), h = (int)(id / a.S % a.nq), b = (int)(id / ((long)a.S * a.nq));
    const int len = window_len(a, a.lens != nullptr ? a.lens[b] : 0);
    const long row = (long)b * a.S;
    const int kh = h / (a.nq / a.nk);
    const T *k = (const T *)a.k + row * a.ldk + (long)kh * a.dh, *v = (const T *)a.v + row * a.ldv + (long)kh * a.dh;
    const long at_q = (row + i) * a.ldq + (long)h * a.dh, at_o = (row + i) * a.ldo + (long)h * a.dh;
    float acc[kCols] = {};
    if (i < len) {
      float dsum = 0.f;
      for (int d = lane; d < a.dh; d += 64) {
        qs[d] = ldf((const T *)a.q + at_q + d);
        gs[d] = ldf((const T *)a.d_o + at_o + d);
        dsum += gs[d] * ldf((const T *)a.o_in + at_o + d);
      }
      dsum = wave_sum(dsum);
      wave_sync();
      if (lane == 0) a.ws[id] = dsum;
      const float L = a.lse[id];
      auto run = [&](int j0, int j1) {
        for (int jb = j0; jb < j1; jb += 64) {
          const int j = jb + lane, cnt = min(64, j1 - jb);
          float ds = 0.f;
          if (j < j1) ds = expf(a.scale * dot(qs, k + (long)j * a.ldk, a.dh) - L) * (dot(gs, v + (long)j * a.ldv, a.dh) - dsum);
          for (int t = 0; t < cnt; ++t) {
            const float w = __shfl(ds, t, 64);
#pragma unroll
            for (int c = 0; c < kCols; ++c)
              if (lane + 64 * c < a.dh) acc[c] += w * ldf(k + (long)(jb + t) * a.ldk + lane + 64 * c);
          }
        }
      };
      const Runs r = runs_of(a, i);
      run(0, r.n0);
      run(r.k1, i + 1);
      wave_sync();
    }
#pragma unroll
    for (int c = 0; c < kCols; ++c)
      if (lane + 64 * c < a.dh) stf((T *)a.dq + at_q + lane + 64 * c, acc[c] * a.scale);
  }
}

// dV_j = sum_i P_ij dO_i;  dK_j = scale * sum_i dS_ij Q_i, over the queries of all heads that read the key's
template <typename T> __global__ __launch_bounds__(256) void window_dkv_simple_kernel(WindowArgs a) {
  __shared__ float rows[4][2 * kMaxDim];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float *ks = rows[wave], *vs = ks + kMaxDim;
  const int group = a.nq / a.nk;
  const long n = (long)a.B * a.nk * a.S;
  for (long id = (long)blockIdx.x * 4 + wave; id < n; id += (long)gridDim.x * 4) {
    const int j = (int)(id % a.S), kh = (int)(id / a.S % a.nk), b = (int)(id / ((long)a.S * a.nk));
    const int len = window_len(a, a.lens != nullptr ? a.lens[b] : 0);
    const long row = (long)b * a.S, at_k = (row + j) * a.ldk + (long)kh * a.dh, at_v = (row + j) * a.ldv + (long)kh * a.dh;
    float dk[kCols] = {}, dv[kCols] = {};
    if (j < len) {
      for (int d = lane; d < a.dh; d += 64) {
        ks[d] = ldf((const T *)a.k + at_k + d);
        vs[d] = ldf((const T *)a.v + at_v + d);
      }
      wave_sync();
      const int i1 = j < a.sinks || a.window > len - j ? len : j + a.window;
      for (int g = 0; g < group; ++g) {
        const int h = kh * group + g;
        const T *q = (const T *)a.q + row * a.ldq + (long)h * a.dh, *d_o = (const T *)a.d_o + row * a.ldo + (long)h * a.dh;
        const float *lse = a.lse + ((long)b * a.nq + h) * a.S, *dsum = a.ws + ((long)b * a.nq + h) * a.S;
        for (int ib = j; ib < i1; ib += 64) {
          const int i = ib + lane, cnt = min(64, i1 - ib);
          float p = 0.f, ds = 0.f;
          if (i < i1) {
            p = expf(a.scale * dot(ks, q + (long)i * a.ldq, a.dh) - lse[i]);
            ds = p * (dot(vs, d_o + (long)i * a.ldo, a.dh) - dsum[i]);
          }
          for (int t = 0; t < cnt; ++t) {
            const float wp = __shfl(p, t, 64), ws = __shfl(ds, t, 64);
#pragma unroll
            for (int c = 0; c < kCols; ++c)
              if (lane + 64 * c < a.dh) {
                dv[c] += wp * ldf(d_o + (long)(ib + t) * a.ldo + lane + 64 * c);
                dk[c] += ws * ldf(q + (long)(ib + t) * a.ldq + lane + 64 * c);
              }
          }
        }
      }
      wave_sync();
    }
#pragma unroll
    for (int c = 0; c < kCols; ++c)
      if (lane + 64 * c < a.dh) {
        stf((T *)a.dk + at_k + lane + 64 * c, dk[c] * a.scale);
        stf((T *)a.dv + at_v + lane + 64 * c, dv[c]);
      }
  }
}

int blocks_for(long rows) {   // four rows a block at a time; a launch has less than 2^32 threads
  const long n = (rows + 3) / 4;
  return (int)(n < (1 << 22) ? n : 1 << 22);
}

}  // namespace

hipError_t launch_window_fwd_simple(int dtype, const WindowArgs &a, hipStream_t s) {
  const int blocks = blocks_for((long)a.B * a.nq * a.S);
  if (dtype == kBF16) hipLaunchKernelGGL((window_fwd_simple_kernel<bf16>), dim3(blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((window_fwd_simple_kernel<float>), dim3(blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_window_bwd_simple(int dtype, const WindowArgs &a, hipStream_t s) {
  const int bq = blocks_for((long)a.B * a.nq * a.S), bk = blocks_for((long)a.B * a.nk * a.S);
  if (dtype == kBF16) {
    hipLaunchKernelGGL((window_dq_simple_kernel<bf16>), dim3(bq), dim3(256), 0, s, a);
    hipLaunchKernelGGL((window_dkv_simple_kernel<bf16>), dim3(bk), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((window_dq_simple_kernel<float>), dim3(bq), dim3(256), 0, s, a);
    hipLaunchKernelGGL((window_dkv_simple_kernel<float>), dim3(bk), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

// ---- which kernels a call runs
static WindowArgs clipped(WindowArgs a) {   // a window that with the first keys covers the sequence: all of it
  if ((long)a.window + a.sinks >= a.S) { a.window = a.S; a.sinks = 0; }
  return a;
}
size_t window_ws_bytes(int dtype, const WindowArgs &args) {
  const WindowArgs a = clipped(args);
  const size_t simple = (size_t)a.B * a.nq * a.S * sizeof(float);
  const size_t matrix = a.S == 0 ? 0 : dtype == kBF16 ? window_mfma_ws_bytes(a) : window_f32_ws_bytes(a);
  return simple > matrix ? simple : matrix;
}
hipError_t launch_window_fwd(int dtype, const WindowArgs &args, hipStream_t s) {
  const WindowArgs a = clipped(args);
  if (dtype == kBF16 && window_mfma_supported(a)) return launch_window_fwd_mfma(a, s);
  if (dtype == kF32 && window_f32_supported(a)) return launch_window_fwd_f32(a, s);
  return launch_window_fwd_simple(dtype, a, s);
}
hipError_t launch_window_bwd(int dtype, const WindowArgs &args, hipStream_t s) {
  const WindowArgs a = clipped(args);
  if (dtype == kBF16 && window_mfma_supported(a)) return launch_window_bwd_mfma(a, s);
  if (dtype == kF32 && window_f32_supported(a)) return launch_window_bwd_f32(a, s);
  return launch_window_bwd_simple(dtype, a, s);
}

}  // namespace dp
