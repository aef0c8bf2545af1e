// What the matrix-core kernels of sliding-window attention share, in bf16 and in fp32: which keys a query sees, the tiles that
// hold them, how the walks of the key blocks are cut into pieces and added up.
#pragma once
#include "attn_tile.h"

namespace dp {

namespace {

constexpr int kCus = 256;

// ---- what a query, or a key, sees ------------------------------------------------------------------
// bits x and up of a 32-bit word (any x)
__device__ __forceinline__ uint32_t bits_from(int x) { return (uint32_t)(0xffffffffull << min(max(x, 0), 32)); }
// the hidden ones of keys jb .. jb+31 for query i
__device__ __forceinline__ uint32_t hidden_keys(int i, int jb, int window, int sinks) {
  return bits_from(i + 1 - jb) | (bits_from(sinks - jb) & ~bits_from(i - window + 1 - jb));
}
// the hidden ones of queries ib .. ib+31 for key j
__device__ __forceinline__ uint32_t hidden_queries(int j, int ib, int window, int sinks) {
  return ~bits_from(j - ib) | (j < sinks ? 0u : bits_from(j + window - ib));
}
// -inf for the hidden ones of a 32x32 result's 16 elements a lane (rows acc_row(e, lane))
__device__ __forceinline__ void hide(f32x16 &v, uint32_t hidden, int hh) {
  const int h = (int)(hidden >> (4 * hh));
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    int m;   // all ones where hidden (written out: the compiler makes a test, a compare and a select of it)
    asm("v_bfe_i32 %0, %1, %2, 1" : "=v"(m) : "v"(h), "n"(8 * (e >> 2) + (e & 3)));
    v[e] = __int_as_float((m & 0xff800000) | (~m & __float_as_int(v[e])));
  }
}

// The key tiles (N keys) that a block of ROWS queries from q0 on walks: the first `head` tiles, which hold first keys, then those
// of its window.
template <int N, int ROWS> struct KeyTiles {
  int head, gap, n;   // n: how many in all; tile t of the walk is t, or t + gap from `head` on
  __device__ __forceinline__ KeyTiles(int q0, int len, int window, int sinks) {
    const int end = (min(q0 + ROWS, len) - 1) / N + 1, w0 = max(q0 - window + 1, 0) / N;
    head = min((sinks + N - 1) / N, w0);
    gap = w0 - head;
    n = end - gap;
  }
  __device__ __forceinline__ int first_key(int t) const { return (t < head ? t : t + gap) * N; }
};

// Rows of sample b that hold a sequence (the same in every lane, and known to be)
__device__ __forceinline__ int sample_len(const WindowArgs &a, int b) {
  return __builtin_amdgcn_readfirstlane(window_len(a, a.lens != nullptr ? a.lens[b] : 0));
}

// How the walks over query tiles (64 queries) are cut.  Key block kb (ROWS keys) of a key head walks, for each query head of its
// group, the tiles from its own first to the end of its window: `parts` pieces.  Key blocks below `first` hold keys that all
// later queries see: the rest of the sequence, `far` pieces more.
// Key blocks below `full` have a whole window of queries after them, the others a shorter walk.  `together`: how many heads' shorter
// walks an XCD takes at a time.
struct KeyWork { int key_blocks, parts, first, far, full, together; };

struct Walk { int t0, nt, begin, end; };   // query tiles t0 .. t0+nt-1 of each head in turn; items begin .. end-1 of that list
template <int ROWS> __host__ __device__ __forceinline__ Walk walk_of(const KeyWork &w, int kb, int piece, int len, int window, int group) {
  const int tiles = (len + BKV - 1) / BKV, t0 = kb * (ROWS / BKV);
  const long last = ((long)kb * ROWS + ROWS - 1 + window - 1) / BKV;   // the last tile of the window
  const int t1 = last + 1 < tiles ? (int)last + 1 : tiles;
  Walk r;
  const bool far = piece >= w.parts;
  r.t0 = far ? (t1 > t0 ? t1 : t0) : t0;
  const int end = far ? tiles : t1;
  r.nt = end > r.t0 ? end - r.t0 : 0;
  const int n = r.nt * group, pieces = far ? w.far : w.parts, chunk = (n + pieces - 1) / pieces, i = far ? piece - w.parts : piece;
  r.begin = i * chunk < n ? i * chunk : n;
  r.end = r.begin + chunk < n ? r.begin + chunk : n;
  return r;
}
// Which piece a workgroup takes.  Workgroup i runs on XCD i % 8, and an XCD starts its own in order.  Whole walks come first, a head
// (its far pieces, then its key blocks) after the other: an XCD gets all of a head's, or where the heads do not go round evenly
// four in a row, so that those that share queries share an L2.  The shorter walks follow, in falling length: they fill the holes
// that the last whole ones leave, on every XCD alike.  (Contiguous shares in head order gave one XCD the ends of the sequence
// alone: 16384 tokens of 4 + 1 heads, window 4096, took 1.2 times as long.)  They go one by one to the XCDs, or, heads going round
// evenly, those of an XCD's own heads, as many heads at a time as fill its CUs or, if that is more, its L2 with their queries.
struct Piece { int head, kb, piece; };
__device__ __forceinline__ Piece piece_at(const KeyWork &w, int i, int heads) {
  const int nfar = w.first * w.far, per_head = nfar + w.full * w.parts, whole = heads * per_head;
  Piece p;
  if (i < whole) {
    const int run = heads % 8 == 0 ? per_head : 4, dealt = whole / (8 * run) * (8 * run);
    const int at = i < dealt ? i / (8 * run) * (8 * run) + i % 8 * run + i / 8 % run : i;
    p.head = at / per_head;
    const int id = at - p.head * per_head;
    p.kb = id < nfar ? id / w.far : (id - nfar) / w.parts;
    p.piece = id < nfar ? w.parts + id % w.far : (id - nfar) % w.parts;
  } else {
    const int id = i - whole, rows = (w.key_blocks - w.full) * w.parts;
    int first = 0, step = 1, n = heads, at = id;   // heads first, first + step ..: n of them together
    if (heads % 8 == 0) {
      const int own = heads / 8, set = id / 8 / (w.together * rows);
      first = id % 8 + 8 * w.together * set;
      step = 8;
      n = min(w.together, own - w.together * set);
      at = id / 8 - w.together * set * rows;
    }
    const int row = at / n;
    p.head = first + step * (at - row * n);
    p.kb = w.full + row / w.parts;
    p.piece = row % w.parts;
  }
  return p;
}
// Where a piece's sums go: a slot of the workspace (two [ROWS][DH] arrays), or -1: it is its block's only one, the result itself.
// The slots of a block's window, and those of the rest, follow each other.
__host__ __device__ __forceinline__ long slot_of(const KeyWork &w, long head, int kb, int piece) {
  if (w.parts == 1) return kb >= w.first ? -1 : (head * w.first + kb) * (1 + (long)w.far) + piece;
  const long windows = (long)w.key_blocks * w.parts;   // slots a head: those of the windows, then the rest's
  return head * (windows + (long)w.first * w.far) +
         (piece < w.parts ? (long)kb * w.parts + piece : windows + (long)kb * w.far + piece - w.parts);
}

// dK, dV of the key blocks whose walk was cut: the pieces' sums, in order.  Block: kSumRows keys of one of the two, DH / 4 lanes a key.
constexpr int kSumRows = 8;
template <typename T, int ROWS, int DH>
__global__ __launch_bounds__(kSumRows * DH / 4) void window_dkv_sum_kernel(WindowArgs a, KeyWork w, const float *__restrict__ sums, int blocks_per_head) {
  constexpr int LANES = DH / 4, PARTS = ROWS / kSumRows;   // lanes a row, blocks a key block and result
  const int group = a.nq / a.nk;
  const int r = (int)(blockIdx.x % PARTS) * kSumRows + (int)threadIdx.x / LANES, which = (blockIdx.x / PARTS) & 1, id = blockIdx.x / (2 * PARTS);
  const int head = id / blocks_per_head, kb = id - head * blocks_per_head;
  const int kh = head % a.nk, b = head / a.nk, len = sample_len(a, b);
  // how many of the two kinds of pieces hold anything (those from some piece on are empty)
  auto held = [&](int first, int pieces) {
    if (pieces == 0) return 0;
    const Walk r = walk_of<ROWS>(w, kb, first, len, a.window, group);
    const int n = r.nt * group, chunk = r.end - r.begin;
    return chunk == 0 ? 0 : (n + chunk - 1) / chunk;
  };
  const bool any = kb * ROWS < len;
  const int near = any ? held(0, w.parts) : 0, far = any && kb < w.first ? held(w.parts, w.far) : 0;
  const long slot = 2 * ROWS * DH;
  const float *pn = sums + slot_of(w, head, kb, 0) * slot + which * ROWS * DH;
  const float *pf = kb < w.first ? sums + slot_of(w, head, kb, w.parts) * slot + which * ROWS * DH : pn;
  const int col = (threadIdx.x % LANES) * 4;
  if (col >= a.dh) return;
  typedef T T4 __attribute__((ext_vector_type(4)));
  const int j = kb * ROWS + r;
  if (j >= a.S) return;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (j < len) {
#pragma unroll 8
    for (int p = 0; p < near; ++p) s += *reinterpret_cast<const f32x4 *>(pn + p * slot + r * DH + col);
#pragma unroll 8
    for (int p = 0; p < far; ++p) s += *reinterpret_cast<const f32x4 *>(pf + p * slot + r * DH + col);
  }
  T4 v;
#pragma unroll
  for (int u = 0; u < 4; ++u) v[u] = (T)(which == 0 ? s[u] * a.scale : s[u]);
  T *out = which == 0 ? (T *)a.dk + ((long)b * a.S + j) * a.ldk : (T *)a.dv + ((long)b * a.S + j) * a.ldv;
  *reinterpret_cast<T4 *>(out + (long)kh * a.dh + col) = v;
}

size_t slots_of(const WindowArgs &a, const KeyWork &w) {
  const size_t heads = (size_t)a.B * a.nk;
  return w.parts == 1 ? heads * w.first * (1 + (size_t)w.far) : heads * ((size_t)w.key_blocks * w.parts + (size_t)w.first * w.far);
}
size_t dots_bytes(const WindowArgs &a) { return ((size_t)a.B * a.nq * a.S * sizeof(float) + 15) & ~(size_t)15; }
int key_blocks_cut(const KeyWork &w) { return w.parts > 1 ? w.key_blocks : w.first; }   // of a head
long pieces_of(const KeyWork &w) { return (long)w.key_blocks * w.parts + (long)w.first * w.far; }

// The cut with the smallest estimated time, in items (64 queries of a head).  `at_once` pieces run side by side, each as long as
// its items and `start` more (its keys, the pipeline's fill, its results).  The whole walks take full rounds; what their last round
// leaves free goes to the shorter ones, and where there are more of those than free places the longest of the rest comes on top.
// A slot is written and read once more, and adding up is a launch: `slot` and `launch`.  More than kSlots slots of workspace are
// taken only where no cut does with fewer.
struct Costs { double start, slot, launch; };   // in items
template <int ROWS> KeyWork key_work(const WindowArgs &a, int at_once, const Costs &cost, int bytes) {
  constexpr size_t kSlots = 4096;
  constexpr int R = ROWS / BKV;
  const int group = a.nq / a.nk, tiles = (a.S + BKV - 1) / BKV, in_window = (ROWS + a.window - 2) / BKV + 1;   // (as walk_of has them)
  const int walk = group * (tiles < in_window ? tiles : in_window), rest = group * (tiles > in_window ? tiles - in_window : 0);
  const double heads = (double)a.B * a.nk;
  KeyWork best{}, w;
  w.key_blocks = (a.S + ROWS - 1) / ROWS;
  w.first = a.sinks > 0 && rest > 0 ? (a.sinks + ROWS - 1) / ROWS : 0;
  w.full = tiles >= in_window ? (tiles - in_window) / R + 1 : 0;
  if (w.full > w.key_blocks) w.full = w.key_blocks;
  const double n_short = w.key_blocks - w.full;   // (tiles left from their own on: an arithmetic series)
  const double whole_items = heads * ((double)w.full * walk + (double)w.first * rest);
  const double short_items = heads * group * n_short * (tiles - R * 0.5 * (w.full + w.key_blocks - 1));
  double best_time = -1;
  auto consider = [&](int length) {   // of a piece, in items, at most
    w.parts = (walk + length - 1) / length;
    w.far = w.first > 0 ? (rest + length - 1) / length : 0;
    const size_t slots = slots_of(a, w), best_slots = best_time < 0 ? 0 : slots_of(a, best);
    if (best_time >= 0 && slots > kSlots && slots >= best_slots) return;
    const double near = (walk + w.parts - 1) / w.parts + cost.start, far = w.far > 0 ? (rest + w.far - 1) / w.far + cost.start : 0;
    const double longest = near > far ? near : far;
    const double whole = heads * ((double)w.full * w.parts + (double)w.first * w.far), shorts = heads * n_short * w.parts;
    const double rounds = (double)(long)(whole / at_once), left = whole - rounds * at_once;
    const double mean = whole > 0 ? whole_items / whole + cost.start : 0;
    double time = (left > 0 ? rounds + 1 : rounds) * mean;
    const double places = left > 0 ? at_once - left : 0;
    if (shorts > places) time += near * (1 - places / shorts);
    if (whole > 0) time += 0.5 * (longest - mean);
    const double even = (whole_items + short_items + cost.start * (whole + shorts)) / at_once + 0.1 * near;
    if (time < even) time = even;
    if (time < longest) time = longest;
    time += (double)slots * cost.slot + (slots > 0 ? cost.launch : 0);
    if (best_time < 0 || time < best_time || best_slots > kSlots) { best = w; best_time = time; }
  };
  consider(walk);
  if (w.first > 0)   // longer pieces for the rest of the sequence than the windows have
    for (int n = 2; (long)walk * (n / 2) < rest; n *= 2) consider((long)walk * n < rest ? walk * n : rest);
  for (int parts = 2; parts <= 64 && parts <= walk; ++parts) consider((walk + parts - 1) / parts);
  // heads whose shorter walks go together on an XCD: sets of one size that fill its CUs, or its L2 (two tensors) if that is more
  const int own = a.B * a.nk / 8, rows = (best.key_blocks - best.full) * best.parts;
  if (own > 0 && rows > 0) {
    const long streamed = (long)a.S * group * a.dh * 2 * bytes;
    long want = (at_once / 8 + rows - 1) / rows;
    if ((4l << 20) / streamed > want) want = (4l << 20) / streamed;
    const long sets = want >= own ? 1 : (own + want - 1) / want;
    best.together = (int)((own + sets - 1) / sets);
  }
  return best;
}

}  // namespace
}  // namespace dp
