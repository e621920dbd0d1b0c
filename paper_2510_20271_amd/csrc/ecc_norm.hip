// Group normalisation with an activation over channels-last features x [batch][points][C], G groups of Cg = C / G channels:
//   xhat = (x - mean) rstd over the points and channels of a group,   v = xhat w_c + b_c,   y = act(v)
// and its derivatives, with dv = dy act'(v) and m = points Cg:
//   db_c = sum dv,   dw_c = sum dv xhat,   dx = rstd (w_c dv - (1/m) sum_g w dv - (xhat / m) sum_g w dv xhat).
//
// Memory bounds all of it: x in and y out, x, dy in and dx out.  A thread keeps its channels: an item is rows of `cols` vectors
// of V elements (16 bytes where the sizes allow), and a thread walks down one column, so that parameters and sums stay in its
// registers.  A row is the C channels, or the least common multiple of C and V elements where V does not divide C (30 channels
// of 2 bytes: 15 vectors a row).
//
// Two ways:
//   fused   the points of some groups of one item fit one block's registers: one launch reads, sums, writes.
//   swept   sums of blocks over runs of rows (partials in the workspace), a joining kernel, and a second sweep that writes,
//           in the opposite order.  (Sweeping items in chunks that the Infinity Cache holds, so that the second sweep reads
//           little from memory, costs more in short launches than it spares: step on 8 x 512^2 x 128 in bfloat16 1407 us in
//           chunks of 128 MiB, 1077 in chunks of 256, 907 whole.)
//
// Squares are summed about a value of the data.  A thread takes its column's first value K and sums x - K and (x - K)^2 in
// float32 over at most 128 rows: what cancels in q - s^2 / n is at most n times the squares about the mean, because K is one
// of the n values, so the result is good to n E however far K lies from the rest (E: half a step of float32).  Means are
// joined in float64, squares about them by the squared differences of the means.
#include "ecc_norm.h"

#include <algorithm>
#include <numeric>

namespace ecc {

constexpr int kNormThreads = 512;      // of a sweep's block, at most
constexpr int kNormFused = 1024;       // of a fused block, at most
constexpr int kNormWide = 512;         // columns of a block, at most
constexpr int kNormRows = 128;         // rows a thread sums, at most
constexpr int kNormJoin = 256;         // of a block that joins a group's partials
constexpr int kJoinThreads = 1024;     // of one that joins its sums of the backward pass
// Partials of an item that every block of the second sweep joins by itself (48 KB from the cache, 2 to 3 us) instead of a launch
// in between (4.5 us, and as much on the host)
constexpr int64_t kNormHere = 2048;
constexpr size_t kNormShared = 64 << 10;  // shared memory of a block, at most

template <int BYTES> struct RawOf;
template <> struct RawOf<16> { using type = uint4; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<4> { using type = unsigned; };
template <> struct RawOf<2> { using type = unsigned short; };

template <typename T, int V>
struct Pack {
  using Raw = typename RawOf<sizeof(T) * V>::type;
  Raw raw;
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const Raw*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Raw*>(p) = raw; }
  __device__ __forceinline__ float get(int i) const {
    T e[V];
    __builtin_memcpy(e, &raw, sizeof(raw));
    return widen(e[i]);
  }
  __device__ __forceinline__ void set(const float (&f)[V]) {
    T e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = narrow<T>(f[i]);
    __builtin_memcpy(&raw, e, sizeof(raw));
  }
};

// How the points of an item, or of a slice of its channels, are shared out.
struct NormGeo {
  int cols;        // vectors of a row
  int wide;        // columns of a block; blocks' column ranges: `passes`
  int passes;
  int lanes;       // rows that a block takes at a time
  int64_t rows;    // rows of an item
  int64_t per;     // rows of a block
  int parts;       // runs of rows
  int channels;    // of a slice (fused), C otherwise
  int64_t stride;  // elements from a row to the next
  int64_t vectors; // of a slice of one item
  bool across;     // groups reach over several column ranges
};

// what a block knows of its group's values
struct Moments { double n, mean, m2; };

// this thread's place
struct NormLane {
  int rl, cl, col;
  bool on;
  __device__ __forceinline__ NormLane(const NormGeo& g, int pass) {
    const int t = threadIdx.x;
    rl = t / g.wide;
    cl = t - rl * g.wide;
    col = pass * g.wide + cl;
    on = rl < g.lanes && col < g.cols;
  }
};

// the largest power of two that is at most n (n >= 1), and at most `most` (a power of two)
__device__ __forceinline__ int power_below(int n, int most) {
  const int p = 1 << (31 - __clz(n));
  return p < most ? p : most;
}

// Count, mean and squares of a group, joined by `team` lanes of a wave (a power of two).  Entries are [lanes][width], 1 << shift
// to a thread, each standing for `unit` values a row; those of the group are first .. first + len - 1 of every lane, and again
// `repeats` times at every `again` (rows that hold the channels several times).
__device__ __forceinline__ Moments join_entries(const double* mean, const float* m2, const int* cnt, int wide, int lanes,
                                                int width, int first, int len, int again, int repeats, int shift, int unit,
                                                int team) {
  const int lane = threadIdx.x & (team - 1), kt = power_below(len, team), rt = team / kt, l0 = lane / kt, k0 = lane & (kt - 1);
  double n = 0.0, s = 0.0;
  for (int rl = l0; rl < lanes; rl += rt)
    for (int rep = 0, at0 = first; rep < repeats; ++rep, at0 += again)
      for (int k = k0; k < len; k += kt) {
        const double c = (double)(cnt[rl * wide + ((at0 + k) >> shift)] * unit);
        n += c;
        if (c > 0.0) s += c * mean[rl * width + at0 + k];
      }
  for (int o = team / 2; o > 0; o >>= 1) {
    n += __shfl_xor(n, o);
    s += __shfl_xor(s, o);
  }
  const double mu = n > 0.0 ? s / n : 0.0;
  double q = 0.0;
  for (int rl = l0; rl < lanes; rl += rt)
    for (int rep = 0, at0 = first; rep < repeats; ++rep, at0 += again)
      for (int k = k0; k < len; k += kt) {
        const double c = (double)(cnt[rl * wide + ((at0 + k) >> shift)] * unit);
        if (c > 0.0) {
          const double d = mean[rl * width + at0 + k] - mu;
          q += (double)m2[rl * width + at0 + k] + c * d * d;
        }
      }
  for (int o = team / 2; o > 0; o >>= 1) q += __shfl_xor(q, o);
  return {n, mu, q};
}

// Sums of one thread's columns about their first values.
template <int V>
struct Column {
  float k[V], s[V], q[V];
  int n = 0;
  template <typename T>
  __device__ __forceinline__ void first(const Pack<T, V>& p) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      k[i] = p.get(i);
      s[i] = k[i] - k[i];  // 0; NaN for a NaN or Inf
      q[i] = 0.0f;
    }
    n = 1;
  }
  template <typename T>
  __device__ __forceinline__ void add(const Pack<T, V>& p) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = p.get(i) - k[i];
      s[i] += d;
      q[i] = fmaf(d, d, q[i]);
    }
    ++n;
  }
  __device__ __forceinline__ double mean(int i, double by) const { return (double)k[i] + (double)s[i] * by; }  // by: 1 / n
  __device__ __forceinline__ float m2(int i, float by) const {
    const float v = q[i] - s[i] * s[i] * by;
    return v < 0.0f ? 0.0f : v;  // (a NaN stays one)
  }
};

// values side by side in a vector that are sure to be of one group
__host__ __device__ __forceinline__ int run_of(int Cg, int V) {
  int run = 1;
  while (run < V && Cg % (2 * run) == 0) run *= 2;
  return run;
}

// The block's moments: `done(group, Moments)` is called by one thread for each group of the block's channels c0 .. cend - 1 (a
// slice, or a column range).  shared: entries [threads][V / run].
template <int V, typename F>
__device__ __forceinline__ void block_moments(const Column<V>& col, const NormGeo& geo, const NormLane& l, int Cg, int c0, int cend,
                                              double* e_mean, float* e_m2, int* e_cnt, const F& done) {
  const int t = threadIdx.x;
  const int unit = run_of(Cg, V), per = V / unit;  // values of one group side by side: one entry for each such run
  if (t < geo.wide * geo.lanes) e_cnt[t] = l.on ? col.n : 0;
  if (l.on && col.n > 0) {
    double mu[V];
    float m2[V];
    const double by = 1.0 / (double)col.n;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      mu[i] = col.mean(i, by);
      m2[i] = col.m2(i, (float)by);
    }
#pragma unroll
    for (int step = 1; step < V; step *= 2) {  // runs of `step` values joined in pairs
      if (step < unit) {
#pragma unroll
        for (int i = 0; i < V; i += 2 * step) {
          const float d = (float)(mu[i + step] - mu[i]);
          m2[i] += m2[i + step] + 0.5f * (float)(col.n * step) * d * d;
          mu[i] = 0.5 * (mu[i] + mu[i + step]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (i % unit == 0) {
        e_mean[t * per + i / unit] = mu[i];
        e_m2[t * per + i / unit] = m2[i];
      }
    }
  }
  __syncthreads();
  // entries of a lane: its columns in order, `per` each; channel c0 is entry 0.  Groups of few entries share a wave.
  const int width = geo.wide * per, again = geo.channels / unit, repeats = geo.passes > 1 ? 1 : width / again;
  const int g0 = c0 / Cg, g1 = (cend - 1) / Cg;
  const int most = geo.lanes * repeats * ((Cg + unit - 1) / unit), shift = 31 - __clz(per);
  int team = 64;
  while (team > 1 && team / 2 >= most) team /= 2;
  const int teams = (int)blockDim.x / team;
  for (int gb = g0; gb <= g1; gb += teams) {  // (whole waves take part: a team without a group repeats the last one's)
    const int g = min(gb + t / team, g1);
    const int lo = max(g * Cg, c0), hi = min((g + 1) * Cg, cend);
    const Moments m = join_entries(e_mean, e_m2, e_cnt, geo.wide, geo.lanes, width, (lo - c0) / unit, (hi - lo) / unit, again,
                                   repeats, shift, unit, team);
    if ((t & (team - 1)) == 0 && gb + t / team <= g1) done(g, m);
  }
}

// ---- swept: first sweep of the forward pass ----------------------------------------------------------------------------
template <typename T, int V>
__global__ __launch_bounds__(kNormThreads) void norm_stats_kernel(NormArgs a, NormGeo geo, int64_t n0, Moments* part) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int Cg = a.C / a.G;
  const int64_t block = blockIdx.x;
  const int p = (int)(block % geo.parts), z = (int)(block / geo.parts % geo.passes);
  const int64_t n = block / geo.parts / geo.passes;
  const NormLane l(geo, z);
  const T* x = static_cast<const T*>(a.x) + (n0 + n) * a.points * a.C;
  Column<V> col;
  if (l.on) {
    const int64_t end = min(geo.rows, (int64_t)(p + 1) * geo.per);
    int64_t r = (int64_t)p * geo.per + l.rl, v = r * geo.cols + l.col;
    const int64_t step = (int64_t)geo.lanes * geo.cols, vend = min(geo.vectors, end * geo.cols);
    if (v < vend) {
      Pack<T, V> q;
      q.load(x + v * V);
      col.first(q);
      v += step;
      for (; v + 3 * step < vend; v += 4 * step) {
        Pack<T, V> w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u].load(x + (v + u * step) * V);
#pragma unroll
        for (int u = 0; u < 4; ++u) col.add(w[u]);
      }
      for (; v < vend; v += step) {
        q.load(x + v * V);
        col.add(q);
      }
    }
  }
  double* e_mean = reinterpret_cast<double*>(smem);
  const int per = V / run_of(Cg, V), entries = geo.wide * geo.lanes * per;
  float* e_m2 = reinterpret_cast<float*>(e_mean + entries);
  int* e_cnt = reinterpret_cast<int*>(e_m2 + entries);
  const int c0 = geo.passes > 1 ? z * geo.wide * V : 0, cend = geo.passes > 1 ? min(a.C, c0 + geo.wide * V) : a.C;
  const int nq = geo.across ? geo.parts * geo.passes : geo.parts, q = geo.across ? z * geo.parts + p : p;
  Moments* out = part + n * a.G * nq;
  if (geo.across) {  // groups that this column range does not reach
    for (int g = threadIdx.x; g < a.G; g += blockDim.x)
      if (g < c0 / Cg || g > (cend - 1) / Cg) out[(int64_t)g * nq + q] = {0.0, 0.0, 0.0};
  }
  block_moments(col, geo, l, Cg, c0, cend, e_mean, e_m2, e_cnt, [&](int g, const Moments& m) {
    out[(int64_t)g * nq + q] = m;
  });
}

__device__ __forceinline__ void block_add(double& u, double& v, double (*room)[2]) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    u += __shfl_xor(u, o);
    v += __shfl_xor(v, o);
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    room[threadIdx.x >> 6][0] = u;
    room[threadIdx.x >> 6][1] = v;
  }
  __syncthreads();
  u = v = 0.0;
  for (int k = 0; k < (int)(blockDim.x >> 6); ++k) {
    u += room[k][0];
    v += room[k][1];
  }
}

// a block for each item and group
__global__ __launch_bounds__(kNormJoin) void norm_join_kernel(const Moments* part, int nq, float eps, double* stats) {
  __shared__ double room[kNormJoin / 64][2];
  const int64_t g = blockIdx.x;
  const Moments* m = part + g * nq;
  double n = 0.0, s = 0.0;
  for (int i = threadIdx.x; i < nq; i += kNormJoin) {
    n += m[i].n;
    s += m[i].n * m[i].mean;
  }
  block_add(n, s, room);
  const double mu = s / n;
  double q = 0.0, zero = 0.0;
  for (int i = threadIdx.x; i < nq; i += kNormJoin) {
    const double d = m[i].mean - mu;
    q += m[i].m2 + m[i].n * d * d;
  }
  block_add(q, zero, room);
  if (threadIdx.x == 0) {
    stats[g * 2] = mu;
    stats[g * 2 + 1] = 1.0 / sqrt(q / n + (double)eps);
  }
}

// Channel values that a thread keeps: v = ((x - hi) - lo) rw + b.  The mean in two floats, so that a mean far above the spread
// costs nothing but x's own digits.
template <int V>
struct Scale {
  float hi[V], lo[V], rw[V], b[V];
  __device__ __forceinline__ void set(const NormArgs& a, int i, int c, double mean, double rstd) {
    hi[i] = (float)mean;
    lo[i] = (float)(mean - (double)hi[i]);
    rw[i] = (float)(rstd * (a.w ? (double)a.w[c] : 1.0));
    b[i] = a.b ? a.b[c] : 0.0f;
  }
  __device__ __forceinline__ float dev(int i, float x) const { return (x - hi[i]) - lo[i]; }
  __device__ __forceinline__ float at(int i, float dev) const { return fmaf(dev, rw[i], b[i]); }
};

// Calls f(vector index) for this thread's vectors of the block's run of rows, U at a time.
template <int U, typename F, typename G>
__device__ __forceinline__ void over_rows(const NormGeo& geo, const NormLane& l, int p, const F& many, const G& one) {
  const int64_t end = min(geo.rows, (int64_t)(p + 1) * geo.per);
  const int64_t step = (int64_t)geo.lanes * geo.cols, vend = min(geo.vectors, end * geo.cols);
  int64_t v = ((int64_t)p * geo.per + l.rl) * geo.cols + l.col;
  for (; v + (U - 1) * step < vend; v += U * step) many(v, step);
  for (; v < vend; v += step) one(v);
}

// ---- swept: second sweep of the forward pass ---------------------------------------------------------------------------
// part: null where norm_join_kernel has left the statistics in `stats`; otherwise every block joins its item's partials itself
template <typename T, int V>
__global__ __launch_bounds__(kNormThreads) void norm_apply_kernel(NormArgs a, NormGeo geo, int64_t n0, const Moments* part,
                                                                  const double* stats) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int64_t block = gridDim.x - 1 - blockIdx.x;  // (what the first sweep read last is still in the caches)
  const int p = (int)(block % geo.parts), z = (int)(block / geo.parts % geo.passes);
  const int64_t n = n0 + block / geo.parts / geo.passes;
  const NormLane l(geo, z);
  const double* own = stats + n * a.G * 2;
  if (part) {
    const int nq = geo.across ? geo.parts * geo.passes : geo.parts, t = threadIdx.x;
    double* gm = reinterpret_cast<double*>(smem);
    const Moments* m = part + (n - n0) * a.G * nq;
    int team = 64;
    while (team > 1 && team / 2 >= nq) team /= 2;
    const int teams = (int)blockDim.x / team, lane = t & (team - 1);
    for (int gb = 0; gb < a.G; gb += teams) {  // (whole waves take part: a team without a group repeats the last one's)
      const int g = min(gb + t / team, a.G - 1);
      double c = 0.0, s = 0.0, q = 0.0;
      for (int i = lane; i < nq; i += team) {
        c += m[g * nq + i].n;
        s += m[g * nq + i].n * m[g * nq + i].mean;
      }
      for (int o = team / 2; o > 0; o >>= 1) {
        c += __shfl_xor(c, o);
        s += __shfl_xor(s, o);
      }
      const double mu = s / c;
      for (int i = lane; i < nq; i += team) {
        const double d = m[g * nq + i].mean - mu;
        q += m[g * nq + i].m2 + m[g * nq + i].n * d * d;
      }
      for (int o = team / 2; o > 0; o >>= 1) q += __shfl_xor(q, o);
      if (lane == 0 && gb + t / team < a.G) {
        gm[g * 2] = mu;
        gm[g * 2 + 1] = 1.0 / sqrt(q / c + (double)a.eps);
        if (a.stats && p == 0 && z == 0) {
          a.stats[(n * a.G + g) * 2] = mu;
          a.stats[(n * a.G + g) * 2 + 1] = gm[g * 2 + 1];
        }
      }
    }
    __syncthreads();
    own = gm;
  }
  if (!l.on) return;
  const T* x = static_cast<const T*>(a.x) + n * a.points * a.C;
  T* y = static_cast<T*>(a.y) + n * a.points * a.C;
  Scale<V> sc;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (l.col * V + i) % a.C;
    const double* st = own + c / (a.C / a.G) * 2;
    sc.set(a, i, c, st[0], st[1]);
  }
  const auto put = [&](const Pack<T, V>& q, int64_t v) {
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = activate(sc.at(i, sc.dev(i, q.get(i))), a.act);
    Pack<T, V> o;
    o.set(f);
    o.store(y + v * V);
  };
  over_rows<4>(geo, l, p,
               [&](int64_t v, int64_t step) {
                 Pack<T, V> w[4];
#pragma unroll
                 for (int u = 0; u < 4; ++u) w[u].load(x + (v + u * step) * V);
#pragma unroll
                 for (int u = 0; u < 4; ++u) put(w[u], v + u * step);
               },
               [&](int64_t v) {
                 Pack<T, V> q;
                 q.load(x + v * V);
                 put(q, v);
               });
}

// ---- sums of the backward pass -----------------------------------------------------------------------------------------
// A thread's sums of dv and dv (x - mean) down its columns, added over the block's rows by halving; then over the repeats of a
// channel in a row.  sum[0][c], sum[1][c] for the local channels, in shared memory at `chan` (2 x channels of the block).
template <int V>
__device__ __forceinline__ void block_columns(float (&sa)[V], float (&sb)[V], const NormGeo& geo, const NormLane& l, int local,
                                              float* room) {
  const int t = threadIdx.x;
  const bool in = l.rl < geo.lanes;
  for (int h = geo.lanes; h > 1;) {
    const int half = (h + 1) / 2;
    __syncthreads();
    if (in && l.rl >= half && l.rl < h) {
      float* to = room + ((l.rl - half) * geo.wide + l.cl) * 2 * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        to[i] = sa[i];
        to[V + i] = sb[i];
      }
    }
    __syncthreads();
    if (in && l.rl + half < h) {
      const float* from = room + t * 2 * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        sa[i] += from[i];
        sb[i] += from[V + i];
      }
    }
    h = half;
  }
  __syncthreads();
  const int width = geo.wide * V;
  if (l.rl == 0) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      room[l.cl * V + i] = l.on ? sa[i] : 0.0f;
      room[width + l.cl * V + i] = l.on ? sb[i] : 0.0f;
    }
  }
  __syncthreads();
  if (width > local && geo.passes == 1) {  // rows that hold the channels several times
    for (int j = t; j < 2 * local; j += (int)blockDim.x) {
      float* q = room + (j / local) * width + j % local;
      float v = q[0];
      for (int k = local; k < width; k += local) v += q[k];
      q[0] = v;
    }
    __syncthreads();
  }
}

template <typename T, int V>
__global__ __launch_bounds__(kNormThreads) void norm_sums_kernel(NormArgs a, NormGeo geo, int64_t n0, float* part) {
  extern __shared__ __align__(16) unsigned char smem[];
  float* room = reinterpret_cast<float*>(smem);
  const int64_t block = blockIdx.x;
  const int p = (int)(block % geo.parts), z = (int)(block / geo.parts % geo.passes);
  const int64_t n = n0 + block / geo.parts / geo.passes;
  const int Cg = a.C / a.G;
  const NormLane l(geo, z);
  float sa[V], sb[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sa[i] = sb[i] = 0.0f;
  if (l.on) {
    const T* x = static_cast<const T*>(a.x) + n * a.points * a.C;
    const T* dy = static_cast<const T*>(a.dy) + n * a.points * a.C;
    Scale<V> sc;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (l.col * V + i) % a.C;
      const double* st = a.stats + (n * a.G + c / Cg) * 2;
      sc.set(a, i, c, st[0], st[1]);
    }
    const auto add = [&](const Pack<T, V>& q, const Pack<T, V>& d) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float dev = sc.dev(i, q.get(i)), dv = d.get(i) * slope(sc.at(i, dev), a.act);
        sa[i] += dv;
        sb[i] = fmaf(dv, dev, sb[i]);
      }
    };
    over_rows<4>(geo, l, p,
                 [&](int64_t v, int64_t step) {
                   Pack<T, V> w[4], d[4];
#pragma unroll
                   for (int u = 0; u < 4; ++u) {
                     w[u].load(x + (v + u * step) * V);
                     d[u].load(dy + (v + u * step) * V);
                   }
#pragma unroll
                   for (int u = 0; u < 4; ++u) add(w[u], d[u]);
                 },
                 [&](int64_t v) {
                   Pack<T, V> q, d;
                   q.load(x + v * V);
                   d.load(dy + v * V);
                   add(q, d);
                 });
  }
  const int c0 = geo.passes > 1 ? z * geo.wide * V : 0, cend = geo.passes > 1 ? min(a.C, c0 + geo.wide * V) : a.C;
  block_columns<V>(sa, sb, geo, l, cend - c0, room);
  float* out = part + (n * geo.parts + p) * 2 * a.C;
  for (int j = threadIdx.x; j < 2 * (cend - c0); j += blockDim.x) {
    const int which = j / (cend - c0), c = j - which * (cend - c0);
    float v = room[which * geo.wide * V + c];
    if (which) v = (float)((double)v * a.stats[(n * a.G + (c0 + c) / Cg) * 2 + 1]);
    out[which * a.C + c0 + c] = v;
  }
}

// dweight, dbias: columns of `rows` rows [2][C] added in float64; 16 columns a block, 64 threads on each
__device__ __forceinline__ void add_params(const NormArgs& a, const float* part, int64_t rows, int block, double* room) {
  const int cl = threadIdx.x & 15, rl = threadIdx.x >> 4, j = block * 16 + cl;
  double s = 0.0;
  if (j < 2 * a.C) {
#pragma unroll 8
    for (int64_t r = rl; r < rows; r += kJoinThreads / 16) s += (double)part[r * 2 * a.C + j];
  }
  room[threadIdx.x] = s;
  __syncthreads();
  for (int o = kJoinThreads / 32; o > 0; o >>= 1) {
    if (rl < o) room[threadIdx.x] += room[threadIdx.x + o * 16];
    __syncthreads();
  }
  if (rl == 0 && j < 2 * a.C) {
    float* to = j < a.C ? a.db : a.dw;
    if (to) to[j < a.C ? j : j - a.C] = (float)room[cl];
  }
}
__global__ __launch_bounds__(kJoinThreads) void norm_params_kernel(NormArgs a, const float* part, int64_t rows) {
  __shared__ double room[kJoinThreads];
  add_params(a, part, rows, (int)blockIdx.x, room);
}

// (1/m) sum w dv and (1/m) sum w dv xhat of every group of items n0 ..: a block each
// (blocks from `groups` on: the gradients of the parameters, where all items are at hand)
__global__ __launch_bounds__(kJoinThreads) void norm_groups_kernel(NormArgs a, const float* part, int parts, int64_t n0,
                                                                   int64_t groups, double* m12) {
  __shared__ double room[kJoinThreads / 64][2];
  __shared__ double columns[kJoinThreads];
  if (blockIdx.x >= groups) {
    add_params(a, part, a.batch * parts, (int)(blockIdx.x - groups), columns);
    return;
  }
  const int Cg = a.C / a.G, g = (int)(blockIdx.x % a.G);
  const int64_t n = n0 + blockIdx.x / a.G;
  const float* p = part + n * parts * 2 * a.C + (int64_t)g * Cg;
  double s1 = 0.0, s2 = 0.0;
  const int kt = power_below(Cg, kJoinThreads), rt = kJoinThreads / kt;
  for (int c = threadIdx.x & (kt - 1); c < Cg; c += kt) {
    const double w = a.w ? (double)a.w[g * Cg + c] : 1.0;
    double u1 = 0.0, u2 = 0.0;
#pragma unroll 4
    for (int64_t r = threadIdx.x / kt; r < parts; r += rt) {
      u1 += (double)p[r * 2 * a.C + c];
      u2 += (double)p[(r * 2 + 1) * a.C + c];
    }
    s1 += w * u1;
    s2 += w * u2;
  }
  block_add(s1, s2, room);
  if (threadIdx.x == 0) {
    const double m = (double)a.points * Cg;
    m12[(n * a.G + g) * 2] = s1 / m;
    m12[(n * a.G + g) * 2 + 1] = s2 / m;
  }
}

// What dx needs beside the scale: dx = rw dv - k1 - (x - mean) k2, with k1 = rstd m1, k2 = rstd^2 m2.
template <int V>
struct Slopes {
  float k1[V], k2[V];
  __device__ __forceinline__ void set(int i, double rstd, double m1, double m2) {
    k1[i] = (float)(rstd * m1);
    k2[i] = (float)(rstd * rstd * m2);
  }
};
template <typename T, int V>
__device__ __forceinline__ void put_dx(const Scale<V>& sc, const Slopes<V>& sl, const Pack<T, V>& q, const Pack<T, V>& d, int act,
                                       T* to) {
  float f[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float dev = sc.dev(i, q.get(i)), dv = d.get(i) * slope(sc.at(i, dev), act);
    f[i] = fmaf(-dev, sl.k2[i], fmaf(dv, sc.rw[i], -sl.k1[i]));
  }
  Pack<T, V> o;
  o.set(f);
  o.store(to);
}

// ---- swept: second sweep of the backward pass --------------------------------------------------------------------------
template <typename T, int V>
__global__ __launch_bounds__(kNormThreads) void norm_dx_kernel(NormArgs a, NormGeo geo, int64_t n0, const double* m12) {
  const int64_t block = gridDim.x - 1 - blockIdx.x;  // (what the first sweep read last is still in the caches)
  const int p = (int)(block % geo.parts), z = (int)(block / geo.parts % geo.passes);
  const int64_t n = n0 + block / geo.parts / geo.passes;
  const NormLane l(geo, z);
  if (!l.on) return;
  const T* x = static_cast<const T*>(a.x) + n * a.points * a.C;
  const T* dy = static_cast<const T*>(a.dy) + n * a.points * a.C;
  T* dx = static_cast<T*>(a.dx) + n * a.points * a.C;
  Scale<V> sc;
  Slopes<V> sl;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (l.col * V + i) % a.C;
    const int64_t g = (n * a.G + c / (a.C / a.G)) * 2;
    sc.set(a, i, c, a.stats[g], a.stats[g + 1]);
    sl.set(i, a.stats[g + 1], m12[g], m12[g + 1]);
  }
  over_rows<4>(geo, l, p,
               [&](int64_t v, int64_t step) {
                 Pack<T, V> w[4], d[4];
#pragma unroll
                 for (int u = 0; u < 4; ++u) {
                   w[u].load(x + (v + u * step) * V);
                   d[u].load(dy + (v + u * step) * V);
                 }
#pragma unroll
                 for (int u = 0; u < 4; ++u) put_dx<T, V>(sc, sl, w[u], d[u], a.act, dx + (v + u * step) * V);
               },
               [&](int64_t v) {
                 Pack<T, V> q, d;
                 q.load(x + v * V);
                 d.load(dy + v * V);
                 put_dx<T, V>(sc, sl, q, d, a.act, dx + v * V);
               });
}

// ---- fused: the points of some groups of one item in a block's registers -------------------------------------------------
template <typename T, int V, int K>
__global__ __launch_bounds__(kNormFused) void norm_fused_kernel(NormArgs a, NormGeo geo, int64_t n0) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int slices = a.C / geo.channels, Cg = a.C / a.G, gc = geo.channels / Cg;
  const int64_t n = n0 + blockIdx.x / slices;
  const int c0 = (int)(blockIdx.x % slices) * geo.channels;
  const NormLane l(geo, 0);
  const int64_t base = n * a.points * a.C + c0;
  const T* x = static_cast<const T*>(a.x) + base;
  T* y = static_cast<T*>(a.y) + base;
  Pack<T, V> keep[K];
  Column<V> col;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t r = l.rl + (int64_t)k * geo.lanes;
    if (l.on && r < geo.rows && r * geo.cols + l.col < geo.vectors) keep[k].load(x + r * geo.stride + l.col * V);
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t r = l.rl + (int64_t)k * geo.lanes;
    if (l.on && r < geo.rows && r * geo.cols + l.col < geo.vectors) {
      if (k == 0) col.first(keep[0]);
      else col.add(keep[k]);
    }
  }
  const int per = V / run_of(Cg, V), entries = geo.wide * geo.lanes * per;
  double* gm = reinterpret_cast<double*>(smem);  // [gc][2]
  double* e_mean = gm + 2 * gc;
  float* e_m2 = reinterpret_cast<float*>(e_mean + entries);
  int* e_cnt = reinterpret_cast<int*>(e_m2 + entries);
  block_moments(col, geo, l, Cg, 0, geo.channels, e_mean, e_m2, e_cnt, [&](int g, const Moments& m) {
    const double rstd = 1.0 / sqrt(m.m2 / m.n + (double)a.eps);
    gm[g * 2] = m.mean;
    gm[g * 2 + 1] = rstd;
    if (a.stats) {
      double* st = a.stats + (n * a.G + c0 / Cg + g) * 2;
      st[0] = m.mean;
      st[1] = rstd;
    }
  });
  __syncthreads();
  if (!l.on) return;
  Scale<V> sc;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (l.col * V + i) % geo.channels;
    sc.set(a, i, c0 + c, gm[c / Cg * 2], gm[c / Cg * 2 + 1]);
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t r = l.rl + (int64_t)k * geo.lanes;
    if (r < geo.rows && r * geo.cols + l.col < geo.vectors) {
      float f[V];
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = activate(sc.at(i, sc.dev(i, keep[k].get(i))), a.act);
      Pack<T, V> o;
      o.set(f);
      o.store(y + r * geo.stride + l.col * V);
    }
  }
}

// part: [batch][2][C], or null where there is one item, whose sums are the gradients
template <typename T, int V, int K>
__global__ __launch_bounds__(kNormFused) void norm_fused_bwd_kernel(NormArgs a, NormGeo geo, int64_t n0, float* part) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int slices = a.C / geo.channels, Cg = a.C / a.G, gc = geo.channels / Cg;
  const int64_t n = n0 + blockIdx.x / slices;
  const int c0 = (int)(blockIdx.x % slices) * geo.channels;
  const NormLane l(geo, 0);
  const int64_t base = n * a.points * a.C + c0;
  const T* x = static_cast<const T*>(a.x) + base;
  const T* dy = static_cast<const T*>(a.dy) + base;
  Pack<T, V> keep[K], up[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t r = l.rl + (int64_t)k * geo.lanes;
    if (l.on && r < geo.rows && r * geo.cols + l.col < geo.vectors) {
      keep[k].load(x + r * geo.stride + l.col * V);
      up[k].load(dy + r * geo.stride + l.col * V);
    }
  }
  const double* st = a.stats + (n * a.G + c0 / Cg) * 2;
  Scale<V> sc;
  float sa[V], sb[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (l.col * V + i) % geo.channels;
    sc.set(a, i, c0 + c, st[c / Cg * 2], st[c / Cg * 2 + 1]);
    sa[i] = sb[i] = 0.0f;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t r = l.rl + (int64_t)k * geo.lanes;
    if (l.on && r < geo.rows && r * geo.cols + l.col < geo.vectors) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float dev = sc.dev(i, keep[k].get(i)), dv = up[k].get(i) * slope(sc.at(i, dev), a.act);
        sa[i] += dv;
        sb[i] = fmaf(dv, dev, sb[i]);
      }
    }
  }
  double* m12 = reinterpret_cast<double*>(smem);  // [gc][2]
  float* room = reinterpret_cast<float*>(m12 + 2 * gc);
  block_columns<V>(sa, sb, geo, l, geo.channels, room);
  const int width = geo.wide * V;
  for (int j = threadIdx.x; j < 2 * geo.channels; j += blockDim.x) {
    const int which = j / geo.channels, c = j - which * geo.channels;
    float v = room[which * width + c];
    if (which) {
      v = (float)((double)v * st[c / Cg * 2 + 1]);
      room[width + c] = v;  // (its own thread's)
    }
    if (part) part[(n * 2 + which) * a.C + c0 + c] = v;
    else if (which ? a.dw != nullptr : a.db != nullptr) (which ? a.dw : a.db)[c0 + c] = v;
  }
  if (!a.dx) return;  // (block-uniform)
  __syncthreads();
  const double m = (double)a.points * Cg;
  for (int g = threadIdx.x >> 6; g < gc; g += (int)(blockDim.x >> 6)) {
    double s1 = 0.0, s2 = 0.0;
    for (int c = g * Cg + (threadIdx.x & 63); c < (g + 1) * Cg; c += 64) {
      const double w = a.w ? (double)a.w[c0 + c] : 1.0;
      s1 += w * (double)room[c];
      s2 += w * (double)room[width + c];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      s1 += __shfl_xor(s1, o);
      s2 += __shfl_xor(s2, o);
    }
    if ((threadIdx.x & 63) == 0) {
      m12[g * 2] = s1 / m;
      m12[g * 2 + 1] = s2 / m;
    }
  }
  __syncthreads();
  if (!l.on) return;
  Slopes<V> sl;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int g = (l.col * V + i) % geo.channels / Cg;
    sl.set(i, st[g * 2 + 1], m12[g * 2], m12[g * 2 + 1]);
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t r = l.rl + (int64_t)k * geo.lanes;
    if (r < geo.rows && r * geo.cols + l.col < geo.vectors)
      put_dx<T, V>(sc, sl, keep[k], up[k], a.act, static_cast<T*>(a.dx) + base + r * geo.stride + l.col * V);
  }
}

// ---- plans ---------------------------------------------------------------------------------------------------------------
constexpr int64_t kNormFew = 256;      // blocks of a sweep: one a compute unit
constexpr int64_t kNormBlocks = 1024;  // of a sweep, about: what the card holds at a time (2048: 924 us for 907, above)

// elements a vector may have: 16 bytes' worth, or fewer where an item's size or an address does not allow it
static int norm_vector(const NormArgs& a, int size) {
  uintptr_t all = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.dy) | reinterpret_cast<uintptr_t>(a.y) |
                  reinterpret_cast<uintptr_t>(a.dx);
  int V = 16 / size;
  while (V > 1 && (a.points * a.C % V || all % ((uintptr_t)V * size))) V /= 2;
  return V;
}

// Rows of a block.  What a block does beside its rows -- scales, the joining of its sums -- is as much as some ten rows, so
// threads take 16 of them; fewer (four at the least) where 16 would leave compute units without a block.  (2 x 83193 x 44 in
// float32 with four rows a thread: sums 28.7 us, second sweep 20.0; with sixteen 14.0 and 15.2.)
static void share_rows(NormGeo& g, int64_t items) {
  g.lanes = (int)std::max<int64_t>(1, std::min<int64_t>(kNormThreads / g.wide, g.rows));
  const auto parts_of = [&](int64_t each) { return std::max<int64_t>(1, (g.rows + g.lanes * each - 1) / (g.lanes * each)); };
  const int64_t over = std::max<int64_t>(1, items * g.passes);
  int64_t parts = std::max(parts_of(16), std::min(parts_of(4), kNormFew / over));
  parts = std::max(parts_of(kNormRows), std::min(parts, std::max<int64_t>(1, kNormBlocks / over)));
  g.per = (g.rows + parts - 1) / parts;
  g.per = (g.per + g.lanes - 1) / g.lanes * g.lanes;
  g.parts = (int)((g.rows + g.per - 1) / g.per);
}

// Columns: rows of lcm(C, V) elements where a block can hold them; else V divides C, and blocks take ranges of columns that
// hold whole groups, or (groups wider than a block) any.
static NormGeo norm_geo(const NormArgs& a, int& V) {
  NormGeo g{};
  const int Cg = a.C / a.G;
  g.channels = a.C;
  int64_t row = std::lcm<int64_t>(a.C, V);
  if (row / V <= kNormWide) {
    g.cols = g.wide = (int)(row / V);
    g.passes = 1;
  } else {
    while (a.C % V) V /= 2;
    row = a.C;
    g.cols = a.C / V;
    const int64_t unit = std::lcm<int64_t>(Cg, V) / V;  // columns after which a group ends with a column
    if (g.cols <= kNormWide) g.wide = g.cols;
    else if (unit <= kNormWide) g.wide = (int)(kNormWide / unit * unit);
    else {
      g.wide = kNormWide;
      g.across = true;
    }
    g.passes = (g.cols + g.wide - 1) / g.wide;
  }
  g.stride = row;
  g.vectors = a.points * a.C / V;
  g.rows = (g.vectors + g.cols - 1) / g.cols;
  share_rows(g, a.batch);
  return g;
}

// Slices for the fused kernels: as many groups as fit, fewer where that gives the card more blocks without cutting a row into
// runs of less than 64 bytes.  K: vectors a thread keeps (0: no slice fits).
static size_t moments_room(int threads, int Cg, int V) { return (size_t)threads * (V / run_of(Cg, V) * 12 + 4); }
static size_t columns_room(const NormGeo& g, int V) {
  return (size_t)std::max(g.wide * ((g.lanes + 1) / 2), g.wide) * 2 * V * sizeof(float);
}
static int norm_fused_plan(const NormArgs& a, int V, int size, int most, NormGeo& best) {
  const int Cg = a.C / a.G;
  if (a.points * Cg > (int64_t)kNormFused * most * V) return 0;
  int found = 0;
  for (int k = 1; k <= a.G; ++k) {
    if (a.G % k) continue;
    const int gc = a.G / k;
    if (gc < a.G && (a.C % V || (int64_t)gc * Cg % V)) continue;
    NormGeo g{};
    g.channels = gc * Cg;
    if (found && g.channels * size < 64) break;
    const int64_t row = gc == a.G ? std::lcm<int64_t>(a.C, V) : g.channels;
    if (row / V > kNormWide) continue;
    g.cols = g.wide = (int)(row / V);
    g.passes = 1;
    g.stride = gc == a.G ? row : a.C;
    g.vectors = a.points * g.channels / V;
    g.rows = (g.vectors + g.cols - 1) / g.cols;
    const int64_t widest = kNormFused / g.wide;
    if (g.rows > widest * most) continue;
    int64_t lanes = std::min<int64_t>(g.rows, std::max(1, 256 / g.wide));
    while ((g.rows + lanes - 1) / lanes > most) lanes = std::min(g.rows, std::min(lanes * 2, widest));
    g.lanes = (int)lanes;
    if ((size_t)gc * 16 + std::max(moments_room(g.wide * g.lanes, Cg, V), columns_room(g, V)) > kNormShared) continue;
    g.per = g.rows;
    g.parts = 1;
    const int K = (int)((g.rows + lanes - 1) / lanes);
    best = g;
    found = K <= 1 ? 1 : K <= 2 ? 2 : K <= 4 ? 4 : 8;
    if (a.batch * k >= 512) break;
  }
  return found;
}

static size_t align256(size_t n) { return (n + 255) / 256 * 256; }
static unsigned waves(int threads) { return (unsigned)((threads + 63) / 64 * 64); }
// Room for either way with any vector: partial moments or sums, then two doubles a group of every item.
static size_t norm_partials(const NormArgs& a) {
  size_t most = 256;
  for (int V = 1; V <= 8; V *= 2) {
    if (a.points * a.C % V) continue;
    int v = V;
    const NormGeo g = norm_geo(a, v);
    const size_t nq = (size_t)g.parts * (g.across ? g.passes : 1);
    most = std::max(most, std::max((size_t)a.batch * a.G * nq * sizeof(Moments), (size_t)a.batch * g.parts * 2 * a.C * sizeof(float)));
  }
  return align256(most);
}
size_t norm_workspace_bytes(int64_t batch, int64_t points, int C, int G) {
  NormArgs a{};
  a.batch = batch; a.points = points; a.C = C; a.G = G;
  return norm_partials(a) + align256((size_t)batch * G * 2 * sizeof(double));
}

// items of a launch: no more threads than a grid may have (below 2^32, the parameters' blocks with them), `item` threads an item in
// the largest of the launches
static int64_t norm_launch(int64_t batch, int64_t item) {
  return std::max<int64_t>(1, std::min(batch, ((int64_t)1 << 31) / item));
}
// threads of an item in the sweeps, or where its groups are joined by blocks of `join` threads
static int64_t norm_threads(const NormGeo& g, unsigned threads, int groups, int join) {
  return std::max<int64_t>((int64_t)g.parts * g.passes * threads, (int64_t)groups * join);
}

template <typename T, int V>
static hipError_t norm_fwd_v(const NormArgs& a, hipStream_t st) {
  const int Cg = a.C / a.G;
  NormGeo f;
  if (const int K = norm_fused_plan(a, V, sizeof(T), 8, f)) {
    const unsigned threads = waves(f.wide * f.lanes);
    const size_t lds = (size_t)(f.channels / Cg) * 16 + moments_room(f.wide * f.lanes, Cg, V);
    const int slices = a.C / f.channels;
    const int64_t each = norm_launch(a.batch, (int64_t)slices * threads);
    for (int64_t n0 = 0; n0 < a.batch; n0 += each) {
      const dim3 grid((unsigned)(std::min(each, a.batch - n0) * slices));
#define ECC_GO(KK) hipLaunchKernelGGL((norm_fused_kernel<T, V, KK>), grid, dim3(threads), lds, st, a, f, n0)
      if (K == 1) ECC_GO(1);
      else if (K == 2) ECC_GO(2);
      else if (K == 4) ECC_GO(4);
      else ECC_GO(8);
#undef ECC_GO
    }
    return hipGetLastError();
  }
  int v = V;
  const NormGeo g = norm_geo(a, v);
  const unsigned threads = waves(g.wide * g.lanes);
  const int nq = g.parts * (g.across ? g.passes : 1);
  Moments* part = static_cast<Moments*>(a.ws);
  double* stats = a.stats ? a.stats : reinterpret_cast<double*>(static_cast<char*>(a.ws) + norm_partials(a));
  const bool here = (int64_t)nq * a.G <= kNormHere;
  const int64_t each = norm_launch(a.batch, norm_threads(g, threads, a.G, kNormJoin));
  for (int64_t n0 = 0; n0 < a.batch; n0 += each) {
    const int64_t items = std::min(each, a.batch - n0);
    const dim3 grid((unsigned)(items * g.parts * g.passes));
    hipLaunchKernelGGL((norm_stats_kernel<T, V>), grid, dim3(threads), moments_room(g.wide * g.lanes, Cg, V), st, a, g, n0, part);
    if (!here)
      hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(items * a.G)), dim3(kNormJoin), 0, st, part, nq, a.eps, stats + n0 * a.G * 2);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;  // (nothing is made of statistics that are not there)
    hipLaunchKernelGGL((norm_apply_kernel<T, V>), grid, dim3(threads), here ? (size_t)a.G * 16 : 0, st, a, g, n0,
                       here ? part : nullptr, stats);
  }
  return hipGetLastError();
}

template <typename T, int V>
static hipError_t norm_bwd_v(const NormArgs& a, hipStream_t st) {
  const int Cg = a.C / a.G;
  const unsigned params = (unsigned)((2 * a.C + 15) / 16);
  float* part = static_cast<float*>(a.ws);
  NormGeo f;
  if (const int K = norm_fused_plan(a, V, sizeof(T), 4, f)) {
    const unsigned threads = waves(f.wide * f.lanes);
    const size_t lds = (size_t)(f.channels / Cg) * 16 + columns_room(f, V);
    const int slices = a.C / f.channels;
    const int64_t each = norm_launch(a.batch, (int64_t)slices * threads);
    float* rows = a.batch > 1 && (a.dw || a.db) ? part : nullptr;
    NormArgs b = a;
    if (a.batch > 1) b.dw = b.db = nullptr;  // (theirs are sums over the items)
    for (int64_t n0 = 0; n0 < a.batch; n0 += each) {
      const dim3 grid((unsigned)(std::min(each, a.batch - n0) * slices));
#define ECC_GO(KK) hipLaunchKernelGGL((norm_fused_bwd_kernel<T, V, KK>), grid, dim3(threads), lds, st, b, f, n0, rows)
      if (K == 1) ECC_GO(1);
      else if (K == 2) ECC_GO(2);
      else ECC_GO(4);
#undef ECC_GO
    }
    if (rows) hipLaunchKernelGGL(norm_params_kernel, dim3(params), dim3(kJoinThreads), 0, st, a, part, a.batch);
    return hipGetLastError();
  }
  int v = V;
  const NormGeo g = norm_geo(a, v);
  const unsigned threads = waves(g.wide * g.lanes);
  double* m12 = reinterpret_cast<double*>(static_cast<char*>(a.ws) + norm_partials(a));
  const int64_t each = norm_launch(a.batch, norm_threads(g, threads, a.G, kJoinThreads));
  for (int64_t n0 = 0; n0 < a.batch; n0 += each) {
    const int64_t items = std::min(each, a.batch - n0);
    const dim3 grid((unsigned)(items * g.parts * g.passes));
    hipLaunchKernelGGL((norm_sums_kernel<T, V>), grid, dim3(threads), columns_room(g, V), st, a, g, n0, part);
    if (!a.dx) continue;
    const bool all = items == a.batch && (a.dw || a.db);
    hipLaunchKernelGGL(norm_groups_kernel, dim3((unsigned)(items * a.G) + (all ? params : 0u)), dim3(kJoinThreads), 0, st, a, part,
                       g.parts, n0, items * a.G, m12);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((norm_dx_kernel<T, V>), grid, dim3(threads), 0, st, a, g, n0, m12);
  }
  if ((a.dw || a.db) && (!a.dx || each < a.batch))
    hipLaunchKernelGGL(norm_params_kernel, dim3(params), dim3(kJoinThreads), 0, st, a, part, a.batch * g.parts);
  return hipGetLastError();
}

// the vector's width: what sizes and addresses allow, and what norm_geo makes of it
template <typename T, bool BWD>
static hipError_t norm_go(const NormArgs& a, hipStream_t st) {
  int V = norm_vector(a, sizeof(T));
  norm_geo(a, V);
#define ECC_GO(VV) return BWD ? norm_bwd_v<T, VV>(a, st) : norm_fwd_v<T, VV>(a, st)
  if (V == 1) ECC_GO(1);
  if (V == 2) ECC_GO(2);
  if (V == 4 || sizeof(T) == 4) ECC_GO(4);
  ECC_GO((16 / (int)sizeof(T)));
#undef ECC_GO
}

hipError_t launch_norm_fwd(const NormArgs& a, int dtype, hipStream_t st) {
  return dtype == kF32 ? norm_go<float, false>(a, st) : dtype == kF16 ? norm_go<half_t, false>(a, st) : norm_go<bf16_t, false>(a, st);
}
hipError_t launch_norm_bwd(const NormArgs& a, int dtype, hipStream_t st) {
  return dtype == kF32 ? norm_go<float, true>(a, st) : dtype == kF16 ? norm_go<half_t, true>(a, st) : norm_go<bf16_t, true>(a, st);
}

}  // namespace ecc
