// Row kernels around the attention (part of rowwise.hip, whose vectors and angles they use):
// the norm of every query and key head with the rotation in the same pass, forward and
// backward, and dropout in front of the residual sum.

namespace {

// ------------------------------------------------------------------ norm and rotation of heads
//   n = x rstd g, rstd = (mean(x^2) + eps)^(-1/2) over a head;  y = A R(pos) n
//   dn = A R(pos)^T dy;  dg = sum over rows and heads of dn x rstd;
//   dx = rstd (dn g - x rstd^2 mean(dn g x))
// A unit is V pairs of a head (two vectors of V elements: the pairs' halves, or neighbours
// where pairs are interleaved or behind the rotated part).  A head is units of one row of
// `group` lanes, K per lane, so that a lane meets the same elements of every head: its
// gains, its pairs' cosines and sines and its part of dg stay in registers, and the sums
// over a head are a few exchanges within the group.  V elements are 16 bytes, in bf16 8, in
// fp32 4 (16 heads of 128 on 4099 rows, half of each rotated, forward and backward: 80 us; with
// units of 8 pairs, whose loads leave gaps between the lanes, 97); any other alignment takes
// single pairs (16/16 heads in bf16 on 8192 rows, forward and backward: heads of 96 67 us, of
// 100 107).
template <typename T, int V, int K, bool INTER>
struct HeadLane {
  int a[K], b[K], pair[K];     // the unit's two vectors; its first pair, -1: not rotated
  bool live[K];
  __device__ __forceinline__ HeadLane(int d, int rot, int u0, int group) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int units = d / (2 * V), turned = rot / (2 * V), u = min(u0 + k * group, units - 1);
      live[k] = u0 + k * group < units;
      const bool turn = u < turned;
      pair[k] = turn ? V * u : -1;
      a[k] = turn ? (INTER ? 2 * V * u : V * u) : rot + 2 * V * (u - turned);
      b[k] = a[k] + (turn && !INTER ? rot / 2 : V);
    }
  }
  // The unit k of a head as floats, 0 where the lane has none.
  __device__ __forceinline__ void get(int k, const RopeVec<T, V>& x, const RopeVec<T, V>& y, float (&f)[2 * V]) const {
    float lo[V], hi[V];
    x.get(lo);
    y.get(hi);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      f[i] = live[k] ? lo[i] : 0.f;
      f[V + i] = live[k] ? hi[i] : 0.f;
    }
  }
  // Pair i of a unit is (f[first(i)], f[second(i)]).
  static __device__ __forceinline__ constexpr int first(int i) { return INTER ? 2 * i : i; }
  static __device__ __forceinline__ constexpr int second(int i) { return INTER ? 2 * i + 1 : V + i; }
};

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// The sum over the aligned group of `group` lanes (a power of two), in every lane of it.
__device__ __forceinline__ float group_sum(float v, int group) {
  if (group > 1) v += dpp<0xB1>(v);       // lane ^ 1
  if (group > 2) v += dpp<0x4E>(v);       // lane ^ 2
  if (group > 4) v += dpp<0x141>(v);      // the other four of eight
  if (group > 8) v += dpp<0x140>(v);      // the other eight of sixteen
  if (group > 16) v += __shfl_xor(v, 16, 64);
  if (group > 32) v += __shfl_xor(v, 32, 64);
  return v;
}

// The row's (cos, sin) of every pair into tab, formed once per row by the wave's lanes; false:
// a row of no document.
__device__ __forceinline__ bool row_angles(const RopeRotate& r, int row, int lane, float2* tab) {
  int64_t pos = row;
  if (r.pk.n_seqs >= 0) {
    const SeqRows s = seq_of_row(r.pk, row, lane);
    if (row >= s.hi) return false;
    pos = row - s.lo;
  }
  if (r.positions && !r.n_axes) pos = r.positions[row];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (int j = lane; j < r.rot / 2; j += 64) {
    if (r.n_axes) pos = r.positions[static_cast<int64_t>(r.axis[j]) * r.tokens + row];
    tab[j] = rope_angle(r, pos, j);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return true;
}

// Bound by memory, one read and one write of the heads: 32/8 heads of 128 in bf16 on 8192 rows
// 33 us (5.1 TB/s).
template <int K>
constexpr int kNormFlight = K == 1 ? 4 : 1;      // heads in flight per lane

template <typename T, int V, int K, bool INTER>
__global__ void __launch_bounds__(256) qk_norm_fwd_kernel(QkNorm p) {
  constexpr int F = kNormFlight<K>;
  __shared__ __attribute__((aligned(16))) float2 table[4][kMaxRopePairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = static_cast<int>(blockIdx.x) * 4 + wave;
  if (row >= p.r.tokens || !row_angles(p.r, row, lane, table[wave])) return;
  const HeadLane<T, V, K, INTER> at(p.r.d_h, p.r.rot, lane % p.group, p.group);
  const int d = p.r.d_h, hps = 64 / p.group, mine = lane / p.group;
  float2 cs[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i) cs[k][i] = at.pair[k] < 0 ? make_float2(1.f, 0.f) : table[wave][at.pair[k] + i];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (t >= p.r.n_tensors) break;
    const RopeHeads& h = p.r.t[t];
    const T* x = static_cast<const T*>(h.x) + row * h.x_ld;
    T* y = static_cast<T*>(h.y) + row * h.y_ld;
    const T* gain = static_cast<const T*>(p.gain[t]);
    float g[K][2 * V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      RopeVec<T, V> lo, hi;
      lo.load(gain + at.a[k]);
      hi.load(gain + at.b[k]);
      at.get(k, lo, hi, g[k]);
    }
    for (int h0 = static_cast<int>(blockIdx.y) * F * hps; h0 < h.heads; h0 += F * hps * p.r.parts) {
      RopeVec<T, V> a[F][K], b[F][K];
#pragma unroll
      for (int f = 0; f < F; ++f) {
        const int head = min(h0 + f * hps + mine, h.heads - 1);
#pragma unroll
        for (int k = 0; k < K; ++k) {
          a[f][k].load(x + head * d + at.a[k]);
          b[f][k].load(x + head * d + at.b[k]);
        }
      }
#pragma unroll
      for (int f = 0; f < F; ++f) {
        if (h0 + f * hps >= h.heads) break;
        const int head = h0 + f * hps + mine;
        float v[K][2 * V], sum = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          at.get(k, a[f][k], b[f][k], v[k]);
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) sum = fmaf(v[k][i], v[k][i], sum);
        }
        const float rstd = rsqrtf(group_sum(sum, p.group) * p.inv_d + p.eps);
#pragma unroll
        for (int k = 0; k < K; ++k) {
          float out[2 * V];
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) v[k][i] = v[k][i] * rstd * g[k][i];
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float x0 = v[k][at.first(i)], x1 = v[k][at.second(i)];
            out[at.first(i)] = x0 * cs[k][i].x - x1 * cs[k][i].y;
            out[at.second(i)] = x1 * cs[k][i].x + x0 * cs[k][i].y;
          }
          if (head < h.heads && at.live[k]) {
            a[f][k].set(out);
            b[f][k].set(out + V);
            a[f][k].store(y + head * d + at.a[k]);
            b[f][k].store(y + head * d + at.b[k]);
          }
        }
      }
    }
  }
}

// The backward's waves walk the rows of one tensor in steps of the grid, each lane with its
// own part of dg; a workgroup's sum goes to its row of `partial`, and qk_norm_gain_kernel adds
// these up: the order is fixed.  128 registers, so that two workgroups of 8 waves run on a CU:
// what the waves have in flight hides the sums' exchanges.  32/8 heads of 128 in bf16 on 8192
// rows, with qk_norm_gain_kernel: 61 us (4.1 TB/s); both tensors in one workgroup 65 (166
// registers), two heads in flight per lane 74 (154 registers), 88 spilled into 128.
template <typename T, int V, int K, bool INTER>
__global__ void __launch_bounds__(kQkNormWaves * 64) __attribute__((amdgpu_waves_per_eu(4, 4))) qk_norm_bwd_kernel(QkNorm p) {
  constexpr int F = V < 8 && K == 1 ? 2 : 1, E = 2 * V;
  extern __shared__ __attribute__((aligned(16))) float2 shared_lds[];       // angles of every wave, then its sums
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const HeadLane<T, V, K, INTER> at(p.r.d_h, p.r.rot, lane % p.group, p.group);
  const int d = p.r.d_h, hps = 64 / p.group, mine = lane / p.group, t = blockIdx.y;
  const RopeHeads& h = p.r.t[t];
  float2* table = shared_lds + wave * (p.r.rot / 2);
  float g[K][E], dg[K][E];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    RopeVec<T, V> lo, hi;
    lo.load(static_cast<const T*>(p.gain[t]) + at.a[k]);
    hi.load(static_cast<const T*>(p.gain[t]) + at.b[k]);
    at.get(k, lo, hi, g[k]);
#pragma unroll
    for (int i = 0; i < E; ++i) dg[k][i] = 0.f;
  }
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * kQkNormWaves + wave; row < p.r.tokens;
       row += static_cast<int64_t>(gridDim.x) * kQkNormWaves) {
    if (!row_angles(p.r, static_cast<int>(row), lane, table)) continue;
    float2 cs[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) cs[k][i] = at.pair[k] < 0 ? make_float2(1.f, 0.f) : table[at.pair[k] + i];
    const T* x = static_cast<const T*>(h.x) + row * h.x_ld;
    const T* dy = static_cast<const T*>(p.dy[t]) + row * p.dy_ld[t];
    T* dx = static_cast<T*>(h.y) + row * h.y_ld;
    for (int h0 = 0; h0 < h.heads; h0 += F * hps) {
      RopeVec<T, V> xa[F][K], xb[F][K], ya[F][K], yb[F][K];
#pragma unroll
      for (int f = 0; f < F; ++f) {
        const int head = min(h0 + f * hps + mine, h.heads - 1);
#pragma unroll
        for (int k = 0; k < K; ++k) {
          xa[f][k].load(x + head * d + at.a[k]);
          xb[f][k].load(x + head * d + at.b[k]);
          ya[f][k].load(dy + head * d + at.a[k]);
          yb[f][k].load(dy + head * d + at.b[k]);
        }
      }
#pragma unroll
      for (int f = 0; f < F; ++f) {
        if (h0 + f * hps >= h.heads) break;
        const int head = h0 + f * hps + mine;
        const bool ok = head < h.heads;
        float v[K][E], dn[K][E], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          float o[E];
          at.get(k, xa[f][k], xb[f][k], v[k]);
          at.get(k, ya[f][k], yb[f][k], o);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float y0 = o[at.first(i)], y1 = o[at.second(i)];
            dn[k][at.first(i)] = y0 * cs[k][i].x + y1 * cs[k][i].y;
            dn[k][at.second(i)] = y1 * cs[k][i].x - y0 * cs[k][i].y;
          }
#pragma unroll
          for (int i = 0; i < E; ++i) s1 = fmaf(v[k][i], v[k][i], s1);
        }
        // x is scaled before anything is multiplied by it: where its squares pass fp32, and rstd is 0,
        // its products with dn would pass it too, and infinity x 0 reach dx and the gain's gradient
        const float rstd = rsqrtf(group_sum(s1, p.group) * p.inv_d + p.eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int i = 0; i < E; ++i) {
            v[k][i] *= rstd;
            s2 = fmaf(dn[k][i] * g[k][i], v[k][i], s2);
          }
        const float c = group_sum(s2, p.group) * p.inv_d * rstd;
#pragma unroll
        for (int k = 0; k < K; ++k) {
          float out[E];
#pragma unroll
          for (int i = 0; i < E; ++i) {
            out[i] = rstd * g[k][i] * dn[k][i] - c * v[k][i];
            dg[k][i] += ok ? dn[k][i] * v[k][i] : 0.f;
          }
          if (ok && at.live[k]) {
            xa[f][k].set(out);
            xb[f][k].set(out + V);
            xa[f][k].store(dx + head * d + at.a[k]);
            xb[f][k].store(dx + head * d + at.b[k]);
          }
        }
      }
    }
  }
  // over the lane groups of the wave, then over the waves
  __syncthreads();
  float* sums = reinterpret_cast<float*>(shared_lds);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      float v = dg[k][i];
      for (int o = p.group; o < 64; o *= 2) v += __shfl_xor(v, o, 64);
      if (mine == 0 && at.live[k]) sums[wave * d + (i < V ? at.a[k] + i : at.b[k] + i - V)] = v;
    }
  __syncthreads();
  for (int e = threadIdx.x; e < d; e += kQkNormWaves * 64) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kQkNormWaves; ++w) v += sums[w * d + e];
    p.partial[(static_cast<int64_t>(blockIdx.x) * 2 + t) * d + e] = v;
  }
}

// d_gain += the column sums of the workgroups' parts, every load in flight.
__global__ void __launch_bounds__(1024) qk_norm_gain_kernel(QkNorm p, int n) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = blockIdx.y, d = p.r.d_h;
  const int col = static_cast<int>(blockIdx.x) * 64 + lane;
  constexpr int R = kQkNormParts / 16;
  float v[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = wave + 16 * i;
    v[i] = r < n && col < d ? p.partial[(static_cast<int64_t>(r) * 2 + t) * d + col] : 0.f;
  }
#pragma unroll
  for (int o = R / 2; o > 0; o /= 2)
#pragma unroll
    for (int i = 0; i < o; ++i) v[i] += v[i + o];
  sums[wave][lane] = v[0];
  __syncthreads();
  if (wave || col >= d) return;
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) s += sums[w][lane];
  p.d_gain[t][col] += s;
}

// ------------------------------------------------------------------ dropout and residual
// y = residual + keep x / (1 - p).  Element e of the whole array (rows of all ranks) is kept
// where word e % 4 of Philox4x32-10 (a published counter-based generator: ten rounds of two
// 32 x 32-bit products each) at counter (e / 4, offset) under the key `seed` is at least
// p 2^32: the backward forms the mask again, none is stored.
struct Words {
  uint32_t w[4];
};
__device__ __forceinline__ Words philox(uint64_t block, uint64_t offset, uint64_t seed) {
  uint32_t x0 = static_cast<uint32_t>(block), x1 = static_cast<uint32_t>(block >> 32);
  uint32_t x2 = static_cast<uint32_t>(offset), x3 = static_cast<uint32_t>(offset >> 32);
  uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = static_cast<uint64_t>(x0) * 0xD2511F53u, b = static_cast<uint64_t>(x2) * 0xCD9E8D57u;
    x0 = static_cast<uint32_t>(b >> 32) ^ x1 ^ k0;
    x1 = static_cast<uint32_t>(b);
    x2 = static_cast<uint32_t>(a >> 32) ^ x3 ^ k1;
    x3 = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Words{{x0, x1, x2, x3}};
}

// The words of the 8 elements from place e on: two counters, or three where e is within one.
struct UnitWords {
  uint32_t w[8];
};
__device__ __forceinline__ UnitWords unit_words(uint64_t e, int shift, uint64_t offset, uint64_t seed) {   // shift = e % 4
  const Words a = philox(e / 4, offset, seed), b = philox(e / 4 + 1, offset, seed);
  UnitWords u{{a.w[0], a.w[1], a.w[2], a.w[3], b.w[0], b.w[1], b.w[2], b.w[3]}};
  if (shift) {
    const Words c = philox(e / 4 + 2, offset, seed);
    const uint32_t all[12] = {a.w[0], a.w[1], a.w[2], a.w[3], b.w[0], b.w[1], b.w[2], b.w[3], c.w[0], c.w[1], c.w[2], c.w[3]};
#pragma unroll
    for (int i = 0; i < 8; ++i) u.w[i] = shift == 1 ? all[i + 1] : shift == 2 ? all[i + 2] : all[i + 3];
  }
  return u;
}
// Units of 8 elements, whole 16-byte vectors; the last one of a single row may be cut.  Every
// row starts as far into a counter as the first one (cols % 8 == 0, or one row).
// Bound by memory: the ten rounds of a counter take about 400 cycles of a wave for 4 x 64
// elements, 1.6e12 elements a second, 9.4 TB/s in bf16.  8192 x 4096 in bf16: forward 35 us
// (5.7 TB/s), backward 26 us; a unit in the middle of counters takes three of them.
template <typename T, bool ADD>
__global__ void __launch_bounds__(256) dropout_kernel(DropoutAdd p) {
  const uint64_t seed = static_cast<uint64_t>(p.rng[0]), offset = static_cast<uint64_t>(p.rng[1]);
  const uint32_t per_row = static_cast<uint32_t>((p.cols + 7) / 8);
  const uint32_t total = static_cast<uint32_t>(p.rows) * per_row;
  const int shift = static_cast<int>(p.first % 4);
  for (uint32_t u = blockIdx.x * 256u + threadIdx.x; u < total; u += gridDim.x * 256u) {
    const uint32_t row = p.rows == 1 ? 0 : u / per_row;
    const int64_t col = static_cast<int64_t>(u - row * per_row) * 8;
    const T* xp = static_cast<const T*>(p.x) + row * p.x_ld + col;
    const T* rp = static_cast<const T*>(p.residual) + row * p.r_ld + col;
    T* yp = static_cast<T*>(p.y) + row * p.y_ld + col;
    const bool whole = col + 8 <= p.cols;
    RopeVec<T, 8> x, r;
    if (whole) {
      x.load(xp);
      if constexpr (ADD) r.load(rp);
    }
    const UnitWords words = unit_words(p.first + static_cast<uint64_t>(row) * p.cols + col, shift, offset, seed);
    if (!whole) {
      for (int i = 0; i < 7 && col + i < p.cols; ++i) {
        float y = words.w[i] >= p.threshold ? to_f32<T>(xp[i]) * p.scale : 0.f;
        if constexpr (ADD) y += to_f32<T>(rp[i]);
        yp[i] = from_f32<T>(y);
      }
      continue;
    }
    float v[8], res[8];
    x.get(v);
    if constexpr (ADD) r.get(res);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float kept = words.w[i] >= p.threshold ? v[i] * p.scale : 0.f;
      v[i] = ADD ? res[i] + kept : kept;
    }
    x.set(v);
    x.store(yp);
  }
}
// Any columns and alignment: a lane per counter, its up to four elements one at a time, each
// with a division for its row (8192 x 4095 of rows 4096 apart in bf16, forward and backward:
// 134 us, whole vectors 65).
template <typename T, bool ADD>
__global__ void __launch_bounds__(256) dropout_any_kernel(DropoutAdd p) {
  const uint64_t seed = static_cast<uint64_t>(p.rng[0]), offset = static_cast<uint64_t>(p.rng[1]);
  const int64_t n = p.rows * p.cols, skip = static_cast<int64_t>(p.first % 4);
  const int64_t blocks = (n + skip + 3) / 4;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < blocks; i += static_cast<int64_t>(gridDim.x) * 256) {
    const Words w = philox(p.first / 4 + i, offset, seed);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t e = 4 * i + j - skip;
      if (e < 0 || e >= n) continue;
      const int64_t row = e / p.cols, col = e - row * p.cols;
      const float x = to_f32<T>(static_cast<const T*>(p.x)[row * p.x_ld + col]);
      float y = w.w[j] >= p.threshold ? x * p.scale : 0.f;
      if constexpr (ADD) y += to_f32<T>(static_cast<const T*>(p.residual)[row * p.r_ld + col]);
      static_cast<T*>(p.y)[row * p.y_ld + col] = from_f32<T>(y);
    }
  }
}

template <typename T, int V, int K>
hipError_t norm_launch(const QkNorm& p, dim3 grid, hipStream_t stream) {
  if (p.backward) {
    const size_t lds = kQkNormWaves * std::max<size_t>(p.r.rot / 2 * sizeof(float2), p.r.d_h * sizeof(float));
    if (p.r.interleaved) hipLaunchKernelGGL((qk_norm_bwd_kernel<T, V, K, true>), grid, dim3(kQkNormWaves * 64), lds, stream, p);
    else hipLaunchKernelGGL((qk_norm_bwd_kernel<T, V, K, false>), grid, dim3(kQkNormWaves * 64), lds, stream, p);
    const dim3 sums((p.r.d_h + 63) / 64, p.r.n_tensors);
    hipLaunchKernelGGL(qk_norm_gain_kernel, sums, dim3(1024), 0, stream, p, static_cast<int>(grid.x));
  } else if (p.r.interleaved) {
    hipLaunchKernelGGL((qk_norm_fwd_kernel<T, V, K, true>), grid, dim3(256), 0, stream, p);
  } else {
    hipLaunchKernelGGL((qk_norm_fwd_kernel<T, V, K, false>), grid, dim3(256), 0, stream, p);
  }
  return hipGetLastError();
}

// Single pairs: as few per lane as cover a head.
template <typename T>
hipError_t norm_pairs(const QkNorm& p, int units, dim3 grid, hipStream_t stream) {
  if (units <= 64) return norm_launch<T, 1, 1>(p, grid, stream);
  return units <= 128 ? norm_launch<T, 1, 2>(p, grid, stream) : norm_launch<T, 1, 4>(p, grid, stream);
}

template <typename T>
hipError_t dropout_launch(const DropoutAdd& p, bool vec, dim3 grid, hipStream_t stream) {
  if (vec && p.residual) hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(256), 0, stream, p);
  else if (vec) hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(256), 0, stream, p);
  else if (p.residual) hipLaunchKernelGGL((dropout_any_kernel<T, true>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((dropout_any_kernel<T, false>), grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

bool aligned16(const void* x, int64_t ld, int size) { return reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld * size % 16 == 0; }

}  // namespace

int32_t qk_norm_parts(int64_t tokens) {
  return static_cast<int32_t>(std::min<int64_t>(kQkNormParts, (tokens + kQkNormWaves - 1) / kQkNormWaves));
}

hipError_t qk_norm_rope(const QkNorm& params, hipStream_t stream) {
  QkNorm p = params;
  const int size = p.r.f32 ? 4 : 2;
  // whole units of two 16-byte vectors, of which a head has at most 64
  const int unit = 32 / size;
  bool vec = p.r.rot % unit == 0 && p.r.d_h % unit == 0;
  for (int t = 0; t < p.r.n_tensors; ++t) {
    const RopeHeads& h = p.r.t[t];
    vec = vec && aligned16(h.x, h.x_ld, size) && aligned16(h.y, h.y_ld, size) && aligned16(p.gain[t], 8, size) &&
          (!p.backward || aligned16(p.dy[t], p.dy_ld[t], size));
  }
  p.inv_d = 1.f / static_cast<float>(p.r.d_h);
  const int units = p.r.d_h / (vec ? unit : 2);
  for (p.group = 1; p.group < std::min(units, 64);) p.group *= 2;
  p.r.parts = 1;
  dim3 grid(static_cast<unsigned>(qk_norm_parts(p.r.tokens)), static_cast<unsigned>(p.r.n_tensors));
  if (!p.backward) {
    const int at_once = (units <= 64 ? kNormFlight<1> : 1) * (64 / p.group);
    int most = p.r.t[0].heads;
    if (p.r.n_tensors > 1) most = std::max(most, p.r.t[1].heads);
    // waves per row: as rope_rotate
    while (static_cast<int64_t>(p.r.tokens) * p.r.parts * 2 <= 8192 && most > at_once * p.r.parts) p.r.parts *= 2;
    grid = dim3(static_cast<unsigned>((p.r.tokens + 3) / 4), static_cast<unsigned>(p.r.parts));
  }
  if (vec) return p.r.f32 ? norm_launch<float, 4, 1>(p, grid, stream) : norm_launch<uint16_t, 8, 1>(p, grid, stream);
  return p.r.f32 ? norm_pairs<float>(p, units, grid, stream) : norm_pairs<uint16_t>(p, units, grid, stream);
}

hipError_t dropout_add(const DropoutAdd& params, hipStream_t stream) {
  DropoutAdd p = params;
  const int size = p.f32 ? 4 : 2;
  if (p.rows == 1 || (p.x_ld == p.cols && p.y_ld == p.cols && (!p.residual || p.r_ld == p.cols))) {    // one row of all elements
    p.cols *= p.rows;
    p.rows = 1;
    p.x_ld = p.y_ld = p.r_ld = 0;
  }
  const bool vec = (p.rows == 1 || p.cols % 8 == 0) && aligned16(p.x, p.x_ld, size) && aligned16(p.y, p.y_ld, size) &&
                   (!p.residual || aligned16(p.residual, p.r_ld, size));
  const int64_t work = vec ? p.rows * ((p.cols + 7) / 8) : (p.rows * p.cols + 6) / 4;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((work + 255) / 256, 1 << 16)));
  return p.f32 ? dropout_launch<float>(p, vec, grid, stream) : dropout_launch<uint16_t>(p, vec, grid, stream);
}
