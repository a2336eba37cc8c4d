// Causal grouped-query attention over packed documents (device code, part of
// attention.hip: it stands on that file's LDS tiles, fragments and products).
//
//   o_i = sum_j p_ij v_j, p_i. = softmax(scale q_i . k_j), j from row i's document's
//   first row to i; the backward recomputes p from the log-sum-exp.  The WINDOW
//   kernels take the rows j of i's window and the document's first ones alone.
//
// Every tile of queries and keys lies within one document (seq_block), so the
// only masks are the causal one, as for a single sequence, and the window's, and
// nothing a document holds (an infinity or NaN in V, say, which a zero probability
// would not hide) can reach another.

template <bool WINDOW>
using AttnArgs = std::conditional_t<WINDOW, WindowAttn, PackedAttn>;

// Tiles with a probability above this keep a second bf16 part of P (dV) and dS (dQ,
// dK) in the backward's products (a wave-wide vote): there single elements decide a
// gradient.  Relative error of dQ, dK, dV on short documents 1.8, 1.7, 1.7e-3, on
// long ones 2.1, 2.1, 2.0e-3 (the output's own rounding is 1.7e-3), without second
// parts 2.8, 2.4, 2.3e-3; for 1% of the backward's time on long documents, 6% on
// short ones (16384 tokens in 160).
constexpr float kLargeP = 1.f / 8;

// Stores 32 rows of D columns (times mul) that a wave holds transposed (the lane's row
// lane % 32, register i of tile dt column 32 dt + acc_row(i)) as bf16, rows [0, n_rows)
// of them, through 64 D bytes of LDS that no other wave uses: stored straight from
// the registers, an instruction wrote 16 bytes to each of 32 rows (16384 tokens in
// documents of 128, 32/8 heads of 128: forward 97 -> 84 us, dQ 152 -> 137, dK/dV 221 ->
// 201).
template <int D>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[D / 32], float mul, uint8_t* lds, uint16_t* out, int64_t ld,
                                           int n_rows, int lane) {
  constexpr int C = D / 8;                       // 16-byte chunks of a row; chunk c of row r sits at c ^ (r % C)
  const int r = lane & 31, upper = lane >> 5;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int jj = 0; jj < 4; jj += 2) {
      // the half-waves hold columns 0-3 and 4-7 of every 8: the lower one collects chunk jj, the upper chunk jj + 1
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = 4 * jj + 2 * k;
        const u32x2 x = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_permlane32_swap(pack2(acc[dt][i] * mul, acc[dt][i + 1] * mul),
                                                    pack2(acc[dt][i + 4] * mul, acc[dt][i + 5] * mul), false, false));
        w[k] = x[0];
        w[k + 2] = x[1];
      }
      const int c = 4 * dt + jj + upper;
      *reinterpret_cast<u32x4*>(lds + r * (2 * D) + ((c ^ (r & (C - 1))) << 4)) = u32x4{w[0], w[1], w[2], w[3]};
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int j = 0; j < 32 * C / 64; ++j) {
    const int row = j * (64 / C) + lane / C, c = lane % C;
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + row * (2 * D) + ((c ^ (row & (C - 1))) << 4));
    if (row < n_rows) *reinterpret_cast<u32x4*>(out + row * ld + c * 8) = v;
  }
}

// Turns a row of D columns that a lane pair holds as in store_rows back by the angles of
// its row tab of the table (and multiplies by their amplitude), still in fp32: the gradient
// with respect to a rotated q or k becomes that of the projection's output, and is rounded once.
template <int D>
__device__ __forceinline__ void turn_back(f32x16 (&acc)[D / 32], const float2* tab, int lane) {
#pragma unroll
  for (int dt = 0; dt < D / 64; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float2 cs = tab[dt * 32 + acc_row(i, lane)];
      const float a = acc[dt][i], b = acc[dt + D / 64][i];
      acc[dt][i] = a * cs.x + b * cs.y;
      acc[dt + D / 64][i] = b * cs.x - a * cs.y;
    }
}

// The query blocks of the forward and of dQ, the i-th to start: those with most keys
// first, where one load shows all documents (32768 tokens in 6 documents, 8/1 heads of 128:
// forward 653 -> 625 us, dQ 933 -> 886; 8192 tokens in 23, 32/8 heads: forward 85 -> 81, dQ
// as it was), else the documents one after another, last blocks first.
template <bool WINDOW>
__device__ __forceinline__ SeqBlock query_block(const AttnArgs<WINDOW>& p, int i, int rows, int lane) {
  return !WINDOW && p.pk.n_seqs > 1 && p.pk.n_seqs < 64 ? ranked_block(p.pk, i, rows, lane)
                                                        : seq_block(p.pk, p.n_slots - 1 - i, rows, lane);
}

// ------------------------------------------------------------------ sliding window, first tokens visible
// WINDOW kernels: key j of a document is visible to query i >= j where i - j < window or
// j is one of the document's first `sinks` rows.  A block of queries walks the tiles of the
// first rows, then those from its first row's window on; the tiles between are never read.
// Masks cost a tile at either end of the window, and one for the first rows.
//
// Bound as the causal kernels are, with the ends of the windows on top.  32768 tokens in 2,
// window 4096, 4 first rows, 8/1 heads of 128: forward 482 us, dQ 672, dK/dV 983, 1.0, 1.1 (three
// products) and 1.0 PFLOP/s (four); 8192 in 5, window 1024, 32/8 heads: 133, 178, 250; 16384 in
// 100, window 128, 16/4 heads of 64: 35, 47, 55, most of it the way to the first products.
// Tried and dropped: first rows and window in one walk of keys (a tile fewer, but tiles
// that start anywhere: forward 2% faster with heads of 128, 8% slower with 64, dQ 2% slower);
// neighbouring blocks on one XCD where kv heads are few (traffic behind the L2s down to a
// third, times within 4% either way); passing by the tiles that a wave's rows do not see in
// blocks of one query head (dQ up to 7% faster there, 2% slower with four heads; the forward spills).
struct KeyTiles {
  int head, skip, n;     // tiles of the first rows; tiles left out behind them; tiles to walk
  // first key of tile t, from the document's first row on
  template <bool WINDOW>
  __device__ __forceinline__ int key(int t, int size) const { return (WINDOW && t >= head ? t + skip : t) * size; }
};
template <bool WINDOW>
__device__ __forceinline__ KeyTiles key_tiles(const AttnArgs<WINDOW>& p, const SeqBlock& blk, int n_keys, int size) {
  const int all = (n_keys + size - 1) / size;
  if constexpr (WINDOW) {
    const int head = min((p.sinks + size - 1) / size, all);
    const int first = max(blk.row0 - blk.lo - p.window + 1, 0) / size;      // the tile of the first row's first key
    const int skip = max(first - head, 0);
    return KeyTiles{head, skip, all - skip};
  } else {
    return KeyTiles{0, 0, all};
  }
}
// Whether the mask of a window cuts the tile of keys k0 .. k0 + size - 1 for one of the rows up to last_q.
__device__ __forceinline__ bool window_cuts(const WindowAttn& p, int lo, int k0, int size, int last_q) {
  return k0 <= last_q - p.window && k0 + size > lo + p.sinks;
}

// Rows that the queries of a block of keys cover, from its first row on: to the last row that
// sees its last key; to far_rows behind the document's first row where the block holds first
// tokens, whose later rows go in chunks of far_chunk rows (attn_packed_dkdv_kernel).
template <bool WINDOW>
__device__ __forceinline__ int block_rows(const AttnArgs<WINDOW>& p, int lo, int hi, int row0) {
  if constexpr (WINDOW) {
    if (row0 - lo < p.sinks) return min(hi, lo + p.far_rows) - row0;
    return min(hi - row0, 127 + p.window);
  } else {
    return hi - row0;
  }
}

// ------------------------------------------------------------------ forward
// One workgroup per block of query rows and hpb query heads of one kv head: 4
// waves x 32 rows, wave w on head w % hpb.  Each lane holds one query's scores
// (S^T = K Q^T), so the softmax statistics are per-lane scalars.
//
// Key tiles of 64; while tile j's softmax runs, the products of tile j + 1's scores
// are issued between its exponentials, and then tile j's P V products.  Two
// buffers each for K and V; 64 KB of LDS and at most 256 registers, two workgroups
// per CU (heads of 64: half the LDS, three; 38 -> 34 us for 16384 tokens in 160
// documents, 16/4 heads).  The output and the row sum are rescaled only on tiles
// where some row's maximum grew (a wave-wide vote).
//
// Long documents are bound by exponentials and other vector work beside the products,
// at a power-limited clock: 32768 tokens in 6, 8/1 heads of 128, 624 us, 1.1 PFLOP/s,
// matrix cores busy 55% at 1.7 GHz.  Short ones by the way to the first products, about
// 4 us of a workgroup's 6 to 20: 8192 tokens in 23, 32/8 heads of 128, 75 us.
template <int D, bool WINDOW>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2, D == 64 ? 3 : 2))) attn_packed_fwd_kernel(AttnArgs<WINDOW> p) {
  constexpr int TB = KT * D * 2;
  __shared__ __attribute__((aligned(16))) uint8_t k0[TB], v0[TB], k1[TB], v1[TB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_hg = p.heads / p.hpb, rows = 128 / p.hpb;
  const int id = static_cast<int>(blockIdx.x), h0 = id % n_hg * p.hpb;
  const SeqBlock blk = query_block<WINDOW>(p, id / n_hg, rows, lane);
  if (blk.row0 >= blk.hi) return;
  const int hq = h0 + wave % p.hpb, hk = h0 / (p.heads / p.kv_heads);
  const int wave_q0 = blk.row0 + wave / p.hpb * 32;
  const int my_q = wave_q0 + (lane & 31);
  const bool q_ok = my_q < blk.hi;
  const int n_keys = min(blk.row0 + rows, blk.hi) - blk.lo;      // keys the block's last row sees
  const int rbase = 4 * (lane >> 5);
  const LaneAddr la = lane_addr<D>(lane);

  const float c = p.scale * kLog2e;
  // a window may hide a whole tile from a row: its maximum then stays finite, and exp2(-inf - m_run) 0
  float m_run = WINDOW ? -FLT_MAX : -INFINITY, l_run = 0.f;
  f32x16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = f32x16{};

  const TileCopy<D, KT> copy_k(p.k_ld, wave, lane), copy_v(p.v_ld, wave, lane);
  const uint32_t ka0 = lds_addr(k0), ka1 = lds_addr(k1), va0 = lds_addr(v0), va1 = lds_addr(v1);
  const KeyTiles tiles = key_tiles<WINDOW>(p, blk, n_keys, KT);
  const int n_tiles = tiles.n;
  const auto copy_tile = [&](const TileCopy<D, KT>& copy, const uint16_t* base, int64_t ld, int t, uint32_t lds)
      __attribute__((always_inline)) {
    const int64_t row = blk.lo + tiles.key<WINDOW>(t, KT);
    if (t < n_tiles) copy(lds, base + row * ld + hk * D, blk.hi - static_cast<int>(row));
  };
  // the first tiles' copies, and under them the queries
  copy_tile(copy_k, p.k, p.k_ld, 0, ka0);
  copy_tile(copy_v, p.v, p.v_ld, 0, va0);
  copy_tile(copy_k, p.k, p.k_ld, 1, ka1);
  bf16x8 qf[D / 16];
  {
    const uint16_t* qb = p.q + static_cast<int64_t>(min(my_q, blk.hi - 1)) * p.q_ld + hq * D;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qb + (2 * kk + (lane >> 5)) * 8);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) settle(qf[kk]);
  }
  const auto row_max = [](const f32x16 (&s)[2]) __attribute__((always_inline)) {
    float m = __builtin_fmaxf(s[0][0], s[0][1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) m = __builtin_fmaxf(__builtin_fmaxf(m, s[0][i]), s[0][i + 1]);
#pragma unroll
    for (int i = 0; i < 16; i += 2) m = __builtin_fmaxf(__builtin_fmaxf(m, s[1][i]), s[1][i + 1]);
    return m;
  };
  // Key tile t, its scores already in s (their maximum in mx): the softmax and
  // O += V^T P, with the next tile's scores (into sn, mxn) computed under the
  // exponentials.  After the last tile sn comes from stale LDS and is never used.
  const auto step = [&](int t, const uint8_t* vt, const uint8_t* kt_next, f32x16 (&s)[2], float mx, f32x16 (&sn)[2],
                        float& mxn) __attribute__((always_inline)) {
    const int kpos0 = blk.lo + tiles.key<WINDOW>(t, KT);
    if (kpos0 + KT - 1 > wave_q0) {                   // the tile reaches past the wave's first row
      const int lim = my_q - kpos0 - rbase;           // last visible key, relative to the lane's first
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (t2 * 32 + 8 * (i >> 2) + (i & 3) > lim) s[t2][i] = -INFINITY;
      mx = row_max(s);
    }
    if constexpr (WINDOW) if (window_cuts(p, blk.lo, kpos0, KT, wave_q0 + 31)) {
      const int out = my_q - p.window - kpos0 - rbase, sink = blk.lo + p.sinks - kpos0 - rbase;   // hidden: sink <= key <= out
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = t2 * 32 + 8 * (i >> 2) + (i & 3);
          if (key >= sink && key <= out) s[t2][i] = -INFINITY;
        }
      mx = row_max(s);
    }
    mx = half_max(mx) * c;
    if (__builtin_amdgcn_ballot_w64(mx > m_run)) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = fast_exp2(m_run - m_new);   // 0 on the first tile, whose own key every row sees
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) o[dt] *= alpha;
      l_run *= alpha;
      m_run = m_new;
    }
    sn[0] = f32x16{};
    sn[1] = f32x16{};
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      sn[0] = mfma(frag_rows<D>(kt_next, 0, kk, la), qf[kk], sn[0]);
      sn[1] = mfma(frag_rows<D>(kt_next, 32, kk, la), qf[kk], sn[1]);
    }
    float rs[2] = {0.f, 0.f};
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float pr = fast_exp2(fmaf(s[t2][i], c, -m_run));
        s[t2][i] = pr;
        rs[i & 1] += pr;
      }
    l_run += rs[0] + rs[1];
    // the score products: an LDS read (kLookFwd ahead), exponentials and their sums between every two
    constexpr int NS = D / 8, NV = D / 32;
    __builtin_amdgcn_sched_group_barrier(0x100, kLookFwd, 0);
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);            // MFMA
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);            // LDS read
      __builtin_amdgcn_sched_group_barrier(0x400, 32 / NS, 0);      // exponentials
      __builtin_amdgcn_sched_group_barrier(0x002, 96 / NS, 0);      // other VALU
    }
    __builtin_amdgcn_sched_barrier(0);
    // P enters the product as bf16, off by at most 2^-8 of each probability: the size
    // of the output's own rounding
    bf16x8 x[2], f[2][NV];
    const auto group = [&](int g) __attribute__((always_inline)) {
      x[g & 1] = frag_acc(s[g >> 1], 8 * (g & 1));
#pragma unroll
      for (int dt = 0; dt < NV; ++dt) f[g & 1][dt] = frag_cols<D>(vt, dt, g, la);
    };
    group(0);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (g < 3) group(g + 1);
      else mxn = row_max(sn);
#pragma unroll
      for (int dt = 0; dt < NV; ++dt) o[dt] = mfma(f[g & 1][dt], x[g & 1], o[dt]);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 16 / NV, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // While tile j is in step, V_j and K_(j+1) are in use, V_(j+1) and K_(j+2) land in
  // the buffers that V_(j-1) and K_j held.
  wait_copies<0>();
  ring_barrier();
  f32x16 sa[2] = {f32x16{}, f32x16{}}, sb[2];
  scores2<D, kLookFwd>(k0, 0, qf, sa[0], k0, 32, qf, sa[1], la);
  float ma = row_max(sa), mb = -INFINITY;
  const auto turn = [&](int t, const uint8_t* vt, uint32_t va_next, uint32_t ka, const uint8_t* kt_next, f32x16 (&s)[2],
                        float mx, f32x16 (&sn)[2], float& mxn) __attribute__((always_inline)) {
    wait_copies<0>();
    ring_barrier();                      // every wave's copies are visible and the two old buffers are free
    copy_tile(copy_v, p.v, p.v_ld, t + 1, va_next);
    copy_tile(copy_k, p.k, p.k_ld, t + 2, ka);
    __builtin_amdgcn_sched_barrier(0);   // the copies go out now, not next to the wait for them
    step(t, vt, kt_next, s, mx, sn, mxn);
  };
  for (int t = 0; t < n_tiles; t += 2) {
    turn(t, v0, va1, ka0, k1, sa, ma, sb, mb);
    if (t + 1 >= n_tiles) break;
    turn(t + 1, v1, va0, ka1, k0, sb, mb, sa, ma);
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  ring_barrier();                        // every wave is done with the tiles: each takes a quarter of a buffer
  uint8_t* mine = (wave == 0 ? k0 : wave == 1 ? k1 : wave == 2 ? v0 : v1);
  store_rows<D>(o, 1.0f / l_tot, mine, p.o + static_cast<int64_t>(wave_q0) * p.o_ld + hq * D, p.o_ld, blk.hi - wave_q0, lane);
  if (q_ok && lane < 32)
    p.lse[static_cast<int64_t>(hq) * p.pk.tokens + my_q] = (m_run + __builtin_amdgcn_logf(l_tot)) * kLn2;
}

// ------------------------------------------------------------------ backward: order of the blocks of keys
// Windows of 128 rows from row 0 on.  Where only some blocks are cut, a cut one has 128
// rows, so it holds the first row of exactly one window: no more second slices than
// windows are listed, and the pass that adds them up finds every cut block from its window.
__host__ __device__ __forceinline__ int packed_windows(const PackedAttn& p) { return (p.pk.tokens + 127) / 128; }

// Slices of a kv head's query heads that the keys of the block from row0 on get, whose document
// goes on for n_rows rows from there (with a window: block_rows): see attn_packed_plan.
template <bool WINDOW>
__device__ __forceinline__ int packed_slices(const AttnArgs<WINDOW>& p, int row0, int n_rows) {
  bool cut = n_rows >= p.cut_rows;
  if constexpr (WINDOW) cut = cut && (row0 >> 7 & p.cut_mask) == 0;
  return cut ? p.n_split : 1;
}

// Workgroup 0 of the dQ pass lists the blocks of keys for the dK/dV pass, longest
// first, as {first row, sign bit: second slice; end of the document} behind their
// number: a counting sort by work in steps of 1/64 octave.  Workgroups start in order
// and last as long as their document has rows left; in the order of the rows, long ones
// started last, and short ones waited behind parts of the chip that held long ones
// (8192 tokens in 23 documents, 32/8 heads of 128: 157 of 256 CUs busy on average).  dK/dV
// 187 -> 152 us there, 1378 -> 1305 for 32768 tokens in 6, 8/1 heads, 90 -> 59 for 16384
// in 160, 16/4 heads of 64.  Without a window the list hides behind the other workgroups'
// dQ.  Its order within a step varies, the sums do not; steps of 1/16 scatter a document's
// neighbours, which read the same rows (1305 -> 1280 us on the long documents).
//
// With a window the entries are {first row, sign bit: second slice; first query row; row
// behind the last one; row behind the first tokens, sign bit: sums in parts}, and behind the
// blocks of a document's first tokens come the chunks of the rows far from them.  A document
// is one thread's, at about 0.4 us a block or chunk: where few documents are long and the
// window is short, the list is what dQ takes (32768 rows, 8/1 heads of 64, window 128: dQ in
// 256 documents 36 us, in one 94, with 4 first tokens, whose 254 chunks are listed too, 202).
constexpr int kOrderBins = 2048;
template <bool WINDOW>
__device__ __forceinline__ void packed_order(const AttnArgs<WINDOW>& p, int* bin) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int room = p.pk.tokens + packed_windows(p);
  if constexpr (WINDOW) room = static_cast<int>(attn_window_items(p) - 1);
  const int group = p.heads / p.kv_heads;
  for (int i = tid; i < kOrderBins; i += 256) bin[i] = 0;
  __syncthreads();
  // a document per thread: one of n blocks takes the pass n^2 tiles (with a window n times a window's), this loop n steps
  const auto each = [&](auto visit) __attribute__((always_inline)) {
    int left = p.list_steps;             // no more blocks than that, whatever starts holds
    for (int i = tid; i < p.pk.n_seqs; i += 256) {
      const int hi = seq_start(p.pk, i + 1);
      const int lo = seq_start(p.pk, i);
      const auto add = [&](int row0, int q0, int n_rows, int slices, int n) __attribute__((always_inline)) {
        const float work = static_cast<float>((n_rows + QT - 1) / QT) * (group / slices);
        visit(lo, hi, row0, q0, n_rows, static_cast<int>(__float_as_uint(work) >> 17) - (127 << 6), n);
      };
      for (int row0 = lo; row0 < hi && left > 0; row0 += 128, --left) {
        const int n_rows = block_rows<WINDOW>(p, lo, hi, row0), slices = packed_slices<WINDOW>(p, row0, n_rows);
        add(row0, row0, n_rows, slices, p.cut_rows ? slices : 1);
      }
      if constexpr (WINDOW)
        for (int q0 = lo + p.far_rows; q0 < hi;) {
          const int end = min(hi, (q0 / p.far_chunk + 1) * p.far_chunk);
          for (int row0 = lo; row0 < lo + p.sinks && left > 0; row0 += 128, --left)
            add(row0, q0, end - q0, p.cut_rows ? 1 : p.n_split, 1);
          if (left <= 0) break;
          q0 = end;
        }
    }
  };
  each([&](int, int, int, int, int, int k, int n) { atomicAdd(&bin[k], n); });
  __syncthreads();
  if (wave == 0) {                       // entries in fuller bins, for every bin
    constexpr int M = kOrderBins / 64;
    int* mine = bin + (63 - lane) * M;
    int sum = 0;
#pragma unroll
    for (int i = M - 1; i >= 0; --i) sum += mine[i];
    int upto = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int x = __shfl_up(upto, d, 64);
      if (lane >= d) upto += x;
    }
    if (lane == 63) p.items[0] = min(upto, room);
    int at = upto - sum;
#pragma unroll
    for (int i = M - 1; i >= 0; --i) {
      const int n = mine[i];
      mine[i] = at;
      at += n;
    }
  }
  __syncthreads();
  each([&](int lo, int hi, int row0, int q0, int n_rows, int k, int n) {
    const int at = atomicAdd(&bin[k], n);
    for (int j = 0; j < n && at + j < room; ++j) {
      const int first = row0 | (j ? INT32_MIN : 0);
      if constexpr (WINDOW)
        reinterpret_cast<int4*>(p.items)[1 + at + j] = make_int4(
            first, q0, q0 + n_rows, (lo + p.sinks) | (row0 - lo < p.sinks && hi - lo > p.far_rows ? INT32_MIN : 0));
      else
        reinterpret_cast<int2*>(p.items)[1 + at + j] = make_int2(first, hi);
    }
  });
}

// ------------------------------------------------------------------ backward: dQ
// The forward's blocks.  Per key tile: S^T = K Q^T and dP^T = V dO^T, then
// dS^T = P^T (dP^T - delta) feeds dQ^T += K^T dS^T from registers.
//
// delta = rowsum(dO * O) is off by rowsum(dO * r), r the rounding of O to bf16.  As
// sum_j dS_ij is 0 for the true delta and the p_ij add up to 1, the sum that comes
// out is that error: it is added to the delta that the dK/dV pass reads.  The first
// 32 rows of a document, which one tile covers, have it before dQ's product too.
// The dQ of later rows uses the uncorrected delta; where the error counts, a
// probability is large and dS enters the product in two parts (kLargeP).
//
// Bound as the forward is: 32768 tokens in 6 documents, 8/1 heads of 128, 886 us (1.1
// PFLOP/s, busy 58% at 1.75 GHz); 8192 in 23, 32/8 heads, 115 us; 16384 in 160, 16/4
// heads of 64, 41 us (48 with two workgroups per CU, here three).
template <int D, bool ROPE, bool WINDOW>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2, D == 64 ? 3 : 2))) attn_packed_dq_kernel(AttnArgs<WINDOW> p) {
  constexpr int KQ = 32;                     // keys per tile
  constexpr int TB = KQ * D * 2;
  __shared__ __attribute__((aligned(16))) uint8_t kbuf[2][TB], vbuf[2][TB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_hg = p.heads / p.hpb, rows = 128 / p.hpb;
  static_assert(sizeof(kbuf) >= kOrderBins * sizeof(int), "the bins lie in the K tiles");
  if (blockIdx.x == 0) return packed_order<WINDOW>(p, reinterpret_cast<int*>(kbuf));
  const int id = static_cast<int>(blockIdx.x) - 1, h0 = id % n_hg * p.hpb;
  const SeqBlock blk = query_block<WINDOW>(p, id / n_hg, rows, lane);
  if (blk.row0 >= blk.hi) return;
  const int hq = h0 + wave % p.hpb, hk = h0 / (p.heads / p.kv_heads);
  const int wave_q0 = blk.row0 + wave / p.hpb * 32;
  const int my_q = wave_q0 + (lane & 31);
  const bool q_ok = my_q < blk.hi;
  const int n_keys = min(blk.row0 + rows, blk.hi) - blk.lo;
  const int rbase = 4 * (lane >> 5);
  const LaneAddr la = lane_addr<D>(lane);

  const TileCopy<D, KQ> copy_k(p.k_ld, wave, lane), copy_v(p.v_ld, wave, lane);
  const KeyTiles tiles = key_tiles<WINDOW>(p, blk, n_keys, KQ);
  const int n_tiles = tiles.n;
  const auto issue = [&](int t, int b) __attribute__((always_inline)) {
    const int64_t r0 = blk.lo + tiles.key<WINDOW>(t, KQ);
    const int valid = blk.hi - static_cast<int>(r0);
    copy_k(lds_addr(kbuf[b]), p.k + r0 * p.k_ld + hk * D, valid);
    copy_v(lds_addr(vbuf[b]), p.v + r0 * p.v_ld + hk * D, valid);
  };
  issue(0, 0);
  bf16x8 qf[D / 16], dof[D / 16];      // under the first tile's copies
  float my_delta = 0.f;
  const int row = min(my_q, blk.hi - 1);
  {
    u32x4 of[D / 16];
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const int dcol = hq * D + (2 * kk + (lane >> 5)) * 8;
      qf[kk] = *reinterpret_cast<const bf16x8*>(p.q + row * p.q_ld + dcol);
      dof[kk] = *reinterpret_cast<const bf16x8*>(p.dout + row * p.do_ld + dcol);
      of[kk] = *reinterpret_cast<const u32x4*>(p.o + row * p.o_ld + dcol);
    }
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const u32x4 g = __builtin_bit_cast(u32x4, dof[kk]);
#pragma unroll
      for (int j = 0; j < 4; ++j) my_delta += lo16(g[j]) * lo16(of[kk][j]) + hi16(g[j]) * hi16(of[kk][j]);
    }
    my_delta += __shfl_xor(my_delta, 32, 64);
  }
  const int64_t sidx = static_cast<int64_t>(hq) * p.pk.tokens + row;
  const float my_lse = p.lse[sidx] * kLog2e;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    settle(qf[kk]);
    settle(dof[kk]);
  }
  settle(my_lse);
  settle(my_delta);
  const float c = p.scale * kLog2e;
  float ds_sum = 0.f;
  f32x16 dq[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dq[i] = f32x16{};

  for (int t = 0; t < n_tiles; ++t) {
    const int b = t & 1;
    wait_copies<0>();
    ring_barrier();
    if (t + 1 < n_tiles) issue(t + 1, b ^ 1);
    __builtin_amdgcn_sched_barrier(0);
    f32x16 sc = f32x16{}, dp = f32x16{};
    scores2<D, kLookDq>(kbuf[b], 0, qf, sc, vbuf[b], 0, dof, dp, la);
    const int kpos0 = blk.lo + tiles.key<WINDOW>(t, KQ);
    if (kpos0 + KQ - 1 > wave_q0) {                         // the tile reaches past the wave's first row
      const int lim = my_q - kpos0 - rbase;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + (i & 3) > lim) sc[i] = -INFINITY;
    }
    if constexpr (WINDOW) if (window_cuts(p, blk.lo, kpos0, KQ, wave_q0 + 31)) {
      const int out = my_q - p.window - kpos0 - rbase, sink = blk.lo + p.sinks - kpos0 - rbase;   // hidden: sink <= key <= out
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 8 * (i >> 2) + (i & 3);
        if (key >= sink && key <= out) sc[i] = -INFINITY;
      }
    }
    float p_max = 0.f, sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float pr = fast_exp2(fmaf(sc[i], c, -my_lse));
      p_max = __builtin_fmaxf(p_max, pr);
      sc[i] = pr;
      dp[i] -= my_delta;
      sum = fmaf(pr, dp[i], sum);
    }
    if (t == 0 && wave_q0 == blk.lo) {     // the document's first rows see no other tile: the sum is complete
      sum += __shfl_xor(sum, 32, 64);
      my_delta += sum;
#pragma unroll
      for (int i = 0; i < 16; ++i) dp[i] -= sum;
      sum = 0.f;
    }
    ds_sum += sum;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] *= dp[i];   // dS^T
    const bf16x8 sf[2] = {frag_acc(sc, 0), frag_acc(sc, 8)};
    accum_t<D, 2, kLookDq>(kbuf[b], sf, dq, la);
    if (__builtin_amdgcn_ballot_w64(p_max > kLargeP)) {
      const bf16x8 lo[2] = {frag_acc_lo(sc, 0, sf[0]), frag_acc_lo(sc, 8, sf[1])};
      accum_t<D, 2, kLookDq>(kbuf[b], lo, dq, la);
    }
  }

  ds_sum += __shfl_xor(ds_sum, 32, 64);
  if (q_ok && lane < 32) {
    p.delta[sidx] = my_delta + ds_sum;
    p.lse2[sidx] = my_lse;
  }
  if constexpr (ROPE) turn_back<D>(dq, p.rope + static_cast<int64_t>(row) * (D / 2), lane);
  ring_barrier();                        // every wave is done with the tiles: each takes a buffer
  store_rows<D>(dq, p.scale, wave < 2 ? kbuf[wave & 1] : vbuf[wave & 1], p.dq + static_cast<int64_t>(wave_q0) * p.dq_ld + hq * D,
                p.dq_ld, blk.hi - wave_q0, lane);
}

// ------------------------------------------------------------------ backward: dK, dV
// One workgroup per (block of 128 keys, kv head, slice of its query heads), 8 waves.
// The 128 keys form four groups of 32, each with two waves on the same SIMD
// (wave w runs on SIMD w % 4):
//  * role 0 holds K, computes S = Q K^T and P = exp(S - lse), hands P (fp32) to
//    its partner through LDS and accumulates dV^T += dO^T P;
//  * role 1 holds V, computes dP = dO V^T, takes P, forms dS = P (dP - delta) and
//    accumulates dK^T += Q^T dS.
// Each then needs one operand and one accumulator block, which fits 256 registers
// (two waves per SIMD), and the softmax of one wave runs under the products of
// the other.  One wave per group doing both (one wave per SIMD) took 2.6 times as long
// (32768 tokens in 6 documents, 8/1 heads of 128), and 2.2 times (8192 tokens in 23,
// 32/8 heads).
//
// Tiles of 32 queries, from the block's own first row to the document's end (with a
// window of w rows to the last row that sees a key of the block), of each head in turn,
// stream through a ring of four stages.  All four groups take every tile, also those that
// the window or the diagonal hides from a group: of (127 + w)/32 tiles, rounded up, a group's
// keys are seen from (31 + w)/32 (8 and 5 at w = 128, 36 and 33 at 1024).  Heads of 64 take 128
// registers and 65 KB: two workgroups per CU (103 -> 90 us for 16384 tokens in 160
// documents, 16/4 heads).
//
// Bound by the chain of a tile (scores, exponentials, handover, products; 1.0 to 1.3 us)
// and on long documents by the clock: 32768 tokens in 6, 8/1 heads of 128, 1287 us
// (1.0 PFLOP/s, matrix cores busy 49% at 1.79 GHz); 8192 in 23, 32/8 heads, 137 us.
template <int D, bool ROPE, bool WINDOW>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2, D == 64 ? 4 : 2))) attn_packed_dkdv_kernel(AttnArgs<WINDOW> p) {
  constexpr int TB = QT * D * 2;
  __shared__ __attribute__((aligned(16))) uint8_t qg[kDkvStages][2][TB];   // per stage: Q tile, then dO tile
  __shared__ __attribute__((aligned(16))) float st[kDkvStages][2][QT];     // lse (base 2), delta
  __shared__ __attribute__((aligned(16))) float4 xp[2][4][QT / 16][2][64]; // P handover: [buffer][group][16 queries][half][lane]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave & 3, role = wave >> 2;
  const int group = p.heads / p.kv_heads;
  // Workgroups go to the 8 XCDs in turn: the kv heads of a block are neighbours, and the
  // slices where all blocks are cut, so that an XCD keeps to the same heads, whose
  // rows it then has in its L2.
  const int id = static_cast<int>(blockIdx.x), cut = p.cut_rows ? 1 : p.n_split, at = id / (p.kv_heads * cut);
  const int n_items = p.items[0];
  int4 item;                             // see packed_order
  if constexpr (WINDOW) {
    item = reinterpret_cast<const int4*>(p.items)[1 + at];
  } else {
    const int2 x = reinterpret_cast<const int2*>(p.items)[1 + at];
    item = make_int4(x.x, x.x & INT32_MAX, x.y, 0);
  }
  if (at >= n_items) return;
  const int hk = id % (p.kv_heads * cut) / cut, split = p.cut_rows ? item.x < 0 : id % cut;
  const struct { int row0, q0, hi; } blk{item.x & INT32_MAX, WINDOW ? item.y : item.x & INT32_MAX, item.z};
  const int n_rows = blk.hi - blk.q0, n_qt = (n_rows + QT - 1) / QT;
  const bool far = WINDOW && blk.q0 != blk.row0;      // rows far from first tokens: their sums go in a part
  const int slices = far ? (p.cut_rows ? 1 : p.n_split) : packed_slices<WINDOW>(p, blk.row0, n_rows);
  const int hps = group / slices, head0 = hk * group + split * hps;
  const int grp_k0 = blk.row0 + grp * 32;
  const int my_key = grp_k0 + (lane & 31);
  const int sink_end = item.w & INT32_MAX;
  const bool key_ok = my_key < blk.hi;
  const int rbase = 4 * (lane >> 5);
  const LaneAddr la = lane_addr<D>(lane);
  // offsets into a stage's [Q | dO] pair: the first product reads Q (role 0) or dO, the second the other
  const LaneAddr la1{la.rows + role * TB, la.cols};
  const LaneAddr la2{la.rows, la.cols + (1 - role) * TB};
  // the role's member by arithmetic: a select of two members' addresses would put the kernel argument on the stack
  const uint64_t role_mask = 0ull - static_cast<uint64_t>(role);
  const auto pick = [&](uint64_t a, uint64_t b) { return a + ((b - a) & role_mask); };
  const auto addr = [](const void* x) { return reinterpret_cast<uint64_t>(x); };

  f32x16 acc[D / 32];                    // role 0: dV^T, role 1: dK^T (d rows, the lane's key)
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = f32x16{};
  const float c = p.scale * kLog2e;
  // waves 0-3 copy the Q tiles and their lse, waves 4-7 the dO tiles and delta
  const int64_t ld = pick(p.q_ld, p.do_ld);
  const TileCopy<D, QT> copy(ld, grp, lane);
  const uint32_t qg_addr = lds_addr(qg) + role * TB, st_addr = lds_addr(st) + (role * QT + grp * (QT / 4)) * 4;
  // the next tile to copy: its first row, its head's statistics from the block's first row on, its query tile, tiles left after it
  uint64_t src = pick(addr(p.q), addr(p.dout)) + (blk.q0 * ld + head0 * D) * 2;
  uint64_t row = pick(addr(p.lse2), addr(p.delta)) + (static_cast<int64_t>(head0) * p.pk.tokens + blk.q0) * 4;
  const int64_t tile_step = QT * ld * 2, head_step = D * 2 - (n_qt - 1) * tile_step;
  int copy_qt = 0, copy_left = hps * n_qt - 1;
  // Copies that tile into stage b, kCopies per wave, and moves on; past the last
  // tile it repeats it, so that the waits count exactly.
  constexpr int kCopies = TileCopy<D, QT>::NKB / 4 + 1;
  auto issue = [&](int b) __attribute__((always_inline)) {
    const int q0 = copy_qt * QT;
    if (lane < QT / 4)
      dma4(reinterpret_cast<const float*>(row), static_cast<uint32_t>(min(q0 + grp * (QT / 4) + lane, n_rows - 1)) * 4u,
           st_addr + b * (2 * QT * 4));
    copy(qg_addr + b * (2 * TB), reinterpret_cast<const uint16_t*>(src), n_rows - q0);
    const bool more = copy_left > 0, wrap = copy_qt + 1 == n_qt;
    src += more ? (wrap ? head_step : tile_step) : 0;
    row += more && wrap ? static_cast<int64_t>(p.pk.tokens) * 4 : 0;
    copy_qt = more ? (wrap ? 0 : copy_qt + 1) : copy_qt;
    copy_left -= more;
  };
  bf16x8 kv[D / 16];                     // role 0: K rows, role 1: V rows of the group's keys
  {
    const uint16_t* kv_row = reinterpret_cast<const uint16_t*>(pick(addr(p.k), addr(p.v))) +
                          static_cast<int64_t>(pick(p.k_ld, p.v_ld)) * min(my_key, blk.hi - 1) + hk * D;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) kv[kk] = *reinterpret_cast<const bf16x8*>(kv_row + (2 * kk + (lane >> 5)) * 8);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) settle(kv[kk]);
  }
  f32x16 s;                  // role 0: S -> P of a tile, role 1: its dP - delta
  bf16x8 x[2], lo[2] = {};   // role 0: P, role 1: dS (bf16), and their second parts
  bool large = false;        // a probability of the tile is above kLargeP
  const auto second_parts = [&](const f32x16& pr, const f32x16& v) __attribute__((always_inline)) {
    float m = __builtin_fmaxf(pr[0], pr[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) m = __builtin_fmaxf(__builtin_fmaxf(m, pr[i]), pr[i + 1]);
    large = __builtin_amdgcn_ballot_w64(m > kLargeP) != 0;
    if (large) {
      lo[0] = frag_acc_lo(v, 0, x[0]);
      lo[1] = frag_acc_lo(v, 8, x[1]);
    }
  };
  // role 0: P = exp(S - lse) of tile qt from its scores in s; bf16 into x, fp32 into handover hb
  auto probs = [&](int qt, const float4 (&ls4)[4], float4 (*hb)[2][64]) __attribute__((always_inline)) {
    const int q0 = blk.q0 + qt * QT;
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      const float4 ls = ls4[jj];
      const float lsv[4] = {ls.x, ls.y, ls.z, ls.w};      // in base 2, as dQ left it
#pragma unroll
      for (int u = 0; u < 4; ++u) s[4 * jj + u] = fast_exp2(fmaf(s[4 * jj + u], c, -lsv[u]));
    }
    bool cuts = q0 < grp_k0 + 31 || q0 + QT > blk.hi;      // the tile straddles the diagonal, or the document ends in it
    int last = blk.hi;
    if constexpr (WINDOW) {
      cuts = cuts || q0 + QT > grp_k0 + p.window;
      if (my_key >= sink_end) last = min(last, my_key + p.window);
    }
    if (cuts) {
      // visible query rows r (relative to the lane's first row): lo <= r <= hi
      const int lo = (key_ok ? my_key - q0 : QT) - rbase, hi = last - 1 - q0 - rbase;
      // one unsigned comparison an element: with a window a quarter of the tiles are cut (16384 tokens in
      // 100 documents, window 128, 16/4 heads of 64: 62 -> 55 us)
      const uint32_t count = static_cast<uint32_t>(max(hi - lo + 1, 0));
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = 8 * (i >> 2) + (i & 3);
        if (WINDOW ? static_cast<uint32_t>(r - lo) >= count : r < lo || r > hi) s[i] = 0.f;
      }
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int i0 = 8 * g;
      x[g] = frag_acc(s, i0);
      hb[g][0][lane] = make_float4(s[i0], s[i0 + 1], s[i0 + 2], s[i0 + 3]);
      hb[g][1][lane] = make_float4(s[i0 + 4], s[i0 + 5], s[i0 + 6], s[i0 + 7]);
    }
    second_parts(s, s);
  };
  // role 1: dS = P (dP - delta) of the tile whose dP - delta is in s, into x
  auto grads = [&](const float4 (*hb)[2][64]) __attribute__((always_inline)) {
    f32x16 pr, ds;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const float4 p0 = hb[g][0][lane], p1 = hb[g][1][lane];
      const float pv[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        pr[8 * g + j] = pv[j];
        ds[8 * g + j] = pv[j] * s[8 * g + j];
      }
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) x[g] = frag_acc(ds, 8 * g);
    second_parts(pr, ds);
  };
  auto minus = [&](const float4 (&d4)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      s[4 * jj] -= d4[jj].x;
      s[4 * jj + 1] -= d4[jj].y;
      s[4 * jj + 2] -= d4[jj].z;
      s[4 * jj + 3] -= d4[jj].w;
    }
  };
  // Both roles run one stream of products over role-selected tiles: the next
  // tile's scores (stage bn) alternating with this tile's accumulation (stage b) of x.
  auto products = [&](int b, int bn, bool accumulate) __attribute__((always_inline)) {
    s = f32x16{};
    const uint8_t* tb = qg[b][0];
    const uint8_t* tn = qg[bn][0];
    constexpr int NS = D / 16, NA = 2 * (D / 32);     // products of either kind (equal)
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      s = mfma(frag_rows<D>(tn, 0, i, la1), kv[i], s);
      if (accumulate) {
        const int g = i / (D / 32), dt = i % (D / 32);
        acc[dt] = mfma(frag_cols<D>(tb, dt, g, la2), x[g], acc[dt]);
      }
    }
    static_assert(NS == NA, "scores and accumulation alternate");
  };

  // One barrier per tile.  Interval j, after the barrier that publishes tile
  // j + 1 and the handover of P_j: role 1 forms dS_j; both roles run tile j's
  // accumulation and tile j + 1's scores; role 0 forms and hands over P_(j+1).
  // The copies of tile j + 3 go out behind the products; past the last tile its
  // scores are computed once more, unused.
  float4 stat[4];            // the lane's rows of the next tile's lse (role 0) or delta (role 1)
  const auto read_stat = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) stat[jj] = *reinterpret_cast<const float4*>(&st[b][role][8 * jj + rbase]);
  };
#pragma unroll
  for (int b = 0; b < kDkvStages - 1; ++b) issue(b);
  wait_copies<(kDkvStages - 2) * kCopies>();
  ring_barrier();
  read_stat(0);
  products(0, 0, false);
  if (role == 0) probs(0, stat, xp[0][grp]);
  else minus(stat);
  int left = hps * n_qt, qt = 0;
  const auto interval = [&](auto stage) __attribute__((always_inline)) {
    constexpr int b = decltype(stage)::value, bn = (b + 1) % kDkvStages;
    wait_copies<(kDkvStages - 3) * kCopies>();
    ring_barrier();
    if (role == 1) grads(xp[b & 1][grp]);
    __builtin_amdgcn_sched_barrier(0);
    products(b, bn, true);
    __builtin_amdgcn_sched_group_barrier(0x100, 3 * 2, 0);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (large) accum_t<D, 2, kLookDq>(qg[b][0], lo, acc, la2);
    read_stat(bn);
    issue((b + kDkvStages - 1) % kDkvStages);     // under the last products
    if (++qt == n_qt) qt = 0;
    if (role == 0) probs(qt, stat, xp[bn & 1][grp]);
    else minus(stat);
  };
  while (true) {
    interval(std::integral_constant<int, 0>{});
    if (--left == 0) break;
    interval(std::integral_constant<int, 1>{});
    if (--left == 0) break;
    interval(std::integral_constant<int, 2>{});
    if (--left == 0) break;
    interval(std::integral_constant<int, 3>{});
    if (--left == 0) break;
  }
  wait_copies<0>();      // no copy may land after the end

  const float mul = role == 1 ? p.scale : 1.f;
  if constexpr (WINDOW) {
    if (item.w < 0) {        // first tokens of a document with rows far from them: joined by attn_sink_reduce_kernel
      const int lo = sink_end - p.sinks, part = far ? blk.q0 / p.far_chunk : (lo + p.far_rows) / p.far_chunk - 1;
      const int64_t half = static_cast<int64_t>(p.far_parts) * p.n_split * p.kv_heads * p.sinks * D;
      if (my_key < sink_end) {
        float* out = p.sink_partial + (role == 1 ? 0 : half) +
                     (((static_cast<int64_t>(part) * p.n_split + split) * p.kv_heads + hk) * p.sinks + my_key - lo) * D;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
          for (int jj = 0; jj < 4; ++jj)
            *reinterpret_cast<float4*>(out + dt * 32 + 8 * jj + rbase) =
                make_float4(acc[dt][4 * jj] * mul, acc[dt][4 * jj + 1] * mul, acc[dt][4 * jj + 2] * mul, acc[dt][4 * jj + 3] * mul);
      }
      if (far) return;
    }
  }
  if (slices > 1) {
    if (!key_ok) return;
    // lane owns key my_key; register i of tile dt is d = 32 dt + acc_row(i)
    const int64_t half = static_cast<int64_t>(p.n_split) * p.pk.tokens * p.kv_heads * D;
    float* out = p.dkv_partial + (role == 1 ? 0 : half) +
                 ((static_cast<int64_t>(split) * p.pk.tokens + my_key) * p.kv_heads + hk) * D;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj)
        *reinterpret_cast<float4*>(out + dt * 32 + 8 * jj + rbase) =
            make_float4(acc[dt][4 * jj] * mul, acc[dt][4 * jj + 1] * mul, acc[dt][4 * jj + 2] * mul, acc[dt][4 * jj + 3] * mul);
    return;
  }
  if constexpr (ROPE)
    if (role == 1) turn_back<D>(acc, p.rope + static_cast<int64_t>(min(my_key, blk.hi - 1)) * (D / 2), lane);
  ring_barrier();          // every wave is done with the ring, which takes the rows now
  uint16_t* out = reinterpret_cast<uint16_t*>(pick(addr(p.dv), addr(p.dk))) +
                  static_cast<int64_t>(pick(p.dv_ld, p.dk_ld)) * grp_k0 + hk * D;
  // a wave's 64 D bytes of the ring
  store_rows<D>(acc, mul, &qg[0][0][0] + wave * (64 * D), out, pick(p.dv_ld, p.dk_ld), blk.hi - grp_k0, lane);
}

// dK, dV = the sum of the slices' fp32 parts in order, for the blocks that were cut:
// a workgroup per block, kv head and quarter of its rows, eight columns per thread.
// Four slices of 32768 rows and one head of 128: 29 us for 151 MB.  It runs wherever a
// block may be cut, as only the GPU knows the documents: 5 us where few or none are.
template <int D, bool ROPE, bool WINDOW>
__global__ void __launch_bounds__(256) attn_packed_reduce_kernel(AttnArgs<WINDOW> p) {
  const int hk = static_cast<int>(blockIdx.y), lane = static_cast<int>(threadIdx.x) & 63, at = static_cast<int>(blockIdx.x) / 4;
  const SeqBlock blk = p.cut_rows ? block_at(p.pk, at * 128, lane) : seq_block(p.pk, at, 128, lane);
  if (blk.row0 >= blk.hi) return;
  const int n_rows = blk.hi - blk.row0, slices = packed_slices<WINDOW>(p, blk.row0, block_rows<WINDOW>(p, blk.lo, blk.hi, blk.row0));
  if (slices == 1) return;
  const int64_t step = static_cast<int64_t>(p.pk.tokens) * p.kv_heads * D;
  constexpr int C = D / 8, R = 256 / C;                  // rows at a time
  const int first = static_cast<int>(blockIdx.x) % 4 * 32;
  const int col = hk * D + static_cast<int>(threadIdx.x) % C * 8;
#pragma unroll
  for (int u = 0; u < 32 / R; ++u) {
    const int r = first + u * R + static_cast<int>(threadIdx.x) / C;
    if (r >= n_rows) return;
    const int64_t row = blk.row0 + r;
    const float* src = p.dkv_partial + row * p.kv_heads * D + col;
    float4 v[2][2];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int h = 0; h < 2; ++h) v[which][h] = *reinterpret_cast<const float4*>(src + which * p.n_split * step + 4 * h);
    for (int s = 1; s < slices; ++s)
#pragma unroll
      for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 x = *reinterpret_cast<const float4*>(src + (which * p.n_split + s) * step + 4 * h);
          v[which][h].x += x.x; v[which][h].y += x.y; v[which][h].z += x.z; v[which][h].w += x.w;
        }
    if constexpr (ROPE) {      // dK turned back; the lane C/2 further holds the pairs' other elements
      const bool upper = static_cast<int>(threadIdx.x) % C >= C / 2;
      const float2* tab = p.rope + row * (D / 2) + static_cast<int>(threadIdx.x) % (C / 2) * 8;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float* x = &v[0][h].x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 cs = tab[4 * h + j];
          const float other = __shfl_xor(x[j], C / 2, 64);
          x[j] = x[j] * cs.x + (upper ? -other : other) * cs.y;
        }
      }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      uint16_t* dst = which ? p.dv + row * p.dv_ld + col : p.dk + row * p.dk_ld + col;
      *reinterpret_cast<u32x4*>(dst) = u32x4{pack2(v[which][0].x, v[which][0].y), pack2(v[which][0].z, v[which][0].w),
                                             pack2(v[which][1].x, v[which][1].y), pack2(v[which][1].z, v[which][1].w)};
    }
  }
}

// dK, dV of first tokens whose document has rows far from them: the sum of their block's own
// part and of those of the far rows, in order, over what attn_packed_dkdv_kernel or
// attn_packed_reduce_kernel stored.  A workgroup per part that may be a document's first and
// kv head, a wave per first token and tensor, sixteen loads in flight (one load after another:
// 51 us for 48 parts of four slices).
template <int D>
__global__ void __launch_bounds__(256) attn_sink_reduce_kernel(WindowAttn p) {
  constexpr int N = D / 64, L = 16;      // columns per lane; loads in flight
  const int lane = static_cast<int>(threadIdx.x) & 63, hk = static_cast<int>(blockIdx.y);
  const int part0 = static_cast<int>(blockIdx.x), base = (part0 + 1) * p.far_chunk;
  // the document whose first far row lies in chunk part0 + 1
  const SeqRows s = seq_of_row(p.pk, base + p.far_chunk - 1 - p.far_rows, lane);
  if (s.i < 0 || s.lo + p.far_rows < base || s.hi <= s.lo + p.far_rows) return;
  const int parts = (s.hi - 1) / p.far_chunk - part0;
  const int64_t step = static_cast<int64_t>(p.kv_heads) * p.sinks * D;       // from one slice to the next
  const int64_t half = static_cast<int64_t>(p.far_parts) * p.n_split * step;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int i = static_cast<int>(blockIdx.z) * 4 + wave; i < 2 * p.sinks; i += 4 * static_cast<int>(gridDim.z)) {
    const int which = i & 1, row = i >> 1;
    const float* src = p.sink_partial + which * half + (static_cast<int64_t>(part0) * p.n_split * p.kv_heads + hk) * p.sinks * D +
                       static_cast<int64_t>(row) * D + lane * N;
    // the own part's slices, then those of every far part
    const int row0 = s.lo + row / 128 * 128, own = packed_slices<true>(p, row0, block_rows<true>(p, s.lo, s.hi, row0));
    const int n = p.cut_rows ? parts : parts * p.n_split;
    const int64_t far_step = p.cut_rows ? p.n_split * step : step;
    float v[N];
#pragma unroll
    for (int u = 0; u < N; ++u) v[u] = src[u];
    for (int c = 1; c < own; ++c)
#pragma unroll
      for (int u = 0; u < N; ++u) v[u] += src[c * step + u];
    src += p.n_split * step;
    for (int left = n; left > 0; left -= L, src += L * far_step) {
      float x[L][N];
#pragma unroll
      for (int j = 0; j < L; ++j)        // loads without a condition: they stay in flight together
#pragma unroll
        for (int u = 0; u < N; ++u) x[j][u] = src[min(j, left - 1) * far_step + u];
#pragma unroll
      for (int j = 0; j < L; ++j)
#pragma unroll
        for (int u = 0; u < N; ++u) v[u] += j < left ? x[j][u] : 0.f;
    }
    uint16_t* dst = (which ? p.dv + (s.lo + row) * p.dv_ld : p.dk + (s.lo + row) * p.dk_ld) + hk * D + lane * N;
    if constexpr (N == 2) *reinterpret_cast<uint32_t*>(dst) = pack2(v[0], v[1]);
    else *dst = f2bf(v[0]);
  }
}

// Blocks of `rows` rows over every packing of `tokens` rows.
int64_t packed_slots(const PackedAttn& p, int rows) { return p.pk.tokens / rows + static_cast<int64_t>(p.pk.n_seqs); }

// Query heads of a kv head taken together by a query block.
int packed_hpb(int heads, int kv_heads) {
  const int group = heads / kv_heads;
  return group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1;
}

template <int D, bool ROPE, bool WINDOW>
hipError_t packed_launch(AttnArgs<WINDOW>& p, int part, hipStream_t stream) {
  if (part == 0 || part == 2) {
    p.hpb = packed_hpb(p.heads, p.kv_heads);
    p.n_slots = static_cast<int32_t>(packed_slots(p, 128 / p.hpb));
    const dim3 grid(static_cast<unsigned>(p.n_slots) * (p.heads / p.hpb) + (part == 2));    // and the workgroup that lists
    if (part == 0) hipLaunchKernelGGL((attn_packed_fwd_kernel<D, WINDOW>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((attn_packed_dq_kernel<D, ROPE, WINDOW>), grid, dim3(256), 0, stream, p);
  } else if (part == 1) {
    int64_t places;
    if constexpr (WINDOW) places = attn_window_places(p);
    else places = attn_packed_places(p);
    const unsigned blocks = static_cast<unsigned>(places) * p.kv_heads;
    hipLaunchKernelGGL((attn_packed_dkdv_kernel<D, ROPE, WINDOW>), dim3(blocks), dim3(512), 0, stream, p);
  } else if (part == 3) {
    if (p.n_split == 1) return hipSuccess;
    const dim3 grid(static_cast<unsigned>(p.cut_rows ? packed_windows(p) : packed_slots(p, 128)) * 4, p.kv_heads);
    hipLaunchKernelGGL((attn_packed_reduce_kernel<D, ROPE, WINDOW>), grid, dim3(256), 0, stream, p);
  } else if constexpr (WINDOW) {
    const dim3 grid(static_cast<unsigned>(p.far_parts - 1), p.kv_heads, std::min((p.sinks + 1) / 2, 16));
    hipLaunchKernelGGL(attn_sink_reduce_kernel<D>, grid, dim3(256), 0, stream, p);
  }
  return hipGetLastError();
}
