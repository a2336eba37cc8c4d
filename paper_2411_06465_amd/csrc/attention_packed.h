// Causal grouped-query attention over packed documents (device code, part of
// attention.hip: it stands on that file's LDS tiles, fragments and products).
//
//   o_i = sum_j p_ij v_j, p_i. = softmax(scale q_i . k_j), j from row i's document's
//   first row to i; the backward recomputes p from the log-sum-exp.
//
// Every tile of queries and keys lies within one document (seq_block), so the
// only mask is the causal one, as for a single sequence, and nothing a document
// holds (an infinity or NaN in V, say, which a zero probability would not hide)
// can reach another.

// ------------------------------------------------------------------ forward
// One workgroup per block of query rows and hpb query heads of one kv head: 4
// waves x 32 rows, wave w on head w % hpb.  Each lane holds one query's scores
// (S^T = K Q^T), so the softmax statistics are per-lane scalars.
template <int D>
__global__ void __launch_bounds__(256) attn_packed_fwd_kernel(PackedAttn p) {
  constexpr int TB = KT * D * 2;
  __shared__ __attribute__((aligned(16))) uint8_t kbuf[2][TB], vbuf[2][TB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_hg = p.heads / p.hpb, rows = 128 / p.hpb;
  const int slot = p.n_slots - 1 - static_cast<int>(blockIdx.x) / n_hg, h0 = static_cast<int>(blockIdx.x) % n_hg * p.hpb;
  const SeqBlock blk = seq_block(p.pk, slot, rows, lane);
  if (blk.row0 >= blk.hi) return;
  const int hq = h0 + wave % p.hpb, hk = h0 / (p.heads / p.kv_heads);
  const int my_q = blk.row0 + wave / p.hpb * 32 + (lane & 31);
  const bool q_ok = my_q < blk.hi;
  const int n_keys = min(blk.row0 + rows, blk.hi) - blk.lo;      // keys the block's last row sees
  const int rbase = 4 * (lane >> 5);
  const LaneAddr la = lane_addr<D>(lane);

  bf16x8 qf[D / 16];
  {
    const uint16_t* qb = p.q + static_cast<int64_t>(min(my_q, blk.hi - 1)) * p.q_ld + hq * D;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qb + (2 * kk + (lane >> 5)) * 8);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) settle(qf[kk]);
  }
  const float c = p.scale * kLog2e;
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = f32x16{};

  const TileCopy<D, KT> copy_k(p.k_ld, wave, lane), copy_v(p.v_ld, wave, lane);
  const int n_tiles = (n_keys + KT - 1) / KT;
  const auto issue = [&](int t, int b) __attribute__((always_inline)) {
    const int64_t row = blk.lo + t * KT;
    const int valid = blk.hi - static_cast<int>(row);
    copy_k(lds_addr(kbuf[b]), p.k + row * p.k_ld + hk * D, valid);
    copy_v(lds_addr(vbuf[b]), p.v + row * p.v_ld + hk * D, valid);
  };
  issue(0, 0);
  for (int t = 0; t < n_tiles; ++t) {
    const int b = t & 1;
    wait_copies<0>();
    ring_barrier();                     // tile t is visible; the other buffers are free
    if (t + 1 < n_tiles) issue(t + 1, b ^ 1);
    __builtin_amdgcn_sched_barrier(0);
    f32x16 s[2] = {f32x16{}, f32x16{}};
    scores2<D, kLookFwd>(kbuf[b], 0, qf, s[0], kbuf[b], 32, qf, s[1], la);
    const int lim = my_q - (blk.lo + t * KT) - rbase;      // last visible key, relative to the lane's first
    float mx = -INFINITY;
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (t2 * 32 + 8 * (i >> 2) + (i & 3) > lim) s[t2][i] = -INFINITY;
        mx = fmaxf(mx, s[t2][i]);
      }
    mx = half_max(mx) * c;
    const float m_new = fmaxf(m_run, mx);
    const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(m_run - m_new);
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) o[dt] *= alpha;
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[t2][i] = fast_exp2(fmaf(s[t2][i], c, -m_use));
        l_run += s[t2][i];
      }
    // P as bf16 for the product: half a step, 2^-9 of each probability, of the size
    // of the output's own rounding
    const bf16x8 x[4] = {frag_acc(s[0], 0), frag_acc(s[0], 8), frag_acc(s[1], 0), frag_acc(s[1], 8)};
    accum_t<D, 4, kLookDq>(vbuf[b], x, o, la);
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  if (!q_ok) return;
  const float inv = 1.0f / l_tot;
  uint16_t* ob = p.o + static_cast<int64_t>(my_q) * p.o_ld + hq * D;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      const int d = dt * 32 + 8 * jj + rbase;
      *reinterpret_cast<u32x2*>(ob + d) = u32x2{pack2(o[dt][4 * jj] * inv, o[dt][4 * jj + 1] * inv),
                                                pack2(o[dt][4 * jj + 2] * inv, o[dt][4 * jj + 3] * inv)};
    }
  if (lane < 32) p.lse[static_cast<int64_t>(hq) * p.pk.tokens + my_q] = (m_run + __builtin_amdgcn_logf(l_tot)) * kLn2;
}

// ------------------------------------------------------------------ backward: dQ
// The forward's blocks.  Per key tile: S^T = K Q^T and dP^T = V dO^T, then
// dS^T = P^T (dP^T - delta) feeds dQ^T += K^T dS^T from registers.  delta =
// rowsum(dO * O) is formed here and written out for the dK/dV pass.
template <int D>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) attn_packed_dq_kernel(PackedAttn p) {
  constexpr int KQ = 32;                     // keys per tile
  constexpr int TB = KQ * D * 2;
  __shared__ __attribute__((aligned(16))) uint8_t kbuf[2][TB], vbuf[2][TB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_hg = p.heads / p.hpb, rows = 128 / p.hpb;
  const int slot = p.n_slots - 1 - static_cast<int>(blockIdx.x) / n_hg, h0 = static_cast<int>(blockIdx.x) % n_hg * p.hpb;
  const SeqBlock blk = seq_block(p.pk, slot, rows, lane);
  if (blk.row0 >= blk.hi) return;
  const int hq = h0 + wave % p.hpb, hk = h0 / (p.heads / p.kv_heads);
  const int wave_q0 = blk.row0 + wave / p.hpb * 32;
  const int my_q = wave_q0 + (lane & 31);
  const bool q_ok = my_q < blk.hi;
  const int n_keys = min(blk.row0 + rows, blk.hi) - blk.lo;
  const int rbase = 4 * (lane >> 5);
  const LaneAddr la = lane_addr<D>(lane);

  bf16x8 qf[D / 16], dof[D / 16];
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
  if (q_ok && lane < 32) p.delta[sidx] = my_delta;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    settle(qf[kk]);
    settle(dof[kk]);
  }
  settle(my_lse);
  settle(my_delta);
  const float c = p.scale * kLog2e;
  f32x16 dq[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dq[i] = f32x16{};

  const TileCopy<D, KQ> copy_k(p.k_ld, wave, lane), copy_v(p.v_ld, wave, lane);
  const int n_tiles = (n_keys + KQ - 1) / KQ;
  const auto issue = [&](int t, int b) __attribute__((always_inline)) {
    const int64_t r0 = blk.lo + t * KQ;
    const int valid = blk.hi - static_cast<int>(r0);
    copy_k(lds_addr(kbuf[b]), p.k + r0 * p.k_ld + hk * D, valid);
    copy_v(lds_addr(vbuf[b]), p.v + r0 * p.v_ld + hk * D, valid);
  };
  issue(0, 0);
  for (int t = 0; t < n_tiles; ++t) {
    const int b = t & 1;
    wait_copies<0>();
    ring_barrier();
    if (t + 1 < n_tiles) issue(t + 1, b ^ 1);
    __builtin_amdgcn_sched_barrier(0);
    f32x16 sc = f32x16{}, dp = f32x16{};
    scores2<D, kLookDq>(kbuf[b], 0, qf, sc, vbuf[b], 0, dof, dp, la);
    if (blk.lo + t * KQ + KQ - 1 > wave_q0) {               // the tile reaches past the wave's first row
      const int lim = my_q - (blk.lo + t * KQ) - rbase;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + (i & 3) > lim) sc[i] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = fast_exp2(fmaf(sc[i], c, -my_lse)) * (dp[i] - my_delta);   // dS^T
    const bf16x8 sf[2] = {frag_acc(sc, 0), frag_acc(sc, 8)};
    accum_t<D, 2, kLookDq>(kbuf[b], sf, dq, la);
  }

  if (!q_ok) return;
  uint16_t* out = p.dq + static_cast<int64_t>(my_q) * p.dq_ld + hq * D;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      const int d = dt * 32 + 8 * jj + rbase;
      *reinterpret_cast<u32x2*>(out + d) =
          u32x2{pack2(dq[dt][4 * jj] * p.scale, dq[dt][4 * jj + 1] * p.scale),
                pack2(dq[dt][4 * jj + 2] * p.scale, dq[dt][4 * jj + 3] * p.scale)};
    }
}

// ------------------------------------------------------------------ backward: dK, dV
// One workgroup per (block of 128 keys, kv head, slice of its query heads): 4
// waves x 32 keys, each lane one key.  Per query tile and head: S = Q K^T and
// dP = dO V^T, then dV^T += dO^T P and dK^T += Q^T dS with P, dS from registers.
template <int D>
__global__ void __launch_bounds__(256) attn_packed_dkdv_kernel(PackedAttn p) {
  constexpr int TB = QT * D * 2;
  __shared__ __attribute__((aligned(16))) uint8_t qbuf[2][TB], gbuf[2][TB];
  __shared__ __attribute__((aligned(16))) float st[2][2][QT];    // lse, delta
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = p.heads / p.kv_heads, hps = group / p.n_split;
  const int nyz = p.kv_heads * p.n_split;
  const int slot = static_cast<int>(blockIdx.x) / nyz, yz = static_cast<int>(blockIdx.x) % nyz;
  const int hk = yz / p.n_split, split = yz % p.n_split, head0 = hk * group + split * hps;
  const SeqBlock blk = seq_block(p.pk, slot, 128, lane);
  if (blk.row0 >= blk.hi) return;
  const int wave_k0 = blk.row0 + wave * 32;
  const int my_key = wave_k0 + (lane & 31);
  const bool key_ok = my_key < blk.hi;
  const int rbase = 4 * (lane >> 5);
  const LaneAddr la = lane_addr<D>(lane);

  bf16x8 kf[D / 16], vf[D / 16];
  {
    const int64_t row = min(my_key, blk.hi - 1);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const int dcol = hk * D + (2 * kk + (lane >> 5)) * 8;
      kf[kk] = *reinterpret_cast<const bf16x8*>(p.k + row * p.k_ld + dcol);
      vf[kk] = *reinterpret_cast<const bf16x8*>(p.v + row * p.v_ld + dcol);
    }
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      settle(kf[kk]);
      settle(vf[kk]);
    }
  }
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dk[i] = dv[i] = f32x16{};
  const float c = p.scale * kLog2e;
  const TileCopy<D, QT> copy_q(p.q_ld, wave, lane), copy_g(p.do_ld, wave, lane);
  const int n_qt = (blk.hi - blk.row0 + QT - 1) / QT, n_tiles = n_qt * hps;    // query tiles from the block's own rows on
  // lse or delta by arithmetic: a select of the members' addresses would put the kernel argument on the stack
  const uint64_t stat0 = reinterpret_cast<uint64_t>(p.lse) +
                         ((reinterpret_cast<uint64_t>(p.delta) - reinterpret_cast<uint64_t>(p.lse)) & (0ull - (wave & 1)));
  const auto issue = [&](int t, int b) __attribute__((always_inline)) {
    const int h = head0 + t / n_qt;
    const int64_t r0 = blk.row0 + t % n_qt * QT;
    const int valid = blk.hi - static_cast<int>(r0);
    copy_q(lds_addr(qbuf[b]), p.q + r0 * p.q_ld + h * D, valid);
    copy_g(lds_addr(gbuf[b]), p.dout + r0 * p.do_ld + h * D, valid);
    // waves 0 and 1 fetch the rows' lse and delta
    const float* stat = reinterpret_cast<const float*>(stat0) + static_cast<int64_t>(h) * p.pk.tokens + r0;
    if (wave < 2 && lane < QT) dma4(stat, static_cast<uint32_t>(min(lane, valid - 1)) * 4u, lds_addr(st[b][wave & 1]));
  };
  issue(0, 0);
  for (int t = 0; t < n_tiles; ++t) {
    const int b = t & 1;
    wait_copies<0>();
    ring_barrier();
    if (t + 1 < n_tiles) issue(t + 1, b ^ 1);
    __builtin_amdgcn_sched_barrier(0);
    const int q0 = blk.row0 + t % n_qt * QT;
    f32x16 s = f32x16{}, dp = f32x16{};
    scores2<D, kLookDq>(qbuf[b], 0, kf, s, gbuf[b], 0, vf, dp, la);
    // visible query rows r (relative to the lane's first row): lo <= r <= hi
    const int lo = my_key - q0 - rbase, hi = blk.hi - 1 - q0 - rbase;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = 8 * (i >> 2) + (i & 3);
      const float pr = fast_exp2(fmaf(s[i], c, -st[b][0][r + rbase] * kLog2e));
      s[i] = r < lo || r > hi ? 0.f : pr;
      dp[i] = r < lo || r > hi ? 0.f : pr * (dp[i] - st[b][1][r + rbase]);
    }
    const bf16x8 x[2] = {frag_acc(s, 0), frag_acc(s, 8)}, y[2] = {frag_acc(dp, 0), frag_acc(dp, 8)};
    accum_t<D, 2, kLookDq>(gbuf[b], x, dv, la);
    accum_t<D, 2, kLookDq>(qbuf[b], y, dk, la);
  }
  if (!key_ok) return;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) dk[dt] *= p.scale;
  if (p.n_split > 1) {
    const int64_t half = static_cast<int64_t>(p.n_split) * p.pk.tokens * p.kv_heads * D;
    float* pk = p.dkv_partial + ((static_cast<int64_t>(split) * p.pk.tokens + my_key) * p.kv_heads + hk) * D;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int d = dt * 32 + 8 * jj + rbase;
        *reinterpret_cast<float4*>(pk + d) =
            make_float4(dk[dt][4 * jj], dk[dt][4 * jj + 1], dk[dt][4 * jj + 2], dk[dt][4 * jj + 3]);
        *reinterpret_cast<float4*>(pk + half + d) =
            make_float4(dv[dt][4 * jj], dv[dt][4 * jj + 1], dv[dt][4 * jj + 2], dv[dt][4 * jj + 3]);
      }
    return;
  }
  uint16_t* ok = p.dk + static_cast<int64_t>(my_key) * p.dk_ld + hk * D;
  uint16_t* ov = p.dv + static_cast<int64_t>(my_key) * p.dv_ld + hk * D;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      const int d = dt * 32 + 8 * jj + rbase;
      *reinterpret_cast<u32x2*>(ok + d) =
          u32x2{pack2(dk[dt][4 * jj], dk[dt][4 * jj + 1]), pack2(dk[dt][4 * jj + 2], dk[dt][4 * jj + 3])};
      *reinterpret_cast<u32x2*>(ov + d) =
          u32x2{pack2(dv[dt][4 * jj], dv[dt][4 * jj + 1]), pack2(dv[dt][4 * jj + 2], dv[dt][4 * jj + 3])};
    }
}

// dK, dV = the sum of the slices' fp32 parts in order, for the rows that belong to
// a document.  Eight columns per thread.
template <int D>
__global__ void __launch_bounds__(256) attn_packed_reduce_kernel(PackedAttn p) {
  const int64_t idx = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t per_row = static_cast<int64_t>(p.kv_heads) * (D / 8);
  const int64_t first = seq_start(p.pk, 0), end = seq_start(p.pk, p.pk.n_seqs);
  const int64_t row = idx / per_row;
  if (row >= p.pk.tokens || row < first || row >= end) return;
  const int64_t col = idx % per_row * 8;                 // hk * D + d
  const int64_t step = static_cast<int64_t>(p.pk.tokens) * p.kv_heads * D;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float* src = p.dkv_partial + which * p.n_split * step + row * p.kv_heads * D + col;
    float4 a = *reinterpret_cast<const float4*>(src), b = *reinterpret_cast<const float4*>(src + 4);
    for (int s = 1; s < p.n_split; ++s) {
      const float4 x = *reinterpret_cast<const float4*>(src + s * step), y = *reinterpret_cast<const float4*>(src + s * step + 4);
      a.x += x.x; a.y += x.y; a.z += x.z; a.w += x.w;
      b.x += y.x; b.y += y.y; b.z += y.z; b.w += y.w;
    }
    uint16_t* dst = which ? p.dv + row * p.dv_ld + col : p.dk + row * p.dk_ld + col;
    *reinterpret_cast<u32x4*>(dst) = u32x4{pack2(a.x, a.y), pack2(a.z, a.w), pack2(b.x, b.y), pack2(b.z, b.w)};
  }
}

// Blocks of `rows` rows over every packing of `tokens` rows.
int64_t packed_slots(const PackedAttn& p, int rows) { return p.pk.tokens / rows + static_cast<int64_t>(p.pk.n_seqs); }

// Query heads of a kv head taken together by a query block.
int packed_hpb(int heads, int kv_heads) {
  const int group = heads / kv_heads;
  return group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1;
}

template <int D>
hipError_t packed_launch(PackedAttn& p, int part, hipStream_t stream) {
  if (part == 0 || part == 2) {
    p.hpb = packed_hpb(p.heads, p.kv_heads);
    p.n_slots = static_cast<int32_t>(packed_slots(p, 128 / p.hpb));
    const dim3 grid(static_cast<unsigned>(p.n_slots) * (p.heads / p.hpb));
    if (part == 0) hipLaunchKernelGGL(attn_packed_fwd_kernel<D>, grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(attn_packed_dq_kernel<D>, grid, dim3(256), 0, stream, p);
  } else if (part == 1) {
    p.n_slots = static_cast<int32_t>(packed_slots(p, 128));
    const dim3 grid(static_cast<unsigned>(p.n_slots) * p.kv_heads * p.n_split);
    hipLaunchKernelGGL(attn_packed_dkdv_kernel<D>, grid, dim3(256), 0, stream, p);
  } else {
    if (p.n_split == 1) return hipSuccess;
    const int64_t n = static_cast<int64_t>(p.pk.tokens) * p.kv_heads * (D / 8);
    hipLaunchKernelGGL(attn_packed_reduce_kernel<D>, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, stream, p);
  }
  return hipGetLastError();
}
