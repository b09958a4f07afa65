// The gated half of a feed-forward block (included by kernels.hip): y = act(x . Wg + bg) * (x . Wu + bu).
//
// Both projections share the operand x and meet element by element, so a workgroup computes
// the same columns of both: half the rows of its weight tile come from Wg, half from Wu (the
// N rows after it), arranged so that one lane holds a gate and the value it multiplies.  Against
// two products and an element-wise operator, x is read once and two results are neither written nor read.
//
// What bounds it: with few rows the weights' bytes, with many the matrix cores.  Measured, fp16, 4096 -> 2 x 12288
// (us; the plain library product of the same size reaches 1350 TFLOP/s): 1 row 34.4 (5.9 TB/s of weights),
// 64 rows 48, 512 rows 109, 4096 rows 680 (1210 TFLOP/s).  Which form runs follows from a table of costs
// (kGatedForms in plan_decoder.cpp).

template <typename T> __device__ __forceinline__ float gate_apply(int act, float x) {
  constexpr bool H = std::is_same<T, half_t>::value;
  // exp and the divisions below: for fp16 results the hardware's (2^-22), else the library's
  auto ex = [](float v) { return H ? __builtin_amdgcn_exp2f(v * 1.44269504088896341f) : expf(v); };
  auto over = [](float n, float d) { return H ? n * __builtin_amdgcn_rcpf(d) : n / d; };
  switch (act) {
    case 0: return over(x, 1.0f + ex(-x));
    case 1: return elt_apply<T>(2, x);
    case 2: {                                               // 0.5 (1 + tanh t) = 1 / (1 + exp(-2 t))
      const float t = 0.79788456080286536f * (x + 0.044715f * x * x * x);
      return over(x, 1.0f + ex(-2.0f * t));
    }
    case 3: return x < 0.f ? 0.f : x;                       // NaN stays, as in the others
    default: return over(1.0f, 1.0f + ex(-x));
  }
}
// Bias of gate and value columns n .. n + 3 (zeros without one).
template <typename T, typename AR>
__device__ __forceinline__ void gated_store4(const AR &a, floatx4 g, floatx4 u, int m, int n) {
  typedef typename Run4<T>::type R;
  if (m >= a.M || n >= a.N) return;
  T *dst = (T *)a.y + (int64_t)m * a.ldy + n;
  T o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = min(n + e, a.N - 1);
    const float bg = a.bias ? a.bias[c] : 0.f, bu = a.bias ? a.bias[(int64_t)a.N + c] : 0.f;
    o[e] = (T)(gate_apply<T>(a.relu, g[e] + bg) * (u[e] + bu));
  }
  if (n + 3 < a.N) {
    *(R *)dst = R{o[0], o[1], o[2], o[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.N) dst[e] = o[e];
  }
}

// Any row length, alignment and operand size: 64 rows x 32 columns per workgroup, operands staged
// through registers at element alignment and with 64-bit addresses.
constexpr int kGatedAnyRow = 144;                          // bytes from one row of a tile to the next: 128 and a skew
template <typename T, typename AR>
__device__ __forceinline__ void gated_any_body(const AR &a, const Blk &b, unsigned char *lds) {
  typedef typename Vec16<T>::type V;
  typedef V VU __attribute__((aligned(sizeof(T))));
  constexpr int VE = Vec16<T>::N, BKE = 8 * VE, ROWB = kGatedAnyRow, BM = 64, BC = 32;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, grp = lane >> 4, r16 = lane & 15;
  int tile_x, tile_y;
  xcd_tile(b, a.div_gx, tile_x, tile_y);
  const int m0 = tile_x * BM, n0 = tile_y * BC;
  // A thread moves a 16-byte chunk of rows `row` and `row` + 32: a gate column and the value it is
  // multiplied with, two rows of the input.  128 bytes of every row per step: with 64 the loads' latency is paid twice as often
  // (fp16, 77 x 1001 x 2000 21.5 -> 16.4 us, 2000 x 1001 x 2000 58.5 -> 54.5; fp32, 300 x 999 x 2000 52.5 -> 49.0,
  // 2000 x 999 x 2000 174 -> 177).
  const int kc = t & 7, row = t >> 3, n = n0 + row;
  const T *wr[2], *xr[2];
  bool xok[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    wr[h] = (const T *)a.w + ((int64_t)h * a.N + min(n, a.N - 1)) * a.ldb;
    xr[h] = (const T *)a.x + (int64_t)min(m0 + row + h * 32, a.M - 1) * a.lda;
    xok[h] = m0 + row + h * 32 < a.M;
  }
  const bool wok = n < a.N;
  V wv[2], xv[2];
  auto load = [&](const T *p, bool ok, int k) {
    V v = {};
    if (ok && k + VE <= a.K) v = *(const VU *)(p + k);
    else if (ok)
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (k + e < a.K) v[e] = p[k + e];
    return v;
  };
  unsigned char (*smem)[2 * 64 * ROWB] = (unsigned char (*)[2 * 64 * ROWB])lds;      // [2][weights, rows]
  auto fetch = [&](int kt) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      wv[h] = load(wr[h], wok, kt * BKE + kc * VE);
      xv[h] = load(xr[h], xok[h], kt * BKE + kc * VE);
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      *(V *)(smem[buf] + (row + h * 32) * ROWB + kc * 16) = wv[h];
      *(V *)(smem[buf] + (64 + row + h * 32) * ROWB + kc * 16) = xv[h];
    }
  };
  floatx4 acc[4];                                           // gate, gate, value, value columns of this wavefront's 16 rows
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int nk = (a.K + BKE - 1) / BKE;
  fetch(0);
  put(0);
  __syncthreads();
  for (int kt = 0; kt < nk; ++kt) {
    const bool more = kt + 1 < nk;
    if (more) fetch(kt + 1);
    const unsigned char *W = smem[kt & 1], *X = W + 64 * ROWB;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const V xf = *(const V *)(X + (wave * 16 + r16) * ROWB + (s * 4 + grp) * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = mma16<T>(*(const V *)(W + (i * 16 + r16) * ROWB + (s * 4 + grp) * 16), xf, acc[i]);
    }
    if (more) put((kt & 1) ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) gated_store4<T>(a, acc[i], acc[i + 2], m0 + wave * 16 + r16, n0 + i * 16 + grp * 4);
}

// Bias of four gate columns and of the four values they multiply.
struct GateBias {
  __amdgpu_buffer_rsrc_t buf;
  int cols;
  template <typename AR> __device__ __forceinline__ GateBias(const AR &a)
      : buf(__builtin_amdgcn_make_buffer_rsrc((void *)a.bias, 0, a.bias ? (int)min((int64_t)a.N * 8, (int64_t)kOperandMaxBytes) : 0, 0x00020000)), cols(a.N) {}
  __device__ __forceinline__ floatx4 gate(int n) const {
    return __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(buf, n * 4, 0, 0));
  }
  __device__ __forceinline__ floatx4 value(int n) const { return gate(cols + n); }
};

// Slot of a 16-byte chunk of a weight row is chunk ^ gated_slot(row): the rows a fragment takes differ in it.
template <int FN> __device__ __forceinline__ int gated_slot(int row) { return (row & 3) | (((row >> (2 + log2_of(FN))) & 1) << 2); }

// Which weight row a tile row holds: of a wavefront's 16 FN rows, run q of 4 FN feeds the lanes of group q; its first
// half are 2 FN gate columns, its second half the values of the same columns.  A lane then ends up with 2 FN
// consecutive columns of a row, gate and value.
template <typename T, int FN, int NW, int LW, int LX, typename AR>
__device__ __forceinline__ void gated_stager(Stager<T, LW, LX> &st, const AR &a, int n0, int m0, int wave, int lane) {
  st.init(a, (const T *)a.w, (const T *)a.x, 0, m0, 0, wave, NW, lane, (lane & 7) ^ gated_slot<FN>(wave * 8 + (lane >> 3)),
          (lane & 7) ^ (lane >> 3));
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int row = (wave + i * NW) * 8 + (lane >> 3), in = row % (4 * FN);
    const int n = n0 + row / (16 * FN) * (8 * FN) + row % (16 * FN) / (4 * FN) * (2 * FN) + in % (2 * FN);
    st.wo[i] = n < a.N ? ((uint32_t)(n + (in >= 2 * FN ? a.N : 0)) * (uint32_t)a.ldb + (uint32_t)st.kw0) * (int)sizeof(T) : kOperandMaxBytes;
  }
}

// Results of a lane: rows m, m + 16 ..., 2 FN columns from n on.
template <typename T, int FN, int FM, typename AR>
__device__ __forceinline__ void gated_finish(const AR &a, const floatx4 (&acc)[FN][FM], int m, int n) {
  typedef typename Vec16<T>::type V;
  typedef V VU __attribute__((aligned(sizeof(T))));
  constexpr int VE = Vec16<T>::N, Q = VE / 4, FH = FN / 2;   // Q: runs of four per 16 bytes
  static_assert(FH % Q == 0, "a lane's columns are whole vectors");
  const GateBias bias(a);
  floatx4 bg[FH], bu[FH];
#pragma unroll
  for (int i = 0; i < FH; ++i) { bg[i] = bias.gate(n + i * 4); bu[i] = bias.value(n + i * 4); }
#pragma unroll
  for (int j = 0; j < FM; ++j) {
    if (m + j * 16 >= a.M) continue;
    T *dst = (T *)a.y + (int64_t)(m + j * 16) * a.ldy + n;
#pragma unroll
    for (int i = 0; i < FH; i += Q) {
      V o;
#pragma unroll
      for (int e = 0; e < VE; ++e)
        o[e] = (T)(gate_apply<T>(a.relu, acc[i + e / 4][j][e % 4] + bg[i + e / 4][e % 4]) *
                   (acc[FH + i + e / 4][j][e % 4] + bu[i + e / 4][e % 4]));
      const int c = n + i * 4;
      if (c + VE <= a.N) {
        *(VU *)(dst + i * 4) = o;
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (c + e < a.N) dst[i * 4 + e] = o[e];
      }
    }
  }
}

// Many rows: BN weight rows (half of them gate columns) x BM rows per workgroup of WN x WM wavefronts, a
// ring of S stages of 128 bytes of K in workgroup memory, S - 1 requested ahead, one barrier per stage.
template <typename T, int BN, int BM, int WN, int WM, int S, typename AR>
__device__ __forceinline__ void gated_tile_body(const AR &a, const Blk &b, unsigned char *lds) {
  typedef typename Vec16<T>::type V;
  constexpr int NW = WN * WM, STAGE = (BN + BM) * 128;
  constexpr int FN = BN / WN / 16, FM = BM / WM / 16;
  constexpr int LW = BN / 8 / NW, LX = BM / 8 / NW, L = LW + LX;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int grp = lane >> 4, r16 = lane & 15;
  const int wn = wave % WN, wm0 = (wave / WN) * (BM / WM);
  int tile_x, tile_y;
  xcd_tile(b, a.div_gx, tile_x, tile_y);
  const int m0 = tile_x * BM, n0 = tile_y * (BN / 2);
  Stager<T, LW, LX> st;
  gated_stager<T, FN, NW>(st, a, n0, m0, wave, lane);
  const uint32_t base = lds_address(lds) + wave * 1024;
  auto issue = [&](int kt, int slot) { st.issue(kt, base + slot * STAGE, base + slot * STAGE + BN * 128, NW * 1024); };
  floatx4 acc[FN][FM];
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int nst = (a.K + Stager<T, LW, LX>::BKE - 1) / Stager<T, LW, LX>::BKE;
#pragma unroll
  for (int s = 0; s < S - 1; ++s)
    if (s < nst) issue(s, s);
  const int wrow = wn * (16 * FN) + (r16 >> 2) * (4 * FN) + (r16 & 3);
  int slot = 0, ahead = S - 1;
#pragma nounroll
  for (int kt = 0; kt < nst; ++kt) {
    if (kt + S - 2 < nst) wait_loads_and_meet<(S - 2) * L>();
    else wait_loads_and_meet<0>();
    if (kt + S - 1 < nst) issue(kt + S - 1, ahead);
    const unsigned char *Wb = lds + slot * STAGE, *Xb = Wb + BN * 128;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      V af[FN], bf[FM];
#pragma unroll
      for (int i = 0; i < FN; ++i) {
        const int row = wrow + i * 4;
        af[i] = *(const V *)(Wb + row * 128 + (((ks * 4 + grp) ^ gated_slot<FN>(row)) * 16));
      }
#pragma unroll
      for (int j = 0; j < FM; ++j) {
        const int row = wm0 + j * 16 + r16;
        bf[j] = *(const V *)(Xb + row * 128 + (((ks * 4 + grp) ^ (row & 7)) * 16));
      }
      mma_block<T>(af, bf, acc);
    }
    slot = slot == S - 1 ? 0 : slot + 1;
    ahead = ahead == S - 1 ? 0 : ahead + 1;
  }
  gated_finish<T, FN, FM>(a, acc, m0 + wm0 + r16, n0 + wn * (8 * FN) + grp * (2 * FN));
}

// Very many rows, fp16: 256 weight rows x 256 rows per workgroup of eight wavefronts, two stages of 64 KB.  Fragments are
// read half a stage ahead of the matrix instructions that take them, and woven between
// those of the half before: a wavefront that reads only when it needs the data leaves the matrix
// cores idle behind every barrier, where all eight read at once.
template <int BN, int BM, int WN, int WM, typename AR>
__device__ __forceinline__ void gated_wide_body(const AR &a, const Blk &b, unsigned char *lds) {
  typedef half_t T;
  typedef half8 V;
  constexpr int NW = WN * WM, STAGE = (BN + BM) * 128;
  constexpr int FN = BN / WN / 16, FM = BM / WM / 16;
  constexpr int LW = BN / 8 / NW, LX = BM / 8 / NW, L = LW + LX;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int grp = lane >> 4, r16 = lane & 15;
  const int wn = wave % WN, wm0 = (wave / WN) * (BM / WM);
  int tile_x, tile_y;
  xcd_tile(b, a.div_gx, tile_x, tile_y);
  {
    // Eight row tiles of every column tile in turn, then the next eight: the 32 workgroups an XCD runs at
    // a time then share 8 + 4 tiles of the operands, not 16 + 2 (4096 x 4096 x 12288: 682 -> 663 us).
    constexpr int G = 8;
    const int lin = tile_y * b.gx + tile_x, per = G * b.gy, run = lin / per, in = lin - run * per, rows = min(G, b.gx - run * G);
    tile_y = in / rows;
    tile_x = run * G + in - tile_y * rows;
  }
  const int m0 = tile_x * BM, n0 = tile_y * (BN / 2);
  Stager<T, LW, LX> st;
  gated_stager<T, FN, NW>(st, a, n0, m0, wave, lane);
  const uint32_t base = lds_address(lds) + wave * 1024;
  auto issue = [&](int kt, int slot) { st.issue(kt, base + slot * STAGE, base + slot * STAGE + BN * 128, NW * 1024); };
  floatx4 acc[FN][FM];
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int nst = (a.K + Stager<T, LW, LX>::BKE - 1) / Stager<T, LW, LX>::BKE;
  issue(0, 0);
  if (nst > 1) issue(1, 1);
  const int wrow = wn * (16 * FN) + (r16 >> 2) * (4 * FN) + (r16 & 3);
  V a0[FN], b0[FM], a1[FN], b1[FM];
  auto read = [&](V (&af)[FN], V (&bf)[FM], int slot, int ks) {
    const unsigned char *Wb = lds + slot * STAGE, *Xb = Wb + BN * 128;
#pragma unroll
    for (int i = 0; i < FN; ++i) {
      const int row = wrow + i * 4;
      af[i] = *(const V *)(Wb + row * 128 + (((ks * 4 + grp) ^ gated_slot<FN>(row)) * 16));
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
      const int row = wm0 + j * 16 + r16;
      bf[j] = *(const V *)(Xb + row * 128 + (((ks * 4 + grp) ^ (row & 7)) * 16));
    }
  };
  auto weave = [&]() {                                        // one read, two matrix instructions, and so on
#pragma unroll
    for (int q = 0; q < FN + FM; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, FN * FM - 2 * (FN + FM), 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  if (nst > 1) wait_loads_and_meet<L>();
  else wait_loads_and_meet<0>();
  read(a0, b0, 0, 0);
  int slot = 0;
#pragma nounroll
  for (int kt = 0; kt < nst; ++kt) {
    read(a1, b1, slot, 1);
    mma_block<T>(a0, b0, acc);
    weave();
    // Everybody has read this stage, and the next one has arrived (requested a whole stage ago).
    wait_loads_and_meet<0>();
    __builtin_amdgcn_sched_barrier(0);
    if (kt + 2 < nst) issue(kt + 2, slot);
    read(a0, b0, slot ^ 1, 0);                                // behind the last stage: read and not used
    mma_block<T>(a1, b1, acc);
    weave();
    slot ^= 1;
  }
  gated_finish<T, FN, FM>(a, acc, m0 + wm0 + r16, n0 + wn * (8 * FN) + grp * (2 * FN));
}

// Few rows: 16 NI weight rows (half of them gate columns) x 16 NJ rows per workgroup, K shared out between its
// four wavefronts in whole 128-byte steps; every wavefront has its own ring of S slots and waits for its own
// loads only, and the partial tiles meet once, at the end.
template <typename T, int NI, int NJ, int S, typename AR>
__device__ __forceinline__ void gated_split_body(const AR &a, const Blk &b, unsigned char *lds) {
  typedef typename Vec16<T>::type V;
  constexpr int WAVES = 4, BN = 16 * NI, BC = BN / 2, BM = 16 * NJ, STEP = (BN + BM) * 128, PITCH = BN + 4;
  constexpr int RING = split_ring_bytes(NI, NJ, S), LW = BN / 8, LX = BM / 8, L = LW + LX;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int grp = lane >> 4, r16 = lane & 15;
  int tile_x, tile_y;
  xcd_tile(b, a.div_gx, tile_x, tile_y);
  const int m0 = tile_x * BM, n0 = tile_y * BC;
  const int nst = (a.K + Stager<T, LW, LX>::BKE - 1) / Stager<T, LW, LX>::BKE;
  const int k_begin = nst * wave / WAVES, k_end = nst * (wave + 1) / WAVES;
  Stager<T, LW, LX> st;
  const int cslot = (lane & 7) ^ (lane >> 3);
  st.init(a, (const T *)a.w, (const T *)a.x, 0, m0, k_begin, 0, 1, lane, cslot, cslot);
#pragma unroll
  for (int i = 0; i < LW; ++i) {                            // tile rows: BC gate columns, then their values
    const int row = i * 8 + (lane >> 3), n = n0 + row % BC;
    st.wo[i] = n < a.N ? ((uint32_t)(n + (row >= BC ? a.N : 0)) * (uint32_t)a.ldb + (uint32_t)st.kw0) * (int)sizeof(T) : kOperandMaxBytes;
  }
  unsigned char *ring = lds + wave * RING;
  const uint32_t base = lds_address(ring);
  auto issue = [&](int kt, int slot) { st.issue(kt, base + slot * STEP, base + slot * STEP + BN * 128, 1024); };
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (k_begin + s < k_end) issue(k_begin + s, s);
  floatx4 acc[NI][NJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  constexpr int PG = BC / 4, PIECES = (BM * PG + 255) / 256;   // runs of four columns per row, per thread
  const GateBias bias(a);
  floatx4 bg[PIECES], bu[PIECES];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int n = n0 + (t + p * 256) % PG * 4;
    bg[p] = bias.gate(n);
    bu[p] = bias.value(n);
  }
  int slot = 0;
#pragma nounroll
  for (int kt = k_begin; kt < k_end; ++kt) {
    if (kt + S - 1 < k_end) wait_loads<(S - 1) * L>();
    else wait_loads<0>();
    const unsigned char *Wb = ring + slot * STEP, *Xb = Wb + BN * 128;
    V af[2][NI], bf[2][NJ];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int c = ((ks * 4 + grp) ^ (r16 & 7)) * 16;
#pragma unroll
      for (int i = 0; i < NI; ++i) af[ks][i] = *(const V *)(Wb + (i * 16 + r16) * 128 + c);
#pragma unroll
      for (int j = 0; j < NJ; ++j) bf[ks][j] = *(const V *)(Xb + (j * 16 + r16) * 128 + c);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");     // the slot has been read: it may be refilled
    if (kt + S < k_end) issue(kt + S, slot);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) mma_block<T>(af[ks], bf[ks], acc);
    slot = slot == S - 1 ? 0 : slot + 1;
  }
  float *part = (float *)ring;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) *(floatx4 *)(part + (j * 16 + r16) * PITCH + i * 16 + grp * 4) = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int idx = t + p * 256, pm = idx / PG, pn = idx % PG * 4, m = m0 + pm, n = n0 + pn;
    if (idx >= BM * PG || m >= a.M || n >= a.N) continue;
    const unsigned char *at = lds + (pm * PITCH + pn) * 4;
    floatx4 g = bg[p], u = bu[p];
#pragma unroll
    for (int q = 0; q < WAVES; ++q) {
      g += *(const floatx4 *)(at + q * RING);
      u += *(const floatx4 *)(at + q * RING + BC * 4);
    }
    typedef typename Run4<T>::type R;
    T o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (T)(gate_apply<T>(a.relu, g[e]) * u[e]);
    T *dst = (T *)a.y + (int64_t)m * a.ldy + n;
    if (n + 3 < a.N) {
      *(R *)dst = R{o[0], o[1], o[2], o[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.N) dst[e] = o[e];
    }
  }
}

// One row: a wavefront reads the two weight rows of a column from one end to the other and adds up its lanes at
// the end.  Taken for few columns, where even 16 of them per workgroup leave most compute units without
// work (fp32, 4096 -> 1024: 11.8 us, split16 15.5; 1024 -> 4096: 9.0 and 7.8), and for rows at odd addresses.
template <typename T, typename AR>
__device__ __forceinline__ void gated_row_body(const AR &a, const Blk &b, unsigned char *) {
  typedef typename Vec16<T>::type V;
  typedef V VU __attribute__((aligned(sizeof(T))));
  constexpr int VE = Vec16<T>::N, U = 2;
  const int lane = threadIdx.x & 63, n = b.x * 4 + (threadIdx.x >> 6);
  if (n >= a.N) return;
  const T *__restrict__ x = (const T *)a.x, *__restrict__ wg = (const T *)a.w + (int64_t)n * a.ldb,
          *__restrict__ wu = (const T *)a.w + ((int64_t)a.N + n) * a.ldb;
  float g = 0.f, u = 0.f;
  auto add = [&](V gv, V uv, int k) {
    const V xv = *(const VU *)(x + k);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      g += (float)gv[e] * (float)xv[e];
      u += (float)uv[e] * (float)xv[e];
    }
  };
  int k = lane * VE;
  for (; k + (U - 1) * 64 * VE + VE <= a.K; k += U * 64 * VE) {
    V gv[U], uv[U];
#pragma unroll
    for (int q = 0; q < U; ++q) { gv[q] = *(const VU *)(wg + k + q * 64 * VE); uv[q] = *(const VU *)(wu + k + q * 64 * VE); }
#pragma unroll
    for (int q = 0; q < U; ++q) add(gv[q], uv[q], k + q * 64 * VE);
  }
  for (; k + VE <= a.K; k += 64 * VE) add(*(const VU *)(wg + k), *(const VU *)(wu + k), k);
  for (int e = k; e < min(k + VE, a.K); ++e) {              // the piece that is not whole: one lane has it
    g += (float)wg[e] * (float)x[e];
    u += (float)wu[e] * (float)x[e];
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    g += __shfl_xor(g, off, 64);
    u += __shfl_xor(u, off, 64);
  }
  if (lane) return;
  if (a.bias) { g += a.bias[n]; u += a.bias[(int64_t)a.N + n]; }
  ((T *)a.y)[n] = (T)(gate_apply<T>(a.relu, g) * u);
}
