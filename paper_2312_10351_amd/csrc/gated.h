// The gated half of a feed-forward block (included by kernels.hip): y = act(x . Wg + bg) * (x . Wu + bu).
//
// Both projections share the operand x and meet element by element, so a workgroup computes
// the same columns of both: half the rows of its weight tile come from Wg, half from Wu (the
// N rows after it), arranged so that one lane holds a gate and the value it multiplies.  Against
// two products and an element-wise operator, x is read once and two results are neither written nor read.

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
    case 3: return fmaxf(x, 0.f);
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
template <typename T, typename AR>
__device__ __forceinline__ void gated_any_body(const AR &a, const Blk &b, unsigned char *lds) {
  typedef typename Vec16<T>::type V;
  typedef V VU __attribute__((aligned(sizeof(T))));
  constexpr int VE = Vec16<T>::N, BKE = 4 * VE, ROWB = 80, BM = 64, BC = 32;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, grp = lane >> 4, r16 = lane & 15;
  int tile_x, tile_y;
  xcd_tile(b, a.div_gx, tile_x, tile_y);
  const int m0 = tile_x * BM, n0 = tile_y * BC;
  const int kc = t & 3, row = t >> 2;                       // 16-byte chunk and tile row this thread moves
  // tile rows 0..31: gate columns, 32..63: the values they multiply
  const int n = n0 + (row & 31), m = m0 + row;
  const T *wr = (const T *)a.w + ((int64_t)(row >> 5) * a.N + min(n, a.N - 1)) * a.ldb;
  const T *xr = (const T *)a.x + (int64_t)min(m, a.M - 1) * a.lda;
  const bool wok = n < a.N, xok = m < a.M;
  V wv, xv;
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
  auto put = [&](int buf) {
    *(V *)(smem[buf] + row * ROWB + kc * 16) = wv;
    *(V *)(smem[buf] + (64 + row) * ROWB + kc * 16) = xv;
  };
  floatx4 acc[4];                                           // gate, gate, value, value columns of this wavefront's 16 rows
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int nk = (a.K + BKE - 1) / BKE;
  wv = load(wr, wok, kc * VE);
  xv = load(xr, xok, kc * VE);
  put(0);
  __syncthreads();
  for (int kt = 0; kt < nk; ++kt) {
    const bool more = kt + 1 < nk;
    if (more) {
      wv = load(wr, wok, (kt + 1) * BKE + kc * VE);
      xv = load(xr, xok, (kt + 1) * BKE + kc * VE);
    }
    const unsigned char *W = smem[kt & 1], *X = W + 64 * ROWB;
    const V xf = *(const V *)(X + (wave * 16 + r16) * ROWB + grp * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = mma16<T>(*(const V *)(W + (i * 16 + r16) * ROWB + grp * 16), xf, acc[i]);
    if (more) put((kt & 1) ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) gated_store4<T>(a, acc[i], acc[i + 2], m0 + wave * 16 + r16, n0 + i * 16 + grp * 4);
}
