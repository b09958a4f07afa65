// The norms around a residual sum (included by kernels.hip):
//   z = N(x) w + b or x;  s = alpha r + beta gate z;  y = N(s) w' + b' (and s), or s.
//
// What bounds it: bytes (x, r and a gate of full size read once, s and y written once), at few rows the
// launch and two reductions one after another.  A row lives in registers between its statistics,
// held by a wavefront or by a workgroup of four; x and r are requested together, so that
// r arrives behind x's reduction.  The statistics are taken over the centred values (two passes over
// registers), in fp32, and y is computed from s as it is before it is rounded.  Chunks are read at element
// alignment, so odd widths take the same path; a row's last chunk goes element by element where it is not whole.

template <typename T, typename P> __device__ __forceinline__ void load_run(const P *src, int col, int cols, float *v) {
  constexpr int VE = Vec16<T>::N;
  constexpr int PE = 16 / (int)sizeof(P);                     // elements of P per 16 bytes
  typedef P PV __attribute__((ext_vector_type(PE), aligned(sizeof(P))));
  if (col + VE <= cols) {
#pragma unroll
    for (int q = 0; q < VE; q += PE) {
      const PV t = *(const PV *)(src + col + q);
#pragma unroll
      for (int e = 0; e < PE; ++e) v[q + e] = (float)t[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] = col + e < cols ? (float)src[col + e] : 0.f;
  }
}
template <typename T> __device__ __forceinline__ void store_run(T *dst, int col, int cols, const float *v) {
  typedef typename Vec16<T>::type V;
  typedef V VU __attribute__((aligned(sizeof(T))));
  constexpr int VE = Vec16<T>::N;
  if (col + VE <= cols) {
    V o;
#pragma unroll
    for (int e = 0; e < VE; ++e) o[e] = (T)v[e];
    *(VU *)(dst + col) = o;
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (col + e < cols) dst[col + e] = (T)v[e];
  }
}

template <typename T, int G, int MAXCH, typename AR>
__device__ __forceinline__ void residual_norm_body(const AR &a, const Blk &b, unsigned char *lds) {
  constexpr int VE = Vec16<T>::N;
  float *scratch = (float *)lds;                              // [4]
  const int gl = threadIdx.x % G, cols = a.cols;
  const int row = b.x * (256 / G) + threadIdx.x / G;
  if (G == 64 && row >= a.rows) return;                       // whole wavefront leaves together
  const int64_t base = (int64_t)row * cols;
  const T *gate = a.g ? (const T *)a.g + (int64_t)fast_div((uint32_t)row, (uint32_t)a.gate_rows, a.div_gate) * cols : nullptr;
  float v[MAXCH][VE], r[MAXCH][VE];
#pragma unroll
  for (int c = 0; c < MAXCH; ++c) {
    const int col = (c * G + gl) * VE;
#pragma unroll
    for (int e = 0; e < VE; ++e) { v[c][e] = 0.f; r[c][e] = 0.f; }
    if (col < cols) {
      load_run<T>((const T *)a.x + base, col, cols, v[c]);
      if (a.r) load_run<T>((const T *)a.r + base, col, cols, r[c]);
    }
  }
  // v -> (v - mean) / sqrt(mean of squares + eps) * w + b over the row's cols elements
  auto norm = [&](const T *w, const float *bias) {
    if (!a.rms) {
      float s = 0.f;
#pragma unroll
      for (int c = 0; c < MAXCH; ++c)
#pragma unroll
        for (int e = 0; e < VE; ++e) s += v[c][e];            // zeros behind the row
      const float mean = group_reduce<G, false>(s, scratch) / (float)cols;
#pragma unroll
      for (int c = 0; c < MAXCH; ++c)
#pragma unroll
        for (int e = 0; e < VE; ++e) v[c][e] = (c * G + gl) * VE + e < cols ? v[c][e] - mean : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < MAXCH; ++c)
#pragma unroll
      for (int e = 0; e < VE; ++e) q += v[c][e] * v[c][e];
    const float k = 1.0f / sqrtf(group_reduce<G, false>(q, scratch) / (float)cols + a.eps);
#pragma unroll
    for (int c = 0; c < MAXCH; ++c) {
      const int col = (c * G + gl) * VE;
      if (col >= cols) continue;
      float wv[VE], bv[VE];
      if (w) load_run<T>(w, col, cols, wv);
      if (bias) load_run<T>(bias, col, cols, bv);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        v[c][e] *= k;
        if (w) v[c][e] *= wv[e];
        if (bias) v[c][e] += bv[e];
      }
    }
  };
  if (a.after) norm((const T *)a.w, a.b);
  const int skip = a.after ? cols : 0;                        // the weights of the second norm follow the first's
#pragma unroll
  for (int c = 0; c < MAXCH; ++c) {
    const int col = (c * G + gl) * VE;
    if (col >= cols) continue;
    float gv[VE];
    if (gate) load_run<T>(gate, col, cols, gv);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float z = col + e < cols ? (gate ? v[c][e] * gv[e] : v[c][e]) : 0.f;
      v[c][e] = a.beta * z;
      if (a.r) v[c][e] += a.alpha * r[c][e];
    }
    if (a.s) store_run<T>((T *)a.s + base, col, cols, v[c]);
  }
  if (!a.before) return;
  norm(a.w ? (const T *)a.w + skip : nullptr, a.b ? a.b + skip : nullptr);
#pragma unroll
  for (int c = 0; c < MAXCH; ++c) {
    const int col = (c * G + gl) * VE;
    if (col < cols) store_run<T>((T *)a.y + base, col, cols, v[c]);
  }
}

// Rows too wide for registers: one workgroup per row, inputs re-read for every statistic.
template <typename T, typename AR>
__device__ __forceinline__ void residual_norm_wide_body(const AR &a, const Blk &b, unsigned char *lds) {
  float *scratch = (float *)lds;                              // [4]
  const int cols = a.cols, row = b.x;
  const int64_t base = (int64_t)row * cols;
  const T *x = (const T *)a.x + base, *r = a.r ? (const T *)a.r + base : nullptr;
  const T *gate = a.g ? (const T *)a.g + (int64_t)fast_div((uint32_t)row, (uint32_t)a.gate_rows, a.div_gate) * cols : nullptr;
  float mean1 = 0.f, k1 = 1.f;
  auto z = [&](int col) {
    float t = (float)x[col];
    if (a.after) {
      t = (t - mean1) * k1;
      if (a.w) t *= (float)((const T *)a.w)[col];
      if (a.b) t += a.b[col];
    }
    return t;
  };
  auto sum = [&](int col) {
    const float t = a.beta * (gate ? z(col) * (float)gate[col] : z(col));
    return r ? t + a.alpha * (float)r[col] : t;
  };
  auto stats = [&](auto value, float &mean, float &k) {
    float p = 0.f;
    mean = 0.f;
    if (!a.rms) {
      for (int col = threadIdx.x; col < cols; col += 256) p += value(col);
      mean = group_reduce<256, false>(p, scratch) / (float)cols;
    }
    p = 0.f;
    for (int col = threadIdx.x; col < cols; col += 256) { const float d = value(col) - mean; p += d * d; }
    k = 1.0f / sqrtf(group_reduce<256, false>(p, scratch) / (float)cols + a.eps);
  };
  if (a.after) stats([&](int col) { return (float)x[col]; }, mean1, k1);
  const int skip = a.after ? cols : 0;
  float mean2 = 0.f, k2 = 1.f;
  if (a.before) stats(sum, mean2, k2);
  for (int col = threadIdx.x; col < cols; col += 256) {
    const float s = sum(col);
    if (a.s) ((T *)a.s)[base + col] = (T)s;
    if (a.before) {
      float t = (s - mean2) * k2;
      if (a.w) t *= (float)((const T *)a.w)[skip + col];
      if (a.b) t += a.b[skip + col];
      ((T *)a.y)[base + col] = (T)t;
    }
  }
}
