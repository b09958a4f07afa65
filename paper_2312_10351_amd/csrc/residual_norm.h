// The norms around a residual sum (included by kernels.hip):
//   z = N(x) w + b or x;  s = alpha r + beta gate z;  y = N(s) w' + b' (and s), or s.
//
// What bounds it: bytes (x, r and a gate of full size read once, s and y written once), at few rows the
// launch and two reductions one after another.  A row lives in registers between its statistics,
// held by a wavefront or by a workgroup of four; x, r and the gate are requested together.  A workgroup takes several
// rows where there are many and keeps the weights (of two norms 48 KB per row of 4096, against 40 KB of
// the row itself).  The statistics are taken over the centred values (two passes over registers), in fp32, and
// y is computed from s as it is before it is rounded.  A row is addressed through a buffer of its length: lanes behind
// it read zeros and write nothing, without a branch around any load.
// Measured (us): fp16, 4096 x 4096, two norms and a gate per channel 28 (134 MB, 4.8 TB/s; a large copy runs at 4.9),
// 64 x 4096 4.2, one row of 768 3.0 (an empty launch: 2.2); fp32 1000 x 1027 with a gate per element 7.9.

// W elements of a row from column col on: 16 bytes of T, or one element where the rows are not made of
// aligned 16-byte pieces.
template <typename P> __device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const P *row, int cols) {
  return __builtin_amdgcn_make_buffer_rsrc((void *)row, 0, row ? cols * (int)sizeof(P) : 0, 0x00020000);
}
template <typename P, int W> struct RowPiece {
  typedef P PV __attribute__((ext_vector_type(16 / sizeof(P))));
  static constexpr int PE = W == 1 ? 1 : 16 / (int)sizeof(P), NV = W / PE;
  typename std::conditional<W == 1, P, PV>::type v[NV];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t buf, int col) {
    const int at = col * (int)sizeof(P);
    if constexpr (W > 1) {
#pragma unroll
      for (int q = 0; q < NV; ++q) v[q] = __builtin_bit_cast(PV, __builtin_amdgcn_raw_buffer_load_b128(buf, at + q * 16, 0, 0));
    } else if constexpr (sizeof(P) == 2) {
      v[0] = __builtin_bit_cast(P, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(buf, at, 0, 0));
    } else {
      v[0] = __builtin_bit_cast(P, __builtin_amdgcn_raw_buffer_load_b32(buf, at, 0, 0));
    }
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (W == 1) return (float)v[0];
    else return (float)v[e / PE][e % PE];
  }
};
template <typename T, int W> __device__ __forceinline__ void store_piece(__amdgpu_buffer_rsrc_t buf, int col, const float *v) {
  const int at = col * (int)sizeof(T);
  if constexpr (W > 1) {
    typename Vec16<T>::type o;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int e = 0; e < W; ++e) o[e] = (T)v[e];
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), buf, at, 0, 0);
  } else if constexpr (sizeof(T) == 2) {
    __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (T)v[0]), buf, at, 0, 0);
  } else {
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v[0]), buf, at, 0, 0);
  }
}

// G lanes hold a row in NP pieces of W elements each; KEEP: the weights stay in registers from row to row.
template <typename T, int G, int NP, int W, bool KEEP, typename AR>
__device__ __forceinline__ void residual_norm_body(const AR &a, const Blk &b, unsigned char *lds) {
  constexpr int RPW = 256 / G;                                // rows of a workgroup at a time
  float *scratch = (float *)lds;                              // [4]
  const int cols = a.cols, col0 = (int)(threadIdx.x % G) * W;
  const float over = 1.0f / (float)cols;
  const bool has_w = a.w != nullptr, has_b = a.b != nullptr, has_g = a.g != nullptr;
  RowPiece<T, W> w[KEEP ? 2 : 1][NP];
  RowPiece<float, W> bias[KEEP ? 2 : 1][NP];
  auto weights = [&](auto which, auto to) {                   // which: 0 of the norm after the block, 1 of the one before the next
    const int64_t skip = decltype(which)::value && a.after ? cols : 0;
    const auto wbuf = row_buffer(has_w ? (const T *)a.w + skip : nullptr, cols);
    const auto bbuf = row_buffer(has_b ? a.b + skip : nullptr, cols);
#pragma unroll
    for (int c = 0; c < NP; ++c) {
      w[decltype(to)::value][c].load(wbuf, col0 + c * G * W);
      bias[decltype(to)::value][c].load(bbuf, col0 + c * G * W);
    }
  };
  typedef std::integral_constant<int, 0> I0;
  typedef std::integral_constant<int, 1> I1;
  typedef std::integral_constant<int, KEEP ? 1 : 0> Last;
  if constexpr (KEEP) {
    if (a.after) weights(I0{}, I0{});
    if (a.before) weights(I1{}, I1{});
  }
  const int step = b.gx * RPW;
  for (int row0 = b.x * RPW + (int)threadIdx.x / G; row0 < a.rows; row0 += step) {   // the same for all lanes of a row
    const int row = __builtin_amdgcn_readfirstlane(row0);
    const int64_t base = (int64_t)row * cols;
    const auto xbuf = row_buffer((const T *)a.x + base, cols);
    const auto rbuf = row_buffer(a.r ? (const T *)a.r + base : nullptr, cols);
    const auto gbuf = row_buffer(has_g ? (const T *)a.g + (int64_t)fast_div((uint32_t)row, (uint32_t)a.gate_rows, a.div_gate) * cols : nullptr, cols);
    RowPiece<T, W> x[NP], r[NP], g[NP];
#pragma unroll
    for (int c = 0; c < NP; ++c) {
      x[c].load(xbuf, col0 + c * G * W);
      r[c].load(rbuf, col0 + c * G * W);
      g[c].load(gbuf, col0 + c * G * W);
    }
    float v[NP][W];
    auto inside = [&](int c) { return col0 + c * G * W < cols; };
    // v -> (v - mean) / sqrt(mean of squares + eps) * w + b; v is zero behind the row
    auto norm = [&](auto which, auto from) {
      if constexpr (!KEEP) weights(which, from);
      if (!a.rms) {
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
          for (int e = 0; e < W; ++e) s += v[c][e];
        const float mean = group_reduce<G, false>(s, scratch) * over;
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
          for (int e = 0; e < W; ++e) v[c][e] = inside(c) ? v[c][e] - mean : 0.f;
      }
      float q = 0.f;
#pragma unroll
      for (int c = 0; c < NP; ++c)
#pragma unroll
        for (int e = 0; e < W; ++e) q += v[c][e] * v[c][e];
      const float k = 1.0f / sqrtf(group_reduce<G, false>(q, scratch) * over + a.eps);
#pragma unroll
      for (int c = 0; c < NP; ++c)
#pragma unroll
        for (int e = 0; e < W; ++e)
          v[c][e] = v[c][e] * k * (has_w ? w[decltype(from)::value][c].at(e) : 1.0f) + bias[decltype(from)::value][c].at(e);
    };
#pragma unroll
    for (int c = 0; c < NP; ++c)
#pragma unroll
      for (int e = 0; e < W; ++e) v[c][e] = x[c].at(e);
    if (a.after) norm(I0{}, I0{});
#pragma unroll
    for (int c = 0; c < NP; ++c)
#pragma unroll
      for (int e = 0; e < W; ++e) v[c][e] = a.beta * (has_g ? v[c][e] * g[c].at(e) : v[c][e]) + a.alpha * r[c].at(e);
    if (a.s) {
      const auto sbuf = row_buffer((T *)a.s + base, cols);
#pragma unroll
      for (int c = 0; c < NP; ++c) store_piece<T, W>(sbuf, col0 + c * G * W, v[c]);
    }
    if (!a.before) continue;
#pragma unroll
    for (int c = 0; c < NP; ++c)
#pragma unroll
      for (int e = 0; e < W; ++e) v[c][e] = inside(c) ? v[c][e] : 0.f;     // 0 * infinity behind the row, if a factor is
    norm(I1{}, Last{});
    const auto ybuf = row_buffer((T *)a.y + base, cols);
#pragma unroll
    for (int c = 0; c < NP; ++c) store_piece<T, W>(ybuf, col0 + c * G * W, v[c]);
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
