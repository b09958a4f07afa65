// Rotary positions (included by kernels.hip).
//
// A pair (u, v) of a head is turned by the angle p * f of its row's position and its frequency.
// The frequency is a 64-bit fraction of a turn per position, so the phase is an integer product
// modulo 2^64: exact at any position, where an fp32 angle of position 2^20 would be off by 0.06
// radians.  Only the phase's top bits become floating point.
//
// What bounds it: bytes (every element read and written once), at few rows the launch.  A thread owns
// eight (fp32: four) columns of one row, computes their sines and cosines once and applies them to
// `heads_each` heads, four loads in flight; adjacent threads hold adjacent columns.  Chunks are read at
// element alignment, so odd widths and strides take the same path; a chunk that is not whole
// goes element by element.
// Measured (us): fp16, 32 heads of 128, one row 3.3 (an empty launch: 2.2), 77 rows 3.5, 4096 rows 14.8 (67 MB),
// 16384 rows 62 (268 MB, 4.3 TB/s; a large copy runs at 4.9); fp32, 4096 rows 32 (134 MB, 4.2 TB/s).

// cos and sin of a phase in units of 2^-64 turns.
template <typename T> __device__ __forceinline__ void turn_of(uint64_t phase, float &c, float &s) {
  if constexpr (std::is_same<T, half_t>::value) {
    // The hardware's sine takes turns; its error (2^-20) is far below the fp16 result's.
    const float turns = (float)(int32_t)(phase >> 32) * 0x1p-32f;
    s = __builtin_amdgcn_sinf(turns);
    c = __builtin_amdgcn_cosf(turns);
  } else {
    // The nearest quarter turn is split off as an integer: what is left keeps all its bits in fp32.
    const uint32_t quarter = (uint32_t)((phase + (1ull << 61)) >> 62);
    const int64_t rest = (int64_t)(phase - ((uint64_t)quarter << 62));      // [-2^61, 2^61)
    float s0, c0;
    sincospif((float)(int32_t)(rest >> 30) * 0x1p-33f, &s0, &c0);           // half turns
    s = quarter & 1 ? c0 : s0;
    c = quarter & 1 ? s0 : c0;
    if (quarter & 2) s = -s;
    if ((quarter + 1) & 2) c = -c;
  }
}

template <typename T, typename AR>
__device__ __forceinline__ void rotary_body(const AR &a, const Blk &b, unsigned char *) {
  typedef typename Vec16<T>::type V;
  typedef V VU __attribute__((aligned(sizeof(T))));
  constexpr int VE = Vec16<T>::N, HU = 4;
  const uint32_t item = (uint32_t)b.x * 256u + threadIdx.x;
  if (item >= a.items) return;
  const uint32_t row = fast_div(item, (uint32_t)a.units, a.div_units);
  const int u = (int)(item - row * (uint32_t)a.units);
  const int h0 = b.y * a.heads_each, h1 = min(a.heads, h0 + a.heads_each);
  const uint64_t p = (uint64_t)(a.positions ? (int64_t)a.positions[row] : (int64_t)a.first + (int64_t)row);
  const T *x = (const T *)a.x + (int64_t)row * a.ldx;
  T *y = (T *)a.y + (int64_t)row * a.ldy;
  const int half = a.rotated / 2;
  auto at = [&](int i, float &c, float &s) {
    turn_of<T>(p * a.turns[i], c, s);
    c *= a.amplitude;
    s *= a.amplitude;
  };
  if (!a.interleaved && u < a.rotated_units) {             // columns i0 .. of the first half of the pairs, and their partners
    const int i0 = u * VE, count = min(VE, half - i0);
    float c[VE], s[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) at(min(i0 + e, half - 1), c[e], s[e]);
    if (count == VE) {
      for (int h = h0; h < h1; h += HU) {
        V lo[HU], hi[HU];
#pragma unroll
        for (int q = 0; q < HU; ++q) {
          const T *src = x + (int64_t)min(h + q, h1 - 1) * a.width + i0;
          lo[q] = *(const VU *)src;
          hi[q] = *(const VU *)(src + half);
        }
#pragma unroll
        for (int q = 0; q < HU; ++q) {
          if (h + q >= h1) break;
          V ylo, yhi;
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            ylo[e] = (T)((float)lo[q][e] * c[e] - (float)hi[q][e] * s[e]);
            yhi[e] = (T)((float)hi[q][e] * c[e] + (float)lo[q][e] * s[e]);
          }
          T *dst = y + (int64_t)(h + q) * a.width + i0;
          *(VU *)dst = ylo;
          *(VU *)(dst + half) = yhi;
        }
      }
    } else {
      for (int h = h0; h < h1; ++h) {
        const T *src = x + (int64_t)h * a.width + i0;
        T *dst = y + (int64_t)h * a.width + i0;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          if (e >= count) break;
          const float lo = (float)src[e], hi = (float)src[e + half];
          dst[e] = (T)(lo * c[e] - hi * s[e]);
          dst[e + half] = (T)(hi * c[e] + lo * s[e]);
        }
      }
    }
    return;
  }
  // Interleaved pairs, or columns behind the rotated ones: both stay inside one chunk.  A pair behind
  // the rotated part has angle zero; elements that are copied keep their bits.
  const int o = a.interleaved ? u * VE : a.rotated + (u - a.rotated_units) * VE, count = min(VE, a.width - o);
  float c[VE / 2], s[VE / 2];
#pragma unroll
  for (int e = 0; e < VE / 2; ++e) {
    c[e] = 1.f;
    s[e] = 0.f;
    if (a.interleaved && o / 2 + e < half) at(o / 2 + e, c[e], s[e]);
  }
  auto turned = [&](const T *in, T *out) {
#pragma unroll
    for (int e = 0; e < VE / 2; ++e) {
      const bool moved = a.interleaved && o / 2 + e < half;
      const float lo = (float)in[2 * e], hi = (float)in[2 * e + 1];
      out[2 * e] = moved ? (T)(lo * c[e] - hi * s[e]) : in[2 * e];
      out[2 * e + 1] = moved ? (T)(hi * c[e] + lo * s[e]) : in[2 * e + 1];
    }
  };
  if (count == VE) {
    for (int h = h0; h < h1; h += HU) {
      V in[HU];
#pragma unroll
      for (int q = 0; q < HU; ++q) in[q] = *(const VU *)(x + (int64_t)min(h + q, h1 - 1) * a.width + o);
#pragma unroll
      for (int q = 0; q < HU; ++q) {
        if (h + q >= h1) break;
        V out;
        turned((const T *)&in[q], (T *)&out);
        *(VU *)(y + (int64_t)(h + q) * a.width + o) = out;
      }
    }
  } else {
    for (int h = h0; h < h1; ++h) {
      T in[VE], out[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) in[e] = e < count ? x[(int64_t)h * a.width + o + e] : (T)0.f;
      turned(in, out);
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (e < count) y[(int64_t)h * a.width + o + e] = out[e];
    }
  }
}
