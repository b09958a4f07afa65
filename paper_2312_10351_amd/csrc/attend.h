// Attention as an operator of its own (included by kernels.hip): Y = softmax(alpha Q K^T, masked) V,
// one pass over the keys with the running maximum and sum of the softmax; scores never leave registers.
//
// The query heads that share a key and value head are further query rows of it (row = i * share +
// head in the share), so that the keys are read once for all of them.  Scores are formed
// transposed, S^T = K Q^T: a lane then holds one query row and a few keys of it, the maximum and sum
// of a row need two shuffles per tile, and its probabilities already lie where the second product wants them,
// O^T += V^T P^T (both operands number the keys of a step alike, in whatever order).
// Statistics and sums are fp32.  Probabilities are rounded to the element type for the matrix cores:
// relative 2^-11 per term in fp16, as the result's own rounding; their sum is taken before that.
//
// rows kernels: sixteen query rows per workgroup, keys dealt to its four wavefronts in tiles of KT;
// each wavefront has its own ring in workgroup memory and its own maximum, sum and result, which meet at
// the end.  Where there are few query rows the keys of a tile are also shared out between `splits`
// workgroups: each leaves (maximum, sum, result) in scratch memory and the last to arrive joins them in
// a fixed order, so the result does not depend on who that is.

constexpr int attend_stages(int dp) { return dp <= 128 ? 2 : 1; }
constexpr int attend_ring_bytes(int dp) { return attend_stages(dp) * 2 * 64 * dp; }      // of one wavefront
constexpr int lds_attend_rows(int dp) { return 4 * attend_ring_bytes(dp) + 16; }

// What one tile of sixteen query rows sees: keys [0, end), row r its first limit(r).
template <typename AR> struct AttendSight {
  int length, end;
  int64_t ahead;                           // query row i of the sequence sees keys j < i + ahead
  bool causal;
  __device__ __forceinline__ AttendSight(const AR &a, int z, int last_row) {
    length = a.lengths ? min(max(a.lengths[z], 0), a.n) : a.n;
    causal = a.causal != 0;
    ahead = a.causal == 2 ? (int64_t)length - a.m + 1 : (int64_t)a.first + 1;
    end = limit(last_row);
  }
  __device__ __forceinline__ int limit(int i) const {      // i: query row of the sequence
    return causal ? (int)max((int64_t)0, min((int64_t)length, i + ahead)) : length;
  }
};

template <typename T, int DP, bool VEC, typename AR>
__device__ __forceinline__ void attend_rows_body(const AR &a, const Blk &b, unsigned char *lds) {
  typedef typename Vec16<T>::type V;
  typedef V VU __attribute__((aligned(sizeof(T))));
  constexpr int VE = Vec16<T>::N, ES = (int)sizeof(T);
  constexpr int KT = 4 * VE;                                // keys per tile: 32 halves or 16 floats deep
  constexpr int CH = DP * ES / 16;                          // 16-byte chunks per key or value row
  constexpr int L = KT * CH / 64;                           // loads of a wavefront per tile of keys, or of values
  constexpr int S = attend_stages(DP), TILE = KT * DP * ES, RING = attend_ring_bytes(DP);
  constexpr int NS = DP / (4 * VE), NQ = KT / 16, NO = DP / 16, PITCH = DP + 4;
  static_assert(RING == 2 * S * TILE && 16 * PITCH * 4 + 128 <= RING, "ring of a wavefront");
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int grp = lane >> 4, r16 = lane & 15;
  const int tile = (int)fast_div((uint32_t)b.x, (uint32_t)a.splits, a.div_splits), split = b.x - tile * a.splits;
  const int g = b.y, z = b.z;
  const int r0 = tile * 16, rows = a.m * a.share;
  const int r = r0 + r16, qi = (int)fast_div((uint32_t)r, (uint32_t)a.share, a.div_share), head = g * a.share + r - qi * a.share;
  const AttendSight<AR> sight(a, z, (int)fast_div((uint32_t)min(rows - 1, r0 + 15), (uint32_t)a.share, a.div_share));
  const int mine = r < rows ? sight.limit(qi) : 0;          // this lane's query row sees keys [0, mine)
  const int tiles = (sight.end + KT - 1) / KT;
  const int t0 = (int)((int64_t)tiles * split / a.splits), t1 = (int)((int64_t)tiles * (split + 1) / a.splits);
  const int bound = min(sight.end, t1 * KT);                // keys of this workgroup end here

  V qf[NS];                                                 // query row r16, elements (s * 4 + grp) * VE ..
  {
    const T *q = (const T *)a.q + z * a.q_s[0] + qi * a.q_s[1] + head * a.q_s[2];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int d = (s * 4 + grp) * VE;
      V v = {};
      if (r < rows) {
        if (d + VE <= a.width) v = *(const VU *)(q + d);
        else
#pragma unroll
          for (int e = 0; e < VE; ++e)
            if (d + e < a.width) v[e] = q[d + e];
      }
      qf[s] = v;
    }
  }
  const T *kbase = (const T *)a.k + z * a.k_s[0] + g * a.k_s[2], *vbase = (const T *)a.v + z * a.v_s[0] + g * a.v_s[2];
  unsigned char *ring = lds + wave * RING;                  // S tiles of keys, then S tiles of values
  // A row's chunk c lies in slot c ^ (row & 7): fragment reads of adjacent rows then differ in their banks.
  const int lrow = lane / CH, lslot = lane % CH;            // row and slot this lane fills (row + l * 64 / CH)
  constexpr int RL = 64 / CH;                               // rows per load
  static_assert(CH <= 64, "a row fits one load");

  auto stage = [&](const T *base, int64_t pitch, int width, int kt, unsigned char *to) {
    if constexpr (VEC) {
      const i32x4 buf = buffer_of(base + (int64_t)kt * KT * pitch, kOperandMaxBytes);
#pragma unroll
      for (int l = 0; l < L; ++l) {
        const int row = l * RL + lrow, chunk = lslot ^ (row & 7);
        const bool in = kt * KT + row < bound && chunk * VE < width;
        lds_load16(buf, in ? ((uint32_t)row * (uint32_t)pitch + (uint32_t)chunk * VE) * ES : kOperandMaxBytes, 0,
                   lds_address(to) + l * 1024);
      }
    } else {
#pragma unroll
      for (int l = 0; l < L; ++l) {
        const int row = l * RL + lrow, chunk = lslot ^ (row & 7), key = kt * KT + row, d = chunk * VE;
        V v = {};
        if (key < bound) {
          const T *src = base + (int64_t)key * pitch + d;
          if (d + VE <= width) v = *(const VU *)src;
          else
#pragma unroll
            for (int e = 0; e < VE; ++e)
              if (d + e < width) v[e] = src[e];
        }
        *(V *)(to + l * 1024 + lane * 16) = v;
      }
    }
  };
  auto stage_k = [&](int kt, int slot) { stage(kbase, a.k_s[1], a.width, kt, ring + slot * TILE); };
  auto stage_v = [&](int kt, int slot) { stage(vbase, a.v_s[1], a.v_width, kt, ring + (S + slot) * TILE); };

  floatx4 o[NO];
#pragma unroll
  for (int j = 0; j < NO; ++j) o[j] = floatx4{0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, sum = 0.f;
  int kt = t0 + wave;
  // Tiles past the range load nothing (zeros), so that the number of loads in flight never varies.
  if constexpr (VEC) {
    if (kt < t1) {
#pragma unroll
      for (int s = 0; s < S; ++s) { stage_k(kt + s * 4, s); stage_v(kt + s * 4, s); }
    }
  }
  int slot = 0;
#pragma nounroll
  for (; kt < t1; kt += 4) {
    if constexpr (VEC) wait_loads<(2 * S - 1) * L>();
    else stage_k(kt, slot);
    // ---- scores of KT keys
    float p[NQ][4];
    {
      const unsigned char *K = ring + slot * TILE;
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const int row = i * 16 + r16;
          acc = mma16<T>(*(const V *)(K + row * (DP * ES) + (((s * 4 + grp) ^ (row & 7)) * 16)), qf[s], acc);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) p[i][e] = kt * KT + i * 16 + grp * 4 + e < mine ? acc[e] * a.scale : -INFINITY;
      }
    }
    if constexpr (VEC) {
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the slot has been read: it may be refilled
      stage_k(kt + S * 4, slot);
    }
    // ---- running maximum and sum
    float most = top;
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) most = fmaxf(most, p[i][e]);
    most = fmaxf(most, __shfl_xor(most, 16, 64));
    most = fmaxf(most, __shfl_xor(most, 32, 64));
    const float from = most == -INFINITY ? 0.f : most;      // a row that has seen nothing yet
    const float shrink = __builtin_amdgcn_exp2f(top - from);
    top = most;
    sum *= shrink;
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[i][e] = __builtin_amdgcn_exp2f(p[i][e] - from);
        sum += p[i][e];
      }
#pragma unroll
    for (int j = 0; j < NO; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] *= shrink;
    // ---- O^T += V^T P^T; key e of a lane's step: 16 * (e / 4) + 4 * grp + e % 4
    if constexpr (VEC) wait_loads<(2 * S - 1) * L>();
    else stage_v(kt, slot);
    const unsigned char *W = ring + (S + slot) * TILE;
    V pf;
#pragma unroll
    for (int e = 0; e < VE; ++e) pf[e] = (T)p[e / 4][e % 4];
    if constexpr (ES == 2) {
#pragma unroll
      for (int j = 0; j < NO; ++j) {
        half4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = h * 16 + grp * 4 + (r16 >> 2);
          v[h] = lds_read_transposed(W + row * (DP * ES) + (((j * 2 + ((r16 >> 1) & 1)) ^ (row & 7)) * 16) + (r16 & 1) * 8);
        }
        o[j] = mma16<T>(__builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7), pf, o[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < NO; ++j) {
        V v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = grp * 4 + e;
          v[e] = *(const T *)(W + row * (DP * ES) + (((j * 4 + (r16 >> 2)) ^ (row & 7)) * 16) + (r16 & 3) * 4);
        }
        o[j] = mma16<T>(v, pf, o[j]);
      }
    }
    if constexpr (VEC) {
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
      stage_v(kt + S * 4, slot);
    }
    slot = slot == S - 1 ? 0 : slot + 1;
  }

  // ---- the four wavefronts meet
  wait_loads<0>();                                          // no load may outlive its ring
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  float *part = (float *)ring, *stat = part + 16 * PITCH;   // result rows, then maxima and sums
#pragma unroll
  for (int j = 0; j < NO; ++j) *(floatx4 *)(part + r16 * PITCH + j * 16 + grp * 4) = o[j];
  if (grp == 0) { stat[r16] = top; stat[16 + r16] = sum; }
  __syncthreads();
  const int pr = t >> 4, pc = (t & 15) * 4;                 // this thread's row and first column
  const float *wave0 = (const float *)lds;
  constexpr int WF = RING / 4;                              // floats from one wavefront's part to the next
  float share[4], all = -INFINITY, total = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) all = fmaxf(all, wave0[w * WF + 16 * PITCH + pr]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float mw = wave0[w * WF + 16 * PITCH + pr];
    share[w] = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - all);
    total += share[w] * wave0[w * WF + 16 * PITCH + 16 + pr];
  }
  const int row = r0 + pr, yi = (int)fast_div((uint32_t)row, (uint32_t)a.share, a.div_share);
  T *y = (T *)a.y + z * a.y_s[0] + yi * a.y_s[1] + (g * a.share + row - yi * a.share) * a.y_s[2];
  auto joined = [&](int col) {
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const floatx4 x = *(const floatx4 *)(wave0 + w * WF + pr * PITCH + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += share[w] * x[e];
    }
    return v;
  };
  auto store = [&](int col, floatx4 v, float total) {
    typedef typename Run4<T>::type R;
    const float inv = total > 0.f ? 1.0f / total : total == 0.f ? 0.f : total;      // nothing seen: zeros; NaN stays
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= inv;
    if (col + 3 < a.v_width) {
      *(R *)(y + col) = R{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < a.v_width) y[col + e] = (T)v[e];
    }
  };
  if (a.splits == 1) {
    if (row < rows)
#pragma unroll
      for (int c = 0; c < DP; c += 64)
        if (c + pc < a.v_width) store(c + pc, joined(c + pc), total);
    return;
  }

  // ---- the workgroups of a tile meet.  Partial results go past the caches that XCDs do not share
  // (agent-scope stores); a workgroup is counted once its stores have completed, and whoever counts last
  // invalidates its caches and reads them all.  As in the persistent executor this rests on
  // gfx950's behaviour (a store that vmcnt has retired has reached the memory side all XCDs
  // share), not on a release fence, which would write back a whole L2 per workgroup.
  const int64_t tile_id = ((int64_t)z * b.gy + g) * a.tiles + tile;
  float *slot0 = a.partials + tile_id * a.splits * (16 * DP + 32), *mineslot = slot0 + (int64_t)split * (16 * DP + 32);
  if (row < rows) {
#pragma unroll
    for (int c = 0; c < DP; c += 64) {
      const floatx4 v = joined(c + pc);
      stg<true, floatx4>(mineslot + pr * DP + c + pc, v);
    }
    if ((t & 15) == 0) {
      stg<true, float>(mineslot + 16 * DP + pr, all);
      stg<true, float>(mineslot + 16 * DP + 16 + pr, total);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  __syncthreads();
  int *last = (int *)(lds + 4 * RING);
  if (t == 0) {
    uint32_t *count = a.counters + tile_id;
    const bool end = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.splits - 1u;
    if (end) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next launch
    *last = end;
  }
  __syncthreads();
  if (!*last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  if (row >= rows) return;
  float most = -INFINITY;
  for (int s = 0; s < a.splits; ++s) most = fmaxf(most, slot0[(int64_t)s * (16 * DP + 32) + 16 * DP + pr]);
  floatx4 v[DP / 64];
#pragma unroll
  for (int c = 0; c < DP / 64; ++c) v[c] = floatx4{0.f, 0.f, 0.f, 0.f};
  float whole = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const float *from = slot0 + (int64_t)s * (16 * DP + 32);
    const float ms = from[16 * DP + pr], f = ms == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms - most);
    whole += f * from[16 * DP + 16 + pr];
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) {
      const floatx4 x = *(const floatx4 *)(from + pr * DP + c * 64 + pc);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[c][e] += f * x[e];
    }
  }
#pragma unroll
  for (int c = 0; c < DP / 64; ++c)
    if (c * 64 + pc < a.v_width) store(c * 64 + pc, v[c], whole);
}
