// Attention as an operator of its own (included by kernels.hip): Y = softmax(alpha Q K^T, masked) V,
// one pass over the keys with the running maximum and sum of the softmax; scores never leave registers.
//
// The query heads that share a key and value head are further query rows of it (row = i * share +
// head in the share), so that the keys are read once for all of them.  Scores are formed
// transposed, S^T = K Q^T: a lane then holds one query row and a few keys of it, the maximum and sum
// of a row need two lane swaps per tile, and its probabilities already lie where the second product wants them,
// O^T += V^T P^T (both operands number the keys of a step alike, in whatever order).
// Statistics and sums are fp32.  The matrix cores take probabilities of the element type, in fp16 rounded by relative
// 2^-11, while their sum is taken before that.  They are formed 2^kAttendLift times too large, a factor that the sum
// has too: fp16 then keeps all bits of weights down to 2^-25 of a row's largest, and below that multiples of 2^-35 of
// it.  (Without it weights below 2^-25 of the largest were lost, which a tail of 2^16 keys and more shows.)
// What the rounding takes off a probability is an fp16 number too (but for 2^-20 of the probability), and a second
// product adds it where bytes and latencies are the bound, in the rows kernels: a result is then off by its own
// rounding alone (1500 keys, root mean square against 64 bits 2.0e-4, without it 2.7e-4; 12 heads of 64 7.2 -> 7.6 us,
// 65536 keys 55.4 us either way).  In the wide kernel, which the matrix cores bound, it is left out: causal, 8192 rows
// 543 us at 2.5e-4, with it 730 at 1.9e-4.
//
// rows kernels: sixteen query rows per workgroup, keys dealt to its four (deep: eight) wavefronts in tiles of KT;
// each wavefront has its own ring in workgroup memory and its own maximum, sum and result, which meet at
// the end.  Where there are few query rows the keys of a tile are also shared out between `splits`
// workgroups: each leaves (maximum, sum, result) in scratch memory and the last to arrive joins them in
// a fixed order, so the result does not depend on who that is.
// What bounds them: few rows over many keys the keys' bytes (fp16, 32 heads over 8 of 128, 65536 keys, one row:
// 55 us, 4.9 TB/s, a large copy runs at 4.9); few rows over few keys latencies, launch, first loads and
// join (12 heads of 64, 1500 keys: 7.6 us, of which an empty launch takes 2.2); many rows in fp32 the matrix
// cores (32 heads over 8 of 128, causal, 2048 rows: 320 to 329 us, 105 to 107 TFLOP/s, a large matrix product reaches 154).
// Lanes hold whole rows of scores in registers: one wavefront works on a tile for about 1 us, 0.4 of it matrix
// instructions, so that several per SIMD are wanted.

constexpr int attend_ring_bytes(int dp) { return 2 * 64 * dp; }      // of one wavefront: a tile of keys, one of values
constexpr int lds_attend_rows(int dp, int waves) { return waves * attend_ring_bytes(dp); }

// A result is scaled down only when its row's maximum has grown by more than 2^kAttendSlack.  Together the two stay below
// fp16's largest power of two, 2^15.  In fp32 there is no lift: values near its largest would leave its range.  A slack of
// 8 leaves 7 for the lift; for scores of standard deviation 1 (causal, 8192 rows) it costs the same, of 8 it takes 525 us
// against 535.
constexpr float kAttendSlack = 4.f, kAttendLift = 11.f;

// A row's 16-byte chunk c lies in slot c ^ attend_slot(row), so that what one fragment read takes at a time lies in
// different banks, which are 256 bytes wide: of keys one chunk of 16 rows; of values in fp16 (read transposed) two
// chunks of 8 rows, in fp32 four chunks of every fourth row.  (With row & 7 for both, each read took
// twice its time: SQ_LDS_BANK_CONFLICT was 23 % of the busy cycles of the wide kernel.)
template <typename T, int DP, bool VALUES> __device__ __forceinline__ constexpr int attend_slot(int row) {
  if constexpr (!VALUES) return DP * sizeof(T) == 128 ? row >> 1 & 7 : row & 15;
  else if constexpr (sizeof(T) == 4) return (row >> 2 & 3) << 2;
  else return DP == 64 ? (row >> 1 & 3) << 1 : (row & 7) << 1;
}

// L loads of a wavefront bring its share of a tile of KT keys (or values) straight into workgroup memory.  Offsets inside a
// tile are worked out once; a tile is a buffer that begins at its first row and ends with the last key, so
// rows behind that arrive as zeros, and a step costs no vector instruction but the loads.
template <typename T, int DP, int KT, int L, bool VALUES> struct KeyStager {
  static constexpr int ES = (int)sizeof(T), CH = DP * ES / 16, RL = 64 / CH;     // chunks per row, rows per load
  uint32_t off[L], row_bytes;
  const unsigned char *at;
  int64_t step_bytes;
  // share: this wavefront's number among those that fill the tile; the tile after next lies `tiles` further on.
  __device__ __forceinline__ void init(const T *base, int64_t pitch, int width, int share, int first_tile, int tiles, int lane) {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      const int row = (share * L + l) * RL + lane / CH, d = ((lane % CH) ^ attend_slot<T, DP, VALUES>(row)) * (16 / ES);
      off[l] = d < width ? ((uint32_t)row * (uint32_t)pitch + (uint32_t)d) * ES : kOperandMaxBytes;
    }
    row_bytes = (uint32_t)pitch * ES;
    at = (const unsigned char *)(base + (int64_t)first_tile * KT * pitch);
    step_bytes = (int64_t)tiles * KT * pitch * ES;
  }
  // left: keys from the tile's first on
  __device__ __forceinline__ void issue(int left, uint32_t lds) {
    const i32x4 buf = buffer_of(at, (uint32_t)__builtin_amdgcn_readfirstlane(min(max(left, 0), KT)) * row_bytes);
    // The clamp is a vector instruction: five wait states from there to the loads, which take the descriptor from
    // scalar registers inside assembly that the compiler does not look into.
    asm volatile("s_nop 4" : : "s"(buf));
#pragma unroll
    for (int l = 0; l < L; ++l) lds_load16(buf, off[l], 0, lds + l * 1024);
    at += step_bytes;
  }
};

// Over the four lanes that hold a query row: i, i ^ 16, i ^ 32, i ^ 48.  Lane swaps stay in the vector unit; a
// shuffle goes through workgroup memory's crossbar.
template <typename F> __device__ __forceinline__ float over_row(float v, F join) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  v = join(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  const u32x2 b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return join(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}
__device__ __forceinline__ float row_max(float v) { return over_row(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float row_sum(float v) { return over_row(v, [](float a, float b) { return a + b; }); }

// What one tile of sixteen query rows sees: keys [0, end), row r its first limit(r).
template <typename AR> struct AttendSight {
  int length, end;
  int64_t ahead;                           // query row i of the sequence sees keys j < i + ahead
  bool causal;
  __device__ __forceinline__ AttendSight(const AR &a, int z, int last_row) {
    length = __builtin_amdgcn_readfirstlane(a.lengths ? min(max(a.lengths[z], 0), a.n) : a.n);
    causal = a.causal != 0;
    ahead = a.causal == 2 ? (int64_t)length - a.m + 1 : (int64_t)a.first + 1;
    end = __builtin_amdgcn_readfirstlane(limit(last_row));   // in a scalar register: loads take what follows from it at once
  }
  __device__ __forceinline__ int limit(int i) const {      // i: query row of the sequence
    return causal ? (int)max((int64_t)0, min((int64_t)length, i + ahead)) : length;
  }
};

// Which tile, share of its keys, key head and sequence a workgroup takes.  Every XCD takes a contiguous range of
// them: its L2 then holds one head's keys for all tiles of query rows.  The tiles of a head in descending order:
// under a causal mask the later rows have more to do.
template <typename AR>
__device__ __forceinline__ void attend_place(const AR &a, const Blk &b, int &tile, int &split, int &g, int &z) {
  const uint32_t total = (uint32_t)(b.gx * b.gy * a.batch), lin = (uint32_t)b.lin + (uint32_t)(b.gx * b.gy) * (uint32_t)b.z;
  const uint32_t xcd = lin % 8u, r = total % 8u, at = xcd * (total / 8u) + (xcd < r ? xcd : r) + lin / 8u;
  const uint32_t head = at / (uint32_t)b.gx;
  const int x = b.gx - 1 - (int)(at - head * (uint32_t)b.gx);
  z = (int)(head / (uint32_t)b.gy);
  g = (int)(head - (uint32_t)z * (uint32_t)b.gy);
  tile = (int)fast_div((uint32_t)x, (uint32_t)a.splits, a.div_splits);
  split = x - tile * a.splits;
}

// Four result columns of one query row; `scale`: one over the sum of its probabilities.
template <typename T, typename AR>
__device__ __forceinline__ void attend_store(const AR &a, int g, int z, int r, int col, floatx4 v, float scale) {
  typedef typename Run4<T>::type R;
  const int i = (int)fast_div((uint32_t)r, (uint32_t)a.share, a.div_share);
  T *y = (T *)a.y + z * a.y_s[0] + i * a.y_s[1] + (g * a.share + r - i * a.share) * a.y_s[2] + col;
  if (col + 3 < a.v_width) {
    *(R *)y = R{(T)(v[0] * scale), (T)(v[1] * scale), (T)(v[2] * scale), (T)(v[3] * scale)};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < a.v_width) y[e] = (T)(v[e] * scale);
  }
}
// One over a sum of probabilities; a row that has seen nothing gives zeros, NaN stays.
__device__ __forceinline__ float attend_inverse(float sum) { return sum > 0.f ? 1.0f / sum : sum == 0.f ? 0.f : sum; }

// A value row that one query row sees and another does not may hold infinities or NaN; a probability of zero does not
// take them out of a product.  Where a tile has such keys its values are looked over first (once per tile of
// query rows under a causal mask), and only if one is not finite, what is not is added to the rows that see
// it and taken out of the tile.
template <typename T, int BYTES> __device__ __forceinline__ bool any_not_finite(const unsigned char *tile, int lane) {
  constexpr uint32_t VALUE = sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu, STEP = sizeof(T) == 2 ? 0x04000400u : 0x00800000u;
  uint32_t found = 0;
#pragma unroll 4
  for (int l = 0; l < BYTES; l += 1024) {
    const i32x4 w = *(const i32x4 *)(tile + l + lane * 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) found |= ((uint32_t)w[e] & VALUE) + STEP;      // an exponent of ones carries into the sign
  }
  return __any((found & ~VALUE) != 0);
}
// tile: KT values from key `first` on; a lane holds result columns j * 16 + grp * 4 .. + 3, at(j, x), of NX query
// rows that see keys below limit(x).
template <typename T, int DP, int KT, int NX, typename F, typename G>
__device__ __forceinline__ void add_infinite(const unsigned char *tile, int first, int grp, F limit, G at) {
  typedef typename Run4<T>::type R;
  constexpr int ES = (int)sizeof(T);
#pragma nounroll
  for (int key = 0; key < KT; ++key)
#pragma unroll
    for (int j = 0; j < DP / 16; ++j) {
      const int byte = (j * 16 + grp * 4) * ES;
      const R v = *(const R *)(tile + key * (DP * ES) + (((byte >> 4) ^ attend_slot<T, DP, true>(key)) << 4) + (byte & 15));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float f = (float)v[e], add = fabsf(f) < INFINITY ? 0.f : f;
#pragma unroll
        for (int x = 0; x < NX; ++x) at(j, x)[e] += first + key < limit(x) ? add : 0.f;
      }
      __builtin_amdgcn_sched_barrier(0);                     // no registers for what hardly ever runs
    }
}
template <typename T, int BYTES> __device__ __forceinline__ void drop_infinite(unsigned char *part, int lane) {
  typedef typename Vec16<T>::type V;
#pragma nounroll
  for (int l = 0; l < BYTES; l += 1024) {
    V v = *(const V *)(part + l + lane * 16);
#pragma unroll
    for (int e = 0; e < Vec16<T>::N; ++e) v[e] = fabsf((float)v[e]) < INFINITY ? v[e] : (T)0;
    *(V *)(part + l + lane * 16) = v;
  }
  asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
}

// The workgroups that share a tile's keys meet.  Each has left a record of R maxima, R sums and R x DP results in
// `slots` with agent-scope stores, which pass the caches that XCDs do not share; it is counted once its stores have
// completed, and whoever counts last invalidates its caches and joins the records in their order.
// As in the persistent executor this rests on gfx950's behaviour (a store that vmcnt has retired has
// reached the memory side all XCDs share), not on a release fence, which would write back a whole L2 per
// workgroup.  place(q): row and column of the q-th run of four results.  lds: R * splits floats, then 16 bytes per thread.
template <typename T, int DP, int R, int NT, typename AR, typename F>
__device__ __forceinline__ void attend_join(const AR &a, int64_t tile_id, const float *slots, int g, int z, int r0, int runs,
                                            unsigned char *lds, F place) {
  constexpr int REC = R * DP + 2 * R;
  const int t = threadIdx.x, S = a.splits, rows = min(R, a.m * a.share - r0);
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  __syncthreads();
  int *last = (int *)lds;
  if (t == 0) {
    uint32_t *count = a.counters + tile_id;
    const bool end = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)S - 1u;
    if (end) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next launch
    *last = end;
  }
  __syncthreads();
  if (!*last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  __syncthreads();                                           // `last` lies where the factors go
  // ---- what every record counts for in a row: LR lanes share the row's records, eight of each lane are requested at
  // once, and with them, where there are few runs of four results, the first eight that a thread adds up
  constexpr int LR = NT / R;
  static_assert(LR >= 1 && LR <= 64 && (LR & (LR - 1)) == 0, "lanes per row");
  float *factor = (float *)lds;                              // [S][R]
  const bool few = runs <= NT;
  const int parts = runs * 8 <= NT ? 8 : runs * 4 <= NT ? 4 : runs * 2 <= NT ? 2 : 1;      // threads that share a run
  const int q = t % (NT / parts), part = t / (NT / parts);
  const float *from = slots + (int64_t)min(q, runs - 1) * 4;
  floatx4 x[8];
  {
    const int row = t / LR, lane = t % LR;
    const float *stat = slots + R * DP + min(row, rows - 1);
    float m[8], e[8];
    auto request = [&](int s0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float *at = stat + (int64_t)min(s0 + i * LR, S - 1) * REC;
        m[i] = at[0];
        e[i] = at[R];
      }
    };
    request(lane);
    if (few)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *(const floatx4 *)(from + (int64_t)min(part + i * parts, S - 1) * REC);
    float most = -INFINITY, total = 0.f;
    for (int s0 = lane; s0 < S; s0 += 8 * LR) {
      if (s0 != lane) request(s0);
#pragma unroll
      for (int i = 0; i < 8; ++i) most = fmaxf(most, m[i]);  // records past the last repeat it
    }
#pragma unroll
    for (int off = LR / 2; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor(most, off, 64));
    for (int s0 = lane; s0 < S; s0 += 8 * LR) {
      if (S > 8 * LR) request(s0);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (s0 + i * LR >= S) break;
        const float f = m[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[i] - most);
        factor[(s0 + i * LR) * R + row] = f;
        total += f * e[i];
      }
    }
#pragma unroll
    for (int off = LR / 2; off > 0; off >>= 1) total += __shfl_xor(total, off, 64);
    const float inverse = attend_inverse(total);
    for (int s = lane; s < S; s += LR) factor[s * R + row] *= inverse;
  }
  __syncthreads();
  // ---- the sums
  if (few) {
    floatx4 *shared = (floatx4 *)(lds + (((size_t)R * S * 4 + 15) & ~(size_t)15));
    int row, col;
    place(min(q, runs - 1), row, col);
    const bool live = q < runs && row < rows && col < a.v_width;
    row = min(row, rows - 1);
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (part + i * parts < S) v += x[i] * factor[(part + i * parts) * R + row];
    for (int s0 = part + 8 * parts; s0 < S; s0 += 8 * parts) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *(const floatx4 *)(from + (int64_t)min(s0 + i * parts, S - 1) * REC);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s0 + i * parts < S) v += x[i] * factor[(s0 + i * parts) * R + row];
    }
    shared[t] = v;
    __syncthreads();
    if (live && part == 0) {
      for (int i = 1; i < parts; ++i) v += shared[i * (NT / parts) + t];
      attend_store<T>(a, g, z, r0 + row, col, v, 1.0f);
    }
    return;
  }
  for (int q0 = t; q0 < runs; q0 += 8 * NT) {
    int row[8];
    floatx4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int c;
      place(min(q0 + i * NT, runs - 1), row[i], c);
      row[i] = min(row[i], rows - 1);                        // rows behind the last are computed and not stored
      v[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    for (int s = 0; s < S; ++s) {
      const float *record = slots + (int64_t)s * REC;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *(const floatx4 *)(record + (int64_t)min(q0 + i * NT, runs - 1) * 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += x[i] * factor[s * R + row[i]];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int at, c;
      place(min(q0 + i * NT, runs - 1), at, c);
      if (q0 + i * NT < runs && at < rows && c < a.v_width) attend_store<T>(a, g, z, r0 + at, c, v[i], 1.0f);
    }
  }
}

// Two probabilities, cut off to fp16, and what that takes off them.  The rest of one that is not zero is not zero
// either (2^-24 at least, 2^-35 of a row's largest), nor negative: an infinite value times both stays what it is.
__device__ __forceinline__ void split_probabilities(float a, float b, uint32_t *cut, uint32_t *rest) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  const auto c = __builtin_amdgcn_cvt_pkrtz(a, b);
  const auto r = __builtin_amdgcn_cvt_pkrtz(__builtin_fmaf((float)c[0], -1.0f, a), __builtin_fmaf((float)c[1], -1.0f, b));
  u16x2 least;                                              // of each half: the compiler makes comparisons of it
  asm("v_pk_min_u16 %0, %1, %2" : "=v"(least) : "v"(c), "s"(0x00010001));
  *cut = __builtin_bit_cast(uint32_t, c);
  *rest = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, r), least));
}

// NW: wavefronts of a workgroup.  They share its keys without the cost of a join, so that few query rows over some
// hundred keys are best served by as many as workgroup memory holds; longer ones by smaller workgroups, of which
// more run at once.
template <typename T, int DP, bool VEC, int NW, typename AR>
__device__ __forceinline__ void attend_rows_body(const AR &a, const Blk &b, unsigned char *lds) {
  typedef typename Vec16<T>::type V;
  typedef V VU __attribute__((aligned(sizeof(T))));
  constexpr int VE = Vec16<T>::N, ES = (int)sizeof(T);
  constexpr int KT = 4 * VE;                                // keys per tile: 32 halves or 16 floats deep
  constexpr int CH = DP * ES / 16;                          // 16-byte chunks per key or value row
  constexpr int L = KT * CH / 64;                           // loads of a wavefront per tile of keys, or of values
  constexpr int TILE = KT * DP * ES, RING = attend_ring_bytes(DP);
  constexpr int NS = DP / (4 * VE), NQ = KT / 16, NO = DP / 16, PITCH = DP + 4;
  static_assert(RING == 2 * TILE && 16 * PITCH * 4 + 128 <= RING, "ring of a wavefront");
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int grp = lane >> 4, r16 = lane & 15;
  int tile, split, g, z;
  attend_place(a, b, tile, split, g, z);
  const int r0 = tile * 16, rows = a.m * a.share;
  const int r = r0 + r16, qi = (int)fast_div((uint32_t)r, (uint32_t)a.share, a.div_share), head = g * a.share + r - qi * a.share;
  const AttendSight<AR> sight(a, z, (int)fast_div((uint32_t)min(rows - 1, r0 + 15), (uint32_t)a.share, a.div_share));
  const int mine = r < rows ? sight.limit(qi) : 0;          // this lane's query row sees keys [0, mine)
  const int every = sight.limit((int)fast_div((uint32_t)r0, (uint32_t)a.share, a.div_share));      // every row sees these
  const int tiles = (sight.end + KT - 1) / KT;
  // Tiles go round the wavefronts of all workgroups that share them: what is read at a time lies together
  // (65536 keys of 8 heads beside each other: 53.2 us; in runs of tiles 61.1).
  const int first = split * NW + wave, step = NW * a.splits;

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
      qf[s] = v * (T)a.sign;
    }
  }
  const T *kbase = (const T *)a.k + z * a.k_s[0] + g * a.k_s[2], *vbase = (const T *)a.v + z * a.v_s[0] + g * a.v_s[2];
  unsigned char *ring = lds + wave * RING;                  // a tile of keys, a tile of values
  KeyStager<T, DP, KT, L, false> keys;
  KeyStager<T, DP, KT, L, true> values;
  if constexpr (VEC) {
    keys.init(kbase, a.k_s[1], a.width, 0, first, step, lane);
    values.init(vbase, a.v_s[1], a.v_width, 0, first, step, lane);
  }
  // Rows at any address and distance: through registers.
  auto copy = [&](const T *base, int64_t pitch, int width, int kt, unsigned char *to, auto values_tag) {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      const int row = l * (64 / CH) + lane / CH, key = kt * KT + row;
      const int d = ((lane % CH) ^ attend_slot<T, DP, decltype(values_tag)::value>(row)) * VE;
      V v = {};
      if (key < sight.end) {
        const T *src = base + (int64_t)key * pitch + d;
        if (d + VE <= width) v = *(const VU *)src;
        else
#pragma unroll
          for (int e = 0; e < VE; ++e)
            if (d + e < width) v[e] = src[e];
      }
      *(V *)(to + l * 1024 + lane * 16) = v;
    }
  };

  floatx4 o[NO];
#pragma unroll
  for (int j = 0; j < NO; ++j) o[j] = floatx4{0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, sum = 0.f;
  int kt = first;
  // Keys are refilled as soon as they have been read, behind them the values: while one product runs
  // the other's operand is on its way.  (Two slots each hold half the workgroups per CU and measured the same.)  Tiles past
  // the last load nothing (zeros), so that the number of loads in flight never varies.
  if constexpr (VEC) {
    if (kt < tiles) {
      keys.issue(sight.end - kt * KT, lds_address(ring));
      values.issue(sight.end - kt * KT, lds_address(ring) + TILE);
    }
  }
#pragma nounroll
  for (; kt < tiles; kt += step) {
    const int left = sight.end - (kt + step) * KT;          // of the tile after this one
    if constexpr (VEC) wait_loads<L>();
    else copy(kbase, a.k_s[1], a.width, kt, ring, std::false_type{});
    // ---- scores of KT keys
    floatx4 p[NQ];
    {
      const unsigned char *K = ring;
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        floatx4 acc = {0.f, 0.f, 0.f, 0.f}, more[3];           // fp32: four chains, so that no instruction waits for the one before
#pragma unroll
        for (int e = 0; e < 3; ++e) more[e] = acc;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const int row = i * 16 + r16;
          const V kf = *(const V *)(K + row * (DP * ES) + (((s * 4 + grp) ^ attend_slot<T, DP, false>(row)) * 16));
          if constexpr (ES == 2) {
            acc = mma16<T>(kf, qf[s], acc);
          } else {
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[0], qf[s][0], acc, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 3; ++e) more[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e + 1], qf[s][e + 1], more[e], 0, 0, 0);
          }
        }
        if constexpr (ES == 4) acc += (more[0] + more[1]) + more[2];
        p[i] = acc;
      }
    }
    if constexpr (VEC) {
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the slot has been read: it may be refilled
      keys.issue(left, lds_address(ring));
    }
    // ---- running maximum and sum
    if (kt * KT + KT > every)                                 // not for everybody
#pragma unroll
      for (int i = 0; i < NQ; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[i][e] = kt * KT + i * 16 + grp * 4 + e < mine ? p[i][e] : -INFINITY;
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) most = fmaxf(most, p[i][e]);
    most = row_max(most) * a.scale - (ES == 2 ? kAttendLift : 0.f);      // a positive factor
    if (__any(most > top + kAttendSlack)) {
      const float now = fmaxf(most, top), shrink = __builtin_amdgcn_exp2f(top - (now == -INFINITY ? 0.f : now));
      top = now;
      sum *= shrink;
#pragma unroll
      for (int j = 0; j < NO; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] *= shrink;
    }
    const float from = top == -INFINITY ? 0.f : top;        // a row that has seen nothing yet
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[i][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i][e], a.scale, -from));
        sum += p[i][e];
      }
    // ---- O^T += V^T P^T; key e of a lane's step: 16 * (e / 4) + 4 * grp + e % 4
    if constexpr (VEC) wait_loads<L>();
    else copy(vbase, a.v_s[1], a.v_width, kt, ring + TILE, std::true_type{});
    const unsigned char *W = ring + TILE;
    V pf, rest;
#pragma unroll
    for (int e = 0; e < VE; e += 2) {                       // fp32: as they are
      if constexpr (ES == 2) split_probabilities(p[e / 4][e % 4], p[e / 4][e % 4 + 1], (uint32_t *)&pf + e / 2, (uint32_t *)&rest + e / 2);
      else { pf[e] = p[e / 4][e % 4]; pf[e + 1] = p[e / 4][e % 4 + 1]; }
    }
    auto value = [&](int j) {
      if constexpr (ES == 2) {
        half4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = h * 16 + grp * 4 + (r16 >> 2);
          v[h] = lds_read_transposed(W + row * (DP * ES) + (((j * 2 + ((r16 >> 1) & 1)) ^ attend_slot<T, DP, true>(row)) * 16) + (r16 & 1) * 8);
        }
        return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
      } else {
        V v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = grp * 4 + e;
          v[e] = *(const T *)(W + row * (DP * ES) + (((j * 4 + (r16 >> 2)) ^ attend_slot<T, DP, true>(row)) * 16) + (r16 & 3) * 4);
        }
        return v;
      }
    };
    if (every < sight.end && kt * KT + KT > every && any_not_finite<T, TILE>(W, lane)) {
      add_infinite<T, DP, KT, 1>(W, kt * KT, grp, [&](int) { return mine; }, [&](int j, int) -> floatx4 & { return o[j]; });
      drop_infinite<T, TILE>(ring + TILE, lane);
    }
#pragma unroll
    for (int j = 0; j < NO; j += 4) {                       // four results at a time: no instruction waits for the one before
      V v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = value(j + i);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[j + i] = mma16<T>(v[i], pf, o[j + i]);
      if constexpr (ES == 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j + i] = mma16<T>(v[i], rest, o[j + i]);
    }
    if constexpr (VEC) {
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
      values.issue(left, lds_address(ring) + TILE);
    }
  }

  // ---- the wavefronts meet
  wait_loads<0>();                                          // no load may outlive its ring
  sum = row_sum(sum);
  float *part = (float *)ring, *stat = part + 16 * PITCH;   // result rows, then maxima and sums
#pragma unroll
  for (int j = 0; j < NO; ++j) *(floatx4 *)(part + r16 * PITCH + j * 16 + grp * 4) = o[j];
  if (grp == 0) { stat[r16] = top; stat[16 + r16] = sum; }
  __syncthreads();
  constexpr int TR = 4 * NW, RUN = 4 * TR;                  // threads per row, the columns that they take at a time
  const int pr = t / TR, pc = t % TR * 4;                   // this thread's row and first column
  const float *wave0 = (const float *)lds;
  constexpr int WF = RING / 4;                              // floats from one wavefront's part to the next
  float share[NW], all = -INFINITY, total = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) all = fmaxf(all, wave0[w * WF + 16 * PITCH + pr]);
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float mw = wave0[w * WF + 16 * PITCH + pr];
    share[w] = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - all);
    total += share[w] * wave0[w * WF + 16 * PITCH + 16 + pr];
  }
  const int row = r0 + pr;
  auto joined = [&](int col) {
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) v += *(const floatx4 *)(wave0 + w * WF + pr * PITCH + col) * share[w];
    return v;
  };
  if (a.splits == 1) {
    const float inverse = attend_inverse(total);
    if (row < rows)
#pragma unroll
      for (int c = 0; c < DP; c += RUN)
        if (c + pc < a.v_width) attend_store<T>(a, g, z, row, c + pc, joined(c + pc), inverse);
    return;
  }
  const int64_t tile_id = ((int64_t)z * b.gy + g) * a.tiles + tile;
  float *slots = a.partials + tile_id * a.splits * (16 * DP + 32), *mineslot = slots + (int64_t)split * (16 * DP + 32);
  if (row < rows) {
#pragma unroll
    for (int c = 0; c < DP; c += RUN)
      if (RUN <= DP || c + pc < DP) stg<true, floatx4>(mineslot + pr * DP + c + pc, joined(c + pc));
    if (pc == 0) {
      stg<true, float>(mineslot + 16 * DP + pr, all);
      stg<true, float>(mineslot + 16 * DP + 16 + pr, total);
    }
  }
  attend_join<T, DP, 16, 64 * NW>(a, tile_id, slots, g, z, r0, min(16, rows - r0) * (DP / 4), lds, [](int q, int &row, int &col) {
    row = q / (DP / 4);
    col = q % (DP / 4) * 4;
  });
}


// wide kernels, fp16: 32 NW query rows per workgroup, 32 per wavefront, the keys in tiles of 64 that all
// wavefronts share, two of them and their values in workgroup memory.
// What bounds it: per tile and wavefront 64 x 32 x 2 widths of matrix work, about as long in vector instructions (at
// a width of 128; exponentials take a quarter of the rate) and 16 KB of fragment reads each for keys and values; two
// wavefronts per SIMD overlap the three, the one at a product first (s_setprio).  16 x 16 matrix instructions:
// with 32 x 32 ones, which need half as many reductions, the same kernel measured 9 % slower.
// Measured, fp16, 32 heads over 8 of 128, 8192 rows (us): causal 543 among other work (1010 TFLOP/s), 568 to 575
// launched back to back, all keys 1046 (1051; a large matrix product reaches 1350); 16 heads of 64, 4096 rows 88 (779).
// Matrix cores busy 49 % of the compute units' cycles (causal), 256 vector instructions for 64 matrix instructions of
// 16 cycles.
constexpr int lds_attend_wide(int dp) { return 4 * 64 * dp * 2; }

template <int DP, int NW, typename AR>
__device__ __forceinline__ void attend_wide_body(const AR &a, const Blk &b, unsigned char *lds) {
  typedef half_t T;
  typedef half8 V;
  typedef V VU __attribute__((aligned(2)));
  constexpr int KT = 64, TILE = KT * DP * 2;                  // keys per tile, bytes
  constexpr int L = TILE / 1024 / NW;                         // loads of a wavefront per tile
  constexpr int NS = DP / 32, NO = DP / 16;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int grp = lane >> 4, r16 = lane & 15;
  int tile, split, g, z;
  attend_place(a, b, tile, split, g, z);
  const int r0 = tile * (32 * NW), rows = a.m * a.share;
  int r[2], qi[2], mine[2];
  V qf[2][NS];
  const AttendSight<AR> sight(a, z, (int)fast_div((uint32_t)min(rows - 1, r0 + 32 * NW - 1), (uint32_t)a.share, a.div_share));
  const int last = min(rows - 1, r0 + wave * 32 + 31);        // of this wavefront; it sees keys below `reach`
  const int reach = r0 + wave * 32 < rows ? sight.limit((int)fast_div((uint32_t)last, (uint32_t)a.share, a.div_share)) : 0;
  const int all = sight.limit((int)fast_div((uint32_t)r0, (uint32_t)a.share, a.div_share));   // every row of the tile sees these
  const int tiles = (sight.end + KT - 1) / KT, full = all / KT;

#pragma unroll
  for (int x = 0; x < 2; ++x) {
    r[x] = r0 + wave * 32 + x * 16 + r16;
    qi[x] = (int)fast_div((uint32_t)r[x], (uint32_t)a.share, a.div_share);
    mine[x] = r[x] < rows ? sight.limit(qi[x]) : 0;
    const T *q = (const T *)a.q + z * a.q_s[0] + qi[x] * a.q_s[1] + (g * a.share + r[x] - qi[x] * a.share) * a.q_s[2];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int d = s * 32 + grp * 8;
      V v = {};
      if (r[x] < rows) {
        if (d + 8 <= a.width) v = *(const VU *)(q + d);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (d + e < a.width) v[e] = q[d + e];
      }
      qf[x][s] = v * (T)a.sign;
    }
  }
  KeyStager<T, DP, KT, L, false> keys;
  KeyStager<T, DP, KT, L, true> values;
  keys.init((const T *)a.k + z * a.k_s[0] + g * a.k_s[2], a.k_s[1], a.width, wave, split, a.splits, lane);
  values.init((const T *)a.v + z * a.v_s[0] + g * a.v_s[2], a.v_s[1], a.v_width, wave, split, a.splits, lane);
  const uint32_t base = lds_address(lds) + wave * L * 1024;
  floatx4 o[NO][2];
#pragma unroll
  for (int j = 0; j < NO; ++j)
#pragma unroll
    for (int x = 0; x < 2; ++x) o[j][x] = floatx4{0.f, 0.f, 0.f, 0.f};
  float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
  auto issue = [&](int kt, int slot) {                        // in increasing order
    keys.issue(sight.end - kt * KT, base + slot * TILE);
    values.issue(sight.end - kt * KT, base + (2 + slot) * TILE);
  };
  auto scores = [&](floatx4 (&s)[4][2], int slot) {
    const unsigned char *K = lds + slot * TILE;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) s[i][x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < NS; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const V kf = *(const V *)(K + (i * 16 + r16) * (DP * 2) + (((d * 4 + grp) ^ attend_slot<T, DP, false>(r16)) * 16));
#pragma unroll
        for (int x = 0; x < 2; ++x) s[i][x] = mma16<T>(kf, qf[x][d], s[i][x]);
      }
  };
  V p[2][2];                               // [step of 32 keys][query block]
  auto soften = [&](floatx4 (&s)[4][2], int kt, auto masked_tag) {
    constexpr bool MASKED = decltype(masked_tag)::value;
    float most[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      most[x] = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (MASKED) s[i][x][e] = kt * KT + i * 16 + grp * 4 + e < mine[x] ? s[i][x][e] * a.scale : -INFINITY;
          most[x] = fmaxf(most[x], s[i][x][e]);
        }
      if constexpr (!MASKED) most[x] *= a.scale;
      most[x] = row_max(most[x]) - kAttendLift;
    }
    if (__any(most[0] > top[0] + kAttendSlack || most[1] > top[1] + kAttendSlack)) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float now = fmaxf(most[x], top[x]), from = now == -INFINITY ? 0.f : now, shrink = __builtin_amdgcn_exp2f(top[x] - from);
        top[x] = now;
        sum[x] *= shrink;
#pragma unroll
        for (int j = 0; j < NO; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[j][x][e] *= shrink;
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float from = top[x] == -INFINITY ? 0.f : top[x];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = __builtin_amdgcn_exp2f(MASKED ? s[i][x][e] - from : __builtin_fmaf(s[i][x][e], a.scale, -from));
          sum[x] += v;
          p[i / 2][x][i % 2 * 4 + e] = (T)v;
        }
    }
  };
  auto value = [&](int slot, int q, int j) {
    half4 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = q * 32 + h * 16 + grp * 4 + (r16 >> 2), chunk = j * 2 + ((r16 >> 1) & 1);
      v[h] = lds_read_transposed(lds + (2 + slot) * TILE + row * (DP * 2) + ((chunk ^ attend_slot<T, DP, true>(row)) * 16) + (r16 & 1) * 8);
    }
    return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto context = [&](int slot) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int j = 0; j < NO; ++j) {
        const V v = value(slot, q, j);
#pragma unroll
        for (int x = 0; x < 2; ++x) o[j][x] = mma16<T>(v, p[q][x], o[j][x]);
      }
  };
  // All wavefronts come here, and read the tile before any of them changes it.
  auto take_infinite = [&](int slot, int kt) {
    add_infinite<T, DP, KT, 2>(lds + (2 + slot) * TILE, kt * KT, grp, [&](int x) { return mine[x]; },
                               [&](int j, int x) -> floatx4 & { return o[j][x]; });
    __syncthreads();
    drop_infinite<T, TILE / NW>(lds + (2 + slot) * TILE + wave * (TILE / NW), lane);
    __syncthreads();
  };

  if (split < tiles) issue(split, 0);
  int slot = 0;
  auto turn = [&](int kt, auto masked_tag) {
    wait_loads_and_meet<0>();
    const int at = slot;
    slot ^= 1;
    if (kt + a.splits < tiles) issue(kt + a.splits, slot);
    bool apart = false;
    if constexpr (decltype(masked_tag)::value) {
      apart = a.causal && any_not_finite<T, TILE>(lds + (2 + at) * TILE, lane);
      if (kt * KT >= reach) {
        if (apart) take_infinite(at, kt);
        return;
      }
    }
    floatx4 s[4][2];
    __builtin_amdgcn_s_setprio(1);
    scores(s, at);
    __builtin_amdgcn_s_setprio(0);
    soften(s, kt, masked_tag);
    if constexpr (decltype(masked_tag)::value)
      if (apart) take_infinite(at, kt);
    __builtin_amdgcn_s_setprio(1);
    context(at);
    __builtin_amdgcn_s_setprio(0);
  };
  int kt = split;
#pragma nounroll
  for (; kt < full; kt += a.splits) turn(kt, std::integral_constant<bool, false>{});
#pragma nounroll
  for (; kt < tiles; kt += a.splits) turn(kt, std::integral_constant<bool, true>{});

  sum[0] = row_sum(sum[0]);
  sum[1] = row_sum(sum[1]);
  if (a.splits == 1) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float inverse = attend_inverse(sum[x]);
      if (r[x] < rows)
#pragma unroll
        for (int j = 0; j < NO; ++j)
          if (j * 16 + grp * 4 < a.v_width) attend_store<T>(a, g, z, r[x], j * 16 + grp * 4, o[j][x], inverse);
    }
    return;
  }
  // A record keeps the results as the lanes hold them, so that they are written and read in whole lines.
  constexpr int R = 32 * NW, REC = R * DP + 2 * R;
  const int64_t tile_id = ((int64_t)z * b.gy + g) * a.tiles + tile;
  float *slots = a.partials + tile_id * a.splits * REC, *mineslot = slots + (int64_t)split * REC;
#pragma unroll
  for (int j = 0; j < NO; ++j)
#pragma unroll
    for (int x = 0; x < 2; ++x) stg<true, floatx4>(mineslot + ((wave * (NO * 2) + j * 2 + x) * 64 + lane) * 4, o[j][x]);
  if (grp == 0)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      stg<true, float>(mineslot + R * DP + wave * 32 + x * 16 + r16, top[x]);
      stg<true, float>(mineslot + R * DP + R + wave * 32 + x * 16 + r16, sum[x]);
    }
  attend_join<T, DP, R, 64 * NW>(a, tile_id, slots, g, z, r0, R * DP / 4, lds, [](int q, int &row, int &col) {
    const int lane = q & 63, run = (q >> 6) % (NO * 2);
    row = (q >> 6) / (NO * 2) * 32 + (run & 1) * 16 + (lane & 15);
    col = (run >> 1) * 16 + (lane >> 4) * 4;
  });
}
