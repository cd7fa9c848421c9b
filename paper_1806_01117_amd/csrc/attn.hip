// Attention whose state decays, in chunks of 64 tokens on the matrix cores.
//
// With lambda^(i-j) between the tokens of a chunk and the state S before it,
//   o_i = sum_{j <= i} lambda^(i-j) (q_i . k_j) v_j + lambda^(i+1) S^T q_i,
//   S' = lambda^m S + sum_j lambda^(m-1-j) k_j v_j^T      (m tokens in the chunk),
// so a chunk is four products and the state passes from chunk to chunk.  The
// gradients are the same recurrence on other operands:
//   dq: do for q, v for k, k for v and S^T for S, forwards;
//   dv: k for q, q for k, do for v; dk: v for q, do for k, q for v; both
//   backwards over the gradient D of the state, with D_{i-1} = lambda A_i.
//
// A long sequence of few heads is cut into segments: a first launch forms each
// segment's own contribution to the state, a second one passes the states from
// segment to segment, and the segments then run side by side.
//
// Rounding.  States, accumulators and sums are fp32, and bf16 operands enter
// the matrix cores as they are.  The fp32 values that go there in the bf16
// kernels are split in bf16 parts: the weighted products lambda^(i-j) (q_i . k_j)
// and the copy of the state that multiplies q in two (16 bits; with one part
// each a result was 1.35 times as far off as its own rounding to bf16 makes
// it), the weighted rows lambda^(m-1-j) k_j, which go into the fp32 state, in
// three (24 bits).
#include "mfma.hpp"
#include "ops.hpp"

namespace ambptt {

namespace {

constexpr int kC = 64;    // tokens per chunk: 16 rows for each of 4 pairs of waves
constexpr int kPad = 16;  // bytes between rows in LDS: 16 rows start in different banks

// Eight waves: wave w has the rows of w % 4, and of the state and the results
// the half w / 4 (backwards: dv or dk), so that its accumulators and fragments
// fit in 256 registers and two waves share a SIMD.
constexpr int kThreads = 512, kSets = 2;

typedef unsigned int u4v __attribute__((ext_vector_type(4)));
typedef unsigned int u2v __attribute__((ext_vector_type(2)));
typedef u4v u4u __attribute__((aligned(2)));  // 16 bytes at any element's address
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// lambda^n
__device__ __forceinline__ float power(float log_decay, int n) { return n == 0 ? 1.0f : expf(float(n) * log_decay); }

__device__ __forceinline__ unsigned pk_bf16(float a, float b) {
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f2{a, b}, bf16x2));
}
__device__ __forceinline__ float lo_f(unsigned p) { return __builtin_bit_cast(float, p << 16); }
__device__ __forceinline__ float hi_f(unsigned p) { return __builtin_bit_cast(float, p & 0xffff0000u); }

// Fragments of 16 x 16 tiles.  A lane l of a wave stands for row (or column)
// l % 16 and for the group l / 16 of the reduction's indices.
//
// Row fragments hold 16 consecutive bytes of a row, group after group: a unit
// of the reduction is 64 bytes of a row.  Token fragments reduce over rows of a
// tile in LDS: a unit is kTiles tiles of 16 rows, and slot (tile, r) of group g
// is row 16 tile + 4 g + r, which is where a product's accumulators lie, so
// that the weighted products are operands of the next product as they stand.
template <class T>
struct Mm;

template <>
struct Mm<__bf16> {
  typedef bf16x8 Frag;
  static constexpr int kTiles = 2, kParts = 3, kHalves = 2;
  static __device__ __forceinline__ f4 mul(const Frag& a, const Frag& b, f4 c) { return mfma_bf16_16x16x32(a, b, c); }
  // column of lane n in tile t: two tiles share 32 columns so that a lane's
  // accumulators of both are 8 neighbours (16 bytes to store)
  static __device__ __forceinline__ int column(int t, int n) { return 32 * (t / 2) + 8 * (n / 4) + 4 * (t % 2) + n % 4; }
  // token fragment of unit u for the columns that `lane` points at (token_lane)
  static __device__ __forceinline__ Frag token(const char* lane, int ld, int u) {
    typedef __attribute__((address_space(3))) bf16x4* Lds;
    const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((Lds)(lane + 32 * u * ld));
    const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((Lds)(lane + (32 * u + 16) * ld));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  // a lane's address for token(): 16 lanes read 4 rows of 16 columns, 4 columns
  // each, and get them transposed
  static __device__ __forceinline__ const char* token_lane(const char* tile, int ld, int l) {
    return tile + (4 * (l / 16) + l % 16 / 4) * ld;
  }
  static __device__ __forceinline__ int token_col(int t, int l) { return 2 * (32 * (t / 2) + 8 * (l % 4) + 4 * (t % 2)); }
  static __device__ __forceinline__ int token_plain_col(int t, int l) { return 2 * (16 * t + 4 * (l % 4)); }
  // accumulators of kTiles tiles as token fragments, in kHalves parts
  static __device__ __forceinline__ void pack(const f4 (&p)[2], Frag (&out)[2]) {
    u4v a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = p[i / 2][i % 2 * 2], y = p[i / 2][i % 2 * 2 + 1];
      a[i] = pk_bf16(x, y);
      b[i] = pk_bf16(x - lo_f(a[i]), y - hi_f(a[i]));
    }
    out[0] = __builtin_bit_cast(Frag, a), out[1] = __builtin_bit_cast(Frag, b);
  }
  // x times the weights, in kParts parts whose sum is exact to 24 bits
  static __device__ __forceinline__ void split(const Frag& x, const float (&w)[8], Frag (&out)[kParts]) {
    const u4v v = __builtin_bit_cast(u4v, x);
    u4v o[kParts];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = lo_f(v[i]) * w[2 * i], b = hi_f(v[i]) * w[2 * i + 1];
#pragma unroll
      for (int p = 0; p < kParts; ++p) {
        const unsigned q = pk_bf16(a, b);
        o[p][i] = q;
        a -= lo_f(q), b -= hi_f(q);
      }
    }
#pragma unroll
    for (int p = 0; p < kParts; ++p) out[p] = __builtin_bit_cast(Frag, o[p]);
  }
  // four accumulators as elements, their parts `apart` bytes from each other
  static __device__ __forceinline__ void put4(char* p, int apart, const f4& v) {
    const u2v a = {pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
    *(u2v*)p = a;
    *(u2v*)(p + apart) = u2v{pk_bf16(v[0] - lo_f(a[0]), v[1] - hi_f(a[0])), pk_bf16(v[2] - lo_f(a[1]), v[3] - hi_f(a[1]))};
  }
};

template <>
struct Mm<float> {
  typedef f4 Frag;
  static constexpr int kTiles = 1, kParts = 1, kHalves = 1;
  static __device__ __forceinline__ f4 mul(const Frag& a, const Frag& b, f4 c) {
#pragma unroll
    for (int r = 0; r < 4; ++r) c = mfma_f32_16x16x4(a[r], b[r], c);
    asm volatile("" ::: "memory");  // loads stay where they are: hoisted, they would spill
    return c;
  }
  static __device__ __forceinline__ int column(int t, int n) { return 16 * t + n; }
  static __device__ __forceinline__ Frag token(const char* lane, int ld, int u) {
    f4 v;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = *(const float*)(lane + (16 * u + r) * ld);
    return v;
  }
  static __device__ __forceinline__ const char* token_lane(const char* tile, int ld, int l) { return tile + 4 * (l / 16) * ld; }
  static __device__ __forceinline__ int token_col(int t, int l) { return 4 * (16 * t + l % 16); }
  static __device__ __forceinline__ int token_plain_col(int t, int l) { return 4 * (16 * t + l % 16); }
  static __device__ __forceinline__ void pack(const f4 (&p)[1], Frag (&out)[1]) { out[0] = p[0]; }
  static __device__ __forceinline__ void split(const Frag& x, const float (&w)[4], Frag (&out)[1]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) out[0][r] = x[r] * w[r];
  }
  static __device__ __forceinline__ void put4(char* p, int, const f4& v) { *(f4*)p = v; }
};

// 64 rows of NX elements on their way from memory to LDS
template <class T, int NX>
constexpr int tile_ld = NX* int(sizeof(T)) + kPad;  // bytes of a row in LDS

template <class T, int NX>
struct Stage {
  static constexpr int kLd = tile_ld<T, NX>;
  static constexpr int kLanes = NX * int(sizeof(T)) / 16;  // lanes per row
  static constexpr int kPer = kThreads / kLanes;           // rows per load
  static constexpr int kLoads = kC / kPer;
  u4v v[kLoads];
  // rows 0 .. m - 1 at p with the row stride `step` (elements), nx of their NX columns; the rest are zeros
  __device__ __forceinline__ void load(const T* p, int64_t step, int m, int nx) {
    const int row = threadIdx.x / kLanes, col = threadIdx.x % kLanes * (16 / int(sizeof(T)));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = row + i * kPer;
      v[i] = r < m && col < nx ? *(const u4u*)(p + r * step + col) : u4v{0, 0, 0, 0};
    }
  }
  __device__ __forceinline__ void put(char* lds) const {
    const int row = threadIdx.x / kLanes, at = threadIdx.x % kLanes * 16;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *(u4v*)(lds + (row + i * kPer) * kLd + at) = v[i];
  }
};

// row fragments of one row (zeros for a row that is not there)
template <class T, int NX>
struct RowFrags {
  static constexpr int kUnits = NX * int(sizeof(T)) / 64;
  typename Mm<T>::Frag f[kUnits];
  __device__ __forceinline__ void load(const T* row, bool there, int nx) {
    const int g = threadIdx.x % 64 / 16;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int col = (u * 64 + g * 16) / int(sizeof(T));
      const u4v v = there && col < nx ? *(const u4u*)(row + col) : u4v{0, 0, 0, 0};
      f[u] = __builtin_bit_cast(typename Mm<T>::Frag, v);
    }
  }
};

struct ChunkArgs {
  View c, u, w, out;        // rows that multiply the state, its updates u w^T, results
  View c2, out2;            // backwards: the rows v and results dk beside k and dv
  int G, na, nb, H, nseg;   // na rows and nb columns of the state
  int64_t T, L;             // tokens per segment, a multiple of kC
  float scale;
  const float* log_decay;
  const int32_t* lengths;
  const float* s0;          // [B][H][nseg][dk dv] states at the segments' starts (backwards: gradients at their ends), NULL = zeros
  float* sn;                // the same of the segments' other ends, or NULL
  int sr, sc;               // element strides of the state's rows and columns
};

struct Where {
  int b, h, seg;
  int64_t t0, t1, end;  // the segment's tokens t0 .. t1 - 1, of which those before `end` count
};

__device__ __forceinline__ Where where(const ChunkArgs& a) {
  Where x;
  const int id = blockIdx.x;
  x.seg = id % a.nseg;
  x.h = id / a.nseg % a.H;
  x.b = id / a.nseg / a.H;
  x.t0 = x.seg * a.L;
  x.t1 = min(x.t0 + a.L, a.T);
  int64_t n = a.T;
  if (a.lengths) n = min(max(int64_t(a.lengths[x.b]), int64_t(0)), a.T);
  x.end = min(n, x.t1);
  return x;
}

template <class T>
__device__ __forceinline__ T* at(const View& v, int b, int64_t t, int h) {
  return static_cast<T*>(v.p) + b * v.batch + t * v.step + h * v.head;
}

// Columns t0 .. of NT tiles of results, times f: eight (bf16) or four (fp32) per lane
template <class T, int NT, int NO>
__device__ __forceinline__ void store_row(T* row, int t0, const f4 (&o)[NO], float f, bool zero, int n) {
  const int g = threadIdx.x % 64 / 16;
#pragma unroll
  for (int t = 0; t < NT; t += Mm<T>::kTiles) {
    u4v v;
    int col = 16 * (t0 + t);
    if constexpr (sizeof(T) == 2) {
      v = u4v{pk_bf16(o[t][0] * f, o[t][1] * f), pk_bf16(o[t][2] * f, o[t][3] * f), pk_bf16(o[t + 1][0] * f, o[t + 1][1] * f),
              pk_bf16(o[t + 1][2] * f, o[t + 1][3] * f)};
      col += 8 * g;
    } else {
      v = __builtin_bit_cast(u4v, f4{o[t][0] * f, o[t][1] * f, o[t][2] * f, o[t][3] * f});
      col += 4 * g;
    }
    if (zero) v = u4v{0, 0, 0, 0};
    if (col < n) *(u4u*)(row + col) = v;
  }
}

// zeros for the results of tokens t .. t1 - 1
template <class T, int NX>
__device__ __forceinline__ void zero_rows(const View& out, int b, int h0, int heads, int64_t t, int64_t t1, int n) {
  constexpr int lanes = NX * int(sizeof(T)) / 16;
  const int col = threadIdx.x % lanes * (16 / int(sizeof(T)));
  for (int64_t r = t + threadIdx.x / lanes; r < t1; r += kThreads / lanes)
    if (col < n)
      for (int g = 0; g < heads; ++g) *(u4u*)(at<T>(out, b, r, h0 + g) + col) = u4v{0, 0, 0, 0};
}

// The state of one segment in the accumulators of a workgroup's waves: wave w
// holds the rows 16 MT (w % 4) .. and the tiles NT (w / 4) .. of columns.
template <class T, int NA, int NB>
struct State {
  static constexpr int MT = NA / 64, NT = NB / 16 / kSets;
  static constexpr int kLd = tile_ld<T, NA>, kPart = NB * kLd;  // of the copy in LDS
  f4 s[MT][NT];

  __device__ __forceinline__ int tile(int t) const { return threadIdx.x / 256 * NT + t; }
  __device__ __forceinline__ int row_tile(int mt) const { return threadIdx.x / 64 % 4 * MT + mt; }
  __device__ __forceinline__ int row(int mt) const { return row_tile(mt) * 16 + threadIdx.x % 64 / 16 * 4; }
  __device__ __forceinline__ int column(int t) const { return Mm<T>::column(tile(t), threadIdx.x % 16); }

  __device__ __forceinline__ void load(const float* p, const ChunkArgs& a) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          s[mt][t][r] = p && row(mt) + r < a.na && column(t) < a.nb ? p[(row(mt) + r) * a.sr + column(t) * a.sc] : 0.0f;
  }
  __device__ __forceinline__ void store(float* p, const ChunkArgs& a) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (row(mt) + r < a.na && column(t) < a.nb) p[(row(mt) + r) * a.sr + column(t) * a.sc] = s[mt][t][r];
  }
  // the transposed copy that multiplies rows, in kHalves parts: line 16 t + n holds column(t, n)
  __device__ __forceinline__ void put(char* lds) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        Mm<T>::put4(lds + (16 * tile(t) + threadIdx.x % 16) * kLd + row(mt) * int(sizeof(T)), kPart, s[mt][t]);
  }
  // s = f s + sum over the chunk's rows of weight u w^T; weight(tile, r) is that of row 16 tile + 4 g + r
  template <class Weight>
  __device__ __forceinline__ void update(float f, const char* u, const char* w, Weight weight) {
    constexpr int lu = tile_ld<T, NA>, lw = tile_ld<T, NB>, tiles = Mm<T>::kTiles, units = kC / (16 * tiles);
    const int l = threadIdx.x % 64;
    typename Mm<T>::Frag a[MT][units][Mm<T>::kParts];
#pragma unroll
    for (int i = 0; i < units; ++i) {
      float by[4 * tiles];
#pragma unroll
      for (int k = 0; k < 4 * tiles; ++k) by[k] = weight(tiles * i + k / 4, k % 4);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const char* p = Mm<T>::token_lane(u, lu, l) + Mm<T>::token_plain_col(row_tile(mt), l);
        Mm<T>::split(Mm<T>::token(p, lu, i), by, a[mt][i]);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      typename Mm<T>::Frag b[units];
#pragma unroll
      for (int i = 0; i < units; ++i) b[i] = Mm<T>::token(Mm<T>::token_lane(w, lw, l) + Mm<T>::token_col(tile(t), l), lw, i);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        f4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < units; ++i)
#pragma unroll
          for (int p = Mm<T>::kParts - 1; p >= 0; --p) sum = Mm<T>::mul(a[mt][i][p], b[i], sum);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[mt][t][r] = fmaf(f, s[mt][t][r], sum[r]);
      }
    }
  }
};

// acc[t] = f times lines 16 (t0 + t) .. of the state's copy times a row's fragments
template <class T, int NA, int NB, int NT, int NO, int NC>
__device__ __forceinline__ void times_state(f4 (&acc)[NO], int t0, const char* copy, const RowFrags<T, NC>& c, float f) {
  constexpr int ld = State<T, NA, NB>::kLd, part = State<T, NA, NB>::kPart, units = RowFrags<T, NA>::kUnits;
  const char* p = copy + (16 * t0 + threadIdx.x % 16) * ld + threadIdx.x % 64 / 16 * 16;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    typename Mm<T>::Frag a[Mm<T>::kHalves][units];
#pragma unroll
    for (int h = 0; h < Mm<T>::kHalves; ++h)
#pragma unroll
      for (int u = 0; u < units; ++u) a[h][u] = *(const typename Mm<T>::Frag*)(p + h * part + 16 * t * ld + 64 * u);
    f4 v = {0, 0, 0, 0};
#pragma unroll
    for (int h = Mm<T>::kHalves - 1; h >= 0; --h)
#pragma unroll
      for (int u = 0; u < units; ++u) v = Mm<T>::mul(a[h][u], c.f[u], v);
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[t][r] = v[r] * f;
  }
}

// acc[t] = f times columns of the state's copy's lines (rows of the state) times a row's fragments
template <class T, int NA, int NB, int NO, int NC>
__device__ __forceinline__ void times_state_back(f4 (&acc)[NO], const char* copy, const RowFrags<T, NC>& c, float f) {
  constexpr int ld = State<T, NA, NB>::kLd, part = State<T, NA, NB>::kPart, units = RowFrags<T, NB>::kUnits;
  const int l = threadIdx.x % 64;
  const char* p = Mm<T>::token_lane(copy, ld, l);
#pragma unroll
  for (int t = 0; t < NA / 16; ++t) {
    typename Mm<T>::Frag a[Mm<T>::kHalves][units];
#pragma unroll
    for (int h = 0; h < Mm<T>::kHalves; ++h)
#pragma unroll
      for (int u = 0; u < units; ++u) a[h][u] = Mm<T>::token(p + h * part + Mm<T>::token_col(t, l), ld, u);
    f4 v = {0, 0, 0, 0};
#pragma unroll
    for (int h = Mm<T>::kHalves - 1; h >= 0; --h)
#pragma unroll
      for (int u = 0; u < units; ++u) v = Mm<T>::mul(a[h][u], c.f[u], v);
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[t][r] = v[r] * f;
  }
}

// the products of 16 rows of a tile in LDS with a row's fragments: row 4 g + r in p[r]
template <class T, int NX, int NC>
__device__ __forceinline__ f4 dots(const char* tile, int jt, const RowFrags<T, NC>& c) {
  constexpr int ld = tile_ld<T, NX>, units = RowFrags<T, NX>::kUnits;
  const char* p = tile + (16 * jt + threadIdx.x % 16) * ld + threadIdx.x % 64 / 16 * 16;
  typename Mm<T>::Frag a[units];
  f4 v = {0, 0, 0, 0};
#pragma unroll
  for (int u = 0; u < units; ++u) a[u] = *(const typename Mm<T>::Frag*)(p + 64 * u);
#pragma unroll
  for (int u = 0; u < units; ++u) v = Mm<T>::mul(a[u], c.f[u], v);
  return v;
}

// acc[t] += tiles t0 + t of a transposed tile of 64 rows times weighted products
template <class T, int NX, int NT, int NO>
__device__ __forceinline__ void times_tile(f4 (&acc)[NO], int t0, const char* tile, int unit,
                                           const typename Mm<T>::Frag (&p)[Mm<T>::kHalves]) {
  constexpr int ld = tile_ld<T, NX>;
  const int l = threadIdx.x % 64;
  const char* q = Mm<T>::token_lane(tile, ld, l);
  typename Mm<T>::Frag a[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) a[t] = Mm<T>::token(q + Mm<T>::token_col(t0 + t, l), ld, unit);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int h = Mm<T>::kHalves - 1; h >= 0; --h) acc[t] = Mm<T>::mul(a[t], p[h], acc[t]);
}

template <class T, int NA, int NB>
constexpr int chunk_lds() {
  return kC * (tile_ld<T, NA> + tile_ld<T, NB>)+Mm<T>::kHalves * State<T, NA, NB>::kPart;
}

// Forwards: results of a segment's tokens (OUT), or the state that the segment
// alone leaves.
template <class T, int NA, int NB, bool OUT>
__global__ __launch_bounds__(kThreads, 2) void forwards(ChunkArgs a) {
  extern __shared__ __align__(16) char lds[];
  constexpr int units = kC / (16 * Mm<T>::kTiles), NT = NB / 16 / kSets;
  char* const ut = lds;
  char* const wt = ut + kC * tile_ld<T, NA>;
  char* const copy = wt + kC * tile_ld<T, NB>;
  const Where x = where(a);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % 4, n = threadIdx.x % 16, g = threadIdx.x % 64 / 16;
  const float ld = a.log_decay[x.h];
  const int64_t state = (int64_t(x.b) * a.H + x.h) * a.nseg + x.seg;

  State<T, NA, NB> S;
  S.load(OUT && a.s0 ? a.s0 + state * a.na * a.nb : nullptr, a);
  const float whole = power(ld, kC);
  // lambda^(i-j) for this lane's row i = 16 wave + n and j = 16 jt + 4 g + r:
  // far[wave - jt] near[r] below the diagonal tile, both with exponents >= 0
  float diag[4], near[4], far[4], after[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    diag[r] = n >= 4 * g + r ? power(ld, n - 4 * g - r) : 0.0f;
    near[r] = power(ld, 15 - 4 * g - r);
    far[r] = power(ld, r ? 16 * r + n - 15 : 0);
    after[r] = power(ld, kC - 16 - 16 * r);
  }
  const float own = power(ld, 16 * wave + n + 1);

  Stage<T, NA> su;
  Stage<T, NB> sw;
  RowFrags<T, NA> c, next;
  const int i = 16 * wave + n;
  auto fetch = [&](int64_t t) {
    const int m = int(min(int64_t(kC), x.end - t));
    su.load(at<T>(a.u, x.b, t, x.h), a.u.step, m, a.na);
    sw.load(at<T>(a.w, x.b, t, x.h), a.w.step, m, a.nb);
  };
  auto fetch_row = [&](int64_t t, int q) { next.load(at<T>(a.c, x.b, t + i, x.h * a.G + q), t + i < x.end, a.na); };
  if (x.t0 < x.end) {
    fetch(x.t0);
    if (OUT) fetch_row(x.t0, 0);
  }
  int64_t t = x.t0;
  for (; t < x.end; t += kC) {
    const int m = int(min(int64_t(kC), x.end - t)), rows = int(min(int64_t(kC), x.t1 - t));
    su.put(ut), sw.put(wt);
    if (OUT) S.put(copy);
    __syncthreads();
    if (t + kC < x.end) fetch(t + kC);
    if (OUT) {
      for (int q = 0; q < a.G; ++q) {
        c = next;
        if (q + 1 < a.G)
          fetch_row(t, q + 1);
        else if (t + kC < x.end)
          fetch_row(t + kC, 0);
        f4 o[NT];
        times_state<T, NA, NB, NT>(o, S.tile(0), copy, c, own);
#pragma unroll
        for (int u = 0; u < units; ++u) {
          if (u * Mm<T>::kTiles > wave) continue;
          f4 p[Mm<T>::kTiles];
#pragma unroll
          for (int k = 0; k < Mm<T>::kTiles; ++k) {
            const int jt = u * Mm<T>::kTiles + k;
            p[k] = f4{0, 0, 0, 0};
            if (jt > wave) continue;
            const f4 v = dots<T, NA>(ut, jt, c);
            const float f = wave - jt == 1 ? far[1] : wave - jt == 2 ? far[2] : far[3];
#pragma unroll
            for (int r = 0; r < 4; ++r)
              p[k][r] = jt == wave ? (n >= 4 * g + r ? v[r] * diag[r] : 0.0f) : v[r] * (f * near[r]);
          }
          typename Mm<T>::Frag pf[Mm<T>::kHalves];
          Mm<T>::pack(p, pf);
          times_tile<T, NB, NT>(o, S.tile(0), wt, u, pf);
        }
        if (i < rows) store_row<T, NT>(at<T>(a.out, x.b, t + i, x.h * a.G + q), S.tile(0), o, a.scale, i >= m, a.nb);
      }
    }
    if (m == kC)
      S.update(whole, ut, wt, [&](int tile, int r) { return after[tile] * near[r]; });
    else
      S.update(power(ld, m), ut, wt, [&](int tile, int r) { return power(ld, max(0, m - 1 - 16 * tile - 4 * g - r)); });
    __syncthreads();
  }
  if (OUT) zero_rows<T, NB>(a.out, x.b, x.h * a.G, a.G, t, x.t1, a.nb);
  if (a.sn) S.store(a.sn + state * a.na * a.nb, a);
}

// One side of a chunk's gradients: o = (scale lambda^(i-j) (rows i of `left` . c))
// summed over the rows of `right`, the rows i >= j of this lane's row j.
template <class T, int NL, int NR, int NO, int NC>
__device__ __forceinline__ void later_rows(f4 (&o)[NO], const char* left, const char* right, const RowFrags<T, NC>& c,
                                           int wave, const float (&diag)[4], const float (&near)[4], const float (&far)[4]) {
  constexpr int units = kC / (16 * Mm<T>::kTiles);
  const int n = threadIdx.x % 16, g = threadIdx.x % 64 / 16;
#pragma unroll
  for (int u = 0; u < units; ++u) {
    if (u * Mm<T>::kTiles + Mm<T>::kTiles - 1 < wave) continue;
    f4 p[Mm<T>::kTiles];
#pragma unroll
    for (int k = 0; k < Mm<T>::kTiles; ++k) {
      const int it = u * Mm<T>::kTiles + k;
      p[k] = f4{0, 0, 0, 0};
      if (it < wave) continue;
      const f4 v = dots<T, NL>(left, it, c);
      const float f = it - wave == 1 ? far[1] : it - wave == 2 ? far[2] : far[3];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        p[k][r] = it == wave ? (4 * g + r >= n ? v[r] * diag[r] : 0.0f) : v[r] * (f * near[r]);
    }
    typename Mm<T>::Frag pf[Mm<T>::kHalves];
    Mm<T>::pack(p, pf);
    times_tile<T, NR, NR / 16>(o, 0, right, u, pf);
  }
}

// Backwards: u = q and w = do of G heads, c = k, c2 = v; out = dv, out2 = dk
// (OUT), or the gradient that the segment alone leaves at its start.  The first
// four waves form dv and the others dk.
template <class T, int NA, int NB, bool OUT>
__global__ __launch_bounds__(kThreads, 2) void backwards(ChunkArgs a) {
  extern __shared__ __align__(16) char lds[];
  constexpr int NX = NA > NB ? NA : NB;
  char* const ut = lds;
  char* const wt = ut + kC * tile_ld<T, NA>;
  char* const copy = wt + kC * tile_ld<T, NB>;
  const Where x = where(a);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % 4, n = threadIdx.x % 16, g = threadIdx.x % 64 / 16;
  const bool first = __builtin_amdgcn_readfirstlane(threadIdx.x / 256) == 0;
  const float ld = a.log_decay[x.h];
  const int64_t state = (int64_t(x.b) * a.H + x.h) * a.nseg + x.seg;

  State<T, NA, NB> D;
  D.load(OUT && a.s0 ? a.s0 + state * a.na * a.nb : nullptr, a);
  // lambda^(i-j) scale for this lane's row j = 16 wave + n and i = 16 it + 4 g + r
  float diag[4], near[4], far[4], after[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    diag[r] = 4 * g + r >= n ? a.scale * power(ld, 4 * g + r - n) : 0.0f;
    near[r] = a.scale * power(ld, 4 * g + r);
    far[r] = power(ld, r ? 16 * r - n : 0);
    after[r] = power(ld, 16 * r + 1);
  }

  Stage<T, NA> su;
  Stage<T, NB> sw;
  RowFrags<T, NX> c, next;
  const int j = 16 * wave + n;
  auto fetch = [&](int64_t t, int q) {
    const int m = int(min(int64_t(kC), x.end - t));
    su.load(at<T>(a.u, x.b, t, x.h * a.G + q), a.u.step, m, a.na);
    sw.load(at<T>(a.w, x.b, t, x.h * a.G + q), a.w.step, m, a.nb);
  };
  auto fetch_rows = [&](int64_t t) {
    next.load(first ? at<T>(a.c, x.b, t + j, x.h) : at<T>(a.c2, x.b, t + j, x.h), t + j < x.end, first ? a.na : a.nb);
  };
  const int64_t past = x.t0 + (max(x.end - x.t0, int64_t(0)) + kC - 1) / kC * kC;
  if (past > x.t0) {
    fetch(past - kC, 0);
    if (OUT) fetch_rows(past - kC);
  }
  for (int64_t t = past - kC; t >= x.t0; t -= kC) {
    const int m = int(min(int64_t(kC), x.end - t)), rows = int(min(int64_t(kC), x.t1 - t));
    f4 o[NX / 16];
    for (int q = 0; q < a.G; ++q) {
      su.put(ut), sw.put(wt);
      if (OUT && q == 0) D.put(copy);
      __syncthreads();
      if (OUT && q == 0) c = next;
      if (q + 1 < a.G) {
        fetch(t, q + 1);
      } else if (t > x.t0) {
        fetch(t - kC, 0);
        if (OUT) fetch_rows(t - kC);
      }
      if (OUT) {
        if (q == 0) {
          const float own = power(ld, max(0, m - 1 - j));
          if (first)
            times_state<T, NA, NB, NB / 16>(o, 0, copy, c, own);
          else
            times_state_back<T, NA, NB>(o, copy, c, own);
        }
        if (first)
          later_rows<T, NA, NB>(o, ut, wt, c, wave, diag, near, far);
        else
          later_rows<T, NB, NA>(o, wt, ut, c, wave, diag, near, far);
      }
      D.update(q ? 1.0f : power(ld, m), ut, wt, [&](int tile, int r) { return after[tile] * near[r]; });
      __syncthreads();
    }
    if (OUT && j < rows) {
      if (first)
        store_row<T, NB / 16>(at<T>(a.out, x.b, t + j, x.h), 0, o, 1.0f, j >= m, a.nb);
      else
        store_row<T, NA / 16>(at<T>(a.out2, x.b, t + j, x.h), 0, o, 1.0f, j >= m, a.na);
    }
  }
  if (OUT) {
    zero_rows<T, NB>(a.out, x.b, x.h, 1, past, x.t1, a.nb);
    zero_rows<T, NA>(a.out2, x.b, x.h, 1, past, x.t1, a.na);
  }
  if (a.sn) D.store(a.sn + state * a.na * a.nb, a);
}

// Passes the states from segment to segment: what each segment alone leaves,
// in ws [B H][nseg][size], gives way to the state it starts from.
struct PassArgs {
  float* ws;
  const float* s0;
  float* sn;
  const float* log_decay;
  const int32_t* lengths;
  int64_t T, L;
  int H, nseg, size;
};
template <bool BACK>
__global__ __launch_bounds__(256) void pass_states(PassArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x, bh = blockIdx.y;
  if (i >= a.size) return;
  const int b = bh / a.H;
  const float ld = a.log_decay[bh % a.H];
  int64_t n = a.T;
  if (a.lengths) n = min(max(int64_t(a.lengths[b]), int64_t(0)), a.T);
  float* p = a.ws + int64_t(bh) * a.nseg * a.size + i;
  float s = a.s0 ? a.s0[int64_t(bh) * a.size + i] : 0.0f;
  const float whole = power(ld, int(a.L));
#pragma unroll 8
  for (int k = 0; k < a.nseg; ++k) {
    const int seg = BACK ? a.nseg - 1 - k : k;
    const int64_t m = min(max(n - seg * a.L, int64_t(0)), a.L);
    float* const at = p + int64_t(seg) * a.size;
    const float add = *at;
    *at = s;
    s = fmaf(m == a.L ? whole : power(ld, int(m)), s, add);
  }
  if (a.sn) a.sn[int64_t(bh) * a.size + i] = s;
}

template <class T, int NA, int NB, bool BACK, bool OUT>
hipError_t run_chunks(const ChunkArgs& a, int B, hipStream_t s) {
  constexpr int lds = chunk_lds<T, NA, NB>();
  void (*const f)(ChunkArgs) = BACK ? backwards<T, NA, NB, OUT> : forwards<T, NA, NB, OUT>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void*)f, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  f<<<unsigned(B) * a.H * a.nseg, kThreads, lds, s>>>(a);
  return hipGetLastError();
}

template <bool BACK, bool OUT>
hipError_t launch_chunks(const ChunkArgs& a, int bf16, int B, hipStream_t s) {
  const int form = (bf16 ? 4 : 0) + (a.na > 64 ? 2 : 0) + (a.nb > 64 ? 1 : 0);
  switch (form) {
    case 0: return run_chunks<float, 64, 64, BACK, OUT>(a, B, s);
    case 1: return run_chunks<float, 64, 128, BACK, OUT>(a, B, s);
    case 2: return run_chunks<float, 128, 64, BACK, OUT>(a, B, s);
    case 3: return run_chunks<float, 128, 128, BACK, OUT>(a, B, s);
    case 4: return run_chunks<__bf16, 64, 64, BACK, OUT>(a, B, s);
    case 5: return run_chunks<__bf16, 64, 128, BACK, OUT>(a, B, s);
    case 6: return run_chunks<__bf16, 128, 64, BACK, OUT>(a, B, s);
    default: return run_chunks<__bf16, 128, 128, BACK, OUT>(a, B, s);
  }
}

// Tokens per segment and segments: as many workgroups as the CUs hold at once.
struct Cut {
  int64_t L;
  int nseg;
};
Cut cut(const AttnArgs& a) {
  const int64_t chunks = (a.T + kC - 1) / kC, states = int64_t(a.B) * a.H;
  int64_t want = (a.dk > 64 || a.dv > 64 ? 256 : 512) / states;
  if (want > chunks / 2) want = chunks / 2;  // a segment of one chunk would only move states
  if (want < 1) want = 1;
  const int64_t per = chunks ? (chunks + want - 1) / want : 1;
  return {per * kC, int(chunks ? (chunks + per - 1) / per : 1)};
}

size_t states_bytes(const AttnArgs& a, const Cut& c) {
  const size_t n = size_t(a.B) * a.H * c.nseg * a.dk * a.dv * 4;
  return c.nseg > 1 ? (n + 255) / 256 * 256 : 0;
}

ChunkArgs base(const AttnArgs& a, const Cut& c) {
  ChunkArgs r{};
  r.G = a.G, r.na = a.dk, r.nb = a.dv, r.H = a.H, r.nseg = c.nseg, r.T = a.T, r.L = c.L, r.scale = a.scale;
  r.log_decay = a.log_decay, r.lengths = a.lengths, r.sr = a.dv, r.sc = 1;
  return r;
}

template <bool BACK>
hipError_t pass(const AttnArgs& a, const Cut& c, float* ws, const float* s0, float* sn, hipStream_t s) {
  const PassArgs p{ws, s0, sn, a.log_decay, a.lengths, a.T, c.L, a.H, c.nseg, a.dk * a.dv};
  pass_states<BACK><<<dim3(unsigned(p.size + 255) / 256, unsigned(a.B) * a.H), 256, 0, s>>>(p);
  return hipGetLastError();
}

#define TRY(expr)                          \
  do {                                     \
    const hipError_t e_ = (expr);          \
    if (e_ != hipSuccess) return e_;       \
  } while (0)

// the states at the segments' starts, in ws, and the last one
hipError_t segment_states(const AttnArgs& a, const Cut& c, float* ws, float* sn, hipStream_t s) {
  ChunkArgs r = base(a, c);
  r.u = a.k, r.w = a.v, r.sn = ws;
  TRY((launch_chunks<false, false>(r, a.bf16, a.B, s)));
  return pass<false>(a, c, ws, a.s0, sn, s);
}

}  // namespace

size_t attn_workspace(const AttnArgs& a, bool backward) {
  const Cut c = cut(a);
  return (backward ? 2 : 1) * states_bytes(a, c);
}

hipError_t launch_attn(const AttnArgs& a, hipStream_t s) {
  const Cut c = cut(a);
  ChunkArgs r = base(a, c);
  r.c = a.q, r.u = a.k, r.w = a.v, r.out = a.o, r.s0 = a.s0, r.sn = a.sn;
  if (c.nseg > 1) {
    float* ws = reinterpret_cast<float*>(a.ws);
    TRY(segment_states(a, c, ws, a.sn, s));
    r.s0 = ws, r.sn = nullptr;
  }
  return launch_chunks<false, true>(r, a.bf16, a.B, s);
}

hipError_t launch_attn_backward(const AttnGradArgs& g, hipStream_t s) {
  const AttnArgs& a = g.a;
  const Cut c = cut(a);
  ChunkArgs f = base(a, c), r = base(a, c);
  // dq: forwards over the transposed states
  f.c = a.o, f.u = a.v, f.w = a.k, f.out = g.dq, f.s0 = a.s0;
  f.na = a.dv, f.nb = a.dk, f.sr = 1, f.sc = a.dv;
  r.c = a.k, r.c2 = a.v, r.u = a.q, r.w = a.o, r.out = g.dv, r.out2 = g.dk, r.s0 = g.dsn, r.sn = g.ds0;
  if (c.nseg > 1) {
    float* ws = reinterpret_cast<float*>(a.ws);
    float* ws2 = reinterpret_cast<float*>(a.ws + states_bytes(a, c));
    TRY(segment_states(a, c, ws, nullptr, s));
    ChunkArgs l = r;
    l.sn = ws2;
    TRY((launch_chunks<true, false>(l, a.bf16, a.B, s)));
    TRY(pass<true>(a, c, ws2, g.dsn, g.ds0, s));
    f.s0 = ws, r.s0 = ws2, r.sn = nullptr;
  }
  TRY((launch_chunks<false, true>(f, a.bf16, a.B, s)));
  return launch_chunks<true, true>(r, a.bf16, a.B, s);
}

}  // namespace ambptt
