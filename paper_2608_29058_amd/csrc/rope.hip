// Rotary positions: rows of queries and keys turned by their positions (rs_rope_apply), and new rows of the cache with
// their keys and queries turned on the way (rs_cache_append_rope).
//
// Pair i of a row at position p turns by a = p f_i:  y_1 = m (x_1 cos a - x_2 sin a), y_2 = m (x_2 cos a + x_1 sin a).
// Every element is read and written once, so memory bounds both calls (and the launch the short ones).  A lane takes 8
// pairs of a row, two vectors of 16 bytes (four in fp32); the workgroup computes each cosine and sine of its rows once, into
// LDS, for all heads, so that they cost little beside the copying: no table of them is read from memory, and positions have
// no upper end.  131072 rows of 32 + 8 heads of 128 in bf16: 492 us, 5.5 TB/s (a large copy: 5.15); a step's few rows:
// the launch.
#include "rope.h"
#include "cache.h"
#include "rope_plan.h"

namespace rs {

namespace {

// Cosine and sine of t turns, t the fp64 product of position and turns per position (good to 2^-52 of itself: at
// position 2^31 and one turn in six positions 10^-7 turns, at 2^18 10^-11).  Less whole quarter turns r is within half of
// one, and r, as fp32, is good to 2^-26 of a quarter turn.  The series of sine and cosine, up to x^9 and x^10, end
// within 2^-29 for |x| <= pi / 4.
__device__ __forceinline__ void turn(double t, float &c, float &s) {
  const double t4 = 4.0 * t, n = __builtin_rint(t4);
  const float x = (float)(t4 - n) * 1.57079632679489662f, z = x * x;
  // n modulo 4, exact for any n (positions times turns may pass 32 bits)
  const int q = (int)(n - 4.0 * __builtin_floor(0.25 * n));
  const float sx = x + x * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
  const float cx = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
  const float a = q & 1 ? sx : cx, b = q & 1 ? cx : sx;
  c = q == 1 || q == 2 ? -a : a;
  s = q >= 2 ? -b : b;
}

// Rows are written past the caches (nontemporal), so that what is read stays in the 256 MB memory-side cache: 8191 fp32 rows
// of 32 heads of 64 35 -> 26 us, 224 MiB of bf16 rows 90 -> 69 us, 90 -> 86 where other rows were read since.  Inputs beyond that
// size are read past them too (NTL): nothing of them is left there, and what is there may be of use (1 GiB between two passes of
// another kernel over it: 404 -> 349 us); smaller ones not (96 MiB: 31 -> 35 us), nor where an instruction reads half
// lines, which would be fetched twice (30001 rows of 32 + 8 heads, with lanes that read so: 122 -> 133 us).
template <bool NTL>
__device__ __forceinline__ u32x4 load16(const char *p) {
  if constexpr (NTL) return __builtin_nontemporal_load((const u32x4 *)p);
  return *(const u32x4 *)p;
}
__device__ __forceinline__ void store16(char *p, u32x4 x) { __builtin_nontemporal_store(x, (u32x4 *)p); }

// 16 elements of a row per lane, as vectors of 16 bytes: NV of them, V elements each.
template <typename T>
struct Raw {
  static constexpr int V = 16 / (int)sizeof(T), NV = 16 / V;
  u32x4 x[NV];
  __device__ __forceinline__ void get(float (&f)[16]) const {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t y = x[k][w];
        if constexpr (V == 8) {
          f[8 * k + 2 * w] = __builtin_bit_cast(float, y << 16);
          f[8 * k + 2 * w + 1] = __builtin_bit_cast(float, y & 0xffff0000u);
        } else {
          f[4 * k + w] = __builtin_bit_cast(float, y);
        }
      }
  }
  __device__ __forceinline__ void set(const float (&f)[16]) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if constexpr (V == 8) x[k][w] = pack_bf16x2(f[8 * k + 2 * w], f[8 * k + 2 * w + 1]);
        else x[k][w] = __builtin_bit_cast(uint32_t, f[4 * k + w]);
      }
  }
};

constexpr int kThreads = kRopeThreads;

// Neighbouring lanes take neighbouring vectors of a row, LPR apart, so that an instruction moves whole lines (with a lane's 16
// elements in one piece, 8191 fp32 rows of 32 heads of 64: 57 us; so, 35).  Where the pairs of a row are then:
//   R_HALF   half layout of the whole head: both in the lane, elements x and 8 + x;
//   R_INTER  interleaved: neighbours; pairs from dim / 2 on stay;
//   R_PART   half layout of a part of the head whose half is made of vectors: the other of each pair in another lane's vector, which
//            passes through LDS (79652 rows of 32 + 8 heads of 128, 32 of each rotated: 297 us, with lanes that read both halves of
//            their pairs, and so parts of lines, 816);
//   R_ANY    half layout of any even dim: the same, element by element (43998 rows of 64 + 8 heads of 128, 126 of each rotated: 331 us, with elements from
//            memory 1100).
enum { R_HALF = 0, R_INTER = 1, R_PART = 2, R_ANY = 3 };

// A lane's cosines and sines and its places in a row.
template <typename T, int MODE, int LPR>
struct Turner {
  static constexpr bool STAGED = MODE == R_PART || MODE == R_ANY;
  static constexpr int V = Raw<T>::V, NV = Raw<T>::NV, E = sizeof(T), NC = STAGED ? 16 : 8;
  static constexpr int kStage = STAGED ? kThreads * 16 * E / 4 : 0;  // floats of LDS
  float c[NC], s[NC];  // of each pair (STAGED: of each element, the sine with the sign that it has there)
  int l, dim;
  int mate[MODE == R_ANY ? 16 : NV];  // STAGED: byte offset of the other element of a pair, R_PART: of a vector of them
  char *stage;                        // STAGED: the row in LDS

  __device__ __forceinline__ Turner(int lane, int rot, char *lds) : l(lane), dim(rot), stage(lds) {
    if constexpr (MODE == R_PART)
#pragma unroll
      for (int k = 0; k < NV; ++k) mate[k] = E * mate_of(V * (l + k * LPR));
    if constexpr (MODE == R_ANY)
#pragma unroll
      for (int x = 0; x < 16; ++x) mate[x] = E * mate_of(element(x));
  }
  __device__ __forceinline__ int off(int k) const { return 16 * (l + k * LPR); }
  __device__ __forceinline__ int element(int x) const { return V * (l + x / V * LPR) + x % V; }
  __device__ __forceinline__ int mate_of(int i) const { return i >= dim ? i : i < dim >> 1 ? i + (dim >> 1) : i - (dim >> 1); }
  // R_HALF, R_INTER: the pair whose turn is c[e], s[e]
  __device__ __forceinline__ int pair_of(int e) const {
    if constexpr (MODE == R_INTER) return V / 2 * (l + e / (V / 2) * LPR) + e % (V / 2);
    return element(e);
  }
  // the lane's pairs from the row's table of cosines, then sines
  __device__ __forceinline__ void take(const float *row) {
    const int half = dim >> 1;
#pragma unroll
    for (int e = 0; e < NC; ++e) {
      int i = STAGED ? element(e) : pair_of(e);
      const bool first = !STAGED || i < half;
      i = STAGED && !first ? i - half : i;
      i = i < half ? i : 0;
      c[e] = row[i], s[e] = STAGED && first ? -row[8 * LPR + i] : row[8 * LPR + i];
    }
  }
  __device__ __forceinline__ void pair(int e, float &x, float &y) const {
    const float u = x * c[e] - y * s[e], v = y * c[e] + x * s[e];
    x = u, y = v;
  }
  __device__ __forceinline__ void turn_raw(Raw<T> &r, const bool (&move)[NV]) const {
    float f[16];
    r.get(f);
    if constexpr (STAGED) {
      // a row's lanes are of one wave, whose accesses of LDS follow each other
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (move[k]) *(u32x4 *)(stage + off(k)) = r.x[k];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
      float g[16];
      if constexpr (MODE == R_PART) {
        Raw<T> o;
#pragma unroll
        for (int k = 0; k < NV; ++k) o.x[k] = *(const u32x4 *)(stage + mate[k]);
        o.get(g);
      } else {
#pragma unroll
        for (int x = 0; x < 16; ++x) g[x] = (float)*(const T *)(stage + mate[x]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
#pragma unroll
      for (int x = 0; x < 16; ++x) f[x] = f[x] * c[x] + g[x] * s[x];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) MODE == R_HALF ? pair(e, f[e], f[8 + e]) : pair(e, f[2 * e], f[2 * e + 1]);
    }
    Raw<T> y;
    y.set(f);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w)  // what stays keeps its bits, those of a NaN too (dim is even: a word of two bf16 turns or stays)
        r.x[k][w] = MODE == R_HALF || V * (l + k * LPR) + w * (V / 4) < dim ? y.x[k][w] : r.x[k][w];
  }
  // Rows of one position: heads h0, h0 + step, ... below `end`, N of them loaded before any is stored.  N = 2 (16 registers)
  // where the heads lie together; apart, one, whose 50 registers leave room for eight waves per SIMD (131072 rows of 32 + 8 heads of
  // 128: 492 us, with four 551).  skip: y is x, and vectors that stay need not move.
  template <int N, bool NTL>
  __device__ __forceinline__ void rows(const char *x, char *y, int64_t sx, int64_t sy, int h0, int step, int end, bool skip) const {
    bool move[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) move[k] = MODE == R_HALF || !skip || off(k) < dim * E;
    for (; h0 + (N - 1) * step < end; h0 += N * step) some_rows<N, NTL>(x, y, sx, sy, h0, step, move);
    if constexpr (N > 1)
      for (; h0 < end; h0 += step) some_rows<1, NTL>(x, y, sx, sy, h0, step, move);
  }
  template <int N, bool NTL>
  __device__ __forceinline__ void some_rows(const char *x, char *y, int64_t sx, int64_t sy, int h0, int step, const bool (&move)[NV]) const {
    Raw<T> r[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const char *p = x + (h0 + n * step) * sx;
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (move[k]) r[n].x[k] = load16<NTL>(p + off(k));
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      turn_raw(r[n], move);
      char *p = y + (h0 + n * step) * sy;
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (move[k]) store16(p + off(k), r[n].x[k]);
    }
  }
};

constexpr int64_t kSideCache = 256ll << 20;  // bytes of the memory-side cache

struct RopePart {
  const char *x;
  char *y;
  int64_t sx_t, sx_h, sy_t, sy_h;  // bytes
  int heads;
  bool inplace;
};
struct RopeArgs {
  rs_rope rope;
  RopePart part[4];
  int nparts, n, lg;  // 1 << lg: groups of heads that share a row
  const int32_t *pos;
  int64_t pos0;
  bool back;
};

// Cosines and sines of the `rows` rows of a workgroup, every one computed once: tab[row] holds 8 LPR of each.  pos(row): its
// position.
template <int LPR, typename F>
__device__ __forceinline__ void angle_table(float *tab, const rs_rope &r, int rows, bool back, F pos) {
  const int half = r.dim >> 1;
  for (int x = threadIdx.x; x < rows * 8 * LPR; x += kThreads) {
    const int row = x / (8 * LPR), i = x % (8 * LPR);
    if (i >= half) continue;
    float c, s;
    turn(pos(row) * r.turns[i], c, s);
    tab[row * 16 * LPR + i] = c * r.mscale;
    tab[row * 16 * LPR + 8 * LPR + i] = s * (back ? -r.mscale : r.mscale);
  }
  __syncthreads();
}

// A workgroup takes 256 / (lanes of a row x groups) rows.
template <typename T, int MODE, int LPR, int N, bool NTL>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeArgs a) {
  __shared__ __align__(16) float tab[kThreads * 16 + Turner<T, MODE, LPR>::kStage];
  const int l = threadIdx.x % LPR, x = threadIdx.x / LPR, groups = 1 << a.lg, g = x & (groups - 1), rows = kThreads / LPR >> a.lg;
  const int r0 = blockIdx.x * rows, r = r0 + (x >> a.lg);
  angle_table<LPR>(tab, a.rope, rows, a.back, [&](int i) {
    const int at = r0 + i < a.n ? r0 + i : a.n - 1;
    return (double)(a.pos ? (int64_t)a.pos[at] : a.pos0 + at);
  });
  if (r >= a.n) return;
  Turner<T, MODE, LPR> t(l, a.rope.dim, (char *)(tab + kThreads * 16) + x * LPR * 16 * (int)sizeof(T));
  t.take(tab + (r - r0) * 16 * LPR);
  int first = g;  // heads of all parts one after the other are dealt to the groups
  for (int k = 0; k < a.nparts; ++k) {
    const RopePart &p = a.part[k];
    t.template rows<N, NTL>(p.x + r * p.sx_t, p.y + r * p.sy_t, p.sx_h, p.sy_h, first, groups, p.heads, p.inplace);
    first = (first - p.heads) & (groups - 1);
  }
}

struct AppendRopeArgs {
  CacheView c;
  rs_rope rope;
  const char *kn, *vn;
  int64_t skt, skh, svt, svh;  // bytes
  RopePart q;                  // heads 0: none
  const int32_t *pos, *start;
  int nrows, max_rows, lg;
};

// As rope_kernel, a sequence's rows: heads of K with those of V, then of Q.  BYROW: the rows are the batch's, and each has a
// sequence of its own, or none.
template <typename T, int MODE, int LPR, int N, bool NTL, bool BYROW>
__global__ __launch_bounds__(kThreads) void append_rope_kernel(const AppendRopeArgs a) {
  __shared__ __align__(16) float tab[kThreads * 16 + Turner<T, MODE, LPR>::kStage];
  __shared__ unsigned long long own[BYROW ? kThreads / LPR : 1];  // sequence and place in it of each row, ~0: none
  const CacheView &c = a.c;
  const int l = threadIdx.x % LPR, x = threadIdx.x / LPR, groups = 1 << a.lg, g = x & (groups - 1), rows = kThreads / LPR >> a.lg;
  const int x0 = blockIdx.x * rows, at = x >> a.lg;
  int b = blockIdx.y, i = x0 + at, len = 0;
  int64_t row = i;
  if constexpr (BYROW) {
    if ((int)threadIdx.x < rows) own[threadIdx.x] = ~0ull;
    __syncthreads();
    for (int s = threadIdx.x; s < c.nseq; s += kThreads) {
      const RowRange rr = new_rows(a.start, s, a.nrows, a.max_rows);
      const int first = rr.first > x0 ? rr.first : x0, end = rr.first + rr.count < x0 + rows ? rr.first + rr.count : x0 + rows;
      // (a row that several sequences claim, which a start that descends allows, is the first one's)
      for (int r = first; r < end; ++r) atomicMin(&own[r - x0], (unsigned long long)s << 32 | (uint32_t)(r - rr.first));
    }
    __syncthreads();
    angle_table<LPR>(tab, a.rope, rows, false, [&](int k) {
      const unsigned long long o = own[k];
      if (o == ~0ull) return 0.0;
      const int s = (int)(o >> 32);
      return (double)(a.pos ? (int64_t)a.pos[x0 + k] : (c.seen ? c.seen[s] : cache_len(c, s)) + (int64_t)(uint32_t)o);
    });
    const unsigned long long o = own[at];
    if (o == ~0ull) return;
    b = (int)(o >> 32), i = (int)(uint32_t)o;
    len = cache_len(c, b);
  } else {
    const RowRange rr = new_rows(a.start, b, a.nrows, a.max_rows);
    if (x0 >= rr.count) return;
    len = cache_len(c, b);
    const int64_t pos0 = c.seen ? c.seen[b] : len;
    angle_table<LPR>(tab, a.rope, rows, false, [&](int k) {
      const int y = x0 + k < rr.count ? x0 + k : rr.count - 1;
      return (double)(a.pos ? (int64_t)a.pos[rr.first + y] : pos0 + y);
    });
    if (i >= rr.count) return;
    row = rr.first + i;
  }
  Turner<T, MODE, LPR> t(l, a.rope.dim, (char *)(tab + kThreads * 16) + x * LPR * 16 * (int)sizeof(T));
  t.take(tab + at * 16 * LPR);
  const int64_t j = (int64_t)len + i;
  const int p = j < c.cap ? page_of(c, (int)j) : 0, id = j < c.cap ? page_id(c, b, p) : -1;
  if (id >= 0) {
    const char *kr = a.kn + row * a.skt, *vr = a.vn + row * a.svt;
    const int64_t ko = k_offset(c, id, p, (int)j, 0), vo = v_offset(c, id, p, (int)j, 0);
    for (int h = g; h < c.hkv; h += groups) {
      Raw<T> v;
#pragma unroll
      for (int k = 0; k < Raw<T>::NV; ++k) v.x[k] = load16<NTL>(vr + h * a.svh + 16 * (l + k * LPR));
      t.template rows<1, NTL>(kr, c.k + ko, a.skh, c.sk_h, h, groups, h + 1, false);
#pragma unroll
      for (int k = 0; k < Raw<T>::NV; ++k) store16(c.v + vo + h * c.sv_h + 16 * (l + k * LPR), v.x[k]);
      if (c.acc && l == 0) c.acc[((int64_t)b * c.hkv + h) * c.cap + j] = 0.f;
    }
  }
  const int first = (g - c.hkv) & (groups - 1);
  t.template rows<N, NTL>(a.q.x + row * a.q.sx_t, a.q.y + row * a.q.sy_t, a.q.sx_h, a.q.sy_h, first, groups, a.q.heads, a.q.inplace);
}

RopePart part_of(const rs_rope_part &p, int e) {
  return RopePart{(const char *)p.x, (char *)p.y, p.sx_t * e, p.sx_h * e, p.sy_t * e, p.sy_h * e, p.heads, p.x == p.y};
}

// f(type, mode, lanes of a row, heads at a time, loads that bypass) of a call over `bytes` of input.
template <typename F>
void by_shape(int dtype, int d, const rs_rope &r, bool tokens, int64_t bytes, F f) {
  using std::integral_constant;
  auto with_n = [&](auto t, auto m, auto l) {
    constexpr int L = decltype(l)::value, many = sizeof(t) == 2 ? 2 : 1;
    auto with_l = [&](auto n) {
      if constexpr (L == 8)  // a row's lanes read whole lines of 128 bytes
        if (bytes > kSideCache) return f(t, m, l, n, std::true_type{});
      f(t, m, l, n, std::false_type{});
    };
    tokens ? with_l(integral_constant<int, many>{}) : with_l(integral_constant<int, 1>{});
  };
  auto with_l = [&](auto t, auto m) {
    d == 128 ? with_n(t, m, integral_constant<int, 8>{}) : with_n(t, m, integral_constant<int, 4>{});
  };
  auto with_m = [&](auto t) {
    if (r.layout == RS_ROPE_INTERLEAVED) with_l(t, integral_constant<int, R_INTER>{});
    else if (r.dim == d) with_l(t, integral_constant<int, R_HALF>{});
    else if (r.dim % (32 / (int)sizeof(t)) == 0) with_l(t, integral_constant<int, R_PART>{});
    else with_l(t, integral_constant<int, R_ANY>{});
  };
  dtype == RS_BF16 ? with_m(bf16{}) : with_m(float{});
}

}  // namespace

rs_status rope_launch(const rs_rope &rope, const rs_rope_rows &rows, bool transpose, hipStream_t st) {
  const int e = rows.dtype == RS_BF16 ? 2 : 4;
  RopeArgs a{};
  a.rope = rope;
  a.nparts = rows.nparts, a.n = rows.n, a.pos = rows.pos, a.pos0 = rows.pos0, a.back = transpose;
  int heads = 0;
  for (int k = 0; k < rows.nparts; ++k) {
    a.part[k] = part_of(rows.part[k], e);
    heads += rows.part[k].heads;
  }
  const bool tokens = rows.part[0].sx_h < rows.part[0].sx_t;
  a.lg = head_groups(rows.n, rows.d, heads, tokens, rope);
  const int per = kThreads / (rows.d / 16) >> a.lg;
  by_shape(rows.dtype, rows.d, rope, tokens, (int64_t)rows.n * heads * rows.d * e, [&](auto t, auto m, auto l, auto n, auto ntl) {
    rope_kernel<decltype(t), decltype(m)::value, decltype(l)::value, decltype(n)::value, decltype(ntl)::value>
        <<<(rows.n + per - 1) / per, kThreads, 0, st>>>(a);
  });
  RS_HIP(hipGetLastError());
  return RS_OK;
}

rs_status append_rope_launch(const CacheView &c, int dtype, int d, const rs_rope &rope, const void *kn, const void *vn,
                             int64_t skt, int64_t skh, int64_t svt, int64_t svh, const rs_rope_part *q, const int32_t *pos,
                             const int32_t *start, int nrows, int max_rows, hipStream_t st) {
  const int e = dtype == RS_BF16 ? 2 : 4;
  AppendRopeArgs a{};
  a.c = c;
  a.rope = rope;
  a.kn = (const char *)kn, a.vn = (const char *)vn;
  a.skt = skt * e, a.skh = skh * e, a.svt = svt * e, a.svh = svh * e;
  if (q) a.q = part_of(*q, e);
  a.pos = pos, a.start = start, a.nrows = nrows, a.max_rows = max_rows;
  const bool tokens = skh < skt;
  const AppendShape sh = append_rope_shape(c.nseq, c.cap, nrows, max_rows, start, d, c.hkv, a.q.heads, tokens, rope);
  a.lg = sh.lg;
  const dim3 grid((unsigned)sh.x, (unsigned)sh.y);
  by_shape(dtype, d, rope, tokens, (int64_t)nrows * (2 * c.hkv + a.q.heads) * d * e, [&](auto t, auto m, auto l, auto n, auto ntl) {
    auto launch = [&](auto byrow) {
      append_rope_kernel<decltype(t), decltype(m)::value, decltype(l)::value, decltype(n)::value, decltype(ntl)::value, decltype(byrow)::value>
          <<<grid, kThreads, 0, st>>>(a);
    };
    sh.byrow ? launch(std::true_type{}) : launch(std::false_type{});
  });
  RS_HIP(hipGetLastError());
  return RS_OK;
}

}  // namespace rs
