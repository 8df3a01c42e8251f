// Rotary positions: rows of queries and keys turned by their positions (rs_rope_apply), and new rows of the cache with
// their keys and queries turned on the way (rs_cache_append_rope).
//
// Pair i of a row at position p turns by a = p f_i:  y_1 = m (x_1 cos a - x_2 sin a), y_2 = m (x_2 cos a + x_1 sin a).
// Every element is read and written once, so memory bounds both calls (and the launch the short ones).  A lane takes 8
// pairs of a row, two 16-byte chunks (four in fp32), computes their cosines and sines once and uses them for head after
// head, so that the angles cost little beside the copying: no table of them is read from memory, and positions have no
// upper end.
#include "rope.h"
#include "cache.h"

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

// What a lane holds of a row: 8 elements each of two chunks, in 32 bits.
struct Piece {
  float a[8], b[8];
};

template <typename T>
struct Raw;  // a chunk as it lies in memory
template <>
struct Raw<bf16> {
  u32x4 x;
  __device__ __forceinline__ void load(const char *p) { x = *(const u32x4 *)p; }
  __device__ __forceinline__ void store(char *p) const { *(u32x4 *)p = x; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t w = x[e];
      f[2 * e] = __builtin_bit_cast(float, w << 16);
      f[2 * e + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = pack_bf16x2(f[2 * e], f[2 * e + 1]);
  }
};
template <>
struct Raw<float> {
  f32x4 x, y;
  __device__ __forceinline__ void load(const char *p) { x = *(const f32x4 *)p, y = *(const f32x4 *)(p + 16); }
  __device__ __forceinline__ void store(char *p) const { *(f32x4 *)p = x, *(f32x4 *)(p + 16) = y; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = x[e], f[4 + e] = y[e];
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = f[e], y[e] = f[4 + e];
  }
};

// How the pairs of a row lie in a lane's two chunks.
//   R_HALF   dim a multiple of 16: lanes below dim / 16 hold elements 8l .. and dim / 2 + 8l .., pair e in element e of
//            both; the others 16 elements that stay as they are;
//   R_INTER  elements 16l .. 16l + 15, pair e in elements 2e and 2e + 1; pairs from dim / 2 on stay;
//   R_ANY    half layout of any even dim: elements one by one, pair 8l + e in elements 8l + e and dim / 2 + 8l + e, and
//            from pair dim / 2 on, two neighbours that stay.
enum { R_HALF = 0, R_INTER = 1, R_ANY = 2 };

// A lane's cosines and sines, its places in a row and the number of its pairs that turn.
template <typename T, int MODE>
struct Turner {
  float c[8], s[8];
  int oa, ob, np;  // byte offsets of the chunks (R_ANY: of the first element of the first and the second kind)

  __device__ __forceinline__ void places(int dim, int l) {
    const int half = dim >> 1;
    np = clampi(half - 8 * l, 0, 8);
    if constexpr (MODE == R_HALF) {
      oa = np ? 8 * l : 16 * l;
      ob = np ? half + 8 * l : 16 * l + 8;
    } else if constexpr (MODE == R_INTER) {
      oa = 16 * l;
      ob = 16 * l + 8;
    } else {
      oa = 8 * l;
      ob = half + 8 * l;
    }
    oa *= (int)sizeof(T);
    ob *= (int)sizeof(T);
  }
  __device__ __forceinline__ void angles(const rs_rope &r, int l, double pos, bool back) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      c[e] = 1.f, s[e] = 0.f;
      if (e < np) {
        turn(pos * r.turns[8 * l + e], c[e], s[e]);
        c[e] *= r.mscale;
        s[e] *= back ? -r.mscale : r.mscale;
      }
    }
  }
  __device__ __forceinline__ void pair(int e, float &x, float &y) const {
    const float u = x * c[e] - y * s[e], v = y * c[e] + x * s[e];
    x = u, y = v;
  }
  __device__ __forceinline__ void turn_piece(Raw<T> &ra, Raw<T> &rb) const {
    if (np == 0) return;  // (what stays keeps its bits)
    Piece p;
    ra.get(p.a);
    rb.get(p.b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (MODE == R_HALF) {
        pair(e, p.a[e], p.b[e]);
      } else {
        float &x = e < 4 ? p.a[2 * e & 7] : p.b[2 * e & 7], &y = e < 4 ? p.a[(2 * e & 7) + 1] : p.b[(2 * e & 7) + 1];
        float u = x, v = y;
        pair(e, u, v);
        x = e < np ? u : x;
        y = e < np ? v : y;
      }
    }
    ra.set(p.a);
    rb.set(p.b);
  }
  // N rows of one position: heads h0, h0 + step, ... below `end`; all are loaded before any is stored, so that the loads
  // are in flight together.  skip: y is x, and lanes whose elements stay have nothing to do.
  template <int N>
  __device__ __forceinline__ void rows(const char *x, char *y, int64_t sx, int64_t sy, int h0, int step, int end, int dim, int d,
                                       int l, bool skip) const {
    if constexpr (MODE == R_ANY) {
      for (int h = h0; h < end; h += step) {
        const T *xr = (const T *)(x + h * sx);
        T *yr = (T *)(y + h * sy);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int i = 8 * l + e, half = dim >> 1;
          if (2 * i >= d) break;
          const int ia = e < np ? i : 2 * i, ib = e < np ? half + i : 2 * i + 1;
          if (e >= np && skip) continue;
          const T xa = xr[ia], xb = xr[ib];
          float a = (float)xa, b = (float)xb;
          pair(e, a, b);
          yr[ia] = e < np ? (T)a : xa;
          yr[ib] = e < np ? (T)b : xb;
        }
      }
    } else {
      if (np == 0 && skip) return;
      for (; h0 < end; h0 += N * step) {
        Raw<T> ra[N], rb[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const char *p = x + (h0 + k * step < end ? h0 + k * step : h0) * sx;
          ra[k].load(p + oa);
          rb[k].load(p + ob);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
          if (h0 + k * step >= end) break;
          turn_piece(ra[k], rb[k]);
          char *p = y + (h0 + k * step) * sy;
          ra[k].store(p + oa);
          rb[k].store(p + ob);
        }
      }
    }
  }
};

constexpr int kThreads = 256;

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
  int nparts, n, d, lg;  // 1 << lg: groups of heads that share a row
  const int32_t *pos;
  int64_t pos0;
  bool back;
};

// A workgroup takes 256 / (lanes of a row x groups) rows.
template <typename T, int MODE, int LPR>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeArgs a) {
  const int l = threadIdx.x % LPR, x = threadIdx.x / LPR, groups = 1 << a.lg, g = x & (groups - 1);
  const int r = blockIdx.x * (kThreads / LPR >> a.lg) + (x >> a.lg);
  if (r >= a.n) return;
  Turner<T, MODE> t;
  t.places(a.rope.dim, l);
  t.angles(a.rope, l, (double)(a.pos ? (int64_t)a.pos[r] : a.pos0 + r), a.back);
  int first = g;  // heads of all parts one after the other are dealt to the groups
  for (int k = 0; k < a.nparts; ++k) {
    const RopePart &p = a.part[k];
    t.template rows<4>(p.x + r * p.sx_t, p.y + r * p.sy_t, p.sx_h, p.sy_h, first, groups, p.heads, a.rope.dim, a.d, l, p.inplace);
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
  int nrows, max_rows, d, lg;
};

// As rope_kernel, a sequence's rows: heads of K with those of V, then of Q.
template <typename T, int MODE, int LPR>
__global__ __launch_bounds__(kThreads) void append_rope_kernel(const AppendRopeArgs a) {
  const CacheView &c = a.c;
  const int l = threadIdx.x % LPR, x = threadIdx.x / LPR, groups = 1 << a.lg, g = x & (groups - 1);
  const int b = blockIdx.y, i = blockIdx.x * (kThreads / LPR >> a.lg) + (x >> a.lg);
  const RowRange rr = new_rows(a.start, b, a.nrows, a.max_rows);
  if (i >= rr.count) return;
  const int len = cache_len(c, b);
  const int64_t row = rr.first + i;
  Turner<T, MODE> t;
  t.places(a.rope.dim, l);
  t.angles(a.rope, l, (double)(a.pos ? (int64_t)a.pos[row] : (int64_t)(c.seen ? c.seen[b] : len) + i), false);
  const int64_t j = (int64_t)len + i;
  const int p = j < c.cap ? page_of(c, (int)j) : 0, id = j < c.cap ? page_id(c, b, p) : -1;
  if (id >= 0) {
    const char *kr = a.kn + row * a.skt, *vr = a.vn + row * a.svt;
    const int64_t ko = k_offset(c, id, p, (int)j, 0), vo = v_offset(c, id, p, (int)j, 0);
    for (int h = g; h < c.hkv; h += groups) {
      Raw<T> va, vb;
      va.load(vr + h * a.svh + 16 * l * (int)sizeof(T));
      vb.load(vr + h * a.svh + (16 * l + 8) * (int)sizeof(T));
      t.template rows<1>(kr, c.k + ko, a.skh, c.sk_h, h, groups, h + 1, a.rope.dim, a.d, l, false);
      char *vp = c.v + vo + h * c.sv_h + 16 * l * (int)sizeof(T);
      va.store(vp);
      vb.store(vp + 8 * sizeof(T));
      if (c.acc && l == 0) c.acc[((int64_t)b * c.hkv + h) * c.cap + j] = 0.f;
    }
  }
  const int first = (g - c.hkv) & (groups - 1);
  t.template rows<4>(a.q.x + row * a.q.sx_t, a.q.y + row * a.q.sy_t, a.q.sx_h, a.q.sy_h, first, groups, a.q.heads, a.rope.dim, a.d,
                     l, a.q.inplace);
}

RopePart part_of(const rs_rope_part &p, int e) {
  return RopePart{(const char *)p.x, (char *)p.y, p.sx_t * e, p.sx_h * e, p.sy_t * e, p.sy_h * e, p.heads, p.x == p.y};
}

// log2 of the groups of heads: a row is split over so many lanes that the rows fill the chip's 2^19 lanes, up to a
// workgroup's 256 or one head each.
int head_groups(int64_t rows, int d, int heads) {
  int lg = 0;
  while (lg < (d == 128 ? 5 : 6) && (1 << lg) < heads && rows * (d / 16) << lg < 1 << 19) ++lg;
  return lg;
}

template <typename F>
void by_shape(int dtype, int d, const rs_rope &r, F f) {
  auto with_l = [&](auto t, auto m) {
    d == 128 ? f(t, m, std::integral_constant<int, 8>{}) : f(t, m, std::integral_constant<int, 4>{});
  };
  auto with_m = [&](auto t) {
    if (r.layout == RS_ROPE_INTERLEAVED) with_l(t, std::integral_constant<int, R_INTER>{});
    else if (r.dim % 16 == 0) with_l(t, std::integral_constant<int, R_HALF>{});
    else with_l(t, std::integral_constant<int, R_ANY>{});
  };
  dtype == RS_BF16 ? with_m(bf16{}) : with_m(float{});
}

}  // namespace

rs_status rope_launch(const rs_rope &rope, const rs_rope_rows &rows, bool transpose, hipStream_t st) {
  const int e = rows.dtype == RS_BF16 ? 2 : 4;
  RopeArgs a{};
  a.rope = rope;
  a.nparts = rows.nparts, a.n = rows.n, a.d = rows.d, a.pos = rows.pos, a.pos0 = rows.pos0, a.back = transpose;
  int heads = 0;
  for (int k = 0; k < rows.nparts; ++k) {
    a.part[k] = part_of(rows.part[k], e);
    heads += rows.part[k].heads;
  }
  a.lg = head_groups(rows.n, rows.d, heads);
  const int per = kThreads / (rows.d / 16) >> a.lg;
  by_shape(rows.dtype, rows.d, rope, [&](auto t, auto m, auto l) {
    rope_kernel<decltype(t), decltype(m)::value, decltype(l)::value><<<(rows.n + per - 1) / per, kThreads, 0, st>>>(a);
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
  a.pos = pos, a.start = start, a.nrows = nrows, a.max_rows = max_rows, a.d = d;
  const int most = max_rows < nrows ? max_rows : nrows;  // rows of a sequence at most
  const int64_t all = (int64_t)c.nseq * most;
  a.lg = head_groups(all < nrows ? all : nrows, d, c.hkv + a.q.heads);
  const int per = kThreads / (d / 16) >> a.lg;
  by_shape(dtype, d, rope, [&](auto t, auto m, auto l) {
    append_rope_kernel<decltype(t), decltype(m)::value, decltype(l)::value>
        <<<dim3((most + per - 1) / per, c.nseq), kThreads, 0, st>>>(a);
  });
  RS_HIP(hipGetLastError());
  return RS_OK;
}

}  // namespace rs
