// Cross attention of many rows per head (prompts) in bf16, at the rate of the matrix instructions.
//
// For rows r (token and query head of one key/value head) and the cached rows j that are seen:
//   l_j = scale q_r . k_j,  p_j = exp(l_j - max l),  O = sum p_j v_j / sum p_j.
// 4 d flops per row and state against 4 d bytes per state and 128 rows: the matrix rate bounds it.
//
// A workgroup takes 128 rows of one sequence and key/value head (all its query heads: the rows of a token lie side by side, so
// that few tokens fill a tile), 32 per wave; two workgroups share a CU, so that one's softmax overlaps the other's products.
// States pass in tiles of 64 through LDS, K and V in two buffers each, copied from memory without registers; a tile lies in one
// page.  Per wave and tile:
//   S^T [64 states x 32 rows] = K Q^T (Q in registers), v_mfma_f32_32x32x16_bf16: a lane holds one row and 32 states;
//   O^T [d x 32 rows] += V^T P^T, V read transposed, P straight from the accumulators of S^T.
// The running maximum is raised only where a sum of 32 weights passes 2^8, so that O is rarely rescaled.  Sums are of the
// weights before their rounding to bf16.  What the key mask hides is the same for all rows: a tile of which nothing is seen is
// left out, and of one seen in part the products of the hidden states start from minus infinity.
// 4096 rows x 32 heads of 128 over 65536 states of 8: 3.75-3.96 ms, 1.11-1.17 PFLOP/s, where the dense prefill runs at 1.11-1.17 and
// a 16384^3 product of torch's at 1.29-1.36: the matrix instructions are at work in 62 % of the cycles, the exponents (two vector
// instructions and a half per score) in most of the others, and the clock falls to 1.75 GHz; on constant operands, at the full clock, 1.5.
// Heads of 64: 2.36 ms, 0.93 PFLOP/s: half the products per exponent.  Where 3.82 ms are taken without a mask, one that hides nothing
// takes 3.89 and one that hides a state of every tile 4.01.
#include "draft_plan.h"

namespace rs {

namespace {

// Lambdas share the accumulators, which only stay in registers where all of them are inlined.
#define RS_INLINE __attribute__((always_inline))

constexpr int kRows = 128, kKeys = 64;  // rows of Q of a workgroup, states of a tile
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

// XOR of the 16-byte chunks of LDS row r: 16 rows' equal chunks (reads of K) and 4 rows' chunk pairs (transposed reads of V)
// lie in different banks.
template <int D>
__device__ __forceinline__ int swz(int r) {
  if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  else return ((r & 3) << 1) | ((r >> 2) & 1);
}

// Barrier after which every wave's copies into LDS and accesses of it are complete.  The wait for the copies (vmcnt(0)) is
// explicit: the fence does not always wait for them.
__device__ __forceinline__ void tile_barrier() {
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
// Barrier after LDS accesses alone.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Groups per piece, from all lengths.
__device__ __forceinline__ int plan_rounds(const DraftArgs &a, const Seq &first, int lane) {
  if (a.slots == 0) return kMaxN;  // one piece each
  auto all = [&](auto f) {  // sum over the sequences
    int x = f(first);
    for (int b0 = 64; b0 < a.c.nseq; b0 += 64) x += f(seq_at<W_CROSS>(a, b0 + lane));
    return wave_sum(x);
  };
  const int items = all([&](const Seq &q) { return items_of<W_CROSS>(a, q); });
  const int work = all([&](const Seq &q) { return items_of<W_CROSS>(a, q) * q.groups; });
  int longest = first.groups;
  for (int b0 = 64; b0 < a.c.nseq; b0 += 64) longest = larger(longest, seq_at<W_CROSS>(a, b0 + lane).groups);
  longest = wave_most(longest);
  return rounds_groups(items, work, longest, a.resident, a.grid, a.least, [&](int per) {
    const float inv = 1.f / (float)per;
    return all([&](const Seq &q) { return items_of<W_CROSS>(a, q) * pieces_by(q.groups, per, inv); });
  });
}

// A tile of the walk: its first state, page, and the states that are seen as bits; j < 0: none.
struct CrossTile {
  int j, id;
  uint64_t see;
};

// The kernel's arguments, read where they are needed: kept in scalar registers through the walk they would not fit.
typedef const __attribute__((address_space(4))) DraftArgs *ArgsPtr;
__device__ __forceinline__ ArgsPtr args_here() {
  ArgsPtr p = (ArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}
// x in scalar registers of its own, not as part of the arguments that were loaded with it.
template <typename T>
__device__ __forceinline__ T own(T x) {
  asm volatile("" : "+s"(x));
  return x;
}

// The LDS of a workgroup: tiles of K and V, what the products of K0 and K1 start from (minus infinity where a state is
// hidden), and whether a wave met what is not finite.
template <int D>
struct CrossLds {
  bf16 *K0, *K1, *V0, *V1;
  float *B0, *B1;
  int *odd;
};

// One piece of an item.  MASK: a key mask may hide states anywhere; without one only the last tile ends early.
// Hidden states may hold infinities and NaN, which a weight of zero and a score of minus infinity do not silence.  They show
// in O or in the sums, so the walk pays nothing for them: it writes nothing and returns false where something is not finite,
// and is then walked again SAFE, with the hidden rows of K and V zeroed in LDS.  (Zeroing them always, after a barrier in the
// middle of a step, took 20 % of a tile's time where a mask hides some of it.)
template <int D, bool MASK, bool SAFE>
__device__ __forceinline__ bool cross_walk(const Item &it, const CrossLds<D> &lds) {
  constexpr int NW = 4, KS = D / 16, DB = D / 32, CPR = D / 8, RPI = 64 / CPR, LPT = kKeys / RPI / NW;
  constexpr int KPF = 4, VPF = 3;  // fragment reads ahead of the products
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // (nothing that one walk derives from it is kept for the other)
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  const int r0 = it.rt * kRows, total = it.len;
  const int ngroups = (total + kGroup - 1) / kGroup, ntiles = (total + kKeys - 1) / kKeys;
  const int g0 = (int)((long long)ngroups * it.piece / it.npieces), g1 = (int)((long long)ngroups * (it.piece + 1) / it.npieces);
  const int t1 = uniform(g1 * (kGroup / kKeys) < ntiles ? g1 * (kGroup / kKeys) : ntiles);

  // this lane's row; rows behind the last are read as the last and not stored
  u32x4 qf[KS];
  {
    const ArgsPtr a = args_here();
    const int G = a->q.hq / a->c.hkv, nr = G * it.t, mine = r0 + 32 * wave + l32, row = mine < nr ? mine : nr - 1, tok = row / G;
    const bf16 *p = (const bf16 *)a->q.q + (it.first + tok) * a->q.sq_t + (it.g * G + row - tok * G) * a->q.sq_h + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const u32x4 *)(p + 16 * ks);
  }

  // ---- the walk: 64 tiles at a time, a lane per tile, those of which nothing is seen left out -----------------------
  int wt = uniform(g0 * (kGroup / kKeys)), wid = 0;  // first tile of the window; lane: page of tile wt + lane
  [[maybe_unused]] uint32_t wlo = 0, whi = 0;        // lane: its states that are seen
  uint64_t todo = 0;
  auto look = [&]() RS_INLINE {
    const ArgsPtr a = args_here();
    const int t = wt + lane, j = t * kKeys;
    bool ok = false;
    if (t < t1) {
      const int p = (int)(((uint64_t)((uint32_t)(j >> 6) * 2u) * a->c.pmul) >> 32);  // as page_of
      const int64_t at = (int64_t)it.b * a->c.max_pages + p;
      const int e = a->c.table ? a->c.table[at] : (int)at;
      wid = e;
      ok = e >= 0 && e < a->c.npages;
      if constexpr (MASK) {
        const uint32_t *m = a->q.mask + (int64_t)it.b * a->q.nwords;
        const auto word = [&](int w) RS_INLINE { return m[w]; };
        const uint64_t see = seen_words(total, j, word);
        wlo = (uint32_t)see;
        whi = (uint32_t)(see >> 32);
        ok = ok && see != 0;
      }
    }
    todo = __ballot(ok);
  };
  look();
  auto next = [&]() RS_INLINE -> CrossTile {
    while (__builtin_expect(todo == 0, 0)) {
      wt += 64;
      if (wt >= t1) return CrossTile{-1, 0, 0};
      look();
    }
    const int b = __builtin_ctzll(todo), j = (wt + b) * kKeys;
    todo &= todo - 1;
    uint64_t see = 0;
    if constexpr (MASK) {
      const uint32_t lo = __builtin_amdgcn_readlane(wlo, b), hi = __builtin_amdgcn_readlane(whi, b);
      see = (uint64_t)hi << 32 | lo;
    }
    return CrossTile{j, __builtin_amdgcn_readlane(wid, b), see};
  };
  // the states of a tile that are seen
  auto seen = [&](const CrossTile &t) RS_INLINE -> uint64_t { return MASK ? t.see : prefix_mask(total - t.j); };
  auto partly = [&](const CrossTile &t) RS_INLINE -> bool { return MASK ? t.see != ~0ull : t.j + kKeys > total; };

  // ---- copies: a wave instruction moves RPI rows; the lane's place among them is the same for every tile ------------
  const int lrow = wave * RPI + lane / CPR, lchunk = 16 * ((lane % CPR) ^ swz<D>(lrow));  // (swz sees row & 15 alone)
  const ArgsPtr a0 = args_here();
  const char *kb = own(a0->c.k + it.g * a0->c.sk_h), *vb = own(a0->c.v + it.g * a0->c.sv_h);
  const int64_t kp = own(a0->c.sk_p), vp = own(a0->c.sv_p);
  const uint32_t bK = own((uint32_t)a0->c.sk_t), bV = own((uint32_t)a0->c.sv_t);  // (rows are at most 16 MiB apart)
  const uint32_t pmul = own(a0->c.pmul), page = own((uint32_t)a0->c.page);
  const uint32_t voK = lrow * bK + lchunk, voV = lrow * bV + lchunk;
  auto copy = [&](bf16 *dst, const CrossTile &t, bool isv) RS_INLINE {
    const uint32_t p = (uint32_t)(((uint64_t)((uint32_t)(t.j >> 6) * 2u) * pmul) >> 32), in = t.j - p * page;
    const uint32_t b = isv ? bV : bK, vo = isv ? voV : voK;
    const char *base = (isv ? vb : kb) + t.id * (isv ? vp : kp) + (uint64_t)in * b;
    const int last = total - 1 - t.j;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        (void *)base, (short)0, (int)((uint32_t)(last < kKeys ? last : kKeys - 1) * b + D * 2), 0x00020000);
    bf16 *dw = dst + wave * RPI * D;
    if (__builtin_expect(last >= kKeys - 1, 1)) {
#pragma unroll
      for (int i = 0; i < LPT; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(dw + i * NW * RPI * D), 16, vo,
                                                 (uint32_t)(i * NW * RPI) * b, 0, 0);
    } else {  // rows behind the end are read as the last
#pragma unroll
      for (int i = 0; i < LPT; ++i) {
        const int r = lrow + i * NW * RPI;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(dw + i * NW * RPI * D), 16,
                                                 (uint32_t)(r < last ? r : last) * b + lchunk, 0, 0, 0);
      }
    }
  };

  // ---- products ------------------------------------------------------------------------------------------------------
  const int kswz = swz<D>(l32);
  const int g16 = lane >> 4, i16 = lane & 15, vrow = 4 * hh + (i16 >> 2);
  const int vsw0 = swz<D>(vrow), vsw1 = swz<D>(vrow + 8);
  int voff[DB], voff1[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int d0 = 32 * db + 16 * (g16 & 1) + 4 * (i16 & 3);
    voff[db] = vrow * D + (((d0 >> 3) ^ vsw0) << 3) + (d0 & 7);
    voff1[db] = (vrow + 8) * D + (((d0 >> 3) ^ vsw1) << 3) + (d0 & 7);
  }
  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;  // in units of the logits; this lane's half of the states
  const float cs = own(a0->q.c);

  // element r of s[mb]: state 32 mb + 8 (r / 4) + 4 hh + r % 4
  auto qk = [&](f32x16 (&s)[2], const bf16 *sK, const float *sB, bool part) RS_INLINE {
#pragma unroll
    for (int mb = 0; mb < 2; ++mb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mb][r] = 0.f;
    if (MASK && part)
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 b = *(const f32x4 *)&sB[32 * mb + 8 * i + 4 * hh];
#pragma unroll
          for (int e = 0; e < 4; ++e) s[mb][4 * i + e] = b[e];
        }
    auto read = [&](int f) RS_INLINE { return *(const u32x4 *)&sK[(32 * (f & 1) + l32) * D + (((2 * (f >> 1) + hh) ^ kswz) << 3)]; };
    u32x4 kb[KPF];
#pragma unroll
    for (int f = 0; f < KPF; ++f) kb[f] = read(f);
#pragma unroll
    for (int f = 0; f < 2 * KS; ++f) {
      s[f & 1] = mfma32(kb[f % KPF], qf[f >> 1], s[f & 1]);
      if (f + KPF < 2 * KS) kb[f % KPF] = read(f + KPF);
    }
    // (the compiler puts each read right before its product otherwise: 4050 -> 3970 us)
    __builtin_amdgcn_sched_group_barrier(0x100, KPF, 0);
#pragma unroll
    for (int f = 0; f < 2 * KS - KPF; ++f) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, KPF, 0);
  };
  u32x4 pb[2][2];
  auto weigh = [&](const f32x16 (&s)[2], float nmc) RS_INLINE -> float {
    float z = 0.f;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mb][8 * h + 2 * w], cs, nmc));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mb][8 * h + 2 * w + 1], cs, nmc));
          z += p0;
          z += p1;
          // P is rounded to bf16 for the product: half a step of each weight, as much as O's own rounding
          pb[mb][h][w] = pack_bf16x2(p0, p1);
        }
    return z;
  };
  auto pv = [&](const bf16 *sV) RS_INLINE {
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
      auto read = [&](int f) RS_INLINE {
        const int h = f / DB, db = f % DB;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16 *)(sV + voff[db] + (32 * mb + 16 * h) * D)));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16 *)(sV + voff1[db] + (32 * mb + 16 * h) * D)));
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
      };
      u32x4 vb[VPF];
#pragma unroll
      for (int f = 0; f < VPF; ++f) vb[f] = read(f);
#pragma unroll
      for (int f = 0; f < 2 * DB; ++f) {
        oacc[f % DB] = mfma32(vb[f % VPF], pb[mb][f / DB], oacc[f % DB]);
        if (f + VPF < 2 * DB) vb[f % VPF] = read(f + VPF);
      }
    }
  };

  // the weights of a tile from its scores: raises the running maximum and rescales what it must, adds to the sum
  auto soften = [&](const f32x16 (&sc)[2]) RS_INLINE {
    float z = weigh(sc, m_run == -INFINITY ? 0.f : -m_run * cs);
    const uint64_t want = __ballot(!(z <= 256.f) || m_run == -INFINITY);
    if (want != 0ull) {
      float mx = -INFINITY;
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[mb][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (((want >> l32) | (want >> (l32 + 32))) & 1ull) {  // both lanes of a row decide alike
        const float m_new = fmaxf(m_run, mx);
        if (m_new > m_run) {
          const float al = __builtin_amdgcn_exp2f((m_run - m_new) * cs);  // 0 for m_run = -inf
          l_run *= al;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[db][r] *= al;
          m_run = m_new;
        }
      }
      z = weigh(sc, m_run == -INFINITY ? 0.f : -m_run * cs);
    }
    l_run += z;
  };
  // zeroes the rows of a tile that are not seen
  auto hide_rows = [&](bf16 *t, uint64_t see) RS_INLINE {
    if (!(see >> (tid >> 2) & 1))
#pragma unroll
      for (int i = 0; i < D / 32; ++i) *(u32x4 *)(t + (tid >> 2) * D + ((tid & 3) * (D / 32) + i) * 8) = u32x4{0u, 0u, 0u, 0u};
  };
  auto hide_keys = [&](float *sB, const CrossTile &t) RS_INLINE {
    if (MASK && t.j >= 0 && partly(t) && tid < kKeys) sB[tid] = seen(t) >> tid & 1 ? 0.f : -INFINITY;
  };

  // ---- one step: softmax and P V of tile tc, then the products of tile tn --------------------------------------------
  // s holds S^T of tc; after the barrier K of tn (kn) and V of tc (vc) are there, and kc and vn are free.
  CrossTile tc = next(), tn{-1, 0, 0};
  // one S where d = 128 (registers): 4 % faster with two where d = 64, 2 % slower where d = 128
  f32x16 s0[2], s1[D == 64 ? 2 : 1];
  auto other = [&]() RS_INLINE -> f32x16 (&)[2] {
    if constexpr (D == 64) return s1;
    else return s0;
  };
  auto step = [&](f32x16 (&s)[2], f32x16 (&sn)[2], bf16 *kc, bf16 *kn, bf16 *vc, bf16 *vn, float *bc, float *bn) RS_INLINE {
    tile_barrier();
    CrossTile t2{-1, 0, 0};
    if (tn.j >= 0) t2 = next();
    if (t2.j >= 0) copy(kc, t2, false);
    if (tn.j >= 0) copy(vn, tn, true);
    hide_keys(bc, t2);
    if constexpr (SAFE) {
      hide_rows(vc, seen(tc));
      if (tn.j >= 0) hide_rows(kn, seen(tn));
      lds_barrier();
    }
    if (!MASK && partly(tc)) {
      // the last tile (a scalar pair holds an element's decision for all lanes: the states of lanes 32 .. 63 lie 4 behind)
      const uint64_t see = seen(tc);
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int x = 32 * mb + 8 * (r >> 2) + (r & 3);
          const uint64_t lanes = (uint64_t)(uint32_t)((int)((uint32_t)(see >> (x + 4)) << 31) >> 31) << 32 | (uint32_t)((int)((uint32_t)(see >> x) << 31) >> 31);
          s[mb][r] = __builtin_amdgcn_inverse_ballot_w64(lanes) ? s[mb][r] : -INFINITY;
        }
    }
    soften(s);
    __builtin_amdgcn_s_setprio(1);  // matrix instructions first: the other workgroup's exponents fill their gaps
    pv(vc);
    if (tn.j >= 0) qk(sn, kn, bn, partly(tn));
    __builtin_amdgcn_s_setprio(0);
    tc = tn;
    tn = t2;
  };
  if (tc.j >= 0) {
    copy(lds.K0, tc, false);
    copy(lds.V0, tc, true);
    tn = next();
    if (tn.j >= 0) copy(lds.K1, tn, false);
    hide_keys(lds.B0, tc);
    hide_keys(lds.B1, tn);
    tile_barrier();
    if constexpr (SAFE) {
      hide_rows(lds.K0, seen(tc));
      lds_barrier();
    }
    qk(s0, lds.K0, lds.B0, partly(tc));
    while (true) {
      step(s0, other(), lds.K0, lds.K1, lds.V0, lds.V1, lds.B0, lds.B1);
      if (tc.j < 0) break;
      step(other(), s0, lds.K1, lds.K0, lds.V1, lds.V0, lds.B1, lds.B0);
      if (tc.j < 0) break;
    }
  }
  if constexpr (!SAFE) {
    bool odd = !(l_run < INFINITY);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) odd = odd || !(__builtin_fabsf(oacc[db][r]) < INFINITY);
    if (tid == 0) *lds.odd = 0;
    lds_barrier();
    if (odd) *lds.odd = 1;
    lds_barrier();
    if (__builtin_expect(uniform(*lds.odd), 0)) return false;
  }

  // ---- the end: lane (row, hh) holds dimensions 32 db + 8 i + 4 hh .. + 3 ---------------------------------------------
  const float z = l_run + __shfl_xor(l_run, 32);
  asm volatile("" : "+v"(tid));  // (places are computed again, not kept)
  const ArgsPtr a = args_here();
  const int h2 = (tid & 63) >> 5, in = 32 * (tid >> 6) + (tid & 31), G = a->q.hq / a->c.hkv, row = r0 + in;
  if (row >= G * it.t) return true;
  if (it.npieces > 1) {
    const int64_t at = (int64_t)(it.slot0 + it.piece * it.per + it.rt * a->c.hkv + it.g) * kRows + in;
    float *po = a->po + at * D + 4 * h2;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4 *)(po + 32 * db + 8 * i) = f32x4{oacc[db][4 * i], oacc[db][4 * i + 1], oacc[db][4 * i + 2], oacc[db][4 * i + 3]};
    if (h2 == 0) {
      a->pml[at * 2] = m_run * cs;  // (the joining kernel's maxima are those of the exponents of 2)
      a->pml[at * 2 + 1] = z;
    }
    return true;
  }
  const int tok = row / G, head = it.g * G + row - tok * G;
  const float inv = z > 0.f ? 1.f / z : z == 0.f ? 0.f : z;
  bf16 *o = (bf16 *)a->o + (it.first + tok) * a->so_t + head * a->so_h + 4 * h2;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(u32x2 *)(o + 32 * db + 8 * i) = u32x2{pack_bf16x2(oacc[db][4 * i] * inv, oacc[db][4 * i + 1] * inv),
                                              pack_bf16x2(oacc[db][4 * i + 2] * inv, oacc[db][4 * i + 3] * inv)};
  if (a->lse && h2 == 0)
    a->lse[(int64_t)head * a->q.nrows + it.first + tok] = z == 0.f ? -INFINITY : (m_run * cs + __builtin_amdgcn_logf(z)) * kLn2;
  return true;
}

template <int D, bool MASK>
__global__ __launch_bounds__(256, 2) void cross_kernel(const DraftArgs) {
  __shared__ __align__(16) bf16 sK0[kKeys * D], sK1[kKeys * D], sV0[kKeys * D], sV1[kKeys * D];
  __shared__ __align__(16) float sB0[kKeys], sB1[kKeys];
  __shared__ int sOdd;
  const int lane = threadIdx.x & 63;
  Item it;
  {
    const DraftArgs a = *(const DraftArgs *)(const void *)args_here();
    const Seq first = seq_at<W_CROSS>(a, lane);
    const int groups = plan_rounds(a, first, lane);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.plan = groups;
    if (!find_piece<W_CROSS>(a, first, groups, blockIdx.x, lane, it)) return;
  }
  it = uniform(it);
  const CrossLds<D> lds{sK0, sK1, sV0, sV1, sB0, sB1, &sOdd};
  if (!cross_walk<D, MASK, false>(it, lds)) cross_walk<D, MASK, true>(it, lds);
}

// Joins the pieces of an item, 32 of its rows per workgroup (grid: items x trows / 32), for this kernel and for those of decode.hip
// that share stages: where there are many rows, of which each would plan for itself there.  A row's D / 4 lanes hold 4 dimensions.
template <int D>
__global__ __launch_bounds__(256) void cross_join_kernel(const DraftArgs a) {
  constexpr int LPR = D / 4, RPI = 256 / LPR, kAhead = 8;
  const int lane = threadIdx.x & 63;
  const Seq head_of = seq_at<W_CROSS>(a, lane);
  const int groups = a.plan ? *a.plan : plan_groups<W_CROSS>(a, head_of, lane);
  int id = blockIdx.x, slot = -1, np = 0, per = 0, first = 0, t = 0, base = 0;
  for (int b0 = 0; b0 < a.c.nseq && slot < 0; b0 += 64) {
    const Seq q = b0 ? seq_at<W_CROSS>(a, b0 + lane) : head_of;
    const int k = q.r.count > 0 ? pieces_of(q.groups, groups) : 0, n = q.r.count > 0 ? items_of<W_CROSS>(a, q) : 0;
    const int si = wave_scan(n), ss = wave_scan(k * n);
    const unsigned long long hit = __ballot(id < si);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      np = __builtin_amdgcn_readlane(k, l);
      per = __builtin_amdgcn_readlane(n, l);
      first = __builtin_amdgcn_readlane(q.r.first, l);
      t = __builtin_amdgcn_readlane(q.r.count, l);
      id -= __builtin_amdgcn_readlane(si, l) - per;  // the item among its sequence's: row tile, then head
      slot = base + __builtin_amdgcn_readlane(ss, l) - np * per + id;
    }
    id -= hit ? 0 : __builtin_amdgcn_readlane(si, 63);
    base += __builtin_amdgcn_readlane(ss, 63);
  }
  // (sequences that share rows, which start does not allow, may have more pieces than there are workgroups)
  if (np <= 1 || slot + (np - 1) * per >= a.grid) return;
  const int rt = id / a.c.hkv, g = id - rt * a.c.hkv, G = a.q.hq / a.c.hkv;
  const int d0 = threadIdx.x % LPR * 4;
  for (int x = 0; x < 32; x += RPI) {
    const int in = blockIdx.y * 32 + x + threadIdx.x / LPR, row = rt * a.trows + in;
    if (row >= G * t) return;
    const float *pml = a.pml + ((int64_t)slot * a.trows + in) * 2, *po = a.po + ((int64_t)slot * a.trows + in) * D + d0;
    const int64_t step = (int64_t)per * a.trows;
    // in one pass, with a running maximum: kAhead pieces are in flight at a time
    float M = -INFINITY, z = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < np; k0 += kAhead) {
      f32x4 p[kAhead];
      float m[kAhead], s[kAhead], top = M;
#pragma unroll
      for (int y = 0; y < kAhead; ++y) {
        const int64_t k = k0 + y < np ? k0 + y : k0;
        p[y] = *(const f32x4 *)(po + k * step * D);
        m[y] = pml[k * step * 2], s[y] = pml[k * step * 2 + 1];
      }
#pragma unroll
      for (int y = 0; y < kAhead; ++y) top = fmaxf(top, m[y]);
      const float ref = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f(M - ref);
      z *= old;
      v *= old;
      M = top;
#pragma unroll
      for (int y = 0; y < kAhead; ++y) {
        if (k0 + y >= np) break;
        const float w = __builtin_amdgcn_exp2f(m[y] - ref);
        z += s[y] * w;
        if (m[y] != -INFINITY) v += p[y] * w;  // (of a piece that saw nothing O is zero; of one of NaN alone z says so)
      }
    }
    const int tok = row / G, head = g * G + row - tok * G;
    const float inv = z > 0.f ? 1.f / z : z == 0.f ? 0.f : z;
    *(u32x2 *)((bf16 *)a.o + (first + tok) * a.so_t + head * a.so_h + d0) = u32x2{pack_bf16x2(v[0] * inv, v[1] * inv), pack_bf16x2(v[2] * inv, v[3] * inv)};
    if (a.lse && d0 == 0)
      a.lse[(int64_t)head * a.q.nrows + first + tok] = z == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(z)) * kLn2;
  }
}

}  // namespace

void cross_prompt_launch(const DraftArgs &a, int d, hipStream_t st) {
  if (a.q.mask) d == 128 ? cross_kernel<128, true><<<a.grid, 256, 0, st>>>(a) : cross_kernel<64, true><<<a.grid, 256, 0, st>>>(a);
  else d == 128 ? cross_kernel<128, false><<<a.grid, 256, 0, st>>>(a) : cross_kernel<64, false><<<a.grid, 256, 0, st>>>(a);
}

void cross_join_launch(const DraftArgs &a, int d, int items, hipStream_t st) {
  const dim3 grid(items, a.trows / 32);
  d == 128 ? cross_join_kernel<128><<<grid, 256, 0, st>>>(a) : cross_join_kernel<64><<<grid, 256, 0, st>>>(a);
}

}  // namespace rs
