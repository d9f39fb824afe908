// Kernels of softmax-free attention on ciphertexts: weighted sums of rotations in the extended basis (rotary positions, slot
// sums, the giant steps of a state's read) and sums of ciphertext products (scores, the state's update and read).
#pragma once
#include "ntt16_kernels.hip.h"
#include "radix4.hip.h"

#define ROT_SUM_TERMS 32   // terms per launch (they travel in the kernel's arguments)

// acc[b][c][t][n] = P w_0[t][n] base[b][c][t][n] (main primes only)
//                 + sum_r w_r[t][n] ( sum_j D_rj[pi_r(n)] evk_r[j][c][id(t)][n] + [c = 0, main primes] P c0_r[b][t][pi_r(n)] ),
// pi_r the evaluation-domain index map of term r. D_rj is digit j of the term's polynomial in the extended basis: d_r itself on
// the limbs that the digit holds, the transformed conversions in ext_r elsewhere. Without weights every w is one. On integer
// moduli acc carries the factor 2^-64 that ModDown's constants expect there (not on rings that go one kernel per step). A launch computes `outs` such
// sums from nterms terms each, the accumulators one after another; base belongs to the first.
struct RotTerm {
  const u64* ext;   // [B][beta][next][N]
  const u64* d;     // limb-vector (b, t) at d + b*d_stride + t*N
  const u64* c0;    // like d; null: no such addend
  const u64* evk;   // [dnum][2][nm][N]
  u32 galois;
};
struct RotSumArgs {
  const u64* base;      // null: none; component c of ciphertext b at base + b*base_stride + c*nlimbs*N
  u64 base_stride;
  const u64* w;         // null: none; weight of term r of set s at w + ((s*w_terms + r + 1)*next + t)*N, of base at r = -1
  u64* acc;             // [outs][B][2][next][N]
  const ModInfo* mods;
  u64 d_stride;
  u32 logN, nlimbs, nq, nm, alpha, beta, next, B, nterms, w_first, w_terms, per_set, accumulate, nfp;
  u32 doubles;          // != 0: ext holds doubles on moduli below 2^50
  // block_sum_kernel, FUSED: twiddles; integer slots from first_special on go through their inverse block pass if `inverse` says so
  const ulonglong2 *tw = nullptr, *twi = nullptr;
  const double* twfp = nullptr;
  u32 first_special = 0, inverse = 0;
  // fin_tq != null: main limbs are finished, out = (sum - NTT(tq)) pinv, instead of stored; tq after the first pass of its transform
  const u64* fin_tq = nullptr;   // [B][2][fin_limbs][N]
  u64* fin_out = nullptr;        // [B][2][fin_limbs][N]
  const ulonglong2* fin_pinv = nullptr;
  u32 fin_limbs = 0;
  unsigned char slots[128];
  RotTerm term[ROT_SUM_TERMS];
};

// Workgroup -> (what: ciphertexts or outputs, block of positions, limb), so that everything that reads the same positions of a limb
// (key and weight slices, factors of many products) runs on one XCD, one after another, and finds them in its L2.
__device__ __forceinline__ void attention_map(u32& what, u32& blk, u32& zi) {
  const u32 lin = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z), units = gridDim.y * gridDim.z, whole = units & ~7u;
  u32 unit;
  if (lin < whole * gridDim.x) {
    const u32 rest = lin >> 3;
    what = rest % gridDim.x;
    unit = (lin & 7) + 8 * (rest / gridDim.x);
  } else {
    const u32 rest = lin - whole * gridDim.x;
    what = rest % gridDim.x;
    unit = whole + rest / gridDim.x;
  }
  blk = unit % gridDim.y;
  zi = unit / gridDim.y;
}

// Moduli below 2^50 where ext holds doubles: sums in doubles (|.| < 2^53 = 8q throughout). A lane owns a position of CB ciphertexts, which
// share the key words, and asks for the next digit while it multiplies this one. What bounds it is the wait for the gathers: two
// rotations of 16 ciphertexts of 20 limbs, 4 digits, 492 us, 2.6 GB (5.2 TB/s), vector units 40 % busy. CB = 2: with 4 there are fewer
// waves (7 % longer), with 1 every ciphertext fetches the keys again (24 %); nothing asked ahead 526 us, a whole term ahead 550.
// Both terms side by side in the order of the Galois map's orbits halve the HBM reads (1.2 GB) and take 593 us; four
// ciphertext pairs of the same positions in a workgroup ask the L2 for a third less, 559; by (ciphertexts, limb) on an XCD 504.
// grid = (outs * ceil(B / CB), N / 256, slots).
template <int CB>
__device__ __forceinline__ void rot_sum_fp(const RotSumArgs& a, u32 what, u32 blk, u32 zi) {
  const size_t N = (size_t)1 << a.logN, pl = (size_t)a.nlimbs * N, comp = (size_t)a.nm * N;
  const u32 groups = (a.B + CB - 1) / CB, o = what / groups, b0 = (what % groups) * CB;
  const u32 n = blk * 256 + threadIdx.x, t = a.slots[zi];
  const bool main_prime = t < a.nlimbs;
  const u32 id = main_prime ? t : t - a.nlimbs + a.nq;
  const ModInfo mi = a.mods[id];
  const double q = mi.qd, qinv = mi.qinv, pm = u2d(mi.pmod);
  u32 bb[CB];   // surplus places repeat the last ciphertext and store nothing
  const u64* w[CB];
  double s0[CB], s1[CB];
#pragma unroll
  for (int k = 0; k < CB; k++) {
    bb[k] = min(b0 + k, a.B - 1);
    w[k] = a.w ? a.w + (((size_t)(bb[k] / a.per_set) * a.w_terms + a.w_first) * a.next + t) * N : nullptr;
    s0[k] = s1[k] = 0.0;
    if (a.base && main_prime && o == 0) {
      const u64* x = a.base + (size_t)bb[k] * a.base_stride + (size_t)t * N + n;
      const double f = a.w ? fp_mulmod_var(pm, u2d(w[k][n]), qinv, q) : pm;
      s0[k] = fp_mulmod_var(u2d(x[0]), f, qinv, q);
      s1[k] = fp_mulmod_var(u2d(x[pl]), f, qinv, q);
    }
  }
  const u32 jo = main_prime ? t / a.alpha : 0xFFFFFFFFu;   // the digit that holds limb t itself
  for (u32 r = 0; r < a.nterms; r++) {
    const RotTerm& term = a.term[o * a.nterms + r];
    const u32 m = galois_src_index(n, term.galois, a.logN);
    const u64* e = uniform_ptr(term.evk) + (size_t)id * N;
    const u64 *ext = uniform_ptr(term.ext), *d = uniform_ptr(term.d), *c0 = term.c0 ? uniform_ptr(term.c0) : nullptr;
    u64 cw[CB], ww[CB];
#pragma unroll
    for (int k = 0; k < CB; k++) {
      cw[k] = c0 && main_prime ? uniform_load(c0 + (size_t)bb[k] * a.d_stride + (size_t)t * N, m * 8) : 0;
      ww[k] = a.w ? uniform_load(w[k] + (size_t)(r + 1) * a.next * N, n * 8) : 0;
    }
    double v0[CB], v1[CB];
#pragma unroll
    for (int k = 0; k < CB; k++) v0[k] = v1[k] = 0.0;
    u64 xn[CB], kn[2];
    auto request = [&](u32 j) {
      const bool own = j == jo;   // uniform: where the digit's words start, and how far its ciphertexts are apart
      const u64* x = own ? d + (size_t)t * N : ext + ((size_t)j * a.next + t) * N;
      const size_t apart = own ? (size_t)a.d_stride : (size_t)a.beta * a.next * N;
#pragma unroll
      for (int k = 0; k < CB; k++) xn[k] = uniform_load(x + bb[k] * apart, m * 8);
      kn[0] = uniform_load(e, n * 8), kn[1] = uniform_load(e + comp, n * 8);
      e += 2 * comp;
    };
    request(0);
    for (u32 j = 0; j < a.beta; j++) {
      u64 xr[CB];
#pragma unroll
      for (int k = 0; k < CB; k++) xr[k] = xn[k];
      const double e0 = u2d(kn[0]), e1 = u2d(kn[1]);
      if (j + 1 < a.beta) request(j + 1);
      __builtin_amdgcn_sched_barrier(0);
      // residues become doubles by setting the exponent and taking 2^52 away, doubles stay what they are
      const u64 bias = j == jo ? 0x4330000000000000ull : 0ull;
      const double less = __longlong_as_double((long long)bias);
#pragma unroll
      for (int k = 0; k < CB; k++) {
        const double v = __longlong_as_double((long long)(xr[k] | bias)) - less;
        v0[k] += fp_mulmod_var(v, e0, qinv, q);
        v1[k] += fp_mulmod_var(v, e1, qinv, q);
        if ((j & 3) == 3) v0[k] = fp_reduce(v0[k], qinv, q), v1[k] = fp_reduce(v1[k], qinv, q);   // 4 products below 0.9 q, a folded sum
      }
    }
#pragma unroll
    for (int k = 0; k < CB; k++) {
      if (c0 && main_prime) v0[k] += fp_mulmod_var(u2d(cw[k]), pm, qinv, q);
      v0[k] = fp_reduce(v0[k], qinv, q);
      v1[k] = fp_reduce(v1[k], qinv, q);
      if (a.w) {
        const double f = u2d(ww[k]);
        v0[k] = fp_mulmod_var(v0[k], f, qinv, q);
        v1[k] = fp_mulmod_var(v1[k], f, qinv, q);
      }
      s0[k] = fp_reduce(s0[k] + v0[k], qinv, q);
      s1[k] = fp_reduce(s1[k] + v1[k], qinv, q);
    }
  }
#pragma unroll
  for (int k = 0; k < CB; k++) {
    if (b0 + k >= a.B) break;
    u64* to = a.acc + (((size_t)o * a.B + bb[k]) * 2 * a.next + t) * N + n;
    if (a.accumulate) s0[k] += u2d(to[0]), s1[k] += u2d(to[(size_t)a.next * N]);
    to[0] = d2u_canon(fp_reduce(s0[k], qinv, q), q);
    to[(size_t)a.next * N] = d2u_canon(fp_reduce(s1[k], qinv, q), q);
  }
}

// All other moduli: residues in ext, Montgomery products, sums below 2m. PLAIN: acc without the factor 2^-64. Grid and lanes as above. A
// position, ciphertext and rotation with 4 digits takes 11 Montgomery products on a special limb (8 with keys, 2 with the weight, 1 that
// prepares it) and 12 on a main one, 10 multiplies each. They cost little on top of the gathers that double-precision limbs wait for: the
// rotations above with 25 limbs of this kind 620 us, with 25 doubles 570, with 20 doubles and 5 special limbs of this kind 575. In
// 128-bit sums with a reduction each the 5 special limbs alone took 163, this way 130.
template <int CB, bool PLAIN>
__device__ __forceinline__ void rot_sum_int(const RotSumArgs& a, u32 what, u32 blk, u32 zi) {
  const size_t N = (size_t)1 << a.logN, pl = (size_t)a.nlimbs * N, comp = (size_t)a.nm * N;
  const u32 groups = (a.B + CB - 1) / CB, o = what / groups, b0 = (what % groups) * CB;
  const u32 n = blk * 256 + threadIdx.x, t = a.slots[zi];
  const bool main_prime = t < a.nlimbs;
  const u32 id = main_prime ? t : t - a.nlimbs + a.nq;
  const ModInfo mi = a.mods[id];
  const u64 q = mi.m, q2 = 2 * mi.m, r2 = a.w || PLAIN ? mont_r2(mi) : 0;
  u32 bb[CB];
  const u64* w[CB];
  u64 s0[CB], s1[CB];
#pragma unroll
  for (int k = 0; k < CB; k++) {
    bb[k] = min(b0 + k, a.B - 1);
    w[k] = a.w ? a.w + (((size_t)(bb[k] / a.per_set) * a.w_terms + a.w_first) * a.next + t) * N + n : nullptr;
    s0[k] = s1[k] = 0;
    if (a.base && main_prime && o == 0) {
      const u64* x = a.base + (size_t)bb[k] * a.base_stride + (size_t)t * N + n;
      const u64 f = a.w ? mont_plain(*w[k], mi.pmod, r2, q, mi.minv) : mi.pmod;
      s0[k] = mont_mul63(x[0], f, q, mi.minv);   // below 2m, with the factor 2^-64 like everything below
      s1[k] = mont_mul63(x[pl], f, q, mi.minv);
    }
  }
  const u32 jo = main_prime ? t / a.alpha : 0xFFFFFFFFu;
  for (u32 r = 0; r < a.nterms; r++) {
    const RotTerm& term = a.term[o * a.nterms + r];
    const u32 m = galois_src_index(n, term.galois, a.logN);
    const u64* e = term.evk + (size_t)id * N + n;
    u64 v0[CB], v1[CB];
#pragma unroll
    for (int k = 0; k < CB; k++) {
      v0[k] = v1[k] = 0;
      if (term.c0 && main_prime) v0[k] = mont_mul63(term.c0[(size_t)bb[k] * a.d_stride + (size_t)t * N + m], mi.pmod, q, mi.minv);
    }
    u64 xn[CB], kn[2];
    auto request = [&](u32 j) {
#pragma unroll
      for (int k = 0; k < CB; k++)
        xn[k] = j == jo ? term.d[(size_t)bb[k] * a.d_stride + (size_t)t * N + m]
                        : term.ext[(((size_t)bb[k] * a.beta + j) * a.next + t) * N + m];
      kn[0] = e[0], kn[1] = e[comp];
      e += 2 * comp;
    };
    request(0);
    for (u32 j = 0; j < a.beta; j++) {
      u64 x[CB];
#pragma unroll
      for (int k = 0; k < CB; k++) x[k] = xn[k];
      const u64 e0 = kn[0], e1 = kn[1];
      if (j + 1 < a.beta) request(j + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < CB; k++) {
        v0[k] = csub(v0[k] + mont_mul63(x[k], e0, q, mi.minv), q2);
        v1[k] = csub(v1[k] + mont_mul63(x[k], e1, q, mi.minv), q2);
      }
    }
#pragma unroll
    for (int k = 0; k < CB; k++) {
      if (a.w) {   // the weight times 2^64 makes up for this product's factor
        const u64 f = csub(mont_mul63(w[k][(size_t)(r + 1) * a.next * N], r2, q, mi.minv), q);
        v0[k] = mont_mul63(v0[k], f, q, mi.minv);
        v1[k] = mont_mul63(v1[k], f, q, mi.minv);
      }
      s0[k] = csub(s0[k] + v0[k], q2);
      s1[k] = csub(s1[k] + v1[k], q2);
    }
  }
#pragma unroll
  for (int k = 0; k < CB; k++) {
    if (b0 + k >= a.B) break;
    u64* to = a.acc + (((size_t)o * a.B + bb[k]) * 2 * a.next + t) * N + n;
    if (PLAIN) s0[k] = mont_mul63(s0[k], r2, q, mi.minv), s1[k] = mont_mul63(s1[k], r2, q, mi.minv);
    if (a.accumulate) s0[k] = csub(s0[k] + to[0], q2), s1[k] = csub(s1[k] + to[(size_t)a.next * N], q2);
    to[0] = csub(s0[k], q);
    to[(size_t)a.next * N] = csub(s1[k], q);
  }
}

// KIND 0: slots of both arithmetic kinds, the first nfp of them double-precision ones; 1: integer ones only; 2: every slot, PLAIN. Both
// kinds share a launch, whose integer workgroups (bound by their products) run into the tail of the others (bound by their gathers), and
// a launch costs more than the registers of the other kind. us, one launch | two: two rotations of 4 ciphertexts of 5 limbs at 2^13
// 62 | 70, of 4 of 24 limbs at 2^16 512 | 524, of 16 of 20 limbs 1653 | 1664; with the kinds mixed block by block 61, 519, 1745.
template <int KIND, int CB>
__global__ void __launch_bounds__(256) rot_sum_kernel(RotSumArgs a) {
  u32 what, blk, zi;
  attention_map(what, blk, zi);
  if (KIND == 0 && zi < a.nfp) rot_sum_fp<CB>(a, what, blk, zi);
  else rot_sum_int<CB, KIND == 2>(a, what, blk, zi);
}

// The unweighted sum of rotations of one decomposition (all terms have the same ext, d, c0) whose Galois maps keep every aligned block of
// 256 positions: g = 1 mod 2N / 256, which all rotations by multiples of the stride are where a head of at most 256 components fills the
// slots. A workgroup takes such a block of CB ciphertexts, puts a digit into LDS once and reads it there for every rotation; a lane owns a
// position and shares the key words among its ciphertexts.
// Doubles: digits within q / 2, key words below q < 2^50, so that four products stay within 2^101 of H = 1.5 * 2^102, in whose binade
// sums are multiples of 2^50 and what a product loses in joining H is exact and goes to L: 4 instructions a term, 6 every fourth.
// 26 ciphertexts of 8 + 3 limbs at 2^16 by 7 rotations and by 7 again took 1337 us in rot_sum_kernel, which fetches a digit's words from
// the caches once for every rotation, and the digits' last passes; in here 981, with the key words requested 4 rotations ahead 850 (6: the
// same; moved through registers instead of an unrolled walk: slower). Four ciphertexts a lane share the key words and take 119 registers:
// two a lane in the integer launches cost 1345 us where four take 1303, and 580 for 552 (64 scores of 7 limbs); tiles of four digits at a
// time (178 registers) 1088 for 981. What bounds it is issue: 8 double-precision instructions a term beside the butterflies, at 2 to 3 TB/s.
#define BLOCK_SUM 256
// The last 8 stages of a transform on a block of 256 elements in one wave, four values a lane: round K (stages 2K, 2K + 1 of the block)
// holds in lane l the elements (l / S) 4S + i S + l % S, S = 64 >> 2K.
__device__ __forceinline__ u32 block_lane() {   // hidden, so that what is derived from it is not kept in registers from digit to digit
  u32 l = threadIdx.x & 63;
  asm volatile("" : "+v"(l));
  return l;
}
__device__ __forceinline__ u32 block_elem(int K, u32 i, u32 l) {
  const u32 s = 6 - 2 * K;
  return ((l >> s) << (s + 2)) + (i << s) + (l & ((1u << s) - 1));
}
template <int FROM, int TO, class T>
__device__ __forceinline__ void block_exchange(T (&x)[4], T* blk) {
  const u32 l = block_lane();
#pragma unroll
  for (int i = 0; i < 4; i++) blk[wl_word(block_elem(FROM, i, l))] = x[i];
  wave_lds_sync();
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = blk[wl_word(block_elem(TO, i, l))];
  wave_lds_sync();
  __builtin_amdgcn_sched_barrier(0);
}
// Twiddles of block h of R, stage s, group g at (1 << s) - 1 + g.
template <class TW>
__device__ __forceinline__ void block_twiddles_fetch(TW* tws, const TW* __restrict__ tw, u32 h, u32 R) {
  const u32 t = min(threadIdx.x, 254u), s = 31 - __clz(t + 1);
  tws[t] = tw[(R << s) + (h << s) + (t + 1 - (1u << s))];
}
template <class TW>
__device__ __forceinline__ void block_twiddles(TW (&w)[3], const TW* tws, int K) {
  const u32 g = block_lane() >> (6 - 2 * K);
  w[0] = tws[(1u << (2 * K)) - 1 + g];
  w[1] = tws[(2u << (2 * K)) - 1 + 2 * g];
  w[2] = tws[(2u << (2 * K)) + 2 * g];
}
// In: round 0's elements, at most 2.64 q (integers: below 16q, SMALL 33q). Out: round 3's, reduced (canonical).
__device__ __forceinline__ void block_forward(double (&x)[4], const double* tws, double q, double qinv, double* blk) {
  double w[3];
  block_twiddles(w, tws, 0);
  radix4_fwd(x, w, q, qinv);
  block_exchange<0, 1>(x, blk);
  block_twiddles(w, tws, 1);
  radix4_fwd(x, w, q, qinv);
  reduce4(x, q, qinv);
  block_exchange<1, 2>(x, blk);
  block_twiddles(w, tws, 2);
  radix4_fwd(x, w, q, qinv);
  block_exchange<2, 3>(x, blk);
  block_twiddles(w, tws, 3);
  radix4_fwd(x, w, q, qinv);
  reduce4(x, q, qinv);
}
template <bool BIG>
__device__ __forceinline__ void block_forward(u64 (&x)[4], const ulonglong2* tws, u64 q, u64 mu, u64* blk) {
  const u64 q2 = lazy_const<BIG>(q);
  ulonglong2 w[3];
  block_twiddles(w, tws, 0);
  radix4_fwd<BIG>(x, w, q, q2);
  block_exchange<0, 1>(x, blk);
  block_twiddles(w, tws, 1);
  radix4_fwd<BIG>(x, w, q, q2);
  block_exchange<1, 2>(x, blk);
  block_twiddles(w, tws, 2);
  radix4_fwd<BIG>(x, w, q, q2);
  block_exchange<2, 3>(x, blk);
  block_twiddles(w, tws, 3);
  radix4_fwd<BIG>(x, w, q, q2);
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = csub(fwd_settle<BIG>(x[i], mu, q), q);
}
// In: round 3's elements, canonical. Out: round 0's, below 8q (SMALL 2q).
template <bool BIG>
__device__ __forceinline__ void block_inverse(u64 (&x)[4], const ulonglong2* tws, u64 q, u64 mu, u64* blk) {
  const u64 q2 = lazy_const<BIG>(q);
  ulonglong2 w[3];
  block_twiddles(w, tws, 3);
  radix4_inv<BIG>(x, w, q, q2);
  block_exchange<3, 2>(x, blk);
  block_twiddles(w, tws, 2);
  radix4_inv<BIG>(x, w, q, BIG ? q2 : q2 << 2);
  block_exchange<2, 1>(x, blk);
  block_twiddles(w, tws, 1);
  radix4_inv<BIG>(x, w, q, BIG ? q2 : q2 << 4);
  block_exchange<1, 0>(x, blk);
  block_twiddles(w, tws, 0);
  radix4_inv<BIG>(x, w, q, BIG ? q2 : q2 << 6);
  if (!BIG) {
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = barrett_lazy(x[i], mu, q);
  }
}
#define BLOCK_SUM_AHEAD 4
// Walks over the terms, digit by digit and rotation by rotation, with the key words requested BLOCK_SUM_AHEAD rotations ahead, across the
// digits' ends (what a workgroup waits for is their way from memory, which the others that share them wait for too). begin(j) puts
// digit j into LDS, term(e0, e1, m) multiplies by the words of both components what lies at index m of the block.
template <class Begin, class Term>
__device__ __forceinline__ void block_sum_terms(const RotSumArgs& a, size_t at, size_t comp, u32 n, Begin begin, Term term) {
  const u32 R = a.nterms;
  u64 k0[BLOCK_SUM_AHEAD], k1[BLOCK_SUM_AHEAD];
  auto request = [&](int u, u32 r, u32 j) {
    if (r >= R || j >= a.beta) return;   // uniform
    const u64* e = uniform_ptr(a.term[r].evk) + (size_t)j * 2 * comp + at;
    k0[u] = e[0], k1[u] = e[comp];
  };
#pragma unroll
  for (int u = 0; u < BLOCK_SUM_AHEAD; u++) request(u, u, 0);
#pragma nounroll
  for (u32 j = 0; j < a.beta; j++) {
    begin(j);
    __builtin_amdgcn_sched_barrier(0);
#pragma nounroll
    for (u32 r = 0; r < R; r += BLOCK_SUM_AHEAD) {
      const bool more = r + BLOCK_SUM_AHEAD < R;
#pragma unroll
      for (int u = 0; u < BLOCK_SUM_AHEAD; u++) {
        if (r + u >= R) break;   // uniform
        term(k0[u], k1[u], galois_src_index(n, a.term[r + u].galois, a.logN) & (BLOCK_SUM - 1));
        request(u, more ? r + BLOCK_SUM_AHEAD + u : u, more ? j : j + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (more) {   // places that the last rotations of a digit leave: the next one's
#pragma unroll
        for (int u = 0; u < BLOCK_SUM_AHEAD; u++)
          if (r + BLOCK_SUM_AHEAD + u >= R) request(u, u, j + 1);
      }
    }
  }
}
// The corrections of CB ciphertexts' accumulators at a block, transformed, to sm[2 k + c][256].
template <int CB, class Forward>
__device__ __forceinline__ void block_corrections(const RotSumArgs& a, u32 b0, u32 blk, u32 t, u64* sm, Forward forward) {
  const size_t N = (size_t)1 << a.logN;
  lds_barrier();   // what was there has been read
  for (u32 u = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); u < 2 * CB; u += 4) {
    const u32 l = block_lane();
    const u64* p = uniform_ptr(a.fin_tq + (((size_t)min(b0 + u / 2, a.B - 1) * 2 + u % 2) * a.fin_limbs + t) * N + blk * BLOCK_SUM);
    u64 x[4];
#pragma unroll
    for (u32 i = 0; i < 4; i++) x[i] = p[block_elem(0, i, l)];
    forward(x, sm + u * BLOCK_SUM);
#pragma unroll
    for (u32 i = 0; i < 4; i++) sm[u * BLOCK_SUM + block_elem(3, i, l)] = x[i];
  }
  lds_barrier();
}
// FUSED: ext comes from the first pass of the digits' transform. A wave takes a block of a ciphertext's digit through the second one on
// its way into LDS, as many digits at a time as there are waves for.
template <int CB, bool FUSED>
constexpr u32 block_sum_fill() { return !FUSED ? 1 : CB == 1 ? 4 : CB == 2 ? 2 : 1; }
// The words of a fill that a lane moves: with FUSED four of its wave's block, else one of each ciphertext.
template <int CB, bool FUSED>
struct BlockFill {
  static constexpr u32 DIGITS = block_sum_fill<CB, FUSED>(), WORDS = FUSED ? 4 : CB;
  u64 w[WORDS];
  u32 b;         // FUSED: the wave's ciphertext, and its digit among those of a fill
  u32 digit;
  bool active;
  __device__ __forceinline__ BlockFill(u32 b0, u32 B) {
    const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    digit = wave / CB;
    active = wave < DIGITS * CB;
    b = min(b0 + wave % CB, B - 1);
  }
  // ext, d: at the block's first word of ciphertext and digit 0
  __device__ __forceinline__ void request(const RotSumArgs& a, const u64* ext, const u64* d, const u32 (&bb)[CB], u32 j, u32 jo) {
    const size_t N = (size_t)1 << a.logN;
    if (FUSED) {
      const u32 jj = min(j + digit, a.beta - 1);
      const u32 l = block_lane();
      const u64* p = uniform_ptr(jj == jo ? d + (size_t)b * a.d_stride : ext + ((size_t)b * a.beta + jj) * a.next * N);
#pragma unroll
      for (u32 i = 0; i < 4; i++) w[i % WORDS] = p[block_elem(0, i, l)];
    } else {
#pragma unroll
      for (int k = 0; k < CB; k++)
        w[k % WORDS] = (j == jo ? d + (size_t)bb[k] * a.d_stride : ext + ((size_t)bb[k] * a.beta + j) * a.next * N)[threadIdx.x];
    }
  }
};
template <int CB, bool FUSED>
__device__ __forceinline__ void block_sum_fp(const RotSumArgs& a, u32 what, u32 blk, u32 zi, u64* sm, ulonglong2* tws_) {
  constexpr double M = 1.5 * 5070602400912917605986812821504.0;   // 1.5 * 2^102
  const size_t N = (size_t)1 << a.logN, pl = (size_t)a.nlimbs * N, comp = (size_t)a.nm * N;
  const u32 tid = threadIdx.x, n = blk * BLOCK_SUM + tid, t = a.slots[zi], b0 = what * CB;
  const bool main_prime = t < a.nlimbs;
  const u32 id = main_prime ? t : t - a.nlimbs + a.nq;
  const ModInfo mi = a.mods[id];
  const double q = mi.qd, qinv = mi.qinv;
  const u64 *ext = a.term[0].ext + (size_t)t * N + blk * BLOCK_SUM, *d = a.term[0].d + (size_t)t * N + blk * BLOCK_SUM;
  const u32 jo = main_prime ? t / a.alpha : 0xFFFFFFFFu;   // the digit that holds limb t itself
  u32 bb[CB];   // surplus places repeat the last ciphertext and store nothing
  double H0[CB], L0[CB], H1[CB], L1[CB];
#pragma unroll
  for (int k = 0; k < CB; k++) {
    bb[k] = min(b0 + k, a.B - 1);
    H0[k] = H1[k] = M;
    L0[k] = L1[k] = 0.0;
  }
  auto settle = [&](double& H, double& L) {
    const double h = H - M;
    L = __builtin_fma(-__builtin_rint(__builtin_fma(L, qinv, h * qinv)), q, h) + L;   // at most 1.3 q
    H = M;
  };
  typedef BlockFill<CB, FUSED> Fill;
  double *tile = (double*)sm, *digit = tile;
  Fill fill(b0, a.B);
  double* const tws = (double*)tws_;
  if (FUSED) block_twiddles_fetch(tws, a.twfp + (size_t)id * N, blk, (u32)(N / BLOCK_SUM));
  const u32 R = a.nterms;
  fill.request(a, ext, d, bb, 0, jo);
  if (FUSED) lds_barrier();
  u32 count = 0;
  block_sum_terms(
      a, (size_t)id * N + n, comp, n,
      [&](u32 j) {
        const u32 place = j % Fill::DIGITS;
        if (place == 0) {
          if (j) tile = (double*)sm + (tile == (double*)sm ? Fill::DIGITS * CB * BLOCK_SUM : 0);
          if (FUSED) {
            if (fill.active) {
              double* to = tile + (threadIdx.x >> 6) * BLOCK_SUM;
              double x[4];
              const u32 l = block_lane();
              if (j + fill.digit == jo) {   // uniform
#pragma unroll
                for (u32 i = 0; i < 4; i++) to[block_elem(0, i, l)] = fp_reduce(u2d(fill.w[i % Fill::WORDS]), qinv, q);
              } else {
#pragma unroll
                for (u32 i = 0; i < 4; i++) x[i] = __longlong_as_double((long long)fill.w[i % Fill::WORDS]);
                block_forward(x, tws, q, qinv, to);
#pragma unroll
                for (u32 i = 0; i < 4; i++) to[block_elem(3, i, l)] = x[i];
              }
            }
          } else {
            const u64 bias = j == jo ? 0x4330000000000000ull : 0ull;   // residues become doubles, doubles stay what they are
            const double less = __longlong_as_double((long long)bias);
#pragma unroll
            for (int k = 0; k < CB; k++) {
              const double v = __longlong_as_double((long long)(fill.w[k % Fill::WORDS] | bias)) - less;
              tile[k * BLOCK_SUM + tid] = j == jo ? fp_reduce(v, qinv, q) : v;
            }
          }
          lds_barrier();   // the other tile's readers are past it, since they have written this one
          if (j + Fill::DIGITS < a.beta) fill.request(a, ext, d, bb, j + Fill::DIGITS, jo);
        }
        digit = tile + place * CB * BLOCK_SUM;
      },
      [&](u64 k0, u64 k1, u32 m) {
        const double e0 = u2d(k0), e1 = u2d(k1);
#pragma unroll
        for (int k = 0; k < CB; k++) {
          const double x = digit[k * BLOCK_SUM + m];
          const double p0 = __builtin_fma(x, e0, H0[k]), h0 = p0 - H0[k];
          L0[k] += __builtin_fma(x, e0, -h0);
          H0[k] = p0;
          const double p1 = __builtin_fma(x, e1, H1[k]), h1 = p1 - H1[k];
          L1[k] += __builtin_fma(x, e1, -h1);
          H1[k] = p1;
        }
        if ((++count & 3) == 0) {
#pragma unroll
          for (int k = 0; k < CB; k++) settle(H0[k], L0[k]), settle(H1[k], L1[k]);
        }
      });
  tile = (double*)sm + (tile == (double*)sm ? Fill::DIGITS * CB * BLOCK_SUM : 0);
  if (main_prime) {   // P (base + sum of the rotated first components), P base
    double v[CB] = {};
    if (a.term[0].c0) {   // uniform
      const u64* c0 = a.term[0].c0 + (size_t)t * N + n;
#pragma unroll
      for (int k = 0; k < CB; k++) tile[k * BLOCK_SUM + tid] = u2d(c0[(size_t)bb[k] * a.d_stride]);
      lds_barrier();
      for (u32 r = 0; r < R; r++) {
        const u32 m = galois_src_index(n, a.term[r].galois, a.logN) & (BLOCK_SUM - 1);
#pragma unroll
        for (int k = 0; k < CB; k++) v[k] += tile[k * BLOCK_SUM + m];
        if ((r & 3) == 3) {
#pragma unroll
          for (int k = 0; k < CB; k++) v[k] = fp_reduce(v[k], qinv, q);
        }
      }
    }
    const double pm = u2d(mi.pmod);
#pragma unroll
    for (int k = 0; k < CB; k++) {
      settle(H0[k], L0[k]);
      settle(H1[k], L1[k]);
      if (a.base) {
        const u64* x = a.base + (size_t)bb[k] * a.base_stride + (size_t)t * N + n;
        v[k] += u2d(x[0]);
        L1[k] += fp_mulmod_var(u2d(x[pl]), pm, qinv, q);
      }
      L0[k] += fp_mulmod_var(fp_reduce(v[k], qinv, q), pm, qinv, q);
    }
  }
  const bool finish = FUSED && main_prime && a.fin_tq;   // uniform
  if (finish)
    block_corrections<CB>(a, b0, blk, t, sm, [&](u64 (&v)[4], u64* to) {
      double y[4];
#pragma unroll
      for (int i = 0; i < 4; i++) y[i] = __longlong_as_double((long long)v[i]);
      block_forward(y, tws, q, qinv, (double*)to);
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] = (u64)__double_as_longlong(y[i]);
    });
#pragma unroll
  for (int k = 0; k < CB; k++) {
    if (b0 + k >= a.B) break;
    settle(H0[k], L0[k]);
    settle(H1[k], L1[k]);
    u64* to = a.acc + ((size_t)bb[k] * 2 * a.next + t) * N + n;
    if (a.accumulate) L0[k] += u2d(to[0]), L1[k] += u2d(to[(size_t)a.next * N]);
    double r0 = fp_reduce(L0[k], qinv, q), r1 = fp_reduce(L1[k], qinv, q);
    if (finish) {
      const double2 pv = ((const double2*)a.fin_pinv)[t];
      r0 = fp_mulmod_const(r0 - __longlong_as_double((long long)sm[2 * k * BLOCK_SUM + tid]), pv.x, pv.y, q);
      r1 = fp_mulmod_const(r1 - __longlong_as_double((long long)sm[(2 * k + 1) * BLOCK_SUM + tid]), pv.x, pv.y, q);
      to = a.fin_out + ((size_t)bb[k] * 2 * a.fin_limbs + t) * N + n;
    }
    to[0] = d2u_canon(r0, q);
    to[(finish ? a.fin_limbs : a.next) * N] = d2u_canon(r1, q);
  }
}
// Integer moduli (PLAIN: all of them, acc without the factor 2^-64): 30-bit halves, 4 multiply-adds a term and carries every
// seventh.
template <int CB, bool PLAIN, bool FUSED>
__device__ __forceinline__ void block_sum_int(const RotSumArgs& a, u32 what, u32 blk, u32 zi, u64* tile, ulonglong2* tws) {
  const size_t N = (size_t)1 << a.logN, pl = (size_t)a.nlimbs * N, comp = (size_t)a.nm * N;
  const u32 tid = threadIdx.x, n = blk * BLOCK_SUM + tid, t = a.slots[zi], b0 = what * CB;
  const bool main_prime = t < a.nlimbs;
  const u32 id = main_prime ? t : t - a.nlimbs + a.nq;
  const ModInfo mi = a.mods[id];
  const u64 q = mi.m, nm = neg_opaque(q);
  const u64 *ext = a.term[0].ext + (size_t)t * N + blk * BLOCK_SUM, *d = a.term[0].d + (size_t)t * N + blk * BLOCK_SUM;
  const u32 jo = main_prime ? t / a.alpha : 0xFFFFFFFFu;
  u64* const sm = tile;
  u32 bb[CB];
  Dot30N s0[CB], s1[CB];
#pragma unroll
  for (int k = 0; k < CB; k++) {
    bb[k] = min(b0 + k, a.B - 1);
    dot30n_init(s0[k]);
    dot30n_init(s1[k]);
  }
  typedef BlockFill<CB, FUSED> Fill;
  u64* digit = tile;
  Fill fill(b0, a.B);
  const bool big = (q >> 52) != 0;   // uniform
  if (FUSED) block_twiddles_fetch(tws, a.tw + (size_t)id * N, blk, (u32)(N / BLOCK_SUM));
  const u32 R = a.nterms;
  fill.request(a, ext, d, bb, 0, jo);
  if (FUSED) lds_barrier();
  u32 count = 0;
  auto carry = [&] {
    if (++count < 7) return;
    count = 0;
#pragma unroll
    for (int k = 0; k < CB; k++) dot30n_settle(s0[k], mi.mu64, nm), dot30n_settle(s1[k], mi.mu64, nm);
  };
  block_sum_terms(
      a, (size_t)id * N + n, comp, n,
      [&](u32 j) {
        const u32 place = j % Fill::DIGITS;
        if (place == 0) {
          if (j) tile = sm + (tile == sm ? Fill::DIGITS * CB * BLOCK_SUM : 0);
          if (FUSED) {
            if (fill.active) {
              u64 *to = tile + (threadIdx.x >> 6) * BLOCK_SUM, x[4];
              const u32 l = block_lane();
#pragma unroll
              for (u32 i = 0; i < 4; i++) x[i] = fill.w[i % Fill::WORDS];
              if (j + fill.digit == jo) {   // uniform
#pragma unroll
                for (u32 i = 0; i < 4; i++) to[block_elem(0, i, l)] = x[i];
              } else {
                if (big) block_forward<true>(x, tws, q, mi.mu64, to);
                else block_forward<false>(x, tws, q, mi.mu64, to);
#pragma unroll
                for (u32 i = 0; i < 4; i++) to[block_elem(3, i, l)] = x[i];
              }
            }
          } else {
#pragma unroll
            for (int k = 0; k < CB; k++) tile[k * BLOCK_SUM + tid] = fill.w[k % Fill::WORDS];
          }
          lds_barrier();
          if (j + Fill::DIGITS < a.beta) fill.request(a, ext, d, bb, j + Fill::DIGITS, jo);
        }
        digit = tile + place * CB * BLOCK_SUM;
      },
      [&](u64 k0, u64 k1, u32 m) {
        const u32 e00 = (u32)k0 & M30, e01 = (u32)(k0 >> 30), e10 = (u32)k1 & M30, e11 = (u32)(k1 >> 30);
#pragma unroll
        for (int k = 0; k < CB; k++) {
          const u64 x = digit[k * BLOCK_SUM + m];
          const u32 x0 = (u32)x & M30, x1 = (u32)(x >> 30);
          dot30n_mac(s0[k], x0, x1, e00, e01);
          dot30n_mac(s1[k], x0, x1, e10, e11);
        }
        carry();
      });
  tile = sm + (tile == sm ? Fill::DIGITS * CB * BLOCK_SUM : 0);
  if (main_prime) {
    const u32 p0 = (u32)mi.pmod & M30, p1 = (u32)(mi.pmod >> 30);
    if (a.term[0].c0) {   // uniform
      const u64* c0 = a.term[0].c0 + (size_t)t * N + n;
#pragma unroll
      for (int k = 0; k < CB; k++) tile[k * BLOCK_SUM + tid] = c0[(size_t)bb[k] * a.d_stride];
      lds_barrier();
      for (u32 r = 0; r < R; r++) {
        const u32 m = galois_src_index(n, a.term[r].galois, a.logN) & (BLOCK_SUM - 1);
#pragma unroll
        for (int k = 0; k < CB; k++) {
          const u64 x = tile[k * BLOCK_SUM + m];
          dot30n_mac(s0[k], (u32)x & M30, (u32)(x >> 30), p0, p1);
        }
        carry();
      }
    }
    if (a.base) {
#pragma unroll
      for (int k = 0; k < CB; k++) {
        const u64* x = a.base + (size_t)bb[k] * a.base_stride + (size_t)t * N + n;
        dot30n_mac(s0[k], (u32)x[0] & M30, (u32)(x[0] >> 30), p0, p1);
        dot30n_mac(s1[k], (u32)x[pl] & M30, (u32)(x[pl] >> 30), p0, p1);
      }
    }
  }
  const bool back = FUSED && a.inverse && t >= a.first_special;   // uniform
  const bool finish = FUSED && main_prime && !back && a.fin_tq;
  if (finish)
    block_corrections<CB>(a, b0, blk, t, sm, [&](u64 (&v)[4], u64* to) {
      if (big) block_forward<true>(v, tws, q, mi.mu64, to);
      else block_forward<false>(v, tws, q, mi.mu64, to);
    });
  if (back) {
    lds_barrier();   // the tiles and the twiddles have been read
    block_twiddles_fetch(tws, a.twi + (size_t)id * N, blk, (u32)(N / BLOCK_SUM));
  }
#pragma unroll
  for (int k = 0; k < CB; k++) {
    u64* to = a.acc + ((size_t)bb[k] * 2 * a.next + t) * N + n;
#pragma unroll
    for (int c = 0; c < 2; c++) {
      Dot30N& s = c ? s1[k] : s0[k];
      dot30n_settle(s, mi.mu64, nm);
      u64 v = PLAIN ? reduce128(dot30n_value(s), mi) : csub(csub(redc(dot30n_value(s), q, mi.minv), q), q);
      u64* o = to + (size_t)c * a.next * N;
      if (a.accumulate && b0 + k < a.B) v = addmod(v, *o, q);
      if (finish) {
        const ulonglong2 pv = a.fin_pinv[t];
        v = shoup(submod(v, sm[(2 * k + c) * BLOCK_SUM + tid], q), pv.x, pv.y, q);
        o = a.fin_out + (((size_t)bb[k] * 2 + c) * a.fin_limbs + t) * N + n;
      }
      if (back) sm[(2 * k + c) * BLOCK_SUM + tid] = v;
      else if (b0 + k < a.B) *o = v;
    }
  }
  if (!back) return;
  lds_barrier();
  for (u32 u = threadIdx.x >> 6; u < 2 * CB; u += 4) {   // a wave for each accumulator of a ciphertext
    if (b0 + u / 2 >= a.B) break;
    u64 *blk_sm = sm + u * BLOCK_SUM, x[4];
    const u32 l = block_lane();
#pragma unroll
    for (u32 i = 0; i < 4; i++) x[i] = blk_sm[block_elem(3, i, l)];
    wave_lds_sync();
    if (big) block_inverse<true>(x, tws, q, mi.mu64, blk_sm);
    else block_inverse<false>(x, tws, q, mi.mu64, blk_sm);
    u64* o = a.acc + (((size_t)(b0 + u / 2) * 2 + u % 2) * a.next + t) * N + blk * BLOCK_SUM;
#pragma unroll
    for (u32 i = 0; i < 4; i++) o[block_elem(0, i, l)] = x[i];
  }
}
// Kinds as for rot_sum_kernel. grid = (ceil(B / CB), N / 256, slots)
template <int KIND, int CB, bool FUSED>
__global__ void __launch_bounds__(BLOCK_SUM) __attribute__((amdgpu_waves_per_eu(4))) block_sum_kernel(RotSumArgs a) {
  __shared__ __attribute__((aligned(16))) u64 sm[2 * block_sum_fill<CB, FUSED>() * CB * BLOCK_SUM];
  __shared__ ulonglong2 tws[FUSED ? BLOCK_SUM - 1 : 1];
  u32 what, blk, zi;
  attention_map(what, blk, zi);
  if (KIND == 0 && zi < a.nfp) block_sum_fp<CB, FUSED>(a, what, blk, zi, sm, tws);
  else block_sum_int<CB, KIND == 2, FUSED>(a, what, blk, zi, sm, tws);
}

// out[i][j][b] = sum_{s < ns} x(j, s)[b] * y(i, s)[b] in three components (+ add in the first two, or in all three), for i0 <= i < i1 and
// j0 <= j < j1. Products of moduli below 2^60 are kept as 128-bit sums, of those below 2^50 in doubles.
struct ProdSumArgs {
  ProdOperand x, y;
  const u64* add;       // null: none; ciphertexts of add_comps components, in the order of the outputs
  const u64* fade;      // not null (nj = 1): every y is multiplied by it ([nlimbs][N]) where it lies, after it has been read
  u64* out;             // [i1 - i0][j1 - j0][B][3][nlimbs][N]
  const ModInfo* mods;
  u32 logN, nlimbs, B, i0, i1, j0, j1, ns, add_comps, add_i;   // add_i: outputs with i below it have an addend
  // triangles: outputs j <= i only, pair (i, j) at place i (i + 1) / 2 + j, places tri_first .. tri_first + tri_out - 1; or terms s <= i
  // only, y's at i (i + 1) / 2 + s - tri_first
  u32 tri_out, tri_sum;
  u64 tri_first;
  unsigned char limbs[128];
};
// Running sum of products of canonical residues of one modulus.
template <bool FP>
struct ProdAcc;
template <>
struct ProdAcc<true> {
  double v = 0.0;
  __device__ __forceinline__ void mac(u64 x, u64 y, const ModInfo& mi) { v += fp_mulmod_var(u2d(x), u2d(y), mi.qinv, mi.qd); }
  __device__ __forceinline__ void fold(const ModInfo& mi) { v = fp_reduce(v, mi.qinv, mi.qd); }
  __device__ __forceinline__ u64 value(const ModInfo& mi) const { return d2u_canon(fp_reduce(v, mi.qinv, mi.qd), mi.qd); }
};
template <>
struct ProdAcc<false> {
  Acc128 v = {0, 0};
  __device__ __forceinline__ void mac(u64 x, u64 y, const ModInfo&) { mac128(v, x, y); }
  __device__ __forceinline__ void fold(const ModInfo& mi) { v = Acc128{reduce128(v, mi), 0}; }
  __device__ __forceinline__ u64 value(const ModInfo& mi) const { return reduce128(v, mi); }
};
template <bool FP>
__device__ __forceinline__ u64 prod_mulmod(u64 x, u64 y, const ModInfo& mi) {
  if (!FP) return mulmod(x, y, mi);
  return d2u_canon(fp_mulmod_var(u2d(x), u2d(y), mi.qinv, mi.qd), mi.qd);
}

// A lane keeps one position of a tile of TI x TJ outputs, so that a word of x serves TI of them and a word of y TJ. FIRST = 2: only the
// third component of every product, [i1 - i0][j1 - j0][B][nlimbs][N].
// What bounds it: memory. At 2^16: the update of 32 outputs from 4 tokens and the read of 32 for 4 tokens, 8 limbs, 1.8 GB in 398 us
// (one output per lane 820); the read of 64 outputs of 9 limbs with their decay, 1.4 GB in 257 us; the third components of 64
// outputs of one token, 0.38 GB in 91 us. A copy of 4 GB runs at 4.8 TB/s on this card. Larger tiles cost the waves that hide the loads.
// grid = (tiles * B, N / 256, limbs)
template <bool FP, int TI, int TJ, int FIRST>
__global__ void __launch_bounds__(256) prod_sum_kernel(ProdSumArgs a) {
  const size_t N = (size_t)1 << a.logN, pl = (size_t)a.nlimbs * N, ct = 2 * pl;
  u32 what, blk, zi;
  attention_map(what, blk, zi);
  const u32 n = blk * 256 + threadIdx.x, l = a.limbs[zi], b = what % a.B;
  const u32 nj = a.j1 - a.j0, tj = (nj + TJ - 1) / TJ;
  u32 tile = what / a.B, i = a.i0 + tile / tj * TI, j = a.j0 + tile % tj * TJ;
  u64 place = (u64)(i - a.i0) * nj + (j - a.j0);   // of the tile's first output
  if (a.tri_out) {
    const u64 pair = a.tri_first + tile;
    i = 0;
    while ((u64)(i + 1) * (i + 2) / 2 <= pair) i++;
    j = (u32)(pair - (u64)i * (i + 1) / 2);
    place = tile;
  }
  const ModInfo mi = a.mods[l];
  const size_t at = (size_t)b * ct + (size_t)l * N + n;
  constexpr int NC = 3 - FIRST;
  ProdAcc<FP> v[TI][TJ][NC];
  const u32 ns = a.tri_sum ? i + 1 : a.ns;
  const u64 tri = a.tri_sum ? ((u64)i * (i + 1) / 2 - a.tri_first) * a.B * ct : 0;
  const u64 fade = a.fade ? a.fade[(size_t)l * N + n] : 0;
  const u32 last_i = a.tri_out ? i : a.i1 - 1, last_j = a.tri_out ? j : a.j1 - 1;   // surplus places repeat the last output
  for (u32 s = 0; s < ns; s++) {
    u64 x[TJ][2], y[TI][2];
#pragma unroll
    for (int f = 0; f < TJ; f++) {
      const u64* p = prod_operand(a.x, min(j + f, last_j), s, ct) + at;
      x[f][0] = p[0], x[f][1] = p[pl];
    }
#pragma unroll
    for (int e = 0; e < TI; e++) {
      const u64* p = prod_operand(a.y, min(i + e, last_i), s, ct) + tri + at;
      y[e][0] = p[0], y[e][1] = p[pl];
    }
#pragma unroll
    for (int e = 0; e < TI; e++) {
      if (a.fade && i + e <= last_i) {
        u64* p = const_cast<u64*>(prod_operand(a.y, i + e, s, ct)) + at;
        p[0] = prod_mulmod<FP>(y[e][0], fade, mi), p[pl] = prod_mulmod<FP>(y[e][1], fade, mi);
      }
#pragma unroll
      for (int f = 0; f < TJ; f++) {
        if (FIRST == 0) {
          v[e][f][0].mac(x[f][0], y[e][0], mi);
          v[e][f][1 % NC].mac(x[f][0], y[e][1], mi);
          v[e][f][1 % NC].mac(x[f][1], y[e][0], mi);
        }
        v[e][f][NC - 1].mac(x[f][1], y[e][1], mi);
      }
    }
    // in doubles a sum takes 6 products below 0.9 q on top of a folded one, 128 bits take 130 products below 2^120
    if (FP ? s % 3 == 2 : (s & 63) == 63) {
#pragma unroll
      for (int e = 0; e < TI; e++)
#pragma unroll
        for (int f = 0; f < TJ; f++)
#pragma unroll
          for (int c = 0; c < NC; c++) v[e][f][c].fold(mi);
    }
  }
#pragma unroll
  for (int e = 0; e < TI; e++)
#pragma unroll
    for (int f = 0; f < TJ; f++) {
      if (i + e > last_i || j + f > last_j) continue;
      const size_t to = (place + (size_t)e * nj + f) * a.B + b;
      u64* o = a.out + to * NC * pl + (size_t)l * N + n;
      const u64* g = a.add && i + e < a.add_i ? a.add + to * a.add_comps * pl + (size_t)l * N + n : nullptr;
#pragma unroll
      for (int c = 0; c < NC; c++) {
        u64 r = v[e][f][c].value(mi);
        if (FIRST == 0 && g && (u32)c < a.add_comps) r = addmod(r, g[c * pl], mi.m);
        o[c * pl] = r;
      }
    }
}

// Up to three batches of ciphertexts one after another: out[k] = in[k] for k < gridDim.y, `words` 16-byte words each.
struct GatherArgs {
  const ulonglong2* in[3];
  ulonglong2* out;
  size_t words;
};
__global__ void __launch_bounds__(256) gather_kernel(GatherArgs a) {
  const size_t i = blockIdx.x * (size_t)256 + threadIdx.x;
  if (i < a.words) a.out[blockIdx.y * a.words + i] = a.in[blockIdx.y][i];
}
