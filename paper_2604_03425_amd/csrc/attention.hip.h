// Kernels of softmax-free attention on ciphertexts: weighted sums of rotations in the extended basis (rotary positions, slot
// sums, the giant steps of a state's read) and sums of ciphertext products (scores, the state's update and read).
#pragma once
#include "ntt16_kernels.hip.h"

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
