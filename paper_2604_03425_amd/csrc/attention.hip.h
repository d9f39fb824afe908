// Kernels of softmax-free attention on ciphertexts: weighted sums of rotations in the extended basis (rotary positions, slot
// sums, the giant steps of a state's read) and sums of ciphertext products (scores, the state's update and read).
#pragma once
#include "modarith.hip.h"

#define ROT_SUM_TERMS 32   // terms per launch (they travel in the kernel's arguments)

// acc[b][c][t][n] = P w_0[t][n] base[b][c][t][n] (main primes only)
//                 + sum_r w_r[t][n] ( sum_j D_rj[pi_r(n)] evk_r[j][c][id(t)][n] + [c = 0, main primes] P c0_r[b][t][pi_r(n)] ),
// pi_r the evaluation-domain index map of term r. D_rj is digit j of the term's polynomial in the extended basis: d_r itself on
// the limbs that the digit holds, the transformed conversions in ext_r elsewhere. Without weights every w is one. On integer
// moduli of the two-pass rings acc carries the factor 2^-64 that ModDown's constants expect there.
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
  u64* acc;             // [B][2][next][N]
  const ModInfo* mods;
  u64 d_stride;
  u32 logN, nlimbs, nq, nm, alpha, beta, next, nterms, w_first, w_terms, per_set, accumulate;
  unsigned char slots[128];
  RotTerm term[ROT_SUM_TERMS];
};

// KIND 0: doubles in ext (moduli < 2^50 of the two-pass rings); 1: residues, Montgomery factor in acc; 2: residues, none
template <int KIND>
__global__ void __launch_bounds__(256) rot_sum_kernel(RotSumArgs a) {
  const size_t N = (size_t)1 << a.logN;
  const u32 b = blockIdx.x, n = blockIdx.y * 256 + threadIdx.x, t = a.slots[blockIdx.z];
  const bool main_prime = t < a.nlimbs;
  const u32 id = main_prime ? t : t - a.nlimbs + a.nq;
  const ModInfo mi = a.mods[id];
  const u64 m = mi.m;
  const size_t pl = (size_t)a.nlimbs * N;
  const u64* w = a.w ? a.w + (((size_t)(b / a.per_set) * a.w_terms + a.w_first) * a.next + t) * N + n : nullptr;
  u64 s0 = 0, s1 = 0;
  if (a.base && main_prime) {
    const u64* x = a.base + (size_t)b * a.base_stride + (size_t)t * N + n;
    const u64 pw = w ? mulmod(mi.pmod, *w, mi) : mi.pmod;
    s0 = mulmod(x[0], pw, mi);
    s1 = mulmod(x[pl], pw, mi);
  }
  for (u32 r = 0; r < a.nterms; r++) {
    const RotTerm& q = a.term[r];
    const u32 k = galois_src_index(n, q.galois, a.logN);
    Acc128 v0 = {0, 0}, v1 = {0, 0};
    for (u32 j = 0; j < a.beta; j++) {
      const u32 lo = j * a.alpha, hi = min(lo + a.alpha, a.nlimbs);
      u64 x;
      if (t >= lo && t < hi) {
        x = q.d[(size_t)b * a.d_stride + (size_t)t * N + k];
      } else {
        x = q.ext[(((size_t)b * a.beta + j) * a.next + t) * N + k];
        if (KIND == 0) x = d2u_canon(__longlong_as_double((long long)x), mi.qd);
      }
      const u64* e = q.evk + ((size_t)j * 2 * a.nm + id) * N + n;
      mac128(v0, x, e[0]);
      mac128(v1, x, e[(size_t)a.nm * N]);
    }
    if (q.c0 && main_prime) mac128(v0, q.c0[(size_t)b * a.d_stride + (size_t)t * N + k], mi.pmod);
    u64 r0 = reduce128(v0, mi), r1 = reduce128(v1, mi);
    if (w) {
      const u64 f = w[(size_t)(r + 1) * a.next * N];
      r0 = mulmod(r0, f, mi);
      r1 = mulmod(r1, f, mi);
    }
    s0 = addmod(s0, r0, m);
    s1 = addmod(s1, r1, m);
  }
  if (KIND == 1) {
    s0 = csub(redc(Acc128{s0, 0}, m, mi.minv), m);
    s1 = csub(redc(Acc128{s1, 0}, m, mi.minv), m);
  }
  u64* o = a.acc + ((size_t)b * 2 * a.next + t) * N + n;
  if (a.accumulate) {
    s0 = addmod(s0, o[0], m);
    s1 = addmod(s1, o[(size_t)a.next * N], m);
  }
  o[0] = s0;
  o[(size_t)a.next * N] = s1;
}

// One operand of a sum of products: the ciphertext of output (i, j), term s. With `rotated` the index i, j or s that it names counts
// the rotations of a ciphertext, the first of which (the ciphertext itself) lies at `first` and the others at `rest`, one
// rotation after another.
enum ProdIndex : u32 { PROD_NONE = 0, PROD_I = 1, PROD_J = 2, PROD_S = 3 };
struct ProdOperand {
  const u64 *first, *rest;
  u64 step[4];   // in ciphertexts: [PROD_I], [PROD_J], [PROD_S] multiply the index; [0] is unused
  u32 rotated;
};
// out[i][j][b] = sum_{s < ns} x(i, j, s)[b] * y(i, j, s)[b] in three components (+ add in the first two, or in all three)
struct ProdSumArgs {
  ProdOperand x, y;
  const u64* add;       // null: none; ciphertexts of add_comps components, in the order of the outputs
  u64* out;             // [ni][nj][B][3][nlimbs][N]
  const ModInfo* mods;
  u32 logN, nlimbs, B, nj, ns, add_comps, add_i;   // add_i: outputs with i below it have an addend
  u32 o_first;          // the first output of the launch; out and add start at it
  // triangles: outputs (i, j) with j <= i only, at i (i + 1) / 2 + j; or terms s <= i only, x's at i (i + 1) / 2 + s
  u32 tri_out, tri_sum;
  u64 tri_base;         // the place in the triangle that x starts at
};
__device__ __forceinline__ const u64* prod_operand(const ProdOperand& p, u32 i, u32 j, u32 s, u64 ct) {
  const u32 r = p.rotated == PROD_I ? i : p.rotated == PROD_J ? j : p.rotated == PROD_S ? s : 0;
  u64 at = p.step[PROD_I] * i + p.step[PROD_J] * j + p.step[PROD_S] * s;
  if (p.rotated && r) return p.rest + (at - p.step[p.rotated]) * ct;
  return p.first + at * ct;
}

// grid = (N / 256, nlimbs, outputs * B)
__global__ void __launch_bounds__(256) prod_sum_kernel(ProdSumArgs a) {
  const size_t N = (size_t)1 << a.logN, pl = (size_t)a.nlimbs * N, ct = 2 * pl;
  const u32 n = blockIdx.x * 256 + threadIdx.x, l = blockIdx.y, o = a.o_first + blockIdx.z / a.B, b = blockIdx.z % a.B;
  u32 i = o / a.nj, j = o % a.nj;
  if (a.tri_out) {
    i = 0;
    while ((i + 1) * (i + 2) / 2 <= o) i++;
    j = o - i * (i + 1) / 2;
  }
  const ModInfo mi = a.mods[l];
  const size_t at = (size_t)b * ct + (size_t)l * N + n;
  Acc128 v0 = {0, 0}, v1 = {0, 0}, v2 = {0, 0};
  const u32 ns = a.tri_sum ? i + 1 : a.ns;
  const u64 tri = a.tri_sum ? ((u64)i * (i + 1) / 2 - a.tri_base) * a.B * ct : 0;
  for (u32 s = 0; s < ns; s++) {
    const u64* x = prod_operand(a.x, i, j, s, ct) + tri + at;
    const u64* y = prod_operand(a.y, i, j, s, ct) + at;
    const u64 x0 = x[0], x1 = x[pl], y0 = y[0], y1 = y[pl];
    mac128(v0, x0, y0);
    mac128(v1, x0, y1);
    mac128(v1, x1, y0);
    mac128(v2, x1, y1);
    if ((s & 63) == 63) {   // at most 129 products below 2^120 in a sum
      v0 = Acc128{reduce128(v0, mi), 0};
      v1 = Acc128{reduce128(v1, mi), 0};
      v2 = Acc128{reduce128(v2, mi), 0};
    }
  }
  u64 r0 = reduce128(v0, mi), r1 = reduce128(v1, mi), r2 = reduce128(v2, mi);
  const size_t to = (size_t)blockIdx.z * 3 * pl + (size_t)l * N + n;
  if (a.add && i < a.add_i) {
    const u64* e = a.add + (size_t)blockIdx.z * a.add_comps * pl + (size_t)l * N + n;
    r0 = addmod(r0, e[0], mi.m);
    r1 = addmod(r1, e[pl], mi.m);
    if (a.add_comps == 3) r2 = addmod(r2, e[2 * pl], mi.m);
  }
  a.out[to] = r0;
  a.out[to + pl] = r1;
  a.out[to + 2 * pl] = r2;
}
