// Kernels of attention over a paged cache of ciphertexts and of the root-mean-square norm: what stands between their key switches.
// All of them take every word of their operands once and are bound by memory: a lane owns two adjacent positions (16-byte accesses) and
// holds the three components of a product there, in doubles below 2^50 and in 128 bits above, reduced once. What one product feeds
// another with (numbers in every slot, negatives, a residual, a second product of the same operand) is done on the way in.
#pragma once
#include "attention.hip.h"

#define DECODER_PAIRS 128   // (query, key) pairs or cache entries per launch (their places travel in the kernel's arguments)

// Ciphertexts in memory: component c of ciphertext b at `at + b * stride + c * comp`, limbs N words apart.
struct CtRef {
  const u64* at;
  u64 stride, comp;
};
// A signed number modulo m.
__device__ __forceinline__ u64 signed_residue(long long v, const ModInfo& mi) {
  const u64 a = v < 0 ? 0 - (u64)v : (u64)v;
  const u64 r = csub(a - mul_hi64(a, mi.mu64) * mi.m, mi.m);
  return v < 0 && r ? mi.m - r : r;
}
__device__ __forceinline__ ulonglong2 word_pair(const u64* p) { return *(const ulonglong2*)p; }
__device__ __forceinline__ ulonglong2 plus_number(ulonglong2 x, u64 a, u64 m) { return {addmod(x.x, a, m), addmod(x.y, a, m)}; }

// x * y in three components for two positions.
template <bool FP>
struct PairAcc {
  ProdAcc<FP> v[2][3];
  __device__ __forceinline__ void mac(const ulonglong2 (&x)[2], const ulonglong2 (&y)[2], const ModInfo& mi) {
    const u64 a[2][2] = {{x[0].x, x[1].x}, {x[0].y, x[1].y}}, b[2][2] = {{y[0].x, y[1].x}, {y[0].y, y[1].y}};
#pragma unroll
    for (int e = 0; e < 2; e++) {
      v[e][0].mac(a[e][0], b[e][0], mi);
      v[e][1].mac(a[e][0], b[e][1], mi);
      v[e][1].mac(a[e][1], b[e][0], mi);
      v[e][2].mac(a[e][1], b[e][1], mi);
    }
  }
  __device__ __forceinline__ void fold(const ModInfo& mi) {
#pragma unroll
    for (int e = 0; e < 2; e++)
#pragma unroll
      for (int c = 0; c < 3; c++) v[e][c].fold(mi);
  }
  __device__ __forceinline__ ulonglong2 value(int c, const ModInfo& mi) const { return {v[0][c].value(mi), v[1][c].value(mi)}; }
};

// Products in three components, where a key switch that divides by P (kept = nlimbs) or by P and the last prime (kept = nlimbs - 1) expects
// them. In the latter case the first two components are divided by that prime on the limbs that stay, and P times their last limb, in the
// form of the accumulators there, starts those.
struct ProductOut {
  u64* out;                 // [..][3][nlimbs][N]
  const ulonglong2* less;   // null: kept = nlimbs; else [nlimbs - 1] Shoup pairs of q_last^-1
  u64* last;                // limb nlimbs - 1 of accumulator c of ciphertext b at last + (2 b + c) * last_stride
  u64 last_stride;
  u32 nlimbs, last_int;     // != 0: the accumulators of that limb are integer ones (times 2^-64) whatever its class
};
template <bool FP>
__device__ __forceinline__ void store_product(const ProductOut& o, size_t b, int c, u32 l, size_t n, size_t N, ulonglong2 w, const ModInfo& mi) {
  if (o.less && c < 2) {
    if (l + 1 == o.nlimbs) {
      if (FP && !o.last_int) w = {prod_mulmod<true>(w.x, mi.pmod, mi), prod_mulmod<true>(w.y, mi.pmod, mi)};
      else w = {csub(mont_mul63(w.x, mi.pmod, mi.m, mi.minv), mi.m), csub(mont_mul63(w.y, mi.pmod, mi.m, mi.minv), mi.m)};
      *(ulonglong2*)(o.last + (2 * b + c) * o.last_stride + n) = w;
      return;
    }
    const ulonglong2 f = o.less[l];
    w = {shoup(w.x, f.x, f.y, mi.m), shoup(w.y, f.x, f.y, mi.m)};
  }
  *(ulonglong2*)(o.out + ((b * 3 + c) * o.nlimbs + l) * N + n) = w;
}

// Scores before their sum over the components: q[row[i]] * key[i] for pair i, keys read in their pages. A row's query comes from the
// caches after its first pair: 4 words read and 3 written a pair, 103 us for 26 pairs of 4 rows, 8 limbs at 2^16 (6.0 TB/s).
struct PairArgs {
  CtRef q;
  u64 key_comp;         // words between the two components of a cached key
  ProductOut o;
  const ModInfo* mods;
  u32 logN, fp_on;
  u32 row[DECODER_PAIRS];
  const u64* key[DECODER_PAIRS];
};
template <bool FP>
__device__ __forceinline__ void pair_products(const PairArgs& a, const ModInfo& mi) {
  const size_t N = (size_t)1 << a.logN, n = (blockIdx.x * 256 + threadIdx.x) * 2, l = blockIdx.y, i = blockIdx.z;
  const u64 *q = a.q.at + a.row[i] * a.q.stride + l * N + n, *k = a.key[i] + l * N + n;
  const ulonglong2 x[2] = {word_pair(q), word_pair(q + a.q.comp)}, y[2] = {word_pair(k), word_pair(k + a.key_comp)};
  PairAcc<FP> s;
  s.mac(x, y, mi);
#pragma unroll
  for (int c = 0; c < 3; c++) store_product<FP>(a.o, i, c, (u32)l, n, N, s.value(c, mi), mi);
}
// grid = (N / 512, limbs, pairs)
__global__ void __launch_bounds__(256) pair_products_kernel(PairArgs a) {
  const ModInfo mi = a.mods[blockIdx.y];
  if (mod_class(mi.m, a.fp_on) == 0) pair_products<true>(a, mi);
  else pair_products<false>(a, mi);
}

// out[r] (+)= sum over the pairs i of row r of (u[i] + bias) * value[i], three components; bias is added to every slot. A lane goes over
// all of its row's pairs, so that the sum alone is written and one relinearisation serves the row; 57 us for 26 pairs of 4 rows, 6 limbs at
// 2^16 (6.1 TB/s). A long row of a small ring leaves the chip empty (32 workgroups for one row of 2 limbs at 2^13), which costs the
// latency of its pairs: 41 us for 64, 94 to 105 for a launch's 128, a fifth of a call on 1024 cached tokens there (3.5 ms).
struct ValueArgs {
  CtRef u;
  u64 value_comp;
  u64* out;             // [rows][3][nlimbs][N]
  const ModInfo* mods;
  long long bias;
  u32 logN, nlimbs, fp_on;
  u32 row[DECODER_PAIRS];                       // row and first pair of each sum of the launch; bit 31 of row: adds to what is there
  u32 begin[DECODER_PAIRS + 1];
  const u64* value[DECODER_PAIRS];
};
template <bool FP>
__device__ __forceinline__ void weighted_values(const ValueArgs& a, const ModInfo& mi) {
  const size_t N = (size_t)1 << a.logN, n = (blockIdx.x * 256 + threadIdx.x) * 2, l = blockIdx.y, r = blockIdx.z;
  const u64 bias = signed_residue(a.bias, mi);
  const u32 first = a.begin[r], end = a.begin[r + 1];
  PairAcc<FP> s;
  for (u32 i = first; i < end; i++) {
    const u64 *u = a.u.at + i * a.u.stride + l * N + n, *v = a.value[i] + l * N + n;
    const ulonglong2 x[2] = {plus_number(word_pair(u), bias, mi.m), word_pair(u + a.u.comp)}, y[2] = {word_pair(v), word_pair(v + a.value_comp)};
    s.mac(x, y, mi);
    // in doubles a sum takes 6 products below 0.9 q on top of a folded one, 128 bits take 130 products below 2^120
    if (FP ? (i - first) % 3 == 2 : ((i - first) & 63) == 63) s.fold(mi);
  }
  u64* o = a.out + ((size_t)(a.row[r] & 0x7FFFFFFFu) * 3 * a.nlimbs + l) * N + n;
  const bool add = a.row[r] >> 31;
#pragma unroll
  for (int c = 0; c < 3; c++) {
    ulonglong2 w = s.value(c, mi);
    ulonglong2* to = (ulonglong2*)(o + c * a.nlimbs * N);
    if (add) {
      const ulonglong2 old = *to;
      w = {addmod(w.x, old.x, mi.m), addmod(w.y, old.y, mi.m)};
    }
    *to = w;
  }
}
// grid = (N / 512, limbs, rows)
__global__ void __launch_bounds__(256) weighted_values_kernel(ValueArgs a) {
  const ModInfo mi = a.mods[blockIdx.y];
  if (mod_class(mi.m, a.fp_on) == 0) weighted_values<true>(a, mi);
  else weighted_values<false>(a, mi);
}

// A ciphertext as a product takes it: itself or its negative, plus the number add - sub in every slot.
struct Affine {
  long long add, sub;
  u32 negative;
};
__device__ __forceinline__ void apply(const Affine& f, ulonglong2 (&v)[2], const ModInfo& mi) {
  const u64 m = mi.m, number = submod(signed_residue(f.add, mi), signed_residue(f.sub, mi), m);
  if (f.negative) {   // uniform
    v[0] = {submod(number, v[0].x, m), submod(number, v[0].y, m)};
    v[1] = {submod(0, v[1].x, m), submod(0, v[1].y, m)};
  } else {
    v[0] = plus_number(v[0], number, m);
  }
}
// factor X * Y + (z_factor Z, 0) for ciphertext b, X, Y and Z what fx, fy and fz make of x, y and z. y null: the same words as x; z null:
// none. plus: x + plus in the place of x, written to `sum` too where that is given (layout of x). second != 0: also Y * Y, as
// ciphertext second + b. 5.5 TB/s over the 8 launches of a norm of 8 ciphertexts of 20 limbs at 2^16 (895 us). Both of Newton's products
// read y once; the residual's sum, eps and the start as kernels of their own took that norm from 7990 to 8190 us.
struct ProductArgs {
  CtRef x, y, z;
  Affine fx, fy, fz;
  const u64* plus;
  u64* sum;
  ProductOut o;
  const ModInfo* mods;
  long long factor, z_factor;
  u32 logN, fp_on, second;
};
template <bool FP>
__device__ __forceinline__ void ct_products(const ProductArgs& a, const ModInfo& mi) {
  const size_t N = (size_t)1 << a.logN, n = (blockIdx.x * 256 + threadIdx.x) * 2, l = blockIdx.y, b = blockIdx.z;
  ulonglong2 x[2], y[2];
#pragma unroll
  for (int c = 0; c < 2; c++) {
    const size_t at = b * a.x.stride + c * a.x.comp + l * N + n;
    x[c] = word_pair(a.x.at + at);
    if (a.plus) {
      const ulonglong2 p = word_pair(a.plus + at);
      x[c] = {addmod(x[c].x, p.x, mi.m), addmod(x[c].y, p.y, mi.m)};
      if (a.sum) *(ulonglong2*)(a.sum + at) = x[c];
    }
    y[c] = a.y.at ? word_pair(a.y.at + b * a.y.stride + c * a.y.comp + l * N + n) : x[c];
  }
  apply(a.fx, x, mi);
  apply(a.fy, y, mi);
  if (a.factor != 1) {
    const u64 f = signed_residue(a.factor, mi);
#pragma unroll
    for (int c = 0; c < 2; c++) x[c] = {prod_mulmod<FP>(x[c].x, f, mi), prod_mulmod<FP>(x[c].y, f, mi)};
  }
  {
    PairAcc<FP> s;
    s.mac(x, y, mi);
    ulonglong2 z[2] = {};
    u64 zf = 0;
    if (a.z.at) {
#pragma unroll
      for (int c = 0; c < 2; c++) z[c] = word_pair(a.z.at + b * a.z.stride + c * a.z.comp + l * N + n);
      apply(a.fz, z, mi);
      zf = signed_residue(a.z_factor, mi);
    }
#pragma unroll
    for (int c = 0; c < 3; c++) {
      ulonglong2 w = s.value(c, mi);
      if (a.z.at && c < 2) w = {addmod(w.x, prod_mulmod<FP>(z[c % 2].x, zf, mi), mi.m), addmod(w.y, prod_mulmod<FP>(z[c % 2].y, zf, mi), mi.m)};
      store_product<FP>(a.o, b, c, (u32)l, n, N, w, mi);
    }
  }
  if (a.second) {
    PairAcc<FP> s;
    s.mac(y, y, mi);
#pragma unroll
    for (int c = 0; c < 3; c++) store_product<FP>(a.o, a.second + b, c, (u32)l, n, N, s.value(c, mi), mi);
  }
}
// grid = (N / 512, limbs, ciphertexts)
__global__ void __launch_bounds__(256) ct_products_kernel(ProductArgs a) {
  const ModInfo mi = a.mods[blockIdx.y];
  if (mod_class(mi.m, a.fp_on) == 0) ct_products<true>(a, mi);
  else ct_products<false>(a, mi);
}

// out = pt (.) x on the first nlimbs limbs of ciphertexts, [B][2][nlimbs][N]; grid = (N / 512, limbs, 2 B). 41 us and 5.9 TB/s for 8
// ciphertexts of 14 limbs at 2^16.
__global__ void __launch_bounds__(256) cut_pmult_kernel(u64* out, CtRef x, const u64* pt, const ModInfo* mods, u32 logN, u32 nlimbs) {
  const size_t N = (size_t)1 << logN, n = (blockIdx.x * 256 + threadIdx.x) * 2 + blockIdx.y * N;
  const ModInfo mi = mods[blockIdx.y];
  const ulonglong2 w = word_pair(pt + n), v = word_pair(x.at + (blockIdx.z / 2) * x.stride + (blockIdx.z & 1) * x.comp + n);
  *(ulonglong2*)(out + (size_t)blockIdx.z * nlimbs * N + n) = {mulmod(v.x, w.x, mi), mulmod(v.y, w.y, mi)};
}

// New tokens into their places in the pages of a cache: the first limbs of both components. Entry i < ntokens is a key, the others
// are values; grid = (N / 512, most limbs, 2 * entries). 20 us and 5.8 TB/s for 4 tokens of 8 and 6 limbs at 2^16.
struct AppendArgs {
  const u64 *k, *v;     // [tokens][2][in_limbs][N]
  u32 logN, in_limbs, k_limbs, v_limbs, ntokens, first;
  u64* to[2 * DECODER_PAIRS];
};
__global__ void __launch_bounds__(256) kv_append_kernel(AppendArgs a) {
  const size_t N = (size_t)1 << a.logN;
  const u32 i = blockIdx.z / 2, c = blockIdx.z & 1, l = blockIdx.y;
  const bool value = i >= a.ntokens;
  const u32 limbs = value ? a.v_limbs : a.k_limbs;
  if (l >= limbs) return;
  const size_t n = (blockIdx.x * 256 + threadIdx.x) * 2;
  const u64* from = (value ? a.v : a.k) + ((((size_t)a.first + (value ? i - a.ntokens : i)) * 2 + c) * a.in_limbs + l) * N + n;
  *(ulonglong2*)(a.to[i] + ((size_t)c * limbs + l) * N + n) = word_pair(from);
}
