// Host side of the calls for softmax-free attention: rotary positions (ckks_rope) and linear attention with decays
// (ckks_linattn_step, ckks_linattn_chunk). Included at the end of ckks_mi355.hip, whose launch sequences it uses.
#pragma once

namespace {

// Takes pieces of a workspace in order; without one it only counts.
struct Carve {
  char* base;
  size_t used = 0;
  char* bytes(size_t n) {
    char* p = base ? base + used : nullptr;
    used += align256(n);
    return p;
  }
  u64* words(size_t n) { return (u64*)bytes(n * 8); }
};

u32 rotation_element(const ckks_ctx* c, u64 steps) {   // 5^steps mod 2N
  const u64 two_n = 2 * (u64)c->N;
  u64 g = 1, b = 5;
  for (; steps; steps >>= 1) {
    if (steps & 1) g = g * b % two_n;
    b = b * b % two_n;
  }
  return (u32)g;
}

// Ring 2^12 has its kernels that hold whole limbs (`whole`: whole_limb's rule, once a call, since the forms below differ) or goes one
// kernel per step like the rings without any: rotary positions of 8 ciphertexts of 4 limbs 38 us that way, by steps 44; 256 of 12 limbs
// in 3 digits 1012 and 880.
// Digits of B polynomials in the extended basis, evaluation domain, at L.ext of the key-switch workspace: (b, limb t) is at
// d + b * d_stride + t * N. Doubles on the double-precision moduli of the two-pass rings and of whole limbs, canonical residues elsewhere.
// last_int (two-pass rings): limb nlimbs - 1 in residues whatever its class; rows_only (there): after the first pass of the transform.
int ext_digits(ckks_ctx* c, const LevelTables* lt, bool whole, const u64* d, u64 d_stride, u32 B, u32 nlimbs, char* ws, hipStream_t st,
               bool last_int = false, bool rows_only = false) {
  int rc;
  FwdInnerArgs unused;
  if (two_pass(c)) return hoist_front16(c, lt, d, d_stride, B, nlimbs, ws, st, unused, last_int, rows_only);
  if (whole) {
    Ks12Args a = ks12_args(c, lt, B, nlimbs, ws);
    a.d = d;
    a.d_stride = d_stride;
    launch_ks12_digits(c, lt, B, nlimbs, a, st);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
  }
  const u32 N = c->N, next = lt->next, beta = lt->beta;
  const KsLayout L = ks_layout(c, B, nlimbs);
  u64 *dcoef = (u64*)(ws + L.dcoef), *ext = (u64*)(ws + L.ext);
  if ((rc = launch_ntt(c, true, d, d_stride, dcoef, (u64)nlimbs * N, B, 0, nlimbs, identity_map(nlimbs), 0, 0, st))) return rc;
  {
    ModUpArgs a{dcoef, ext, c->d_mods, lt->up_inv, lt->up_mat, c->logN, nlimbs, c->nq, c->alpha, beta, next};
    ProfScope ps(c, PK_MODUP, st);
    launch_modup<false>(c, lt, a, beta, B, st);
    HIP_TRY(hipGetLastError());
  }
  return launch_ntt(c, false, ext, (u64)next * N, ext, (u64)next * N, B * beta, 0, next, ext_map(c, nlimbs), beta, nlimbs, st);
}

// ModDown of both accumulators [B][2][next][N] (their special limbs are overwritten) to out [B][2][nlimbs][N].
int ext_mod_down(ckks_ctx* c, const LevelTables* lt, bool whole, u64* acc, u64* out, u32 B, u32 nlimbs, char* ws, hipStream_t st) {
  int rc;
  if (two_pass(c)) {
    KsIo io{nullptr, 0, 0, out, {0, 0}, nullptr, 0};
    return ks16_finish(c, lt, io, B, nlimbs, ws, st, acc);
  }
  if (whole) {
    Ks12Args a = ks12_args(c, lt, B, nlimbs, ws);
    a.sums = a.acc = acc;
    a.out = out;
    const dim3 block(WL_THREADS), grid(2 * B, nlimbs);
    {
      ProfScope ps(c, PK_KS12_SPECIAL, st);
      hipLaunchKernelGGL(ks12_special_sums_kernel, dim3(2 * B, c->np), block, 0, st, a);
    }
    ProfScope ps(c, PK_KS12_FINAL, st);
    if (lt->narrow_dn) hipLaunchKernelGGL(ks12_final_sums_kernel<true>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(ks12_final_sums_kernel<false>, grid, block, 0, st, a);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
  }
  const u32 N = c->N, next = lt->next, K = c->np;
  u64* tq = (u64*)(ws + ks_layout(c, B, nlimbs).tq);
  LimbMap pmap;
  for (u32 k = 0; k < CKKS_MAX_SLOTS; k++) pmap.id[k] = (unsigned char)(k < K ? c->nq + k : 0);
  if ((rc = launch_ntt(c, true, acc, (u64)next * N, acc, (u64)next * N, B * 2, nlimbs, K, pmap, 0, 0, st))) return rc;
  {
    ModDownArgs a{acc, tq, c->d_mods, lt->dn_inv, lt->dn_mat, c->logN, nlimbs, c->nq, K, next, nlimbs, c->nq};
    ProfScope ps(c, PK_MODDOWN, st);
    launch_moddown<false>(c, lt, a, B * 2, lt->narrow_dn, st);
    HIP_TRY(hipGetLastError());
  }
  if ((rc = launch_ntt(c, false, tq, (u64)nlimbs * N, tq, (u64)nlimbs * N, B * 2, 0, nlimbs, identity_map(nlimbs), 0, 0, st)))
    return rc;
  FinalArgs a{acc, tq, out, c->d_mods, lt->pinv, c->logN, nlimbs, next, 0};
  ProfScope ps(c, PK_FINAL, st);
  hipLaunchKernelGGL(ks_final_kernel, dim3(N / 256, nlimbs, B * 2), dim3(256), 0, st, a);
  HIP_TRY(hipGetLastError());
  return CKKS_OK;
}

// Everything about rot_sum_kernel's arguments that the context and the level fix.
RotSumArgs rot_sum_args(const ckks_ctx* c, const LevelTables* lt, bool whole, u32 nlimbs, u64* acc, u64 d_stride) {
  RotSumArgs a;
  a.base = a.w = nullptr;
  a.base_stride = 0;
  a.acc = acc;
  a.mods = c->d_mods;
  a.d_stride = d_stride;
  a.logN = c->logN;
  a.nlimbs = nlimbs;
  a.nq = c->nq;
  a.nm = c->nm;
  a.alpha = c->alpha;
  a.beta = lt->beta;
  a.next = lt->next;
  a.nterms = a.w_first = a.w_terms = a.accumulate = 0;
  a.per_set = 1;
  a.doubles = two_pass(c) || whole;
  return a;
}
template <int KIND>
void launch_rot_sum_of(u32 outs, u32 slots, const RotSumArgs& a, hipStream_t st) {
  const dim3 block(256);
  if (a.B > 1) hipLaunchKernelGGL((rot_sum_kernel<KIND, 2>), dim3(outs * ((a.B + 1) / 2), (1u << a.logN) / 256, slots), block, 0, st, a);
  else hipLaunchKernelGGL((rot_sum_kernel<KIND, 1>), dim3(outs, (1u << a.logN) / 256, slots), block, 0, st, a);
}
template <int CB>
void launch_block_sum_of(u32 slots, const RotSumArgs& a, hipStream_t st) {
  const dim3 grid((a.B + CB - 1) / CB, (1u << a.logN) / BLOCK_SUM, slots), block(BLOCK_SUM);
  if (a.tw && a.nfp) hipLaunchKernelGGL((block_sum_kernel<0, CB, true>), grid, block, 0, st, a);
  else if (a.tw) hipLaunchKernelGGL((block_sum_kernel<1, CB, true>), grid, block, 0, st, a);
  else if (!a.doubles) hipLaunchKernelGGL((block_sum_kernel<2, CB, false>), grid, block, 0, st, a);
  else if (a.nfp == 0) hipLaunchKernelGGL((block_sum_kernel<1, CB, false>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((block_sum_kernel<0, CB, false>), grid, block, 0, st, a);
}
// Whether all rotations keep the blocks that block_sum_kernel holds.
bool rotations_near(const ckks_ctx* c, const u32* galois, u32 R) {
  for (u32 r = 0; r < R; r++)
    if (galois[r] % (2 * c->N / BLOCK_SUM) != 1) return false;
  return R != 0;
}
// near: block_sum_kernel (rotations_near); last_int: limb nlimbs - 1 in integers; extended limbs from `from` to `to` only.
int launch_rot_sum(const ckks_ctx* c, RotSumArgs& a, u32 B, hipStream_t st, u32 outs = 1, bool near = false, bool last_int = false,
                   u32 from = 0, u32 to = ~0u) {
  a.B = B;
  const LimbMap emap = ext_map(c, a.nlimbs);
  u32 cnt = 0;
  for (int fp = 1; fp >= 0; fp--) {   // double-precision slots first
    for (u32 s = from; s < std::min(to, a.next); s++)
      if ((a.doubles && host_class(c, c->mod[emap.id[s]]) == 0 && !(last_int && s + 1 == a.nlimbs)) == (fp == 1)) a.slots[cnt++] = (unsigned char)s;
    if (fp) a.nfp = cnt;
  }
  ProfScope ps(c, near ? PK_BLOCK_SUM : PK_ROT_SUM, st);
  if (near) {
    const u32 groups = (B + 3) / 4;
    switch ((B + groups - 1) / groups) {   // ciphertexts a lane, as even as possible
      case 1: launch_block_sum_of<1>(cnt, a, st); break;
      case 2: launch_block_sum_of<2>(cnt, a, st); break;
      case 3: launch_block_sum_of<3>(cnt, a, st); break;
      default: launch_block_sum_of<4>(cnt, a, st); break;
    }
  } else if (!a.doubles) launch_rot_sum_of<2>(outs, cnt, a, st);
  else if (a.nfp == 0) launch_rot_sum_of<1>(outs, cnt, a, st);
  else launch_rot_sum_of<0>(outs, cnt, a, st);
  HIP_TRY(hipGetLastError());
  return CKKS_OK;
}

// acc = P w_0 ct + sum_r w_{r+1} (accumulators of the rotation of ct by galois[r]); ws: a key-switch workspace for B.
int rotations_to_ext(ckks_ctx* c, const LevelTables* lt, bool whole, const u64* ct, u32 B, u32 nlimbs, const u32* galois,
                     const u64* const* evks, u32 R, const u64* w, u32 per_set, u64* acc, char* ws, hipStream_t st, bool last_int = false) {
  int rc;
  const u64 pl = (u64)nlimbs * c->N;
  const bool near = !w && rotations_near(c, galois, R);
  if (R && (rc = ext_digits(c, lt, whole, ct + pl, 2 * pl, B, nlimbs, ws, st, last_int))) return rc;
  const u64* ext = (const u64*)(ws + ks_layout(c, B, nlimbs).ext);
  RotSumArgs a = rot_sum_args(c, lt, whole, nlimbs, acc, 2 * pl);
  a.base = ct;
  a.base_stride = 2 * pl;
  a.w = w;
  a.w_terms = R + 1;
  a.per_set = per_set;
  for (u32 r0 = 0; r0 == 0 || r0 < R; r0 += ROT_SUM_TERMS) {
    a.nterms = std::min<u32>(ROT_SUM_TERMS, R - r0);
    a.w_first = r0;
    for (u32 r = 0; r < a.nterms; r++) a.term[r] = RotTerm{ext, ct + pl, ct, evks[r0 + r], galois[r0 + r]};
    if ((rc = launch_rot_sum(c, a, B, st, 1, near, last_int))) return rc;
    a.base = nullptr;
    a.accumulate = 1;
  }
  return CKKS_OK;
}

// What near_sums decomposes (limb t of number b at d + b * d_stride + t * N), rotates beside it (c0, the same stride; null: nothing) and
// adds as it is (two components, N nlimbs words apart).
struct NearIn {
  const u64 *d, *c0;
  u64 d_stride;
  const u64* base;
  u64 base_stride;
};
// out = base + the rotations by galois[r] with one ModDown, by P or (drop) by P q_{nlimbs-1}; R > 0, ws: a key-switch workspace for B.
// Unweighted near rotations on two-pass rings: digits go through their last stages and the special limbs through their first inverse ones
// in the sums' kernel, which comes first for the special limbs and then for the main ones, whose sums it finishes: neither the
// transformed digits nor the main limbs' sums reach memory. Up to BLOCK_SUM_TOGETHER workgroups, four times what the chip holds of them
// (four to a compute unit), the limbs go together and the assembly is a kernel of its own: a part of a last round twice costs more there
// than the main limbs' sums in memory. us, together | apart: attention of four ragged sequences at 2^13, 672 workgroups, 318 | 336; norms of
// 5 ciphertexts at 2^14, 1280, 604 | 611, of one of 12 limbs at 2^16, 4096, 1151 | 1161; 26 pairs of 64 components there, 19 712,
// 3829 | 3579.
#define BLOCK_SUM_TOGETHER 4096
int near_sums(ckks_ctx* c, const LevelTables* lt, u64* out, const NearIn& in, u32 B, u32 nlimbs, const u32* galois, const u64* const* evks,
              u32 R, bool drop, char* ws, hipStream_t st) {
  int rc;
  const KsLayout L = ks_layout(c, B, nlimbs);
  u64 *acc = (u64*)(ws + L.acc), *tq = (u64*)(ws + L.tq);
  const u64* ext = (const u64*)(ws + L.ext);
  const DropForm form = drop ? drop_form(c, lt, nlimbs) : APART;
  const bool last_int = form == JOINED_FORCED;
  const u32 keep = drop ? nlimbs - 1 : nlimbs;
  if ((rc = ext_digits(c, lt, false, in.d, in.d_stride, B, nlimbs, ws, st, last_int, true))) return rc;
  RotSumArgs a = rot_sum_args(c, lt, false, nlimbs, acc, in.d_stride);
  a.base_stride = in.base_stride;
  a.tw = c->d_tw_fwd;
  a.twi = c->d_tw_inv;
  a.twfp = c->d_twfp_fwd;
  a.first_special = form == APART ? nlimbs : keep;
  a.fin_out = out;
  a.fin_pinv = drop ? lt->dm_pinv2 : lt->pinv2;
  a.fin_limbs = keep;
  auto sums = [&](u32 from, u32 to) {
    a.base = in.base;
    a.accumulate = 0;
    for (u32 r0 = 0; r0 < R; r0 += ROT_SUM_TERMS) {
      a.nterms = std::min<u32>(ROT_SUM_TERMS, R - r0);
      a.inverse = r0 + a.nterms == R;
      a.fin_tq = to <= keep && a.inverse ? tq : nullptr;
      for (u32 r = 0; r < a.nterms; r++) a.term[r] = RotTerm{ext, in.d, in.c0, evks[r0 + r], galois[r0 + r]};
      if (int e = launch_rot_sum(c, a, B, st, 1, true, last_int, from, to)) return e;
      a.base = nullptr;
      a.accumulate = 1;
    }
    return CKKS_OK;
  };
  const u32 groups = (B + 3) / 4;
  if ((u64)groups * (c->N / BLOCK_SUM) * lt->next <= BLOCK_SUM_TOGETHER) {
    if ((rc = sums(0, lt->next))) return rc;
    if (drop) rc = ks16_drop_rows(c, lt, B, nlimbs, acc, tq, st, true);
    else rc = ks16_moddown_rows(c, lt, B, nlimbs, acc, tq, st, true);
    if (rc) return rc;
    if (drop) return ks16_drop_assemble(c, lt, out, B, nlimbs, acc, tq, st);
    KsIo io{nullptr, 0, 0, out, {0, 0}, nullptr, 0};
    return ks16_assemble(c, lt, io, B, nlimbs, acc, tq, st);
  }
  if ((rc = sums(keep, lt->next))) return rc;
  if (drop) rc = ks16_drop_rows(c, lt, B, nlimbs, acc, tq, st, true);
  else rc = ks16_moddown_rows(c, lt, B, nlimbs, acc, tq, st, true);
  if (rc) return rc;
  return sums(0, keep);
}
// The sum of a ciphertext and its rotations this way, if they are near ones on a two-pass ring. Otherwise *done is false and nothing happens.
int sum_near_rotations(ckks_ctx* c, const LevelTables* lt, u64* out, const u64* ct, u32 B, u32 nlimbs, const u32* galois,
                       const u64* const* evks, u32 R, bool drop, char* ws, hipStream_t st, bool* done) {
  *done = two_pass(c) && rotations_near(c, galois, R);
  if (!*done) return CKKS_OK;
  const u64 pl = (u64)nlimbs * c->N;
  return near_sums(c, lt, out, NearIn{ct + pl, ct, 2 * pl, ct, 2 * pl}, B, nlimbs, galois, evks, R, drop, ws, st);
}

// ---- linear attention ----
// Ciphertexts that one key switch of the calls below works on at a time: all that the call has to switch at once (components of the
// state; groups of the read; all rotations and what they are taken from, side by side; scores), up to what fills the chip many times over
// (a pass over 128 of 9 limbs at 2^16 is two dozen rounds of workgroups) or the B of a token: more would only take workspace. 128 of 24
// limbs at 2^16 take 31 GB in all, the 4 of a step with 4 components 1 GB.
u32 linattn_slice(const ckks_ctx* c, bool scores, u32 C, u32 B, u32 n1, u32 n2) {
  const u64 keyed = (u64)C * B, rotated = std::max<u64>(2 * (u64)(n1 - 1) + n2 - 1, 3) * keyed;
  const u64 needed = std::max<u64>({(u64)n1 * n2 * B, n2 * keyed, n1 * n2 > 1 ? rotated : 0, scores ? keyed * (C + 1) / 2 : 0});
  return (u32)std::min<u64>(needed, std::max<u32>(B, std::min(1024u, 128u << (c->logN < 16 ? 16 - c->logN : 0))));
}

// Tokens up to which the key switches of a state's update form the first two terms of the sums of products themselves. us, that way |
// by the kernel of the products, 32 components at 2^16, 8 limbs, 1, 2, 4, 8 tokens: 1934 | 2012, 2665 | 2699, 4415 | 4363, 9338 | 8961;
// 16 at 2^15, 5 60-bit limbs, 2, 5, 8: 1607 | 1618, 3424 | 3353, 5954 | 5785. Beyond two every output fetches factors that a tile shares.
#define LINATTN_MAPPED_TOKENS 2
// Words of a component of a read's products up to which all their groups are relinearised from the same launches. us, so | by the fused
// kernels: a token of 4 components at 2^13, 5 limbs (2^16 words) 263 | 286, of 16 at 2^15, 6 limbs (2^19.6) 603 | 631, 9 limbs
// (2^20.2) 761 | 775, three of 16 at 2^14 (2^20.4) 831 | 835, eight (2^21.8) 1734 | 1721, one of 16 at 2^16, 8 groups (2^22.2) 1551 | 1534.
#define LINATTN_BESIDE_WORDS (1ull << 21)

struct LinAttn {
  const ckks_ctx* cc;      // for sizes
  ckks_ctx* c;
  const LevelTables* lt;
  bool whole;              // ring 2^12: the kernels for whole limbs
  u32 C, B, nlimbs, n1, n2;
  u64 pl, ct;              // words of a polynomial, of a ciphertext
  u32 slice, tokens;       // ciphertexts per key switch; tokens whose ciphertexts make at most that many
  const u64 *mult_key;
  const u64 *const *baby_keys, *const *giant_keys, *const *value_keys;
  std::vector<u32> baby, giant, value;   // Galois elements
  hipStream_t st;
  // workspace
  u64 *rot_a, *rot_b;      // rotations 1.. of keys or queries, and of values
  const u64 *q_rest = nullptr, *k_rest = nullptr, *v_rest = nullptr;   // those of all three, where a call makes them at once
  u32 turn_step = 0;       // ciphertexts from one rotation of a key to the next
  u64 *d, *y, *p, *sums, *extra, *total;  // products in three components, ciphertexts, scores and their inner sums, the terms from
                                          // inside the chunk, the read's sum in the extended basis
  u64* acc;                // accumulators of rotations, [slice][2][next][N]
  char* ks;                // a key-switch workspace for `slice` ciphertexts
  size_t ks_bytes;

  void shape(const ckks_ctx* c_, bool scores, u32 C_, u32 B_, u32 nlimbs_, u32 n1_, u32 n2_) {
    cc = c_, C = C_, B = B_, nlimbs = nlimbs_, n1 = n1_, n2 = n2_;
    pl = (u64)nlimbs * cc->N, ct = 2 * pl;
    slice = linattn_slice(cc, scores, C, B, n1, n2);
    tokens = std::min<u32>(C, slice / B);
    whole = whole_limb(cc, C * B, nlimbs, false);
  }
  // pieces of the workspace of a step (scores = false) or of a chunk
  size_t carve(char* ws, bool scores) {
    Carve w{ws};
    const u64 ext_ct = 2 * (u64)(nlimbs + cc->np) * cc->N;
    const size_t group = (size_t)tokens * B;               // ciphertexts of the read's queries at a time
    const size_t keyed = (size_t)C * B;
    rot_a = w.words(std::max<size_t>((n1 - 1) * keyed, joint(true) || joint(false) ? slice : 0) * ct);
    rot_b = w.words((n2 - 1) * keyed * ct);
    const size_t most = std::max<size_t>({(size_t)slice, group * n2, scores ? keyed : 0});   // (a call's inputs side by side too)
    d = w.words(most * 3 * pl);
    y = w.words(most * ct);
    p = w.words(scores ? std::max<size_t>(slice, keyed) * ct : 0);
    sums = w.words(scores ? slice * ct : 0);
    extra = w.words(scores ? group * 3 * pl : 0);
    total = w.words(group * ext_ct);
    acc = w.words(slice * ext_ct);
    ks_bytes = ckks_workspace_bytes(cc, CKKS_OP_KEYSWITCH, slice, nlimbs, 0);
    ks = w.bytes(ks_bytes);
    return w.used;
  }

  // out[r][..] = rotations of n ciphertexts, one rotation out_stride words after another. The digits are shared by all rotations of a
  // ciphertext, and P sigma(c0) joins the accumulators, so that one ModDown serves all rotations of all ciphertexts at once
  // (a ModDown of one ciphertext of 9 limbs at 2^16 takes 50 us, of seven 150).
  int rotate(u64* out, u64 out_stride, const u64* in, u32 n, const std::vector<u32>& elements, const u64* const* keys) {
    int rc;
    const u32 R = (u32)elements.size();
    if (!R) return CKKS_OK;
    const u64 ext_ct = 2 * (u64)lt->next * c->N;
    const u32 nb = std::min(n, std::max(1u, slice / R));
    for (u32 i = 0; i < n; i += nb) {
      const u32 cnt = std::min(nb, n - i), per = std::min<u32>(R, slice / cnt);
      const u64* ext = (const u64*)(ks + ks_layout(c, cnt, nlimbs).ext);
      for (u32 r0 = 0; r0 < R; r0 += per) {   // (ModDown's scratch takes the digits' place, so a further pass converts again)
        if ((rc = ext_digits(c, lt, whole, in + i * ct + pl, ct, cnt, nlimbs, ks, st))) return rc;
        const u32 rots = std::min(per, R - r0);
        if ((rc = rotations_apart(acc, ext, in + i * ct, cnt, elements.data() + r0, keys + r0, rots))) return rc;
        if (out_stride == (u64)cnt * ct) {
          if ((rc = ext_mod_down(c, lt, whole, acc, out + r0 * out_stride, rots * cnt, nlimbs, ks, st))) return rc;
          continue;
        }
        for (u32 r = 0; r < rots; r++)
          if ((rc = ext_mod_down(c, lt, whole, acc + (u64)r * cnt * ext_ct, out + (r0 + r) * out_stride + i * ct, cnt, nlimbs, ks, st)))
            return rc;
      }
    }
    return CKKS_OK;
  }
  // The accumulators of each rotation of n ciphertexts `in`, whose digits are at `ext`, rotation by rotation.
  int rotations_apart(u64* to, const u64* ext, const u64* in, u32 n, const u32* elements, const u64* const* keys, u32 R) {
    int rc;
    const u64 stride = n * 2 * (u64)lt->next * c->N;
    // the kernel that keeps a position's digits for all rotations: a chunk of 4 tokens of 32 components 4236 us, by sums of one term each
    // 4395; a token of 64 components, whose keys are read once either way, 3395 and 3357
    const bool streamed = two_pass(c) && lt->beta <= INNER16_ROT_MAX_BETA;
    const u32 most = streamed ? KS_MULTI_MAX : ROT_SUM_TERMS;
    for (u32 r0 = 0; r0 < R; r0 += most) {
      const u32 rots = std::min(most, R - r0);
      if (streamed) {
        FwdInnerArgs ia = hoisted_args(c, lt, in + pl, ct, ext, nlimbs);
        ia.c0 = in;
        ia.c0_poly_stride = ct;
        if ((rc = launch_inner_rot(c, lt, ia, n, nlimbs, elements + r0, keys + r0, rots, to + r0 * stride, stride, st))) return rc;
        continue;
      }
      RotSumArgs a = rot_sum_args(c, lt, whole, nlimbs, to + r0 * stride, ct);
      a.nterms = 1;
      for (u32 r = 0; r < rots; r++) a.term[r] = RotTerm{ext, in + pl, in, keys[r0 + r], elements[r0 + r]};
      if ((rc = launch_rot_sum(c, a, n, st, rots))) return rc;
    }
    return CKKS_OK;
  }
  // All rotations of a call at once, where they are few: queries (if the state is read), keys and values side by side go through one
  // decomposition and one ModDown, which takes a third of the launches. us, all at once | one after another: a token of 4 components at
  // 2^13 288 | 378, of 16 at 2^14 833 | 933, of 64 at 2^16 3395 | 3425; a chunk of 4 tokens of 32 components 4236 | 4452.
  bool joint(bool with_q) const {
    const u64 baby_cts = (with_q ? 2 : 1) * (u64)(n1 - 1), all = (baby_cts + n2 - 1) * C * B;
    return all && all <= slice && (with_q ? 3u : 2u) * (u64)C * B <= slice;
  }
  int rotate_all(const u64* q, const u64* k, const u64* v, bool with_q) {
    int rc;
    const u32 n = C * B, turned = (with_q ? 2 : 1) * n;   // ciphertexts that take the baby steps
    const u64 ext_ct = 2 * (u64)lt->next * c->N;
    GatherArgs g{{(const ulonglong2*)(with_q ? q : k), (const ulonglong2*)(with_q ? k : v), (const ulonglong2*)v}, (ulonglong2*)d, n * ct / 2};
    {
      ProfScope ps(c, PK_GATHER, st);
      hipLaunchKernelGGL(gather_kernel, dim3((unsigned)((g.words + 255) / 256), with_q ? 3 : 2), dim3(256), 0, st, g);
      HIP_TRY(hipGetLastError());
    }
    if ((rc = ext_digits(c, lt, whole, d + pl, ct, turned + n, nlimbs, ks, st))) return rc;
    const u64* ext = (const u64*)(ks + ks_layout(c, turned + n, nlimbs).ext);
    u64* to = acc;
    if ((rc = rotations_apart(to, ext, d, turned, baby.data(), baby_keys, n1 - 1))) return rc;
    to += (u64)(n1 - 1) * turned * ext_ct;
    if ((rc = rotations_apart(to, ext + (u64)turned * lt->beta * lt->next * c->N, d + (u64)turned * ct, n, value.data(), value_keys, n2 - 1)))
      return rc;
    if ((rc = ext_mod_down(c, lt, whole, acc, rot_a, (n1 - 1) * turned + (n2 - 1) * n, nlimbs, ks, st))) return rc;
    q_rest = rot_a;
    k_rest = rot_a + (with_q ? n * ct : 0);
    v_rest = rot_a + (u64)(n1 - 1) * turned * ct;
    turn_step = turned;
    return CKKS_OK;
  }
  int relin(u64* out, const u64* in, size_t n) {
    int rc;
    for (size_t i = 0; i < n; i += slice)
      if ((rc = ckks_relin(c, (uint64_t*)out + i * ct, (const uint64_t*)in + i * 3 * pl, (u32)std::min<size_t>(slice, n - i), nlimbs,
                           (const uint64_t*)mult_key, ks, ks_bytes, st)))
        return rc;
    return CKKS_OK;
  }
  template <int TI, int TJ, int FIRST = 0>
  void launch_products(bool fp, u32 tiles, u32 cnt, const ProdSumArgs& a) {
    const dim3 grid(tiles * B, c->N / 256, cnt), block(256);
    if (fp) hipLaunchKernelGGL((prod_sum_kernel<true, TI, TJ, FIRST>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((prod_sum_kernel<false, TI, TJ, FIRST>), grid, block, 0, st, a);
  }
  int products(ProdSumArgs a, bool third_only = false) {
    a.mods = c->d_mods;
    a.logN = c->logN;
    a.nlimbs = nlimbs;
    a.B = B;
    for (int fp = 1; fp >= 0; fp--) {
      u32 cnt = 0;
      for (u32 l = 0; l < nlimbs; l++)
        if ((c->logN <= 16 && host_class(c, c->mod[l]) == 0) == (fp == 1)) a.limbs[cnt++] = (unsigned char)l;
      if (!cnt) continue;
      ProfScope ps(c, PK_PROD_SUM, st);
      const u32 ni = a.i1 - a.i0, nj = a.j1 - a.j0;
      if (third_only && a.tri_out) launch_products<1, 1, 2>(fp, a.tri_out, cnt, a);
      else if (third_only) launch_products<2, 4, 2>(fp, (ni + 1) / 2 * ((nj + 3) / 4), cnt, a);
      else if (a.tri_out) launch_products<1, 1>(fp, a.tri_out, cnt, a);
      else if (a.tri_sum || (ni == 1 && nj == 1)) launch_products<1, 1>(fp, ni * nj, cnt, a);
      else if (nj == 1) launch_products<4, 1>(fp, (ni + 3) / 4, cnt, a);
      else launch_products<2, 4>(fp, (ni + 1) / 2 * ((nj + 3) / 4), cnt, a);
    }
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
  }

  // out = add + Relin(products of a) on the two-pass rings: only the third terms of the products go through memory, at d; the key
  // switch forms the other two where it assembles its result.
  int relin_products(u64* out, const u64* add, const ProdSumArgs& a) {
    int rc;
    if ((rc = products(a, true))) return rc;
    const u32 cnt = (a.tri_out ? a.tri_out : (a.i1 - a.i0) * (a.j1 - a.j0)) * B;
    KsIo io{a.out, pl, 0, out, {add ? 1u : 0u, add ? 1u : 0u}, nullptr, 0};
    io.add2 = add;
    io.more = KS_MAPPED;
    KsMore& m = io.more_args;
    m.B = B;
    m.i0 = a.i0;
    m.j0 = a.j0;
    m.nj = a.j1 - a.j0;
    m.ns = a.ns;
    m.tri = a.tri_out;
    m.tri_first = a.tri_first;
    m.x = a.x;
    m.y = a.y;
    return keyswitch_impl(c, io, cnt, nlimbs, mult_key, ks, st);
  }

  // state_out = state_in + Relin(sum_s K_s[b] * V_s[g]), then times decay. state_out may be state_in.
  int update(u64* state_out, const u64* state_in, const u64* k, const u64* v, const u64* decay) {
    int rc;
    const u64 keyed = (u64)C * B;
    if (!k_rest) {
      if ((rc = rotate(rot_a, keyed * ct, k, C * B, baby, baby_keys))) return rc;
      if ((rc = rotate(rot_b, keyed * ct, v, C * B, value, value_keys))) return rc;
    }
    ProdSumArgs a{};
    a.x = ProdOperand{k, k_rest ? k_rest : rot_a, k_rest ? turn_step : keyed, B, 1};
    a.y = ProdOperand{v, k_rest ? v_rest : rot_b, keyed, B, 1};
    a.ns = C;
    a.out = d;
    a.add_comps = 2;
    a.add_i = n2;
    // whole rows of the state, as many as make a slice, or pieces of one row
    const u32 rows = std::max(1u, slice / (n1 * B)), cols = std::min(n1, slice / B);
    for (u32 g = 0; g < n2; g += rows)
      for (u32 b = 0; b < n1; b += cols) {
        a.i0 = g, a.i1 = std::min(n2, g + rows);
        a.j0 = b, a.j1 = std::min(n1, b + cols);
        const u64 at = ((u64)g * n1 + b) * B * ct;
        if (C <= LINATTN_MAPPED_TOKENS && two_pass(c) && c->tune[3] != 1) {
          // the key switch forms the first two terms of the products where it assembles its result, with the state's addend
          if ((rc = relin_products(state_out + at, state_in ? state_in + at : nullptr, a))) return rc;
          continue;
        }
        a.add = state_in ? state_in + at : nullptr;   // Relin(d) + S = Relin(d + (S, 0))
        if ((rc = products(a))) return rc;
        if ((rc = relin(state_out + at, d, (size_t)(a.i1 - a.i0) * (a.j1 - a.j0) * B))) return rc;
      }
    return decay ? multiply(state_out, decay) : CKKS_OK;
  }
  int multiply(u64* state, const u64* decay) {
    int rc;
    const u32 all = n1 * n2 * B;
    for (u32 i = 0; i < all; i += 16384)
      if ((rc = ckks_pmult(c, (uint64_t*)state + i * ct, (const uint64_t*)state + i * ct, (const uint64_t*)decay,
                           std::min(16384u, all - i), nlimbs, st)))
        return rc;
    return CKKS_OK;
  }

  // o of T <= tokens tokens: see the header. extra (three components) holds their terms from inside the chunk. fade (T = 1): the state is
  // multiplied by it where it lies, once it has been read, which saves the product a pass of its own its read of the state.
  int read(u64* o, const u64* q, u32 T, const u64* state, const u64* extra, const u64* fade = nullptr) {
    int rc;
    const u32 n = T * B;
    if (!state) return relin(o, extra, n);
    if (!q_rest && (rc = rotate(rot_a, (u64)n * ct, q, n, baby, baby_keys))) return rc;
    ProdSumArgs a{};
    a.x = ProdOperand{q, q_rest ? q_rest : rot_a, B, q_rest ? turn_step : n, 2};
    a.y = ProdOperand{state, nullptr, (u64)n1 * B, B, 0};
    a.i1 = n2;
    a.j1 = T;
    a.ns = n1;
    a.fade = fade;
    a.out = d;
    a.add = extra;
    a.add_comps = 3;
    a.add_i = 1;
    if ((rc = products(a))) return rc;
    // The sum of the first group's relinearisation and the others' rotations in the extended basis. Where they are few, the other groups
    // are relinearised beside the first one, from the same launches; else by the fused kernels, which move less.
    const bool beside = n2 > 1 && (u64)n2 * n <= slice && (u64)n2 * n * nlimbs * c->N <= LINATTN_BESIDE_WORDS;
    const u32 first = beside ? n2 * n : n;
    u64* sum = beside ? acc : total;
    if (!beside && (rc = relin(y, d + (u64)n * 3 * pl, (size_t)(n2 - 1) * n))) return rc;
    if ((rc = ext_digits(c, lt, whole, d + 2 * pl, 3 * pl, first, nlimbs, ks, st))) return rc;
    RotSumArgs r = rot_sum_args(c, lt, whole, nlimbs, sum, 3 * pl);
    r.base = d;
    r.base_stride = 3 * pl;
    r.nterms = 1;
    r.term[0] = RotTerm{(const u64*)(ks + ks_layout(c, first, nlimbs).ext), d + 2 * pl, nullptr, mult_key, 1};
    if ((rc = launch_rot_sum(c, r, first, st))) return rc;
    if (beside && (rc = ext_mod_down(c, lt, whole, sum + (u64)n * 2 * lt->next * c->N, y, (n2 - 1) * n, nlimbs, ks, st))) return rc;
    const u32 others = n2 - 1, per = std::min<u32>(ROT_SUM_TERMS, slice / n);
    for (u32 g0 = 0; g0 < others; g0 += per) {
      const u32 cnt = std::min(per, others - g0);
      const u64* yg = y + (u64)g0 * n * ct;
      if ((rc = ext_digits(c, lt, whole, yg + pl, ct, cnt * n, nlimbs, ks, st))) return rc;
      const u64* ext = (const u64*)(ks + ks_layout(c, cnt * n, nlimbs).ext);
      RotSumArgs s = rot_sum_args(c, lt, whole, nlimbs, sum, ct);
      s.accumulate = 1;
      s.nterms = cnt;
      for (u32 g = 0; g < cnt; g++)
        s.term[g] = RotTerm{ext + (u64)g * n * lt->beta * lt->next * c->N, yg + (u64)g * n * ct + pl, yg + (u64)g * n * ct,
                            giant_keys[g0 + g], giant[g0 + g]};
      if ((rc = launch_rot_sum(c, s, n, st))) return rc;
    }
    return ext_mod_down(c, lt, whole, sum, o, n, nlimbs, ks, st);
  }

  // out = in + its rotations by the elements, one ModDown for all of them; n <= slice ciphertexts
  int sum_rotations(u64* out, const u64* in, u32 n, const std::vector<u32>& elements, const u64* const* keys) {
    int rc;
    bool done;
    if ((rc = sum_near_rotations(c, lt, out, in, n, nlimbs, elements.data(), keys, (u32)elements.size(), false, ks, st, &done)) || done)
      return rc;
    u64* acc = (u64*)(ks + ks_layout(c, n, nlimbs).acc);
    if ((rc = rotations_to_ext(c, lt, whole, in, n, nlimbs, elements.data(), keys, (u32)elements.size(), nullptr, 1, acc, ks, st))) return rc;
    return ext_mod_down(c, lt, whole, acc, out, n, nlimbs, ks, st);
  }

  // d = sum_{s <= t} p_ts * v_s for tokens [t0, t0 + T)
  int scored(u64* out, const u64* q, const u64* k, const u64* v, u32 t0, u32 T) {
    int rc;
    for (u32 t = t0; t < t0 + T;) {
      // rows t .. u-1 of the triangle of pairs, whole rows that make at most a slice
      u32 u = t + 1;
      u64 pairs = t + 1;
      while (u < t0 + T && (pairs + u + 1) * B <= std::max<u64>(slice, (u64)C * B)) {
        u++;
        pairs += u;
      }
      const u64 first = (u64)t * (t + 1) / 2;
      ProdSumArgs a{};
      a.x = ProdOperand{k, nullptr, B, 0, 0};
      a.y = ProdOperand{q, nullptr, B, 0, 0};
      a.j1 = a.i1 = 1;
      a.ns = 1;
      const u32 per = slice / B;
      for (u64 i = 0; i < pairs; i += per) {
        const u32 cnt = (u32)std::min<u64>(per, pairs - i);
        a.out = d;
        a.tri_first = first + i;
        a.tri_out = cnt;
        u64* to = p + i * B * ct;
        u64* stage = n1 > 1 || n2 > 1 ? y : to;
        if (two_pass(c) && c->tune[3] != 1) {
          if ((rc = relin_products(stage, nullptr, a))) return rc;
        } else {
          if ((rc = products(a))) return rc;
          if ((rc = relin(stage, d, (size_t)cnt * B))) return rc;
        }
        if (n1 > 1) {
          u64* next = n2 > 1 ? sums : to;
          if ((rc = sum_rotations(next, stage, cnt * B, baby, baby_keys))) return rc;
          stage = next;
        }
        if (n2 > 1 && (rc = sum_rotations(to, stage, cnt * B, giant, giant_keys))) return rc;
      }
      ProdSumArgs e{};
      e.x = ProdOperand{v, nullptr, 0, B, 0};
      e.y = ProdOperand{p, nullptr, 0, B, 0};
      e.i0 = t;
      e.i1 = u;
      e.j1 = 1;
      e.tri_sum = 1;
      e.tri_first = first;
      e.out = out + (u64)(t - t0) * B * 3 * pl;
      if ((rc = products(e))) return rc;
      t = u;
    }
    return CKKS_OK;
  }
};

int linattn_check(const ckks_ctx* c, u32 C, u32 B, u32 nlimbs, u32 n1, u32 n2) {
  int rc = check_common(c, B, nlimbs);
  if (rc) return rc;
  if (C == 0 || n1 == 0 || n2 == 0) return fail(CKKS_ESHAPE, "tokens, n1 and n2 must be positive");
  if (C > 4096 || n1 > 4096 || n2 > 4096 || (u64)C * B > 32767 || (u64)n1 * n2 * B > 32767 * 64ull || (u64)n2 * C * B > 65535 ||
      (u64)B * std::max<u32>(2, c->dnum) > 65535)
    return fail(CKKS_ESHAPE, "too many ciphertexts for one call");
  return CKKS_OK;
}

struct LinAttnCall {
  uint64_t *o_out, *state_out;
  const uint64_t *q, *k, *v, *state_in, *decay;
};
int linattn_run(bool chunk, ckks_ctx* c, const LinAttnCall& io, u32 C, u32 B, u32 nlimbs, u32 n1, u32 n2, u32 stride,
                const uint64_t* evk_mult, const uint64_t* const* evk_baby, const uint64_t* const* evk_giant,
                const uint64_t* const* evk_value, void* ws, size_t ws_bytes, void* stream) {
  int rc = linattn_check(c, C, B, nlimbs, n1, n2);
  if (rc) return rc;
  if (stride == 0) return fail(CKKS_ESHAPE, "stride must be positive");
  if (!io.o_out || !io.state_out || !io.q || !io.k || !io.v || !evk_mult) return fail(CKKS_EINVAL, "null argument");
  if ((n1 > 1 && !evk_baby) || (n2 > 1 && (!evk_giant || !evk_value))) return fail(CKKS_EINVAL, "null key array");
  for (u32 b = 1; b < n1; b++)
    if (!evk_baby[b - 1]) return fail(CKKS_EINVAL, "null baby-step key");
  for (u32 g = 1; g < n2; g++)
    if (!evk_giant[g - 1] || !evk_value[g - 1]) return fail(CKKS_EINVAL, "null giant-step or value key");
  const size_t ct_bytes = (size_t)2 * nlimbs * c->N * 8, in_bytes = (size_t)C * B * ct_bytes, state_bytes = (size_t)n1 * n2 * B * ct_bytes;
  for (const uint64_t* x : {io.q, io.k, io.v})
    if (overlap(io.o_out, in_bytes, x, in_bytes) || overlap(io.state_out, state_bytes, x, in_bytes))
      return fail(CKKS_EINVAL, "an output overlaps q, k or v");
  if (overlap(io.o_out, in_bytes, io.state_out, state_bytes)) return fail(CKKS_EINVAL, "the outputs overlap each other");
  if (io.state_in && (overlap(io.o_out, in_bytes, io.state_in, state_bytes) ||
                      (io.state_in != io.state_out && overlap(io.state_out, state_bytes, io.state_in, state_bytes))))
    return fail(CKKS_EINVAL, "state_in must be state_out itself or not overlap the outputs");
  if (io.decay && (overlap(io.o_out, in_bytes, io.decay, ct_bytes / 2) || overlap(io.state_out, state_bytes, io.decay, ct_bytes / 2)))
    return fail(CKKS_EINVAL, "an output overlaps decay");
  LinAttn f;
  f.shape(c, chunk, C, B, nlimbs, n1, n2);
  f.c = c;
  if (!ws || ((uintptr_t)ws & 255)) return fail(CKKS_EWORKSPACE, "workspace is null or not 256-byte aligned");
  const size_t need = f.carve((char*)ws, chunk);
  if (ws_bytes < need)
    return fail(CKKS_EWORKSPACE, "workspace too small: need " + std::to_string(need) + " bytes, got " + std::to_string(ws_bytes));
  if ((rc = get_level(c, nlimbs, &f.lt))) return rc;
  DeviceGuard guard(c->device);
  if (!guard.ok) return fail(CKKS_EHIP, "cannot select the context's device");
  f.st = (hipStream_t)stream;
  f.mult_key = (const u64*)evk_mult;
  f.baby_keys = (const u64* const*)evk_baby;
  f.giant_keys = (const u64* const*)evk_giant;
  f.value_keys = (const u64* const*)evk_value;
  const u64 slots = c->N / 2;
  for (u32 b = 1; b < n1; b++) f.baby.push_back(rotation_element(c, (u64)b * stride % slots));
  for (u32 g = 1; g < n2; g++) {
    const u64 steps = (u64)g * n1 % slots * stride % slots;
    f.giant.push_back(rotation_element(c, steps));
    f.value.push_back(rotation_element(c, slots - steps));
  }
  const u64 *q = (const u64*)io.q, *k = (const u64*)io.k, *v = (const u64*)io.v, *S = (const u64*)io.state_in, *decay = (const u64*)io.decay;
  u64 *o = (u64*)io.o_out, *out = (u64*)io.state_out;
  const bool with_q = !chunk || S;
  if (f.joint(with_q) && (rc = f.rotate_all(q, k, v, with_q))) return rc;
  if (!chunk) {
    if ((rc = f.update(out, S, k, v, nullptr))) return rc;
    return f.read(o, q, 1, out, nullptr, decay);
  }
  for (u32 t = 0; t < C; t += f.tokens) {   // all reads of the old state come before the update, which may overwrite it
    const u32 T = std::min(f.tokens, C - t);
    if ((rc = f.scored(f.extra, q, k, v, t, T))) return rc;
    if ((rc = f.read(o + (u64)t * B * f.ct, q + (u64)t * B * f.ct, T, S, f.extra))) return rc;
  }
  return f.update(out, S, k, v, decay);
}

// Runs a call's body; what it may throw (memory for its host arrays) becomes an error code.
template <class F>
int guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(CKKS_EINVAL, std::string("host error: ") + e.what());
  }
}

}  // namespace

extern "C" {

int ckks_rope(ckks_ctx* c, uint64_t* ct_out, const uint64_t* ct_in, uint32_t B, uint32_t nlimbs, const uint64_t* pt_ext, uint32_t npt,
              const uint32_t* galois_elts, const uint64_t* const* evks, uint32_t R, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    int rc = check_common(c, B, nlimbs);
    if (rc) return rc;
    if (!ct_out || !ct_in || !pt_ext || (R && (!galois_elts || !evks))) return fail(CKKS_EINVAL, "null argument");
    if (npt == 0 || B % npt) return fail(CKKS_ESHAPE, "the batch must be a multiple of the number of weight sets");
    for (u32 r = 0; r < R; r++) {
      if (!evks[r]) return fail(CKKS_EINVAL, "null key");
      if (!(galois_elts[r] & 1) || galois_elts[r] >= 2 * c->N) return fail(CKKS_EINVAL, "galois_elt must be odd and < 2N");
    }
    const LevelTables* lt;
    if ((rc = get_level(c, nlimbs, &lt))) return rc;
    if ((u64)B * std::max<u32>(2, lt->beta) > 65535) return fail(CKKS_ESHAPE, "batch too large for one call");
    if ((rc = check_ws(c, CKKS_OP_ROPE, B, nlimbs, 0, ws, ws_bytes))) return rc;
    const size_t ct_bytes = (size_t)B * 2 * nlimbs * c->N * 8;
    const size_t pt_bytes = (size_t)npt * (R + (size_t)1) * lt->next * c->N * 8;
    if (overlap(ct_out, ct_bytes, ct_in, ct_bytes) || overlap(ct_out, ct_bytes, pt_ext, pt_bytes))
      return fail(CKKS_EINVAL, "ct_out overlaps an input");
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(CKKS_EHIP, "cannot select the context's device");
    hipStream_t st = (hipStream_t)stream;
    const u64* in = (const u64*)ct_in;
    const bool whole = whole_limb(c, B, nlimbs, false);
    if (R == 1 && two_pass(c) && c->tune[3] != 1) {
      // One rotation: the weights join the fused kernels of a key switch, whose digits never reach memory in the evaluation domain. us,
      // that way | through sums of rotations: 24 limbs at 2^16, 1, 4, 16, 64 ciphertexts 147 | 185, 367 | 462, 1287 | 1596, 5105 |
      // 6416; 5 limbs at 2^13, 1, 8, 64: 52 | 55, 63 | 72, 140 | 194; 8 60-bit limbs at 2^15, 1, 8: 76 | 74, 165 | 186. They hold
      // one rotation's digits and sums; two rotations go through the sums of rotations, the only form there is for them.
      const u64 pl = (u64)nlimbs * c->N;
      KsIo io{in + pl, 2 * pl, galois_elts[0], (u64*)ct_out, {0, 0}, in, galois_elts[0]};
      io.more = KS_WEIGHTED;
      io.more_args.w = (const u64*)pt_ext;
      io.more_args.per_set = B / npt;
      return keyswitch_impl(c, io, B, nlimbs, (const u64*)evks[0], (char*)ws, st);
    }
    u64* acc = (u64*)((char*)ws + ks_layout(c, B, nlimbs).acc);
    if ((rc = rotations_to_ext(c, lt, whole, (const u64*)ct_in, B, nlimbs, galois_elts, (const u64* const*)evks, R, (const u64*)pt_ext,
                               B / npt, acc, (char*)ws, st)))
      return rc;
    return ext_mod_down(c, lt, whole, acc, (u64*)ct_out, B, nlimbs, (char*)ws, st);
  });
}

size_t ckks_linattn_workspace_bytes(const ckks_ctx* c, int op, uint32_t tokens, uint32_t B, uint32_t nlimbs, uint32_t n1, uint32_t n2) {
  size_t bytes = 0;
  guarded([&]() -> int {
    if ((op != CKKS_OP_LINATTN_STEP && op != CKKS_OP_LINATTN_CHUNK) || (op == CKKS_OP_LINATTN_STEP && tokens != 1))
      return fail(CKKS_EINVAL, "not a linear-attention operation");
    const int rc = linattn_check(c, tokens, B, nlimbs, n1, n2);
    if (rc) return rc;
    LinAttn f;
    const bool scores = op == CKKS_OP_LINATTN_CHUNK;
    f.shape(c, scores, tokens, B, nlimbs, n1, n2);
    bytes = f.carve(nullptr, scores);
    return CKKS_OK;
  });
  return bytes;
}

int ckks_linattn_step(ckks_ctx* c, uint64_t* o_out, uint64_t* state_out, const uint64_t* q, const uint64_t* k, const uint64_t* v,
                      const uint64_t* state_in, const uint64_t* decay, uint32_t B, uint32_t nlimbs, uint32_t n1, uint32_t n2,
                      uint32_t stride, const uint64_t* evk_mult, const uint64_t* const* evk_baby, const uint64_t* const* evk_giant,
                      const uint64_t* const* evk_value, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&] {
    return linattn_run(false, c, {o_out, state_out, q, k, v, state_in, decay}, 1, B, nlimbs, n1, n2, stride, evk_mult, evk_baby,
                       evk_giant, evk_value, ws, ws_bytes, stream);
  });
}

int ckks_linattn_chunk(ckks_ctx* c, uint64_t* o_out, uint64_t* state_out, const uint64_t* q, const uint64_t* k, const uint64_t* v,
                       const uint64_t* state_in, const uint64_t* decay, uint32_t tokens, uint32_t B, uint32_t nlimbs, uint32_t n1,
                       uint32_t n2, uint32_t stride, const uint64_t* evk_mult, const uint64_t* const* evk_baby,
                       const uint64_t* const* evk_giant, const uint64_t* const* evk_value, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&] {
    return linattn_run(true, c, {o_out, state_out, q, k, v, state_in, decay}, tokens, B, nlimbs, n1, n2, stride, evk_mult, evk_baby,
                       evk_giant, evk_value, ws, ws_bytes, stream);
  });
}

}  // extern "C"
