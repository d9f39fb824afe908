// Host side of attention over a paged cache (ckks_kv_append, ckks_attn_paged) and of the root-mean-square norm (ckks_rmsnorm). Included
// at the end of ckks_mi355.hip, whose launch sequences it uses.
#pragma once
#include "attention_calls.hip.h"

namespace {

// ModDown by P q_{nlimbs-1} of both accumulators [B][2][next][N] (what lies from limb nlimbs - 1 on is overwritten) to out
// [B][2][nlimbs - 1][N]: that limb joins the special ones as a source of the conversion.
int ext_mod_down_more(ckks_ctx* c, const LevelTables* lt, bool whole, u64* acc, u64* out, u32 B, u32 nlimbs, char* ws, hipStream_t st) {
  int rc;
  if (whole) {
    Ks12Args a = ks12_args(c, lt, B, nlimbs, ws);
    a.sums = a.acc = acc;
    a.out = out;
    ks12_drop(a, lt);
    const dim3 block(WL_THREADS), grid(2 * B, a.keep);
    {
      ProfScope ps(c, PK_KS12_SPECIAL, st);
      hipLaunchKernelGGL(ks12_special_sums_kernel, dim3(2 * B, a.next - a.keep), block, 0, st, a);
    }
    ProfScope ps(c, PK_KS12_FINAL, st);
    if (lt->narrow_dm) hipLaunchKernelGGL(ks12_final_sums_kernel<true>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(ks12_final_sums_kernel<false>, grid, block, 0, st, a);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
  }
  const u32 N = c->N, next = lt->next, K = c->np, keep = nlimbs - 1;
  u64* tq = (u64*)(ws + ks_layout(c, B, nlimbs).tq);
  if (two_pass(c)) {
    if ((rc = ks16_drop_rows(c, lt, B, nlimbs, acc, tq, st, false))) return rc;
    return ks16_drop_assemble(c, lt, out, B, nlimbs, acc, tq, st);
  }
  LimbMap sources = identity_map(0);
  sources.id[0] = (unsigned char)keep;
  for (u32 k = 0; k < K; k++) sources.id[k + 1] = (unsigned char)(c->nq + k);
  if ((rc = launch_ntt(c, true, acc, (u64)next * N, acc, (u64)next * N, B * 2, keep, K + 1, sources, 0, 0, st))) return rc;
  {
    ProfScope ps(c, PK_MODDOWN, st);
    launch_wide(drop_wide_args(c, lt, acc, tq, nlimbs), 1, B * 2, st);
    HIP_TRY(hipGetLastError());
  }
  if ((rc = launch_ntt(c, false, tq, (u64)keep * N, tq, (u64)keep * N, B * 2, 0, keep, identity_map(keep), 0, 0, st))) return rc;
  FinalArgs a{acc, tq, out, c->d_mods, lt->dm_pinv, c->logN, keep, next, 0};
  ProfScope ps(c, PK_FINAL, st);
  hipLaunchKernelGGL(ks_final_kernel, dim3(N / 256, keep, B * 2), dim3(256), 0, st, a);
  HIP_TRY(hipGetLastError());
  return CKKS_OK;
}

// Ciphertexts that one key switch of the calls below works on at a time (see linattn_slice).
u32 decoder_slice(const ckks_ctx* c, u64 needed) {
  return (u32)std::min<u64>(needed, std::min(1024u, 128u << (c->logN < 16 ? 16 - c->logN : 0)));
}

// What both operators share: key switches of up to `slice` ciphertexts in one workspace.
struct Decoder {
  const ckks_ctx* cc;      // for sizes
  ckks_ctx* c = nullptr;
  hipStream_t st = nullptr;
  u32 nlimbs, n1, n2, slice;
  const u64* mult_key = nullptr;
  const u64 *const *baby_keys = nullptr, *const *giant_keys = nullptr;
  std::vector<u32> baby, giant;   // Galois elements
  u64 *d, *y[2];           // [slice]: products in three components, ciphertexts
  char* ks;                // a key-switch workspace
  size_t ks_bytes;

  u64 poly(u32 limbs) const { return (u64)limbs * cc->N; }
  u64 fp_on() const { return cc->logN <= 16 && cc->tune[1] == 0; }
  CtRef cts(const u64* at, u32 limbs) const { return CtRef{at, 2 * poly(limbs), poly(limbs)}; }
  void carve_common(Carve& w) {
    d = w.words(slice * 3 * poly(nlimbs));
    for (u64*& x : y) x = w.words(slice * 2 * poly(nlimbs));
    ks_bytes = ckks_workspace_bytes(cc, CKKS_OP_KEYSWITCH, slice, nlimbs, 0);
    ks = w.bytes(ks_bytes);
  }
  void keys(ckks_ctx* c_, u32 stride, const uint64_t* mult, const uint64_t* const* b, const uint64_t* const* g, void* stream) {
    c = c_;
    st = (hipStream_t)stream;
    mult_key = (const u64*)mult;
    baby_keys = (const u64* const*)b;
    giant_keys = (const u64* const*)g;
    const u64 slots = c->N / 2;
    for (u32 i = 1; i < n1; i++) baby.push_back(rotation_element(c, (u64)i * stride % slots));
    for (u32 i = 1; i < n2; i++) giant.push_back(rotation_element(c, (u64)i * n1 % slots * stride % slots));
  }
  // Ring 2^12: whether n ciphertexts go through the kernels that hold whole limbs.
  bool whole(const LevelTables* lt, u32 n, u32 limbs) const { return lt->dm_off12 && whole_limb(cc, n, limbs, false); }
  // Whether a relinearisation that divides by the last prime too takes the fused kernels of a key switch; products for one go where it
  // wants them (`more` of product_out). Against a step of sums and a division of their own, us: a norm of 8 ciphertexts of 20 limbs at 2^16
  // 10 498 -> 9 100, 64 scores of 7 limbs squared twice 2 524 -> 2 370; 2^12: a token of 4 pairs 166 -> 156.
  bool fused(const LevelTables* lt, u32 n, u32 limbs) const { return two_pass(cc) ? cc->tune[3] != 1 && !few(lt, n) : whole(lt, n, limbs); }
  // Two-pass rings: whether n ciphertexts are so few that the sum of one rotation, by nothing, is sooner there than the fused kernels of a
  // key switch, which end in longer ones. In blocks of 256 words, us fused | as a sum: a norm of one ciphertext at 2^13 (relinearisations
  // of up to 512) 381 | 331, at 2^14 (up to 1152) 419 | 383, at 2^15 (up to 2816) 527 | 503 (516 without those above 1536), of 3 at 2^14
  // (up to 1920) 490 | 487; attention of one token with itself at 2^13 186 | 162. Above: 13 ciphertexts at 2^13 (2912, 2496) 312 | 306, 5 at
  // 2^14 (2560) 601 | 603, 4 of 60-bit primes at 2^15 (4096) 1099 | 1106.
  bool few(const LevelTables* lt, u32 n) const { return two_pass(cc) && (u64)n * (cc->N / BLOCK_SUM) * lt->next <= 2048; }
  int product_out(ProductOut* o, u64* out, u32 n, u32 limbs, bool more) const {
    int rc;
    *o = ProductOut{out, nullptr, nullptr, 0, limbs, 0};
    if (!more) return CKKS_OK;
    const LevelTables* lt;
    if ((rc = get_level(c, limbs, &lt))) return rc;
    if (!fused(lt, n, limbs)) return CKKS_OK;
    o->less = lt->rs_qinv;
    o->last = (u64*)(ks + ks_layout(c, n, limbs).acc) + poly(limbs - 1);
    o->last_stride = poly(lt->next);
    o->last_int = drop_form(cc, lt, limbs) == JOINED_FORCED;
    return CKKS_OK;
  }
  // Relin of products in three components (at `limbs` limbs); more: dividing by the last prime too.
  int relin(u64* out, const u64* in, u32 n, u32 limbs, bool more) {
    int rc;
    const LevelTables* lt;
    if ((rc = get_level(c, limbs, &lt))) return rc;
    const u64 pl = poly(limbs);
    const u32 nothing = 1;   // as a Galois element
    if (few(lt, n)) return near_sums(c, lt, out, NearIn{in + 2 * pl, nullptr, 3 * pl, in, 3 * pl}, n, limbs, &nothing, &mult_key, 1, more, ks, st);
    if (!more) return ckks_relin(c, (uint64_t*)out, (const uint64_t*)in, n, limbs, (const uint64_t*)mult_key, ks, ks_bytes, st);
    if (fused(lt, n, limbs)) {
      KsIo io{in + 2 * pl, 3 * pl, 0, out, {1, 1}, nullptr, 0};
      io.add2 = in;
      io.add2_three = true;
      io.drop = true;
      return keyswitch_impl(c, io, n, limbs, mult_key, ks, st);
    }
    const KsLayout L = ks_layout(c, n, limbs);
    const bool last_int = drop_form(c, lt, limbs) == JOINED_FORCED;
    if ((rc = ext_digits(c, lt, false, in + 2 * pl, 3 * pl, n, limbs, ks, st, last_int))) return rc;
    u64* acc = (u64*)(ks + L.acc);
    RotSumArgs r = rot_sum_args(c, lt, false, limbs, acc, 3 * pl);
    r.base = in;
    r.base_stride = 3 * pl;
    r.nterms = 1;
    r.term[0] = RotTerm{(const u64*)(ks + L.ext), in + 2 * pl, nullptr, mult_key, 1};
    if ((rc = launch_rot_sum(c, r, n, st, 1, false, last_int))) return rc;
    return ext_mod_down_more(c, lt, false, acc, out, n, limbs, ks, st);
  }
  int sum_rotations(u64* out, const u64* in, u32 n, const std::vector<u32>& elements, const u64* const* rot_keys, bool more) {
    int rc;
    const LevelTables* lt;
    if ((rc = get_level(c, nlimbs, &lt))) return rc;
    bool done;
    if ((rc = sum_near_rotations(c, lt, out, in, n, nlimbs, elements.data(), rot_keys, (u32)elements.size(), more, ks, st, &done)) || done)
      return rc;
    u64* acc = (u64*)(ks + ks_layout(c, n, nlimbs).acc);
    const bool by_limbs = whole(lt, n, nlimbs);
    if ((rc = rotations_to_ext(c, lt, by_limbs, in, n, nlimbs, elements.data(), rot_keys, (u32)elements.size(), nullptr, 1, acc, ks, st,
                               more && drop_form(c, lt, nlimbs) == JOINED_FORCED)))
      return rc;
    return more ? ext_mod_down_more(c, lt, by_limbs, acc, out, n, nlimbs, ks, st)
                : ext_mod_down(c, lt, by_limbs, acc, out, n, nlimbs, ks, st);
  }
  // The sum over the components of a lane of products d (nlimbs limbs), less a limb, in every slot of the lane. In one of y; where is
  // returned in `out`.
  int slot_sum(u64*& out, u32 n) {
    int rc, at = 0;
    if ((rc = relin(y[0], d, n, nlimbs, n1 == 1 && n2 == 1))) return rc;
    if (n1 > 1) {
      if ((rc = sum_rotations(y[1 - at], y[at], n, baby, baby_keys, n2 == 1))) return rc;
      at = 1 - at;
    }
    if (n2 > 1) {
      if ((rc = sum_rotations(y[1 - at], y[at], n, giant, giant_keys, true))) return rc;
      at = 1 - at;
    }
    out = y[at];
    return CKKS_OK;
  }
  // to d, for relin() of n ciphertexts (2 n with `second`)
  int products(ProductArgs a, u32 n, u32 limbs, bool more) {
    int rc;
    if ((rc = product_out(&a.o, d, a.second ? 2 * n : n, limbs, more))) return rc;
    a.mods = c->d_mods;
    a.logN = c->logN;
    a.fp_on = (u32)fp_on();
    ProfScope ps(c, PK_CT_PRODUCTS, st);
    hipLaunchKernelGGL(ct_products_kernel, dim3(c->N / 512, limbs, n), dim3(256), 0, st, a);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
  }
};

int decoder_check(const ckks_ctx* c, u32 B, u32 nlimbs, u32 n1, u32 n2) {
  int rc = check_common(c, B, nlimbs);
  if (rc) return rc;
  if (c->np == 0) return fail(CKKS_ESHAPE, "the context has no special primes");
  if (n1 == 0 || n2 == 0 || n1 > 4096 || n2 > 4096) return fail(CKKS_ESHAPE, "n1 and n2 must be in [1, 4096]");
  return CKKS_OK;
}
int decoder_check_keys(u32 n1, u32 n2, u32 stride, const uint64_t* mult, const uint64_t* const* baby, const uint64_t* const* giant) {
  if (stride == 0) return fail(CKKS_ESHAPE, "stride must be positive");
  if (!mult || (n1 > 1 && !baby) || (n2 > 1 && !giant)) return fail(CKKS_EINVAL, "null key");
  for (u32 b = 1; b < n1; b++)
    if (!baby[b - 1]) return fail(CKKS_EINVAL, "null baby-step key");
  for (u32 g = 1; g < n2; g++)
    if (!giant[g - 1]) return fail(CKKS_EINVAL, "null giant-step key");
  return CKKS_OK;
}
int decoder_check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (!ws || ((uintptr_t)ws & 255)) return fail(CKKS_EWORKSPACE, "workspace is null or not 256-byte aligned");
  if (ws_bytes < need)
    return fail(CKKS_EWORKSPACE, "workspace too small: need " + std::to_string(need) + " bytes, got " + std::to_string(ws_bytes));
  return CKKS_OK;
}

// ---- attention over a paged cache ----
struct PagedAttn : Decoder {
  u32 rows, squarings, limbs_out;
  u64* sums;               // [rows]: sums of weighted values in three components
  struct Pair {
    u32 row;
    bool first;            // of its row
    const u64 *k, *v;
  };
  std::vector<Pair> pairs; // of the slice that is being gathered

  void shape(const ckks_ctx* c_, u32 rows_, u64 npairs, u32 nlimbs_, u32 n1_, u32 n2_, u32 squarings_) {
    cc = c_, rows = rows_, nlimbs = nlimbs_, n1 = n1_, n2 = n2_, squarings = squarings_;
    limbs_out = nlimbs - 1 - squarings;
    slice = decoder_slice(cc, std::max<u64>(npairs, rows));
  }
  size_t carve(char* ws) {
    Carve w{ws};
    sums = w.words((size_t)rows * 3 * poly(limbs_out));
    carve_common(w);
    return w.used;
  }
  // Scores of the gathered pairs and their weighted values.
  int flush(const u64* q, u32 k_limbs, u32 v_limbs, int64_t bias) {
    int rc;
    const u32 n = (u32)pairs.size();
    for (u32 i = 0; i < n; i += DECODER_PAIRS) {
      const u32 cnt = std::min<u32>(DECODER_PAIRS, n - i);
      PairArgs a;
      a.q = cts(q, nlimbs);
      a.key_comp = poly(k_limbs);
      if ((rc = product_out(&a.o, d + i * 3 * poly(nlimbs), n, nlimbs, n1 == 1 && n2 == 1))) return rc;
      a.o.last += 2 * i * a.o.last_stride;
      a.mods = c->d_mods;
      a.logN = c->logN;
      a.fp_on = (u32)fp_on();
      for (u32 k = 0; k < cnt; k++) a.row[k] = pairs[i + k].row, a.key[k] = pairs[i + k].k;
      ProfScope ps(c, PK_PAIR_PRODUCTS, st);
      hipLaunchKernelGGL(pair_products_kernel, dim3(c->N / 512, nlimbs, cnt), dim3(256), 0, st, a);
      HIP_TRY(hipGetLastError());
    }
    u64* u;
    if ((rc = slot_sum(u, n))) return rc;
    u32 limbs = nlimbs - 1;
    long long add = bias;
    for (u32 s = 0; s < squarings; s++) {
      ProductArgs a{};
      a.x = cts(u, limbs);
      a.factor = 1;
      a.fx.add = a.fy.add = add;
      if ((rc = products(a, n, limbs, true))) return rc;
      if ((rc = relin(u, d, n, limbs, true))) return rc;
      add = 0;
      limbs--;
    }
    for (u32 i = 0; i < n; i += DECODER_PAIRS) {
      const u32 cnt = std::min<u32>(DECODER_PAIRS, n - i);
      ValueArgs a;
      a.u = cts(u + i * 2 * poly(limbs), limbs);
      a.value_comp = poly(v_limbs);
      a.out = sums;
      a.mods = c->d_mods;
      a.bias = add;
      a.logN = c->logN;
      a.nlimbs = limbs;
      a.fp_on = (u32)fp_on();
      u32 r = 0;
      for (u32 k = 0; k < cnt; k++) {
        const Pair& p = pairs[i + k];
        if (k == 0 || p.first) a.begin[r] = k, a.row[r++] = p.row | (p.first ? 0 : 1u << 31);
        a.value[k] = p.v;
      }
      a.begin[r] = cnt;
      ProfScope ps(c, PK_WEIGHTED_VALUES, st);
      hipLaunchKernelGGL(weighted_values_kernel, dim3(c->N / 512, limbs, r), dim3(256), 0, st, a);
      HIP_TRY(hipGetLastError());
    }
    pairs.clear();
    return CKKS_OK;
  }
};

// The cached tokens that the query at position t sees: [0, head) and [tail, t].
struct Visible {
  u32 head, tail;
  Visible(u32 t, u32 window, u32 sinks) {
    tail = window == 0 || t < window ? 0 : t - window + 1;
    head = std::min(sinks, tail);
  }
  u64 count(u32 t) const { return (u64)head + (t - tail + 1); }
};

struct CacheArgs {
  uint32_t seqs;
  const uint32_t *new_lens, *lens;
  uint32_t page_tokens, k_limbs, v_limbs;
};
// Checks a cache's description; rows: all new tokens.
int cache_check(const ckks_ctx* c, const CacheArgs& a, const void* k_pages, const void* v_pages, u64* rows) {
  if (!a.new_lens || !a.lens || !k_pages || !v_pages) return fail(CKKS_EINVAL, "null argument");
  if (a.page_tokens == 0) return fail(CKKS_ESHAPE, "page_tokens must be positive");
  if (a.k_limbs == 0 || a.k_limbs > c->nq || a.v_limbs == 0 || a.v_limbs > c->nq)
    return fail(CKKS_ESHAPE, "k_limbs and v_limbs must be in [1, L+1]");
  *rows = 0;
  for (u32 b = 0; b < a.seqs; b++) {
    if (a.new_lens[b] > a.lens[b]) return fail(CKKS_ESHAPE, "a sequence has more new tokens than tokens");
    if (a.lens[b] > 0x7FFFFFFFu) return fail(CKKS_ESHAPE, "a sequence is too long");
    *rows += a.new_lens[b];
  }
  if (*rows > 32767) return fail(CKKS_ESHAPE, "too many new tokens for one call");
  return CKKS_OK;
}

// ---- root-mean-square norm ----
struct RmsNorm : Decoder {
  u32 B, iterations, limbs_out;
  u64 *h, *uw, *g_in, *g;  // [part] each: the sum with the residual, Newton's two products, the weighted input and it rescaled
  char* rs;
  size_t rs_bytes;
  u32 part;                // ciphertexts of the batch worked on at a time

  void shape(const ckks_ctx* c_, u32 B_, u32 nlimbs_, u32 n1_, u32 n2_, u32 iterations_) {
    cc = c_, B = B_, nlimbs = nlimbs_, n1 = n1_, n2 = n2_, iterations = iterations_;
    limbs_out = nlimbs - 1 - 2 * iterations;
    slice = decoder_slice(cc, 2 * (u64)B);
    part = std::max(1u, slice / 2);
    slice = 2 * part;
  }
  size_t carve(char* ws) {
    Carve w{ws};
    h = w.words((size_t)part * 2 * poly(nlimbs));
    uw = w.words((size_t)2 * part * 2 * poly(nlimbs));
    g_in = w.words((size_t)part * 2 * poly(limbs_out + 1));
    g = w.words((size_t)part * 2 * poly(limbs_out));
    rs_bytes = ckks_workspace_bytes(cc, CKKS_OP_RESCALE, part, limbs_out + 1, 0);
    rs = w.bytes(rs_bytes);
    carve_common(w);
    return w.used;
  }
  // A part of the batch.
  int run(u64* out, u64* h_out, const u64* x, const u64* res, const u64* gain, int64_t square, int64_t eps, int64_t start,
          const int64_t* factors, u32 n) {
    int rc;
    const u64* in = res ? h_out ? h_out : h : x;
    ProductArgs a{};
    a.x = cts(x, nlimbs);
    a.plus = res;
    a.sum = res ? const_cast<u64*>(in) : nullptr;
    a.factor = square;
    if ((rc = products(a, n, nlimbs, n1 == 1 && n2 == 1))) return rc;
    u64* mean;   // without eps, which the products add
    if ((rc = slot_sum(mean, n))) return rc;
    u32 limbs = nlimbs - 1;
    // y: start - (mean + eps) until the first step has put it where the mean is not
    u64 *next = mean == y[0] ? y[1] : y[0], *v = mean;
    Affine fy{start, eps, 1};
    for (u32 k = 0; k < iterations; k++) {
      ProductArgs p{};
      p.x = cts(mean, nlimbs - 1);
      p.fx.add = eps;
      if (v != mean) p.y = cts(v, limbs);
      p.fy = fy;
      p.factor = 1;
      p.second = n;
      if ((rc = products(p, n, limbs, true))) return rc;
      if ((rc = relin(uw, d, 2 * n, limbs, true))) return rc;
      ProductArgs s{};
      s.x = cts(uw, limbs - 1);
      s.y = cts(uw + n * 2 * poly(limbs - 1), limbs - 1);
      s.factor = -1;
      s.z = cts(v, limbs);
      s.fz = fy;
      s.z_factor = factors[k];
      if ((rc = products(s, n, limbs - 1, true))) return rc;
      if ((rc = relin(next, d, n, limbs - 1, true))) return rc;
      v = next;
      fy = Affine{0, 0, 0};
      limbs -= 2;
    }
    ProductArgs e{};
    e.x = cts(in, nlimbs);
    e.y = cts(v, limbs);
    e.fy = fy;
    e.factor = 1;
    if (gain) {
      {
        ProfScope ps(c, PK_CUT_PMULT, st);
        hipLaunchKernelGGL(cut_pmult_kernel, dim3(c->N / 512, limbs + 1, 2 * n), dim3(256), 0, st, g_in, e.x, gain, c->d_mods, c->logN,
                           limbs + 1);
        HIP_TRY(hipGetLastError());
      }
      if ((rc = ckks_rescale(c, (uint64_t*)g, (const uint64_t*)g_in, n, limbs + 1, rs, rs_bytes, st))) return rc;
      e.x = cts(g, limbs);
    }
    if ((rc = products(e, n, limbs, false))) return rc;
    return relin(out, d, n, limbs, false);
  }
};
int norm_check(const ckks_ctx* c, u32 B, u32 nlimbs, u32 n1, u32 n2, u32 iterations) {
  int rc = decoder_check(c, B, nlimbs, n1, n2);
  if (rc) return rc;
  if (B > 32767) return fail(CKKS_ESHAPE, "batch must be in [1, 32767]");
  if (iterations > 64 || nlimbs < 2 + 2 * iterations) return fail(CKKS_ESHAPE, "the norm takes 1 + 2 iterations limbs and leaves one or more");
  return CKKS_OK;
}

}  // namespace

extern "C" {

int ckks_kv_append(ckks_ctx* c, const uint64_t* k, const uint64_t* v, uint32_t in_limbs, uint32_t seqs, const uint32_t* new_lens,
                   const uint32_t* lens, uint64_t* const* k_pages, uint64_t* const* v_pages, uint32_t page_tokens, uint32_t k_limbs,
                   uint32_t v_limbs, void* stream) {
  return guarded([&]() -> int {
    int rc = check_common(c, 1, in_limbs);
    if (rc) return rc;
    u64 rows;
    if ((rc = cache_check(c, {seqs, new_lens, lens, page_tokens, k_limbs, v_limbs}, k_pages, v_pages, &rows))) return rc;
    if (k_limbs > in_limbs || v_limbs > in_limbs) return fail(CKKS_ESHAPE, "the cache keeps more limbs than the new tokens have");
    if (rows == 0) return CKKS_OK;
    if (!k || !v) return fail(CKKS_EINVAL, "null argument");
    const size_t in_bytes = (size_t)rows * 2 * in_limbs * c->N * 8;
    std::vector<u64*> to[2];
    std::vector<std::pair<uintptr_t, uintptr_t>> ranges;
    size_t page = 0;
    for (u32 b = 0; b < seqs; b++) {
      for (u32 t = lens[b] - new_lens[b]; t < lens[b]; t++)
        for (int i = 0; i < 2; i++) {
          u64* p = (u64*)(i ? v_pages : k_pages)[page + t / page_tokens];
          if (!p) return fail(CKKS_EINVAL, "null page for a new token");
          const u64 words = 2 * (u64)(i ? v_limbs : k_limbs) * c->N;
          p += (u64)(t % page_tokens) * words;
          if (overlap(p, words * 8, k, in_bytes) || overlap(p, words * 8, v, in_bytes)) return fail(CKKS_EINVAL, "a page overlaps k or v");
          to[i].push_back(p);
          ranges.push_back({(uintptr_t)p, (uintptr_t)(p + words)});
        }
      page += (lens[b] + (size_t)page_tokens - 1) / page_tokens;
    }
    std::sort(ranges.begin(), ranges.end());
    for (size_t i = 1; i < ranges.size(); i++)
      if (ranges[i].first < ranges[i - 1].second) return fail(CKKS_EINVAL, "two new tokens have the same place");
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(CKKS_EHIP, "cannot select the context's device");
    for (u32 i = 0; i < rows; i += DECODER_PAIRS) {
      const u32 cnt = std::min<u32>(DECODER_PAIRS, (u32)rows - i);
      AppendArgs a;
      a.k = (const u64*)k;
      a.v = (const u64*)v;
      a.logN = c->logN;
      a.in_limbs = in_limbs;
      a.k_limbs = k_limbs;
      a.v_limbs = v_limbs;
      a.ntokens = cnt;
      a.first = i;
      for (u32 t = 0; t < cnt; t++) a.to[t] = to[0][i + t], a.to[cnt + t] = to[1][i + t];
      ProfScope ps(c, PK_KV_APPEND, (hipStream_t)stream);
      hipLaunchKernelGGL(kv_append_kernel, dim3(c->N / 512, std::max(k_limbs, v_limbs), 4 * cnt), dim3(256), 0, (hipStream_t)stream, a);
      HIP_TRY(hipGetLastError());
    }
    return CKKS_OK;
  });
}

size_t ckks_attn_workspace_bytes(const ckks_ctx* c, uint32_t rows, uint64_t pairs, uint32_t nlimbs, uint32_t n1, uint32_t n2,
                                 uint32_t squarings) {
  size_t bytes = 0;
  guarded([&]() -> int {
    const int rc = decoder_check(c, 1, nlimbs, n1, n2);
    if (rc) return rc;
    if (rows == 0 || rows > 32767 || pairs < rows) return fail(CKKS_ESHAPE, "every new token sees itself at least");
    if (nlimbs < 2 || squarings > nlimbs - 2) return fail(CKKS_ESHAPE, "the scores take 1 + squarings limbs and leave one or more");
    PagedAttn f;
    f.shape(c, rows, pairs, nlimbs, n1, n2, squarings);
    bytes = f.carve(nullptr);
    return CKKS_OK;
  });
  return bytes;
}

int ckks_attn_paged(ckks_ctx* c, uint64_t* o_out, const uint64_t* q, uint32_t nlimbs, uint32_t seqs, const uint32_t* new_lens,
                    const uint32_t* lens, const uint64_t* const* k_pages, const uint64_t* const* v_pages, uint32_t page_tokens,
                    uint32_t k_limbs, uint32_t v_limbs, uint32_t window, uint32_t sinks, int64_t bias, uint32_t squarings, uint32_t n1,
                    uint32_t n2, uint32_t stride, const uint64_t* evk_mult, const uint64_t* const* evk_baby,
                    const uint64_t* const* evk_giant, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    int rc = decoder_check(c, 1, nlimbs, n1, n2);
    if (rc) return rc;
    if (nlimbs < 2 || squarings > nlimbs - 2) return fail(CKKS_ESHAPE, "the scores take 1 + squarings limbs and leave one or more");
    u64 rows;
    if ((rc = cache_check(c, {seqs, new_lens, lens, page_tokens, k_limbs, v_limbs}, k_pages, v_pages, &rows))) return rc;
    if (k_limbs < nlimbs || v_limbs < nlimbs - 1 - squarings) return fail(CKKS_ESHAPE, "the cache has fewer limbs than the call needs");
    if ((rc = decoder_check_keys(n1, n2, stride, evk_mult, evk_baby, evk_giant))) return rc;
    if (rows == 0) return CKKS_OK;
    if (!o_out || !q) return fail(CKKS_EINVAL, "null argument");
    u64 npairs = 0;
    size_t page = 0;
    const size_t out_bytes = (size_t)rows * 2 * (nlimbs - 1 - squarings) * c->N * 8;
    if (overlap(o_out, out_bytes, q, (size_t)rows * 2 * nlimbs * c->N * 8)) return fail(CKKS_EINVAL, "o_out overlaps q");
    const u64 k_words = 2 * (u64)k_limbs * c->N, v_words = 2 * (u64)v_limbs * c->N;
    for (u32 b = 0; b < seqs; b++) {
      const size_t npages = (lens[b] + (size_t)page_tokens - 1) / page_tokens;
      if (new_lens[b]) {
        const u32 t0 = lens[b] - new_lens[b];
        for (u32 t = t0; t < lens[b]; t++) npairs += Visible(t, window, sinks).count(t);
        // the first new token sees the oldest of the window, the last one the most sinks
        const u32 head = Visible(lens[b] - 1, window, sinks).head, tail = Visible(t0, window, sinks).tail;
        for (size_t i = 0; i < npages; i++) {
          if (i * page_tokens >= head && (i + 1) * page_tokens <= tail) continue;   // nobody reads this page
          const uint64_t *kp = k_pages[page + i], *vp = v_pages[page + i];
          if (!kp || !vp) return fail(CKKS_EINVAL, "null page that a new token sees");
          if (overlap(o_out, out_bytes, kp, page_tokens * k_words * 8) || overlap(o_out, out_bytes, vp, page_tokens * v_words * 8))
            return fail(CKKS_EINVAL, "o_out overlaps a page");
        }
      }
      page += npages;
    }
    PagedAttn f;
    f.shape(c, (u32)rows, npairs, nlimbs, n1, n2, squarings);
    if ((rc = decoder_check_ws(ws, ws_bytes, f.carve((char*)ws)))) return rc;
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(CKKS_EHIP, "cannot select the context's device");
    f.keys(c, stride, evk_mult, evk_baby, evk_giant, stream);
    f.pairs.reserve(f.slice);
    u32 row = 0;
    page = 0;
    for (u32 b = 0; b < seqs; b++) {
      for (u32 t = lens[b] - new_lens[b]; t < lens[b]; t++, row++) {
        const Visible see(t, window, sinks);
        bool first = true;
        for (u32 s = see.head ? 0 : see.tail; s <= t; s = s + 1 == see.head ? see.tail : s + 1) {
          const u64 *kp = (const u64*)k_pages[page + s / page_tokens], *vp = (const u64*)v_pages[page + s / page_tokens];
          f.pairs.push_back({row, first, kp + (u64)(s % page_tokens) * k_words, vp + (u64)(s % page_tokens) * v_words});
          first = false;
          if (f.pairs.size() == f.slice && (rc = f.flush((const u64*)q, k_limbs, v_limbs, bias))) return rc;
        }
      }
      page += (lens[b] + (size_t)page_tokens - 1) / page_tokens;
    }
    if (!f.pairs.empty() && (rc = f.flush((const u64*)q, k_limbs, v_limbs, bias))) return rc;
    for (u32 r = 0; r < rows; r += f.slice) {
      const u32 n = std::min(f.slice, (u32)rows - r);
      if ((rc = f.relin((u64*)o_out + r * 2 * f.poly(f.limbs_out), f.sums + r * 3 * f.poly(f.limbs_out), n, f.limbs_out, false))) return rc;
    }
    return CKKS_OK;
  });
}

size_t ckks_rmsnorm_workspace_bytes(const ckks_ctx* c, uint32_t B, uint32_t nlimbs, uint32_t n1, uint32_t n2, uint32_t iterations) {
  size_t bytes = 0;
  guarded([&]() -> int {
    const int rc = norm_check(c, B, nlimbs, n1, n2, iterations);
    if (rc) return rc;
    RmsNorm f;
    f.shape(c, B, nlimbs, n1, n2, iterations);
    bytes = f.carve(nullptr);
    return CKKS_OK;
  });
  return bytes;
}

int ckks_rmsnorm(ckks_ctx* c, uint64_t* ct_out, uint64_t* h_out, const uint64_t* ct_x, const uint64_t* ct_res, const uint64_t* gain,
                 int64_t square, int64_t eps, int64_t start, const int64_t* factors, uint32_t iterations, uint32_t B, uint32_t nlimbs,
                 uint32_t n1, uint32_t n2, uint32_t stride, const uint64_t* evk_mult, const uint64_t* const* evk_baby,
                 const uint64_t* const* evk_giant, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    int rc = norm_check(c, B, nlimbs, n1, n2, iterations);
    if (rc) return rc;
    if ((rc = decoder_check_keys(n1, n2, stride, evk_mult, evk_baby, evk_giant))) return rc;
    if (!ct_out || !ct_x || (iterations && !factors)) return fail(CKKS_EINVAL, "null argument");
    if (h_out && !ct_res) return fail(CKKS_EINVAL, "h_out is the sum with a residual, which is not given");
    const u32 L = nlimbs - 1 - 2 * iterations;
    const size_t in_bytes = (size_t)B * 2 * nlimbs * c->N * 8, out_bytes = (size_t)B * 2 * L * c->N * 8, gain_bytes = (size_t)(L + 1) * c->N * 8;
    if (overlap(ct_out, out_bytes, ct_x, in_bytes) || (ct_res && overlap(ct_out, out_bytes, ct_res, in_bytes)) ||
        (gain && overlap(ct_out, out_bytes, gain, gain_bytes)))
      return fail(CKKS_EINVAL, "ct_out overlaps an input");
    if (h_out) {
      if (overlap(h_out, in_bytes, ct_out, out_bytes) || (gain && overlap(h_out, in_bytes, gain, gain_bytes)))
        return fail(CKKS_EINVAL, "h_out overlaps ct_out or gain");
      for (const uint64_t* x : {ct_x, ct_res})
        if (h_out != x && overlap(h_out, in_bytes, x, in_bytes)) return fail(CKKS_EINVAL, "h_out must be an input itself or not overlap it");
    }
    RmsNorm f;
    f.shape(c, B, nlimbs, n1, n2, iterations);
    if ((rc = decoder_check_ws(ws, ws_bytes, f.carve((char*)ws)))) return rc;
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(CKKS_EHIP, "cannot select the context's device");
    f.keys(c, stride, evk_mult, evk_baby, evk_giant, stream);
    const u64 ct = 2 * f.poly(nlimbs), ct_o = 2 * f.poly(L);
    for (u32 b = 0; b < B; b += f.part)
      if ((rc = f.run((u64*)ct_out + b * ct_o, h_out ? (u64*)h_out + b * ct : nullptr, (const u64*)ct_x + b * ct,
                      ct_res ? (const u64*)ct_res + b * ct : nullptr, (const u64*)gain, square, eps, start, factors,
                      std::min(f.part, B - b))))
        return rc;
    return CKKS_OK;
  });
}

}  // extern "C"
