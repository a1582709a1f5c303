// Attention of new tokens over the compacted cache (what the target does with it after the mask was applied), with an account of the softmax
// weight that every cached token gets.
//
// Three steps.  attend_wave_kernel and, for more than 32 queries per key, attend_block_kernel: waves take shares of a row's keys (a row's new tokens
// are few, its keys many) and leave, for each query, the share's reference m (a logit), its sum l of 2^(c (s - m)), c = log2(e) / sqrt(D), and its
// output, not divided yet, in fp32.  attend_finish_kernel: shares are joined, in order, and where the logits were kept, every key's probabilities are added
// to the account.  attend_account_kernel: where they were not (many queries), they are computed once more.  Rows of few keys go through
// attend_row_kernel, which does all of it.  No sum's order depends on timing.
//
// A tile is 32 keys.  S^T = K Q^T on 16 x 16 x 32 matrix instructions: a lane has one query (column) and 8 of the keys, so that a softmax needs
// nothing from other lanes but a sum over four of them at the end, and its probabilities are the second product's operand as they lie (O^T =
// V^T P^T); V is transposed on its way out of LDS.  K and V go into LDS without registers, two stages ahead.
#include "common.hpp"
#include "kernels.hpp"

namespace pkv {
namespace {

template <int D>
constexpr float kScale = 1.4426950408889634f / (D == 64 ? 8.0f : 11.313708498984761f);  // of logits, for exponents of 2
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLow = -3.4028235e38f;  // the reference of no logits: none lies below
// Up to here an exponent c s - m is one fma, m a scaled reference or log-sum-exp: rounding m leaves 2^-13 of a probability at most.  Beyond, it
// would soon leave whole powers of 2, and the exponent is that of a difference of logits, c (s - r).
constexpr float kFar = 4096.0f;
constexpr int kTile = 32;               // keys per step of a wave
constexpr int kXcds = 8;
constexpr int kMerge = 4;               // waves that are joined in LDS
constexpr int64_t kKeptQueries = 32;    // up to this many queries per key, logits are kept for the account

template <bool F16>
struct Elem {
  static __device__ __forceinline__ uint16_t narrow(float f) {
    if constexpr (F16) return __builtin_bit_cast(uint16_t, (_Float16)f);
    else return f32_to_bf16_bits(f);
  }
  static __device__ __forceinline__ u32x2 narrow4(f32x4 y) {
    return u32x2{narrow(y[0]) | (uint32_t)narrow(y[1]) << 16, narrow(y[2]) | (uint32_t)narrow(y[3]) << 16};
  }
  static constexpr uint32_t kExp = F16 ? 0x7c00u : 0x7f80u;  // all ones: not finite
  static constexpr uint32_t kOne = F16 ? 0x3c00u : 0x3f80u;
  // Probabilities are relative to their query's reference, which moves so that the largest is 2^kTop.
  // fp16: when a lane's eight come to more than kMost.  Its steps are 2^-24 at the low end, 2^-36 of the largest then.
  // bf16: when all of a lane's so far do, to where those are no more than 2^kSum: a query's in four waves are less than 1, and its output no larger
  // than its values, which may be as large as fp32 holds.  (From 2^-13 to 2^-5 a move is rare; with 2^-9 and 2^-12 for the largest, 512 new tokens on 10 343
  // keys took 140 to 145 us in the blocks of eight waves, 136 so.)
  static constexpr float kTop = F16 ? 11.0f : -16.0f, kSum = -13.0f, kMost = F16 ? 32768.0f : 0.03125f;
  // 2^-kTop: a wave leaves a reference near its largest logit, sums by that, and outputs 2^kTop of those
  static constexpr float kUnit = F16 ? 1.0f / 2048.0f : 65536.0f;
  static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (F16) return mfma_f16_16x16x32(as_f16x8(a), as_f16x8(b), c);
    else return mfma_bf16_16x16x32(as_bf16x8(a), as_bf16x8(b), c);
  }
  // Two probabilities as sums of two 16-bit values each: rounded, and what that leaves.
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ uint32_t first(float p0, float p1) {
    if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0, p1}), f16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0, p1}), bf16x2));
  }
  static __device__ __forceinline__ uint32_t rest(float p0, float p1, uint32_t hi) {
    if constexpr (F16) {
      const f16x2 h = __builtin_bit_cast(f16x2, hi);
      return first(p0 - (float)h[0], p1 - (float)h[1]);
    } else {
      return first(p0 - __uint_as_float(hi << 16), p1 - __uint_as_float(hi & 0xffff0000u));
    }
  }
};

// Tokens of a row of `most`: what the device array says, kept inside the row.
__device__ __forceinline__ int row_len(const int32_t* lens, int64_t row, int64_t most) {
  if (lens == nullptr) return (int)most;
  const int n = lens[row];
  return n < 0 ? 0 : n < most ? n : (int)most;
}
// Own tokens that new token t of T sees: the T new ones are the row's last.
__device__ __forceinline__ int seen(int len, int T, int t) {
  const int n = len - T + 1 + t;
  return n < 0 ? 0 : n;
}

// m % T for 0 <= m < 2^23, which a float holds: inv = 1 / T is off by 2^-24 relative, so the quotient by one at most
__device__ __forceinline__ int remainder_of(int m, int T, float inv) {
  int r = m - (int)((float)m * inv) * T;
  r += r < 0 ? T : 0;
  return r >= T ? r - T : r;
}

// One kind of keys (shared or own) in a launch: `rows` rows of `n` keys, each seen by m queries, in `tiles` tiles of 16 * ct * waves, and cut into
// `splits` shares of `chunk` keys, which `merge` waves cut once more.
struct Keys {
  int64_t rows, n, m, score_stride;
  int splits, chunk, tiles, ct, waves, merge, blocks, first_split, parts;
  float* scores;  // [rows, m, score_stride] logits, or null
};
struct Plan {
  Keys shared, own;
  int64_t queries;
  int splits;      // of both kinds together
  bool one_launch; // few keys: attend_row_kernel
  float* ml;       // [splits, queries] pairs
  float* o;        // [splits, queries, D]
  float* lse;      // [queries] log2(sum 2^(c s)) in the order of q, and behind them in the shared keys' order
  float2* parts;   // the same, as a reference and log2 of the sum by it
  float* part_sums;  // accounts of parts of the queries
};

// A query's reference (a logit), the sum of probabilities by it, and its log2; of nothing +infinity, by which nothing gets a probability.
struct Joined {
  float ref, l, log2;
};
__device__ __forceinline__ float log2_of(float l) { return l == 0.0f ? -kNegInf : __builtin_amdgcn_logf(l); }

// Where query m of a row's m queries lies in q.  Shared keys: row = head, queries (sequence, group head, token).
__device__ __forceinline__ int64_t query_at(bool shared, int64_t row, int m, int per, int64_t heads) {
  return shared ? ((int64_t)(m / per) * heads + row) * per + m % per : row * per + m;
}

template <int D>
__device__ __forceinline__ int swizzle(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }

// A step's 16-bit values transposed: fragment d has features 16 d + lane % 16 of keys 4 (lane / 16) + 0..3 and those 16 further on.  `at`: LDS
// bytes of this lane's piece of fragment 0; the pieces of fragment d lie (d << 5) away by exclusive or, 16 keys further on `next` bytes.  The
// waits are in the same block as the reads (the compiler, with its own reads, waits for all loads under way as well: they might write there).
template <int NEXT>
__device__ __forceinline__ void read_transposed(uint32_t at, int d0, u32x4 (&f)[4]) {
  u32x2 x[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
      : "v"(at ^ (uint32_t)(d0 << 5)), "v"(at ^ (uint32_t)((d0 + 1) << 5)), "v"(at ^ (uint32_t)((d0 + 2) << 5)), "v"(at ^ (uint32_t)((d0 + 3) << 5)),
        "n"(NEXT)
      : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = u32x4{x[2 * i][0], x[2 * i][1], x[2 * i + 1][0], x[2 * i + 1][1]};
}

// A block's share: keys [begin, end) of a row for 16 * CT * W queries.  V = 1: each of the W waves has 16 * CT of them, and the waves share the
// keys' tiles.  W = 1: each of the V waves has all of them and keys of its own, and what the waves have is joined in LDS.
template <int D, bool F16, int CT, int W, int V>
struct Part {
  static_assert(W == 1 || V == 1, "waves share keys or queries");
  static constexpr int SUB = W > 1 ? 2 : 1, KEYS = kTile * SUB;  // tiles, keys of a stage
  using E = Elem<F16>;
  static constexpr int CPR = D / 8, KK = D / 32, DT = D / 16;  // 16-byte pieces per key; products' steps; output tiles
  static constexpr int NL = KEYS * CPR / 64;                   // a stage's loads of K, by a wave
  static constexpr bool PIPE = W == 8;  // products a tile ahead of their exponentials
  static constexpr int STAGES = PIPE ? 4 : 2, STAGE = 2 * NL * 64;
  static constexpr int MINE = 2 * NL / W;                      // loads of a wave per stage
  static_assert(MINE * W == 2 * NL, "the waves share a stage's loads");

  // WHOLE: the share is all of a row, whose outputs are written and whose queries' references and sums are left in `fin`.
  template <bool WHOLE = false>
  static __device__ __forceinline__ void run(const AttendArgs& a, const Plan& p, const Keys& ks, bool shared, int64_t row, int split, int tile0, u32x4* lds,
                                             Joined* fin = nullptr) {
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
    const int member = V == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lds += member * (STAGES * STAGE);
    const int per = (int)(a.group * a.T), T = (int)a.T, M = (int)ks.m;
    const int b0 = tile0 * 16 * CT * W, m0 = b0 + wave * 16 * CT;
    constexpr float c = kScale<D>;
    const int len = row_len(shared ? a.shared_lens : a.lens, row, ks.n);
    // keys that all, and that any, of the block's queries see
    int64_t query[CT];
    int see[CT];
    int least = len, most = len;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int m = m0 + ct * 16 + col, mc = m < M ? m : M - 1;
      query[ct] = query_at(shared, row, mc, per, a.heads);
      see[ct] = shared ? len : seen(len, T, mc % T);
    }
    if (!shared) {
      const int b1 = (b0 + 16 * CT * W < M ? b0 + 16 * CT * W : M) - 1;
      const bool one = b0 / T == b1 / T;  // tokens of one head, in order
      most = seen(len, T, one ? b1 % T : T - 1);
      least = seen(len, T, one ? b0 % T : 0);
    }
    const int begin0 = split * ks.chunk, end0 = begin0 + ks.chunk < most ? begin0 + ks.chunk : most;
    const int mine = V == 1 ? ks.chunk : (ks.chunk / V + kTile - 1) / kTile * kTile;
    const int begin = begin0 + member * mine, end = begin + mine < end0 ? begin + mine : end0;
    const int n_stages = end > begin ? (end - begin + KEYS - 1) / KEYS : 0;

    float m_run[CT], l_run[CT];  // (a reference is scaled, and kTop less than the logit that gets 2^kTop; if `far`, it is that logit)
    bool far = false;
    f32x4 o[DT][CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      m_run[ct] = kLow;
      l_run[ct] = 0.0f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d][ct] = f32x4{0, 0, 0, 0};
    }
    if (n_stages > 0) {
      u32x4 bq[CT][KK];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) bq[ct][kk] = *reinterpret_cast<const u32x4*>((const uint16_t*)a.q + query[ct] * D + kk * 32 + quad * 8);
      const uint8_t* kb = (const uint8_t*)(shared ? a.k_shared : a.k) + ((size_t)row * ks.n + begin) * (D * 2);
      const uint8_t* vb = (const uint8_t*)(shared ? a.v_shared : a.v) + ((size_t)row * ks.n + begin) * (D * 2);
      typedef const __attribute__((address_space(1))) void* gptr_t;
      typedef __attribute__((address_space(3))) void* lptr_t;
      // Stage t straight into LDS, a key's pieces exchanged (swizzle) so that fragments are read from all banks.  Keys behind the last are the
      // last one again: nothing behind it is touched.
      const int r0 = wave * (64 / CPR) + lane / CPR, piece = (lane % CPR) ^ swizzle<D>(r0);
      auto fetch = [&](int t, int stage) __attribute__((always_inline)) {
        u32x4* st = lds + stage * STAGE + wave * 64;
        const int last = end - 1 - begin - t * KEYS;
        const uint8_t *kt = kb + (size_t)t * (KEYS * D * 2), *vt = vb + (size_t)t * (KEYS * D * 2);
        static_for<NL / W>([&](auto ic) __attribute__((always_inline)) {
          constexpr int i = decltype(ic)::value, step = i * W * (64 / CPR), turn = D == 128 ? step & 15 : (step >> 1) & 7;  // (its bits are not r0's)
          const int r = r0 + step, at = (r < last ? r : last) * (D * 2) + (piece ^ turn) * 16;
          __builtin_amdgcn_global_load_lds((gptr_t)(kt + at), (lptr_t)(st + i * W * 64), 16, 0, 0);
          __builtin_amdgcn_global_load_lds((gptr_t)(vt + at), (lptr_t)(st + (NL + i * W) * 64), 16, 0, 0);
        });
      };
      // S^T of a tile: a lane has the logits of its query (column) with keys 4 quad + r and 16 + 4 quad + r
      auto read_k = [&](const u32x4* st, u32x4 (&f)[2][KK]) __attribute__((always_inline)) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            const int r = kt * 16 + col;
            f[kt][kk] = st[r * CPR + ((kk * 4 + quad) ^ swizzle<D>(r))];
          }
      };
      auto logits = [&](const u32x4 (&f)[2][KK], f32x4 (&s)[2][CT]) __attribute__((always_inline)) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) s[kt][ct] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[kt][ct] = E::mfma(f[kt][kk], bq[ct][kk], s[kt][ct]);
      };
      // Probabilities by the reference that there is; only where a lane's come to more than kMost are the logits' maxima taken, the
      // reference moved and the probabilities computed again (at first always).
      auto probabilities = [&](const f32x4 (&s)[2][CT], int ct, float (&pf)[8]) __attribute__((always_inline)) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          pf[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 2][ct][i & 3], c, -m_run[ct]));
          sum += pf[i];
        }
        return sum;
      };
      auto keep_reference = [&](const f32x4 (&s)[2][CT], float (&pf)[CT][8], float (&sum)[CT]) __attribute__((always_inline)) {
        bool much = false;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) much = much || !((F16 ? sum[ct] : l_run[ct] + sum[ct]) <= E::kMost);
        if (__builtin_expect(far || __builtin_amdgcn_ballot_w64(much) != 0, 0)) {
          float top[CT];
          bool huge = false;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            top[ct] = max3f(s[0][ct][0], s[0][ct][1], s[0][ct][2]);
            top[ct] = max3f(top[ct], s[0][ct][3], s[1][ct][0]);
            top[ct] = max3f(top[ct], s[1][ct][1], s[1][ct][2]);
            top[ct] = quads_max(__builtin_fmaxf(top[ct], s[1][ct][3]));
            huge = huge || (__builtin_fabsf(top[ct]) * c > kFar && top[ct] != kNegInf);
          }
          const bool was = far;
          far = was || __builtin_amdgcn_ballot_w64(huge) != 0;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            const float up = F16 ? 0.0f : __builtin_fmaxf(__builtin_amdgcn_logf(quads_max(l_run[ct])) - E::kSum, 0.0f);  // (log2)
            float f;
            if (far) {
              const float old = was ? m_run[ct] : (m_run[ct] + E::kTop) * (1.0f / c), r = max3f(old + up / c, top[ct], kLow);
              f = __builtin_amdgcn_exp2f(was ? (old - r) * c : __builtin_fmaf(-r, c, m_run[ct] + E::kTop));
              m_run[ct] = r;
              sum[ct] = 0.0f;
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                pf[ct][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 2][ct][i & 3] - r, c, E::kTop));
                sum[ct] += pf[ct][i];
              }
            } else {
              const float m = __builtin_fmaxf(m_run[ct] + up, top[ct] * c - E::kTop);
              f = __builtin_amdgcn_exp2f(m_run[ct] - m);
              m_run[ct] = m;
              sum[ct] = probabilities(s, ct, pf[ct]);
            }
            l_run[ct] *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d][ct] *= f;
          }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) l_run[ct] += sum[ct];
      };
      auto place_v = [&](const u32x4* vst) __attribute__((always_inline)) {  // this lane's piece of the first transposed fragment
        const int vr = quad * 4 + (col >> 2);
        return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)(vst + vr * CPR + (((col >> 1) & 1) ^ swizzle<D>(vr))) + (col & 1) * 8;
      };
      auto tile = [&](int n0, const u32x4* st, auto cut_c) __attribute__((always_inline)) {  // keys from n0 on
        constexpr bool cut = decltype(cut_c)::value;
        f32x4 s[2][CT];
        {
          u32x4 f[2][KK];
          read_k(st, f);
          logits(f, s);
        }
        if (W == 1 && ks.scores != nullptr) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            const int m = m0 + ct * 16 + col;
            if (m < M) {
              float* at = ks.scores + ((size_t)row * M + m) * ks.score_stride + n0 + quad * 4;
              *reinterpret_cast<f32x4*>(at) = s[0][ct];
              *reinterpret_cast<f32x4*>(at + 16) = s[1][ct];
            }
          }
        }
        u32x4 hi[CT], lo[CT];
        float pf[CT][8], sum[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          if constexpr (cut) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              s[i >> 2][ct][i & 3] = n0 + (i >> 2) * 16 + quad * 4 + (i & 3) < see[ct] ? s[i >> 2][ct][i & 3] : kNegInf;
          }
          sum[ct] = probabilities(s, ct, pf[ct]);
        }
        keep_reference(s, pf, sum);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            hi[ct][i] = E::first(pf[ct][2 * i], pf[ct][2 * i + 1]);
            lo[ct][i] = E::rest(pf[ct][2 * i], pf[ct][2 * i + 1], hi[ct][i]);
          }
        // O^T += V^T P^T: 16 features by the keys that the lane's probabilities belong to
        const uint32_t at = place_v(st + NL * 64);
        bool bad = false;
#pragma unroll
        for (int d0 = 0; d0 < DT; d0 += 4) {
          u32x4 v[4];
          read_transposed<16 * D * 2>(at, d0, v);
          if constexpr (cut) {
            // values that are not finite must not meet the zero probabilities of queries that do not see them
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const uint32_t x = v[i >> 2][i & 3];
              const bool x0 = (x & E::kExp) == E::kExp, x1 = (x >> 16 & E::kExp) == E::kExp;
              bad = bad || x0 || x1;
              v[i >> 2][i & 3] = x & ((x0 ? 0u : 0xffffu) | (x1 ? 0u : 0xffff0000u));
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) o[d0 + i][ct] = E::mfma(v[i], hi[ct], o[d0 + i][ct]);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) o[d0 + i][ct] = E::mfma(v[i], lo[ct], o[d0 + i][ct]);
        }
        if constexpr (cut) {
          if (__builtin_expect(__builtin_amdgcn_ballot_w64(bad) != 0, 0)) {
            // How many values of plus and of minus infinity (a NaN is both) each output would have met: products of ones, by queries that see the key.
            uint32_t ones[CT][4];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int n = n0 + (i >> 1) * 16 + quad * 4 + (i & 1) * 2;
                ones[ct][i] = (n < see[ct] ? E::kOne : 0u) | (n + 1 < see[ct] ? E::kOne << 16 : 0u);
              }
#pragma unroll
            for (int d0 = 0; d0 < DT; d0 += 4) {
              u32x4 v[4];
              read_transposed<16 * D * 2>(at, d0, v);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                u32x4 up, down;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  uint32_t u = 0, w = 0;
#pragma unroll
                  for (int sh = 0; sh < 32; sh += 16) {
                    const uint32_t x = v[i][j] >> sh & 0xffffu;
                    const bool odd = (x & E::kExp) == E::kExp;
                    u |= odd && x != (E::kExp | 0x8000u) ? E::kOne << sh : 0u;
                    w |= odd && x != E::kExp ? E::kOne << sh : 0u;
                  }
                  up[j] = u;
                  down[j] = w;
                }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                  const u32x4 m = {ones[ct][0], ones[ct][1], ones[ct][2], ones[ct][3]};
                  const f32x4 tu = E::mfma(up, m, f32x4{0, 0, 0, 0}), td = E::mfma(down, m, f32x4{0, 0, 0, 0});
#pragma unroll
                  for (int e = 0; e < 4; ++e) o[d0 + i][ct][e] += (tu[e] > 0.0f ? -kNegInf : 0.0f) + (td[e] > 0.0f ? kNegInf : 0.0f);
                }
              }
            }
          }
        }
      };
      // Behind the whole tiles, in which an infinite value meets the two parts of a probability, of which the second may be 0 or negative, so that any
      // output that is not finite may have come of one: it is what the row's first `keys` values of its feature say, which all queries see.
      auto infinite = [&](int keys) __attribute__((always_inline)) {
        float odd = 0.0f;  // or NaN
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int e = 0; e < 4; ++e) odd = __builtin_fmaf(o[d][ct][e], 0.0f, odd);
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd != 0.0f) == 0, 1)) return;
        uint32_t up = 0, down = 0;  // bit 4 d + e: some value of feature 16 d + 4 quad + e is infinite upwards, downwards (a NaN is both)
#pragma unroll 1
        for (int n = col; n < keys; n += 16)
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(vb + (size_t)n * (D * 2) + d * 32 + quad * 8);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t v = x[e >> 1] >> (e & 1) * 16 & 0xffffu;
              const bool not_finite = (v & E::kExp) == E::kExp;
              up |= not_finite && v != (E::kExp | 0x8000u) ? 1u << (4 * d + e) : 0u;
              down |= not_finite && v != E::kExp ? 1u << (4 * d + e) : 0u;
            }
          }
#pragma unroll
        for (int off = 1; off < 16; off *= 2) {
          up |= (uint32_t)__shfl_xor((int)up, off, 64);
          down |= (uint32_t)__shfl_xor((int)down, off, 64);
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const float l = quads_sum(l_run[ct]);
          if (l != l) continue;  // (a logit that is not a number: nor is any output)
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool u = up >> (4 * d + e) & 1u, w = down >> (4 * d + e) & 1u;
              o[d][ct][e] = u && w ? __builtin_nanf("") : u ? -kNegInf : w ? kNegInf : o[d][ct][e];
            }
        }
      };
      // A wave alone has two stages under way; waves that share them ask for the next one when all of them have read the one before.
      // (The waits are on every path: it is where the compiler knows that the queries have landed, for which it otherwise waits in every
      // stage, and for the stages under way with them.)
      fetch(0, 0);
      if (W == 1 && n_stages > 1) fetch(1, 1);
      __builtin_amdgcn_s_waitcnt(W == 1 ? MINE == 16 ? 0x4F70 : 0x0F70 | MINE : 0x0F70);
      auto turn = [&](int t) __attribute__((always_inline)) {
          if constexpr (W == 1) {  // stage t has landed; the loads of stage t + 1 may be under way
            __builtin_amdgcn_s_waitcnt(MINE == 16 ? 0x4F70 : 0x0F70 | MINE);
            if (t + 1 == n_stages) __builtin_amdgcn_s_waitcnt(0x0F70);
            asm volatile("" ::: "memory");
          } else {
            __builtin_amdgcn_s_waitcnt(0x0F70);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();  // everyone's part has, and everyone has read the stage whose place takes stage t + 1
            asm volatile("" ::: "memory");
            if (t + 1 < n_stages) fetch(t + 1, (t + 1) % STAGES);
          }
      };
      auto stages = [&](int t0, int t1, auto cut) __attribute__((always_inline)) {
        for (int t = t0; t < t1; ++t) {
          const int stage = t % STAGES;
          turn(t);
#pragma unroll 1
          for (int sub = 0; sub < SUB; ++sub) {
            const int n0 = begin + t * KEYS + sub * kTile;
            if (!decltype(cut)::value || n0 < end) tile(n0, lds + stage * STAGE + sub * (kTile * CPR), cut);
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // all of stage t has been read
          if (W == 1 && t + 2 < n_stages) fetch(t + 2, stage);
        }
      };
      // whole stages that all of the block's queries see, and those behind them (a loop each: where one loop has both kinds of tiles, the
      // compiler moves the outputs from register to register in every tile)
      const int whole = least < end ? least : end, full = whole > begin ? (whole - begin) / KEYS : 0;
      if constexpr (PIPE) {
        // A step has the products of one tile's keys (f, read a step ahead) between the exponentials of the tile before, then that one's products with
        // V: one after the other, matrix and vector instructions of a SIMD's waves take turns.  `ahead` reads the next keys in front of the latter.
        auto step = [&](u32x4 (&f)[2][KK], const u32x4* vst, const f32x4 (&s)[2][CT], f32x4 (&next)[2][CT], auto more, auto ahead)
            __attribute__((always_inline)) {
          float pf[CT][8], sum[CT];
          if constexpr (decltype(more)::value) logits(f, next);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) sum[ct] = probabilities(s, ct, pf[ct]);
          if constexpr (decltype(more)::value) {
#pragma unroll
            for (int i = 0; i < 2 * CT * KK; ++i) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
              __builtin_amdgcn_sched_group_barrier(0x002, 24 / (2 * KK), 0);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          keep_reference(s, pf, sum);
          u32x4 hi[CT], lo[CT];
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              hi[ct][i] = E::first(pf[ct][2 * i], pf[ct][2 * i + 1]);
              lo[ct][i] = E::rest(pf[ct][2 * i], pf[ct][2 * i + 1], hi[ct][i]);
            }
          __builtin_amdgcn_sched_barrier(0);
          ahead();
          __builtin_amdgcn_sched_barrier(0);
          const uint32_t at = place_v(vst);
#pragma unroll
          for (int d0 = 0; d0 < DT; d0 += 4) {
            u32x4 x[4];
            read_transposed<16 * D * 2>(at, d0, x);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
              for (int ct = 0; ct < CT; ++ct) o[d0 + d][ct] = E::mfma(x[d], hi[ct], o[d0 + d][ct]);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
              for (int ct = 0; ct < CT; ++ct) o[d0 + d][ct] = E::mfma(x[d], lo[ct], o[d0 + d][ct]);
            __builtin_amdgcn_sched_barrier(0);
          }
        };
        // behind its barrier stage t may be read
        auto turn_ahead = [&](int t) __attribute__((always_inline)) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_s_barrier();  // everyone's part of stage t has landed, and everyone has read stage t - 2, whose place takes stage t + 2
          asm volatile("" ::: "memory");
          if (t + 2 < n_stages) fetch(t + 2, (t + 2) % STAGES);
        };
        // this wave's part of stage t + 1 has landed; its loads of stage t + 2 may be under way
        auto next_landed = [&](int t) __attribute__((always_inline)) {
          __builtin_amdgcn_s_waitcnt(0x0F70 | MINE);
          if (t + 2 >= n_stages) __builtin_amdgcn_s_waitcnt(0x0F70);
          asm volatile("" ::: "memory");
        };
        int done = 0;
        if (full > 0) {
          static_assert(SUB == 2, "two tiles by name");
          constexpr int TILE = kTile * CPR;
          f32x4 sa[2][CT], sb[2][CT];
          u32x4 f[2][KK];
          if (n_stages > 1) fetch(1, 1);
          next_landed(n_stages > 1 ? -1 : 0);
          turn_ahead(0);
          read_k(lds, f);
          logits(f, sa);
          read_k(lds + TILE, f);
#pragma unroll 1
          for (; done + 1 < full; ++done) {  // sa: of the first tile of stage `done`, f: the second one's keys
            const u32x4 *st = lds + done % STAGES * STAGE, *on = lds + (done + 1) % STAGES * STAGE;
            next_landed(done);
            step(f, st + NL * 64, sa, sb, std::integral_constant<bool, true>{}, [&]() __attribute__((always_inline)) {
              turn_ahead(done + 1);
              read_k(on, f);
            });
            step(f, st + NL * 64 + TILE, sb, sa, std::integral_constant<bool, true>{}, [&]() __attribute__((always_inline)) { read_k(on + TILE, f); });
          }
          const u32x4* st = lds + done % STAGES * STAGE;
          step(f, st + NL * 64, sa, sb, std::integral_constant<bool, true>{}, []() {});
          step(f, st + NL * 64 + TILE, sb, sa, std::integral_constant<bool, false>{}, []() {});
          ++done;
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          infinite(full * KEYS);
        }
        stages(done, n_stages, std::integral_constant<bool, true>{});
      } else {
        stages(0, full, std::integral_constant<bool, false>{});
        if (full > 0) infinite(full * KEYS);
        stages(full, n_stages, std::integral_constant<bool, true>{});
      }
    }
    float own[CT];  // from here on references are logits; what rounding them leaves
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const float r = far ? m_run[ct] : __builtin_fmaxf((m_run[ct] + E::kTop) * (1.0f / c), kLow);
      own[ct] = far ? 1.0f : __builtin_amdgcn_exp2f(__builtin_fmaf(-r, c, m_run[ct] + E::kTop));
      m_run[ct] = r;
    }
    const size_t at = (size_t)(ks.first_split + split) * p.queries;
    if constexpr (V == 1) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const float l = quads_sum(l_run[ct]) * own[ct] * E::kUnit;
        if (m0 + ct * 16 + col < M) {
          if (quad == 0) reinterpret_cast<float2*>(p.ml)[at + query[ct]] = float2{m_run[ct], l};
          if (n_stages > 0) {
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(p.o + (at + query[ct]) * D + d * 16 + quad * 4) = o[d][ct] * own[ct];
          }
        }
      }
    } else {
      // Every member's outputs by the largest reference, then their sum, in the members' order.
      constexpr int Q = 16 * CT, LINE = D + 4;  // (a line's first bank differs from query to query)
      static_assert(V * (Q * LINE + 2 * Q) * 4 <= V * STAGES * STAGE * 16, "the joined outputs lie where the stages were");
      float* all = reinterpret_cast<float*>(lds - member * (STAGES * STAGE));
      float2* ml = reinterpret_cast<float2*>(all + V * Q * LINE);
      __syncthreads();  // everyone has read its last stage
      float l_own[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        l_own[ct] = quads_sum(l_run[ct]) * own[ct] * E::kUnit;
        if (quad == 0) ml[member * Q + ct * 16 + col] = float2{m_run[ct], l_own[ct]};
      }
      __syncthreads();
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float m = kLow, l = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) m = __builtin_fmaxf(m, ml[v * Q + ct * 16 + col].x);
#pragma unroll
        for (int v = 0; v < V; ++v) l = __builtin_fmaf(ml[v * Q + ct * 16 + col].y, __builtin_amdgcn_exp2f((ml[v * Q + ct * 16 + col].x - m) * c), l);
        const float f = __builtin_amdgcn_exp2f((m_run[ct] - m) * c) * own[ct];
#pragma unroll
        for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(all + (member * Q + ct * 16 + col) * LINE + d * 16 + quad * 4) = o[d][ct] * f;
        if (member == 0 && quad == 0) {
          if constexpr (WHOLE) fin[ct * 16 + col] = Joined{m, l, log2_of(m0 + ct * 16 + col < M ? l : 0.0f)};
          else if (m0 + ct * 16 + col < M) reinterpret_cast<float2*>(p.ml)[at + query[ct]] = float2{m, l};
        }
      }
      __syncthreads();
      if (WHOLE || end0 > begin0) {
#pragma unroll
        for (int i = 0; i < Q * D / 4 / (64 * V); ++i) {
          const int x = i * 64 * V + threadIdx.x, q = x / (D / 4), d = x % (D / 4) * 4;
          f32x4 sum = *reinterpret_cast<const f32x4*>(all + q * LINE + d);
#pragma unroll
          for (int v = 1; v < V; ++v) sum += *reinterpret_cast<const f32x4*>(all + (v * Q + q) * LINE + d);
          if constexpr (WHOLE) {
            const float l = fin[q].l;
            const u32x2 r = l == 0.0f ? u32x2{0, 0} : E::narrow4(sum / l * E::kUnit);
            if (m0 + q < M) *reinterpret_cast<u32x2*>((uint16_t*)a.out + query_at(shared, row, m0 + q, per, a.heads) * D + d) = r;
          } else if (m0 + q < M) {
            *reinterpret_cast<f32x4*>(p.o + (at + query_at(shared, row, m0 + q, per, a.heads)) * D + d) = sum;
          }
        }
      }
    }
  }
};

// Blocks that share keys (tiles of one row's queries) follow each other on one XCD, whose L2 then has the keys.
// false: nothing to do
__device__ __forceinline__ bool share_of(int b, const Keys& ks, int64_t& row, int& split, int& tile) {
  const int64_t share = (int64_t)(b / (kXcds * ks.tiles)) * kXcds + b % kXcds;
  tile = b / kXcds % ks.tiles;
  row = share / ks.splits;
  // turned from row to row: with a number of shares that eight divides, one XCD would get every row's first, another every row's last, which
  // rows that are not full do not have (256 rows of up to 8192 keys in 16 shares, 144 us, turned 132)
  split = (int)((share + row) % ks.splits);
  return share < ks.rows * ks.splits;
}

// Few queries per row: V waves for a share of its keys.  CT: of the kind of keys that has the larger tiles.  Bound by reading the cache: 256 rows of up
// to 8192 keys, 4 queries, 540 MB in 116 us (4.6 TB/s; a large copy reaches 5.2), 8 rows of 10 240 in 10.5.  Waves of their own, five of
// which fit a compute unit's LDS, rather than blocks: nothing waits for anything but its own loads.  From 17 queries on what a share leaves is a quarter
// of what it reads, and four waves are joined first (64 rows of up to 4001 keys of 64, 20 queries: 16 us).
template <int D, bool F16, int CT, int V>
__global__ __launch_bounds__(64 * V, CT == 1 ? 2 : 1) void attend_wave_kernel(AttendArgs a, Plan p) {
  __shared__ u32x4 lds[V * Part<D, F16, CT, 1, V>::STAGES * Part<D, F16, CT, 1, V>::STAGE];
  const bool shared = (int)blockIdx.x < p.shared.blocks;
  const Keys& ks = shared ? p.shared : p.own;
  int64_t row;
  int split, tile;
  if (!share_of(shared ? blockIdx.x : blockIdx.x - p.shared.blocks, ks, row, split, tile)) return;
  if (CT == 1 || ks.ct == 1) Part<D, F16, 1, 1, V>::run(a, p, ks, shared, row, split, tile, lds);
  else Part<D, F16, CT, 1, V>::run(a, p, ks, shared, row, split, tile, lds);
}

// Many: W waves of 32 queries share the keys.  2048 queries on 10 343 keys of 128 for each of 8 heads (W = 8), 8.7e10 flop and half as many again for the
// second part of the probabilities, take 139 us, 256 on 32 768 58 (0.94 and 0.89 PFLOP/s with those; a large library product reaches 1.25).  The matrix
// unit is busy for 48 % of that, and no one thing bounds the rest: without the reads of K out of LDS it would be 4 us less, without those of V 8, without exponentials
// 12, without the products with the second part 17.  Half of the waves half a step behind the others, and that part worked out between the products
// with the first, were 2 % slower; other orders of products and exponentials or wave priorities made no difference.
// W = 2: 64 queries on 10 240 keys of 8 rows 19.9 us, W = 4: 128 queries 22.9, where reading the keys alone takes 8 (they ask for a stage when the one
// before has landed, and leave 11 and 21 MB of outputs for 42 MB of keys).
template <int D, bool F16, int W>
__global__ __launch_bounds__(64 * W, W == 2 ? 1 : 2) void attend_block_kernel(AttendArgs a, Plan p, bool shared) {
  __shared__ u32x4 lds[Part<D, F16, 2, W, 1>::STAGES * Part<D, F16, 2, W, 1>::STAGE];
  const Keys& ks = shared ? p.shared : p.own;
  int64_t row;
  int split, tile;
  if (!share_of(blockIdx.x, ks, row, split, tile)) return;
  Part<D, F16, 2, W, 1>::run(a, p, ks, shared, row, split, tile, lds);
}

// Joins the shares' outputs: D / 4 threads hold a share's row, so that a block takes 8 queries of up to four shares (QB = 8), 4 of up to eight, or one
// query's 256 / (D / 4) shares at a time.  Bound by reading them: 16 384 queries of four shares, 36 MB and 4.5 MB written, 9 us (with QB = 4, where half
// of the reads are another's share once more, 12).
template <int D, bool F16, int QB>
__device__ __forceinline__ void join_outputs(const AttendArgs& a, const Plan& p, int block) {
  constexpr int LPR = D / 4, G = 256 / LPR / QB;  // threads per row; shares at a time
  __shared__ float part[256 / LPR][D];
  __shared__ float2 part_ml[256 / LPR];
  constexpr float c = kScale<D>;
  const int tid = threadIdx.x, g = tid / LPR, at = tid % LPR * 4, per = (int)(a.group * a.T);
  const int64_t mine = (int64_t)block * QB + g / G, query = mine < p.queries ? mine : p.queries - 1;
  const float down = (float)__builtin_clz(p.splits) - 32.0f;  // each share 2^down of what it has: their sum is finite where every one is
  float m = kLow, l = 0.0f;
  f32x4 x = {0, 0, 0, 0};
  constexpr int U = 4;
  for (int s0 = g % G; s0 < p.splits; s0 += G * U) {
    float2 ml[U];
    f32x4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // (a share behind the last reads that one and counts nothing; one without keys has left no output)
      const int s = s0 + u * G < p.splits ? s0 + u * G : p.splits - 1;
      ml[u] = reinterpret_cast<const float2*>(p.ml)[(size_t)s * p.queries + query];
      o[u] = *reinterpret_cast<const f32x4*>(p.o + ((size_t)s * p.queries + query) * D + at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u * G >= p.splits || ml[u].y == 0.0f) continue;
      const float top = __builtin_fmaxf(m, ml[u].x), f = __builtin_amdgcn_exp2f((m - top) * c), f2 = __builtin_amdgcn_exp2f(__builtin_fmaf(ml[u].x - top, c, down));
      l = l * f + ml[u].y * f2;
      x = x * f + o[u] * f2;
      m = top;
    }
  }
  if constexpr (G > 1) {
    *reinterpret_cast<f32x4*>(&part[g][at]) = x;
    if (at == 0) part_ml[g] = float2{m, l};
    __syncthreads();
    if (g % G != 0) return;
    for (int i = 1; i < G; ++i) {
      const float2 ml = part_ml[g + i];
      const float top = __builtin_fmaxf(m, ml.x), f = __builtin_amdgcn_exp2f((m - top) * c), f2 = __builtin_amdgcn_exp2f((ml.x - top) * c);
      l = l * f + ml.y * f2;
      x = x * f + *reinterpret_cast<const f32x4*>(&part[g + i][at]) * f2;
      m = top;
    }
  }
  if (mine >= p.queries) return;
  const bool none = l == 0.0f;
  const u32x2 r = none ? u32x2{0, 0} : Elem<F16>::narrow4(x / l * Elem<F16>::kUnit);
  *reinterpret_cast<u32x2*>((uint16_t*)a.out + query * D + at) = r;
  if (at == 0 && p.lse != nullptr) {
    const float2 part = {m, log2_of(l) - down};
    const float v = __builtin_fmaf(m, c, part.y);
    const int64_t row = query / per;  // (sequence, head)
    const int64_t at_shared = p.queries + (row % a.heads * a.batch + row / a.heads) * per + query % per;
    p.lse[query] = p.lse[at_shared] = v;
    p.parts[query] = p.parts[at_shared] = part;
  }
}

// The account of 256 * KP keys of a row from logits that were kept, of up to MQ queries: a chain of loads (lengths; logits, sums and the account; then
// the store) that takes 3 us where little is to be done, otherwise bound by reading the logits (256 rows of up to 8192, 34 MB, 12 us with the outputs).
template <int D, int MQ, int KP>
__device__ __forceinline__ void account_kept(const AttendArgs& a, const Plan& p, const Keys& ks, bool shared, int b) {
  constexpr float c = kScale<D>;
  typedef float keys_t __attribute__((ext_vector_type(KP)));
  __shared__ float2 parts[MQ];
  const int per = (int)(a.group * a.T), M = (int)ks.m, T = (int)a.T;
  const int blocks = (int)((ks.n + 256 * KP - 1) / (256 * KP)), n = b % blocks * (256 * KP) + threadIdx.x * KP;
  const int64_t row = b / blocks;
  const int len = row_len(shared ? a.shared_lens : a.lens, row, ks.n);
  if (b % blocks * (256 * KP) >= len) return;
  // (asked for before the joins: score rows have room for a whole quad)
  keys_t s[MQ];
  static_for<MQ / 4>([&](auto four) __attribute__((always_inline)) {
    constexpr int q = decltype(four)::value * 4;
    if (q >= M) return;
#pragma unroll
    for (int m = q; m < q + 4; ++m)
      s[m] = *reinterpret_cast<const keys_t*>(ks.scores + ((size_t)row * M + (m < M ? m : M - 1)) * ks.score_stride + (n < len ? n : 0));
  });
  float* w = (shared ? a.weight_shared : a.weight) + row * ks.n;
  float x[KP];
#pragma unroll
  for (int e = 0; e < KP; ++e) x[e] = w[n + e < len ? n + e : len - 1];
  {  // 256 / MQ threads join a query's shares
    constexpr int G = 256 / MQ;
    const int m = threadIdx.x / G, g = threadIdx.x % G;
    const int64_t query = query_at(shared, row, m < M ? m : M - 1, per, a.heads);
    float top = kLow, l = 0.0f;
#pragma unroll 4
    for (int i = g; i < p.splits; i += G) {
      const float2 y = reinterpret_cast<const float2*>(p.ml)[(size_t)i * p.queries + query];
      const float t = __builtin_fmaxf(top, y.x);
      l = l * __builtin_amdgcn_exp2f((top - t) * c) + y.y * __builtin_amdgcn_exp2f((y.x - t) * c);
      top = t;
    }
#pragma unroll
    for (int off = G / 2; off; off >>= 1) {
      const float m2 = __shfl_xor(top, off, 64), l2 = __shfl_xor(l, off, 64), t = __builtin_fmaxf(top, m2);
      l = l * __builtin_amdgcn_exp2f((top - t) * c) + l2 * __builtin_amdgcn_exp2f((m2 - t) * c);
      top = t;
    }
    if (g == 0) parts[m] = float2{top, log2_of(m < M ? l : 0.0f)};
  }
  __syncthreads();
  float sum[KP] = {};
  int t = 0;  // m % T
  static_for<MQ / 4>([&](auto four) __attribute__((always_inline)) {
    constexpr int q = decltype(four)::value * 4;
    if (q >= M) return;
#pragma unroll
    for (int m = q; m < q + 4; ++m) {
      const float2 part = parts[m];
      const int see = m < M ? shared ? len : seen(len, T, t) : 0;
      t = t + 1 == T ? 0 : t + 1;
#pragma unroll
      for (int e = 0; e < KP; ++e) sum[e] += n + e < see ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][e] - part.x, c, -part.y)) : 0.0f;
    }
  });
#pragma unroll
  for (int e = 0; e < KP; ++e)
    if (n + e < len) w[n + e] = x[e] + sum[e];
}

// Blocks below `query_blocks` join outputs, those behind them keep the account.
template <int D, bool F16, int QB, int MQ, int KP>
__global__ __launch_bounds__(256) void attend_finish_kernel(AttendArgs a, Plan p, int query_blocks, int shared_blocks) {
  const int b = (int)blockIdx.x - query_blocks;
  if (b < 0) return join_outputs<D, F16, QB>(a, p, blockIdx.x);
  if constexpr (MQ > 0) {
    const bool shared = b < shared_blocks;
    account_kept<D, MQ, KP>(a, p, shared ? p.shared : p.own, shared, shared ? b : b - shared_blocks);
  }
}

// A row of few keys and its queries from beginning to end, in one launch: four waves have a quarter of the keys each and are joined in LDS, and the logits,
// for the account, come out of the compute unit's own cache.  A chain of waits: 4 rows of up to 512 keys 9.1 us, of 256 6.9.
template <int D, bool F16>
__global__ __launch_bounds__(64 * kMerge) void attend_row_kernel(AttendArgs a, Plan p) {
  using P = Part<D, F16, 1, 1, kMerge>;
  __shared__ u32x4 lds[kMerge * P::STAGES * P::STAGE];
  const int64_t row = blockIdx.x;
  const int M = (int)p.own.m;
  __shared__ Joined fin[16];
  P::template run<true>(a, p, p.own, false, row, 0, 0, lds, fin);
  if (a.weight == nullptr) return;
  // the account, four keys a thread, from the logits that the block has kept
  const int T = (int)a.T, len = row_len(a.lens, row, a.N);
  constexpr float c = kScale<D>;
  float* w = a.weight + row * a.N;
  const float* scores = p.own.scores + (size_t)row * M * p.own.score_stride;
  for (int n = threadIdx.x * 4; n < len; n += 64 * kMerge * 4) {
    f32x4 s[16];
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = w[n + e < len ? n + e : len - 1];
    static_for<4>([&](auto quarter) __attribute__((always_inline)) {
      constexpr int q = decltype(quarter)::value * 4;
      if (q >= M) return;
#pragma unroll
      for (int m = q; m < q + 4; ++m) s[m] = *reinterpret_cast<const f32x4*>(scores + (size_t)(m < M ? m : M - 1) * p.own.score_stride + n);
    });
    float sum[4] = {};
    int t = 0;  // m % T
    static_for<4>([&](auto quarter) __attribute__((always_inline)) {
      constexpr int q = decltype(quarter)::value * 4;
      if (q >= M) return;
#pragma unroll
      for (int m = q; m < q + 4; ++m) {
        const float2 part = {fin[m].ref, fin[m].log2};
        const int see = m < M ? seen(len, T, t) : 0;
        t = t + 1 == T ? 0 : t + 1;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += n + e < see ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][e] - part.x, c, -part.y)) : 0.0f;
      }
    });
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < len) w[n + e] = x[e] + sum[e];
  }
}

// The account where the logits were not kept: a block takes 256 keys of a row, 64 in each wave's registers, and walks the queries that see
// them, or one of `parts` parts of those, 64 at a time, through LDS.  S: a lane has the logits of its key (column) with queries 4 quad + r, so
// that a key's sum stays in the lane until the end.  The products of 16 queries are spread between the exponentials of the 16 before: one
// after the other, matrix and vector instructions of a SIMD's waves take turns.  Sums of parts are added up by attend_add_kernel.
// 2048 queries on 10 343 keys of 128 for 8 heads, 4.3e10 flop and 1.7e8 exponentials, take 63 us, 256 on 32 768 31, with the vector unit busy for 53 % of
// the time and the matrix unit for 34.  Three blocks per compute unit, 1 to 8 parts, and 32 x 32 products with the exponentials spread from step to step
// took as long (the last at a clock of 2.03 GHz where this has 2.2).
template <int D, bool F16>
__global__ __launch_bounds__(256, 2) void attend_account_kernel(AttendArgs a, Keys ks, bool shared, const float* __restrict__ lse,
                                                                const float2* __restrict__ lse_parts, int parts, float* __restrict__ part_sums) {
  using E = Elem<F16>;
  constexpr int CPR = D / 8, KK = D / 32, QS = 64, STAGE = QS * CPR + QS / 4, LOADS = QS * CPR / 256;  // queries, 16-byte units and a wave's loads of a step
  __shared__ u32x4 lds[3 * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
  const int per = (int)(a.group * a.T), T = (int)a.T, M = (int)ks.m, blocks = (int)((ks.n + 255) / 256);
  // a row's last keys first: those that only some queries see take longest
  const int rows = (int)ks.rows, part = blockIdx.x % parts, b0 = (blocks - 1 - (int)(blockIdx.x / parts / rows)) * 256, n0 = b0 + wave * 64;
  const int64_t row = blockIdx.x / parts % rows;
  const float inv_T = 1.0f / (float)T;
  const int len = row_len(shared ? a.shared_lens : a.lens, row, ks.n);
  if (b0 >= len) return;
  const int all = (M + QS - 1) / QS, first = (int)((int64_t)all * part / parts), steps = (int)((int64_t)all * (part + 1) / parts) - first;  // (parts <= all)
  constexpr float c = kScale<D>;
  typedef const __attribute__((address_space(1))) void* gptr_t;
  typedef __attribute__((address_space(3))) void* lptr_t;
  // This lane's pieces of a step: query r of it, whose row in q moves on by QS queries: a whole number of sequences and `turn` queries of the next.
  const int heads = shared ? (int)a.heads : 1, each = shared ? per : M;
  const uint8_t* qb = (const uint8_t*)a.q + (size_t)row * each * (D * 2);
  uint32_t at[LOADS];
  int of[LOADS];  // which of its sequence's queries
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = (i * 4 + wave) * (64 / CPR) + lane / CPR, m = first * QS + r < M ? first * QS + r : M - 1;
    of[i] = m % each;
    at[i] = (uint32_t)(((m / each) * heads * each + of[i]) * (D * 2) + ((lane % CPR) ^ swizzle<D>(r)) * 16);
  }
  const int turn = QS % each, on = (QS / each * heads * each + turn) * (D * 2), wrap = (heads - 1) * each * (D * 2);
  int fetched = first;
  auto fetch = [&](int stage) __attribute__((always_inline)) {  // the next step
    u32x4* st = lds + stage * STAGE;
    const int left = M - 1 - fetched * QS;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      __builtin_amdgcn_global_load_lds((gptr_t)(qb + at[i]), (lptr_t)(st + (i * 4 + wave) * 64), 16, 0, 0);
      const int r = (i * 4 + wave) * (64 / CPR) + lane / CPR;
      if (r + QS <= left) {  // (a query behind the last: the same row again, which counts nowhere)
        of[i] += turn;
        const bool over = of[i] >= each;
        of[i] -= over ? each : 0;
        at[i] += (uint32_t)(on + (over ? wrap : 0));
      }
    }
    // every wave, so that all have as many loads under way
    const int m = fetched * QS + lane < M ? fetched * QS + lane : M - 1;
    __builtin_amdgcn_global_load_lds((gptr_t)(lse + row * M + m), (lptr_t)(st + QS * CPR), 4, 0, 0);
    ++fetched;
  };
  u32x4 bk[4][KK];
#pragma unroll
  for (int kt = 0; kt < 4; ++kt) {
    const int n = n0 + kt * 16 + col;
    const uint16_t* k = (const uint16_t*)(shared ? a.k_shared : a.k) + ((size_t)row * ks.n + (n < len ? n : len - 1)) * D + quad * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) bk[kt][kk] = *reinterpret_cast<const u32x4*>(k + kk * 32);
  }
  struct Logits {
    f32x4 s[4], ref;
  };
  float sum[4] = {};
  auto read = [&](u32x4 (&fq)[KK], const u32x4* st, int u) __attribute__((always_inline)) {
    const int r = u * 16 + col;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) fq[kk] = st[r * CPR + ((kk * 4 + quad) ^ swizzle<D>(r))];
  };
  auto products = [&](const u32x4 (&fq)[KK], Logits& x) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) x.s[kt] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) x.s[kt] = E::mfma(fq[kk], bk[kt][kk], x.s[kt]);
  };
  auto add = [&](const Logits& x) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[kt] += __builtin_amdgcn_exp2f(__builtin_fmaf(x.s[kt][e], c, -x.ref[e]));
  };
  // waits until this wave's part of step t has landed
  auto landed = [&](int t) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0F70 | (LOADS + 1));  // (on every path: it is where the compiler knows of the keys)
    if (t + 1 >= steps) __builtin_amdgcn_s_waitcnt(0x0F70);
    asm volatile("" ::: "memory");
  };
  fetch(0);
  if (steps > 1) fetch(1);
  landed(0);  // and with it the resident keys: where the compiler does not know, it waits for all loads in front of every step's products
  int stage = 0;
  for (int t = 0; t < steps; ++t) {
    landed(t);
    const u32x4* st = lds + stage * STAGE;
    const float some = __builtin_fabsf(reinterpret_cast<const float*>(st + QS * CPR)[lane]);  // (this wave's own load)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();  // everyone's has, and everyone has read step t - 1, whose place takes step t + 2
    asm volatile("" ::: "memory");
    if (t + 2 < steps) fetch(stage == 0 ? 2 : stage - 1);
    const bool far = __builtin_amdgcn_ballot_w64(some > kFar && some != -kNegInf) != 0;  // some of the step's queries have logits far from 0
    const f32x4* refs = reinterpret_cast<const f32x4*>(st + QS * CPR) + quad;
    // whether all the step's queries see all of this wave's keys
    const int q0 = (first + t) * QS, q1 = q0 + QS - 1;
    const int t0 = shared ? 0 : q0 % T;
    const int least = shared ? len : seen(len, T, t0 + QS <= T ? t0 : 0);
    auto work = [&](auto cut_c) __attribute__((always_inline)) {
      constexpr bool cut = decltype(cut_c)::value;
      u32x4 fq[2][KK];
      Logits x[2];
      read(fq[0], st, 0);
      read(fq[1], st, 1);
      x[0].ref = refs[0];
      products(fq[0], x[0]);
      static_for<4>([&](auto uc) __attribute__((always_inline)) {
        constexpr int u = decltype(uc)::value, cur = u & 1, nxt = cur ^ 1;
        if constexpr (u < 3) {
          x[nxt].ref = refs[(u + 1) * 4];
          if constexpr (u < 2) read(fq[cur], st, u + 2);
          if constexpr (!cut) __builtin_amdgcn_sched_barrier(0);
          products(fq[nxt], x[nxt]);
        }
        if constexpr (cut) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int m = q0 + u * 16 + quad * 4 + e, see = m >= M ? 0 : shared ? len : seen(len, T, remainder_of(m, T, inv_T));
            float2 part = {0.0f, 0.0f};
            if (far) part = lse_parts[row * M + (m < M ? m : M - 1)];
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
              const float y = __builtin_amdgcn_exp2f(far ? __builtin_fmaf(x[cur].s[kt][e] - part.x, c, -part.y) : __builtin_fmaf(x[cur].s[kt][e], c, -x[cur].ref[e]));
              sum[kt] += n0 + kt * 16 + col < see ? y : 0.0f;
            }
          }
        } else {
          add(x[cur]);
          if constexpr (u < 3) {
#pragma unroll
            for (int i = 0; i < 4 * KK; ++i) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);              // one product
              __builtin_amdgcn_sched_group_barrier(0x002, 48 / (4 * KK), 0);  // its share of 16 fma, 16 exponentials and 16 additions
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      });
    };
    const int any = shared ? len : seen(len, T, t0 + QS <= T ? t0 + QS - 1 : T - 1);  // keys that some of the step's queries see
    if (__builtin_expect(q1 < M && n0 + 64 <= least && !far, 1)) work(std::integral_constant<bool, false>{});
    else if (n0 < any) work(std::integral_constant<bool, true>{});
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    stage = stage == 2 ? 0 : stage + 1;
  }
  float* w = (shared ? a.weight_shared : a.weight) + row * ks.n;
  float* mine = part_sums + ((size_t)part * ks.rows + row) * ks.n;
#pragma unroll
  for (int kt = 0; kt < 4; ++kt) {
    const int n = n0 + kt * 16 + col;
    const float x = quads_sum(sum[kt]);
    if (quad == 0 && n < len) {
      if (parts > 1) mine[n] = x;
      else w[n] += x;
    }
  }
}

__global__ __launch_bounds__(256) void attend_add_kernel(float* __restrict__ weight, const float* __restrict__ part_sums, const int32_t* __restrict__ lens,
                                                         int64_t rows, int64_t n, int parts) {
  const int blocks = (int)((n + 255) / 256);
  const int64_t row = blockIdx.x / blocks;
  const int i = blockIdx.x % blocks * 256 + threadIdx.x;
  if (i >= row_len(lens, row, n)) return;
  float x = 0.0f;
  for (int p = 0; p < parts; ++p) x += part_sums[((size_t)p * rows + row) * n + i];
  weight[row * n + i] += x;
}

// Parts of the queries in attend_account_kernel: where a row's keys are few blocks, the last turn on the compute units is mostly empty.
// Though adding up the parts is one more launch: 256 queries on 8 rows of 1000 keys in two parts 39.7 us a call, in one 44.1; 2048 on one row of 4000 in four 57.9 and 111.
// (No more blocks than 16 turns have: behind those an empty one is little.  It also bounds the sums that the parts leave.)
constexpr int64_t kPartBlocks = 4096;
int account_parts(const Keys& k) {
  const int64_t blocks = k.rows * ((k.n + 255) / 256), steps = (k.m + 63) / 64;
  int best = 1;
  double least = 1e30;
  for (int p = 1; p <= 8 && p <= steps && (p == 1 || blocks * p <= kPartBlocks); ++p) {
    const double turns = (double)((blocks * p + 255) / 256) * (double)((steps + p - 1) / p) + 1.0 * p;
    if (turns < least) {
      least = turns;
      best = p;
    }
  }
  return best;
}

constexpr int64_t kMergedKeys = 512;  // of a share (64 rows of up to 4001 keys, 20 queries: 22.1 us, 256 keys 28.7; 8 of 9830, 32 queries, with 64 of 512: 24.1 and 31.6)
constexpr int64_t kMostSplits = 512;
// One launch instead of two (which takes the host 3.5 us less of about 17) where a block per row is not much slower on the device: us, one and two
// launches, 4 query heads: 4 rows of 256 keys 6.9 and 8.1, 4 of up to 512 9.1 and 8.5 (in a graph, where the host does not count, two would be faster there), 256 of
// 512 15.7 and 17.5; but 8 of 1024 13.1 and 8.5, and with more rows than compute units (a block has most of one's LDS) 1024 of 128 28.3 and 18.8.
constexpr int64_t kShortKeys = 512, kShortRows = 256;

Keys keys_of(int64_t rows, int64_t n, int64_t m, int merge, int64_t more, bool account) {
  Keys k = {};
  k.rows = rows;
  k.n = n;
  k.m = m;
  k.merge = 1;
  if (n == 0) {
    k.tiles = 1;
    return k;
  }
  k.ct = m <= 16 ? 1 : 2;
  k.waves = m <= 32 ? 1 : m <= 64 ? 2 : m <= 128 ? 4 : 8;
  if (k.waves == 1) k.merge = merge;
  const int64_t tile = 16 * k.ct * k.waves, jobs = rows * ((m + tile - 1) / tile);
  k.tiles = (int)((m + tile - 1) / tile);
  int64_t splits, least;
  if (k.waves > 1) {
    splits = (2048 / k.waves + jobs - 1) / jobs;
    least = 256;
  } else if (k.merge > 1) {
    splits = more == 0 ? 1 : (n + kMergedKeys - 1) / kMergedKeys * more;
    least = 256;
  } else {
    least = jobs * n <= 64 * 256 ? 64 : jobs * n <= 128 * 1024 ? 128 : 384;
    splits = kMostSplits;
  }
  const int64_t most = (n + least - 1) / least;
  splits = splits < most ? splits : most;
  splits = splits < kMostSplits ? splits : kMostSplits;
  const int64_t step = kTile * k.merge;
  k.chunk = (int)(((n + splits - 1) / splits + step - 1) / step * step);
  k.splits = (int)((n + k.chunk - 1) / k.chunk);
  k.blocks = (int)((rows * k.splits + kXcds - 1) / kXcds * kXcds * k.tiles);
  k.parts = account && m > kKeptQueries ? account_parts(k) : 1;
  k.score_stride = account && m <= kKeptQueries ? (n + kTile - 1) / kTile * kTile : 0;
  return k;
}

Plan plan_of(const AttendArgs& a, uint8_t* scratch) {
  const int64_t per = a.group * a.T, rows = a.batch * a.heads;
  Plan p = {};
  p.queries = rows * per;
  const bool short_rows = a.P == 0 && per <= 16 && a.N <= kShortKeys && rows <= kShortRows;
  const int64_t m_shared = a.P > 0 ? a.batch * per : 0, m_own = a.N > 0 ? per : 0;
  // waves are joined in LDS where they leave outputs of more than 16 queries: those would be a quarter of what is read
  const int merge = short_rows || (m_shared > 16 && m_shared <= 32) || (m_own > 16 && m_own <= 32) ? kMerge : 1;
  const int64_t blocks = (m_shared <= 32 ? a.heads * ((a.P + kMergedKeys - 1) / kMergedKeys) : 0) + (m_own <= 32 ? rows * ((a.N + kMergedKeys - 1) / kMergedKeys) : 0);
  const int64_t more = short_rows ? 0 : blocks > 0 && blocks < 256 ? 256 / blocks : 1;
  p.one_launch = short_rows;
  p.shared = keys_of(a.heads, a.P, m_shared, merge, more, a.weight_shared != nullptr);
  p.own = keys_of(rows, a.N, m_own, merge, more, a.weight != nullptr);
  p.own.first_split = p.shared.splits;
  p.splits = p.shared.splits + p.own.splits;
  size_t at = 0;
  auto take = [&](size_t floats) {
    float* r = (float*)(scratch + at);
    at += (floats * 4 + 255) / 256 * 256;
    return r;
  };
  p.ml = take((size_t)p.splits * p.queries * 2);
  p.o = take((size_t)p.splits * p.queries * a.D);
  p.lse = take((size_t)p.queries * 2);
  p.parts = (float2*)take((size_t)p.queries * 4);
  const size_t sums_shared = p.shared.parts > 1 ? (size_t)(p.shared.parts * p.shared.rows * p.shared.n) : 0;
  const size_t sums_own = p.own.parts > 1 ? (size_t)(p.own.parts * p.own.rows * p.own.n) : 0;
  p.part_sums = take(sums_shared > sums_own ? sums_shared : sums_own);
  if (p.shared.score_stride) p.shared.scores = take((size_t)(p.shared.rows * p.shared.m * p.shared.score_stride));
  if (p.own.score_stride) p.own.scores = take((size_t)(p.own.rows * p.own.m * p.own.score_stride));
  return p;
}

template <int D, bool F16>
hipError_t launch_attend_of(const AttendArgs& a, void* scratch, hipStream_t stream) {
  const Plan p = plan_of(a, (uint8_t*)scratch);
  hipError_t e = hipSuccess;
  if (p.one_launch) {
    attend_row_kernel<D, F16><<<(unsigned)p.own.rows, 64 * kMerge, 0, stream>>>(a, p);
    return hipGetLastError();
  }
  auto many = [&](const Keys& k, bool shared) {
    if (e != hipSuccess || k.waves <= 1) return;
    if (k.waves == 2) attend_block_kernel<D, F16, 2><<<(unsigned)k.blocks, 128, 0, stream>>>(a, p, shared);
    else if (k.waves == 4) attend_block_kernel<D, F16, 4><<<(unsigned)k.blocks, 256, 0, stream>>>(a, p, shared);
    else attend_block_kernel<D, F16, 8><<<(unsigned)k.blocks, 512, 0, stream>>>(a, p, shared);
    e = hipGetLastError();
  };
  many(p.shared, true);
  many(p.own, false);
  Plan few = p;
  if (p.shared.waves > 1) few.shared.blocks = 0;
  if (p.own.waves > 1) few.own.blocks = 0;
  const unsigned blocks = (unsigned)(few.shared.blocks + few.own.blocks);
  if (e == hipSuccess && blocks > 0) {
    if (p.shared.merge > 1 || p.own.merge > 1) attend_wave_kernel<D, F16, 2, kMerge><<<blocks, 64 * kMerge, 0, stream>>>(a, few);
    else attend_wave_kernel<D, F16, 1, 1><<<blocks, 64, 0, stream>>>(a, few);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  const int64_t kept_shared = p.shared.scores ? p.shared.m : 0, kept_own = p.own.scores ? p.own.m : 0, kept = kept_shared > kept_own ? kept_shared : kept_own;
  const int64_t kept_keys = (p.shared.scores ? p.shared.rows * p.shared.n : 0) + (p.own.scores ? p.own.rows * p.own.n : 0);
  auto finish = [&](auto qb, auto mq, auto kp) {
    constexpr int QB = decltype(qb)::value, MQ = decltype(mq)::value, KP = decltype(kp)::value;
    const int query_blocks = (int)((p.queries + QB - 1) / QB);
    auto key_blocks = [&](const Keys& k) { return k.scores ? k.rows * ((k.n + 256 * KP - 1) / (256 * KP)) : 0; };
    const int64_t shared_blocks = key_blocks(p.shared), own_blocks = key_blocks(p.own);
    attend_finish_kernel<D, F16, QB, MQ, KP><<<(unsigned)(query_blocks + shared_blocks + own_blocks), 256, 0, stream>>>(a, p, query_blocks, (int)shared_blocks);
  };
  auto finish_of = [&](auto qb) {
    // Four keys a thread where most compute units still get a block (us a call, four and one: 2.1e6 keys of 128, 4 queries 130.0 and 135.3; 256 064, 20 queries,
    // of 64 22.1 and 22.6, of 128 34.2 and 34.8; 163 840, 32 queries 41.0 and 40.0, 8 queries 22.0 and 21.7; 111 408, 32 queries 25.2 and 24.2).
    auto with = [&](auto mq) {
      if (kept_keys >= 192 * 1024) finish(qb, mq, std::integral_constant<int, 4>{});
      else finish(qb, mq, std::integral_constant<int, 1>{});
    };
    if (kept == 0) finish(qb, std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
    else if (kept <= 4) with(std::integral_constant<int, 4>{});
    else if (kept <= 8) with(std::integral_constant<int, 8>{});
    else if (kept <= 16) with(std::integral_constant<int, 16>{});
    else with(std::integral_constant<int, 32>{});
  };
  if (p.splits <= 4) finish_of(std::integral_constant<int, 8>{});
  else if (p.splits <= 8) finish_of(std::integral_constant<int, 4>{});
  else finish_of(std::integral_constant<int, 1>{});
  e = hipGetLastError();
  auto account = [&](const Keys& k, bool shared, float* weight, const int32_t* lens) {
    if (e != hipSuccess || weight == nullptr || k.n == 0 || k.scores) return;
    const int64_t blocks = k.rows * ((k.n + 255) / 256), first = shared ? p.queries : 0;
    attend_account_kernel<D, F16><<<(unsigned)(blocks * k.parts), 256, 0, stream>>>(a, k, shared, p.lse + first, p.parts + first, k.parts, p.part_sums);
    e = hipGetLastError();
    if (e == hipSuccess && k.parts > 1) {
      attend_add_kernel<<<(unsigned)blocks, 256, 0, stream>>>(weight, p.part_sums, lens, k.rows, k.n, k.parts);
      e = hipGetLastError();
    }
  };
  account(p.shared, true, a.weight_shared, a.shared_lens);
  account(p.own, false, a.weight, a.lens);
  return e;
}

}  // namespace

// Not what this call's plan takes (fewer rows are split more often, so that would shrink and grow), but what none of no more rows, sequences and
// tokens takes: so one call of the largest size makes room for all.
size_t attend_scratch_bytes(const AttendArgs& a) {
  const int64_t per = a.group * a.T, rows = a.batch * a.heads, queries = rows * per;
  int64_t outputs = 0, scores = 0, sums = 0;
  auto shares = [&](int64_t rows, int64_t n, int64_t m, bool account) {  // bounds of keys_of's choices, each growing in rows, n and m
    if (n == 0) return;
    if (m <= kKeptQueries) {
      const int64_t s = (n + 383) / 384, many = rows * (s < kMostSplits ? s : kMostSplits), few = rows + 1024;  // (shares of 64 or 128 keys: of up to 2^17 in all)
      outputs += m * (many > few ? many : few);
      scores += account ? rows * m * ((n + kTile - 1) / kTile * kTile) + 64 : 0;
    } else {
      const int64_t tile = m <= 64 ? 64 : m <= 128 ? 128 : 256;
      outputs += rows * ((m + tile - 1) / tile * tile) + 2048 * 32;
      sums = account ? kPartBlocks * 256 : sums;
    }
  };
  shares(rows, a.N, per, a.weight != nullptr);
  shares(a.heads, a.P, a.batch * per, a.weight_shared != nullptr);
  if (a.batch * per > kKeptQueries) shares(a.heads, a.P, kKeptQueries, a.weight_shared != nullptr);  // a smaller batch
  return (size_t)(outputs * (a.D + 2) + scores + sums + queries * 6) * 4 + 7 * 256;
}

hipError_t launch_attend(const AttendArgs& a, void* scratch, hipStream_t stream) {
  if (a.D == 64) return a.f16 ? launch_attend_of<64, true>(a, scratch, stream) : launch_attend_of<64, false>(a, scratch, stream);
  return a.f16 ? launch_attend_of<128, true>(a, scratch, stream) : launch_attend_of<128, false>(a, scratch, stream);
}

}  // namespace pkv
