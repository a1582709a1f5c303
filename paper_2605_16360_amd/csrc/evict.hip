// Eviction from the cache by the account of attention weight that attend.hip keeps.  A row of n tokens with a budget of b < n keeps its `recent`
// last ones and, of the n - recent candidates in front of them, the keep = b - recent heaviest.  Rotary positions are in the keys, so
// where a kept token lies does not matter to attention: a candidate that is kept in one of the first `keep` slots stays there,
// those kept further back move, in order, into the slots that were given up, in order, and only the recent tokens are moved up as a
// block.  (In order throughout, nearly all of the row would move: 256 of 4352 tokens evicted, 512 recent, about 740 of 4096 tokens move so.)
#include "common.hpp"
#include "kernels.hpp"

namespace pkv {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kBins = 2048, kCopies = 8;  // of a digit's histogram: accounts share their high digits, and lanes that meet in a word take turns
constexpr int kFew = 256;                 // keys that are ranked by comparing all with all
// Words: moves, candidates, keep, recent tokens to move up (0: nothing to do); then, in order, the places that change: the slots given up, and
// behind those, as many, the places of the tokens that take them.
constexpr int kPlanHead = 4;

// Larger key <=> heavier.  NaN maps to 0 (below every number), -0.0 onto +0.0.
__device__ __forceinline__ uint32_t weight_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);
  const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return f == f ? k : 0u;
}

// One workgroup per row: the keep-th heaviest candidate by a radix select of 11, 11 and 10 bits, which ends where few keys are left in a bin, the list of
// places that change, then the moves of the account and the positions themselves.  A wave has consecutive candidates, 64 at a time, so that ranks need one exchange
// between waves.  Bound by the chain of its phases, or, for long rows, by what one compute unit can do with a row (30 001 tokens: 44 us, of
// which the digits take 9, the places 9 and the account's moves 6 at the median length); 8 rows of 1088 9.3 us in the trace, 256 of 4352 12.9.
// STEPS > 0: a lane keeps its candidates' keys, STEPS of them, in registers; 0: they are read again for each use.
template <int STEPS>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(float* __restrict__ weight, int32_t* __restrict__ positions,
                                                                   int32_t* __restrict__ lens, const int32_t* __restrict__ budgets, int64_t N,
                                                                   int budget, int recent, int32_t* __restrict__ plans, int64_t plan_words) {
  __shared__ u32x4 hist4[kBins * kCopies / 4];
  __shared__ int s_wave[kSelWaves];
  __shared__ u32x4 few4[kFew / 4];
  __shared__ uint32_t few_rank[kFew], s_few, s_prefix, s_left, s_equal;
  uint32_t *hist = reinterpret_cast<uint32_t*>(hist4), *few = reinterpret_cast<uint32_t*>(few4);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = blockIdx.x;
  int32_t* plan = plans + r * plan_words;
  int32_t* list = plan + kPlanHead;
  float* w = weight + r * N;
  uint32_t keys[STEPS > 0 ? STEPS : 1];
  auto ask = [&](int end) __attribute__((always_inline)) {  // (no branch around a load; what lies behind the last candidate counts nowhere)
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
      const int i = wave * (STEPS * 64) + lane + j * 64;
      keys[j] = __float_as_uint(w[i < end ? i : end - 1]);
    }
  };
  constexpr bool kAtOnce = STEPS > 0 && STEPS <= 5;  // before the row's length is known: few steps are one wait anyway
  if constexpr (kAtOnce) ask((int)N);
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBins * kCopies / 4 / kSelThreads; ++i) hist4[i * kSelThreads + tid] = u32x4{0, 0, 0, 0};
  };
  clear();
  if (tid < kFew) few_rank[tid] = 0;
  if (tid == 0) s_few = 0;
  int n = lens[r], b = budget;
  n = n < 0 ? 0 : n < N ? n : (int)N;
  if (budgets != nullptr) {
    b = budgets[r];
    b = b < recent ? recent : b < N ? b : (int)N;
  }
  if (n <= b) {
    if (tid < kPlanHead) plan[tid] = 0;
    return;
  }
  const int cand = n - recent, keep = b - recent;
  int moves = 0;
  if (keep > 0) {
    const int steps = STEPS > 0 ? STEPS : (cand + kSelThreads - 1) / kSelThreads, first = wave * steps * 64 + lane;
    if constexpr (STEPS > 0) {
      if constexpr (!kAtOnce) ask(cand);
#pragma unroll
      for (int j = 0; j < STEPS; ++j) keys[j] = weight_key(__uint_as_float(keys[j]));
    }
    // f(place, key) for this lane's places, in order; a place behind the last candidate has place >= cand
    auto again = [&](auto f) __attribute__((always_inline)) {
      constexpr int U = 8;
#pragma unroll 1
      for (int j0 = 0; j0 < steps; j0 += U) {
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = w[first + (j0 + u) * 64 < cand ? first + (j0 + u) * 64 : cand - 1];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (j0 + u < steps) f(first + (j0 + u) * 64, weight_key(x[u]));
      }
    };
    auto each = [&](auto f) __attribute__((always_inline)) {
      if constexpr (STEPS > 0) {
#pragma unroll
        for (int j = 0; j < STEPS; ++j) f(first + j * 64, keys[j]);
      } else {
        again(f);
      }
    };
    uint32_t prefix = 0, left = (uint32_t)keep, equal = kFew + 1;  // of the key's bits known so far, how many keys have them
    int known = 32;                                                // and how many are not
    static_for<3>([&](auto digit) __attribute__((always_inline)) {
      constexpr int shift = decltype(digit)::value == 0 ? 21 : decltype(digit)::value == 1 ? 10 : 0, bits = decltype(digit)::value == 2 ? 10 : 11;
      if (equal <= kFew) return;
      if constexpr (shift != 21) clear();
      __syncthreads();
      each([&](int i, uint32_t k) __attribute__((always_inline)) {
        if (i < cand && (shift == 21 || (k >> (shift + bits < 32 ? shift + bits : 31)) == (prefix >> (shift + bits < 32 ? shift + bits : 31))))
          atomicAdd(&hist[((k >> shift) & ((1u << bits) - 1u)) * kCopies + (lane & (kCopies - 1))], 1u);
      });
      __syncthreads();
      // thread t has the bins 2047 - 2 t and 2046 - 2 t: how many keys lie above them, from the highest downwards
      uint32_t h[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const u32x4 x = hist4[(kBins - 1 - 2 * tid - e) * 2], y = hist4[(kBins - 1 - 2 * tid - e) * 2 + 1];
        h[e] = x[0] + x[1] + x[2] + x[3] + y[0] + y[1] + y[2] + y[3];
      }
      uint32_t upto = h[0] + h[1];
      for (int off = 1; off < 64; off *= 2) {
        const uint32_t o = __shfl_up(upto, off, 64);
        upto += lane >= off ? o : 0u;
      }
      if (lane == 63) s_wave[wave] = (int)upto;
      __syncthreads();
      for (int x = 0; x < kSelWaves; ++x) upto += x < wave ? (uint32_t)s_wave[x] : 0u;
      uint32_t above = upto - h[0] - h[1];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (above < left && above + h[e] >= left) {
          s_prefix = prefix | (uint32_t)(kBins - 1 - 2 * tid - e) << shift;
          s_left = left - above;
          s_equal = h[e];
        }
        above += h[e];
      }
      __syncthreads();
      prefix = s_prefix;
      left = s_left;
      equal = s_equal;
      known = shift;
    });
    if (known > 0) {  // the few keys that agree so far: thread t compares the (t % 256)-th with a quarter of them
      each([&](int i, uint32_t k) __attribute__((always_inline)) {
        if (i < cand && (k ^ prefix) >> known == 0) few[atomicAdd(&s_few, 1u) % kFew] = k;  // (no more than `equal`)
      });
      __syncthreads();
      const uint32_t x = (uint32_t)tid % kFew, mine = few[x], c = equal;
      if (x < c) {
        uint32_t rank = 0;  // greater ones, and equal ones 2^16 each
        for (uint32_t i = (uint32_t)tid / kFew * 4; i < c; i += kSelThreads / kFew * 4) {
          const u32x4 y = few4[i / 4];
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e) rank += i + e < c ? y[e] > mine ? 1u : y[e] == mine ? 1u << 16 : 0u : 0u;
        }
        atomicAdd(&few_rank[x], rank);
      }
      __syncthreads();
      if ((uint32_t)tid < c) {
        const uint32_t greater = few_rank[tid] & 0xffffu, same = few_rank[tid] >> 16;
        if (greater < left && greater + same >= left) {  // (of equal keys, all write the same)
          s_prefix = mine;
          s_left = left - greater;
          s_equal = same;
        }
      }
      __syncthreads();
      prefix = s_prefix;
      left = s_left;
      equal = s_equal;
    }
    // kept: above the key, or equal to it and among the first `left` of those.  A place changes that is kept behind the first `keep` ones, or
    // given up among them; walk(f): f(place, kept) for this lane's places in order
    auto places = [&](auto walk) __attribute__((always_inline)) {
      int count = 0;
      walk([&](int i, bool kept) __attribute__((always_inline)) { count += __popcll(__builtin_amdgcn_ballot_w64(kept != (i < keep) && i < cand)); });
      if (lane == 0) s_wave[wave] = count;
      __syncthreads();
      int before = 0;
      for (int x = 0; x < kSelWaves; ++x) {
        before += x < wave ? s_wave[x] : 0;
        moves += s_wave[x];
      }
      moves /= 2;
      walk([&](int i, bool kept) __attribute__((always_inline)) {
        const bool changes = kept != (i < keep) && i < cand;
        const uint64_t all = __builtin_amdgcn_ballot_w64(changes);
        if (changes) list[before + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0))] = i;
        before += __popcll(all);
      });
    };
    if (equal == left) {  // all of those that equal the key
      places([&](auto f) __attribute__((always_inline)) {
        each([&](int i, uint32_t k) __attribute__((always_inline)) { f(i, k >= prefix); });
      });
    } else {  // some: by their ranks (masks of a lane's many places take more code than the row's second reading takes time)
      auto stream = [&](auto f) __attribute__((always_inline)) {
        if constexpr (STEPS > 10) again(f);
        else each(f);
      };
      int count = 0;
      stream([&](int i, uint32_t k) __attribute__((always_inline)) { count += __popcll(__builtin_amdgcn_ballot_w64(i < cand && k == prefix)); });
      if (lane == 0) s_wave[wave] = count;
      __syncthreads();
      int rank0 = 0;
      for (int x = 0; x < kSelWaves; ++x) rank0 += x < wave ? s_wave[x] : 0;
      __syncthreads();
      places([&](auto f) __attribute__((always_inline)) {
        int rank = rank0;
        stream([&](int i, uint32_t k) __attribute__((always_inline)) {
          const uint64_t eq = __builtin_amdgcn_ballot_w64(i < cand && k == prefix);
          const int mine = rank + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(eq >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)eq, 0));
          rank += __popcll(eq);
          f(i, k > prefix || (k == prefix && mine < (int)left));
        });
      });
    }
    __syncthreads();
  }
  if (tid == 0) {
    plan[0] = moves;
    plan[1] = cand;
    plan[2] = keep;
    plan[3] = recent;
  }
  int32_t* pos = positions == nullptr ? nullptr : positions + r * N;
  for (int j0 = tid; j0 < moves; j0 += 4 * kSelThreads) {  // (sources lie behind the first `keep` places, targets among them)
    int y[4], z[4];
    float x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int j = j0 + u * kSelThreads < moves ? j0 + u * kSelThreads : j0;  // (again the first: the same value once more)
      y[u] = list[j];
      z[u] = list[moves + j];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = w[z[u]];
    if (pos != nullptr) {
#pragma unroll
      for (int u = 0; u < 4; ++u) z[u] = pos[z[u]];
#pragma unroll
      for (int u = 0; u < 4; ++u) pos[y[u]] = z[u];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) w[y[u]] = x[u];
  }
  __syncthreads();
  // a recent token never moves back, so what a step stores is behind nothing that a later one reads
  for (int j0 = 0; j0 < recent; j0 += kSelThreads) {
    const int j = j0 + tid;
    float x = 0.0f;
    int32_t p = 0;
    if (j < recent) {
      x = w[cand + j];
      if (pos != nullptr) p = pos[cand + j];
    }
    asm volatile("" : "+v"(x), "+v"(p));  // arrived, not only asked for
    __syncthreads();
    if (j < recent) {
      w[keep + j] = x;
      if (pos != nullptr) pos[keep + j] = p;
    }
  }
  if (tid == 0) lens[r] = b;
}

// The planned moves of K and V.  K and V, and the slices of a token, are independent, so each gets workgroups of its own.  A candidate's new
// place is nothing that is read any more, but the recent tokens' new places, keep .. b - 1, are the old places of the first moves.  Those
// and the recent tokens are one list, which one workgroup walks in order, a step's loads under way while the one before is stored:
// what a step stores lies on nothing that a later step reads (a recent token's new place is the old one of an earlier entry), so each
// waits only for its own loads, in all threads, before it stores.  Moves from behind the budget are anybody's: blockIdx.z > 0, free_tokens each.
// Bound by HBM: 256 rows of 4352 tokens to 4096, 512 recent, 194 MB in 36 us (5.3 TB/s; a large copy reaches 5.2), 112 of up to 30 001 to 9999 365 MB
// in 83 us (4.4).
// grid (rows, 2 * slices, 1 + blocks for the free moves), 256 threads; cpr = 16-byte pieces per token, cps those of a slice.
constexpr int kPer = 4;
__global__ __launch_bounds__(256) void evict_move_kernel(u32x4* __restrict__ k, u32x4* __restrict__ v, const int32_t* __restrict__ plans,
                                                         int64_t plan_words, int64_t N, int cpr, int cps, int free_tokens) {
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, step = 256 * kPer / cps;  // tokens at a time
  const int32_t* plan = plans + r * plan_words;
  const int moves = plan[0], cand = plan[1], keep = plan[2], recent = plan[3], b = keep + recent;
  const int32_t *to = plan + kPlanHead, *from = to + plan[0];
  int bound = 0;  // moves from in front of the budget's end: those come first
  for (int lo = 0, hi = moves;;) {
    if (lo >= hi) {
      bound = lo;
      break;
    }
    const int mid = (lo + hi) / 2;
    if (from[mid] < b) lo = mid + 1;
    else hi = mid;
  }
  u32x4* base = ((blockIdx.y & 1) ? v : k) + (size_t)r * N * cpr + (blockIdx.y >> 1) * cps;
  const bool free = blockIdx.z > 0;
  const int64_t begin64 = free ? bound + ((int64_t)blockIdx.z - 1) * free_tokens : 0;
  const int64_t end64 = free ? (begin64 + free_tokens < moves ? begin64 + free_tokens : moves) : (int64_t)bound + recent;
  if (begin64 >= end64) return;
  const int begin = (int)begin64, end = (int)end64;
  auto places = [&](int j, int& src, int& dst) __attribute__((always_inline)) {  // of entry j; the free moves have no recent tokens
    const int jm = j < moves ? j : moves > 0 ? moves - 1 : 0;
    const bool move = free || j < bound;
    const int x = from[jm], y = to[jm];
    src = move ? x : cand + j - bound;
    dst = move ? y : keep + j - bound;
  };
  int tok[kPer], ch[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int piece = tid + 256 * u;
    tok[u] = evict_token(piece, step, cps);
    ch[u] = piece % cps;
  }
  auto load = [&](int j0, u32x4 (&x)[kPer], int (&dst)[kPer]) __attribute__((always_inline)) {  // (a piece behind the end reads the last token's and stores nothing)
    int src[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int j = tok[u] < end - j0 ? j0 + tok[u] : end - 1;
      places(j, src[u], dst[u]);
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) x[u] = base[(size_t)src[u] * cpr + ch[u]];
  };
  auto store = [&](int j0, const u32x4 (&x)[kPer], const int (&dst)[kPer]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (tok[u] < end - j0) base[(size_t)dst[u] * cpr + ch[u]] = x[u];
  };
  auto meet = [&](u32x4 (&x)[kPer]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) asm volatile("" : "+v"(x[u]));  // arrived, not only asked for
    __syncthreads();
  };
  u32x4 x0[kPer], x1[kPer];
  int d0[kPer], d1[kPer];
  load(begin, x0, d0);
  for (int j = begin; j < end; j += 2 * step) {  // (two steps by name: moving x1 to x0 would wait for it)
    if (j + step < end) load(j + step, x1, d1);
    meet(x0);
    store(j, x0, d0);
    if (j + step >= end) break;
    if (j + 2 * step < end) load(j + 2 * step, x0, d0);
    meet(x1);
    store(j + step, x1, d1);
  }
}

// No more candidates than half of a row can change places: those that are kept behind the first `keep` slots are as many as the slots given
// up, and both are candidates.
int64_t plan_words_of(int64_t N) { return (kPlanHead + 2 * (N / 2 + 1) + 3) / 4 * 4; }

}  // namespace

size_t evict_scratch_bytes(int64_t rows, int64_t N) { return (size_t)(rows * plan_words_of(N)) * 4; }

hipError_t launch_evict(void* k, void* v, float* weight, int32_t* positions, int32_t* lens, const int32_t* budgets, int64_t rows, int64_t N,
                        int64_t budget, int64_t recent, int64_t row_bytes, void* scratch, hipStream_t stream) {
  const int64_t words = plan_words_of(N), most = N - recent;  // (candidates of a row)
  auto select = [&](auto steps) {
    evict_select_kernel<decltype(steps)::value><<<(unsigned)rows, kSelThreads, 0, stream>>>(weight, positions, lens, budgets, N, (int)budget, (int)recent,
                                                                                          (int32_t*)scratch, words);
  };
  if (most <= 2 * kSelThreads) select(std::integral_constant<int, 2>{});
  else if (most <= 5 * kSelThreads) select(std::integral_constant<int, 5>{});
  else if (most <= 10 * kSelThreads) select(std::integral_constant<int, 10>{});
  else if (most <= 20 * kSelThreads) select(std::integral_constant<int, 20>{});
  else if (most <= 40 * kSelThreads) select(std::integral_constant<int, 40>{});
  else select(std::integral_constant<int, 0>{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int cpr = (int)(row_bytes / 16), slices = cpr % 8 == 0 ? cpr / 8 : 1;
  // free moves of a row: kept candidates from behind the budget, no more than places in front of the recent ones, nor than candidates there
  int64_t free = budgets != nullptr ? N / 2 : budget - recent < N - recent - budget ? budget - recent : N - recent - budget;
  free = free > 0 ? free : 0;
  const int64_t free_tokens = free <= 256 * 4096 ? 256 : (free + 4095) / 4096;
  free = (free + free_tokens - 1) / free_tokens;
  evict_move_kernel<<<dim3((unsigned)rows, (unsigned)(2 * slices), (unsigned)(1 + free)), 256, 0, stream>>>((u32x4*)k, (u32x4*)v, (const int32_t*)scratch,
                                                                                                          words, N, cpr, cpr / slices, (int)free_tokens);
  return hipGetLastError();
}

}  // namespace pkv
