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
constexpr int kPlanHead = 4;  // words: moves, candidates, keep, recent tokens to move up (0: nothing to do)

// Larger key <=> heavier.  NaN maps to 0 (below every number), -0.0 onto +0.0.
__device__ __forceinline__ uint32_t weight_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);
  const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return f == f ? k : 0u;
}

// One workgroup per row: the keep-th heaviest candidate by a radix select of four digits, the lists of moves in order, then the moves of
// the account and the positions themselves.
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(float* __restrict__ weight, int32_t* __restrict__ positions,
                                                                   int32_t* __restrict__ lens, const int32_t* __restrict__ budgets, int64_t N,
                                                                   int budget, int recent, int32_t* __restrict__ plans, int64_t plan_words) {
  __shared__ uint32_t hist[256];
  __shared__ int s_eq[kSelWaves], s_list[kSelWaves];
  __shared__ uint32_t s_prefix, s_left;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = blockIdx.x;
  int32_t* plan = plans + r * plan_words;
  const int cap = (int)((plan_words - kPlanHead) / 2);
  int32_t *from = plan + kPlanHead, *to = from + cap;
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
  float* w = weight + r * N;
  const int cand = n - recent, keep = b - recent;
  int moves = 0;
  if (keep > 0) {
    uint32_t prefix = 0, left = (uint32_t)keep;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = tid; i < cand; i += kSelThreads) {
        const uint32_t k = weight_key(w[i]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (wave == 0) {  // lane l has bins 255 - 4 l downwards
        uint32_t h[4], sum = 0;
        for (int e = 0; e < 4; ++e) sum += h[e] = hist[255 - 4 * lane - e];
        uint32_t upto = sum;
        for (int off = 1; off < 64; off *= 2) {
          const uint32_t o = __shfl_up(upto, off, 64);
          upto += lane >= off ? o : 0u;
        }
        uint32_t above = upto - sum;
        if (above < left && upto >= left)
          for (int e = 0; e < 4; ++e) {
            if (above < left && above + h[e] >= left) {
              s_prefix = prefix | (uint32_t)(255 - 4 * lane - e) << shift;
              s_left = left - above;
            }
            above += h[e];
          }
      }
      __syncthreads();
      prefix = s_prefix;
      left = s_left;
    }
    // kept: above the key, or equal to it and among the first `left` of those
    uint32_t equal = 0;
    int holes = 0;
    for (int i0 = 0; i0 < cand; i0 += kSelThreads) {
      const int i = i0 + tid;
      const uint32_t k = i < cand ? weight_key(w[i]) : 0u;
      const bool eq = i < cand && k == prefix;
      const uint64_t eq_mask = __builtin_amdgcn_ballot_w64(eq), below = (1ull << lane) - 1;
      if (lane == 0) s_eq[wave] = __popcll(eq_mask);
      __syncthreads();
      uint32_t rank = equal + __popcll(eq_mask & below);
      for (int x = 0; x < kSelWaves; ++x) {
        rank += x < wave ? s_eq[x] : 0;
        equal += s_eq[x];
      }
      const bool kept = i < cand && (k > prefix || (eq && rank < left));
      const bool hole = i < keep && !kept, filler = i >= keep && kept;
      const uint64_t hole_mask = __builtin_amdgcn_ballot_w64(hole), fill_mask = __builtin_amdgcn_ballot_w64(filler);
      if (lane == 0) s_list[wave] = __popcll(hole_mask) | __popcll(fill_mask) << 16;
      __syncthreads();
      int h = holes + __popcll(hole_mask & below), f = moves + __popcll(fill_mask & below);
      for (int x = 0; x < kSelWaves; ++x) {
        const int c = s_list[x];
        h += x < wave ? c & 0xffff : 0;
        f += x < wave ? c >> 16 : 0;
        holes += c & 0xffff;
        moves += c >> 16;
      }
      if (hole) to[h] = i;
      if (filler) from[f] = i;
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
  for (int j = tid; j < moves; j += kSelThreads) {
    w[to[j]] = w[from[j]];
    if (pos != nullptr) pos[to[j]] = pos[from[j]];
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

// The planned moves of K and V.  K and V, and the slices of a token, are independent, so each gets a workgroup.  First the candidates, whose new
// places nothing else reads; their old places may be the recent tokens' new ones, so every one of them has been read before those are stored.
// grid (rows, 2 * slices), 256 threads; cpr = 16-byte pieces per token, cps = those of a slice.
template <int PER>
__global__ __launch_bounds__(256) void evict_move_kernel(u32x4* __restrict__ k, u32x4* __restrict__ v, const int32_t* __restrict__ plans,
                                                         int64_t plan_words, int64_t N, int cpr, int cps) {
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const int32_t* plan = plans + r * plan_words;
  const int moves = plan[0], cand = plan[1], keep = plan[2], recent = plan[3];
  const int32_t *from = plan + kPlanHead, *to = from + (plan_words - kPlanHead) / 2;
  u32x4* base = ((blockIdx.y & 1) ? v : k) + (size_t)r * N * cpr + (blockIdx.y >> 1) * cps;
  for (int64_t i0 = 0; i0 < (int64_t)moves * cps; i0 += 256 * PER) {
    u32x4 x[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int64_t i = i0 + u * 256 + tid;
      if (i < (int64_t)moves * cps) x[u] = base[(size_t)from[i / cps] * cpr + i % cps];
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int64_t i = i0 + u * 256 + tid;
      if (i < (int64_t)moves * cps) base[(size_t)to[i / cps] * cpr + i % cps] = x[u];
    }
  }
  __syncthreads();
  for (int64_t i0 = 0; i0 < (int64_t)recent * cps; i0 += 256 * PER) {
    u32x4 x[PER] = {};
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int64_t i = i0 + u * 256 + tid;
      if (i < (int64_t)recent * cps) x[u] = base[(size_t)(cand + i / cps) * cpr + i % cps];
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) asm volatile("" : "+v"(x[u]));  // arrived, not only asked for
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int64_t i = i0 + u * 256 + tid;
      if (i < (int64_t)recent * cps) base[(size_t)(keep + i / cps) * cpr + i % cps] = x[u];
    }
  }
}

// No more candidates than half of a row can change places: those that are kept behind the first `keep` slots are as many as the slots given
// up, and both are candidates.
int64_t plan_words_of(int64_t N) { return (kPlanHead + 2 * (N / 2 + 1) + 3) / 4 * 4; }

}  // namespace

size_t evict_scratch_bytes(int64_t rows, int64_t N) { return (size_t)(rows * plan_words_of(N)) * 4; }

hipError_t launch_evict(void* k, void* v, float* weight, int32_t* positions, int32_t* lens, const int32_t* budgets, int64_t rows, int64_t N,
                        int64_t budget, int64_t recent, int64_t row_bytes, void* scratch, hipStream_t stream) {
  const int64_t words = plan_words_of(N);
  evict_select_kernel<<<(unsigned)rows, kSelThreads, 0, stream>>>(weight, positions, lens, budgets, N, (int)budget, (int)recent, (int32_t*)scratch, words);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int cpr = (int)(row_bytes / 16), slices = cpr % 8 == 0 ? cpr / 8 : 1;
  evict_move_kernel<8><<<dim3((unsigned)rows, (unsigned)(2 * slices)), 256, 0, stream>>>((u32x4*)k, (u32x4*)v, (const int32_t*)scratch, words, N, cpr,
                                                                                       cpr / slices);
  return hipGetLastError();
}

}  // namespace pkv
