// Attention of new tokens over the compacted cache (what the target does with it after the mask was applied), with an account of the softmax
// weight that every cached token gets.
#include "common.hpp"
#include "kernels.hpp"

namespace pkv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -__builtin_huge_valf();

template <bool F16>
__device__ __forceinline__ float to_f32(uint16_t b) {
  if constexpr (F16) return (float)__builtin_bit_cast(_Float16, b);
  else return bf16_bits_to_f32(b);
}
template <bool F16>
__device__ __forceinline__ uint16_t from_f32(float f) {
  if constexpr (F16) return __builtin_bit_cast(uint16_t, (_Float16)f);
  else return f32_to_bf16_bits(f);
}

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

// One workgroup per query: its waves take 64 keys at a time, a lane one of them, with a running maximum and sum.
template <int D, bool F16>
__global__ __launch_bounds__(256) void attend_query_kernel(AttendArgs a, float* __restrict__ lse) {
  __shared__ float q[D], part_o[4][D], part_m[4], part_l[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t query = blockIdx.x, row = query / (a.group * a.T), head = row % a.heads;
  const int t = (int)(query % a.T);
  const float c = kLog2e / __builtin_sqrtf((float)D);
  if (tid < D) q[tid] = to_f32<F16>(((const uint16_t*)a.q)[query * D + tid]);
  __syncthreads();
  float m = kNone, l = 0.0f, o[D / 64] = {};
  auto segment = [&](const uint16_t* k, const uint16_t* v, int n_seen) {
    for (int n0 = wave * 64; n0 < n_seen; n0 += 256) {
      const int n = n0 + lane, many = n_seen - n0 < 64 ? n_seen - n0 : 64;
      float s = kNone;
      if (n < n_seen) {
        s = 0.0f;
        for (int i = 0; i < D; ++i) s = __builtin_fmaf(q[i], to_f32<F16>(k[(size_t)n * D + i]), s);
        s *= c;
      }
      float top = s;
      for (int off = 32; off; off >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, off, 64));
      top = __builtin_fmaxf(top, m);
      const float p = n < n_seen ? __builtin_amdgcn_exp2f(s - top) : 0.0f, old = l > 0.0f ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
      float sum = p;
      for (int off = 32; off; off >>= 1) sum += __shfl_xor(sum, off, 64);
      m = top;
      l = l * old + sum;
      for (int e = 0; e < D / 64; ++e) o[e] *= old;
      for (int j = 0; j < many; ++j) {
        const float pj = __shfl(p, j, 64);
        for (int e = 0; e < D / 64; ++e) o[e] = __builtin_fmaf(pj, to_f32<F16>(v[(size_t)(n0 + j) * D + e * 64 + lane]), o[e]);
      }
    }
  };
  if (a.P > 0)
    segment((const uint16_t*)a.k_shared + (size_t)head * a.P * D, (const uint16_t*)a.v_shared + (size_t)head * a.P * D, row_len(a.shared_lens, head, a.P));
  if (a.N > 0) segment((const uint16_t*)a.k + (size_t)row * a.N * D, (const uint16_t*)a.v + (size_t)row * a.N * D, seen(row_len(a.lens, row, a.N), (int)a.T, t));
  for (int e = 0; e < D / 64; ++e) part_o[wave][e * 64 + lane] = o[e];
  if (lane == 0) {
    part_m[wave] = m;
    part_l[wave] = l;
  }
  __syncthreads();
  float top = part_m[0], sum = 0.0f, f[4];
  for (int w = 1; w < 4; ++w) top = __builtin_fmaxf(top, part_m[w]);
  for (int w = 0; w < 4; ++w) {
    f[w] = part_l[w] != 0.0f ? __builtin_amdgcn_exp2f(part_m[w] - top) : 0.0f;
    sum += f[w] * part_l[w];
  }
  const bool none = sum == 0.0f;
  if (tid < D) {
    float x = 0.0f;
    for (int w = 0; w < 4; ++w) x += f[w] * part_o[w][tid];
    ((uint16_t*)a.out)[query * D + tid] = from_f32<F16>(none ? 0.0f : x / sum);
  }
  if (tid == 0 && lse != nullptr) lse[query] = none ? -kNone : top + __builtin_amdgcn_logf(sum);
}

// weight[n] += sum over the queries that see key n of 2^(c <q, k_n> - lse).  One thread per key; shared keys are seen by every
// sequence's queries of their head, own ones by their row's.
template <int D, bool F16, bool SHARED>
__global__ __launch_bounds__(256) void attend_weight_kernel(AttendArgs a, const float* __restrict__ lse) {
  const int64_t row = blockIdx.y + (int64_t)blockIdx.z * gridDim.y, rows = SHARED ? a.heads : a.batch * a.heads;
  if (row >= rows) return;
  const int64_t most = SHARED ? a.P : a.N;
  const int len = row_len(SHARED ? a.shared_lens : a.lens, row, most), n = blockIdx.x * 256 + threadIdx.x, T = (int)a.T;
  if (n >= len) return;
  const uint16_t* k = (const uint16_t*)(SHARED ? a.k_shared : a.k) + ((size_t)row * most + n) * D;
  const float c = kLog2e / __builtin_sqrtf((float)D);
  const int64_t per = a.group * a.T;
  float w = 0.0f;
  for (int64_t b = 0; b < (SHARED ? a.batch : 1); ++b)
    for (int64_t g = 0; g < per; ++g) {
      const int64_t query = (SHARED ? b * a.heads + row : row) * per + g;
      if (!SHARED && n >= seen(len, T, (int)(g % T))) continue;
      const uint16_t* q = (const uint16_t*)a.q + query * D;
      float s = 0.0f;
      for (int i = 0; i < D; ++i) s = __builtin_fmaf(to_f32<F16>(q[i]), to_f32<F16>(k[i]), s);
      w += __builtin_amdgcn_exp2f(c * s - lse[query]);
    }
  (SHARED ? a.weight_shared : a.weight)[row * most + n] += w;
}

template <int D, bool F16>
hipError_t launch_attend_of(const AttendArgs& a, float* lse, hipStream_t stream) {
  const int64_t rows = a.batch * a.heads;
  attend_query_kernel<D, F16><<<(unsigned)(rows * a.group * a.T), 256, 0, stream>>>(a, lse);
  hipError_t e = hipGetLastError();
  auto grid = [](int64_t n, int64_t r) { return dim3((unsigned)((n + 255) / 256), (unsigned)(r < 65535 ? r : 65535), (unsigned)((r + 65534) / 65535)); };
  if (e == hipSuccess && a.weight != nullptr && a.N > 0) {
    attend_weight_kernel<D, F16, false><<<grid(a.N, rows), 256, 0, stream>>>(a, lse);
    e = hipGetLastError();
  }
  if (e == hipSuccess && a.weight_shared != nullptr && a.P > 0) {
    attend_weight_kernel<D, F16, true><<<grid(a.P, a.heads), 256, 0, stream>>>(a, lse);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

size_t attend_scratch_bytes(const AttendArgs& a) { return (size_t)(a.batch * a.heads * a.group * a.T) * 4; }

hipError_t launch_attend(const AttendArgs& a, void* scratch, hipStream_t stream) {
  if (a.D == 64) return a.f16 ? launch_attend_of<64, true>(a, (float*)scratch, stream) : launch_attend_of<64, false>(a, (float*)scratch, stream);
  return a.f16 ? launch_attend_of<128, true>(a, (float*)scratch, stream) : launch_attend_of<128, false>(a, (float*)scratch, stream);
}

}  // namespace pkv
