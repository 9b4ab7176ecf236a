// Softmax attention within packed sequences.
//
// Query head j of row r of a sequence reads key head j / (heads / kv_heads) of the rows of that sequence, all of them or (causal) those up to r:
//
//   z_k = scale q . key_k,  o = sum_k e^(z_k - lse) value_k,  lse = log sum_k e^(z_k)
//
// One pass over the keys with the running maximum and sum of the softmax: a block holds 128 queries of one head, 32 to each of
// its four wavefronts, and walks the sequence's keys in panels that lie in LDS two at a time.  Scores, probabilities and results stay in
// registers (attention_common.hpp has the layout).  Scores, statistics and sums are fp32; with bf16 operands the probabilities are rounded to
// bf16 for the product with the values, relative to their running maximum, which is an error of 2^-9 of each term.
#include "attention_common.hpp"
#include "detag_internal.h"

namespace detag {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kHigh = 32 * kWaves;  // queries of a block
constexpr float kSlack = 8.f;  // how far (in powers of two) a maximum may grow before what was summed is scaled again

template <class T, int WIDTH, bool Direct>
__global__ __launch_bounds__(kThreads) void attention_kernel(AttentionArgs a) {
  constexpr int kRows = sizeof(T) == 2 ? 64 : 32, kScores = kRows / 32;
  using Keys = Panel<T, WIDTH, kRows, kThreads, Direct>;
  __shared__ __attribute__((aligned(1024))) char lds_[4 * Keys::kBytes];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds_));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
  const int groups = a.heads / a.kv_heads;
  const int64_t runs = part_runs(a.rows, a.parts, kHigh), blocks = attention_blocks(a.kv_heads, runs * groups);
  const uint32_t along = Keys::along_base(), across = Keys::across_base();
  for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
    const Work w = work_of(block, a.kv_heads, runs, groups);
    if (w.run < 0) continue;
    // causal: the last runs of a sequence see the most keys and start first
    const Run run = run_of(a.offsets, a.parts, a.rows, kHigh, int(a.causal ? runs - 1 - w.run : w.run));
    if (run.part < 0) continue;
    const int head = w.kv * groups + w.group, length = run.hi - run.lo;
    const int first = run.first - run.lo + 32 * wave, query = first + p;  // within the sequence
    const int upto = a.causal && run.first - run.lo + kHigh < length ? run.first - run.lo + kHigh : length;  // keys that the block reads
    const int mine = a.causal && first + 32 < length ? first + 32 : first < length ? length : 0;             // and the wavefront
    const int panels = (upto + kRows - 1) / kRows;

    u32x4 q[Keys::kSteps];
    load_operand<T>(q, static_cast<const T *>(a.q) + head * a.width, a.ldq, int64_t(run.lo) + query, query < length, a.width);
    Keys keys, values;
    keys.init(static_cast<const T *>(a.k) + run.lo * a.ldk + w.kv * a.width, a.ldk, a.width);
    values.init(static_cast<const T *>(a.v) + run.lo * a.ldv + w.kv * a.width, a.ldv, a.width);

    f32x16 acc[Keys::kBlocks];
#pragma unroll
    for (int b = 0; b < Keys::kBlocks; ++b) acc[b] = f32x16{};
    float top = -INFINITY, base = 0.f, sum = 0.f;  // the largest score, what exponents are taken relative to (scale2 * a maximum), this half's sum

    __syncthreads();  // the block before is done with the panels
    auto request = [&](int t) {
      const uint32_t to = lds + (t & 1) * 2 * Keys::kBytes;
      keys.request(t * kRows, length, to), values.request(t * kRows, length, to + Keys::kBytes);
    };
    auto deliver = [&](int t) {
      const uint32_t to = lds + (t & 1) * 2 * Keys::kBytes;
      keys.deliver(to), values.deliver(to + Keys::kBytes);
    };
    request(0), deliver(0);
    for (int t = 0; t < panels; ++t) {
      wait_all();
      __builtin_amdgcn_s_barrier();  // panel t is there, and all have read panel t - 1
      asm volatile("" ::: "memory");
      if (t + 1 < panels) request(t + 1);
      const uint32_t here = lds + (t & 1) * 2 * Keys::kBytes;
      const int key0 = t * kRows;
      if (key0 < mine) {
        f32x16 s[kScores];
#pragma unroll
        for (int b = 0; b < kScores; ++b) s[b] = f32x16{};
#pragma unroll
        for (int k = 0; k < Keys::kSteps; ++k)
#pragma unroll
          for (int b = 0; b < kScores; ++b) s[b] = multiply32<T>(Keys::along(along, here, b, k), q[k], s[b]);
        const int last = a.causal && query < length ? query : length - 1;
        if (key0 + kRows > (a.causal ? first + 1 : length)) {  // some of the wavefront's lanes do not see all
#pragma unroll
          for (int b = 0; b < kScores; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = key0 + 32 * b + 8 * (r / 4) + 4 * h + r % 4 <= last ? s[b][r] : -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int b = 0; b < kScores; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) most = fmaxf(most, s[b][r]);
        most = fmaxf(most, other_half(most));
        if (__ballot(!(most * a.scale2 <= base + kSlack) || top == -INFINITY)) {
          top = fmaxf(top, most);
          const float now = top == -INFINITY ? 0.f : top * a.scale2, factor = __builtin_amdgcn_exp2f(base - now);
          base = now, sum *= factor;
#pragma unroll
          for (int b = 0; b < Keys::kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[b][r] *= factor;
        }
#pragma unroll
        for (int b = 0; b < kScores; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[b][r] = __builtin_amdgcn_exp2f(s[b][r] * a.scale2 - base);
            sum += s[b][r];
          }
#pragma unroll
        for (int b = 0; b < kScores; ++b)
#pragma unroll
          for (int g = 0; g < Keys::kGroups; ++g) {
            const u32x4 prob = as_operand<T>(s[b], g);
#pragma unroll
            for (int c = 0; c < Keys::kBlocks; ++c)
              acc[c] = multiply32<T>(Keys::across(across, here + Keys::kBytes, c, 32 * b, g), prob, acc[c]);
          }
      }
      if (t + 1 < panels) deliver(t + 1);
    }
    if (query < length) {
      sum += other_half(sum);
      const int64_t row = int64_t(run.lo) + query;
      store_row(static_cast<T *>(a.out) + row * a.ldo + head * a.width, acc, 1.f / sum, a.width);
      if (a.lse && h == 0) a.lse[head * int64_t(a.rows) + row] = base * kLn2 + logf(sum);
    }
  }
}

template <class T, int WIDTH>
int attention(const AttentionArgs &a, bool direct, hipStream_t st) {
  int64_t blocks = attention_blocks(a.kv_heads, part_runs(a.rows, a.parts, kHigh) * (a.heads / a.kv_heads));
  if (blocks > 1 << 20) blocks = 1 << 20;
  if (direct) attention_kernel<T, WIDTH, true><<<dim3(uint32_t(blocks)), kThreads, 0, st>>>(a);
  else attention_kernel<T, WIDTH, false><<<dim3(uint32_t(blocks)), kThreads, 0, st>>>(a);
  return hip_rc(hipGetLastError());
}

}  // namespace

int launch_attention(const AttentionArgs &a, bool bf16, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const bool direct = panels_direct(a.k, a.ldk, a.width, e) && panels_direct(a.v, a.ldv, a.width, e);
  if (bf16) return a.width <= 64 ? attention<bf16_t, 64>(a, direct, st) : attention<bf16_t, 128>(a, direct, st);
  return a.width <= 64 ? attention<float, 64>(a, direct, st) : attention<float, 128>(a, direct, st);
}

}  // namespace detag
