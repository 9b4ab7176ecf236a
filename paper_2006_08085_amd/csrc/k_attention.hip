// Softmax attention within packed sequences.
//
// Query head j of row r of a sequence reads key head j / (heads / kv_heads) of the rows of that sequence, all of them or (causal) those up to r:
//
//   z_k = scale q . key_k,  o = sum_k e^(z_k - lse) value_k,  lse = log sum_k e^(z_k)
//
// One pass over the keys with the running maximum and sum of the softmax: a block holds 128 queries of one head, 32 to each of its four
// wavefronts, and walks the sequence's keys in panels, two of which lie in LDS: one is read while the next arrives.  Scores, probabilities and
// results stay in registers (attention_common.hpp has the layout).  Scores, statistics and sums are fp32; with bf16 operands the probabilities
// are rounded to bf16 for the product with the values, relative to their running maximum, which is an error of 2^-8 of each term at most.
//
// What bounds the long ones is the matrix cores and what power leaves of their clock.  bf16, 32 heads of 128 with 8 key heads, two sequences
// of 8192 rows, causal: 980 to 1095 us from card to card, 1.12 to 1.0 PFLOP/s (a large library product 1.22); the clock falls from 1.9 to
// 1.55 GHz meanwhile.  Results leave through LDS as whole rows: 24 uneven sequences of 8192 rows in all, 16 heads of 128 with 4 key heads,
// 46.5 us; 50.5 with each lane storing its own row's parts and operands by 64-bit addresses.  Scores of the next panel taken during the softmax of this one
// needed more registers than they hid (1537 us for 1230 at the time); a wavefront's priority changed nothing.  Few queries are bound by one
// walk over the keys: hence Split (attention_common.hpp has both sides).
#include "attention_common.hpp"
#include "detag_internal.h"

namespace detag {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kSlack = 8.f;  // how far (in powers of two) a maximum may grow before what was summed is scaled again

// Split: the block's wavefronts have the same 32 queries and 32 keys of a panel each, and join their results at the end.
template <class T, bool Split>
struct Cut {
  static constexpr int kHigh = Split ? 32 : 32 * kWaves;                      // queries of a block
  static constexpr int kRows = Split ? 32 * kWaves : sizeof(T) == 2 ? 64 : 32;  // keys of a panel
  static constexpr int kStages = Split ? 1 : 2;                               // panels in LDS
};

template <class T, int WIDTH, bool Direct, bool Split>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 && !Split ? 2 : 1) void attention_kernel(AttentionArgs a, WorkGrid grid) {
  using C = Cut<T, Split>;
  constexpr int kHigh = C::kHigh, kRows = C::kRows, kScores = Split ? 1 : kRows / 32;
  using Keys = Panel<T, WIDTH, kRows, kThreads, Direct>;
  __shared__ __attribute__((aligned(1024))) char lds_[2 * C::kStages * Keys::kBytes];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds_));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, p = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
  const int groups = a.heads / a.kv_heads;
  const uint32_t along = Keys::along_base(), across = Keys::across_base();
  for_work(grid, [&](int kv, uint32_t piece) {
    const int turn = piece / groups;
    const Run run = run_in_turn(a, kHigh, turn, grid.each / groups, a.causal);
    if (run.part < 0) return;
    const int head = kv * groups + int(piece - turn * groups), length = run.hi - run.lo;
    const int own = Split ? wave : 0;  // the wavefront's keys of a panel: from 32 * own on
    const int first = run.first - run.lo + (Split ? 0 : 32 * wave), query = first + p;  // within the sequence
    const int upto = a.causal && run.first - run.lo + kHigh < length ? run.first - run.lo + kHigh : length;  // keys that the block reads
    const int mine = a.causal && first + 32 < length ? first + 32 : first < length ? length : 0;             // and the wavefront
    const int panels = (upto + kRows - 1) / kRows;

    u32x4 q[Keys::kSteps];
    load_operand<T, Direct>(q, static_cast<const T *>(a.q) + run.first * a.ldq + head * a.width, a.ldq, query - (run.first - run.lo), query < length, a.width);
    Keys keys, values;
    keys.init(static_cast<const T *>(a.k) + run.lo * a.ldk + kv * a.width, a.ldk, a.width, length);
    values.init(static_cast<const T *>(a.v) + run.lo * a.ldv + kv * a.width, a.ldv, a.width, length);

    f32x16 acc[Keys::kBlocks];
#pragma unroll
    for (int b = 0; b < Keys::kBlocks; ++b) acc[b] = f32x16{};
    float top = -INFINITY, base = 0.f, sum = 0.f;  // the largest score, what exponents are taken relative to (scale2 * a maximum), this half's sum

    __syncthreads();  // the block before is done with the panels
    auto stage = [&](int odd) { return lds + odd * 2 * Keys::kBytes; };
    auto request = [&](int odd) { keys.request(stage(odd)), values.request(stage(odd) + Keys::kBytes); };
    auto deliver = [&](int odd) { keys.deliver(stage(odd)), values.deliver(stage(odd) + Keys::kBytes); };
    auto meet = [] {
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    request(0), deliver(0);
    // One panel; its stage is a constant, and so are all offsets into LDS.  Two stages: the next panel is under way meanwhile.  One (Split,
    // for two blocks of a compute unit): the next keys from when all have read these, and likewise the values.
    auto panel = [&](auto odd_, int t) {
      constexpr int odd = Split ? 0 : decltype(odd_)::value;
      if constexpr (Split && Direct) wait_loads<Keys::kLoads>();  // the keys
      else wait_all();
      wait_lds();
      meet();  // panel t is there (its keys), and all have read panel t - 1
      const int key0 = t * kRows + 32 * own;
      // (requested when the scores' products have been issued, which take longer than that)
      auto next_keys = [&] {
        if constexpr (Split) {
          wait_all();  // the values
          meet();
          if (t + 1 < panels) keys.request(lds);
        } else if (t + 1 < panels) {
          request(odd ^ 1);
        }
      };
      if (key0 >= mine) next_keys();
      if (key0 < mine) {
        // A panel's fragments are requested before they are needed: the scores' all at once, the values' while the softmax runs.
        u32x4 x[kScores][Keys::kSteps], y[Keys::kGroups][Keys::kBlocks];
#pragma unroll
        for (int k = 0; k < Keys::kSteps; ++k)
#pragma unroll
          for (int b = 0; b < kScores; ++b) x[b][k] = Keys::along(along, stage(odd), own + b, k);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        f32x16 s[kScores];
#pragma unroll
        for (int b = 0; b < kScores; ++b) s[b] = f32x16{};
#pragma unroll
        for (int k = 0; k < Keys::kSteps; ++k)
#pragma unroll
          for (int b = 0; b < kScores; ++b)
            if (sizeof(T) == 2 || 2 * k * Keys::kElems < a.width) s[b] = multiply32<T>(x[b][k], q[k], s[b]);  // (fp32 products take long)
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        next_keys();
#pragma unroll
        for (int g = 0; g < Keys::kGroups; ++g)
#pragma unroll
          for (int c = 0; c < Keys::kBlocks; ++c) y[g][c] = Keys::across(across, stage(odd) + Keys::kBytes, c, 32 * own, g);
        __builtin_amdgcn_sched_barrier(0);
        const int last = a.causal && query < length ? query : length - 1;
        if (key0 + 32 * kScores > (a.causal ? first + 1 : length)) {  // some of the wavefront's lanes do not see all
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
          // What has been summed is relative to a smaller base, or is nothing: then base is still 0, and the scores may lie far below it.
          const float now = top == -INFINITY ? 0.f : top * a.scale2, factor = __builtin_amdgcn_exp2f(fminf(base - now, 0.f));
          base = now, sum *= factor;
#pragma unroll
          for (int b = 0; b < Keys::kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[b][r] *= factor;
        }
        u32x4 prob[kScores][Keys::kGroups];
#pragma unroll
        for (int b = 0; b < kScores; ++b) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[b][r] = __builtin_amdgcn_exp2f(s[b][r] * a.scale2 - base);
            sum += s[b][r];
          }
#pragma unroll
          for (int g = 0; g < Keys::kGroups; ++g) prob[b][g] = as_operand<T>(s[b], g);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int b = 0; b < kScores; ++b)
#pragma unroll
          for (int g = 0; g < Keys::kGroups; ++g) {
#pragma unroll
            for (int c = 0; c < Keys::kBlocks; ++c) acc[c] = multiply32<T>(y[g][c], prob[b][g], acc[c]);
            if (b + 1 < kScores)
#pragma unroll
              for (int c = 0; c < Keys::kBlocks; ++c) y[g][c] = Keys::across(across, stage(odd) + Keys::kBytes, c, 32 * (b + 1), g);
          }
        __builtin_amdgcn_s_setprio(0);
      }
      if constexpr (Split) {
        wait_lds();
        meet();  // all have read the values
        if (t + 1 < panels) keys.deliver(lds), values.request(lds + Keys::kBytes), values.deliver(lds + Keys::kBytes);
      } else {
        if (t + 1 < panels) deliver(odd ^ 1);
      }
    };
    for (int t = 0; t < panels; t += 2) {
      panel(std::integral_constant<int, 0>{}, t);
      if (t + 1 < panels) panel(std::integral_constant<int, 1>{}, t + 1);
    }
    sum += other_half(sum);
    const int64_t row = int64_t(run.lo) + query;
    if constexpr (Split) {
      // parts relative to the largest of their bases, added up in the wavefronts' order; every wavefront takes some of the columns
      __shared__ float shares[2][kWaves][32];
      if (h == 0) shares[0][wave][p] = top == -INFINITY ? -INFINITY : base, shares[1][wave][p] = sum;
#pragma unroll
      for (int b = 0; b < Keys::kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          *reinterpret_cast<__attribute__((address_space(3))) float *>(lds + (((wave * Keys::kBlocks + b) * 16 + r) * 64 + lane) * 4) = acc[b][r];
      __syncthreads();
      base = -INFINITY;
#pragma unroll
      for (int w2 = 0; w2 < kWaves; ++w2) base = fmaxf(base, shares[0][w2][p]);
      if (base == -INFINITY) base = 0.f;
      sum = 0.f;
      float factor[kWaves];
#pragma unroll
      for (int w2 = 0; w2 < kWaves; ++w2) {
        factor[w2] = __builtin_amdgcn_exp2f(shares[0][w2][p] - base);
        sum += shares[1][w2][p] * factor[w2];
      }
      if (query < length) {
        const float inverse = 1.f / sum;
        T *const to = static_cast<T *>(a.out) + row * a.ldo + head * a.width;
        for (int b = wave; b < Keys::kBlocks; b += kWaves) {
          f32x16 part[1] = {f32x16{}};
#pragma unroll
          for (int w2 = 0; w2 < kWaves; ++w2)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              part[0][r] += factor[w2] * *reinterpret_cast<__attribute__((address_space(3))) float *>(lds + (((w2 * Keys::kBlocks + b) * 16 + r) * 64 + lane) * 4);
          store_row(to + 32 * b, part, inverse, a.width - 32 * b);
        }
        if (a.lse && h == 0 && wave == 0) a.lse[head * int64_t(a.rows) + row] = base * kLn2 + logf(sum);
      }
    } else {
      if constexpr (Direct) {
        static_assert(Split || kWaves * 32 * WIDTH * sizeof(T) <= sizeof(lds_), "the rows fit the panels");
        __syncthreads();  // all have read the last panel
        store_rows(static_cast<T *>(a.out) + (int64_t(run.lo) + first) * a.ldo + head * a.width, a.ldo, length - first,
                   lds + wave * 32 * WIDTH * int(sizeof(T)), acc, 1.f / sum, a.width);
      } else if (query < length) {
        store_row(static_cast<T *>(a.out) + row * a.ldo + head * a.width, acc, 1.f / sum, a.width);
      }
      if (query < length && a.lse && h == 0) a.lse[head * int64_t(a.rows) + row] = base * kLn2 + logf(sum);
    }
  });
}

template <class T, int WIDTH, bool Split>
int launch_cut(const AttentionArgs &a, bool direct, hipStream_t st) {
  const WorkGrid grid = work_grid(a.kv_heads, part_runs(a.rows, a.parts, Cut<T, Split>::kHigh) * (a.heads / a.kv_heads));
  if (direct) attention_kernel<T, WIDTH, true, Split><<<work_blocks(grid), kThreads, 0, st>>>(a, grid);
  else attention_kernel<T, WIDTH, false, Split><<<work_blocks(grid), kThreads, 0, st>>>(a, grid);
  return hip_rc(hipGetLastError());
}

template <class T, int WIDTH>
int attention(const AttentionArgs &a, bool direct, hipStream_t st) {
  return attention_splits(a, sizeof(T) == 2) ? launch_cut<T, WIDTH, true>(a, direct, st) : launch_cut<T, WIDTH, false>(a, direct, st);
}

}  // namespace

int launch_attention(const AttentionArgs &a, bool bf16, void *stream) {
  const size_t e = bf16 ? 2 : 4;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const bool direct = panels_direct(a.q, a.ldq, a.width, e) && panels_direct(a.k, a.ldk, a.width, e) && panels_direct(a.v, a.ldv, a.width, e);
  if (bf16) return a.width <= 64 ? attention<bf16_t, 64>(a, direct, st) : attention<bf16_t, 128>(a, direct, st);
  return a.width <= 64 ? attention<float, 64>(a, direct, st) : attention<float, 128>(a, direct, st);
}

}  // namespace detag
