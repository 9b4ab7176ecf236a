// The gradient of attention (k_attention.hip): from q, k, v, the result o, lse and dO,
//
//   p_k = e^(z_k - lse),  delta = dO . o,  dz_k = p_k (dO . v_k - delta) scale
//   dq = sum_k dz_k key_k;   dkey_k = sum over the queries that read it, of every query head that shares it, of dz_k q;  dv_k = sum p_k dO
//
// Two kernels, neither of which stores a probability, and no sum whose order changes.  The first has 128 queries of a head in a block, 32
// to a wavefront, and walks the keys (scores, dO V^T, dq); it takes delta first and leaves it for the second, which has 64 keys of a key
// head in a block and walks the queries of all the heads that share it (scores, dO V^T, dv, dk).  Scores and dO V^T are computed
// in both: seven products instead of five, in place of atomics or of a pass over fp32 parts.  With bf16 operands p and dz are rounded to bf16
// for the products that follow; all sums are fp32 and rounded once.
#include "attention_common.hpp"
#include "detag_internal.h"

namespace detag {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kHigh = 32 * kWaves;  // queries, or keys, of a block
constexpr int kRows = 32;                                               // of a panel

template <class T, int WIDTH, bool Direct>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void attention_grad_query_kernel(AttentionArgs a, WorkGrid grid) {
  using Keys = Panel<T, WIDTH, kRows, kThreads, Direct>;
  __shared__ __attribute__((aligned(1024))) char lds_[4 * Keys::kBytes];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds_));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
  const int groups = a.heads / a.kv_heads;
  const uint32_t along = Keys::along_base(), across = Keys::across_base();
  for_work(grid, [&](int kv, uint32_t piece) {
    const int turn = piece / groups, number = a.causal ? grid.each / groups - 1 - turn : turn;
    const Run run = run_of(a.offsets, a.parts, a.rows, kHigh, number);
    if (run.part < 0) return;
    const int head = kv * groups + int(piece - turn * groups), length = run.hi - run.lo;
    const int first = run.first - run.lo + 32 * wave, query = first + p;
    const int upto = a.causal && run.first - run.lo + kHigh < length ? run.first - run.lo + kHigh : length;
    const int mine = a.causal && first + 32 < length ? first + 32 : first < length ? length : 0;
    const int panels = (upto + kRows - 1) / kRows;
    const int64_t row = int64_t(run.lo) + query;
    const bool there = query < length;

    __syncthreads();  // the block before is done with the panels
    Keys keys, values;
    keys.init(static_cast<const T *>(a.k) + run.lo * a.ldk + kv * a.width, a.ldk, a.width, length);
    values.init(static_cast<const T *>(a.v) + run.lo * a.ldv + kv * a.width, a.ldv, a.width, length);
    auto request = [&](int t) {
      const uint32_t to = lds + (t & 1) * 2 * Keys::kBytes;
      keys.request(to), values.request(to + Keys::kBytes);
    };
    auto deliver = [&](int t) {
      const uint32_t to = lds + (t & 1) * 2 * Keys::kBytes;
      keys.deliver(to), values.deliver(to + Keys::kBytes);
    };
    request(0), deliver(0);
    u32x4 q[Keys::kSteps], g[Keys::kSteps];
    load_operand<T>(q, static_cast<const T *>(a.q) + head * a.width, a.ldq, row, there, a.width);
    load_operand<T>(g, static_cast<const T *>(a.d_o) + head * a.width, a.ld_do, row, there, a.width);
    float delta = 0.f;
    {
      u32x4 o[Keys::kSteps];
      load_operand<T>(o, static_cast<const T *>(a.o) + head * a.width, a.ldo, row, there, a.width);
#pragma unroll
      for (int s = 0; s < Keys::kSteps; ++s)
#pragma unroll
        for (int e = 0; e < Keys::kElems; ++e) delta += element<T>(o[s], e) * element<T>(g[s], e);
    }
    delta += other_half(delta);
    const int64_t at = head * int64_t(a.rows) + row;
    if (there && h == 0) a.delta[at] = delta;
    const float level = there ? a.lse[at] * (1.f / kLn2) : 0.f;  // in powers of two

    f32x16 acc[Keys::kBlocks];
#pragma unroll
    for (int b = 0; b < Keys::kBlocks; ++b) acc[b] = f32x16{};
    for (int t = 0; t < panels; ++t) {
      wait_all();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (t + 1 < panels) request(t + 1);
      const uint32_t here = lds + (t & 1) * 2 * Keys::kBytes;
      const int key0 = t * kRows;
      if (key0 < mine) {
        f32x16 s{}, ds{};
#pragma unroll
        for (int k = 0; k < Keys::kSteps; ++k) {
          s = multiply32<T>(Keys::along(along, here, 0, k), q[k], s);
          ds = multiply32<T>(Keys::along(along, here + Keys::kBytes, 0, k), g[k], ds);
        }
        const int last = a.causal && there ? query : length - 1;
        const bool all = key0 + kRows <= (a.causal ? first + 1 : length);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float prob = __builtin_amdgcn_exp2f(s[r] * a.scale2 - level);
          ds[r] = prob * (ds[r] - delta);
          if (!all) ds[r] = key0 + 8 * (r / 4) + 4 * h + r % 4 <= last ? ds[r] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < Keys::kGroups; ++j) {
          const u32x4 dz = as_operand<T>(ds, j);
#pragma unroll
          for (int c = 0; c < Keys::kBlocks; ++c) acc[c] = multiply32<T>(Keys::across(across, here, c, 0, j), dz, acc[c]);
        }
      }
      if (t + 1 < panels) deliver(t + 1);
    }
    if (there) store_row(static_cast<T *>(a.dq) + row * a.ld_dq + head * a.width, acc, a.scale, a.width);
  });
}

// A block's four wavefronts are two times two: 32 of its 64 keys each, and every other panel of queries, whose parts of dk and dv are added up
// at the end.  A panel is 32 queries of one of the heads that share the key head; the panels of all these heads are taken one after the
// other, two at a time.
constexpr int kSplit = 2, kKeysHigh = 32 * kWaves / kSplit;

template <class T, int WIDTH, bool Direct>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void attention_grad_key_kernel(AttentionArgs a, WorkGrid grid) {
  using Queries = Panel<T, WIDTH, kRows, kThreads, Direct>;
  constexpr int kStage = 2 * kSplit * Queries::kBytes;
  static_assert(2 * kStage >= (kWaves / kSplit) * 2 * Queries::kBlocks * 16 * 64 * 4, "the parts of dk and dv fit the panels");
  __shared__ __attribute__((aligned(1024))) char lds_[2 * kStage];
  __shared__ __attribute__((aligned(16))) float levels_[2][kSplit][2][kRows];  // lse in powers of two, delta
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds_));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, p = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
  const int keys = wave % (kWaves / kSplit), split = wave / (kWaves / kSplit);
  const int groups = a.heads / a.kv_heads;
  const uint32_t along = Queries::along_base(), across = Queries::across_base();
  for_work(grid, [&](int kv, uint32_t piece) {
    const Run run = run_of(a.offsets, a.parts, a.rows, kKeysHigh, piece);  // causal: the first runs of a sequence are read by the most queries
    if (run.part < 0) return;
    const int length = run.hi - run.lo, first = run.first - run.lo + 32 * keys, key = first + p;
    const int start = a.causal ? run.first - run.lo : 0;  // first query that reads the block's keys
    const int64_t row = int64_t(run.lo) + key;
    const bool there = key < length;
    const int panels = (length - start + kRows - 1) / kRows, steps = panels * groups;

    __syncthreads();  // the block before is done with the panels
    Queries queries, grads;
    queries.init(static_cast<const T *>(a.q) + run.lo * a.ldq + int64_t(kv) * groups * a.width, a.ldq, a.width, length);
    grads.init(static_cast<const T *>(a.d_o) + run.lo * a.ld_do + int64_t(kv) * groups * a.width, a.ld_do, a.width, length);
    // Where a step is: a head of the group, and a panel of its queries.
    struct Step {
      int head, panel;
      __device__ __forceinline__ void on(int by, int panels) {
        panel += by;
        while (panel >= panels) panel -= panels, ++head;
      }
    };
    const Queries queries0 = queries, grads0 = grads;
    Queries queries2 = queries, grads2 = grads;  // (their registers, if they have any)
    float held = 0.f;
    auto request = [&](Step s, int stage) {
      const uint32_t to = lds + stage * kStage;
      int heads[kSplit], at[kSplit];
#pragma unroll
      for (int i = 0; i < kSplit; ++i, s.on(1, panels)) {
        heads[i] = s.head, at[i] = start + s.panel * kRows;
        if (s.head >= groups) {
          at[i] = length;  // no such step
          continue;
        }
        const int64_t over = int64_t(s.head) * a.width * int64_t(sizeof(T));
        Queries &qs = i ? queries2 : queries, &gs = i ? grads2 : grads;
        qs.from = queries0.from + over, qs.left = queries0.left, gs.from = grads0.from + over, gs.left = grads0.left;
        qs.skip(at[i]), gs.skip(at[i]);
        qs.request(to + 2 * i * Queries::kBytes), gs.request(to + (2 * i + 1) * Queries::kBytes);
      }
      if (threadIdx.x < 2 * kRows * kSplit) {
        const int i = threadIdx.x / (2 * kRows), r = (i ? at[1] : at[0]) + int(threadIdx.x % kRows);
        const int64_t from = (kv * groups + (i ? heads[1] : heads[0])) * int64_t(a.rows) + run.lo + r;
        held = r < length ? (threadIdx.x / kRows % 2 == 0 ? a.lse[from] * (1.f / kLn2) : a.delta[from]) : 0.f;
      }
    };
    auto deliver = [&](int stage) {
      const uint32_t to = lds + stage * kStage;
      queries.deliver(to), grads.deliver(to + Queries::kBytes);
      queries2.deliver(to + 2 * Queries::kBytes), grads2.deliver(to + 3 * Queries::kBytes);
      if (threadIdx.x < 2 * kRows * kSplit) (&levels_[stage][0][0][0])[threadIdx.x] = held;
    };
    Step next{0, 0}, mine{0, 0};
    mine.on(split, panels);
    request(next, 0), deliver(0);
    u32x4 k[Queries::kSteps], v[Queries::kSteps];
    load_operand<T>(k, static_cast<const T *>(a.k) + kv * a.width, a.ldk, row, there, a.width);
    load_operand<T>(v, static_cast<const T *>(a.v) + kv * a.width, a.ldv, row, there, a.width);
    f32x16 dk[Queries::kBlocks], dv[Queries::kBlocks];
#pragma unroll
    for (int b = 0; b < Queries::kBlocks; ++b) dk[b] = f32x16{}, dv[b] = f32x16{};
    for (int t = 0, stage = 0; t < steps; t += kSplit, stage ^= 1) {
      wait_all();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      next.on(kSplit, panels);
      if (t + kSplit < steps) request(next, stage ^ 1);
      const uint32_t here = lds + stage * kStage + 2 * split * Queries::kBytes;
      const int query0 = start + mine.panel * kRows;
      if (first < length && mine.head < groups && (!a.causal || query0 + kRows > first)) {
        f32x16 s{}, ds{};
#pragma unroll
        for (int j = 0; j < Queries::kSteps; ++j) {
          s = multiply32<T>(Queries::along(along, here, 0, j), k[j], s);
          ds = multiply32<T>(Queries::along(along, here + Queries::kBytes, 0, j), v[j], ds);
        }
        const bool all = query0 + kRows <= length && (!a.causal || query0 >= first + 31);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float prob = __builtin_amdgcn_exp2f(s[r] * a.scale2 - levels_[stage][split][0][8 * (r / 4) + 4 * h + r % 4]);
          ds[r] = prob * (ds[r] - levels_[stage][split][1][8 * (r / 4) + 4 * h + r % 4]);
          if (!all) {
            const int at = query0 + 8 * (r / 4) + 4 * h + r % 4;
            const bool reads = at < length && (!a.causal || at >= key);
            prob = reads ? prob : 0.f, ds[r] = reads ? ds[r] : 0.f;
          }
          s[r] = prob;
        }
#pragma unroll
        for (int j = 0; j < Queries::kGroups; ++j) {
          const u32x4 prob = as_operand<T>(s, j), dz = as_operand<T>(ds, j);
#pragma unroll
          for (int c = 0; c < Queries::kBlocks; ++c) {
            dv[c] = multiply32<T>(Queries::across(across, here + Queries::kBytes, c, 0, j), prob, dv[c]);
            dk[c] = multiply32<T>(Queries::across(across, here, c, 0, j), dz, dk[c]);
          }
        }
      }
      mine.on(kSplit, panels);
      if (t + kSplit < steps) deliver(stage ^ 1);
    }
    __syncthreads();  // all have read the last panels
    auto part = [&](int i) { return reinterpret_cast<__attribute__((address_space(3))) float *>(lds + ((keys * 32 * Queries::kBlocks + i) * 64 + lane) * 4); };
    if (split)
#pragma unroll
      for (int b = 0; b < Queries::kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) *part(32 * b + r) = dk[b][r], *part(32 * b + 16 + r) = dv[b][r];
    __syncthreads();
    if (split == 0 && there) {
#pragma unroll
      for (int b = 0; b < Queries::kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[b][r] += *part(32 * b + r), dv[b][r] += *part(32 * b + 16 + r);
      store_row(static_cast<T *>(a.dk) + row * a.ld_dk + kv * a.width, dk, a.scale, a.width);
      store_row(static_cast<T *>(a.dv) + row * a.ld_dv + kv * a.width, dv, 1.f, a.width);
    }
  });
}

template <class T, int WIDTH>
int attention_grad(const AttentionArgs &a, hipStream_t st) {
  const WorkGrid by_query = work_grid(a.kv_heads, part_runs(a.rows, a.parts, kHigh) * (a.heads / a.kv_heads));
  const WorkGrid by_key = work_grid(a.kv_heads, part_runs(a.rows, a.parts, kKeysHigh));
  if (panels_direct(a.k, a.ldk, a.width, sizeof(T)) && panels_direct(a.v, a.ldv, a.width, sizeof(T)))
    attention_grad_query_kernel<T, WIDTH, true><<<work_blocks(by_query), kThreads, 0, st>>>(a, by_query);
  else attention_grad_query_kernel<T, WIDTH, false><<<work_blocks(by_query), kThreads, 0, st>>>(a, by_query);
  if (const int rc = hip_rc(hipGetLastError())) return rc;
  if (panels_direct(a.q, a.ldq, a.width, sizeof(T)) && panels_direct(a.d_o, a.ld_do, a.width, sizeof(T)))
    attention_grad_key_kernel<T, WIDTH, true><<<work_blocks(by_key), kThreads, 0, st>>>(a, by_key);
  else attention_grad_key_kernel<T, WIDTH, false><<<work_blocks(by_key), kThreads, 0, st>>>(a, by_key);
  return hip_rc(hipGetLastError());
}

}  // namespace

int launch_attention_grad(const AttentionArgs &a, bool bf16, void *stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (bf16) return a.width <= 64 ? attention_grad<bf16_t, 64>(a, st) : attention_grad<bf16_t, 128>(a, st);
  return a.width <= 64 ? attention_grad<float, 64>(a, st) : attention_grad<float, 128>(a, st);
}

}  // namespace detag
