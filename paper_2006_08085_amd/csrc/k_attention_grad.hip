// The gradient of attention (k_attention.hip): from q, k, v, the result o, lse and dO,
//
//   p_k = e^(z_k - lse),  delta = dO . o,  dz_k = p_k (dO . v_k - delta) scale
//   dq = sum_k dz_k key_k;   dkey_k = sum over the queries that read it, of every query head that shares it, of dz_k q;  dv_k = sum p_k dO
//
// Two kernels, neither of which stores a probability, and no sum whose order changes.  The first has 128 queries of a head in a block, 32
// to a wavefront, and walks the keys (scores, dO V^T, dq); it takes delta first and leaves it for the second, which has 64 or 128 keys of a
// key head in a block and walks the queries of all the heads that share it (scores, dO V^T, dv, dk).  Scores and dO V^T are computed
// in both: seven products instead of five, in place of atomics or of a pass over fp32 parts.  With bf16 operands p and dz are rounded to bf16
// for the products that follow, and the second kernel makes dz of the rounded p; all sums are fp32 and rounded once.  The error against 64
// bits is 0.0027 of the result's size (the packed sequences below), where fp32 throughout and one rounding at the end leave 0.0019.
//
// What bounds them: LDS, which feeds four products a step and of whose rows each is read along and across, and, with uneven sequences, the longest
// walk.  One bf16 sequence of 8192 rows, not causal, 8 heads of 128: the first 413 us (1.0 PFLOP/s), the second 740 (0.74).  24 uneven
// sequences of 8192 rows in all, 16 heads of 128 with 4 key heads, causal: 67 and 114 us alone, 161 to 169 back to back; a third of the second's
// time is its blocks' beginnings and ends, since LDS holds one at a time.
#include "attention_common.hpp"
#include "detag_internal.h"

namespace detag {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRows = 32;                                               // of a panel

// Split: the block's wavefronts have the same 32 queries and 32 keys of a panel each, and add up their parts of dq at the end.
template <class T, int WIDTH, bool Split>
struct QueryCut {
  static constexpr int kPanel = Split ? kWaves * kRows : kRows, kHigh = Split ? 32 : 32 * kWaves;  // keys of a panel, queries of a block
  static constexpr int kStages = 4 * kPanel * WIDTH * int(sizeof(T)) <= 131072 ? 2 : 1;
};

template <class T, int WIDTH, bool Direct, bool Split>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 && !Split ? 2 : 1) void attention_grad_query_kernel(AttentionArgs a, WorkGrid grid) {
  using C = QueryCut<T, WIDTH, Split>;
  using Keys = Panel<T, WIDTH, C::kPanel, kThreads, Direct>;
  constexpr int kHigh = C::kHigh, kStages = C::kStages;
  __shared__ __attribute__((aligned(1024))) char lds_[2 * kStages * Keys::kBytes];
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
    const int first = run.first - run.lo + (Split ? 0 : 32 * wave), query = first + p;
    const int upto = a.causal && run.first - run.lo + kHigh < length ? run.first - run.lo + kHigh : length;
    const int mine = a.causal && first + 32 < length ? first + 32 : first < length ? length : 0;
    const int panels = (upto + C::kPanel - 1) / C::kPanel;
    const int64_t row = int64_t(run.lo) + query;
    const bool there = query < length;

    __syncthreads();  // the block before is done with the panels
    Keys keys, values;
    keys.init(static_cast<const T *>(a.k) + run.lo * a.ldk + kv * a.width, a.ldk, a.width, length);
    values.init(static_cast<const T *>(a.v) + run.lo * a.ldv + kv * a.width, a.ldv, a.width, length);
    auto stage_of = [&](int t) { return lds + t % kStages * 2 * Keys::kBytes; };
    auto request = [&](int t) {
      const uint32_t to = stage_of(t);
      keys.request(to), values.request(to + Keys::kBytes);
    };
    auto deliver = [&](int t) {
      const uint32_t to = stage_of(t);
      keys.deliver(to), values.deliver(to + Keys::kBytes);
    };
    request(0), deliver(0);
    u32x4 q[Keys::kSteps], g[Keys::kSteps];
    load_operand<T, Direct>(q, static_cast<const T *>(a.q) + run.first * a.ldq + head * a.width, a.ldq, query - (run.first - run.lo), there, a.width);
    load_operand<T, Direct>(g, static_cast<const T *>(a.d_o) + run.first * a.ld_do + head * a.width, a.ld_do, query - (run.first - run.lo), there, a.width);
    float delta = 0.f;
    {
      u32x4 o[Keys::kSteps];
      load_operand<T, Direct>(o, static_cast<const T *>(a.o) + run.first * a.ldo + head * a.width, a.ldo, query - (run.first - run.lo), there, a.width);
#pragma unroll
      for (int s = 0; s < Keys::kSteps; ++s)
#pragma unroll
        for (int e = 0; e < Keys::kElems; ++e) delta += element<T>(o[s], e) * element<T>(g[s], e);
    }
    delta += other_half(delta);
    const int64_t at = head * int64_t(a.rows) + row;
    if (there && h == 0 && own == 0) a.delta[at] = delta;
    const float level = there ? a.lse[at] * (1.f / kLn2) : 0.f;  // in powers of two

    f32x16 acc[Keys::kBlocks];
#pragma unroll
    for (int b = 0; b < Keys::kBlocks; ++b) acc[b] = f32x16{};
    // One panel; its stage is a constant, and so are all offsets into LDS (a variable one: 83 us instead of 72).
    auto panel = [&](auto odd_, int t) {
      constexpr int odd = decltype(odd_)::value;
      wait_all();
      wait_lds();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const uint32_t here = lds + odd * 2 * Keys::kBytes;
      const int key0 = t * C::kPanel + 32 * own;
      if (kStages == 2 && key0 >= mine && t + 1 < panels) request(t + 1);
      if (key0 < mine) {
        f32x16 s{}, ds{};
#pragma unroll
        for (int k = 0; k < Keys::kSteps; ++k) {
          if (sizeof(T) == 4 && 2 * k * Keys::kElems >= a.width) break;  // (fp32 products take long)
          s = multiply32<T>(Keys::along(along, here, own, k), q[k], s);
          ds = multiply32<T>(Keys::along(along, here + Keys::kBytes, own, k), g[k], ds);
        }
        if (kStages == 2 && t + 1 < panels) request(t + 1);  // (while the products run)
        u32x4 y[Keys::kGroups][Keys::kBlocks];
#pragma unroll
        for (int j = 0; j < Keys::kGroups; ++j)
#pragma unroll
          for (int c = 0; c < Keys::kBlocks; ++c) y[j][c] = Keys::across(across, here, c, 32 * own, j);
        __builtin_amdgcn_sched_barrier(0);
        const int last = a.causal && there ? query : length - 1;
        const bool all = key0 + kRows <= (a.causal ? first + 1 : length);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float prob = __builtin_amdgcn_exp2f(s[r] * a.scale2 - level);
          ds[r] = prob * (ds[r] - delta);
        }
        if (!all)
#pragma unroll
          for (int r = 0; r < 16; ++r) ds[r] = key0 + 8 * (r / 4) + 4 * h + r % 4 <= last ? ds[r] : 0.f;
#pragma unroll
        for (int j = 0; j < Keys::kGroups; ++j) {
          const u32x4 dz = as_operand<T>(ds, j);
#pragma unroll
          for (int c = 0; c < Keys::kBlocks; ++c) acc[c] = multiply32<T>(y[j][c], dz, acc[c]);
        }
      }
      if (kStages == 1 && t + 1 < panels) {
        wait_lds();
        __builtin_amdgcn_s_barrier();  // all have read the panel
        asm volatile("" ::: "memory");
        request(t + 1);
      }
      if (t + 1 < panels) deliver(t + 1);
    };
    for (int t = 0; t < panels; t += kStages) {
      panel(std::integral_constant<int, 0>{}, t);
      if constexpr (kStages == 2)
        if (t + 1 < panels) panel(std::integral_constant<int, 1>{}, t + 1);
    }
    if constexpr (Split) {  // every wavefront adds up some of the columns
      auto part = [&](int w, int b, int r) {
        return reinterpret_cast<__attribute__((address_space(3))) float *>(lds + (((w * Keys::kBlocks + b) * 16 + r) * 64 + lane) * 4);
      };
      static_assert(kWaves * Keys::kBlocks * 4096 <= 2 * kStages * Keys::kBytes, "the parts fit the panels");
      __syncthreads();  // all have read the last panel
#pragma unroll
      for (int b = 0; b < Keys::kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) *part(wave, b, r) = acc[b][r];
      __syncthreads();
      for (int b = wave; b < Keys::kBlocks; b += kWaves) {
        f32x16 sum[1] = {f32x16{}};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
          for (int r = 0; r < 16; ++r) sum[0][r] += *part(w, b, r);
        if (there) store_row(static_cast<T *>(a.dq) + row * a.ld_dq + head * a.width + 32 * b, sum, a.scale, a.width - 32 * b);
      }
      return;
    }
    if constexpr (Direct) {
      static_assert(Split || kWaves * 32 * WIDTH * sizeof(T) <= 2 * kStages * Keys::kBytes, "the rows fit the panels");
      __syncthreads();  // all have read the last panel
      store_rows(static_cast<T *>(a.dq) + (int64_t(run.lo) + first) * a.ld_dq + head * a.width, a.ld_dq, length - first,
                 lds + wave * 32 * WIDTH * int(sizeof(T)), acc, a.scale, a.width);
    } else if (there) {
      store_row(static_cast<T *>(a.dq) + row * a.ld_dq + head * a.width, acc, a.scale, a.width);
    }
  });
}

// Eight wavefronts in pairs.  The first of a pair takes the scores, the probabilities and dv of 32 keys, the second, a step later, dO V^T, dz
// and dk, with the probabilities that the first has left in LDS (as it multiplied them: of bf16 they are rounded).  The sums of one alone
// leave registers for a panel's fragments to be read before they are needed.  A step is a panel of 32 queries of one of the heads that share
// the key head; the panels of all these heads are taken one after the other.  Two pairs have the same keys and take them in turn, so that the
// longest sequence does not hold up the launch for as long, and join their sums at the end (fp32 heads of more than 64: one, for LDS).  8192
// rows in 24 uneven sequences, 16 heads of 128 with 4 key heads, causal: both sums in one wavefront 217 us, pairs with keys of their own 168,
// this 114.
template <class T, int WIDTH, bool Direct>
struct KeyCut {
  static constexpr int kSplit = sizeof(T) * WIDTH > 256 ? 1 : 2, kKeys = kWaves / kSplit, kHigh = 32 * kKeys;  // keys of a block
  using Queries = Panel<T, WIDTH, kRows, kThreads / kSplit, Direct>;
  // LDS: stages of panels, probabilities as they are multiplied (two steps' of every pair), and a few steps' levels (of every wavefront)
  static constexpr int kPanels = 2 * kSplit * Queries::kBytes, kProb = Queries::kGroups * 1024, kLevel = 2 * kWaves * 256;
  static constexpr int kFit = (163840 - 2 * kWaves * kProb - 4 * kLevel) / kPanels, kStages = kFit < 6 ? kFit : 6;
  static constexpr int kAhead = Direct ? kStages - 2 : 1, kSlots = kAhead <= 2 ? 4 : 8;
  static constexpr int kProbs = kStages * kPanels, kLevels = kProbs + 2 * kWaves * kProb, kLds = kLevels + kSlots * kLevel;
  static_assert(kStages >= 3 && kAhead + 2 <= kSlots && kLds <= 163840, "a step's levels stay until its second wavefronts have read them");
};
template <class T, int WIDTH>
constexpr int kKeysHigh = KeyCut<T, WIDTH, true>::kHigh;

template <class T, int WIDTH, bool Direct>
__global__ __launch_bounds__(2 * kThreads, 2) void attention_grad_key_kernel(AttentionArgs a, WorkGrid grid) {
  using C = KeyCut<T, WIDTH, Direct>;
  using Queries = typename C::Queries;
  constexpr int kStages = C::kStages, kAhead = C::kAhead, kSplit = C::kSplit, kStage = C::kPanels;
  __shared__ __attribute__((aligned(1024))) char lds_[C::kLds];
  const uint32_t lds = uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds_));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, p = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
  const int pair = wave % kWaves, second = wave / kWaves, keys = pair % C::kKeys, split = pair / C::kKeys;
  const int groups = a.heads / a.kv_heads;
  const uint32_t along = Queries::along_base(), across = Queries::across_base();
  for_work(grid, [&](int kv, uint32_t piece) {
    const Run run = run_in_turn(a, C::kHigh, piece, grid.each, false);  // causal: the first runs of a sequence are read by the most queries
    if (run.part < 0) return;
    const int length = run.hi - run.lo, first = run.first - run.lo + 32 * keys, key = first + p;
    const int start = a.causal ? run.first - run.lo : 0;  // first query that reads the block's keys
    const int64_t row = int64_t(run.lo) + key;
    const bool there = key < length;
    const int panels = (length - start + kRows - 1) / kRows, steps = (panels * groups + kSplit - 1) / kSplit;

    __syncthreads();  // the block before is done with LDS
    // The first wavefronts of the pairs that take a panel fetch its queries and their lse, the second ones dO and delta.
    Queries own;
    own.init(second ? static_cast<const T *>(a.d_o) + (int64_t(run.lo) + start) * a.ld_do + int64_t(kv) * groups * a.width
                    : static_cast<const T *>(a.q) + (int64_t(run.lo) + start) * a.ldq + int64_t(kv) * groups * a.width,
             second ? a.ld_do : a.ldq, a.width, length - start);
    const uint64_t from0 = own.from;
    const int64_t left0 = own.left;
    const float *const level0 = (second ? a.delta : a.lse) + int64_t(kv) * groups * a.rows + run.lo + start;
    int next_head = 0, next_panel = 0, next_stage = 0, asked = 0, next_rows;  // rows: of the head from the next panel on, none past the last head
    uint64_t next_level;
    auto on = [&](int &head, int &panel, int by) {
      for (panel += by; panel >= panels; panel -= panels) ++head;
    };
    auto begin = [&] {
      const bool some = next_head < groups;  // or zeros: the loads under way are counted
      const int from = next_panel * kRows;
      next_rows = some ? length - start - from : 0;
      next_level = reinterpret_cast<uint64_t>(level0 + next_head * int64_t(a.rows) + from);
      own.from = from0 + int64_t(next_head) * a.width * int64_t(sizeof(T)), own.left = some ? left0 : 0;
      own.skip(from);
    };
    on(next_head, next_panel, split), begin();
    auto request = [&] {
      load_floats_to_lds(u32x4{uint32_t(next_level), uint32_t(next_level >> 32), uint32_t(next_rows < 64 ? next_rows : 64) * 4u, 0x00020000u},
                         lds + C::kLevels + asked++ % C::kSlots * C::kLevel + wave * 256);
      own.request(lds + next_stage * kStage + (2 * split + second) * Queries::kBytes);
      if (next_panel + kSplit < panels) {
        next_panel += kSplit, next_rows -= kSplit * kRows, next_level += kSplit * kRows * 4;
        own.skip((kSplit - 1) * kRows);
      } else {
        on(next_head, next_panel, kSplit), begin();
      }
    };
    auto deliver = [&] {
      own.deliver(lds + next_stage * kStage + (2 * split + second) * Queries::kBytes);
      next_stage = next_stage + 1 == kStages ? 0 : next_stage + 1;
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (k < steps) request(), deliver();
    u32x4 kv_[Queries::kSteps];
    if (second) load_operand<T, Direct>(kv_, static_cast<const T *>(a.v) + run.first * a.ldv + kv * a.width, a.ldv, 32 * keys + p, there, a.width);
    else load_operand<T, Direct>(kv_, static_cast<const T *>(a.k) + run.first * a.ldk + kv * a.width, a.ldk, 32 * keys + p, there, a.width);
    f32x16 acc[Queries::kBlocks];
#pragma unroll
    for (int b = 0; b < Queries::kBlocks; ++b) acc[b] = f32x16{};
    int panel = 0, head = 0, stage = 0;  // of the wavefront's step
    on(head, panel, split);
    // The last products of a step: fragments y across a panel with z, probabilities or dz.  The second wavefronts do them at the start of their
    // next step, while the first ones read LDS; bf16 fragments are read as soon as the products before have left their registers (fp32 has none for
    // that, and reads each before its product).
    constexpr bool kHeld = sizeof(T) == 2;
    u32x4 y[kHeld ? Queries::kGroups : 1][kHeld ? Queries::kBlocks : 1], z[Queries::kGroups];
    bool pending = false;
    auto get_y = [&](int stage, int j, int c) { return Queries::across(across, lds + stage * kStage + (2 * split + 1 - second) * Queries::kBytes, c, 0, j); };
    auto products = [&](int stage) {
#pragma unroll
      for (int j = 0; j < Queries::kGroups; ++j)
#pragma unroll
        for (int c = 0; c < Queries::kBlocks; ++c) {
          if constexpr (kHeld) acc[c] = multiply32<T>(y[j][c], z[j], acc[c]);
          else acc[c] = multiply32<T>(get_y(stage, j, c), z[j], acc[c]);
        }
    };
    for (int t = 0; t <= steps; ++t) {
      // panel t has arrived; those after it may be under way
      if (Direct && t > 0 && t + kAhead <= steps) wait_loads<(kAhead - 1) * (Queries::kLoads + 1)>();
      else wait_all();
      wait_lds();
      __builtin_amdgcn_s_barrier();  // in all wavefronts, and they are done with the stage that is filled next
      asm volatile("" ::: "memory");
      const bool more = t + kAhead < steps;
      const int query0 = start + panel * kRows;
      if (pending) products(0), pending = false;
      const bool active = t >= second && head < groups && first < length && (!a.causal || query0 + kRows > first);
      if (!active && more) request();
      if (active) {
        const uint32_t probs = lds + C::kProbs + (((t - second) & 1) * kWaves + pair) * C::kProb + lane * 16;
        const uint32_t levels = lds + C::kLevels + (t - second) % C::kSlots * C::kLevel + wave * 256 + 16 * h;
        u32x4 x[Queries::kSteps];
#pragma unroll
        for (int j = 0; j < Queries::kSteps; ++j) x[j] = Queries::along(along, lds + stage * kStage + (2 * split + second) * Queries::kBytes, 0, j);
        __builtin_amdgcn_sched_barrier(0);
        f32x16 s{};
#pragma unroll
        for (int j = 0; j < Queries::kSteps; ++j)
          if (sizeof(T) == 2 || 2 * j * Queries::kElems < a.width) s = multiply32<T>(x[j], kv_[j], s);  // (fp32 products take long)
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kHeld)
#pragma unroll
          for (int j = 0; j < Queries::kGroups; ++j)
#pragma unroll
            for (int c = 0; c < Queries::kBlocks; ++c) y[j][c] = get_y(stage, j, c);
        if (more) request();  // (while the products run)
        f32x4 level[4];
        u32x4 prob[Queries::kGroups];
#pragma unroll
        for (int r = 0; r < 4; ++r) level[r] = read_lds<f32x4>(levels + 32 * r);
        if (second)
#pragma unroll
          for (int j = 0; j < Queries::kGroups; ++j) prob[j] = read_lds<u32x4>(probs + 1024 * j);
        __builtin_amdgcn_sched_barrier(0);
        const bool all = query0 + kRows <= length && (!a.causal || query0 >= first + 31);
        if (second) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = element<T>(prob[r / (16 / Queries::kGroups)], r % (16 / Queries::kGroups)) * (s[r] - level[r / 4][r % 4]);
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] * a.scale2 - level[r / 4][r % 4] * (1.f / kLn2));
        }
        if (!all) {
          int from = query0 + 4 * h, upto = a.causal ? key : 0;
          asm volatile("" : "+v"(from), "+v"(upto));  // (as in store_rows)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int at = from + 8 * (r / 4) + r % 4;
            s[r] = at < length && at >= upto ? s[r] : 0.f;
          }
        }
#pragma unroll
        for (int j = 0; j < Queries::kGroups; ++j) z[j] = as_operand<T>(s, j);
        if (!second)
#pragma unroll
          for (int j = 0; j < Queries::kGroups; ++j) *reinterpret_cast<__attribute__((address_space(3))) u32x4 *>(probs + 1024 * j) = z[j];
        if (kHeld && second) pending = true;
        else products(stage);
      }
      if (t >= second) {
        on(head, panel, kSplit);
        stage = stage + 1 == kStages ? 0 : stage + 1;
      }
      if (more) deliver();
    }
    if (pending) products(0);
    if constexpr (kSplit > 1) {
      static_assert(kSplit == 1 || (kSplit - 1) * C::kKeys * 2 * Queries::kBlocks * 4096 <= C::kProbs, "the parts fit the panels");
      int at = lane * 16;
      asm volatile("" : "+v"(at));  // (as in store_rows)
      auto part = [&](int b, int r) {  // four registers
        return reinterpret_cast<__attribute__((address_space(3))) f32x4 *>(lds + (((second * C::kKeys + keys) * Queries::kBlocks + b) * 16 + r) * 256 + at);
      };
      __syncthreads();  // all have read the last panels
      if (split)
#pragma unroll
        for (int b = 0; b < Queries::kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 16; r += 4) *part(b, r) = f32x4{acc[b][r], acc[b][r + 1], acc[b][r + 2], acc[b][r + 3]};
      __syncthreads();
      if (split) return;
#pragma unroll
      for (int b = 0; b < Queries::kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const f32x4 other = *part(b, r);
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[b][r + k] += other[k];
        }
    }
    T *const to = static_cast<T *>(second ? a.dk : a.dv) + kv * a.width;
    const int64_t pitch = second ? a.ld_dk : a.ld_dv;
    const float factor = second ? a.scale : 1.f;
    if constexpr (Direct) {
      constexpr int kMine = 32 * WIDTH * int(sizeof(T)), kParts = (kSplit - 1) * C::kKeys * 2 * Queries::kBlocks * 4096;
      static_assert(kParts + 2 * C::kKeys * kMine <= C::kLds, "the rows fit beside the parts");
      if constexpr (kSplit == 1) __syncthreads();  // all have read the last panels
      store_rows(to + (int64_t(run.lo) + first) * pitch, pitch, length - first, lds + kParts + (second * C::kKeys + keys) * kMine, acc, factor, a.width);
    } else if (there) {
      store_row(to + row * pitch, acc, factor, a.width);
    }
  });
}

template <class T>
bool attention_grad_direct(const AttentionArgs &a) {
  auto direct = [&](const void *p, int64_t pitch) { return panels_direct(p, pitch, a.width, sizeof(T)); };
  return direct(a.q, a.ldq) && direct(a.k, a.ldk) && direct(a.v, a.ldv) && direct(a.o, a.ldo) && direct(a.d_o, a.ld_do);
}

template <class T, int WIDTH, bool Split>
int launch_queries(const AttentionArgs &a, hipStream_t st) {
  const WorkGrid grid = work_grid(a.kv_heads, part_runs(a.rows, a.parts, QueryCut<T, WIDTH, Split>::kHigh) * (a.heads / a.kv_heads));
  if (attention_grad_direct<T>(a)) attention_grad_query_kernel<T, WIDTH, true, Split><<<work_blocks(grid), kThreads, 0, st>>>(a, grid);
  else attention_grad_query_kernel<T, WIDTH, false, Split><<<work_blocks(grid), kThreads, 0, st>>>(a, grid);
  return hip_rc(hipGetLastError());
}

template <class T, int WIDTH>
int attention_grad(const AttentionArgs &a, hipStream_t st) {
  const WorkGrid by_key = work_grid(a.kv_heads, part_runs(a.rows, a.parts, kKeysHigh<T, WIDTH>));
  const bool split = attention_splits(a, sizeof(T) == 2);
  if (const int rc = split ? launch_queries<T, WIDTH, true>(a, st) : launch_queries<T, WIDTH, false>(a, st)) return rc;
  if (attention_grad_direct<T>(a)) attention_grad_key_kernel<T, WIDTH, true><<<work_blocks(by_key), 2 * kThreads, 0, st>>>(a, by_key);
  else attention_grad_key_kernel<T, WIDTH, false><<<work_blocks(by_key), 2 * kThreads, 0, st>>>(a, by_key);
  return hip_rc(hipGetLastError());
}

}  // namespace

int launch_attention_grad(const AttentionArgs &a, bool bf16, void *stream) {
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (bf16) return a.width <= 64 ? attention_grad<bf16_t, 64>(a, st) : attention_grad<bf16_t, 128>(a, st);
  return a.width <= 64 ? attention_grad<float, 64>(a, st) : attention_grad<float, 128>(a, st);
}

}  // namespace detag
