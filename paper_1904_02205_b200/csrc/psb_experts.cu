// Routing of rows to experts, and the weighted sum of what the experts give back.
//
// route: a row's experts are those of the top_k largest select values.  Near the border two values may differ by less
// than fp32 resolves, and a row sent to another expert is a wrong answer, so the comparison is exact: without a bias the
// scores are monotone in the logits and the logits themselves are compared; otherwise fp32 values decide wherever
// they are further apart than their error bound (kRound), and the row is done again in 64 bits where they are not (equal
// logits with equal biases are equal, and need no second look).
// The order of the choices is a counting sort: blocks of consecutive rows count their choices per expert, a second launch
// adds up the counts of the blocks before each (from 37741 rows on a launch between them does) and places the choices, the rank inside
// a block being the number of earlier rows that chose the same expert (bit masks over the block's rows).  Nothing depends on the order of atomics.
// Up to 64 rows one block does all three.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "psb_common.cuh"

namespace psb {

namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;
// (16384 rows over 256 experts in groups, unsorted: 28 us with 768 threads, 30 with 1024 of 64 registers, 31 to 38 with 512; over 512
// experts 25 us with 512 threads, 41 with 256; 4096 over 1024 experts 15.5 with either, and the scratch of 16 warps with as many groups
// as experts would pass a block's shared memory)
template <int EL> constexpr uint32_t kRouteThreads = EL <= 8 ? 768u : EL == 16 ? 512u : 256u;
constexpr uint32_t kMaxBlockRows = 1024;   // rows of a counting block: 32 words of a bit mask
// The most dynamic shared memory of a launch, which every launch sets as its kernel's limit: the limit belongs to a kernel on a device, not to a
// context, and host threads that set each call's own size would lower it under one another's launches.
constexpr int kMaxSmem = 160 * 1024;
template <int EL> constexpr uint32_t kMostRouteSmem = kRouteThreads<EL> / 32u * (2u * 32u * EL) * 8u + 3u * 32u * EL * 4u;   // (as many groups as experts)
static_assert(kMostRouteSmem<8> <= kMaxSmem && kMostRouteSmem<16> <= kMaxSmem && kMostRouteSmem<32> <= kMaxSmem, "scratch of the warps");
static_assert(1024u * (1u + kMaxBlockRows / 32u) * 4u <= kMaxSmem, "bits of a block's rows, counts in words");
static_assert(1024u * (1u + 8u) * 4u + 2u * 4u * 1024u * 4u <= kMaxSmem, "bits of a block's rows, counts in bytes");
// Two fp32 select values are told apart if they differ by more than unit + kRound * (|v| + |w|).  The bounds that CUDA publishes are 2 + 1.173 |z| units
// in the last place for __expf(z) and 2 for __fdividef, a unit being at most 2^-23 of the number; sums and differences round to half a unit.
// A sigmoid p is off by p (1 - p) of exp's error, p 2^-24 of the sum's and the quotient's: 2.99e-7 at most.  Two values, hence twice.
// A softmax, in parts of the row's largest score: exp and its argument's rounding are off by 2.4e-7 at most (at the top; e^-d (2.4 + 2 d) 1e-7 falls), the
// quotient by 2.4e-7, twice for two values.  The sum's error is common to both values and moves them apart by that part of their difference,
// hence once: the mean of exp's errors by scores, 2.4e-7 + 2e-7 d n e^-d / (1 + n e^-d) for n scores of e^-d beside the top (d times its quotient is 3.4 at
// most for 256 experts, 4.5 for 1024), and the roundings of `el` numbers a lane and five levels of lanes.  In all 1.9e-6 for 32 experts, 2.7e-6
// for 256, 4.3e-6 for 1024, where softmax_unit is 2.3e-6, 3.1e-6 and 6e-6.  The bias rounds once, 2^-24 of the value.
constexpr float kSigmoidUnit = 6e-7f, kRound = 1.2e-7f;
__host__ __device__ constexpr float softmax_unit(int el) { return 2.0f * (8e-7f + 6e-8f * (float)(el + 5)); }

struct RouteArgs {
  const void* logits;
  const float* bias;
  const uint8_t* mask;
  uint32_t in_dtype, sigmoid, tokens, experts, top_k, groups, top_groups, group_best, renormalise;
  float scaling;
  uint64_t logit_stride;
  int32_t *ids, *offsets, *order, *slot;
  float* weights;
  uint32_t* counts;        // [blocks + 1][experts]
  uint32_t block_rows, blocks;
  uint32_t alone;            // one block has all rows and places them itself
  uint32_t wide;             // rows of logits start at multiples of 16 bytes
  uint32_t groups_of_counts; // counts are bytes, and so many threads add up the counts of four experts; 0: words, added up by scan_kernel
  uint32_t lanes_per_group;  // a power of two where groups are the experts of whole lanes, else 0
};

__host__ __device__ __forceinline__ uint32_t round_up4(uint32_t n) { return (n + 3u) & ~3u; }

// Monotone map of fp32 numbers onto words, kNone below all of them; and of fp64 numbers, 0 below all of them.
constexpr int kNone = (int)0x80000000;
__device__ __forceinline__ int key_of(float v) {
  const int u = __float_as_int(v);
  return u ^ ((u >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float value_of(int key) { return __int_as_float(key ^ ((key >> 31) & 0x7FFFFFFF)); }
__device__ __forceinline__ unsigned long long key_of(double v) {
  const unsigned long long u = (unsigned long long)__double_as_longlong(v);
  return (u >> 63) ? ~u : (u | (1ull << 63));
}
__device__ __forceinline__ double value_of(unsigned long long key) {
  return __longlong_as_double((long long)((key >> 63) ? (key & ~(1ull << 63)) : ~key));
}
__device__ __forceinline__ int warp_max(int v) { return __reduce_max_sync(kAll, v); }
__device__ __forceinline__ unsigned long long warp_max(unsigned long long v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const unsigned long long o = __shfl_xor_sync(kAll, v, d);
    v = o > v ? o : v;
  }
  return v;
}
template <typename F> __device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  return v;
}

__device__ __forceinline__ float load_logit(const RouteArgs& a, uint64_t at) {
  if (a.in_dtype == PSB_DT_F32) return ((const float*)a.logits)[at];
  if (a.in_dtype == PSB_DT_BF16) return __bfloat162float(((const __nv_bfloat16*)a.logits)[at]);
  return __half2float(((const __half*)a.logits)[at]);
}

// A logit as it counts: NaN where the expert is not available.
__device__ __forceinline__ float clean(float v) { return v == INFINITY ? 3.402823466e38f : v == -INFINITY ? NAN : v; }
__device__ __forceinline__ float load_clean(const RouteArgs& a, uint64_t at) { return clean(load_logit(a, at)); }

// The lane's logits, experts lane * EL ...; NaN where there is no such expert or it is not available.
template <int EL>
__device__ __forceinline__ void load_logits(const RouteArgs& a, uint32_t t, uint32_t lane, float (&x)[EL]) {
  const uint32_t e0 = lane * EL;
  const uint64_t at = (uint64_t)t * a.logit_stride + e0;
  const bool whole = e0 + EL <= a.experts;
  if (EL >= 4 && a.wide && whole && a.in_dtype == PSB_DT_F32) {
#pragma unroll
    for (int i = 0; i < EL / 4; ++i) {
      const float4 w = *reinterpret_cast<const float4*>((const float*)a.logits + at + 4 * i);
      x[4 * i] = w.x;
      x[4 * i + 1] = w.y;
      x[(4 * i + 2) % EL] = w.z;
      x[(4 * i + 3) % EL] = w.w;
    }
  } else if (EL >= 4 && a.wide && whole) {
#pragma unroll
    for (int i = 0; i < EL / 4; ++i) {
      const uint2 w = *reinterpret_cast<const uint2*>((const uint16_t*)a.logits + at + 4 * i);
      const uint32_t h[4] = {w.x & 0xFFFFu, w.x >> 16, w.y & 0xFFFFu, w.y >> 16};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x[(4 * i + j) % EL] = a.in_dtype == PSB_DT_BF16 ? __uint_as_float(h[j] << 16) : __half2float(__ushort_as_half((uint16_t)h[j]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < EL; ++i) x[i] = e0 + i < a.experts ? load_logit(a, at + i) : NAN;
  }
#pragma unroll
  for (int i = 0; i < EL; ++i) x[i] = clean(x[i]);
}

// Two experts of a row, e chosen before o by fp32 values: 1 if that is right, -1 if the other way round is, 0 if it takes the whole row.
__device__ __noinline__ int exact_order(const RouteArgs& a, float xmax, uint32_t t, uint32_t e, uint32_t o) {
  const uint64_t row = (uint64_t)t * a.logit_stride;
  const float x = load_clean(a, row + e), y = load_clean(a, row + o);
  const float b = a.bias ? __ldca(a.bias + e) : 0.0f, c = a.bias ? __ldca(a.bias + o) : 0.0f;
  const int by_index = e < o ? 1 : -1;
  if (b == c && x == y) return by_index;
  if (!a.sigmoid) {
    if (a.bias) return 0;
    // The scores are monotone in the logits, but in 64 bits they may be equal (0 from 745 below the largest logit on; arguments of exp that round to
    // the same), and then the index counts.  exp of more than -700, divided by at most 1024, is a normal number, its argument is off by
    // 2^-44 at most and the score by as much: logits that are 1e-9 apart have different scores.
    const int by_logit = x > y ? 1 : -1;
    const double low = (double)fminf(x, y), high = (double)fmaxf(x, y);
    return by_logit == by_index || (low - (double)xmax > -700.0 && high - low > 1e-9) ? by_logit : 0;
  }
  if (!a.bias && x > y && by_index > 0) return 1;
  double v[2];
#pragma unroll 1
  for (int i = 0; i < 2; ++i) v[i] = 1.0 / (1.0 + exp(-(double)(i ? y : x))) + (double)(i ? c : b);
  return v[0] > v[1] ? 1 : v[0] < v[1] ? -1 : by_index;
}

// The two largest keys of a run of experts, put together with those of another run.
template <typename Key>
__device__ __forceinline__ void merge_best(Key& first, Key& second, Key f, Key s) {
  const Key low = f < first ? f : first;
  first = f > first ? f : first;
  second = s > second ? s : second;
  second = low > second ? low : second;
}

// The choices of one row, by a warp; lane l holds experts l * EL ...  Lane j < top_k receives choice j (id -1: none).
// Returns whether the comparisons were certain (if not: choose_exactly).
template <int EL>
__device__ __forceinline__ bool choose(const RouteArgs& a, const float (&x)[EL], const float (&bias)[EL], float xmax, uint32_t t,
                                       uint32_t lane, int* scratch, int& my_id) {
  const bool by_logit = !a.bias && a.groups == 1u;      // scores are monotone in the logits
  int key[EL];
  bool sure = true;
  float unit = kSigmoidUnit;
  if (by_logit) {
#pragma unroll
    for (int i = 0; i < EL; ++i) key[i] = x[i] == x[i] ? key_of(x[i] + 0.0f) : kNone;     // (-0 and 0 are equal)
  } else {
    float p[EL];
    if (a.sigmoid) {
#pragma unroll
      for (int i = 0; i < EL; ++i) p[i] = __fdividef(1.0f, 1.0f + __expf(-x[i]));
    } else {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < EL; ++i) {
        p[i] = __expf(x[i] - xmax);
        sum += x[i] == x[i] ? p[i] : 0.0f;
      }
      sum = warp_sum(sum);
      unit = softmax_unit(EL) / sum;      // (the largest score is 1 / sum)
#pragma unroll
      for (int i = 0; i < EL; ++i) p[i] = __fdividef(p[i], sum);
    }
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const float sel = p[i] + bias[i];         // (NaN where x is)
      key[i] = sel == sel ? key_of(sel + 0.0f) : kNone;
    }
    if (a.groups > 1u) {
      const uint32_t size = a.experts / a.groups;
      uint32_t stay = 0;       // bit i: my expert i stays
      if (a.lanes_per_group) {
        // a group is the experts of 1, 2, 4 ... lanes: every lane learns its group's strength
        int first = kNone, second = kNone;
#pragma unroll
        for (int i = 0; i < EL; ++i) merge_best(first, second, key[i], kNone);
        for (uint32_t d = 1; d < a.lanes_per_group; d <<= 1) {
          const int f = __shfl_xor_sync(kAll, first, (int)d), s = __shfl_xor_sync(kAll, second, (int)d);
          merge_best(first, second, f, s);
        }
        const bool two = second != kNone && a.group_best > 1u;
        const float v1 = value_of(first), v2 = two ? value_of(second) : 0.0f;
        const uint32_t head = lane & ~(a.lanes_per_group - 1u);
        const bool real = lane < a.groups * a.lanes_per_group;
        const int mine = first == kNone || !real ? kNone : key_of(v1 + v2);
        uint32_t before = 0;
        for (uint32_t from = 0; from < a.groups * a.lanes_per_group; from += a.lanes_per_group) {
          const int k = __shfl_sync(kAll, mine, (int)from);
          before += (k > mine || (k == mine && from < head)) ? 1u : 0u;
        }
        stay = before < a.top_groups ? 0xFFFFFFFFu : 0u;
        if (a.top_groups < a.groups) {
          // the weakest group that stays against the strongest that does not
          const int in = ~warp_max(real && stay ? ~mine : kNone), out = warp_max(real && !stay ? mine : kNone);
          const float far = value_of(warp_max(mine != kNone ? key_of(fabsf(v1) + fabsf(v2)) : 0));
          if (in != kNone && out != kNone) sure = value_of(in) - value_of(out) > 2.0f * unit + 4.0f * kRound * far;
        }
      } else {
        // strengths through shared memory: lane g takes groups g, g + 32, ...
        int* all = scratch;                                    // [experts]
#pragma unroll
        for (int i = 0; i < EL; ++i)
          if (lane * EL + i < a.experts) all[lane * EL + i] = key[i];
        __syncwarp();
        int* group = all + a.experts;                          // [groups]
        float* size_of = reinterpret_cast<float*>(group + a.groups);   // [groups] magnitudes behind the strengths
        for (uint32_t g = lane; g < a.groups; g += 32u) {
          int first = kNone, second = kNone;
          for (uint32_t j = 0; j < size; ++j) merge_best(first, second, all[g * size + j], kNone);
          const bool two = second != kNone && a.group_best > 1u;
          const float v1 = value_of(first), v2 = two ? value_of(second) : 0.0f;
          group[g] = first == kNone ? kNone : key_of(v1 + v2 + 0.0f);
          size_of[g] = fabsf(v1) + fabsf(v2);
        }
        __syncwarp();
        // a group stays if fewer than top_groups are stronger, or as strong and before it
        for (uint32_t g0 = 0; g0 < a.groups; g0 += 32u) {
          const uint32_t g = g0 + lane;
          const int mine = g < a.groups ? group[g] : kNone;
          uint32_t before = 0;
          for (uint32_t o = 0; o < a.groups; ++o) {
            const int k = group[o];
            before += (k > mine || (k == mine && o < g)) ? 1u : 0u;
            if (o != g && mine != kNone && k != kNone)
              sure = sure && fabsf(value_of(k) - value_of(mine)) > 2.0f * unit + 2.0f * kRound * (size_of[g] + size_of[o]);
          }
          const uint32_t in = __ballot_sync(kAll, g < a.groups && before < a.top_groups);
#pragma unroll
          for (int i = 0; i < EL; ++i) {
            const uint32_t mg = min(lane * EL + i, a.experts - 1u) / size;
            if (mg >= g0 && mg < g0 + 32u && ((in >> (mg - g0)) & 1u)) stay |= 1u << i;
          }
        }
        __syncwarp();
      }
#pragma unroll
      for (int i = 0; i < EL; ++i)
        if (!((stay >> i) & 1u)) key[i] = kNone;
    }
  }
  // the lane's two best; the third is looked for only where both have been taken
  int best = kNone, next = kNone;
  uint32_t at = 0, next_at = 0;
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    if (key[i] > best) { next = best; next_at = at; best = key[i]; at = (uint32_t)i; }
    else if (key[i] > next) { next = key[i]; next_at = (uint32_t)i; }
  }
  uint32_t taken = 0;          // bit i: my expert i
  my_id = -1;
  int my_key = kNone;
  // two rounds more than there are choices: is the last choice certain against the first that is left out
  const uint32_t rounds = a.top_k + (by_logit || a.top_k > 30u ? 0u : 2u);
  for (uint32_t j = 0; j < rounds; ++j) {
    const int top = warp_max(best);
    if (top == kNone) break;
    const uint32_t from = (uint32_t)__ffs((int)__ballot_sync(kAll, best == top)) - 1u;     // the lowest lane, the lowest expert
    const uint32_t id = from * EL + __shfl_sync(kAll, at, (int)from);
    if (lane == j) { my_id = (int)id; my_key = top; }
    if (lane == from) {
      taken |= 1u << at;
      best = next;
      at = next_at;
      next = kNone;
      if (best == kNone && EL > 2) {
#pragma unroll
        for (int i = 0; i < EL; ++i)
          if (!((taken >> i) & 1u) && key[i] > best) { best = key[i]; at = (uint32_t)i; }
      }
    }
  }
  if (!by_logit) {
    // each choice against the next
    const int other = __shfl_down_sync(kAll, my_key, 1), other_id = __shfl_down_sync(kAll, my_id, 1);
    const float v = value_of(my_key), w = value_of(other);
    const bool pair = lane < 31u && my_id >= 0 && other_id >= 0 && lane <= a.top_k;
    const uint32_t doubts = __ballot_sync(kAll, pair && !(v - w > unit + kRound * (fabsf(v) + fabsf(w))));
    if (doubts) {
      // Pairs that are right as they stand settle everything between the first and the last of them.  One that is not is turned round
      // if its neighbours are certain.  Two in doubt at the border: others behind them may be as close, so the whole row is done again.
      bool swap = false;
      if (((doubts >> lane) & 1u) && lane < a.top_k) {
        const int order = exact_order(a, xmax, t, (uint32_t)my_id, (uint32_t)other_id);
        swap = order < 0;
        const bool border = lane == a.top_k - 1u && ((doubts >> lane >> 1) & 1u);
        if (order == 0 || border || (swap && (((doubts >> 1) | (doubts << 1)) >> lane & 1u))) sure = false;
      }
      const uint32_t swaps = __ballot_sync(kAll, swap);
      const int above = __shfl_up_sync(kAll, my_id, 1);
      if ((swaps >> lane) & 1u) my_id = other_id;
      else if (lane && ((swaps >> (lane - 1u)) & 1u)) my_id = above;
    }
    if (a.top_k > 30u) sure = false;           // (no lanes for those that are left out)
  }
  if (lane >= a.top_k) my_id = -1;
  return __all_sync(kAll, sure);
}

// The choices of one row in 64 bits, from memory again.  The rare case: its code is met cold, line by line, by the one warp
// that needs it, while the other warps of the launch finish, so it is short (loops through shared memory, two copies of exp
// and not one for each of the lane's experts: 30 us of a launch otherwise).  `keys`: [experts + groups].
__device__ __noinline__ int choose_exactly(const RouteArgs& a, float xmax, uint32_t t, uint32_t lane, unsigned long long* keys) {
  typedef unsigned long long Key;
  const uint64_t row = (uint64_t)t * a.logit_stride;
  double sum = 0.0;
  __syncwarp();           // (the groups' strengths of the 32-bit choice have been read)
  // (the loads together; the lane's own places)
#pragma unroll 4
  for (uint32_t e = lane; e < a.experts; e += 32u) keys[e] = (Key)__float_as_uint(load_clean(a, row + e));
#pragma unroll 1
  for (uint32_t pass = a.sigmoid ? 1u : 0u; pass < 2u; ++pass) {
#pragma unroll 2
    for (uint32_t e = lane; e < a.experts; e += 32u) {
      const double x = (double)__uint_as_float((uint32_t)keys[e]), v = exp(a.sigmoid ? -x : x - (double)xmax);
      if (pass == 0u) {
        if (x == x) sum += v;
      } else {
        const double sel = (a.sigmoid ? 1.0 : v) / (a.sigmoid ? 1.0 + v : sum) + (a.bias ? (double)__ldca(a.bias + e) : 0.0);
        keys[e] = x == x && sel == sel ? key_of(sel + 0.0) : (Key)0;
      }
    }
    if (pass == 0u) sum = warp_sum(sum);
  }
  __syncwarp();
  const uint32_t size = a.experts / a.groups;
  if (a.groups > 1u) {
    Key* group = keys + a.experts;
#pragma unroll 1
    for (uint32_t g = lane; g < a.groups; g += 32u) {
      Key first = 0, second = 0;
#pragma unroll 4
      for (uint32_t j = 0; j < size; ++j) merge_best(first, second, keys[g * size + j], (Key)0);
      group[g] = !first ? (Key)0 : key_of((second && a.group_best > 1u ? value_of(first) + value_of(second) : value_of(first)) + 0.0);
    }
    __syncwarp();
#pragma unroll 1
    for (uint32_t g = lane; g < a.groups; g += 32u) {
      uint32_t before = 0;
#pragma unroll 4
      for (uint32_t o = 0; o < a.groups; ++o) before += (group[o] > group[g] || (group[o] == group[g] && o < g)) ? 1u : 0u;
      if (before >= a.top_groups) {
#pragma unroll 4
        for (uint32_t j = 0; j < size; ++j) keys[g * size + j] = 0;
      }
    }
    __syncwarp();
  }
  int id = -1;
#pragma unroll 1
  for (uint32_t j = 0; j < a.top_k; ++j) {
    Key best = 0;
    uint32_t at = 0xFFFFFFFFu;
#pragma unroll 4
    for (uint32_t e = lane; e < a.experts; e += 32u)
      if (keys[e] > best) { best = keys[e]; at = e; }
    const Key top = warp_max(best);
    if (!top) break;
    const uint32_t e = __reduce_min_sync(kAll, best == top ? at : 0xFFFFFFFFu);
    if (lane == j) id = (int)e;
    if (e % 32u == lane) keys[e] = 0;
    __syncwarp();
  }
  return id;
}

// One row: its choices and their weights, by a warp.
template <int EL>
__device__ __forceinline__ void route_row(const RouteArgs& a, uint32_t t, const float (&x)[EL], const float (&bias)[EL], uint32_t lane,
                                          double* scratch, int& id, float& w) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < EL; ++i) m = fmaxf(m, x[i]);      // (NaN counts as absent)
  m = value_of(warp_max(key_of(m)));
  if (!choose<EL>(a, x, bias, m, t, lane, reinterpret_cast<int*>(scratch), id))
    id = choose_exactly(a, m, t, lane, reinterpret_cast<unsigned long long*>(scratch));
  const bool mine = id >= 0;
  const float logit = mine ? load_clean(a, (uint64_t)t * a.logit_stride + (uint32_t)id) : 0.0f;
  float s = 0.0f;
  if (a.renormalise) {
    // ratios of scores, without under- or overflow: softmax exp(x - top) and sigmoid
    // exp(min(x, 0) - min(top, 0)) / (1 + exp(-|x|)) up to factors that the choices share
    const float top = value_of(warp_max(mine ? key_of(logit) : kNone));
    if (mine) s = a.sigmoid ? expf(fminf(logit, 0.0f) - fminf(top, 0.0f)) / (1.0f + expf(-fabsf(logit))) : expf(logit - top);
    const float sum = warp_sum(s);
    s = mine ? s / sum : 0.0f;
  } else if (a.sigmoid) {
    s = mine ? (logit >= 0.0f ? 1.0f / (1.0f + expf(-logit)) : expf(logit) / (1.0f + expf(logit))) : 0.0f;
  } else {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < EL; ++i) sum += x[i] == x[i] ? expf(x[i] - m) : 0.0f;
    sum = warp_sum(sum);
    s = mine ? expf(logit - m) / sum : 0.0f;
  }
  w = mine ? s * a.scaling : 0.0f;
}

// The choices of rows [lo, hi) are placed in two steps, so that other work may lie between them.  Shared memory: bits
// [experts][words], zeros at first, a bit for each of the rows; place [experts], the first place of each expert for these rows.
// `id`: the thread's first choice.
__device__ __forceinline__ int first_choice(const RouteArgs& a, uint32_t lo, uint32_t hi) {
  return threadIdx.x < (hi - lo) * a.top_k ? __ldcg(a.ids + (size_t)lo * a.top_k + threadIdx.x) : -1;
}
__device__ __forceinline__ void mark_choices(const RouteArgs& a, uint32_t lo, uint32_t hi, int id, uint32_t* bits, uint32_t words) {
  const uint32_t choices = (hi - lo) * a.top_k;
  for (uint32_t i = threadIdx.x; i < choices; i += blockDim.x) {
    if (i != threadIdx.x) id = __ldcg(a.ids + (size_t)lo * a.top_k + i);
    const uint32_t r = i / a.top_k;
    if (id >= 0) atomicOr(&bits[(uint32_t)id * words + r / 32u], 1u << (r & 31u));
  }
}
__device__ __forceinline__ void place_choices(const RouteArgs& a, uint32_t lo, uint32_t hi, int id, const uint32_t* place, const uint32_t* bits,
                                              uint32_t words) {
  const uint32_t choices = (hi - lo) * a.top_k;
  for (uint32_t i = threadIdx.x; i < choices; i += blockDim.x) {
    if (i != threadIdx.x) id = __ldcg(a.ids + (size_t)lo * a.top_k + i);
    const uint32_t r = i / a.top_k;
    int at = -1;
    if (id >= 0) {
      uint32_t rank = __popc(bits[(uint32_t)id * words + r / 32u] & ((1u << (r & 31u)) - 1u));
      for (uint32_t w = 0; w < r / 32u; ++w) rank += __popc(bits[(uint32_t)id * words + w]);
      at = (int)(place[id] + rank);
      a.order[at] = (int32_t)(lo + r);
    }
    a.slot[(size_t)lo * a.top_k + i] = at;
  }
}

// Sums before each of up to blockDim.x numbers; all threads take part.  `total`: their sum.
__device__ __forceinline__ uint32_t sum_before(uint32_t mine, uint32_t* warp_total, uint32_t& total) {
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  uint32_t up = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t o = __shfl_up_sync(kAll, up, d);
    if (lane >= (uint32_t)d) up += o;
  }
  if (lane == 31u) warp_total[warp] = up;
  __syncthreads();
  uint32_t base = 0;
  total = 0;
  for (uint32_t w = 0; w < blockDim.x / 32u; ++w) {
    if (w < warp) base += warp_total[w];
    total += warp_total[w];
  }
  __syncthreads();
  return base + up - mine;
}

// Rows of a block one after another by its warps.  Dynamic shared memory: counts [experts]; where one block has all
// rows, the bits of place_choices; then per warp the scratch of groups.
template <int EL>
__global__ void __launch_bounds__(kRouteThreads<EL>) route_kernel(const RouteArgs a) {
  pdl_prologue();
  extern __shared__ __align__(16) unsigned char route_smem[];
  __shared__ uint32_t warp_total[32];
  uint32_t* hist = reinterpret_cast<uint32_t*>(route_smem);
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, words = (a.block_rows + 31u) / 32u;
  const uint32_t ints = a.experts * (a.alone ? 1u + words : 1u);
  double* scratch = reinterpret_cast<double*>(route_smem + ((ints * 4u + 15u) & ~15u)) + (size_t)warp * (a.experts + a.groups);
  for (uint32_t e = threadIdx.x; e < ints; e += blockDim.x) hist[e] = 0u;
  float bias[EL];
#pragma unroll
  // (through L1: every warp of the machine asking L2 for the same few lines took 20 us)
  for (int i = 0; i < EL; ++i) bias[i] = a.bias && lane * EL + i < a.experts ? __ldca(a.bias + lane * EL + i) : 0.0f;
  __syncthreads();
  const uint32_t lo = blockIdx.x * a.block_rows, hi = min(lo + a.block_rows, a.tokens), step = blockDim.x >> 5;
  float x[EL];
  if (lo + warp < hi) load_logits<EL>(a, lo + warp, lane, x);
  for (uint32_t t = lo + warp; t < hi; t += step) {
    const bool on = !a.mask || a.mask[t] != 0u;
    int id = -1;
    float w = 0.0f, next[EL];
    if (t + step < hi) load_logits<EL>(a, t + step, lane, next);
    if (on) route_row<EL>(a, t, x, bias, lane, scratch, id, w);
#pragma unroll
    for (int i = 0; i < EL; ++i) x[i] = next[i];
    if (lane < a.top_k) {
      a.ids[(size_t)t * a.top_k + lane] = id;
      a.weights[(size_t)t * a.top_k + lane] = w;
      if (id >= 0) atomicAdd(&hist[id], 1u);
    }
  }
  if (!a.order) return;
  __syncthreads();
  if (!a.alone) {
    for (uint32_t e = threadIdx.x; e < a.experts; e += blockDim.x) {
      if (a.groups_of_counts) ((uint8_t*)a.counts)[(size_t)blockIdx.x * round_up4(a.experts) + e] = (uint8_t)hist[e];
      else a.counts[(size_t)blockIdx.x * a.experts + e] = hist[e];
    }
    return;
  }
  uint32_t carry = 0;
  for (uint32_t e0 = 0; e0 < a.experts; e0 += blockDim.x) {
    const uint32_t e = e0 + threadIdx.x;
    uint32_t total;
    const uint32_t before = carry + sum_before(e < a.experts ? hist[e] : 0u, warp_total, total);
    if (e < a.experts) {
      hist[e] = before;
      a.offsets[e] = (int32_t)before;
    }
    carry += total;
  }
  if (threadIdx.x == 0u) a.offsets[a.experts] = (int32_t)carry;
  __syncthreads();
  const int id = first_choice(a, lo, hi);
  mark_choices(a, lo, hi, id, hist + a.experts, words);
  __syncthreads();
  place_choices(a, lo, hi, id, hist, hist + a.experts, words);
  for (uint32_t i = carry + threadIdx.x; i < a.tokens * a.top_k; i += blockDim.x) a.order[i] = -1;
}

// Turns the counts of the blocks into the numbers of rows before each block, expert by expert, and adds the sums as one row more.
// 32 experts a block of threads, the counting blocks dealt out to 32 threads each.  (Where counts are words: every placing block adding
// them up took 12 us, 148 SMs on the same 150 KB.)
__global__ void __launch_bounds__(1024) scan_kernel(const RouteArgs a) {
  pdl_prologue();
  __shared__ uint32_t sums[32][33];
  const uint32_t x = threadIdx.x & 31u, y = threadIdx.x >> 5, e = blockIdx.x * 32u + x;
  const uint32_t lo = a.blocks * y / 32u, hi = a.blocks * (y + 1u) / 32u;
  uint32_t sum = 0;
  if (e < a.experts) {
#pragma unroll 8
    for (uint32_t b = lo; b < hi; ++b) sum += __ldcg(a.counts + (size_t)b * a.experts + e);
  }
  sums[y][x] = sum;
  __syncthreads();
  if (e >= a.experts) return;
  uint32_t before = 0;
  for (uint32_t q = 0; q < y; ++q) before += sums[q][x];
#pragma unroll 8
  for (uint32_t b = lo; b < hi; ++b) {
    uint32_t* at = a.counts + (size_t)b * a.experts + e;
    const uint32_t c = __ldcg(at);
    *at = before;
    before += c;
  }
  if (y == 31u) a.counts[(size_t)a.blocks * a.experts + e] = before;
}

// Places the choices of each block.  Dynamic shared memory: places [experts], the bits of place_choices, sums of bytes
// [groups_of_counts][2][experts].
__global__ void __launch_bounds__(1024) order_kernel(const RouteArgs a) {
  pdl_prologue();
  extern __shared__ uint32_t order_smem[];
  __shared__ uint32_t warp_total[32];
  const uint32_t words = (a.block_rows + 31u) / 32u;
  uint32_t *place = order_smem, *bits = place + a.experts;
  const uint32_t lo = blockIdx.x * a.block_rows, hi = min(lo + a.block_rows, a.tokens), e = threadIdx.x;
  const int id = first_choice(a, lo, hi);
  for (uint32_t i = threadIdx.x; i < a.experts * words; i += blockDim.x) bits[i] = 0u;
  uint32_t all = 0u, earlier = 0u;
  if (a.groups_of_counts) {
    // four experts in a word, added up in 16 bits: 148 blocks of at most 255 rows
    const uint32_t quads = round_up4(a.experts) / 4u, q = threadIdx.x % quads, g = threadIdx.x / quads;
    uint32_t* sums = bits + a.experts * words;
    if (g < a.groups_of_counts) {
      const uint32_t b_lo = a.blocks * g / a.groups_of_counts, b_hi = a.blocks * (g + 1u) / a.groups_of_counts;
      uint32_t sum[2] = {0u, 0u}, before[2] = {0u, 0u};
#pragma unroll 10
      for (uint32_t b = b_lo; b < b_hi; ++b) {
        const uint32_t w = __ldcg(a.counts + (size_t)b * quads + q);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t pair = (w >> (8 * h)) & 0x00FF00FFu;
          sum[h] += pair;
          before[h] += b < blockIdx.x ? pair : 0u;
        }
      }
#pragma unroll
      for (uint32_t k = 0; k < 4u; ++k) {
        sums[(2u * g) * quads * 4u + 4u * q + k] = (sum[k & 1u] >> (16u * (k >> 1))) & 0xFFFFu;
        sums[(2u * g + 1u) * quads * 4u + 4u * q + k] = (before[k & 1u] >> (16u * (k >> 1))) & 0xFFFFu;
      }
    }
    __syncthreads();
    if (e < a.experts) {
      for (uint32_t k = 0; k < a.groups_of_counts; ++k) {
        all += sums[2u * k * quads * 4u + e];
        earlier += sums[(2u * k + 1u) * quads * 4u + e];
      }
    }
  } else if (e < a.experts) {
    all = __ldcg(a.counts + (size_t)a.blocks * a.experts + e);
    earlier = __ldcg(a.counts + (size_t)blockIdx.x * a.experts + e);
  }
  __syncthreads();
  mark_choices(a, lo, hi, id, bits, words);
  uint32_t used;
  const uint32_t start = sum_before(all, warp_total, used);      // (at most 1024 experts: a thread each)
  if (e < a.experts) {
    place[e] = start + earlier;
    if (blockIdx.x == 0u) a.offsets[e] = (int32_t)start;
  }
  if (blockIdx.x == 0u && threadIdx.x == 0u) a.offsets[a.experts] = (int32_t)used;
  __syncthreads();
  place_choices(a, lo, hi, id, place, bits, words);
  // behind the last
  const uint64_t end = (uint64_t)a.tokens * a.top_k;
  for (uint64_t i = used + (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < end; i += (uint64_t)gridDim.x * blockDim.x) a.order[i] = -1;
}

uint32_t rows_of_a_block(const psb_route_desc& d) {
  // a block per SM; up to 64 rows one block alone, which spares a launch or two
  if (d.tokens <= 64u) return 64u;
  const uint32_t rows = (d.tokens + kSms - 1u) / kSms;
  return rows < 8u ? 8u : rows < kMaxBlockRows ? rows : kMaxBlockRows;
}

// ---- combine -------------------------------------------------------------------------------------------------------------

template <typename T> __device__ __forceinline__ float as_f32(T v);
template <> __device__ __forceinline__ float as_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float as_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float as_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

struct CombineArgs {
  const void* y;
  const float* weights;
  const int32_t* slot;
  void* out;
  uint32_t* err;
  uint32_t tokens, top_k, n, rows, chunks, wide;   // chunks: pieces of 16 input bytes in a row
  uint32_t row_blocks, threads, pieces;            // blocks for a row, their threads, pieces a thread
  uint64_t y_stride, out_stride;
};

// A thread owns kPieces times 16 input bytes of an output row; eight loads of the chosen rows go out together: eight choices of one
// piece, or four of two (two choices of rows of 4096 in bf16 for 8192 rows: 73 us with one piece, 43 with two).
template <typename TI, typename TO, int kPieces>
__global__ void __launch_bounds__(256, 4) combine_kernel(const CombineArgs a) {
  pdl_prologue();
  constexpr int kPer = 16 / sizeof(TI), kChoices = 8 / kPieces;
  const uint32_t t = blockIdx.x / a.row_blocks, first = (blockIdx.x - t * a.row_blocks) * blockDim.x * kPieces + threadIdx.x;
  if (first >= a.chunks) return;
  float sum[kPieces][kPer];
#pragma unroll
  for (int q = 0; q < kPieces; ++q)
#pragma unroll
    for (int e = 0; e < kPer; ++e) sum[q][e] = 0.0f;
  for (uint32_t j0 = 0; j0 < a.top_k; j0 += kChoices) {
    // all places and weights first: a row's address waits for its place, and must not hold up the next place
    uint4 v[kChoices][kPieces];
    float w[kChoices];
    int s[kChoices];
#pragma unroll
    for (int j = 0; j < kChoices; ++j) {
      const bool there = j0 + j < a.top_k;
      s[j] = there ? a.slot[(size_t)t * a.top_k + j0 + j] : -1;
      w[j] = there ? a.weights[(size_t)t * a.top_k + j0 + j] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kChoices; ++j) {
      if (s[j] >= 0 && (uint32_t)s[j] >= a.rows) {
        atomicOr(a.err, kDevErrRange);
        s[j] = -1;
      }
#pragma unroll
      for (int q = 0; q < kPieces; ++q) {
        const uint32_t c = (first + q * blockDim.x) * kPer;
        if (s[j] < 0 || c >= a.n) continue;
        const TI* row = (const TI*)a.y + (uint64_t)s[j] * a.y_stride + c;
        if (a.wide && c + kPer <= a.n) {
          v[j][q] = *reinterpret_cast<const uint4*>(row);
        } else {
          TI* parts = reinterpret_cast<TI*>(&v[j][q]);
#pragma unroll
          for (int e = 0; e < kPer; ++e) parts[e] = c + e < a.n ? row[e] : from_f32<TI>(0.0f);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kChoices; ++j) {
      if (s[j] < 0) continue;
#pragma unroll
      for (int q = 0; q < kPieces; ++q) {
        if ((first + q * blockDim.x) * kPer >= a.n) continue;
        const TI* parts = reinterpret_cast<const TI*>(&v[j][q]);
#pragma unroll
        for (int e = 0; e < kPer; ++e) sum[q][e] = __fmaf_rn(w[j], as_f32<TI>(parts[e]), sum[q][e]);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < kPieces; ++q) {
    const uint32_t c = (first + q * blockDim.x) * kPer;
    TO* out = (TO*)a.out + t * a.out_stride + c;
    if (a.wide && c + kPer <= a.n) {
      constexpr int kBytes = kPer * (int)sizeof(TO);      // 8, 16 or 32
      alignas(16) TO parts[kPer];
#pragma unroll
      for (int e = 0; e < kPer; ++e) parts[e] = from_f32<TO>(sum[q][e]);
      if (kBytes == 8) {
        *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(parts);
      } else {
#pragma unroll
        for (int b = 0; b < kBytes / 16; ++b) reinterpret_cast<uint4*>(out)[b] = reinterpret_cast<const uint4*>(parts)[b];
      }
    } else {
      for (int e = 0; e < kPer; ++e)
        if (c + e < a.n) out[e] = from_f32<TO>(sum[q][e]);
    }
  }
}

template <typename TI, typename TO>
cudaError_t launch_combine_as(const CombineArgs& a, cudaStream_t s) {
  return launched(a.pieces == 2u ? launch_pdl(combine_kernel<TI, TO, 2>, a.tokens * a.row_blocks, a.threads, 0, s, a)
                                 : launch_pdl(combine_kernel<TI, TO, 1>, a.tokens * a.row_blocks, a.threads, 0, s, a));
}
template <typename TI>
cudaError_t launch_combine_from(const CombineArgs& a, uint32_t out_dtype, cudaStream_t s) {
  if (out_dtype == PSB_DT_F32) return launch_combine_as<TI, float>(a, s);
  if (out_dtype == PSB_DT_BF16) return launch_combine_as<TI, __nv_bfloat16>(a, s);
  return launch_combine_as<TI, __half>(a, s);
}

}  // namespace

size_t route_scratch_bytes(const psb_route_desc& d) {
  const uint32_t rows = rows_of_a_block(d);
  return (size_t)((d.tokens + rows - 1u) / rows + 1u) * d.experts * sizeof(uint32_t);      // and the sums
}

cudaError_t launch_route(const void* logits, const float* bias, const uint8_t* mask, const psb_route_desc& d, int32_t* ids,
                         float* weights, int32_t* offsets, int32_t* order, int32_t* slot, void* counts, cudaStream_t s) {
  RouteArgs a;
  a.logits = logits;
  a.bias = bias;
  a.mask = mask;
  a.in_dtype = d.in_dtype;
  a.sigmoid = d.score == PSB_SCORE_SIGMOID;
  a.tokens = d.tokens;
  a.experts = d.experts;
  a.top_k = d.top_k;
  a.groups = d.groups;
  a.top_groups = d.top_groups;
  a.group_best = d.group_best;
  a.renormalise = d.renormalise;
  a.scaling = d.scaling;
  a.logit_stride = d.logit_stride;
  a.ids = ids;
  a.weights = weights;
  a.offsets = offsets;
  a.order = order;
  a.slot = slot;
  a.counts = (uint32_t*)counts;
  a.block_rows = rows_of_a_block(d);
  a.blocks = (d.tokens + a.block_rows - 1u) / a.block_rows;
  a.alone = a.blocks == 1u;
  a.wide = (((uintptr_t)logits | d.logit_stride * (d.in_dtype == PSB_DT_F32 ? 4u : 2u)) & 15u) == 0u;
  // a block's counts in bytes: every placing block adds up those of all 148 itself (16384 rows over 256 experts 27.3 us, 28.2 with scan_kernel
  // between, and a launch less for the host)
  const uint32_t quads = round_up4(d.experts) / 4u;
  a.groups_of_counts = a.block_rows > 255u || a.blocks > kSms ? 0u : 1024u / quads < 16u ? 1024u / quads : 16u;
  uint32_t el = 1;
  while (el * 32u < d.experts) el *= 2u;
  const uint32_t size = d.experts / d.groups, lanes = size / el;
  a.lanes_per_group = size % el == 0u && (lanes & (lanes - 1u)) == 0u ? lanes : 0u;
  const uint32_t ints = d.experts * (a.alone ? 1u + (a.block_rows + 31u) / 32u : 1u);
  // (a launch that fails is the last: those behind it take the choices as indices)
  auto go = [&](auto kernel, uint32_t blocks, uint32_t threads, size_t smem) {
    cudaError_t e = cudaSuccess;
    if (smem > 48u * 1024u) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
    return launched(e == cudaSuccess ? launch_pdl(kernel, blocks, threads, smem, s, a) : e);
  };
  auto route = [&](auto kernel, uint32_t threads) {
    return go(kernel, a.blocks, threads, ((ints * 4u + 15u) & ~15u) + sizeof(double) * (threads / 32u) * (d.experts + d.groups));
  };
  cudaError_t e = el == 1u    ? route(route_kernel<1>, kRouteThreads<1>)
                  : el == 2u  ? route(route_kernel<2>, kRouteThreads<2>)
                  : el == 4u  ? route(route_kernel<4>, kRouteThreads<4>)
                  : el == 8u  ? route(route_kernel<8>, kRouteThreads<8>)
                  : el == 16u ? route(route_kernel<16>, kRouteThreads<16>)
                              : route(route_kernel<32>, kRouteThreads<32>);
  if (e == cudaSuccess && order && !a.alone) {
    if (!a.groups_of_counts) e = go(scan_kernel, (d.experts + 31u) / 32u, 1024, 0);
    if (e == cudaSuccess)
      e = go(order_kernel, a.blocks, 1024,
             sizeof(uint32_t) * (d.experts * (1u + (a.block_rows + 31u) / 32u) + 2u * a.groups_of_counts * round_up4(d.experts)));
  }
  return e;
}

cudaError_t launch_combine(const void* y, const float* weights, const int32_t* slot, const psb_combine_desc& d, void* out,
                           uint32_t* err, cudaStream_t s) {
  CombineArgs a;
  a.y = y;
  a.weights = weights;
  a.slot = slot;
  a.out = out;
  a.err = err;
  a.tokens = d.tokens;
  a.top_k = d.top_k;
  a.n = d.n;
  a.rows = d.rows;
  a.y_stride = d.y_stride;
  a.out_stride = d.out_stride;
  const uint32_t in = d.in_dtype == PSB_DT_F32 ? 4u : 2u, to = d.out_dtype == PSB_DT_F32 ? 4u : 2u;
  a.chunks = (d.n + 16u / in - 1u) / (16u / in);
  a.pieces = d.top_k <= 4u && a.chunks >= 256u ? 2u : 1u;
  const uint32_t share = (a.chunks + a.pieces - 1u) / a.pieces;
  a.threads = share < 256u ? round_up(share, 32u) : 256u;
  a.row_blocks = (share + a.threads - 1u) / a.threads;
  a.wide = (((uintptr_t)y | (uintptr_t)out | d.y_stride * in | d.out_stride * to) & 15u) == 0u;
  if (d.in_dtype == PSB_DT_F32) return launch_combine_from<float>(a, d.out_dtype, s);
  if (d.in_dtype == PSB_DT_BF16) return launch_combine_from<__nv_bfloat16>(a, d.out_dtype, s);
  return launch_combine_from<__half>(a, d.out_dtype, s);
}

}  // namespace psb
