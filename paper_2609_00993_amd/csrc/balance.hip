// The router's load-balance loss, per-expert counts and gradient
// (include/moepd_balance.h).
//
// Both directions read the logits once; what bounds them is that stream, or, for
// small batches, the launches and dependent loads.  65,536 x 256 float32: the pieces 15 us
// (4.5 TB/s), their join 7.7, the gradient 25 (5.4 TB/s); 12,001 x 512 in 37 sequences 10.6,
// 8.3 and 12.3; 64 x 8 in one launch 4.1.  One wave takes a token at a time, its logits in
// registers (runs of four neighbouring experts to a lane), with wave-wide maxima and sums in
// cross-lane moves; lanes accumulate their own experts' probabilities, so the sum
// over tokens crosses lanes only once per piece.
//
// Pieces: the tokens are cut into chunks of equal length, a workgroup each, and a
// chunk is cut where sequences end.  Chunk c and sequence s meet at most once,
// and as tokens ascend either c or s does, so c + s numbers the pieces without a
// gap in order: a piece's sums go to slot c + s, at most chunks + S - 1 slots.
// The second kernel adds each sequence's slots in a fixed order, so the
// results do not depend on scheduling, and its last workgroup adds the sequences'
// losses.  The work is dealt by tokens, so long sequences share the GPU however many there
// are; but a chunk takes its sequences one after another, and where short ones crowd beside
// a long one, whose tokens make the chunks long, few workgroups have them all: 65,536 x 256 in 99
// sequences of one token and one of the rest 149 us (loss alone; 100 even sequences 27),
// 1099 and one 162 (there one wave also adds all the long one's slots; even 26).
#include <math.h>

#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "moepd_balance.h"
#include "pipeline.h"

namespace moepd {

namespace {

struct BalanceArgs {
  const void* logits;
  const uint8_t* mask;   // null: all live
  const int32_t* seq;    // null: one sequence of all tokens
  long long stride;
  int S, T, E, k;
  float coef;
};

__device__ __forceinline__ int seq_begin(const BalanceArgs& g, int s) {
  if (!g.seq) return s <= 0 ? 0 : g.T;
  const int v = g.seq[s];
  return v < 0 ? 0 : v < g.T ? v : g.T;
}

// The first sequence that ends past token t (S if none does).  The wave's lanes look
// at 64 boundaries at a time, so that up to 64 sequences take one load and up to 4096
// two, where a binary search would take one for each halving.
__device__ __forceinline__ int seq_of(const BalanceArgs& g, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = g.S;  // the answer lies in [lo, lo + n]
  while (n > 0) {
    const int step = (n + kWave - 1) / kWave;
    const int last = min((lane + 1) * step, n) - 1;  // of this lane's run of `step`
    const uint64_t past = __ballot(lane * step < n && seq_begin(g, lo + last + 1) > t);
    if (!past) return lo + n;
    const int i = __builtin_ctzll(past);
    lo += i * step;
    if (step == 1) return lo;
    n = min(step, n - i * step) - 1;  // its last one does: the answer at the latest
  }
  return lo;
}

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, ROW_MASK, 0xF, false));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = dpp_add<0xB1, 0xF>(v);   // as wave_extremum_u32
  v = dpp_add<0x4E, 0xF>(v);
  v = dpp_add<0x124, 0xF>(v);
  v = dpp_add<0x128, 0xF>(v);
  v = dpp_add<0x142, 0xA>(v);
  v = dpp_add<0x143, 0xC>(v);
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_max(float v) {
  const uint32_t low = 0xff800000u;  // minus infinity
  return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(low, __float_as_uint(v), CTRL, ROW_MASK, 0xF, false)));
}
__device__ __forceinline__ float wave_max(float v) {
  v = dpp_max<0xB1, 0xF>(v);
  v = dpp_max<0x4E, 0xF>(v);
  v = dpp_max<0x124, 0xF>(v);
  v = dpp_max<0x128, 0xF>(v);
  v = dpp_max<0x142, 0xA>(v);
  v = dpp_max<0x143, 0xC>(v);
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// A lane's EPL experts of a row: runs of V neighbours (16 bytes of float32), lane by lane.
template <int EPL>
constexpr int kRun = EPL < 4 ? EPL : 4;
template <int EPL>
__device__ __forceinline__ int expert_of(int i) {
  constexpr int V = kRun<EPL>;
  return i / V * (kWave * V) + (int)(threadIdx.x & 63) * V + i % V;
}

template <int EPL, bool BF16>
__device__ __forceinline__ void load_logits(const BalanceArgs& g, int t, float (&x)[EPL]) {
  constexpr int V = kRun<EPL>;
#pragma unroll
  for (int i = 0; i < EPL; i += V) {
    const int e = expert_of<EPL>(i);
    const long long at = t * g.stride + e;
    if (V == 4 && e + V <= g.E) {
      if constexpr (BF16) {
        typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));
        const u16x4 q = *reinterpret_cast<const u16x4*>(static_cast<const uint16_t*>(g.logits) + at);
#pragma unroll
        for (int j = 0; j < V; ++j) x[i + j] = bf16_to_f32(q[j]);
      } else {
        const u32x4 q = *reinterpret_cast<const u32x4_any*>(static_cast<const float*>(g.logits) + at);
#pragma unroll
        for (int j = 0; j < V; ++j) x[i + j] = __uint_as_float(q[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        x[i + j] = -INFINITY;
        if (e + j < g.E) {
          if constexpr (BF16) x[i + j] = bf16_to_f32(static_cast<const uint16_t*>(g.logits)[at + j]);
          else x[i + j] = static_cast<const float*>(g.logits)[at + j];
        }
      }
    }
  }
}

// Probabilities of a row in place; all zero where every logit is minus infinity,
// NaN where one is NaN or plus infinity (the sum of the exponentials then is).
// e^(x - m) as 2^((x - m) log2 e): the two roundings and the constant's cost at most 2.2
// |x - m| 2^-24 relative, so little where the probability is not small.
template <int EPL>
__device__ __forceinline__ void softmax(float (&x)[EPL]) {
  constexpr float kLog2e = 1.44269504f;
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < EPL; ++i) m = fmaxf(m, x[i]);
  m = wave_max(m);
  m = m == -INFINITY ? 0.f : m;  // minus infinity against itself would be NaN
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    x[i] = __builtin_amdgcn_exp2f((x[i] - m) * kLog2e);
    s += x[i];
  }
  s = wave_sum(s);
  const float inv = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
  for (int i = 0; i < EPL; ++i) x[i] *= inv;
}

constexpr int kBalanceWaves = 8;
// Tokens that a wave has in flight at a time.
template <int EPL>
constexpr int kTokens = EPL <= 4 ? 4 : 2;

// A slot: E sums of probabilities, E counts, the live tokens, each part on lines of its own.
__host__ __device__ inline int slot_counts(int E) { return (E + 31) / 32 * 32; }
__host__ __device__ inline int slot_live(int E) { return 2 * slot_counts(E); }
__host__ __device__ inline int slot_words(int E) { return slot_live(E) + 32; }

// LDS of a workgroup that adds up a piece.
template <int EPL, int WAVES>
struct PieceSums {
  float sums[WAVES][EPL * kWave];
  int counts[EPL * kWave];
  int live[WAVES];
};

// Tokens [lo, hi) of one sequence: every wave's sums and live tokens, and the counts, in LDS.
template <int EPL, bool BF16, int WAVES>
__device__ __forceinline__ void add_piece(const BalanceArgs& g, const int32_t* __restrict__ idx, int lo, int hi,
                                          PieceSums<EPL, WAVES>& lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int e = threadIdx.x; e < g.E; e += 64 * WAVES) lds.counts[e] = 0;
  __syncthreads();
  float acc[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) acc[i] = 0.f;
  int live = 0;
  constexpr int N = kTokens<EPL>;
  for (int t0 = lo + wave * N; t0 < hi; t0 += WAVES * N) {
    float p[N][EPL];
    int e[N];
    bool on[N];
    // the mask and what it may mask are read together
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int t = min(t0 + j, hi - 1);
      on[j] = t0 + j < hi && !(g.mask && !g.mask[t]);
      load_logits<EPL, BF16>(g, t, p[j]);
      e[j] = lane < g.k ? idx[(long long)t * g.k + lane] : -1;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (!on[j]) continue;
      ++live;
      if ((uint32_t)e[j] < (uint32_t)g.E) atomicAdd(&lds.counts[e[j]], 1);
      softmax<EPL>(p[j]);
#pragma unroll
      for (int i = 0; i < EPL; ++i) acc[i] += p[j][i];
    }
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) lds.sums[wave][expert_of<EPL>(i)] = acc[i];
  if (lane == 0) lds.live[wave] = live;
  __syncthreads();
}
template <int EPL, int WAVES>
__device__ __forceinline__ float piece_sum(const PieceSums<EPL, WAVES>& lds, int e) {
  float v = lds.sums[0][e];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) v += lds.sums[w][e];
  return v;
}
template <int EPL, int WAVES>
__device__ __forceinline__ int piece_live(const PieceSums<EPL, WAVES>& lds) {
  int n = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) n += lds.live[w];
  return n;
}

// f P = (E c / (k T_s)) (p / T_s) of an expert of a sequence with n live tokens
// (counts and lengths are exact in float32 up to 2^24).
__device__ __forceinline__ float load_of(const BalanceArgs& g, float p, int cnt, int n) {
  return n ? (float)g.E * (float)cnt / ((float)g.k * (float)n) * (p * (1.f / (float)n)) : 0.f;
}

template <int EPL, bool BF16>
__global__ __launch_bounds__(64 * kBalanceWaves) void balance_pieces_kernel(BalanceArgs g,
                                                                            const int32_t* __restrict__ idx, int chunk,
                                                                            uint32_t* __restrict__ slots,
                                                                            int32_t* __restrict__ ticket) {
  __shared__ PieceSums<EPL, kBalanceWaves> lds;
  if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
  const int c = blockIdx.x;
  const int begin = c * chunk, end = min(begin + chunk, g.T);
  int s = seq_of(g, begin);
  for (int first = s < g.S ? seq_begin(g, s) : end; s < g.S && first < end; ++s) {
    const int next = seq_begin(g, s + 1), lo = max(begin, first), hi = min(end, next);
    first = next;
    if (lo >= hi) {  // an empty sequence: past all that follow it at once
      s = max(s, seq_of(g, max(begin, first)) - 1);
      continue;
    }
    add_piece<EPL, BF16>(g, idx, lo, hi, lds);
    uint32_t* slot = slots + (long long)(c + s) * slot_words(g.E);
    for (int e = threadIdx.x; e < g.E; e += 64 * kBalanceWaves) {
      slot[e] = __float_as_uint(piece_sum(lds, e));
      slot[slot_counts(g.E) + e] = (uint32_t)lds.counts[e];
    }
    if (threadIdx.x == 0) slot[slot_live(g.E)] = (uint32_t)piece_live(lds);
    __syncthreads();  // the LDS is free for the next piece
  }
}

// One sequence of few tokens: one workgroup does it all, with one launch (64 tokens of 8
// experts 4.4 us, two launches 8.4; 256 of 1024, 16 values to a lane, would take 24 and 9).
constexpr int kSmallWaves = 16, kSmallRows = 256;
template <int EPL, bool BF16>
__global__ __launch_bounds__(64 * kSmallWaves) void balance_small_kernel(BalanceArgs g, const int32_t* __restrict__ idx,
                                                                       float* __restrict__ loss,
                                                                       int32_t* __restrict__ counts,
                                                                       int32_t* __restrict__ live) {
  __shared__ PieceSums<EPL, kSmallWaves> lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lo = seq_begin(g, 0), hi = seq_begin(g, 1);
  add_piece<EPL, BF16>(g, idx, lo, hi, lds);
  const int n = piece_live(lds);
  float v = 0.f;
  for (int e = threadIdx.x; e < g.E; e += 64 * kSmallWaves) {
    const int cnt = lds.counts[e];
    counts[e] = cnt;
    v += load_of(g, piece_sum(lds, e), cnt, n);
  }
  v = wave_sum(v);
  __syncthreads();
  if (lane == 0) lds.sums[0][wave] = v;  // the experts' sums have been read
  __syncthreads();
  if (threadIdx.x == 0) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) sum += lds.sums[0][w];
    *loss = n ? g.coef * sum : 0.f;
    live[0] = n;
    live[1] = n > 0;
  }
}

// A lane's expert e of sequence s: its sum, count and the live tokens over slots first,
// first + step, ... of the sequence's, eight in flight (past the last one that again).
__device__ __forceinline__ void add_slots(const BalanceArgs& g, int chunk, const uint32_t* __restrict__ slots, int s,
                                          int e, int first, int step, float& p, int& cnt, int& n) {
  const int lo = seq_begin(g, s), hi = seq_begin(g, s + 1);
  if (lo >= hi) return;
  constexpr int N = 8;
  const int c1 = (hi - 1) / chunk;
  const int at = e < g.E ? e : 0;
  for (int c0 = lo / chunk + first; c0 <= c1; c0 += step * N) {
    float pv[N];
    int cv[N], nv[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t* slot = slots + (long long)(min(c0 + j * step, c1) + s) * slot_words(g.E);
      pv[j] = __uint_as_float(slot[at]);
      cv[j] = (int)slot[slot_counts(g.E) + at];
      nv[j] = (int)slot[slot_live(g.E)];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const bool in = c0 + j * step <= c1;
      p += in ? pv[j] : 0.f;
      cnt += in ? cv[j] : 0;
      n += in ? nv[j] : 0;
    }
  }
}

constexpr int kJoinWaves = 16;
struct JoinSums {
  float p[kJoinWaves][kWave];
  int counts[kJoinWaves][kWave], live[kJoinWaves];
};

// A workgroup adds all sequences' losses, in an order that its size alone decides.
__device__ __forceinline__ void add_losses(const BalanceArgs& g, int groups, const float* parts, float* loss, int32_t* live,
                                           JoinSums& lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  float sum = 0.f;
  int alive = 0;
  for (int i = threadIdx.x; i < groups * g.S; i += 64 * waves)
    sum += __hip_atomic_load(&parts[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  for (int i = threadIdx.x; i < g.S; i += 64 * waves)
    alive += __hip_atomic_load(&live[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) > 0;
  lds.p[wave][lane] = sum;
  lds.counts[wave][lane] = alive;
  __syncthreads();
  if (wave == 0) {
    sum = 0.f;
    alive = 0;
    for (int w = 0; w < waves; ++w) {
      sum += lds.p[w][lane];
      alive += lds.counts[w][lane];
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) alive += __shfl_xor(alive, off, kWave);
    if (lane == 0) {
      *loss = alive ? g.coef * (sum / (float)alive) : 0.f;
      live[g.S] = alive;
    }
  }
}

// Workgroup (x, s): 64 experts of sequence s.  Its waves deal the sequence's slots
// among them, their sums meet in LDS in wave order, and the last workgroup to finish adds
// the losses.  16 waves, or 4 where the sequences' workgroups fill the GPU by themselves.
__global__ __launch_bounds__(64 * kJoinWaves) void balance_join_kernel(BalanceArgs g, int chunk,
                                                                      const uint32_t* __restrict__ slots,
                                                                      float* __restrict__ parts, int32_t* ticket,
                                                                      float* __restrict__ loss,
                                                                      int32_t* __restrict__ counts, int32_t* live) {
  __shared__ JoinSums lds;
  __shared__ int last;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int eg = blockIdx.x, groups = gridDim.x, s = blockIdx.y;
  const int e = eg * kWave + lane;
  float p = 0.f;
  int cnt = 0, n = 0;
  add_slots(g, chunk, slots, s, e, wave, waves, p, cnt, n);
  lds.p[wave][lane] = p;
  lds.counts[wave][lane] = cnt;
  if (lane == 0) lds.live[wave] = n;
  __syncthreads();
  if (wave == 0) {
    p = 0.f;
    cnt = n = 0;
    for (int w = 0; w < waves; ++w) {
      p += lds.p[w][lane];
      cnt += lds.counts[w][lane];
      n += lds.live[w];
    }
    if (e < g.E) counts[(long long)s * g.E + e] = cnt;
    const float v = wave_sum(e < g.E ? load_of(g, p, cnt, n) : 0.f);
    if (lane == 0) {
      __hip_atomic_store(&parts[s * groups + eg], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (eg == 0) __hip_atomic_store(&live[s], n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // What the last workgroup reads is stored and loaded at the device's point of coherence, so
      // all the ticket has to follow is those stores' completion: a release and an acquire for
      // the whole device would write back and drop every XCD's L2 on the way (12 us for 7).
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      wait_vmcnt_lgkm0<0>();
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups * g.S - 1;
    }
  }
  __syncthreads();
  if (last) add_losses(g, groups, parts, loss, live, lds);
}

// Many sequences: a wave each for 64 experts of a sequence, and a launch of its own for
// the losses, since thousands of tickets on one word would take longer.
__global__ __launch_bounds__(256) void balance_join_each_kernel(BalanceArgs g, int chunk,
                                                               const uint32_t* __restrict__ slots,
                                                               float* __restrict__ parts, int32_t* __restrict__ counts,
                                                               int32_t* __restrict__ live) {
  const int lane = threadIdx.x & 63;
  const int eg = blockIdx.x, groups = gridDim.x, s = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (s >= g.S) return;  // whole wave leaves together
  const int e = eg * kWave + lane;
  float p = 0.f;
  int cnt = 0, n = 0;
  add_slots(g, chunk, slots, s, e, 0, 1, p, cnt, n);
  if (e < g.E) counts[(long long)s * g.E + e] = cnt;
  const float v = wave_sum(e < g.E ? load_of(g, p, cnt, n) : 0.f);
  if (lane == 0) {
    parts[s * groups + eg] = v;
    if (eg == 0) live[s] = n;
  }
}
__global__ __launch_bounds__(64 * kJoinWaves) void balance_total_kernel(BalanceArgs g, int groups, const float* parts,
                                                                       float* loss, int32_t* live) {
  __shared__ JoinSums lds;
  add_losses(g, groups, parts, loss, live, lds);
}

// One wave takes a run of consecutive tokens, so that a sequence's f stays in its registers.
template <int EPL, bool BF16>
__global__ __launch_bounds__(64 * kBalanceWaves) void balance_backward_kernel(BalanceArgs g, int run,
                                                                              const int32_t* __restrict__ counts,
                                                                              const int32_t* __restrict__ live,
                                                                              const float* __restrict__ grad,
                                                                              void* dlogits, long long dstride,
                                                                              bool accumulate) {
  const int wave = threadIdx.x >> 6;
  const long long first = ((long long)blockIdx.x * kBalanceWaves + wave) * run;
  if (first >= g.T) return;
  const int begin = (int)first, end = (int)(first + run < g.T ? first + run : g.T);
  constexpr int N = EPL <= 4 ? 4 : 2;
  float d[N][EPL];
  uint8_t mask[N];
  auto load = [&](int t0) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int t = min(t0 + j, end - 1);
      mask[j] = g.mask ? g.mask[t] : 1;
      load_logits<EPL, BF16>(g, t, d[j]);
    }
  };
  load(begin);  // beside the loads that find its sequence
  const int seqs = live[g.S];
  const float scale = (grad ? *grad : 1.f) * g.coef;
  int s = seq_of(g, begin);
  int s_begin = s < g.S ? seq_begin(g, s) : g.T, s_end = s < g.S ? seq_begin(g, s + 1) : g.T;
  float f[EPL], weight = 0.f;
  auto enter = [&] {
    const int n = s < g.S ? live[s] : 0;
    weight = n > 0 && seqs > 0 ? scale / ((float)n * (float)seqs) : 0.f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = expert_of<EPL>(i);
      f[i] = e < g.E && n > 0 ? (float)g.E * (float)counts[(long long)s * g.E + e] / ((float)g.k * (float)n) : 0.f;
    }
  };
  enter();
  for (int t0 = begin; t0 < end; t0 += N) {
    if (t0 != begin) load(t0);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int t = t0 + j;
      if (t >= end) break;
      if (t >= s_end && s < g.S) {
        ++s;
        if (s < g.S) s_end = seq_begin(g, s + 1);
        if (s < g.S && t >= s_end) {  // empty sequences: past all of them at once
          s = max(s, seq_of(g, t));
          if (s < g.S) s_end = seq_begin(g, s + 1);
        }
        s_begin = s < g.S ? seq_begin(g, s) : g.T;
        enter();
      }
      const bool on = s < g.S && t >= s_begin && mask[j];
      if (!on && accumulate) continue;
      if (on) {
        softmax<EPL>(d[j]);
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) dot = __builtin_fmaf(f[i], d[j][i], dot);
        dot = wave_sum(dot);
#pragma unroll
        for (int i = 0; i < EPL; ++i) d[j][i] = weight * (d[j][i] * (f[i] - dot));
      } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i) d[j][i] = 0.f;
      }
      constexpr int V = kRun<EPL>;
#pragma unroll
      for (int i = 0; i < EPL; i += V) {
        const int e = expert_of<EPL>(i);
        const long long at = t * dstride + e;
        if (V == 4 && !BF16 && !accumulate && e + V <= g.E) {
          // a gradient is written once, past the caches' keeping
          const u32x4_any q = {__float_as_uint(d[j][i]), __float_as_uint(d[j][i + 1 % V]), __float_as_uint(d[j][i + 2 % V]),
                               __float_as_uint(d[j][i + 3 % V])};
          __builtin_nontemporal_store(q, reinterpret_cast<u32x4_any*>(static_cast<float*>(dlogits) + at));
          continue;
        }
#pragma unroll
        for (int c = 0; c < V; ++c) {
          if (e + c >= g.E) continue;
          const float v = d[j][i + c];
          if constexpr (BF16) {
            uint16_t* o = static_cast<uint16_t*>(dlogits) + at + c;
            *o = f32_to_bf16(accumulate ? bf16_to_f32(*o) + v : v);
          } else {
            float* o = static_cast<float*>(dlogits) + at + c;
            *o = accumulate ? *o + v : v;
          }
        }
      }
    }
  }
}

// Tokens of a chunk: at most 512 chunks (two workgroups to a CU; every slot is
// written and read again), of whole rounds of its waves, one at least.  A chunk's
// sequences are taken one after another, 2 to 3 us each, so where sequences are shorter than
// a round a chunk holds about two of them, and many sequences may have up to 4096 chunks (342
// tokens in 126 sequences: 41 us with chunks of 32 tokens, 19 with 5; 60,000 tokens in 9000 sequences 179 and 52, with the
// join of its own for many sequences).
int chunk_of(int T, int S) {
  const int most = S < 512 ? 512 : S < 4096 ? S : 4096, round = 4 * kBalanceWaves;
  const int c = (T + most - 1) / most;
  const long long two = S > 1 ? 2LL * T / S : round;
  const int least = two < 4 ? 4 : two < round ? (int)two : round;
  return c <= least ? least : c < round ? c : (c + round - 1) / round * round;
}

constexpr int kTicketBytes = 128;

int64_t workspace_bytes(int T, int E, int S) {
  const int chunk = chunk_of(T, S);
  const int64_t slots = (T + chunk - 1) / chunk + (int64_t)S;
  return kTicketBytes + slots * slot_words(E) * 4 + (int64_t)S * ((E + 63) / 64) * 4;
}

template <class F>
hipError_t by_experts(int E, F&& f) {
  if (E <= 64) f(std::integral_constant<int, 1>{});
  else if (E <= 128) f(std::integral_constant<int, 2>{});
  else if (E <= 256) f(std::integral_constant<int, 4>{});
  else if (E <= 512) f(std::integral_constant<int, 8>{});
  else f(std::integral_constant<int, 16>{});
  return hipGetLastError();
}

bool valid(int32_t dtype, int64_t* stride, const int32_t* seq, int32_t S, int32_t T, int32_t E, int32_t k,
           hipStream_t stream) {
  if (!stream || (dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16)) return false;
  if (T < 0 || T > (1 << 24) || E < 1 || E > kMaxExperts || k < 1 || k > kMaxTopK || k > E) return false;
  if (S < 1 || S > 65536 || (!seq && S != 1) || (uintptr_t)seq % 4) return false;
  if (*stride == 0) *stride = E;
  return *stride >= E;
}

bool aligned(const void* p, int32_t dtype) { return (uintptr_t)p % (dtype == MOE_DTYPE_F32 ? 4 : 2) == 0; }

}  // namespace
}  // namespace moepd

using namespace moepd;

extern "C" {

int moe_balance_workspace(int32_t T, int32_t E, int32_t S, int64_t* bytes) {
  if (!bytes || T < 0 || T > (1 << 24) || E < 1 || E > kMaxExperts || S < 1 || S > 65536) return MOE_ERR_INVALID_ARG;
  *bytes = workspace_bytes(T, E, S);
  return MOE_OK;
}

int moe_balance_loss(const void* logits, int32_t logits_dtype, int64_t logits_stride, const int32_t* topk_idx,
                     const uint8_t* token_mask, const int32_t* seq_offsets, int32_t S, int32_t T, int32_t E, int32_t k,
                     float coef, float* loss, int32_t* counts, int32_t* live, void* workspace, int64_t ws_bytes,
                     hipStream_t stream) {
  if (!valid(logits_dtype, &logits_stride, seq_offsets, S, T, E, k, stream)) return MOE_ERR_INVALID_ARG;
  if (!loss || !counts || !live || !workspace || (uintptr_t)workspace % 256 ||
      ((uintptr_t)loss | (uintptr_t)counts | (uintptr_t)live | (uintptr_t)topk_idx) % 4)
    return MOE_ERR_INVALID_ARG;
  if (T > 0 && (!logits || !topk_idx || !aligned(logits, logits_dtype))) return MOE_ERR_INVALID_ARG;
  if (ws_bytes < workspace_bytes(T, E, S)) return MOE_ERR_CAPACITY;
  const BalanceArgs g{logits, token_mask, seq_offsets, logits_stride, S, T, E, k, coef};
  const int chunk = chunk_of(T, S), chunks = T > 0 ? (T + chunk - 1) / chunk : 1, groups = (E + 63) / 64;
  int32_t* ticket = static_cast<int32_t*>(workspace);
  uint32_t* slots = reinterpret_cast<uint32_t*>(static_cast<char*>(workspace) + kTicketBytes);
  float* parts = reinterpret_cast<float*>(slots + ((T + chunk - 1) / chunk + (long long)S) * slot_words(E));
  if (S == 1 && T * ((E + 63) / 64) <= kSmallRows) {
    auto small = [&](auto epl) {
      constexpr int EPL = decltype(epl)::value;
      if (logits_dtype == MOE_DTYPE_BF16)
        balance_small_kernel<EPL, true><<<1, 64 * kSmallWaves, 0, stream>>>(g, topk_idx, loss, counts, live);
      else
        balance_small_kernel<EPL, false><<<1, 64 * kSmallWaves, 0, stream>>>(g, topk_idx, loss, counts, live);
    };
    return by_experts(E, small) == hipSuccess ? MOE_OK : MOE_ERR_HIP;
  }
  auto pieces = [&](auto epl) {
    constexpr int EPL = decltype(epl)::value;
    if (logits_dtype == MOE_DTYPE_BF16)
      balance_pieces_kernel<EPL, true><<<chunks, 64 * kBalanceWaves, 0, stream>>>(g, topk_idx, chunk, slots, ticket);
    else
      balance_pieces_kernel<EPL, false><<<chunks, 64 * kBalanceWaves, 0, stream>>>(g, topk_idx, chunk, slots, ticket);
  };
  if (by_experts(E, pieces) != hipSuccess) return MOE_ERR_HIP;
  if ((long long)groups * S > 4096) {
    balance_join_each_kernel<<<dim3(groups, (S + 3) / 4), 256, 0, stream>>>(g, chunk, slots, parts, counts, live);
    balance_total_kernel<<<1, 64 * kJoinWaves, 0, stream>>>(g, groups, parts, loss, live);
  } else {
    const int waves = groups * S > 512 ? 4 : kJoinWaves;
    balance_join_kernel<<<dim3(groups, S), 64 * waves, 0, stream>>>(g, chunk, slots, parts, ticket, loss, counts, live);
  }
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_balance_loss_backward(const void* logits, int32_t logits_dtype, int64_t logits_stride,
                              const uint8_t* token_mask, const int32_t* seq_offsets, int32_t S, int32_t T, int32_t E,
                              int32_t k, float coef, const int32_t* counts, const int32_t* live, const float* grad,
                              void* dlogits, int64_t dlogits_stride, int32_t accumulate, hipStream_t stream) {
  if (!valid(logits_dtype, &logits_stride, seq_offsets, S, T, E, k, stream)) return MOE_ERR_INVALID_ARG;
  if (dlogits_stride == 0) dlogits_stride = E;
  if (dlogits_stride < E) return MOE_ERR_INVALID_ARG;
  if (dlogits == logits && dlogits && (accumulate || dlogits_stride != logits_stride)) return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!logits || !counts || !live || !dlogits || !aligned(logits, logits_dtype) || !aligned(dlogits, logits_dtype) ||
      ((uintptr_t)counts | (uintptr_t)live | (uintptr_t)grad) % 4)
    return MOE_ERR_INVALID_ARG;
  const BalanceArgs g{logits, token_mask, seq_offsets, logits_stride, S, T, E, k, coef};
  // 4096 waves or one token each
  const int run = (T + 4095) / 4096;
  const int blocks = (int)(((T + run - 1) / run + kBalanceWaves - 1) / kBalanceWaves);
  auto go = [&](auto epl) {
    constexpr int EPL = decltype(epl)::value;
    if (logits_dtype == MOE_DTYPE_BF16)
      balance_backward_kernel<EPL, true><<<blocks, 64 * kBalanceWaves, 0, stream>>>(g, run, counts, live, grad, dlogits,
                                                                                   dlogits_stride, accumulate != 0);
    else
      balance_backward_kernel<EPL, false><<<blocks, 64 * kBalanceWaves, 0, stream>>>(g, run, counts, live, grad, dlogits,
                                                                                    dlogits_stride, accumulate != 0);
  };
  return by_experts(E, go) == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
