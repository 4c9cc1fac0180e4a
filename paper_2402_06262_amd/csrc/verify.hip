// Verification of drafted trees against the target's probabilities.
//
// A node's continuations are tried in their order.  After k of them have been rejected the target's distribution there is
//   p_k = max(p_(k-1) - q_(k-1), 0), normalised,   q_k the distribution that the next one was drawn from,
// which is max(p - c_k q, 0) / N_k with one number c_k, since q_k is q times a number where it is not zero: c_0 = 0, N_0 = 1,
// c_(k+1) = c_k + N_k / (1 - Q_k), N_k = sum max(p - c_k q, 0), Q_k what q gives to the earlier ones if all are distinct (else 0).
// So a decision takes two probabilities and N, and N a pass over one row of p and of q.  (Without q, which is then 1 for the drafted token, a
// rejection takes the token's p from N, and the token from the row.)
//
//   verify_pass   : the sums of a request's next pass, of blocks of kVerifyBlock tokens, a wave each.  Every workgroup adds the sums of the pass before and
//                   decides for itself, from where the walk was then, what this one is; one of them leaves the walk behind, and in the first round
//                   the nodes' probabilities, which lie in as many places.
//   verify_choose : one workgroup per request.  The passes that are left (trees; one workgroup alone with a row), the accepted path, and the next
//                   token: the block, and in it the token, where the sums pass a share `choose` of N.
// Measured, fp32: 64 chains of 8 nodes over 100003 tokens 26 to 28 us (52 MB have to be read: 7 us at the 7.0 TB/s of reads alone), 32 trees of 32 nodes over
// 65536 51 to 62 us, in 7 rounds of up to 7.5 us by trace, waits for memory three times over; before the walks were left behind, 27 and 74 to 82.  The same of bf16
// 21 and 49.  Without q, 57 trees of 18 over 2727, five continuations each, 20 us (50 with every element compared with every rejected token in a loop of its own).
// Sums are held in 64 bits: with 32 a token in some thousands would be another than the numbers say (2^17 borders, each 2^-24 off).
#include <algorithm>

#include "common.hpp"
#include "profile.hpp"

namespace roco {
namespace {

constexpr int kPassThreads = 256, kPassWaves = kPassThreads / kWave;
constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / kWave;
constexpr int kMostBlocks = kMaxVocab / kVerifyBlock + 1;

__device__ __forceinline__ double from_lane(double v, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(b), lane), hi = __builtin_amdgcn_readlane(static_cast<int>(b >> 32), lane);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int s = 1; s < kWave; s *= 2) v += __shfl_xor(v, s, kWave);
  return v;
}
__device__ __forceinline__ double sum_of(const double* sums, int blocks) {  // in a fixed order
  double v = 0.0;
  for (int i = threadIdx.x & (kWave - 1); i < blocks; i += kWave) v += sums[i];
  return wave_sum(v);
}

template <bool BF16> __device__ __forceinline__ float element(const void* row, int64_t i) {
  return BF16 ? bf16_to_f32(static_cast<const uint16_t*>(row)[i]) : static_cast<const float*>(row)[i];
}
__device__ __forceinline__ float probability(float v) { return __builtin_amdgcn_fmed3f(v, 0.0f, INFINITY); }  // (NaN: zero; one instruction)

// A request's tree, node i in lane i.
template <bool BF16> struct Tree {
  int parent, token, n;
  float accept;
  double pr, qr;
  // found: a pass before has left the nodes behind, so that nobody gathers their probabilities again
  __device__ __forceinline__ Tree(const VerifyArgs& a, int r, bool found) {
    const int lane = threadIdx.x & (kWave - 1), i = min(lane, a.nodes - 1);
    if (found) {
      const VerifyNode& node = a.found[static_cast<size_t>(r) * a.nodes + i];
      const int4 words = *reinterpret_cast<const int4*>(&node.parent);
      const double2 probabilities = *reinterpret_cast<const double2*>(&node.p);
      parent = lane < a.nodes ? words.x : -1;
      token = words.y;
      accept = __int_as_float(words.z);
      n = __builtin_amdgcn_readfirstlane(words.w);
      pr = probabilities.x;
      qr = probabilities.y;
      return;
    }
    n = __builtin_amdgcn_readfirstlane(a.n_nodes != nullptr ? min(max(a.n_nodes[r], 0), a.nodes) : a.nodes);
    parent = a.parent != nullptr ? a.parent[static_cast<size_t>(r) * a.nodes + i] : i - 1;
    token = a.tokens[static_cast<size_t>(r) * a.nodes + i];
    accept = a.accept[static_cast<size_t>(r) * a.nodes + i];
    if (lane >= n || lane == 0 || parent < 0 || parent >= lane || token < 0 || token >= a.vocab) parent = -1;  // such a node is never accepted
    pr = qr = 0.0;
    if (parent >= 0) {
      pr = probability(element<BF16>(a.p, r * a.p_request + parent * a.p_row + token));
      if (a.q != nullptr) qr = probability(element<BF16>(a.q, r * a.q_request + parent * a.q_row + token));
    }
  }
  __device__ __forceinline__ void leave(const VerifyArgs& a, int r) const {
    const int lane = threadIdx.x & (kWave - 1);
    if (lane < a.nodes) a.found[static_cast<size_t>(r) * a.nodes + lane] = VerifyNode{parent, token, accept, n, pr, qr};
  }
  __device__ __forceinline__ VerifyWalk start(const VerifyArgs& a) const {
    VerifyWalk w = {};
    w.left = 1.0;
    w.tried = 1;
    w.length = n > 0 ? 1 : 0;
    w.phase = n > 0 ? kVerifyWalks : kVerifyNothing;
    return w;
  }
  // As far as it goes without another sum; total: what the pass that it waits for has found, if it waits for one.
  __device__ __forceinline__ void advance(const VerifyArgs& a, VerifyWalk& w, double total) const {
    if (w.phase == kVerifyRejected) {
      w.left = total;
      w.phase = kVerifyWalks;
    } else if (w.phase == kVerifyEnds) {
      if (total > 0.0) {
        w.phase = kVerifyDone;
        return;
      }
      w.times = 0.0;  // nothing is left: the row as it was
      w.rejected = 0;
      w.phase = kVerifyEndsWhole;
      return;
    } else if (w.phase == kVerifyEndsWhole) {
      w.phase = kVerifyDone;
      return;
    }
    while (w.phase == kVerifyWalks) {
      const uint64_t next = __builtin_amdgcn_ballot_w64(parent == w.node && parent >= 0) & ~w.tried;
      if (next == 0 || w.length >= a.max_path) {
        w.phase = kVerifyEnds;
        return;
      }
      if (w.stale != 0) {  // the sum of the row before the last rejection will not do for another continuation
        w.stale = 0;
        w.phase = kVerifyRejected;
        return;
      }
      const int i = __builtin_ctzll(next);
      w.tried |= 1ull << i;
      const double u = from_lane(static_cast<double>(accept), i), p = from_lane(pr, i), q = from_lane(qr, i);
      bool good;
      if (a.q != nullptr) {
        const double rest = 1.0 - w.gone;
        good = __dmul_rn(__dmul_rn(u, q), w.left) < __dmul_rn(fmax(__dsub_rn(p, __dmul_rn(w.times, q)), 0.0), rest);
        if (__builtin_amdgcn_readfirstlane(!good && rest > 0.0 ? 1 : 0) != 0) {
          w.times += w.left / rest;
          if (a.distinct) w.gone += q;
          w.stale = 1;
        }
      } else {
        // (a token that is among those rejected has nothing left)
        const int x = __builtin_amdgcn_readlane(token, i);
        const bool again = (__builtin_amdgcn_ballot_w64(token == x) & w.rejected) != 0;
        good = !again && __dmul_rn(u, w.left) < p;
        if (!good) {
          if (!again) w.left -= p;
          w.rejected |= 1ull << i;
        }
      }
      if (__builtin_amdgcn_readfirstlane(good ? 1 : 0) != 0) {
        w.node = i;
        w.times = w.gone = 0.0;
        w.rejected = 0;
        w.left = 1.0;
        w.stale = 0;
        ++w.length;
      }
    }
  }
  // This lane's place in the path, or -1.
  __device__ __forceinline__ int place_of(const VerifyWalk& w) const {
    int at = -1, node = w.node;
    for (int k = w.length - 1; k >= 0; --k) {
      if (static_cast<int>(threadIdx.x & (kWave - 1)) == node) at = k;
      node = k > 0 ? __builtin_amdgcn_readlane(parent, node) : 0;
    }
    return at;
  }
};
__device__ __forceinline__ bool waits(const VerifyWalk& w) { return w.phase == kVerifyRejected || w.phase == kVerifyEnds || w.phase == kVerifyEndsWhole; }
__device__ __forceinline__ uint64_t uniform(uint64_t v) {
  return static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v >> 32)))) << 32 | static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v)));
}
__device__ __forceinline__ void uniform(VerifyWalk& w) {
  w.rejected = uniform(w.rejected);
  w.tried = uniform(w.tried);
  w.node = __builtin_amdgcn_readfirstlane(w.node);
  w.length = __builtin_amdgcn_readfirstlane(w.length);
  w.phase = __builtin_amdgcn_readfirstlane(w.phase);
  w.stale = __builtin_amdgcn_readfirstlane(w.stale);
}

// The weights of a block, one wave's: 16 bytes of a row at a time, f(index, weight) for those of the vocabulary.  The blocks begin where 16 bytes do.
template <bool BF16> struct Row {
  static constexpr int PER = BF16 ? 8 : 4, kSteps = kVerifyBlock / (kWave * PER);
  const char *p, *q;
  int before;          // elements between the last multiple of 16 bytes and the row
  bool together;       // the rows of p and q lie alike
  const VerifyArgs& a;
  const VerifyWalk& w;
  int rejected_token;  // lane i: node i's, if it has been rejected
  __device__ __forceinline__ Row(const VerifyArgs& a_, int r, const VerifyWalk& w_, int token) : a(a_), w(w_) {
    constexpr int E = BF16 ? 2 : 4;
    p = static_cast<const char*>(a.p) + (r * a.p_request + w.node * a.p_row) * E;
    q = a.q != nullptr && w.times != 0.0 ? static_cast<const char*>(a.q) + (r * a.q_request + w.node * a.q_row) * E : nullptr;
    before = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15u) / E;
    together = q == nullptr || ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15u) == 0;
    rejected_token = (w.rejected >> (threadIdx.x & (kWave - 1))) & 1 ? token : -1;
  }
  __device__ __forceinline__ int first_of(int block) const { return block * kVerifyBlock - before; }
  // PER elements from i on, zeros outside the row
  __device__ __forceinline__ void elements(const char* row, bool aligned, int i, float* f) const {
    if (aligned && i >= 0 && i + PER <= a.vocab) {
      unpack16<BF16 ? kBF16 : kF32>(load16(row + static_cast<int64_t>(i) * (BF16 ? 2 : 4)), f);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e) f[e] = i + e >= 0 && i + e < a.vocab ? element<BF16>(row, i + e) : 0.0f;
    }
  }
  __device__ __forceinline__ double weight(float x, float y) const {
    const double v = q != nullptr ? __dsub_rn(static_cast<double>(x), __dmul_rn(w.times, static_cast<double>(probability(y)))) : static_cast<double>(x);
    return v > 0.0 ? v : 0.0;  // (NaN: none)
  }
  // Zeros for the rejected tokens (without q, whose weights are p): token after token, so that an element costs a comparison and nothing else.  index(k): that of f[k].
  template <int N, class Index> __device__ __forceinline__ void take_out(float (&f)[N], Index index) const {
#pragma unroll 1
    for (uint64_t left = w.rejected; left != 0; left &= left - 1) {
      const int out = __builtin_amdgcn_readlane(rejected_token, __builtin_ctzll(left));
#pragma unroll
      for (int k = 0; k < N; ++k) f[k] = index(k) == out ? 0.0f : f[k];
    }
  }
  __device__ __forceinline__ double block_sum(int block) const {
    const int lane = threadIdx.x & (kWave - 1), first = first_of(block);
    float x[kSteps * PER], y[kSteps][PER];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) elements(p, true, first + (s * kWave + lane) * PER, x + s * PER);
    if (q != nullptr) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) elements(q, together, first + (s * kWave + lane) * PER, y[s]);
    }
    take_out(x, [&](int k) { return first + (k / PER * kWave + lane) * PER + k % PER; });
    double sum = 0.0;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int e = 0; e < PER; ++e) sum += weight(x[s * PER + e], q != nullptr ? y[s][e] : 0.0f);
    return wave_sum(sum);
  }
};

template <bool BF16> __global__ __launch_bounds__(kPassThreads) void verify_pass(VerifyArgs a, int round) {
  const int r = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int block = blockIdx.x * kPassWaves + wave;
  if (block >= a.blocks) return;
  const auto sums = [&](int pass) { return a.sums + (static_cast<size_t>(pass) * a.requests + r) * a.blocks; };
  VerifyWalk w;
  double total = 0.0;
  if (round > 0) {
    w = a.walks[static_cast<size_t>(round - 1) * a.requests + r];
    total = sum_of(sums(round - 1), a.blocks);
    uniform(w);
  }
  const Tree<BF16> tree(a, r, round > 0);
  if (round == 0) w = tree.start(a);
  const bool over = w.phase >= kVerifyDone;
  tree.advance(a, w, total);
  if (!over) w.pass = round - 1;
  if (block == 0) {
    if (round == 0) tree.leave(a, r);
    if ((threadIdx.x & (kWave - 1)) == 0) a.walks[static_cast<size_t>(round) * a.requests + r] = w;
  }
  if (!waits(w)) return;
  const Row<BF16> row(a, r, w, tree.token);
  const double sum = row.block_sum(block);
  if ((threadIdx.x & (kWave - 1)) == 0) sums(round)[block] = sum;
}

template <bool BF16> __global__ __launch_bounds__(kChooseThreads) void verify_choose(VerifyArgs a) {
  __shared__ double block_s[kMostBlocks];          // sums of the last pass
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  // (every wave walks by itself, to the same end)
  VerifyWalk w = a.walks[static_cast<size_t>(a.rounds - 1) * a.requests + r];
  uniform(w);
  // (a round that had nothing to do has left no sums: the last ones are those of the pass that ended the walk)
  const double* sums = a.sums + (static_cast<size_t>(w.phase == kVerifyDone ? w.pass : a.rounds - 1) * a.requests + r) * a.blocks;
  double all = sum_of(sums, a.blocks);
  const Tree<BF16> tree(a, r, true);
  tree.advance(a, w, all);
  while (waits(w)) {
    const Row<BF16> row(a, r, w, tree.token);
    for (int block = wave; block < a.blocks; block += kChooseWaves) {
      const double sum = row.block_sum(block);
      if (lane == 0) block_s[block] = sum;
    }
    __syncthreads();
    sums = block_s;
    all = sum_of(block_s, a.blocks);
    __syncthreads();
    tree.advance(a, w, all);
  }
  if (wave != 0) return;
  const int path_at = tree.place_of(w);
  int32_t* const path = a.path + static_cast<size_t>(r) * a.max_path;
  if (path_at >= 0) path[path_at] = lane;
  if (lane >= w.length && lane < a.max_path) path[lane] = -1;
  if (lane == 0) a.n_path[r] = w.length;
  if (w.length == 0 || !(all > 0.0)) {
    if (lane == 0) a.next[r] = -1;
    return;
  }
  // the block: each lane has `per` of them side by side
  const int per = (a.blocks + kWave - 1) / kWave;
  const auto before_of = [&](double mine, double& total) {  // exclusive prefix over the lanes
    double v = mine;
#pragma unroll
    for (int s = 1; s < kWave; s *= 2) {
      const double o = __shfl_up(v, s, kWave);
      if (lane >= s) v += o;
    }
    total = __shfl(v, kWave - 1, kWave);
    const double b = __shfl_up(v, 1, kWave);
    return lane == 0 ? 0.0 : b;
  };
  double mine = 0.0, total;
  for (int b = lane * per; b < min(a.blocks, (lane + 1) * per); ++b) mine += sums[b];
  double before = before_of(mine, total);
  const double goal = static_cast<double>(a.choose[r]) * total;
  int found = -1, last = -1;     // the first block whose end lies above the goal, the last one of any weight
  double found_before = 0.0, last_before = 0.0;
  for (int b = lane * per; b < min(a.blocks, (lane + 1) * per); ++b) {
    const double v = sums[b];
    if (v > 0.0) {
      last = b;
      last_before = before;
      if (found < 0 && before + v > goal) {
        found = b;
        found_before = before;
      }
    }
    before += v;
  }
  // (the goal is a share below one of the total; where rounding has it at the total, the last weight is meant)
  const auto pick = [&](int& at, int other, double& b, double other_b) {
    const uint64_t some = __builtin_amdgcn_ballot_w64(at >= 0);
    if (some != 0) {
      const int l = __builtin_ctzll(some);
      at = __shfl(at, l, kWave);
      b = __shfl(b, l, kWave);
    } else {
      const uint64_t any_weight = __builtin_amdgcn_ballot_w64(other >= 0);
      const int l = any_weight != 0 ? 63 - __builtin_clzll(any_weight) : 0;
      at = __shfl(other, l, kWave);
      b = __shfl(other_b, l, kWave);
    }
  };
  pick(found, last, found_before, last_before);
  // the token: each lane has kVerifyBlock / 64 of the block's side by side
  constexpr int kMine = kVerifyBlock / kWave, PER = Row<BF16>::PER;
  const Row<BF16> row(a, r, w, tree.token);
  const int first = row.first_of(found) + lane * kMine;
  float x[kMine], y[kMine];
#pragma unroll
  for (int s = 0; s < kMine / PER; ++s) row.elements(row.p, true, first + s * PER, x + s * PER);
#pragma unroll
  for (int e = 0; e < kMine; ++e) y[e] = 0.0f;
  if (row.q != nullptr) {
#pragma unroll
    for (int s = 0; s < kMine / PER; ++s) row.elements(row.q, row.together, first + s * PER, y + s * PER);
  }
  row.take_out(x, [&](int k) { return first + k; });
  double weights[kMine];
  mine = 0.0;
#pragma unroll
  for (int e = 0; e < kMine; ++e) {
    weights[e] = row.weight(x[e], y[e]);
    mine += weights[e];
  }
  before = found_before + before_of(mine, total);
  int token = -1;
  last = -1;
#pragma unroll
  for (int e = 0; e < kMine; ++e) {
    if (weights[e] > 0.0) {
      last = first + e;
      if (token < 0 && before + weights[e] > goal) token = first + e;
    }
    before += weights[e];
  }
  double unused = 0.0;
  pick(token, last, unused, 0.0);
  if (lane == 0) a.next[r] = token;
}

}  // namespace

hipError_t launch_tree_verify(const VerifyArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.blocks + kPassWaves - 1) / kPassWaves), static_cast<unsigned>(a.requests));
  for (int round = 0; round < a.rounds; ++round) {
    ProfScope ps(kProfVerifyPass, s);
    if (a.bf16) hipLaunchKernelGGL((verify_pass<true>), grid, dim3(kPassThreads), 0, s, a, round);
    else hipLaunchKernelGGL((verify_pass<false>), grid, dim3(kPassThreads), 0, s, a, round);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  ProfScope ps(kProfVerifyChoose, s);
  if (a.bf16) hipLaunchKernelGGL((verify_choose<true>), dim3(a.requests), dim3(kChooseThreads), 0, s, a);
  else hipLaunchKernelGGL((verify_choose<false>), dim3(a.requests), dim3(kChooseThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace roco
