// Verification of drafted trees against the target's probabilities.
//
// A node's continuations are tried in their order.  After k of them have been rejected the target's distribution there is
//   p_k = max(p_(k-1) - q_(k-1), 0), normalised,   q_k the distribution that the next one was drawn from,
// which is max(p - c_k q, 0) / N_k with one number c_k, since q_k is q times a number where it is not zero: c_0 = 0, N_0 = 1,
// c_(k+1) = c_k + N_k / (1 - Q_k), N_k = sum max(p - c_k q, 0), Q_k what q gives to the earlier ones if all are distinct (else 0).
// So a decision takes two probabilities and N, and N a pass over one row of p and of q.  (Without q, which is then 1 for the drafted token, a
// rejection takes the token's p from N, and the token from the row.)
//
//   verify_pass   : the sums of a request's next pass, of blocks of kVerifyBlock tokens, a wave each.  Every workgroup decides for itself what that pass
//                   is, from the sums of the passes before: no launch in between.
//   verify_choose : one workgroup per request.  The passes that are left (trees; one workgroup alone with a row), the accepted path, and the next
//                   token: the block, and in it the token, where the sums pass a share `choose` of N.
// Sums are held in 64 bits: with 32 a token in some thousands would be another than the numbers say (2^17 borders, each 2^-24 off).
#include <algorithm>

#include "common.hpp"
#include "profile.hpp"

namespace roco {
namespace {

constexpr int kPassThreads = 256, kPassWaves = kPassThreads / kWave;
constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / kWave;
constexpr int kMostNodes = kMaxTreeNodes;
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

// What a walk has come to: the node whose row is wanted, and of the row max(p - times q, 0), or, without q, p without the rejected tokens.
struct Wanted {
  int node;
  double times;
  uint64_t rejected;  // nodes whose tokens are left out (without q)
  int pass;           // number of the pass whose sums these are
  int length;         // of the path
  bool known;         // those sums are there: the walk is done
};

// The walk over a request's tree by one wave, node i in lane i: what can be decided with the sums of `passes` passes, totals of which are in `left_of`.
template <bool BF16> struct Tree {
  int parent, token, n;
  float accept;
  double pr, qr;
  __device__ __forceinline__ Tree(const VerifyArgs& a, int r) {
    const int lane = threadIdx.x & (kWave - 1), i = min(lane, a.nodes - 1);
    n = __builtin_amdgcn_readfirstlane(a.n_nodes != nullptr ? min(max(a.n_nodes[r], 0), a.nodes) : a.nodes);
    parent = a.parent != nullptr ? a.parent[static_cast<size_t>(r) * a.nodes + i] : i - 1;
    token = a.tokens[static_cast<size_t>(r) * a.nodes + i];
    accept = a.accept[static_cast<size_t>(r) * a.nodes + i];
    if (lane >= n || lane == 0 || parent < 0 || parent >= lane || token < 0 || token >= a.vocab) parent = -1;  // such a node is never accepted
    pr = qr = 0.0;
    if (parent >= 0) {
      pr = element<BF16>(a.p, r * a.p_request + parent * a.p_row + token);
      if (a.q != nullptr) qr = element<BF16>(a.q, r * a.q_request + parent * a.q_row + token);
    }
  }
  // path_at: this lane's place in the path, or -1.  left_of(pass): the total of a pass.
  template <class LeftOf> __device__ __forceinline__ Wanted walk(const VerifyArgs& a, int passes, LeftOf left_of, int& path_at) const {
    const int lane = threadIdx.x & (kWave - 1);
    Wanted w = {0, 0.0, 0, 0, n > 0 ? 1 : 0, false};
    path_at = n > 0 && lane == 0 ? 0 : -1;
    double left = 1.0, gone = 0.0;
    bool stale = false;  // `left` is that of the row before the last rejection
    uint64_t tried = 1;
    while (w.length > 0 && w.length < a.max_path) {
      const uint64_t next = __builtin_amdgcn_ballot_w64(parent == w.node && parent >= 0) & ~tried;
      if (next == 0) break;
      const int i = __builtin_ctzll(next);
      if (stale) {
        if (w.pass >= passes) return w;
        left = left_of(w.pass++);
        stale = false;
      }
      tried |= 1ull << i;
      const double u = from_lane(static_cast<double>(accept), i), p = from_lane(pr, i), q = from_lane(qr, i);
      bool good;
      if (a.q != nullptr) {
        const double rest = 1.0 - gone;
        good = __dmul_rn(__dmul_rn(u, q), left) < __dmul_rn(fmax(__dsub_rn(p, __dmul_rn(w.times, q)), 0.0), rest);
        if (!good && rest > 0.0) {
          w.times += left / rest;
          if (a.distinct) gone += q;
          stale = true;
        }
      } else {
        // (a token that is among those rejected has nothing left)
        const int x = __builtin_amdgcn_readlane(token, i);
        const bool again = (__builtin_amdgcn_ballot_w64(token == x) & w.rejected) != 0;
        good = !again && __dmul_rn(u, left) < p;
        if (!good) {
          if (!again) left -= p;
          w.rejected |= 1ull << i;
        }
      }
      if (good) {
        w.node = i;
        w.times = 0.0;
        w.rejected = 0;
        left = 1.0;
        gone = 0.0;
        stale = false;
        if (lane == i) path_at = w.length;
        ++w.length;
      }
    }
    w.known = w.pass < passes;
    if (w.known && !(left_of(w.pass) > 0.0)) {  // nothing is left: the row as it was
      w.times = 0.0;
      w.rejected = 0;
      w.known = ++w.pass < passes;
    }
    return w;
  }
};

// The weights of a block, one wave's: 16 bytes of a row at a time, f(index, weight) for those of the vocabulary.  The blocks begin where 16 bytes do.
template <bool BF16> struct Row {
  static constexpr int PER = BF16 ? 8 : 4, kSteps = kVerifyBlock / (kWave * PER);
  const char *p, *q;
  int before;          // elements between the last multiple of 16 bytes and the row
  bool together;       // the rows of p and q lie alike
  const VerifyArgs& a;
  const Wanted& w;
  int rejected_token;  // lane i: node i's, if it has been rejected
  __device__ __forceinline__ Row(const VerifyArgs& a_, int r, const Wanted& w_, int token) : a(a_), w(w_) {
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
    const double v = q != nullptr ? __dsub_rn(static_cast<double>(x), __dmul_rn(w.times, static_cast<double>(y))) : static_cast<double>(x);
    return v > 0.0 ? v : 0.0;  // (NaN: none)
  }
  __device__ __forceinline__ bool left_out(int i) const {
    bool out = false;
    for (uint64_t left = w.rejected; left != 0; left &= left - 1) out |= __builtin_amdgcn_readlane(rejected_token, __builtin_ctzll(left)) == i;
    return out;
  }
  __device__ __forceinline__ double block_sum(int block) const {
    const int lane = threadIdx.x & (kWave - 1), first = first_of(block);
    float x[kSteps][PER], y[kSteps][PER];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) elements(p, true, first + (s * kWave + lane) * PER, x[s]);
    if (q != nullptr) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) elements(q, together, first + (s * kWave + lane) * PER, y[s]);
    }
    double sum = 0.0;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        double v = weight(x[s][e], q != nullptr ? y[s][e] : 0.0f);
        if (w.rejected != 0 && left_out(first + (s * kWave + lane) * PER + e)) v = 0.0;
        sum += v;
      }
    return wave_sum(sum);
  }
};

template <bool BF16> __global__ __launch_bounds__(kPassThreads) void verify_pass(VerifyArgs a, int round) {
  const int r = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int block = blockIdx.x * kPassWaves + wave;
  if (block >= a.blocks) return;
  const Tree<BF16> tree(a, r);
  int path_at;
  const auto sums = [&](int pass) { return a.sums + (static_cast<size_t>(pass) * a.requests + r) * a.blocks; };
  const Wanted w = tree.walk(a, round, [&](int pass) { return sum_of(sums(pass), a.blocks); }, path_at);
  if (w.known || w.length == 0) return;
  const Row<BF16> row(a, r, w, tree.token);
  const double sum = row.block_sum(block);
  if ((threadIdx.x & (kWave - 1)) == 0) a.sums[(static_cast<size_t>(round) * a.requests + r) * a.blocks + block] = sum;
}

template <bool BF16> __global__ __launch_bounds__(kChooseThreads) void verify_choose(VerifyArgs a) {
  __shared__ double block_s[kMostBlocks];          // sums of the last pass
  __shared__ double left_s[kMostNodes + 2];        // totals of the passes
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const Tree<BF16> tree(a, r);
  // (every wave walks by itself, to the same end)
  for (int pass = wave; pass < a.rounds; pass += kChooseWaves) {
    // what a pass that was not wanted has left there is not looked at
    const double total = sum_of(a.sums + (static_cast<size_t>(pass) * a.requests + r) * a.blocks, a.blocks);
    if (lane == 0) left_s[pass] = total;
  }
  __syncthreads();
  int passes = a.rounds, path_at;
  Wanted w;
  for (;;) {
    w = tree.walk(a, passes, [&](int pass) { return left_s[pass]; }, path_at);
    if (w.known || w.length == 0 || passes >= kMostNodes + 2) break;
    const Row<BF16> row(a, r, w, tree.token);
    for (int block = wave; block < a.blocks; block += kChooseWaves) {
      const double sum = row.block_sum(block);
      if (lane == 0) block_s[block] = sum;
    }
    __syncthreads();
    const double total = sum_of(block_s, a.blocks);
    if (tid == 0) left_s[passes] = total;
    ++passes;
    __syncthreads();
  }
  if (wave != 0) return;
  int32_t* const path = a.path + static_cast<size_t>(r) * a.max_path;
  if (path_at >= 0) path[path_at] = lane;
  if (lane >= w.length && lane < a.max_path) path[lane] = -1;
  if (lane == 0) a.n_path[r] = w.length;
  const bool any = w.known && left_s[min(w.pass, kMostNodes + 1)] > 0.0;
  if (w.length == 0 || !any) {
    if (lane == 0) a.next[r] = -1;
    return;
  }
  // the block: each lane has `per` of them side by side
  const double* const sums = w.pass < a.rounds ? a.sums + (static_cast<size_t>(w.pass) * a.requests + r) * a.blocks : block_s;
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
  double weights[kMine];
  mine = 0.0;
#pragma unroll
  for (int e = 0; e < kMine; ++e) {
    weights[e] = row.weight(x[e], y[e]);
    if (w.rejected != 0 && row.left_out(first + e)) weights[e] = 0.0;
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
