// layer_paged_evict.hip -- part of liblram: eviction from the cache in pages by accumulated attention weight.
//
// Of n keys of a head the `budget` of the highest rank stay: (newest ones first, weight, lowest position) as one 64-bit number
// whose order is theirs, found by a radix selection from the top digit down.  Attention asks for no order of its keys (their
// positions are stored beside them), so only keys that stay and lie past the budget move, into the slots below it that
// are left: budget - n moves at most, and one where a step adds one key.

#include "layer_paged.h"

namespace {

constexpr int EVICT_THREADS = 1024, EVICT_WAVES = EVICT_THREADS / WAVE;

struct Evict {
  Pool p;
  int64_t budget, recent;
  int64_t most;   // entries of a list
  int32_t* lists; // [batch][kv_heads][2][most]: slots that move, and where they go
};

// A slot of no page below the budget counts as taken: nothing can move there.
__device__ __forceinline__ uint64_t rank_of(const Pool& p, int b, int head, int slot, int64_t newest, int budget) {
  const int page = page_of(p, b, slot);
  if (page < 0) return slot < budget ? ~(uint64_t)0 : 0;
  const int64_t at = page_rows(p, page, head) + (slot & (p.page - 1));
  const int position = p.position[at];
  const float w = p.weight[at] + 0.0f;  // -0 is 0
  const uint32_t bits = __builtin_bit_cast(uint32_t, w), up = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
  const uint32_t high = position >= newest ? 0xffffffffu : w != w ? 0u : up;
  return (uint64_t)high << 32 | (0x7fffffffu - (uint32_t)position);  // 0x7fffffff - position >= 0
}

// How many of the workgroup's threads before this one (in order) say yes, and all that do.
__device__ __forceinline__ int before(bool yes, int* sums, int& all) {
  const uint64_t votes = __builtin_amdgcn_ballot_w64(yes);
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  __syncthreads();  // the last sums have been read
  if (lane == 0) sums[wave] = __popcll(votes);
  __syncthreads();
  int n = __popcll(votes & (((uint64_t)1 << lane) - 1));
  all = 0;
#pragma unroll
  for (int w = 0; w < EVICT_WAVES; ++w) {
    n += w < wave ? sums[w] : 0;
    all += sums[w];
  }
  return n;
}

// One key to another slot, by a wave.
template <typename T, int D>
__device__ __forceinline__ void move_key(const Pool& p, int b, int head, int from, int to) {
  using Ti = PageTile<T>;
  constexpr int E = Ti::E;
  const int lane = threadIdx.x % WAVE;
  const int pf = page_of(p, b, from), pt = page_of(p, b, to);
  if (pf < 0 || pt < 0) return;
  const int tf = from & (p.page - 1), tt = to & (p.page - 1);
  const int64_t f = page_rows(p, pf, head), t = page_rows(p, pt, head);
  if (lane < D / E)
    *(uint4*)((T*)p.k + t * D + ((int64_t)(tt / 16 * (D / E) + lane) * 16 + tt % 16) * E) =
        *(const uint4*)((const T*)p.k + f * D + ((int64_t)(tf / 16 * (D / E) + lane) * 16 + tf % 16) * E);
  const auto place = [](int t, int d) {
    return ((t / Ti::KEYS * (D / 16) + d / 16) * 64 + t % 16 / 4 * 16 + d % 16) * E + t % Ti::KEYS / 16 * 4 + t % 4;
  };
  for (int d = lane; d < D; d += WAVE) ((T*)p.v)[t * D + place(tt, d)] = ((const T*)p.v)[f * D + place(tf, d)];
  if (lane == 0) {
    p.position[t + tt] = p.position[f + tf];
    p.weight[t + tt] = p.weight[f + tf];
  }
}

template <typename T, int D>
__global__ __launch_bounds__(EVICT_THREADS) void k_paged_evict(Evict a) {
  __shared__ int bins[256], sums[EVICT_WAVES], chosen[3];
  const Pool& p = a.p;
  const int head = blockIdx.x % p.kv_heads, b = blockIdx.x / p.kv_heads;
  const int64_t most = p.width << p.log_page;
  const int n = (int)min((int64_t)max(p.used[b], 0), most);
  if (n <= a.budget) return;
  const int budget = (int)a.budget;
  const int64_t newest = (int64_t)p.seen[b] - a.recent;
  // the digits of the lowest rank that stays, from the top
  uint64_t mask = 0, prefix = 0;
  int want = budget;  // of the ranks that begin with prefix
  bool all = false;   // these are all there are
  for (int shift = 56; shift >= 0 && !all; shift -= 8) {
    if (threadIdx.x < 256) bins[threadIdx.x] = 0;
    __syncthreads();
    for (int slot = threadIdx.x; slot < n; slot += EVICT_THREADS) {
      const uint64_t r = rank_of(p, b, head, slot, newest, budget);
      if ((r & mask) == prefix) atomicAdd(&bins[r >> shift & 255], 1);
    }
    __syncthreads();
    if (threadIdx.x < WAVE) {  // lane l: the bins 255 - 4 l and the three below
      int sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += bins[255 - 4 * threadIdx.x - i];
      int above = sum;
#pragma unroll
      for (int o = 1; o < WAVE; o *= 2) {
        const int x = __shfl_up(above, o);
        above += (int)threadIdx.x >= o ? x : 0;
      }
      if (above >= want && above - sum < want) {  // one lane
        int left = want - (above - sum), bin = 255 - 4 * threadIdx.x;
        while (bins[bin] < left) left -= bins[bin--];
        chosen[0] = bin, chosen[1] = left, chosen[2] = bins[bin];
      }
    }
    __syncthreads();
    prefix |= (uint64_t)chosen[0] << shift;
    mask |= (uint64_t)255 << shift;
    want = chosen[1];
    all = want == chosen[2];
  }
  int32_t* const from = a.lists + ((int64_t)b * p.kv_heads + head) * 2 * a.most;
  int32_t* const to = from + a.most;
  int equal = 0, sources = 0, holes = 0;
  for (int base = 0; base < n; base += EVICT_THREADS) {
    const int slot = base + threadIdx.x;
    const uint64_t r = slot < n ? rank_of(p, b, head, slot, newest, budget) & mask : 0;
    bool stays = slot < n && r >= prefix;
    int more;
    if (!all) {  // equal ranks: the first ones
      const bool same = slot < n && r == prefix;
      const int earlier = equal + before(same, sums, more);
      equal += more;
      stays = stays && !(same && earlier >= want);
    }
    const bool moves = stays && slot >= budget, hole = !stays && slot < budget;
    const int i = sources + before(moves, sums, more);
    sources += more;
    const int j = holes + before(hole, sums, more);
    holes += more;
    if (moves && i < a.most) from[i] = slot;
    if (hole && j < a.most) to[j] = slot;
  }
  __syncthreads();
  const int count = (int)min((int64_t)min(sources, holes), a.most);
  for (int i = threadIdx.x / WAVE; i < count; i += EVICT_WAVES) move_key<T, D>(p, b, head, from[i], to[i]);
}

int64_t list_of(const lram_paged& p, int64_t budget) {
  return std::max<int64_t>(0, std::min(budget, p.width * p.page - budget));
}

int check_evict(const lram_paged& p, int64_t budget, int64_t recent) {
  if (int rc = check_pool(p, false)) return rc;
  if (budget < 1 || recent < 0 || recent > budget || (p.pages && !p.weight)) return LRAM_EINVAL;
  if ((int64_t)p.batch * p.kv_heads > ((int64_t)1 << 32) / EVICT_THREADS - 1) return LRAM_EINVAL;
  return LRAM_OK;
}

}  // namespace

extern "C" {

int lram_paged_evict_workspace_bytes(const lram_paged* p, int64_t budget, size_t* bytes) {
  if (!p || !bytes) return LRAM_EINVAL;
  if (int rc = check_evict(*p, budget, 0)) return rc;
  *bytes = (size_t)p->batch * p->kv_heads * 2 * list_of(*p, budget) * sizeof(int32_t);
  return LRAM_OK;
}

int lram_paged_evict(const lram_paged* p, int64_t budget, int64_t recent, void* workspace, size_t ws_bytes, void* stream) {
  if (!p) return LRAM_EINVAL;
  if (int rc = check_evict(*p, budget, recent)) return rc;
  Evict a{};
  a.p = pool_of(*p);
  a.budget = budget, a.recent = recent, a.most = list_of(*p, budget);
  if (p->batch == 0 || a.most == 0) return LRAM_OK;  // nothing can be over the budget
  const size_t need = (size_t)p->batch * p->kv_heads * 2 * a.most * sizeof(int32_t);
  if (!workspace || off_align(workspace, 16) || ws_bytes < need) return LRAM_EWORKSPACE;
  a.lists = (int32_t*)workspace;
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p->batch * p->kv_heads)), dim3(EVICT_THREADS), 0, (hipStream_t)stream, a);
    return layer_launched();
  };
  return by_form(p->dtype, p->head_dim, [&](auto t, auto d) { return go(k_paged_evict<decltype(t), decltype(d)::value>); });
}

}  // extern "C"
